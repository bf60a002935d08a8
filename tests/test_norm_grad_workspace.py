"""Where layer norm's gradient needs a workspace (no GPU): from the first row on that one
workgroup does not hold, which a call without the bytes tells of."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVAL, WORKSPACE = 1, 3
F32, BF16 = 0, 1
FAR = 1 << 28


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(os.path.join(ROOT, "paper_1810_10045_amd", "liblmzipf.so")):
        from paper_1810_10045_amd import build
        build.build()
    from paper_1810_10045_amd import lmzipf
    return lmzipf.lib()


def rows_of_a_workgroup(D, dtype):
    """256 threads, a row by as many lanes as it has 16-byte vectors, up to whole waves."""
    vectors = -(-D * (2 if dtype == BF16 else 4) // 16)
    for lanes in (8, 16, 32, 64):
        if vectors <= lanes:
            return 256 // lanes
    return 4 if D <= 512 else 2 if D <= 1024 else 1


# Both sides of each change of form
@pytest.mark.parametrize("D", [1, 7, 32, 33, 64, 65, 128, 129, 256, 257, 512, 513, 1024, 1025, 2048,
                               2049, 4096, 4097, 8192, 8193, 16384])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_one_workgroup_holds(lib, D, dtype):
    need = lib.lm_layer_norm_grad_workspace_bytes
    rows = rows_of_a_workgroup(D, dtype)

    def call(rows, ws, ws_bytes):
        # dh over rstd: refused before anything is launched, behind the workspace's check
        return lib.lm_layer_norm_grad(FAR, D, 2 * FAR, D, None, 0, rows, D, dtype, 3 * FAR, 4 * FAR,
                                      5 * FAR, 0.0, 1, None, 4 * FAR, D, None, 0, 7 * FAR, 8 * FAR,
                                      0, ws, ws_bytes, None)
    for n in {1, rows}:
        assert need(n, D, dtype) == 0
        assert call(n, 9 * FAR, 0) == INVAL == call(n, None, 0)
    for n in (rows + 1, 2 * rows, 2 * rows + 1):
        parts = -(-n // rows)
        assert need(n, D, dtype) == parts * 2 * D * 4
        assert call(n, 9 * FAR, 0) == WORKSPACE
        assert call(n, 9 * FAR, parts * 2 * D * 4 - 1) == WORKSPACE
        assert call(n, 9 * FAR, parts * 2 * D * 4) == INVAL == call(n, None, 1 << 30)
