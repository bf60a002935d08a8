"""The extension module of the short calls is a shorter way to the same library: without it
every call is there, and takes the ctypes way."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

IMPORT = """
import sys, warnings
class Absent:
    def find_spec(self, name, path=None, target=None):
        if name.endswith("_lmzipf_calls"):
            raise {error}
sys.meta_path.insert(0, Absent())
with warnings.catch_warnings(record=True) as told:
    warnings.simplefilter("always")
    from paper_1810_10045_amd import lmzipf as lz
assert any("_lmzipf_calls" in str(w.message) for w in told), told
assert lz.lib().lm_unique_workspace_bytes(1000, 0, 100) > 0
import torch
for f in (lambda: lz.dropout(torch.zeros(2, 3), 0.5, 1), lambda: lz.layer_norm(torch.zeros(2, 3)),
          lambda: lz.token_logprobs(torch.zeros(2, 3))):
    try:
        f()
    except lz.LmError:
        continue
    raise AssertionError("a tensor on the CPU")
print("imported")
"""


@pytest.mark.parametrize("error", ["ModuleNotFoundError(\"No module named '_lmzipf_calls'\")",
                                   "ImportError('_lmzipf_calls.so: undefined symbol')"])
def test_the_library_without_the_extension(error):
    if not os.path.exists(os.path.join(ROOT, "paper_1810_10045_amd", "liblmzipf.so")):
        from paper_1810_10045_amd import build
        build.build()
    r = subprocess.run([sys.executable, "-c", IMPORT.format(error=error)], cwd=ROOT, text=True,
                       capture_output=True, timeout=300)
    assert r.returncode == 0 and "imported" in r.stdout, r.stderr


def test_a_build_without_the_extension(monkeypatch, tmp_path):
    """Where the extension cannot be compiled the library is linked all the same, and the build says
    what failed."""
    sys.path.insert(0, ROOT)
    from paper_1810_10045_amd import build

    def compiler(cmd, check):
        open(cmd[cmd.index("-o") + 1], "w").close()

    def no_headers(verbose):
        raise RuntimeError("no headers")
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path / "objects"))
    monkeypatch.setattr(build.subprocess, "run", compiler)
    monkeypatch.setattr(build, "build_calls", no_headers)
    with pytest.raises(RuntimeError, match="no headers"):
        build.build()
    assert os.path.exists(tmp_path / "lib.so")


@pytest.mark.gpu
def test_the_same_results_without_the_extension(monkeypatch):
    import torch
    from paper_1810_10045_amd import lmzipf as lz
    gen = torch.Generator(device="cuda").manual_seed(3)
    assert lz._calls is not None
    x, add, dy = torch.randn(3, 40, 70, generator=gen, device="cuda").unbind()
    w, b = torch.randn(2, 70, generator=gen, device="cuda").unbind()
    t = torch.randint(0, 70, (40,), generator=gen, device="cuda")

    def run():
        f = lz.layer_norm(x, w, b, add=add, p=0.2, seed=5)
        r = lz.token_logprobs(x, t, top=3)
        return [lz.dropout(x, 0.5, 4, add=add), *f,
                *lz.layer_norm_grad(dy, f.h, f.mean, f.rstd, w, add=add, p=0.2, seed=5), *r,
                lz.token_logprobs_grad(x, t, r.peak, r.log_sum, r.logp)]
    want = run()
    monkeypatch.setattr(lz, "_calls", None)
    assert all(torch.equal(p, q) for p, q in zip(run(), want))
