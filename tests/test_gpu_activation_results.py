"""What the results of dropout, layer norm and the token log probabilities keep to whatever
their inputs are: signs, and memory that is not theirs."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import activations_ref as A  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lz():
    from paper_1810_10045_amd import lmzipf
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return lmzipf


# ---------------------------------------------------------------------------
# Log probabilities are at most 0
# ---------------------------------------------------------------------------
# Rows in some lanes, in a wave's, by a workgroup each, and cut into parts
@pytest.mark.parametrize("N,V", [(512, 3), (512, 98), (512, 1500), (1100, 3001), (24, 9000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", [-INF, -30.0])
def test_log_probabilities_are_not_above_0(lz, N, V, dtype, rest):
    """One word left of each row, or one far above the others: it contributes e^0 to the sum, so
    the sum's logarithm is 0 or more and no probability is above 1."""
    top = torch.linspace(-32, 32, N, device=DEV) + torch.arange(N, device=DEV) % 7 * 0.013
    top = top.to(dtype).to(F32)
    at = torch.arange(N, device=DEV) * 31 % V
    for scale in (1.0, 1 / 0.7, 0.37, 3.0):
        x = (top[:, None] + rest / scale).expand(N, V).to(dtype).contiguous()
        x[torch.arange(N, device=DEV), at] = top.to(dtype)
        r = lz.token_logprobs(x, at, scale=scale, top=2)
        s = float(np.float32(scale))
        ref = A.logprobs(x.double().cpu().numpy(), at.cpu().numpy(), s, 2)
        assert bool((r.log_sum >= 0).all()) and bool((r.entropy >= 0).all())
        assert bool((r.logp <= 0).all()) and bool((r.top_logp <= 0).all())
        assert torch.equal(r.top_logp[:, 0], r.logp)
        for name in ("log_sum", "logp", "top_logp", "entropy"):
            want, tol = ref[name]
            got = getattr(r, name).double().cpu().numpy()
            same = got == want
            with np.errstate(invalid="ignore"):
                assert (same | (np.abs(got - want) <= tol + A.TINY)).all(), (scale, name)
