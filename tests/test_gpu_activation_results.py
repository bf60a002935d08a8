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


# ---------------------------------------------------------------------------
# More logits at the border of the alternatives than are ranked at once
# ---------------------------------------------------------------------------
# Rows of no two equal logits: in lanes' registers (about half of them with 64 alternatives have
# more than 256 candidates, all of them where lanes are left without a logit), by a workgroup each
# and cut into parts
@pytest.mark.parametrize("N,V", [(300, 257), (300, 300), (300, 511), (300, 1000), (40, 2048),
                                 (1030, 2100), (3, 9000)])
@pytest.mark.parametrize("top", [60, 62, 63, 64])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_candidates(lz, N, V, top, dtype):
    gen = torch.Generator(device=DEV).manual_seed(V + top)
    x = torch.stack([torch.randperm(V, generator=gen, device=DEV) for _ in range(N)])
    x = (x - V // 2).to(F32)
    # different bf16 numbers: each integer's own bits, its sign kept
    x = (x.sign() * 2.0 ** (x.abs() // 128 - 40) * (1 + x.abs() % 128 / 128)).to(dtype)
    assert int(torch.unique(x[0]).numel()) >= V - 1  # (0 and the smallest at most are one)
    r = lz.token_logprobs(x, top=top)
    ref = A.logprobs(x.double().cpu().numpy(), None, 1.0, top)
    assert np.array_equal(r.top_ids.cpu().numpy(), ref["top_ids"][0])
    want, tol = ref["top_logp"]
    assert (np.abs(r.top_logp.double().cpu().numpy() - want) <= tol + A.TINY).all()


@pytest.mark.parametrize("V", [1500, 4099, 80_001])
@pytest.mark.parametrize("live", [65, 300, 1100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_alternatives_in_a_few_parts_of_a_row(lz, V, live, dtype):
    """Words left in a few stretches: parts of the row without any, so that every word left is a
    candidate."""
    gen = torch.Generator(device=DEV).manual_seed(V + live)
    for N in (5, 1040):
        x = torch.full((N, V), -INF, dtype=dtype, device=DEV)
        place = torch.arange(live, device=DEV)
        place = place // 8 % 3 * 8 * 64 + place % 8 + place // 24 * 8 * 64 * 3  # a lane's vectors
        place = place[place < V]
        x[:, place] = torch.randn(N, len(place), generator=gen, device=DEV).to(dtype)
        r = lz.token_logprobs(x, top=64)
        rows = [0, 1, N // 2, N - 1]
        ref = A.logprobs(x[rows].double().cpu().numpy(), None, 1.0, 64)
        assert np.array_equal(r.top_ids[rows].cpu().numpy(), ref["top_ids"][0])
        want, tol = ref["top_logp"]
        got = r.top_logp[rows].double().cpu().numpy()
        with np.errstate(invalid="ignore"):
            assert ((got == want) | (np.abs(got - want) <= tol + A.TINY)).all()
