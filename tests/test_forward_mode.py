"""Tensors with a forward-mode tangent: a call that autograd does not record would drop it, so
it is refused as one on tensors that require grad is."""
import os

import pytest

torch = pytest.importorskip("torch")
from torch.autograd import forward_ad  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lz():
    if not os.path.exists(os.path.join(ROOT, "paper_1810_10045_amd", "liblmzipf.so")):
        from paper_1810_10045_amd import build
        build.build()
    from paper_1810_10045_amd import lmzipf
    return lmzipf


def calls(lz, device, dual):
    """The calls with one operand after another given its tangent by `dual`."""
    x, v, w = (torch.ones(*s, device=device) for s in ((4, 8), (4,), (8,)))
    t = torch.zeros(4, dtype=torch.int64, device=device)
    b = lz.rel_buckets(8, 16)
    table, scores = torch.ones(8, 2, device=device), torch.ones(1, 2, 3, 5, device=device)
    return [lambda: lz.dropout(dual(x), 0.5, 1), lambda: lz.dropout(x, 0.5, 1, add=dual(x)),
            lambda: lz.layer_norm(dual(x)), lambda: lz.layer_norm(x, dual(w)),
            lambda: lz.layer_norm(x, w, dual(w)), lambda: lz.layer_norm(x, add=dual(x)),
            lambda: lz.layer_norm(x, out=dual(x)),
            lambda: lz.layer_norm_grad(dual(x), x, v, v), lambda: lz.layer_norm_grad(x, dual(x), v, v),
            lambda: lz.layer_norm_grad(x, x, v, v, dual(w)),
            lambda: lz.layer_norm_grad(x, x, dual(v), v), lambda: lz.layer_norm_grad(x, x, v, dual(v)),
            lambda: lz.layer_norm_grad(x, x, v, v, add=dual(x)),
            lambda: lz.token_logprobs(dual(x), t),
            lambda: lz.token_logprobs_grad(dual(x), t, v, v, v),
            lambda: lz.token_logprobs_grad(x, t, v, v, dual(v)),
            lambda: lz.token_logprobs_grad(x, t, dual(v), v, v),
            lambda: lz.token_logprobs_grad(x, t, v, dual(v), v),
            lambda: lz.token_logprobs_grad(x, t, v, v, v, entropy=v, dentropy=dual(v)),
            lambda: lz.token_logprobs_grad(x, t, v, v, v, entropy=dual(v), dentropy=v),
            lambda: lz.rel_bias(dual(table), b, 3, 5), lambda: lz.rel_bias(table, b, 3, 5, add=dual(scores)),
            lambda: lz.rel_bias_grad(dual(scores), b)]


def refused(lz, device):
    dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
    for grad in (True, False):  # no_grad is of reverse mode only
        with forward_ad.dual_level(), torch.set_grad_enabled(grad):
            for call in calls(lz, device, dual):
                with pytest.raises(lz.LmError, match="tangent"):
                    call()


def test_tangents_are_refused(lz):
    refused(lz, "cpu")  # before anything else is looked at


@pytest.mark.gpu
def test_tangents_are_refused_on_the_gpu(lz):
    """Where most of these calls go through the extension module; and tensors without a tangent,
    one that ended with its level, and inference mode are taken as before."""
    refused(lz, "cuda")
    x = torch.randn(4, 8, device="cuda")
    want = lz.layer_norm(x)
    with forward_ad.dual_level():
        d = forward_ad.make_dual(x, torch.ones_like(x))
        assert all(torch.equal(p, q) for p, q in zip(lz.layer_norm(x), want))
        plain = forward_ad.unpack_dual(d).primal
        assert all(torch.equal(p, q) for p, q in zip(lz.layer_norm(plain), want))
        with torch.inference_mode():
            assert all(torch.equal(p, q) for p, q in zip(lz.layer_norm(d), want))
    assert all(torch.equal(p, q) for p, q in zip(lz.layer_norm(d), want))


@pytest.mark.gpu
def test_a_function_with_a_forward_derivative(lz):
    """An autograd.Function around a call has a jvp of its own: dropout is linear."""
    class Drop(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return lz.dropout(x, 0.5, 3)

        @staticmethod
        def jvp(ctx, tangent):
            return lz.dropout(tangent, 0.5, 3)
    x, v = torch.randn(2, 6, 16, device="cuda").unbind()
    with forward_ad.dual_level():
        y, dy = forward_ad.unpack_dual(Drop.apply(forward_ad.make_dual(x, v)))
        assert torch.equal(y, lz.dropout(x, 0.5, 3)) and torch.equal(dy, lz.dropout(v, 0.5, 3))
