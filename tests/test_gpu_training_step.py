"""A training step of the entry points together: Unique, Seg-Sum and the 8-bit
step of the embedding's touched rows; the relative position bias added to the
attention scores, its gradient, and one AdamW step over the bias table and the
dense parameters. Eager against 64 bits, and captured into a graph against eager."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import moments_ref as R  # noqa: E402
from paper_1810_10045_amd import synth  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda"
B, H, L, DH, V, NB = 2, 4, 70, 16, 900, 32
D = H * DH


@pytest.fixture(scope="module")
def lz():
    from paper_1810_10045_amd import lmzipf
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.device_powers(torch)
    return lmzipf


class Model:
    """One causal attention layer: embedding, the output's weight, the bias table."""

    def __init__(self, lz, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.lz = lz
        self.embed = torch.randn(V, D, generator=gen, device=DEV) * 0.3
        self.weight = torch.randn(D, D, generator=gen, device=DEV) * 0.3
        self.table = torch.randn(NB, H, generator=gen, device=DEV)
        self.target = torch.randn(B, L, D, generator=gen, device=DEV)
        self.buckets = lz.rel_buckets(NB, 40, "causal")
        z = lambda *n: torch.zeros(*n, dtype=torch.uint8, device=DEV)  # noqa: E731
        nb = R.blocks(D)
        self.rows = [z(V, D), z(V, D), z(V, nb), z(V, nb)]
        self.grads = [torch.zeros_like(self.weight), torch.zeros_like(self.table)]
        params = [self.weight, self.table]
        state = [[z(p.numel()) for p in params] for _ in range(2)]
        scales = [[z(R.blocks(p.numel())) for p in params] for _ in range(2)]
        self.dense = [*state[0], *state[1], *scales[0], *scales[1]]
        self.copies = [torch.zeros(p.shape, dtype=torch.bfloat16, device=DEV) for p in params]
        self.plan = lz.adamw_plan(params, self.grads, *state, m_scale=scales[0], v_scale=scales[1],
                                  copies=self.copies, decay=[True, False])
        self.ids = torch.zeros(B * L, dtype=torch.int32, device=DEV)
        self.unique = lz.unique_buffers(B * L, V, torch.int32, torch.device(DEV))
        self.sums = torch.zeros(B * L, D, device=DEV)
        self.err = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.ws = lz.Workspace(DEV)
        self.ws.get(1 << 20)

    def state(self):
        return [self.embed, self.weight, self.table, *self.rows, *self.dense, *self.copies]

    def step(self, n):
        """One step on self.ids; returns the scores with their bias and the gradients used."""
        lz = self.lz
        x = self.embed[self.ids.long()].view(B, L, H, DH).transpose(1, 2).contiguous()
        scores = torch.matmul(x, x.transpose(2, 3).contiguous()) * DH ** -0.5
        biased = lz.rel_bias(self.table, self.buckets, L, L, add=scores)
        p = biased.softmax(-1)
        y = torch.matmul(p, x)
        flat = y.transpose(1, 2).reshape(B * L, D).contiguous()
        dout = (flat @ self.weight - self.target.view(B * L, D)) * (1.0 / (B * L))
        self.grads[0].copy_(flat.t().contiguous() @ dout)
        dy = (dout @ self.weight.t().contiguous()).view(B, L, H, DH).transpose(1, 2).contiguous()
        dp = torch.matmul(dy, x.transpose(2, 3).contiguous())
        ds = p * (dp - (p * dp).sum(-1, keepdim=True))
        lz.rel_bias_grad(ds, self.buckets, out=self.grads[1], ws=self.ws)
        dx = torch.matmul(p.transpose(2, 3).contiguous(), dy)
        dscaled = ds * DH ** -0.5
        dx = dx + torch.matmul(dscaled, x) + torch.matmul(dscaled.transpose(2, 3).contiguous(), x)
        rows = dx.transpose(1, 2).reshape(B * L, D).contiguous()
        u = lz.unique(self.ids, V, out=self.unique, ws=self.ws)
        lz.segsum(rows, u.perm, u.inverse, u.offsets, u.num_unique, out=self.sums,
                  dev_err=self.err, ws=self.ws)
        lz.sparse_apply_q8(self.embed, u.uniq, u.num_unique, self.sums, *self.rows, lr=1e-2,
                           step=n, seed=2 * n, dev_err=self.err)
        lz.adamw(self.plan, lr=1e-2, weight_decay=0.1, step=n, seed=2 * n + 1, dev_err=self.err)
        return biased


def _autograd(m):
    """The same loss's gradients in 64 bits, by torch, from the formula of the bias."""
    embed, weight, table = (t.double().cpu().requires_grad_() for t in (m.embed, m.weight, m.table))
    ids = m.ids.long().cpu()
    x = embed[ids].view(B, L, H, DH).transpose(1, 2)
    i = torch.arange(L)
    d = (i[:, None] - i).clamp(min=0)
    near = NB // 2
    far = near + (torch.log(d.clamp(min=1).double() / near) / np.log(40 / near) * near + 1e-9).floor().long()
    bucket = torch.where(d < near, d, far.clamp(max=NB - 1))
    bias = table[bucket].permute(2, 0, 1).masked_fill(i[:, None] < i, -float("inf"))
    biased = x @ x.transpose(2, 3) * DH ** -0.5 + bias
    y = (biased.softmax(-1) @ x).transpose(1, 2).reshape(B * L, D)
    loss = 0.5 * ((y @ weight - m.target.double().cpu().view(B * L, D)) ** 2).sum() / (B * L)
    return biased.detach(), torch.autograd.grad(loss, (embed, weight, table))


def test_training_step(lz):
    m = Model(lz, 1)
    for n in (1, 2, 3):
        m.ids.copy_(torch.from_numpy(synth.zipf_ids(B * L, V, 1.0, 10 + n, np.int32)))
        want, (ge, gw, gt) = _autograd(m)
        before = [t.cpu().numpy() for t in (m.weight, m.table, m.embed, *m.dense, *m.rows)]
        biased = m.step(n)
        torch.cuda.synchronize()
        lz.check(m.err)
        lz.check(m.unique.dev_err)
        # fp32 chains of sums of at most 140 terms, a softmax and two products between: the
        # norm of the difference is under 1000 half steps of the gradient's own norm
        fin = torch.isfinite(want)
        assert torch.equal(fin, torch.isfinite(biased.cpu()))
        near = lambda a, b: float((a - b).norm()) <= 1000 * R.U32 * float(b.norm())  # noqa: E731
        assert near(biased.double().cpu()[fin], want[fin])
        assert near(m.grads[0].double().cpu(), gw) and near(m.grads[1].double().cpu(), gt)
        U = int(m.unique.num_unique)
        uniq = m.unique.uniq[:U].long().cpu()
        assert near(m.sums[:U].double().cpu(), ge[uniq])
        # the optimizer's steps from the gradients as they were computed: bit for bit
        first = 0
        for i, (p, g, wd) in enumerate(((before[0], m.grads[0], 0.1), (before[1], m.grads[1], 0.0))):
            k = p.size
            old = [before[3 + i + 2 * j] for j in range(4)]
            hyper = (1e-2, 0.9, 0.999, 1e-8, wd, n)
            ref, bound, m8, v8, ms8, vs8, _ = R.step8(
                p.reshape(-1), g.cpu().numpy().reshape(-1), *old, hyper, first + np.arange(k), 2 * n + 1)
            first += R.blocks(k) * 32
            for j, x in enumerate((m8, v8, ms8, vs8)):
                assert np.array_equal(m.dense[i + 2 * j].cpu().numpy(), x), (n, i, j)
            new = (m.weight, m.table)[i]
            assert (np.abs(new.cpu().numpy().reshape(-1).astype(np.float64) - ref) <= bound).all()
            assert torch.equal(m.copies[i], new.bfloat16())
        at = uniq.numpy()
        ref, bound, *state, _ = R.step8(before[2][at], m.sums[:U].cpu().numpy(),
                                        *[x[at] for x in before[11:]],
                                        (1e-2, 0.9, 0.999, 1e-8, 0.0, n),
                                        at[:, None] * D + np.arange(D), 2 * n)
        for x, want_x in zip(m.rows, state):
            assert np.array_equal(x.cpu().numpy()[at], want_x), n
        assert (np.abs(m.embed.cpu().numpy()[at].astype(np.float64) - ref) <= bound).all()
        rest = np.setdiff1d(np.arange(V), at)
        assert np.array_equal(m.embed.cpu().numpy()[rest], before[2][rest])


def test_training_step_in_a_graph(lz):
    """The whole step captured and replayed on new ids and state, eager steps of another
    model between the replays (on another workspace): each replay is the eager step."""
    m, other = Model(lz, 2), Model(lz, 3)
    m.step(5)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        m.step(5)
    for i in range(4):
        ids = torch.from_numpy(synth.zipf_ids(B * L, V, 1.0, 40 + i, np.int32))
        m.ids.copy_(ids)
        other.ids.copy_(ids)
        m.weight.normal_(0, 0.3)
        before = [t.clone() for t in m.state()]
        torch.cuda.synchronize()
        graph.replay()
        other.step(i + 1)
        torch.cuda.synchronize()
        lz.check(m.err)
        after = [t.clone() for t in m.state()]
        [t.copy_(x) for t, x in zip(m.state(), before)]
        two = lz.segsum_two_launches(True)  # the form that a capture takes: the same order of sums
        m.step(5)
        lz.segsum_two_launches(two)
        torch.cuda.synchronize()
        lz.check(other.err)
        assert all(torch.equal(a, b) for a, b in zip(m.state(), after)), i
