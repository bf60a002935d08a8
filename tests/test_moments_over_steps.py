"""8-bit moments over many steps: the numpy form beside 64 bits (CPU), and the kernels beside
the numpy form, bit for bit, and beside fp32 moments (GPU).

The second moment is kept as its root r, rounded without bias, so the mean of r^2 is above v by
the rounding's variance, s^2 f (1 - f) with s the step of the grid and f the place between two
codes. r was a code before the step, so f (1 - f) s is at most the distance moved, |r' - r| =
c |g^2 - v| / (r' + r), c = 1 - beta2, and s at most r' / 8 in the grid's normal range: the
variance is at most c |g^2 - v| / 16 where r' is near r, under c (E g^2 + v) / 16 in the mean.
With v = beta2 v + c E g^2 + variance that is E g^2 <= v <= (1 + 1/16) / (1 - 1/16) E g^2 =
1.133 E g^2; r' / (r' + r) up to 0.52 instead of a half makes it 1.15. For normal gradients
E |g^2 - v| is 0.97 E g^2 and s about r / 11: 4 to 5% are expected."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import moments_ref as M  # noqa: E402

HIGH = 1.15
DEV = "cuda"


def test_second_moment_over_many_steps():
    """From zero, beside 64 bits: the mean of v between E g^2 and the bound above it, its root
    unbiased to half of that, in every place of a block's normal range."""
    rng = np.random.default_rng(1)
    nb, b2, steps = 256, np.float32(0.99), 2500
    c2 = np.float32(1) - b2
    size = np.exp2(-np.repeat(np.arange(4) * 4.0, nb // 4))[:, None] * np.ones((1, 32))
    size[:, :2] = 1.0  # these set the block's scale; the others lie 0, 4, 8 or 12 bits below
    v, vs = np.zeros(nb * 32, np.uint8), np.zeros(nb, np.uint8)
    total, roots, n = np.zeros((nb, 32)), np.zeros((nb, 32)), 0
    for t in range(steps):
        g = (rng.normal(0, 1, (nb, 32)) * size).astype(np.float32).ravel()
        r = M.decode(v, vs).astype(np.float32)
        v1 = (r * r) * b2 + (g * c2) * g
        v, vs = M.encode(np.sqrt(v1), rng.integers(0, 1 << 20, nb * 32) / 2.0 ** 20, True)
        if t >= 800:  # 0.99^800 = 3e-4 of the start is left
            x = M.decode(v, vs).reshape(nb, 32) / size
            total, roots, n = total + x * x, roots + x, n + 1
    # v scatters by under 0.5 of itself, over some 200 steps at once: 64 x 30 values, 1,700 steps
    noise = 6 * 0.5 / np.sqrt(64 * 30 * (steps - 800) / 200)
    for k in range(4):
        at = slice(k * nb // 4, (k + 1) * nb // 4)
        mean = total[at, 2:].mean() / n
        assert 1 - noise <= mean <= HIGH + noise, (k, mean)
        root = roots[at, 2:].mean() / n
        assert mean - root ** 2 <= 0.25 ** 2, "the root scatters by a quarter of itself"


@pytest.mark.gpu
def test_adamw8_many_steps_bit_for_bit():
    torch = pytest.importorskip("torch")
    from paper_1810_10045_amd import lmzipf as lz
    M.device_powers(torch)
    rng = np.random.default_rng(2)
    n, steps = 32 * 40 + 5, 200
    size = np.exp(rng.normal(-5, 3, n))
    p = rng.normal(0, 0.02, n).astype(np.float32)
    state = [np.zeros(k, np.uint8) for k in (n, n, M.blocks(n), M.blocks(n))]
    t = [torch.from_numpy(x).to(DEV) for x in (p, np.zeros(n, np.float32), *state)]
    plan = lz.adamw_plan([t[0]], [t[1]], [t[2]], [t[3]], m_scale=[t[4]], v_scale=[t[5]])
    for step in range(1, steps + 1):
        g = (rng.normal(0, 1, n) * size).astype(np.float32)
        t[1].copy_(torch.from_numpy(g))
        hyper = (1e-3, 0.9, 0.99, 1e-8, 0.01, step)
        lz.adamw(plan, lr=1e-3, beta1=0.9, beta2=0.99, weight_decay=0.01, step=step, seed=step)
        ref, bound, *state, _ = M.step8(p, g, *state, hyper, np.arange(n), step)
        for got, want in zip(t[2:], state):
            assert np.array_equal(got.cpu().numpy(), want), step
        p = t[0].cpu().numpy()
        assert (np.abs(p.astype(np.float64) - ref) <= bound).all(), step


@pytest.mark.gpu
def test_adamw8_beside_fp32_moments():
    """2,000 steps on the same gradients: second moments as bounded above, first moments
    without bias."""
    torch = pytest.importorskip("torch")
    from paper_1810_10045_amd import lmzipf as lz
    n, kw = 1 << 16, dict(lr=1e-4, beta1=0.9, beta2=0.99)
    gen = torch.Generator(device=DEV).manual_seed(3)
    size = torch.exp2(-torch.arange(8, device=DEV).repeat_interleave(n // 8) * 2.0)  # whole blocks
    z = lambda d=torch.float32, k=n: torch.zeros(k, dtype=d, device=DEV)  # noqa: E731
    u8, g = torch.uint8, z()
    p8, p32, m32, v32, m8, v8 = z(), z(), z(), z(), z(u8), z(u8)
    ms, vs = z(u8, n // 32), z(u8, n // 32)
    a = lz.adamw_plan([p8], [g], [m8], [v8], m_scale=[ms], v_scale=[vs])
    b = lz.adamw_plan([p32], [g], [m32], [v32])
    means = []
    for step in range(1, 2001):
        g.normal_(generator=gen).mul_(size)
        lz.adamw(a, step=step, seed=step, **kw)
        lz.adamw(b, step=step, **kw)
        if step > 800 and step % 200 == 0:
            r = M.decode(v8.cpu().numpy(), vs.cpu().numpy())
            m = M.decode(m8.cpu().numpy(), ms.cpu().numpy())
            means.append([(r * r / size.double().cpu().numpy() ** 2).mean(),
                          (v32 / size ** 2).mean().item(),
                          ((m - m32.double().cpu().numpy()) / size.double().cpu().numpy()).mean()])
    v8m, v32m, off = np.mean(means, 0)
    # 2^16 values 6 times, 200 steps apart: v8's and v32's own scatter are under 0.5
    noise = 6 * 2 * 0.5 / np.sqrt(6 * n)
    assert v32m * (1 - noise) <= v8m <= v32m * (HIGH + noise), (v8m, v32m)
    # m is 0.23 of the gradient's size; a rounding is within |m| / 8, the last 10 count
    assert abs(off) <= 6 * 0.23 / 8 * np.sqrt(5.3) / np.sqrt(6 * n), off
