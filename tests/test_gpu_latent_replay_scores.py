"""Replay attention of latent layers with scores of any size that 32 bits hold: one key has the weight 1 whatever its score is, keys far apart
leave the largest alone, and differences count where the scores are large.

Queries are 1 in one column of each part, keys a number in it, the scale is 1: scores and their differences are exact.  A largest score's
weight may be any power of two near 1 as long as all keys share it, rounded to bf16 (2^-8), as the output is: 2^-7 of the values.  The
log-sum-exp is a score times log2 e and back, two rounded constants and two products, 4 * 2^-24 of it, one more where a logarithm is added, and
2^-20 for that logarithm.  The gradients' weights are exponentials of score - lse, lse off by that much, and of its product with log2 e:
2^-22 of it (and 2^-8 for bf16)."""
import numpy as np
import pytest

from test_gpu_latent_replay import Case

pytestmark = pytest.mark.gpu
SIZES = [1.375 * 2.0 ** e for e in (3, 10, 13, 23, 25, 30, 34, 60, 100, 126)]
HALF = 2.0 ** -8


def _case(D, T, H=2, **kw):
    c = Case(51, 2, T, H, D, **kw)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.kv[..., :D] = 0
    c.rope.zero_()
    c.scale = 1.0
    return c


def _forward(c):
    b = c.buffers()
    c.forward(b)
    return b["out"].double(), b["lse"].double()


def _lse_tol(score):
    return abs(score) * 5 * 2.0 ** -24 + 2.0 ** -20


@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 40, 200])
def test_one_key(D, T, sign):
    """Every position sees itself alone."""
    import torch
    c = _case(D, T, death=np.tile(np.arange(T) + 1, (2, 1)))
    v = c.kv[..., D:].double()
    for size in SIZES:
        c.kv[..., 0] = sign * size
        out, lse = _forward(c)
        assert bool(((out - v).abs() <= 2 * HALF * v.abs()).all()), size
        assert bool(((lse - sign * size).abs() <= _lse_tol(size)).all()), size
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("D", [64, 128])
def test_the_largest_of_many(D, sign):
    """Keys at 9/8 of a size, but one at the size itself: below zero that one is the largest from its position on, and those before share;
    above zero the others share."""
    import torch
    T, at = 200, 77
    c = _case(D, T)
    v = c.kv[..., D:].double()
    count = torch.arange(1, T + 1, device="cuda").view(1, T, 1, 1).double()
    without = v.clone()
    without[:, at] = 0
    for size in SIZES[1:-1]:
        c.kv[..., 0] = sign * size * 1.125
        c.kv[:, at, :, 0] = sign * size
        out, lse = _forward(c)
        others = (without.cumsum(1), without.abs().cumsum(1)) if sign > 0 else (v.cumsum(1), v.abs().cumsum(1))
        n = count - (count > at).double() if sign > 0 else count
        want, mag = others[0] / n, others[1] / n
        top, keys = torch.full((T,), sign * size * 1.125, dtype=torch.float64, device="cuda"), n.view(T)
        if sign < 0:
            want[:, at:], mag[:, at:] = v[:, at:at + 1], v[:, at:at + 1].abs()
            top[at:], keys = -size, torch.where(torch.arange(T, device="cuda") < at, keys, torch.ones_like(keys))
        assert bool(((out - want).abs() <= 2 * HALF * mag + HALF * want.abs()).all()), size
        assert bool(((lse - (top + keys.log())).abs() <= _lse_tol(1.125 * size)).all()), size


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("base", [0.0, 1024.0, 4096.0, 2.0 ** 15, -2.0 ** 20, 2.0 ** 20])
def test_differences_count(D, base):
    """Scores of a size and a multiple of 1/8, in eight columns' sum: the weights are those of the differences.  Rows whose scores rise, too."""
    import torch
    T = 200
    for rising in (False, True):
        c = _case(D, T)
        c.q[..., D] = 1.0                       # (of the rotary part)
        gen = torch.Generator(device="cuda").manual_seed(5)
        add = torch.randint(-16, 17, (2, T), generator=gen, device="cuda") / 8
        if rising:
            add = torch.arange(T, device="cuda").expand(2, T) * 0.5
        c.kv[..., 0] = base
        c.rope[..., 0] = add
        assert torch.equal(c.rope[..., 0].float(), add.float())
        out, lse = _forward(c)
        x = add.double().unsqueeze(1).expand(2, T, T).masked_fill(torch.arange(T, device="cuda").unsqueeze(1) < torch.arange(T, device="cuda"), -np.inf)
        p = torch.softmax(x, -1)
        v = c.kv[..., D:].double()
        for h in range(c.H):
            want, mag = torch.bmm(p, v[:, :, h].contiguous()), torch.bmm(p, v[:, :, h].abs().contiguous())
            # (the weights' sum, and what a moved reference leaves of 2^-12 in the weights before it: below 2^-19)
            assert bool(((out[:, :, h] - want).abs() <= mag * (HALF + 2.0 ** -14) * (1 + HALF) + HALF * want.abs()).all()), (rising, h)
        z = torch.logsumexp(x, -1) + base
        assert bool(((lse - z.unsqueeze(1)).abs() <= _lse_tol(abs(base) + 100)).all()), rising


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("base", [0.0, -1024.0, 4096.0, 2.0 ** 15])
def test_gradient_of_the_values(D, base):
    """dV = P^T dO, P from the scores and lse."""
    import torch
    T = 200
    c = _case(D, T)
    c.q[..., D] = 1.0
    gen = torch.Generator(device="cuda").manual_seed(6)
    add = torch.randint(-16, 17, (2, T), generator=gen, device="cuda") / 8
    c.kv[..., 0] = base
    c.rope[..., 0] = add
    b = c.run()
    x = add.double().unsqueeze(1).expand(2, T, T).masked_fill(torch.arange(T, device="cuda").unsqueeze(1) < torch.arange(T, device="cuda"), -np.inf)
    pt = torch.softmax(x, -1).transpose(1, 2).contiguous()
    e = (abs(base) + 4) * 2.0 ** -22 + 2.0 ** -20
    for h in range(c.H):
        g = c.dout[:, :, h].double().contiguous()
        want, mag = torch.bmm(pt, g), torch.bmm(pt, g.abs())
        got = b["dkv"][:, :, h, D:].double()
        assert bool(((got - want).abs() <= mag * (HALF + e) * (1 + HALF) + HALF * want.abs()).all()), h


@pytest.mark.parametrize("D", [64, 128])
def test_large_scales(D):
    """Scales up to the largest that is accepted: the largest score alone is left."""
    import torch
    T, at = 130, 40
    c = _case(D, T)
    v = c.kv[..., D:].double()
    c.kv[..., 0] = 2.0 ** -4
    c.kv[:, at:, :, 0] = 2.0 ** -3
    c.kv[:, at + 1:, :, 0] = 2.0 ** -5
    for scale in (2.0 ** 13, 2.0 ** 40, 2.0 ** 126):
        c.scale = scale
        out, lse = _forward(c)
        assert bool(((out[:, at:] - v[:, at:at + 1]).abs() <= 2 * HALF * v[:, at:at + 1].abs()).all()), scale
        n = torch.arange(1, at + 1, device="cuda").view(1, at, 1, 1)
        want, mag = v[:, :at].cumsum(1) / n, v[:, :at].abs().cumsum(1) / n
        assert bool(((out[:, :at] - want).abs() <= 2 * HALF * mag + HALF * want.abs()).all()), scale
        assert bool(((lse[:, :, at:] - scale / 8).abs() <= _lse_tol(scale / 8)).all()), scale
