"""Scores of any size that 32 bits hold: one key has the weight 1 whatever its score is, keys far apart leave the largest alone, and
differences count where the scores are large.

Queries are 1 in one column, keys a number in it: scores and their differences are exact.  A largest score's weight may be any power of two
near 1 (the exponents' reference is rounded) as long as all keys share it: its three parts times a value, added, are off by 3 * 2^-23 of the
value, the quotient by 2^-23, what the parts leave out is 2^-24: less than 5 * 2^-23 together.  The log-sum-exp is a score times log2 e
and back: two rounded constants and two products, 4 * 2^-24 of it, one more where the logarithm of several keys is added, and 2^-20
for that logarithm (below 8.3, a few units in its last place)."""
import numpy as np
import pytest

from test_gpu_tree_attn import MANY, Case

pytestmark = pytest.mark.gpu
GEOMETRIES = [(3, 2, 4, 5, 128), (2, 2, 8, 16, 64), (40, 4, 2, 16, 128)] + MANY[:3] + MANY[6:8]
SIZES = [1.375 * 2.0 ** e for e in (10, 23, 24, 25, 30, 34, 60, 100, 126)]


def _case(B, H, G, W, D, lens, cap, **kw):
    c = Case(B=B, H=H, G=G, D=D, W=W, lens=lens, cap=cap, shape="star", **kw)
    c.q.zero_()
    c.q[..., 0] = 1.0
    return c


VALUE_TOL = 5 * 2.0 ** -23


def _same(got, value):
    return ((got - value).abs() <= VALUE_TOL * value.abs()).all()


def _lse_ok(lse, score, keys=1):
    assert np.abs(lse.double().cpu().numpy() - (score + np.log(keys))).max() <= abs(score) * 5 * 2.0 ** -24 + 2.0 ** -20


@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("B,H,G,W,D", GEOMETRIES)
def test_one_key(B, H, G, W, D, sign):
    """Empty caches and nothing but roots: every node sees itself."""
    c = _case(B, H, G, W, D, (0,), 4)
    torch = c.torch
    c.parents.fill_(-1)
    want = c.vd[0].float().repeat_interleave(G, 2)
    for size in SIZES:
        c.kd.zero_()
        c.kd[..., 0] = sign * size
        c.run(scale=1.0)
        torch.cuda.synchronize()
        assert _same(c.out[0], want), size
        _lse_ok(c.lse[0], sign * size)


@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("B,H,G,W,D", GEOMETRIES)
@pytest.mark.parametrize("page", [0, 32])
def test_the_largest_of_many(B, H, G, W, D, page, sign):
    """Cached keys at 9/8 of a size, but one at the size itself; below zero that one is the largest, above zero the others share.
    Keys of one value leave the mean of their values: three products a key, each added to a sum below 5 n with an error of 2^-23 of it, and
    the sum divided by n: 3 n * 5 * 2^-23."""
    n, at = 300, 217
    c = _case(B, H, G, W, D, (n,), 320, page=page, seed=7)
    torch = c.torch
    c.kd.zero_()
    c.parents.fill_(-1)
    v = np.stack([np.stack([c.rows(0, b, h)[1] for h in range(H)]) for b in range(B)]).astype(np.float64)      # [B, H, n, D]
    others = np.delete(v, at, 2).mean(2) if sign > 0 else v[:, :, at]
    for size in SIZES[1:]:
        if page:
            pages = c.cache.table[0, :, :, :-(-n // page)].long()
            k = torch.zeros(B, H, pages.shape[2] * page, D, device="cuda", dtype=torch.bfloat16)
            k[:, :, :, 0] = sign * size * 1.125
            k[:, :, at, 0] = sign * size
            c.cache.k_pool[pages.flatten()] = k.view(-1, page, D)
        else:
            c.cache.k[0, :, :, :n] = 0
            c.cache.k[0, :, :, :n, 0] = sign * size * 1.125
            c.cache.k[0, :, :, at, 0] = sign * size
        c.kd[..., 0] = -1.5 * size           # and the drafts below all of them
        c.run(scale=1.0)
        torch.cuda.synchronize()
        got = c.out[0].cpu().numpy().reshape(B, W, H, G, D)
        want = others[:, None, :, None]
        assert (np.abs(got - want) <= (3 * n * 5 * 2.0 ** -23 if sign > 0 else VALUE_TOL * np.abs(want))).all(), size
        _lse_ok(c.lse[0], size * 1.125 if sign > 0 else -size, n - 1 if sign > 0 else 1)


@pytest.mark.parametrize("B,H,G,W,D", GEOMETRIES)
def test_shared_segments(B, H, G, W, D):
    """The partials of workgroups, and of their waves, are joined at the same size."""
    n = 1800
    c = _case(B, H, G, W, D, (n,), 1801, seed=9)
    torch = c.torch
    c.kd.zero_()
    c.parents.fill_(-1)
    for size in (1.375 * 2.0 ** 26, 1.375 * 2.0 ** 40, 1.375 * 2.0 ** 100):
        for at in (0, 700, n - 1):
            c.cache.k[0, :, :, :n] = 0
            c.cache.k[0, :, :, :n, 0] = -1.25 * size
            c.cache.k[0, :, :, at, 0] = -size
            c.kd[..., 0] = -1.5 * size
            c.run(scale=1.0)
            torch.cuda.synchronize()
            assert _same(c.out[0], c.cache.v[0, :, :, at].float().repeat_interleave(G, 1).unsqueeze(1))
            _lse_ok(c.lse[0], -size)


def test_a_chain_is_what_decode_steps_give():
    """Large scores of general inputs: the same key wins."""
    c = Case(B=3, H=2, G=4, W=6, shape="chain", lens=(37, 64, 1), cap=300, seed=23)
    ngc, torch = c.ngc, c.torch
    c.cache.k.mul_(2.0 ** 60)
    c.kd.mul_(2.0 ** 60)
    c.run()
    ws = ngc.allocate_workspace(c.cache, 1)
    out = torch.zeros(3, 8, c.D, device="cuda")
    for i in range(6):
        ngc.ngc_decode_step(c.cache, 0, c.kd[0, :, i].contiguous(), c.vd[0, :, i].contiguous(), None, c.q[0, :, i].contiguous(),
                            c.D ** -0.5, 0, out, ws)
        assert torch.isfinite(out).all() and torch.allclose(out, c.out[0, :, i], atol=1e-5)
