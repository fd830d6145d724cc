"""The probabilities enter the second product in three bf16 parts, 24 bits: a test that two parts do not pass.

Two cached keys, scores 0 (value 0) and -a (value v), and the node itself at -128 a with the value 0: out = v p / (1 + p), p = e^-a,
1 <= a < 4.  Queries and keys have one column each, so scores are exact.  Relative to the output:
    log2 e rounded to 32 bits      4 * 2^-24          (the exponent times ln 2: a of it)
    the exponent, below 8          ln 2 * 2^-22
    2^x                            2^-23              (one unit in the last place)
    1 + p                          2^-24
    p in three parts               2^-24              (three roundings by at most 2^-8 of what is left, 24 bits; 2^-17 with two)
    three products added           3 * 2^-23
    the quotient                   2^-23              (one unit)
together 1.12e-6.  What p loses shrinks by 1 / (1 + p) in the quotient, so this is an upper bound.  With two parts the largest loss over
these a, computed here, is several times as large."""
import numpy as np
import pytest

from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu
BOUND = 4 * 2.0 ** -24 + np.log(2) * 2.0 ** -22 + 2.0 ** -23 + 2.0 ** -24 + 2.0 ** -24 + 3 * 2.0 ** -23 + 2.0 ** -23
SCORES = np.concatenate([1 + np.arange(128) / 128, 2 + np.arange(128) / 64])


def _rounded(x):
    """To bf16, to nearest, ties to even."""
    u = x.astype(np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).view(np.float32)


def test_two_parts_would_lose_more():
    p = np.exp(-SCORES).astype(np.float32)
    first = _rounded(p)
    second = _rounded(p - first)
    lost = np.abs(p.astype(np.float64) - first - second) / p
    assert lost.max() * 1 / (1 + np.exp(-1.0)) > 3 * BOUND


@pytest.mark.parametrize("B,H,G,W,D", [(4, 2, 4, 8, 128), (4, 2, 4, 8, 64), (130, 2, 1, 33, 128), (88, 2, 2, 64, 128), (400, 2, 4, 16, 64),
                                       (100, 2, 4, 64, 64)])
def test_three_parts(B, H, G, W, D):
    c = Case(B=B, H=H, G=G, D=D, W=W, lens=(2,), cap=8, shape="star", seed=W)
    torch = c.torch
    c.parents.fill_(-1)
    rows = B * W * H * G
    a = np.resize(SCORES, rows).reshape(B, W, H * G)
    c.q.zero_()
    c.q[0, ..., 0] = torch.from_numpy(a).cuda().bfloat16()
    assert (c.q[0, ..., 0].double().cpu().numpy() == a).all()
    c.cache.k[0, :, :, :2] = 0
    c.cache.k[0, :, :, 1, 0] = -1.0
    c.cache.v[0, :, :, 0] = 0
    c.kd.zero_()
    c.kd[..., 0] = -128.0
    c.vd.zero_()
    c.run(scale=1.0)
    torch.cuda.synchronize()
    p = np.exp(-a)
    v = c.cache.v[0, :, :, 1].double().cpu().numpy().repeat(G, 1)[:, None]           # [B, 1, Hq, D]
    want = v * (p / (1 + p))[..., None]
    got = c.out[0].double().cpu().numpy()
    assert (np.abs(got - want) <= BOUND * np.abs(want)).all()
