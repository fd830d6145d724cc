"""Replay attention of latent layers at the longest trajectories that it takes: outputs and gradients of some positions against the formulas,
those of keys over all queries that see them."""
import numpy as np
import pytest

from test_gpu_latent_replay import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["window", "none evicted at the ends"])
def test_the_longest(D, kind):
    import torch
    T = 131072
    death = np.arange(T) + 200 + (np.arange(T) % 7) * 31
    if kind != "window":                        # a few keys live to the end, others die late
        death[:70] = 1 << 30
        death[5000:5032] = T
        death[T - 3000:] = 1 << 30
    c = Case(81, 1, T, 1, D, death=death[None])
    b = c.run()
    f = lambda x: x[0, :, 0].double()           # noqa: E731
    q, g, k, v = f(c.q), f(c.dout), torch.cat([c.kv[0, :, 0, :D], c.rope[0]], -1).double(), c.kv[0, :, 0, D:].double()
    out, lse, dq, dk, dv = f(b["out"]), b["lse"][0, 0].double(), f(b["dq"]), b["dkv"][0, :, 0, :D].double(), b["dkv"][0, :, 0, D:].double()
    d, at = c.death[0].long(), torch.arange(T, device="cuda")
    half = 2.0 ** -8
    for i in (0, 31, 32, 4095, 65535, 65536, 99999, 131039, 131040, 131071):
        j = torch.nonzero((at <= i) & (d > i)).flatten()
        x = k[j] @ q[i] * c.scale
        p = torch.softmax(x, 0)
        want = p @ v[j]
        # Weights and the output are rounded to bf16.  Scores, of D + E products whose magnitudes add up to 12 or less, are off by 12 (D + E + 4) 2^-23
        # < 2^-11, and a weight, by its exponent and lse, by twice that.
        assert bool(((out[i] - want).abs() <= (p @ v[j].abs()) * (half + 2.0 ** -10) * (1 + half) + half * want.abs()).all()), i
        assert abs(float(lse[i] - torch.logsumexp(x, 0))) < 2.0 ** -11, i
        ds = p * (v[j] @ g[i] - g[i] @ out[i])  # (of the output as it is stored)
        want = ds @ k[j] * c.scale
        slack = (p * (v[j].abs() @ g[i].abs() + g[i].abs() @ out[i].abs())) @ k[j].abs() * 2.0 ** -10
        assert bool(((dq[i] - want).abs() <= ((ds.abs() @ k[j].abs()) * half + slack) * (1 + half) * c.scale + half * want.abs()).all()), i
    delta = (g * out).sum(-1)
    for j in (0, 31, 69, 5000, 5031, 4096, 65535, 65536, 131000, 131039, 131040, 131071):
        i = torch.arange(j, min(int(d[j]), T), device="cuda")
        p = torch.exp(q[i] @ k[j] * c.scale - lse[i])
        want, mag = p @ g[i], p @ g[i].abs()
        steps = 2.0 ** -10 + len(i) * 2.0 ** -24             # the exponents' and the sums' own
        assert bool(((dv[j] - want).abs() <= mag * (half + steps) * (1 + half) + half * want.abs()).all()), j
        ds = p * (g[i] @ v[j] - delta[i])
        size = p * (g[i].abs() @ v[j].abs() + (g[i] * out[i]).abs().sum(-1))
        for got, want, qq in ((dk[j], ds @ q[i][:, :D], q[i][:, :D]), (b["drope"][0, j].double(), ds @ q[i][:, D:], q[i][:, D:])):
            want = want * c.scale
            bound = (ds.abs() * half + size * steps) @ qq.abs() * c.scale
            assert bool(((got - want).abs() <= bound * (1 + half) + half * want.abs()).all()), j
