"""Replay attention of latent layers where one input is not finite: outputs and gradients are finite exactly where the formulas' are, wherever
the value lies (next to the diagonal, among keys that die midway, far before its queries), and entries that the formulas leave alone
keep their bits."""
import numpy as np
import pytest

from test_gpu_latent_replay import Case

pytestmark = pytest.mark.gpu


def formulas(c):
    """The definitions in 64 bits, pair by pair (what a query does not see is not multiplied by 0 but left out); first trajectory."""
    D, n = c.D, c.lens[0]
    g = lambda x: x[0].double().cpu().numpy()             # noqa: E731
    q, kv, rope, dout = g(c.q), g(c.kv), g(c.rope), g(c.dout)
    death = c.death[0].cpu().numpy()
    r = dict(out=np.zeros((c.T, c.H, D)), lse=np.full((c.H, c.T), -np.inf), dq=np.zeros(q.shape), dkv=np.zeros(kv.shape), drope=np.zeros((c.T, c.E)))
    with np.errstate(all="ignore"):
        for h in range(c.H):
            k, v = np.concatenate([kv[:, h, :D], rope], 1), kv[:, h, D:]
            for i in range(n):
                j = np.flatnonzero((np.arange(c.T) <= i) & (death > i))
                if not len(j):
                    continue
                x = (k[j] * q[i, h]).sum(1) * c.scale
                top = np.nanmax(x) if not np.isnan(x).all() else np.nan
                e = np.exp(x - top)
                p = e / e.sum()
                if top > -np.inf or np.isnan(top):         # (else zeros and -inf, and gradients of weights that are NaN)
                    r["lse"][h, i] = top + np.log(e.sum())
                    r["out"][i, h] = (p[:, None] * v[j]).sum(0)
                ds = p * ((v[j] * dout[i, h]).sum(1) - (dout[i, h] * r["out"][i, h]).sum()) * c.scale
                r["dq"][i, h] = (ds[:, None] * k[j]).sum(0)
                dk = ds[:, None] * q[i, h]
                r["dkv"][j, h, :D] += dk[:, :D]
                r["dkv"][j, h, D:] += p[:, None] * dout[i, h]
                r["drope"][j] += dk[:, D:]
    return r


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("part", ["value", "key", "rope", "query", "dout"])
@pytest.mark.parametrize("at", [1, 31, 70, 128, 179])
def test_one_value(D, part, at):
    T, n = 200, 180
    death = np.full((1, T), 1 << 30)
    death[0, 70], death[0, 32:64], death[0, 1] = 150, 64, 100
    c = Case(71, 1, T, 2, D, n=[n], death=death)
    clean, want_clean = c.run(), formulas(c)
    where = {"value": (c.kv, (0, at, 1, 2 * D - 3)), "key": (c.kv, (0, at, 1, 5)), "rope": (c.rope, (0, at, 3)), "query": (c.q, (0, at, 0, D + 2)),
             "dout": (c.dout, (0, at, 0, 7))}[part]
    kept = where[0][where[1]].clone()
    for odd in (float("nan"), float("inf"), -float("inf")):
        where[0][where[1]] = odd
        got, want = c.run(), formulas(c)
        where[0][where[1]] = kept
        for name in want:
            a = got[name][0].double().cpu().numpy()
            b, a0, b0 = want[name], clean[name][0].double().cpu().numpy(), want_clean[name]
            real = (slice(None), slice(0, n)) if name == "lse" else slice(0, n)
            a, b, a0, b0 = a[real], b[real], a0[real], b0[real]
            assert np.array_equal(np.isfinite(a), np.isfinite(b)), (name, odd, np.argwhere(np.isfinite(a) != np.isfinite(b))[:4])
            if part == "value" and name in ("out", "lse"):
                assert np.array_equal(np.isnan(a), np.isnan(b)), (name, odd)       # an infinity is one
            same = np.isfinite(b) & (b == b0)
            assert np.array_equal(a[same], a0[same]), (name, odd)
