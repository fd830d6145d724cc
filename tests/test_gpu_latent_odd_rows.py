"""Attention over latent rows where one of them is not finite: every token that sees it has it in its output and in lse, however few rows share
its tile, its key group or its workgroup, and no other token has."""
import pytest

from test_gpu_latent_attn import Case
from test_gpu_latent_wide import shape

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")

# D, heads, sequences, hint, (row groups, workgroups for a sequence): none share a sequence, and some do, in both shapes
CALLS = [(576, 16, 1, 1, (1, 1)), (576, 16, 1, 257, (1, 5)), (576, 16, 1, 1025, (1, 17)), (576, 128, 2, 257, (1, 5)), (576, 128, 40, 257, (4, 1)),
         (576, 128, 12, 8000, (4, 10)), (288, 16, 1, 1, (1, 1)), (288, 16, 1, 1025, (1, 17)), (288, 128, 100, 257, (4, 1)), (288, 128, 12, 2000, (4, 8))]


@pytest.mark.parametrize("D,Hq,B,hint,want", CALLS)
@pytest.mark.parametrize("n", [1, 17, 65, 129, 257, 641, 1025])
def test_the_newest_row(D, Hq, B, hint, want, n):
    """A row that is the only one of its tile, of its key group or of its share (lengths one above a multiple of 16, 64 ..)."""
    import torch
    c = Case(n, B, Hq, D, 32, [n + 3 * (b % 2) for b in range(B)], max_pages=256)
    assert shape(c, hint) == want
    clean, clean_lse = c.run(hint=hint)
    page, at = int(c.pc.table[0, 0, 0, (n - 1) // 32]), (n - 1) % 32
    kept = c.pc.k_pool[page, at].clone()
    for col in (0, c.R - 1, D - 1):
        for odd in (NAN, INF, -INF):
            c.pc.k_pool[page, at, col] = odd
            out, lse = c.run(hint=hint)
            assert torch.equal(out[0, 1:], clean[0, 1:]) and torch.equal(lse[0, 1:], clean_lse[0, 1:])
            out, lse = out[0, 0, 0].float(), lse[0, 0, 0]
            up = c.q[0, 0, 0, :, col].float() * odd          # the score, but for its finite parts
            assert bool((up != 0).all())
            gone = ~(up < 0)                                 # NaN or infinite: so are the weights
            assert bool(torch.isnan(out[gone]).all()) and not bool(torch.isfinite(lse[gone]).any()), (col, odd)
            if col < c.R:
                assert not bool(torch.isfinite(out[:, col]).any()), (col, odd)
            c.pc.k_pool[page, at] = kept


@pytest.mark.parametrize("D,Hq,B,hint,want", CALLS)
def test_queries_that_are_not_finite(D, Hq, B, hint, want):
    import torch
    c = Case(41, B, Hq, D, 32, [(1, 65, 300)[b % 3] for b in range(B)], max_pages=256)
    assert shape(c, hint) == want
    clean, clean_lse = c.run(hint=hint)
    c.q[0, :, 0, 3, 5] = NAN
    out, lse = c.run(hint=hint)
    assert bool(torch.isnan(out[0, :, 0, 3].float()).all()) and bool(torch.isnan(lse[0, :, 0, 3]).all())
    rest = [h for h in range(Hq) if h != 3]
    assert torch.equal(out[..., rest, :], clean[..., rest, :]) and torch.equal(lse[..., rest], clean_lse[..., rest])


@pytest.mark.parametrize("D,Hq,B,hint,want", CALLS)
def test_a_row_far_below_the_others(D, Hq, B, hint, want):
    """Weights of its whole share that are zero in 32 bits next to the others'."""
    import torch
    n = 1040
    c = Case(42, B, Hq, D, 32, [n] * B, max_pages=256)
    assert shape(c, hint) == want
    pages = c.pc.table[0, 0, 0, :-(-n // 32)].long()
    flat = c.pc.k_pool[pages].reshape(-1, D)
    flat[:, 0] = 200.0
    flat[n - 16:, 0] = -200.0                                # scores 230 and more below the rest's
    flat[n - 7, 1] = NAN
    c.pc.k_pool[pages] = flat.view(-1, 32, D)
    c.q[..., 0] = 8.0
    out, lse = c.run(hint=hint)
    assert bool(torch.isnan(out[0, 0].float()).all()) and bool(torch.isnan(lse[0, 0]).all())
    assert B == 1 or bool(torch.isfinite(out[0, 1:].float()).all())


def formula(rows, q, scale, R):
    """All rows seen, in 64 bits, term by term: a score of minus infinity is a weight of 0 (and 0 times infinity NaN)."""
    import torch
    x = (q.unsqueeze(1) * rows).sum(-1) * scale
    p = torch.softmax(x, 1)
    out = torch.stack([(p[h].unsqueeze(1) * rows[:, :R]).sum(0) for h in range(q.shape[0])])
    return x, out, torch.logsumexp(x, 1)


@pytest.mark.parametrize("n", [60, 150])
@pytest.mark.parametrize("D,Hq,B,hint,want", CALLS + [(576, 40, 32, 257, (4, 1)), (288, 65, 32, 257, (4, 1))])
def test_as_the_formula_has_it(D, Hq, B, hint, want, n):
    """Finite where the formula is, whether all of the workgroup's queries see the tile or not; and there within the bounds of the other rows."""
    import torch
    from _latent import attention
    W = 1 if (Hq, B) not in ((40, 32), (65, 32)) else 4
    c = Case(43, B, Hq, D, 32, [n] * B, W, max_pages=256)
    assert shape(c, hint) == want
    clean, clean_lse = c.run(hint=hint)
    for at in (3, n - 23, n - 21, n - 7, n - 3, n - 1):
        page, row = int(c.pc.table[0, 0, 0, at // 32]), at % 32
        kept = c.pc.k_pool[page, row].clone()
        for col in (7, c.R - 1, c.R, D - 2):
            for odd in (NAN, INF, -INF):
                c.pc.k_pool[page, row, col] = odd
                out, lse = c.run(hint=hint)
                rows = c.rows(0, 0)
                c.pc.k_pool[page, row] = kept
                assert torch.equal(out[0, 1:], clean[0, 1:]) and torch.equal(lse[0, 1:], clean_lse[0, 1:])
                for i in range(W):
                    limit = n - W + i + 1
                    if at >= limit:                      # not seen
                        assert torch.equal(out[0, 0, i], clean[0, 0, i]) and torch.equal(lse[0, 0, i], clean_lse[0, 0, i])
                        continue
                    q = c.q[0, 0, i].double()
                    x, o, z = formula(rows[:limit], q, c.scale, c.R)
                    assert torch.equal(torch.isfinite(out[0, 0, i].float()), torch.isfinite(o)), (at, col, odd, i)
                    assert torch.equal(torch.isfinite(lse[0, 0, i]), torch.isfinite(z)), (at, col, odd, i)
                    left = x[:, at] == -INF              # heads without this row
                    others = torch.cat([rows[:at], rows[at + 1:limit]])
                    o, z, tol, tol_z = attention(others, q[left], torch.full((int(left.sum()),), limit - 1, device="cuda"), c.scale, c.R)
                    good = (out[0, 0, i, left].double() - o).abs() <= tol
                    good[:, col:col + 1] |= col < c.R    # (NaN there)
                    assert bool(good.all()) and bool(((lse[0, 0, i, left].double() - z).abs() <= tol_z).all()), (at, col, odd, i)
