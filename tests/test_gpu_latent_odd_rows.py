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
