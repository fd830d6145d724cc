"""Attention over latent rows in the shape that was meant: four row groups of queries a workgroup, or one, with and without a share of a
sequence for several workgroups.  Which one a call takes follows from its sizes alone, and every test here asks for it first."""
import numpy as np
import pytest

from test_gpu_latent_attn import Case

pytestmark = pytest.mark.gpu

LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 191, 192, 193, 255, 256, 257, 300, 383, 385, 1000, 1025, 4097]


def shape(c, hint):
    from paper_2604_18002_amd.probe import ngc_probe_latent_shape
    return ngc_probe_latent_shape(c.D, c.Hq, c.W, c.L * c.B, hint)


def lengths(B, turn=0):
    return [LENGTHS[(i + turn) % len(LENGTHS)] for i in range(B)]


# D, heads, sequences, hint, new tokens, workgroups for a sequence: by sizes that take four row groups
FOUR = [(576, 128, 40, 257, 1, 1), (576, 128, 12, 8000, 1, 10), (576, 128, 4, 16000, 1, 32), (576, 40, 100, 257, 1, 1), (576, 65, 20, 2000, 1, 6),
        (576, 17, 48, 4000, 1, 5), (576, 40, 32, 257, 4, 1), (576, 17, 12, 8000, 4, 10), (288, 128, 100, 257, 1, 1), (288, 128, 12, 2000, 1, 8),
        (288, 64, 48, 4000, 1, 5), (288, 40, 24, 8000, 1, 10), (288, 65, 32, 257, 4, 1), (288, 17, 16, 4000, 4, 8)]


@pytest.mark.parametrize("D,Hq,B,hint,W,splits", FOUR)
def test_lengths(D, Hq, B, hint, W, splits):
    page = 32 if D == 576 else 64
    for turn in range(0, len(LENGTHS), B):
        n_new = None if W == 1 else [(3 * i + turn) % (W + 1) for i in range(B)]
        c = Case(D + turn, B, Hq, D, page, lengths(B, turn), W, n_new, max_pages=16384 // page)
        assert shape(c, hint) == (4, splits)
        c.check(*c.run(hint=hint))


@pytest.mark.parametrize("D,Hq,B,hint,splits", [(576, 128, 12, 8000, 10), (576, 128, 40, 257, 1), (288, 128, 12, 2000, 8), (288, 128, 100, 257, 1)])
def test_large_and_rising_scores(D, Hq, B, hint, splits):
    """Scores far apart, and each row's above all before it: the reference of the exponents moves on every tile."""
    import torch
    c = Case(31, B, Hq, D, 32, lengths(B, 9), spread=30.0, max_pages=512)
    assert shape(c, hint) == (4, splits)
    c.check(*c.run(hint=hint))
    c = Case(32, B, Hq, D, 32, lengths(B, 5), max_pages=512)
    for b in range(B):
        n = int(c.lens[0, b])
        pages = c.pc.table[0, b, 0, :-(-n // 32)].long()
        flat = c.pc.k_pool[pages].reshape(-1, D)
        flat[:, 0] = (torch.arange(flat.shape[0], device="cuda") / 4).bfloat16()
        c.pc.k_pool[pages] = flat.view(-1, 32, D)
    c.q[..., 0] = 8.0
    assert shape(c, hint) == (4, splits)
    c.check(*c.run(hint=hint))


@pytest.mark.parametrize("D,Hq,B,lo,hi", [(576, 64, 64, (1000, (1, 1)), (2000, (4, 4))), (288, 40, 64, (300, (1, 1)), (1000, (4, 4))),
                                          (576, 128, 12, (64, (1, 1)), (2000, (4, 8))), (288, 128, 20, (257, (1, 1)), (1000, (4, 4)))])
def test_both_sides_of_the_rule(D, Hq, B, lo, hi):
    """Sizes that differ in the hint alone take one row group and four."""
    c = Case(33, B, Hq, D, 32, [min(n, 1025) for n in lengths(B)], max_pages=64)
    for hint, want in (lo, hi):
        assert shape(c, hint) == want
        c.check(*c.run(hint=hint))


@pytest.mark.parametrize("D,Hq,lens,hint,want", [(576, 128, [20011], 20011, (1, 32)), (576, 128, [4097, 20011], 64000, (4, 63)), (576, 16, [20011], 20011, (1, 63)),
                                                 (288, 128, [20011, 4097], 20011, (1, 32)), (288, 128, [20011, 513], 64000, (4, 63)), (576, 128, [4097, 20011] + [1] * 38, 257, (4, 1)),
                                                 (288, 128, [4097, 20011] + [65] * 98, 257, (4, 1))])
def test_every_row_is_there_once(D, Hq, lens, hint, want):
    """A row's rotary part is its number in binary, one of +-1 a place, and a head's query that of one row, 512 times: the row's score is at
    least 2 512 scale = 60 above any other's, so the head's output is its latent part as it is, and lse its score.  A row that is left out
    changes all of the output, one that is taken twice lse by log 2."""
    import torch
    c = Case(34, len(lens), Hq, D, 32, lens, max_pages=2048)
    assert shape(c, hint) == want
    E = D - c.R
    bits = torch.arange(E, device="cuda") % 16
    code = lambda j: (((j.unsqueeze(-1) >> bits) & 1) * 2 - 1).bfloat16()          # noqa: E731
    for b, n in enumerate(lens):
        pages = c.pc.table[0, b, 0, :-(-n // 32)].long()
        flat = c.pc.k_pool[pages].reshape(-1, D)
        flat[:, :c.R], flat[:, c.R:] = flat[:, :c.R].sign() * (1 + flat[:, :c.R].abs().clamp(max=8)), code(torch.arange(flat.shape[0], device="cuda"))
        c.pc.k_pool[pages] = flat.view(-1, 32, D)
    c.q.zero_()
    rows = [c.rows(0, b)[:, :c.R].bfloat16() for b in range(len(lens))]
    score = 512.0 * E * c.scale
    assert 2 * 512 * c.scale > 60 and E % 16 == 0
    for at in range(0, max(lens), Hq):
        j = [(at + torch.arange(Hq, device="cuda")) % n for n in lens]
        c.q[0, :, 0, :, c.R:] = torch.stack([512 * code(x) for x in j])
        out, lse = c.run(hint=hint)
        assert bool(((lse - score).abs() < score * 2.0 ** -20).all()), at
        for b in range(len(lens)):
            assert torch.equal(out[0, b, 0], rows[b][j[b]]), (at, b)


@pytest.mark.parametrize("D,Hq,W,lens,n_new,groups", [(576, 128, 200, [700, 77], [200, 77], 4), (288, 128, 130, [1000, 129, 400], [130, 1, 70], 4), (576, 40, 1024, [1024], [1024], 4),
                                                      (288, 20, 300, [2500, 300], [299, 300], 4), (576, 8, 17, [5000], [17], 1), (288, 8, 33, [64, 40], [33, 17], 1)])
def test_prompts_behind_a_prefix(D, Hq, W, lens, n_new, groups):
    c = Case(35, len(lens), Hq, D, 32, lens, W, n_new)
    assert shape(c, c.pc.cap)[0] == groups
    c.check(*c.run())
