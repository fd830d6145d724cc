"""Infinities in V that a node does see: weights are positive, so by the formula the output is that infinity (NaN where both signs or a
NaN meet), in those columns and in no others, wherever the row stands and however small its weight is."""
import pytest

from _drafts import ancestors
from test_gpu_tree_attn import MANY, Case

pytestmark = pytest.mark.gpu
INF = float("inf")

# one workgroup, several that share a segment, and workgroups of 64 and 128 query rows
GEOMETRIES = [(2, 2, 4, 3, 128), (2, 2, 4, 9, 64), (1, 2, 8, 40, 128)] + MANY[:3] + MANY[6:8]


def _rows(c, b, h):
    """K and V rows of a cached segment as [n, D] views, and their number."""
    n = int(c.lens[0, b, h])
    if hasattr(c.cache, "table"):
        P = c.cache.k_pool.shape[1]
        pages = c.cache.table[0, b, h, :-(-n // P)].long().tolist()
        return n, lambda x, j: getattr(c.cache, x + "_pool")[pages[j // P], j % P]
    return n, lambda x, j: getattr(c.cache, x)[0, b, h, j]


def _same(got, want):
    import torch
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("lens", [(1, 33, 64, 130), (1, 900, 700, 37)])
@pytest.mark.parametrize("B,H,G,W,D", GEOMETRIES)
def test_cached_rows(B, H, G, W, D, lens, page):
    c = Case(B=B, H=H, G=G, D=D, W=W, lens=lens, cap=960, page=page, seed=W)
    c.run()
    c.check()
    clean = c.out.clone()
    touched = [(b, h) for b in range(B) for h in range(H)][:6]
    want = clean.clone()
    for b, h in touched:
        n, row = _rows(c, b, h)
        row("v", n - 1)[3] = INF                  # the last row, whose copies fill up the tile
        row("v", 0)[5] = -INF
        row("v", n // 2)[8] = INF
        row("v", n // 3)[D - 1] = float("nan")
        row("v", 0)[20] = INF                     # the same infinity twice
        row("v", n - 1)[20] = INF
        heads = want[0, b, :, h * G:(h + 1) * G]
        heads[..., 3], heads[..., 5], heads[..., 8], heads[..., D - 1], heads[..., 20] = INF, -INF, INF, float("nan"), INF
        if n > 1:
            row("v", 0)[22] = INF                 # both signs
            row("v", n - 1)[22] = -INF
            heads[..., 22] = float("nan")
    c.run()
    c.torch.cuda.synchronize()
    _same(c.out, want)


@pytest.mark.parametrize("B,H,G,W,D", GEOMETRIES)
def test_drafted_rows_beside_cached_ones(B, H, G, W, D):
    c = Case(B=B, H=H, G=G, D=D, W=W, lens=(900, 37, 0), cap=901, seed=W + 1)
    c.run()
    c.check()
    clean = c.out.clone()
    node = W - 1
    sees = c.torch.from_numpy(ancestors(c.parent[0])[:, node]).cuda()
    n, row = _rows(c, 0, 0)
    assert n == 900
    c.vd[0, 0, node, 0, 4] = INF
    c.vd[0, 0, node, 0, 6] = INF
    row("v", 2)[6] = -INF
    row("v", 899)[7] = -INF
    c.run()
    c.torch.cuda.synchronize()
    want = clean.clone()
    heads = want[0, 0, :, :G]
    heads[sees, :, 4] = INF
    heads[..., 6] = -INF
    heads[sees, :, 6] = float("nan")
    heads[..., 7] = -INF
    _same(c.out, want)


@pytest.mark.parametrize("B,H,G,W,D", [(1, 1, 4, 3, 128), (130, 2, 1, 33, 128), (88, 2, 2, 64, 128)])
def test_weights_that_are_nothing_in_32_bits(B, H, G, W, D):
    """Key 0 has the score -400, the others 0: e^-400 is 0 in 32 bits and is not 0.  It is in another wave's tile, and in another
    workgroup's, than most keys."""
    c = Case(B=B, H=H, G=G, D=D, W=W, lens=(1500,), cap=1501, seed=3)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.cache.k[0, :, :, :1500] = 0
    c.cache.k[0, :, :, 0, 0] = -400.0
    c.kd.zero_()
    c.cache.v[0, 0, 0, 0, 9] = INF
    c.vd[0, 0, 0, 0, 11] = -INF                   # node 0, seen by all in this tree but with a weight of e^-600
    c.kd[0, 0, 0, 0, 0] = -600.0
    c.run(scale=1.0)
    c.torch.cuda.synchronize()
    sees = c.torch.from_numpy(ancestors(c.parent[0])[:, 0]).cuda()
    got = c.out[0, 0, :, :G]
    assert (got[:, :, 9] == INF).all() and (got[sees][:, :, 11] == -INF).all()
    rest = [d for d in range(D) if d not in (9, 11)]
    assert c.torch.isfinite(got[:, :, rest]).all()
    assert c.torch.isfinite(got[~sees][:, :, 11]).all()
