"""What a drafted row that is not finite does to the nodes that do not see it: nothing, whichever node it is and whichever kernel runs.
The last drafted node is the one whose row fills up the rest of a tile, so it is tried with counts that are no multiple of a tile.
Nodes that do not see the row have to be equal to the run without it: where they had P = 0 times a number they still have 0."""
import numpy as np
import pytest

from _drafts import ancestors
from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu

# few segments (workgroups of 32 query rows), and more row blocks than the chip holds at once (workgroups of 64 and of 128), D = 128 and 64
GEOMETRIES = [(9, 2, 4, 64, 128), (9, 2, 2, 12, 64), (130, 2, 1, 64, 128), (130, 2, 2, 32, 128), (88, 2, 2, 64, 128), (66, 1, 4, 64, 128),
              (400, 2, 4, 16, 64), (400, 2, 1, 64, 64), (260, 2, 5, 14, 64), (100, 2, 4, 64, 64)]
COUNTS = (1, 2, 8, 15, 16, 17, 31, 32, 33, 40, 63, 64)


def _counts(B, W):
    """Ragged: every count that fits; the others W."""
    fit = [n for n in COUNTS if n <= W]
    return np.array([fit[b % len(fit)] if b % 2 else W for b in range(B)], dtype=np.int32)


@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("ragged", [True, False])
@pytest.mark.parametrize("B,H,G,W,D", GEOMETRIES)
def test_the_last_node(B, H, G, W, D, ragged, page):
    nd = _counts(B, W) if ragged else np.full(B, W - 1 if W % 32 == 0 else W, dtype=np.int32)
    c = Case(B=B, H=H, G=G, D=D, W=W, lens=(40, 0, 129, 64), cap=160, nd=nd, page=page, shape="star", seed=B + W)
    torch = c.torch
    c.run()
    c.check()
    clean = c.out.clone()
    seq, last = torch.arange(B, device="cuda"), torch.from_numpy(nd - 1).long().cuda()
    vd, kd = c.vd.clone(), c.kd.clone()
    # [b, i]: node i sees the last one; in a star that is the last one itself
    sees = torch.arange(W, device="cuda") == last.unsqueeze(1)
    real = torch.arange(W, device="cuda") < (last + 1).unsqueeze(1)
    for bad in (float("nan"), float("inf"), -float("inf")):
        for column, key in ((None, False), (D - 1, False), (None, True)):
            c.vd.copy_(vd)
            c.kd.copy_(kd)
            if column is None:
                c.vd[0, seq, last] = bad
            else:
                c.vd[0, seq, last, :, column] = bad
            if key:
                c.kd[0, seq, last] = bad
            c.out.fill_(77.0)
            c.run()
            torch.cuda.synchronize()
            assert torch.equal(c.out[0][real & ~sees], clean[0][real & ~sees])
            assert (c.out[0][~real] == 77.0).all()
            got = c.out[0][sees]
            if column is None:
                assert not torch.isfinite(got).any()
            else:
                hit = got[:, :, column]
                assert (torch.isnan(hit) if bad != bad else hit == bad).all()
                got[:, :, column] = clean[0][sees][:, :, column]
                assert torch.equal(got, clean[0][sees])


@pytest.mark.parametrize("B,H,G,W,D", [(9, 2, 4, 40, 128), (88, 2, 2, 47, 128), (100, 2, 4, 33, 64)])
def test_any_node_of_a_tree(B, H, G, W, D):
    c = Case(B=B, H=H, G=G, D=D, W=W, lens=(40, 0, 129), cap=130, seed=W)
    torch = c.torch
    c.run()
    torch.cuda.synchronize()
    clean, vd = c.out.clone(), c.vd.clone()
    rng = np.random.default_rng(W)
    seq = np.arange(B)
    for bad in (float("nan"), float("inf")):
        node = rng.integers(0, W, size=B)
        node[::5] = W - 1
        sees = torch.from_numpy(np.stack([ancestors(c.parent[b])[:, node[b]] for b in seq])).cuda()
        c.vd.copy_(vd)
        c.vd[0, torch.from_numpy(seq).cuda(), torch.from_numpy(node).cuda()] = bad
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.out[0][~sees], clean[0][~sees])
        got = c.out[0][sees]
        assert (torch.isnan(got) if bad != bad else got == bad).all()
