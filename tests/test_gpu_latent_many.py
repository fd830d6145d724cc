"""Attention over latent rows of more sequences than a launch's second dimension counts: all layers of a large batch in one call."""
import numpy as np
import pytest

from _latent import attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,Hq", [(288, 1), (576, 2)])
def test_more_than_65535_sequences(D, Hq):
    import torch
    from paper_2604_18002_amd import binding as ngc
    L, B, pages = 2, 35000, 97
    rng = np.random.default_rng(61)
    pc = ngc.PagedCache.allocate_latent(L, B, Hq, D, 32, 1, pages)
    gen = torch.Generator(device="cuda").manual_seed(61)
    pc.k_pool.normal_(generator=gen)
    pc.table.copy_(torch.from_numpy(rng.integers(0, pages, (L, B, 1, 1)).astype(np.int32)))
    pc.len.copy_(torch.from_numpy(rng.integers(0, 33, (L, B, 1)).astype(np.int32)))
    q = torch.randn(L, B, 1, Hq, D, generator=gen, device="cuda").bfloat16()
    ws, scale, R = ngc.allocate_latent_workspace(pc), (D / 3) ** -0.5, D // 9 * 8
    out, lse = torch.full((L, B, 1, Hq, R), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((L, B, 1, Hq), 7.0, device="cuda")
    ngc.ngc_latent_attn(pc, -1, None, 1, q, scale, 0, out, ws, lse_out=lse)
    assert ngc.read_status(ws)[ngc.STATUS_EMPTY_ATTN] == int((pc.len == 0).sum())
    for l in range(L):
        o, z = torch.full_like(out[l], 3.0), torch.full_like(lse[l], 3.0)
        ngc.ngc_latent_attn(pc, l, None, 1, q[l], scale, 0, o, ws, lse_out=z)
        assert torch.equal(o, out[l]) and torch.equal(z, lse[l])
    for l, b in [(0, 0), (1, 65535 - B), (1, 65536 - B), (1, B - 1)] + [(int(i) // B, int(i) % B) for i in rng.integers(0, L * B, 200)]:
        n = int(pc.len[l, b, 0])
        rows = pc.k_pool[int(pc.table[l, b, 0, 0])][:n].double()
        want, z, tol, tol_z = attention(rows, q[l, b, 0].double(), torch.full((Hq,), n, device="cuda"), scale, R)
        assert bool(((out[l, b, 0].double() - want).abs() <= tol).all()), (l, b)
        assert n == 0 or bool(((lse[l, b, 0].double() - z).abs() <= tol_z).all()), (l, b)
