"""Pages, tables, lengths and slots from request lengths, and the rows that go there, against the plain form."""
import numpy as np
import pytest

from _latent import extend

pytestmark = pytest.mark.gpu


def make(rng, L, B, H, page, max_pages, lens, spare, D=64, latent=False, pos=False):
    import torch
    from paper_2604_18002_amd import binding as ngc
    lens = np.asarray(lens, np.int32).reshape(L, B, H)
    used = np.where((lens < 0) | (lens > page * max_pages), 0, -(-lens // page))
    total = int(used.sum())
    order = rng.permutation(total + spare).astype(np.int32)
    table = np.full((L, B, H, max_pages), -1, np.int32)
    table[np.arange(max_pages) < used[..., None]] = order[:total]
    stack = np.concatenate([order[total:], order[:total]]).astype(np.int32)
    pc = ngc.PagedCache.allocate_latent(L, B, 16, D, page, max_pages, total + spare, with_pos=pos) if latent else \
        ngc.PagedCache.allocate(L, B, H, H, D, page, max_pages, total + spare, with_pos=pos)
    pc.table.copy_(torch.from_numpy(table))
    pc.len.copy_(torch.from_numpy(lens))
    pc.free_stack.copy_(torch.from_numpy(stack))
    pc.free_count.fill_(spare)
    ws = ngc.allocate_latent_workspace(pc) if latent else ngc.allocate_paged_workspace(pc)
    return pc, ws, table, lens, stack, spare


def check(pc, ws, table, lens, stack, spare, page, n_new, T, layer=-1, slot=None, start=None):
    import torch
    from paper_2604_18002_amd import binding as ngc
    L, B, H, _ = table.shape
    n_layers = L if layer < 0 else 1
    slot = torch.full((n_layers, H, T), 77, dtype=torch.int32, device="cuda") if slot is None else slot
    start = torch.full((B + 1,), 77, dtype=torch.int32, device="cuda") if start is None else start
    new = None if n_new is None else torch.as_tensor(np.asarray(n_new, np.int32)).cuda()
    before = ngc.read_status(ws)
    ngc.ngc_paged_extend(pc, layer, new, T, slot, start, ws)
    w_table, w_len, w_slot, w_start, w_count, counts = extend(table, lens, stack, spare, page, n_new, T, layer)
    np.testing.assert_array_equal(start.cpu().numpy(), w_start)
    np.testing.assert_array_equal(pc.len.cpu().numpy(), w_len)
    np.testing.assert_array_equal(slot.cpu().numpy(), w_slot)
    np.testing.assert_array_equal(pc.table.cpu().numpy(), w_table)
    np.testing.assert_array_equal(pc.free_stack.cpu().numpy(), stack)
    assert int(pc.free_count) == w_count
    status = [x - y for x, y in zip(ngc.read_status(ws), before)]
    assert status[ngc.STATUS_APPEND_FULL] == counts["full"]
    assert status[ngc.STATUS_LEN_CLAMPED] == counts["clamped"]
    assert sum(status) == counts["full"] + counts["clamped"]
    return slot, start, w_table, w_len, w_count


@pytest.mark.parametrize("L,B,H,page,lens,new", [
    (1, 1, 1, 32, (0, 0), (1, 1)),
    (1, 1, 1, 32, (32, 32), (1, 1)),
    (2, 3, 2, 32, (0, 200), (0, 70)),
    (3, 5, 3, 64, (0, 130), (0, 500)),
    (1, 130, 1, 128, (1, 300), (1, 1)),
    (28, 16, 2, 32, (300, 700), (1, 1)),
    (4, 300, 2, 32, (0, 64), (0, 40)),
    (1, 2000, 1, 32, (0, 40), (0, 3)),
    (2, 2, 1, 256, (0, 0), (3000, 5000)),
])
def test_growth(L, B, H, page, lens, new):
    rng = np.random.default_rng(L * 1000 + B)
    n = np.broadcast_to(rng.integers(lens[0], lens[1] + 1, (L, B, 1)), (L, B, H))
    n_new = rng.integers(new[0], new[1] + 1, B)
    max_pages = -(-(lens[1] + new[1]) // page)
    T = max(1, int(n_new.sum()) + int(rng.integers(0, 70)))
    c = make(rng, L, B, H, page, max_pages, n, int(L * B * H * (new[1] // page + 2)))
    check(*c, page, n_new, T)


def test_lengths_that_differ_by_head_and_layer_and_one_layer_at_a_time():
    rng = np.random.default_rng(7)
    L, B, H, page = 3, 9, 4, 32
    c = make(rng, L, B, H, page, 12, rng.integers(0, 200, (L, B, H)), 900)
    pc, ws, table, lens, stack, spare = c
    for layer in (1, 0, 2):
        _, _, table, lens, spare = check(pc, ws, table, lens, stack, spare, page, rng.integers(0, 60, B), 600, layer)


def test_one_token_each_without_counts():
    rng = np.random.default_rng(8)
    c = make(rng, 2, 33, 2, 32, 4, rng.integers(30, 34, (2, 33, 2)), 200)
    check(*c, 32, None, 40)


def test_full_sequences_dry_stack_and_odd_counts():
    rng = np.random.default_rng(9)
    B, page, cap = 12, 32, 96
    lens = np.array([0, 96, 95, 97, -1, 31, 32, 33, 64, 10, 0, 50])
    new = np.array([100, 5, 3, 4, 4, -7, 64, 1, 40, 0, 200, 31])
    for spare in (0, 1, 5, 100):
        c = make(rng, 1, B, 1, page, cap // page, lens, spare)
        check(*c, page, new, 460)
    c = make(rng, 1, B, 1, page, cap // page, lens, 40)
    check(*c, page, new, 150)                   # fewer places than tokens
    c = make(rng, 1, B, 1, page, cap // page, lens, 40)
    check(*c, page, np.full(B, 2 ** 31 - 1), 300)
    c = make(rng, 1, B, 1, page, cap // page, lens, 40)
    check(*c, page, np.full(B, -(2 ** 31)), 3)


def test_a_height_of_the_stack_out_of_range_and_a_page_outside_the_pool():
    import torch
    from paper_2604_18002_amd import binding as ngc
    rng = np.random.default_rng(10)
    pc, ws, table, lens, stack, spare = make(rng, 1, 2, 1, 32, 4, [[20], [40]], 6)
    pc.table[0, 1, 0, 1] = 10 ** 6
    slot, start = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (10, 3))
    ngc.ngc_paged_extend(pc, 0, torch.tensor([3, 4], dtype=torch.int32, device="cuda"), 10, slot, start, ws)
    p = int(table[0, 0, 0, 0]) * 32
    assert slot.tolist() == [p + 20, p + 21, p + 22, -1, -1, -1, -1, -1, -1, -1]
    assert ngc.read_status(ws)[ngc.STATUS_POOL_BOUNDS] == 4
    pc.free_count.fill_(-5)
    ngc.ngc_paged_extend(pc, 0, torch.tensor([30, 0], dtype=torch.int32, device="cuda"), 30, torch.zeros(30, dtype=torch.int32, device="cuda"),
                         start, ws)
    assert pc.len.flatten().tolist() == [32, 44] and int(pc.free_count) == 0
    status = ngc.read_status(ws)
    assert status[ngc.STATUS_POOL_BOUNDS] == 5 and status[ngc.STATUS_APPEND_FULL] == 21


@pytest.mark.parametrize("latent,H,D", [(False, 2, 128), (False, 3, 64), (True, 1, 576), (True, 1, 288)])
@pytest.mark.parametrize("layer", [-1, 1])
def test_rows_reach_their_slots_and_nothing_else_changes(latent, H, D, layer):
    import torch
    from paper_2604_18002_amd import binding as ngc
    rng = np.random.default_rng(H * D)
    L, B, page, T = 2, 5, 32, 333
    pc, ws, table, lens, stack, spare = make(rng, L, B, H, page, 8, np.broadcast_to(rng.integers(0, 90, (L, B, 1)), (L, B, H)), 400, D, latent, True)
    n_layers = L if layer < 0 else 1
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()       # noqa: E731
    pc.k_pool.copy_(new(*pc.k_pool.shape))
    if not latent:
        pc.v_pool.copy_(new(*pc.v_pool.shape))
    n_new = np.array([70, 0, 100, 33, 98])
    slot, *_ = check(pc, ws, table, lens, stack, spare, page, n_new, T, layer)
    k_new = new(n_layers, T, H, D)
    v_new = None if latent else new(n_layers, T, H, D)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") + 1000
    slot[0, 0, 5], slot[-1, H - 1, 17] = -3, pc.k_pool.shape[0] * page         # left out; beyond the pool
    want_k, want_v, want_pos = pc.k_pool.clone().view(-1, D), None if latent else pc.v_pool.clone().view(-1, D), pc.pos_pool.clone().view(-1)
    for l in range(n_layers):
        for h in range(H):
            ok = (slot[l, h] >= 0) & (slot[l, h] < want_k.shape[0])
            at = slot[l, h][ok].long()
            want_k[at] = k_new[l, ok, h]
            want_pos[at] = pos[ok]
            if not latent:
                want_v[at] = v_new[l, ok, h]
    before = ngc.read_status(ws)[ngc.STATUS_POOL_BOUNDS]
    ngc.ngc_paged_fill(pc, layer, k_new, v_new, pos, slot, T, ws)
    assert torch.equal(pc.k_pool.view(-1, D), want_k) and torch.equal(pc.pos_pool.view(-1), want_pos)
    assert latent or torch.equal(pc.v_pool.view(-1, D), want_v)
    assert ngc.read_status(ws)[ngc.STATUS_POOL_BOUNDS] == before + 1
    ngc.ngc_paged_fill(pc, layer, k_new, v_new, None, slot, T, ws)             # positions stay
    assert torch.equal(pc.pos_pool.view(-1), want_pos)


def test_a_prompt_decodes_like_one_entered_token_by_token():
    """The same rows by extend and fill as by one append a token: the attention over them has the same bits."""
    import torch
    from paper_2604_18002_amd import binding as ngc
    B, H, Hq, D, T0 = 3, 2, 12, 128, 75
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn(T0, B, H, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(B, Hq, D, generator=gen, device="cuda").bfloat16()
    one, many = (ngc.PagedCache.allocate(1, B, H, Hq, D, 32, 4, 40) for _ in range(2))
    ws = ngc.allocate_paged_workspace(one)
    for t in range(T0):
        ngc.ngc_paged_append(one, 0, k[t], v[t], None, ws)
    slot = torch.zeros(H, B * T0, dtype=torch.int32, device="cuda")
    start = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    ngc.ngc_paged_extend(many, 0, torch.full((B,), T0, dtype=torch.int32, device="cuda"), B * T0, slot, start, ws)
    packed = [x.transpose(0, 1).reshape(B * T0, H, D).contiguous() for x in (k, v)]
    ngc.ngc_paged_fill(many, 0, *packed, None, slot, B * T0, ws)
    out = [torch.zeros(B, Hq, D, device="cuda") for _ in range(2)]
    for pc, o in zip((one, many), out):
        ngc.ngc_paged_decode_attn(pc, 0, q, D ** -0.5, 0, o, ws)
    assert torch.equal(one.len, many.len) and torch.equal(*out)
