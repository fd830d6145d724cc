"""Commits of drafted rows, and forks, ends and packing of a paged cache's sequences, against plain numpy models.  Nothing is
computed: everything has to be equal."""
import numpy as np
import pytest

from _drafts import PagedModel

pytestmark = pytest.mark.gpu


def _drafted(rng, L, B, W, H, D):
    import torch
    x = torch.from_numpy(rng.standard_normal((2, L, B, W, H, D), dtype=np.float32)).cuda().bfloat16()
    return x[0].contiguous(), x[1].contiguous()


def _paths(rng, B, W, most):
    n = rng.integers(0, min(W, most) + 1, size=B).astype(np.int32)
    path = np.full((B, W), -1, dtype=np.int32)
    for b in range(B):
        path[b, :n[b]] = np.sort(rng.permutation(W)[:n[b]])
    return path, n


@pytest.mark.parametrize("L,B,H,D,cap,W,layer", [(3, 5, 2, 128, 90, 8, -1), (2, 3, 4, 64, 33, 64, 1), (1, 1, 1, 64, 1, 1, 0), (2, 40, 3, 128, 64, 17, 0)])
@pytest.mark.parametrize("with_pos", [True, False])
def test_dense_commits(L, B, H, D, cap, W, layer, with_pos):
    import torch
    from paper_2604_18002_amd import binding as ngc
    rng = np.random.default_rng(cap + W)
    cache = ngc.Cache.allocate(L, B, H, H, D, cap, with_pos=with_pos)
    cache.k.normal_()
    cache.v.normal_()
    lens = rng.integers(0, cap + 1, size=(L, B, H)).astype(np.int32)
    cache.len.copy_(torch.from_numpy(lens))
    layers = range(L) if layer < 0 else [layer]
    kd, vd = _drafted(rng, len(layers), B, W, H, D)
    path, n_path = _paths(rng, B, W, 9)
    pos = rng.integers(0, 1000, size=(B, W)).astype(np.int32)
    k, v, p = cache.k.clone(), cache.v.clone(), None if not with_pos else cache.pos.clone()
    full = 0
    for i, l in enumerate(layers):
        for b in range(B):
            for h in range(H):
                n = lens[l, b, h]
                m = min(n_path[b], cap - n)
                full += n_path[b] - m
                for j in range(m):
                    k[l, b, h, n + j], v[l, b, h, n + j] = kd[i, b, path[b, j], h], vd[i, b, path[b, j], h]
                    if with_pos:
                        p[l, b, h, n + j] = int(pos[b, path[b, j]])
                lens[l, b, h] += m
    ws = ngc.allocate_workspace(cache, 1)
    cut = (lambda t: t) if layer < 0 else (lambda t: t[0])
    ngc.ngc_tree_commit(cache, layer, cut(kd), cut(vd), torch.from_numpy(pos).cuda() if with_pos else None,
                        torch.from_numpy(path).cuda(), torch.from_numpy(n_path).cuda(), W, ws)
    torch.cuda.synchronize()
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v) and cache.len.cpu().numpy().tolist() == lens.tolist()
    if with_pos:
        assert torch.equal(cache.pos, p)
    status = ngc.read_status(ws)
    assert status[ngc.STATUS_APPEND_FULL] == full and sum(status) == full


def test_commits_with_what_is_out_of_range():
    import torch
    from paper_2604_18002_amd import binding as ngc
    rng = np.random.default_rng(1)
    cache = ngc.Cache.allocate(1, 4, 2, 2, 64, 20)
    cache.len.copy_(torch.tensor([[[5, 5], [-3, 25], [2, 2], [7, 7]]]))
    kd, vd = _drafted(rng, 1, 4, 6, 2, 64)
    path = torch.tensor([[0, 1, 2, 3, 4, 5]] * 2 + [[0, 9, -2, 1, -1, -1]] + [[0] * 6], dtype=torch.int32, device="cuda")
    n_path = torch.tensor([99, 2, 4, -5], dtype=torch.int32, device="cuda")
    ws = ngc.allocate_workspace(cache, 1)
    ngc.ngc_tree_commit(cache, 0, kd[0], vd[0], None, path, n_path, 6, ws)
    torch.cuda.synchronize()
    assert cache.len.cpu().tolist() == [[[11, 11], [-3, 25], [6, 6], [7, 7]]]
    assert torch.equal(cache.k[0, 0, 1, 5:11], kd[0, 0, :, 1])
    s = ngc.read_status(ws)
    assert s[ngc.STATUS_LEN_CLAMPED] == 2 and s[ngc.STATUS_APPEND_FULL] == 4 and s[ngc.STATUS_BAD_TREE] == 2 + 2


def _pool(rng, L, B, H, D, P, max_pages, lens, spare, with_pos=True):
    """A cache on scattered pages and its model."""
    import torch
    from paper_2604_18002_amd import binding as ngc
    used = -(-lens // P)
    num = int(used.sum()) + spare
    order = rng.permutation(num).astype(np.int32)
    table = np.full((L, B, H, max_pages), -7, dtype=np.int32)
    at = 0
    for s in np.ndindex(L, B, H):
        table[s][:used[s]] = order[at:at + used[s]]
        at += used[s]
    stack = np.concatenate([order[at:], np.full(at, -9, dtype=np.int32)])
    cache = ngc.PagedCache.allocate(L, B, H, H, D, P, max_pages, num, with_pos=with_pos)
    cache.k_pool.normal_()
    cache.v_pool.normal_()
    if with_pos:
        cache.pos_pool.copy_(torch.arange(num * P).view(num, P))
    cache.table.copy_(torch.from_numpy(table))
    cache.len.copy_(torch.from_numpy(lens))
    cache.free_stack.copy_(torch.from_numpy(stack))
    cache.free_count.fill_(spare)
    host = lambda t: t.float().cpu().numpy()     # noqa: E731
    model = PagedModel(table, lens, stack, spare, P, host(cache.k_pool), host(cache.v_pool),
                       cache.pos_pool.cpu().numpy() if with_pos else None)
    return ngc, cache, model, ngc.allocate_tree_workspace(cache, 64)


def _same(cache, model):
    import torch
    torch.cuda.synchronize()
    assert cache.len.cpu().numpy().tolist() == model.len.tolist()
    assert int(cache.free_count) == model.count
    assert cache.free_stack[:model.count].cpu().tolist() == model.stack[:model.count].tolist()
    table = cache.table.cpu().numpy()
    owned = []
    for s in np.ndindex(*model.len.shape):
        n = model.pages(model.len[s])
        assert table[s][:n].tolist() == model.table[s][:n].tolist(), s
        owned += table[s][:n].tolist()
    owned += model.stack[:model.count].tolist()
    assert sorted(owned) == list(range(len(model.stack)))          # every page is in one place
    k, v = cache.k_pool.float().cpu().numpy(), cache.v_pool.float().cpu().numpy()
    assert np.array_equal(k, model.k) and np.array_equal(v, model.v)
    if model.pos is not None:
        assert np.array_equal(cache.pos_pool.cpu().numpy(), model.pos)


GEOMETRIES = [(2, 6, 2, 128, 32, 6), (1, 16, 4, 64, 64, 3), (3, 4, 1, 64, 128, 2), (2, 700, 1, 64, 32, 2)]


@pytest.mark.parametrize("L,B,H,D,P,max_pages", GEOMETRIES)
@pytest.mark.parametrize("spare", [0, 3, 5000])
@pytest.mark.parametrize("layer", [-1, 0])
def test_paged_commits(L, B, H, D, P, max_pages, spare, layer):
    import torch
    rng = np.random.default_rng(P + spare)
    lens = rng.integers(0, max_pages * P + 1, size=(L, B, H)).astype(np.int32)
    lens[0, 0, 0], lens[-1, -1, -1] = max_pages * P - 1, max_pages * P
    ngc, cache, model, ws = _pool(rng, L, B, H, D, P, max_pages, lens, spare)
    W = 64
    kd, vd = _drafted(rng, L if layer < 0 else 1, B, W, H, D)
    pos = rng.integers(0, 1000, size=(B, W)).astype(np.int32)
    for most in (W, 5):
        path, n_path = _paths(rng, B, W, most)
        model.commit(layer, kd.float().cpu().numpy(), vd.float().cpu().numpy(), pos, path, n_path)
        ngc.ngc_paged_tree_commit(cache, layer, kd if layer < 0 else kd[0], vd if layer < 0 else vd[0], torch.from_numpy(pos).cuda(),
                                  torch.from_numpy(path).cuda(), torch.from_numpy(n_path).cuda(), W, ws)
        _same(cache, model)
    status = ngc.read_status(ws)
    assert status[ngc.STATUS_APPEND_FULL] == model.full == sum(status)


def test_a_commit_never_leaves_the_pool():
    import torch
    rng = np.random.default_rng(4)
    ngc, cache, model, ws = _pool(rng, 1, 2, 1, 64, 32, 4, np.int32([[[40], [10]]]), 2)
    cache.table[0, 0, 0, 1] = 9999
    kd, vd = _drafted(rng, 1, 2, 4, 1, 64)
    path = torch.tensor([[0, 1, 2, 3]] * 2, dtype=torch.int32, device="cuda")
    n_path = torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    ngc.ngc_paged_tree_commit(cache, 0, kd[0], vd[0], None, path, n_path, 4, ws)
    torch.cuda.synchronize()
    assert cache.len.cpu().tolist() == [[[40], [12]]]
    s = ngc.read_status(ws)
    assert s[ngc.STATUS_POOL_BOUNDS] == 1 and s[ngc.STATUS_APPEND_FULL] == 3


@pytest.mark.parametrize("L,B,H,D,P,max_pages", GEOMETRIES)
@pytest.mark.parametrize("spare", [0, 17, 5000])
@pytest.mark.parametrize("layer", [-1, 0])
def test_forks(L, B, H, D, P, max_pages, spare, layer):
    import torch
    rng = np.random.default_rng(B + spare)
    lens = rng.integers(0, max_pages * P + 1, size=(L, B, H)).astype(np.int32)
    lens[:, 1] = 0
    ngc, cache, model, ws = _pool(rng, L, B, H, D, P, max_pages, lens, spare)
    for _ in range(3):
        keeps = rng.random(B) < 0.4
        keeps[rng.integers(0, B)] = True
        source = np.where(keeps, rng.choice([-1, -5], size=B), rng.choice(np.nonzero(keeps)[0], size=B)).astype(np.int32)
        own = np.nonzero(keeps)[0][0]
        source[own] = own
        model.fork(layer, source)
        ngc.ngc_paged_fork(cache, layer, torch.from_numpy(source).cuda(), ws)
        _same(cache, model)
    status = ngc.read_status(ws)
    assert status[ngc.STATUS_APPEND_FULL] == model.full == sum(status)


def test_forks_of_what_is_replaced_are_refused():
    import torch
    rng = np.random.default_rng(3)
    lens = rng.integers(1, 100, size=(2, 5, 2)).astype(np.int32)
    ngc, cache, model, ws = _pool(rng, 2, 5, 2, 64, 32, 4, lens, 50)
    source = np.int32([-1, 0, 1, 5, 2])
    model.fork(-1, source)
    ngc.ngc_paged_fork(cache, -1, torch.from_numpy(source).cuda(), ws)
    _same(cache, model)
    assert model.invalid == 3 == ngc.read_status(ws)[ngc.STATUS_BAD_FORK]


@pytest.mark.parametrize("L,B,H,D,P,max_pages", GEOMETRIES)
def test_sequences_that_end(L, B, H, D, P, max_pages):
    import torch
    rng = np.random.default_rng(B)
    lens = rng.integers(0, max_pages * P + 1, size=(L, B, H)).astype(np.int32)
    ngc, cache, model, ws = _pool(rng, L, B, H, D, P, max_pages, lens, 2)
    for layer in (0, -1, -1):
        drop = (rng.random(B) < 0.5).astype(np.int32) * 3
        model.free(layer, drop)
        ngc.ngc_paged_free(cache, layer, torch.from_numpy(drop).cuda(), ws)
        _same(cache, model)
    assert sum(ngc.read_status(ws)) == 0


@pytest.mark.parametrize("L,B,H,D,P,max_pages", GEOMETRIES)
@pytest.mark.parametrize("spare", [0, 1, 40, 3000])
def test_packing(L, B, H, D, P, max_pages, spare):
    import torch
    rng = np.random.default_rng(B + spare)
    lens = rng.integers(0, max_pages * P + 1, size=(L, B, H)).astype(np.int32)
    ngc, cache, model, ws = _pool(rng, L, B, H, D, P, max_pages, lens, spare, with_pos=spare != 40)
    for drop_share in (0.0, 0.5, 1.0):
        drop = (rng.random(B) < drop_share).astype(np.int32)
        model.free(-1, drop)
        ngc.ngc_paged_free(cache, -1, torch.from_numpy(drop).cuda(), ws)
        model.compact()
        ngc.ngc_paged_compact(cache, ws)
        _same(cache, model)
        used = len(model.stack) - model.count
        for s in np.ndindex(L, B, H):
            assert (model.table[s][:model.pages(model.len[s])] < used).all()
    assert sum(ngc.read_status(ws)) == 0


def test_packing_a_table_that_names_no_page():
    import torch
    rng = np.random.default_rng(8)
    ngc, cache, model, ws = _pool(rng, 1, 3, 1, 64, 32, 4, np.int32([[[100], [30], [64]]]), 6)
    cache.table[0, 0, 0, 2] = 1 << 20
    cache.table[0, 2, 0, 1] = -4
    cache.len[0, 1, 0] = 99999
    cache.table[0, 1, 0, 1:] = -1
    ngc.ngc_paged_compact(cache, ws)
    torch.cuda.synchronize()
    s = ngc.read_status(ws)
    assert s[ngc.STATUS_POOL_BOUNDS] == 2 + 3 + 1 and s[ngc.STATUS_LEN_CLAMPED] == 1


def test_pages_of_a_gibibyte():
    import torch
    from paper_2604_18002_amd import binding as ngc
    P = 1 << 22                             # 256 bytes each: K and V of a page are 2^31 bytes
    cache = ngc.PagedCache.allocate(1, 2, 1, 1, 128, P, 1, 3, with_pos=True)
    for pool in (cache.k_pool, cache.v_pool):
        pool.random_(-100, 100)
    cache.pos_pool.random_(0, 1000)
    cache.table.copy_(torch.tensor([2, 0]).view(1, 2, 1, 1))
    cache.len.copy_(torch.tensor([P - 1, 0]).view(1, 2, 1))
    cache.free_stack.copy_(torch.tensor([1, 0, -9]))
    cache.free_count.fill_(2)
    pools = (cache.k_pool, cache.v_pool, cache.pos_pool)
    was = [t[2].clone() for t in pools]
    ws = ngc.allocate_tree_workspace(cache, 1)
    ngc.ngc_paged_fork(cache, -1, torch.tensor([0, 0], dtype=torch.int32, device="cuda"), ws)
    torch.cuda.synchronize()
    assert cache.table.flatten().tolist() == [2, 0] and cache.len.flatten().tolist() == [P - 1, P - 1]
    assert all(torch.equal(t[0], w) and torch.equal(t[2], w) for t, w in zip(pools, was))
    ngc.ngc_paged_free(cache, -1, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), ws)
    for t in pools:
        t[0].zero_()
    ngc.ngc_paged_compact(cache, ws)
    torch.cuda.synchronize()
    assert cache.table.flatten().tolist()[0] == 0 and cache.free_stack.tolist()[:2] == [2, 1] and int(cache.free_count) == 2
    assert all(torch.equal(t[0], w) for t, w in zip(pools, was)) and sum(ngc.read_status(ws)) == 0


def test_captured_page_operations():
    import torch
    rng = np.random.default_rng(6)
    lens = rng.integers(1, 200, size=(2, 8, 2)).astype(np.int32)
    lens[:, 1::2] = 0
    ngc, cache, model, ws = _pool(rng, 2, 8, 2, 128, 32, 8, lens, 200)
    start = [t.clone() for t in (cache.table, cache.len, cache.free_stack, cache.free_count, cache.k_pool, cache.v_pool)]
    source = np.int32([-1, 0, -1, 2, -1, 4, -1, 6])
    drop = np.int32([1, 0, 0, 0, 1, 1, 0, 0])
    src, gone = torch.from_numpy(source).cuda(), torch.from_numpy(drop).cuda()
    kd, vd = _drafted(rng, 2, 8, 5, 2, 128)
    path, n_path = _paths(rng, 8, 5, 5)
    args = torch.from_numpy(path).cuda(), torch.from_numpy(n_path).cuda()

    def work():
        ngc.ngc_paged_fork(cache, -1, src, ws)
        ngc.ngc_paged_tree_commit(cache, -1, kd, vd, None, *args, 5, ws)
        ngc.ngc_paged_free(cache, -1, gone, ws)
        ngc.ngc_paged_compact(cache, ws)
    model.fork(-1, source)
    model.commit(-1, kd.float().cpu().numpy(), vd.float().cpu().numpy(), None, path, n_path)
    model.free(-1, drop)
    model.compact()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        work()
    for _ in range(3):
        for t, x in zip((cache.table, cache.len, cache.free_stack, cache.free_count, cache.k_pool, cache.v_pool), start):
            t.copy_(x)
        cache.pos_pool.copy_(torch.arange(cache.pos_pool.numel()).view_as(cache.pos_pool))
        torch.cuda.synchronize()
        g.replay()
        _same(cache, model)
