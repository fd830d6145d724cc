"""Attention of drafted tokens over the dense and the paged cache, against the definition in 64 bits.

Tolerance: a score is D products, exact in fp32, added with at most D roundings of partial sums that stay below about
4 sqrt(D) for the N(0,1) inputs used here: D * 4 sqrt(D) * 2^-24 / sqrt(D) <= 3e-5 in the exponent at D = 128, and as
much relative in a probability; a quotient of two such sums is off by at most twice that, times |V| <= 5 of the output:
3e-4.  The log-sum-exp is off by at most one exponent's error: 3e-5, and its own size (up to 12) times 2^-23."""
import numpy as np
import pytest

from _drafts import make_tree, tree_attention

pytestmark = pytest.mark.gpu
OUT_TOL, LSE_TOL = 3e-4, 4e-5


def _bf16(x, torch):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to("cuda").bfloat16()


def _host(t):
    return t.float().cpu().numpy()


class Case:
    def __init__(self, *, L=1, B=2, H=2, G=4, D=128, cap=200, lens=(100, 57), W=8, shape="tree", page=0, nd=None, seed=0,
                 with_lse=True, ws="tree"):
        import torch
        from paper_2604_18002_amd import binding as ngc
        self.ngc, self.torch = ngc, torch
        rng = np.random.default_rng(seed)
        self.rng, self.L, self.B, self.H, self.G, self.D, self.W = rng, L, B, H, G, D, W
        self.lens = np.zeros((L, B, H), dtype=np.int32)
        for l in range(L):
            for b in range(B):
                for h in range(H):
                    self.lens[l, b, h] = lens[(b * H + h + l) % len(lens)]
        self.parent = make_tree(rng, B, W, shape)
        self.nd = np.full(B, W, dtype=np.int32) if nd is None else np.asarray(nd, dtype=np.int32)
        dev = dict(device="cuda")
        self.n_draft = None if nd is None else torch.from_numpy(self.nd).cuda()
        n = lambda *s: torch.from_numpy(rng.standard_normal(s, dtype=np.float32)).cuda().bfloat16()     # noqa: E731
        self.kd, self.vd, self.q = n(L, B, W, H, D), n(L, B, W, H, D), n(L, B, W, H * G, D)
        if page:
            max_pages = -(-cap // page)
            used = -(-self.lens // page)
            num = int(used.sum()) + 3
            order = rng.permutation(num)
            table = np.full((L, B, H, max_pages), 7 * num, dtype=np.int32)        # what is not in use names no page
            at = 0
            for s in np.ndindex(L, B, H):
                table[s][:used[s]] = order[at:at + used[s]]
                at += used[s]
            self.cache = ngc.PagedCache(n(num, page, D), n(num, page, D), None, torch.from_numpy(table).cuda(),
                                        torch.from_numpy(self.lens).cuda(), torch.zeros(num, dtype=torch.int32, **dev),
                                        torch.zeros(1, dtype=torch.int32, **dev), H * G)
            k, v = _host(self.cache.k_pool), _host(self.cache.v_pool)
            self.rows = lambda l, b, h: tuple(                                              # noqa: E731
                x[table[l, b, h][:used[l, b, h]]].reshape(-1, D)[:self.lens[l, b, h]] for x in (k, v))
            self.call = ngc.ngc_paged_tree_attn
        else:
            self.cache = ngc.Cache(n(L, B, H, cap, D), n(L, B, H, cap, D), torch.from_numpy(self.lens).cuda(), None, H * G)
            for s in np.ndindex(L, B, H):      # rows behind the last one hold anything
                self.cache.k[s][self.lens[s]:] = float("nan")
                self.cache.v[s][self.lens[s]:] = float("nan")
            self.rows = lambda l, b, h: tuple(_host(x[l, b, h, :self.lens[l, b, h]]) for x in (self.cache.k, self.cache.v))  # noqa: E731
            self.call = ngc.ngc_tree_attn
        for b in range(B):                     # so do the drafts behind the last one
            self.kd[:, b, self.nd[b]:] = float("nan")
            self.vd[:, b, self.nd[b]:] = float("nan")
        self.out = torch.full((L, B, W, H * G, D), 77.0, **dev)
        self.lse = torch.full((L, B, W, H * G), 77.0, **dev) if with_lse else None
        self.parents = torch.from_numpy(self.parent).cuda()
        if ws == "tree":
            self.ws = ngc.allocate_tree_workspace(self.cache, W)
        elif page:
            self.ws = ngc.allocate_paged_workspace(self.cache)
        else:
            self.ws = ngc.allocate_workspace(self.cache, 1)

    def run(self, layer=-1, hint=0, stream=None, scale=None):
        cut = (lambda t: t) if layer < 0 else (lambda t: None if t is None else t[layer])
        self.call(self.cache, layer, cut(self.kd), cut(self.vd), self.parents, self.n_draft, self.W, cut(self.q),
                  scale or self.D ** -0.5, hint, cut(self.out), self.ws, stream=stream, lse_out=cut(self.lse))

    def check(self, layers=None, scale=None, tol=OUT_TOL):
        self.torch.cuda.synchronize()
        out = self.out.cpu().numpy()
        lse = None if self.lse is None else self.lse.cpu().numpy()
        q, kd, vd = _host(self.q), _host(self.kd), _host(self.vd)
        for l in range(self.L) if layers is None else layers:
            for b in range(self.B):
                w = self.nd[b]
                assert (out[l, b, w:] == 77.0).all()
                if lse is not None:
                    assert (lse[l, b, w:] == 77.0).all()
                for h in range(self.H):
                    heads = slice(h * self.G, (h + 1) * self.G)
                    k, v = self.rows(l, b, h)
                    o, z = tree_attention(k, v, kd[l, b, :w, h], vd[l, b, :w, h], self.parent[b, :w], q[l, b, :w, heads],
                                          scale or self.D ** -0.5)
                    assert np.abs(out[l, b, :w, heads] - o).max(initial=0) < tol, (l, b, h)
                    if lse is not None:
                        assert np.abs(lse[l, b, :w, heads] - z).max(initial=0) < LSE_TOL, (l, b, h)


EDGES = (0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130)


@pytest.mark.parametrize("page", [0, 32, 64, 128])
@pytest.mark.parametrize("D,G,W", [(128, 4, 8), (64, 4, 3), (128, 7, 9), (64, 16, 5), (128, 6, 33), (64, 1, 64), (128, 1, 1),
                                   (128, 16, 2)])
def test_lengths_around_the_tiles(page, D, G, W):
    c = Case(B=3, H=4, G=G, D=D, W=W, cap=256, lens=EDGES, page=page, seed=D + G + W + page)
    c.run()
    c.check()
    assert c.ngc.read_status(c.ws)[:8] == [0] * 8


@pytest.mark.parametrize("shape", ["chain", "star", "forest", "tree"])
@pytest.mark.parametrize("W", [2, 31, 32, 33, 64])
def test_shapes_of_trees(shape, W):
    c = Case(B=3, H=1, G=2, W=W, shape=shape, lens=(0, 5, 90), nd=(W, W // 2, 1), seed=W)
    c.run()
    c.check()


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("nd", [(0, 3, 11), (11, 0, 0), (1, 10, 0)])
def test_ragged_drafts_leave_the_others_as_they_were(page, nd):
    c = Case(B=3, H=2, G=3, W=11, lens=(70, 300, 0), cap=320, nd=nd, page=page, seed=5)
    c.run()
    c.check()


@pytest.mark.parametrize("lens,B,H,G,W", [((2500,), 1, 2, 4, 5), ((1900, 33), 2, 4, 7, 64), ((5000, 1, 777), 3, 2, 16, 10),
                                          ((700, 64, 0, 1500), 2, 2, 16, 64),
                                          ((900, 1100, 40), 40, 4, 2, 16)])
@pytest.mark.parametrize("ws", ["tree", "cache"])
def test_long_caches_shared_by_workgroups(lens, B, H, G, W, ws):
    c = Case(B=B, H=H, G=G, W=W, lens=lens, cap=max(lens) + 7, ws=ws, seed=B + W)
    for hint in (0, max(lens), 64):        # the hint never changes what is computed
        c.out.fill_(77.0)
        c.run(hint=hint)
        c.check()


def test_layers_one_by_one_and_all_at_once():
    c = Case(L=3, B=2, H=2, G=4, W=6, lens=(80, 3, 150, 64), nd=(6, 4), seed=9)
    c.run(layer=1)
    c.check(layers=[1])
    assert (c.out[0] == 77).all() and (c.out[2] == 77).all()
    one = c.out[1].clone()
    c.run(layer=-1)
    c.check()
    assert c.torch.allclose(c.out[1], one, atol=1e-5)


def test_nothing_is_drafted():
    c = Case(B=2, H=2, G=4, W=5, lens=(80, 300), cap=400, nd=(0, 0), seed=8)
    c.run()
    c.check()
    assert c.ngc.read_status(c.ws)[:8] == [0] * 8


def test_a_full_cache_and_an_odd_capacity():
    for cap in (1, 37, 95, 161):
        c = Case(B=2, H=2, G=5, W=4, lens=(cap, cap - 1), cap=cap, seed=cap)
        c.run()
        c.check()


def test_values_that_are_not_seen_stay_out():
    """A drafted row full of NaN and infinities reaches the nodes that see it, and nobody else."""
    for bad in (float("nan"), float("inf"), -float("inf")):
        c = Case(B=2, H=2, G=4, W=12, shape="tree", lens=(40, 0), seed=3)
        c.run()
        c.torch.cuda.synchronize()
        clean = c.out.clone()
        node = 5
        c.vd[0, :, node] = bad
        c.kd[0, :, node] = bad if bad != bad else 3.0e38
        c.run()
        c.torch.cuda.synchronize()
        from _drafts import ancestors
        for b in range(2):
            sees = ancestors(c.parent[b])[:, node]
            assert 0 < sees.sum() < 12
            assert c.torch.allclose(c.out[0, b][~sees], clean[0, b][~sees], atol=OUT_TOL)
            assert not c.torch.isfinite(c.out[0, b][sees]).any()


def test_scores_that_span_the_exponents():
    """Large scores: the running maximum moves many times, and all weight may end on one key."""
    c = Case(B=2, H=2, G=4, W=9, lens=(300, 75), cap=300, seed=11)
    c.cache.k[0, 0, 0, :300] *= c.torch.linspace(0.1, 12, 300, device="cuda").bfloat16().unsqueeze(1)
    c.q *= 4
    c.run()
    # scores reach 12 * 4 * 5 times those of N(0,1): so does the error of an exponent
    c.torch.cuda.synchronize()
    q, kd, vd = _host(c.q), _host(c.kd), _host(c.vd)
    k, v = c.rows(0, 0, 0)
    o, z = tree_attention(k, v, kd[0, 0, :, 0], vd[0, 0, :, 0], c.parent[0], q[0, 0, :, :4], c.D ** -0.5)
    assert np.abs(c.out[0, 0, :, :4].cpu().numpy() - o).max() < 48 * OUT_TOL
    assert np.abs(c.lse[0, 0, :, :4].cpu().numpy() - z).max() < 48 * LSE_TOL


def test_a_chain_is_what_decode_steps_give():
    c = Case(B=3, H=2, G=4, W=6, shape="chain", lens=(37, 64, 0), cap=300, seed=21)
    c.run()
    ngc, torch = c.ngc, c.torch
    ws = ngc.allocate_workspace(c.cache, 1)
    out = torch.zeros(3, 8, c.D, device="cuda")
    lse = torch.zeros(3, 8, device="cuda")
    for i in range(6):
        ngc.ngc_decode_step(c.cache, 0, c.kd[0, :, i].contiguous(), c.vd[0, :, i].contiguous(), None,
                            c.q[0, :, i].contiguous(), c.D ** -0.5, 0, out, ws, lse_out=lse)
        assert torch.allclose(out, c.out[0, :, i], atol=2 * OUT_TOL)
        assert torch.allclose(lse, c.lse[0, :, i], atol=2 * LSE_TOL)


def test_parents_and_counts_out_of_range_are_counted():
    c = Case(B=2, H=2, G=2, W=5, lens=(20,), nd=(9, -3), seed=1)
    c.parents[0] = c.torch.tensor([-1, 0, 2, 99, -7])
    c.parent[0] = [-1, 0, -1, -1, -1]
    c.nd[:] = (5, 0)
    c.run()
    c.check()
    assert c.ngc.read_status(c.ws)[c.ngc.STATUS_BAD_TREE] == 2 + 3


def test_lengths_out_of_range_are_clamped_and_counted():
    c = Case(B=2, H=1, G=2, W=4, cap=50, lens=(50, 0), seed=2)
    c.cache.len.copy_(c.torch.tensor([[[77], [-5]]]))
    c.run()
    c.check()
    assert c.ngc.read_status(c.ws)[c.ngc.STATUS_LEN_CLAMPED] == 2


def test_offsets_beyond_32_bits():
    import torch
    from paper_2604_18002_amd import binding as ngc
    B, H, D, cap, W = 70, 4, 128, 66000, 3
    k = torch.zeros(1, B, H, cap, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[0, B - 1, H - 1, :300].normal_()
    v[0, B - 1, H - 1, :300].normal_()
    length = torch.zeros(1, B, H, dtype=torch.int32, device="cuda")
    length[0, B - 1, H - 1] = 300
    cache = ngc.Cache(k, v, length, None, H * 2)
    kd, vd = (torch.randn(B, W, H, D, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(B, W, H * 2, D, device="cuda").bfloat16()
    parent = torch.tensor([[-1, 0, 0]] * B, dtype=torch.int32, device="cuda")
    out = torch.zeros(B, W, H * 2, D, device="cuda")
    ngc.ngc_tree_attn(cache, 0, kd, vd, parent, None, W, q, D ** -0.5, 0, out, ngc.allocate_tree_workspace(cache, W))
    o, _ = tree_attention(_host(k[0, -1, -1, :300]), _host(v[0, -1, -1, :300]), _host(kd[-1, :, -1]), _host(vd[-1, :, -1]),
                          [-1, 0, 0], _host(q[-1, :, -2:]), D ** -0.5)
    assert np.abs(out[-1, :, -2:].cpu().numpy() - o).max() < OUT_TOL


def test_captured_and_on_another_stream():
    c = Case(B=2, H=2, G=4, W=8, lens=(900, 70), cap=1000, seed=31)
    torch = c.torch
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(stream=side)
    side.synchronize()
    c.check()
    want = c.out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    for _ in range(3):
        c.out.fill_(77.0)
        c.lse.fill_(77.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want)


def test_the_workspace_serves_decode_in_between():
    c = Case(B=2, H=2, G=4, W=8, lens=(900, 1200), cap=1300, seed=41)
    ngc, torch = c.ngc, c.torch
    q = torch.randn(2, 8, c.D, device="cuda").bfloat16()
    a, b = torch.zeros(2, 8, c.D, device="cuda"), torch.zeros(2, 8, c.D, device="cuda")
    ngc.ngc_decode_attn(c.cache, 0, q, c.D ** -0.5, 0, a, c.ws)
    for _ in range(3):
        c.run()
        ngc.ngc_decode_attn(c.cache, 0, q, c.D ** -0.5, 0, b, c.ws)
        assert torch.equal(a, b)
    c.check()


# More row blocks of 32 than workgroups that the chip holds at once (the last three: three times as many): workgroups of several row blocks
MANY = [(130, 2, 1, 33, 128), (260, 1, 4, 16, 64), (88, 2, 2, 64, 128), (176, 1, 7, 10, 64), (66, 1, 4, 64, 128), (30, 2, 5, 57, 64),
        (400, 2, 4, 16, 64), (260, 2, 5, 14, 64), (100, 2, 4, 64, 64)]


@pytest.mark.parametrize("page", [0, 32, 128])
@pytest.mark.parametrize("B,H,G,W,D", MANY)
def test_many_segments(B, H, G, W, D, page):
    nd = np.random.default_rng(B).integers(0, W + 1, size=B)
    nd[:4] = (0, 1, W, W - 1)
    c = Case(B=B, H=H, G=G, D=D, W=W, cap=256, lens=EDGES, page=page, nd=nd, seed=B + W + page)
    c.run()
    c.check()
    assert c.ngc.read_status(c.ws)[:8] == [0] * 8


@pytest.mark.parametrize("B,H,G,W,D", MANY)
def test_many_segments_shared_by_workgroups(B, H, G, W, D):
    c = Case(B=B, H=H, G=G, D=D, W=W, cap=900, lens=(0, 890, 64, 300, 449), seed=B + W)
    for hint in (0, 200):
        c.out.fill_(77.0)
        c.run(hint=hint)
        c.check()


@pytest.mark.parametrize("B,H,G,W,D", MANY)
def test_many_segments_with_values_that_are_not_seen(B, H, G, W, D):
    from _drafts import ancestors
    for bad in (float("nan"), float("inf")):
        c = Case(B=B, H=H, G=G, D=D, W=W, lens=(40, 0), seed=3)
        c.run()
        c.torch.cuda.synchronize()
        clean = c.out.clone()
        node = W // 2
        c.vd[0, :, node] = bad
        c.kd[0, :, node] = bad if bad != bad else 3.0e38
        c.run()
        c.torch.cuda.synchronize()
        for b in range(0, B, 7):
            sees = ancestors(c.parent[b])[:, node]
            assert 0 < sees.sum() < W
            assert c.torch.allclose(c.out[0, b][~sees], clean[0, b][~sees], atol=OUT_TOL)
            assert not c.torch.isfinite(c.out[0, b][sees]).any()


def test_many_segments_with_parents_counts_and_lengths_out_of_range():
    c = Case(B=264, H=1, G=2, W=17, cap=50, lens=(50, 0, 20), nd=[17] * 262 + [40, -1], seed=1)
    c.parents[0, :5] = c.torch.tensor([-1, 0, 2, 99, -7])
    c.parent[0, :5] = [-1, 0, -1, -1, -1]
    c.nd[262:] = (17, 0)
    c.kd[:, 262:], c.vd[:, 262:] = c.kd[:, :2], c.vd[:, :2]
    c.cache.len[0, 0, 0] = 51
    c.cache.len[0, 1, 0] = -1
    c.run()
    c.check()
    s = c.ngc.read_status(c.ws)
    assert s[c.ngc.STATUS_BAD_TREE] == 2 + 3 and s[c.ngc.STATUS_LEN_CLAMPED] == 2


def test_many_segments_captured():
    c = Case(B=88, H=2, G=2, W=64, lens=(700, 70, 899), cap=1000, seed=31)
    torch = c.torch
    c.run()
    c.check()
    want = c.out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    for _ in range(3):
        c.out.fill_(77.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want)
