"""Verification of drafted tokens, against the definition in 64 bits.  Outputs are whole numbers and have to be equal: two 64-bit
sums of the same numbers in another order differ by 1e-16 of their size per term, so a random number would have to fall into
1e-11 of the unit interval for them to disagree."""
import numpy as np
import pytest

from _drafts import make_tree, verify

pytestmark = pytest.mark.gpu


def _case(seed, B, W, V, shape="tree", drafted=True, sharp=2.0, nd=None, pad=0, near=0.5):
    rng = np.random.default_rng(seed)
    logits = rng.standard_normal((B, W, V)) * sharp
    guess = logits + near * rng.standard_normal((B, W, V))

    def soft(x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return (e / e.sum(-1, keepdims=True)).astype(np.float32)
    target, draft = soft(logits), soft(guess) if drafted else None
    parent = make_tree(rng, B, W, shape)
    token = np.zeros((B, W), dtype=np.int32)
    for b in range(B):
        for i in range(1, W):
            row = max(int(parent[b, i]), 0)
            if drafted:
                token[b, i] = rng.choice(V, p=draft[b, row].astype(np.float64) / draft[b, row].astype(np.float64).sum())
            else:
                rank = sum(parent[b, j] == parent[b, i] for j in range(i))
                token[b, i] = np.argsort(-guess[b, row], kind="stable")[rank % V]
    nd = np.full(B, W, dtype=np.int32) if nd is None else np.asarray(nd, dtype=np.int32)
    u, us = rng.random((B, W), dtype=np.float32), rng.random(B, dtype=np.float32)
    return dict(target=target, draft=draft, token=token, parent=parent, nd=nd, u=u, us=us, pad=pad)


def _run(c, ws=None, stream=None):
    import torch
    from paper_2604_18002_amd import binding as ngc
    B, W, V = c["target"].shape

    def rows(x):
        if x is None:
            return None
        t = torch.full((B * W * (V + c["pad"]) + 1,), float("nan"), device="cuda")       # rows at odd places
        t = t[1:] if c["pad"] else t[:-1]
        t.view(B, W, V + c["pad"])[:, :, :V] = torch.from_numpy(x).cuda()
        return t
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()     # noqa: E731
    path = torch.full((B, W), 99, dtype=torch.int32, device="cuda")
    n, nxt = torch.full((B,), 99, dtype=torch.int32, device="cuda"), torch.full((B,), 99, dtype=torch.int32, device="cuda")
    if ws is None:
        ws = torch.zeros(ngc.ngc_verify_workspace_bytes(B, V), dtype=torch.uint8, device="cuda")
    args = (rows(c["target"]), rows(c["draft"]), V + c["pad"], dev(c["token"]), dev(c["parent"]), dev(c["nd"]), B, W, V, dev(c["u"]),
            dev(c["us"]), path, n, nxt, ws)
    ngc.ngc_tree_verify(*args, stream=stream)
    torch.cuda.synchronize()
    assert ws[256:].count_nonzero() == 0 and ws[32:256].count_nonzero() == 0        # as it was found
    return path.cpu().numpy(), n.cpu().numpy(), nxt.cpu().numpy(), ngc.read_status(ws), args


def _check(c, got):
    path, n, nxt = got[:3]
    B, W, V = c["target"].shape
    for b in range(B):
        p, t = verify(c["target"][b], None if c["draft"] is None else c["draft"][b], c["token"][b], c["parent"][b], int(c["nd"][b]),
                      c["u"][b], c["us"][b])
        assert n[b] == len(p) and path[b].tolist() == p + [-1] * (W - len(p)), b
        assert nxt[b] == t, b


@pytest.mark.parametrize("V", [1, 2, 5, 63, 1000, 1023, 1024, 1025, 4099, 20001])
@pytest.mark.parametrize("drafted", [True, False])
def test_vocabularies(V, drafted):
    c = _case(V, 6, 7, V, drafted=drafted, pad=V % 2)
    got = _run(c)
    _check(c, got)
    assert got[3][:8] == [0] * 8


@pytest.mark.parametrize("shape", ["chain", "star", "tree", "forest"])
@pytest.mark.parametrize("W", [1, 2, 33, 64])
@pytest.mark.parametrize("drafted", [True, False])
def test_shapes(shape, W, drafted):
    c = _case(W, 12, W, 301, shape=shape, drafted=drafted, near=1.5, nd=[W] * 10 + [1, 0], pad=3)
    _check(c, _run(c))


@pytest.mark.parametrize("B", [1, 40, 216, 217, 300, 600])
def test_batches(B):
    c = _case(B, B, 3, 2500, shape="star", sharp=1.0, near=2.0)
    _check(c, _run(c))


def test_numbers_at_the_ends():
    for u, us in ((0.0, 0.0), (1 - 2 ** -24, 1 - 2 ** -24), (0.0, 1 - 2 ** -24), (1 - 2 ** -24, 0.0)):
        for drafted in (True, False):
            c = _case(3, 8, 6, 777, drafted=drafted)
            c["target"][:, :, ::3] = 0                       # tokens that cannot be
            c["u"][:], c["us"][:] = u, us
            got = _run(c)
            _check(c, got)
            assert (c["target"][np.arange(8), got[0][np.arange(8), got[1] - 1], got[2]] > 0).all()


def test_greedy_by_one_hot_rows():
    c = _case(5, 20, 8, 50, drafted=False, near=0.3)
    best = c["target"].argmax(-1)
    c["target"][:] = np.eye(50, dtype=np.float32)[best]
    got = _run(c)
    _check(c, got)
    for b in range(20):
        assert got[2][b] == best[b, got[0][b, got[1][b] - 1]]


def test_the_draft_is_the_target():
    """Everything is accepted, and the residual behind a refusal that rounding may bring is empty: then p itself serves."""
    c = _case(6, 10, 5, 333, shape="chain")
    c["draft"] = c["target"].copy()
    got = _run(c)
    _check(c, got)
    assert (got[1] == 5).all()
    c["u"][:] = 1.0                                           # outside [0, 1): u q < p fails, nothing is left
    got = _run(c)
    _check(c, got)
    assert (got[1] == 1).all()


def test_the_same_token_twice_among_siblings():
    for drafted in (True, False):
        c = _case(7, 12, 6, 40, shape="star", drafted=drafted, near=3.0)
        c["token"][:, 1:] = c["token"][:, 1:2]
        c["u"][:] = 0.999
        _check(c, _run(c))


def test_rows_without_probability():
    c = _case(8, 4, 3, 2000, shape="chain", drafted=False)
    c["target"][1] = 0
    c["target"][2] = np.nan
    c["target"][3, :, 5:] = np.nan
    got = _run(c)
    _check(c, got)
    assert got[2][1] == -1 and got[2][2] == -1 and 0 <= got[2][3] < 5
    assert got[3][6] == 2


@pytest.mark.parametrize("shape", ["chain", "star", "tree"])
def test_draft_values_below_zero_and_nan_count_as_zero(shape):
    c = _case(29, 24, 9, 300, shape=shape, near=1.0)
    rng = np.random.default_rng(30)
    raw = c["draft"].copy()
    odd = rng.random(raw.shape)
    raw[odd < 0.1] = -0.25
    raw[odd > 0.9] = np.nan
    for b in range(0, 24, 3):               # proposed tokens among them
        raw[b, np.maximum(c["parent"][b], 0), c["token"][b]] = -1.0 if b % 2 else np.nan
    got = _run(dict(c, draft=raw))
    _check(dict(c, draft=np.maximum(np.nan_to_num(raw, nan=0.0), 0.0)), got)
    assert got[3][:8] == [0] * 8


def test_what_is_out_of_range_is_counted():
    c = _case(9, 3, 6, 100, shape="chain", drafted=False)
    c["token"][0, 2], c["token"][1, 3], c["token"][2, 0] = 100, -1, -50     # the last is the pending token: not looked at
    c["parent"][2, 4] = 5
    ref = {k: (v.copy() if isinstance(v, np.ndarray) else v) for k, v in c.items()}
    ref["parent"][2, 4] = -1
    c["nd"][0] = 99
    got = _run(c)
    _check(ref, got)
    assert got[3][6] == 4


@pytest.mark.parametrize("drafted", [True, False])
def test_emitted_tokens_have_the_target_s_distribution(drafted):
    """Two drafted children of one node; the token that follows node 0 is the accepted child's or the drawn one.  30000
    sequences: a frequency f is off by less than five standard deviations, 5 sqrt(f (1 - f) / 30000)."""
    rng = np.random.default_rng(12)
    V, B = 6, 30000
    p, q = rng.dirichlet(np.ones(V)).astype(np.float32), rng.dirichlet(np.ones(V)).astype(np.float32)
    W = 3
    token = np.zeros((B, W), dtype=np.int32)
    token[:, 1:] = rng.choice(V, size=(B, 2), p=q / q.astype(np.float64).sum()) if drafted else [2, 4]
    c = dict(target=np.broadcast_to(p, (B, W, V)).copy(), draft=np.broadcast_to(q, (B, W, V)).copy() if drafted else None, token=token,
             parent=np.tile(np.int32([-1, 0, 0]), (B, 1)), nd=np.full(B, W, dtype=np.int32), u=rng.random((B, W), dtype=np.float32),
             us=rng.random(B, dtype=np.float32), pad=0)
    path, n, nxt = _run(c)[:3]
    first = np.where(n > 1, token[np.arange(B), path[:, 1] * (n > 1)], nxt)
    f = np.bincount(first, minlength=V) / B
    assert (np.abs(f - p) < 5 * np.sqrt(p * (1 - p) / B) + 1e-6).all()


@pytest.mark.parametrize("B", [2, 60, 300])
def test_what_the_workspace_holds_does_not_matter(B):
    """Other calls leave their scratch behind; only the status words have to be as they leave them."""
    import torch
    from paper_2604_18002_amd import binding as ngc
    c = _case(B, B, 4, 3000, shape="star", near=2.0)
    ws = torch.full((ngc.ngc_verify_workspace_bytes(B, 3000),), 0xA5, dtype=torch.uint8, device="cuda")
    ws[:256] = 0
    _check(c, _run(c, ws=ws))


def test_captured_on_another_stream_and_in_a_cache_s_workspace():
    import torch
    from paper_2604_18002_amd import binding as ngc
    c = _case(13, 5, 6, 5000)
    side = torch.cuda.Stream()
    cache = ngc.Cache.allocate(1, 2, 2, 4, 64, 64)
    cache.len.fill_(64)
    cache.k.normal_()
    cache.v.normal_()
    ws = ngc.allocate_tree_workspace(cache, 6, 5000)
    ws = torch.zeros(max(ws.numel(), ngc.ngc_verify_workspace_bytes(5, 5000)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    got = _run(c, ws=ws, stream=side)
    _check(c, got)
    args = got[4]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ngc.ngc_tree_verify(*args)
    q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    a, b = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 4, 64, device="cuda")
    ngc.ngc_decode_attn(cache, 0, q, 0.125, 0, a, ws)
    for _ in range(3):
        for t in args[11:14]:
            t.fill_(99)
        g.replay()
        ngc.ngc_decode_attn(cache, 0, q, 0.125, 0, b, ws)
        torch.cuda.synchronize()
        _check(c, [t.cpu().numpy() for t in args[11:14]])
        assert torch.equal(a, b)
