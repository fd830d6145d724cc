"""Drafted generation as a program runs it: fork the prompt, attend, verify, commit, evict; the tokens are those of generation
one by one."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


class Model:
    """One attention layer between random embeddings and random logits."""

    def __init__(self, V, H, G, D, seed):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = lambda *s: torch.randn(*s, generator=g, device="cuda")     # noqa: E731
        self.q, self.k, self.v = n(V, H * G, D).bfloat16(), n(V, H, D).bfloat16(), n(V, H, D).bfloat16()
        self.head = n(H * G * D, V)

    def logits(self, out):      # [..., Hq, D]
        return out.flatten(-2) @ self.head


def _chains(rng, history, W, V):
    """Drafts: after the pending token what followed it last time, and two random branches."""
    B = len(history)
    parent, token = np.full((B, W), -1, dtype=np.int32), rng.integers(0, V, size=(B, W)).astype(np.int32)
    for b, seq in enumerate(history):
        token[b, 0] = seq[-1]
        for i in range(1, W):
            parent[b, i] = i - 1 if i < W - 2 else 0
    return parent, token


@pytest.mark.parametrize("paged", [False, True])
def test_drafted_generation_emits_what_single_steps_emit(paged):
    import torch
    from paper_2604_18002_amd import binding as ngc
    V, H, G, D, B, W, prompt, steps = 50, 2, 4, 64, 4, 7, 20, 12
    model = Model(V, H, G, D, 5)
    rng = np.random.default_rng(2)
    first = rng.integers(0, V, size=prompt + 1)
    rows_k, rows_v = model.k[torch.from_numpy(first[:-1]).cuda()], model.v[torch.from_numpy(first[:-1]).cuda()]     # [prompt, H, D]

    def fresh():
        cache = ngc.Cache.allocate(1, B, H, H * G, D, 256)
        cache.k[0, :, :, :prompt], cache.v[0, :, :, :prompt] = rows_k.transpose(0, 1), rows_v.transpose(0, 1)
        cache.len.fill_(prompt)
        return cache

    # one by one
    cache = fresh()
    ws = ngc.allocate_workspace(cache, 1)
    out = torch.zeros(B, H * G, D, device="cuda")
    # sequences differ in a second prompt token
    pending = torch.from_numpy(np.int64([first[-1], 3, 7, 11])).cuda()
    single = [pending.tolist()]
    for _ in range(steps * W):
        ngc.ngc_decode_step(cache, 0, model.k[pending], model.v[pending], None, model.q[pending], D ** -0.5, 0, out, ws)
        pending = model.logits(out).argmax(-1)
        single.append(pending.tolist())
    single = np.int64(single).T

    # drafted; over the paged layout the prompt is stored once and forked
    if paged:
        cache = ngc.PagedCache.allocate(1, B, H, H * G, D, 32, 8, 8 * B * H)
        ws = ngc.allocate_tree_workspace(cache, W, V)
        path = torch.arange(prompt, dtype=torch.int32, device="cuda").repeat(B, 1)
        n_path = torch.tensor([prompt] + [0] * (B - 1), dtype=torch.int32, device="cuda")
        kd, vd = (x.unsqueeze(0).repeat(B, 1, 1, 1) for x in (rows_k, rows_v))
        ngc.ngc_paged_tree_commit(cache, 0, kd, vd, None, path, n_path, prompt, ws)
        ngc.ngc_paged_fork(cache, -1, torch.tensor([-1, 0, 0, 0], dtype=torch.int32, device="cuda"), ws)
        attn, commit = ngc.ngc_paged_tree_attn, ngc.ngc_paged_tree_commit
    else:
        cache = fresh()
        ws = ngc.allocate_tree_workspace(cache, W, V)
        attn, commit = ngc.ngc_tree_attn, ngc.ngc_tree_commit
    history = [[int(x)] for x in single[:, 0]]
    out = torch.zeros(B, W, H * G, D, device="cuda")
    path = torch.zeros(B, W, dtype=torch.int32, device="cuda")
    n_path, nxt = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    accepted = 0
    for _ in range(steps):
        parent, token = _chains(rng, history, W, V)
        for b in range(B):      # a drafter that is right for three tokens
            at = len(history[b])
            token[b, 1:4] = single[b, at:at + 3]
        parent_t, token_t = torch.from_numpy(parent).cuda(), torch.from_numpy(token).cuda()
        ids = token_t.long()
        kd, vd = model.k[ids], model.v[ids]
        attn(cache, 0, kd, vd, parent_t, None, W, model.q[ids], D ** -0.5, 0, out, ws)
        best = model.logits(out).argmax(-1)
        target = torch.nn.functional.one_hot(best, V).float()
        ngc.ngc_tree_verify(target, None, V, token_t, parent_t, None, B, W, V, torch.rand(B, W, device="cuda"),
                            torch.rand(B, device="cuda"), path, n_path, nxt, ws)
        commit(cache, 0, kd, vd, None, path, n_path, W, ws)
        for b in range(B):
            n = int(n_path[b])
            accepted += n - 1
            history[b] += [int(token[b, i]) for i in path[b, 1:n].tolist()] + [int(nxt[b])]
    assert accepted >= 3 * steps * B
    for b in range(B):
        assert history[b] == single[b, :len(history[b])].tolist()
        assert cache.len[0, b].tolist() == [prompt + len(history[b]) - 1] * H
    assert sum(ngc.read_status(ws)) == 0
    # the cache goes on as any other: an eviction round, then single steps
    keep = torch.full((1, B, H), 1 if paged else 16, dtype=torch.int32, device="cuda")
    kept = torch.zeros(1, B, H, 16, dtype=torch.int32, device="cuda")
    if paged:
        logits = torch.randn(1, B, H, 8, device="cuda")
        ngc.ngc_paged_evict(cache, -1, logits, 8, keep, ngc.make_params(block=32, seed=1), 16, kept, None, None, ws)
        ngc.ngc_paged_free(cache, -1, torch.tensor([0, 1, 0, 0], dtype=torch.int32, device="cuda"), ws)
        ngc.ngc_paged_compact(cache, ws)
        assert int(cache.free_count) == 8 * B * H - 3 * H and int(cache.table[0, [0, 2, 3], :, 0].max()) == 3 * H - 1
    else:
        logits = torch.randn(1, B, H, 256, device="cuda")
        ngc.ngc_evict(cache, -1, logits, keep, ngc.make_params(seed=1), 16, kept, None, None, ws)
        assert (cache.len == 16).all()
    assert sum(ngc.read_status(ws)) == 0
