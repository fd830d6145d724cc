"""Prompts, growth, attention, eviction and release of a cache of latent rows as a rollout uses them, and the replay of that rollout."""
import numpy as np
import pytest

from _latent import attention, extend, replay, widths

pytestmark = pytest.mark.gpu

FOREVER = 1 << 30


class Rollout:
    """B sequences of latents, the same tokens for the cache (absorbed: each head's queries reach the latent) and for the replay
    (expanded: each head's keys and values are made of the latent).  The matrices between them pick entries, so both are exact."""

    def __init__(self, D, B, H, T, seed):
        import torch
        self.B, self.H, self.T, self.D = B, H, T, D
        self.R, self.E = widths(D)
        self.Dh = 2 * self.E
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()       # noqa: E731
        self.c = normal(B, T, D)
        self.q = normal(B, T, H, self.Dh + self.E)
        self.pick_k, self.pick_v = (torch.stack([torch.randperm(self.R, generator=gen, device="cuda")[:self.Dh] for _ in range(H)]) for _ in range(2))
        self.absorbed = torch.zeros(B, T, H, D, dtype=torch.bfloat16, device="cuda")
        self.absorbed[..., self.R:] = self.q[..., self.Dh:]
        self.absorbed.scatter_(3, self.pick_k.expand(B, T, H, self.Dh), self.q[..., :self.Dh])
        latent = self.c[..., :self.R]
        self.kv = torch.cat([latent[:, :, self.pick_k], latent[:, :, self.pick_v]], -1).contiguous()
        self.scale = (self.Dh + self.E) ** -0.5
        self.death = np.full((B, T), FOREVER, np.int32)


@pytest.mark.parametrize("D,H,page", [(288, 6, 32), (576, 16, 32), (576, 40, 64)])
def test_a_rollout_with_evictions_answers_like_its_replay(D, H, page):
    import torch
    from paper_2604_18002_amd import binding as ngc
    B, prompts, steps, every = 3, [70, 33, 5], 60, 20
    T = max(prompts) + steps
    r = Rollout(D, B, H, T, D + H)
    rng = np.random.default_rng(D + H)
    max_pages = -(-T // page) + 1
    pc = ngc.PagedCache.allocate_latent(1, B, H, D, page, max_pages, B * max_pages + 2, with_pos=True)
    pc.free_stack.copy_(torch.from_numpy(rng.permutation(B * max_pages + 2).astype(np.int32)))
    pc.free_count.fill_(B * max_pages + 2)
    W = max(prompts)
    ws = ngc.allocate_latent_workspace(pc, W)
    outs, lses = torch.zeros(B, T, H, r.R, device="cuda"), torch.zeros(B, T, H, device="cuda")
    held = [[] for _ in range(B)]                          # positions of the cached rows

    def enter(first, counts):
        """Rows of counts[b] tokens from first[b] on, and their attention."""
        n_new = torch.tensor(counts, dtype=torch.int32, device="cuda")
        total = sum(counts)
        slot = torch.full((1, total + 3), 7, dtype=torch.int32, device="cuda")
        start = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        ngc.ngc_paged_extend(pc, 0, n_new, total + 3, slot, start, ws)
        rows = torch.zeros(total + 3, 1, D, dtype=torch.bfloat16, device="cuda")
        pos = torch.zeros(total + 3, dtype=torch.int32, device="cuda")
        at = 0
        for b, w in enumerate(counts):
            assert int(start[b]) == at
            rows[at:at + w, 0] = r.c[b, first[b]:first[b] + w]
            pos[at:at + w] = torch.arange(first[b], first[b] + w, dtype=torch.int32, device="cuda")
            at += w
            held[b] += range(first[b], first[b] + w)
        ngc.ngc_paged_fill(pc, 0, rows, None, pos, slot, total + 3, ws)
        w_most = max(counts)
        q = torch.zeros(B, w_most, H, D, dtype=torch.bfloat16, device="cuda")
        for b, w in enumerate(counts):
            q[b, :w] = r.absorbed[b, first[b]:first[b] + w]
        out = torch.zeros(B, w_most, H, r.R, dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros(B, w_most, H, device="cuda")
        ngc.ngc_latent_attn(pc, 0, n_new, w_most, q, r.scale, 0, out, ws, lse_out=lse)
        for b, w in enumerate(counts):
            outs[b, first[b]:first[b] + w], lses[b, first[b]:first[b] + w] = out[b, :w].float(), lse[b, :w]

    enter([0] * B, prompts)
    for step in range(steps):
        if step % every == every - 1:                      # half the pages go
            logits = torch.from_numpy(rng.standard_normal((B, max_pages)).astype(np.float32)).cuda()
            keep = [-(-len(h) // page) // 2 + 1 for h in held]
            kept = torch.zeros(B, max(keep), dtype=torch.int32, device="cuda")
            ngc.ngc_paged_evict(pc, 0, logits, max_pages, torch.tensor(keep, dtype=torch.int32, device="cuda"),
                                ngc.make_params(block=page, noise_scale=0.0, round=step), max(keep), kept, None, None, ws)
            for b in range(B):
                pages = set(kept[b, :min(keep[b], -(-len(held[b]) // page))].tolist())
                gone = [p for i, p in enumerate(held[b]) if i // page not in pages]
                held[b] = [p for i, p in enumerate(held[b]) if i // page in pages]
                r.death[b, gone] = prompts[b] + step
        enter([p + step for p in prompts], [1] * B)
    assert pc.len.flatten().tolist() == [len(h) for h in held]
    assert int(pc.free_count) == B * max_pages + 2 - sum(-(-len(h) // page) for h in held)
    assert sum(ngc.read_status(ws)) == 0 and (r.death < FOREVER).any()
    for b in range(B):                                     # the cached rows and positions are those that are held
        at = [int(pc.table[0, b, 0, i // page]) * page + i % page for i in range(len(held[b]))]
        assert pc.pos_pool.flatten()[at].tolist() == held[b]
        assert torch.equal(pc.k_pool.view(-1, D)[at], r.c[b, held[b]])

    # the same tokens replayed
    lens = [p + steps for p in prompts]
    n, death = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.from_numpy(r.death).cuda()
    rope = r.c[..., r.R:]
    out = torch.zeros(B, T, H, r.Dh, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(B, H, T, device="cuda")
    ngc.ngc_latent_replay_attn(r.q, r.kv, rope, D, death, n, B, T, H, r.Dh, r.scale, out, lse)
    dout = torch.randn(B, T, H, r.Dh, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    dq, dkv, drope = torch.zeros_like(r.q), torch.zeros_like(r.kv), torch.zeros(B, T, r.E, dtype=torch.bfloat16, device="cuda")
    ws2 = torch.empty(ngc.ngc_latent_replay_workspace_bytes(B, T, H, r.Dh), dtype=torch.uint8, device="cuda")
    ngc.ngc_latent_replay_attn_backward(r.q, r.kv, rope, D, death, n, out, lse, dout, B, T, H, r.Dh, r.scale, dq, dkv, drope, ws2)

    def near(name, got, want, tol):
        assert bool(((got.double() - want).abs() <= tol).all()), (name, float(((got.double() - want).abs() / tol).max()))

    for b in range(B):
        m = lens[b]
        ref = replay(r.q[b].double(), r.kv[b].double(), rope[b].double(), death[b], m, r.scale, dout[b].double())
        near("replayed", out[b, :m].transpose(0, 1), ref["out"], ref["tol_out"])
        near("replayed lse", lse[b, :, :m], ref["lse"], ref["tol_lse"])
        for name, got in (("dq", dq[b, :m]), ("dk", dkv[b, :m, :, :r.Dh]), ("dv", dkv[b, :m, :, r.Dh:])):
            near(name, got.transpose(0, 1), ref[name], ref["tol_" + name])
        near("drope", drope[b, :m], ref["drope"], ref["tol_drope"])
        for i in range(m):                                 # the cache's answers, against the rows that this token saw
            seen = torch.nonzero(death[b, :i + 1] > i).flatten()
            w_out, w_lse, tol_out, tol_lse = attention(r.c[b, seen].double(), r.absorbed[b, i].double(),
                                                       torch.full((H,), len(seen), device="cuda"), r.scale, r.R)
            near("cached", outs[b, i], w_out, tol_out)
            near("cached lse", lses[b, i], w_lse, tol_lse)
            near("one and the other", torch.gather(w_out, 1, r.pick_v), ref["out"][:, i], torch.full_like(ref["out"][:, i], 1e-9))

    # a sequence ends, its pages come back, and a longer prompt takes its place
    drop = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
    ngc.ngc_paged_free(pc, 0, drop, ws)
    held[1] = []
    assert pc.len.flatten().tolist() == [len(h) for h in held]
    enter([0, 0, 0], [0, 90, 0])
    assert pc.len.flatten().tolist() == [len(h) for h in held] and sum(ngc.read_status(ws)) == 0
    for i in (0, 31, 32, 89):
        w_out, w_lse, tol_out, tol_lse = attention(r.c[1, :i + 1].double(), r.absorbed[1, i].double(), torch.full((H,), i + 1, device="cuda"),
                                                   r.scale, r.R)
        near("again", outs[1, i], w_out, tol_out)
        near("again lse", lses[1, i], w_lse, tol_lse)


def test_a_decoding_step_of_latent_rows_under_graph_capture():
    import torch
    from paper_2604_18002_amd import binding as ngc
    L, B, H, D, page = 2, 5, 16, 288, 32
    gen = torch.Generator(device="cuda").manual_seed(4)
    steps = 5
    rows = torch.randn(steps, L, B, 1, D, generator=gen, device="cuda").bfloat16()
    qs = torch.randn(steps, L, B, 1, H, D, generator=gen, device="cuda").bfloat16()

    class State:
        def __init__(self):
            self.pc = ngc.PagedCache.allocate_latent(L, B, H, D, page, 4, 44)
            self.pc.free_stack.copy_(torch.arange(44, dtype=torch.int32, device="cuda"))
            self.pc.free_count.fill_(44)
            self.ws = ngc.allocate_latent_workspace(self.pc)
            self.slot, self.start = torch.zeros(L, 1, B, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda")
            self.row, self.q = rows[0].clone(), qs[0].clone()
            self.out = torch.zeros(L, B, 1, H, 256, dtype=torch.bfloat16, device="cuda")
            prompt = torch.tensor([30, 0, 31, 64, 95], dtype=torch.int32, device="cuda")
            slot, start = torch.zeros(L, 1, 220, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda")
            ngc.ngc_paged_extend(self.pc, -1, prompt, 220, slot, start, self.ws)
            cached = torch.randn(L, 220, 1, D, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda").bfloat16()
            ngc.ngc_paged_fill(self.pc, -1, cached, None, None, slot, 220, self.ws)

        def step(self):
            ngc.ngc_paged_extend(self.pc, -1, None, B, self.slot, self.start, self.ws)
            ngc.ngc_paged_fill(self.pc, -1, self.row, None, None, self.slot, B, self.ws)
            ngc.ngc_latent_attn(self.pc, -1, None, 1, self.q, 0.1, 0, self.out, self.ws)

    ref, got = State(), State()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        State().step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got.step()
    for i in range(steps):
        for s in (ref, got):
            s.row.copy_(rows[i])
            s.q.copy_(qs[i])
        ref.step()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("slot", "start", "out"):
            assert torch.equal(getattr(ref, name), getattr(got, name)), (i, name)
        for name in ("len", "free_count", "k_pool"):
            assert torch.equal(getattr(ref.pc, name), getattr(got.pc, name)), (i, name)
    assert got.pc.len[0].flatten().tolist() == [35, 5, 36, 69, 100] and ngc.read_status(got.ws) == ngc.read_status(ref.ws)


def test_more_segments_than_a_thread_holds_and_a_long_tail():
    """Extension of segments of which a thread takes more than one batch, with places left behind the last sequence."""
    import torch
    from paper_2604_18002_amd import binding as ngc
    rng = np.random.default_rng(3)
    L, B, H, page, max_pages, T = 20, 70, 4, 32, 4, 4000
    lens = np.broadcast_to(rng.integers(0, 40, (L, B, 1)), (L, B, H)).astype(np.int32)
    used = -(-lens // page)
    total = int(used.sum())
    spare = total + 900                                    # too few for the last of them
    order = rng.permutation(total + spare).astype(np.int32)
    table = np.full((L, B, H, max_pages), -1, np.int32)
    table[np.arange(max_pages) < used[..., None]] = order[:total]
    stack = np.concatenate([order[total:], order[:total]]).astype(np.int32)
    pc = ngc.PagedCache.allocate(L, B, H, H, 64, page, max_pages, total + spare)
    for to, x in ((pc.table, table), (pc.len, lens.copy()), (pc.free_stack, stack)):
        to.copy_(torch.from_numpy(x))
    pc.free_count.fill_(spare)
    ws = ngc.allocate_paged_workspace(pc)
    n_new = rng.integers(0, 60, B).astype(np.int32)
    full = 0
    for _ in range(3):                                     # (the stack is dry in the end)
        slot, start = torch.full((L, H, T), 7, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        ngc.ngc_paged_extend(pc, -1, torch.from_numpy(n_new).cuda(), T, slot, start, ws)
        w_table, w_len, w_slot, w_start, w_count, counts = extend(table, lens, stack, spare, page, n_new, T)
        np.testing.assert_array_equal(slot.cpu().numpy(), w_slot)
        np.testing.assert_array_equal(start.cpu().numpy(), w_start)
        np.testing.assert_array_equal(pc.len.cpu().numpy(), w_len)
        np.testing.assert_array_equal(pc.table.cpu().numpy(), w_table)
        full += counts["full"]
        assert int(pc.free_count) == w_count and ngc.read_status(ws)[ngc.STATUS_APPEND_FULL] == full
        table, lens, spare = w_table, w_len, w_count
    assert full > 0 and spare == 0 and int(n_new.sum()) < T - 1000
