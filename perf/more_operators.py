"""The operators of prompts and of latent caches: what they compute, on what, and how long it takes.

A program that serves prompts gives every sequence of a paged cache as many rows as its request is long: the pages, the
page tables and the slots of the packed tokens are found on the GPU (`extend`), and every layer writes its rows there
(`fill`).  A model whose layers keep one latent vector a token reads such rows with all its query heads at once, one or
a few new tokens a sequence (`attn`, the absorbed form); it is trained on keys and values that are expanded from the
latent vectors, under the mask of what the rollout had evicted (`replay`, and `train` with its gradient).

`run` is one pass through one operator: with `own` through the public binding, otherwise as elementary torch operations.
`listed()` holds the named cases, `draw(rng)` gives further ones of the same ranges, `prepare` makes what a program has
in hand before the call, `work` what the pass cannot do without, `exact` the same outputs in 64 bits.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEV = "cuda"


# ------------------------------------------------------------------ cases ---

def listed():
    return [
        # a decoding step of the paper's rollout group: 16 sequences grow by a token, in all layers
        dict(name="extend_step", kind="extend", L=28, B=16, Hkv=2, page=32, max_pages=24, n_lo=300, n_hi=700, new_lo=1, new_hi=1),
        # prompts of a batch of 64 enter an empty cache, all layers
        dict(name="extend_prompts", kind="extend", L=28, B=64, Hkv=2, page=32, max_pages=40, n_lo=0, n_hi=0, new_lo=300, new_hi=1000),
        # one layer's keys and values of those prompts
        dict(name="fill_prompts", kind="fill", latent=False, B=64, Hkv=2, D=128, page=32, n_lo=0, n_hi=0, new_lo=300, new_hi=1000),
        # latent rows of a few long prompts that continue cached ones
        dict(name="fill_latent", kind="fill", latent=True, B=8, Hkv=1, D=576, page=64, n_lo=100, n_hi=2000, new_lo=1000, new_hi=4096),
        # one new token of one short sequence: pure latency
        dict(name="attn_tiny", kind="attn", B=1, Hq=16, D=288, page=32, n_lo=300, n_hi=300, W=1, ragged=False, lse=False),
        # a layer's share of 16 heads, a batch of 64 in the middle of a period
        dict(name="attn_heads16", kind="attn", B=64, Hq=16, D=576, page=32, n_lo=1000, n_hi=2000, W=1, ragged=False, lse=False),
        # all 128 heads on one card, a large ragged batch: bytes and products in balance
        dict(name="attn_heads128", kind="attn", B=128, Hq=128, D=576, page=64, n_lo=1894, n_hi=3533, W=1, ragged=False, lse=True),
        # a few long sequences with drafted tokens, the length split over the chip
        dict(name="attn_long", kind="attn", B=4, Hq=40, D=576, page=64, n_lo=20000, n_hi=32000, W=3, ragged=True, lse=False),
        # training forward over rollouts of the paper's length, pages evicted every 256 tokens
        dict(name="replay_group", kind="replay", B=16, T=1050, Hq=16, D=128, n_lo=700, n_hi=1050, delta=256, keep=0.5),
        # a long prompt, nothing evicted
        dict(name="replay_long", kind="replay", B=1, T=8192, Hq=16, D=128, n_lo=8192, n_hi=8192, delta=0, keep=1.0),
        # training step over a few short rollouts of a small model
        dict(name="train_short", kind="train", B=4, T=350, Hq=8, D=64, n_lo=200, n_hi=350, delta=64, keep=0.5),
        # training step over the longest responses, pages evicted every 512 tokens
        dict(name="train_long", kind="train", B=2, T=3850, Hq=16, D=128, n_lo=3000, n_hi=3850, delta=512, keep=0.75),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the kinds of the list with sizes, widths and options spread over their ranges."""
    kind = rng.choice(["extend", "fill", "attn", "attn", "attn", "replay", "train", "train"])
    page = rng.choice([32, 64, 128])
    if kind == "extend":
        L, B, Hkv = rng.choice([1, 4, 28]), _log_int(rng, 1, 200), rng.choice([1, 2, 4, 8])
        new_hi = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 64, 2000)])
        n_hi = rng.choice([0, _log_int(rng, 1, 2000)])
        while B > 1 and L * Hkv * B * (new_hi + n_hi / 4) > 2.5e6:
            B //= 2
        return dict(kind=kind, L=L, B=B, Hkv=Hkv, page=page, max_pages=-(-(n_hi + new_hi) // page) + rng.choice([0, 1, 8]),
                    n_lo=n_hi // 2, n_hi=n_hi, new_lo=min(new_hi, rng.choice([0, 1, new_hi // 2])), new_hi=new_hi)
    if kind == "fill":
        latent = rng.random() < 0.5
        Hkv, D = (1, rng.choice([576, 288])) if latent else rng.choice([(2, 64), (2, 128), (4, 128), (8, 128), (3, 64)])
        B, new_hi, n_hi = _log_int(rng, 1, 128), _log_int(rng, 1, 4096), rng.choice([0, _log_int(rng, 1, 2000)])
        while B > 1 and B * Hkv * D * new_hi * (2 if latent else 4) > 6.0e7:
            B //= 2
        return dict(kind=kind, latent=latent, B=B, Hkv=Hkv, D=D, page=page, n_lo=n_hi // 2, n_hi=n_hi,
                    new_lo=max(1, new_hi // rng.choice([1, 2, 10])), new_hi=new_hi)
    if kind == "attn":
        B, Hq, W, n_hi = _log_int(rng, 1, 128), rng.choice([8, 16, 20, 32, 40, 64, 128]), rng.choice([1, 1, _log_int(rng, 1, 16)]), _log_int(rng, 20, 32000)
        D = rng.choice([576, 576, 288])
        while B > 1 and (B * n_hi * D > 2.0e8 or B * n_hi * W * Hq * D > 2.5e10):
            B //= 2
        while W > 1 and B * n_hi * W * Hq * D > 2.5e10:
            W //= 2
        return dict(kind=kind, B=B, Hq=Hq, D=D, page=page, n_lo=max(W, int(n_hi * rng.choice([1.0, 0.5, 0.1]))), n_hi=max(W, n_hi), W=W,
                    ragged=rng.random() < 0.4, lse=rng.random() < 0.4)
    B, T, Hq, D = _log_int(rng, 1, 16), _log_int(rng, 30, 5000), rng.choice([4, 5, 8, 16, 32]), rng.choice([64, 128, 128])
    while B > 1 and B * Hq * T * T > 3.5e8:
        B //= 2
    while Hq > 4 and B * Hq * T * T > 3.5e8:
        Hq //= 2
    evict = rng.random() < 0.6
    return dict(kind=kind, B=B, T=T, Hq=Hq, D=D, n_lo=max(1, int(T * rng.choice([1.0, 0.5, 0.1]))), n_hi=T,
                delta=rng.choice([64, 256, 512]) if evict else 0, keep=rng.choice([0.25, 0.5, 0.75]) if evict else 1.0)


# ----------------------------------------------------------------- inputs ---

def _latent(D):
    """The latent and the rotary width of a cached row of D values."""
    return D * 8 // 9, D // 9


def _tables(rs, L, B, H, lens, page, max_pages, num):
    """Tables of scattered pages, and the stack of those that are left (its first entries count)."""
    used = -(-lens // page)
    total = int(used.sum())
    order = rs.permutation(num).astype(np.int32)
    table = np.full((L * B * H, max_pages), -1, dtype=np.int32)
    table[np.arange(max_pages)[None, :] < used.reshape(-1, 1)] = order[:total]
    stack = np.concatenate([order[total:], order[:total]]).astype(np.int32)
    return torch.from_numpy(table.reshape(L, B, H, max_pages)).to(DEV), torch.from_numpy(stack).to(DEV), num - total


def prepare(c, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed * 9973 + 29)
    rs = np.random.RandomState((seed * 7919 + 11) % (1 << 31))
    s = SimpleNamespace(c=c, ws=None)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.bfloat16)

    if c["kind"] in ("replay", "train"):
        return _prepare_replay(c, s, normal, gen, rs)
    L, B, H, P = c.get("L", 1), c["B"], c.get("Hkv", 1), c["page"]
    lens = np.broadcast_to(rs.randint(c["n_lo"], c["n_hi"] + 1, size=(L, B, 1)), (L, B, H)).astype(np.int32)
    grown = c.get("new_hi", 0)
    max_pages = c.get("max_pages", -(-(c["n_hi"] + grown) // P))
    num = L * B * H * (-(-(c["n_hi"] + grown) // P) + 1)
    s.table, s.stack, spare = _tables(rs, L, B, H, lens, P, max_pages, num)
    # the lengths and the height of the stack of free pages, side by side
    s.state0 = torch.from_numpy(np.concatenate([lens.reshape(-1), [spare]]).astype(np.int32)).to(DEV)
    s.state = s.state0.clone()
    s.len, s.count = s.state[:-1].view(L, B, H), s.state[-1:]
    if c["kind"] == "attn":
        W, D = c["W"], c["D"]
        s.rows = normal(num, P, D)
        s.q = normal(B, W, c["Hq"], D)
        n_new = np.minimum(rs.randint(1, W + 1, size=B) if c["ragged"] else W, lens[0, :, 0]).astype(np.int32)
        s.n_new = torch.from_numpy(n_new).to(DEV)
        s.out = torch.zeros(B, W, c["Hq"], _latent(D)[0], dtype=torch.bfloat16, device=DEV)
        s.lse = torch.zeros(B, W, c["Hq"], dtype=torch.float32, device=DEV) if c["lse"] else None
        # what a program keeps beside such a cache, for every layer and every call
        s.ws = torch.zeros(256 << 20, dtype=torch.uint8, device=DEV)
        return s
    n_new = rs.randint(c["new_lo"], c["new_hi"] + 1, size=B).astype(np.int32)
    s.n_new = torch.from_numpy(n_new).to(DEV)
    # the packed tokens of a step lie in a buffer of a round size
    s.T = -(-int(B * c["new_hi"]) // 64) * 64
    s.ws = torch.zeros(16 << 20, dtype=torch.uint8, device=DEV)
    if c["kind"] == "extend":
        # a pool whose rows nobody looks at here, as wide as the library takes them
        s.rows = torch.zeros(num, P, 64, dtype=torch.bfloat16, device=DEV)
        s.slot = torch.zeros(L, H, s.T, dtype=torch.int32, device=DEV)
        s.start = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
        return s
    D = c["D"]
    s.k, s.v = normal(num, P, D), None if c["latent"] else normal(num, P, D)
    s.k_new, s.v_new = normal(s.T, H, D), None if c["latent"] else normal(s.T, H, D)
    _, s.slot, _ = _plain_extend(s, L, B, H, P)
    return s


def _prepare_replay(c, s, normal, gen, rs):
    B, T, H, D = c["B"], c["T"], c["Hq"], c["D"]
    E = D // 2
    n = rs.randint(c["n_lo"], c["n_hi"] + 1, size=B).astype(np.int32)
    n[rs.randint(B)] = c["n_hi"]
    s.n = torch.from_numpy(n).to(DEV)
    s.q, s.kv = normal(B, T, H, D + E), normal(B, T, H, 2 * D)
    # the rotary keys lie in the latent rows, as the cache holds them
    s.latent = normal(B, T, 9 * E)
    s.rope = s.latent[:, :, 8 * E:]
    s.death = None
    if c["delta"]:
        s.death = _deaths(c, gen)
    s.out = torch.zeros(B, T, H, D, dtype=torch.bfloat16, device=DEV)
    s.lse = torch.zeros(B, H, T, dtype=torch.float32, device=DEV)
    if c["kind"] == "train":
        s.dout = normal(B, T, H, D)
        s.dq, s.dkv = torch.zeros_like(s.q), torch.zeros_like(s.kv)
        s.drope = torch.zeros(B, T, E, dtype=torch.bfloat16, device=DEV)
        s.ws = torch.zeros(B * H * T * (E + 2) * 4 + (1 << 20), dtype=torch.uint8, device=DEV)
    return s


BLOCK = 32


def _deaths(c, gen):
    """The position at which every key was evicted: every `delta` tokens each whole block of 32 goes with 1 - keep."""
    B, T, delta = c["B"], c["T"], c["delta"]
    blocks, rounds = -(-T // BLOCK), -(-T // delta)
    at = (torch.arange(rounds, device=DEV) + 1) * delta
    whole = (torch.arange(blocks, device=DEV) + 1) * BLOCK
    goes = (torch.rand(B, blocks, rounds, generator=gen, device=DEV) >= c["keep"]) & (at >= whole.unsqueeze(1))
    death = torch.where(goes, at, torch.full_like(at, 1 << 30)).amin(-1)
    return death.repeat_interleave(BLOCK, 1)[:, :T].contiguous().int()


# ------------------------------------------------------------------- work ---

def work(c):
    if c["kind"] == "extend":
        tokens = c["B"] * 0.5 * (c["new_lo"] + c["new_hi"])
        segments, heads = c["L"] * c["B"] * c["Hkv"], c["L"] * c["Hkv"]
        capacity = -(-c["B"] * c["new_hi"] // 64) * 64
        return {"bytes": float(segments * 8 + c["B"] * 8 + heads * capacity * 4 + heads * tokens / c["page"] * 8), "flops": 0.0}
    if c["kind"] == "fill":
        rows = c["B"] * 0.5 * (c["new_lo"] + c["new_hi"]) * c["Hkv"]
        return {"bytes": float(rows * ((4 if c["latent"] else 8) * c["D"] + 4)), "flops": 0.0}
    if c["kind"] == "attn":
        R, E = _latent(c["D"])
        n = 0.5 * (c["n_lo"] + c["n_hi"])
        w = (c["W"] + 1) / 2 if c["ragged"] else c["W"]
        rows = c["B"] * w * c["Hq"]
        return {"bytes": float(c["B"] * n * c["D"] * 2 + rows * (c["D"] + R) * 2 + (rows * 4 if c["lse"] else 0)),
                "flops": float(rows * (n - (w - 1) / 2) * (4 * R + 2 * E))}
    B, T, H, D = c["B"], 0.5 * (c["n_lo"] + c["n_hi"]), c["Hq"], c["D"]
    E = D // 2
    # the pairs that are seen: a block that is j rounds old is left with keep^j
    pairs = 0.5 * T * T
    if c["delta"]:
        pairs = sum(max(0.0, min(T, i + c["delta"]) - i) ** 2 / 2 for i in range(0, int(T), c["delta"]))
        rounds = [min(T, i + c["delta"]) - i for i in range(0, int(T), c["delta"])]
        pairs += sum(rounds[i] * rounds[j] * c["keep"] ** (i - j) for i in range(len(rounds)) for j in range(i))
    tokens = B * T
    inputs = tokens * (H * (3 * D + E) + E) * 2
    if c["kind"] == "replay":
        return {"bytes": float(inputs + tokens * H * (D * 2 + 4)), "flops": float(2 * B * H * pairs * (2 * D + E))}
    # forward, then scores again and four products for the gradients
    return {"bytes": float(2 * inputs + tokens * H * (D * 6 + 8)),
            "flops": float(2 * B * H * pairs * (2 * D + E) + 2 * B * H * pairs * (3 * (D + E) + 2 * D))}


# -------------------------------------------------------------------- run ---

def run(s):
    c = s.c
    if c["kind"] == "extend":
        s.state.copy_(s.state0)         # every pass begins at the same lengths and the same free pages
        return _run_extend(s, c)
    if c["kind"] == "fill":
        return _run_fill(s, c)
    if c["kind"] == "attn":
        return _run_attn(s, c)
    return _run_replay(s, c)


def _run_extend(s, c):
    L, B, H, P = c["L"], c["B"], c["Hkv"], c["page"]
    if own:
        from paper_2604_18002_amd import binding as ngc
        cache = ngc.PagedCache(s.rows, s.rows, None, s.table, s.len, s.stack, s.count, H)
        ngc.ngc_paged_extend(cache, -1, s.n_new, s.T, s.slot, s.start, s.ws)
        return s.table, s.len, s.slot, s.start, s.count
    after, slot, start = _plain_extend(s, L, B, H, P)
    s.len.copy_(after)
    return s.table, s.len, slot, start, s.count


def _plain_extend(s, L, B, H, P):
    """Pages for the new rows from the top of the stack, segments in ascending order; the new lengths, the slots of the packed tokens and
    where every sequence's tokens begin."""
    n, new = s.len.long(), s.n_new.long()
    have, want = -(-n // P), -(-(n + new.view(1, B, 1)) // P)
    table = s.table.view(-1, s.table.shape[-1])
    entry = torch.arange(table.shape[1], device=DEV)
    granted = (entry >= have.view(-1, 1)) & (entry < want.view(-1, 1))
    rank = granted.view(-1).cumsum(0).view(granted.shape) - 1
    table.copy_(torch.where(granted, s.stack[(s.count.long() - 1 - rank).clamp(0, s.stack.numel() - 1)], table))
    s.count.sub_(granted.sum().int())
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), new.cumsum(0)])
    token = torch.arange(s.T, device=DEV)
    seq = (token.unsqueeze(1) >= start[1:]).sum(1)
    real, seq = seq < B, seq.clamp(max=B - 1)
    row = n[:, seq] + (token - start[seq]).view(1, -1, 1)                    # [L, T, H]
    page = torch.gather(s.table[:, seq], 3, (row // P).clamp(max=s.table.shape[3] - 1).unsqueeze(-1)).squeeze(-1).long()
    slot = torch.where(real.view(1, -1, 1), page * P + row % P, torch.full_like(row, -1))
    return (n + new.view(1, B, 1)).int(), slot.transpose(1, 2).contiguous().int(), start.int()


def _run_fill(s, c):
    if own:
        from paper_2604_18002_amd import binding as ngc
        cache = ngc.PagedCache(s.k, s.v, None, s.table, s.len, s.stack, s.count, c["Hkv"])
        ngc.ngc_paged_fill(cache, 0, s.k_new, s.v_new, None, s.slot[0], s.T, s.ws)
        return s.k if c["latent"] else (s.k, s.v)
    slot = s.slot[0].t()                # [T, H]
    real = slot >= 0
    at = slot[real].long()
    s.k.view(-1, c["D"])[at] = s.k_new[real]
    if c["latent"]:
        return s.k
    s.v.view(-1, c["D"])[at] = s.v_new[real]
    return s.k, s.v


def _expanded_width(D):
    """Width of the keys that the absorbed queries stand for: the scores' scale goes by it."""
    return D // 3


def _run_attn(s, c):
    B, W, Hq, D, P = c["B"], c["W"], c["Hq"], c["D"], c["page"]
    R = _latent(D)[0]
    scale = _expanded_width(D) ** -0.5
    if own:
        from paper_2604_18002_amd import binding as ngc
        cache = ngc.PagedCache(s.rows, None, None, s.table, s.len, s.stack, s.count, Hq)
        ngc.ngc_latent_attn(cache, 0, s.n_new, W, s.q, scale, c["n_hi"], s.out, s.ws, lse_out=s.lse)
        return (s.out, s.lse) if c["lse"] else s.out
    top = c["n_hi"]
    rows = s.rows[s.table[0, :, 0, :-(-top // P)].long().clamp(min=0)].reshape(B, -1, D)[:, :top].float()
    scores = s.q.float().view(B, W * Hq, D) @ rows.transpose(1, 2).contiguous() * scale
    # token i of the new ones sees the rows up to its own
    sees = s.len[0].long() - s.n_new.long().unsqueeze(1) + 1 + torch.arange(W, device=DEV)      # [B, W]
    hidden = (torch.arange(top, device=DEV) >= sees.unsqueeze(-1)).unsqueeze(2)
    scores.view(B, W, Hq, top).masked_fill_(hidden, -math.inf)
    peak = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - peak)
    total = p.sum(-1, keepdim=True)
    out = (p @ rows[..., :R].contiguous() / total).view(B, W, Hq, R)
    real = torch.arange(W, device=DEV) < s.n_new.unsqueeze(1)
    out = torch.where(real.view(B, W, 1, 1), out, torch.zeros_like(out)).bfloat16()
    if not c["lse"]:
        return out
    lse = (peak + torch.log(total)).view(B, W, Hq)
    return out, torch.where(real.unsqueeze(-1), lse, torch.zeros_like(lse))


def _run_replay(s, c):
    B, T, H, D = c["B"], c["T"], c["Hq"], c["D"]
    E = D // 2
    scale = (D + E) ** -0.5
    train = c["kind"] == "train"
    if own:
        from paper_2604_18002_amd import binding as ngc
        ngc.ngc_latent_replay_attn(s.q, s.kv, s.rope, 9 * E, s.death, s.n, B, T, H, D, scale, s.out, s.lse)
        if not train:
            return s.out, s.lse
        ngc.ngc_latent_replay_attn_backward(s.q, s.kv, s.rope, 9 * E, s.death, s.n, s.out, s.lse, s.dout, B, T, H, D, scale,
                                            s.dq, s.dkv, s.drope, s.ws)
        return s.out, s.lse, s.dq, s.dkv, s.drope
    pos = torch.arange(T, device=DEV)
    real = pos < s.n.unsqueeze(1)                                               # [B, T]
    sees = (pos.unsqueeze(1) >= pos) & real.unsqueeze(-1)                       # [B, query, key]
    if s.death is not None:
        sees = sees & (pos.unsqueeze(1) < s.death.unsqueeze(1))
    sees = sees.unsqueeze(1)
    q = s.q.float().transpose(1, 2).contiguous()
    k = torch.cat([s.kv[..., :D].float(), s.rope.float().unsqueeze(2).expand(B, T, H, E)], -1).transpose(1, 2).contiguous()
    v = s.kv[..., D:].float().transpose(1, 2).contiguous()
    scores = (q @ k.transpose(2, 3).contiguous() * scale).masked_fill_(~sees, -math.inf)
    peak = scores.amax(-1, keepdim=True)
    peak = torch.where(peak > -math.inf, peak, torch.zeros_like(peak))          # rows that see nothing
    p = scores.sub_(peak).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    out = p @ v
    lse = torch.where(real.unsqueeze(1), (peak + torch.log(total)).squeeze(-1), torch.zeros(1, device=DEV))
    out_bf16 = out.transpose(1, 2).contiguous().bfloat16()
    if not train:
        return out_bf16, lse
    dout = torch.where(real.view(B, T, 1, 1), s.dout.float(), torch.zeros(1, device=DEV)).transpose(1, 2).contiguous()
    dv = p.transpose(2, 3).contiguous() @ dout
    delta = (out * dout).sum(-1, keepdim=True)
    ds = p.mul_((dout @ v.transpose(2, 3).contiguous()).sub_(delta)).mul_(scale)
    dq = ds @ k
    dk = ds.transpose(2, 3).contiguous() @ q
    dkv = torch.cat([dk[..., :D], dv], -1).transpose(1, 2).contiguous()
    return out_bf16, lse, dq.transpose(1, 2).contiguous().bfloat16(), dkv.bfloat16(), dk[..., D:].sum(1).bfloat16()


# ------------------------------------------------------------------ exact ---

def exact(c, seed):
    if c["kind"] in ("extend", "fill"):
        return None             # page numbers, lengths and rows, moved as they are
    s = prepare(c, seed)
    if c["kind"] == "attn":
        return _exact_attn(s, c)
    return _exact_replay(s, c)


def _exact_attn(s, c):
    B, W, Hq, D, P = c["B"], c["W"], c["Hq"], c["D"], c["page"]
    R = _latent(D)[0]
    out = torch.zeros(B, W, Hq, R, dtype=torch.float64, device=DEV)
    lse = torch.zeros(B, W, Hq, dtype=torch.float64, device=DEV)
    lens, new = s.len[0, :, 0].tolist(), s.n_new.tolist()
    for b in range(B):
        n, w = lens[b], new[b]
        rows = s.rows[s.table[0, b, 0, :-(-n // P)].long()].reshape(-1, D)[:n].double()
        for i in range(w):
            m = n - w + i + 1
            x = torch.mm(s.q[b, i].double(), rows[:m].t()) / math.sqrt(_expanded_width(D))
            z = torch.logsumexp(x, 1)
            out[b, i] = torch.mm(torch.exp(x - z.unsqueeze(1)), rows[:m, :R])
            lse[b, i] = z
    return (out, lse) if c["lse"] else out


def _exact_replay(s, c):
    B, T, H, D = c["B"], c["T"], c["Hq"], c["D"]
    E = D // 2
    f8 = dict(dtype=torch.float64, device=DEV)
    out, lse = torch.zeros(B, T, H, D, **f8), torch.zeros(B, H, T, **f8)
    dq, dkv, drope = torch.zeros(B, T, H, D + E, **f8), torch.zeros(B, T, H, 2 * D, **f8), torch.zeros(B, T, E, **f8)
    for b in range(B):
        n = int(s.n[b])
        at = torch.arange(n, device=DEV)
        hidden = at.unsqueeze(0) > at.unsqueeze(1)
        if s.death is not None:
            hidden |= at.unsqueeze(1) >= s.death[b, :n].unsqueeze(0)
        empty = hidden.all(1)
        rope = s.rope[b, :n].double()
        for h in range(H):
            q, v = s.q[b, :n, h].double(), s.kv[b, :n, h, D:].double()
            k = torch.cat([s.kv[b, :n, h, :D].double(), rope], 1)
            x = (torch.mm(q, k.t()) / math.sqrt(D + E)).masked_fill_(hidden, -math.inf)
            z = torch.logsumexp(x, 1)
            p = torch.exp(x - torch.where(empty, torch.zeros_like(z), z).unsqueeze(1))
            out[b, :n, h], lse[b, h, :n] = torch.mm(p, v), z
            if c["kind"] == "train":
                g = s.dout[b, :n, h].double()
                dp = torch.mm(g, v.t())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(D + E)
                dq[b, :n, h] = torch.mm(ds, k)
                dk = torch.mm(ds.t(), q)
                dkv[b, :n, h] = torch.cat([dk[:, :D], torch.mm(p.t(), g)], 1)
                drope[b, :n] += dk[:, D:]
    return (out, lse, dq, dkv, drope) if c["kind"] == "train" else (out, lse)
