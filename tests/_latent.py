"""Plain 64-bit forms of the operators on prompts and latent caches, from their definitions, and what their tests share."""
import math

import numpy as np


def widths(D):
    """Latent and rotary part of a row of D values."""
    return {576: (512, 64), 288: (256, 32)}[D]


# ------------------------------------------------------------------ extend ---

def extend(table, length, stack, count, page_rows, n_new, T, layer=-1):
    """-> table, len, slots [layers, Hkv, T], start, count, {rows left out, clamped}; the arguments stay as they are."""
    L, B, H, max_pages = table.shape
    table, length = table.copy(), length.copy()
    cap, pages = page_rows * max_pages, lambda n: -(-int(n) // page_rows)
    new = np.ones(B, np.int64) if n_new is None else np.asarray(n_new, np.int64)
    start, clamped, full = [0], 0, 0
    for x in new:
        nxt = min(T, start[-1] + max(0, int(x)))
        clamped += nxt - start[-1] != x
        start.append(nxt)
    layers = range(L) if layer < 0 else [layer]
    slot = np.full((len(layers), H, T), -1, np.int64)
    asked = 0
    for i, l in enumerate(layers):
        for b in range(B):
            for h in range(H):
                n, w = int(length[l, b, h]), start[b + 1] - start[b]
                if n < 0 or n > cap:
                    clamped += 1
                    full += w
                    continue
                m = min(w, cap - n)
                need = pages(n + m) - pages(n)
                got = max(0, min(need, count - asked))
                for j in range(got):
                    table[l, b, h, pages(n) + j] = stack[count - 1 - asked - j]
                if got < need:
                    m = (pages(n) + got) * page_rows - n
                asked += need
                full += w - m
                for t in range(m):
                    p = int(table[l, b, h, (n + t) // page_rows])
                    slot[i, h, start[b] + t] = p * page_rows + (n + t) % page_rows
                length[l, b, h] = n + m
    return table, length, slot, np.array(start), max(0, count - asked), dict(full=full, clamped=clamped)


# --------------------------------------------------------------- attention ---

def attention(rows, q, limits, scale, R):
    """rows [n, D], q [M, D] (float64 tensors), limits [M] -> out [M, R], lse [M], and bounds of their errors.

    A weight is rounded to bf16 (half a step: 2^-8 of it), the output again.  A score is a sum of D products in 32 bits: it
    is off by at most (D + 2) 2^-24 of the sum of their magnitudes, and so is the exponent."""
    import torch
    n, M, D = rows.shape[0], q.shape[0], q.shape[1]
    out, lse = torch.zeros(M, R, dtype=torch.float64, device=q.device), torch.full((M,), -math.inf, dtype=torch.float64, device=q.device)
    tol_out, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    if n == 0:
        return out, lse, tol_out, tol_lse
    x = torch.mm(q, rows.t()) * scale
    delta = torch.mm(q.abs(), rows.abs().t()).amax(1) * scale * (D + 2) * 2.0 ** -24
    hidden = torch.arange(n, device=q.device) >= limits.unsqueeze(1)
    x = x.masked_fill(hidden, -math.inf)
    some = limits > 0
    z = torch.where(some, torch.logsumexp(x, 1), torch.zeros_like(lse))
    p = torch.exp(x - z.unsqueeze(1))
    out = torch.mm(p, rows[:, :R])
    magnitude = torch.mm(p, rows[:, :R].abs())
    lse = torch.where(some, z, lse)
    # weights: rounding, the exponent's error twice (of the weight and of their sum), the exponential's and the sum's own steps
    slack = 2 * torch.expm1(delta) + (n + 64) * 2.0 ** -23
    tol_out = magnitude * (2.0 ** -8 + slack.unsqueeze(1)) * (1 + 2.0 ** -8) + 2.0 ** -8 * out.abs()
    tol_lse = delta + (n + 64) * 2.0 ** -24 + 2.0 ** -22 * z.abs() + 2.0 ** -21
    return out, lse, tol_out, tol_lse


# ------------------------------------------------------------------ replay ---

def replay(q, kv, rope, death, n, scale, dout=None):
    """One trajectory, all heads, float64 tensors: q [T, H, D + E], kv [T, H, 2 D], rope [T, E], death [T] or None, n positions.

    -> dict of values, and of bounds of the kernels' errors.  The kernels round P and dS to bf16 for their products, and every
    result: half a step, 2^-8, each.  The scores' products are exact and their sums in 32 bits, so an exponent is off by at
    most `eps_x`, and so is lse; out enters delta rounded to bf16."""
    import torch
    T, H, DE = q.shape
    D = kv.shape[2] // 2
    at = torch.arange(n, device=q.device)
    hidden = at.unsqueeze(0) > at.unsqueeze(1)
    if death is not None:
        hidden = hidden | (at.unsqueeze(1) >= death[:n].unsqueeze(0))
    empty = hidden.all(1)
    k = torch.cat([kv[:n, :, :D], rope[:n].unsqueeze(1).expand(n, H, DE - D)], -1).transpose(0, 1).contiguous()
    v, qq = kv[:n, :, D:].transpose(0, 1).contiguous(), q[:n].transpose(0, 1).contiguous()
    x = (qq @ k.transpose(1, 2).contiguous() * scale).masked_fill(hidden, -math.inf)
    half, f32 = 2.0 ** -8, 2.0 ** -23
    eps_x = (qq.abs() @ k.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True) * scale * (DE + 4) * 2.0 ** -24 * 2 + (n + 64) * f32
    z = torch.logsumexp(x, -1, keepdim=True)
    p = torch.exp(x - torch.where(empty.view(1, n, 1), torch.zeros_like(z), z))
    out, mag = p @ v, p @ v.abs()
    slack = 2 * torch.expm1(eps_x)
    r = dict(out=out, lse=z[..., 0], tol_out=mag * (half + slack) * (1 + half) + half * out.abs(),
             tol_lse=eps_x[..., 0] + (z[..., 0].abs() * 2.0 ** -22).nan_to_num(posinf=0.0) + 2.0 ** -21, empty=empty)
    if dout is None:
        return r
    g = dout[:n].transpose(0, 1).contiguous()
    t = lambda a: a.transpose(1, 2).contiguous()      # noqa: E731
    dp, dp_mag = g @ t(v), g.abs() @ t(v.abs())
    delta = (g * out).sum(-1, keepdim=True)
    e_delta = (g.abs() * r["tol_out"]).sum(-1, keepdim=True) + (g * out).abs().sum(-1, keepdim=True) * (D + 2) * f32
    ds = p * (dp - delta)
    e_p = p * (slack + half)
    e_ds = p * (dp_mag * (D + 2) * f32 + e_delta) + (dp - delta).abs() * p * slack * 2 + half * ds.abs() * (1 + half)
    dv = t(p) @ g
    dq, dk = ds @ k * scale, t(ds) @ qq * scale
    acc = (n + 64) * f32                              # the long sums' own steps
    r.update(dv=dv, tol_dv=(t(e_p) @ g.abs() + acc * (t(p) @ g.abs())) * (1 + half) + half * dv.abs(),
             dq=dq, tol_dq=(e_ds @ k.abs() + acc * (ds.abs() @ k.abs())) * scale * (1 + half) + half * dq.abs())
    e_k = (t(e_ds) @ qq.abs() + acc * (t(ds.abs()) @ qq.abs())) * scale * (1 + half)
    drope = dk[..., D:].sum(0)
    r.update(dk=dk[..., :D], tol_dk=(e_k + half * dk.abs())[..., :D], drope=drope, tol_drope=e_k[..., D:].sum(0) * (1 + H * f32) + half * drope.abs())
    return r
