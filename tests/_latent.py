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
