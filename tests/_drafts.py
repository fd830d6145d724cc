"""Plain 64-bit forms of the operators on drafted tokens and on a paged cache's sequences, from their definitions."""
import numpy as np


def make_tree(rng, B, W, shape):
    parent = np.full((B, W), -1, dtype=np.int32)
    for b in range(B):
        for i in range(1, W):
            if shape == "chain":
                parent[b, i] = i - 1
            elif shape == "star":
                parent[b, i] = 0
            elif shape == "forest":
                parent[b, i] = rng.integers(-1, i)
            else:
                parent[b, i] = rng.integers(max(0, i - 5), i)
    return parent


def ancestors(parent):
    """sees[i, j]: node j is node i or lies on its way from the root."""
    W = len(parent)
    sees = np.zeros((W, W), dtype=bool)
    for i in range(W):
        if 0 <= parent[i] < i:
            sees[i] = sees[parent[i]]
        sees[i, i] = True
    return sees


def tree_attention(k, v, kd, vd, parent, q, scale):
    """One KV head of one sequence.  k, v [n, D]; kd, vd [w, D]; q [w, G, D] -> out [w, G, D], lse [w, G]."""
    w, G, D = q.shape
    sees = np.concatenate([np.ones((w, len(k)), dtype=bool), ancestors(parent)], 1)
    keys, values = np.concatenate([k, kd]).astype(np.float64), np.concatenate([v, vd]).astype(np.float64)
    out, lse = np.zeros((w, G, D)), np.zeros((w, G))
    for i in range(w):
        kk, vv = keys[sees[i]], values[sees[i]]
        x = q[i].astype(np.float64) @ kk.T * scale
        top = x.max(1, keepdims=True)
        e = np.exp(x - top)
        out[i] = e @ vv / e.sum(1, keepdims=True)
        lse[i] = top[:, 0] + np.log(e.sum(1))
    return out, lse


def verify(target, draft, token, parent, nd, u_accept, u_sample):
    """One sequence -> path (list), next token."""
    W, V = target.shape
    if nd == 0:
        return [], -1
    node, path = 0, [0]
    while True:
        p = np.maximum(np.nan_to_num(target[node].astype(np.float64), nan=0.0), 0.0)
        q = None if draft is None else draft[node].astype(np.float64)
        r, whole, c, taken = p.copy(), 1.0, 0.0, -1
        for x in range(node + 1, nd):
            if parent[x] != node or not 0 <= token[x] < V:
                continue
            t = token[x]
            u = float(u_accept[x])
            if u * whole * (1.0 if q is None else q[t]) < r[t]:
                taken = x
                break
            if q is None:
                whole = max(whole - r[t], 0.0)
                r[t] = 0.0
            else:
                c += whole
                r = np.maximum(p - c * q, 0.0)
                whole = r.sum()
        if taken < 0:
            break
        node = taken
        path.append(node)
    if not r.sum() > 0:
        r = p
    upto = np.cumsum(r)
    if not upto[-1] > 0:
        return path, -1
    above = np.nonzero((upto > float(u_sample) * upto[-1]) & (r > 0))[0]
    return path, int(above[0]) if len(above) else int(np.nonzero(r)[0][-1])


class PagedModel:
    """Tables, stack and pools of a paged cache as numpy arrays."""

    def __init__(self, table, length, stack, count, page_rows, k, v, pos=None):
        self.table, self.len, self.stack, self.count, self.P = table.copy(), length.copy(), stack.copy(), int(count), page_rows
        self.k, self.v, self.pos = k.copy(), v.copy(), None if pos is None else pos.copy()
        self.full = self.invalid = 0

    def pages(self, n):
        return -(-int(n) // self.P)

    def segments(self, layer):
        L, B, H = self.len.shape
        return [(l, b, h) for l in (range(L) if layer < 0 else [layer]) for b in range(B) for h in range(H)]

    def commit(self, layer, kd, vd, draft_pos, path, n_path):
        cap = self.table.shape[3] * self.P
        segs = self.segments(layer)
        first_layer = segs[0][0]
        take = {}
        count = self.count
        asked = 0
        for s in segs:
            n = self.len[s]
            m = min(int(n_path[s[1]]), cap - n)
            need = self.pages(n + m) - self.pages(n)
            got = max(0, min(need, count - asked))
            for j in range(got):
                self.table[s][self.pages(n) + j] = self.stack[count - 1 - asked - j]
            if got < need:
                m = (self.pages(n) + got) * self.P - n
            asked += need
            take[s] = m
            self.full += int(n_path[s[1]]) - m
        self.count = max(0, count - asked)
        for s in segs:
            l, b, h = s
            for i in range(take[s]):
                r = self.len[s] + i
                page, row = self.table[s][r // self.P], r % self.P
                node = path[b, i]
                self.k[page, row], self.v[page, row] = kd[l - first_layer, b, node, h], vd[l - first_layer, b, node, h]
                if self.pos is not None and draft_pos is not None:
                    self.pos[page, row] = draft_pos[b, node]
            self.len[s] += take[s]

    def release(self, segs):
        for s in segs:
            for j in range(self.pages(self.len[s])):
                self.stack[self.count] = self.table[s][j]
                self.count += 1

    def free(self, layer, drop):
        segs = [s for s in self.segments(layer) if drop[s[1]]]
        self.release(segs)
        for s in segs:
            self.len[s] = 0

    def fork(self, layer, source):
        B = self.len.shape[1]
        valid = {}
        for b in range(B):
            s = int(source[b])
            if s < 0 or s == b:
                continue
            if s < B and (source[s] < 0 or source[s] == s):
                valid[b] = s
            else:
                self.invalid += 1
        segs = [s for s in self.segments(layer) if s[1] in valid]
        self.release(segs)
        height, asked = self.count, 0
        granted = 0
        for l, b, h in segs:
            src = (l, valid[b], h)
            need = self.pages(self.len[src])
            if need and asked + need > height:
                self.full += 1
                self.len[l, b, h] = 0
            else:
                for j in range(need):
                    to, of = self.stack[height - 1 - asked - j], self.table[src][j]
                    self.table[l, b, h, j] = to
                    self.k[to], self.v[to] = self.k[of], self.v[of]
                    if self.pos is not None:
                        self.pos[to] = self.pos[of]
                granted += need
                self.len[l, b, h] = self.len[src]
            asked += need
        self.count = height - granted

    def compact(self):
        num = len(self.stack)
        U = num - self.count
        owner = {}
        for s in self.segments(-1):
            for j in range(self.pages(self.len[s])):
                owner[int(self.table[s][j])] = (s, j)
        holes = [p for p in range(U) if p not in owner]
        movers = sorted(p for p in owner if p >= U)
        for to, of in zip(holes, movers):
            self.k[to], self.v[to] = self.k[of], self.v[of]
            if self.pos is not None:
                self.pos[to] = self.pos[of]
            s, j = owner[of]
            self.table[s][j] = to
        self.stack[:self.count] = np.arange(num - 1, U - 1, -1)
