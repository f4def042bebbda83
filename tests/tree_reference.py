"""Plain statements of the calls on drafted trees and on the pages of a cache (test infrastructure only)."""
import math

import numpy as np
import torch

D = 128


def ancestors(parents):
    """bool [n, n]: row t: t and its ancestors; depths.  parents: a list, -1 for roots."""
    n = len(parents)
    sees, depth = np.zeros((n, n), dtype=bool), np.zeros(n, dtype=np.int64)
    for t in range(n):
        x, steps = t, 0
        while x >= 0:
            sees[t, x] = True
            x = parents[x]
            steps += 1
        depth[t] = steps - 1
    return sees, depth


def pack(sees, words, T, starts):
    """int32 [T, words] from a list of bool [n, n]; rows of no unit are all ones."""
    out = np.full((T, words), 0xffffffff, dtype=np.uint32)
    for u, s in enumerate(sees):
        n = s.shape[0]
        bits = np.zeros((n, 32 * words), dtype=np.uint64)
        m = min(n, 32 * words)
        bits[:, :m] = s[:, :m]
        out[starts[u]:starts[u + 1]] = (bits.reshape(n, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    return torch.from_numpy(out.view(np.int32))


def attend(q, starts, rows, sees, scale=None):
    """out [T, H, d], lse [T, H] in float64: token i of unit u sees rows below len - n of rows[u][g] = (k, v), and row len - n + t
    where sees[u][i, t].  Tokens of no unit are left NaN; hidden rows may hold anything."""
    T, H, _ = q.shape
    Hkv = len(rows[0])
    G = H // Hkv
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out = torch.full((T, H, D), float("nan"), dtype=torch.float64, device=q.device)
    lse = torch.full((T, H), float("nan"), dtype=torch.float64, device=q.device)
    for u in range(len(rows)):
        a, b = starts[u], starts[u + 1]
        n = b - a
        for g in range(Hkv):
            k, v = (x.to(q.device).double() for x in rows[u][g])
            L = k.shape[0]
            base = L - n
            see = torch.ones(n, L, dtype=torch.bool, device=q.device)
            tree = torch.as_tensor(sees[u], device=q.device)
            if L:
                see[:, max(base, 0):] = tree[:, max(-base, 0):]
            x = torch.einsum("nhd,ld->nhl", q[a:b, g * G:(g + 1) * G].double(), k.nan_to_num(0, 0, 0)) * scale
            x = x.masked_fill(~see[:, None], -math.inf)
            l = torch.logsumexp(x, -1) if L else torch.full(x.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
            p = torch.exp(x - torch.where(torch.isfinite(l), l, torch.zeros_like(l))[..., None])
            out[a:b, g * G:(g + 1) * G] = torch.einsum("nhl,ld->nhd", p, v.nan_to_num(0, 0, 0))
            lse[a:b, g * G:(g + 1) * G] = l
    return out, lse


class Pages:
    """The state that the page calls keep, in numpy, and the calls one entry at a time.  Rows are not part of it: `reserve` says
    which pages were copied."""

    def __init__(self, P, refs, held, table, lengths):
        self.P, self.refs, self.held, self.table, self.lengths = P, refs.copy(), held.copy(), table.copy(), lengths.copy()

    def reserve(self, new_rows, layers=1):
        Nu, Hkv, width = self.table.shape
        free = [int(p) for p in np.flatnonzero(self.refs == 0)]
        got, copies, held, old = [], [], self.held.copy(), self.refs.copy()
        seqs = Nu // layers
        for u in range(Nu):
            for g in range(Hkv):
                n = int(new_rows[u * Hkv + g] if len(new_rows) != seqs else new_rows[u % seqs])
                if n <= 0:
                    continue
                L = int(self.lengths[u, g])
                slots = min(-(-(L + n) // self.P), width)
                for s in range(L // self.P, slots):
                    if s < self.held[u, g]:
                        if old[self.table[u, g, s]] > 1:
                            copies.append((u, g, s, int(self.table[u, g, s]), len(got), L % self.P if s == L // self.P else 0))
                            got.append((u, g, s))
                    else:
                        got.append((u, g, s))
                held[u, g] = max(held[u, g], slots)
        if len(got) > len(free):
            return (len(free), len(got) - len(free)), []
        for (u, g, s), p in zip(got, free):
            if s < self.held[u, g]:
                self.refs[self.table[u, g, s]] -= 1
            self.table[u, g, s] = p
            self.refs[p] = 1
        self.held = held
        return (len(free) - len(got), 0), [(src, free[i], rows) for _, _, _, src, i, rows in copies]

    def trim(self, lengths=None):
        for u, g in np.ndindex(*self.held.shape):
            keep = 0 if lengths is None else -(-int(lengths[u, g]) // self.P)
            for s in range(keep, int(self.held[u, g])):
                self.refs[self.table[u, g, s]] -= 1
            self.held[u, g] = min(self.held[u, g], keep)

    def fork(self, parents, layers=1, keep_old=False, fill=0):
        Nu, Hkv, width = self.table.shape
        seqs, n = Nu // layers, len(parents)
        new = Pages(self.P, self.refs, np.zeros((layers * n, Hkv), np.int32), np.full((layers * n, Hkv, width), fill, np.int32),
                    np.zeros((layers * n, Hkv), np.int32))
        for l in range(layers):
            for s, p in enumerate(parents):
                if p < 0:
                    continue
                a, b = l * seqs + p, l * n + s
                new.lengths[b], new.held[b] = self.lengths[a], self.held[a]
                for g in range(Hkv):
                    h = int(self.held[a, g])
                    new.table[b, g, :h] = self.table[a, g, :h]
                    new.refs[self.table[a, g, :h]] += 1
        if not keep_old:
            for u, g in np.ndindex(*self.held.shape):
                np.subtract.at(new.refs, self.table[u, g, :int(self.held[u, g])], 1)
        return new
