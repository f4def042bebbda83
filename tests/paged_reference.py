"""Plain 64-bit statements of the paged-cache operators, and a cache to try them on (test infrastructure only)."""
import math

import torch

D = 128


def turn(x, positions, inv_freq=None, w=None, eps=1e-6, interleaved=False, scale=1.0):
    """x [T, heads, d] normed and rotated, float64."""
    y = x.double().clone()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
    if inv_freq is None or inv_freq.numel() == 0:
        return y
    half = inv_freq.numel()
    angle = positions.double()[:, None, None] * inv_freq.double()
    c, s = scale * torch.cos(angle), scale * torch.sin(angle)
    out = y.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        out[..., a] = y[..., a] * c[..., i] - y[..., b] * s[..., i]
        out[..., b] = y[..., b] * c[..., i] + y[..., a] * s[..., i]
    return out


class Cache:
    """A paged cache whose rows are known: rows[u][g] = (k [len, d], v [len, d]); the rest of the pool is poison."""

    def __init__(self, lens, page, max_extra=0, dtype=torch.bfloat16, device="cpu", seed=0, poison=float("nan"), row_pad=0,
                 spare=2, k_scale=1.0):
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.P = lens, page
        Nu, Hkv = len(lens), len(lens[0])
        need = [[-(-(x + max_extra) // page) for x in row] for row in lens]
        self.max_pages = max(1, max(max(r) for r in need))
        total = sum(map(sum, need))
        n_pages = total + spare
        perm = torch.randperm(n_pages, generator=gen).int()
        table = torch.full((Nu, Hkv, self.max_pages), 0x7ffffff0, dtype=torch.int32)   # entries of no row are never read
        at = 0
        width = D + row_pad
        self.pools = []
        for _ in range(2):
            self.pools.append(torch.full((n_pages, page, width), poison, dtype=dtype))
        self.rows = [[None] * Hkv for _ in range(Nu)]
        for u in range(Nu):
            for g in range(Hkv):
                m = need[u][g]
                table[u, g, :m] = perm[at:at + m]
                at += m
                kv = []
                for pool, mul in zip(self.pools, (k_scale, 1.0)):
                    x = (torch.randn(lens[u][g], D, generator=gen) * mul).to(dtype)
                    for j in range(0, lens[u][g], page):
                        pool[int(table[u, g, j // page]), :min(page, lens[u][g] - j), :D] = x[j:j + page]
                    kv.append(x)
                self.rows[u][g] = tuple(kv)
        self.table = table.to(device)
        self.pools = [p.to(device) for p in self.pools]
        self.k_pages, self.v_pages = (p[..., :D] for p in self.pools)
        self.lengths = torch.tensor(lens, dtype=torch.int32, device=device)


def attend(q, starts, rows, causal=True, scale=None):
    """out [T, H, d], lse [T, H] in float64; rows[u][g] = (k, v).  Rows of no unit are left NaN."""
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
            x = torch.einsum("nhd,ld->nhl", q[a:b, g * G:(g + 1) * G].double(), k) * scale
            if causal:
                hide = torch.arange(L, device=q.device)[None] > (L - n + torch.arange(n, device=q.device))[:, None]
                x = x.masked_fill(hide[:, None], -math.inf)
            l = torch.logsumexp(x, -1) if L else torch.full(x.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
            p = torch.exp(x - torch.where(torch.isfinite(l), l, torch.zeros_like(l))[..., None])
            out[a:b, g * G:(g + 1) * G] = torch.einsum("nhl,ld->nhd", p, v)
            lse[a:b, g * G:(g + 1) * G] = l
    return out, lse
