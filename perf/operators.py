"""The operators around the retention pass that a decoder runs on a paged cache, and what they are measured on.

  rotate   norms of queries and keys for each head and their position rotation, in place of a prefill's own
           (it makes the rotated queries and keys that the retention pass reads)
  gather   the rows that the retention pass kept, copied from the prompt's K and V into the pages of a cache
           whose page table and lengths are per sequence AND per KV head (heads keep different numbers of rows)
  append   new tokens' keys (normed, rotated) and values written behind those rows, their queries normed and rotated
  attend   attention of the new tokens of every sequence over its pages, causal inside the chunk

``run`` computes each in its plain form (elementary torch operations, 32 bits, rounded once at the end), or, where
``own`` is true, makes the calls that a user of ``paper_2602_08686_b200.binding`` makes.  ``exact`` states the same
outputs in 64 bits.  Notation as in include/ckv.h: Nu units, H query heads, Hkv KV heads, G = H / Hkv, d = 128.
"""
import math
import random

import torch

own = False
D = 128
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def _case(name, op, dtype, units, q_heads, kv_heads, new=1, cached=0, page=64, ragged=False, rot=128, interleaved=False,
          norm=False, start=0, pad=0, window=32, budget=512):
    c = {"op": op, "dtype": dtype, "units": units, "q_heads": q_heads, "kv_heads": kv_heads, "new": new, "cached": cached,
         "page": page, "ragged": ragged, "rot": rot, "interleaved": interleaved, "norm": norm, "start": start, "pad": pad,
         "window": window, "budget": budget}
    return dict({"name": name}, **c) if name else c


def listed():
    return [
        # a 32k prompt of the Llama-3-8B-shaped layer before the retention pass reads it: one pass over 0.34 GB
        _case("rotate prompt 32k", "rotate", "bf16", 1, 32, 8, new=32768),
        # three sequences' next tokens in a model with query and key norms and interleaved pairs: latency
        _case("rotate 3 tokens f32", "rotate", "f32", 3, 28, 4, norm=True, interleaved=True, start=65536),
        # the pass over eight layers of a 32k prompt hands 512 rows a head to the decoder's pages
        _case("gather 8 layers 32k", "gather", "bf16", 8, 32, 8, cached=32768, page=64, budget=512),
        # one fp32 layer, ragged heads, a small page
        _case("gather 1 layer f32", "gather", "f32", 1, 8, 2, cached=2048, page=16, ragged=True, budget=512),
        # a decode step of a batch of 16 on compressed caches: one token each, far behind the rows it is stored after
        _case("append decode 16", "append", "bf16", 16, 32, 8, cached=512, ragged=True, start=32768),
        # chunked prefill of ragged sequences, query/key norms, positions past 2^17
        _case("append chunk ragged", "append", "bf16", 7, 28, 4, new=2048, cached=4096, page=16, ragged=True, norm=True,
              start=131072, pad=13),
        # the smallest step: one sequence, one token, 512 rows a head kept of its prompt
        _case("attend decode 1x512", "attend", "bf16", 1, 32, 8, cached=512, ragged=True),
        # a decode step of a serving batch whose 32k prompts were not compressed
        _case("attend decode 16x32k", "attend", "bf16", 16, 32, 8, cached=32768, page=64),
        # five drafted tokens a sequence checked at once, ragged lengths, seven query heads a KV head, small pages
        _case("attend verify 8x16k", "attend", "bf16", 8, 28, 4, new=5, cached=16384, page=16, ragged=True),
        # a 2048-token chunk of a prompt over the 32k tokens before it
        _case("attend chunk 2048", "attend", "bf16", 1, 32, 8, new=2048, cached=32768, page=128),
        # chunks and single tokens in one call, an idle sequence among them, padding rows behind the last
        _case("attend mixed ragged", "attend", "bf16", 8, 32, 8, new=512, cached=16384, page=64, ragged=True, pad=11),
        # the fp32 layer, decoded after a 2048-token prompt
        _case("attend decode f32", "attend", "f32", 4, 8, 2, cached=2048, page=32, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["rotate", "gather", "append", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    q_heads, kv_heads = rng.choice([(32, 8), (28, 4), (8, 2), (16, 16), (24, 2), (8, 1)])
    c = dict(page=rng.choice([16, 32, 64, 128, 256]), ragged=rng.random() < 0.6, rot=rng.choice([128, 128, 64, 96]),
             interleaved=rng.random() < 0.3, norm=rng.random() < 0.5, start=_log(rng, 1, 1 << 20), pad=rng.choice([0, 0, 1, 17]))
    if op == "rotate":
        return _case(None, op, dtype, rng.randint(1, 8), q_heads, kv_heads, new=_log(rng, 1, 2000), **c)
    if op == "gather":
        cached = _log(rng, 300, 32768)
        return _case(None, op, dtype, rng.randint(1, 6), q_heads, min(kv_heads, 8), cached=cached, window=rng.choice([16, 32, 64]),
                     budget=min(cached, _log(rng, 100, 2048)), **c)
    if op == "append":
        return _case(None, op, dtype, _log(rng, 1, 32), q_heads, kv_heads, new=_log(rng, 1, 500), cached=_log(rng, 1, 8000), **c)
    kind = rng.choice(["decode", "verify", "chunk"]) if dtype == "bf16" else rng.choice(["decode", "verify"])
    if kind == "decode":
        units, new = _log(rng, 1, 32), 1
        cached = _log(rng, 1, 32768 * 16 // (units * max(kv_heads, 4)))
    elif kind == "verify":
        units, new = _log(rng, 1, 16), rng.randint(2, 16)
        cached = _log(rng, 16, 8192 * 16 // (units * max(kv_heads, 4)))
    else:
        units, new = rng.randint(1, 3), _log(rng, 17, 1024)
        cached = _log(rng, 1, 8192)
    return _case(None, op, dtype, units, q_heads, kv_heads, new=new, cached=cached, **c)


def _plan(c):
    """What the case alone decides: new tokens of every unit and rows cached for every (unit, KV head)."""
    r = random.Random("%(units)d %(kv_heads)d %(new)d %(cached)d %(page)d" % c)
    Nu, Hkv = c["units"], c["kv_heads"]
    if c["op"] == "gather":      # budgets of the pass: each head keeps its window and a share that adds up to the total
        L, W = c["cached"], c["window"]
        B = max(min(c["budget"], L), min(W, L))
        lens = []
        for _ in range(Nu):
            row = [B] * Hkv
            if c["ragged"]:
                for g in range(0, Hkv - 1, 2):
                    x = r.randint(0, min(B - min(W, L), L - B))
                    row[g], row[g + 1] = row[g] - x, row[g + 1] + x
            lens.append(row)
        return [0] * Nu, lens
    n = [c["new"]] * Nu
    if c["ragged"] and c["new"] > 1:
        n = [r.choice([0, 1, 1, r.randint(1, c["new"]), c["new"]]) if c["new"] > 16 else r.randint(1, c["new"]) for _ in range(Nu)]
        n[r.randrange(Nu)] = c["new"]
    full = [r.randint(c["cached"] // 3, c["cached"]) if c["ragged"] and Nu > 1 else c["cached"] for _ in range(Nu)]
    lens = [[f if not c["ragged"] else r.randint(f - f // 4, f) for _ in range(Hkv)] for f in full]
    return n, lens


# ----------------------------------------------------------------------------------------------- inputs
def _pages(c, rows, gen):
    """A pool of pages, a random assignment of them to the (unit, KV head) rows, and a few pages nobody has."""
    P = c["page"]
    need = [[-(-x // P) for x in row] for row in rows]
    max_pages = max(1, max(max(row) for row in need))
    total = sum(sum(row) for row in need)
    n_pages = total + 3
    perm = torch.randperm(n_pages, generator=gen, device=DEV).int()
    table = torch.zeros(c["units"], c["kv_heads"], max_pages, dtype=torch.int32, device=DEV)
    have = torch.arange(max_pages, device=DEV) < torch.tensor(need, device=DEV)[..., None]
    table[have] = perm[:total]
    return table, n_pages


def _pool(n_pages, P, dt, gen):
    return torch.randn(n_pages, P, D, generator=gen, device=DEV, dtype=torch.float32).to(dt) if n_pages * P < 1 << 22 else \
        torch.randn(n_pages, P, D, generator=gen, device=DEV, dtype=dt)


def prepare(case, seed):
    c, dt = case, DT[case["dtype"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    Nu, H, Hkv, P = c["units"], c["q_heads"], c["kv_heads"], c["page"]
    n, lens = _plan(c)
    s = {"c": c, "rows": lens}
    if c["op"] == "gather":
        L, W = c["cached"], min(c["window"], c["cached"])
        B = max(min(c["budget"], L), W)
        s["k"], s["v"] = (torch.randn(Nu, Hkv, L, D, generator=gen, device=DEV, dtype=dt) for _ in range(2))
        s["budgets"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["offsets"] = torch.zeros(Nu, Hkv + 1, dtype=torch.int32, device=DEV)
        s["offsets"][:, 1:] = s["budgets"].cumsum(1)
        # the kept positions: a random choice of the prefix, ascending, then the window
        order = torch.rand(Nu, Hkv, L, generator=gen, device=DEV)
        order[..., L - W:] = -1.0
        rank = order.argsort(-1).argsort(-1)
        keep = rank < s["budgets"][..., None]
        s["indices"] = torch.arange(L, device=DEV, dtype=torch.int32).expand(Nu, Hkv, L)[keep].view(Nu, Hkv * B)
        s["table"], s["n_pages"] = _pages(c, lens, gen)
        s["k_pages"], s["v_pages"] = (torch.zeros(s["n_pages"], P, D, device=DEV, dtype=dt) for _ in range(2))
        s["lengths"] = torch.zeros(Nu, Hkv, dtype=torch.int32, device=DEV)
        if own:
            from paper_2602_08686_b200 import binding as b
            s["shape"] = b.make_shape(torch.empty(Nu, H, W, D, device=DEV, dtype=dt), s["k"])
            s["params"] = b.make_params(b.Params(budget_per_head=B, floor_per_head=0), None, None)
            s["paged"] = b.make_paged(s["k_pages"], s["table"], n_q_heads=H)
            s["ws"] = b.alloc_paged_workspace(s["paged"], DEV)
        return s
    T = sum(n) + c["pad"]
    s["n"], s["valid"] = n, sum(n)
    s["starts"] = torch.tensor([sum(n[:u]) for u in range(Nu + 1)], dtype=torch.int32, device=DEV)
    s["scale"] = 1.0 / math.sqrt(D)
    if c["op"] in ("rotate", "append"):
        # the fused projection's output, [T, H + 2 Hkv, d]: queries, keys and values are views of it
        qkv = torch.randn(max(T, 1), H + 2 * Hkv, D, generator=gen, device=DEV).to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        rot = c["rot"]
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot))
        s["qw"], s["kw"] = ((1.0 + 0.1 * torch.randn(D, generator=gen, device=DEV)) if c["norm"] else None for _ in range(2))
        first = torch.randint(0, c["start"] + 1, (Nu,), generator=gen, device=DEV) // 2 + c["start"] // 2
        s["positions"] = torch.zeros(max(T, 1), dtype=torch.int32, device=DEV)
        unit = torch.repeat_interleave(torch.arange(Nu, device=DEV), torch.tensor(n, device=DEV))
        s["positions"][:s["valid"]] = (first[unit] + torch.arange(s["valid"], device=DEV) - s["starts"].long()[unit]).int()
        s["q_out"] = torch.zeros(max(T, 1), H, D, device=DEV, dtype=dt)
        s["unit"] = unit
    if c["op"] == "rotate":
        s["k_out"] = torch.zeros(max(T, 1), Hkv, D, device=DEV, dtype=dt)
        if own:
            from paper_2602_08686_b200 import binding as b
            s["paged"] = b.make_packed(s["q"], s["k"], n_units=Nu)
            s["rotary"] = b.make_rotary(s["inv_freq"], interleaved=c["interleaved"], q_norm_w=s["qw"], k_norm_w=s["kw"])
        return s
    rows = [[x + n[u] for x in lens[u]] for u in range(Nu)]      # after the chunk
    s["table"], s["n_pages"] = _pages(c, rows, gen)
    s["k_pages"], s["v_pages"] = _pool(s["n_pages"], P, dt, gen), _pool(s["n_pages"], P, dt, gen)
    if c["op"] == "append":
        s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["new_lengths"] = torch.zeros(Nu, Hkv, dtype=torch.int32, device=DEV)
        if own:
            from paper_2602_08686_b200 import binding as b
            s["paged"] = b.make_paged(s["k_pages"], s["table"], q=s["q"], k_new=s["k"], max_new=c["new"])
            s["rotary"] = b.make_rotary(s["inv_freq"], interleaved=c["interleaved"], q_norm_w=s["qw"], k_norm_w=s["kw"])
            s["ws"] = b.alloc_paged_workspace(s["paged"], DEV)
        return s
    s["rows"] = rows
    s["lengths"] = torch.tensor(rows, dtype=torch.int32, device=DEV)
    q = torch.randn(T, H, D, generator=gen, device=DEV)
    s["q"] = q.to(dt)
    # an attention sink in row 0 of every head, along the mean query of its group
    mean = torch.stack([q[sum(n[:u]):sum(n[:u]) + max(n[u], 1)].mean(0) for u in range(Nu)]) if T else q.new_zeros(Nu, H, D)
    mean = mean.view(Nu, Hkv, H // Hkv, D).mean(2)
    s["k_pages"][s["table"][:, :, 0].long(), 0] = (2.0 * math.sqrt(D) * mean / mean.norm(dim=-1, keepdim=True).clamp_min(1e-6)).to(dt)
    s["out"] = torch.zeros(T, H, D, device=DEV, dtype=dt)
    s["lse"] = torch.zeros(T, H, device=DEV)
    if own:
        from paper_2602_08686_b200 import binding as b
        s["paged"] = b.make_paged(s["k_pages"], s["table"], q=s["q"], max_new=c["new"])
        s["ws"] = b.alloc_paged_workspace(s["paged"], DEV)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _turned(x, w, positions, inv_freq, interleaved):
    """x [T, heads, d] in 32 bits: root-mean-square norm (where there is a weight), then the rotation by position."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6) * w
    angle = positions.double()[:, None] * inv_freq            # 64 bits: far positions turn by many thousand radians
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    rot = 2 * inv_freq.numel()
    a, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        e, o = a[..., 0::2], a[..., 1::2]
        a = torch.stack((e * cos - o * sin, o * cos + e * sin), -1).flatten(-2)
    else:
        e, o = a[..., :rot // 2], a[..., rot // 2:]
        a = torch.cat((e * cos - o * sin, o * cos + e * sin), -1)
    return torch.cat((a, rest), -1)


def _places(table, rows_first, count, P):
    """Flat pool rows of cache rows rows_first + (0 .. count-1) of every (unit, head): [Nu, Hkv, count] (clamped table)."""
    j = rows_first + torch.arange(count, device=DEV)
    page = torch.gather(table.long(), 2, (j // P).clamp(max=table.shape[2] - 1).expand(table.shape[0], table.shape[1], count))
    return page * P + j % P


def _plain_gather(s):
    c, P = s["c"], s["c"]["page"]
    Nu, Hkv = c["units"], c["kv_heads"]
    rows = s["indices"].shape[1]
    at = torch.arange(rows, device=DEV).expand(Nu, rows)
    head = torch.searchsorted(s["offsets"][:, 1:].contiguous(), at.int().contiguous(), right=True)
    row = at - torch.gather(s["offsets"].long(), 1, head)
    u = torch.arange(Nu, device=DEV)[:, None]
    place = s["table"][u, head, row // P].long() * P + row % P
    for name in ("k", "v"):
        s[name + "_pages"].view(-1, D)[place] = s[name][u, head, s["indices"].long()]
    s["lengths"].copy_(s["budgets"])


def _plain_append(s):
    c, P, v = s["c"], s["c"]["page"], s["valid"]
    unit, pos = s["unit"], s["positions"][:v]
    s["q_out"][:v] = _turned(s["q"][:v], s["qw"], pos, s["inv_freq"], c["interleaved"]).to(s["q"].dtype)
    k = _turned(s["k"][:v], s["kw"], pos, s["inv_freq"], c["interleaved"]).to(s["k"].dtype)
    row = s["lengths"].long()[unit] + (torch.arange(v, device=DEV) - s["starts"].long()[unit])[:, None]     # [T, Hkv]
    page = s["table"][unit[:, None], torch.arange(c["kv_heads"], device=DEV), row // P].long()
    s["k_pages"].view(-1, D)[page * P + row % P] = k
    s["v_pages"].view(-1, D)[page * P + row % P] = s["v"][:v]
    s["new_lengths"].copy_(s["lengths"] + (s["starts"][1:] - s["starts"][:-1])[:, None])


def _plain_attend(s):
    c, P = s["c"], s["c"]["page"]
    Nu, H, Hkv = c["units"], c["q_heads"], c["kv_heads"]
    G, nmax, Lmax = H // Hkv, max(s["n"]), max(max(r) for r in s["rows"])
    place = _places(s["table"], 0, Lmax, P)                                    # [Nu, Hkv, Lmax]
    j = torch.arange(Lmax, device=DEV)
    there = j < s["lengths"][..., None]
    K = s["k_pages"].view(-1, D)[place].float()
    V = torch.where(there[..., None], s["v_pages"].view(-1, D)[place].float(), 0.0)
    starts, count = s["starts"].long(), (s["starts"][1:] - s["starts"][:-1]).long()
    i = torch.arange(nmax, device=DEV)
    token = (starts[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)             # [Nu, nmax]
    q = s["q"][token].float().view(Nu, nmax, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(Nu, Hkv, G * nmax, D)
    x = torch.matmul(q, K.transpose(-1, -2)).mul_(s["scale"]).view(Nu, Hkv, G, nmax, Lmax)
    # token i of a unit's n sees the rows up to its own, the (length - n + i)-th
    limit = s["lengths"][..., None].long() - count[:, None, None] + i          # [Nu, Hkv, nmax]
    hidden = j > limit[..., None]
    x.masked_fill_(hidden[:, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)                                      # [Nu, Hkv, G, nmax]
    o = torch.matmul(x.view(Nu, Hkv, G * nmax, Lmax), V).view(Nu, Hkv, G, nmax, D)
    o = o / torch.where(total > 0, total, 1.0)
    mine = i < count[:, None]                                                  # [Nu, nmax]
    s["out"][token[mine]] = o.permute(0, 3, 1, 2, 4).reshape(Nu, nmax, H, D)[mine].to(s["q"].dtype)
    s["lse"][token[mine]] = lse.permute(0, 3, 1, 2).reshape(Nu, nmax, H)[mine]


# -------------------------------------------------------------------------------------------------- run
def run(s):
    c = s["c"]
    if own:
        from paper_2602_08686_b200 import binding as b
    if c["op"] == "rotate":
        if own:
            b.ckv_rotate(s["paged"], s["rotary"], s["q"], s["k"], s["positions"], s["starts"], s["q_out"], s["k_out"])
        else:
            v, pos = s["valid"], s["positions"][:s["valid"]]
            for x, w in (("q", s["qw"]), ("k", s["kw"])):
                s[x + "_out"][:v] = _turned(s[x][:v], w, pos, s["inv_freq"], c["interleaved"]).to(s[x].dtype)
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["op"] == "gather":
        if own:
            b.ckv_gather_pages(s["shape"], s["params"], s["paged"], s["k"], s["v"], s["indices"], s["budgets"], s["offsets"],
                               s["table"], s["k_pages"], s["v_pages"], s["lengths"], s["ws"])
        else:
            _plain_gather(s)
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "lengths": s["lengths"]}
    if c["op"] == "append":
        if own:
            b.ckv_append(s["paged"], s["rotary"], s["k"], s["v"], s["positions"], s["starts"], s["lengths"], s["table"],
                         s["k_pages"], s["v_pages"], s["ws"], q=s["q"], q_out=s["q_out"], new_lengths=s["new_lengths"])
        else:
            _plain_append(s)
        return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"], "lengths": s["new_lengths"]}
    if own:
        b.ckv_paged_attend(s["paged"], s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["starts"], s["out"],
                           s["ws"], lse=s["lse"])
    else:
        _plain_attend(s)
    return {"out": s["out"], "lse": s["lse"]}


def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    n, lens = _plan(c)
    H, Hkv, T = c["q_heads"], c["kv_heads"], sum(n)
    if c["op"] == "rotate":
        return {"bytes": 2 * T * (H + Hkv) * D * e + 4 * T, "flops": 6 * T * (H + Hkv) * D}
    if c["op"] == "append":
        return {"bytes": 2 * T * (H + 2 * Hkv) * D * e + 4 * T, "flops": 6 * T * (H + Hkv) * D}
    if c["op"] == "gather":
        kept = sum(sum(r) for r in lens)
        return {"bytes": kept * (4 * D * e + 4), "flops": 0}
    # rows a unit without tokens holds are not read; pairs: what each query sees
    rows = sum(x + n[u] for u in range(c["units"]) if n[u] for x in lens[u])
    pairs = sum(H // Hkv * sum(x + i + 1 for i in range(n[u])) for u in range(c["units"]) for x in lens[u])
    return {"bytes": 2 * rows * D * e + 2 * T * H * D * e + 4 * T * H, "flops": 4 * D * pairs}


# ------------------------------------------------------------------------------------------------ exact
def _turn64(x, w, positions, inv_freq, interleaved):
    y = x.to(torch.float64, copy=True)
    if w is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + 1e-6) * w.double()
    half = inv_freq.numel()
    z = torch.polar(torch.ones_like(positions, dtype=torch.float64)[:, None].expand(-1, half).contiguous(),
                    positions.double()[:, None] * inv_freq)[:, None]
    first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    t = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * z
    y[..., first], y[..., second] = t.real, t.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    c, P = case, case["page"]
    Nu, H, Hkv = c["units"], c["q_heads"], c["kv_heads"]
    if c["op"] == "rotate":
        v, got = s["valid"], {}
        for x, w in (("q", s["qw"]), ("k", s["kw"])):
            got[x] = s[x + "_out"].double()
            got[x][:v] = _turn64(s[x][:v], w, s["positions"][:v], s["inv_freq"], c["interleaved"])
        return got
    if c["op"] == "gather":
        got = {x: torch.zeros(s[x].shape, dtype=torch.float64, device=DEV) for x in ("k_pages", "v_pages")}
        for u in range(Nu):
            for g in range(Hkv):
                m = s["rows"][u][g]
                kept = s["indices"][u, int(s["offsets"][u, g]):][:m].long()
                pages = s["table"][u, g, :-(-m // P)].long()
                for x in ("k", "v"):
                    block = torch.zeros(pages.numel() * P, D, dtype=torch.float64, device=DEV)
                    block[:m] = s[x][u, g, kept].double()
                    got[x + "_pages"][pages] = block.view(-1, P, D)
        return {**got, "lengths": None}
    if c["op"] == "append":
        q, kp = s["q_out"].double(), s["k_pages"].double()
        v = s["valid"]
        q[:v] = _turn64(s["q"][:v], s["qw"], s["positions"][:v], s["inv_freq"], c["interleaved"])
        k = _turn64(s["k"][:v], s["kw"], s["positions"][:v], s["inv_freq"], c["interleaved"])
        for u in range(Nu):
            a, m = int(s["starts"][u]), s["n"][u]
            for g in range(Hkv):
                r = s["rows"][u][g] + torch.arange(m, device=DEV)
                kp[s["table"][u, g, r // P].long(), r % P] = k[a:a + m, g]
        return {"q": q, "k_pages": kp, "v_pages": None, "lengths": None}
    out, lse = s["out"].double(), s["lse"].double()
    G = H // Hkv
    for u in range(Nu):
        a, m = int(s["starts"][u]), s["n"][u]
        for g in range(Hkv if m else 0):
            length = s["rows"][u][g]
            pages = s["table"][u, g, :-(-length // P)].long()
            K = s["k_pages"][pages].reshape(-1, D)[:length].double()
            V = s["v_pages"][pages].reshape(-1, D)[:length].double()
            sees = torch.arange(length, device=DEV)[None] <= (length - m + torch.arange(m, device=DEV))[:, None]
            for h in range(g * G, (g + 1) * G):
                x = (s["q"][a:a + m, h].double() @ K.T / math.sqrt(D)).masked_fill(~sees, -math.inf)
                lse[a:a + m, h] = torch.logsumexp(x, -1)
                out[a:a + m, h] = torch.softmax(x, -1) @ V
    return {"out": out, "lse": lse}
