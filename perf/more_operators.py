"""Operators of a decoder that drafts trees of tokens on the paged cache and shares, grows and prunes its pages.

  masks    the ancestors of every drafted token as bits, and the tokens' positions, from the trees' parents
  attend   attention of the drafted tokens over the cache: each sees the rows before the tree and its own ancestors
  keep     rows moved together inside the pages: the accepted path of a tree, or the rows a retention pass chose
  reserve  pages for the rows to come (the lowest free ones), and the pages that hold no rows any more given back
  fork     a batch's sequences continued by new ones that share their pages; the first write copies the page it goes to;
           then the new ones end

``run`` computes each in its plain form (elementary torch operations, 32 bits, rounded once at the end), or, where ``own`` is
true, makes the calls that a user of ``paper_2602_08686_b200.binding`` makes.  ``exact`` states the attention in 64 bits; the
others move and count.  Notation as in include/ckv.h: Nu units (layer by layer: unit = layer * sequences + sequence), H query
heads, Hkv KV heads, G = H / Hkv, d = 128; a cache's state is its pages, the page table, the heads' lengths, the pages each
head holds (held) and, for each page, how many hold it (refs; 0: free).
"""
import math
import random

import torch

own = False
D = 128
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEV = "cuda"


# ------------------------------------------------------------------------------------------------ cases
def _case(name, op, dtype="bf16", seqs=1, layers=1, q_heads=32, kv_heads=8, cached=512, new=0, page=64, ragged=False, chain=0.3,
          path=0, budget=0, children=0, pool=0, pad=0):
    c = {"op": op, "dtype": dtype, "seqs": seqs, "layers": layers, "q_heads": q_heads, "kv_heads": kv_heads, "cached": cached,
         "new": new, "page": page, "ragged": ragged, "chain": chain, "path": path, "budget": budget, "children": children,
         "pool": pool, "pad": pad}
    return dict({"name": name}, **c) if name else c


def listed():
    return [
        # eight drafted tokens of one sequence whose prompt was compressed to 512 rows a head: latency
        _case("tree attend 1x8 on 512", "attend", seqs=1, new=8, cached=512, ragged=True),
        # a batch's trees of up to 63 tokens, ragged, a few padding rows behind the last
        _case("tree attend 16x63 on 8k", "attend", seqs=16, new=63, cached=8192, ragged=True, pad=5),
        # wide trees on prompts that were not compressed, seven query heads a KV head
        _case("tree attend 4x256 on 32k", "attend", seqs=4, q_heads=28, kv_heads=4, new=256, cached=32768, page=128),
        # the fp32 layer
        _case("tree attend f32 4x24 on 2k", "attend", "f32", seqs=4, q_heads=8, kv_heads=2, new=24, cached=2048, page=32, ragged=True),
        # the trees of a batch, once a step
        _case("tree masks 16x63", "masks", seqs=16, new=63, ragged=True),
        # few branches, deep: 512 tokens a sequence
        _case("tree masks 64x512 deep", "masks", seqs=64, new=512, chain=0.97),
        # up to eight of 63 drafted rows accepted, in all 32 layers of 16 sequences at once
        _case("keep path 16x32 layers", "keep", seqs=16, layers=32, new=63, path=8, cached=512, ragged=True),
        # 32k prompts in the cache of eight layers pruned to 4096 rows a head, where they lie
        _case("keep 4096 of 32k, 8 layers", "keep", seqs=1, layers=8, cached=32768, budget=4096, ragged=True),
        # one step of a batch of 32 in 32 layers, ragged heads: few of them need a page
        _case("reserve a step 32x32", "reserve", seqs=32, layers=32, cached=1024, new=1, page=32, ragged=True, pool=20000),
        # the pages of two prompts of 16k rows in 32 layers, from a pool of a million pages of which most are taken
        _case("reserve 2 prompts 16k", "reserve", seqs=2, layers=32, cached=0, new=16384, page=64, pool=1000000),
        # four samples of one prompt in one layer, and their first token's page
        _case("fork 1 to 4", "fork", seqs=1, layers=1, cached=2000, new=1, children=4, ragged=True),
        # eight samples of each of four prompts in 32 layers, and their first tokens' pages
        _case("fork 4 to 32, 32 layers", "fork", seqs=4, layers=32, cached=8000, new=5, children=32, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["attend", "attend", "attend", "masks", "keep", "keep", "reserve", "fork"])
    q_heads, kv_heads = rng.choice([(32, 8), (28, 4), (8, 2), (16, 16), (24, 2), (8, 1)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c = dict(dtype=dtype, q_heads=q_heads, kv_heads=kv_heads, page=rng.choice([16, 32, 64, 128, 256]), ragged=rng.random() < 0.6,
             chain=rng.choice([0.0, 0.3, 0.9]), pad=rng.choice([0, 0, 1, 17]))
    if op == "masks":
        return _case(None, op, seqs=_log(rng, 1, 64), new=_log(rng, 1, 512), **c)
    if op == "attend":
        seqs = _log(rng, 1, 16)
        new = _log(rng, 1, (256 if dtype == "bf16" else 32))
        return _case(None, op, seqs=seqs, new=new, cached=_log(rng, 1, min(32768, 65536 * 8 // (seqs * max(kv_heads, 4)))), **c)
    if op == "keep":
        layers = _log(rng, 1, 16)
        if rng.random() < 0.5:
            new = _log(rng, 2, 256)
            return _case(None, op, seqs=_log(rng, 1, 16), layers=layers, new=new, path=rng.randint(1, min(new, 12)), cached=_log(rng, 1, 2000), **c)
        cached = _log(rng, 100, 32768 // layers)
        return _case(None, op, seqs=1, layers=layers, cached=cached, budget=_log(rng, 10, cached), **c)
    if op == "reserve":
        return _case(None, op, seqs=_log(rng, 1, 16), layers=_log(rng, 1, 32), cached=_log(rng, 1, 2000), new=_log(rng, 1, 1000),
                     pool=_log(rng, 1, 200000), **c)
    seqs = rng.randint(1, 4)
    return _case(None, op, seqs=seqs, layers=_log(rng, 1, 16), cached=_log(rng, 1, 4000), new=_log(rng, 1, 64),
                 children=_log(rng, 1, 32), **c)


def _words(c):
    return (c["new"] + 31) // 32


def _plan(c):
    """What the case alone decides: drafted tokens of every sequence, rows cached (before them) for every (unit, KV head), and
    how many rows the lists of `keep` have."""
    r = random.Random("%(seqs)d %(layers)d %(kv_heads)d %(new)d %(cached)d %(path)d %(budget)d" % c)
    S, Nu, Hkv = c["seqs"], c["seqs"] * c["layers"], c["kv_heads"]
    n = [c["new"]] * S
    if c["ragged"] and c["new"] > 1 and S > 1:
        n = [r.randint((c["new"] + 1) // 2, c["new"]) if r.random() < 0.9 else r.randint(1, c["new"]) for _ in range(S)]
        n[r.randrange(S)] = c["new"]
    low = c["cached"] - c["cached"] // 4
    lens = [[r.randint(low, c["cached"]) if c["ragged"] else c["cached"] for _ in range(Hkv)] for _ in range(Nu)]
    if c["path"]:
        counts = [r.randint(1, min(c["path"], n[s])) for s in range(S)]
    else:
        counts = [r.randint(c["budget"] - c["budget"] // 2, c["budget"]) if c["ragged"] else c["budget"] for _ in range(Nu * Hkv)]
        counts = [min(m, lens[i // Hkv][i % Hkv]) for i, m in enumerate(counts)]
    return n, lens, counts


# ----------------------------------------------------------------------------------------------- inputs
def _table(c, rows, max_rows, gen, spare):
    """Pages of a pool, in random order, for the (unit, head) rows; `spare` more pages, half of them held by nobody here."""
    P = c["page"]
    held = (torch.tensor(rows, device=DEV) + P - 1) // P                       # [Nu, Hkv]
    max_pages = max(1, -(-max_rows // P))
    total = int(held.sum())
    n_pages = total + spare
    perm = torch.randperm(n_pages, generator=gen, device=DEV).int()
    table = torch.zeros(*held.shape, max_pages, dtype=torch.int32, device=DEV)
    table[torch.arange(max_pages, device=DEV) < held[..., None]] = perm[:total]
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[perm[:total].long()] = 1
    return table, held.int(), refs, perm[total:].long()


def _pools(c, n_pages, gen, filled=True):
    dt, P = DT[c["dtype"]], c["page"]
    if not filled:
        return tuple(torch.empty(n_pages, P, D, device=DEV, dtype=dt) for _ in range(2))
    return tuple(torch.randn(n_pages, P, D, generator=gen, device=DEV, dtype=dt) for _ in range(2))


def _trees(n, chain, gen):
    """Parents of the packed tokens inside their sequence (-1: a root), sequence and place of each token."""
    count = torch.tensor(n, device=DEV)
    seq = torch.repeat_interleave(torch.arange(len(n), device=DEV), count)
    first = torch.cumsum(count, 0) - count
    place = torch.arange(sum(n), device=DEV) - first[seq]
    x, y = torch.rand(2, sum(n), generator=gen, device=DEV)
    earlier = (x * (place + 1)).long().clamp(max=place.max() if sum(n) else 0).minimum(place) - 1    # -1 .. place - 1
    return torch.where(y < chain, place - 1, earlier).int(), seq, place


def _bits(parents, seq, place, n, words):
    """Ancestors (the token included) of every packed token as bits: int32 [T, words]."""
    S, most = len(n), max(n)
    up = torch.full((S, most + 1), most, dtype=torch.long, device=DEV)       # place `most`: above the roots
    up[seq, place] = torch.where(parents < 0, most, parents.long())
    sees = torch.zeros(S, most + 1, 32 * words, dtype=torch.bool, device=DEV)
    sees[seq, place, place] = True
    depth = torch.zeros(S, most + 1, dtype=torch.long, device=DEV)
    depth[seq, place] = (parents >= 0).long()
    for _ in range(max(most - 1, 1).bit_length()):                             # ancestors' ancestors
        sees = sees | torch.gather(sees, 1, up[..., None].expand(-1, -1, 32 * words))
        depth = depth + torch.gather(depth, 1, up)
        up = torch.gather(up, 1, up)
    at = sees[seq, place].view(-1, words, 32)
    word = (at.long() << torch.arange(32, device=DEV)).sum(-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).int(), depth[seq, place].int()


def prepare(case, seed):
    c, dt = case, DT[case["dtype"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    S, Nu, H, Hkv, P = c["seqs"], c["seqs"] * c["layers"], c["q_heads"], c["kv_heads"], c["page"]
    n, lens, counts = _plan(c)
    s = {"c": c, "n": n, "lens": lens}
    if own:
        from paper_2602_08686_b200 import binding as b
    if c["op"] in ("masks", "attend"):
        T, words = sum(n) + c["pad"], _words(c)
        s["starts"] = torch.tensor([sum(n[:u]) for u in range(S + 1)], dtype=torch.int32, device=DEV)
        parents, s["seq"], s["place"] = _trees(n, c["chain"], gen)
        s["valid"] = sum(n)
    if c["op"] == "masks":
        s["parents"] = torch.zeros(T, dtype=torch.int32, device=DEV)
        s["parents"][:s["valid"]] = parents
        s["first"] = torch.randint(0, 100000, (S,), generator=gen, device=DEV, dtype=torch.int32)
        s["masks"] = torch.zeros(T, words, dtype=torch.int32, device=DEV)
        s["positions"] = torch.zeros(T, dtype=torch.int32, device=DEV)
        if own:
            s["ws"] = torch.zeros(256, dtype=torch.uint8, device=DEV)
        return s
    if c["op"] == "attend":
        rows = [[x + n[u] for x in lens[u]] for u in range(S)]                 # the drafted tokens' own rows included
        s["rows"] = rows
        s["table"], _, refs, _ = _table(c, rows, max(map(max, rows)), gen, 3)
        s["k_pages"], s["v_pages"] = _pools(c, refs.numel(), gen)
        s["lengths"] = torch.tensor(rows, dtype=torch.int32, device=DEV)
        s["masks"] = torch.zeros(T, words, dtype=torch.int32, device=DEV)
        s["masks"][:s["valid"]] = _bits(parents, s["seq"], s["place"], n, words)[0]
        q = torch.randn(T, H, D, generator=gen, device=DEV)
        s["q"] = q.to(dt)
        # an attention sink in row 0 of every head, along the mean query of its group
        mean = torch.stack([q[sum(n[:u]):sum(n[:u]) + n[u]].mean(0) for u in range(S)]).view(S, Hkv, H // Hkv, D).mean(2)
        s["k_pages"][s["table"][:, :, 0].long(), 0] = (2.0 * math.sqrt(D) * mean / mean.norm(dim=-1, keepdim=True).clamp_min(1e-6)).to(dt)
        s["out"] = torch.zeros(T, H, D, device=DEV, dtype=dt)
        s["lse"] = torch.zeros(T, H, device=DEV)
        s["scale"] = 1.0 / math.sqrt(D)
        if own:
            s["paged"] = b.make_paged(s["k_pages"], s["table"], q=s["q"], max_new=c["new"])
            s["ws"] = b.alloc_paged_workspace(s["paged"])
        return s
    if c["op"] == "keep":
        tail = torch.tensor(n if c["path"] else [0], device=DEV)
        rows = [[x + (n[u % S] if c["path"] else 0) for x in lens[u]] for u in range(Nu)]
        s["table"], s["held"], refs, _ = _table(c, rows, max(map(max, rows)), gen, 3)
        s["refs"] = refs
        s["k_pages"], s["v_pages"] = _pools(c, refs.numel(), gen)
        s["lengths"] = torch.tensor(rows, dtype=torch.int32, device=DEV)
        s["new_lengths"] = torch.zeros_like(s["lengths"])
        # ascending lists: a path's places in its tree, or the rows of a head that are kept (its first four always)
        span = tail if c["path"] else s["lengths"].flatten().long()
        count = torch.tensor(counts, device=DEV)
        order = torch.rand(len(counts), int(span.max()), generator=gen, device=DEV)
        if not c["path"]:
            order[:, :4] = -1.0
        order.masked_fill_(torch.arange(order.shape[1], device=DEV) >= span[:, None], 2.0)
        chosen = order.argsort(-1).argsort(-1) < count[:, None]
        s["list"] = chosen.nonzero()[:, 1].int()
        s["counts"] = count.int()
        s["begins"] = (torch.cumsum(count, 0) - count).int()
        s["tails"] = tail.int() if c["path"] else None
        s["most"] = max(counts)
        if own:
            s["paged"] = b.make_paged(s["k_pages"], s["table"], n_q_heads=H)
            s["ws"] = b.alloc_pages_workspace(s["paged"])
        return s
    S2 = c["children"] if c["op"] == "fork" else S
    more = [[max(0, -(-(x + c["new"]) // P) - x // P) for x in row] for row in lens]    # pages that growing takes at most
    spare = 3 + sum(map(sum, more)) * (-(-S2 // S)) + c["pool"]
    s["table"], s["held"], s["refs"], others = _table(c, lens, max(map(max, lens)) + c["new"], gen, spare)
    # of the pages that growing can do without, the larger part is held by other batches
    taken = others[torch.randperm(others.numel(), generator=gen, device=DEV)[:c["pool"] * 7 // 8]]
    s["refs"][taken] = 1
    s["k_pages"], s["v_pages"] = _pools(c, s["refs"].numel(), gen, filled=c["op"] == "fork")
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["room"] = torch.zeros(2, dtype=torch.int32, device=DEV)
    s["new_rows"] = torch.tensor(n if c["op"] == "reserve" else [c["new"]] * S2, dtype=torch.int32, device=DEV)
    if c["op"] == "fork":
        parents = torch.arange(S2, device=DEV) * S // S2                       # every sequence goes on, as evenly as may be
        s["parents"] = parents[torch.randperm(S2, generator=gen, device=DEV)].int()
        s["table2"] = torch.zeros(S2 * c["layers"], Hkv, s["table"].shape[2], dtype=torch.int32, device=DEV)
        s["lengths2"], s["held2"] = (torch.zeros(S2 * c["layers"], Hkv, dtype=torch.int32, device=DEV) for _ in range(2))
    if own:
        s["paged"] = b.make_paged(s["k_pages"], s["table"], n_q_heads=H)
        s["ws"] = b.alloc_pages_workspace(s["paged"])
        if c["op"] == "fork":
            s["paged2"] = b.make_paged(s["k_pages"], s["table2"], n_q_heads=H)
            s["ws"] = b.alloc_pages_workspace(s["paged2"])
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_masks(s):
    v = s["valid"]
    bits, depth = _bits(s["parents"][:v], s["seq"], s["place"], s["n"], s["masks"].shape[1])
    s["masks"][:v] = bits
    s["positions"][:v] = s["first"][s["seq"]] + depth


def _plain_attend(s):
    c, P = s["c"], s["c"]["page"]
    Nu, H, Hkv = c["seqs"], c["q_heads"], c["kv_heads"]
    G, nmax, Lmax = H // Hkv, max(s["n"]), max(map(max, s["rows"]))
    j = torch.arange(Lmax, device=DEV)
    page = torch.gather(s["table"].long(), 2, (j // P).expand(Nu, Hkv, Lmax))
    place = page * P + j % P
    K = s["k_pages"].view(-1, D)[place].float()                                # [Nu, Hkv, Lmax, D]
    V = torch.where((j < s["lengths"][..., None])[..., None], s["v_pages"].view(-1, D)[place].float(), 0.0)
    count = (s["starts"][1:] - s["starts"][:-1]).long()
    i = torch.arange(nmax, device=DEV)
    token = (s["starts"][:-1].long()[:, None] + i).clamp(max=s["q"].shape[0] - 1)          # [Nu, nmax]
    q = s["q"][token].float().view(Nu, nmax, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(Nu, Hkv, G * nmax, D)
    x = torch.matmul(q, K.transpose(-1, -2)).mul_(s["scale"]).view(Nu, Hkv, G, nmax, Lmax)
    # the rows before the tree, and of the tree's those whose bit is set
    t = j - (s["lengths"].long() - count[:, None])[..., None]                  # [Nu, Hkv, Lmax]: which drafted token's row it is
    bits = (s["masks"][token][..., None] >> torch.arange(32, device=DEV) & 1).bool().flatten(2)          # [Nu, nmax, 32 words]
    hit = torch.gather(bits[:, None].expand(-1, Hkv, -1, -1), 3, t.clamp(0, bits.shape[2] - 1)[:, :, None].expand(-1, -1, nmax, -1))
    sees = (t < 0)[:, :, None] | (hit & (t < count[:, None, None])[:, :, None])            # [Nu, Hkv, nmax, Lmax]
    x.masked_fill_(~sees[:, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)                                      # [Nu, Hkv, G, nmax]
    o = torch.matmul(x.view(Nu, Hkv, G * nmax, Lmax), V).view(Nu, Hkv, G, nmax, D)
    o = o / torch.where(total > 0, total, 1.0)
    v = s["valid"]
    s["out"][:v] = o.permute(0, 3, 1, 2, 4).reshape(Nu, nmax, H, D)[s["seq"], s["place"]].to(s["q"].dtype)
    s["lse"][:v] = lse.permute(0, 3, 1, 2).reshape(Nu, nmax, H)[s["seq"], s["place"]]


def _plain_keep(s):
    c, P = s["c"], s["c"]["page"]
    Nu, Hkv, S = c["seqs"] * c["layers"], c["kv_heads"], c["seqs"]
    per_pair = torch.arange(Nu * Hkv, device=DEV) if s["tails"] is None else \
        (torch.arange(Nu, device=DEV) % S)[:, None].expand(Nu, Hkv).reshape(-1)            # which list is a head's
    length = s["lengths"].flatten().long()
    base = torch.zeros_like(length) if s["tails"] is None else length - s["tails"].long()[per_pair]
    count, begin = s["counts"].long()[per_pair], s["begins"].long()[per_pair]
    i = torch.arange(s["most"], device=DEV).expand(Nu * Hkv, -1)
    i = torch.where(i < count[:, None], i, 0)                                  # behind the list: its first entry again
    src = base[:, None] + s["list"].long()[begin[:, None] + i]
    dst = base[:, None] + i
    none = count[:, None] == 0
    src, dst = (torch.where(none, (length - 1)[:, None], x) for x in (src, dst))
    table = s["table"].long().view(Nu * Hkv, -1)
    src, dst = (torch.gather(table, 1, x // P) * P + x % P for x in (src, dst))
    for pool in (s["k_pages"], s["v_pages"]):
        flat = pool.view(-1, D)
        flat[dst] = flat[src]
    s["new_lengths"].copy_((base + count).view(Nu, Hkv))


def _plain_reserve(s, table, lengths, held, new_rows):
    """Pages for rows length .. length + new - 1 of every head; shared ones among them are replaced by copies."""
    P, refs = s["c"]["page"], s["refs"]
    Nu, Hkv, slots = table.shape
    new = new_rows[torch.arange(Nu, device=DEV) % new_rows.numel()][:, None]
    j = torch.arange(slots, device=DEV)
    want = torch.where(new > 0, (lengths + new + P - 1) // P, 0)
    first = lengths // P
    mine = j < held[..., None]
    shared = mine & (j >= first[..., None]) & (j < want[..., None]) & (refs[table.long()] > 1)
    need = shared | (~mine & (j < want[..., None]))
    rank = torch.cumsum(need.flatten(), 0) - 1
    free = refs == 0
    order = torch.cumsum(free, 0) - 1
    n = refs.numel()
    by_rank = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    by_rank.scatter_(0, torch.where(free, order, n), torch.arange(n, dtype=torch.int32, device=DEV))
    asked, there = rank[-1] + 1, order[-1] + 1
    enough = asked <= there
    got = by_rank[rank.clamp(0, n - 1)].view(need.shape)
    fresh = torch.where(need & enough, got, table)
    if s["c"]["op"] == "fork":                                                 # only a shared page has rows to copy
        at = first.clamp(max=slots - 1)[..., None].long()
        old, to = torch.gather(table, 2, at).flatten().long(), torch.gather(fresh, 2, at).flatten().long()
        rows = (torch.arange(P, device=DEV) < (lengths - first * P).view(-1, 1))[..., None]
        moves = torch.gather(shared, 2, at).flatten()[:, None, None]
        to = torch.where(moves[:, 0, 0], to, old)
        for pool in (s["k_pages"], s["v_pages"]):
            pool[to] = torch.where(rows & moves, pool[old], pool[to])
    refs.scatter_add_(0, table.flatten().long(), -(shared & enough).flatten().int())
    refs.scatter_add_(0, fresh.flatten().long(), (need & enough).flatten().int())
    table.copy_(fresh)
    held.copy_(torch.where(enough, torch.maximum(held, want), held))
    s["room"].copy_(torch.stack((torch.where(enough, there - asked, there), torch.where(enough, 0, asked - there))))


def _plain_trim(s, table, lengths, held):
    P = s["c"]["page"]
    keep = torch.zeros_like(held) if lengths is None else torch.minimum(held, (lengths + P - 1) // P)
    j = torch.arange(table.shape[2], device=DEV)
    gone = (j >= keep[..., None]) & (j < held[..., None])
    s["refs"].scatter_add_(0, table.flatten().long(), -gone.flatten().int())
    held.copy_(keep)


def _plain_fork(s):
    c = s["c"]
    S, layers, p = c["seqs"], c["layers"], s["parents"].long()
    src = (torch.arange(layers, device=DEV)[:, None] * S + p).flatten()
    s["lengths2"].copy_(s["lengths"][src])
    s["held2"].copy_(s["held"][src])
    j = torch.arange(s["table"].shape[2], device=DEV)
    s["table2"].copy_(torch.where(j < s["held2"][..., None], s["table"][src], s["table2"]))
    children = torch.zeros(S, dtype=torch.int32, device=DEV).scatter_add_(0, p, torch.ones_like(s["parents"]))
    more = torch.where(j < s["held"][..., None], children.repeat(layers)[:, None, None], 0)
    s["refs"].scatter_add_(0, s["table"].flatten().long(), more.flatten().int())


# -------------------------------------------------------------------------------------------------- run
def run(s):
    c = s["c"]
    if own:
        from paper_2602_08686_b200 import binding as b
    if c["op"] == "masks":
        if own:
            b.ckv_tree_masks(s["parents"], s["starts"], s["masks"], s["ws"], positions=s["positions"], first_positions=s["first"])
        else:
            _plain_masks(s)
        return {"masks": s["masks"], "positions": s["positions"]}
    if c["op"] == "attend":
        if own:
            b.ckv_tree_attend(s["paged"], s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["starts"], s["masks"],
                              s["out"], s["ws"], lse=s["lse"])
        else:
            _plain_attend(s)
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "keep":
        if own:
            b.ckv_keep_rows(s["paged"], s["list"], s["begins"], s["counts"], s["lengths"], s["table"], s["k_pages"], s["v_pages"],
                            s["new_lengths"], s["ws"], tails=s["tails"], refs=s["refs"], layers=c["layers"])
        else:
            _plain_keep(s)
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "lengths": s["new_lengths"]}
    if c["op"] == "reserve":     # a step's pages, and given back: its rows were not kept
        if own:
            b.ckv_pages_reserve(s["paged"], s["new_rows"], s["lengths"], s["held"], s["table"], s["refs"], s["k_pages"], s["v_pages"],
                                s["ws"], room=s["room"], layers=c["layers"])
            b.ckv_pages_trim(s["paged"], s["lengths"], s["held"], s["table"], s["refs"], s["ws"])
        else:
            _plain_reserve(s, s["table"], s["lengths"], s["held"], s["new_rows"])
            _plain_trim(s, s["table"], s["lengths"], s["held"])
        return {"table": s["table"], "held": s["held"], "refs": s["refs"], "room": s["room"]}
    if own:
        b.ckv_pages_fork(s["paged"], s["parents"], s["lengths"], s["held"], s["table"], s["refs"], s["lengths2"], s["held2"],
                         s["table2"], s["ws"], layers=c["layers"], keep_old=True)
        b.ckv_pages_reserve(s["paged2"], s["new_rows"], s["lengths2"], s["held2"], s["table2"], s["refs"], s["k_pages"], s["v_pages"],
                            s["ws"], room=s["room"], layers=c["layers"])
        b.ckv_pages_trim(s["paged2"], None, s["held2"], s["table2"], s["refs"], s["ws"])
    else:
        _plain_fork(s)
        _plain_reserve(s, s["table2"], s["lengths2"], s["held2"], s["new_rows"])
        _plain_trim(s, s["table2"], None, s["held2"])
    return {"table": s["table2"], "lengths": s["lengths2"], "held": s["held2"], "refs": s["refs"], "room": s["room"],
            "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    n, lens, counts = _plan(c)
    S, Nu, H, Hkv, P, T = c["seqs"], c["seqs"] * c["layers"], c["q_heads"], c["kv_heads"], c["page"], sum(n)
    if c["op"] == "masks":
        return {"bytes": T * (8 + 4 * _words(c)) + 8 * S, "flops": 0}
    if c["op"] == "attend":
        rows = sum(x + n[u] for u in range(S) for x in lens[u])
        pairs = sum(H // Hkv * n[u] * (x + 1) for u in range(S) for x in lens[u])      # the rows before the tree, and its own
        return {"bytes": 2 * rows * D * e + 2 * T * H * D * e + 4 * T * H + 4 * T * _words(c), "flops": 4 * D * pairs}
    if c["op"] == "keep":
        moved = sum(counts) * (c["layers"] * Hkv if c["path"] else 1)
        return {"bytes": moved * 4 * D * e + 4 * sum(counts) + 12 * Nu * Hkv, "flops": 0}
    held = sum(-(-x // P) for row in lens for x in row)
    if c["op"] == "reserve":
        new = sum(-(-(x + n[u % S]) // P) - -(-x // P) for u in range(Nu) for x in lens[u])
        other = 3 + sum(max(0, -(-(x + c["new"]) // P) - x // P) for row in lens for x in row) + c["pool"]
        return {"bytes": 4 * (held + other) + 24 * Nu * Hkv + 24 * new, "flops": 0}    # every page's count read, new pages' table and counts there and back
    times = c["children"] / S
    copied = sum(x % P for row in lens for x in row) * times
    return {"bytes": 4 * D * e * copied + held * (12 + 16 * times) + 24 * Nu * Hkv * times, "flops": 0}


# ------------------------------------------------------------------------------------------------ exact
def exact(case, seed):
    """The attention from its definition in 64 bits, head by head; the other operators move and count."""
    if case["op"] != "attend":
        return None
    s = prepare(case, seed)
    H, Hkv = case["q_heads"], case["kv_heads"]
    out, lse = s["out"].double(), s["lse"].double()
    masks = s["masks"].cpu().numpy().view("uint32")
    for u in range(case["seqs"]):
        a, m = int(s["starts"][u]), s["n"][u]
        tree = torch.tensor([[bool(masks[a + i, t // 32] >> (t % 32) & 1) for t in range(m)] for i in range(m)], device=DEV)
        for g in range(Hkv):
            length = s["rows"][u][g]
            pages = s["table"][u, g, :-(-length // case["page"])].long()
            K = s["k_pages"][pages].reshape(-1, D)[:length].double()
            V = s["v_pages"][pages].reshape(-1, D)[:length].double()
            sees = torch.ones(m, length, dtype=torch.bool, device=DEV)
            sees[:, length - m:] = tree
            for h in range(g * (H // Hkv), (g + 1) * (H // Hkv)):
                x = (s["q"][a:a + m, h].double() @ K.T / math.sqrt(D)).masked_fill(~sees, -math.inf)
                lse[a:a + m, h] = torch.logsumexp(x, -1)
                out[a:a + m, h] = torch.softmax(x, -1) @ V
    return {"out": out, "lse": lse}
