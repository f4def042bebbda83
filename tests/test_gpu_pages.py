"""GPU tests of the calls that manage the pages of a cache, against statements of them one entry at a time (tests/tree_reference.py);
rows are compared bit by bit.  Then the calls together, as a decoder makes them."""
import os
import random

import numpy as np
import pytest
import torch

import tree_reference as TR

pytestmark = pytest.mark.gpu
D = 128
EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2602_08686_b200 import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


class Cache:
    """A state at random: pages of a pool handed out in random order, some shared between neighbouring units."""

    def __init__(self, B, layers, seqs, Hkv, P, width, spare, dtype=torch.bfloat16, seed=0, share=0.0, row_pad=0, most=None, other=0.4):
        rng = np.random.RandomState(seed)
        Nu = layers * seqs
        held = rng.randint(0, (width if most is None else most) + 1, (Nu, Hkv)).astype(np.int32)
        total = int(held.sum())
        n_pages = total + spare
        perm = rng.permutation(n_pages)
        refs = np.zeros(n_pages, np.int32)
        refs[perm[total:]] = rng.rand(spare) < other                   # pages of other batches
        table = np.full((Nu, Hkv, width), 0x7ffffff0, np.int32)
        lengths = np.zeros((Nu, Hkv), np.int32)
        at = 0
        for u in range(Nu):
            for g in range(Hkv):
                h = int(held[u, g])
                table[u, g, :h] = perm[at:at + h]
                at += h
                if u and share:
                    both = min(h, int(held[u - 1, g]))
                    mine = rng.rand(both) < share
                    table[u, g, :both][mine] = table[u - 1, g, :both][mine]
                refs_of = table[u, g, :h]
                np.add.at(refs, refs_of, 1)
                lengths[u, g] = rng.randint(0, h * P + 1) if h else 0
        refs[perm[:total]] = 0
        for u, g in np.ndindex(Nu, Hkv):
            np.add.at(refs, table[u, g, :held[u, g]], 1)
        self.ref = TR.Pages(P, refs, held, table, lengths)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        pools = [torch.randn(n_pages, P, D + row_pad, generator=gen, device="cuda").to(dtype) for _ in range(2)]
        self.pools, (self.k, self.v) = pools, (p[..., :D] for p in pools)
        self.refs, self.held, self.table, self.lengths = (i32(x) for x in (refs, held, table, lengths))
        self.layers, self.Hkv, self.n_pages = layers, Hkv, n_pages
        self.pg = B.make_paged(self.k, self.table)
        n = B.ckv_pages_workspace_bytes(self.pg)
        self.guard = torch.full((n + 512,), 0xAB, dtype=torch.uint8, device="cuda")
        self.ws = self.guard[256:256 + n]

    def fine(self, B, status=0):
        assert B.ckv_device_status(self.ws) == status
        assert (self.guard[:256] == 0xAB).all() and (self.guard[256 + self.ws.numel():] == 0xAB).all()

    def same(self):
        for name in ("refs", "held", "table"):
            got, want = getattr(self, name).cpu().numpy(), getattr(self.ref, name)
            assert np.array_equal(got, want), (name, np.argwhere(got != want)[:5])


SHAPES = [  # layers, sequences, KV heads, page, width, spare pages, share
    (1, 1, 1, 16, 3, 2, 0.0), (1, 1, 8, 64, 9, 70, 0.0), (2, 3, 4, 16, 5, 200, 0.5), (4, 8, 8, 32, 7, 3000, 0.3), (32, 4, 8, 16, 4, 9000, 0.4),
    (3, 5, 1, 256, 6, 5000, 0.2), (1, 700, 2, 16, 3, 400, 0.6), (16, 64, 8, 16, 2, 30000, 0.1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layers,seqs,Hkv,P,width,spare,share", SHAPES)
def test_reserve_and_trim(B, dtype, layers, seqs, Hkv, P, width, spare, share):
    if dtype == torch.float32 and layers * seqs * Hkv > 4000:
        pytest.skip("rows are moved alike")
    rng = np.random.RandomState(P + seqs)
    for step, per_head in enumerate((False, True, False)):
        c = Cache(B, layers, seqs, Hkv, P, width, spare, dtype, seed=step, share=share, row_pad=8 * step, most=max(1, width - step))
        for more_rows in (1, 2 * P + 3):
            most = [rng.randint(0, more_rows + 1) for _ in range(layers * seqs * Hkv if per_head else seqs)]
            most = np.minimum(most, max(1, (width * P - int(c.ref.lengths.max()))))      # inside the table
            room = torch.full((2,), -3, dtype=torch.int32, device="cuda")
            before = [p.clone() for p in c.pools]
            B.ckv_pages_reserve(c.pg, i32(most), c.lengths, c.held, c.table, c.refs, c.k, c.v, c.ws, room=room, layers=layers)
            each = np.reshape(most, c.ref.lengths.shape) if per_head else np.tile(most, layers)[:, None]
            full = bool(((each > 0) & (c.ref.lengths + each > width * P)).any())
            want_room, copies = c.ref.reserve(most, layers)
            c.fine(B, B.ERR_PAGE if full else 0)
            assert tuple(room.tolist()) == want_room
            c.same()
            for src, dst, rows in copies:
                for p, old in zip(c.pools, before):
                    old[dst, :rows, :D] = old[src, :rows, :D]
            for p, old in zip(c.pools, before):
                assert torch.equal(p, old)
        # some heads lose rows, some units end
        lengths = np.maximum(c.ref.lengths - rng.randint(0, 2 * P, c.ref.lengths.shape), 0).astype(np.int32)
        lengths[::3] = 0
        B.ckv_pages_trim(c.pg, i32(lengths), c.held, c.table, c.refs, c.ws)
        c.ref.trim(lengths)
        c.fine(B), c.same()
        B.ckv_pages_trim(c.pg, None, c.held, c.table, c.refs, c.ws)
        c.ref.trim()
        c.fine(B), c.same()


def test_reserve_is_all_or_nothing(B):
    for seqs in (2, 900):
        c = Cache(B, 1, seqs, 2, 16, 40, 50, seed=3, most=2, other=0.0)
        need = sum(-(-(int(x) + 200) // 16) - int(h) for x, h in zip(c.ref.lengths.flatten(), c.ref.held.flatten()))
        room, more = torch.zeros(2, dtype=torch.int32, device="cuda"), i32([200] * seqs)
        B.ckv_pages_reserve(c.pg, more, c.lengths, c.held, c.table, c.refs, c.k, c.v, c.ws, room=room)
        free = int((c.ref.refs == 0).sum())
        if need <= free:
            assert seqs == 2
            c.ref.reserve([200] * seqs)
            assert room.tolist() == [free - need, 0]
        else:
            assert room.tolist() == [free, need - free]
        c.fine(B), c.same()
        # exactly as many as there are, and one fewer
        free = int((c.ref.refs == 0).sum())
        one = Cache(B, 1, 1, 1, 16, free + 2, free, seed=4, most=0, other=0.0)
        for rows, want in ((16 * free + 1, [free, 1]), (16 * free, [0, 0])):
            B.ckv_pages_reserve(one.pg, i32([rows]), one.lengths, one.held, one.table, one.refs, one.k, one.v, one.ws, room=room)
            assert room.tolist() == want
            one.ref.reserve([rows])
            one.fine(B), one.same()


def test_reserve_from_a_large_pool(B):
    """Two million pages, most of them taken; a pool past 2^32 bytes whose far end is written."""
    n, P = 2100000, 16
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    rng = np.random.RandomState(1)
    refs = (rng.rand(n) < 0.98).astype(np.int32)
    refs[-300:] = 0
    k, v = (torch.empty(n, P, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for Nu, Hkv, width, rows in ((2, 2, 10, 150), (40, 8, 90, 1400), (300, 3, 6, 70)):
        held = np.zeros((Nu, Hkv), np.int32)
        held[0, 0] = 1
        table = np.full((Nu, Hkv, width), -9, np.int32)
        table[0, 0, 0] = n - 1
        refs[n - 1] = 2                                                    # shared, with five rows
        lengths = np.zeros((Nu, Hkv), np.int32)
        lengths[0, 0] = 5
        k[n - 1], v[n - 1] = 3.0, 4.0
        ref = TR.Pages(P, refs, held, table, lengths)
        d = [i32(x) for x in (lengths, held, table, refs)]
        pg = B.make_paged(k, d[2])
        ws, room = B.alloc_pages_workspace(pg), torch.zeros(2, dtype=torch.int32, device="cuda")
        B.ckv_pages_reserve(pg, i32([rows] * Nu), *d, k, v, ws, room=room)
        want, copies = ref.reserve([rows] * Nu)
        assert B.ckv_device_status(ws) == B.OK and tuple(room.tolist()) == want and want[1] == 0
        for x, y in zip(d[1:], (ref.held, ref.table, ref.refs)):
            assert np.array_equal(x.cpu().numpy(), y)
        (src, dst, m), = copies
        assert src == n - 1 and (k[dst, :m] == 3).all() and (v[dst, :m] == 4).all()


def test_reserve_says_what_is_wrong(B):
    """Rows past the table, pages outside the pool, negative lengths and counts: reported, the rest is done."""
    for seqs in (3, 700):
        c = Cache(B, 1, seqs, 1, 16, 4, 5000, seed=8, most=3, other=0.0)
        more = np.full(seqs, 2, np.int32)
        more[0] = 1000                                                      # more than the table has room for
        B.ckv_pages_reserve(c.pg, i32(more), c.lengths, c.held, c.table, c.refs, c.k, c.v, c.ws)
        c.ref.reserve(more)
        c.fine(B, B.ERR_PAGE), c.same()
        assert int(c.held[0, 0]) == 4
        # a page number outside the pool where a row would be written: that page is left alone
        u = next(i for i in range(seqs) if c.ref.lengths[i, 0] // 16 < c.ref.held[i, 0])
        s = int(c.ref.lengths[u, 0]) // 16
        keep = int(c.table[u, 0, s])
        c.table[u, 0, s] = c.n_pages
        B.ckv_pages_reserve(c.pg, i32([1] * seqs), c.lengths, c.held, c.table, c.refs, c.k, c.v, c.ws)
        c.fine(B, B.ERR_PAGE)
        assert int(c.table[u, 0, s]) == c.n_pages
        c.table[u, 0, s] = keep
        c.ref.reserve([1] * seqs)
        c.same()
        lengths = c.lengths.clone()
        lengths[1, 0] = -1
        B.ckv_pages_reserve(c.pg, i32([0] * seqs), lengths, c.held, c.table, c.refs, c.k, c.v, c.ws)
        c.fine(B, B.ERR_PAGE), c.same()
        B.ckv_pages_trim(c.pg, lengths, c.held, c.table, c.refs, c.ws)      # the others are trimmed
        other = c.ref.lengths.copy()
        other[1, 0] = 64
        c.ref.trim(other)
        c.fine(B, B.ERR_PAGE), c.same()
        # a page that nobody holds is given back
        u = next(i for i in range(seqs) if c.ref.held[i, 0] > 0)
        c.refs[c.table[u, 0, 0].long()] = 0
        B.ckv_pages_trim(c.pg, None, c.held, c.table, c.refs, c.ws)
        c.fine(B, B.ERR_PAGE)
        c.ref.refs[c.ref.table[u, 0, 0]] = 1
        c.ref.trim()
        c.same()                                                            # counts of others, and none below zero


@pytest.mark.parametrize("keep_old", [False, True])
@pytest.mark.parametrize("layers,seqs,Hkv,P,width,n_new", [
    (1, 1, 1, 16, 3, 1), (1, 1, 8, 64, 40, 4), (2, 3, 4, 16, 50, 7), (32, 4, 8, 32, 5, 32), (3, 70, 2, 16, 3, 90), (1, 5, 2, 16, 300, 0)])
def test_fork(B, keep_old, layers, seqs, Hkv, P, width, n_new):
    rng = np.random.RandomState(n_new)
    c = Cache(B, layers, seqs, Hkv, P, width, 20, seed=n_new, share=0.3)
    for turn in range(3):
        parents = rng.randint(-1, seqs, n_new)
        if turn == 1:
            parents[:] = np.arange(n_new) % seqs                            # as they are, as far as they go
        new = [torch.full(s, 7, dtype=torch.int32, device="cuda") for s in
               ((layers * n_new, Hkv), (layers * n_new, Hkv), (layers * n_new, Hkv, width))]
        B.ckv_pages_fork(c.pg, i32(parents), c.lengths, c.held, c.table, c.refs, *new, c.ws, layers=layers, keep_old=keep_old)
        ref = c.ref.fork(parents, layers, keep_old, fill=7)
        c.fine(B)
        for x, y in zip(new + [c.refs], (ref.lengths, ref.held, ref.table, ref.refs)):
            assert np.array_equal(x.cpu().numpy(), y)
        assert (ref.refs >= 0).all()
        if n_new:                                                           # the new ones end; the old ones are back
            pg = B.make_paged(c.k, new[2])
            B.ckv_pages_trim(pg, None, new[1], new[2], c.refs, c.ws)
            ref.trim()
            assert np.array_equal(c.refs.cpu().numpy(), ref.refs) and (new[1] == 0).all()
        c.refs.copy_(i32(c.ref.refs))


def test_fork_says_what_is_wrong(B):
    c = Cache(B, 1, 3, 2, 16, 4, 9, seed=1)
    new = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((4, 2), (4, 2), (4, 2, 4))]
    B.ckv_pages_fork(c.pg, i32([1, 3, -2, 1]), c.lengths, c.held, c.table, c.refs, *new, c.ws, keep_old=True)
    ref = c.ref.fork([1, -1, -1, 1], 1, True)
    c.fine(B, B.ERR_PAGE)
    for x, y in zip(new + [c.refs], (ref.lengths, ref.held, ref.table, ref.refs)):
        assert np.array_equal(x.cpu().numpy(), y)


# -------------------------------------------------------------------------------------------------- keep
def kept(c, lengths, table, lists, base):
    """The pools after the lists' rows have been moved, from copies of them; lists[u][g] counts from base[u][g]."""
    out = [p.clone() for p in c.pools]
    P = c.ref.P
    for u, row in enumerate(lists):
        for g, chosen in enumerate(row):
            src = base[u][g] + np.asarray(chosen, dtype=np.int64)
            dst = base[u][g] + np.arange(len(chosen))
            at = lambda r: (torch.as_tensor(table[u, g, r // P].astype(np.int64), device="cuda"), torch.as_tensor(r % P, device="cuda"))
            for new, old in zip(out, c.pools):
                if len(chosen):
                    new[(*at(dst), slice(0, D))] = old[(*at(src), slice(0, D))]
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layers,seqs,Hkv,P,width,tail,most", [
    (1, 1, 1, 16, 3, 5, 3), (1, 2, 8, 64, 9, 63, 8), (32, 3, 4, 32, 4, 20, 20), (2, 40, 2, 16, 10, 100, 90), (5, 1, 1, 256, 4, 300, 1), (4, 4, 8, 16, 6, 1, 1)])
def test_keep_a_path(B, dtype, layers, seqs, Hkv, P, width, tail, most):
    """A list a sequence, counted from its drafted rows; the heads hold different numbers of rows."""
    rng = np.random.RandomState(tail)
    c = Cache(B, layers, seqs, Hkv, P, width, 10, dtype, seed=tail, most=0, row_pad=8)
    n = rng.randint(0, tail + 1, seqs)
    n[0] = tail
    length = np.zeros((layers * seqs, Hkv), np.int32)
    for u, g in np.ndindex(*length.shape):
        length[u, g] = rng.randint(n[u % seqs], width * P + 1)
    need = int((-(-length // P)).sum())
    c = Cache(B, layers, seqs, Hkv, P, width, need + 10, dtype, seed=tail, most=0, row_pad=8, other=0.0)
    B.ckv_pages_reserve(c.pg, i32(length.flatten()), c.lengths, c.held, c.table, c.refs, c.k, c.v, c.ws, layers=layers)
    c.ref.reserve(length.flatten(), layers)
    c.fine(B), c.same()
    lists = [sorted(rng.choice(n[s], rng.randint(0, min(n[s], most) + 1), replace=False).tolist()) if n[s] else [] for s in range(seqs)]
    if most > 2:
        lists[0] = list(range(min(n[0], most)))                             # nothing moves
    rows, begins = [-1], []
    for x in lists:
        begins.append(len(rows))
        rows += x
    for pad in (0, 60 * seqs):                                              # a longer array: lists may be long
        lengths, out = i32(length), torch.full((layers * seqs, Hkv), 99, dtype=torch.int32, device="cuda")
        base = length - np.tile(n, layers)[:, None]
        want = kept(c, length, c.ref.table, [[lists[u % seqs]] * Hkv for u in range(layers * seqs)], base)
        B.ckv_keep_rows(c.pg, i32(rows + [1 << 30] * pad), i32(begins), i32([len(x) for x in lists]), lengths, c.table, c.k, c.v, out, c.ws,
                        tails=i32(n), refs=c.refs, layers=layers)
        c.fine(B), c.same()
        for x, y in zip(c.pools, want):
            assert torch.equal(x, y)
        assert np.array_equal(out.cpu().numpy(), base + np.tile([len(x) for x in lists], layers)[:, None])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Nu,Hkv,P,L,share", [(1, 1, 16, 40, 0.5), (1, 8, 64, 3000, 0.125), (2, 4, 32, 1000, 0.9), (3, 2, 256, 5000, 0.01), (90, 8, 16, 100, 0.3),
                                              (1, 2, 128, 20000, 0.5)])
def test_keep_rows_of_each_head(B, dtype, Nu, Hkv, P, L, share):
    """A list a head over all its rows, as a retention pass leaves them; heads with all and with none of their rows among them."""
    rng = np.random.RandomState(L)
    width = -(-L // P)
    length = rng.randint(max(L // 2, 1), L + 1, (Nu, Hkv)).astype(np.int32)
    c = Cache(B, 1, Nu, Hkv, P, width, int((-(-length // P)).sum()) + 3, dtype, seed=L, most=0, other=0.0)
    B.ckv_pages_reserve(c.pg, i32(length.flatten()), c.lengths, c.held, c.table, c.refs, c.k, c.v, c.ws)
    c.ref.reserve(length.flatten())
    lists = [[np.flatnonzero(rng.rand(length[u, g]) < share) for g in range(Hkv)] for u in range(Nu)]
    lists[0][-1] = np.arange(length[0, -1])
    if Nu > 1:
        lists[1][0] = np.arange(0)
    want = kept(c, length, c.ref.table, lists, np.zeros_like(length))
    flat = np.concatenate([x for row in lists for x in row])
    counts = np.array([len(x) for row in lists for x in row])
    out = torch.zeros(Nu, Hkv, dtype=torch.int32, device="cuda")
    B.ckv_keep_rows(c.pg, i32(flat), i32(np.cumsum(counts) - counts), i32(counts), i32(length), c.table, c.k, c.v, out, c.ws, refs=c.refs)
    c.fine(B), c.same()
    for x, y in zip(c.pools, want):
        assert torch.equal(x, y)
    assert np.array_equal(out.cpu().numpy().flatten(), counts)
    B.ckv_pages_trim(c.pg, out, c.held, c.table, c.refs, c.ws)
    c.ref.trim(out.cpu().numpy())
    c.fine(B), c.same()


@pytest.mark.parametrize("pad", [0, 4000])
def test_keep_leaves_what_it_may_not_move(B, pad):
    """Lists that do not ascend or leave their span, pages outside the pool and pages that others hold: the head stays as it is."""
    P, n, Hkv = 16, 20, 2
    good = [0, 2, 5, 19]
    for what in ("twice", "down", "past", "negative", "count", "begin", "tail", "page", "shared"):
        c = Cache(B, 1, 3, Hkv, P, 5, 40, seed=5, most=0, other=0.0)
        length = np.full((3, Hkv), 50, np.int32)
        B.ckv_pages_reserve(c.pg, i32([50] * 3), c.lengths, c.held, c.table, c.refs, c.k, c.v, c.ws)
        c.ref.reserve([50] * 3)
        lists, counts, begins, tails, table = [list(good) for _ in range(3)], [4] * 3, [0, 4, 8], [n] * 3, c.table.clone()
        if what == "twice":
            lists[1][2] = 2
        elif what == "down":
            lists[1][1] = 6
        elif what == "past":
            lists[1][3] = n
        elif what == "negative":
            lists[1][0] = -1
        elif what == "count":
            counts[1] = -1
        elif what == "begin":
            begins[1] = 12 + pad
        elif what == "tail":
            tails[1] = 51
        elif what == "page":
            table[1, :, 2] = c.n_pages
        else:
            c.refs[c.table[1, :, 2].long()] = 2
        want = kept(c, length, c.ref.table, [[good if u != 1 else []] * Hkv for u in range(3)], length - n)
        refs, out = c.refs.clone(), torch.zeros(3, Hkv, dtype=torch.int32, device="cuda")
        B.ckv_keep_rows(c.pg, i32(sum(lists, []) + [0] * pad), i32(begins), i32(counts), i32(length), table, c.k, c.v, out, c.ws, tails=i32(tails), refs=c.refs)
        assert B.ckv_device_status(c.ws) == B.ERR_PAGE, what
        for x, y in zip(c.pools, want):
            assert torch.equal(x, y), what
        assert out[:, 0].tolist() == [34, 50, 34] and out[:, 1].tolist() == [34, 50, 34] and torch.equal(refs, c.refs)
    # a shared page behind and in front of the rows that are written is no hindrance
    c.refs[c.table[1, :, 2].long()] = 1
    c.refs[c.table[1, :, 3].long()] = 2
    c.refs[c.table[1, :, 0].long()] = 2
    want = kept(c, length, c.ref.table, [[[0, 1]] * Hkv if u == 1 else [[]] * Hkv for u in range(3)], length - n)
    B.ckv_keep_rows(c.pg, i32([0, 2] + [9] * pad), i32([0, 0, 0]), i32([0, 2, 0]), i32(length), c.table, c.k, c.v, out, c.ws, tails=i32([n] * 3), refs=c.refs)
    assert B.ckv_device_status(c.ws) == B.OK and out[:, 0].tolist() == [30, 32, 30]


# ------------------------------------------------------------------------------------- as they are used together
@pytest.mark.parametrize("dtype,H,Hkv,P,seqs,samples,n", [(torch.bfloat16, 8, 2, 16, 2, 3, 12), (torch.bfloat16, 32, 8, 64, 1, 2, 40), (torch.float32, 4, 2, 16, 2, 2, 5)])
def test_drafting_on_shared_prompts(B, dtype, H, Hkv, P, seqs, samples, n):
    """Prompts of one layer, forked to samples, and steps of tree drafting for each: reserve, append, attend, keep the accepted
    path, trim; the step runs as one captured graph.  Every sample's rows are followed in a list of its own."""
    rng = random.Random(n)
    gen = torch.Generator(device="cuda").manual_seed(n)
    S, width, words, T = seqs * samples, 12, (n + 31) // 32, seqs * samples * n
    n_pages = 4 + S * Hkv * width
    k_pages, v_pages = (torch.full((n_pages, P, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    refs, table0, held0, len0 = z(n_pages), z(seqs, Hkv, width), z(seqs, Hkv), z(seqs, Hkv)
    # the prompts: ragged heads, written row by row through ckv_append
    m = [rng.randint(P, 3 * P) for _ in range(seqs)]
    st = [sum(m[:u]) for u in range(seqs + 1)]
    kv = [torch.randn(sum(m), Hkv, D, generator=gen, device="cuda").to(dtype) for _ in range(2)]
    pg0 = B.make_paged(k_pages, table0, k_new=kv[0], n_q_heads=H)
    ws0 = B.alloc_pages_workspace(pg0)
    B.ckv_pages_reserve(pg0, i32(m), len0, held0, table0, refs, k_pages, v_pages, ws0)
    grown = z(seqs, Hkv)
    B.ckv_append(pg0, None, kv[0], kv[1], None, i32(st), len0, table0, k_pages, v_pages, ws0, new_lengths=grown)
    assert B.ckv_device_status(ws0) == B.OK
    rows = [[tuple(x[st[s // samples]:st[s // samples + 1], g].clone() for x in kv) for g in range(Hkv)] for s in range(S)]
    # the samples
    lengths, held, table = z(S, Hkv), z(S, Hkv), z(S, Hkv, width)
    B.ckv_pages_fork(pg0, i32([s // samples for s in range(S)]), grown, held0, table0, refs, lengths, held, table, ws0)
    assert B.ckv_device_status(ws0) == B.OK and int(refs.max()) == samples
    # a step's inputs and buffers
    q, k, v = (torch.zeros(T, h, D, dtype=dtype, device="cuda") for h in (H, Hkv, Hkv))
    parents, starts, news, paths, counts = z(T), z(S + 1), z(S), z(S * n), z(S)
    begins = i32([s * n for s in range(S)])
    masks, positions, out, lse, longer, room = z(T, words), z(T), torch.zeros_like(q), torch.zeros(T, H, device="cuda"), z(S, Hkv), z(2)
    pg = B.make_paged(k_pages, table, q=q, k_new=k, max_new=n)
    ws = torch.empty(max(B.ckv_pages_workspace_bytes(pg), B.ckv_paged_workspace_bytes(pg)), dtype=torch.uint8, device="cuda")

    def draft():
        B.ckv_tree_masks(parents, starts, masks, ws, positions=positions, first_positions=lengths[:, 0].contiguous())
        B.ckv_pages_reserve(pg, news, lengths, held, table, refs, k_pages, v_pages, ws, room=room)
        B.ckv_append(pg, None, k, v, None, starts, lengths, table, k_pages, v_pages, ws, new_lengths=longer)
        B.ckv_tree_attend(pg, q, k_pages, v_pages, table, longer, starts, masks, out, ws, lse=lse)

    def accept():
        B.ckv_keep_rows(pg, paths, begins, counts, longer, table, k_pages, v_pages, lengths, ws, tails=news, refs=refs)
        B.ckv_pages_trim(pg, lengths, held, table, refs, ws)

    state = [x.clone() for x in (refs, held, table, lengths, k_pages, v_pages)]
    draft(), accept()                                                       # warm-up on empty trees
    for x, y in zip((refs, held, table, lengths), state):
        assert torch.equal(x, y)
    torch.cuda.synchronize()
    graphs = []
    for f in (draft, accept):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    for step in range(5):
        c = [rng.randint(0, n) if step else n for _ in range(S)]
        at = [sum(c[:u]) for u in range(S + 1)]
        trees = [[rng.randint(-1, t - 1) if rng.random() < 0.6 else t - 1 for t in range(x)] for x in c]
        parents[:at[-1]] = i32(sum(trees, [])) if at[-1] else z(0)
        starts.copy_(i32(at)), news.copy_(i32(c))
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        graphs[0].replay()
        sees = [TR.ancestors(t)[0] for t in trees]
        now = [[tuple(torch.cat((x, y[at[s]:at[s + 1], g])) for x, y in zip(rows[s][g], (k, v))) for g in range(Hkv)] for s in range(S)]
        want, want_lse = TR.attend(q[:at[-1]], at, now, sees)
        vmax = max(float(y.double().abs().max()) for row in now for _, y in row)
        norms = float(q.double().norm(dim=-1).max()) * max(float(x.double().norm(dim=-1).max()) for row in now for x, _ in row)
        r = 132 * EPS * norms / D ** 0.5 + 2.0 ** -20 + 300 * EPS
        assert ((out[:at[-1]].double() - want).abs() <= eps * (vmax + want.abs()) + EPS * want.abs() + 2 * r * vmax).all()
        assert ((lse[:at[-1]].double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs()).all()
        for s in range(S):
            depth = TR.ancestors(trees[s])[1]
            assert (positions[at[s]:at[s + 1]].cpu().numpy() == depth + rows[s][0][0].shape[0]).all()
        # a path: from some node up
        chosen = []
        for s in range(S):
            t, path = (rng.randint(-1, c[s] - 1) if c[s] else -1), []
            while t >= 0:
                path.insert(0, t)
                t = trees[s][t]
            chosen.append(path)
            paths[s * n:s * n + len(path)] = i32(path) if path else z(0)
            rows[s] = [tuple(torch.cat((x[:x.shape[0] - c[s]], x[x.shape[0] - c[s]:][path])) for x in now[s][g]) for g in range(Hkv)]
        counts.copy_(i32([len(p) for p in chosen]))
        graphs[1].replay()
        assert room[1] == 0 and B.ckv_device_status(ws) == B.OK
        assert lengths.tolist() == [[rows[s][g][0].shape[0] for g in range(Hkv)] for s in range(S)]
        for s in range(S):
            for g in range(Hkv):
                L = int(lengths[s, g])
                pages = table[s, g, :-(-L // P)].long()
                assert int(held[s, g]) == -(-L // P) and (refs[pages] > 0).all()
                for pool, x in zip((k_pages, v_pages), rows[s][g]):
                    assert torch.equal(pool[pages].reshape(-1, D)[:L], x)
        total = int(held.sum())
        assert int(refs.sum()) == total                                     # nothing is lost
    B.ckv_pages_trim(pg, None, held, table, refs, ws)
    assert not refs.any() and not held.any() and B.ckv_device_status(ws) == B.OK


def test_two_streams_with_states_of_their_own(B):
    """Two caches managed at the same time from two streams, each with its own work space, ten steps long."""
    caches = [Cache(B, 8, 4, 4, 16, 30, 12000, seed=s, share=0.2, most=4) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in caches]
    torch.cuda.synchronize()
    more = i32([3, 40, 0, 17])
    for _ in range(10):
        for c, s in zip(caches, streams):
            B.ckv_pages_reserve(c.pg, more, c.lengths, c.held, c.table, c.refs, c.k, c.v, c.ws, layers=8, stream=s)
            B.ckv_pages_trim(c.pg, c.lengths, c.held, c.table, c.refs, c.ws, stream=s)
    torch.cuda.synchronize()
    for c in caches:
        for _ in range(10):
            c.ref.reserve([3, 40, 0, 17], 8)
            c.ref.trim(c.ref.lengths)
        c.fine(B), c.same()


def test_the_readme_s_step_that_drafts_trees(B):
    """The lines under "A step that drafts trees", twice; the second time the sequences are those that the first forked."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        lines = f.read().split("A step that drafts trees")[1].split("\n\n")[1].split("\n")
    assert len(lines) == 7 and all(x.startswith("    ckv.ckv_") for x in lines)
    P, H, Hkv, S, n, width = 16, 8, 2, 2, 6, 8
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    kp, vp = (torch.randn(64, P, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
    qkv = torch.randn(S * n, H + 2 * Hkv, D, generator=gen, device="cuda").bfloat16()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    q_rot, out, lse = torch.zeros(S * n, H, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(S * n, H, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(S * n, H, device="cuda")
    parents = [-1, 0, 0, 1, 2, -1]
    names = dict(ckv=B, k_pages=kp, v_pages=vp, q=q, k=k, v=v, q_rot=q_rot, out=out, lse=lse, refs=z(64), held=z(S, Hkv), page_table=z(S, Hkv, width), lengths=z(S, Hkv),
                 longer=z(S, Hkv), room=z(2), parents=i32(parents * S), token_starts=i32([0, n, 2 * n]), masks=z(S * n, 1), positions=z(S * n), next_position=i32([0, 0]),
                 new=i32([n, n]), path=i32([0, 1, 3, 5]), begins=i32([0, 3]), counts=i32([3, 1]), lengths2=z(S, Hkv), held2=z(S, Hkv), page_table2=z(S, Hkv, width),
                 parent_of_each=i32([0, 0]), rotary=B.make_rotary(10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)))
    for turn in range(2):
        pg = names["pg"] = B.make_paged(kp, names["page_table"], q=q, k_new=k, max_new=n)
        names["pg_rot"] = B.make_paged(kp, names["page_table"], q=q_rot, max_new=n)
        names["ws"] = torch.empty(max(B.ckv_paged_workspace_bytes(pg), B.ckv_pages_workspace_bytes(pg)), dtype=torch.uint8, device="cuda")
        before = names["lengths"].clone()
        exec("\n".join(x[4:] for x in lines), names)
        assert B.ckv_device_status(names["ws"]) == B.OK and names["room"][1] == 0
        assert torch.equal(names["lengths"], before + names["counts"][:, None])
        assert torch.equal(names["lengths2"], names["lengths"][:1].expand(S, Hkv))       # both go on from the first
        assert names["positions"].tolist() == [int(p) + d for p in names["next_position"] for d in (0, 1, 1, 2, 2, 0)]
        # the rows kept are the path's, turned by their positions
        L = int(before[0, 0])
        angle = names["positions"][:n].double()[:, None, None] * names["rotary"]._keep[0]
        a, b = k[:n, :, :64].double(), k[:n, :, 64:].double()
        want = torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)
        for i, t in enumerate((0, 1, 3)):
            row = kp[names["page_table"][0, :, (L + i) // P].long(), (L + i) % P]
            # rounded to bf16 once, of an fp32 angle and products (40 * 2^-24 of a pair's sizes)
            assert ((row.double() - want[t]).abs() <= 2.0 ** -8 * want[t].abs() + 40 * EPS * 2 * want[t].abs().max()).all()
        assert int(names["refs"].sum()) == int(names["held2"].sum())
        for x, y in (("lengths", "lengths2"), ("held", "held2"), ("page_table", "page_table2")):
            names[x], names[y] = names[y], names[x]
        names["next_position"] = names["lengths"][:, 0].contiguous()
