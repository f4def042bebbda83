"""GPU tests of the calls on drafted trees: ancestor bits against a walk from parent to parent, attention against its 64-bit statement
(tests/tree_reference.py).

Tolerances are those of the attention over pages, counted in roundings: a logit is off by dx <= 132 * 2^-24 * |q| |k| * scale, the
exponential of it by a factor 1 + dx + 2^-22, sums of non-negative terms over `depth` additions by depth * 2^-24.  With
r = dx + 2^-20 + depth * 2^-24 the lse is off by at most r + 2^-23 |lse|, the output by 2 r max|v| + 2^-24 |out|; in bf16 each
probability is rounded for its product (2^-8 max|v| at the worst) and the output once more (2^-8 |out|).
"""
import copy
import math
import random

import numpy as np
import pytest
import torch

import paged_reference as R
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


def starts_of(counts, lead=0):
    s = [lead]
    for c in counts:
        s.append(s[-1] + c)
    return s


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def status_ws():
    return torch.full((256,), 0xAB, dtype=torch.uint8, device="cuda")


def random_parents(n, rng, chain=0.3, shuffled=False):
    p = [t - 1 if rng.random() < chain else rng.randint(-1, t - 1) for t in range(n)]
    if shuffled:                                           # parents behind their children
        at = list(range(n))
        rng.shuffle(at)
        q = [0] * n
        for t in range(n):
            q[at[t]] = -1 if p[t] < 0 else at[p[t]]
        p = q
    return p


# ------------------------------------------------------------------------------------------------- masks
@pytest.mark.parametrize("counts,words,chain,shuffled", [
    ([1], 1, 0.0, False), ([2, 0, 1], 1, 1.0, False), ([8], 1, 0.3, False), ([31, 32, 5], 1, 0.3, True), ([33, 64, 1], 2, 0.3, False),
    ([63] * 16, 2, 0.5, True), ([65, 96], 3, 0.9, True), ([100, 7], 5, 1.0, True), ([512, 300, 511], 16, 0.97, False),
    ([1024, 1, 1023], 32, 1.0, True), ([1000, 1000], 32, 0.0, True), ([40, 0, 0, 20], 32, 0.5, False), ([3] * 700, 1, 0.5, True)])
def test_masks(B, counts, words, chain, shuffled):
    rng = random.Random(len(counts) + words)
    st = starts_of(counts, 3)
    T = st[-1] + 2
    parents, sees, depth = torch.full((T,), -99, dtype=torch.int32), [], []
    for u, n in enumerate(counts):
        p = random_parents(n, rng, chain, shuffled)
        parents[st[u]:st[u + 1]] = torch.tensor(p, dtype=torch.int32)
        s, d = TR.ancestors(p)
        sees.append(s), depth.append(d)
    want = TR.pack(sees, words, T, st)
    ws = status_ws()
    for first in (None, i32([1000 * u - 5 for u in range(len(counts))])):
        masks, positions = torch.full((T, words), -1, dtype=torch.int32, device="cuda"), torch.full((T,), 77, dtype=torch.int32, device="cuda")
        B.ckv_tree_masks(parents.cuda(), i32(st), masks, ws, positions=positions, first_positions=first)
        assert B.ckv_device_status(ws) == B.OK
        assert torch.equal(masks.cpu(), want)
        pos = positions.cpu()
        assert (pos[:st[0]] == 77).all() and (pos[st[-1]:] == 77).all()
        for u in range(len(counts)):
            assert (pos[st[u]:st[u + 1]].numpy() == depth[u] + (0 if first is None else 1000 * u - 5)).all()
    masks.zero_()
    B.ckv_tree_masks(parents.cuda(), i32(st), masks, ws)                   # positions are not asked for
    assert torch.equal(masks[st[0]:st[-1]].cpu(), want[st[0]:st[-1]])


def test_masks_report_what_is_no_tree(B):
    ws = status_ws()
    for parents, words, want in (([-1, 0, 5], 1, [1, 3, 4]), ([-1, 0, -2], 1, [1, 3, 4]),           # no token of the unit: as a root
                                 ([1, 0, -1, 2], 1, [3, 3, 4, 12]), ([-1, 1, 1], 1, [1, 2, 6])):    # its own ancestor
        n = len(parents)
        masks, pos = torch.zeros(n, words, dtype=torch.int32, device="cuda"), torch.full((n,), 9, dtype=torch.int32, device="cuda")
        B.ckv_tree_masks(i32(parents), i32([0, n]), masks, ws, positions=pos)
        assert B.ckv_device_status(ws) == B.ERR_PAGE and B.ckv_device_status(ws) == B.OK
        assert masks[:, 0].tolist() == want
        assert all(0 <= x < n for x in pos.tolist())
    # more tokens than words
    n = 40
    masks, pos = torch.full((n, 1), 5, dtype=torch.int32, device="cuda"), torch.full((n,), 9, dtype=torch.int32, device="cuda")
    B.ckv_tree_masks(i32([t - 1 for t in range(n)]), i32([0, n]), masks, ws, positions=pos)
    assert B.ckv_device_status(ws) == B.ERR_PAGE
    assert [x & 0xffffffff for x in masks[:32, 0].tolist()] == [(2 << t) - 1 for t in range(32)] and (masks[32:] == 0).all()
    assert pos[:32].tolist() == list(range(32)) and (pos[32:] == 0).all()


# ------------------------------------------------------------------------------------------------ attend
def run_attend(B, c, q, starts, masks, scale=0.0, max_new=0, lse=True):
    pg = B.make_paged(c.k_pages, c.table, q=q, scale=scale, max_new=max_new)
    n = B.ckv_paged_workspace_bytes(pg)
    ws = torch.full((n + 512,), 0xAB, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 11.0, device="cuda").to(q.dtype)
    l = torch.full(q.shape[:2], 11.0, device="cuda") if lse else None
    B.ckv_tree_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, i32(starts), masks, out, ws[256:256 + n], lse=l)
    assert B.ckv_device_status(ws[256:256 + n]) == B.OK
    assert (ws[:256] == 0xAB).all() and (ws[256 + n:] == 0xAB).all()
    return out, l


def r_of(q, k, length, scale=1 / math.sqrt(D)):
    """The r of this file's first lines, for these queries and keys (rows of the last dimension)."""
    norm = lambda x: float(x.double().nan_to_num(0, 0, 0).norm(dim=-1).max()) if x.numel() else 0.0
    return 132 * EPS * norm(q) * norm(k) * scale + 2.0 ** -20 + (length / 8 + 256) * EPS


def widened(c, H):
    """The same cache under a table so wide that fp32 calls of more than 16 query rows a head go to the tensor cores."""
    Nu, Hkv, width = c.table.shape
    wide = torch.full((Nu, Hkv, max(width, 80000 // (c.P * Nu * Hkv) + 1)), 0x7ffffff0, dtype=torch.int32, device="cuda")
    wide[:, :, :width] = c.table
    other = copy.copy(c)
    other.table = wide
    return other


def caches(c, H, counts):
    """c, and widened where that picks another kernel."""
    return [c, widened(c, H)] if c.k_pages.dtype == torch.float32 and max(counts) * H // c.table.shape[1] > 16 else [c]


def check_attend(c, q, starts, sees, out, lse, scale=None):
    want, want_lse = TR.attend(q, starts, c.rows, sees, scale)
    live = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    live[starts[0]:starts[-1]] = True
    s = 1 / math.sqrt(D) if scale is None else abs(scale)
    vmax = max([float(v.double().nan_to_num(0, 0, 0).abs().max()) for row in c.rows for _, v in row if v.shape[0]] + [0.0])
    r = r_of(q[live], torch.cat([k for row in c.rows for k, _ in row]), max(max(r) for r in c.lens), s)
    tol = 2 * r * vmax + (2.0 ** -8 * (vmax + want.abs()) if q.dtype == torch.bfloat16 else EPS * want.abs())
    err = (out.double() - want).abs()
    assert (err <= tol)[live].all(), float((err / tol)[live].max())
    if lse is not None:
        none = torch.isinf(want_lse)
        assert torch.equal((lse == -math.inf)[live], none[live])
        seen = live[:, None] & ~none
        assert ((lse.double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs())[seen].all()
        assert (out[live][none[live]] == 0).all()
        assert (lse[~live] == 11.0).all()
    assert (out[~live] == 11.0).all()


def some_sees(counts, kind, rng):
    """Trees, any bits at all, bits that leave every third token nothing of the tree, or whole chunks."""
    sees = []
    for n in counts:
        if kind == "tree":
            sees.append(TR.ancestors(random_parents(n, rng, 0.3, rng.random() < 0.5))[0])
        elif kind == "bits":
            sees.append(np.array([[rng.random() < 0.4 for _ in range(n)] for _ in range(n)], dtype=bool).reshape(n, n))
        elif kind == "gaps":
            s = TR.ancestors(random_parents(n, rng, 0.8))[0]
            s[::3] = False
            sees.append(s)
        else:
            sees.append(np.ones((n, n), dtype=bool))
    return sees


CASES = [
    # H, Hkv, page, tokens per unit, rows per (unit, head) with the tokens'
    (8, 2, 16, [1], [[1, 1]]),
    (8, 2, 16, [1], [[0, 5]]),
    (32, 8, 64, [8], [[512, 400, 8, 63, 64, 65, 127, 129]]),
    (28, 4, 16, [1, 4, 2], [[100, 0, 17, 256], [4, 5, 6, 7], [700, 701, 699, 15]]),
    (28, 4, 32, [5, 3, 0, 1], [[300, 5, 31, 33], [64, 65, 3, 3], [9, 9, 9, 9], [128, 127, 129, 1]]),
    (16, 16, 128, [2, 7], [[130] * 16, [200] * 16]),
    (24, 2, 64, [3], [[1000, 37]]),
    (40, 1, 64, [4, 1], [[333], [90]]),
    (8, 1, 256, [16], [[5000]]),
    (4, 4, 16, [33, 1, 70], [[33, 40, 1000, 64], [9, 8, 7, 6], [70, 71, 300, 128]]),
    (32, 8, 64, [63], [[63, 64, 127, 128, 129, 640, 1000, 2000]]),
    (28, 4, 16, [19, 200], [[19, 20, 500, 128], [200, 255, 256, 1100]]),
    (6, 2, 128, [257, 1, 64], [[300, 1500], [1500, 1], [64, 65]]),
    (128, 1, 64, [5], [[77]]),
    (130, 1, 64, [3], [[77]]),
    (8, 2, 64, [7], [[3, 6]]),                       # more tokens than rows: only some of the tree's rows are there
    (8, 2, 64, [300], [[100, 290]]),
]


@pytest.mark.parametrize("kind", ["tree", "bits", "gaps", "whole"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,page,counts,lens", CASES)
def test_attend(B, dtype, kind, H, Hkv, page, counts, lens):
    """Rows behind the lengths, pages of nobody and padding tokens are NaN; table entries of no row point far outside; bits past a
    unit's tokens are set."""
    rng = random.Random(H + len(kind))
    c = R.Cache(lens, page, dtype=dtype, device="cuda", seed=H + page, row_pad=8 if page == 32 else 0)
    st = starts_of(counts, 2)
    g = torch.Generator(device="cuda").manual_seed(len(counts))
    qkv = torch.randn(st[-1] + 3, H + 4, D, generator=g, device="cuda").to(dtype)
    qkv[:2] = float("nan")
    qkv[st[-1]:] = float("nan")
    q = qkv[:, 1:1 + H]
    sees = some_sees(counts, kind, rng)
    words = (max(counts) + 31) // 32 + rng.randint(0, 1)
    padded = []
    for s in sees:
        n = s.shape[0]
        wide = np.ones((n, 32 * words), dtype=bool)
        wide[:, :n] = s
        padded.append(wide)
    masks = torch.full((q.shape[0], words), -1, dtype=torch.int32)
    for u, s in enumerate(padded):
        bits = (s.reshape(-1, words, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
        masks[st[u]:st[u + 1]] = torch.from_numpy(bits.view(np.int32))
    for cache in caches(c, H, counts):
        for max_new in (0, max(counts)):
            out, lse = run_attend(B, cache, q, st, masks.cuda(), max_new=max_new)
            check_attend(c, q, st, sees, out, lse)


@pytest.mark.parametrize("dtype,Nu,Hkv,H,n,rows", [
    (torch.bfloat16, 3, 2, 8, 4, 9000), (torch.bfloat16, 2, 2, 8, 63, 9000), (torch.bfloat16, 40, 4, 16, 20, 700),
    (torch.bfloat16, 1, 1, 7, 300, 20000), (torch.float32, 2, 2, 8, 5, 9000), (torch.float32, 40, 4, 8, 3, 300), (torch.float32, 1, 2, 14, 70, 5000),
    (torch.float32, 30, 2, 8, 33, 400), (torch.float32, 1, 1, 8, 32, 16000)])
def test_attend_long_and_many(B, dtype, Nu, Hkv, H, n, rows):
    """Caches whose work is split over the SMs, and more heads than there are SMs."""
    rng = random.Random(n)
    lens = [[rows + n - rng.randint(0, rows // 2) for _ in range(Hkv)] for _ in range(Nu)]
    counts = [n if u == 0 else rng.randint(0, n) for u in range(Nu)]
    c = R.Cache(lens, 64, dtype=dtype, device="cuda", seed=n)
    st = starts_of(counts)
    q = torch.randn(st[-1], H, D, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").to(dtype)
    sees = some_sees(counts, "tree", rng)
    out, lse = run_attend(B, c, q, st, TR.pack(sees, (n + 31) // 32, st[-1], st).cuda(), max_new=n)
    check_attend(c, q, st, sees, out, lse)


@pytest.mark.parametrize("Nu,Hkv,H,n,rows", [(6, 4, 16, 200, 1500), (2, 1, 8, 250, 6000), (12, 4, 28, 140, 900), (1, 2, 2, 600, 3000), (40, 2, 8, 130, 500)])
def test_shares_of_units_with_several_blocks(B, Nu, Hkv, H, n, rows):
    """Shares that begin inside an item, hold whole ones and end in another: fewer items than SMs, about as many, more."""
    rng = random.Random(n)
    lens = [[rows + n - rng.randint(0, 200) for _ in range(Hkv)] for _ in range(Nu)]
    counts = [n if u == 0 else n - rng.randint(0, n // 2) for u in range(Nu)]
    c = R.Cache(lens, 16, dtype=torch.bfloat16, device="cuda", seed=n)
    st = starts_of(counts)
    q = torch.randn(st[-1], H, D, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").bfloat16()
    sees = some_sees(counts, "tree", rng)
    out, lse = run_attend(B, c, q, st, TR.pack(sees, (n + 31) // 32, st[-1], st).cuda(), max_new=n)
    check_attend(c, q, st, sees, out, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [4, 12, 90])
def test_a_chain_is_a_causal_chunk(B, dtype, n):
    """Tokens that each follow the one before see what ckv_paged_attend with causal = 1 shows them."""
    c = R.Cache([[n + 300, n, n + 5000, n + 1]], 32, dtype=dtype, device="cuda", seed=n)
    q = torch.randn(n, 8, D, device="cuda").to(dtype)
    sees = [np.tril(np.ones((n, n), dtype=bool))]
    out, lse = run_attend(B, c, q, [0, n], TR.pack(sees, (n + 31) // 32, n, [0, n]).cuda(), max_new=n)
    check_attend(c, q, [0, n], sees, out, lse)
    pg = B.make_paged(c.k_pages, c.table, q=q, max_new=n)
    out2, lse2 = torch.zeros_like(q), torch.zeros(n, 8, device="cuda")
    B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, i32([0, n]), out2, B.alloc_paged_workspace(pg), lse=lse2)
    vmax = max(float(v.double().abs().max()) for _, v in c.rows[0])
    r = r_of(q, torch.cat([k for k, _ in c.rows[0]]), n + 5000)        # each is off by what check_attend allows
    assert (out.double() - out2.double()).abs().max() <= (4 * 2.0 ** -8 * (dtype == torch.bfloat16) + 4 * r + 2 * EPS) * vmax
    assert ((lse - lse2).double().abs() <= 2 * (r + 2 * EPS * lse.double().abs())).all()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 3), (torch.bfloat16, 8), (torch.bfloat16, 70), (torch.bfloat16, 200), (torch.float32, 9), (torch.float32, 40)])
def test_values_that_are_not_finite(B, dtype, n, bad):
    """A value element of a drafted token's row that is not finite reaches the tokens that see the row, in that element, and no
    others; the row's key, where it is not finite either, the tokens that see it and no others."""
    rng = random.Random(n)
    H, Hkv, base = 8, 2, 61
    c = R.Cache([[n + base, n + 200]], 32, dtype=dtype, device="cuda", seed=n)
    sees = some_sees([n], "tree", rng)
    q = torch.randn(n, H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(dtype)
    masks = TR.pack(sees, (n + 31) // 32, n, [0, n]).cuda()
    hit = sorted({0, n // 2, n - 1})
    clean = [tuple(x.clone() for x in row) for row in c.rows[0]]
    for g in range(Hkv):
        k, v = (x.clone() for x in c.rows[0][g])
        for t in hit:
            j = c.lens[0][g] - n + t
            v[j, 5 * g + 3] = bad
            c.v_pages[int(c.table[0, g, j // 32]), j % 32, 5 * g + 3] = bad
        c.rows[0][g] = (k, v)
    touched = torch.from_numpy(sees[0][:, hit].any(1)).cuda()
    for max_new, cache in [(m, x) for m in (0, n) for x in caches(c, H, [n])]:
        out, lse = run_attend(B, cache, q, [0, n], masks, max_new=max_new)
        for g in range(Hkv):
            mine = out[:, 4 * g:4 * g + 4]
            assert not torch.isfinite(mine[touched][:, :, 5 * g + 3]).any()
            mine[touched, :, 5 * g + 3] = 0.0
        assert torch.isfinite(out).all()
        keep, c.rows[0] = c.rows[0], clean
        want, _ = TR.attend(q, [0, n], c.rows, sees)
        for g in range(Hkv):
            w = want[:, 4 * g:4 * g + 4]
            w[touched, :, 5 * g + 3] = 0.0
        vmax = max(float(v.double().abs().max()) for _, v in clean)
        r = r_of(q, torch.cat([k for k, _ in clean]), n + 200)
        assert ((out.double() - want).abs() <= (2.0 ** -8 * (vmax + want.abs()) if dtype == torch.bfloat16 else EPS * want.abs()) + 2 * r * vmax).all()
        c.rows[0] = keep
    # keys that are not finite, of rows that only some tokens see
    t = hit[-1]
    for g in range(Hkv):
        j = c.lens[0][g] - n + t
        c.k_pages[int(c.table[0, g, j // 32]), j % 32] = float("nan")
        for x in hit:
            j = c.lens[0][g] - n + x
            c.v_pages[int(c.table[0, g, j // 32]), j % 32] = clean[g][1][j].cuda()
    for cache in caches(c, H, [n]):
        out, lse = run_attend(B, cache, q, [0, n], masks, max_new=n)
        ill = torch.from_numpy(sees[0][:, t]).cuda()
        assert torch.isnan(lse[ill]).all() and torch.isnan(out[ill]).all()
        assert torch.isfinite(lse[~ill]).all() and torch.isfinite(out[~ill]).all()


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype,n", [(torch.float32, 3), (torch.float32, 20), (torch.float32, 40), (torch.bfloat16, 3), (torch.bfloat16, 20), (torch.bfloat16, 70)])
def test_largest_finite_numbers(B, dtype, n, sign):
    """Rows of the type's largest number, keys and values: tokens that do not see them have what they would have without; in tokens that
    see a value of that size (their sums may pass the type's range before they are divided) it stays of its sign."""
    H, Hkv, base = 8, 2, 90
    c = R.Cache([[n + base, n + 200]], 32, dtype=dtype, device="cuda", seed=n)
    sees = some_sees([n], "tree", random.Random(n))
    q = torch.randn(n, H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(dtype)
    masks = TR.pack(sees, (n + 31) // 32, n, [0, n]).cuda()
    want, want_lse = TR.attend(q, [0, n], c.rows, sees)
    vmax = max(float(v.double().abs().max()) for _, v in c.rows[0])
    r = r_of(q, torch.cat([k for k, _ in c.rows[0]]), n + 200)
    tol = (2.0 ** -8 * (vmax + want.abs()) if dtype == torch.bfloat16 else EPS * want.abs()) + 2 * r * vmax
    hit = sorted({n // 2, n - 1}) if n > 3 else [2]                        # so that some tokens see none
    clear = ~torch.from_numpy(sees[0][:, hit].any(1)).cuda()
    assert clear.any() and (~clear).any()
    for pool in (c.v_pages, c.k_pages):
        for g in range(Hkv):
            for t in hit:
                j = c.lens[0][g] - n + t
                pool[int(c.table[0, g, j // 32]), j % 32] = sign * torch.finfo(dtype).max
        for cache in caches(c, H, [n]):
            out, lse = run_attend(B, cache, q, [0, n], masks, max_new=n)
            assert ((out.double() - want).abs() <= tol)[clear].all()
            assert ((lse.double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs())[clear].all()
            if pool is c.v_pages:
                assert (out[~clear] * sign > vmax).all()


@pytest.mark.parametrize("bits", [0x7fffffff, -1, 0x7f800001, -0x7fffff])      # quiet and signalling, of both signs
def test_every_nan(B, bits):
    """A drafted token's key, or value, of NaNs with this pattern: NaN in the tokens that see it and nothing of it in the others."""
    n, H, Hkv = 20, 8, 2
    sees = some_sees([n], "tree", random.Random(n))
    masks = TR.pack(sees, 1, n, [0, n]).cuda()
    q = torch.randn(n, H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))
    ill = torch.from_numpy(sees[0][:, n // 2]).cuda()
    assert ill.any() and (~ill).any()
    for name in ("k_pages", "v_pages"):
        c = R.Cache([[n + 90, n + 200]], 32, dtype=torch.float32, device="cuda", seed=n)
        want, _ = TR.attend(q, [0, n], c.rows, sees)
        vmax = max(float(v.double().abs().max()) for _, v in c.rows[0])
        tol = EPS * want.abs() + 2 * vmax * r_of(q, torch.cat([k for k, _ in c.rows[0]]), n + 200)
        for g in range(Hkv):
            j = c.lens[0][g] - n + n // 2
            getattr(c, name).view(torch.int32)[int(c.table[0, g, j // 32]), j % 32] = bits
        for cache in caches(c, H, [n]):
            out, lse = run_attend(B, cache, q, [0, n], masks, max_new=n)
            assert torch.isnan(out[ill]).all() and ((out.double() - want).abs() <= tol)[~ill].all()
            assert torch.isnan(lse[ill]).all() if name == "k_pages" else torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype,n", [(torch.float32, 3), (torch.float32, 20), (torch.bfloat16, 3), (torch.bfloat16, 20), (torch.bfloat16, 70)])
def test_infinite_keys_and_values_of_the_prefix(B, dtype, n):
    """Rows that every token sees.  A key with an infinity gives the logit its product with the query has: minus infinity is a row of no
    weight, plus infinity makes the token NaN.  A value with an infinity makes that element infinite."""
    H, Hkv, base = 8, 2, 150
    c = R.Cache([[n + base, n + base + 60]], 32, dtype=dtype, device="cuda", seed=n)
    q = torch.randn(n, H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(dtype)
    q[:, :, 5] = q[:, :, 5].abs() + 0.5
    q[-1, :, 5] *= -1                                                       # one token that meets the infinity with the other sign
    sees = some_sees([n], "tree", random.Random(n))
    masks = TR.pack(sees, 3, n, [0, n]).cuda()
    place = lambda j, g: (int(c.table[0, g, j // 32]), j % 32)
    for g in range(Hkv):
        k, v = (x.clone() for x in c.rows[0][g])
        k[17, 5], v[33, 9] = -math.inf, math.inf
        c.k_pages[place(17, g)][5], c.v_pages[place(33, g)][9] = -math.inf, math.inf
        c.rows[0][g] = (k, v)
    for cache in caches(c, H, [n]):
        out, lse = run_attend(B, cache, q, [0, n], masks, max_new=n)
        assert torch.isnan(lse[-1]).all() and torch.isnan(out[-1]).all()
        assert torch.isfinite(lse[:-1]).all() and not torch.isfinite(out[:-1, :, 9]).any()
        rest = [d for d in range(D) if d != 9]
        clean = [[(torch.cat((k[:17], k[18:])), torch.cat((v[:17], v[18:])).nan_to_num(0, 0, 0)) for k, v in c.rows[0]]]
        want, want_lse = TR.attend(q, [0, n], clean, sees)
        vmax = max(float(v.double().abs().max()) for _, v in clean[0])
        r = r_of(q, torch.cat([k for k, _ in clean[0]]), n + 300)
        tol = (2.0 ** -8 * (vmax + want.abs()) if dtype == torch.bfloat16 else EPS * want.abs()) + 2 * r * vmax
        assert ((out.double() - want).abs() <= tol)[:-1][:, :, rest].all()
        assert ((lse.double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs())[:-1].all()


@pytest.mark.parametrize("dtype,n,pages", [(torch.float32, 6, 3), (torch.float32, 40, 700), (torch.bfloat16, 6, 3), (torch.bfloat16, 40, 4), (torch.bfloat16, 40, 2)])
def test_rows_past_the_table_and_bad_pages(B, dtype, n, pages):
    """Rows the table has no page for, and rows of a page outside the pool, are left out (drafted ones among them), and said."""
    P, H = 16, 4
    lens = [[pages * P + 5, pages * P + 30]]
    room = pages * P
    c = R.Cache(lens, P, dtype=dtype, device="cuda", seed=n)
    rng = random.Random(n)
    sees = some_sees([n], "tree", rng)
    q = torch.randn(n, H, D, device="cuda").to(dtype)
    masks = TR.pack(sees, 2, n, [0, n]).cuda()
    table = c.table[:, :, :pages].contiguous()
    table[0, 1, 1] = c.k_pages.shape[0]
    pg = B.make_paged(c.k_pages, table, q=q, max_new=n)
    ws = B.alloc_paged_workspace(pg)
    out, lse = torch.zeros_like(q), torch.zeros(n, H, device="cuda")
    B.ckv_tree_attend(pg, q, c.k_pages, c.v_pages, table, c.lengths, i32([0, n]), masks, out, ws, lse=lse)
    assert B.ckv_device_status(ws) == B.ERR_PAGE
    for g in range(2):
        k, v = (x.cuda().double() for x in c.rows[0][g])
        L = lens[0][g]
        see = torch.ones(n, L, dtype=torch.bool, device="cuda")
        see[:, max(L - n, 0):] = torch.from_numpy(sees[0]).cuda()[:, max(n - L, 0):]
        see[:, room:] = False
        if g == 1:
            see[:, P:2 * P] = False
        x = torch.einsum("nhd,ld->nhl", q[:, 2 * g:2 * g + 2].double(), k) / math.sqrt(D)
        x = x.masked_fill(~see[:, None], -math.inf)
        want = torch.einsum("nhl,ld->nhd", torch.softmax(x, -1).nan_to_num(0), v)
        r = r_of(q, k, L)
        tol = (2.0 ** -8 * (v.abs().max() + want.abs()) if dtype == torch.bfloat16 else EPS * want.abs()) + 2 * r * v.abs().max()
        assert ((out[:, 2 * g:2 * g + 2].double() - want).abs() <= tol).all()
        want_lse = torch.logsumexp(x, -1)
        got = lse[:, 2 * g:2 * g + 2].double()
        assert torch.equal(got == -math.inf, want_lse == -math.inf)
        assert ((got - want_lse).abs() <= r + 2 * EPS * want_lse.abs())[want_lse > -math.inf].all()


def test_words_that_do_not_reach_all_tokens(B):
    """Tokens past 32 * words are seen by nobody, themselves included."""
    for dtype, n in ((torch.float32, 50), (torch.bfloat16, 50), (torch.bfloat16, 3), (torch.bfloat16, 33)):
        c = R.Cache([[n + 40, n]], 16, dtype=dtype, device="cuda", seed=n)
        q = torch.randn(n, 4, D, device="cuda").to(dtype)
        sees = [np.ones((n, n), dtype=bool)]
        sees[0][:, 32:] = False
        for cache in caches(c, 4, [n]):
            out, lse = run_attend(B, cache, q, [0, n], torch.full((n, 1), -1, dtype=torch.int32, device="cuda"), max_new=n)
            check_attend(c, q, [0, n], sees, out, lse)


@pytest.mark.parametrize("scale", [0.5, -0.09, 2.0 ** -20])
def test_scales(B, scale):
    for dtype, n in ((torch.float32, 5), (torch.bfloat16, 5), (torch.bfloat16, 70)):
        c = R.Cache([[n + 700, n + 10]], 64, dtype=dtype, device="cuda", seed=n)
        q = torch.randn(n, 8, D, device="cuda").to(dtype)
        sees = some_sees([n], "tree", random.Random(n))
        for cache in caches(c, 8, [n]):
            out, lse = run_attend(B, cache, q, [0, n], TR.pack(sees, 3, n, [0, n]).cuda(), scale=scale, max_new=n)
            check_attend(c, q, [0, n], sees, out, lse, scale=scale)


@pytest.mark.parametrize("size", [1.0, 30.0, 1000.0])
@pytest.mark.parametrize("dtype,n", [(torch.float32, 3), (torch.float32, 24), (torch.bfloat16, 70)])
def test_large_logits(B, dtype, n, size):
    """Logits that rise along the cache, to thousands: the running maximum moves at every tile."""
    L = n + 900
    c = R.Cache([[L, L - 33]], 32, dtype=dtype, device="cuda", seed=n)
    q = torch.randn(n, 8, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)).to(dtype)
    for g in range(2):
        k, v = c.rows[0][g]
        rise = torch.linspace(0, size / 10, k.shape[0])[:, None] * q[0, 4 * g].float().cpu() / D ** 0.5
        k = (k.float() * min(size, 3.0) + rise).to(dtype)
        c.rows[0][g] = (k, v)
        for j in range(0, k.shape[0], 32):
            c.k_pages[int(c.table[0, g, j // 32]), :min(32, k.shape[0] - j)] = k[j:j + 32].cuda()
    sees = some_sees([n], "tree", random.Random(n))
    for cache in caches(c, 8, [n]):
        out, lse = run_attend(B, cache, q, [0, n], TR.pack(sees, 3, n, [0, n]).cuda(), max_new=n)
        check_attend(c, q, [0, n], sees, out, lse)


def test_fp32_is_as_exact_as_multiplications_in_fp32(B):
    """The three-product form against the plain kernel's: 2-norms of the errors against 64 bits."""
    n, H = 24, 8
    c = R.Cache([[n + 4000, n + 3500]], 64, dtype=torch.float32, device="cuda", seed=1)
    q = torch.randn(n, H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    sees = some_sees([n], "tree", random.Random(n))
    masks = TR.pack(sees, 1, n, [0, n]).cuda()
    want, want_lse = TR.attend(q, [0, n], c.rows, sees)
    out, lse = run_attend(B, widened(c, H), q, [0, n], masks, max_new=n)
    # roundings of a product's two halves (2^-22 each) and of the unit's sums (a unit in the last place each, few in a row): a few 2^-23,
    # and not the 2^-12 of a product of two tf32 numbers
    assert (out.double() - want).norm() <= 8 * 2.0 ** -23 * want.norm()
    assert (lse.double() - want_lse).norm() <= 4 * 2.0 ** -23 * want_lse.norm()


def test_same_bits_again_on_two_streams_and_in_a_graph(B):
    rng = random.Random(3)
    for counts in ([3, 2], [60, 9]):
        c = R.Cache([[3000, 100], [777, 2500]], 64, dtype=torch.bfloat16, device="cuda")
        q = torch.randn(sum(counts), 16, D, device="cuda").bfloat16()
        st = starts_of(counts)
        sees = some_sees(counts, "tree", rng)
        masks, start = TR.pack(sees, 2, sum(counts), st).cuda(), i32(st)
        pg = B.make_paged(c.k_pages, c.table, q=q, max_new=max(counts))
        streams, ws = [torch.cuda.Stream() for _ in range(2)], [B.alloc_paged_workspace(pg) for _ in range(2)]
        outs = [torch.zeros_like(q) for _ in range(2)]
        torch.cuda.synchronize()
        first = None
        for _ in range(4):
            for s, w, o in zip(streams, ws, outs):
                B.ckv_tree_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, start, masks, o, w, stream=s)
            torch.cuda.synchronize()
            first = outs[0].clone() if first is None else first
            assert torch.equal(outs[0], first) and torch.equal(outs[1], first)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.ckv_tree_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, start, masks, outs[0], ws[0])
        # the trees change between replays
        sees = some_sees(counts, "tree", rng)
        masks.copy_(TR.pack(sees, 2, sum(counts), st))
        outs[0].fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        B.ckv_tree_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, start, masks, outs[1], ws[1])
        assert torch.equal(outs[0], outs[1]) and not torch.equal(outs[0], first)
