"""GPU tests of the paged-cache operators against plain 64-bit statements of them (tests/paged_reference.py).

Tolerances count roundings.  An output in bf16 is off by at most half a step of its value, 2^-8 relative (`finfo.eps / 2`); fp32
arithmetic contributes multiples of 2^-24.
  rotate: fp32 angle of a fraction of a turn (2^-25 turns: 1.9e-7 rad) and its sine and cosine, three products and a sum, and
    with norms a 128-term sum of squares (relative 2^-24 * 8, a shuffle tree), a root and a division: at most 40 * 2^-24 of
    |a| + |b| of the pair.
  attend: a logit is a dot product of 128 terms in fp32: off by dx <= 132 * 2^-24 * |q| |k| * scale (Cauchy-Schwarz on the
    absolute products); the exponential of it moves by a factor 1 + dx + 2^-22 (exp2f and its argument, |x| <= 64); sums of
    non-negative terms over at most `depth` sequential additions add depth * 2^-24.  With r = dx + 2^-20 + depth * 2^-24:
    lse is off by at most r + 2^-23 |lse|; the output by 2 r max|v| (numerator and denominator) + 2^-24 |out|.
    In bf16 the probabilities are rounded for the product with v, 2^-8 relative each, so at most 2^-8 max|v| in the worst
    case, and the output once more, 2^-8 |out|.  Those roundings are independent: over all outputs the 2-norm of the error is
    bounded by 2 * 2^-8 of the outputs' 2-norm wherever no single key carries the row, and never by more than the first bound.
"""
import math

import pytest
import torch

import paged_reference as R
from paper_2602_08686_b200 import inputs as gen

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


# ------------------------------------------------------------------------------------------------ rotate
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,Hkv,T,rot,interleaved,norm,in_place", [
    (32, 8, 1, 128, False, False, False), (28, 4, 3, 128, True, True, False), (8, 1, 17, 64, False, True, True),
    (5, 5, 33, 96, True, False, True), (16, 2, 2500, 128, False, True, False), (1, 1, 2371, 16, False, False, False),
    (7, 7, 9, 0, False, True, False), (64, 64, 5, 32, True, True, True), (3, 1, 4, 112, False, False, False)])
def test_rotate(B, dtype, H, Hkv, T, rot, interleaved, norm, in_place):
    g = torch.Generator(device="cuda").manual_seed(T + rot)
    lead, pad = (1, 2) if T > 4 else (0, 0)       # padding rows before the first and behind the last unit
    qkv = torch.randn(T, H + 2 * Hkv, D, generator=g, device="cuda").to(dtype)
    before = qkv.clone()
    q, k = qkv[:, :H], qkv[:, H:H + Hkv]
    pos = torch.randint(-5, 1 << 20, (T,), generator=g, device="cuda", dtype=torch.int32)
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1)) if rot else None
    w = [1 + 0.2 * torch.randn(D, generator=g, device="cuda") if norm else None for _ in range(2)]
    starts = starts_of([T - lead - pad], lead)
    rotary = B.make_rotary(inv, interleaved=interleaved, q_norm_w=w[0], k_norm_w=w[1], rot_scale=1.25, norm_eps=1e-5)
    outs = (q, k) if in_place else (torch.full((T, H, D), 7.0, device="cuda").to(dtype), torch.full((T, Hkv, D), 7.0, device="cuda").to(dtype))
    B.ckv_rotate(B.make_packed(q, k, 1), rotary, q, k, pos, i32(starts), *outs)
    for x, wt, out in ((before[:, :H], w[0], outs[0]), (before[:, H:H + Hkv], w[1], outs[1])):
        live = slice(lead, T - pad)
        want = R.turn(x, pos, inv, wt, 1e-5, interleaved, 1.25)
        size = want.abs() + R.turn(x, pos, inv, wt, 1e-5, interleaved, 1.25).roll(1, -1).abs().amax(-1, keepdim=True)
        tol = 40 * EPS * size + (2.0 ** -8 if dtype == torch.bfloat16 else 2 * EPS) * want.abs()
        assert ((out.double() - want).abs() <= tol)[live].all(), ((out.double() - want).abs() / tol)[live].max()
        for rows in (slice(0, lead), slice(T - pad, T)):
            assert torch.equal(out[rows], x[rows] if in_place else torch.full_like(out[rows], 7.0))
    if in_place:
        assert torch.equal(qkv[:, H + Hkv:], before[:, H + Hkv:])     # the values between are untouched


def test_rotate_one_side_only_and_plain_copies(B):
    x = torch.randn(6, 4, D, device="cuda")
    inv = 10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64, device="cuda") / 128)
    pos, st = torch.arange(6, dtype=torch.int32, device="cuda"), i32([0, 6])
    out = torch.zeros_like(x)
    B.ckv_rotate(B.make_packed(x, None, 1), B.make_rotary(inv), x, None, pos, st, out, None)
    ref = R.turn(x, pos, inv)
    assert (out.double() - ref).abs().max() <= 40 * EPS * 2 * x.abs().max()
    out2 = torch.zeros_like(x)
    B.ckv_rotate(B.make_packed(None, x, 1), B.make_rotary(inv), None, x, pos, st, None, out2)
    assert torch.equal(out, out2)
    B.ckv_rotate(B.make_packed(x, None, 1), B.make_rotary(None), x, None, pos, st, out, None)
    assert torch.equal(out, x)                              # no norm, no rotation: the same bits


@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("layout", ["token, kind, head", "token, head, kind", "kind, token, head", "kind, head, token", "head, kind, token"])
def test_rotate_in_place_in_any_layout(B, layout, T):
    """Queries and keys as views of one projection, turned where they lie, whatever the order of its dimensions."""
    H = 4
    sizes = dict(token=T, kind=3, head=H)
    order = layout.split(", ")
    x = torch.randn(*[sizes[n] for n in order], D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(T))
    was = x.clone()
    view = lambda y, i: y.permute(*[order.index(n) for n in ("token", "kind", "head")], 3)[:, i]
    q, k = view(x, 0), view(x, 1)
    inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") + 5
    B.ckv_rotate(B.make_packed(q, k, 1), B.make_rotary(inv), q, k, pos, i32([0, T]), q, k)
    for i in range(2):
        want = R.turn(view(was, i), pos, inv)
        assert ((view(x, i).double() - want).abs() <= 80 * EPS * want.abs().amax(-1, keepdim=True) + 2 * EPS * want.abs()).all()
    assert torch.equal(view(x, 2), view(was, 2))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,Hkv,norm", [(889, 12, 12, False), (1783, 32, 8, True), (3553, 28, 4, True), (4575, 32, 8, False)])
def test_rotate_where_the_last_cta_is_not_full(B, dtype, T, H, Hkv, norm):
    """Two, four and eight tokens a CTA with one to seven in the last, more heads than the first batch of rows."""
    g = torch.Generator(device="cuda").manual_seed(T)
    qkv = torch.randn(T, H + 2 * Hkv, D, generator=g, device="cuda").to(dtype)
    q, k = qkv[:, :H], qkv[:, H:H + Hkv]
    pos = torch.randint(0, 1 << 17, (T,), generator=g, device="cuda", dtype=torch.int32)
    inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    w = [1 + 0.2 * torch.randn(D, generator=g, device="cuda") if norm else None for _ in range(2)]
    outs = torch.zeros(T, H, D, device="cuda", dtype=dtype), torch.zeros(T, Hkv, D, device="cuda", dtype=dtype)
    B.ckv_rotate(B.make_packed(q, k, 2), B.make_rotary(inv, q_norm_w=w[0], k_norm_w=w[1]), q, k, pos, i32([0, T // 2, T]), *outs)
    for x, wt, out in ((q, w[0], outs[0]), (k, w[1], outs[1])):
        want = R.turn(x, pos, inv, wt)
        tol = 80 * EPS * want.abs().amax(-1, keepdim=True) + (2.0 ** -8 if dtype == torch.bfloat16 else 2 * EPS) * want.abs()
        assert ((out.double() - want).abs() <= tol).all()


# ------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,Hkv,page,counts,lens,rot,norm", [
    (32, 8, 64, [1], [[0]], 128, False), (8, 2, 16, [1, 0, 5], [[15, 16], [3, 4], [31, 0]], 128, True),
    (28, 4, 32, [40, 1, 2], [[0, 1, 31, 32], [33, 63, 64, 65], [5, 6, 7, 8]], 64, True),
    (4, 4, 256, [300, 2], [[255, 256, 257, 0], [511, 1, 2, 3]], 0, False), (2, 1, 128, [2000], [[77]], 128, False)])
def test_append(B, dtype, H, Hkv, page, counts, lens, rot, norm):
    lens = [row if len(row) == Hkv else row * Hkv for row in lens]
    g = torch.Generator(device="cuda").manual_seed(sum(counts) + page)
    pad = 3
    c = R.Cache(lens, page, max_extra=max(counts), dtype=dtype, device="cuda", poison=3.0, row_pad=8 if page == 32 else 0)
    starts = starts_of(counts)
    T = starts[-1] + pad
    qkv = torch.randn(T, H + 2 * Hkv, D, generator=g, device="cuda").to(dtype)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    pos = torch.randint(0, 1 << 18, (T,), generator=g, device="cuda", dtype=torch.int32)
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1)) if rot else None
    w = [1 + 0.2 * torch.randn(D, generator=g, device="cuda") if norm else None for _ in range(2)]
    rotary = B.make_rotary(inv, q_norm_w=w[0], k_norm_w=w[1]) if rot or norm else None
    pg = B.make_paged(c.k_pages, c.table, q=q, k_new=k, max_new=max(counts))
    ws = B.alloc_paged_workspace(pg)
    q_out = torch.full((T, H, D), 5.0, device="cuda").to(dtype)
    new = torch.full((len(counts), Hkv), -1, dtype=torch.int32, device="cuda")
    want_k, want_v = (p.double().clone() for p in c.pools)
    size_k = want_k.abs()
    tk = R.turn(k, pos, inv, w[1])
    for u in range(len(counts)):
        for gg in range(Hkv):
            for i in range(counts[u]):
                j = lens[u][gg] + i
                at = int(c.table[u, gg, j // page]), j % page
                want_k[at][:D], want_v[at][:D] = tk[starts[u] + i, gg], v[starts[u] + i, gg].double()
                size_k[at][:D] = 2 * tk[starts[u] + i, gg].abs().max()
    B.ckv_append(pg, rotary, k, v, pos, i32(starts), c.lengths, c.table, c.k_pages, c.v_pages, ws, q=q, q_out=q_out, new_lengths=new)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2 * EPS
    assert torch.equal(c.pools[1].double(), want_v)
    assert ((c.pools[0].double() - want_k).abs() <= 40 * EPS * size_k + half * want_k.abs()).all()
    untouched = want_k == 3.0
    assert torch.equal(c.pools[0].double()[untouched], want_k[untouched])
    tq = R.turn(q, pos, inv, w[0])
    live = slice(0, starts[-1])
    assert ((q_out.double() - tq).abs() <= 80 * EPS * tq.abs().amax(-1, keepdim=True) + half * tq.abs())[live].all()
    assert (q_out[starts[-1]:] == 5.0).all()
    assert torch.equal(new, c.lengths + i32(counts)[:, None])
    assert B.ckv_device_status(ws) == B.OK
    # without queries and new lengths: the same pages
    again = [p.clone() for p in c.pools]
    B.ckv_append(pg, rotary, k, v, pos, i32(starts), c.lengths, c.table, c.k_pages, c.v_pages, ws)
    assert torch.equal(again[0], c.pools[0]) and torch.equal(again[1], c.pools[1])


@pytest.mark.parametrize("Nu,per", [(600, 1), (520, 5), (33, 100), (3, 0)])
def test_append_many_units(B, Nu, per):
    """Units found among many starts, empty ones among them; a call without tokens still hands the lengths on."""
    counts = [(u * 7) % (per + 1) if per != 1 else 1 for u in range(Nu)]
    st = starts_of(counts)
    lens = [[(u * 5) % 40] for u in range(Nu)]
    c = R.Cache(lens, 16, max_extra=max(max(counts), 1), dtype=torch.float32, device="cuda", poison=3.0)
    k = torch.randn(st[-1], 1, D, device="cuda")
    v = torch.randn(st[-1], 1, D, device="cuda")
    pg = B.make_paged(c.k_pages, c.table, k_new=k)
    ws = B.alloc_paged_workspace(pg)
    new = torch.full((Nu, 1), -1, dtype=torch.int32, device="cuda")
    B.ckv_append(pg, None, k, v, None, i32(st), c.lengths, c.table, c.k_pages, c.v_pages, ws, new_lengths=new)
    assert torch.equal(new, c.lengths + i32(counts)[:, None]) and B.ckv_device_status(ws) == B.OK
    for u in range(Nu):
        for i in range(counts[u]):
            j = lens[u][0] + i
            assert torch.equal(c.k_pages[int(c.table[u, 0, j // 16]), j % 16], k[st[u] + i, 0]), (u, i)
            assert torch.equal(c.v_pages[int(c.table[u, 0, j // 16]), j % 16], v[st[u] + i, 0]), (u, i)
            if u > 40:
                break
    assert int((c.pools[0] != 3.0).any(-1).sum()) == sum(x[0] for x in lens) + sum(counts)


def test_append_leaves_out_rows_that_have_no_page_and_says_so(B):
    c = R.Cache([[20, 3]], 16, max_extra=4, dtype=torch.float32, device="cuda", poison=3.0)
    k = torch.randn(4, 2, D, device="cuda")
    pg = B.make_paged(c.k_pages, c.table, k_new=k)
    ws = torch.randint(0, 255, (B.ckv_paged_workspace_bytes(pg),), dtype=torch.uint8, device="cuda")   # nobody cleared it
    args = lambda table, lengths: (pg, None, k, k, None, i32([0, 4]), lengths, table, c.k_pages, c.v_pages, ws)
    before = c.pools[0].clone()
    for bad in (torch.full_like(c.table, -1), torch.full_like(c.table, 1 << 30)):
        B.ckv_append(*args(bad, c.lengths))
        assert B.ckv_device_status(ws) == B.ERR_PAGE and B.ckv_device_status(ws) == B.OK
    for lengths in (i32([[-4, -9]]), i32([[2147483647, 1 << 30]])):
        B.ckv_append(*args(c.table, lengths))
        assert B.ckv_device_status(ws) == B.ERR_PAGE
    assert torch.equal(before, c.pools[0])
    B.ckv_append(*args(c.table, c.lengths))
    assert B.ckv_device_status(ws) == B.OK
    assert torch.equal(c.k_pages[c.table[0, 1, 0].long(), 3:7], k[:, 1])


@pytest.mark.parametrize("layout", ["page, kind, row", "page, row, kind", "kind, page, row"])
@pytest.mark.parametrize("n", [1, 60])
def test_interleaved_pools(B, layout, n):
    """Keys and values as views of one pool."""
    P, pages = 32, 9
    order = layout.split(", ")
    sizes = dict(page=pages, row=P, kind=2)
    pool = torch.full([sizes[x] for x in order] + [D], float("nan"), dtype=torch.bfloat16, device="cuda")
    kp, vp = (pool.permute(*[order.index(x) for x in ("kind", "page", "row")], 3)[i] for i in range(2))
    table = torch.arange(8, dtype=torch.int32, device="cuda").flip(0).view(1, 2, 4).contiguous()
    x, v = (torch.randn(n + 50, 2, D, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(n, 8, D, device="cuda").bfloat16()
    grown = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    pk, pq = B.make_paged(kp, table, k_new=x), B.make_paged(kp, table, q=q)
    ws = B.alloc_paged_workspace(pq)
    B.ckv_append(pk, None, x, v, None, i32([0, n + 50]), i32([[0, 0]]), table, kp, vp, ws, new_lengths=grown)
    out, lse = torch.zeros_like(q), torch.zeros(n, 8, device="cuda")
    B.ckv_paged_attend(pq, q, kp, vp, table, grown, i32([0, n]), out, ws, lse=lse)
    assert B.ckv_device_status(ws) == B.OK
    want, want_lse = R.attend(q, [0, n], [[(x[:, g], v[:, g]) for g in range(2)]])
    assert (out.double() - want).norm() <= 2 * 2.0 ** -8 * want.norm() and (lse.double() - want_lse).abs().max() <= 1e-3
    assert torch.isnan(kp[8]).all() and torch.isnan(vp[8]).all()


# ---------------------------------------------------------------------------------------- gather into pages
@pytest.mark.parametrize("cfg_name,page,L", [("c1", 16, 2048), ("c2", 64, 4096), ("c5", 256, 1111)])
def test_gather_pages(B, cfg_name, page, L):
    from test_gpu_parity import params_of, problem_of
    cfg = gen.shrink(gen.CONFIGS[cfg_name], n_layers=2, batch=1, seq_len=L, budget_per_head=128, n_needles=4)
    b = gen.make_batch(cfg, "cuda")
    P = params_of(B, problem_of(cfg, 2))
    out = B.compress(b["q"], b["k"], b["v"], b["head_w"], b["sens"], P)
    shape, params = B.make_shape(b["q"], b["k"]), B.make_params(P, b["head_w"], b["sens"])
    bud = out["budgets"].tolist()
    c = R.Cache(bud, page, dtype=b["k"].dtype, device="cuda", poison=9.0)
    for p in c.pools:
        p.fill_(9.0)
    pg = B.make_paged(c.k_pages, c.table, n_q_heads=cfg.n_q_heads)
    ws = B.alloc_paged_workspace(pg)
    lengths = torch.full_like(out["budgets"], -1)
    B.ckv_gather_pages(shape, params, pg, b["k"], b["v"], out["indices"], out["budgets"], out["offsets"], c.table, c.k_pages,
                       c.v_pages, lengths, ws)
    assert torch.equal(lengths, out["budgets"]) and B.ckv_device_status(ws) == B.OK
    off = out["offsets"].tolist()
    for pool, src in zip((c.k_pages, c.v_pages), ("k_out", "v_out")):
        want = torch.full_like(pool, 9.0)
        for u in range(2):
            for g in range(cfg.n_kv_heads):
                for j in range(bud[u][g]):
                    want[int(c.table[u, g, j // page]), j % page] = out[src][u, off[u][g] + j]
        assert torch.equal(pool, want)
    short = torch.full_like(c.table, -1)
    B.ckv_gather_pages(shape, params, pg, b["k"], b["v"], out["indices"], out["budgets"], out["offsets"], short, c.k_pages,
                       c.v_pages, lengths, ws)
    assert B.ckv_device_status(ws) == B.ERR_PAGE


# ------------------------------------------------------------------------------------------------ attend
def run_attend(B, c, q, starts, causal=True, scale=0.0, max_new=0, lse=True):
    pg = B.make_paged(c.k_pages, c.table, q=q, causal=causal, scale=scale, max_new=max_new)
    n = B.ckv_paged_workspace_bytes(pg)
    ws = torch.full((n + 512,), 0xAB, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 11.0, device="cuda").to(q.dtype)
    l = torch.full(q.shape[:2], 11.0, device="cuda") if lse else None
    B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, i32(starts), out, ws[256:256 + n], lse=l)
    assert B.ckv_device_status(ws[256:256 + n]) == B.OK
    assert (ws[:256] == 0xAB).all() and (ws[256 + n:] == 0xAB).all()
    return out, l


def check_attend(c, q, starts, out, lse, causal=True, scale=None, spread=True):
    want, want_lse = R.attend(q, starts, c.rows, causal, scale)
    live = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    live[starts[0]:starts[-1]] = True
    s = 1 / math.sqrt(D) if scale is None else abs(scale)
    kmax = max([float(k.double().norm(dim=-1).max()) for row in c.rows for k, _ in row if k.shape[0]] + [0.0])
    vmax = max([float(v.double().abs().max()) for row in c.rows for _, v in row if v.shape[0]] + [0.0])
    depth = max(max(r) for r in c.lens) / 8 + 256
    r = 132 * EPS * float(q[live].double().norm(dim=-1).max()) * kmax * s + 2.0 ** -20 + depth * EPS
    tol = 2 * r * vmax + (2.0 ** -8 * (vmax + want.abs()) if q.dtype == torch.bfloat16 else EPS * want.abs())
    err = (out.double() - want).abs()
    assert (err <= tol)[live].all(), float((err / tol)[live].max())
    if q.dtype == torch.bfloat16 and spread and bool(live.any()):
        assert err[live].norm() <= 2 * 2.0 ** -8 * want[live].norm() + 2 * r * vmax * math.sqrt(err[live].numel())
    if lse is not None:
        none = torch.isinf(want_lse)
        assert torch.equal((lse == -math.inf)[live], none[live])
        seen = live[:, None] & ~none
        assert ((lse.double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs())[seen].all()
        assert (lse[~live] == 11.0).all()
    assert (out[~live] == 11.0).all()


CASES = [
    # H, Hkv, page, tokens per unit, rows per (unit, head) after the tokens
    (8, 2, 16, [1], [[1, 1]]),
    (8, 2, 16, [1], [[0, 5]]),
    (32, 8, 64, [1], [[512, 400, 1, 63, 64, 65, 127, 129]]),
    (28, 4, 16, [1, 1, 1], [[100, 0, 17, 256], [1, 2, 3, 4], [700, 701, 699, 15]]),
    (28, 4, 32, [5, 3, 0, 1], [[300, 5, 31, 33], [64, 65, 3, 3], [9, 9, 9, 9], [128, 127, 129, 1]]),
    (16, 16, 128, [2, 7], [[130] * 16, [200] * 16]),
    (24, 2, 64, [3], [[1000, 37]]),
    (40, 1, 64, [4, 1], [[333], [90]]),
    (8, 1, 256, [16], [[5000]]),
    (4, 4, 16, [33, 1, 70], [[33, 40, 1000, 64], [9, 8, 7, 6], [70, 71, 300, 128]]),
    (32, 8, 64, [130], [[130, 131, 200, 256, 257, 640, 1000, 2000]]),
    (28, 4, 16, [19, 200], [[19, 20, 500, 128], [200, 255, 256, 1100]]),
    (6, 2, 128, [257, 1, 64], [[300, 1500], [1500, 1], [64, 65]]),
    (8, 8, 32, [128, 129], [[128, 129, 130, 500, 140, 150, 160, 170], [129, 300, 301, 302, 303, 304, 305, 306]]),
    (128, 1, 64, [5], [[77]]),
    (130, 1, 64, [3], [[77]]),
    (8, 2, 64, [7], [[3, 6]]),                       # more tokens than rows: the first ones see nothing
    (8, 2, 64, [300], [[100, 290]]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hkv,page,counts,lens", CASES)
def test_attend(B, dtype, causal, H, Hkv, page, counts, lens):
    """Rows behind the lengths, pages of nobody and padding tokens are NaN; table entries of no row point far outside."""
    c = R.Cache(lens, page, dtype=dtype, device="cuda", seed=H + page, row_pad=8 if page == 32 else 0)
    starts = starts_of(counts, 2)
    g = torch.Generator(device="cuda").manual_seed(len(counts))
    qkv = torch.randn(starts[-1] + 3, H + 4, D, generator=g, device="cuda").to(dtype)
    qkv[:2] = float("nan")
    qkv[starts[-1]:] = float("nan")
    q = qkv[:, 1:1 + H]
    for max_new in (0, max(counts)):
        out, lse = run_attend(B, c, q, starts, causal, max_new=max_new)
        check_attend(c, q, starts, out, lse, causal)


MANY = {
    # more (unit, KV head) pairs than one warp schedules, units without tokens among them, short and long caches
    "decode short": (40, 8, 8, 16, lambda u: 1 if u % 7 else 0, lambda u, g: 3 + (37 * u + 11 * g) % 200),
    "decode long": (33, 4, 8, 64, lambda u: u % 2, lambda u, g: 1200 + (97 * u + 501 * g) % 1500),
    "verify": (50, 3, 9, 32, lambda u: (u * 5) % 4, lambda u, g: 4 + (61 * u + 17 * g) % 1300),
    "chunks": (36, 4, 8, 16, lambda u: (0, 1, 40, 3)[u % 4], lambda u, g: 40 + (53 * u + 29 * g) % 300),
    "one head": (700, 1, 4, 16, lambda u: 1, lambda u, g: 1 + (u * 13) % 90),
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("name", list(MANY))
def test_attend_many_heads(B, dtype, name):
    Nu, Hkv, H, page, count, length = MANY[name]
    counts = [count(u) for u in range(Nu)]
    lens = [[length(u, g) for g in range(Hkv)] for u in range(Nu)]
    c = R.Cache(lens, page, dtype=dtype, device="cuda", seed=Nu)
    st = starts_of(counts)
    q = torch.randn(st[-1] + 1, H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).to(dtype)
    for max_new in (0, max(counts), 1):          # the last one may be less than the truth: it only picks kernels
        out, lse = run_attend(B, c, q, st, max_new=max_new)
        check_attend(c, q, st, out, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("counts,length", [([1], 40000), ([1, 1], 9000), ([6], 20000), ([100], 9000), ([700], 3000)])
def test_attend_long(B, dtype, counts, length):
    """Items split over many CTAs."""
    lens = [[length - 7 * u, length // 3] for u in range(len(counts))]
    c = R.Cache(lens, 64, dtype=dtype, device="cuda", seed=length)
    q = torch.randn(sum(counts), 8, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype)
    st = starts_of(counts)
    out, lse = run_attend(B, c, q, st, max_new=max(counts))
    check_attend(c, q, st, out, lse)
    out2, lse2 = run_attend(B, c, q, st, max_new=max(counts), lse=False)
    assert torch.equal(out, out2)


@pytest.mark.parametrize("causal", [True, False])
def test_attend_wide_group_on_a_long_cache(B, causal):
    """More query heads per KV head than a tensor-core block has rows: blocks of 32 rows, split along the keys."""
    c = R.Cache([[12000], [9001]], 64, device="cuda", seed=4)
    q = torch.randn(4, 150, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).bfloat16()
    for max_new in (0, 3, 1):
        out, lse = run_attend(B, c, q, [0, 1, 4], causal, max_new=max_new)
        check_attend(c, q, [0, 1, 4], out, lse, causal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Nu,Hkv,H,counts,extra", [
    (1, 1, 4, [1100], 40),                                   # the blocks of one head spread over the threads
    (3, 2, 8, [257, 0, 600], 300),
    (30, 8, 16, [0, 70, 129, 1, 260], 20),                   # a few hundred heads of up to three blocks
    (60, 8, 8, [300, 1, 0, 33], 0),                          # more heads than threads
    (5, 4, 32, [512, 64, 65, 1, 200], 700),                  # whole items first, then shares
    (4, 8, 32, [700, 650, 800, 1], 0),                       # items of one key tile and of many
    (1, 1, 200, [21], 300),                                  # more query heads than a tensor-core block has rows
    (7, 2, 8, [16, 3, 0, 9], 250),                           # a head's blocks shared out to clusters
])
def test_attend_schedules(B, dtype, Nu, Hkv, H, counts, extra):
    """Long chunks of many shapes: whatever max_new says, the same rows come out."""
    counts = [counts[u % len(counts)] for u in range(Nu)]
    lens = [[n + (extra * (u + 3 * g)) % (2 * extra + 1) for g in range(Hkv)] for u, n in enumerate(counts)]
    c = R.Cache(lens, 32, dtype=dtype, device="cuda", seed=Nu + Hkv)
    st = starts_of(counts)
    q = torch.randn(st[-1], H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).to(dtype)
    for max_new in (0, max(counts), 40, 1):
        out, lse = run_attend(B, c, q, st, max_new=max_new)
        check_attend(c, q, st, out, lse)


@pytest.mark.parametrize("n", [5, 20, 64, 90, 300])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_attend_infinite_values_inside_a_chunk(B, n, bad):
    """A value row with one element that is not finite reaches the tokens that see it, in that element, and no others."""
    lens = [[n + 200, n + 61]]
    c = R.Cache(lens, 32, device="cuda", seed=n)
    rows = []
    for g in range(2):
        k, v = c.rows[0][g]
        hit = sorted({lens[0][g] - x for x in (1, 2, n // 2 + 1, n // 3 + 1, 3 * n // 4 + 1, n - 1)})
        v = v.clone()
        for j in hit:
            v[j, 7 * g + 3] = bad
            c.v_pages[int(c.table[0, g, j // 32]), j % 32, 7 * g + 3] = bad
        rows.append((k, v, hit[0]))
    q = torch.randn(n, 8, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).bfloat16()
    for max_new in (0, n):
        out, lse = run_attend(B, c, q, [0, n], max_new=max_new)
        for g in range(2):
            first = rows[g][2] - (lens[0][g] - n)              # the first token that sees a bad row
            mine = out[:, 4 * g:4 * g + 4]
            assert not torch.isfinite(mine[first:, :, 7 * g + 3]).any()
            mine[first:, :, 7 * g + 3] = 0.0
            assert torch.isfinite(mine).all()
        # the element aside, the outputs are those of the clean cache
        want, want_lse = R.attend(q, [0, n], c.rows)
        for g in range(2):
            first = rows[g][2] - (lens[0][g] - n)
            want[first:, 4 * g:4 * g + 4, 7 * g + 3] = 0.0
        vmax = max(float(v.double().abs().max()) for _, v in c.rows[0])
        kmax = max(float(k.double().norm(dim=-1).max()) for k, _ in c.rows[0])
        r = 132 * EPS * float(q.double().norm(dim=-1).max()) * kmax / math.sqrt(D) + 2.0 ** -20 + (lens[0][0] / 8 + 256) * EPS
        assert ((out.double() - want).abs() <= 2.0 ** -8 * (vmax + want.abs()) + 2 * r * vmax).all()
        assert ((lse.double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("counts", [[1], [40], [200]])
def test_attend_large_logits_and_scales(B, dtype, counts):
    """One key far above the others, negative and tiny scales, and logits of hundreds that grow along the cache (the running
    maximum moves at every tile)."""
    n = counts[0]
    c = R.Cache([[n + 900, n + 130]], 32, dtype=dtype, device="cuda", seed=3)
    for g in range(2):
        k, v = c.rows[0][g]
        ramp = torch.linspace(0.0, 6.0, k.shape[0]).double()[:, None]
        k2 = (k.double() * ramp).to(dtype)
        c.rows[0][g] = (k2, v)
        for j in range(k.shape[0]):
            c.k_pages[int(c.table[0, g, j // 32]), j % 32] = k2[j].cuda()
    q = torch.randn(n, 8, D, device="cuda").to(dtype)
    for scale in (0.0, 1.0, -0.7, 1e-3):
        out, lse = run_attend(B, c, q, [0, n], scale=scale)
        check_attend(c, q, [0, n], out, lse, scale=scale or None, spread=False)


@pytest.mark.parametrize("size", [1e21, 4e27])
@pytest.mark.parametrize("dtype,counts,rows", [
    (torch.float32, [3], 1500), (torch.bfloat16, [1], 700), (torch.bfloat16, [4], 12000), (torch.bfloat16, [40], 20000),
    (torch.bfloat16, [90], 20000), (torch.bfloat16, [300], 9000), (torch.bfloat16, [700], 800)])
def test_attend_large_values_under_rising_logits(B, dtype, counts, rows, size):
    """Values up to 2^94 stay in range in every kernel while the logits climb by 41 (a factor of 2^59) over 256 keys and fall again,
    over and over, so that each of the parts a cache is cut into sees a rise."""
    n = counts[0]
    c = R.Cache([[n + rows, n + rows // 3]], 32, dtype=dtype, device="cuda", seed=n)
    q = torch.randn(n, 8, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).mul_(0.1)
    q[..., 0] = 8.0
    q = q.to(dtype)
    for g in range(2):
        k, v = c.rows[0][g]
        L = k.shape[0]
        k = k.clone()
        wave = torch.cat((torch.zeros(128), torch.linspace(0.0, 41.0 * math.sqrt(D) / 8.0, 256), torch.zeros(128)))
        k[:, 0] = wave.repeat(L // 512 + 1)[:L].to(dtype)
        v = (v.double() * size).clamp(-2.0 ** 94, 2.0 ** 94).to(dtype)
        c.rows[0][g] = (k, v)
        for pool, x in ((c.k_pages, k), (c.v_pages, v)):
            for j in range(0, L, 32):
                pool[int(c.table[0, g, j // 32]), :min(32, L - j)] = x[j:j + 32].cuda()
    for causal in (True, False):
        out, lse = run_attend(B, c, q, [0, n], causal)
        assert torch.isfinite(out).all()
        check_attend(c, q, [0, n], out, lse, causal, spread=False)


@pytest.mark.parametrize("counts", [[1], [5], [150]])
def test_attend_masked_infinities(B, counts):
    """Infinite and NaN keys and values behind what a token sees do not reach it."""
    n = counts[0]
    for poison in (float("inf"), float("-inf"), float("nan"), torch.finfo(torch.bfloat16).min):
        c = R.Cache([[n + 50, n + 64]], 64, dtype=torch.bfloat16, device="cuda", poison=poison)
        # the chunk's last token is poison too: only its own query may see it
        q = torch.randn(n, 8, D, device="cuda").bfloat16()
        if n > 1:
            for g in range(2):
                j = c.lens[0][g] - 1
                c.k_pages[int(c.table[0, g, j // 64]), j % 64] = poison
                c.v_pages[int(c.table[0, g, j // 64]), j % 64] = poison
        out, lse = run_attend(B, c, q, [0, n])
        seen = n - 1 if n > 1 else 1
        rows = [[(k, v) for k, v in c.rows[0]]]
        want, want_lse = R.attend(q, [0, n], rows)
        assert (out.double() - want).abs()[:seen].max() <= 0.03
        assert (lse.double() - want_lse).abs()[:seen].max() <= 1e-3


@pytest.mark.parametrize("where", ["query", "keys"])
@pytest.mark.parametrize("counts,rows,width", [
    ([1], [[300, 90]], 0), ([1], [[9000, 700]], 0), ([1, 1, 1], [[500, 40], [33, 1], [600, 600]], 900),    # clusters, split, wide tables
    ([5], [[400, 77]], 0), ([5, 2], [[16000, 3000], [900, 2]], 0), ([7], [[400, 77]], 900),
    ([30], [[300, 31]], 0), ([100], [[100, 700]], 0), ([90], [[9000, 8000]], 0), ([400, 3], [[3000, 400], [70, 3]], 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attend_carries_nan(B, dtype, counts, rows, width, where):
    """A NaN in a query, or in every key a token sees, reaches that token's output and lse, and nobody else's: only a token that
    sees no row gets zeros.  More tokens than rows among them, whose first see nothing."""
    H, Hkv = 8, 2
    c = R.Cache(rows, 32, dtype=dtype, device="cuda", seed=sum(counts), max_extra=0)
    if width:
        wide = torch.full((len(rows), Hkv, width), 0x7ffffff0, dtype=torch.int32, device="cuda")
        wide[:, :, :c.max_pages] = c.table
        c.table, c.max_pages = wide, width
    st = starts_of(counts)
    q = torch.randn(st[-1], H, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).to(dtype)
    sick = torch.zeros(st[-1], H, dtype=torch.bool, device="cuda")
    clean = q.clone()
    if where == "query":
        for t in {0, st[-1] // 2, st[-1] - 1}:
            for h in (1, 6):
                q[t, h, (7 * t + h) % D] = float("nan")
                sick[t, h] = True
    else:                                              # unit 0, head 0: every key
        k, v = c.rows[0][0]
        c.rows[0][0] = (torch.full_like(k, float("nan")), v)
        for j in range(0, k.shape[0], 32):
            c.k_pages[int(c.table[0, 0, j // 32]), :min(32, k.shape[0] - j)] = float("nan")
        sick[:st[1], :H // Hkv] = True
    for causal in (True, False):
        out, lse = run_attend(B, c, q, st, causal, max_new=max(counts))
        want, want_lse = R.attend(q, st, c.rows, causal)
        ill = sick.clone()
        for u in range(len(counts)):                   # tokens that see nothing stay as they are
            for g in range(Hkv):
                for i in range(max(0, min(counts[u], counts[u] - rows[u][g])) if causal else 0):
                    ill[st[u] + i, g * (H // Hkv):(g + 1) * (H // Hkv)] = False
        assert torch.equal(torch.isnan(lse), ill)
        assert torch.equal(torch.isnan(out).all(-1), ill) and torch.equal(torch.isnan(out).any(-1), ill)
        well = ~ill
        assert torch.equal((lse == -math.inf)[well], torch.isinf(want_lse)[well])
        seen = well & ~torch.isinf(want_lse)
        # (as check_attend, for the tokens that are well)
        kmax = max(float(k.double().nan_to_num().norm(dim=-1).max()) for row in c.rows for k, _ in row)
        vmax = max(float(v.double().abs().max()) for row in c.rows for _, v in row)
        r = 132 * EPS * float(clean.double().norm(dim=-1).max()) * kmax / math.sqrt(D) + 2.0 ** -20 + (max(map(max, rows)) / 8 + 256) * EPS
        assert ((lse.double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs())[seen].all()
        tol = 2 * r * vmax + (2.0 ** -8 * (vmax + want.abs()) if dtype == torch.bfloat16 else EPS * want.abs())
        assert ((out.double() - want).abs() <= tol)[seen].all()
        assert (out[well & torch.isinf(want_lse)] == 0).all()


@pytest.mark.parametrize("dtype,counts", [(torch.float32, [2]), (torch.bfloat16, [2]), (torch.bfloat16, [90])])
def test_attend_leaves_out_bad_pages_and_says_so(B, dtype, counts):
    n = counts[0]
    c = R.Cache([[n + 200, n + 77]], 16, dtype=dtype, device="cuda")
    q = torch.randn(n, 4, D, device="cuda").to(dtype)
    pg = B.make_paged(c.k_pages, c.table, q=q, causal=False)
    ws = B.alloc_paged_workspace(pg)
    out, lse = torch.zeros_like(q), torch.zeros(n, 4, device="cuda")
    table = c.table.clone()
    table[0, 0, 2] = -1
    table[0, 1, 0] = c.k_pages.shape[0]
    B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, table, c.lengths, i32([0, n]), out, ws, lse=lse)
    assert B.ckv_device_status(ws) == B.ERR_PAGE and B.ckv_device_status(ws) == B.OK
    keep = [torch.cat((k[:32], k[48:])) for k in c.rows[0][0]], [k[16:] for k in c.rows[0][1]]
    want, want_lse = R.attend(q, [0, n], [[tuple(keep[0]), tuple(keep[1])]], causal=False)
    assert (out.double() - want).abs().max() <= 0.03 and (lse.double() - want_lse).abs().max() <= 1e-3
    # a length past the table's pages ends at its last page
    B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, i32([[1 << 30, -5]]), i32([0, n]), out, ws, lse=lse)
    assert B.ckv_device_status(ws) == B.ERR_PAGE
    assert (out[:, 2:] == 0).all() and (lse[:, 2:] == -math.inf).all()
    # token starts that run off the tokens or backwards are never followed
    B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, i32([-7, 1 << 30]), out, ws, lse=lse)
    B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, i32([n, 0]), out, ws, lse=lse)
    assert B.ckv_device_status(ws) == B.OK


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("counts,pages", [([1], 4), ([5], 4), ([5], 400), ([40], 20), ([300], 30), ([90, 7], 300)])
def test_attend_leaves_out_rows_past_the_table(B, dtype, causal, counts, pages):
    """Lengths past the table's last page (an append that ran out of pages): the rows it has no place for are left out, every
    other row is seen by the tokens that the lengths say see it."""
    room = 32 * pages
    c = R.Cache([[room, room] for _ in counts], 32, dtype=dtype, device="cuda", seed=pages)
    q = torch.randn(sum(counts), 8, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(dtype)
    st = starts_of(counts)
    more = [[max(1, n // 2), max(1, n - 1)] for n in counts]
    pg = B.make_paged(c.k_pages, c.table, q=q, causal=causal)
    ws = B.alloc_paged_workspace(pg)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, i32([[room + x for x in m] for m in more]), i32(st), out, ws, lse=lse)
    assert B.ckv_device_status(ws) == B.ERR_PAGE and B.ckv_device_status(ws) == B.OK
    for u, n in enumerate(counts):
        for g in range(2):
            k, v = (x.cuda().double() for x in c.rows[u][g])
            qs = q[st[u]:st[u + 1], 4 * g:4 * g + 4].double()
            x = torch.einsum("nhd,ld->nhl", qs, k) / math.sqrt(D)
            if causal:
                sees = room + more[u][g] - n + torch.arange(n, device="cuda")
                x = x.masked_fill((torch.arange(room, device="cuda")[None] > sees[:, None])[:, None], -math.inf)
            want = torch.einsum("nhl,ld->nhd", torch.softmax(x, -1), v)
            r = 132 * EPS * float(q.double().norm(dim=-1).max()) * float(k.norm(dim=-1).max()) / math.sqrt(D) + 2.0 ** -20 + (room / 8 + 256) * EPS
            tol = 2 * r * v.abs().max() + (2.0 ** -8 * (v.abs().max() + want.abs()) if dtype == torch.bfloat16 else EPS * want.abs())
            assert ((out[st[u]:st[u + 1], 4 * g:4 * g + 4].double() - want).abs() <= tol).all()
            want_lse = torch.logsumexp(x, -1)
            assert ((lse[st[u]:st[u + 1], 4 * g:4 * g + 4].double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs()).all()


def test_attend_same_bits_again_and_on_two_streams(B):
    for counts in ([1, 1], [60, 3]):
        c = R.Cache([[3000, 100], [777, 2500]], 64, dtype=torch.bfloat16, device="cuda")
        q = torch.randn(sum(counts), 16, D, device="cuda").bfloat16()
        st = i32(starts_of(counts))
        pg = B.make_paged(c.k_pages, c.table, q=q, max_new=max(counts))
        streams = [torch.cuda.Stream() for _ in range(2)]
        ws = [B.alloc_paged_workspace(pg) for _ in range(2)]
        outs = [torch.zeros_like(q) for _ in range(2)]
        torch.cuda.synchronize()
        first = None
        for _ in range(5):
            for s, w, o in zip(streams, ws, outs):
                B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, st, o, w, stream=s)
            torch.cuda.synchronize()
            first = outs[0].clone() if first is None else first
            assert torch.equal(outs[0], first) and torch.equal(outs[1], first)


def test_attend_same_bits_whatever_ran_before(B):
    """Groups that do not fill a tensor-core block leave rows of it to what shared memory held: no token's bits depend on it."""
    n = 100
    c = R.Cache([[n + 900] * 4], 32, device="cuda", seed=8)
    other = R.Cache([[n + 900] * 4], 32, device="cuda", seed=9)
    q = torch.randn(n, 28, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6)).bfloat16()
    big = torch.randn(n, 32, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)).bfloat16()
    seen = []
    for factor in (0.0, 300.0, 1.0, 3e4):
        run_attend(B, other, big * factor, [0, n])
        seen.append(run_attend(B, c, q, [0, n]))
    for out, lse in seen[1:]:
        assert torch.equal(out, seen[0][0]) and torch.equal(lse, seen[0][1])
    check_attend(c, q, [0, n], *seen[0])


def test_two_graphs_share_a_work_space(B):
    """Two captured steps of different shapes on one work space, replayed in turn: neither leaves anything the other trips over."""
    cases = []
    for counts, lens in (([1, 1], [[3000, 100], [777, 2500]]), ([60], [[2000, 333]]), ([1], [[40, 17]])):
        c = R.Cache(lens, 64, dtype=torch.bfloat16, device="cuda", seed=sum(counts))
        q = torch.randn(sum(counts), 16, D, device="cuda").bfloat16()
        pg = B.make_paged(c.k_pages, c.table, q=q, max_new=max(counts))
        cases.append((c, q, pg, i32(starts_of(counts)), torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda"), counts))
    ws = torch.randint(0, 255, (max(B.ckv_paged_workspace_bytes(x[2]) for x in cases),), dtype=torch.uint8, device="cuda")
    graphs = []
    for c, q, pg, st, out, lse, _ in cases:
        B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, st, out, ws, lse=lse)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, st, out, ws, lse=lse)
        graphs.append(g)
    first = []
    for c, q, pg, st, out, lse, counts in cases:
        want, want_lse = R.attend(q, starts_of(counts), c.rows)
        assert (out.double() - want).norm() <= 2 * 2.0 ** -8 * want.norm() and (lse.double() - want_lse).abs().max() <= 1e-3
        first.append(out.clone())
        out.fill_(5.0)
    for turn in range(6):
        for g in (graphs if turn % 2 else graphs[::-1]):
            g.replay()
    torch.cuda.synchronize()
    for x, want in zip(cases, first):
        assert torch.equal(x[4], want)
    assert B.ckv_device_status(ws) == B.OK


def test_offsets_past_32_bits(B):
    """A pool of more than 2^32 bytes and 2^31 elements: appended to and read at its far end."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    P, n_pages = 256, 70000            # 2.29e9 elements, 4.6 GB a pool
    kp, vp = (torch.empty(n_pages, P, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[[n_pages - 1, 3, n_pages - 2]]], dtype=torch.int32, device="cuda")
    x = torch.randn(600, 1, D, device="cuda").bfloat16()
    v = torch.randn(600, 1, D, device="cuda").bfloat16()
    for n in (600, 1):
        q = torch.randn(n, 4, D, device="cuda").bfloat16()
        pg = B.make_paged(kp, table, q=q)
        pk = B.make_paged(kp, table, k_new=x)
        ws = B.alloc_paged_workspace(pg)
        new = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
        B.ckv_append(pk, None, x, v, None, i32([0, 600]), i32([[0]]), table, kp, vp, ws, new_lengths=new)
        assert torch.equal(kp[n_pages - 1], x[:P, 0]) and torch.equal(vp[n_pages - 2, :88], v[512:, 0])
        out, lse = torch.zeros_like(q), torch.zeros(n, 4, device="cuda")
        B.ckv_paged_attend(pg, q, kp, vp, table, new, i32([0, n]), out, ws, lse=lse)
        want, want_lse = R.attend(q, [0, n], [[(x[:, 0], v[:, 0])]])
        assert (out.double() - want).abs().max() <= 0.05 and (lse.double() - want_lse).abs().max() <= 1e-3


# ------------------------------------------------------------------------------------- as they are used together
@pytest.mark.parametrize("cfg_name,chunk", [("c2", 1), ("c2", 80), ("c5", 3), ("c1", 2)])
def test_prompt_to_decode(B, cfg_name, chunk):
    """rotate -> the retention pass -> gather_pages -> (append -> attend) over several steps, the steps as one captured graph
    replayed with new tokens; against the 64-bit statement on the rows the pass kept."""
    from test_gpu_parity import params_of, problem_of
    Nu, L = 2, 1500
    cfg = gen.shrink(gen.CONFIGS[cfg_name], n_layers=Nu, batch=1, seq_len=L, budget_per_head=160, n_needles=4)
    H, Hkv, W = cfg.n_q_heads, cfg.n_kv_heads, cfg.window
    dt = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
    b = gen.make_batch(cfg, "cuda")
    qkv = torch.randn(Nu * L, H + 2 * Hkv, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).to(dt)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    pos = torch.arange(L, dtype=torch.int32, device="cuda").repeat(Nu)
    inv = 500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    rotary = B.make_rotary(inv, q_norm_w=torch.ones(D, device="cuda"), k_norm_w=torch.ones(D, device="cuda"))
    B.ckv_rotate(B.make_packed(q, k, Nu), rotary, q, k, pos, i32([0, L, 2 * L]), q, k)
    kd, vd = k.unflatten(0, (Nu, L)).transpose(1, 2), v.unflatten(0, (Nu, L)).transpose(1, 2)
    qw = q.unflatten(0, (Nu, L))[:, L - W:].transpose(1, 2)
    P = params_of(B, problem_of(cfg, Nu))
    kept = B.compress(qw, kd, vd, b["head_w"], b["sens"], P)
    shape, params = B.make_shape(qw, kd), B.make_params(P, b["head_w"], b["sens"])
    bud = kept["budgets"].tolist()
    steps = 3
    c = R.Cache(bud, 32, max_extra=steps * chunk, dtype=dt, device="cuda")
    T = Nu * chunk
    new = torch.zeros(T, H + 2 * Hkv, D, device="cuda", dtype=dt)
    nq, nk, nv = new[:, :H], new[:, H:H + Hkv], new[:, H + Hkv:]
    pg = B.make_paged(c.k_pages, c.table, q=nq, k_new=nk, max_new=chunk)
    po = B.make_paged(c.k_pages, c.table, q=torch.empty(T, H, D, device="cuda", dtype=dt), max_new=chunk)
    ws = B.alloc_paged_workspace(pg)
    lengths, grown = torch.zeros(Nu, Hkv, dtype=torch.int32, device="cuda"), torch.zeros(Nu, Hkv, dtype=torch.int32, device="cuda")
    npos, st = torch.zeros(T, dtype=torch.int32, device="cuda"), i32(starts_of([chunk] * Nu))
    q_out, out = torch.zeros(T, H, D, device="cuda", dtype=dt), torch.zeros(T, H, D, device="cuda", dtype=dt)
    lse = torch.zeros(T, H, device="cuda")

    def step():
        B.ckv_append(pg, rotary, nk, nv, npos, st, lengths, c.table, c.k_pages, c.v_pages, ws, q=nq, q_out=q_out, new_lengths=grown)
        B.ckv_paged_attend(po, q_out, c.k_pages, c.v_pages, c.table, grown, st, out, ws, lse=lse)
        lengths.copy_(grown)

    off = kept["offsets"].tolist()
    rows = [[[kept[x][u, off[u][g]:off[u][g] + bud[u][g]].double() for x in ("k_out", "v_out")] for g in range(Hkv)] for u in range(Nu)]
    graph = torch.cuda.CUDAGraph()
    step()                                          # warm-up on an empty cache; its rows are overwritten below
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    B.ckv_gather_pages(shape, params, pg, kd, vd, kept["indices"], kept["budgets"], kept["offsets"], c.table, c.k_pages, c.v_pages,
                       lengths, ws)
    for s in range(steps):
        new.copy_(torch.randn(new.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(50 + s)))
        npos.copy_((L + s * chunk + torch.arange(chunk, device="cuda", dtype=torch.int32)).repeat(Nu))
        graph.replay()
        rk = R.turn(nk, npos, inv, torch.ones(D, device="cuda")).to(dt)
        rq = R.turn(nq, npos, inv, torch.ones(D, device="cuda"))
        for u in range(Nu):
            for g in range(Hkv):
                kk, vv = rows[u][g]
                rows[u][g] = [torch.cat((kk, rk[u * chunk:(u + 1) * chunk, g].double())),
                              torch.cat((vv, nv[u * chunk:(u + 1) * chunk, g].double()))]
        want, want_lse = R.attend(rq.to(dt), [0, chunk, 2 * chunk], rows)
        # a key or query that rounds the other way moves a logit by 2 * 2^-8 * |q| |k| / sqrt(d) / sqrt(d) in the mean: 0.05 in bf16
        bf = dt == torch.bfloat16
        assert (out.double() - want).abs().max() <= (0.1 if bf else 1e-4)
        assert (out.double() - want).norm() <= (3 * 2.0 ** -8 if bf else 1e-5) * want.norm()
        assert (lse.double() - want_lse).abs().max() <= (0.02 if bf else 1e-4)
    assert grown.tolist() == [[x + steps * chunk for x in r] for r in bud]
    assert B.ckv_device_status(ws) == B.OK


def test_the_readme_s_step_of_a_decoder(B):
    """The example as it is printed, twice, on a batch of three sequences."""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        lines = f.read().split("A step of a decoder")[1].split("\n\n")[1].split("\n")
    assert lines and all(x.startswith("    ") for x in lines)
    H, Hkv, Nu = 8, 2, 3
    c = R.Cache([[40, 33], [7, 64], [100, 1]], 32, device="cuda", max_extra=1)
    qkv = torch.randn(Nu, H + 2 * Hkv, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    names = dict(k_pages=c.k_pages, v_pages=c.v_pages, page_table=c.table, q=q, k=k, v=v, inv_freq=inv, qw=torch.ones(D, device="cuda"),
                 kw=torch.ones(D, device="cuda"), positions=i32([500, 600, 700]), token_starts=i32([0, 1, 2, 3]), lengths=c.lengths,
                 new_lengths=torch.zeros_like(c.lengths), q_rot=torch.zeros(Nu, H, D, dtype=torch.bfloat16, device="cuda"),
                 out=torch.zeros(Nu, H, D, dtype=torch.bfloat16, device="cuda"), lse=torch.zeros(Nu, H, device="cuda"))
    for _ in range(2):
        exec("\n".join(x[4:] for x in lines), names)
    one = torch.ones(D, device="cuda")
    tk = R.turn(k, names["positions"], inv, one).bfloat16()
    rows = [[tuple(torch.cat((x.cuda(), y[u:u + 1, g])) for x, y in zip(c.rows[u][g], (tk, v))) for g in range(Hkv)] for u in range(Nu)]
    want, want_lse = R.attend(names["q_rot"], [0, 1, 2, 3], rows)
    assert B.ckv_device_status(names["ws"]) == B.OK
    assert torch.equal(names["new_lengths"], c.lengths + 1)
    # a key that rounds the other way moves a logit by 2^-8 |q| |k| / sqrt(d) at most
    assert (names["lse"].double() - want_lse).abs().max() <= 0.05
    assert (names["out"].double() - want).norm() <= 3 * 2.0 ** -8 * want.norm()


# ------------------------------------------------------------------------------------- at the ends of the documented ranges
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 40])
def test_attend_the_longest_cache(B, dtype, n):
    """2^24 rows of one head, the same eight pages over and over: the output is that of the pages taken once, the lse larger by the
    logarithm of how often they are taken."""
    P, pages = 64, 8
    c = R.Cache([[P * pages]], P, dtype=dtype, device="cuda", seed=1)
    reps = (1 << 24) // (P * pages)
    c.table = c.table.repeat(1, 1, reps)
    c.lengths = i32([[1 << 24]])
    q = torch.randn(n, 2, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype)
    out, lse = run_attend(B, c, q, [0, n], causal=False)
    want, want_lse = R.attend(q, [0, n], c.rows, causal=False)
    vmax = float(c.rows[0][0][1].double().abs().max())
    # a thread adds up no more than 2^24 / 148 / 16 rows in turn (tensor cores: a row's sum, 64 of them at a time)
    r = 132 * EPS * float(q.double().norm(dim=-1).max()) * float(c.rows[0][0][0].double().norm(dim=-1).max()) / math.sqrt(D) + 2.0 ** -20 + 7200 * EPS
    assert ((lse.double() - want_lse - math.log(reps)).abs() <= r + 2 * EPS * (want_lse.abs() + math.log(reps))).all()
    tol = 2 * r * vmax + (2.0 ** -8 * (vmax + want.abs()) if dtype == torch.bfloat16 else EPS * want.abs())
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_as_many_units_as_there_may_be(B, dtype):
    """65536 sequences of one head: a token appended and attended for each, up to 16 rows."""
    Nu, P, H = 65536, 16, 2
    g = torch.Generator(device="cuda").manual_seed(2)
    kp, vp = (torch.randn(Nu + 3, P, D, device="cuda", generator=g).to(dtype) for _ in range(2))
    table = torch.randperm(Nu + 3, device="cuda", generator=g)[:Nu].int().view(Nu, 1, 1).contiguous()
    lengths = torch.randint(0, P, (Nu, 1), device="cuda", generator=g, dtype=torch.int32)
    st = torch.arange(Nu + 1, device="cuda", dtype=torch.int32)
    q, k, v = (torch.randn(Nu, h, D, device="cuda", generator=g).to(dtype) for h in (H, 1, 1))
    pg = B.make_paged(kp, table, q=q, k_new=k, max_new=1)
    ws, grown, out, lse = B.alloc_paged_workspace(pg), torch.zeros_like(lengths), torch.zeros_like(q), torch.zeros(Nu, H, device="cuda")
    before = kp.clone()
    B.ckv_append(pg, None, k, v, None, st, lengths, table, kp, vp, ws, new_lengths=grown)
    B.ckv_paged_attend(pg, q, kp, vp, table, grown, st, out, ws, lse=lse)
    assert B.ckv_device_status(ws) == B.OK and torch.equal(grown, lengths + 1)
    at = table.view(Nu).long(), lengths.view(Nu).long()
    assert torch.equal(kp[at], k[:, 0]) and torch.equal(vp[at], v[:, 0])
    kp[at] = before[at]
    assert torch.equal(kp, before)
    kp[at] = k[:, 0]
    pages = table.view(Nu).long()
    x = torch.einsum("uhd,ujd->uhj", q.double(), kp[pages].double()) / math.sqrt(D)
    x = x.masked_fill((torch.arange(P, device="cuda")[None] > lengths)[:, None], -math.inf)
    want = torch.einsum("uhj,ujd->uhd", torch.softmax(x, -1), vp[pages].double())
    vmax = vp[pages].double().abs().amax((1, 2))[:, None, None]
    r = 132 * EPS * 20 * 20 / math.sqrt(D) + 2.0 ** -20 + 300 * EPS
    assert ((lse.double() - torch.logsumexp(x, -1)).abs() <= r + 2 * EPS * 8).all()
    assert ((out.double() - want).abs() <= 2 * r * vmax + (2.0 ** -8 * (vmax + want.abs()) if dtype == torch.bfloat16 else EPS * want.abs())).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 4, 30, 200])
def test_attend_queries_head_by_head(B, dtype, n):
    """q as a view of [H, T, d]."""
    c = R.Cache([[n + 300, n + 31]], 64, dtype=dtype, device="cuda", seed=n)
    q = torch.randn(8, n, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(dtype).transpose(0, 1)
    for max_new in (0, n):
        out, lse = run_attend(B, c, q, [0, n], max_new=max_new)
        check_attend(c, q, [0, n], out, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("counts,rows", [([1], 500), ([1], 20000), ([4], 900), ([40], 700), ([300], 2000), ([90], 20000)])
def test_attend_logits_of_any_size(B, dtype, counts, rows):
    """Logits of 1e11, where one step of fp32 is thousands: the largest takes the row, as it does in 64 bits."""
    n = counts[0]
    c = R.Cache([[n + rows, n + rows]], 32, dtype=dtype, device="cuda", seed=n, k_scale=1e5)
    q = (1e5 * torch.randn(n, 8, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n))).to(dtype)
    for causal in (True, False):
        out, lse = run_attend(B, c, q, [0, n], causal)
        bad = int((~torch.isfinite(out)).sum()), int((~torch.isfinite(lse)).sum())
        assert bad == (0, 0)
        for g in range(2):
            k, v = (x.cuda().double() for x in c.rows[0][g])
            x = torch.einsum("nhd,ld->nhl", q[:, 4 * g:4 * g + 4].double(), k) / math.sqrt(D)
            if causal:
                x = x.masked_fill((torch.arange(k.shape[0], device="cuda")[None] > rows + torch.arange(n, device="cuda")[:, None])[:, None], -math.inf)
            two = x.topk(2, -1)
            # a logit is off by at most 132 * 2^-24 |q| |k| / sqrt(d)
            off = 132 * EPS * float(q.double().norm(dim=-1).max()) * float(k.norm(dim=-1).max()) / math.sqrt(D)
            sure = two.values[..., 0] - two.values[..., 1] > 2 * off + 200
            assert sure.float().mean() > 0.9
            want = v[two.indices[..., 0]]
            got = out[:, 4 * g:4 * g + 4].double()
            assert ((got - want).abs() <= (2.0 ** -7 if dtype == torch.bfloat16 else 2 * EPS) * want.abs())[sure].all()
            assert ((lse[:, 4 * g:4 * g + 4].double() - two.values[..., 0]).abs() <= off + 4 * EPS * two.values[..., 0].abs() + 1)[sure].all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [7, 950])
def test_append_in_place_queries_behind_padding(B, dtype, T):
    """q_out == q in a fused projection, rows of no unit before the first unit and behind the last, an idle unit between."""
    H, Hkv, lead, pad = 10, 5, 2, 1
    a = (T - lead - pad) // 2
    starts = [lead, lead + a, lead + a, T - pad]
    c = R.Cache([[3, 0, 31, 32, 40], [1] * 5, [64, 9, 2, 0, 5]], 32, max_extra=T, dtype=dtype, device="cuda", poison=3.0)
    qkv = torch.randn(T, H + 2 * Hkv, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(T)).to(dtype)
    was = qkv.clone()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    pg = B.make_paged(c.k_pages, c.table, q=q, k_new=k)
    ws, new = B.alloc_paged_workspace(pg), torch.zeros_like(c.lengths)
    B.ckv_append(pg, B.make_rotary(inv), k, v, pos, i32(starts), c.lengths, c.table, c.k_pages, c.v_pages, ws, q=q, q_out=q, new_lengths=new)
    assert B.ckv_device_status(ws) == B.OK
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2 * EPS
    tq, tk = R.turn(was[:, :H], pos, inv), R.turn(was[:, H:H + Hkv], pos, inv)
    live = slice(lead, T - pad)
    assert ((q.double() - tq).abs() <= 80 * EPS * tq.abs().amax(-1, keepdim=True) + half * tq.abs())[live].all()
    assert torch.equal(qkv[:lead], was[:lead]) and torch.equal(qkv[T - pad:], was[T - pad:]) and torch.equal(qkv[:, H:], was[:, H:])
    for u in range(3):
        n = starts[u + 1] - starts[u]
        for g in range(Hkv):
            L = c.lens[u][g]
            assert int(new[u, g]) == L + n
            j = torch.arange(L, L + n, device="cuda")
            at = c.table[u, g, j // 32].long(), j % 32
            want = tk[starts[u]:starts[u + 1], g]
            assert ((c.k_pages[at].double() - want).abs() <= 80 * EPS * want.abs().amax(-1, keepdim=True) + half * want.abs()).all()
            assert torch.equal(c.v_pages[at], was[starts[u]:starts[u + 1], H + Hkv + g])


@pytest.mark.parametrize("kind", ["elastic", "all"])
def test_gather_pages_of_other_selections(B, kind):
    """The shared elastic selection, which may keep fewer rows than its share, and a budget that keeps everything."""
    from test_gpu_parity import params_of, problem_of
    cfg = gen.shrink(gen.CONFIGS["c2"], n_layers=2, batch=1, seq_len=900, budget_per_head=128, n_needles=4)
    b = gen.make_batch(cfg, "cuda")
    P = params_of(B, problem_of(cfg, 2))
    if kind == "elastic":
        P.shared_elastic = True
        b["sens"] = b["sens"] * 0 + 1e4                 # a threshold that leaves few candidates
    else:
        P.budget_per_head = 5000
    out = B.compress(b["q"], b["k"], b["v"], b["head_w"], b["sens"], P)
    shape, params = B.make_shape(b["q"], b["k"]), B.make_params(P, b["head_w"], b["sens"])
    bud, off = out["budgets"].tolist(), out["offsets"].tolist()
    assert (max(map(max, bud)) < 128) if kind == "elastic" else all(x == 900 for r in bud for x in r)
    c = R.Cache(bud, 16, dtype=b["k"].dtype, device="cuda", poison=9.0)
    for p in c.pools:
        p.fill_(9.0)
    pg = B.make_paged(c.k_pages, c.table, n_q_heads=cfg.n_q_heads)
    ws, lengths = B.alloc_paged_workspace(pg), torch.full_like(out["budgets"], -1)
    B.ckv_gather_pages(shape, params, pg, b["k"], b["v"], out["indices"], out["budgets"], out["offsets"], c.table, c.k_pages, c.v_pages,
                       lengths, ws)
    assert torch.equal(lengths, out["budgets"]) and B.ckv_device_status(ws) == B.OK
    for pool, src in zip((c.k_pages, c.v_pages), ("k_out", "v_out")):
        want = torch.full_like(pool, 9.0)
        for u in range(2):
            for g in range(cfg.n_kv_heads):
                j = torch.arange(bud[u][g], device="cuda")
                want[c.table[u, g, j // 16].long(), j % 16] = out[src][u, off[u][g]:off[u][g] + bud[u][g]]
        assert torch.equal(pool, want)
