"""The paged-cache entry points on the host: argument errors are reported before anything is launched, the binding
compares every tensor with the layout its struct was made for.  No GPU needed: no call below passes validation."""
import ctypes as C
import subprocess

import pytest
import torch

import host_cuda
from paper_2602_08686_b200 import binding as B
from paper_2602_08686_b200 import build as ckv_build


@pytest.fixture(scope="module", autouse=True)
def built():
    ckv_build.build_lib()


FAKE = 256 * 1024          # never dereferenced
BIG = 1 << 40


def paged(**kw):
    base = dict(n_units=2, n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=B.BF16, n_tokens=10, max_new=5, causal=1,
                page_size=64, n_pages=100, max_pages=9, scale=0.0, q_stride_tok=48 * 128, q_stride_head=128,
                kv_stride_tok=48 * 128, kv_stride_head=128, page_stride=64 * 128, page_stride_row=128)
    base.update(kw)
    pg = B.ckv_paged()
    for k, v in base.items():
        setattr(pg, k, v)
    return pg


def rotary(**kw):
    base = dict(inv_freq=FAKE, q_norm_w=FAKE, k_norm_w=FAKE, rot_dim=128, interleaved=0, rot_scale=1.0, norm_eps=1e-6)
    base.update(kw)
    return B.ckv_rotary(*[base[k] for k, _ in B.ckv_rotary._fields_])


BAD_TOKENS = [(dict(n_units=0), B.ERR_INVALID_ARG), (dict(n_q_heads=30), B.ERR_INVALID_ARG), (dict(n_tokens=-1), B.ERR_INVALID_ARG),
              (dict(dtype=2), B.ERR_INVALID_ARG), (dict(head_dim=64), B.ERR_UNSUPPORTED), (dict(max_new=-1), B.ERR_INVALID_ARG),
              (dict(n_kv_heads=128, n_q_heads=128), B.ERR_UNSUPPORTED), (dict(n_tokens=(1 << 20) + 1), B.ERR_UNSUPPORTED),
              (dict(n_units=8193), B.ERR_UNSUPPORTED)]
BAD_PAGES = [(dict(page_size=0), B.ERR_INVALID_ARG), (dict(page_size=48), B.ERR_UNSUPPORTED), (dict(page_size=8), B.ERR_UNSUPPORTED),
             (dict(page_size=512), B.ERR_UNSUPPORTED), (dict(n_pages=0), B.ERR_INVALID_ARG), (dict(max_pages=0), B.ERR_INVALID_ARG),
             (dict(max_pages=1 << 20), B.ERR_UNSUPPORTED), (dict(page_stride=64 * 128 - 8), B.ERR_INVALID_ARG),
             (dict(page_stride_row=120), B.ERR_INVALID_ARG), (dict(page_stride_row=130), B.ERR_INVALID_ARG),
             (dict(causal=2), B.ERR_INVALID_ARG), (dict(scale=float("nan")), B.ERR_INVALID_ARG),
             (dict(scale=float("inf")), B.ERR_INVALID_ARG)]
BAD_Q = [(dict(q_stride_tok=4), B.ERR_INVALID_ARG), (dict(q_stride_head=0), B.ERR_INVALID_ARG), (dict(q_stride_tok=0), B.ERR_INVALID_ARG),
         (dict(q_stride_tok=-128), B.ERR_INVALID_ARG)]


def call(name, pg, rot=None, **over):
    L = B.lib()
    far = lambda i: FAKE + i * (1 << 30)
    a = dict(q=far(1), k=far(2), v=far(3), positions=far(4), starts=far(5), lengths=far(6), table=far(7), q_out=far(8),
             k_out=far(9), k_pages=far(10), v_pages=far(11), new_lengths=far(12), out=far(13), lse=far(14), ws=far(15), ws_bytes=BIG)
    a.update(over)
    p = C.byref(pg)
    r = None if rot is None else C.byref(rot)
    if name == "rotate":
        return L.ckv_rotate(p, r, a["q"], a["k"], a["positions"], a["starts"], a["q_out"], a["k_out"], None)
    if name == "append":
        return L.ckv_append(p, r, a["q"], a["k"], a["v"], a["positions"], a["starts"], a["lengths"], a["table"], a["q_out"],
                            a["k_pages"], a["v_pages"], a["new_lengths"], a["ws"], a["ws_bytes"], None)
    return L.ckv_paged_attend(p, a["q"], a["k_pages"], a["v_pages"], a["table"], a["lengths"], a["starts"], a["out"], a["lse"],
                              a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("change,want", BAD_TOKENS + BAD_PAGES)
def test_bad_shapes(change, want):
    pg = paged(**change)
    assert B.ckv_paged_workspace_bytes(pg) == 0
    assert call("append", pg, rotary()) == want
    assert call("attend", pg) == want
    if "page" not in str(change) and "causal" not in change and "scale" not in change:
        assert call("rotate", pg, rotary()) == want


@pytest.mark.parametrize("change,want", BAD_Q)
def test_bad_strides(change, want):
    for name in ("rotate", "append", "attend"):
        assert call(name, paged(**change), rotary()) == want, name
    kv = {k.replace("q_", "kv_"): v for k, v in change.items()}
    for name in ("rotate", "append"):
        assert call(name, paged(**kv), rotary()) == want, name


@pytest.mark.parametrize("change,want", [(dict(rot_dim=-16), B.ERR_INVALID_ARG), (dict(rot_dim=144), B.ERR_INVALID_ARG),
                                         (dict(rot_dim=24), B.ERR_UNSUPPORTED), (dict(interleaved=2), B.ERR_INVALID_ARG),
                                         (dict(inv_freq=None), B.ERR_INVALID_ARG), (dict(inv_freq=FAKE + 4), B.ERR_INVALID_ARG),
                                         (dict(norm_eps=-1.0), B.ERR_INVALID_ARG), (dict(norm_eps=float("nan")), B.ERR_INVALID_ARG),
                                         (dict(rot_scale=float("inf")), B.ERR_INVALID_ARG), (dict(q_norm_w=FAKE + 2), B.ERR_INVALID_ARG)])
def test_bad_rotary(change, want):
    assert call("rotate", paged(), rotary(**change)) == want
    assert call("append", paged(), rotary(**change)) == want


def test_bad_pointers_and_work_space():
    pg, rot = paged(), rotary()
    assert B.ckv_paged_workspace_bytes(pg) > 256
    assert call("rotate", pg, None) == B.ERR_INVALID_ARG
    for name, ptrs in (("rotate", "positions starts q_out k_out"), ("append", "k v positions starts lengths table q_out k_pages v_pages"),
                       ("attend", "q k_pages v_pages table lengths starts out")):
        for x in ptrs.split():
            assert call(name, pg, rot, **{x: None}) == B.ERR_INVALID_ARG, (name, x)
            assert call(name, pg, rot, **{x: FAKE + (1 << 34) + 2}) == B.ERR_INVALID_ARG, (name, x)
    assert call("rotate", pg, rot, q=None, k=None) == B.ERR_INVALID_ARG
    for name in ("append", "attend"):
        assert call(name, pg, rot, ws=None) == B.ERR_WORKSPACE
        assert call(name, pg, rot, ws=FAKE + (1 << 34) + 16) == B.ERR_WORKSPACE
        need = 256 if name == "append" else B.ckv_paged_workspace_bytes(pg)       # append only uses the status section
        assert call(name, pg, rot, ws_bytes=need - 1) == B.ERR_WORKSPACE
    assert call("append", pg, rot, k_pages=FAKE, v_pages=FAKE) == B.ERR_INVALID_ARG
    # outputs on top of inputs
    assert call("append", pg, rot, new_lengths=FAKE + 6 * (1 << 30)) == B.ERR_INVALID_ARG
    assert call("append", pg, rot, new_lengths=FAKE + 6 * (1 << 30) + 60) == B.ERR_INVALID_ARG
    assert call("attend", pg, out=FAKE + 1 * (1 << 30)) == B.ERR_INVALID_ARG
    assert call("attend", pg, out=FAKE + 10 * (1 << 30) + 64) == B.ERR_INVALID_ARG       # the pages
    assert call("attend", pg, out=FAKE + (1 << 36) + 16) == B.ERR_INVALID_ARG            # off its 32-byte boundary
    assert call("rotate", pg, rot, q_out=FAKE + 1 * (1 << 30) + 16) == B.ERR_INVALID_ARG
    assert call("rotate", pg, rot, q_out=FAKE + 2 * (1 << 30)) == B.ERR_INVALID_ARG      # the keys' input
    assert call("rotate", pg, rot, q_out=FAKE + 9 * (1 << 30) + 256) == B.ERR_INVALID_ARG  # the keys' output


def test_calls_without_tokens_are_empty():
    pg = paged(n_tokens=0)
    assert call("rotate", pg, rotary(), q=None, k=None, positions=None) == B.OK
    assert call("attend", pg, q=None, out=None) == B.OK
    assert call("append", pg, rotary(), q=None, k=None, v=None, positions=None, new_lengths=None) == B.OK


def test_gather_pages_refusals():
    s = B.ckv_shape(2, 32, 8, 128, 4096, 32, B.BF16, 0, 32 * 32 * 128, 32 * 128, 128, 8 * 4096 * 128, 4096 * 128, 128)
    p = B.make_params(B.Params(), None, None)
    far = [FAKE + i * (1 << 30) for i in range(20)]

    def go(pg, k=far[1], k_pages=far[6], lengths=far[8], ws_bytes=BIG, shape=s):
        return B.lib().ckv_gather_pages(C.byref(shape), C.byref(p), C.byref(pg), k, far[2], far[3], far[4], far[5], far[9], k_pages,
                                        far[7], lengths, far[10], ws_bytes, None)

    for change in (dict(n_units=3), dict(n_kv_heads=4), dict(dtype=B.F32)):
        assert go(paged(**change)) == B.ERR_INVALID_ARG, change
    assert go(paged(page_size=48)) == B.ERR_UNSUPPORTED
    assert go(paged(), k=None) == B.ERR_INVALID_ARG
    assert go(paged(), k_pages=far[6] + 8) == B.ERR_INVALID_ARG
    assert go(paged(), lengths=far[4]) == B.ERR_INVALID_ARG
    assert go(paged(), ws_bytes=16) == B.ERR_WORKSPACE
    bad = B.ckv_shape(2, 32, 8, 64, 4096, 32, B.BF16, 0, 32 * 32 * 128, 32 * 128, 128, 8 * 4096 * 128, 4096 * 128, 128)
    assert go(paged(), shape=bad) == B.ERR_INVALID_ARG


def test_the_binding_compares_layouts():
    kp = torch.zeros(6, 16, 128, dtype=torch.bfloat16)
    table = torch.zeros(1, 2, 3, dtype=torch.int32)
    qkv = torch.zeros(4, 12, 128, dtype=torch.bfloat16)
    q, k = qkv[:, :8], qkv[:, 8:10]
    pg = B.make_paged(kp, table, q=q, k_new=k, max_new=4)
    assert (pg.n_units, pg.n_q_heads, pg.n_kv_heads, pg.n_tokens, pg.max_pages, pg.page_size) == (1, 8, 2, 4, 3, 16)
    assert pg.q_stride_tok == 12 * 128 and pg.page_stride == 16 * 128
    starts, lengths = torch.zeros(2, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32)
    out, ws = torch.zeros(4, 8, 128, dtype=torch.bfloat16), torch.zeros(1 << 20, dtype=torch.uint8)

    def attend(**kw):
        a = dict(q=q, k_pages=kp, v_pages=kp.clone(), page_table=table, lengths=lengths, token_starts=starts, out=out, ws=ws)
        a.update(kw)
        B.ckv_paged_attend(pg, **a)

    for kw in (dict(q=q.contiguous()), dict(q=q.float()), dict(q=q[:3]), dict(v_pages=kp.transpose(0, 1)), dict(v_pages=kp.float()),
               dict(page_table=table.long()), dict(page_table=table[:, :1]), dict(lengths=lengths[0]),
               dict(token_starts=starts.long()), dict(token_starts=torch.zeros(3, dtype=torch.int32)), dict(out=out[:3]),
               dict(out=out.float()), dict(out=torch.zeros(4, 128, 8, dtype=torch.bfloat16).transpose(1, 2)),
               dict(lse=torch.zeros(4, 8, 1)), dict(ws=ws[::2]), dict(ws=ws.to(torch.int8))):
        with pytest.raises(ValueError):
            attend(**kw)
    with pytest.raises(ValueError):
        B.make_paged(kp, table.long(), q=q)
    with pytest.raises(ValueError):
        B.make_paged(kp.transpose(1, 2), table, q=q)
    with pytest.raises(ValueError):
        B.make_paged(kp, table, q=q.float())
    with pytest.raises(ValueError):
        B.make_rotary(torch.zeros(64))
    with pytest.raises(ValueError):
        B.make_rotary(torch.zeros(64, dtype=torch.float64), q_norm_w=torch.zeros(64))
    with pytest.raises(TypeError):
        B.make_packed(q.half(), k.half(), 1)


def test_the_binding_names_what_is_missing():
    """A struct that was made without pages, a token array without its output, or nothing at all: ValueError."""
    kp, table = torch.zeros(6, 16, 128), torch.zeros(1, 2, 3, dtype=torch.int32)
    x, k = torch.zeros(4, 8, 128), torch.zeros(4, 2, 128)
    ints = lambda *n: torch.zeros(*n, dtype=torch.int32)
    ws, rot = torch.zeros(1 << 16, dtype=torch.uint8), B.make_rotary(torch.zeros(64, dtype=torch.float64))
    full, tokens = B.make_paged(kp, table, q=x, k_new=k), B.make_packed(x, k, 1)
    append = lambda pg, **kw: B.ckv_append(pg, rot, **dict(dict(k=k, v=k.clone(), positions=ints(4), token_starts=ints(2), lengths=ints(1, 2),
                                                               page_table=table, k_pages=kp, v_pages=kp.clone(), ws=ws), **kw))
    for call_ in (lambda: B.ckv_rotate(full, rot, x, None, ints(4), ints(2), None, None),
                  lambda: B.ckv_rotate(full, rot, None, k, ints(4), ints(2), None, None),
                  lambda: B.ckv_rotate(full, rot, x, None, None, ints(2), x, None),
                  lambda: append(full, q=x), lambda: append(tokens), lambda: append(full, k=None), lambda: append(full, lengths=None),
                  lambda: append(full, v_pages=None),
                  lambda: append(full, ws=None),
                  lambda: B.ckv_paged_attend(tokens, x, kp, kp.clone(), table, ints(1, 2), ints(2), x.clone(), ws),
                  lambda: B.ckv_paged_attend(full, None, kp, kp.clone(), table, ints(1, 2), ints(2), x.clone(), ws),
                  lambda: B.ckv_paged_attend(full, x, kp, kp.clone(), table, ints(1, 2), ints(2), None, ws),
                  lambda: B.ckv_gather_pages(B.make_shape(torch.zeros(1, 8, 16, 128), torch.zeros(1, 2, 64, 128)),
                                             B.make_params(B.Params(), None, None), tokens, torch.zeros(1, 2, 64, 128),
                                             torch.zeros(1, 2, 64, 128), ints(1, 128), ints(1, 2), ints(1, 3), table, kp, kp.clone(),
                                             ints(1, 2), ws),
                  lambda: B.ckv_paged_workspace_bytes(tokens) or B.alloc_paged_workspace(tokens, "cpu")):
        with pytest.raises((ValueError, B.CkvError)):
            call_()


def test_outputs_and_pages_apart_from_inputs():
    pg, rot = paged(), rotary()
    far = lambda i: FAKE + i * (1 << 30)
    for x in ("q", "k", "v", "q_out"):
        for pool in (10, 11):
            assert call("append", pg, rot, **{x: far(pool) + 99 * 64 * 256}) == B.ERR_INVALID_ARG, (x, pool)   # the last page
    assert call("attend", pg, lse=far(13) + 10 * 32 * 256 - 4) == B.ERR_INVALID_ARG
    s = B.ckv_shape(2, 32, 8, 128, 4096, 32, B.BF16, 0, 32 * 32 * 128, 32 * 128, 128, 8 * 4096 * 128, 4096 * 128, 128)
    p = B.make_params(B.Params(), None, None)
    for k, v in ((far(6) - 256, far(2)), (far(1), far(7) + 99 * 64 * 256), (far(6) - 2 * 8 * 4096 * 256 + 256, far(2))):
        assert B.lib().ckv_gather_pages(C.byref(s), C.byref(p), C.byref(pg), k, v, far(3), far(4), far(5), far(9), far(6), far(7),
                                        far(8), far(10), BIG, None) == B.ERR_INVALID_ARG


def test_rows_written_in_place_are_apart():
    """A row that is two (token, head) pairs', or a query's and a key's, would be turned twice at once."""
    far = lambda i: FAKE + i * (1 << 30)
    rot = rotary()
    in_place = dict(rotate=dict(q_out=far(1), k_out=far(2)), append=dict(q_out=far(1)))
    for name, outs in in_place.items():
        for strides in (dict(q_stride_tok=128), dict(q_stride_tok=31 * 128), dict(q_stride_head=9 * 128, q_stride_tok=128),
                        dict(q_stride_head=256, q_stride_tok=384)):
            assert call(name, paged(**strides), rot, **outs) == B.ERR_INVALID_ARG, (name, strides)
    for strides in (dict(kv_stride_tok=128), dict(kv_stride_tok=7 * 128), dict(kv_stride_head=9 * 128, kv_stride_tok=128)):
        assert call("rotate", paged(**strides), rot, k_out=far(2)) == B.ERR_INVALID_ARG, strides
    # the keys (append: or the values) start inside the queries' rows, or are the queries
    for shift in (0, 256, 31 * 256, 48 * 256, -7 * 256, 3 * 48 * 256 + 64, -9 * 48 * 256):
        at = far(1) + shift
        assert call("rotate", paged(), rot, q_out=far(1), k=at) == B.ERR_INVALID_ARG, shift
        assert call("rotate", paged(), rot, k=at, k_out=at) == B.ERR_INVALID_ARG, shift
        assert call("append", paged(), rot, q_out=far(1), k=at) == B.ERR_INVALID_ARG, shift
        assert call("append", paged(), rot, q_out=far(1), v=at) == B.ERR_INVALID_ARG, shift
    pg = paged(kv_stride_tok=50 * 128)                 # other token strides over the same memory
    assert call("rotate", pg, rot, q_out=far(1), k=far(1) + 32 * 256) == B.ERR_INVALID_ARG


def test_the_two_pools_are_apart():
    """A page row that is both pools' would take a key and a value at once."""
    far = lambda i: FAKE + i * (1 << 30)
    s = B.ckv_shape(2, 32, 8, 128, 4096, 32, B.BF16, 0, 32 * 32 * 128, 32 * 128, 128, 8 * 4096 * 128, 4096 * 128, 128)
    p = B.make_params(B.Params(), None, None)

    def gather(pg, v_pages):
        return B.lib().ckv_gather_pages(C.byref(s), C.byref(p), C.byref(pg), far(1), far(2), far(3), far(4), far(5), far(9), far(10),
                                        v_pages, far(8), far(15), BIG, None)

    page = 64 * 256
    for layout, shifts in ((dict(), (0, 256, page, 99 * page, -page, 64, -99 * page - 16)),
                           (dict(page_stride=2 * 64 * 128), (256, page - 16, 2 * page, 2 * page - 256)),
                           (dict(page_stride=2 * 64 * 128, page_stride_row=256), (512, 16, 128, 2 * page + 512, -512)),
                           (dict(page_stride=64 * 136, page_stride_row=136), (16, 64 * 272, 272))):
        for shift in shifts:
            assert call("append", paged(**layout), rotary(), v_pages=far(10) + shift) == B.ERR_INVALID_ARG, (layout, shift)
            assert gather(paged(**layout), far(10) + shift) == B.ERR_INVALID_ARG, (layout, shift)


def test_outputs_apart_from_all_that_a_call_reads_and_writes():
    """Every output against every input and every other output: last byte on first byte, and the other way round."""
    far = lambda i: FAKE + i * (1 << 30)
    pg, rot = paged(), B.ckv_rotary(far(16), far(17), far(18), 128, 0, 1.0, 1e-6)
    at = dict(q=1, k=2, v=3, positions=4, starts=5, lengths=6, table=7, q_out=8, k_out=9, k_pages=10, v_pages=11, new_lengths=12, out=13,
              lse=14, ws=15)
    row, need = 256, B.ckv_paged_workspace_bytes(pg)
    size = dict(q=(9 * 48 + 32) * row, k=(9 * 48 + 8) * row, v=(9 * 48 + 8) * row, positions=40, starts=12, lengths=64, table=2 * 8 * 9 * 4,
                q_out=10 * 32 * row, k_out=10 * 8 * row, k_pages=100 * 64 * row, v_pages=100 * 64 * row, new_lengths=64, out=10 * 32 * row,
                lse=10 * 32 * 4, inv_freq=512, q_norm_w=512, k_norm_w=512)
    place = {n: far(i) for n, i in at.items()}
    place.update(inv_freq=far(16), q_norm_w=far(17), k_norm_w=far(18))
    turned = "inv_freq q_norm_w k_norm_w positions starts".split()
    calls = dict(rotate=("q_out k_out", "q k".split() + turned, 0),
                 append=("q_out k_pages v_pages new_lengths ws", "q k v lengths table".split() + turned, 256),
                 attend=("out lse ws", "q k_pages v_pages table lengths starts".split(), need))
    for name, (outs, ins, ws) in calls.items():
        outs = outs.split()
        size["ws"] = ws
        for o in outs:
            step = dict(ws=256, out=32, q_out=16, k_out=16, k_pages=16, v_pages=16).get(o, 4)
            for x in ins + [y for y in outs if y != o]:
                first = (place[x] + size[x] - 1) // step * step             # begins on x's last bytes
                last = -(-(place[x] + 1 - size[o]) // step) * step          # ends on its first
                for where in (first, last):
                    assert where < place[x] + size[x] and where + size[o] > place[x]
                    assert call(name, pg, rot, **{o: where}) == B.ERR_INVALID_ARG, (name, o, x)
    s = B.ckv_shape(2, 32, 8, 128, 4096, 32, B.BF16, 0, 32 * 32 * 128, 32 * 128, 128, 8 * 4096 * 128, 4096 * 128, 128)
    p = B.make_params(B.Params(), None, None)                              # 512 rows a head
    names = "k v indices budgets offsets table k_pages v_pages lengths ws".split()
    size = dict(k=2 * 8 * 4096 * row, v=2 * 8 * 4096 * row, indices=2 * 8 * 512 * 4, budgets=64, offsets=72, table=2 * 8 * 9 * 4,
                k_pages=100 * 64 * row, v_pages=100 * 64 * row, lengths=64, ws=256)
    place = {n: far(i + 1) for i, n in enumerate(names)}

    def gather(**over):
        a = dict(place, **over)
        return B.lib().ckv_gather_pages(C.byref(s), C.byref(p), C.byref(pg), *[a[n] for n in names], BIG, None)

    for o, step in dict(k_pages=16, v_pages=16, lengths=4, ws=256).items():
        for x in names:
            if x != o:
                for where in ((place[x] + size[x] - 1) // step * step, -(-(place[x] + 1 - size[o]) // step) * step):
                    assert gather(**{o: where}) == B.ERR_INVALID_ARG, (o, x)


APART = r"""
#include "host_cuda.h"
#include <random>
#include "paged_api.cu"
namespace ckv {
PagedWs paged_ws(const ckv_paged&) { return {}; }
cudaError_t launch_rotate(const ckv_paged&, const ckv_rotary*, const void*, const void*, const void*, const int32_t*, const int32_t*, void*, void*,
                          const int32_t*, const int32_t*, void*, void*, int32_t*, int*, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t launch_gather_pages(const ckv_shape&, const ckv_params&, const ckv_paged&, const void*, const void*, const int32_t*, const int32_t*,
                                const int32_t*, const int32_t*, void*, void*, int32_t*, int*, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t launch_paged_attend(const ckv_paged&, const void*, const void*, const void*, const int32_t*, const int32_t*, const int32_t*, void*,
                                float*, char*, cudaStream_t) { return cudaErrorUnknown; }
}
extern "C" size_t ckv_workspace_bytes(const ckv_shape*, const ckv_params*) { return 0; }
int main() {
  std::mt19937 rng(1);
  auto any = [&](int lo, int hi) { return (int64_t)(lo + rng() % (hi - lo + 1)); };
  int yes = 0, no = 0, careful = 0;
  for (int c = 0; c < 200000; ++c) {
    const int64_t esz = any(0, 1) ? 2 : 4, n = any(1, 5), outer = any(16, 16 * 14) * 8, q = 128;
    auto heads = [&] { return any(0, 2) ? q * any(1, 4) : any(16, 60) * 8; };
    const int64_t inner = heads();
    Rows a{(char*)0 + (1 << 20), n, outer, any(1, 5), inner, esz}, b{(char*)0 + (1 << 20) + 16 * any(-900, 900), n, outer, any(1, 5), inner, esz};
    if (any(0, 3) == 0) b.inner = heads();
    const bool alike = any(0, 9) != 0;
    if (!alike) b.outer = any(16, 16 * 14) * 8;
    auto at = [](const Rows& x, int64_t i, int64_t j) { return (int64_t)(intptr_t)x.base + (i * x.outer + j * x.inner) * x.esz; };
    bool meet = false, self = false;
    for (int64_t i = 0; i < a.n_outer; ++i)
      for (int64_t j = 0; j < a.n_inner; ++j) {
        for (int64_t k = 0; k < b.n_outer; ++k)
          for (int64_t l = 0; l < b.n_inner; ++l) meet |= llabs(at(a, i, j) - at(b, k, l)) < 128 * esz;
        for (int64_t k = 0; k < a.n_outer; ++k)
          for (int64_t l = 0; l < a.n_inner; ++l) self |= (i != k || j != l) && llabs(at(a, i, j) - at(a, k, l)) < 128 * esz;
      }
    const bool said = apart(a, b);
    if (said && meet) return printf("said apart\n"), 1;
    if (!said && !meet) {
      if (alike && outer >= 128) return printf("said not apart\n"), 1;
      ++careful;
    }
    if (a.apart_from_itself() && self) return printf("said apart from itself\n"), 1;
    said ? ++yes : ++no;
  }
  printf("%d apart, %d not, %d of them only to be careful\n", yes, no, careful);
  return yes < 10000 || no < 10000;
}
"""


def test_which_arrays_count_as_apart(tmp_path):
    """The host's check of overlapping rows against every row of small arrays."""
    p = subprocess.run([host_cuda.build(str(tmp_path), APART)], stdout=subprocess.PIPE)
    assert p.returncode == 0, p.stdout.decode()


@pytest.mark.parametrize("heads,kv_heads,tokens", [(65472, 64, 1 << 20), (65535, 1, 1 << 15), (2048, 8, (1 << 19) + 1)])
def test_more_query_rows_than_any_memory_holds(heads, kv_heads, tokens):
    """T * H above 2^30 (256 GB of bf16 rows): row indices are 32-bit."""
    pg = paged(n_units=1, n_q_heads=heads, n_kv_heads=kv_heads, n_tokens=tokens, q_stride_tok=heads * 128)
    assert B.ckv_paged_workspace_bytes(pg) == 0
    for name in ("rotate", "append", "attend"):
        assert call(name, pg, rotary()) == B.ERR_UNSUPPORTED
