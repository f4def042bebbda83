"""The calls on drafted trees and on the pages of a cache on the host: argument errors are reported before anything is launched, and
the binding compares every tensor with the layout its struct was made for.  No GPU needed: no call below passes validation."""
import ctypes as C

import pytest
import torch

from paper_2602_08686_b200 import binding as B
from paper_2602_08686_b200 import build as ckv_build


@pytest.fixture(scope="module", autouse=True)
def built():
    ckv_build.build_lib()


BIG = 1 << 40
far = lambda i: 256 * 1024 + i * (1 << 30)          # never dereferenced


def paged(**kw):
    base = dict(n_units=6, n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=B.BF16, n_tokens=10, max_new=5, causal=1, page_size=64,
                n_pages=100, max_pages=9, scale=0.0, q_stride_tok=48 * 128, q_stride_head=128, kv_stride_tok=48 * 128,
                kv_stride_head=128, page_stride=64 * 128, page_stride_row=128)
    base.update(kw)
    pg = B.ckv_paged()
    for k, v in base.items():
        setattr(pg, k, v)
    return pg


ORDER = {
    "masks": "n_units n_tokens words parents starts first masks positions ws ws_bytes stream",
    "attend": "pg q k_pages v_pages table lengths starts masks words out lse ws ws_bytes stream",
    "keep": "pg layers rows n_rows begins counts n_lists tails refs lengths table k_pages v_pages new_lengths ws ws_bytes stream",
    "reserve": "pg layers new_rows n_lists lengths held table refs k_pages v_pages room ws ws_bytes stream",
    "trim": "pg lengths held table refs ws ws_bytes stream",
    "fork": "pg layers n_new parents lengths held table refs keep_old new_lengths new_held new_table ws ws_bytes stream",
}
NAMES = {"masks": "ckv_tree_masks", "attend": "ckv_tree_attend", "keep": "ckv_keep_rows", "reserve": "ckv_pages_reserve", "trim": "ckv_pages_trim",
         "fork": "ckv_pages_fork"}
POINTERS = ("parents starts first masks positions ws q k_pages v_pages table lengths out lse rows begins counts tails refs new_lengths new_rows "
            "held room new_held new_table").split()
PLACE = {n: far(i + 1) for i, n in enumerate(POINTERS)}
PLAIN = dict(n_units=6, n_tokens=10, words=2, layers=2, n_rows=40, n_lists=3, n_new=4, keep_old=0, ws_bytes=BIG, stream=None)


def call(name, pg=None, **over):
    a = dict(PLAIN, **PLACE)
    a["pg"] = C.byref(paged() if pg is None else pg)
    a.update(over)
    return getattr(B.lib(), NAMES[name])(*[a[x] for x in ORDER[name].split()])


CACHES = ("attend", "keep", "reserve", "trim", "fork")
BAD = [(dict(n_units=0), B.ERR_INVALID_ARG), (dict(n_q_heads=30), B.ERR_INVALID_ARG), (dict(dtype=2), B.ERR_INVALID_ARG),
       (dict(head_dim=64), B.ERR_UNSUPPORTED), (dict(n_kv_heads=128, n_q_heads=128), B.ERR_UNSUPPORTED), (dict(n_units=8194), B.ERR_UNSUPPORTED),
       (dict(page_size=0), B.ERR_INVALID_ARG), (dict(page_size=48), B.ERR_UNSUPPORTED), (dict(n_pages=0), B.ERR_INVALID_ARG),
       (dict(max_pages=0), B.ERR_INVALID_ARG), (dict(max_pages=1 << 20), B.ERR_UNSUPPORTED), (dict(page_stride=64 * 128 - 8), B.ERR_INVALID_ARG),
       (dict(page_stride_row=120), B.ERR_INVALID_ARG), (dict(page_stride_row=130), B.ERR_INVALID_ARG)]


@pytest.mark.parametrize("change,want", BAD)
def test_bad_caches(change, want):
    pg = paged(**change)
    assert B.ckv_pages_workspace_bytes(pg) == 0
    for name in CACHES:
        assert call(name, pg) == want, name


def test_missing_and_misaligned_pointers():
    optional = {"masks": "first positions", "attend": "lse", "keep": "tails refs", "reserve": "room", "trim": "lengths", "fork": ""}
    for name, order in ORDER.items():
        for x in order.split():
            if x not in PLACE or x == "ws":
                continue
            if x not in optional[name].split():
                assert call(name, **{x: None}) == B.ERR_INVALID_ARG, (name, x)
            assert call(name, **{x: PLACE[x] + 2}) == B.ERR_INVALID_ARG, (name, x)
            if x in ("k_pages", "v_pages", "q"):
                assert call(name, **{x: PLACE[x] + 8}) == B.ERR_INVALID_ARG, (name, x)
    assert call("attend", out=PLACE["out"] + 16) == B.ERR_INVALID_ARG


def test_work_space():
    pg = paged()
    need = {"masks": 256, "attend": B.ckv_paged_workspace_bytes(pg), "keep": 256, "reserve": B.ckv_pages_workspace_bytes(pg), "trim": 256, "fork": 256}
    assert need["reserve"] > 256
    for name in ORDER:
        assert call(name, ws=None) == B.ERR_WORKSPACE, name
        assert call(name, ws=PLACE["ws"] + 16) == B.ERR_WORKSPACE, name
        assert call(name, ws_bytes=need[name] - 1) == B.ERR_WORKSPACE, name


def test_counts():
    for bad in (dict(n_units=0), dict(n_tokens=-1), dict(words=0), dict(words=-3)):
        assert call("masks", **bad) == B.ERR_INVALID_ARG, bad
    for bad in (dict(n_units=65537), dict(n_tokens=(1 << 20) + 1), dict(words=33)):
        assert call("masks", **bad) == B.ERR_UNSUPPORTED, bad
    assert call("attend", words=0) == B.ERR_INVALID_ARG
    assert call("attend", words=(1 << 15) + 1) == B.ERR_UNSUPPORTED
    for name in ("keep", "reserve", "fork"):
        for layers in (0, -1, 4, 12):                       # six units
            assert call(name, layers=layers) == B.ERR_INVALID_ARG, (name, layers)
    for name in ("keep", "reserve"):
        for n in (0, -1, 2, 6, 47, 49):                     # three sequences, 48 heads
            assert call(name, n_lists=n) == B.ERR_INVALID_ARG, (name, n)
    assert call("keep", n_rows=-1) == B.ERR_INVALID_ARG
    assert call("fork", n_new=-1) == B.ERR_INVALID_ARG
    assert call("fork", n_new=4097) == B.ERR_UNSUPPORTED   # 2 layers x 4097 x 8 heads
    for keep_old in (-1, 2):
        assert call("fork", keep_old=keep_old) == B.ERR_INVALID_ARG


def test_bad_query_strides():
    for change in (dict(q_stride_tok=4), dict(q_stride_head=0), dict(q_stride_tok=0), dict(q_stride_tok=-128)):
        assert call("attend", paged(**change)) == B.ERR_INVALID_ARG, change


def test_what_is_written_is_apart():
    """Every output, page pool, table that is written, and the work space, on the first and last bytes of everything else."""
    row, pg = 256, paged()
    size = dict(parents=40, starts=28, first=24, masks=80, positions=40, q=(9 * 48 + 31) * row + row, k_pages=100 * 64 * row, v_pages=100 * 64 * row,
                table=6 * 8 * 9 * 4, lengths=192, out=10 * 32 * row, lse=1280, rows=160, begins=12, counts=12, tails=12, refs=400, new_lengths=192,
                new_rows=12, held=192, room=8)
    new = dict(new_lengths=2 * 4 * 8 * 4, new_held=2 * 4 * 8 * 4, new_table=2 * 4 * 8 * 9 * 4, parents=16)
    written = {"masks": "masks positions ws", "attend": "out lse ws", "keep": "k_pages v_pages new_lengths ws", "reserve": "held table refs k_pages v_pages room ws",
               "trim": "held refs ws", "fork": "refs new_lengths new_held new_table ws"}
    step = dict(k_pages=16, v_pages=16, out=32, ws=256)
    ws = {"masks": 256, "attend": B.ckv_paged_workspace_bytes(pg), "keep": 256, "reserve": B.ckv_pages_workspace_bytes(pg), "trim": 256, "fork": 256}
    for name, order in ORDER.items():
        sizes = dict(size, ws=ws[name], **(new if name == "fork" else {}))
        arrays = [x for x in order.split() if x in PLACE]
        for o in written[name].split():
            for x in arrays:
                if x == o:
                    continue
                s = step.get(o, 4)
                last = (PLACE[x] + sizes[x] - 1) // s * s                  # begins on x's last bytes
                first = -(-(PLACE[x] + 1 - sizes[o]) // s) * s             # ends on its first
                for where in (first, last):
                    assert where < PLACE[x] + sizes[x] and where + sizes[o] > PLACE[x]
                    assert call(name, **{o: where}) == B.ERR_INVALID_ARG, (name, o, x)


def test_calls_without_tokens_are_empty():
    assert call("masks", n_tokens=0) == B.OK
    assert call("attend", paged(n_tokens=0)) == B.OK


def test_the_binding_names_what_does_not_fit():
    z = lambda *s: torch.zeros(*s, dtype=torch.int32)
    kp, vp = (torch.zeros(20, 16, 128, dtype=torch.bfloat16) for _ in range(2))
    table, q = z(4, 2, 5), torch.zeros(7, 4, 128, dtype=torch.bfloat16)
    pg = B.make_paged(kp, table, q=q)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    out, masks, lens = torch.zeros_like(q), z(7, 1), z(4, 2)
    fine = dict(
        attend=lambda **k: B.ckv_tree_attend(*[k.get(n, d) for n, d in dict(pg=pg, q=q, kp=kp, vp=vp, table=table, lengths=lens, starts=z(5), masks=masks, out=out, ws=ws).items()]),
        masks=lambda **k: B.ckv_tree_masks(k.get("parents", z(7)), k.get("starts", z(5)), k.get("masks", masks), k.get("ws", ws), positions=k.get("positions", z(7)),
                                           first_positions=k.get("first", z(4))),
        keep=lambda **k: B.ckv_keep_rows(pg, k.get("rows", z(9)), k.get("begins", z(4)), k.get("counts", z(4)), k.get("lengths", lens), k.get("table", table), k.get("kp", kp),
                                         k.get("vp", vp), k.get("new", z(4, 2)), k.get("ws", ws), tails=k.get("tails", z(4)), refs=k.get("refs", z(20))),
        reserve=lambda **k: B.ckv_pages_reserve(pg, k.get("more", z(4)), k.get("lengths", lens), k.get("held", z(4, 2)), k.get("table", table), k.get("refs", z(20)), k.get("kp", kp),
                                                k.get("vp", vp), k.get("ws", ws), room=k.get("room", z(2))),
        trim=lambda **k: B.ckv_pages_trim(pg, k.get("lengths", lens), k.get("held", z(4, 2)), k.get("table", table), k.get("refs", z(20)), k.get("ws", ws)),
        fork=lambda **k: B.ckv_pages_fork(pg, k.get("parents", z(3)), k.get("lengths", lens), k.get("held", z(4, 2)), k.get("table", table), k.get("refs", z(20)),
                                          k.get("new", z(3, 2)), k.get("new_held", z(3, 2)), k.get("new_table", z(3, 2, 5)), k.get("ws", ws)))
    for name, f in fine.items():
        with pytest.raises(ValueError, match="CUDA tensors"):               # all is as it should be, but for the device
            f()
    wrong = dict(attend=dict(q=q[:5], masks=z(6, 1), lengths=z(4, 3), starts=z(4), out=out.float(), table=z(4, 2, 6), kp=kp[:9], ws=ws.float()),
                 masks=dict(parents=z(8), starts=z(5).long(), masks=masks.long(), positions=z(6), first=z(5), ws=None),
                 keep=dict(rows=z(3, 3), begins=z(5), counts=z(3), tails=z(1), refs=z(19), new=z(2, 4), lengths=lens.long(), vp=vp.float()),
                 reserve=dict(more=z(4).float(), held=z(8), refs=z(21), room=z(3), table=table[:, :, :4], ws=None),
                 trim=dict(lengths=z(4), held=z(4, 3), refs=z(20).long(), table=None),
                 fork=dict(parents=z(3, 1), new=z(4, 2), new_held=z(3, 3), new_table=z(3, 2, 4), refs=None, held=z(4, 2).T))
    for name, cases in wrong.items():
        for key, value in cases.items():
            with pytest.raises(ValueError) as e:
                fine[name](**{key: value})
            assert "CUDA tensors" not in str(e.value), (name, key)
    with pytest.raises(ValueError, match="masks must be"):
        fine["attend"](masks=z(7))
    with pytest.raises(ValueError, match="made without pages"):
        B.ckv_pages_trim(B.make_packed(q, None, 4), None, z(4, 2), table, z(20), ws)


def test_marshalled_arguments():
    """What csrc/marshal.cpp hands over: integers of any width and null for None, by number of arguments; and what it refuses."""
    B.lib()
    m = B._m
    L = C.CDLL(None)
    fn = C.cast(L.abs, C.c_void_p).value
    assert m.call(fn, -7) == 7
    many = C.CFUNCTYPE(C.c_int, *[C.c_int64] * 18)(lambda *a: sum(i * x for i, x in enumerate(a)) % 1000003)
    at = C.cast(many, C.c_void_p).value
    args = [(1 << 40) + 3 * i if i % 2 else -i for i in range(18)]
    assert m.call(at, *args) == sum(i * x for i, x in enumerate(args)) % 1000003
    none = C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_int32)(lambda p, x: (p is None) * 100 + x)
    assert m.call(C.cast(none, C.c_void_p).value, None, -1) == 99
    with pytest.raises(TypeError):
        m.call(fn, 1.5)
    with pytest.raises(TypeError):
        m.call()
    t = torch.zeros(3, 4, dtype=torch.int32)
    for args in ((t, (3, 4), torch.int32, -1), (t, (3, 4), torch.int32, 0), (None, (3, 4), torch.int32, 0), (t, [3, 4], torch.int32, 0), (t,)):
        assert m.dense(*args) is None                                       # not a CUDA tensor, or not a tensor at all
    assert m.same(t, (t.shape, t.stride(), t.dtype, 0)) is None and m.same(t, None) is None
