"""GPU test of a captured step that drafts trees where the pool has too few pages: the lines of the README, its guard among them."""
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def B():
    from paper_2602_08686_b200 import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def readme_lines():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        text = f.read().split("A step that drafts trees")[1]
    code = [[x[4:] for x in block.split("\n")] for block in text.split("\n\n") if block.startswith("    ")]
    step, guard = code[0], code[1]
    assert "ckv_pages_reserve" in step[1] and "ckv_pages_fork" in step[6] and "room" in guard[0]
    return step[:2], guard, step[2:6]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_step_without_pages_is_one_without_tokens(B, dtype):
    """A sequence of 20 rows goes on as three, on one and a half shared pages.  With pages for two of them the captured step leaves every
    row, count and length as it is, as often as it runs; with one page given back it runs as ever."""
    before, guard, after = readme_lines()
    P, H, Hkv, S, n, width, L = 16, 8, 1, 3, 6, 4, 20
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(5)
    n_pages = 2 + S + 1
    kp, vp = (torch.randn(n_pages, P, D, generator=gen, device="cuda").to(dtype) for _ in range(2))
    refs, table, held, lengths = z(n_pages), z(S, Hkv, width), z(S, Hkv), z(S, Hkv)
    # pages 3 and 5 are the prompt's, shared by all; page 0, which entries past `held` name, and page 1 are another batch's
    table[:, 0, :2] = i32([3, 5])
    held[:], lengths[:], refs[3], refs[5], refs[0], refs[1] = 2, L, S, S, 1, 1
    qkv = torch.randn(S * n, H + 2 * Hkv, D, generator=gen, device="cuda").to(dtype)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    starts, new, counts = i32([0, n, 2 * n, 3 * n]), i32([n] * S), i32([3, 1, 0])
    names = dict(ckv=B, k_pages=kp, v_pages=vp, q=q, k=k, v=v, q_rot=torch.zeros(S * n, H, D, dtype=dtype, device="cuda"),
                 out=torch.full((S * n, H, D), 11.0, device="cuda").to(dtype), lse=torch.zeros(S * n, H, device="cuda"), refs=refs, held=held, page_table=table,
                 lengths=lengths, longer=z(S, Hkv), room=z(2), parents=i32([-1, 0, 0, 1, 2, -1] * S), token_starts=starts, masks=z(S * n, 1),
                 positions=z(S * n), next_position=i32([L] * S), new=new, path=i32([0, 1, 3, 5]), begins=i32([0, 3, 0]), counts=counts,
                 rotary=B.make_rotary(10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)))
    pg = names["pg"] = B.make_paged(kp, table, q=q, k_new=k, max_new=n)
    names["pg_rot"] = B.make_paged(kp, table, q=names["q_rot"], max_new=n)
    names["ws"] = torch.zeros(max(B.ckv_paged_workspace_bytes(pg), B.ckv_pages_workspace_bytes(pg)), dtype=torch.uint8, device="cuda")
    inputs = [x.clone() for x in (starts, new, counts)]
    code = compile("\n".join(before + guard + after), "README.md", "exec")
    state = [x.clone() for x in (kp, vp, refs, held, table, lengths, names["out"])]
    now = lambda: (kp, vp, refs, held, table, lengths, names["out"])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        exec(code, names)                                                   # also the warm-up
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        exec(code, names)
    for _ in range(3):
        for x, y in zip((starts, new, counts), inputs):
            x.copy_(y)
        graph.replay()
        assert names["room"].tolist() == [2, 1] and B.ckv_device_status(names["ws"]) == B.OK
        for x, y in zip(now(), state):
            assert torch.equal(x, y)
    # the other batch gives a page back
    refs[1] = 0
    for x, y in zip((starts, new, counts), inputs):
        x.copy_(y)
    graph.replay()
    assert names["room"].tolist() == [0, 0] and B.ckv_device_status(names["ws"]) == B.OK
    assert lengths[:, 0].tolist() == [L + 3, L + 1, L] and held[:, 0].tolist() == [2, 2, 2]
    assert table[:, 0, :2].tolist() == [[3, 1], [3, 2], [3, 4]] and refs.tolist() == [1, 1, 1, 3, 1, 0]
    for pool, old in ((kp, state[0]), (vp, state[1])):
        assert torch.equal(pool[0], old[0]) and torch.equal(pool[3], old[3])
        for page in (1, 2, 4):
            assert torch.equal(pool[page, :L - P], old[5, :L - P])
    for s, kept in ((0, [0, 1, 3]), (1, [5])):
        assert torch.equal(vp[table[s, 0, 1].long(), L - P:L - P + len(kept)], v[s * n:(s + 1) * n][kept][:, 0])
    assert torch.isfinite(names["out"]).all() and not (names["out"] == 11.0).all(-1).any()
