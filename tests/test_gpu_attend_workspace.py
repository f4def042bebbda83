"""GPU test of ckv_paged_attend in fp32 on the least work space that it takes, bytes around it looked over.  Tolerances as in tests/test_gpu_tree.py."""
import pytest
import torch

import paged_reference as R
from test_attend_workspace_host import of_rows
from test_gpu_tree import EPS, i32, r_of, starts_of

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("counts,lens,H,Hkv", [([1, 1], [[9000, 4000], [300, 7000]], 8, 2), ([9], [[8000]], 4, 1), ([200], [[1000, 1100]], 8, 2), ([1], [[400]], 4, 1)])
def test_least_work_space(counts, lens, H, Hkv):
    from paper_2602_08686_b200 import binding as B
    c = R.Cache(lens, 64, dtype=torch.float32, device="cuda", seed=len(lens))
    st = starts_of(counts)
    q = torch.randn(st[-1], H, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    pg = B.make_paged(c.k_pages, c.table, q=q, max_new=max(counts))
    n = of_rows(4)
    guard = torch.full((n + 512,), 0xAB, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 11.0), torch.zeros(st[-1], H, device="cuda")
    B.ckv_paged_attend(pg, q, c.k_pages, c.v_pages, c.table, c.lengths, i32(st), out, guard[256:256 + n], lse=lse)
    assert B.ckv_device_status(guard[256:256 + n]) == B.OK
    assert (guard[:256] == 0xAB).all() and (guard[256 + n:] == 0xAB).all()
    want, want_lse = R.attend(q, st, c.rows)
    vmax = max(float(v.double().abs().max()) for row in c.rows for _, v in row)
    r = r_of(q, torch.cat([k for row in c.rows for k, _ in row]), max(map(max, lens)))
    assert ((out.double() - want).abs() <= 2 * r * vmax + EPS * want.abs()).all()
    assert ((lse.double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs()).all()
