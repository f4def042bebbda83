"""GPU tests of attention of drafted trees of more than a thousand tokens, whose rows fill many key tiles: values that are not finite reach
the tokens that see their row and no others, wherever in the tree the row is.  Tolerances as in tests/test_gpu_tree.py."""
import random

import numpy as np
import pytest
import torch

import paged_reference as R
import tree_reference as TR
from test_gpu_tree import EPS, i32, r_of, random_parents, run_attend, starts_of

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def B():
    from paper_2602_08686_b200 import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def sees_of(n, kind, rng):
    if kind == "tree":
        return TR.ancestors(random_parents(n, rng, 0.3, True))[0]
    return np.random.RandomState(rng.randint(0, 1 << 30)).rand(n, n) < 0.4


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("kind", ["tree", "bits"])
@pytest.mark.parametrize("H,Hkv,page,counts,base", [
    (8, 2, 32, [1024] * 10, 61),                     # nine key tiles a tree, whole items and shares of items
    (8, 2, 64, [1024] * 10, 0),                      # eight of them
    (8, 2, 16, [2100, 1500, 2100, 1100], 77),        # up to 18
    (16, 1, 128, [2100], 300),                       # shares of fifteen tiles
    (8, 2, 32, [600] * 15, 100)])                    # six
def test_values_that_are_not_finite_in_large_trees(B, H, Hkv, page, counts, base, kind, bad):
    """Every 97th token's value row has an element that is not finite, each in a dimension of its own: exactly the tokens that see
    the row have it there, and what is finite is right."""
    rng = random.Random(len(counts) + base)
    G, Nu = H // Hkv, len(counts)
    c = R.Cache([[base + n] * Hkv for n in counts], page, dtype=torch.bfloat16, device="cuda", seed=base)
    st = starts_of(counts)
    q = torch.randn(st[-1], H, D, generator=torch.Generator(device="cuda").manual_seed(base), device="cuda").bfloat16()
    sees = [sees_of(n, kind, rng) for n in counts]
    masks = TR.pack(sees, (max(counts) + 31) // 32, st[-1], st).cuda()
    clean = [[tuple(x.clone() for x in pair) for pair in row] for row in c.rows]
    hits = [list(range(5 + 3 * u, n, 97)) for u, n in enumerate(counts)]
    for u in range(Nu):
        for g in range(Hkv):
            for i, t in enumerate(hits[u]):
                j = base + t
                c.v_pages[int(c.table[u, g, j // page]), j % page, 5 * i + g] = bad
    out, lse = run_attend(B, c, q, st, masks, max_new=max(counts))
    want, want_lse = TR.attend(q, st, clean, sees)
    lost = 0
    for u in range(Nu):
        see = torch.from_numpy(sees[u]).cuda()
        for g in range(Hkv):
            mine, theirs = (x[st[u]:st[u + 1], g * G:(g + 1) * G] for x in (out, want))
            for i, t in enumerate(hits[u]):
                touched = see[:, t][:, None].expand(-1, G)
                lost += int((torch.isfinite(mine[:, :, 5 * i + g]) == touched).sum())
                mine[:, :, 5 * i + g][touched] = 0.0
                theirs[:, :, 5 * i + g][touched] = 0.0
    assert lost == 0, f"{lost} elements are finite where they should not be, or the other way round"
    vmax = max(float(v.double().abs().max()) for row in clean for _, v in row)
    r = r_of(q, torch.cat([k for row in clean for k, _ in row]), base + max(counts))
    off = (out.double() - want).abs() > 2.0 ** -8 * (vmax + want.abs()) + 2 * r * vmax
    assert not off.any(), f"{int(off.sum())} elements"
    assert ((lse.double() - want_lse).abs() <= r + 2 * EPS * want_lse.abs()).all()
