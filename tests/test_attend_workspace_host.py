"""How much work space the attention calls ask for.  No GPU needed: a call with enough of it is refused for a missing query."""
import pytest

from paper_2602_08686_b200 import binding as B
from test_paged_host import call, paged
import test_pages_refusals_host as trees
from paper_2602_08686_b200 import build as ckv_build


@pytest.fixture(scope="module", autouse=True)
def built():
    ckv_build.build_lib()


def up256(x):
    return -(-x // 256) * 256


def of_rows(rows):
    """148 CTAs, each with two slots of `rows` query rows: 128 numbers, a maximum and a sum each, beside what the CTA leaves in them."""
    return 256 + up256(148 * 16) + up256(148 * 2 * rows * 8) + up256(148 * 2 * rows * 128 * 4)


@pytest.mark.parametrize("tokens", [1, 10, 1000])
@pytest.mark.parametrize("max_pages", [9, 5000])
def test_fp32(tokens, max_pages):
    """Chunks are worked on in blocks of four query rows and need room for those; trees in up to 64."""
    pg = paged(dtype=B.F32, n_tokens=tokens, max_new=tokens, max_pages=max_pages)
    small, large = of_rows(4), of_rows(64)
    assert B.ckv_paged_workspace_bytes(pg) == large
    assert call("attend", pg, q=None, ws_bytes=small - 1) == B.ERR_WORKSPACE
    assert call("attend", pg, q=None, ws_bytes=small) == B.ERR_INVALID_ARG
    assert trees.call("attend", pg, q=None, ws_bytes=large - 1) == B.ERR_WORKSPACE
    assert trees.call("attend", pg, q=None, ws_bytes=large) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("tokens,rows", [(1, 32), (4, 32), (1000, 256)])
def test_bf16(tokens, rows):
    pg = paged(n_tokens=tokens, max_new=tokens)
    assert B.ckv_paged_workspace_bytes(pg) == of_rows(rows)
    for f in (call, trees.call):
        assert f("attend", pg, q=None, ws_bytes=of_rows(rows) - 1) == B.ERR_WORKSPACE
        assert f("attend", pg, q=None, ws_bytes=of_rows(rows)) == B.ERR_INVALID_ARG
