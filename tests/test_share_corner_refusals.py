"""Refusals of the calls for caches that sequences share, before anything is launched (no GPU needed): what is written overlaps
lengths, groups, lists or tables that are read."""
import pytest

from test_cache_refusals import A, EINVAL, OK, lib  # noqa: F401
from test_share_refusals import M, half

X = A + 32 * M
TABLE = A + 16 * M         # of half(): 3 rows of 5 pages or more


def table_bytes(pages):
    return 3 * pages._obj.max_pages * 4


@pytest.mark.parametrize("at", ["out", "lse", "ws"])
@pytest.mark.parametrize("what", ["lens", "table", "cu", "shared"])
def test_shared_attention_overlaps(lib, at, what):  # noqa: F811
    pages = half()
    a = dict(q=X, lens=X + M, cu=X + M + 64, shared=X + M + 128, out=X + 2 * M, lse=X + 3 * M, ws=X + 4 * M)
    read = TABLE if what == "table" else a[what]
    for shift in (0, -16, (table_bytes(pages) if what == "table" else 12 if what == "cu" else 8) - 8):
        b = dict(a)
        b[at] = (read + shift) & ~15
        rc = lib.retopk_shared_attention(pages, 3, 1, 4, b["lens"], 2, b["cu"], b["shared"], b["q"], 512, 1.0, b["out"], b["lse"], b["ws"], 1 << 20, None)
        assert rc == EINVAL, (at, what, shift)


@pytest.mark.parametrize("at", ["out", "lse", "ws"])
@pytest.mark.parametrize("what", ["lens", "table", "list"])
def test_block_attention_overlaps(lib, at, what):  # noqa: F811
    pages = half()
    a = dict(q=X, lens=X + M, list=X + M + 64, out=X + 2 * M, lse=X + 3 * M, ws=X + 4 * M)
    read = TABLE if what == "table" else a[what]
    a[at] = read & ~15
    assert lib.retopk_block_attention(pages, 16, 3, 1, 4, a["lens"], 4, a["list"], a["q"], 512, 1.0, a["out"], a["lse"], a["ws"], 1 << 20, None) == EINVAL


@pytest.mark.parametrize("at", ["out", "ws"])
@pytest.mark.parametrize("what", ["lens", "table"])
def test_select_overlaps(lib, at, what):  # noqa: F811
    pages = half()
    a = dict(q=X, lens=X + M, out=X + 2 * M, ws=X + 3 * M, bounds=X + 5 * M)
    a[at] = TABLE if what == "table" else a[what]
    rc = lib.retopk_block_select(pages, 64, a["bounds"], 3, 1, 4, a["lens"], a["q"], 512, 4, 1, 2, a["out"], a["ws"], M, None)
    assert rc == EINVAL


def test_update_overlaps(lib):  # noqa: F811
    assert lib.retopk_block_update(half(), 64, X, 3, X + 64, 5, None) == EINVAL
    assert lib.retopk_block_update(half(), 64, TABLE, 3, X, 5, None) == EINVAL
    assert lib.retopk_block_update(half(), 64, X, 3, X, 0, None) == OK


@pytest.mark.parametrize("scale", [3.0e38, -2.4e38, 3.4028234e38])
def test_scale_beyond_fp32(lib, scale):  # noqa: F811
    """As a power of two it would be infinite, and 0 times it no number."""
    args = (X, 512, scale, X + 2 * M, None, X + 4 * M, 1 << 20, None)
    assert lib.retopk_shared_attention(half(), 3, 1, 4, X + M, 0, None, None, *args) == EINVAL
    assert lib.retopk_block_attention(half(), 16, 3, 1, 4, X + M, 4, X + M + 64, *args) == EINVAL
