"""Calls for caches that sequences share that are refused before anything is launched (no GPU needed)."""
import ctypes as C
import math

import pytest

from test_cache_refusals import A, BAD_PAGES, EINVAL, EUNSUPPORTED, OK, lib, pages  # noqa: F401


class Pool(C.Structure):
    _fields_ = [("refs", C.c_void_p), ("scratch", C.c_void_p), ("n_pages", C.c_int64), ("page_size", C.c_int)]


M = 1 << 20     # distance between arrays that are never followed


def pool(**kw):
    p = dict(refs=A, scratch=A + 8 * M, n_pages=100, page_size=16)
    p.update(kw)
    return C.byref(Pool(**p))


def half(**kw):
    """16-bit pages whose tensors lie apart."""
    return pages(**{**dict(format=0, k=A, v=A + 8 * M, k_scale=None, v_scale=None, block_table=A + 16 * M), **kw})


BAD_POOLS = [(dict(refs=None), EINVAL), (dict(scratch=None), EINVAL), (dict(n_pages=0), EINVAL), (dict(page_size=0), EINVAL),
             (dict(n_pages=(1 << 20) + 1, scratch=A + 64 * M), EUNSUPPORTED), (dict(scratch=A + 396), EINVAL)]


@pytest.mark.parametrize("kw,want", BAD_POOLS)
def test_bad_pools(lib, kw, want):  # noqa: F811
    L, T, X = A + 16 * M, A + 17 * M, A + 18 * M
    assert lib.retopk_pool_reserve(pool(**kw), 3, L, L, T, 5, None) == want
    assert lib.retopk_pool_fork(pool(**kw), 3, L, T, 5, 1, X, X, X + 64, X + 128, X + 192, None) == want
    assert lib.retopk_pool_free(pool(**kw), 3, L, T, 5, 3, None, None) == want
    assert lib.retopk_pool_compact(pool(**kw), 3, L, T, 5, X, X + 4096, None) == want


def test_pool_refusals(lib):  # noqa: F811
    L, T, X = A + 16 * M, A + 17 * M, A + 18 * M
    for B, lens, table, width, want in ((0, L, T, 5, EINVAL), (3, None, T, 5, EINVAL), (3, L, None, 5, EINVAL), (3, L, T, 0, EINVAL),
                                        (3, L, T, 1 << 28, EINVAL), (70000, L, T + 8 * M, 1, EUNSUPPORTED), (3, T, T, 5, EINVAL),
                                        (3, A, T, 5, EINVAL), (3, L, A + 8 * M, 5, EINVAL)):
        assert lib.retopk_pool_reserve(pool(), B, lens, L, table, width, None) == want
        assert lib.retopk_pool_free(pool(), B, lens, table, width, 1, X, None) == want
        assert lib.retopk_pool_compact(pool(), B, lens, table, width, X, X + 4096, None) == want
        assert lib.retopk_pool_fork(pool(), B, lens, table, width, 1, X, X + 16, X + 64, X + 128, X + 192, None) == want
    assert lib.retopk_pool_reserve(pool(), 3, L, None, T, 5, None) == EINVAL
    assert lib.retopk_pool_reserve(pool(), 3, L, T + 4, T, 5, None) == EINVAL

    def fork(n=2, p=X, c=X + 16, s=X + 64, d=X + 128, r=X + 192):
        return lib.retopk_pool_fork(pool(), 3, L, T, 5, n, p, c, s, d, r, None)

    for kw in (dict(n=-1), dict(p=None), dict(c=None), dict(s=None), dict(d=None), dict(r=None), dict(s=X), dict(d=X + 68), dict(r=X + 16), dict(s=L), dict(p=T)):
        assert fork(**kw) == EINVAL, kw
    assert fork(n=70000) == EUNSUPPORTED and fork(n=0) == OK
    assert lib.retopk_pool_free(pool(), 3, L, T, 5, 2, None, None) == EINVAL
    assert lib.retopk_pool_free(pool(), 3, L, T, 5, -1, X, None) == EINVAL
    assert lib.retopk_pool_free(pool(), 3, L, T, 5, 2, T, None) == EINVAL
    assert lib.retopk_pool_free(pool(), 3, L, T, 5, 0, X, None) == OK
    for s, d in ((None, X), (X, None), (X, X + 4), (T, X), (X, L)):
        assert lib.retopk_pool_compact(pool(), 3, L, T, 5, s, d, None) == EINVAL
    assert lib.retopk_pool_compact(pool(n_pages=1), 3, L, T, 5, None, None, None) == OK


@pytest.mark.parametrize("kw,want", [x for x in BAD_PAGES if "k_scale" not in x[0] and "v_scale" not in x[0] and x[0].get("page_size") != 24])
def test_bad_pages(lib, kw, want):  # noqa: F811
    X = A + 32 * M
    if "block_table" not in kw and "max_pages" not in kw:
        assert lib.retopk_pages_copy(half(**kw), 2, X, X + 64, None, None) == want
    assert lib.retopk_shared_attention(half(**kw), 3, 1, 4, X, 0, None, None, X, 512, 1.0, X + M, None, X + 2 * M, 1 << 30, None) == want
    assert lib.retopk_block_update(half(**kw), 16, X, 3, X, 5, None) == want
    assert lib.retopk_block_select(half(**kw), 16, X, 3, 1, 4, X, X, 512, 4, 1, 2, X + M, X + 2 * M, 1 << 30, None) == want
    assert lib.retopk_block_attention(half(**kw), 16, 3, 1, 4, X, 4, X, X, 512, 1.0, X + M, None, X + 2 * M, 1 << 30, None) == want


def test_copy_refusals(lib):  # noqa: F811
    X = A + 32 * M
    for args in ((-1, X, X, None), (2, None, X, None), (2, X, None, None), (2, A, X, None), (2, X, A + 64, None), (2, X, X, A + 8 * M)):
        assert lib.retopk_pages_copy(half(), *args, None) == EINVAL
    assert lib.retopk_pages_copy(half(v=A + 64), 2, X, X, None, None) == EINVAL
    assert lib.retopk_pages_copy(half(), 0, None, None, None, None) == OK
    assert lib.retopk_pages_copy(half(), (1 << 20) + 1, X, X, None, None) == EUNSUPPORTED
    assert lib.retopk_block_copy(half(), 64, X, 2, None, X, None) == EINVAL
    assert lib.retopk_block_copy(half(), 64, X, 2, X, A + 64 * M, None) == EINVAL
    assert lib.retopk_block_copy(half(), 24, X, 2, X + M, X + M, None) == EUNSUPPORTED
    assert lib.retopk_block_copy(half(), 128, X, 2, X + M, X + M, None) == EINVAL
    assert lib.retopk_block_copy(half(), 64, A + 64, 2, X + M, X + M, None) == EINVAL
    assert lib.retopk_block_copy(half(), 64, X, 0, None, None, None) == OK


def test_attention_refusals(lib):  # noqa: F811
    X = A + 32 * M

    def shared(pg=None, B=3, T=1, Hq=4, lens=X, n=0, cu=None, sh=None, q=X, qs=512, scale=1.0, out=X + M, lse=None, ws=X + 2 * M, nb=1 << 30):
        return lib.retopk_shared_attention(half() if pg is None else pg, B, T, Hq, lens, n, cu, sh, q, qs, scale, out, lse, ws, nb, None)

    def blocks(pg=None, B=3, T=1, Hq=4, lens=X, q=X, qs=512, scale=1.0, out=X + M, lse=None, ws=X + 2 * M, nb=1 << 30, block=16, keep=4, list=X):
        return lib.retopk_block_attention(half() if pg is None else pg, block, B, T, Hq, lens, keep, list, q, qs, scale, out, lse, ws, nb, None)

    for call in (shared, blocks):
        for kw in (dict(B=0), dict(T=0), dict(Hq=0), dict(Hq=3), dict(lens=None), dict(q=None), dict(q=X + 2), dict(qs=256), dict(qs=514),
                   dict(scale=math.nan), dict(scale=math.inf), dict(out=None), dict(ws=None), dict(ws=X + 2 * M + 4), dict(nb=0),
                   dict(pg=pages()), dict(out=X + 16), dict(out=A), dict(lse=X), dict(lse=X + M), dict(ws=X), dict(ws=X + M), dict(out=X + M + 8)):
            assert call(**kw) == EINVAL, kw
        for kw in (dict(T=17), dict(Hq=34, qs=34 * 128), dict(B=2049), dict(pg=half(max_pages=16385)),
                   dict(pg=half(n_pages=1 << 26, v=A + (1 << 44)))):
            assert call(**kw) == EUNSUPPORTED, kw
    for kw in (dict(n=-1), dict(n=4), dict(n=2), dict(n=2, cu=X), dict(n=2, sh=X)):
        assert shared(**kw) == EINVAL, kw
    for kw in (dict(keep=0), dict(list=None), dict(block=128), dict(list=X + M), dict(list=X + 2 * M)):
        assert blocks(**kw) == EINVAL, kw
    assert blocks(block=8) == EUNSUPPORTED
    assert lib.retopk_shared_attention_workspace(3, 4, 1, 4, 2, 128, 1000) == EINVAL
    assert lib.retopk_block_attention_workspace(3, 1, 4, 2, 96, 4, 16) == EUNSUPPORTED


def test_select_refusals(lib):  # noqa: F811
    X = A + 32 * M

    def call(pg=None, block=64, bounds=X + 4 * M, B=3, T=1, Hq=4, lens=X, q=X, qs=512, keep=4, first=1, last=2, out=X + M, ws=X + 2 * M, nb=M):
        return lib.retopk_block_select(half() if pg is None else pg, block, bounds, B, T, Hq, lens, q, qs, keep, first, last, out, ws, nb, None)

    for kw in (dict(B=0), dict(T=0), dict(Hq=3), dict(lens=None), dict(q=None), dict(q=X + 8), dict(qs=256), dict(keep=0), dict(first=-1), dict(last=0),
               dict(first=3), dict(out=None), dict(ws=None), dict(nb=8), dict(bounds=None), dict(bounds=X + 4 * M + 2), dict(bounds=A),
               dict(block=128), dict(pg=pages()), dict(out=X), dict(out=X + 2 * M), dict(ws=X), dict(ws=X + 4 * M), dict(last=2 ** 31 - 1, first=2 ** 31 - 1)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(block=48), dict(T=17), dict(Hq=34, qs=34 * 128), dict(B=2049), dict(pg=half(max_pages=16385))):
        assert call(**kw) == EUNSUPPORTED, kw
    assert lib.retopk_block_select_workspace(3, 1, 4, 2, 128, 0) == EINVAL
    assert lib.retopk_block_select_workspace(3, 1, 4, 2, 128, 1 << 21) == EUNSUPPORTED
    assert lib.retopk_block_update(half(), 16, X, 3, None, 5, None) == EINVAL
    assert lib.retopk_block_update(half(), 16, X, 3, X, -1, None) == EINVAL
    assert lib.retopk_block_update(half(), 16, X, 3, X, 0, None) == OK
