"""Calls around the KV cache whose outputs overlap what they read or each other (no GPU needed: all are refused)."""
import ctypes as C

import pytest
import torch

EINVAL, EUNSUPPORTED = -1, -2
M = 1 << 20
# the pages' tensors a megabyte apart: 8 pages of 2 heads, 64 rows of 128 channels
K, V, KS, VS = (M * (16 + i) for i in range(4))
TABLE, LENS, FREE = M * 8, M * 9, M * 32
ROWS4, ROWS16 = 8 * 2 * 64 * 64, 8 * 2 * 64 * 256
SCALE = 8 * 2 * 64 * 8


@pytest.fixture(scope="module")
def lib():
    from paper_2607_27692_b200 import build, retopk
    build.build()
    return retopk.load()


@pytest.fixture(scope="module")
def rope(lib):
    from paper_2607_27692_b200 import paged
    h = C.c_void_p()
    assert lib.retopk_rope_create(C.byref(h), C.byref(paged._RopeConfig(128, 128, 0, 0, 10000.0, 1.0, 0, 0, 0, 0, 0, 0))) == 0
    yield h
    lib.retopk_rope_destroy(h)


def pages(fmt=2, **kw):
    from paper_2607_27692_b200 import paged
    q4 = fmt == 2
    p = dict(format=fmt, H_kv=2, d=128, page_size=64, n_pages=8, k=K, v=V, k_scale=KS if q4 else None, v_scale=VS if q4 else None,
             block_table=TABLE, max_pages=4)
    p.update(kw)
    return C.byref(paged._Pages(**p))


@pytest.mark.parametrize("kw", [
    # keys, values, queries and rotated queries that reach into the pages, from below and from above
    dict(k=K), dict(k=K - 16), dict(k=K + ROWS4 - 16), dict(v=V), dict(v=VS + SCALE - 16), dict(v=KS - 3 * 512 + 16),
    dict(q=K, qo=FREE), dict(qo=V), dict(qo=KS - 16), dict(qo=VS), dict(q=V + 1024, qo=V + 1024),
    dict(fmt=0, k=K + ROWS16 - 16), dict(fmt=0, qo=V + ROWS16 - 16), dict(fmt=0, v=K),
    # pages that share memory
    dict(pg=dict(v=K)), dict(pg=dict(v=K + ROWS4 - 16)), dict(pg=dict(k_scale=K)), dict(pg=dict(v_scale=KS)), dict(pg=dict(v_scale=KS + SCALE - 16)),
    dict(pg=dict(k_scale=V + 16)), dict(fmt=0, pg=dict(v=K)), dict(fmt=0, pg=dict(v=K + ROWS16 - 16)),
])
def test_append(lib, rope, kw):
    kw = dict(kw)
    fmt, pg = kw.pop("fmt", 2), kw.pop("pg", {})
    p = dict(k=FREE, v=FREE + M, q=FREE + 2 * M, qo=FREE + 3 * M)
    p.update(kw)
    n, H_q = 3, 4
    assert lib.retopk_kv_append(pages(fmt, **pg), 3, LENS, None, n, 0, p["k"], 256, p["v"], 256, rope, p["q"], 512, p["qo"], 512, H_q, None) == EINVAL


@pytest.mark.parametrize("dtype,fmt", [(0, 2), (1, 2), (2, 2), (0, 0), (2, 0)])
def test_gather(lib, dtype, fmt):
    out = 3 * 2 * 5 * 128 * (4 if dtype == 2 else 2)
    rows = ROWS4 if fmt == 2 else ROWS16

    def call(k, v, **pg):
        return lib.retopk_kv_gather(pages(fmt, **pg), 3, LENS, None, 5, dtype, k, v, None)

    for k, v in ((K, FREE), (K + rows - 16, FREE), (K - out + 16, FREE), (FREE, K), (FREE, V + 1024), (V - 16, None), (None, V),
                 (FREE, FREE), (FREE, FREE + out - 16), (FREE + 16, FREE)):
        assert call(k, v) == EINVAL, (hex(k or 0), hex(v or 0))
    if fmt == 2:
        for k, v in ((KS, None), (None, VS + SCALE - 16), (KS - out + 16, FREE)):
            assert call(k, v) == EINVAL


def test_attention(lib):
    B, T, H_q = 3, 2, 4
    size, lse, ws = B * T * H_q * 128 * 2, B * T * H_q * 4, 1 << 26
    base = dict(q=FREE, qs=512, out=FREE + M, lse=FREE + 2 * M, ws=M * 128)

    def call(**kw):
        p = {**base, **kw}
        return lib.retopk_q4_attention(pages(), B, T, H_q, LENS, 0, p["q"], p["qs"], 1.0, 0, p["out"], p["lse"], p["ws"], ws, None)

    for kw in (dict(out=FREE + 16), dict(out=FREE + size - 16), dict(out=FREE - size + 16), dict(qs=1024, out=FREE), dict(out=K), dict(out=VS),
               dict(lse=FREE), dict(lse=FREE + size - 16), dict(lse=FREE + M + size - 16), dict(lse=V + 16), dict(lse=KS - lse + 16),
               dict(ws=FREE), dict(ws=M), dict(ws=M * 16), dict(ws=FREE + 2 * M), dict(ws=FREE + M + 16), dict(lse=M * 128 + ws - 16)):
        assert call(**kw) == EINVAL, {k: hex(v) for k, v in kw.items()}
    # limits come first, as before
    assert lib.retopk_q4_attention(pages(max_pages=16385), B, T, H_q, LENS, 0, FREE, 512, 1.0, 0, FREE + 16, None, M * 128, ws, None) == EUNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where nothing can be launched")
def test_neighbours_are_not_overlaps(lib, rope):
    """The same calls with memory that touches end to end pass the checks (and find no device)."""
    ecuda = lib.retopk_kv_gather(pages(), 3, LENS, None, 5, 0, FREE, FREE + M, None)
    assert ecuda not in (0, EINVAL, EUNSUPPORTED)
    n, row = 3, 2 * 128 * 2
    assert lib.retopk_kv_append(pages(), 3, LENS, None, n, 0, K - n * row, 256, K + ROWS4, 256, rope, V - n * 2 * row, 512, V + ROWS4, 512, 4, None) == ecuda
    assert lib.retopk_kv_append(pages(v=K + ROWS4, k_scale=K - SCALE, v_scale=K - 2 * SCALE), 3, LENS, None, n, 0, FREE, 256, FREE, 256, None,
                                None, 0, None, 0, 0, None) == ecuda
    out = 3 * 2 * 5 * 128 * 2
    assert lib.retopk_kv_gather(pages(), 3, LENS, None, 5, 0, K - out, K + ROWS4, None) == ecuda
    assert lib.retopk_kv_gather(pages(), 3, LENS, None, 5, 0, FREE, FREE + out, None) == ecuda
    size, ws = 3 * 2 * 4 * 128 * 2, 1 << 26
    for q, qs, o, lse in ((FREE, 512, FREE, FREE + size), (FREE, 512, FREE + size, FREE + 2 * size), (FREE, 1024, FREE + 2 * size, None),
                          (FREE, 512, K - size, K + ROWS4)):
        assert lib.retopk_q4_attention(pages(), 3, 2, 4, LENS, 0, q, qs, 1.0, 0, o, lse, M * 128, ws, None) == ecuda
