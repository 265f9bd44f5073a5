"""Calls around the KV cache that are refused before anything is launched (no GPU needed)."""
import ctypes as C
import math

import pytest

OK, EINVAL, EUNSUPPORTED = 0, -1, -2


@pytest.fixture(scope="module")
def lib():
    from paper_2607_27692_b200 import build, retopk
    build.build()
    return retopk.load()


def config(**kw):
    from paper_2607_27692_b200 import paged
    p = dict(d=128, rot_dim=128, layout=0, scaling=0, base=10000.0, factor=1.0, original_len=0.0, low_freq_factor=0.0,
             high_freq_factor=0.0, beta_fast=0.0, beta_slow=0.0, attn_factor=0.0)
    p.update(kw)
    return paged._RopeConfig(**p)


def create(lib, **kw):
    h = C.c_void_p()
    rc = lib.retopk_rope_create(C.byref(h), C.byref(config(**kw)))
    assert (h.value is not None) == (rc == OK)
    return rc, h


@pytest.mark.parametrize("kw,want", [
    (dict(rot_dim=0), EINVAL), (dict(rot_dim=7), EINVAL), (dict(rot_dim=130), EINVAL), (dict(layout=2), EINVAL),
    (dict(scaling=5), EINVAL), (dict(scaling=-1), EINVAL), (dict(base=1.0), EINVAL), (dict(base=math.nan), EINVAL),
    (dict(base=math.inf), EINVAL), (dict(attn_factor=-1.0), EINVAL), (dict(scaling=1, factor=0.5), EINVAL),
    (dict(scaling=1, factor=math.nan), EINVAL), (dict(scaling=2, factor=2.0, rot_dim=2), EINVAL),
    (dict(scaling=3, factor=2.0), EINVAL), (dict(scaling=4, factor=2.0), EINVAL),
    (dict(scaling=3, factor=2.0, original_len=8192.0, low_freq_factor=4.0, high_freq_factor=4.0), EINVAL),
    (dict(scaling=4, factor=2.0, original_len=8192.0, beta_fast=1.0, beta_slow=2.0), EINVAL),
    (dict(d=96, rot_dim=96), EUNSUPPORTED), (dict(d=256, rot_dim=128), EUNSUPPORTED),
    (dict(), OK), (dict(rot_dim=2), OK), (dict(scaling=4, factor=2.0, original_len=4096.0), OK),
])
def test_rope_create(lib, kw, want):
    rc, h = create(lib, **kw)
    assert rc == want
    if rc == OK:
        assert lib.retopk_rope_destroy(h) == OK


def test_rope_null(lib):
    assert lib.retopk_rope_create(None, C.byref(config())) == EINVAL
    h = C.c_void_p()
    assert lib.retopk_rope_create(C.byref(h), None) == EINVAL and h.value is None
    assert lib.retopk_rope_destroy(None) == EINVAL
    assert lib.retopk_rope_frequencies(None, None, None) == EINVAL


@pytest.mark.parametrize("scaling,factor", [(None, 1.0), ("linear", 4.0), ("ntk", 4.0), ("llama3", 8.0), ("yarn", 4.0)])
@pytest.mark.parametrize("rot", [2, 10, 64, 128])
def test_frequencies(lib, scaling, factor, rot):
    from paper_2607_27692_b200 import paged
    import cache_reference as ref
    if scaling == "ntk" and rot == 2:
        pytest.skip("undefined for one pair")
    kw = {} if scaling is None else dict(scaling=scaling, factor=factor, original_len=8192)
    got, amp = paged.Rope(128, rot, base=500000.0, **kw).frequencies()
    want, want_amp = ref.frequencies(rot, 500000.0, scaling, factor, 8192)
    assert len(got) == rot // 2
    # a power, a logarithm and a few products in 64 bits
    for g, w in zip(got, want):
        assert abs(g - w) <= 2.0 ** -48 * w
    assert abs(amp - want_amp) <= 2.0 ** -50
    assert paged.Rope(128, rot, attn_factor=1.25).frequencies()[1] == 1.25


A = 1 << 20      # an aligned address that is never followed: every call below is refused (or has nothing to do)


def apply_args(**kw):
    p = dict(dtype=0, n=4, pos=A, q=A, qs=512, qo=A + (1 << 16), qos=512, Hq=4, k=None, ks=0, ko=None, kos=0, Hk=0, inv=0)
    p.update(kw)
    return [p[x] for x in ("dtype", "n", "pos", "q", "qs", "qo", "qos", "Hq", "k", "ks", "ko", "kos", "Hk", "inv")] + [None]


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(dtype=-1), dict(n=-1), dict(pos=None), dict(q=None), dict(q=A + 2), dict(qs=500), dict(qs=504),
    dict(qo=None), dict(qo=A + 8 + (1 << 16)), dict(qos=256), dict(Hq=0), dict(inv=2), dict(qo=A + 64), dict(qo=A, qos=1024),
    dict(k=A, ks=512, ko=None, kos=512, Hk=4), dict(k=A, ks=512, ko=A + 16, kos=512, Hk=4),
    # an output on the other tensor's input or output: all of it, part of each token, another stride
    dict(k=A + (1 << 16), ks=512, ko=A + (1 << 17), kos=512, Hk=4), dict(k=A + (1 << 17), ks=512, ko=A, kos=512, Hk=4),
    dict(k=A + (1 << 17), ks=512, ko=A + (1 << 16), kos=512, Hk=4),
    dict(qs=1024, qo=A, qos=1024, k=A + 512, ks=1024, ko=A + 512, kos=1024, Hk=2),
    dict(qs=1024, qo=A, qos=1024, k=A + 1024, ks=1536, ko=A + 1024, kos=1536, Hk=2),
    dict(qs=1024, qo=A, qos=1024, k=A + 1024 - 2048, ks=1024, ko=A + 1024 - 2048, kos=1024, Hk=5),
])
def test_rope_apply_refusals(lib, kw):
    rc, h = create(lib)
    assert lib.retopk_rope_apply(h, *apply_args(**kw)) == EINVAL
    lib.retopk_rope_destroy(h)


def test_rope_apply_nothing_to_do(lib):
    rc, h = create(lib)
    assert lib.retopk_rope_apply(None, *apply_args()) == EINVAL
    assert lib.retopk_rope_apply(h, *apply_args(n=0)) == OK
    lib.retopk_rope_destroy(h)


def pages(**kw):
    from paper_2607_27692_b200 import paged
    p = dict(format=2, H_kv=2, d=128, page_size=64, n_pages=8, k=A, v=A, k_scale=A, v_scale=A, block_table=A, max_pages=4)
    p.update(kw)
    return C.byref(paged._Pages(**p))


BAD_PAGES = [
    (dict(format=3), EINVAL), (dict(format=-1), EINVAL), (dict(H_kv=0), EINVAL), (dict(page_size=0), EINVAL),
    (dict(page_size=24), EINVAL), (dict(n_pages=0), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
    (dict(k=A + 8), EINVAL), (dict(v=A + 4), EINVAL), (dict(k_scale=None), EINVAL), (dict(v_scale=A + 4), EINVAL),
    (dict(max_pages=0), EINVAL), (dict(max_pages=1 << 26), EINVAL), (dict(d=96), EUNSUPPORTED),
    (dict(block_table=None, n_pages=2), EINVAL),
]


@pytest.mark.parametrize("kw,want", BAD_PAGES)
def test_bad_pages(lib, kw, want):
    B, lens = 3, A
    assert lib.retopk_kv_append(pages(**kw), B, lens, None, 3, 0, A, 256, A, 256, None, None, 0, None, 0, 0, None) == want
    assert lib.retopk_kv_gather(pages(**kw), B, lens, None, 5, 0, A, A, None) == want
    assert lib.retopk_q4_attention(pages(**kw), B, 1, 4, lens, 0, A, 512, 1.0, 0, A, None, A, 1 << 30, None) == want


def test_append_refusals(lib):
    rc, h = create(lib)
    rc, h64 = create(lib, d=64, rot_dim=64)

    def call(pg=None, B=3, lens=A, cu=None, n=3, dtype=0, k=A, ks=256, v=A, vs=256, rope=None, q=None, qs=0, qo=None, qos=0, Hq=0):
        return lib.retopk_kv_append(pages() if pg is None else pg, B, lens, cu, n, dtype, k, ks, v, vs, rope, q, qs, qo, qos, Hq, None)

    assert lib.retopk_kv_append(None, 3, A, None, 3, 0, A, 256, A, 256, None, None, 0, None, 0, 0, None) == EINVAL
    for kw in (dict(B=0), dict(lens=None), dict(n=-1), dict(n=4), dict(dtype=2), dict(k=None), dict(v=None), dict(k=A + 2),
               dict(ks=128), dict(vs=260), dict(rope=h64), dict(q=A, qs=512, qo=A, qos=512, Hq=4),
               dict(rope=h, q=A, qs=512, qo=None, qos=512, Hq=4), dict(rope=h, q=A, qs=512, qo=A + 64, qos=512, Hq=4),
               dict(rope=h, q=A, qs=512, qo=A, qos=512, Hq=0), dict(pg=pages(format=1)), dict(pg=pages(format=0), dtype=1)):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(k=A + 4096), dict(v=A + 4096), dict(k=A + 1024, ks=512), dict(v=A + 512, vs=512)):     # q_out on k_new, v_new
        assert call(**{**dict(rope=h, q=A, qs=512, qo=A, qos=512, Hq=4, n=30, B=30, k=A + (1 << 20), v=A + (1 << 20)), **kw}) == EINVAL, kw
    assert call(B=70000, n=70000) == EUNSUPPORTED
    assert call(rope=h, q=A, qs=70000 * 128, qo=A, qos=70000 * 128, Hq=70000) == EUNSUPPORTED
    assert call(n=0) == OK
    lib.retopk_rope_destroy(h)
    lib.retopk_rope_destroy(h64)


def test_gather_refusals(lib):
    def call(pg=None, B=3, lens=A, rows=5, dtype=0, k=A, v=A):
        return lib.retopk_kv_gather(pages() if pg is None else pg, B, lens, None, rows, dtype, k, v, None)

    for kw in (dict(B=0), dict(lens=None), dict(rows=-1), dict(dtype=3), dict(dtype=-1), dict(k=None, v=None), dict(k=A + 8),
               dict(v=A + 2), dict(pg=pages(format=0), dtype=1), dict(pg=pages(format=1), dtype=0)):
        assert call(**kw) == EINVAL, kw
    assert call(B=70000) == EUNSUPPORTED
    assert call(rows=0) == OK


def test_attention_refusals(lib):
    def call(pg=None, B=3, T=1, Hq=4, lens=A, dtype=0, q=A, qs=512, scale=1.0, window=0, out=A, ws=A, nb=1 << 30):
        return lib.retopk_q4_attention(pages() if pg is None else pg, B, T, Hq, lens, dtype, q, qs, scale, window, out, None, ws, nb, None)

    for kw in (dict(B=0), dict(T=0), dict(Hq=0), dict(Hq=3), dict(lens=None), dict(dtype=2), dict(q=None), dict(q=A + 2), dict(qs=256),
               dict(qs=514), dict(scale=math.nan), dict(scale=math.inf), dict(window=-1), dict(out=None), dict(ws=None), dict(ws=A + 4),
               dict(pg=pages(format=0))):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(T=17), dict(Hq=34, qs=34 * 128), dict(B=2049), dict(pg=pages(max_pages=16385))):
        assert call(**kw) == EUNSUPPORTED, kw
    for args, want in (((0, 1, 4, 2, 128), EINVAL), ((1, 1, 5, 2, 128), EINVAL), ((1, 1, 4, 2, 96), EUNSUPPORTED),
                       ((1, 17, 4, 2, 128), EUNSUPPORTED), ((1, 1, 34, 2, 128), EUNSUPPORTED), ((4097, 1, 1, 1, 64), EUNSUPPORTED)):
        assert lib.retopk_q4_attention_workspace(*args) == want


def test_binding_refuses_host_tensors():
    import torch
    from paper_2607_27692_b200 import paged
    rope = paged.Rope(64)
    x = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        rope.apply(x, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        paged.KVPages(2, 2, 16, 64, "q4", device="cpu")
    with pytest.raises(ValueError):
        paged.KVPages(2, 2, 16, 64, "int4", device="cpu")
    with pytest.raises(ValueError):
        paged.Rope(64, scaling="dynamic")
