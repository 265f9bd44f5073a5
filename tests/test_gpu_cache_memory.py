"""Whose memory the calls around the KV cache read and write."""
import pytest
import torch

from test_gpu_cache_ops import BF, FP, filled, gen, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def paged():
    from paper_2607_27692_b200 import build, paged
    build.build()
    return paged


def calls_of(cache, d, H):
    x = torch.zeros(2, H, d, dtype=BF, device="cuda")
    lens, table = ints([1, 1]), ints([[0], [1]])
    rows = torch.zeros(2, H, 1, d, dtype=BF, device="cuda")
    calls = [lambda: cache.append(x, x, lens, table), lambda: cache.gather(rows, None, lens, table)]
    return calls + ([lambda: cache.attend(x, lens, table)] if cache.fmt == "q4" else [])


@pytest.mark.parametrize("fmt", ["q4", "bf16"])
def test_tensors_of_a_cache_that_change(paged, fmt):
    """A cache holds its tensors; one that gets other memory or another size is refused, not followed."""
    d, H, page = 64, 2, 16
    names = ["k", "v", "k_scale", "v_scale"] if fmt == "q4" else ["k", "v"]
    for name in names:
        def fresh():
            cache = paged.KVPages(2, H, page, d, fmt)
            return cache, getattr(cache, name)

        cache, t = fresh()
        with pytest.raises(AttributeError):
            setattr(cache, name, t.clone())
        for call in calls_of(cache, d, H):
            call()
        for change in (lambda t: t.set_(t.clone()), lambda t: t.resize_(4, *t.shape[1:]), lambda t: t.resize_(1, *t.shape[1:]),
                       lambda t: t.set_(torch.zeros(0, dtype=t.dtype, device="cuda")), lambda t: t.untyped_storage().resize_(0)):
            cache, t = fresh()
            change(t)
            for call in calls_of(cache, d, H):
                with pytest.raises(paged._rt.RetopkError, match="wrap"):
                    call()


def test_a_cache_keeps_its_tensors(paged):
    """Wrapped tensors that the caller lets go of stay the cache's."""
    d, H, page = 64, 1, 16
    k = torch.zeros(1, H, page, d, dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    cache = paged.KVPages.wrap(k, v)
    at = (k.data_ptr(), v.data_ptr())
    del k, v
    x = torch.randn(3, H, d, generator=gen(601), device="cuda").to(BF)
    junk = [torch.full((1, H, page, d), 7.0, dtype=BF, device="cuda") for _ in range(8)]
    cache.append(x, x, ints([3]))
    assert (cache.k.data_ptr(), cache.v.data_ptr()) == at and all((j == 7.0).all() for j in junk)
    assert torch.equal(cache.k[0, 0, :3], x[:, 0]) and torch.equal(cache.v[0, 0, :3], x[:, 0])


@pytest.mark.parametrize("G,T,d", [(1, 1, 64), (4, 1, 128), (8, 1, 64), (16, 1, 128), (4, 4, 64), (16, 16, 64)])
def test_attention_in_place(paged, G, T, d):
    """out = q: sequences that one CTA works on, that many share, and empty ones."""
    lens, page = [0, T, 100, 3000, 40000, 17], 16
    cache, table = filled(paged, lens, page, 2, d, 611)
    q = torch.randn(len(lens), T, 2 * G, d, generator=gen(612), device="cuda").to(FP)
    want = cache.attend(q, ints(lens), table)
    for _ in range(3):
        x = q.clone()
        assert cache.attend(x, ints(lens), table, out=x) is x
        assert torch.equal(x, want)


def test_outputs_on_inputs_are_refused(paged):
    """Through the binding: overlaps of outputs, pages and inputs that are views of one tensor; neighbours are fine."""
    d, H, page = 64, 2, 16
    error = paged._rt.RetopkError
    pool = torch.zeros(5, 2, H, page, d, dtype=BF, device="cuda")
    flat = pool.view(-1, H, d)
    cache = paged.KVPages.wrap(pool[0], pool[1])
    lens = ints([1, 1])
    with pytest.raises(error):
        cache.append(flat[1:3], flat[:2] + 1, lens)
    with pytest.raises(error):
        cache.append(flat[:2] + 1, flat[page + 1:page + 3], lens)
    with pytest.raises(error):
        cache.gather(pool[1], None, lens)
    with pytest.raises(error):
        cache.gather(pool[2], pool[2], lens)
    with pytest.raises(error):
        paged.KVPages.wrap(pool[0], pool[0]).append(flat[-2:], flat[-2:], lens)
    assert (pool == 0).all()
    x = torch.randn(2, H, d, generator=gen(621), device="cuda").to(BF)
    flat[4 * page:4 * page + 2] = x                          # pool[2] begins here
    cache.append(flat[4 * page:4 * page + 2], flat[4 * page:4 * page + 2], lens)
    cache.gather(pool[3], pool[4], lens)
    assert torch.equal(pool[0, :, :, 0], x) and torch.equal(pool[3, :, :, 0], x) and torch.equal(pool[4, :, :, 0], x)
    q4, table = filled(paged, [30, 30], page, H, d, 622)
    wide = torch.randn(5, 4, d, generator=gen(623), device="cuda").to(BF)
    for q, out in ((wide[:2], wide[1:3]), (wide[1:3], wide[:2]), (wide[:4:2], wide[1:3])):
        with pytest.raises(error):
            q4.attend(q, ints([30, 30]), table, out=out)
    want = q4.attend(wide[:2].clone(), ints([30, 30]), table)
    assert torch.equal(q4.attend(wide[:2], ints([30, 30]), table, out=wide[2:4]), want)


def test_in_place_operators_on_the_attributes(paged):
    """cache.k |= 1 assigns the same tensor: fine; another one is refused."""
    cache = paged.KVPages(1, 1, 16, 64, "q4")
    cache.k |= 0x11
    cache.v_scale += 1
    cache.k = cache.k
    assert (cache.k == 0x11).all() and (cache.v_scale == 1).all()
    with pytest.raises(AttributeError):
        cache.k = cache.k | 1
