"""Whose memory the calls around the KV cache read and write."""
import pytest
import torch

from test_gpu_cache_ops import BF, gen, ints

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
