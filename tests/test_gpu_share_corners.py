"""Corners of the calls for caches that sequences share: many short sequences, lengths below the number of draft tokens, numbers
that are not finite, sizes at the stated limits, rows that shrink.  Against plain forms in 64 bits."""
import math
import random

import pytest
import torch

import cache_reference as ref
import share_reference as sref
from share_reference import ints

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def paged():
    from paper_2607_27692_b200 import build, paged
    build.build()
    return paged


def randn(seed, *shape, dtype=BF, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device="cuda")).to(dtype)


# ---------------------------------------------------------------------------------------
# Many short sequences to a CTA
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
@pytest.mark.parametrize("T,G", [(1, 4), (10, 8)])
def test_attend_many_lines_of_one_tile(paged, dtype, d, T, G):
    """A CTA's lines have one tile each, of which the second half of its warps has none, until one has two or three: that
    one's keys, of which a part counts, are told from the others'.  (Few rows, whole tiles; 80 rows, halves of tiles.)"""
    rng = random.Random(T)
    lens = [rng.randint(130, 380) if i % 11 == 10 else rng.randint(1, 127) for i in range(300)]
    k, v, table, _, _ = sref.grouped_cache([1] * 300, [0] * 300, lens, 16, 8, d, dtype)
    cache = paged.KVPages.wrap(k, v)
    q = randn(5, 300, T, 8 * G, d, dtype=dtype)
    want = cache.attend_shared(q, ints(lens), table)
    for b in [*range(10, 300, 11), *range(0, 300, 7)]:
        sref.check_attention(want[b:b + 1], None, q[b:b + 1], k, v, table[b:b + 1], lens[b:b + 1], 16, d ** -0.5, case=str(b))
    for _ in range(30):
        assert torch.equal(cache.attend_shared(q, ints(lens), table), want)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
@pytest.mark.parametrize("T,G", [(1, 4), (10, 8)])
def test_attend_many_lines_of_a_few_tiles(paged, dtype, d, T, G):
    """Lines of one to five tiles in any order: what one stream gives back of the ring while the other stream's product
    still reads the tile before it."""
    rng = random.Random(T + d)
    lens = [rng.randint(1, rng.choice([100, 128, 300, 640])) for _ in range(400)]
    k, v, table, _, _ = sref.grouped_cache([1] * 400, [0] * 400, lens, 16, 8, d, dtype)
    cache = paged.KVPages.wrap(k, v)
    q = randn(6, 400, T, 8 * G, d, dtype=dtype)
    want = cache.attend_shared(q, ints(lens), table)
    for b in range(0, 400, 5):
        sref.check_attention(want[b:b + 1], None, q[b:b + 1], k, v, table[b:b + 1], lens[b:b + 1], 16, d ** -0.5, case=str(b))
    for _ in range(30):
        assert torch.equal(cache.attend_shared(q, ints(lens), table), want)
