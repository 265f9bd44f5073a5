"""How far the 4-bit attention may be from 64 bits where one part of its work could hide in another's rounding."""
import math

import pytest
import torch

import cache_reference as ref
from test_gpu_cache_ops import BF, FP, filled, gen, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def paged():
    from paper_2607_27692_b200 import build, paged
    build.build()
    return paged


def score_bound(q, k_scale, scale):
    """Scores of queries that enter exactly: 16 roundings of 2^-24 of values up to (15 step + |minimum|) * sum |q|."""
    ks, km = k_scale[..., 0].double().abs().max().item(), k_scale[..., 1].double().abs().max().item()
    return abs(scale) * 2.0 ** -20 * q.double().abs().sum(-1).max().item() * (15 * ks + km)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T", [(1, 1), (4, 1), (2, 2), (8, 1)])
def test_query_elements_far_below_the_largest(paged, dtype, d, G, T):
    """One channel of the query is a thousand times the others, and the keys hold nothing there: the others decide."""
    lens, page, big = [40, 700, 2049], 16, 5
    cache, table = filled(paged, lens, page, 1, d, 401, wild=False)
    cache.k_scale[..., 1] = 0.0
    cache.k[..., big // 2] &= 0x0f                  # code 0 in the odd channel 5
    q = 0.5 * torch.randn(len(lens), T, G, d, generator=gen(402), device="cuda")
    q[..., big] = 512.0
    q = q.to(dtype)
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, lse=lse)
    scale = d ** -0.5
    e = score_bound(q, cache.k_scale, scale)
    for b, n in enumerate(lens):
        k = ref.rows_of(cache.k, cache.k_scale, table, b, n, page)
        v = ref.rows_of(cache.v, cache.v_scale, table, b, n, page)
        assert (k[..., big] == 0).all()
        want, want_lse = ref.attention(q[b], k, v, scale)
        off = (lse[b].double() - want_lse).abs()
        # the sum of exponentials and its logarithm: a few fp32 steps of values about ln n, as for whole scores
        assert (off <= e + 2.0 ** -20 * (1 + math.log(n))).all(), f"lse off by {off.max().item()}, scores by {e} at most"
        assert ((out[b].double() - want).abs() <= ref.half_step(dtype) * (1 + 2.0 ** -10) * want.abs() + 2 * (e + 2.0 ** -15) * v.abs().max()).all()


@pytest.mark.parametrize("G,T", [(4, 1), (1, 3), (8, 2)])
def test_lengths_that_the_block_table_cannot_hold(paged, G, T):
    """They do not say which rows hold keys (cut off at the table they moved the tokens' causal limits): no key counts."""
    page, d, cap = 16, 64, 64
    cache, table = filled(paged, [cap] * 4, page, 2, d, 411, wild=False)
    q = torch.randn(4, T, 2 * G, d, generator=gen(412), device="cuda").to(BF)
    lse, fits = torch.empty(q.shape[:-1], device="cuda"), torch.empty(q.shape[:-1], device="cuda")
    want = cache.attend(q, ints([cap] * 4), table, lse=fits)
    out = cache.attend(q, ints([cap, cap + 1, 2 ** 31 - 1, -2 ** 31]), table, lse=lse)
    assert torch.equal(out[0], want[0]) and torch.equal(lse[0], fits[0]) and torch.isfinite(lse[0]).all()
    assert (out[1:] == 0).all() and (lse[1:] == -math.inf).all()


@pytest.mark.parametrize("T", [1, 16])
def test_windows_wider_than_any_sequence(paged, T):
    """Up to the largest 64-bit number, with sequences shorter than the tokens: as without a window."""
    lens, d = [0, 1, 5, T, 300], 64
    cache, table = filled(paged, lens, 16, 1, d, 421)
    q = torch.randn(len(lens), T, 2, d, generator=gen(422), device="cuda").to(BF)
    lse = torch.empty(q.shape[:-1], device="cuda")
    want = cache.attend(q, ints(lens), table, lse=lse)
    for window in (1 << 20, (1 << 20) + 1, (1 << 31) - 1, 1 << 31, 1 << 62, (1 << 63) - 1):
        got_lse = torch.empty_like(lse)
        assert torch.equal(cache.attend(q, ints(lens), table, window=window, lse=got_lse), want) and torch.equal(got_lse, lse)
