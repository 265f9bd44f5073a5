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


def pattern(cache, table, lens, kind):
    """Key minima that make the scores flat, grow along the sequence, or fall."""
    for b, n in enumerate(lens):
        j = torch.arange(n, device="cuda")
        x = j.double() / n
        m = {"flat": 0 * x, "grow": 6 * x, "fall": 6 - 6 * x}[kind]
        cache.k_scale[table[b].long()[j // cache.page_size], :, j % cache.page_size, :, 1] = m.to(BF)[:, None, None]


def against_64_bits(cache, table, q, lens, scale, out, lse, bound):
    """bound(n, v, e): what an output may be off beyond its rounding, e: what a score may be."""
    e = score_bound(q, cache.k_scale, scale)
    for b, n in enumerate(lens):
        k = ref.rows_of(cache.k, cache.k_scale, table, b, n, cache.page_size)
        v = ref.rows_of(cache.v, cache.v_scale, table, b, n, cache.page_size)
        want, want_lse = ref.attention(q[b], k, v, scale)
        assert ((lse[b].double() - want_lse).abs() <= e + 2.0 ** -20 * (1 + math.log(n)) + 2.0 ** -23 * want_lse.abs()).all()
        over = (out[b].double() - want).abs() - (ref.half_step(q.dtype) * (1 + 2.0 ** -10) * want.abs() + bound(n, v, e))
        assert over.max().item() <= 0, f"sequence {b}: {over.max().item()} beyond the bound"


@pytest.mark.parametrize("kind", ["flat", "grow", "fall"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 8, 16])
@pytest.mark.parametrize("step,low", [(2.0 ** -57, 2.0 ** -54), (2.0 ** 54, 2.0 ** 35), (1.0, 2.0 ** 35), (0.0, 2.0 ** 35)])
def test_values_at_the_ends_of_their_range(paged, kind, d, G, step, low):
    """Steps of 2^-57..2^-56 and of 2^54..2^55, minima of up to 2^36: as exact, relative to them, as any."""
    lens, page = [40, 3000, 50000], 16
    cache, table = filled(paged, lens, page, 1, d, 431, wild=False)
    g = gen(432)
    top = 1 - 2.0 ** -8
    cache.v_scale[..., 0] = (step * (1 + top * torch.rand(cache.v_scale.shape[:-1], generator=g, device="cuda", dtype=torch.float64))).to(BF)
    cache.v_scale[..., 1] = (2 * top * low * (2 * torch.rand(cache.v_scale.shape[:-1], generator=g, device="cuda", dtype=torch.float64) - 1)).to(BF)
    pattern(cache, table, lens, kind)
    q = torch.full((len(lens), 1, G, d), 0.5, device="cuda") + 0.1 * torch.randn(len(lens), 1, G, d, generator=g, device="cuda")
    q = q.to(BF)
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, lse=lse)
    vs, vm = cache.v_scale[..., 0].double().max().item(), cache.v_scale[..., 1].double().abs().max().item()
    # as for any values (attention_bounds): weights off by e, their two parts by 2^-16, 24 sums cut off at
    # 2^-23 of at most 16 steps and rounded ones in between, sums of minima rounded to 2^-24 of them
    against_64_bits(cache, table, q, lens, d ** -0.5, out, lse,
                    lambda n, v, e: 2 * (e + 2.0 ** -16) * v.abs().max() + (n / 384 + 88) * 2.0 ** -23 * 16 * vs + (n / 32 + 64) * 2.0 ** -24 * vm)


@pytest.mark.parametrize("part,x", [(0, 2.0 ** 100), (1, 2.0 ** 126), (1, -2.0 ** 126)])
@pytest.mark.parametrize("G", [4, 16])
def test_values_beyond_their_range_are_not_hidden(paged, part, x, G):
    """A sum that leaves the fp32 range is NaN or infinite, not some finite number."""
    lens, d = [3000], 64
    cache, table = filled(paged, lens, 16, 1, d, 441, wild=False)
    pattern(cache, table, lens, "flat")
    cache.v_scale[..., part] = x
    cache.v |= 0x11                                  # no code is 0
    q = torch.randn(1, 1, G, d, generator=gen(442), device="cuda").to(BF)
    out = cache.attend(q, ints(lens), table)
    assert not torch.isfinite(out).any()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T", [(4, 1), (8, 1), (16, 1), (4, 4), (16, 4)])
def test_error_on_average(paged, d, G, T):
    """Root mean square errors, far below the worst case: a part of the weights or of the sums that went missing shows."""
    lens, page = [20, 100, 1003, 30000], 16
    cache, table = filled(paged, lens, page, 2, d, 451)
    q = torch.randn(len(lens), T, 2 * G, d, generator=gen(452), device="cuda").to(FP)
    out = cache.attend(q, ints(lens), table)
    e = score_bound(q, cache.k_scale.nan_to_num(), d ** -0.5)
    for b, n in enumerate(lens):
        k = ref.rows_of(cache.k, cache.k_scale, table, b, n, page)
        v = ref.rows_of(cache.v, cache.v_scale, table, b, n, page)
        want, _ = ref.attention(q[b], k, v, d ** -0.5)
        rms = (out[b].double() - want).square().mean().sqrt().item()
        # one rounding, uniform within half a step of numbers between powers of two; scores off by e move
        # the result by e times the spread of the values; the weights' second part leaves out 2^-16 of each;
        # 24 sums are cut off at 2^-23 of at most 16 steps, half of that on average (steps up to 0.41)
        size, spread = want.square().mean().sqrt().item(), v.std().item()
        limit = 2.0 ** -11 / math.sqrt(3) * 1.02 * size + e * spread + 2.0 ** -16 * v.square().mean().sqrt().item() + 24 * 2.0 ** -23 * 8 * 0.41
        assert rms <= limit, f"sequence {b}: rms {rms}, limit {limit}"


@pytest.mark.parametrize("d,G,T", [(64, 4, 1), (64, 8, 1), (64, 16, 1), (128, 16, 1), (128, 4, 4), (128, 8, 3)])
def test_long_flat_sums(paged, d, G, T):
    """A quarter of a million keys of much the same weight, in every layout of the columns: the little that large sums leave."""
    lens, page = [262144], 128
    cache, table = filled(paged, lens, page, 1, d, 461)
    q = (0.05 * torch.randn(1, T, G, d, generator=gen(462), device="cuda")).to(FP)
    out = cache.attend(q, ints(lens), table)
    k, v = (ref.rows_of(t, s, table, 0, lens[0], page) for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    want, _ = ref.attention(q[0], k, v, d ** -0.5)
    rms = (out[0].double() - want).square().mean().sqrt().item()
    # one rounding of the output; 12 tiles of one or two products, each sum cut off by at most 2^-23 of a
    # partial sum that grows to 16 steps (half on average); steps are 0.21 on average here
    sums = 12 if T * G <= 4 else 24
    assert rms <= ref.half_step(FP) * want.square().mean().sqrt().item() + sums * 2.0 ** -23 * 8 * 0.21
