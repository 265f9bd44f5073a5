"""Attention over long shared caches against 64 bits, with bounds that follow the weights: a wrong tile shows."""
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


# What the tensor core cuts off in all, of a sum of one sign, at 2^-23 for each product that it adds: 8192 in bf16, 1024 in fp16.
CUT = {BF: 2.0 ** -10, FP: 2.0 ** -13}


def exact(q, k, v, scale):
    """One KV head: q [rows, d], k, v [n, d] -> outputs, log-sum-exps and the bounds on both errors.

    Scores: products of 16-bit numbers are exact in fp32, d of them are added, each addition off by at most 2^-23 of
    sum |q| |k_j|, and three more operations at 2^-24 of that; the exponential and powers of two 2^-21: e_j.  Weights: off by 1 + e_j,
    half a step of the type in the product with the values only, and in fp16 2^-25 of the reference's weight, whose sum is at least
    that of exp(s_j - max).  Sums: CUT of sum p_j |v_j|, and 2^-20 where they are added in fp32 (up to 40 parts, 2^-24 each, next to
    sums of weights in 1024 steps whose errors have either sign).  The output is rounded once.
    """
    half = ref.half_step(q.dtype)
    kd, vd = k.double(), v.double()
    s = q.double() @ kd.t() * scale
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    p = p / total
    want = p @ vd
    e = abs(scale) * (q.shape[-1] + 3) * 2.0 ** -23 * (q.double().abs() @ kd.abs().t()) + 2.0 ** -21
    pe = p * e
    mean = pe.sum(-1, keepdim=True)
    size = p @ vd.abs()
    limit = half * want.abs() + (half + CUT[q.dtype] + 2.0 ** -20) * size + pe @ vd.abs() + (mean + 2.0 ** -20) * want.abs() + 2.0 ** -25
    if q.dtype == FP:
        limit += 2.0 ** -25 * vd.abs().sum(0) / total
    lse = (top + torch.log(total)).squeeze(-1)
    return want, limit, lse, mean.squeeze(-1) + 2.0 ** -20 + 2.0 ** -23 * lse.abs()


def pages_that_differ(sizes, shared, lens, page, H, d, dtype, seed=1):
    """Keys whose scores and values whose means differ from page to page; shared rows end with a page."""
    assert all(n % page == 0 for n in shared)
    k, v, table, cu, sh = sref.grouped_cache(sizes, shared, lens, page, H, d, dtype, seed)
    k[:, :, :, 0] = randn(seed + 50, k.shape[0], H, 1, dtype=dtype, scale=2.0)
    v += randn(seed + 51, v.shape[0], H, 1, d, dtype=dtype, scale=3.0)
    return k, v, table, cu, sh


def check(paged, sizes, shared, lens, page, G, H, d, T, dtype, seed=1, which=None, tokens=None):
    k, v, table, cu, sh = pages_that_differ(sizes, shared, lens, page, H, d, dtype, seed)
    cache = paged.KVPages.wrap(k, v)
    q = randn(seed + 5, len(lens), T, H * G, d, dtype=dtype)
    q[..., 0] = 8.0
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    out = cache.attend_shared(q, ints(lens), table, cu, sh, lse=lse)
    scale, told = d ** -0.5, 0
    for b in which if which is not None else range(len(lens)):
        rk, rv = (ref.rows_of(x, None, table, b, lens[b], page).to(dtype) for x in (k, v))
        for t in tokens if tokens is not None else range(T):
            seen = lens[b] - T + 1 + t
            for h in range(H):
                rows = q[b, t, h * G:(h + 1) * G]
                want, limit, want_lse, lse_limit = exact(rows, rk[h, :seen], rv[h, :seen], scale)
                err = (out[b, t, h * G:(h + 1) * G].double() - want).abs()
                assert bool((err <= limit).all()), (b, t, h, float((err / limit).max()))
                assert bool(((lse[b, t, h * G:(h + 1) * G].double() - want_lse).abs() <= lse_limit).all()), (b, t, h)
                # the bound tells: outputs of zero, and two tiles of values that have changed places
                assert bool((want.abs() > limit).any())
                if t == 0 and seen >= 1024:
                    tile = random.Random(told).randrange(seen // 128 - 4)
                    a, z = slice(tile * 128, tile * 128 + 128), slice((tile + 3) * 128, (tile + 3) * 128 + 128)
                    other = rv[h, :seen].clone()
                    other[a], other[z] = rv[h, z], rv[h, a]
                    p = torch.softmax(rows.double() @ rk[h, :seen].double().t() * scale, -1)
                    told += bool(((p @ other.double() - want).abs() > limit).any())
    return told


@pytest.mark.parametrize("dtype", [BF, FP])
def test_long_prefixes(paged, dtype):
    assert check(paged, [5, 1], [20032, 9024], [20043, 20600, 23000, 20033, 20500, 30001], 64, 4, 2, 128, 1, dtype) >= 6
    assert check(paged, [2], [70016], [70100, 70018], 64, 2, 1, 64, 2, dtype) >= 1


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64), (FP, 128)])
@pytest.mark.parametrize("members,G,T", [(1, 1, 1), (2, 4, 2), (8, 4, 1), (11, 3, 1), (17, 4, 1), (40, 4, 1), (3, 16, 4)])
def test_lines_in_many_parts(paged, dtype, d, members, G, T):
    """A line in every CTA's hands, copies of few rows that become one or do not, one and two streams' rows."""
    rng = random.Random(members)
    lens = [9024 + T + rng.randint(0, 300) for _ in range(members)]
    assert check(paged, [members], [9024], lens, 32, G, 1, d, T, dtype, which=sorted({0, members // 2, members - 1})) >= 1


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
@pytest.mark.parametrize("T,G", [(1, 4), (3, 1)])
def test_small_group_in_large_batch(paged, dtype, d, T, G):
    rng = random.Random(T)
    sizes, shared = [2, 66], [9008, 304]
    lens = [n + T + rng.randint(0, 200) for m, n in zip(sizes, shared) for _ in range(m)]
    assert check(paged, sizes, shared, lens, 16, G, 1, d, T, dtype, which=[0, 1, 2, 30, 67]) >= 1


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("members,T,G", [(3, 2, 2), (2, 1, 16), (70, 1, 4)])
def test_more_tiles_than_a_chunk(paged, dtype, members, T, G):
    lens = [132096 + T + 40 * i for i in range(members)] + [140001]
    check(paged, [members, 1], [132096, 0], lens, 128, G, 1, 64, T, dtype, which=[0, members - 1, members])


# ---------------------------------------------------------------------------------------
# Long lines in one CTA
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("d,G,T", [(64, 16, 16), (128, 16, 10), (64, 16, 8), (64, 16, 3)])
def test_sums_of_long_lines_in_fp16(paged, d, G, T):
    """Whole lines of 128K keys, values of one sign: what the tensor core cuts off has one sign too and stays far below half a step.

    At 2^-23 for each of the 1024 products that it adds before the sum is taken over, 2^-13 on average.  Beside that the
    error's mean over N outputs has roundings of the output, within 2^-11 and of either sign: 2^-11 / sqrt(3 N), of which six are
    allowed; roundings of weights are 2^-11 of a row's weights each, of either sign, and vanish among 10^5 keys.
    """
    B, H, n = 19, 8, 131072
    k, v = (torch.empty(B, H, n, d, device="cuda", dtype=FP) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    for b in range(B):
        k[b] = 0.3 * torch.randn(H, n, d, generator=g, device="cuda")
        v[b] = torch.rand(H, n, d, generator=g, device="cuda") + 0.5
    q = randn(3, B, T, H * G, d, dtype=FP)
    out = paged.KVPages.wrap(k, v).attend_shared(q, ints([n] * B))
    errors = []
    for b in range(0, B, 6):
        for h in (0, 3, 7):
            s = q[b, 0, h * G:(h + 1) * G].double() @ k[b, h, :n - T + 1].double().t() * d ** -0.5
            want = torch.softmax(s, -1) @ v[b, h, :n - T + 1].double()
            errors.append(((out[b, 0, h * G:(h + 1) * G].double() - want) / want).flatten())
    e = torch.cat(errors)
    assert abs(float(e.mean())) <= 2.0 ** -13 + 6 * 2.0 ** -11 / math.sqrt(3 * e.numel()), float(e.mean())


@pytest.mark.parametrize("B,H,n,d,G,T", [(75, 2, 20000, 64, 16, 16), (38, 4, 40000, 64, 16, 8), (20, 8, 36000, 128, 13, 16), (26, 1, 400000, 64, 16, 3)])
def test_pieces_that_follow_one_another(paged, B, H, n, d, G, T):
    """fp16 lines of which a CTA has more than its tensor core adds up at once: what one piece leaves, the next one adds to.  Of
    256, 128, 208 and 48 query rows; of the last ones copies, which become one."""
    rng = random.Random(B)
    lens = [n - rng.randint(0, 200) for _ in range(B)]
    check(paged, [1] * B, [0] * B, lens, 32, G, H, d, T, FP, which=[0, B // 3, B - 1], tokens=[0, T - 1])


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("G,T", [(16, 16), (16, 3)])
def test_long_lines_whose_scores_grow(paged, dtype, G, T):
    """References that grow from piece to piece, pages out of range for longer than a piece, NaN in the last key."""
    B, n, page, d = (150, 20480, 64, 64) if G * T > 128 else (24, 163840, 64, 64)
    k, v, table, _, _ = pages_that_differ([1] * B, [0] * B, [n] * B, page, 1, d, dtype)
    for b in range(B):
        k[table[b].long(), 0, :, 0] = torch.linspace(0, 24, n // page, device="cuda").unsqueeze(1).to(dtype)
    gone = slice(n // page // 8, n // page // 8 + (320 if G * T > 128 else 2400) // (page // 64))
    table[1::2, gone] = -1                                # 160 tiles of half the sequences; of few rows, 1200
    cache = paged.KVPages.wrap(k, v)
    q = randn(7, B, T, G, d, dtype=dtype)
    q[..., 0] = 4.0
    lens = ints([n] * B)
    out = cache.attend_shared(q, lens, table)
    for b in (0, 1, B - 2, B - 1):
        rows = torch.arange(n - T + 1, device="cuda")
        ids = table[b].long()[rows // page]
        rows, ids = rows[ids >= 0], ids[ids >= 0]
        want, limit, _, _ = exact(q[b, 0], k[ids, 0, rows % page], v[ids, 0, rows % page], d ** -0.5)
        err = (out[b, 0].double() - want).abs()
        assert bool((err <= limit).all()), (b, float((err / limit).max()))
    k[table[0, -1].long(), 0, 0, 5] = math.nan            # a key of the first sequence's last tile
    again = cache.attend_shared(q, lens, table)
    assert again[0].isnan().all() and torch.equal(again[1:], out[1:])
