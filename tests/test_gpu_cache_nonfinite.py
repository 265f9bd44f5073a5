"""NaN and infinities around the KV cache: where they must have no influence, and where they must not disappear."""
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


def put(cache, table, b, rows, name, part, x, group=None):
    """Step (part 0) or minimum (1) of rows of a sequence becomes x, in one group or in all."""
    j = torch.tensor(list(rows), device="cuda", dtype=torch.long)
    g = slice(None) if group is None else group
    getattr(cache, name)[table[b].long()[j // cache.page_size], :, j % cache.page_size, g, part] = x


WILD = [("v_scale", 0, math.nan), ("v_scale", 0, math.inf), ("v_scale", 1, math.nan), ("v_scale", 1, -math.inf),
        ("k_scale", 0, math.nan), ("k_scale", 1, math.inf)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T,window", [(4, 1, 20), (8, 1, 20), (16, 1, 33), (1, 3, 0), (4, 3, 0), (1, 4, 17), (5, 2, 100), (16, 16, 40)])
def test_rows_that_a_token_does_not_see(paged, d, G, T, window):
    """Before the window and in later draft tokens' rows anything may lie."""
    lens, page = [T, 50, 131, 1003, 2049], 16
    cache, table = filled(paged, lens, page, 2, d, 301)
    q = torch.randn(len(lens), T, 2 * G, d, generator=gen(302), device="cuda").to(BF)
    lse = torch.empty(q.shape[:-1], device="cuda")
    want = cache.attend(q, ints(lens), table, window=window, lse=lse)
    assert torch.isfinite(want.float()).all()
    start = {n: getattr(cache, n).clone() for n in ("k_scale", "v_scale")}
    for name, part, x in WILD:
        for n in start:
            getattr(cache, n).copy_(start[n])
        if window:
            for b, n in enumerate(lens):
                first = n - T + 1 - window          # of the first token's window
                put(cache, table, b, range(max(0, first - 40), max(0, first)), name, part, x)
            got_lse = torch.empty_like(lse)
            got = cache.attend(q, ints(lens), table, window=window, lse=got_lse)
            assert torch.equal(got, want) and torch.equal(got_lse, lse), f"{name}[{part}] = {x} before the window"
        for t in range(T - 1):                      # token t does not see rows from len - T + 1 + t on
            for n in start:
                getattr(cache, n).copy_(start[n])
            for b, n in enumerate(lens):
                put(cache, table, b, range(n - T + 1 + t, n), name, part, x)
            got_lse = torch.empty_like(lse)
            got = cache.attend(q, ints(lens), table, window=window, lse=got_lse)
            assert torch.equal(got[:, :t + 1], want[:, :t + 1]) and torch.equal(got_lse[:, :t + 1], lse[:, :t + 1]), \
                f"{name}[{part}] = {x} behind token {t}"


@pytest.mark.parametrize("d,group", [(64, 0), (128, 0), (128, 1)])
@pytest.mark.parametrize("G,T", [(1, 1), (4, 1), (8, 1), (4, 4), (16, 2)])
def test_values_that_are_seen(paged, d, group, G, T):
    """A live row's wild value step or minimum shows in its 64 channels, for every token that sees it; nowhere else."""
    lens, page = [T, 50, 1003, 3000], 16
    cache, table = filled(paged, lens, page, 2, d, 311)
    q = torch.randn(len(lens), T, 2 * G, d, generator=gen(312), device="cuda").to(FP)
    lse = torch.empty(q.shape[:-1], device="cuda")
    want = cache.attend(q, ints(lens), table, lse=lse)
    start = cache.v_scale.clone()
    for part, x in ((0, math.nan), (0, math.inf), (1, math.nan), (1, math.inf), (1, -math.inf)):
        for far in (0.0, 0.4, 1.0):                 # the first row, one in the middle, the last token's own
            cache.v_scale.copy_(start)
            rows = [int(far * (n - 1)) for n in lens]
            for b, r in enumerate(rows):
                put(cache, table, b, [r], "v_scale", part, x, group)
            got_lse = torch.empty_like(lse)
            got = cache.attend(q, ints(lens), table, lse=got_lse)
            assert torch.equal(got_lse, lse)
            other = [g for g in range(d // 64) if g != group]
            for b, (n, r) in enumerate(zip(lens, rows)):
                for t in range(T):
                    y, w = got[b, t].unflatten(-1, (-1, 64)), want[b, t].unflatten(-1, (-1, 64))
                    if r < n - T + 1 + t:
                        assert not torch.isfinite(y[:, group]).any(), f"sequence {b}, token {t}: row {r} is not to be seen"
                        assert torch.equal(y[:, other], w[:, other])
                    else:
                        assert torch.equal(y, w)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T", [(1, 1), (4, 1), (8, 1), (4, 4)])
def test_queries_that_are_not_finite(paged, dtype, d, G, T):
    """A row whose query holds NaN or an infinity is NaN, not the row of a sequence without keys; others are as before."""
    lens, page = [0, T, 50, 1003, 40000], 16
    cache, table = filled(paged, lens, page, 2, d, 321)
    q = torch.randn(len(lens), T, 2 * G, d, generator=gen(322), device="cuda").to(dtype)
    lse = torch.empty(q.shape[:-1], device="cuda")
    want = cache.attend(q, ints(lens), table, lse=lse)
    for x in (math.nan, math.inf, -math.inf):
        wild, got_lse = q.clone(), torch.empty_like(lse)
        wild[:, T - 1, G, 5] = x
        got = cache.attend(wild, ints(lens), table, lse=got_lse)
        hit = torch.zeros(lse.shape, dtype=torch.bool, device="cuda")
        hit[1:, T - 1, G] = True
        assert torch.isnan(got[hit]).all() and torch.isnan(got_lse[hit]).all()
        assert torch.equal(got[~hit], want[~hit]) and torch.equal(got_lse[~hit], lse[~hit])
        assert (got[0] == 0).all() and (got_lse[0] == -math.inf).all()


@pytest.mark.parametrize("d,group", [(64, 0), (128, 1)])
@pytest.mark.parametrize("G,T", [(1, 1), (4, 1), (8, 1), (4, 4)])
def test_keys_that_are_not_finite(paged, d, group, G, T):
    """One live key without a finite step or minimum: every row that sees it is NaN; an infinite score is never a masked one."""
    lens, page, H = [T, 50, 1003, 40000], 16, 2
    cache, table = filled(paged, lens, page, H, d, 331)
    q = torch.randn(len(lens), T, H * G, d, generator=gen(332), device="cuda").to(BF)
    lse = torch.empty(q.shape[:-1], device="cuda")
    want = cache.attend(q, ints(lens), table, lse=lse)
    start = cache.k_scale.clone()
    for part, x in ((0, math.nan), (0, math.inf), (0, -math.inf), (1, math.nan), (1, math.inf), (1, -math.inf)):
        for far in (0.0, 0.4, 1.0):
            cache.k_scale.copy_(start)
            rows = [int(far * (n - 1)) for n in lens]
            for b, r in enumerate(rows):
                put(cache, table, b, [r], "k_scale", part, x, group)
            got_lse = torch.empty_like(lse)
            got = cache.attend(q, ints(lens), table, lse=got_lse)
            for b, (n, r) in enumerate(zip(lens, rows)):
                for t in range(T):
                    if r < n - T + 1 + t:
                        assert torch.isnan(got[b, t]).all() and torch.isnan(got_lse[b, t]).all()
                    else:
                        assert torch.equal(got[b, t], want[b, t]) and torch.equal(got_lse[b, t], lse[b, t])


@pytest.mark.parametrize("G", [4, 8])
@pytest.mark.parametrize("low", [-1.0e38, -2.2e38, 2.2e38])
def test_scores_near_the_end_of_the_range(paged, G, low):
    """One key with a score near the largest fp32 number: it has all the weight, whatever its sign."""
    d = 64
    cache, table = filled(paged, [1], 16, 1, d, 341, wild=False)
    row = (table[0, 0].item(), 0, 0)
    cache.k_scale[row][:, 0] = 0.0
    cache.k_scale[row][:, 1] = 1.0e36
    q = torch.full((1, G, d), -1.0, device="cuda").to(BF)
    scale = -low / (64 * cache.k_scale[row][0, 1].item())
    lse = torch.empty(1, G, device="cuda")
    out = cache.attend(q, ints([1]), table, scale=scale, lse=lse)
    n = torch.stack((cache.v[row] & 15, cache.v[row] >> 4), -1).flatten().double()
    want = n * cache.v_scale[row][0, 0].double() + cache.v_scale[row][0, 1].double()
    # the weight is 1 and its two parts are exact; one product and sum in fp32, and the rounding to bf16
    assert ((out[0].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs() + 2.0 ** -20).all()
    assert ((lse.double() - low).abs() <= 2.0 ** -20 * abs(low)).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
def test_groups_that_hold_no_finite_numbers(paged, dtype, d):
    """NaN and infinities in keys and values of a 4-bit cache: their 64 channels read back as NaN, all others as ever."""
    n, H, page = 45, 2, 16
    x = torch.randn(n, H, d, generator=gen(351), device="cuda").to(dtype)
    hit = torch.zeros(n, H, d // 64, dtype=torch.bool, device="cuda")
    row = 0
    for at in (0, 7, 8, 31, 32, 63):                # channels in different lanes and chunks
        for v in (math.nan, math.inf, -math.inf):
            for g in range(d // 64):
                x[row % n, row // n, 64 * g + at] = v
                hit[row % n, row // n, g] = True
                row += 1
    for v in (math.nan, math.inf, -math.inf):       # a whole group, and both infinities in one
        x[row % n, row // n, d - 64:] = v
        hit[row % n, row // n, -1] = True
        row += 1
    x[row % n, row // n, :2] = torch.tensor([math.inf, -math.inf])
    hit[row % n, row // n, 0] = True
    if dtype == BF:                                 # a span that fp32 does not hold
        x[row % n, row // n + 1, :2] = torch.tensor([3.0e38, -3.0e38])
        hit[row % n, row // n + 1, 0] = True
    assert row < 2 * n - 45 and not hit.all()
    codes, step, low = ref.quantise(torch.where(hit.repeat_interleave(64, -1), 0, x))
    table = ints([[2, 0, 1]])
    cache = paged.KVPages(3, H, page, d, "q4")
    cache.append(x, x.flip(0).contiguous(), ints([n]), table)
    want = ref.values(ref.pack(codes), torch.stack((step, low), -1)).unflatten(-1, (-1, 64))
    for out in (torch.float32, BF, FP):
        k, v = (torch.zeros(1, H, n, d, dtype=out, device="cuda") for _ in "kv")
        cache.gather(k, v, ints([n]), table)
        for got, w, h in ((k, want, hit), (v, want.flip(0), hit.flip(0))):
            got = got[0].transpose(0, 1).unflatten(-1, (-1, 64))
            assert torch.isnan(got[h]).all()
            tol = 2.0 ** -23 if out == torch.float32 else ref.half_step(out) * (1 + 2.0 ** -10)
            assert ((got[~h].double() - w[~h]).abs() <= tol * w[~h].abs() + 2.0 ** -24).all()
    # and the attention over them does not hide them
    q = torch.randn(1, H, d, generator=gen(352), device="cuda").to(dtype)
    out = cache.attend(q, ints([n]), table)[0]
    for h in range(H):
        assert torch.isnan(out[h]).all() if hit[:, h].any() else torch.isfinite(out[h]).all()


def test_a_rotated_key_that_is_not_finite(paged):
    """An infinity in a key spreads to its pair and to their groups, rotated on the way into 4 bits; other heads stay."""
    n, H, d = 20, 2, 128
    x = torch.randn(n, H, d, generator=gen(361), device="cuda").to(BF)
    wild = x.clone()
    wild[3, 0, 5] = math.inf                        # paired with channel 69: both groups
    wild[4, 1, 70] = math.nan
    rope = paged.Rope(d)
    outs = []
    for k in (x, wild):
        cache = paged.KVPages(2, H, 16, d, "q4")
        cache.append(k, x, ints([n]), ints([[0, 1]]), rope=rope)
        got = torch.zeros(1, H, n, d, device="cuda")
        cache.gather(got, None, ints([n]), ints([[0, 1]]))
        outs.append(got[0])
    assert torch.isnan(outs[1][0, 3]).all() and torch.isnan(outs[1][1, 4]).all()
    outs[1][0, 3], outs[1][1, 4] = outs[0][0, 3], outs[0][1, 4]
    assert torch.equal(outs[0], outs[1])


def same_numbers(got, want, dtype):
    """got is `want` (fp64) rounded: NaN where it is, the same infinities, half a step elsewhere."""
    rounded = want.to(dtype)
    assert torch.equal(torch.isnan(got), torch.isnan(rounded))
    wild = torch.isinf(rounded)
    assert torch.equal(got[wild], rounded[wild]) and torch.equal(torch.isinf(got), wild)
    ok = torch.isfinite(rounded)
    assert ((got[ok].double() - want[ok]).abs() <= ref.half_step(dtype) * (1 + 2.0 ** -10) * want[ok].abs() + 2.0 ** -24).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (128, 64, True), (128, 10, False), (64, 64, False), (64, 48, True), (64, 50, False)])
def test_rotation_of_infinities(paged, dtype, d, rot, interleaved):
    """x cos - y sin and x sin + y cos as IEEE arithmetic has them; positions whose cosine or sine is 0 or 1 among them."""
    n, H = 40, 3
    x = torch.randn(n, H, d, generator=gen(371), device="cuda").to(dtype)
    g = torch.Generator().manual_seed(372)
    for i in range(n):
        for _ in range(4):
            x[i, int(torch.randint(0, H, (1,), generator=g)), int(torch.randint(0, d, (1,), generator=g))] = \
                (math.inf, -math.inf, math.nan)[int(torch.randint(0, 3, (1,), generator=g))]
    x[5] = math.inf
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 97
    w, _ = ref.frequencies(rot)
    rope = paged.Rope(d, rot, interleaved=interleaved)
    for inverse in (False, True):
        same_numbers(rope.apply(x, pos, inverse=inverse), ref.rotate(x, pos, w, 1.0, interleaved, inverse), dtype)
    # on the way into a 16-bit cache: token i goes to position i
    cache = paged.KVPages(1, H, n, d, "bf16" if dtype == BF else "fp16")
    q = cache.append(x, x, ints([n]), rope=rope, q=x.flip(1).contiguous())
    want = ref.rotate(x, torch.arange(n, device="cuda"), w, 1.0, interleaved)
    same_numbers(cache.k[0].transpose(0, 1), want, dtype)
    same_numbers(q, want.flip(1), dtype)
    same_numbers(cache.v[0].transpose(0, 1), x.double(), dtype)


def test_rotation_that_overflows(paged):
    """fp16 rows whose rotated values are beyond the type: infinities, of the right sign."""
    n, H, d = 64, 2, 64
    x = (60000 * torch.randn(n, H, d, generator=gen(381), device="cuda").sign() * torch.rand(n, H, d, generator=gen(382), device="cuda")).to(FP)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    want = ref.rotate(x, pos, ref.frequencies(d)[0])
    assert (want.abs() > 65536).any()
    # within 2^-12 of the border both roundings are right
    want = torch.where((want.abs() - 65520).abs() < 16, 0.0, want)
    got = paged.Rope(d).apply(x, pos)
    same_numbers(torch.where(want == 0, 0, got), want, FP)
