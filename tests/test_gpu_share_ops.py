"""Pages that sequences share, attention over shared prefixes and over selected blocks, against plain forms (64 bits)."""
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
# Pool
# ---------------------------------------------------------------------------------------
class Both:
    """The pool on the device and on the host, step by step."""

    def __init__(self, paged, n_pages, page, B, width):
        self.host = sref.Pool(n_pages, page, B, width)
        self.pool = paged.PagePool(n_pages, page)
        self.table, self.lens = ints(self.host.table), ints(self.host.lens)

    def same(self):
        assert self.pool.refs.tolist() == self.host.refs
        assert self.table.tolist() == self.host.table
        assert self.lens.tolist() == self.host.lens
        assert self.pool.missing.item() == self.host.missing

    def reserve(self, new):
        self.pool.reserve(self.table, self.lens, ints(new))
        self.host.reserve(self.host.lens, new)
        self.same()

    def grow(self, new):
        """Reserve, and take the new lengths where there was room."""
        before = [list(r) for r in self.host.table]
        self.reserve(new)
        for b, n in enumerate(new):
            h = self.host
            if n > h.lens[b] and h.held(n) <= h.width and -1 not in h.table[b][h.held(h.lens[b]):h.held(n)]:
                h.lens[b] = n
        self.lens.copy_(ints(self.host.lens))
        return before

    def fork(self, parents, children):
        src, dst, rows = self.pool.fork(self.table, self.lens, ints(parents), ints(children))
        want = self.host.fork(parents, children)
        self.same()
        assert list(zip(src.tolist(), dst.tolist(), rows.tolist())) == want
        return src, dst, rows

    def free(self, rows=None):
        self.pool.free(self.table, self.lens, None if rows is None else ints(rows))
        self.host.free(range(len(self.host.lens)) if rows is None else rows)
        self.same()

    def compact(self):
        src, dst = self.pool.compact(self.table, self.lens)
        want = self.host.compact()
        self.same()
        n = self.host.refs.__len__() // 2
        assert list(zip(src.tolist(), dst.tolist())) == want + [(-1, -1)] * (n - len(want))
        return src, dst


@pytest.mark.parametrize("n_pages,page,B,width", [(1, 1, 1, 1), (7, 4, 3, 5), (64, 16, 9, 12), (5000, 16, 40, 200), (4097, 1, 33, 400),
                                                  (9000, 64, 1100, 30), (300, 24, 12, 40)])
def test_pool_random_walk(paged, n_pages, page, B, width):
    """Any order of calls, until pages run out and beyond."""
    rng = random.Random(n_pages * 31 + page)
    both = Both(paged, n_pages, page, B, width)
    for step in range(60):
        what = rng.choice(["grow", "grow", "fork", "fork", "free", "compact"])
        if what == "grow":
            most = width * page + (page if rng.random() < 0.2 else 0)
            both.grow([n + rng.choice([0, 0, 1, rng.randint(0, max(1, most - max(n, 0)))]) if rng.random() < 0.5 else n for n in both.host.lens])
        elif what == "fork":
            n = rng.randint(1, min(B, 20))
            both.fork([rng.randrange(-1, B + 1) for _ in range(n)], [rng.randrange(-1, B + 1) for _ in range(n)])
        elif what == "free":
            both.free([rng.randrange(-2, B + 2) for _ in range(rng.randint(1, max(1, B // 3)))])
        else:
            both.compact()
    both.free()
    assert max(both.host.refs) <= 0


def test_pool_many_forks(paged):
    """More forks than a CTA has threads, some without a page."""
    both = Both(paged, 700, 8, 1200, 6)
    both.grow([37, 40, 1] + [0] * 1197)
    both.fork([i % 3 for i in range(1100)], [3 + i for i in range(1100)])
    assert both.host.missing > 0
    both.free([3 + 2 * i for i in range(500)])
    both.compact()
    both.free()


def test_pool_edges(paged):
    both = Both(paged, 16, 4, 4, 4)
    both.lens.copy_(ints([-3, 0, 0, 0]))                      # an idle row may be negative
    both.host.lens[0] = -3
    both.grow([5, 16, 17, 0])                                 # the third does not fit its row
    assert both.host.table[2] == [-1] * 4 and both.host.missing == 5
    both.pool.missing.zero_()
    both.host.missing = 0
    both.fork([1], [3])                                       # ends with a full page: nothing to copy
    both.fork([0, 0], [2, 2])                                 # one child twice
    both.fork([0], [0])
    both.free([1, 1, 3])                                      # one row twice
    both.compact()
    old = both.table.clone()
    both.pool.reserve(both.table, both.lens, both.lens)       # nothing to do, one array
    assert torch.equal(old, both.table)
    # a table that holds numbers that are no pages
    both.table[0, 1] = 99
    both.host.table[0][1] = 99
    both.free([2])
    src, dst, rows = both.pool.fork(both.table, both.lens, ints([0]), ints([2]))
    assert src.tolist() == [99] and rows.tolist() == [1]
    both.pool.free(both.table, both.lens)
    assert both.lens.tolist() == [0] * 4


# ---------------------------------------------------------------------------------------
# Copies
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,H,page,d", [("bf16", 2, 16, 64), ("fp16", 1, 7, 128), ("bf16", 8, 64, 128), ("bf16", 3, 1, 64),
                                          ("q4", 2, 16, 64), ("q4", 5, 48, 128), ("q4", 1, 32, 64)])
@pytest.mark.parametrize("with_rows", [False, True])
def test_copy_pages(paged, fmt, H, page, d, with_rows):
    n_pages = 40
    cache = paged.KVPages(n_pages, H, page, d, fmt)
    g = torch.Generator(device="cuda").manual_seed(page + d)
    parts = [t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]
    for t in parts:
        b = t.view(torch.uint8) if t.dtype != torch.uint8 else t
        b.copy_(torch.randint(0, 256, b.shape, generator=g, device="cuda", dtype=torch.uint8))
    src = [3, 5, -1, 7, 3, 40, 2, 11, 9, 100000]
    dst = [20, 21, 22, -1, 23, 24, 2, 39, 0, 30]
    rows = [page, 1, page, page, max(1, page - 1), page, 1, 0, page + 5, -4]
    rows[9] = -4 if with_rows else page
    want = [t.clone().view(torch.int16 if t.dtype != torch.uint8 else torch.uint8) for t in parts]
    for s, e, r in zip(src, dst, rows):
        if 0 <= s < n_pages and 0 <= e < n_pages:
            r = max(0, min(r, page)) if with_rows else page
            for w in want:
                w[e, :, :r] = w[s, :, :r]
    cache.copy_pages(ints(src), ints(dst), ints(rows) if with_rows else None)
    for t, w in zip(parts, want):
        assert torch.equal(t.view(w.dtype), w)


def test_copy_many_pages(paged):
    """More pairs than CTAs, and pages behind 4 GiB."""
    cache = paged.KVPages(33000, 2, 128, 128, "bf16")              # 2.2 GB for keys
    ids = torch.arange(33000, device="cuda", dtype=torch.int32)
    cache.k.copy_((ids % 251).view(-1, 1, 1, 1).expand_as(cache.k))
    cache.v.copy_((ids % 241).view(-1, 1, 1, 1).expand_as(cache.v))
    order = torch.randperm(16000, device="cuda", dtype=torch.int32)
    cache.copy_pages(order, ids[17000:])
    for x, m in ((cache.k, 251), (cache.v, 241)):
        want = torch.cat((ids[:17000] % m, order % m)).to(BF)
        assert torch.equal(x.amax((1, 2, 3)), want) and torch.equal(x.amin((1, 2, 3)), want)


# ---------------------------------------------------------------------------------------
# Attention over 16-bit pages
# ---------------------------------------------------------------------------------------
def run_shared(paged, sizes, shared, lens, page, H_q, H, d, T, dtype, scale=None, seed=1, groups=True):
    k, v, table, cu, sh = sref.grouped_cache(sizes, shared, lens, page, H, d, dtype, seed)
    cache = paged.KVPages.wrap(k, v)
    q = randn(seed + 5, len(lens), T, H_q, d, dtype=dtype)
    lse = torch.full((len(lens), T, H_q), 7.0, device="cuda")
    out = cache.attend_shared(q, ints(lens), table, cu if groups else None, sh if groups else None, scale=scale, lse=lse)
    sref.check_attention(out, lse, q, k, v, table, lens, page, d ** -0.5 if scale is None else scale, case=f"{sizes} {shared} {lens}")
    return cache, q, table, cu, sh, out, lse


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("H_q,H,d", [(4, 4, 64), (8, 2, 128), (16, 1, 128), (5, 1, 64), (3, 3, 128)])
@pytest.mark.parametrize("T", [1, 3])
def test_attend_heads(paged, dtype, H_q, H, d, T):
    run_shared(paged, [3, 2], [100, 37], [130, 101, 260, 40, 300], 16, H_q, H, d, T, dtype)


@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 128, 256, 1000])
def test_attend_page_sizes(paged, page):
    run_shared(paged, [2, 1, 3], [200, 0, 513], [201, 333, 129, 700, 514, 640], page, 8, 2, 64, 2, BF)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 384, 1000, 5000])
def test_attend_lengths(paged, n):
    """No sharing at all: tile ends."""
    run_shared(paged, [1, 1], [0, 0], [n, max(1, n - 1)], 16, 4, 2, 128, 1, FP)
    run_shared(paged, [1, 1], [0, 0], [n, max(1, n - 1)], 16, 4, 2, 128, 1, FP, groups=False)


@pytest.mark.parametrize("shared", [1, 16, 100, 127, 128, 129, 500, 512])
@pytest.mark.parametrize("own", [0, 1, 130])
def test_attend_prefix_ends(paged, shared, own):
    run_shared(paged, [3], [shared], [shared + own, shared + 1, shared + 2 * own], 16, 8, 2, 128, 1, BF)


@pytest.mark.parametrize("members,G,T", [(31, 4, 1), (32, 4, 1), (33, 4, 1), (64, 4, 1), (65, 4, 1), (9, 16, 2), (3, 16, 16), (130, 2, 1), (40, 8, 3)])
def test_attend_many_members(paged, members, G, T):
    """Rows below, at and above one and two tiles of queries."""
    rng = random.Random(members)
    lens = [300 + T + rng.randint(0, 90) for _ in range(members)]
    run_shared(paged, [members], [300], lens, 32, 2 * G, 2, 64, T, BF)


def test_attend_long(paged):
    run_shared(paged, [5, 1], [20000, 9000], [20011, 20600, 23000, 20001, 20500, 30001], 64, 8, 2, 128, 1, BF)
    run_shared(paged, [2], [70000], [70100, 70001], 64, 2, 1, 128, 2, FP)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
@pytest.mark.parametrize("members,G,T", [(1, 1, 1), (2, 4, 2), (8, 4, 1), (11, 3, 1), (16, 4, 1), (7, 2, 4), (17, 4, 1)])
def test_attend_lines_in_many_parts(paged, dtype, d, members, G, T):
    """A few query rows and one head: parts of a line in every CTA, whose copies of the rows become one."""
    rng = random.Random(members)
    run_shared(paged, [members], [9000], [9000 + T + rng.randint(0, 300) for _ in range(members)], 32, G, 1, d, T, dtype)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
@pytest.mark.parametrize("T,G", [(1, 4), (2, 4), (4, 4), (3, 1)])
def test_attend_small_group_in_large_batch(paged, dtype, d, T, G):
    """Two sequences with a long prefix next to many with a short one."""
    rng = random.Random(T)
    sizes, shared = [2, 66], [9000, 300]
    lens = [n + T + rng.randint(0, 200) for m, n in zip(sizes, shared) for _ in range(m)]
    run_shared(paged, sizes, shared, lens, 16, G, 1, d, T, dtype)


@pytest.mark.parametrize("members,T,G", [(3, 2, 2), (2, 1, 16), (70, 1, 4)])
def test_attend_more_tiles_than_a_chunk(paged, members, T, G):
    """Lines of more than 1024 tiles of 128 keys: of a group and of one sequence alone."""
    lens = [132000 + T + 40 * i for i in range(members)] + [140001]
    run_shared(paged, [members, 1], [132000, 0], lens, 128, G, 1, 64, T, BF)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [2, 5, 16])
def test_attend_draft_tokens_in_place(paged, d, T):
    """Outputs in the place of the queries, which are read for the draft tokens' own keys until the last."""
    lens = [330, T, 900, 301 + T, 0, T - 1]
    k, v, table, cu, sh = sref.grouped_cache([4, 2], [300, 0], lens, 16, 3, d, BF)
    cache = paged.KVPages.wrap(k, v)
    q = randn(4, 6, T, 12, d)
    results = []
    for _ in range(5):
        x = q.clone()
        assert cache.attend_shared(x, ints(lens), table, cu, sh, out=x) is x
        sref.check_attention(x, None, q, k, v, table, lens, 16, d ** -0.5)
        results.append(x)
    assert all(torch.equal(x, results[0]) for x in results)


def test_attend_repeats_itself(paged):
    """The same call gives the same bits, on a busy device too."""
    lens = [5000 + 37 * i for i in range(20)]
    k, v, table, cu, sh = sref.grouped_cache([20], [4900], lens, 16, 2, 128, BF)
    cache = paged.KVPages.wrap(k, v)
    q = randn(4, 20, 1, 8, 128)
    want = cache.attend_shared(q, ints(lens), table, cu, sh)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        with torch.cuda.stream(other):
            cache.k.sum(dtype=torch.float32)
        assert torch.equal(cache.attend_shared(q, ints(lens), table, cu, sh), want)
    torch.cuda.synchronize()


def test_attend_idle_and_short_members(paged):
    """Empty sequences, lengths that the table cannot hold, members that are shorter than the shared rows."""
    k, v, table, cu, sh = sref.grouped_cache([4, 3], [64, 80], [90, 64, 130, 100, 200, 81, 80], 16, 2, 64, BF)
    cache = paged.KVPages.wrap(k, v)
    q = randn(3, 7, 2, 8, 64)
    for lens in ([90, 0, 130, 100, 200, 81, 80], [0, 64, 130, -5, 200, 81, 80], [90, 64, 1, 100, 0, 0, 0], [0] * 7, [90, 10 ** 9, 130, 2, 200, 3, 1]):
        lse = torch.zeros(7, 2, 8, device="cuda")
        out = cache.attend_shared(q, ints(lens), table, cu, sh, lse=lse)
        held = [n if 0 <= n <= table.shape[1] * 16 else 0 for n in lens]
        sref.check_attention(out, lse, q, k, v, table, held, 16, 64 ** -0.5, case=str(lens))


def test_attend_groups_are_a_hint(paged):
    """Groupings that do not ascend from 0 to B stand for none; shared lengths beyond a sequence are cut."""
    k, v, table, cu, sh = sref.grouped_cache([2, 2], [64, 64], [90, 100, 130, 70], 16, 2, 64, BF)
    cache, lens = paged.KVPages.wrap(k, v), [90, 100, 130, 70]
    q = randn(3, 4, 1, 8, 64)
    for bad in ([0, 3, 3], [1, 2, 4], [0, 5, 4], [0, -7, 4], [2 ** 31 - 1, 0, 4]):
        out = cache.attend_shared(q, ints(lens), table, ints(bad), sh)
        sref.check_attention(out, None, q, k, v, table, lens, 16, 64 ** -0.5, case=str(bad))
    for few in ([-5, 0], [64, -2 ** 31], [64, 3]):
        out = cache.attend_shared(q, ints(lens), table, cu, ints(few))
        sref.check_attention(out, None, q, k, v, table, lens, 16, 64 ** -0.5, case=str(few))
    # one sequence of a group, an empty group
    out = cache.attend_shared(q, ints(lens), table, ints([0, 1, 1, 4]), ints([10 ** 9, 5, 0]))
    sref.check_attention(out, None, q, k, v, table, lens, 16, 64 ** -0.5)


def test_attend_pages_out_of_range(paged):
    """Keys of pages that are none do not count."""
    k, v, table, cu, sh = sref.grouped_cache([3], [96], [150, 97, 200], 16, 2, 64, BF)
    cache, lens = paged.KVPages.wrap(k, v), [150, 97, 200]
    q = randn(3, 3, 1, 4, 64)
    table[:, 2] = -1                                              # a shared page, in every row
    table[2, 7] = 10 ** 6
    out = cache.attend_shared(q, ints(lens), table, cu, sh)
    for b, n in enumerate(lens):
        gone = [2] + ([7] if b == 2 else [])
        rows = torch.tensor([j for j in range(n) if j // 16 not in gone], device="cuda")
        ids = table[b].long()[rows // 16]
        rk, rv = (x[ids, :, rows % 16].double().transpose(0, 1) for x in (k, v))
        want, _ = ref.attention(q[b], rk, rv, 64 ** -0.5)
        limit = sref.attention_bound(q[b], rk, rv, 64 ** -0.5, n, BF)[1] + ref.half_step(BF) * want.abs()
        assert bool(((out[b].double() - want).abs() <= limit).all())
    table[:] = -1
    lse = torch.zeros(3, 1, 4, device="cuda")
    out = cache.attend_shared(q, ints(lens), table, cu, sh, lse=lse)
    assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_attend_scales(paged, scale):
    run_shared(paged, [2, 1], [50, 10], [60, 51, 300], 16, 8, 2, 128, 2, BF, scale=scale)


def test_attend_large_scores(paged):
    """A maximum that keeps growing along the keys, and one large key among small ones."""
    lens = [1000, 777]
    k, v, table, cu, sh = sref.grouped_cache([2], [500], lens, 16, 1, 64, BF)
    ramp = torch.linspace(0, 12, 500, device="cuda")
    for j in range(500):
        k[table[0, j // 16].long(), 0, j % 16] = ramp[j].to(BF)
    if table[0, 31] != table[1, 31]:
        k[table[1, 31].long(), 0, :4] = k[table[0, 31].long(), 0, :4]
    k[table[0, 50].long(), 0, 3] = 20.0
    cache = paged.KVPages.wrap(k, v)
    q = randn(8, 2, 1, 4, 64, scale=2.0)
    lse = torch.zeros(2, 1, 4, device="cuda")
    out = cache.attend_shared(q, ints(lens), table, cu, sh, lse=lse)
    sref.check_attention(out, lse, q, k, v, table, lens, 16, 64 ** -0.5)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_attend_nonfinite(paged, dtype):
    """What a token does not see has no influence; what it sees shows in its row alone."""
    lens = [300, 260]
    k, v, table, cu, sh = sref.grouped_cache([2], [200], lens, 16, 2, 64, dtype)
    cache = paged.KVPages.wrap(k, v)
    q = randn(8, 2, 4, 4, 64, dtype=dtype)
    want = cache.attend_shared(q, ints(lens), table, cu, sh)
    sref.check_attention(want, None, q, k, v, table, lens, 16, 64 ** -0.5)
    used = torch.zeros(k.shape[0], 16, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        for j in range(n):
            used[table[b, j // 16].long(), j % 16] = True
    hidden = ~used.unsqueeze(1).unsqueeze(-1).expand_as(k)
    for value in (math.nan, math.inf):
        k.masked_fill_(hidden, value)
        v.masked_fill_(hidden, value)
        assert torch.equal(cache.attend_shared(q, ints(lens), table, cu, sh), want)
    # the last draft token's key and value: seen by itself alone
    j = lens[0] - 1
    for x, value in ((k, math.nan), (v, math.nan), (k, math.inf), (v, -math.inf)):
        keep = x[table[0, j // 16].long(), :, j % 16].clone()
        x[table[0, j // 16].long(), :, j % 16] = value
        got = cache.attend_shared(q, ints(lens), table, cu, sh)
        assert torch.equal(got[1], want[1]) and torch.equal(got[0, :3], want[0, :3])
        if x is v:
            assert not torch.isfinite(got[0, 3]).any()
        elif math.isnan(value):
            assert torch.isnan(got[0, 3]).all()
        x[table[0, j // 16].long(), :, j % 16] = keep
    # a key of the prefix with NaN: every row of that head group; a query with NaN: its row
    page, at = table[0, 3].long(), 5
    keep = k[page, 1, at].clone()
    k[page, 1, at, 7] = math.nan
    got = cache.attend_shared(q, ints(lens), table, cu, sh)
    assert torch.isnan(got[:, :, 2:]).all() and torch.equal(got[:, :, :2], want[:, :, :2])
    k[page, 1, at] = keep
    q[1, 2, 1, 9] = math.nan
    got = cache.attend_shared(q, ints(lens), table, cu, sh)
    assert torch.isnan(got[1, 2, 1]).all()
    got[1, 2, 1] = want[1, 2, 1]
    assert torch.equal(got, want)
    # scores of -inf are weights of 0, and a row of nothing else is NaN; +inf is NaN
    q[1, 2, 1] = randn(9, 64, dtype=dtype)
    q[:, :, :, 0] = 1.0
    want = cache.attend_shared(q, ints(lens), table, cu, sh)
    k[table[0, 2].long(), :, 4, 0] = -math.inf
    got = cache.attend_shared(q, ints(lens), table, cu, sh)
    assert torch.isfinite(got).all() and not torch.equal(got, want)
    k[table[0, 2].long(), :, 4, 0] = math.inf
    assert torch.isnan(cache.attend_shared(q, ints(lens), table, cu, sh)).all()


def test_attend_strides_in_place_and_three_dims(paged):
    lens = [70, 90]
    k, v, table, cu, sh = sref.grouped_cache([2], [64], lens, 16, 2, 64, BF)
    cache = paged.KVPages.wrap(k, v)
    wide = randn(4, 2, 9, 64)
    q = wide[:, :4]
    a = cache.attend_shared(q, ints(lens), table, cu, sh)
    b = cache.attend_shared(q.contiguous().unsqueeze(1), ints(lens), table, cu, sh)
    assert a.shape == (2, 4, 64) and torch.equal(a, b[:, 0])
    c = q.contiguous()
    version = c._version
    assert cache.attend_shared(c, ints(lens), table, cu, sh, out=c) is c and torch.equal(c, a) and c._version > version
    # the contiguous cache of the decode step
    kc, vc = randn(5, 2, 2, 96, 64), randn(6, 2, 2, 96, 64)
    flat = paged.KVPages.wrap(kc, vc)
    out = flat.attend_shared(q, ints(lens))
    sref.check_attention(out.unsqueeze(1), None, q.unsqueeze(1), kc, vc, None, lens, 96, 64 ** -0.5)
    assert cache.attend_shared(q[:0], ints([]), table[:0]).shape == (0, 4, 64)


def test_attend_many_sequences(paged):
    """Thousands of short sequences, in groups of every size."""
    rng = random.Random(4)
    sizes = []
    while sum(sizes) < 2000:
        sizes.append(rng.choice([1, 1, 2, 5, 40, 130]))
    sizes[-1] -= sum(sizes) - 2000
    sizes = [m for m in sizes if m > 0]
    shared = [rng.choice([0, 3, 16, 50]) for _ in sizes]
    lens = [shared[i] + rng.randint(1, 40) for i, m in enumerate(sizes) for _ in range(m)]
    k, v, table, cu, sh = sref.grouped_cache(sizes, shared, lens, 16, 2, 64, BF)
    cache = paged.KVPages.wrap(k, v)
    q = randn(3, 2000, 1, 4, 64)
    for b in range(0, 2000, 3):
        lens[b] = 0
    out = cache.attend_shared(q, ints(lens), table, cu, sh)
    assert torch.equal(out, cache.attend_shared(q, ints(lens), table, cu, sh))
    for b in list(range(0, 2000, 37)) + [1998, 1999]:
        sref.check_attention(out[b:b + 1], None, q[b:b + 1], k, v, table[b:b + 1], lens[b:b + 1], 16, 64 ** -0.5, case=str(b))


# ---------------------------------------------------------------------------------------
# Blocks
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("page,block,d,H", [(16, 16, 64, 2), (64, 64, 128, 3), (64, 16, 128, 1), (96, 32, 64, 4), (256, 128, 128, 2)])
def test_block_update(paged, dtype, page, block, d, H):
    lens = [5 * page, 3 * page + block + 3, block - 1, 0, -4, block]
    rows, total = sref.scattered([max(0, -(-n // page)) for n in lens], 2, 3)
    table = ints([r + [0] * (6 - len(r)) for r in rows])
    k = randn(3, total, H, page, d, dtype=dtype)
    k[table[0, 1].long(), 0, 3, 5] = math.nan
    k[table[0, 2].long(), 0, 3, 5] = math.inf
    cache = paged.KVPages.wrap(k, randn(4, total, H, page, d, dtype=dtype))
    every = sref.bounds_of(k, block)
    for n_new in (None, 1, 2, block, block + 1, 2 * page + 1):
        index = paged.BlockIndex(cache, block)
        index.bounds.fill_(7.0)
        index.update(ints(lens), table, n_new)
        want = torch.full_like(index.bounds, 7.0)
        for b, n in enumerate(lens):
            for j in range(max(0, n - (n_new or n)) // block, max(n, 0) // block):
                p, at = table[b, j * block // page].long(), j * block % page // block
                want[p, :, at] = every[p, :, at]
        assert torch.equal(torch.nan_to_num(index.bounds, nan=99.0), torch.nan_to_num(want, nan=99.0)), n_new
    index.update(ints(lens), table, 0)


def make_blocks(paged, lens, page, block, H, d, dtype, seed=1):
    rows, total = sref.scattered([max(0, -(-n // page)) for n in lens], 1, seed)
    width = max(len(r) for r in rows) + 1
    table = ints([r + [0] * (width - len(r)) for r in rows])
    k = randn(seed, total, H, page, d, dtype=dtype)
    k += randn(seed + 1, total, H, 1, d, dtype=dtype)
    cache = paged.KVPages.wrap(k, randn(seed + 2, total, H, page, d, dtype=dtype))
    index = paged.BlockIndex(cache, block)
    index.update(ints(lens), table)
    return cache, index, table


def check_select(index, table, q, lens, blocks, keep, first, last, page):
    picks = []
    for b, n in enumerate(lens):
        picks.append([sref.select(q[b, t], index.bounds, table, b, n - q.shape[1] + 1 + t, page, index.block, keep, first, last)
                      for t in range(q.shape[1])])
        for t in range(q.shape[1]):
            for h, want in enumerate(picks[b][t]):
                assert blocks[b, t, h].tolist() == want + [-1] * (keep - len(want)), (b, t, h)
    return picks


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("H_q,H,d,T,page,block", [(8, 2, 128, 1, 64, 64), (4, 4, 64, 1, 16, 16), (16, 1, 128, 3, 64, 32), (6, 2, 64, 2, 128, 16),
                                                  (8, 2, 64, 1, 128, 128)])
def test_select_and_attend(paged, dtype, H_q, H, d, T, page, block):
    lens = [40 * block + 5, 17 * block, 3, 0, 9 * block + 1, 100 * block - 1, T]
    cache, index, table = make_blocks(paged, lens, page, block, H, d, dtype)
    q = randn(9, len(lens), T, H_q, d, dtype=dtype)
    for keep, first, last in ((9, 1, 2), (1, 0, 1), (4, 0, 1), (3, 1, 2), (40, 2, 3), (200, 1, 1)):
        blocks = index.select(q, ints(lens), table, keep=keep, first=first, last=last)
        picks = check_select(index, table, q, lens, blocks, keep, first, last, page)
        lse = torch.zeros(len(lens), T, H_q, device="cuda")
        out = index.attend(q, ints(lens), blocks, table, lse=lse)
        sref.check_attention(out, lse, q, cache.k, cache.v, table, lens, page, d ** -0.5, picks, block, case=f"keep {keep}")
    # all blocks: dense attention
    dense = cache.attend_shared(q, ints(lens), table)
    every = index.select(q, ints(lens), table, keep=101)
    sref.check_attention(index.attend(q, ints(lens), every, table), None, q, cache.k, cache.v, table, lens, page, d ** -0.5)
    sref.check_attention(dense, None, q, cache.k, cache.v, table, lens, page, d ** -0.5)


def test_select_ties_and_nonfinite(paged):
    """Equal scores go to the lower number; NaN comes first, pages out of range last."""
    lens = [64 * 50, 64 * 50 + 1]
    cache, index, table = make_blocks(paged, lens, 64, 64, 2, 64, BF)
    index.bounds.zero_()
    q = randn(9, 2, 1, 4, 64)
    blocks = index.select(q, ints(lens), table, keep=10, first=2, last=3)
    assert blocks[0, 0, 0].tolist() == list(range(7)) + [47, 48, 49]
    assert blocks[1, 0, 1].tolist() == list(range(7)) + [48, 49, 50]
    index.bounds[table[0, 20].long(), 1, 0, 0, 3] = math.nan
    index.bounds[table[0, 30].long(), 1] = 1e30
    index.bounds[table[0, 40].long(), 1] = -1e30
    blocks = index.select(q, ints(lens), table, keep=10, first=2, last=3)
    picks = check_select(index, table, q, lens, blocks, 10, 2, 3, 64)
    assert 20 in picks[0][0][1]
    index.bounds.fill_(-1.0)
    table[0, 5:] = -1
    blocks = index.select(q, ints(lens), table, keep=8, first=1, last=1)
    assert blocks[0, 0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 49]
    # scores that differ in the last bits of their sums only
    index.bounds.copy_(randn(11, *index.bounds.shape).sort(3).values)
    table = ints([list(range(50)) + [0] * 2, list(range(51)) + [0]])
    index.bounds[1::2] = index.bounds[0:-1:2].clone()
    q = randn(12, 2, 1, 4, 64)
    blocks = index.select(q, ints(lens), table, keep=20, first=0, last=1)
    check_select(index, table, q, lens, blocks, 20, 0, 1, 64)


def test_select_many_blocks(paged):
    """Tens of thousands of blocks, most of them equal."""
    n = 16 * 40000 + 7
    k = torch.zeros(1, 1, 16 * 40001, 64, dtype=BF, device="cuda")
    k[0, 0, :, :8] = randn(5, 16 * 40001, 8).clamp(-0.5, 0.5)
    cache = paged.KVPages.wrap(k, k.clone())
    index = paged.BlockIndex(cache, 16)
    index.update(ints([n]))
    q = randn(6, 1, 1, 2, 64)
    for keep in (64, 2000, 39000):
        blocks = index.select(q, ints([n]), keep=keep)
        check_select(index, None, q, [n], blocks, keep, 1, 2, k.shape[2])
    out = index.attend(q, ints([n]), blocks)
    picks = [[[[x for x in blocks[0, 0, 0].tolist()]]]]
    sref.check_attention(out, None, q, k, cache.v, None, [n], k.shape[2], 64 ** -0.5, picks, 16)


@pytest.mark.parametrize("dtype,key,query", [(FP, 2.0 ** -20, 1.0), (FP, 2.0 ** -23, 2.0 ** -20), (BF, 2.0 ** -130, 1.0), (BF, 2.0 ** -100, 2.0 ** -30),
                                             (FP, 2.0 ** 12, 2.0 ** 12), (BF, 2.0 ** 100, 2.0 ** 20), (BF, 2.0 ** 120, 2.0 ** 120)])
def test_select_small_and_large_numbers(paged, dtype, key, query):
    """Subnormal numbers and products, sums near and beyond the largest: the order of the scores rounded to fp32 holds."""
    lens = [16 * 300, 16 * 700 + 3]
    cache, index, table = make_blocks(paged, lens, 32, 16, 2, 64, dtype)
    cache.k.copy_((cache.k.float() * key).to(dtype))
    index.update(ints(lens), table)
    q = (randn(9, 2, 1, 6, 64).float() * query).to(dtype)
    for keep in (20, 250):
        blocks = index.select(q, ints(lens), table, keep=keep, first=1, last=2)
        check_select(index, table, q, lens, blocks, keep, 1, 2, 32)


def test_select_infinite_queries(paged):
    """Infinities and NaN in a query: a score that is no number counts as the largest."""
    lens = [16 * 60, 16 * 60]
    cache, index, table = make_blocks(paged, lens, 32, 16, 2, 64, BF)
    q = randn(9, 2, 1, 4, 64)
    q[0, 0, 1, 5] = math.inf
    q[0, 0, 2, 7] = -math.inf
    q[1, 0, 0, 3] = math.nan
    blocks = index.select(q, ints(lens), table, keep=9, first=1, last=2)
    check_select(index, table, q, lens, blocks, 9, 1, 2, 32)


def test_attend_many_selected_blocks(paged):
    """One token whose blocks are in many parts."""
    lens = [16 * 900 + 5]
    cache, index, table = make_blocks(paged, lens, 64, 16, 1, 128, BF)
    q = randn(9, 1, 1, 4, 128)
    blocks = index.select(q, ints(lens), table, keep=700)
    picks = check_select(index, table, q, lens, blocks, 700, 1, 2, 64)
    sref.check_attention(index.attend(q, ints(lens), blocks, table), None, q, cache.k, cache.v, table, lens, 64, 128 ** -0.5, picks, 16)


def test_attend_lists(paged):
    """Lists of the caller's own: any order, numbers that are no blocks, a block twice."""
    lens = [300, 170]
    cache, index, table = make_blocks(paged, lens, 32, 32, 2, 64, BF)
    q = randn(9, 2, 1, 4, 64)
    lists = [[[7, 2, 9], [0, 0, 3]], [[5, 1, -1], [6, 1000000, -9]]]
    blocks = ints(lists).unsqueeze(1)
    lse = torch.zeros(2, 1, 4, device="cuda")
    out = index.attend(q, ints(lens), blocks, table, lse=lse)
    picks = [[[[x for x in l if 0 <= x] for l in row]] for row in lists]
    sref.check_attention(out, lse, q, cache.k, cache.v, table, lens, 32, 64 ** -0.5, picks, 32)
    assert not out[1, 0, 2:].any() and bool((lse[1, 0, 2:] == -math.inf).all())


# ---------------------------------------------------------------------------------------
# All of it together
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,page,block", [(BF, 64, 16), (FP, 16, 16)])
def test_serving_run(paged, dtype, page, block):
    """A prompt, forks, tokens to each, frees, a compaction; two layers over one table; against 64 bits throughout."""
    H_q, H, d, B, width, n_pages = 8, 2, 64, 6, 40, 120
    rope = paged.Rope(d)
    both = Both(paged, n_pages, page, B, width)
    layers = [paged.KVPages(n_pages, H, page, d, "bf16" if dtype == BF else "fp16") for _ in range(2)]
    indexes = [paged.BlockIndex(c, block) for c in layers]
    w, _ = ref.frequencies(d)
    truth = [[[torch.zeros(H, 0, d, dtype=dtype, device="cuda") for _ in range(2)] for _ in range(B)] for _ in layers]
    seed = [100]

    def append(new):
        """new[b] tokens for each sequence; T is one number for the batch, idle ones have length 0."""
        both.grow([n + m for n, m in zip(both.host.lens, new)])
        cu = [sum(new[:i]) for i in range(B + 1)]
        for cache, index, rows in zip(layers, indexes, truth):
            seed[0] += 3
            k, v = randn(seed[0], cu[-1], H, d, dtype=dtype), randn(seed[0] + 1, cu[-1], H, d, dtype=dtype)
            cache.append(k, v, both.lens, both.table, ints(cu), rope=rope)
            index.update(both.lens, both.table, max(new))
            for b, n in enumerate(both.host.lens):
                pos = torch.arange(n - new[b], n, device="cuda")
                turned = ref.rotate(k[cu[b]:cu[b + 1]], pos, w).to(dtype)
                for i, x in enumerate((turned, v[cu[b]:cu[b + 1]])):
                    rows[b][i] = torch.cat((rows[b][i], x.transpose(0, 1)), 1)

    def fork(parents, children):
        src, dst, n = both.fork(parents, children)
        for cache, index, rows in zip(layers, indexes, truth):
            cache.copy_pages(src, dst, n)
            index.copy_pages(src, dst)
            for p, c in zip(parents, children):
                rows[c] = list(rows[p])

    def check(cu, shared, keep=5):
        lens = both.host.lens
        q = randn(seed[0] + 2, B, 1, H_q, d, dtype=dtype)
        for cache, index, rows in zip(layers, indexes, truth):
            out = cache.attend_shared(q, both.lens, both.table, ints(cu), ints(shared))
            blocks = index.select(q, both.lens, both.table, keep=keep)
            sparse = index.attend(q, both.lens, blocks, both.table)
            for b, n in enumerate(lens):
                if n == 0:
                    assert not out[b].any()
                    continue
                rk, rv = rows[b]
                # the cache holds what was appended (a key is rounded once from a rotation within 2^-23)
                have = ref.rows_of(cache.k, None, both.table, b, n, page)
                assert torch.allclose(have, rk.double(), rtol=2 * ref.half_step(dtype), atol=2.0 ** -20)
                assert torch.equal(ref.rows_of(cache.v, None, both.table, b, n, page), rv.double())
            sref.check_attention(out, None, q, cache.k, cache.v, both.table, lens, page, d ** -0.5)
            picks = check_select(index, both.table, q, lens, blocks.view(B, 1, H, keep), keep, 1, 2, page)
            for b, n in enumerate(lens):                          # bounds of the full blocks are those of their keys
                for j in range(n // block):
                    p, at = both.table[b, j * block // page].long(), j * block % page // block
                    x = cache.k[p, :, at * block:(at + 1) * block]
                    assert torch.equal(index.bounds[p, :, at, 0], x.amin(1)) and torch.equal(index.bounds[p, :, at, 1], x.amax(1))
            sref.check_attention(sparse, None, q, cache.k, cache.v, both.table, lens, page, d ** -0.5, picks, block)

    append([203, 0, 0, 0, 90, 0])
    check([0, 4, 6], [0, 0])
    fork([0, 0, 4], [1, 2, 5])
    for step in range(3):
        append([1, 1, 1, 0, 1, 1])
        check([0, 4, 6], [203, 90])
    append([20, 1, 33, 0, 2, 70])
    both.free([0, 4])
    for rows in truth:
        rows[0] = rows[4] = [torch.zeros(H, 0, d, dtype=dtype, device="cuda")] * 2
    check([0, 4, 6], [203, 90])
    src, dst = both.compact()
    for cache, index in zip(layers, indexes):
        cache.copy_pages(src, dst)
        index.copy_pages(src, dst)
    check([0, 4, 6], [203, 90])
    fork([2, 1], [0, 3])
    append([1, 1, 1, 1, 0, 1])
    check([0, 4, 6], [203, 0])


def test_graphs_and_streams(paged):
    """Two captured graphs with workspaces of their own, replayed at once; replays follow the device's numbers."""
    cases = []
    for i in range(2):
        lens = [700 + i, 650, 900]
        k, v, table, cu, sh = sref.grouped_cache([3], [600], lens, 16, 2, 128, BF, seed=i + 1)
        cache = paged.KVPages.wrap(k, v)
        index = paged.BlockIndex(cache, 16)
        n = ints(lens)
        q = randn(i + 3, 3, 8, 128)

        def step(cache=cache, index=index, q=q, n=n, table=table, cu=cu, sh=sh):
            index.update(n, table, 40)
            blocks = index.select(q, n, table, keep=12)
            return cache.attend_shared(q, n, table, cu, sh), index.attend(q, n, blocks, table), blocks

        index.update(n, table)
        cases.append((step, n, [x.clone() for x in step()]))
    streams = [torch.cuda.Stream() for _ in range(2)]
    graphs, outs = [], []
    torch.cuda.synchronize()
    for (step, _, _), s in zip(cases, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(step())
        graphs.append(graph)
    for _ in range(20):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for (_, _, want), out in zip(cases, outs):
        assert all(torch.equal(a, b) for a, b in zip(want, out))
    for step, n, want in cases:
        n.copy_(ints([640, 0, 850]))
    fresh = [[x.clone() for x in step()] for step, _, _ in cases]
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(fresh, outs):
        assert all(torch.equal(x, y) for x, y in zip(a, b)) and not b[0][1].any()
    results = []
    for _ in range(10):
        results = []
        for (step, _, _), s in zip(cases, streams):
            with torch.cuda.stream(s):
                results.append(step())
    torch.cuda.synchronize()
    for a, b in zip(fresh, results):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_pool_graph(paged):
    """A captured fork and free: replays take the pages that are free then."""
    both = Both(paged, 64, 16, 5, 8)
    both.grow([100, 37, 0, 0, 0])
    parents, children = ints([0, 1, 0]), ints([2, 3, 4])
    cache = paged.KVPages(64, 2, 16, 64, "bf16")
    cache.k.copy_(randn(1, *cache.k.shape))
    cache.copy_pages(*both.pool.fork(both.table, both.lens, parents, children))
    both.host.fork([0, 1, 0], [2, 3, 4])
    both.free([2, 3, 4])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        moves = both.pool.fork(both.table, both.lens, parents, children)
        cache.copy_pages(*moves)
    graph.replay()
    both.host.fork([0, 1, 0], [2, 3, 4])
    both.same()
    both.free([2, 4])
    both.free([3, 1])
    graph.replay()                                            # row 1 is empty now: its fork is not made
    both.host.fork([0, 1, 0], [2, 3, 4])
    both.same()
    assert moves[1].tolist()[1] == -1
    page = both.table[2, 6].long()
    assert torch.equal(cache.k[page, :, :4], cache.k[both.table[0, 6].long(), :, :4])


def test_binding_refusals(paged):
    cache, q4 = paged.KVPages(4, 2, 16, 64, "bf16"), paged.KVPages(4, 2, 16, 64, "q4")
    q = torch.zeros(2, 4, 64, dtype=BF, device="cuda")
    lens, table = ints([1, 1]), ints([[0], [1]])
    E = paged._rt.RetopkError
    with pytest.raises(TypeError):
        q4.attend_shared(q, lens, table)
    with pytest.raises(TypeError):
        cache.attend_shared(q.half(), lens, table)
    with pytest.raises(ValueError):
        cache.attend_shared(q, lens, table, ints([0, 2]))
    with pytest.raises(ValueError):
        cache.attend_shared(q, lens, table, ints([0, 2]), ints([1, 1]))
    with pytest.raises(ValueError):
        cache.attend_shared(q, lens, table, ints([0, 1, 1, 2]), ints([1, 1, 1]))
    with pytest.raises(TypeError):
        cache.attend_shared(q, lens, table, ints([0, 2]).long(), ints([1]))
    with pytest.raises(E):
        cache.attend_shared(q[:, :3].contiguous(), lens, table)
    with pytest.raises(E):
        cache.attend_shared(q.requires_grad_(), lens, table)
    q = q.detach()
    with pytest.raises(E):
        cache.attend_shared(q, lens, table, out=cache.k.view(-1)[:512].view(2, 4, 64))
    with pytest.raises(TypeError):
        cache.attend_shared(q, lens, table, out=q.float())
    with pytest.raises(E):
        cache.attend_shared(q, lens, table, scale=math.inf)
    with pytest.raises(TypeError):
        paged.BlockIndex(q4, 16)
    for block in (8, 24, 32, 0):
        with pytest.raises(ValueError):
            paged.BlockIndex(cache, block)
    index = paged.BlockIndex(cache, 16)
    with pytest.raises(ValueError):
        paged.BlockIndex.wrap(cache, index.bounds[:, :, :, 0])
    with pytest.raises(ValueError):
        index.select(q, lens, table, keep=2, first=1, last=2)
    with pytest.raises(ValueError):
        index.select(q, lens, table, keep=4, first=1, last=0)
    with pytest.raises(ValueError):
        index.attend(q, lens, torch.zeros(2, 1, 3, dtype=torch.int32, device="cuda"), table)
    with pytest.raises(TypeError):
        index.attend(q, lens, torch.zeros(2, 2, 3, dtype=torch.int64, device="cuda"), table)
    with pytest.raises(E):
        index.update(lens, table, -1)
    index.bounds = index.bounds[:2]
    with pytest.raises(ValueError):
        index.update(lens, table)
    with pytest.raises(ValueError):
        cache.copy_pages(ints([0, 1]), ints([2]))
    with pytest.raises(TypeError):
        cache.copy_pages(torch.tensor([0]), ints([2]))
    with pytest.raises(E):
        cache.copy_pages(cache.k.view(torch.int32).view(-1)[:4], ints([1, 2, 3, 0]))
    for bad in (torch.zeros(4, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda"), ints([])):
        with pytest.raises(TypeError):
            paged.PagePool.wrap(bad, 16)
    with pytest.raises(ValueError):
        paged.PagePool(4, 0)
    pool = paged.PagePool(8, 16)
    with pytest.raises(ValueError):
        pool.reserve(table, lens, ints([1]))
    with pytest.raises(TypeError):
        pool.reserve(table.long(), lens, lens)
    with pytest.raises(ValueError):
        pool.fork(table, lens, ints([0]), ints([0, 1]))
    with pytest.raises(E):
        pool.free(table, table[:, 0])                          # the lengths lie in the table
    assert [t.numel() for t in pool.fork(table, lens, ints([]), ints([]))] == [0, 0, 0]
    pool.free(table, lens, ints([]))
