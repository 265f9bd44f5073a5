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


# ---------------------------------------------------------------------------------------
# Draft tokens whose keys are late ones, with numbers that are not finite
# ---------------------------------------------------------------------------------------
def formula(q, k, v, scale):
    """The definition as IEEE arithmetic takes it, 64 bits: q [T, H_q, d], k, v [H, n, d] -> out, lse."""
    T, H_q, d = q.shape
    H, n, _ = k.shape
    out, lse = torch.zeros(T, H_q, d, dtype=torch.float64, device="cuda"), torch.full((T, H_q), -math.inf, dtype=torch.float64, device="cuda")
    for t in range(T):
        seen = n - T + 1 + t
        for h in range(H_q):
            if seen > 0:
                s = (k[h * H // H_q, :seen].double() * q[t, h].double()).sum(-1) * scale
                w = torch.exp(s - s.max())
                out[t, h] = (w.unsqueeze(1) * v[h * H // H_q, :seen].double()).sum(0) / w.sum()
                lse[t, h] = s.max() + (torch.log(w.sum()) if s.max() > -math.inf else 0.0)
    return out, lse


def check_formula(paged, q, k, v, lens, scale):
    """k, v [B, H, rows, d], a page for each sequence.  Where values are not finite, outputs are NaN or infinite, as
    the tensor cores add them up."""
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    out = paged.KVPages.wrap(k, v).attend_shared(q, ints(lens), scale=scale, lse=lse)
    exact = bool(v.isfinite().all())
    for b, n in enumerate(lens):
        want, want_lse = formula(q[b], k[b, :, :n], v[b, :, :n], scale)
        keys, values = k[b, :, :n].nan_to_num(0, 0, 0), v[b, :, :n].nan_to_num(0, 0, 0)
        e_lse, e_out = sref.attention_bound(q[b].nan_to_num(0), keys, values, scale, n, q.dtype)
        assert not exact or torch.equal(out[b].isnan(), want.isnan()), b
        assert torch.equal(lse[b].isnan(), want_lse.isnan()), b
        fine = want.isfinite()
        assert torch.equal(out[b].isfinite(), fine)
        assert bool(((out[b].double() - want).abs() <= e_out + ref.half_step(q.dtype) * want.abs() + 2.0 ** -25)[fine].all()), b
        assert torch.equal(lse[b] == -math.inf, want_lse == -math.inf), b
        fine = want_lse.isfinite()
        assert bool(((lse[b].double() - want_lse).abs() <= e_lse + 2.0 ** -23 * want_lse.abs())[fine].all()), b


@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
@pytest.mark.parametrize("T,lens", [(2, [1, 2, 1, 3, 0]), (5, [1, 4, 5, 3, 6]), (16, [15, 1, 16, 9, 200])])
def test_late_keys_that_are_not_finite(paged, dtype, d, T, lens):
    """Rows whose only keys are late ones: NaN in a key or a query shows, as it does in a tile; -inf is a weight of 0."""
    scale = d ** -0.5
    k, v = randn(1, 5, 2, 256, d, dtype=dtype), randn(2, 5, 2, 256, d, dtype=dtype)
    q = randn(3, 5, T, 4, d, dtype=dtype)
    check_formula(paged, q, k, v, lens, scale)
    for where in (0, max(0, T - 3)):
        for value in (math.nan, math.inf, -math.inf):
            x = k.clone()
            x[:, :, where, 5] = value
            check_formula(paged, q, x, v, lens, scale)
            y = v.clone()
            y[:, :, where, 5] = value
            check_formula(paged, q, k, y, lens, scale)
            if not math.isnan(value):                     # a weight of 0 times an infinite value
                check_formula(paged, q, x, y, lens, scale)
    x = q.clone()
    x[:, T - 1, 2, 7] = math.nan
    check_formula(paged, x, k, v, lens, scale)


@pytest.mark.parametrize("where", [0, 1, 4])
def test_late_keys_with_a_scale_of_zero(paged, where):
    """0 counts as the smallest normal number, of late keys as of others: a score of -inf is a weight of 0."""
    q = randn(3, 3, 5, 4, 64).abs()
    k, v = randn(1, 3, 2, 64, 64), randn(2, 3, 2, 64, 64)
    k[:, :, where, 9] = -math.inf
    lens = [3, 5, 9]
    out = paged.KVPages.wrap(k, v).attend_shared(q, ints(lens), scale=0.0)
    for b, n in enumerate(lens):
        want, _ = formula(q[b], k[b, :, :n], v[b, :, :n], 2.0 ** -126)
        assert torch.equal(out[b].isnan(), want.isnan())
        fine = want.isfinite()
        assert bool(((out[b].double() - want).abs()[fine] <= 3 * ref.half_step(BF) * v.abs().max()).all())


# ---------------------------------------------------------------------------------------
# Pages
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_pages,width,page,old,new", [(3, 12, 4, [0, 1], [36, 1]), (10, 32, 16, [1, 40], [321, 40]), (1, 300, 1, [0, 0], [300, 0]),
                                                        (3, 12, 4, [0, 1], [49, 1])])
def test_reserve_more_than_there_are(paged, n_pages, width, page, old, new):
    """A growth by more pages than the pool has, whose row has room for it or not: none of its new entries keeps a number of
    another sequence's page, and what is missing is counted whole."""
    pool = paged.PagePool(n_pages, page)
    table, lens = torch.zeros(2, width, dtype=torch.int32, device="cuda"), ints(old)
    pool.reserve(table, ints([0, 0]), lens)
    had = [-(-n // page) for n in old]
    table[0, had[0]:] = n_pages - 1                       # left from an earlier sequence
    refs, keep = pool.refs.clone(), table.clone()
    pool.reserve(table, lens, ints(new))
    get = -(-new[0] // page)
    keep[0, had[0]:min(get, width)] = -1
    assert torch.equal(table, keep) and torch.equal(pool.refs, refs)
    assert pool.missing.item() == get - had[0]
    pool.free(table, ints(new), ints([0]))
    refs[table[0, :had[0]].long()] -= 1
    assert torch.equal(pool.refs, refs)


def test_missing_pages_stay_at_the_largest_number(paged):
    pool = paged.PagePool(4, 1)
    table, zero, many = torch.zeros(3, 4, dtype=torch.int32, device="cuda"), ints([0, 0, 0]), ints([2 ** 31 - 1] * 3)
    for _ in range(3):
        pool.reserve(table, zero, many)
        assert pool.missing.item() == 2 ** 31 - 1 and bool((table == -1).all()) and not pool.refs.any()
    pool.missing.zero_()
    pool.reserve(table, zero, ints([4, 1, 2]))            # the second finds none, nor does the third
    assert table.tolist() == [[0, 1, 2, 3], [-1] * 4, [-1] * 4] and pool.missing.item() == 3
    pool.missing.zero_()
    pool.reserve(table, ints([4, 0, 0]), ints([4, 2, 0]))
    assert pool.missing.item() == 2


def test_forks_that_find_no_page_are_counted(paged):
    pool = paged.PagePool(6, 4)
    table, lens = torch.zeros(8, 2, dtype=torch.int32, device="cuda"), ints([5, 3] + [0] * 6)
    pool.reserve(table, torch.zeros_like(lens), lens)
    refs = pool.refs.clone()
    pool.missing.fill_(2 ** 31 - 2)
    src, dst, rows = pool.fork(table, lens, ints([0, 1, 0, 1, 0]), ints([2, 3, 4, 5, 6]))
    assert dst.tolist() == [3, 4, 5, -1, -1] and rows.tolist() == [1, 3, 1, 0, 0] and lens.tolist() == [5, 3, 5, 3, 5, 0, 0, 0]
    assert pool.missing.item() == 2 ** 31 - 1
    assert pool.refs.tolist() == [3, 1, 1, 1, 1, 1]
    pool.free(table, lens, ints([2, 3, 4]))
    assert torch.equal(pool.refs, refs)


def test_copy_pages_of_more_than_2_gib_a_head(paged):
    """Pages as long as a sequence: whole ones, and the first rows of one."""
    page = (1 << 23) + 5
    k, v = (torch.empty(2, 2, page, 128, dtype=BF, device="cuda") for _ in range(2))           # 8.6 GB each
    for x, seed in ((k, 1), (v, 2)):
        x.view(torch.int16).random_(-2 ** 15, 2 ** 15, generator=torch.Generator(device="cuda").manual_seed(seed))
    cache = paged.KVPages.wrap(k, v)
    last = [x[1, :, page - 3:].clone().view(torch.int16) for x in (k, v)]
    cache.copy_pages(ints([0]), ints([1]), ints([page - 3]))
    for x, tail in zip((k, v), last):
        bits = x.view(torch.int16)
        assert torch.equal(bits[0, :, :page - 3], bits[1, :, :page - 3]) and torch.equal(bits[1, :, page - 3:], tail)
        assert not torch.equal(bits[0, :, page - 3:], tail)
    cache.copy_pages(ints([1]), ints([0]))
    for x in (k, v):
        assert torch.equal(x[0].view(torch.int16), x[1].view(torch.int16))


# ---------------------------------------------------------------------------------------
# Many tokens with blocks of their own
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,T,H,G,keep", [(4096, 16, 1, 1, 2), (4095, 16, 1, 2, 1), (512, 1, 2, 4, 3), (100, 4, 3, 2, 5)])
def test_block_attention_of_many_tokens(paged, B, T, H, G, keep):
    """Up to the stated limits: 4096 sequences of one KV head, 16 tokens each."""
    rng = random.Random(B)
    lens = [rng.randint(0, 95) for _ in range(B)]
    pages = 97
    k, v = randn(1, pages, H, 16, 64), randn(2, pages, H, 16, 64)
    table = ints([[rng.randrange(pages) for _ in range(6)] for _ in range(B)])
    cache = paged.KVPages.wrap(k, v)
    index = paged.BlockIndex.wrap(cache, sref.bounds_of(k, 16))
    q = randn(3, B, T, H * G, 64)
    blocks = index.select(q, ints(lens), table, keep=keep, first=0, last=1)
    lse = torch.full((B, T, H * G), 7.0, device="cuda")
    out = index.attend(q, ints(lens), blocks, table, lse=lse)
    some = sorted({*range(0, B, max(1, B // 40)), B - 1})
    for b in some:
        picks = [[sref.select(q[b, t], index.bounds, table, b, lens[b] - T + 1 + t, 16, 16, keep, 0, 1) for t in range(T)]]
        assert [[x.tolist() for x in row] for row in blocks[b]] == [[x + [-1] * (keep - len(x)) for x in row] for row in picks[0]], b
        sref.check_attention(out[b:b + 1], lse[b:b + 1], q[b:b + 1], k, v, table[b:b + 1], [lens[b]], 16, 0.125, picks, 16, case=str(b))
    assert torch.equal(out, index.attend(q, ints(lens), blocks, table))
    assert bool((out.isfinite()).all())


# ---------------------------------------------------------------------------------------
# Sequences that shrink
# ---------------------------------------------------------------------------------------
class Rows:
    """The pool on the host, with lengths that go either way."""

    def __init__(self, paged, n_pages, page, B, width):
        self.host = sref.Pool(n_pages, page, B, width)
        self.pool = paged.PagePool(n_pages, page)
        self.table, self.lens = ints(self.host.table), ints(self.host.lens)

    def reserve(self, new):
        """New lengths are taken where there was room."""
        h = self.host
        self.pool.reserve(self.table, self.lens, ints(new))
        for b, (o, n) in enumerate(zip(h.lens, new)):
            for s in range(min(h.held(n), h.width), min(h.held(o), h.width)):
                if 0 <= h.table[b][s] < len(h.refs):
                    h.refs[h.table[b][s]] -= 1
                h.table[b][s] = -1
        h.reserve(h.lens, new)
        assert self.table.tolist() == h.table and self.pool.refs.tolist() == h.refs and self.pool.missing.item() == h.missing
        for b, n in enumerate(new):
            if h.held(n) <= h.width and -1 not in h.table[b][:h.held(n)]:
                h.lens[b] = n
        self.lens.copy_(ints(h.lens))


@pytest.mark.parametrize("n_pages,page,B,width", [(7, 4, 3, 5), (64, 16, 9, 12), (3000, 16, 40, 100), (5000, 8, 1100, 20)])
def test_reserve_for_rows_that_shrink(paged, n_pages, page, B, width):
    rng = random.Random(n_pages)
    rows = Rows(paged, n_pages, page, B, width)
    for step in range(40):
        rows.reserve([rng.choice([n, n, n + rng.randint(0, 3 * page), max(0, n - rng.randint(0, 3 * page)), rng.randint(-1, width * page)]) for n in rows.host.lens])
        idle = [b for b, n in enumerate(rows.host.lens) if n <= 0]
        busy = [b for b, n in enumerate(rows.host.lens) if n > 0]
        if step % 3 == 0 and idle and busy:               # shared pages: one holder less
            p, c = rng.choice(busy), rng.choice(idle)
            rows.pool.fork(rows.table, rows.lens, ints([p]), ints([c]))
            rows.host.fork([p], [c])
            assert rows.table.tolist() == rows.host.table and rows.lens.tolist() == rows.host.lens
    rows.pool.free(rows.table, rows.lens)
    assert not rows.pool.refs.any()


def test_draft_tokens_that_are_not_accepted(paged):
    """Eight rows more in every step, of which some stay: no page is lost, and a page may go to another sequence at once."""
    rows, page = Rows(paged, 12, 4, 2, 12), 4
    rng = random.Random(3)
    lens = [5, 9]
    rows.reserve(lens)
    while max(lens) <= 16:
        rows.reserve([n + 8 for n in lens])
        lens = [n + rng.randint(1, 3) for n in lens]
        rows.reserve(lens)
        assert rows.pool.missing.item() == 0 and int(rows.pool.refs.sum()) == sum(-(-n // page) for n in lens)
    rows.reserve([48, 0])                                 # all pages, the other's among them
    assert rows.pool.missing.item() == 0 and rows.pool.refs.tolist() == [1] * 12 and rows.table[1].tolist() == [-1] * 5 + rows.table[1, 5:].tolist()
    rows.reserve([-3, 48])
    assert rows.pool.missing.item() == 0 and rows.pool.refs.tolist() == [1] * 12


def test_lengths_beyond_the_row_that_shrink(paged):
    pool = paged.PagePool(8, 4)
    table = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    pool.reserve(table, ints([0]), ints([12]))
    pool.reserve(table, ints([400]), ints([30]))          # both beyond: nothing is held less
    assert table.tolist() == [[0, 1, 2]] and pool.refs.tolist() == [1, 1, 1] + [0] * 5
    pool.reserve(table, ints([400]), ints([5]))
    assert table.tolist() == [[0, 1, -1]] and pool.refs.tolist() == [1, 1] + [0] * 6
    table[0, 1] = 99                                      # no page
    pool.reserve(table, ints([8]), ints([0]))
    assert table.tolist() == [[-1] * 3] and pool.refs.tolist() == [0, 1] + [0] * 6 and pool.missing.item() == 0


def test_tables_without_room(paged):
    """A table of no places is refused by every call, where lengths would have been left as they were; one of no rows has nothing to do."""
    pool, lens = paged.PagePool(4, 4), ints([3, 0])
    table, one = torch.zeros(2, 0, dtype=torch.int32, device="cuda"), ints([0])
    for call in (lambda: pool.reserve(table, lens, lens), lambda: pool.fork(table, lens, one, ints([1])), lambda: pool.free(table, lens),
                 lambda: pool.free(table, lens, one), lambda: pool.compact(table, lens)):
        with pytest.raises(ValueError):
            call()
    none, empty = torch.zeros(0, 5, dtype=torch.int32, device="cuda"), ints([])
    pool.reserve(none, empty, empty)
    pool.free(none, empty)
    pool.free(none, empty, one)
    assert [x.numel() for x in pool.fork(none, empty, empty, empty)] == [0, 0, 0]
    with pytest.raises(ValueError):
        pool.fork(none, empty, one, one)
    with pytest.raises(ValueError):
        pool.compact(none, empty)
    assert lens.tolist() == [3, 0] and not pool.refs.any() and pool.missing.item() == 0


def test_more_sequences_than_the_interface_counts(paged):
    """2^32 + 1 rows are not one."""
    pool = paged.PagePool(4, 4)
    lens = torch.zeros(2 ** 32 + 1, dtype=torch.int32, device="cuda")
    lens[0] = 3
    table = torch.zeros(2 ** 32 + 1, 1, dtype=torch.int32, device="cuda")
    with pytest.raises(paged._rt.RetopkError):
        pool.free(table, lens, ints([0]))
    with pytest.raises(paged._rt.RetopkError):
        pool.reserve(table, lens, lens)
    cache = paged.KVPages(4, 1, 16, 64, "bf16")
    with pytest.raises(paged._rt.RetopkError):
        paged.BlockIndex(cache, 16).update(lens, table)
    assert lens[0].item() == 3


def test_pool_at_its_limits(paged):
    """2^20 pages, 65 535 sequences, 65 535 forks, against a model of whole arrays."""
    import numpy as np
    n_pages, B, page, width = 1 << 20, 65535, 16, 17
    rng = np.random.default_rng(1)
    pool = paged.PagePool(n_pages, page)
    table_d, lens_d = torch.zeros(B, width, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    table, lens, refs = np.zeros((B, width), np.int64), np.zeros(B, np.int64), np.zeros(n_pages, np.int64)
    place = np.arange(width)

    def same():
        assert np.array_equal(table_d.cpu().numpy(), table) and np.array_equal(lens_d.cpu().numpy(), lens)
        assert np.array_equal(pool.refs.cpu().numpy(), refs)

    def reserve(new):
        had, get = -(-lens // page), -(-new // page)
        back = (place >= get[:, None]) & (place < had[:, None])
        np.subtract.at(refs, table[back], 1)
        table[back] = -1
        grown = (place >= had[:, None]) & (place < get[:, None])
        pages = np.flatnonzero(refs <= 0)[:grown.sum()]
        table[grown] = pages
        refs[pages] = 1
        new_d = torch.from_numpy(new).to(device="cuda", dtype=torch.int32)
        pool.reserve(table_d, lens_d, new_d)
        lens[:] = new
        lens_d.copy_(new_d)
        same()

    reserve(rng.integers(0, 16 * page, B))
    reserve(rng.integers(1, 17 * page, B))
    gone = rng.permutation(B)[:B // 2]
    np.subtract.at(refs, table[gone][place < (-(-lens[gone] // page))[:, None]], 1)
    lens[gone] = 0
    pool.free(table_d, lens_d, torch.from_numpy(gone).to(device="cuda", dtype=torch.int32))
    same()
    # every empty row continues a sequence; the other forks have children that are not empty
    parents = rng.choice(np.flatnonzero(lens > 0), B)
    children = np.arange(B)
    made = (lens[children] <= 0) & (lens[parents] > 0)
    made &= ~np.isin(parents, children)                   # (all rows are children: none is made)
    moves = pool.fork(table_d, lens_d, *(torch.from_numpy(x).to(device="cuda", dtype=torch.int32) for x in (parents, children)))
    assert not made.any() and [m.min().item() for m in moves] == [-1, -1, 0] and [m.max().item() for m in moves] == [-1, -1, 0]
    same()
    children = np.where(lens <= 0, np.arange(B), -1)      # forks without a child are left out
    made = children >= 0
    moves = pool.fork(table_d, lens_d, *(torch.from_numpy(x).to(device="cuda", dtype=torch.int32) for x in (parents, children)))
    full, rest = lens[parents] // page, lens[parents] % page
    takes = made & (rest > 0)
    pages = np.full(B, -1)
    pages[takes] = np.flatnonzero(refs <= 0)[:takes.sum()]
    want_src = np.where(takes, table[parents, np.minimum(full, width - 1)], -1)
    assert np.array_equal(moves[0].cpu().numpy(), want_src) and np.array_equal(moves[1].cpu().numpy(), pages)
    assert np.array_equal(moves[2].cpu().numpy(), np.where(takes, rest, 0))
    whole = made[:, None] & (place < full[:, None])
    shared = table[parents]
    np.add.at(refs, shared[whole], 1)
    refs[pages[takes]] = 1
    for mask, values in ((whole, shared), (takes[:, None] & (place == full[:, None]), np.broadcast_to(pages[:, None], (B, width)))):
        rows = np.broadcast_to(children[:, None], (B, width))
        table[rows[mask], np.broadcast_to(place, (B, width))[mask]] = values[mask]
    lens[children[made]] = lens[parents[made]]
    same()
    gone = np.arange(0, B, 3)
    np.subtract.at(refs, table[gone][place < (-(-lens[gone] // page))[:, None]], 1)
    lens[gone] = 0
    pool.free(table_d, lens_d, torch.from_numpy(gone).to(device="cuda", dtype=torch.int32))
    used = refs > 0
    U = int(used.sum())
    movers, holes = np.flatnonzero(used[U:]) + U, np.flatnonzero(~used[:U])
    to = np.arange(n_pages)
    to[movers] = holes
    held = place < (-(-lens // page))[:, None]
    table[held] = to[table[held]]
    refs[holes], refs[movers] = refs[movers], 0
    src, dst = (x.cpu().numpy() for x in pool.compact(table_d, lens_d))
    assert np.array_equal(src[:len(movers)], movers) and np.array_equal(dst[:len(holes)], holes) and (src[len(movers):] == -1).all()
    same()
    reserve(np.minimum(lens + rng.integers(-40, 40, B), width * page).clip(0))
    assert pool.missing.item() == 0


# ---------------------------------------------------------------------------------------
# Caches without a table
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d", [(BF, 128), (FP, 64)])
@pytest.mark.parametrize("rows", [1, 7, 127, 129, 300, 1001])
def test_contiguous_caches_of_any_size(paged, dtype, d, rows):
    """Tiles that end behind a sequence's last row, where the next head's and the next sequence's rows follow."""
    lens = [rows, rows - 1, max(1, rows - 130), rows, 1]
    k, v = randn(1, 5, 3, rows, d, dtype=dtype), randn(2, 5, 3, rows, d, dtype=dtype)
    q = randn(3, 5, 2, 6, d, dtype=dtype)
    cache = paged.KVPages.wrap(k, v)
    lse = torch.full((5, 2, 6), 7.0, device="cuda")
    want = cache.attend_shared(q, ints(lens), lse=lse)
    sref.check_attention(want, lse, q, k, v, None, lens, rows, d ** -0.5)
    for value in (math.nan, math.inf):                    # other heads and sequences, rows behind the last
        x, y = k.clone(), v.clone()
        x[:, 1], y[:, 1] = value, value
        for b, n in enumerate(lens):
            x[b, :, n:], y[b, :, n:] = value, value
        got = paged.KVPages.wrap(x, y).attend_shared(q, ints(lens))
        assert torch.equal(got[:, :, :2], want[:, :, :2]) and torch.equal(got[:, :, 4:], want[:, :, 4:])
    if rows % 16 == 0 or rows < 16:
        return
    # selected blocks in a cache whose size is a multiple of the block
    k, v = k[:, :, :rows // 16 * 16].contiguous(), v[:, :, :rows // 16 * 16].contiguous()
    lens = [min(n, k.shape[2]) for n in lens]
    index = paged.BlockIndex(paged.KVPages.wrap(k, v), 16)
    index.update(ints(lens))
    blocks = index.select(q, ints(lens), keep=4, first=1, last=1)
    picks = [[sref.select(q[b, t], index.bounds, None, b, n - 1 + t, k.shape[2], 16, 4, 1, 1) for t in range(2)] for b, n in enumerate(lens)]
    sref.check_attention(index.attend(q, ints(lens), blocks), None, q, k, v, None, lens, k.shape[2], d ** -0.5, picks, 16)
