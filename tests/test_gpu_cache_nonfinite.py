"""NaN and infinities around the KV cache: where they must have no influence, and where they must not disappear."""
import math

import pytest
import torch

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
