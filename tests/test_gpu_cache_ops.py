"""Rotation, append, read-back and attention over 4-bit pages against plain 64-bit forms."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def paged():
    from paper_2607_27692_b200 import build, paged
    build.build()
    return paged


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def close_to_rounding(got, want, dtype):
    """got is `want` (fp64, itself exact to about 2^-45) rounded once, by way of fp32."""
    if want.numel() == 0:
        return
    tiny = torch.finfo(dtype).smallest_normal * ref.half_step(dtype) + 2.0 ** -40 * want.abs().max().item()
    err = (got.double() - want).abs() - (ref.half_step(dtype) * (1 + 2.0 ** -10) * want.abs() + tiny)
    assert err.max().item() <= 0.0, f"off by {err.max().item()} beyond half a step"


# ---------------------------------------------------------------------------------------
# Rotation
# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,rot,interleaved", [
    (128, 128, False), (128, 128, True), (128, 64, False), (128, 32, True), (128, 96, False), (128, 2, False), (128, 10, False),
    (128, 126, True), (64, 64, False), (64, 64, True), (64, 16, False), (64, 40, False), (64, 6, True)])
@pytest.mark.parametrize("n", [1, 37])
def test_rotation(paged, dtype, d, rot, interleaved, n):
    rope = paged.Rope(d, rot, base=500000.0, interleaved=interleaved, scaling="yarn", factor=4.0, original_len=8192)
    w, amp = ref.frequencies(rot, 500000.0, "yarn", 4.0, 8192)
    g = gen(d + rot + n)
    q = torch.randn(n, 5, d, generator=g, device="cuda").to(dtype)
    k = torch.randn(n, 3, d, generator=g, device="cuda").to(dtype)
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = (1 << 20) - 1
    for inverse in (False, True):
        qo, ko = rope.apply_pair(q, k, pos, inverse=inverse)
        close_to_rounding(qo, ref.rotate(q, pos, w, amp, interleaved, inverse), dtype)
        close_to_rounding(ko, ref.rotate(k, pos, w, amp, interleaved, inverse), dtype)
        assert torch.equal(qo[..., rot:], q[..., rot:])


@pytest.mark.parametrize("scaling,factor", [(None, 1.0), ("linear", 4.0), ("ntk", 2.0), ("llama3", 8.0), ("yarn", 4.0)])
def test_rotation_scalings_and_positions(paged, scaling, factor):
    kw = {} if scaling is None else dict(scaling=scaling, factor=factor, original_len=8192)
    rope = paged.Rope(128, **kw)
    w, amp = ref.frequencies(128, 10000.0, scaling, factor, 8192)
    pos = ints([0, 1, -1, 8191, 131071, -131072, (1 << 20) - 1, 2 ** 31 - 1, -2 ** 31])
    x = torch.randn(len(pos), 2, 128, generator=gen(3), device="cuda").to(BF)
    got = rope.apply(x, pos)
    # the reference's angle pos * w in 64 bits is itself off by 2^-53 of up to 2^31
    want = ref.rotate(x, pos, w, amp)
    err = (got.double() - want).abs() - (2.0 ** -8 * (1 + 2.0 ** -10) * want.abs() + 2.0 ** -20)
    assert err.max().item() <= 0
    assert scaling == "yarn" or torch.equal(got[0], x[0])


def test_rotation_many_tokens_strided_and_in_place(paged):
    """Tokens enough for several per CTA; q and k as slices of one projection, rotated where they lie."""
    n, H_q, H_k, d = 9001, 4, 2, 64
    rope = paged.Rope(d, 48, interleaved=False)
    w, amp = ref.frequencies(48)
    qkv = torch.randn(n, H_q + 2 * H_k, d, generator=gen(5), device="cuda").to(BF)
    before = qkv.clone()
    q, k, v = qkv.split([H_q, H_k, H_k], 1)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    apart = rope.apply_pair(q, k, pos)
    rope.apply_pair(q, k, pos, q_out=q, k_out=k)
    assert torch.equal(q, apart[0]) and torch.equal(k, apart[1]) and torch.equal(v, before[:, H_q + H_k:])
    close_to_rounding(q, ref.rotate(before[:, :H_q], pos, w, amp), BF)
    close_to_rounding(k, ref.rotate(before[:, H_q:H_q + H_k], pos, w, amp), BF)
    # an odd rotated part, whose partners cross lanes, in place too
    rope = paged.Rope(d, 50)
    x = before[:, :3].clone()
    assert torch.equal(rope.apply(x, pos, out=x), rope.apply(before[:, :3].contiguous(), pos))
    assert rope.apply(x[:0], pos[:0]).shape == (0, 3, d)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_gradient(paged, interleaved):
    """inverse=True is the gradient: of the 64-bit formula by autograd, and by differences of the kernel."""
    n, H, d, rot = 7, 3, 64, 32
    rope = paged.Rope(d, rot, interleaved=interleaved, scaling="yarn", factor=4.0, original_len=64)
    w, amp = ref.frequencies(rot, 10000.0, "yarn", 4.0, 64)
    g = gen(11)
    x = torch.randn(n, H, d, generator=g, device="cuda").to(FP)
    up = torch.randn(n, H, d, generator=g, device="cuda").to(FP)
    pos = ints(list(range(100, 100 + n)))
    y = x.double().requires_grad_()
    (ref.rotate(y, pos, w, amp, interleaved) * up.double()).sum().backward()
    got = rope.apply(up, pos, inverse=True)
    close_to_rounding(got, y.grad, FP)
    # the map is linear: f(x + h) - f(x - h) = 2 f(h), so powers of two give differences without a remainder
    for c in (0, 1, rot // 2, rot - 1, d - 1):
        e = torch.zeros_like(x)
        e[..., c] = 0.5
        diff = (rope.apply(e, pos).double() - rope.apply(-e, pos).double()) * up.double()
        # each output is rounded once: 2^-11 of each term
        bound = 2.0 ** -10 * diff.abs().sum(-1) + 2.0 ** -11 * got[..., c].double().abs() + 2.0 ** -14
        assert ((diff.sum(-1) - got[..., c].double()).abs() <= bound).all()


# ---------------------------------------------------------------------------------------
# Append and read back
# ---------------------------------------------------------------------------------------
def table_for(lens, page, seed, spare=3):
    need = [max(1, -(-n // page)) for n in lens]
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(sum(need) + spare, generator=g).tolist()
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [10 ** 9] * (max(need) - n))       # beyond a sequence: never looked at
        at += n
    return ints(table), sum(need) + spare


def new_rows(news, H_q, H, d, dtype, seed, pad=0):
    n = sum(news) + pad
    x = torch.randn(n, H_q + 2 * H, d, generator=gen(seed), device="cuda")
    x[:, H_q, :3] *= 8
    return x.to(dtype).split([H_q, H, H], 1)


def sentinel(pages):
    for t in (pages.k, pages.v, pages.k_scale, pages.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(0x5A)


@pytest.mark.parametrize("fmt,dtype", [("bf16", BF), ("fp16", FP), ("q4", BF), ("q4", FP)])
@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (128, 64, False), (128, 32, True), (128, 20, False), (64, 64, True), (64, 16, False)])
@pytest.mark.parametrize("news,pasts,page", [([1, 1, 1], [0, 15, 700], 16), ([5, 0, 130, 1, 17], [0, 9, 31, 63, 2000], 64)])
def test_append(paged, fmt, dtype, d, rot, interleaved, news, pasts, page):
    H_q, H, pad = 6, 2, 3
    B, lens = len(news), [a + b for a, b in zip(news, pasts)]
    table, total = table_for(lens, page, 7)
    cache = paged.KVPages(total, H, page, d, fmt)
    sentinel(cache)
    start = {n: getattr(cache, n).clone() for n in ("k", "v", "k_scale", "v_scale") if getattr(cache, n) is not None}
    q, k, v = new_rows(news, H_q, H, d, dtype, 21, pad)
    cu = ints([sum(news[:b]) for b in range(B + 1)])
    rope = paged.Rope(d, rot, interleaved=interleaved)
    w, amp = ref.frequencies(rot)
    q_out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
    assert cache.append(k, v, ints(lens), table, cu, rope=rope, q=q, q_out=q_out) is q_out
    n = sum(news)
    pos = ints([p + i for p, m in zip(pasts, news) for i in range(m)])
    close_to_rounding(q_out[:n], ref.rotate(q[:n], pos, w, amp, interleaved), dtype)
    assert (q_out[n:] == 7.0).all(), "rows behind the last sequence were written"
    k_rot = ref.rotate(k[:n], pos, w, amp, interleaved)
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(news, device="cuda"))
    ids, row = table[seq, pos.long() // page].long(), pos.long() % page
    touched = torch.zeros(cache.k.shape[:3], dtype=torch.bool, device="cuda")
    touched[ids, :, row] = True
    for name, x in start.items():
        assert torch.equal(getattr(cache, name)[~touched], x[~touched]), f"{name}: rows of other tokens changed"
    if fmt != "q4":
        close_to_rounding(cache.k[ids, :, row], k_rot, dtype)
        assert torch.equal(cache.v[ids, :, row], v[:n])
        return
    # exact but for keys whose 64-bit rotation lies within 2^-45 of a rounding border: none of these
    for x, name in ((k_rot.to(dtype), "k"), (v[:n], "v")):
        codes, step, low = ref.quantise(x)
        got_scale = getattr(cache, name + "_scale")[ids, :, row].double()
        assert torch.equal(got_scale[..., 0], step) and torch.equal(got_scale[..., 1], low)
        assert torch.equal(getattr(cache, name)[ids, :, row], ref.pack(codes))
        # and what a code stands for is within half a step of what was stored, plus what rounding the
        # minimum (half a bf16 step of it) and a rounded-down step (15 codes of 2^-8 of it) leave out
        vals = ref.values(ref.pack(codes), got_scale).unflatten(-1, (-1, 64))
        slack = (0.5 + 15 * 2.0 ** -8) * step + 2.0 ** -8 * low.abs()
        assert ((vals - x.double().unflatten(-1, (-1, 64))).abs() <= slack.unsqueeze(-1) * (1 + 2.0 ** -20)).all()


@pytest.mark.parametrize("dtype", [BF, FP])
def test_quantiser_corners(paged, dtype):
    """Constant groups, zeros, tiny and huge spans, exact ties."""
    d, rows = 64, []
    f = torch.finfo(dtype)
    rows.append(torch.zeros(d))
    rows.append(torch.full((d,), 3.14159))
    rows.append(torch.full((d,), -f.smallest_normal))
    rows.append(torch.linspace(-1, 1, d) * f.smallest_normal)
    rows.append(torch.linspace(-0.4, 0.4, d) * min(f.max, 1e38))
    rows.append(torch.arange(d).float() / 4 - 8)                      # step 1.0625: ties where the type allows them
    rows.append((torch.arange(d) % 31).float() / 2)                   # span 15, step 1: every other value is a tie
    rows.append(torch.cat((torch.full((d - 1,), 1.0), torch.tensor([1.0 + f.eps]))))
    x = torch.stack(rows).to(dtype).cuda().view(len(rows), 1, d)
    cache = paged.KVPages(1, 1, 16, d, "q4")
    cache.append(x, x, ints([len(rows)]))
    codes, step, low = ref.quantise(x)
    for name in ("k", "v"):
        got = getattr(cache, name + "_scale")[0, 0, :len(rows)].double()
        assert torch.equal(got[..., 0], step[:, 0]) and torch.equal(got[..., 1], low[:, 0])
        assert torch.equal(getattr(cache, name)[0, 0, :len(rows)], ref.pack(codes)[:, 0])
    assert step[0].item() == 0 and codes[0].max() == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
def test_quantiser_many_values(paged, dtype, d):
    """Four million values of steps from 2^-100 to 2^100: every code as a 64-bit division rounds it, ties among them."""
    n, H, page = 4096, 8 * 64 // d * 2, 64
    g = gen(d)
    x = torch.randn(n, H, d, generator=g, device="cuda")
    if dtype == BF:
        x = x * torch.exp2(torch.randint(-100, 100, (n, H, 1), generator=g, device="cuda").float())
    else:
        x = x * torch.exp2(torch.randint(-12, 12, (n, H, 1), generator=g, device="cuda").float())
    x[: n // 2] = (x[: n // 2] * 4).round() / 4 * x[: n // 2, :, :1].abs().clamp_min(2.0 ** -90)     # coarse grids: ties
    x[::3] += 5 * x[::3, :, :1]                                                                       # minima far from zero
    x = x.to(dtype)
    cache = paged.KVPages(n // page, H, page, d, "q4")
    cache.append(x, x.flip(0).contiguous(), ints([n]), torch.arange(n // page, dtype=torch.int32, device="cuda")[None])
    codes, step, low = ref.quantise(x)
    # infinities, and spans beyond the fp32 range, are outside what is specified: their groups are left out
    span = x.float().unflatten(-1, (-1, 64)).amax(-1) - low.float()
    fine = torch.isfinite(x).unflatten(-1, (-1, 64)).all(-1) & torch.isfinite(span)
    assert fine.float().mean().item() > 0.8
    for name, c, s, m, ok in (("k", codes, step, low, fine), ("v", codes.flip(0), step.flip(0), low.flip(0), fine.flip(0))):
        got = getattr(cache, name).transpose(1, 2).reshape(n, H, d // 64, 32)
        scale = getattr(cache, name + "_scale").transpose(1, 2).reshape(n, H, d // 64, 2).double()
        assert torch.equal(scale[..., 0][ok], s[ok]) and torch.equal(scale[..., 1][ok], m[ok])
        assert torch.equal(got[ok], ref.pack(c).unflatten(-1, (-1, 32))[ok])


@pytest.mark.parametrize("fmt", ["bf16", "q4"])
def test_append_what_points_outside_is_left_out(paged, fmt):
    """Idle sequences, bad pages and positions beyond the table: skipped, nothing else changes."""
    H, d, page = 2, 128, 16
    table = ints([[0, 1], [2, -1], [99, 3], [4, 5], [2 ** 31 - 1, -2 ** 31]])
    lens = ints([0, 17, 2, 40, 3])              # idle | bad second page | bad first page | beyond 32 rows | bad pages
    cache = paged.KVPages(6, H, page, d, fmt)
    sentinel(cache)
    start = [t.clone() for t in (cache.k, cache.v)]
    rope = paged.Rope(d)
    q, k, v = new_rows([2] * 5, 4, H, d, BF, 31)
    q_out = torch.full(q.shape, 7.0, dtype=BF, device="cuda")
    cache.append(k, v, lens, table, rope=rope, q=q, q_out=q_out)
    assert (q_out[:2] == 7.0).all() and not (q_out[2:] == 7.0).all(-1).any()
    touched = torch.zeros(cache.k.shape[:3], dtype=torch.bool, device="cuda")
    touched[2, :, 15] = True                    # sequence 1: position 15 is stored, 16 is not
    assert torch.equal(cache.k[~touched], start[0][~touched]) and torch.equal(cache.v[~touched], start[1][~touched])
    assert not torch.equal(cache.v[touched], start[1][touched])
    # as long as the length minus the new tokens is negative, the first of them have no place
    cache.append(k[:5], v[:5], ints([1, 1, 1, 1, 1]), table)
    assert not torch.equal(cache.k[0, :, 0], start[0][0, :, 0])


@pytest.mark.parametrize("fmt,src", [("bf16", BF), ("fp16", FP), ("q4", BF)])
@pytest.mark.parametrize("out", [BF, FP, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_gather(paged, fmt, src, out, d):
    H, page, lens = 3, 48, [0, 1, 47, 48, 49, 333]
    table, total = table_for(lens, page, 9)
    cache = paged.KVPages(total, H, page, d, fmt)
    _, k, v = new_rows(lens, 1, H, d, src, 41)
    cu = ints([sum(lens[:b]) for b in range(len(lens) + 1)])
    cache.append(k, v, ints(lens), table, cu)
    first = [0, 0, 5, 48, 48, 100]
    rows = 200
    ko = torch.full((len(lens), H, rows, d), 7.0, dtype=out, device="cuda")
    vo = ko.clone()
    if fmt != "q4" and out not in (src, torch.float32):
        with pytest.raises(Exception):
            cache.gather(ko, vo, ints(lens), table)
        return
    cache.gather(ko, vo, ints(lens), table, first=ints(first))
    for b, n in enumerate(lens):
        m = min(max(0, n - first[b]), rows)
        for got, name in ((ko, "k"), (vo, "v")):
            want = ref.rows_of(getattr(cache, name), getattr(cache, name + "_scale"), table, b, n, page)[:, first[b]:first[b] + m]
            if out == torch.float32:
                assert ((got[b, :, :m].double() - want).abs() <= 2.0 ** -24 * want.abs()).all()
            elif fmt != "q4":
                assert torch.equal(got[b, :, :m].double(), want)
            else:
                close_to_rounding(got[b, :, :m], want, out)
            assert (got[b, :, m:] == 7.0).all(), "rows beyond the sequence were written"
    # rows before the first: left alone, the rest of the sequence behind them, beyond the table's width too
    wide = torch.full((len(lens), H, 400, d), 7.0, dtype=out, device="cuda")
    cache.gather(wide, None, ints(lens), table, first=ints([-60] * len(lens)))
    assert (wide[:, :, :60] == 7.0).all() and torch.equal(wide[5, :, 160:360], ko[5]) and (wide[5, :, 393:] == 7.0).all()
    # one output alone, and pages that do not exist
    ko2 = torch.full_like(ko, 7.0)
    cache.gather(ko2, None, ints(lens), table, first=ints(first))
    assert torch.equal(ko2, ko)
    bad = table.clone()
    bad[5, 3] = total
    ko2.fill_(7.0)
    cache.gather(ko2, None, ints(lens), bad, first=ints(first))
    assert (ko2[5, :, 144 - 100:192 - 100] == 7.0).all() and torch.equal(ko2[5, :, :44], ko[5, :, :44])


# ---------------------------------------------------------------------------------------
# Attention over 4 bits
# ---------------------------------------------------------------------------------------
def filled(paged, lens, page, H, d, seed, wild=True):
    """A cache with random rows; rows behind a sequence's end hold NaN patterns."""
    table, total = table_for(lens, page, seed)
    cache = paged.KVPages(total, H, page, d, "q4")
    g = gen(seed)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    for t in (cache.k_scale, cache.v_scale):
        t[..., 0] = torch.rand(t.shape[:-1], generator=g, device="cuda").mul(0.4).add(0.01).to(BF)
        t[..., 1] = torch.randn(t.shape[:-1], generator=g, device="cuda").sub(2.0).to(BF)
    if wild:
        for b, n in enumerate(lens):
            if n % page:
                for t in (cache.k_scale, cache.v_scale):
                    t[table[b, n // page].item(), :, n % page:] = math.nan
                for t in (cache.k, cache.v):
                    t[table[b, n // page].item(), :, n % page:] = 255
    return cache, table


def check_attention(cache, q, lens, table, out, lse, scale, window=0, bad=None):
    page, d = cache.page_size, cache.d
    T = q.shape[1]
    for b, n in enumerate(lens):
        k = ref.rows_of(cache.k, cache.k_scale, table, b, n, page)
        v = ref.rows_of(cache.v, cache.v_scale, table, b, n, page)
        ok = None if bad is None else ~bad[b][:n]
        want, want_lse = ref.attention(q[b], k, v, scale, window, ok)
        if n == 0:
            assert (out[b] == 0).all() and (lse is None or (lse[b] == -math.inf).all())
            continue
        ids = table[b, :-(-n // page)].long()
        ids = ids[(ids >= 0) & (ids < cache.n_pages)]
        ks, vs = cache.k_scale[ids].nan_to_num(), cache.v_scale[ids].nan_to_num()
        if ok is not None:
            v = v * ok[None, :, None]
        e_lse, e_out = ref.attention_bounds(q[b], ks, vs, v, scale, n, q.dtype)
        err = (out[b].double() - want).abs() - (ref.half_step(q.dtype) * (1 + 2.0 ** -10) * want.abs() + e_out)
        assert err.max().item() <= 0, f"sequence {b} of {n} keys: off by {err.max().item()} beyond the bound"
        # far below the worst case on average: one rounding of the output and the weights' 2^-16
        rms = (out[b].double() - want).square().mean().sqrt().item()
        size = want.square().mean().sqrt().item()
        assert rms <= ref.half_step(q.dtype) * size + e_out, f"sequence {b}: rms {rms} of {size}"
        if lse is not None:
            none = want_lse == -math.inf
            assert torch.equal(lse[b] == -math.inf, none)
            assert ((lse[b].double() - want_lse).abs()[~none] <= e_lse + 2.0 ** -23 * want_lse.abs()[~none]).all()


LENS = [0, 1, 15, 16, 17, 127, 128, 129, 300, 1025]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,G,T", [(2, 1, 1), (2, 4, 1), (3, 3, 1), (1, 8, 1), (2, 16, 1), (2, 5, 1), (1, 4, 3), (2, 1, 7), (2, 6, 2),
                                   (1, 16, 2), (1, 3, 11), (1, 16, 16)])
def test_attention(paged, dtype, d, H, G, T):
    page = 48
    cache, table = filled(paged, LENS, page, H, d, 51)
    q = torch.randn(len(LENS), T, H * G, d, generator=gen(52), device="cuda").to(dtype)
    lse = torch.full(q.shape[:-1], 7.0, device="cuda")
    out = torch.full_like(q, 7.0)
    assert cache.attend(q, ints(LENS), table, out=out, lse=lse) is out
    check_attention(cache, q, LENS, table, out, lse, d ** -0.5)


@pytest.mark.parametrize("T,window", [(1, 1), (1, 16), (1, 100), (1, 5000), (4, 1), (4, 33), (3, 1 << 40)])
@pytest.mark.parametrize("d,G", [(64, 4), (128, 8)])
def test_attention_window(paged, T, window, d, G):
    lens, page = [1, 2, 40, 130, 1000, 2049], 16
    cache, table = filled(paged, lens, page, 2, d, 61)
    q = torch.randn(len(lens), T, 2 * G, d, generator=gen(62), device="cuda").to(BF)
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, scale=0.3, window=window, lse=lse)
    check_attention(cache, q, lens, table, out, lse, 0.3, window)


@pytest.mark.parametrize("page", [16, 112, 4096])
@pytest.mark.parametrize("lens", [[40000], [20000, 3, 0, 9000, 129], [100] * 40, [0, 0, 0], [5000, 4999] * 4])
def test_attention_shares(paged, page, lens):
    """Sequences that many CTAs share, CTAs that work on many sequences, nothing to do at all."""
    cache, table = filled(paged, lens, page, 2, 128, 71)
    q = torch.randn(len(lens), 1, 8, 128, generator=gen(72), device="cuda").to(BF)
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, lse=lse)
    check_attention(cache, q, lens, table, out, lse, 128 ** -0.5)
    again = cache.attend(q, ints(lens), table)
    assert torch.equal(out, again), "not bit-reproducible"


@pytest.mark.parametrize("B", [129, 300, 2000])
def test_many_sequences(paged, B):
    """More sequences than a warp looks at at once: append, read back and attend, empty and idle ones among them."""
    H, d, page = 2, 64, 16
    g = torch.Generator().manual_seed(B)
    news = torch.randint(0, 4, (B,), generator=g).tolist()
    pasts = [0 if i % 7 == 0 else int(x) for i, x in enumerate(torch.randint(0, 90, (B,), generator=g))]
    news[0] = news[-1] = 0
    lens = [a + b for a, b in zip(news, pasts)]
    cache, table = filled(paged, [100] * B, page, H, d, 111, wild=False)
    _, k, v = new_rows(news, 1, H, d, BF, 112)
    cu = ints([0] + torch.tensor(news).cumsum(0).tolist())
    cache.append(k, v, ints(lens), table, cu)
    most = max(news)
    ko, vo = torch.zeros(B, H, most, d, device="cuda"), torch.zeros(B, H, most, d, device="cuda")
    cache.gather(ko, vo, ints(lens), table, first=ints(pasts))
    at = torch.cat([torch.arange(n) for n in news]).cuda()
    seq = torch.repeat_interleave(torch.arange(B), torch.tensor(news)).cuda()
    for x, out in ((k, ko), (v, vo)):
        c, st, m = ref.quantise(x)
        want = ref.values(ref.pack(c), torch.stack((st, m), -1))
        assert ((out[seq, :, at].double() - want).abs() <= 2.0 ** -23 * want.abs()).all()
    q = torch.randn(B, 1, 2 * H, d, generator=gen(113), device="cuda").to(BF)
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, lse=lse)
    some = sorted({0, 1, 2, 127, 128, B // 2, B - 2, B - 1} | set(range(0, B, 97)))
    check_attention(cache, q[some], [lens[b] for b in some], table[some], out[some], lse[some], d ** -0.5)
    assert torch.equal(out, cache.attend(q, ints(lens), table)) and torch.isfinite(out.float()).all()


def test_attention_weights_of_far_keys(paged):
    """Scores that grow along the sequence and others that fall: the running reference has to move, late and often."""
    lens, page, d = [3000, 3000, 3000], 32, 64
    cache, table = filled(paged, lens, page, 1, d, 81)
    ramp = torch.linspace(0, 1, 3000, device="cuda")
    for b, r in enumerate((ramp, 1 - ramp, (ramp * 40).frac())):
        j = torch.arange(3000, device="cuda")
        cache.k_scale[table[b].long()[j // page], 0, j % page, 0, 1] = (r * 4).to(BF)
    q = torch.full((3, 1, 4, d), 0.9, device="cuda").to(BF)
    q[:, :, 1] *= -1
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, lse=lse)
    check_attention(cache, q, lens, table, out, lse, d ** -0.5)


@pytest.mark.parametrize("dtype,G", [(FP, 4), (BF, 4), (FP, 7)])
def test_attention_long_flat(paged, dtype, G):
    """A quarter of a million keys of much the same weight: the result is the little that is left of large sums."""
    lens, page, d = [262144], 128, 128
    cache, table = filled(paged, lens, page, 1, d, 85)
    q = (0.05 * torch.randn(1, 1, G, d, generator=gen(86), device="cuda")).to(dtype)
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, lse=lse)
    check_attention(cache, q, lens, table, out, lse, d ** -0.5)
    want, _ = ref.attention(q[0], *(ref.rows_of(t, s, table, 0, lens[0], page) for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))), d ** -0.5)
    # systematic part: 12 additions cut off by 2^-23 at most, of sums that grow to 16 steps (half on
    # average); steps are 0.21 on average here
    rms = (out[0].double() - want).square().mean().sqrt().item()
    assert rms <= ref.half_step(dtype) * want.square().mean().sqrt().item() + 12 * 2.0 ** -23 * 8 * 0.21


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
@pytest.mark.parametrize("G", [1, 7])
def test_attention_scales(paged, scale, G):
    lens = [5, 260]
    cache, table = filled(paged, lens, 16, 2, 64, 89)
    q = torch.randn(2, 1, 2 * G, 64, generator=gen(90), device="cuda").to(BF)
    q[0, 0, 0] = 0.0
    q[1, 0, 0] *= 2.0 ** -40
    q[1, 0, G] *= 2.0 ** 20 if scale == 0.0 else 1.0
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, scale=scale, lse=lse)
    check_attention(cache, q, lens, table, out, lse, scale)


def test_attention_pages_out_of_range(paged):
    lens, page, d = [200, 64, 33], 16, 128
    cache, table = filled(paged, lens, page, 2, d, 91)
    table = table.clone()
    table[0, 3], table[0, 7], table[1, :] = -1, cache.n_pages, 2 ** 31 - 1
    bad = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in lens]
    bad[0][48:64], bad[0][112:128] = True, True
    bad[1][:] = True
    q = torch.randn(3, 2, 8, d, generator=gen(92), device="cuda").to(BF)
    lse = torch.empty(q.shape[:-1], device="cuda")
    out = cache.attend(q, ints(lens), table, lse=lse)
    safe = table.clamp(0, cache.n_pages - 1)
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    keep = [0, 2]
    check_attention(cache, q[keep], [lens[b] for b in keep], safe[keep], out[keep], lse[keep], d ** -0.5, 0, [bad[b] for b in keep])
    # lengths beyond the block table end with it, negative ones are empty
    short = cache.attend(q, ints([64, -5, 10 ** 9]), table[:, :4].contiguous())
    assert (short[1] == 0).all() and torch.isfinite(short.float()).all()


def test_attention_strided_queries_and_contiguous_cache(paged):
    """Queries as a slice of a projection; a cache without a block table; one head's row alone."""
    B, H, G, d = 3, 2, 4, 64
    lens = [50, 128, 31]
    cache, table = filled(paged, [128] * B, 128, H, d, 95, wild=False)
    plain = paged.KVPages.wrap(*(t[table[:, 0].long()].contiguous() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
    qkv = torch.randn(B, H * G + 2 * H, d, generator=gen(96), device="cuda").to(BF)
    q = qkv[:, :H * G]
    a = plain.attend(q, ints(lens))
    b = cache.attend(q.contiguous(), ints(lens), table)
    assert torch.equal(a, b) and a.shape == (B, H * G, d)
    four = qkv.unsqueeze(1)[:, :, :H * G]
    assert torch.equal(plain.attend(four, ints(lens))[:, 0], a)
    with pytest.raises(ValueError):
        plain.attend(qkv[:, ::2], ints(lens))


def test_offsets_beyond_32_bits(paged):
    """Pages more than 4 GiB into the codes: append, read back, attend."""
    H, page, d, dt = 8, 64, 128, BF
    n_pages = (5 << 30) // (H * page * d // 2)
    k = torch.empty((n_pages, H, page, d // 2), dtype=torch.uint8, device="cuda")
    v = torch.empty_like(k)
    ks = torch.empty((n_pages, H, page, d // 64, 2), dtype=BF, device="cuda")
    cache = paged.KVPages.wrap(k, v, ks, torch.empty_like(ks))
    lens = [100, 64]
    table = ints([[n_pages - 1, n_pages - 3], [n_pages - 2, 0]])
    q, kn, vn = new_rows(lens, 8, H, d, dt, 97)
    cache.append(kn, vn, ints(lens), table, ints([0, 100, 164]))
    want_k, want_v = (ref.values(ref.pack(c), torch.stack((s, m), -1)) for c, s, m in map(ref.quantise, (kn, vn)))
    ko = torch.zeros(2, H, 100, d, device="cuda")
    cache.gather(ko, None, ints(lens), table)
    assert ((ko[0].double() - want_k[:100].transpose(0, 1)).abs() <= 2.0 ** -23 * want_k[:100].transpose(0, 1).abs()).all()
    x = q[:2].unsqueeze(1).contiguous()
    out = cache.attend(x, ints(lens), table)
    check_attention(cache, x, lens, table, out, None, d ** -0.5)


# ---------------------------------------------------------------------------------------
# As they are used
# ---------------------------------------------------------------------------------------
def test_decode_loop_in_four_bits(paged):
    """Prompt, then single tokens, then draft tokens: rotate, append, attend; against 64 bits throughout."""
    H_q, H, d, page, B = 8, 2, 128, 16, 3
    rope = paged.Rope(d, base=500000.0, scaling="llama3", factor=8.0, original_len=8192)
    w, amp = ref.frequencies(d, 500000.0, "llama3", 8.0, 8192)
    table, total = table_for([200] * B, page, 5)
    cache = paged.KVPages(total, H, page, d, "q4")
    prompts, lens = [37, 160, 5], [0, 0, 0]
    hist = [[[], []] for _ in range(B)]
    for step, news in enumerate([prompts, [1] * 3, [1] * 3, [4] * 3, [1] * 3]):
        lens = [a + b for a, b in zip(lens, news)]
        q, k, v = new_rows(news, H_q, H, d, BF, 100 + step)
        cu = ints([sum(news[:b]) for b in range(B + 1)])
        even = len(set(news)) == 1
        qr = cache.append(k, v, ints(lens), table, None if even else cu, rope=rope, q=q)
        pos = ints([n - m + i for n, m in zip(lens, news) for i in range(m)])
        kr = ref.rotate(k, pos, w, amp).to(BF)
        for b in range(B):
            lo, hi = sum(news[:b]), sum(news[:b + 1])
            for x, h in ((kr, hist[b][0]), (v, hist[b][1])):
                c, s, m = ref.quantise(x[lo:hi])
                h.append(ref.values(ref.pack(c), torch.stack((s, m), -1)))
        if not even:
            continue
        T = news[0]
        qq = qr.view(B, T, H_q, d)
        lse = torch.empty(B, T, H_q, device="cuda")
        out = cache.attend(qq, ints(lens), table, lse=lse)
        check_attention(cache, qq, lens, table, out, lse, d ** -0.5)
        for b in range(B):          # and what the cache holds is what was quantised from the start
            want, _ = ref.attention(qq[b], torch.cat(hist[b][0]).transpose(0, 1), torch.cat(hist[b][1]).transpose(0, 1), d ** -0.5)
            assert (out[b].double() - want).abs().max().item() <= 2.0 ** -8 * want.abs().max().item() + 2e-3


def test_feeds_the_retopk_decode_step(paged):
    """Prompt and tokens appended, rotated, into the decode step's cache; and brought there from 4-bit pages."""
    from paper_2607_27692_b200 import retopk as rt
    B, H_q, H, d, S = 2, 8, 2, 128, 512
    rope = paged.Rope(d)
    w, amp = ref.frequencies(d)
    k_cache = torch.zeros(B, H, S, d, dtype=BF, device="cuda")
    v_cache = torch.zeros_like(k_cache)
    cache = paged.KVPages.wrap(k_cache, v_cache)
    want_k, want_v = torch.zeros_like(k_cache), torch.zeros_like(k_cache)
    ours = rt.ReTopK(B, H_q, H, d, 16, 2, 32, 64, 0.85, 16, S)
    other = rt.ReTopK(B, H_q, H, d, 16, 2, 32, 64, 0.85, 16, S)
    n = 300
    _, k, v = new_rows([n] * B, H_q, H, d, BF, 201)
    cache.append(k, v, ints([n] * B), rope=rope)
    want_k[:, :, :n] = ref.rotate(k, ints(list(range(n)) * B), w, amp).to(BF).view(B, n, H, d).transpose(1, 2)
    want_v[:, :, :n] = v.reshape(B, n, H, d).transpose(1, 2)
    for step in range(6):
        q, k, v = new_rows([1] * B, H_q, H, d, BF, 300 + step)
        n += 1
        qr = cache.append(k, v, ints([n] * B), rope=rope, q=q)
        want_k[:, :, n - 1] = ref.rotate(k, ints([n - 1] * B), w, amp).to(BF)
        want_v[:, :, n - 1] = v
        want_q = ref.rotate(q, ints([n - 1] * B), w, amp).to(BF).contiguous()
        assert torch.equal(k_cache, want_k) and torch.equal(v_cache, want_v) and torch.equal(qr, want_q)
        assert torch.equal(ours.decode_step(qr, k_cache, v_cache, n), other.decode_step(want_q, want_k, want_v, n))
    # 4-bit pages -> the decode step's cache; a support of all keys makes it dense attention
    lens = [150, 150]
    q4, table = filled(paged, lens, 16, H, d, 210)
    q4.gather(k_cache, v_cache, ints(lens), table)
    dense = rt.ReTopK(B, H_q, H, d, 4, 1, 0, 256, 2.0, 0, S)
    got = dense.exact_topk_decode(qr, k_cache, v_cache, 150)
    wide = q4.attend(qr, ints(lens), table)
    for b in range(B):
        want, _ = ref.attention(qr[b:b + 1], k_cache[b, :, :150].double(), v_cache[b, :, :150].double(), d ** -0.5)
        assert ((got[b].double() - want[0]).abs() <= 2e-2 + 1e-2 * want[0].abs()).all()
        # the same values before their rounding to bf16: scores move by 2^-8 of sum |q k|
        k64 = ref.rows_of(q4.k, q4.k_scale, table, b, 150, 16)
        shift = 2.0 ** -8 * (qr[b].double().abs().view(H, -1, d) @ k64.abs().transpose(1, 2)).max().item() * d ** -0.5
        spread = 2 * k_cache[b].abs().max().item() + 2 * v_cache[b].abs().max().item()
        assert ((wide[b].double() - want[0]).abs() <= (2 * shift + 2.0 ** -7) * spread).all()


def test_streams_and_graphs(paged):
    """A captured run of the operators replays like the eager one, and two streams at once do not meet."""
    H_q, H, d, page, B = 8, 2, 128, 16, 2
    rope = paged.Rope(d)
    lens0 = [1000, 77]
    caches = [filled(paged, [1200, 1200], page, H, d, s, wild=False) for s in (1, 2)]
    x = [torch.randn(B, H_q + 2 * H, d, generator=gen(s), device="cuda").to(BF) for s in (3, 4)]
    lens = [ints(lens0) for _ in range(2)]

    def step(i):
        c, t = caches[i]
        q, k, v = x[i].split([H_q, H, H], 1)
        return c.attend(c.append(k, v, lens[i], t, rope=rope, q=q), lens[i], t)

    want = [step(i).clone() for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(i))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i])
    # replays follow the lengths on the device
    for i in range(2):
        lens[i].copy_(ints([1001, 500]))
    fresh = [step(i).clone() for i in range(2)]
    for i in range(2):
        graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], fresh[i]) and not torch.equal(outs[i], want[i])
    # eager calls on two streams at once
    res = [None, None]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                res[i] = step(i)
    torch.cuda.synchronize()
    assert torch.equal(res[0], fresh[0]) and torch.equal(res[1], fresh[1])


def test_binding_refusals(paged):
    cache = paged.KVPages(4, 2, 16, 64, "q4")
    half = paged.KVPages(4, 2, 16, 64, "bf16")
    q = torch.zeros(2, 4, 64, dtype=BF, device="cuda")
    k = torch.zeros(2, 2, 64, dtype=BF, device="cuda")
    lens, table = ints([1, 1]), ints([[0], [1]])
    with pytest.raises(TypeError):
        half.attend(q, lens, table)
    with pytest.raises(TypeError):
        cache.attend(q.float(), lens, table)
    with pytest.raises(TypeError):
        cache.attend(q, lens.long(), table)
    with pytest.raises(ValueError):
        cache.attend(q, lens, table[:1])
    with pytest.raises(ValueError):
        cache.attend(q[..., :32], lens, table)
    with pytest.raises(paged._rt.RetopkError):
        cache.attend(q[:, :3].contiguous(), lens, table)
    with pytest.raises(paged._rt.RetopkError):
        half.append(k.half(), k.half(), lens, table)
    with pytest.raises(ValueError):
        cache.append(k, k, lens, table, q=q)
    with pytest.raises(ValueError):
        cache.append(k[:1], k[:1], lens, table)
    with pytest.raises(ValueError):
        cache.append(k.transpose(0, 1), k, lens, table)
    with pytest.raises(ValueError):
        paged.KVPages.wrap(cache.k, cache.v)
    with pytest.raises(TypeError):
        cache.gather(torch.zeros(2, 2, 4, 64, device="cuda", dtype=torch.float64), None, lens, table)
    with pytest.raises(ValueError):
        cache.gather(None, None, lens, table)
    with pytest.raises(TypeError):
        cache.attend(q, [1, 1], table)
    rope = paged.Rope(64)
    wide = torch.zeros(3, 4, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        cache.append(k, k, lens, table, rope=paged.Rope(128))
    with pytest.raises(ValueError):
        rope.apply(q, ints([0]))
    with pytest.raises(paged._rt.RetopkError):
        rope.apply(wide[:2], lens, out=wide[1:])            # overlaps without being the same
    rope.close()
    for call in (lambda: rope.apply(q, lens), lambda: cache.append(k, k, lens, table, rope=rope), rope.frequencies):
        with pytest.raises(paged._rt.RetopkError):
            call()
