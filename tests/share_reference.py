"""Plain forms of the calls for caches that sequences share, and the error bounds of the kernels."""
import math
import random

import torch

import cache_reference as ref

BF, FP = torch.bfloat16, torch.float16


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    """The pool on the host: page counts, a table and lengths as lists."""

    def __init__(self, n_pages, page, B, width):
        self.refs, self.page, self.width = [0] * n_pages, page, width
        self.table, self.lens, self.missing = [[0] * width for _ in range(B)], [0] * B, 0

    def held(self, n):
        return -(-n // self.page) if n > 0 else 0

    def free_pages(self):
        return [p for p, r in enumerate(self.refs) if r <= 0]

    def reserve(self, old, new):
        free, want = self.free_pages(), 0
        for b, (o, n) in enumerate(zip(old, new)):
            had, get = self.held(o), self.held(n)
            if get <= had:
                continue
            lack = min(get - had, len(self.refs) + 1)
            if get > self.width:
                self.missing += lack
                for s in range(min(had, self.width), self.width):
                    self.table[b][s] = -1
                continue
            at, want = want, want + lack
            if want > len(free):
                self.missing += lack
                self.table[b][had:get] = [-1] * (get - had)
                continue
            self.table[b][had:get] = free[at:want]
            for p in free[at:want]:
                self.refs[p] = 1

    def fork(self, parents, children):
        B, capacity = len(self.lens), self.width * self.page
        lens, made, moves = list(self.lens), [], []
        for i, (p, c) in enumerate(zip(parents, children)):
            ok = 0 <= p < B and 0 <= c < B and c not in children[:i] and p not in children
            ok = ok and 0 < lens[p] <= capacity and lens[c] <= 0
            made.append(ok)
        free, at = self.free_pages(), 0
        for i, (p, c) in enumerate(zip(parents, children)):
            if not made[i]:
                moves.append((-1, -1, 0))
                continue
            full, rest = divmod(lens[p], self.page)
            self.table[c][:full] = self.table[p][:full]
            dst = -1
            if rest:
                if at >= len(free):
                    self.missing += 1
                    moves.append((-1, -1, 0))
                    continue
                dst, at = free[at], at + 1
                self.table[c][full] = dst
                self.refs[dst] = 1
            for x in self.table[c][:full]:
                if 0 <= x < len(self.refs):
                    self.refs[x] += 1
            self.lens[c] = lens[p]
            moves.append((self.table[p][full], dst, rest) if rest else (-1, -1, 0))
        return moves

    def free(self, rows):
        for b in rows:
            if 0 <= b < len(self.lens):
                for p in self.table[b][:min(self.held(self.lens[b]), self.width)]:
                    if 0 <= p < len(self.refs):
                        self.refs[p] -= 1
                self.lens[b] = 0

    def compact(self):
        used = [p for p, r in enumerate(self.refs) if r > 0]
        U = len(used)
        place = dict(zip([p for p in used if p >= U], [p for p in range(U) if self.refs[p] <= 0]))
        for b, row in enumerate(self.table):
            n = min(self.held(self.lens[b]), self.width)
            row[:n] = [place.get(p, p) for p in row[:n]]
        for p, to in place.items():
            self.refs[to], self.refs[p] = self.refs[p], 0
        return list(place.items())


def scattered(need, extra, seed):
    """Rows of a block table over shuffled pages; number of pages."""
    total = sum(need) + extra
    order = list(range(total))
    random.Random(seed).shuffle(order)
    rows, at = [], 0
    for n in need:
        rows.append(order[at:at + n])
        at += n
    return rows, total


def grouped_cache(sizes, shared, lens, page, H, d, dtype, seed=1):
    """Cache of sequences in groups of `sizes` that share `shared` rows; k, v, table, cu_groups."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    first = [sum(sizes[:i]) for i in range(len(sizes))]
    of = [i for i, m in enumerate(sizes) for _ in range(m)]
    common = [min(shared[i], max([lens[b] for b in range(len(lens)) if of[b] == i] + [0])) // page for i in range(len(sizes))]
    need = [max(0, -(-n // page) - common[of[b]]) for b, n in enumerate(lens)]
    rows, total = scattered(need + common, 3, seed)
    width = max(max(n + common[of[b]] for b, n in enumerate(need)), 1)
    table = []
    for b in range(len(lens)):
        row = rows[len(lens) + of[b]] + rows[b]
        table.append(row + [0] * (width - len(row)))
    k, v = (torch.randn(total, H, page, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    for b, n in enumerate(lens):                                   # the partial page of the prefix is a copy
        i = of[b]
        rest = shared[i] - common[i] * page
        owner = max(range(first[i], first[i] + sizes[i]), key=lambda x: lens[x])
        if b != owner and 0 < rest and common[i] * page < n and common[i] * page < lens[owner]:
            rest = min(rest, page)
            src, dst = table[owner][common[i]], table[b][common[i]]
            if src != dst:
                for x in (k, v):
                    x[dst, :, :rest] = x[src, :, :rest]
    return k, v, ints(table), ints(first + [len(lens)]), ints(shared)


def attention_bound(q, k, v, scale, n, dtype):
    """(bound on |lse error|, absolute part of the bound on |out error|).

    Scores: products of 16-bit numbers are exact in fp32; d of them are added, each addition off by at most
    2^-23 (cut off) of partial sums below sum |q| |k|; scaling and the exponential's argument are three more
    operations on values of that size, 2^-24 each.  Weights: off by 1 + e with e the error of the score plus 2^-21
    for the exponential and the rescaling by powers; rounded once to the type for the product (half a step; in fp16 below 2^-14
    half a step of 2^-24 absolute, next to sums of at least 1: n * 2^-25 in all).  The sums of weights and of
    products: at most n additions, each off by 2^-23 of a partial sum, and 200 for joining parts.
    """
    if not k.numel():
        return 0.0, 0.0
    size = (q.double().abs().amax(0).amax(0) @ k.double().abs().amax(0).amax(0)).item()
    e = abs(scale) * (q.shape[-1] + 3) * 2.0 ** -23 * size + 2.0 ** -21
    sums = (n + 200) * 2.0 ** -23
    vmax = v.double().abs().max().item()
    return e + sums + 2.0 ** -21 * (1 + math.log(max(n, 2))), (ref.half_step(dtype) + 2 * e + 2 * sums) * vmax


def check_attention(got, lse, q, k, v, table, lens, page, scale, picks=None, block=0, case=""):
    """Compare every sequence with 64 bits; k, v pages; picks [B][T][H] lists of blocks or None.  q [B, T, H_q, d]."""
    B, T, H_q, d = q.shape
    H = k.shape[1]
    G = H_q // H
    for b in range(B):
        n = max(0, lens[b])
        rk, rv = (ref.rows_of(x, None, table, b, n, page) for x in (k, v))
        if picks is None:
            want, want_lse = ref.attention(q[b], rk, rv, scale)
        else:
            want = torch.zeros(T, H_q, d, dtype=torch.float64, device="cuda")
            want_lse = torch.full((T, H_q), -math.inf, dtype=torch.float64, device="cuda")
            for t in range(T):
                seen = n - T + 1 + t
                for h in range(H):
                    keys = [j for x in picks[b][t][h] if 0 <= x * block < seen for j in range(x * block, min(seen, (x + 1) * block))]
                    if keys:
                        j = torch.tensor(keys, device="cuda")
                        s = q[b, t, h * G:(h + 1) * G].double() @ rk[h, j].t() * scale
                        want[t, h * G:(h + 1) * G] = torch.softmax(s, -1) @ rv[h, j]
                        want_lse[t, h * G:(h + 1) * G] = torch.logsumexp(s, -1)
        e_lse, e_out = attention_bound(q[b], rk, rv, scale, n, q.dtype)
        err = (got[b].double() - want).abs()
        limit = e_out + ref.half_step(q.dtype) * want.abs() + 2.0 ** -25
        assert bool((err <= limit).all()), (case, b, float((err - limit).max()), float(err.max()))
        if lse is not None:
            none = torch.isinf(want_lse)
            assert torch.equal(torch.isinf(lse[b]) & (lse[b] < 0), none), (case, b)
            diff = (lse[b].double() - want_lse)[~none].abs()
            assert diff.numel() == 0 or float(diff.max()) <= e_lse + 2.0 ** -23 * float(want_lse[~none].abs().max()), (case, b, float(diff.max()), e_lse)


def bounds_of(k, block):
    """Pages [n, H, page, d] -> bounds [n, H, page / block, 2, d]."""
    x = k.unflatten(2, (-1, block)).double()
    return torch.stack((x.amin(3), x.amax(3)), 3).to(k.dtype)


def select(q, bounds, table, b, n, page, block, keep, first, last):
    """Blocks of one token: q [H_q, d] -> lists per KV head."""
    N = -(-n // block) if n > 0 else 0
    H = bounds.shape[1]
    if N <= keep:
        return [list(range(N)) for _ in range(H)]
    j = torch.arange(N, device="cuda") * block
    ids = torch.full_like(j, b) if table is None else table[b].long()[j // page]
    inside = (ids >= 0) & (ids < bounds.shape[0])
    x = bounds[ids.clamp(0, bounds.shape[0] - 1), :, j % page // block].double()          # [N, H, 2, d]
    qq = q.double().view(H, -1, 1, q.shape[-1])
    low, high = x[:, :, 0].transpose(0, 1).unsqueeze(1), x[:, :, 1].transpose(0, 1).unsqueeze(1)
    s = torch.maximum(qq * low, qq * high).sum(-1).float()                                # [H, G, N]
    s = torch.where(torch.isnan(s), torch.inf, s).amax(1)
    s = torch.where(inside, s, -torch.inf).cpu().tolist()
    out = []
    for h in range(H):
        middle = sorted(range(first, N - last), key=lambda i: (-s[h][i], i))[:keep - first - last]
        out.append(sorted(middle + list(range(first)) + list(range(N - last, N))))
    return out
