"""Cases for paged caches that sequences share: pages, attention over a shared prefix, block-sparse attention.

Five operators, each named by a case's ``"op"``:

* ``fork``: drop old continuations of some sequences and make new ones: full pages shared, the last page copied;
* ``compact``: move the pages in use to the front of the cache;
* ``shared``: decode attention of a batch whose groups of sequences share a prefix;
* ``bounds``: least and largest key of every block of rows, channel by channel;
* ``sparse``: select blocks by their bounds for each query, and attend over them.

``run`` computes them in plain torch operations, or, where ``own`` is true, through the package.
A page that ``refs`` counts 0 block-table entries for is free; new pages are the lowest free ones.
"""
import math
import random

import torch

own = False

GROUP = 64                       # channels that share a step and a minimum in a 4-bit cache
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------
def _fork(name, parents, children, length, H_kv, d, fmt, page, spare, plan):
    return dict(name=name, op="fork", parents=parents, children=children, length=length, H_kv=H_kv, d=d, fmt=fmt, page=page,
                spare=spare, plan=plan)


def _compact(name, batch, length, H_kv, d, fmt, page, spare, plan):
    return dict(name=name, op="compact", batch=batch, length=length, H_kv=H_kv, d=d, fmt=fmt, page=page, spare=spare, plan=plan)


def _shared(name, groups, members, prefix, suffix, T, H_q, H_kv, d, fmt, page, plan):
    return dict(name=name, op="shared", groups=groups, members=members, prefix=prefix, suffix=suffix, T=T, H_q=H_q, H_kv=H_kv,
                d=d, fmt=fmt, page=page, plan=plan)


def _bounds(name, batch, length, ragged, new, H_kv, d, fmt, page, block, plan):
    return dict(name=name, op="bounds", batch=batch, length=length, ragged=ragged, new=new, H_kv=H_kv, d=d, fmt=fmt, page=page,
                block=block, plan=plan)


def _sparse(name, batch, length, ragged, T, H_q, H_kv, d, fmt, page, block, keep, plan):
    return dict(name=name, op="sparse", batch=batch, length=length, ragged=ragged, T=T, H_q=H_q, H_kv=H_kv, d=d, fmt=fmt, page=page,
                block=block, keep=keep, plan=plan)


def listed():
    return [
        # three samples of one short conversation: latency
        _fork("fork_one_short", 1, 3, 1000, 8, 128, "bf16", 64, 64, 11),
        # 16 prompts of mixed length, four beams each, short pages
        _fork("fork_beams_ragged", 16, 64, 32768, 8, 64, "fp16", 16, 512, 12),
        # a cache of 2 GB that is mostly empty after a peak: its live pages move to the front
        _compact("compact_after_peak", 24, 16384, 8, 128, "bf16", 64, 4096, 13),
        # a small 4-bit cache; its values are read back
        _compact("compact_4bit", 5, 3001, 4, 128, "q4", 32, 700, 14),
        # four samples of a short prompt: latency
        _shared("shared_four_short", 1, 4, 700, 60, 1, 32, 8, 128, "bf16", 16, 21),
        # a serving batch behind one system prompt of 32K
        _shared("shared_batch32_32k", 1, 32, 32768, 1024, 1, 32, 8, 128, "bf16", 64, 22),
        # three documents, questions of mixed number to each, four draft tokens at once
        _shared("shared_documents_draft", 3, 13, 9001, 700, 4, 16, 4, 64, "fp16", 16, 23),
        # 64 continuations of a 128K context
        _shared("shared_batch64_128k", 1, 64, 131072, 2048, 1, 32, 8, 128, "bf16", 64, 24),
        # bounds of all blocks of four 128K prompts
        _bounds("bounds_prompts_128k", 4, 131072, False, 0, 8, 128, "bf16", 64, 64, 31),
        # a few draft tokens at the end of mixed lengths: only the blocks that they fill
        _bounds("bounds_draft_ragged", 16, 20011, True, 20, 4, 64, "fp16", 32, 16, 32),
        # the 128K decode step of four sequences over 64 blocks of 64 keys
        _sparse("sparse_batch4_128k", 4, 131072, False, 1, 32, 8, 128, "bf16", 64, 64, 64, 41),
        # a serving batch of mixed lengths, two draft tokens, small blocks
        _sparse("sparse_ragged_draft", 16, 65521, True, 2, 16, 4, 64, "fp16", 128, 16, 128, 42),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["fork", "compact", "shared", "shared", "shared", "bounds", "sparse", "sparse"])
    d = rng.choice([64, 128, 128])
    H_kv = rng.choice([1, 2, 4, 8])
    H_q = H_kv * rng.choice([1, 2, 4, 4] + ([8] if H_kv < 8 else []))
    fmt = rng.choice(["bf16", "bf16", "fp16"])
    page = rng.choice([16, 32, 64, 128])
    plan = rng.randrange(1 << 30)
    if op == "fork":
        parents = rng.randint(1, 16)
        return _fork("", parents, parents * rng.randint(1, 4), _log_int(rng, 20, 32768), H_kv, d, fmt, page, rng.randint(80, 600), plan)
    if op == "compact":
        batch = rng.randint(1, 16)
        if rng.random() < 0.3:
            fmt, length = "q4", _log_int(rng, 20, 4000)
        else:
            length = _log_int(rng, 20, 16384)
        return _compact("", batch, length, H_kv, d, fmt, page, rng.randint(8, 32000 // page), plan)
    if op == "shared":
        T = rng.choice([1, 1, 1, 2, 4])
        groups = rng.choice([1, 1, 2, 3, 5])
        members = rng.randint(1, max(1, 64 // groups))
        return _shared("", groups, members, _log_int(rng, 16, 131072 // groups), _log_int(rng, 4, 2048), T, H_q if T == 1 else H_kv * 2,
                       H_kv, d, fmt, rng.choice([page, page, 24]), plan)
    block = rng.choice([b for b in (16, 32, 64, 128) if b <= page])
    batch = rng.choice([1, 2, 3, 4, 7, 8, 16])
    length = _log_int(rng, 200, 524288 // batch // 4)
    if op == "bounds":
        return _bounds("", batch, length, rng.random() < 0.6, rng.choice([0, 0, rng.randint(1, 150)]), H_kv, d, fmt, page, block, plan)
    return _sparse("", batch, length, rng.random() < 0.6, rng.choice([1, 1, 1, 2, 4]), H_q, H_kv, d, fmt, page, block,
                   rng.randint(4, max(4, 4096 // block)), plan)


FIRST, LAST = 1, 2               # blocks at both ends of a sequence that are always kept


def _fork_plan(case):
    """Lengths of the parents, and for each child its parent."""
    rng = random.Random(case["plan"])
    n, length = case["parents"], case["length"]
    lens = [length if n == 1 else _log_int(rng, max(1, length // 16), length) for _ in range(n)]
    if n > 2:
        lens[1] -= lens[1] % case["page"]                          # one ends with a full page
    return lens, [i * n // case["children"] for i in range(case["children"])]


def _lengths(case):
    rng = random.Random(case["plan"])
    B, length = case["batch"], case["length"]
    if case["op"] == "compact":
        return [_log_int(rng, max(1, length // 8), length) for _ in range(B)]
    return [_log_int(rng, max(8, length // 64), length) for _ in range(B)] if case["ragged"] else [length] * B


def _group_plan(case):
    """Members of each group, shared rows of each group, and all keys of each sequence."""
    rng = random.Random(case["plan"])
    sizes, prefix, lens = [], [], []
    for g in range(case["groups"]):
        sizes.append(case["members"] if g == 0 else rng.randint(1, case["members"]))
        prefix.append(case["prefix"] if g == 0 else _log_int(rng, max(1, case["prefix"] // 8), case["prefix"]))
        lens += [prefix[-1] + case["T"] - 1 + _log_int(rng, 1, case["suffix"]) for _ in range(sizes[-1])]
    return sizes, prefix, lens


def _row_bytes(case):
    return case["d"] // 2 + case["d"] // GROUP * 4 if case["fmt"] == "q4" else 2 * case["d"]


def _moves(case):
    """Pages that a compaction moves, for a layout as `_scattered` makes it."""
    need = sum(-(-n // case["page"]) for n in _lengths(case))
    order = list(range(need + case["spare"]))
    random.Random(case["plan"] + 1).shuffle(order)
    return sum(p >= need for p in order[:need]), need + case["spare"]


def work(case):
    d, H = case["d"], case["H_kv"]
    if case["op"] == "fork":
        lens, parent = _fork_plan(case)
        rows = sum(lens[p] % case["page"] for p in parent)
        held = sum(-(-lens[p] // case["page"]) for p in parent)
        return {"bytes": rows * H * 4 * _row_bytes(case) + held * 4 * 4, "flops": 0}
    if case["op"] == "compact":
        moved, total = _moves(case)
        byt = moved * case["page"] * H * 4 * _row_bytes(case) + total * 8
        if case["fmt"] == "q4":
            byt += total * case["page"] * H * 2 * (_row_bytes(case) + 4 * d)
        return {"bytes": byt, "flops": 0}
    if case["op"] == "shared":
        sizes, prefix, lens = _group_plan(case)
        B, T, H_q = len(lens), case["T"], case["H_q"]
        shared = [p for p, m in zip(prefix, sizes) for _ in range(m)]
        rows = sum(prefix) + sum(n - p for n, p in zip(lens, shared))
        pairs = sum(n - T + 1 + t for n in lens for t in range(T))
        return {"bytes": rows * H * 4 * d + 4 * B * T * H_q * d, "flops": 4 * pairs * H_q * d}
    lens, block = _lengths(case), case["block"]
    if case["op"] == "bounds":
        new = case["new"] or max(lens)
        blocks = sum(n // block - max(0, n - new) // block for n in lens)
        return {"bytes": blocks * H * (block * 2 * d + 4 * d), "flops": blocks * H * block * 2 * d}
    T, H_q = case["T"], case["H_q"]
    seen = [n - T + 1 + t for n in lens for t in range(T)]
    scored = sum(-(-n // block) for n in lens if -(-n // block) > case["keep"])
    pairs = sum(min(n, case["keep"] * block) for n in seen)
    return {"bytes": scored * H * 4 * d + pairs * H * 4 * d + 4 * len(lens) * T * H_q * d,
            "flops": (scored * T * 4 + pairs * 4) * H_q * d}


# ---------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)


def _rand(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _scattered(need, total, seed):
    """A table over pages in no order, as a server that hands pages out and takes them back leaves it."""
    order = list(range(total))
    random.Random(seed).shuffle(order)
    width, at, table = max(need), 0, []
    for n in need:
        table.append(order[at:at + n] + [0] * (width - n))
        at += n
    return table


def _filled(g, shape, fmt):
    """Random keys or values of a cache, filled in pieces."""
    if fmt == "q4":
        codes = torch.randint(0, 256, shape[:-1] + (shape[-1] // 2,), generator=g, device="cuda", dtype=torch.uint8)
        scale = _rand(g, *shape[:-1], shape[-1] // GROUP, 2)
        return codes, scale.abs_().bfloat16()
    x = torch.empty(shape, dtype=TYPES[fmt], device="cuda")
    for part in x.split(max(1, (1 << 25) // math.prod(shape[1:]))):
        part.copy_(_rand(g, *part.shape))
    return x, None


def _towards(g, st, B, T, H, G, d):
    """Queries that lean towards some key of their own sequence, as trained ones do."""
    case, q = st["case"], _rand(g, B, T, H, G, d)
    for b, n in enumerate(st["host_lens"]):
        j = torch.randint(0, n, (T, H, G), generator=g, device="cuda")
        ids = st["table"][b].long()[j // case["page"]]
        h = torch.arange(H, device="cuda").view(1, H, 1)
        q[b] = 0.8 * q[b] + 0.4 * st["k"][ids, h, j % case["page"]].float()
    return q.view(B, T, H * G, d).to(TYPES[case["fmt"]])


def prepare(case, seed):
    st = {"case": case}
    g = _gen(seed)
    H, d, page, op = case["H_kv"], case["d"], case["page"], case["op"]
    if op == "fork":
        lens, parent = _fork_plan(case)
        need = [-(-n // page) for n in lens]
        total = sum(need) + case["spare"]
        width = max(need) + 4
        table = [row + [0] * (width - len(row)) for row in _scattered(need, total, case["plan"] + 1)]
        st["host_table"], st["host_lens"], st["host_parent"] = table, lens, parent
        st["table"] = _ints(table + [[0] * width for _ in parent])
        st["lens"] = _ints(lens + [0] * len(parent))
        st["parents"] = _ints(parent)
        st["children"] = _ints([len(lens) + i for i in range(len(parent))])
    elif op == "compact":
        lens = _lengths(case)
        need = [-(-n // page) for n in lens]
        total = sum(need) + case["spare"]
        st["host_table"], st["host_need"] = _scattered(need, total, case["plan"] + 1), need
        st["table0"], st["lens"] = _ints(st["host_table"]), _ints(lens)
        st["table"] = st["table0"].clone()
    elif op == "shared":
        sizes, prefix, lens = _group_plan(case)
        # whole pages of the prefix are shared; the one in which it ends is a copy in every member
        need, shared = [], []
        for m, p in zip(sizes, prefix):
            shared += [p // page] * m
        need = [-(-n // page) - s for n, s in zip(lens, shared)]
        rows = _scattered(need + [p // page for p in prefix], sum(need) + sum(p // page for p in prefix), case["plan"] + 1)
        width, table, cu = max(n + s for n, s in zip(need, shared)), [], [0]
        for i, m in enumerate(sizes):
            for b in range(cu[-1], cu[-1] + m):
                row = rows[len(lens) + i][:shared[b]] + rows[b][:need[b]]
                table.append(row + [0] * (width - len(row)))
            cu.append(cu[-1] + m)
        total = sum(need) + sum(p // page for p in prefix)
        st["host_lens"], st["lens"], st["table"], st["cu"] = lens, _ints(lens), _ints(table), _ints(cu)
        st["prefix"] = _ints(prefix)
        st["host_cu"], st["host_prefix"] = cu, prefix
    else:
        lens = _lengths(case)
        need = [-(-n // page) for n in lens]
        total = sum(need)
        st["host_lens"], st["lens"], st["table"] = lens, _ints(lens), _ints(_scattered(need, total, case["plan"] + 1))

    st["k"], st["k_scale"] = _filled(g, (total, H, page, d), case["fmt"])
    st["v"], st["v_scale"] = _filled(g, (total, H, page, d), case["fmt"])
    if op == "sparse":                                             # keys near one another are alike
        for part in st["k"].split(max(1, (1 << 25) // (H * page * d))):
            part.add_(0.7 * _rand(g, part.shape[0], H, 1, d).to(part.dtype))
    if op == "shared":
        for b, n in enumerate(prefix[i] for i, m in enumerate(sizes) for _ in range(m)):
            first = st["host_cu"][max(i for i in range(len(sizes)) if st["host_cu"][i] <= b)]
            if n % page and b != first:                            # the copied page of the prefix
                src, dst = st["table"][first, n // page].long(), st["table"][b, n // page].long()
                for x in (st["k"], st["v"]):
                    x[dst, :, :n % page] = x[src, :, :n % page]
    if op in ("fork", "compact"):
        refs = [0] * total
        for row, n in zip(st["host_table"], need):
            for p in row[:n]:
                refs[p] += 1
        st["host_refs"], st["refs0"] = refs, _ints(refs)
        st["refs"] = st["refs0"].clone()
    if op in ("shared", "sparse"):
        st["q"] = _towards(g, st, len(lens), case["T"], H, case["H_q"] // H, d)
    if op == "compact" and case["fmt"] == "q4":
        st["k_out"] = torch.zeros((total, H, page, d), dtype=torch.float32, device="cuda")
        st["v_out"] = torch.zeros_like(st["k_out"])
        st["all"], st["full"] = torch.arange(total, dtype=torch.int32, device="cuda").view(-1, 1), _ints([page] * total)
    if op in ("bounds", "sparse"):
        st["bounds"] = torch.zeros((total, H, page // case["block"], 2, d), dtype=st["k"].dtype, device="cuda")
        if op == "sparse" and not own:
            x = st["k"].unflatten(2, (-1, case["block"]))
            st["bounds"][..., 0, :], st["bounds"][..., 1, :] = x.amin(3), x.amax(3)
    if own:
        from paper_2607_27692_b200 import paged
        st["pages"] = paged.KVPages.wrap(st["k"], st["v"], st["k_scale"], st["v_scale"])
        if op in ("fork", "compact"):
            st["pool"] = paged.PagePool.wrap(st["refs"], page)
        if op in ("bounds", "sparse"):
            st["index"] = paged.BlockIndex.wrap(st["pages"], st["bounds"])
            if op == "sparse":
                st["index"].update(st["lens"], st["table"])
    return st


# ---------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    case, table, lens = st["case"], st["table"], st["lens"]
    if case["op"] == "fork":
        st["pool"].free(table, lens, st["children"])
        src, dst, rows = st["pool"].fork(table, lens, st["parents"], st["children"])
        st["pages"].copy_pages(src, dst, rows)
        return table, lens, st["refs"], st["k"], st["v"]
    if case["op"] == "compact":
        table.copy_(st["table0"])
        st["refs"].copy_(st["refs0"])
        src, dst = st["pool"].compact(table, lens)
        st["pages"].copy_pages(src, dst)
        if case["fmt"] == "q4":
            st["pages"].gather(st["k_out"], st["v_out"], st["full"], st["all"])
            return table, st["refs"], st["k_out"], st["v_out"]
        return table, st["refs"], st["k"], st["v"]
    if case["op"] == "shared":
        return st["pages"].attend_shared(st["q"], lens, table, st["cu"], st["prefix"])
    if case["op"] == "bounds":
        st["index"].update(lens, table, case["new"] or None)
        return st["bounds"]
    blocks = st["index"].select(st["q"], lens, table, keep=case["keep"], first=FIRST, last=LAST)
    return blocks, st["index"].attend(st["q"], lens, blocks, table)


def _values(codes, scale):
    """Packed codes [..., d/2] and (step, minimum) [..., d/64, 2] -> fp32 values [..., d]."""
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float().unflatten(-1, (-1, GROUP))
    s, m = scale.float().unbind(-1)
    return (n * s.unsqueeze(-1) + m.unsqueeze(-1)).flatten(-2)


def _plain_fork(st):
    case, table, lens, refs = st["case"], st["table"], st["lens"], st["refs"]
    page, parents, children = case["page"], st["parents"].long(), st["children"].long()
    slot = torch.arange(table.shape[1], device="cuda")
    held = slot < ((lens[children] + page - 1) // page).unsqueeze(1)
    refs.index_add_(0, table[children].long().flatten(), -held.int().flatten())
    n = lens[parents]
    full, rest = (n // page).long(), n % page
    old = table[parents]
    whole = slot < full.unsqueeze(1)
    refs.index_add_(0, old.long().flatten(), whole.int().flatten())
    lowest = torch.sort((refs > 0).int(), stable=True).indices
    some = rest > 0
    fresh = lowest[(some.long().cumsum(0) - 1).clamp_min(0)]
    last = (slot == full.unsqueeze(1)) & some.unsqueeze(1)
    row = torch.where(whole, old, table[children])
    table[children] = torch.where(last, fresh.int().unsqueeze(1), row)
    refs.index_add_(0, fresh, some.int())
    lens[children] = n
    src = old.gather(1, full.clamp_max(table.shape[1] - 1).unsqueeze(1)).squeeze(1).long()
    src = torch.where(some, src, old[:, 0].long())
    dst = torch.where(some, fresh, src)                            # (a page onto itself)
    copied = (torch.arange(page, device="cuda") < rest.unsqueeze(1)).view(-1, 1, page, 1)
    for x in (st["k"], st["v"]):
        x[dst] = torch.where(copied, x[src], x[dst])
    return table, lens, refs, st["k"], st["v"]


def _plain_compact(st):
    case, page = st["case"], st["case"]["page"]
    table, refs = st["table"], st["refs"]
    table.copy_(st["table0"])
    refs.copy_(st["refs0"])
    p = torch.arange(refs.numel(), device="cuda")
    used = refs > 0
    U = used.sum()
    src, dst = torch.nonzero(used & (p >= U)).squeeze(1), torch.nonzero(~used & (p < U)).squeeze(1)
    moved = p.clone()
    moved[src] = dst
    held = torch.arange(table.shape[1], device="cuda") < ((st["lens"] + page - 1) // page).unsqueeze(1)
    table.copy_(torch.where(held, moved[table.long()].int(), table))
    refs[dst], refs[src] = refs[src], torch.zeros_like(refs[src])
    for x in (st["k"], st["v"], st["k_scale"], st["v_scale"]):
        if x is not None:
            x[dst] = x[src]
    if case["fmt"] == "q4":
        st["k_out"].copy_(_values(st["k"], st["k_scale"]))
        st["v_out"].copy_(_values(st["v"], st["v_scale"]))
        return table, refs, st["k_out"], st["v_out"]
    return table, refs, st["k"], st["v"]


def _rows(st, b, n, name):
    """fp32 [H_kv, n, d]: the first n rows of sequence b."""
    ids = st["table"][b, :-(-n // st["case"]["page"])].long()
    return st[name][ids].transpose(0, 1).flatten(1, 2)[:, :n].float()


def _plain_attention(q, k, v, hidden=None):
    """q [H, rows, d], k, v [H, keys, d], all fp32."""
    s = torch.matmul(q, k.transpose(1, 2)) * q.shape[-1] ** -0.5
    if hidden is not None:
        s = s.masked_fill(hidden, float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    return torch.matmul(p, v) / p.sum(-1, keepdim=True)


def _run_plain(st):
    case = st["case"]
    if case["op"] == "fork":
        return _plain_fork(st)
    if case["op"] == "compact":
        return _plain_compact(st)
    H, d, page = case["H_kv"], case["d"], case["page"]
    if case["op"] == "bounds":
        block = case["block"]
        for b, n in enumerate(st["host_lens"]):
            lo, hi = max(0, n - (case["new"] or n)) // block, n // block
            if hi > lo:
                x = _rows(st, b, hi * block, "k")[:, lo * block:].unflatten(1, (-1, block))
                j = torch.arange(lo, hi, device="cuda") * block
                ids, at = st["table"][b].long()[j // page], j % page // block
                st["bounds"][ids, :, at, 0] = x.amin(2).transpose(0, 1).to(st["bounds"].dtype)
                st["bounds"][ids, :, at, 1] = x.amax(2).transpose(0, 1).to(st["bounds"].dtype)
        return st["bounds"]
    T, H_q = case["T"], case["H_q"]
    G = H_q // H
    out = torch.empty_like(st["q"])
    if case["op"] == "shared":
        for b, n in enumerate(st["host_lens"]):
            k, v = _rows(st, b, n, "k"), _rows(st, b, n, "v")
            q = st["q"][b].float().view(T, H, G, d).permute(1, 0, 2, 3).reshape(H, T * G, d)
            hidden = None
            if T > 1:
                last = torch.arange(n - T, n, device="cuda").repeat_interleave(G).unsqueeze(1)
                hidden = torch.arange(n, device="cuda") > last
            o = _plain_attention(q, k, v, hidden)
            out[b] = o.view(H, T, G, d).permute(1, 0, 2, 3).reshape(T, H_q, d).to(out.dtype)
        return out
    keep, block = case["keep"], case["block"]
    blocks = torch.full((len(st["host_lens"]), T, H, keep), -1, dtype=torch.int32, device="cuda")
    for b, length in enumerate(st["host_lens"]):
        bounds = st["bounds"][st["table"][b].long()].transpose(0, 1).flatten(1, 2)       # [H, blocks, 2, d]
        k, v = _rows(st, b, length, "k"), _rows(st, b, length, "v")
        for t in range(T):
            n = length - T + 1 + t
            N = -(-n // block)
            q = st["q"][b, t].view(H, G, d)
            if N <= keep:
                pick = torch.arange(N, device="cuda").expand(H, N)
            else:
                # 64 bits: the order of blocks whose scores are close
                low, high = bounds[:, FIRST:N - LAST].double().unbind(2)
                s = torch.matmul(q.double().clamp_min(0), high.transpose(1, 2)) + torch.matmul(q.double().clamp_max(0), low.transpose(1, 2))
                s = s.float().amax(1)
                best = torch.sort(s, dim=-1, descending=True, stable=True).indices[:, :keep - FIRST - LAST] + FIRST
                ends = torch.cat((torch.arange(FIRST, device="cuda"), torch.arange(N - LAST, N, device="cuda")))
                pick = torch.cat((best, ends.expand(H, -1)), 1).sort(-1).values
            blocks[b, t, :, :pick.shape[1]] = pick.int()
            j = (pick.unsqueeze(-1) * block + torch.arange(block, device="cuda")).flatten(1)
            inside = (j < n).unsqueeze(1)
            j = j.clamp_max(n - 1).unsqueeze(-1).expand(-1, -1, d)
            out[b, t] = _plain_attention(q.float(), k.gather(1, j), v.gather(1, j), ~inside).view(H_q, d).to(out.dtype)
    return blocks, out


# ---------------------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------
def _exact_fork(case, st):
    """Page by page, decided on the host."""
    k, v = st["k"].clone(), st["v"].clone()
    page, refs, width = case["page"], list(st["host_refs"]), st["table"].shape[1]
    table, lens = [list(r) for r in st["host_table"]], list(st["host_lens"])
    free = [p for p, r in enumerate(refs) if r == 0]
    for p in st["host_parent"]:
        full, row = lens[p] // page, [0] * width
        for i in range(full):
            row[i] = table[p][i]
            refs[row[i]] += 1
        if lens[p] % page:
            row[full] = free.pop(0)
            refs[row[full]] = 1
            for x in (k, v):
                x[row[full], :, :lens[p] % page] = st["k" if x is k else "v"][table[p][full], :, :lens[p] % page]
        table.append(row)
        lens.append(lens[p])
    return _ints(table), _ints(lens), _ints(refs), k, v


def _exact_compact(case, st):
    refs, table = list(st["host_refs"]), [list(r) for r in st["host_table"]]
    U = sum(r > 0 for r in refs)
    holes = [p for p in range(U) if refs[p] == 0]
    place = dict(zip([p for p in range(U, len(refs)) if refs[p] > 0], holes))
    for row, n in zip(table, st["host_need"]):
        row[:n] = [place.get(p, p) for p in row[:n]]
    for p, to in place.items():
        refs[to], refs[p] = refs[p], 0
    was = list(range(len(refs)))
    for p, to in place.items():
        was[to] = p
    at, outs = torch.tensor(was, device="cuda"), []
    if case["fmt"] != "q4":
        return _ints(table), _ints(refs), st["k"][at], st["v"][at]
    for name in ("k", "v"):
        packed, scale = st[name][at], st[name + "_scale"][at].double()
        x = torch.empty(packed.shape[:3] + (case["d"],), dtype=torch.float64, device="cuda")
        x[..., 0::2], x[..., 1::2] = (packed % 16).double(), torch.div(packed, 16, rounding_mode="floor").double()
        for c in range(case["d"] // GROUP):
            x[..., c * GROUP:(c + 1) * GROUP].mul_(scale[..., c, 0:1]).add_(scale[..., c, 1:2])
        outs.append(x)
    return _ints(table), _ints(refs), outs[0], outs[1]


def _exact_sequence(st, b, j, name):
    """fp64 [H_kv, len(j), d]: rows j of sequence b."""
    page = st["case"]["page"]
    return st[name][st["table"][b].long()[j // page], :, j % page].double().transpose(0, 1)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "fork":
        return _exact_fork(case, st)
    if case["op"] == "compact":
        return _exact_compact(case, st)
    H, d, page = case["H_kv"], case["d"], case["page"]
    if case["op"] == "bounds":
        out, block = torch.zeros(st["bounds"].shape, dtype=torch.float64, device="cuda"), case["block"]
        for b, n in enumerate(st["host_lens"]):
            first = max(0, n - case["new"]) // block if case["new"] else 0
            for at in range(page // block):                        # blocks at one place of their pages
                j = torch.arange(n // block, device="cuda")
                j = j[(j >= first) & (j % (page // block) == at)]
                if j.numel():
                    ids = st["table"][b].long()[j // (page // block)]
                    x = st["k"][ids, :, at * block:(at + 1) * block].double()
                    out[ids, :, at, 0], out[ids, :, at, 1] = x.min(2).values, x.max(2).values
        return out
    T, H_q = case["T"], case["H_q"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    if case["op"] == "shared":
        for b, length in enumerate(st["host_lens"]):
            j = torch.arange(length, device="cuda")
            k, v = _exact_sequence(st, b, j, "k"), _exact_sequence(st, b, j, "v")
            for t in range(T):
                n = length - T + 1 + t
                q = st["q"][b, t].double().view(H, H_q // H, d)
                p = torch.softmax(q @ k[:, :n].transpose(1, 2) / math.sqrt(d), -1)
                out[b, t] = (p @ v[:, :n]).view(H_q, d)
        return out
    keep, block = case["keep"], case["block"]
    blocks = torch.full((len(st["host_lens"]), T, H, keep), -1, dtype=torch.int32, device="cuda")
    for b, length in enumerate(st["host_lens"]):
        whole = length // block
        keys = _exact_sequence(st, b, torch.arange(whole * block, device="cuda"), "k").unflatten(1, (whole, block))
        low, high = keys.min(2).values, keys.max(2).values
        for t in range(T):
            n = length - T + 1 + t
            N = (n + block - 1) // block
            q = st["q"][b, t].double().view(H, H_q // H, d)
            for h in range(H):
                if N <= keep:
                    pick = list(range(N))
                else:
                    score = None
                    for x in q[h]:
                        s = torch.maximum(x * low[h, FIRST:N - LAST], x * high[h, FIRST:N - LAST]).sum(-1).float()
                        score = s if score is None else torch.maximum(score, s)
                    order = torch.argsort(-score, stable=True)[:keep - FIRST - LAST] + FIRST
                    pick = sorted(order.tolist() + list(range(FIRST)) + list(range(N - LAST, N)))
                blocks[b, t, h, :len(pick)] = _ints(pick)
                j = torch.cat([torch.arange(i * block, min(n, (i + 1) * block)) for i in pick]).cuda()
                ids = st["table"][b].long()[j // page]
                k, v = st["k"][ids, h, j % page].double(), st["v"][ids, h, j % page].double()
                p = torch.softmax(q[h] @ k.t() / math.sqrt(d), -1)
                out[b, t].view(H, H_q // H, d)[h] = p @ v
    return blocks, out
