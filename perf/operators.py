"""Cases for the operators around the decode step's KV cache: rotation, append, gather, 4-bit attention.

Four operators, each named by a case's ``"op"``:

* ``rope``: rotary positions on queries and keys (and the transposed rotation, its gradient);
* ``append``: rotate new keys and queries and store keys and values in a cache, in 16 or in 4 bits;
* ``gather``: read rows of a paged 4-bit cache back into the contiguous 16-bit cache of the decode step;
* ``attend``: decode attention that reads the paged 4-bit cache.

``run`` computes them in plain torch operations, or, where ``own`` is true, through the package.
A 4-bit cache holds, per row and group of 64 channels, a scale ``s`` and a minimum ``m`` in bf16 and
codes ``n`` in 0..15 (low nibble = even channel); the group stands for ``s * n + m``.
"""
import math
import random

import torch

own = False

GROUP = 64                       # channels that share a scale and a minimum
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------
def _rope(name, tokens, H_q, H_kv, d, dtype, first, rot, layout, scaling, factor, inverse):
    return dict(name=name, op="rope", tokens=tokens, H_q=H_q, H_kv=H_kv, d=d, dtype=dtype, first=first, rot=rot,
                layout=layout, scaling=scaling, factor=factor, inverse=inverse)


def _append(name, batch, new, past, ragged, H_q, H_kv, d, dtype, fmt, page, rot, layout, lens_seed):
    return dict(name=name, op="append", batch=batch, new=new, past=past, ragged=ragged, H_q=H_q, H_kv=H_kv, d=d,
                dtype=dtype, fmt=fmt, page=page, rot=rot, layout=layout, lens_seed=lens_seed)


def _gather(name, batch, length, ragged, H_kv, d, page, out, lens_seed):
    return dict(name=name, op="gather", batch=batch, length=length, ragged=ragged, H_kv=H_kv, d=d, page=page, out=out,
                lens_seed=lens_seed)


def _attend(name, batch, length, ragged, T, H_q, H_kv, d, dtype, page, window, lens_seed):
    return dict(name=name, op="attend", batch=batch, length=length, ragged=ragged, T=T, H_q=H_q, H_kv=H_kv, d=d,
                dtype=dtype, page=page, window=window, lens_seed=lens_seed)


def listed():
    return [
        # one new token of one sequence at the end of a 128K context: a launch's latency
        _rope("rope_one_token", 1, 32, 8, 128, "bf16", 131071, 128, "half", "llama3", 16.0, False),
        # a whole 16K prompt at the far end of a context stretched to 128K
        _rope("rope_prompt_16k", 16384, 32, 8, 128, "bf16", 114688, 128, "half", "llama3", 16.0, False),
        # gradient of an interleaved rotation over half the head, an odd number of tokens
        _rope("rope_gradient_odd", 5003, 16, 4, 64, "fp16", 0, 32, "interleaved", "yarn", 4.0, True),
        # decode step of 16 sequences of mixed length: rotate q and k, store k and v in 4 bits
        _append("append_decode_4bit", 16, 1, 32768, True, 32, 8, 128, "bf16", "q4", 64, 128, "half", 11),
        # seven prompts of mixed length in one call, short pages
        _append("append_ragged_4bit", 7, 4001, 0, True, 16, 4, 64, "fp16", "q4", 16, 64, "half", 12),
        # a 16K prompt into the contiguous cache that the ReTopK decode step reads
        _append("append_prompt_16bit", 1, 16384, 0, False, 32, 8, 128, "bf16", "bf16", 16896, 128, "half", 13),
        # three short sequences read back in full precision
        _gather("gather_short_fp32", 3, 1531, True, 8, 128, 16, "fp32", 23),
        # four sequences of 32K brought back to 16 bits for the decode step
        _gather("gather_batch_32k", 4, 32768, False, 8, 128, 64, "bf16", 22),
        # one short sequence: latency
        _attend("attend_one_short", 1, 777, False, 1, 32, 8, 128, "bf16", 16, 0, 31),
        # the 128K decode step of four sequences
        _attend("attend_batch4_128k", 4, 131584, False, 1, 32, 8, 128, "bf16", 64, 0, 32),
        # a serving batch of mixed lengths, the shortest a hundred keys
        _attend("attend_ragged_batch32", 32, 65536, True, 1, 32, 8, 128, "bf16", 32, 0, 33),
        # four draft tokens checked at once in a layer with a sliding window
        _attend("attend_draft_window", 8, 32768, True, 4, 32, 8, 64, "fp16", 64, 8192, 34),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "append", "gather", "attend", "attend"])
    d = rng.choice([64, 128, 128])
    H_kv = rng.choice([1, 2, 4, 8])
    H_q = H_kv * rng.choice([1, 2, 4, 4, 8])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    page = rng.choice([16, 32, 64, 128])
    seed = rng.randrange(1 << 30)
    rot = d // rng.choice([1, 1, 1, 2, 4])
    layout = rng.choice(["half", "interleaved"])
    if op == "rope":
        tokens = _log_int(rng, 1, 16384)
        scaling = rng.choice(["none", "linear", "ntk", "llama3", "yarn"])
        return _rope("", tokens, H_q, H_kv, d, dtype, rng.randrange(0, 114688), rot, layout, scaling,
                     1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]), rng.random() < 0.3)
    if op == "append":
        batch = rng.randint(1, 24)
        if rng.random() < 0.5:           # decode or a few draft tokens
            new, past = rng.randint(1, 4), _log_int(rng, 32, 16384)
        else:                            # prompts
            new, past = _log_int(rng, 8, max(8, 16384 // batch)), rng.choice([0, rng.randint(1, 2000)])
        fmt = rng.choice(["q4", "q4", dtype])
        return _append("", batch, new, past, rng.random() < 0.6, H_q, H_kv, d, dtype, fmt, page, rot, layout, seed)
    if op == "gather":
        batch = rng.randint(1, 8)
        return _gather("", batch, _log_int(rng, 16, 131072 // batch), rng.random() < 0.6, H_kv, d, page,
                       rng.choice(["bf16", "fp16", "fp32"]), seed)
    batch = rng.choice([1, 2, 3, 4, 7, 8, 16, 31])
    length = _log_int(rng, 16, min(131072, 524288 // batch))
    T = rng.choice([1, 1, 1, 2, 3, 4])
    window = rng.choice([0, 0, 0, rng.randint(1, length)])
    return _attend("", batch, length, rng.random() < 0.6, T, H_q, H_kv, d, dtype, page, window, seed)


def _lengths(case):
    """Per sequence: keys in the cache (new ones included) and new tokens."""
    rng = random.Random(case["lens_seed"])
    B = case["batch"]
    if case["op"] == "append":
        past, new = case["past"], case["new"]
        if not case["ragged"]:
            return [past + new] * B, [new] * B
        pasts = [_log_int(rng, max(1, past // 64), past) if past else 0 for _ in range(B)]
        if new > 4:
            news = [_log_int(rng, max(1, new // 16), new) for _ in range(B)]
        else:
            news = [new] * B
        return [p + n for p, n in zip(pasts, news)], news
    if not case["ragged"]:
        return [case["length"]] * B, [0] * B
    shortest = max(case.get("T", 1), case["length"] // 640, 1)
    return [_log_int(rng, min(shortest, case["length"]), case["length"]) for _ in range(B)], [0] * B


def work(case):
    if case["op"] == "rope":
        n = case["tokens"] * (case["H_q"] + case["H_kv"]) * case["d"]
        return {"bytes": 4 * n + 4 * case["tokens"], "flops": 3 * n}
    lens, news = _lengths(case)
    d, H_kv = case["d"], case["H_kv"]
    packed = 2 * (d // 2 + d // GROUP * 4)                         # key and value of one row
    if case["op"] == "append":
        tok = sum(news)
        byt = tok * (case["H_q"] * d * 4 + H_kv * d * 4)           # q in and out, k and v in
        if case["fmt"] == "q4":
            byt += tok * H_kv * (2 * packed + 2 * d * 4)           # codes out, read back as fp32 values
        else:
            byt += tok * H_kv * d * 4
        return {"bytes": byt, "flops": tok * (case["H_q"] * 3 + H_kv * 8) * d}
    if case["op"] == "gather":
        rows = sum(lens) * H_kv
        size = 4 if case["out"] == "fp32" else 2
        return {"bytes": rows * (packed + 2 * d * size), "flops": rows * 4 * d}
    T, H_q, win = case["T"], case["H_q"], case["window"]
    keys = sum(min(n, win + T - 1) if win else n for n in lens)
    pairs = sum(min(n - T + 1 + t, win) if win else n - T + 1 + t for n in lens for t in range(T))
    return {"bytes": keys * H_kv * packed + 4 * case["batch"] * T * H_q * d, "flops": 4 * pairs * H_q * d}


# ---------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)


def _rand(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _rope_settings(case):
    """Keyword arguments of the rotation, as a model's configuration states them."""
    scaling = case.get("scaling", "none")
    kw = dict(d=case["d"], rot_dim=case["rot"], base=500000.0, interleaved=case["layout"] == "interleaved")
    if scaling != "none":
        kw.update(scaling=scaling, factor=case["factor"], original_len=8192)
    return kw


def _tables(case, lens):
    """Block table over shuffled pages, as a server that hands out pages leaves it."""
    page = case["page"]
    need = [(n + page - 1) // page for n in lens]
    width, total = max(need), sum(need)
    order = list(range(total))
    random.Random(case["lens_seed"] + 1).shuffle(order)
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [0] * (width - n))
        at += n
    return torch.tensor(table, dtype=torch.int32, device="cuda"), total


def _quantise(x):
    """fp32 [..., d] -> codes [..., d] (fp32 whole numbers), (s, m) [..., d/64, 2] bf16."""
    g = x.unflatten(-1, (-1, GROUP))
    low = g.amin(-1).bfloat16()
    span = g.amax(-1) - low.float()
    step = (span / torch.full_like(span, 15.0)).clamp_min(0).bfloat16()   # tensor: a scalar divisor becomes a product
    s, m = step.float().unsqueeze(-1), low.float().unsqueeze(-1)
    n = torch.where(s > 0, torch.round((g - m) / s).clamp(0, 15), torch.zeros_like(g))
    return n.flatten(-2), torch.stack((step, low), -1)


def _pack(n):
    n = n.to(torch.uint8)
    return n[..., 0::2] | (n[..., 1::2] << 4)


def _filled_pages(case, seed, total):
    """4-bit pages whose keys have the clusters that attention meets; also the cluster centres."""
    g = _gen(seed)
    H, page, d = case["H_kv"], case["page"], case["d"]
    centres = 2.0 * _rand(g, H, 64, d)
    k = torch.empty((total, H, page, d // 2), dtype=torch.uint8, device="cuda")
    v = torch.empty_like(k)
    ks = torch.empty((total, H, page, d // GROUP, 2), dtype=torch.bfloat16, device="cuda")
    vs = torch.empty_like(ks)
    step = max(1, (1 << 25) // (H * page * d))
    for at in range(0, total, step):
        n = min(step, total - at)
        x = _rand(g, n, H, page, d)
        which = torch.randint(0, 256, (n, H, page), generator=g, device="cuda")
        near = which < 64                                           # a quarter of the keys lies near a centre
        pick = centres[torch.arange(H, device="cuda").view(1, H, 1), which.clamp_max(63)]
        x = torch.where(near.unsqueeze(-1), pick + 0.5 * x, x)
        codes, ks[at:at + n] = _quantise(x)
        k[at:at + n] = _pack(codes)
        codes, vs[at:at + n] = _quantise(_rand(g, n, H, page, d))
        v[at:at + n] = _pack(codes)
    return k, v, ks, vs, centres, g


def prepare(case, seed):
    dtype = TYPES[case["dtype"]] if "dtype" in case else None
    st = {"case": case}
    if case["op"] == "rope":
        g = _gen(seed)
        n = case["tokens"]
        st["q"] = _rand(g, n, case["H_q"], case["d"]).to(dtype)
        st["k"] = _rand(g, n, case["H_kv"], case["d"]).to(dtype)
        st["pos"] = torch.arange(case["first"], case["first"] + n, dtype=torch.int32, device="cuda")
        if own:
            from paper_2607_27692_b200 import paged
            st["rope"] = paged.Rope(**_rope_settings(case))
        return st

    lens, news = _lengths(case)
    B, H, d, page = case["batch"], case["H_kv"], case["d"], case["page"]
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    st["host_lens"] = lens
    st["table"], total = _tables(case, lens)
    if case["op"] == "append":
        g = _gen(seed)
        tok = sum(news)
        # q, k and v come as slices of one projection's output
        qkv = _rand(g, tok, case["H_q"] + 2 * H, d)
        qkv[:, case["H_q"]:case["H_q"] + H, :2] *= 4.0              # a few channels of a key are larger
        qkv = qkv.to(dtype)
        st["q"], st["k"], st["v"] = qkv.split([case["H_q"], H, H], 1)
        cu = [0]
        for n in news:
            cu.append(cu[-1] + n)
        st["host_cu"], st["host_news"] = cu, news
        st["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
        st["first"] = torch.tensor([n - m for n, m in zip(lens, news)], dtype=torch.int32, device="cuda")
        st["uniform"] = len(set(news)) == 1
        if case["fmt"] == "q4":
            st["k_pages"] = torch.zeros((total, H, page, d // 2), dtype=torch.uint8, device="cuda")
            st["v_pages"] = torch.zeros_like(st["k_pages"])
            st["k_scale"] = torch.zeros((total, H, page, d // GROUP, 2), dtype=torch.bfloat16, device="cuda")
            st["v_scale"] = torch.zeros_like(st["k_scale"])
            st["k_out"] = torch.zeros((B, H, max(news), d), dtype=torch.float32, device="cuda")
            st["v_out"] = torch.zeros_like(st["k_out"])
        else:
            st["k_pages"] = torch.zeros((total, H, page, d), dtype=dtype, device="cuda")
            st["v_pages"] = torch.zeros_like(st["k_pages"])
            st["k_scale"] = st["v_scale"] = None
        if own:
            from paper_2607_27692_b200 import paged
            st["rope"] = paged.Rope(**_rope_settings(case))
            st["pages"] = paged.KVPages.wrap(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
        return st

    st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], centres, g = _filled_pages(case, seed, total)
    if case["op"] == "gather":
        out = TYPES[case["out"]]
        st["k_out"] = torch.zeros((B, H, max(lens), d), dtype=out, device="cuda")
        st["v_out"] = torch.zeros_like(st["k_out"])
    else:
        G = case["H_q"] // H
        q = _rand(g, B, case["T"], H, G, d)
        towards = torch.randint(0, 64, (B, case["T"], H, G), generator=g, device="cuda")
        q = 0.7 * q + 0.25 * centres[torch.arange(H, device="cuda").view(1, 1, H, 1), towards]
        st["q"] = q.view(B, case["T"], case["H_q"], d).to(dtype)
    if own:
        from paper_2607_27692_b200 import paged
        st["pages"] = paged.KVPages.wrap(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
    return st


# ---------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    case = st["case"]
    if case["op"] == "rope":
        return st["rope"].apply_pair(st["q"], st["k"], st["pos"], inverse=case["inverse"])
    if case["op"] == "append":
        q = st["pages"].append(st["k"], st["v"], st["lens"], st["table"], None if st["uniform"] else st["cu"],
                               rope=st["rope"], q=st["q"])
        if case["fmt"] != "q4":
            return q, st["k_pages"], st["v_pages"]
        st["pages"].gather(st["k_out"], st["v_out"], st["lens"], st["table"], first=st["first"])
        return q, st["k_out"], st["v_out"]
    if case["op"] == "gather":
        st["pages"].gather(st["k_out"], st["v_out"], st["lens"], st["table"])
        return st["k_out"], st["v_out"]
    return st["pages"].attend(st["q"], st["lens"], st["table"], window=case["window"])


def _frequencies(case):
    """Radians per position of each pair (fp64), and the factor on cosine and sine."""
    kw = _rope_settings(case)
    rot, base = kw["rot_dim"], kw["base"]
    scaling, f, orig = kw.get("scaling", "none"), kw.get("factor", 1.0), kw.get("original_len", 0)
    i = torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot
    if scaling == "ntk":
        base = base * f ** (rot / (rot - 2))
    w = base ** -i
    if scaling == "linear":
        w = w / f
    elif scaling == "llama3":                                      # low and high frequency factors 1 and 4
        blend = ((orig * w / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        w = (1.0 - blend) * w / f + blend * w
    elif scaling == "yarn":                                        # 32 and 1 rotations over the original length
        def pair_of(turns):
            return rot * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), rot - 1)
        ramp = ((torch.arange(rot // 2, dtype=torch.float64, device="cuda") - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
        w = ramp * w / f + (1.0 - ramp) * w
        return w, 0.1 * math.log(f) + 1.0
    return w, 1.0


def _turn(x, pos, w, factor, layout, inverse=False):
    """Rotate x [N, H, d] at positions [N]; 64 bits, because rounding to codes and far angles need them."""
    angle = pos.double().unsqueeze(-1) * w
    cos, sin = (factor * angle.cos()).unsqueeze(1), (factor * angle.sin()).unsqueeze(1)
    if inverse:
        sin = -sin
    rot = 2 * w.numel()
    y = x.double()
    out = y.clone()
    if layout == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        out[..., :rot // 2], out[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    return out.to(x.dtype)


def _values(codes, scale):
    """Packed codes [..., d/2] and (s, m) [..., d/64, 2] -> fp32 values [..., d]."""
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float().unflatten(-1, (-1, GROUP))
    s, m = scale.float().unbind(-1)
    return (n * s.unsqueeze(-1) + m.unsqueeze(-1)).flatten(-2)


def _rows(st, b, n, name):
    """fp32 [H_kv, n, d]: the first n rows of sequence b in the 4-bit cache."""
    page = st["case"]["page"]
    ids = st["table"][b, :(n + page - 1) // page].long()
    x = _values(st[name + "_pages"][ids], st[name + "_scale"][ids])
    return x.transpose(0, 1).flatten(1, 2)[:, :n]


def _run_plain(st):
    case = st["case"]
    if case["op"] == "rope":
        w, factor = _frequencies(case)
        return tuple(_turn(st[x], st["pos"], w, factor, case["layout"], case["inverse"]) for x in ("q", "k"))
    if case["op"] == "append":
        w, factor = _frequencies(case)
        cu, page = st["host_cu"], case["page"]
        news = st["cu"][1:] - st["cu"][:-1]
        seq = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"), news, output_size=cu[-1])
        at = torch.arange(cu[-1], device="cuda") - st["cu"][seq]
        pos = st["first"][seq] + at
        q = _turn(st["q"], pos, w, factor, case["layout"])
        k, v = _turn(st["k"], pos, w, factor, case["layout"]), st["v"]
        ids, row = st["table"][seq, pos // page].long(), pos % page
        if case["fmt"] != "q4":
            st["k_pages"][ids, :, row], st["v_pages"][ids, :, row] = k, v
            return q, st["k_pages"], st["v_pages"]
        for x, name in ((k, "k"), (v, "v")):
            codes, scale = _quantise(x.float())
            st[name + "_pages"][ids, :, row], st[name + "_scale"][ids, :, row] = _pack(codes), scale
            st[name + "_out"][seq, :, at] = _values(st[name + "_pages"][ids, :, row], st[name + "_scale"][ids, :, row])
        return q, st["k_out"], st["v_out"]
    if case["op"] == "gather":
        for b, n in enumerate(st["host_lens"]):
            for name in ("k", "v"):
                st[name + "_out"][b, :, :n] = _rows(st, b, n, name).to(st[name + "_out"].dtype)
        return st["k_out"], st["v_out"]
    B, T, H, d = case["batch"], case["T"], case["H_kv"], case["d"]
    G = case["H_q"] // H
    out = torch.empty_like(st["q"])
    for b, n in enumerate(st["host_lens"]):
        lo = max(0, n - T + 1 - case["window"]) if case["window"] else 0
        k, v = _rows(st, b, n, "k")[:, lo:], _rows(st, b, n, "v")[:, lo:]
        q = st["q"][b].float().view(T, H, G, d).permute(1, 0, 2, 3).reshape(H, T * G, d)
        s = torch.matmul(q, k.transpose(1, 2)) * d ** -0.5
        if T > 1 or case["window"]:
            key = torch.arange(lo, n, device="cuda")
            at = torch.arange(n - T, n, device="cuda").repeat_interleave(G).unsqueeze(1)
            hidden = key > at
            if case["window"]:
                hidden = hidden | (key <= at - case["window"])
            s = s.masked_fill(hidden, float("-inf"))
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
        out[b] = o.view(H, T, G, d).permute(1, 0, 2, 3).reshape(T, case["H_q"], d).to(out.dtype)
    return out


# ---------------------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------
def _exact_rotation(case, x, pos, inverse=False):
    """Each pair is a complex number, multiplied by a * exp(i * pos * w)."""
    kw = _rope_settings(case)
    rot, base, kind = kw["rot_dim"], kw["base"], kw.get("scaling", "none")
    f, orig = kw.get("factor", 1.0), kw.get("original_len", 0)
    amplitude = 0.1 * math.log(f) + 1.0 if kind == "yarn" else 1.0
    if kind == "ntk":
        base *= f ** (rot / (rot - 2.0))
    speeds = []
    for i in range(rot // 2):
        w = math.pow(base, -2.0 * i / rot)
        if kind == "linear":
            w /= f
        elif kind == "llama3":
            wavelength = 2.0 * math.pi / w
            if wavelength > orig / 1.0:
                w /= f
            elif wavelength > orig / 4.0:
                t = (orig / wavelength - 1.0) / 3.0
                w = (1.0 - t) * w / f + t * w
        elif kind == "yarn":
            lo = max(0, math.floor(rot * math.log(orig / (32.0 * 2.0 * math.pi)) / (2.0 * math.log(base))))
            hi = min(rot - 1, math.ceil(rot * math.log(orig / (2.0 * math.pi)) / (2.0 * math.log(base))))
            t = min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))
            w = t * w / f + (1.0 - t) * w
        speeds.append(w)
    angle = pos.double()[:, None] * torch.tensor(speeds, dtype=torch.float64, device=x.device)[None]
    spin = torch.polar(torch.full_like(angle, amplitude), -angle if inverse else angle)[:, None]
    y = x.double()
    if case["layout"] == "half":
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * spin
        turned = torch.cat((z.real, z.imag), -1)
    else:
        turned = torch.view_as_real(torch.view_as_complex(y[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * spin).flatten(-2)
    return torch.cat((turned, y[..., rot:]), -1)


def _exact_code_values(x):
    """The values that a row stands for once it is held in 4 bits (x: the stored type's values, fp64)."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[-1], GROUP):
        g = x[..., c:c + GROUP]
        m = g.min(-1, keepdim=True).values.to(torch.bfloat16).double()
        s = (g.max(-1, keepdim=True).values - m).clamp_min(0.0)
        s = torch.div(s, torch.full_like(s, 15.0)).to(torch.bfloat16).double()
        n = ((g - m) / torch.where(s > 0, s, torch.ones_like(s))).round().clamp(0.0, 15.0) * (s > 0)
        out[..., c:c + GROUP] = s * n + m
    return out


def _exact_sequence(st, b, n, name):
    """fp64 [H_kv, n, d] of a sequence in the 4-bit cache, page by page order of its table row."""
    case = st["case"]
    ids = st["table"][b].long()
    j = torch.arange(n, device="cuda")
    packed = st[name + "_pages"][ids[j // case["page"]], :, j % case["page"]]          # [n, H, d/2]
    scale = st[name + "_scale"][ids[j // case["page"]], :, j % case["page"]].double()  # [n, H, d/64, 2]
    x = torch.empty(packed.shape[:2] + (case["d"],), dtype=torch.float64, device="cuda")
    x[..., 0::2] = (packed % 16).double()
    x[..., 1::2] = torch.div(packed, 16, rounding_mode="floor").double()
    for c in range(case["d"] // GROUP):
        part = x[..., c * GROUP:(c + 1) * GROUP]
        part.mul_(scale[..., c, 0:1]).add_(scale[..., c, 1:2])
    return x.transpose(0, 1)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return tuple(_exact_rotation(case, st[x], st["pos"], case["inverse"]) for x in ("q", "k"))
    if case["op"] == "append":
        lens, news, cu = st["host_lens"], st["host_news"], st["host_cu"]
        pos = torch.tensor([n - m + i for n, m in zip(lens, news) for i in range(m)], device="cuda")
        q, k = _exact_rotation(case, st["q"], pos), _exact_rotation(case, st["k"], pos)
        v = st["v"].double()
        if case["fmt"] == "q4":
            outs = [torch.zeros(st["k_out"].shape, dtype=torch.float64, device="cuda") for _ in "kv"]
            rows = [_exact_code_values(k.to(st["k"].dtype).double()), _exact_code_values(v)]
            for b, n in enumerate(news):
                for out, x in zip(outs, rows):
                    out[b, :, :n] = x[cu[b]:cu[b + 1]].transpose(0, 1)
            return q, outs[0], outs[1]
        outs = [torch.zeros(st["k_pages"].shape, dtype=torch.float64, device="cuda") for _ in "kv"]
        for b, n in enumerate(news):
            p = pos[cu[b]:cu[b + 1]]
            ids = st["table"][b].long()[p // case["page"]]
            for out, x in zip(outs, (k, v)):
                out[ids, :, p % case["page"]] = x[cu[b]:cu[b + 1]]
        return q, outs[0], outs[1]
    if case["op"] == "gather":
        outs = [torch.zeros(st["k_out"].shape, dtype=torch.float64, device="cuda") for _ in "kv"]
        for b, n in enumerate(st["host_lens"]):
            for out, name in zip(outs, "kv"):
                out[b, :, :n] = _exact_sequence(st, b, n, name)
        return outs[0], outs[1]
    T, H_q, H, d = case["T"], case["H_q"], case["H_kv"], case["d"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(st["host_lens"]):
        k, v = _exact_sequence(st, b, n, "k"), _exact_sequence(st, b, n, "v")
        for t in range(T):
            last = n - T + t
            lo = max(0, last + 1 - case["window"]) if case["window"] else 0
            q = st["q"][b, t].double().view(H, H_q // H, d)
            p = torch.softmax(q @ k[:, lo:last + 1].transpose(1, 2) / math.sqrt(d), -1)
            out[b, t] = (p @ v[:, lo:last + 1]).view(H_q, d)
    return out
