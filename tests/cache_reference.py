"""Plain 64-bit forms of the operators around the KV cache, and the error bounds of the kernels."""
import math

import torch

GROUP = 64


def half_step(dtype):
    """Largest relative error of one rounding to dtype."""
    return torch.finfo(dtype).eps / 2


def frequencies(rot, base=10000.0, scaling=None, factor=1.0, original_len=0, low=1.0, high=4.0, fast=32.0, slow=1.0):
    """Radians per position of each pair, amplitude (formulas of include/retopk.h, pair by pair)."""
    out = []
    b = base * factor ** (rot / (rot - 2.0)) if scaling == "ntk" else base
    for i in range(rot // 2):
        w = b ** (-2.0 * i / rot)
        if scaling == "linear":
            w /= factor
        elif scaling == "llama3":
            wavelength = 2 * math.pi / w
            if wavelength > original_len / low:
                w /= factor
            elif wavelength >= original_len / high:
                t = (original_len / wavelength - low) / (high - low)
                w = (1 - t) * w / factor + t * w
        elif scaling == "yarn":
            lo = max(math.floor(rot * math.log(original_len / (fast * 2 * math.pi)) / (2 * math.log(base))), 0)
            hi = min(math.ceil(rot * math.log(original_len / (slow * 2 * math.pi)) / (2 * math.log(base))), rot - 1)
            t = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            w = t * w / factor + (1 - t) * w
        out.append(w)
    return out, (0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0)


def rotate(x, pos, w, amp=1.0, interleaved=False, inverse=False):
    """x [n, heads, d] (any type) -> fp64, unrounded; differentiable."""
    y = x.double()
    ang = pos.double()[:, None] * torch.tensor(w, dtype=torch.float64, device=x.device)[None]
    c, s = amp * torch.cos(ang)[:, None], amp * torch.sin(ang)[:, None]
    if inverse:
        s = -s
    rot = 2 * len(w)
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat((a * c - b * s, a * s + b * c), -1)
    return torch.cat((turned, y[..., rot:]), -1)


def quantise(x):
    """16-bit tensor [..., d] -> codes [..., d] (int64), step and minimum [..., d/64] (fp64)."""
    g = x.double().unflatten(-1, (-1, GROUP))
    low = g.amin(-1).to(torch.bfloat16).double()
    span = (g.amax(-1) - low).clamp_min(0)
    step = (span / torch.full_like(span, 15)).to(torch.bfloat16).double()
    s = step.unsqueeze(-1)
    n = ((g - low.unsqueeze(-1)) / torch.where(s > 0, s, torch.ones_like(s))).round().clamp(0, 15) * (s > 0)
    return n.long().flatten(-2), step, low


def pack(n):
    n = n.to(torch.uint8)
    return n[..., 0::2] | (n[..., 1::2] << 4)


def values(codes, scale):
    """Packed codes [..., d/2] uint8, scale [..., d/64, 2] -> fp64 values."""
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).double().unflatten(-1, (-1, GROUP))
    sc = scale.double()
    return (n * sc[..., 0:1] + sc[..., 1:2]).flatten(-2)


def rows_of(pages, scale, table, b, n, page_size):
    """fp64 [H_kv, n, d] of sequence b (table None: page b)."""
    j = torch.arange(n, device=pages.device)
    ids = torch.full_like(j, b) if table is None else table[b].long()[j // page_size]
    x = pages[ids, :, j % page_size]
    x = x.double() if scale is None else values(x, scale[ids, :, j % page_size])
    return x.transpose(0, 1)


def attention(q, k, v, scale, window=0, ok=None):
    """q [T, H_q, d], k / v fp64 [H_kv, n, d] -> out [T, H_q, d], lse [T, H_q] (fp64); ok [n]: keys that count."""
    T, H_q, d = q.shape
    H, n = k.shape[:2]
    out = torch.zeros(T, H_q, d, dtype=torch.float64, device=q.device)
    lse = torch.full((T, H_q), -math.inf, dtype=torch.float64, device=q.device)
    j = torch.arange(n, device=q.device)
    for t in range(T):
        last = n - T + t
        m = j <= last
        if window:
            m &= j > last - window
        if ok is not None:
            m &= ok
        if not bool(m.any()):
            continue
        s = (q[t].double().view(H, H_q // H, d) @ k[:, m].transpose(1, 2)) * scale
        lse[t] = torch.logsumexp(s, -1).flatten()
        out[t] = (torch.softmax(s, -1) @ v[:, m]).view(H_q, d)
    return out, lse


def attention_bounds(q, k_scale, v_scale, v, scale, n, dtype):
    """(bound on |lse error|, absolute part of the bound on |out error|); q [.., d].

    Scores.  Queries may become whole numbers of a unit that puts the largest element of a row between
    2^13.99 and 2^15 of them: element c is off by e_c = |q_c - unit * round(q_c / unit)|, worked out here,
    and a group's sum of codes (at most 15) times step by 15 * step * sum of e_c.  Whole-number sums are
    exact.  Or they stay 16-bit numbers: at most 8 additions in fp32, each off by 2^-23 (truncation) of
    partial sums below 15 * sum |q|.  Then a conversion and at most 7 fp32 operations, 2^-24 each, on
    values up to (15 * step + |minimum|) * sum |q|: 16 * 2^-24 in all cover both.
    The exponential: off by e in the score is off by the factor 1 + e; lse adds its own fp32 steps.

    Output.  Weights off by 1 + e on both sides of the quotient: 2 e * max |v|; weights as two truncated
    bf16 parts: 2^-16, likewise.  Sums of codes: at most 12 products in a row in the tensor core, each
    addition off by 2^-23 of a partial sum below 16 * step (bytes up to 255, divided by 16 at the end), for
    weights that sum to 1; then n / 192 rounded additions, 2^-24 each; joining warps and CTAs is within
    64 more.  Sums of minima: n / 32 rounded additions to a lane, of partial sums below |minimum|.
    """
    q = q.double()
    sumq = q.abs().sum(-1).max().item()
    big = q.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -126)
    unit = torch.exp2(torch.floor(torch.log2(big)) - 14)
    unit = torch.where(big / unit > 32512, 2 * unit, unit)
    rounded = (q - unit * torch.round(q / unit)).abs().sum(-1).max().item()
    ks, km = k_scale[..., 0].double().abs().max().item(), k_scale[..., 1].double().abs().max().item()
    vs, vm = v_scale[..., 0].double().abs().max().item(), v_scale[..., 1].double().abs().max().item()
    err = abs(scale) * (15 * ks * rounded + 2.0 ** -20 * sumq * (15 * ks + km))
    vmax = v.abs().max().item() if v.numel() else 0.0
    out = 2 * (err + 2.0 ** -16) * vmax + (n / 384 + 76) * 2.0 ** -23 * 16 * vs + (n / 32 + 64) * 2.0 ** -24 * vm
    return err + 2.0 ** -20 * (1 + abs(math.log(max(n, 2)))), out
