"""Rotary positions, paged key/value caches and attention over a 4-bit cache (binding).

What a decode loop needs around :class:`paper_2607_27692_b200.retopk.ReTopK`::

    rope = Rope(128, base=500000.0, scaling="llama3", factor=8.0, original_len=8192)

    # the contiguous cache of ReTopK.decode_step: sequence b owns page b
    cache = KVPages.wrap(k_cache, v_cache)                # [B, H_kv, max_seq_len, d]
    q = cache.append(k_new, v_new, seq_lens, rope=rope, q=q_new)
    out = ctx.decode_step(q, k_cache, v_cache, seq_len)

    # a cache in 4 bits, in pages
    cache = KVPages(n_pages, H_kv, 64, 128, "q4")
    q = cache.append(k_new, v_new, seq_lens, block_table, rope=rope, q=q_new)
    out = cache.attend(q, seq_lens, block_table)

The arithmetic runs in ``libretopk.so`` (``include/retopk.h`` states it); this module checks the
tensors and passes pointers.  Work is enqueued on the current stream of the tensors' device; nothing
is kept between calls, so calls on several streams and captured graphs do not share anything here.
As with any kernel, the library's first call on a device loads code: make it before capturing.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import retopk as _rt
from .retopk import _check, _vp

_TYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_HALF = (torch.bfloat16, torch.float16)
_FORMATS = {"bf16": (0, torch.bfloat16), "fp16": (1, torch.float16), "q4": (2, torch.uint8)}
_SCALINGS = {None: 0, "linear": 1, "ntk": 2, "llama3": 3, "yarn": 4}
GROUP = 64      # channels that share a step and a minimum in the 4-bit format


class _RopeConfig(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("d", "rot_dim", "layout", "scaling")] +
                [(n, C.c_double) for n in ("base", "factor", "original_len", "low_freq_factor", "high_freq_factor",
                                           "beta_fast", "beta_slow", "attn_factor")])


class _Pages(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("format", "H_kv", "d", "page_size")] + [("n_pages", C.c_int64)] +
                [(n, _vp) for n in ("k", "v", "k_scale", "v_scale", "block_table")] + [("max_pages", C.c_int64)])


# Both cost a tenth of a microsecond; the public forms cost three, as much as a launch.
_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


def _call(device, fn, *args):
    """fn(*args, stream) on the current stream of `device`, which is made current for the call."""
    index = device.index
    if _current_device() == index:
        return fn(*args, _current_stream(index))
    with torch.cuda.device(device):
        return fn(*args, _current_stream(index))


def _rows(t, what, device, dtype, n, heads, d):
    """Pointer and token stride of a token-major [n, heads, d] tensor whose heads lie d apart."""
    if t.device != device or t.dtype != dtype:
        raise TypeError(f"{what}: expected {dtype} on {device}, got {t.dtype} on {t.device}")
    if t.dim() != 3 or t.shape != (n, heads, d):
        raise ValueError(f"{what}: expected shape {(n, heads, d)}, got {tuple(t.shape)}")
    s = t.stride()
    if s[2] != 1 or (heads > 1 and s[1] != d):
        raise ValueError(f"{what}: the heads of a token have to lie {d} elements apart, strides are {s}")
    return t.data_ptr(), (s[0] if n > 1 else heads * d)


def _ints(t, what, device, shape):
    if t.device != device or t.dtype != torch.int32 or not t.is_contiguous():
        raise TypeError(f"{what}: expected a contiguous int32 tensor on {device}, got {t.dtype} on {t.device}")
    if t.shape != shape:
        raise ValueError(f"{what}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _half_rows(t, what):
    if not t.is_cuda or t.dtype not in _HALF:
        raise TypeError(f"{what}: expected a bf16 or fp16 CUDA tensor, got {t.dtype} on {t.device}")
    if t.dim() != 3:
        raise ValueError(f"{what}: expected [tokens, heads, d], got {tuple(t.shape)}")


class Rope:
    """Rotary positions of one model (wraps a ``retopk_rope*``; host memory only, any device).

    ``rot_dim`` channels of a head of ``d`` are rotated (default: all), paired in halves or, with
    ``interleaved``, as neighbours.  ``scaling``: None, "linear", "ntk", "llama3" or "yarn".
    """

    def __init__(self, d, rot_dim=None, base=10000.0, interleaved=False, scaling=None, factor=1.0, original_len=0,
                 low_freq_factor=0.0, high_freq_factor=0.0, beta_fast=0.0, beta_slow=0.0, attn_factor=0.0):
        self.h = None
        if scaling not in _SCALINGS:
            raise ValueError(f"scaling: one of {list(_SCALINGS)}, got {scaling!r}")
        self.lib = _rt.load()
        self.d, self.rot_dim = d, d if rot_dim is None else rot_dim
        cfg = _RopeConfig(d, self.rot_dim, int(bool(interleaved)), _SCALINGS[scaling], base, factor, original_len,
                          low_freq_factor, high_freq_factor, beta_fast, beta_slow, attn_factor)
        h = _vp()
        _check(self.lib.retopk_rope_create(C.byref(h), C.byref(cfg)), "retopk_rope_create")
        self.h = h

    def close(self):
        if self.h is not None:
            self.lib.retopk_rope_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def frequencies(self):
        """Radians per position of each pair (list), and the factor on cosine and sine."""
        w, a = (C.c_double * (self.rot_dim // 2))(), C.c_double()
        _check(self.lib.retopk_rope_frequencies(self.h, w, C.byref(a)), "retopk_rope_frequencies")
        return list(w), float(a.value)

    def apply(self, x, positions, out=None, inverse=False):
        """Rotate x [tokens, heads, d] at int32 ``positions``; ``out`` may be x itself."""
        return self.apply_pair(x, None, positions, out, None, inverse)[0]

    def apply_pair(self, q, k, positions, q_out=None, k_out=None, inverse=False):
        """Rotate queries and keys in one launch.  ``inverse``: the transpose, i.e. the gradient."""
        _half_rows(q, "q")
        (n, H_q, d), dev, dt = q.shape, q.device, q.dtype
        qp, qs = _rows(q, "q", dev, dt, n, H_q, self.d)
        if q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            qop, qos = q_out.data_ptr(), H_q * d
        else:
            qop, qos = _rows(q_out, "q_out", dev, dt, n, H_q, d)
        kp, ks, kop, kos, H_k = None, 0, None, 0, 0
        if k is not None:
            H_k = k.shape[1] if k.dim() == 3 else 0
            kp, ks = _rows(k, "k", dev, dt, n, H_k, d)
            if k_out is None:
                k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
                kop, kos = k_out.data_ptr(), H_k * d
            else:
                kop, kos = _rows(k_out, "k_out", dev, dt, n, H_k, d)
        pos = _ints(positions, "positions", dev, (n,))
        if n == 0:
            return q_out, k_out
        rc = _call(dev, self.lib.retopk_rope_apply, self.h, _TYPE[dt], n, pos, qp, qs, qop, qos, H_q, kp, ks, kop, kos,
                   H_k, 1 if inverse else 0)
        if rc:
            _check(rc, "retopk_rope_apply")
        return q_out, k_out


class KVPages:
    """Keys and values of one layer in pages of ``page_size`` rows.

    ``fmt`` "bf16" / "fp16": ``k``, ``v`` [n_pages, H_kv, page_size, d].  "q4": ``k``, ``v`` uint8
    [.., d/2], two codes to a byte, even channel low, and ``k_scale``, ``v_scale`` bf16 [.., d/64, 2]:
    step and minimum of each group of 64 channels.
    """

    def __init__(self, n_pages, H_kv, page_size, d, fmt="q4", device="cuda"):
        if fmt not in _FORMATS:
            raise ValueError(f"fmt: one of {list(_FORMATS)}, got {fmt!r}")
        q4 = fmt == "q4"
        shape = (n_pages, H_kv, page_size)
        k = torch.zeros(shape + (d // 2 if q4 else d,), dtype=_FORMATS[fmt][1], device=device)
        scale = torch.zeros(shape + (d // GROUP, 2), dtype=torch.bfloat16, device=device) if q4 else None
        self._set(k, torch.zeros_like(k), scale, None if scale is None else torch.zeros_like(scale))

    @classmethod
    def wrap(cls, k, v, k_scale=None, v_scale=None):
        """Use existing tensors, among them the [B, H_kv, max_seq_len, d] cache of ReTopK.decode_step."""
        self = cls.__new__(cls)
        self._set(k, v, k_scale, v_scale)
        return self

    def _set(self, k, v, k_scale, v_scale):
        self.lib = _rt.load()
        if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype:
            raise ValueError(f"k and v: two tensors [n_pages, H_kv, page_size, ..], got {tuple(k.shape)} and {tuple(v.shape)}")
        q4 = k.dtype == torch.uint8
        if not q4 and k.dtype not in _HALF:
            raise TypeError(f"k and v: bf16, fp16 or uint8 (4 bits), got {k.dtype}")
        self.n_pages, self.H_kv, self.page_size = k.shape[:3]
        self.d = k.shape[3] * 2 if q4 else k.shape[3]
        if q4:
            want = (self.n_pages, self.H_kv, self.page_size, self.d // GROUP, 2)
            for name, s in (("k_scale", k_scale), ("v_scale", v_scale)):
                if s is None or s.dtype != torch.bfloat16 or s.shape != want:
                    raise ValueError(f"{name}: a 4-bit cache needs bf16 {want}")
        elif k_scale is not None or v_scale is not None:
            raise ValueError("k_scale, v_scale: only a 4-bit cache has them")
        for t in (k, v, k_scale, v_scale):
            if t is not None and (not t.is_cuda or t.device != k.device or not t.is_contiguous()):
                raise TypeError("the tensors of a cache have to be contiguous on one CUDA device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.fmt = "q4" if q4 else ("bf16" if k.dtype == torch.bfloat16 else "fp16")
        self.device = k.device
        self._needs = {}             # workspace bytes by (B, T, H_q)
        self._head = (_FORMATS[self.fmt][0], self.H_kv, self.d, self.page_size, self.n_pages, k.data_ptr(), v.data_ptr(),
                      k_scale.data_ptr() if q4 else None, v_scale.data_ptr() if q4 else None)

    def _pages(self, B, block_table):
        if block_table is None:
            return C.byref(_Pages(*self._head, None, 0))
        if block_table.dim() != 2:
            raise ValueError(f"block_table: expected [{B}, pages], got {tuple(block_table.shape)}")
        width = block_table.shape[1]
        return C.byref(_Pages(*self._head, _ints(block_table, "block_table", self.device, (B, width)), width))

    def append(self, k_new, v_new, seq_lens, block_table=None, cu_new=None, rope=None, q=None, q_out=None):
        """Store new keys and values [tokens, H_kv, d], rotated by ``rope`` on the way.

        ``seq_lens`` int32 [B] counts each sequence's keys including the new ones.  Sequence b's new
        tokens are rows cu_new[b]:cu_new[b+1] (int32 [B + 1]); without ``cu_new`` every sequence has
        the same number.  With ``q`` the queries are rotated in the same launch and returned; rows of
        ``q_out`` that belong to no token are left as they were.
        """
        _half_rows(k_new, "k_new")
        dev, dt, n, d = self.device, k_new.dtype, k_new.shape[0], self.d
        if seq_lens.dim() != 1:
            raise ValueError(f"seq_lens: expected one length per sequence, got {tuple(seq_lens.shape)}")
        B = seq_lens.shape[0]
        lens = _ints(seq_lens, "seq_lens", dev, (B,))
        kp, ks = _rows(k_new, "k_new", dev, dt, n, self.H_kv, d)
        vp, vs = _rows(v_new, "v_new", dev, dt, n, self.H_kv, d)
        cu = None if cu_new is None else _ints(cu_new, "cu_new", dev, (B + 1,))
        if cu is None and B > 0 and n % B:
            raise ValueError(f"{n} new tokens do not divide among {B} sequences: pass cu_new")
        qp, qs, qop, qos, H_q = None, 0, None, 0, 0
        if q is not None:
            if rope is None:
                raise ValueError("q is rotated with the keys: pass rope")
            _half_rows(q, "q")
            H_q = q.shape[1]
            qp, qs = _rows(q, "q", dev, dt, n, H_q, d)
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                qop, qos = q_out.data_ptr(), H_q * d
            else:
                qop, qos = _rows(q_out, "q_out", dev, dt, n, H_q, d)
        pages = self._pages(B, block_table)
        if n == 0:
            return q_out
        rc = _call(dev, self.lib.retopk_kv_append, pages, B, lens, cu, n, _TYPE[dt], kp, ks, vp, vs,
                   None if rope is None else rope.h, qp, qs, qop, qos, H_q)
        if rc:
            _check(rc, "retopk_kv_append")
        return q_out

    def gather(self, k_out, v_out, seq_lens, block_table=None, first=None):
        """Read rows back into k_out / v_out [B, H_kv, rows, d] (either may be None).

        Row i of sequence b is the cache's row first[b] + i, up to seq_lens[b]; others stay as they are.
        """
        ref = k_out if k_out is not None else v_out
        if ref is None:
            raise ValueError("gather: pass k_out, v_out or both")
        if ref.dim() != 4 or ref.shape[1] != self.H_kv or ref.shape[3] != self.d:
            raise ValueError(f"k_out, v_out: expected [B, {self.H_kv}, rows, {self.d}], got {tuple(ref.shape)}")
        B, rows, dt = ref.shape[0], ref.shape[2], ref.dtype
        if dt not in _TYPE:
            raise TypeError(f"k_out, v_out: bf16, fp16 or fp32, got {dt}")
        for t in (k_out, v_out):
            if t is not None and (t.device != self.device or t.dtype != dt or t.shape != ref.shape or not t.is_contiguous()):
                raise TypeError(f"k_out, v_out: contiguous {dt} {tuple(ref.shape)} on {self.device}")
        lens = _ints(seq_lens, "seq_lens", self.device, (B,))
        start = None if first is None else _ints(first, "first", self.device, (B,))
        pages = self._pages(B, block_table)
        if ref.numel() == 0:
            return k_out, v_out
        rc = _call(self.device, self.lib.retopk_kv_gather, pages, B, lens, start, rows, _TYPE[dt],
                   None if k_out is None else k_out.data_ptr(), None if v_out is None else v_out.data_ptr())
        if rc:
            _check(rc, "retopk_kv_gather")
        return k_out, v_out

    def attend(self, q, seq_lens, block_table=None, scale=None, window=0, out=None, lse=None):
        """Attention of the last T tokens of every sequence over a 4-bit cache.

        q [B, H_q, d] (one token) or [B, T, H_q, d]; the result has q's shape and type.  ``scale``
        defaults to d ** -0.5; ``window`` > 0 limits a token to its last ``window`` keys; ``lse``
        fp32, of q's shape without d, takes the logarithm of the sum of exponentials.
        """
        if self.fmt != "q4":
            raise TypeError(f"attend reads 4-bit pages, this cache holds {self.fmt}")
        dev = self.device
        if q.device != dev or q.dtype not in _HALF:
            raise TypeError(f"q: expected bf16 or fp16 on {dev}, got {q.dtype} on {q.device}")
        if q.dim() not in (3, 4) or q.shape[-1] != self.d:
            raise ValueError(f"q: expected [B, H_q, {self.d}] or [B, T, H_q, {self.d}], got {tuple(q.shape)}")
        B, T, H_q = q.shape[0], q.shape[1] if q.dim() == 4 else 1, q.shape[-2]
        s = q.stride()
        if s[-1] != 1 or (H_q > 1 and s[-2] != self.d) or (q.dim() == 4 and T > 1 and B > 1 and s[0] != T * s[1]):
            raise ValueError(f"q: tokens have to lie one stride apart and heads {self.d} elements apart, strides are {s}")
        q_stride = H_q * self.d if B * T <= 1 else (s[0] if q.dim() == 3 or T == 1 else s[1])
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.device != dev or out.dtype != q.dtype or out.shape != q.shape or not out.is_contiguous():
            raise TypeError(f"out: contiguous {q.dtype} {tuple(q.shape)} on {dev}")
        if lse is not None and (lse.device != dev or lse.dtype != torch.float32 or lse.shape != q.shape[:-1] or
                                not lse.is_contiguous()):
            raise TypeError(f"lse: contiguous fp32 {tuple(q.shape[:-1])} on {dev}")
        lens = _ints(seq_lens, "seq_lens", dev, (B,))
        pages = self._pages(B, block_table)
        if B == 0:
            return out
        rc = _call(dev, self._attend, pages, B, T, H_q, lens, _TYPE[q.dtype], q.data_ptr(), q_stride,
                   self.d ** -0.5 if scale is None else scale, window, out.data_ptr(), None if lse is None else lse.data_ptr())
        if rc:
            _check(rc, "retopk_q4_attention")
        return out

    def _attend(self, pages, B, T, H_q, *rest):
        # (with the device current: the workspace's size depends on it)
        need = self._needs.get((B, T, H_q))
        if need is None:
            need = self.lib.retopk_q4_attention_workspace(B, T, H_q, self.H_kv, self.d)
            if need < 0:
                return int(need)
            self._needs[B, T, H_q] = need
        # from torch's allocator: tied to this stream (and, under capture, to the graph's own pool)
        ws = self.k.new_empty(need)
        return self.lib.retopk_q4_attention(pages, B, T, H_q, *rest[:-1], ws.data_ptr(), need, rest[-1])
