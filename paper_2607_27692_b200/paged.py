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

The rotation is differentiable.  The calls of a cache are for serving: they have no gradient and refuse
tensors that require one unless under ``torch.no_grad()``.

The arithmetic runs in ``libretopk.so`` (``include/retopk.h`` states it); ``_paged.so``
(``csrc/paged_binding.cpp``) checks the tensors and passes pointers.  Work is enqueued on the current stream of the tensors' device; nothing
is kept between calls, so calls on several streams and captured graphs do not share anything here.
As with any kernel, the library's first call on a device loads code: make it before capturing.  A rotation's
backward pass may be captured with its forward pass; as for any operator of torch, no eager graph of the same
leaves may be alive then (torch's gradient accumulators remember the stream that they were made on).
"""
from __future__ import annotations

import ctypes as C
import importlib
import os

import torch

from . import build as _build
from . import retopk as _rt
from .retopk import _check, _vp

_HALF = (torch.bfloat16, torch.float16)
_FORMATS = {"bf16": (0, torch.bfloat16), "fp16": (1, torch.float16), "q4": (2, torch.uint8)}
_SCALINGS = {None: 0, "linear": 1, "ntk": 2, "llama3": 3, "yarn": 4}
GROUP = 64      # channels that share a step and a minimum in the 4-bit format


class _RopeConfig(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("d", "rot_dim", "layout", "scaling")] +
                [(n, C.c_double) for n in ("base", "factor", "original_len", "low_freq_factor", "high_freq_factor",
                                           "beta_fast", "beta_slow", "attn_factor")])


class _Pages(C.Structure):
    """``retopk_pages_t``, for callers of the C interface."""

    _fields_ = ([(n, C.c_int) for n in ("format", "H_kv", "d", "page_size")] + [("n_pages", C.c_int64)] +
                [(n, _vp) for n in ("k", "v", "k_scale", "v_scale", "block_table")] + [("max_pages", C.c_int64)])


_module = None


def _binding():
    """Load ``_paged.so`` (must have been built)."""
    global _module
    if _module is None:
        _rt.load()
        if not os.path.exists(_build.BINDING_PATH):
            raise _rt.RetopkError(f"{_build.BINDING_PATH} is missing: build it with `python -m paper_2607_27692_b200.build`")
        again = "build it again with `python -m paper_2607_27692_b200.build`"
        try:
            module = importlib.import_module("._paged", __package__)
        except ImportError as e:
            raise _rt.RetopkError(f"{_build.BINDING_PATH} does not load ({e}): {again}") from e
        if module.built_for != _build.binding_target():
            raise _rt.RetopkError(f"{_build.BINDING_PATH} was built for {module.built_for}, this is {_build.binding_target()}: {again}")
        module.set_error(_rt.RetopkError)
        _module = module
    return _module


class _Rotation(torch.autograd.Function):
    """The rotation of one or two tensors; its backward pass is the transposed one."""

    @staticmethod
    def forward(ctx, rope, inverse, positions, *tensors):
        ctx.rope, ctx.inverse = rope, inverse
        ctx.save_for_backward(positions)
        out = rope._call(rope.h, rope.d, tensors[0], tensors[1] if len(tensors) > 1 else None, positions, None, None, inverse)
        return out[:len(tensors)]

    @staticmethod
    def backward(ctx, *grads):
        wanted = [i for i in range(len(grads)) if ctx.needs_input_grad[3 + i]]
        turned = ctx.rope._rotate([grads[i].contiguous() for i in wanted], ctx.saved_tensors[0], not ctx.inverse)
        out = [None] * len(grads)
        for i, g in zip(wanted, turned):
            out[i] = g
        return (None, None, None, *out)


class Rope:
    """Rotary positions of one model (wraps a ``retopk_rope*``; host memory only, any device).

    ``rot_dim`` channels of a head of ``d`` are rotated (default: all), paired in halves or, with
    ``interleaved``, as neighbours.  ``scaling``: None, "linear", "ntk", "llama3" or "yarn".
    """

    def __init__(self, d, rot_dim=None, base=10000.0, interleaved=False, scaling=None, factor=1.0, original_len=0,
                 low_freq_factor=0.0, high_freq_factor=0.0, beta_fast=0.0, beta_slow=0.0, attn_factor=0.0):
        self.h = 0
        if scaling not in _SCALINGS:
            raise ValueError(f"scaling: one of {list(_SCALINGS)}, got {scaling!r}")
        self.lib, self._call = _rt.load(), _binding().rope_apply
        self.d, self.rot_dim = d, d if rot_dim is None else rot_dim
        self._config = (d, rot_dim, base, interleaved, scaling, factor, original_len, low_freq_factor, high_freq_factor, beta_fast,
                        beta_slow, attn_factor)
        cfg = _RopeConfig(d, self.rot_dim, int(bool(interleaved)), _SCALINGS[scaling], base, factor, original_len,
                          low_freq_factor, high_freq_factor, beta_fast, beta_slow, attn_factor)
        h = _vp()
        _check(self.lib.retopk_rope_create(C.byref(h), C.byref(cfg)), "retopk_rope_create")
        self.h = h.value

    def close(self):
        if self.h:
            self.lib.retopk_rope_destroy(self.h)
            self.h = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __reduce__(self):
        """Copies (and pickles) are made from the settings: each has a handle of its own to destroy."""
        if not self.h:
            raise _rt.RetopkError("the rotation was closed")
        return type(self), self._config

    def frequencies(self):
        """Radians per position of each pair (list), and the factor on cosine and sine."""
        w, a = (C.c_double * (self.rot_dim // 2))(), C.c_double()
        _check(self.lib.retopk_rope_frequencies(self.h, w, C.byref(a)), "retopk_rope_frequencies")
        return list(w), float(a.value)

    def apply(self, x, positions, out=None, inverse=False):
        """Rotate x [tokens, heads, d] at int32 ``positions``; ``out`` may be x itself.

        Differentiable (twice, too), but not into a given ``out``: that is refused for tensors that
        require a gradient, unless under ``torch.no_grad()``.
        """
        r = self._call(self.h, self.d, x, None, positions, out, None, inverse)
        return self._rotate([x], positions, inverse)[0] if r is None else r[0]

    def apply_pair(self, q, k, positions, q_out=None, k_out=None, inverse=False):
        """Rotate queries and keys in one launch.  ``inverse``: the transpose, i.e. the gradient.

        Differentiable as ``apply`` is; the backward pass is one launch, too.
        """
        r = self._call(self.h, self.d, q, k, positions, q_out, k_out, inverse)
        return self._rotate([q, k], positions, inverse) if r is None else r

    def _rotate(self, tensors, positions, inverse):
        return _Rotation.apply(self, bool(inverse), positions, *tensors)


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
        self._fast = _binding()
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
        self._tensors = (k, v, k_scale, v_scale)
        self.fmt = "q4" if q4 else ("bf16" if k.dtype == torch.bfloat16 else "fp16")
        self.device = k.device
        self._cache = self._fast.cache_new(_FORMATS[self.fmt][0], self.H_kv, self.d, self.page_size, self.n_pages, k, v, k_scale, v_scale)

    def _part(i):
        def get(self):
            return self._tensors[i]

        def set(self, value):
            if value is not self._tensors[i]:       # cache.k *= 2 assigns the tensor that is there
                raise AttributeError("a cache keeps its tensors: write into them, or wrap others")

        return property(get, set)

    # The kernels use the memory that these tensors had when the cache was made; every call checks that it is
    # still theirs.
    k, v, k_scale, v_scale = _part(0), _part(1), _part(2), _part(3)
    del _part

    def append(self, k_new, v_new, seq_lens, block_table=None, cu_new=None, rope=None, q=None, q_out=None):
        """Store new keys and values [tokens, H_kv, d], rotated by ``rope`` on the way.

        ``seq_lens`` int32 [B] counts each sequence's keys including the new ones.  Sequence b's new
        tokens are rows cu_new[b]:cu_new[b+1] (int32 [B + 1]); without ``cu_new`` every sequence has
        the same number.  With ``q`` the queries are rotated in the same launch and returned.  Rows that
        belong to no token (of an idle sequence, or behind cu_new[B]) are not written: they stay as they
        were in ``q_out``, and without ``q_out`` they are uninitialised memory.
        """
        if rope is None:
            return self._fast.append(self._cache, k_new, v_new, seq_lens, block_table, cu_new, 0, q, q_out)
        if not rope.h:
            raise _rt.RetopkError("the rotation was closed")
        if rope.d != self.d:
            raise ValueError(f"the rotation is of heads of {rope.d}, the cache of {self.d}")
        return self._fast.append(self._cache, k_new, v_new, seq_lens, block_table, cu_new, rope.h, q, q_out)

    def gather(self, k_out, v_out, seq_lens, block_table=None, first=None):
        """Read rows back into k_out / v_out [B, H_kv, rows, d] (either may be None).

        Row i of sequence b is the cache's row first[b] + i, up to seq_lens[b]; others stay as they are.
        """
        self._fast.gather(self._cache, k_out, v_out, seq_lens, block_table, first)
        return k_out, v_out

    def attend(self, q, seq_lens, block_table=None, scale=None, window=0, out=None, lse=None):
        """Attention of the last T tokens of every sequence over a 4-bit cache.

        q [B, H_q, d] (one token) or [B, T, H_q, d]; the result has q's shape and type.  ``scale``
        defaults to d ** -0.5; ``window`` > 0 limits a token to its last ``window`` keys; ``lse``
        fp32, of q's shape without d, takes the logarithm of the sum of exponentials; ``out`` may be q
        where q is contiguous.  Rows without keys, and sequences whose length is negative or more than the
        block table holds, give 0 and -inf; NaN and infinities in what a token sees show in its row.
        """
        return self._fast.attend(self._cache, q, seq_lens, block_table, scale, window, out, lse)
