"""Rotary positions, paged key/value caches that sequences share, and attention over them (binding).

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

    # sequences that continue one prompt: pages are shared, and so is the work on them
    pool = PagePool(n_pages, 64)
    pool.reserve(block_table, old_lens, seq_lens)
    cache.copy_pages(*pool.fork(block_table, seq_lens, parents, children))
    out = cache.attend_shared(q, seq_lens, block_table, cu_groups, prompt_lens)

    # attention over the blocks of keys that can score highest
    index = BlockIndex(cache, 64)
    index.update(seq_lens, block_table)
    blocks = index.select(q, seq_lens, block_table, keep=64)
    out = index.attend(q, seq_lens, blocks, block_table)

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

    def attend_shared(self, q, seq_lens, block_table=None, cu_groups=None, shared_lens=None, scale=None, out=None, lse=None):
        """Attention of the last T tokens of every sequence over 16-bit pages, shared prefixes read once.

        q, ``out``, ``lse`` and the result as in ``attend``; q has the cache's type.  Sequences
        cu_groups[g]:cu_groups[g+1] (int32 [groups + 1], from 0 to B) share their first shared_lens[g] rows
        (int32 [groups]): the same pages, as ``PagePool.fork`` leaves them, or equal rows.  The result is that
        of each sequence alone, which is also what is computed without ``cu_groups``.
        """
        return self._fast.attend_shared(self._cache, q, seq_lens, block_table, cu_groups, shared_lens, scale, out, lse)

    def copy_pages(self, src, dst, rows=None):
        """Copy pages src[i] to dst[i] (int32 [n]), with ``rows`` the first rows[i] rows of each.

        Pairs with a negative number are left out.  A page that is written twice, or written and read, is
        unspecified afterwards.
        """
        self._fast.copy_pages(self._cache, src, dst, rows)


class PagePool:
    """Which pages of a cache (of all layers over one block table) are in use.

    ``refs`` int32 [n_pages] counts the entries of block tables that hold a page; new pages are the free ones
    with the lowest numbers.  A sequence of n rows holds the first ceil(n / page_size) entries of its row of
    ``block_table``.  Everything is on the device and nothing is waited for: pages that were missing are
    counted in ``missing`` (int32 [1], to read or clear).  One call at a time may change a pool and its tables.
    """

    def __init__(self, n_pages, page_size, device="cuda"):
        self._set(torch.zeros(n_pages, dtype=torch.int32, device=device), page_size)

    @classmethod
    def wrap(cls, refs, page_size):
        """Use existing counts (int32 [n_pages])."""
        self = cls.__new__(cls)
        self._set(refs, page_size)
        return self

    def _set(self, refs, page_size):
        self._fast = _binding()
        if refs.dim() != 1 or refs.numel() < 1 or refs.dtype != torch.int32 or not refs.is_cuda or not refs.is_contiguous():
            raise TypeError(f"refs: expected a contiguous int32 CUDA tensor [n_pages], got {refs.dtype} {tuple(refs.shape)} on {refs.device}")
        if page_size < 1:
            raise ValueError(f"page_size: at least 1, got {page_size}")
        self.refs, self.page_size, self.n_pages = refs, int(page_size), refs.numel()
        self._scratch = torch.zeros(self.n_pages + 4, dtype=torch.int32, device=refs.device)      # RETOPK_POOL_SCRATCH

    @property
    def missing(self):
        return self._scratch[:1]

    def reserve(self, block_table, old_lens, new_lens):
        """Enter the pages that sequences lack to grow from ``old_lens`` to ``new_lens`` rows (int32 [B]).

        Those that shrink (draft tokens that were not accepted) give back the pages behind their new length first.  In the
        order of the sequences; one that finds too few pages, or no room in its row, gets -1 in its new entries, and so do
        those behind one that finds too few.  A sequence that shrinks to a length inside a page that others hold too is not
        to be appended to there; a fork of it has a page of its own.
        """
        self._fast.pool_reserve(self.refs, self._scratch, self.page_size, block_table, old_lens, new_lens)

    def fork(self, block_table, seq_lens, parents, children):
        """Let the empty rows ``children`` (int32 [n]) continue the sequences ``parents``.

        Full pages are shared, a partial last one gets a page of its own; ``seq_lens`` of the children are set.
        Returns (src, dst, rows), what ``copy_pages`` has to copy in each layer.  A fork that cannot be made (a child
        that is not empty, is named twice or is a parent too, an empty parent, no free page) is left out.
        """
        return self._fast.pool_fork(self.refs, self._scratch, self.page_size, block_table, seq_lens, parents, children)

    def free(self, block_table, seq_lens, rows=None):
        """Give back the pages of sequences ``rows`` (int32 [n], default all) and set their lengths to 0."""
        self._fast.pool_free(self.refs, self._scratch, self.page_size, block_table, seq_lens, rows)

    def compact(self, block_table, seq_lens):
        """Renumber the pages so that those in use come first; ``block_table`` follows.

        Returns (src, dst), the moves that ``copy_pages`` has to make in each layer, -1 behind the last.  All
        entries that hold pages have to be in ``block_table``.
        """
        return self._fast.pool_compact(self.refs, self._scratch, self.page_size, block_table, seq_lens)


class BlockIndex:
    """Bounds of blocks of ``block`` keys (16, 32, 64 or 128) of a 16-bit cache, and attention over selected blocks.

    ``bounds`` [n_pages, H_kv, page_size / block, 2, d], of the cache's type: least and largest key of each
    block, channel by channel.
    """

    def __init__(self, cache, block):
        if block not in (16, 32, 64, 128) or cache.page_size % block:
            raise ValueError(f"block: 16, 32, 64 or 128 and a divisor of page_size {cache.page_size}, got {block}")
        shape = (cache.n_pages, cache.H_kv, cache.page_size // block, 2, cache.d)
        self._set(cache, torch.zeros(shape, dtype=cache.k.dtype, device=cache.device))

    @classmethod
    def wrap(cls, cache, bounds):
        """Use an existing tensor of bounds."""
        self = cls.__new__(cls)
        self._set(cache, bounds)
        return self

    def _set(self, cache, bounds):
        if cache.fmt == "q4":
            raise TypeError("a block index reads 16-bit pages, this cache holds 4-bit values")
        if bounds.dim() != 5 or bounds.shape[2] < 1 or cache.page_size % bounds.shape[2]:
            raise ValueError(f"bounds: expected [n_pages, H_kv, page_size / block, 2, d], got {tuple(bounds.shape)}")
        self.cache, self.bounds, self.block = cache, bounds, cache.page_size // bounds.shape[2]
        if self.block not in (16, 32, 64, 128):
            raise ValueError(f"bounds: blocks of 16, 32, 64 or 128 keys, got {self.block}")
        self._fast = _binding()

    def update(self, seq_lens, block_table=None, n_new=None):
        """Work out the bounds of the full blocks that overlap the last ``n_new`` rows (default: of all)."""
        self._fast.block_update(self.cache._cache, self.bounds, self.block, seq_lens, block_table, (1 << 62) if n_new is None else n_new)

    def select(self, q, seq_lens, block_table=None, keep=64, first=1, last=2, out=None):
        """Blocks for each token and KV head, int32 [B, H_kv, keep] or [B, T, H_kv, keep], ascending, -1 behind the last.

        The ``first`` and ``last`` blocks of a sequence are always among them; the others are those with the
        largest upper bound of a query's products with the block's keys (any head of the group), ties to
        the lower number.  For a ``scale`` above 0.
        """
        return self._fast.block_select(self.cache._cache, self.bounds, self.block, q, seq_lens, block_table, keep, first, last, out)

    def attend(self, q, seq_lens, blocks, block_table=None, scale=None, out=None, lse=None):
        """Attention over the keys of ``blocks``, as ``select`` returns them; the rest as ``KVPages.attend_shared``.

        Entries that are no block of the sequence do not count, a block that is named twice counts twice.
        """
        return self._fast.block_attend(self.cache._cache, self.block, q, seq_lens, blocks, block_table, scale, out, lse)

    def copy_pages(self, src, dst):
        """The bounds follow ``KVPages.copy_pages``."""
        self._fast.block_copy(self.cache._cache, self.bounds, self.block, src, dst)
