"""The language model's side of the library: what happens to the kept tokens
between the reduction and the model's answer (the tr_attn calls of include/tr.h).

* kept_positions          - (time, height, width) of kept tokens in their image;
* Attention.rotate        - norm of each head and rotation by position, one pass,
                            with a graph where its inputs have one;
* Attention.rotate_backward - its gradients, for calls without autograd;
* Attention.append        - the same on the way of new keys into a paged cache;
* Attention.attend        - attention of the new tokens over that cache.

As elsewhere in the package this module only marshals torch tensors and the
stream into the C ABI.
"""
from __future__ import annotations

import ctypes
import math
from array import array
from itertools import chain
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from . import _lib
from ._lib import AttnParams, Cache, Heads, StepArgs

# Small calls are bound by this module's own work (one decoded token: 9 us a call
# against 12.5 us on the device), so each tensor is looked at once, devices are
# compared as indices, and streams are asked for as plain handles.

_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") \
    else lambda index: torch.cuda.current_stream(index).cuda_stream
_DTYPES = {torch.float32: _lib.TR_FP32, torch.bfloat16: _lib.TR_BF16}
_NONE = Heads(None, 0, 0)


def _check(status: int, where: str):
    if status:
        from . import TRError
        raise TRError(status, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _empty(shape, dtype, device, stream):
    """A new tensor from the memory of the stream that will write it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class KVCache(NamedTuple):
    """A paged cache: k and v [pages, page_size, kv_heads, head_dim], of any (the
    same) strides with the elements of a head side by side."""
    k: torch.Tensor
    v: torch.Tensor


class Step(NamedTuple):
    """The sequences of one call: sequence b's new tokens are the packed rows
    q_start[b] .. q_start[b + 1] - 1 and the last of its kv_len[b] tokens; token
    j of it lies in page table[b, j // page_size].  All int32 on the device."""
    q_start: torch.Tensor          # [seqs + 1]
    kv_len: torch.Tensor           # [seqs]
    table: torch.Tensor            # [seqs, width]


def kept_positions(idx: torch.Tensor, K: Sequence[int], grid: Sequence[Tuple[int, int, int]],
                   start: Sequence[Tuple[int, int, int]], *, dst: Optional[Sequence[int]] = None,
                   out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Positions of kept tokens, int32 [3, columns]: start[b] + (t, h, w) for the
    K[b] kept tokens of image b (idx: their image-local indices, as
    ReduceResult.idx) in its grid of (frames, rows, columns) tokens.

    The images' columns are packed, or begin at dst[b] of `out`, whose other
    columns (a prompt's text) stay as they are.
    """
    lib = _lib.load()
    B = len(K)
    counts = array("i", K)
    kept = sum(counts)
    if not isinstance(idx, torch.Tensor) or not idx.is_cuda or idx.dtype is not torch.int32 or idx.dim() != 1 \
            or not idx.is_contiguous() or idx.numel() != kept:
        raise ValueError("idx must be a contiguous int32 [sum K] tensor on a ROCm device")
    if len(grid) != B or len(start) != B or (dst is not None and len(dst) != B):
        raise ValueError("grid, start and dst must have one entry for each image")
    if B and (set(map(len, grid)) != {3} or set(map(len, start)) != {3}):
        raise ValueError("entries of grid and start must be (time, height, width)")
    if out is None:
        if dst is not None:
            raise ValueError("dst needs out")
        out = _empty((3, kept), torch.int32, idx.device, stream)
    elif out.device != idx.device or out.dtype is not torch.int32 or out.dim() != 2 or out.shape[0] != 3 \
            or (out.shape[1] > 1 and out.stride(1) != 1):
        raise ValueError("out must be an int32 [3, columns] tensor with unit column stride on %s" % idx.device)
    elif out.shape[1] and out.stride(0) < out.shape[1]:
        raise ValueError("out has rows that overlap")
    columns = out.shape[1]
    to = None if dst is None else array("q", dst)
    if to is None:
        if kept > columns:
            raise ValueError("the images' columns do not fit out")
    elif any(d < 0 or d + k > columns for d, k in zip(to, counts)):
        raise ValueError("the images' columns do not fit out")
    shape, first = array("i", chain.from_iterable(grid)), array("i", chain.from_iterable(start))
    args = (idx.data_ptr(), B, counts.buffer_info()[0], shape.buffer_info()[0], first.buffer_info()[0],
            None if to is None else to.buffer_info()[0], out.data_ptr(), out.stride(0) if columns else 0)
    index = idx.get_device()
    handle = _raw_stream(index) if stream is None else stream.cuda_stream
    if index == torch.cuda.current_device():
        status = lib.tr_kept_positions(*args, handle)
    else:
        with torch.cuda.device(index):
            status = lib.tr_kept_positions(*args, handle)
    _check(status, "tr_kept_positions")
    return out


class _Rotated(torch.autograd.Function):
    """Attention.rotate with a graph."""

    @staticmethod
    def forward(ctx, attention, q, k, pos, wq, wk):
        ctx.attention, norm = attention, attention.norm
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(q if norm else None, k if norm else None, pos, wq, wk)
        return attention._rotate(q, k, pos, wq, wk, None, None, None)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *g):
        q, k, pos, wq, wk = ctx.saved_tensors
        _, need_q, need_k, _, need_wq, need_wk = ctx.needs_input_grad
        # an expanded gradient (of a sum) has no unit stride
        gq, gk = (x if x is None or x.stride(-1) == 1 else x.contiguous() for x in g)
        gq, gk = gq if need_q or need_wq else None, gk if need_k or need_wk else None
        if gq is None and gk is None:
            return (None,) * 6
        dq, dk, dwq, dwk = ctx.attention.rotate_backward(gq, gk, q, k, pos, wq=wq, wk=wk)
        dwq, dwk = (d.to(w.dtype) if need and d is not None else None for d, w, need in ((dwq, wq, need_wq), (dwk, wk, need_wk)))
        return None, dq if need_q else None, dk if need_k else None, None, dwq, dwk


class Attention:
    """An attention layer's geometry on one device.

    The first rot_dim elements of a head (all by default) turn in pairs: pair i
    by pos[axis] * inv_freq[i], inv_freq[i] = base ** (-2 i / rot_dim) unless
    given.  `sections` gives each axis (row of pos) its number of consecutive
    pairs; `pair_axis` names each pair's axis instead; without either there is
    one axis.  adjacent pairs are elements (2 i, 2 i + 1), otherwise
    (i, i + rot_dim / 2).  norm: heads are divided by their root mean square
    (eps added to its square) and multiplied by a weight before they rotate.

    Layers of one geometry can share an Attention: it holds no weights, only the
    scratch of rotate_backward and attend (up to 68 MB).  That scratch is for one
    stream (and one thread) at a time: a call on another stream has to wait for
    those before it, by an event or wait_stream.
    """

    def __init__(self, heads: int, kv_heads: Optional[int] = None, head_dim: int = 128,
                 dtype: torch.dtype = torch.bfloat16, *, rot_dim: Optional[int] = None, base: float = 10000.0,
                 inv_freq: Optional[Sequence[float]] = None, sections: Optional[Sequence[int]] = None,
                 pair_axis: Optional[Sequence[int]] = None, adjacent: bool = False, norm: bool = False,
                 eps: float = 1e-6, device=None):
        if dtype not in _DTYPES:
            raise TypeError("dtype must be torch.float32 or torch.bfloat16")
        self.heads, self.kv_heads = int(heads), int(heads if kv_heads is None else kv_heads)
        self.head_dim, self.dtype, self.norm = int(head_dim), dtype, bool(norm)
        self.rot_dim = self.head_dim if rot_dim is None else int(rot_dim)
        pairs = self.rot_dim // 2
        if sections is not None and pair_axis is not None:
            raise ValueError("give sections or pair_axis, not both")
        if sections is not None:
            if any(int(s) < 0 for s in sections) or sum(map(int, sections)) != pairs:
                raise ValueError("sections must be >= 0 and add up to rot_dim / 2 = %d" % pairs)
            pair_axis = [a for a, n in enumerate(sections) for _ in range(int(n))]
            self.axes = len(sections)
        else:
            if pair_axis is not None and len(pair_axis) != pairs:
                raise ValueError("pair_axis must have rot_dim / 2 = %d entries" % pairs)
            self.axes = 1 + max(map(int, pair_axis)) if pair_axis else 1
        if inv_freq is not None and len(inv_freq) != pairs:
            raise ValueError("inv_freq must have rot_dim / 2 = %d entries" % pairs)
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2607_13500_amd needs a ROCm GPU (gfx950)")
        self.device = torch.device("cuda", torch.cuda.current_device() if device is None
                                   else torch.device(device).index or 0)
        self._index = self.device.index
        self.lib = _lib.load()
        freq = None if inv_freq is None else (ctypes.c_double * max(pairs, 1))(*map(float, inv_freq))
        axis = None if pair_axis is None else (ctypes.c_int32 * max(pairs, 1))(*map(int, pair_axis))
        p = AttnParams(heads=self.heads, kv_heads=self.kv_heads, head_dim=self.head_dim, rot_dim=self.rot_dim,
                       axes=self.axes, adjacent=int(bool(adjacent)), dtype=_DTYPES[dtype], norm=int(self.norm),
                       eps=float(eps), base=float(base), inv_freq=ctypes.cast(freq, ctypes.c_void_p) if freq else None,
                       pair_axis=ctypes.cast(axis, ctypes.c_void_p) if axis else None)
        ctx = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(self.lib.tr_attn_create(ctypes.byref(p), ctypes.byref(ctx)), "tr_attn_create")
        self._ctx = ctx

    # -- helpers ----------------------------------------------------------
    def _stream(self, stream):
        return _raw_stream(self._index) if stream is None else stream.cuda_stream

    def _heads(self, name, t, heads, tokens) -> Heads:
        if not isinstance(t, torch.Tensor) or t.get_device() != self._index:
            raise ValueError("%s must be a tensor on %s" % (name, self.device))
        if t.dtype is not self.dtype:
            raise TypeError("%s must be %s, got %s" % (name, self.dtype, t.dtype))
        if t.shape == (tokens, heads, self.head_dim):
            token, head, unit = t.stride()
            if unit == 1 or self.head_dim == 1:
                return Heads(t.data_ptr(), token, head)
        raise ValueError("%s must be a [%s, %d, %d] tensor with unit element stride, got %s of strides %s"
                         % (name, tokens, heads, self.head_dim, tuple(t.shape), t.stride()))

    def _out(self, name, t, tokens, heads, stream):
        if t is None:
            dim = self.head_dim
            t = _empty((tokens, heads, dim), self.dtype, self.device, stream)
            return t, Heads(t.data_ptr(), heads * dim, dim)
        return t, self._heads(name, t, heads, tokens)

    def _pos(self, pos, tokens):
        if not isinstance(pos, torch.Tensor) or pos.get_device() != self._index or pos.dtype is not torch.int32:
            raise ValueError("pos must be an int32 tensor on %s" % self.device)
        if pos.dim() == 1 and self.axes == 1:
            pos = pos[None]
        if pos.shape == (self.axes, tokens):
            row, unit = pos.stride()
            if unit == 1 or tokens <= 1:
                return pos.data_ptr(), row
        raise ValueError("pos must be [%d, %d] with unit column stride, got %s" % (self.axes, tokens, tuple(pos.shape)))

    def _weight(self, name, w):
        if w is None:
            return None
        if not isinstance(w, torch.Tensor) or w.get_device() != self._index or w.dtype is not self.dtype \
                or w.shape != (self.head_dim,) or not w.is_contiguous():
            raise ValueError("%s must be a contiguous %s [%d] tensor on %s" % (name, self.dtype, self.head_dim, self.device))
        return w.data_ptr()

    def _cache(self, cache: KVCache) -> Cache:
        k, v = cache
        for name, t in (("cache.k", k), ("cache.v", v)):
            if not isinstance(t, torch.Tensor) or t.get_device() != self._index or t.dtype is not self.dtype:
                raise ValueError("%s must be a %s tensor on %s" % (name, self.dtype, self.device))
        shape, stride = k.shape, k.stride()
        if len(shape) != 4 or shape[2] != self.kv_heads or shape[3] != self.head_dim or (self.head_dim > 1 and stride[3] != 1):
            raise ValueError("cache.k must be [pages, page_size, %d, %d] with unit element stride, got %s of strides %s"
                             % (self.kv_heads, self.head_dim, tuple(shape), stride))
        if shape != v.shape or stride != v.stride():
            raise ValueError("cache.k and cache.v must have the same shape and strides")
        return Cache(k.data_ptr(), v.data_ptr(), shape[0], shape[1], stride[0], stride[1], stride[2])

    def _step(self, step: Step) -> StepArgs:
        for name, t in zip(Step._fields, step):
            if not isinstance(t, torch.Tensor) or t.get_device() != self._index or t.dtype is not torch.int32:
                raise ValueError("step.%s must be an int32 tensor on %s" % (name, self.device))
        q_start, kv_len, table = step
        if kv_len.dim() == 1 and table.dim() == 2:
            seqs, (rows, width), (row, unit) = kv_len.shape[0], table.shape, table.stride()
            if q_start.shape == (seqs + 1,) and rows == seqs and (unit == 1 or width <= 1) and q_start.is_contiguous() \
                    and kv_len.is_contiguous():
                return StepArgs(seqs, width, row, q_start.data_ptr(), kv_len.data_ptr(), table.data_ptr())
        raise ValueError("step must hold q_start [seqs + 1], kv_len [seqs] and table [seqs, width], rows contiguous")

    # -- the operators ------------------------------------------------------
    def rotate(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor], pos: torch.Tensor, *,
               wq: Optional[torch.Tensor] = None, wk: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream=None):
        """(q_out, k_out): heads q [tokens, heads, head_dim] and k [tokens,
        kv_heads, head_dim] normed (with norm) and rotated to pos [axes, tokens]
        (rows may coincide: text.expand(axes, -1)).  Either may be None; the
        outputs may be the inputs themselves.  Where autograd records and q, k or
        a weight requires a gradient, the outputs are the call's own and have one."""
        if torch.is_grad_enabled():
            for t in (q, k, wq, wk):
                if t is not None and t.requires_grad:
                    if q_out is not None or k_out is not None:
                        raise RuntimeError("q_out and k_out take no gradient: leave them out, or call rotate without recording")
                    with torch.cuda.stream(stream):      # the gradient's stream too
                        return _Rotated.apply(self, q, k, pos, wq, wk)
        return self._rotate(q, k, pos, wq, wk, q_out, k_out, stream)

    def _rotate(self, q, k, pos, wq, wk, q_out, k_out, stream):
        if q is None and k is None:
            raise ValueError("nothing to rotate")
        tokens = (q if q is not None else k).shape[0]
        hq = hk = oq = ok = _NONE
        if q is not None:
            hq = self._heads("q", q, self.heads, tokens)
            q_out, oq = self._out("q_out", q_out, tokens, self.heads, stream)
        if k is not None:
            hk = self._heads("k", k, self.kv_heads, tokens)
            k_out, ok = self._out("k_out", k_out, tokens, self.kv_heads, stream)
        at, ldpos = self._pos(pos, tokens)
        _check(self.lib.tr_rotate(self._ctx, tokens, hq, hk, self._weight("wq", wq), self._weight("wk", wk), at, ldpos,
                                  oq, ok, self._stream(stream)), "tr_rotate")
        return (q_out if q is not None else None), (k_out if k is not None else None)

    def rotate_backward(self, gq: Optional[torch.Tensor], gk: Optional[torch.Tensor], q: Optional[torch.Tensor],
                        k: Optional[torch.Tensor], pos: torch.Tensor, *, wq: Optional[torch.Tensor] = None,
                        wk: Optional[torch.Tensor] = None, dq: Optional[torch.Tensor] = None,
                        dk: Optional[torch.Tensor] = None, stream=None):
        """(dq, dk, dwq, dwk): the gradients of rotate's inputs from those of its
        outputs (gq, gk; either may be None).  q and k are rotate's inputs (not
        read without norm).  dwq and dwk are float32 [head_dim], with norm only;
        a weight that was None has the gradient of a weight of ones."""
        if gq is None and gk is None:
            raise ValueError("nothing to compute")
        tokens = (gq if gq is not None else gk).shape[0]
        g, x, d, dw = [_NONE, _NONE], [_NONE, _NONE], [_NONE, _NONE], [None, None]
        outs = [dq, dk]
        for i, (grad, inp, heads) in enumerate(((gq, q, self.heads), (gk, k, self.kv_heads))):
            if grad is None:
                outs[i] = None
                continue
            name = "qk"[i]
            g[i] = self._heads("g" + name, grad, heads, tokens)
            if self.norm:
                x[i] = self._heads(name, inp, heads, tokens)
                dw[i] = _empty((self.head_dim,), torch.float32, self.device, stream)
            outs[i], d[i] = self._out("d" + name, outs[i], tokens, heads, stream)
        at, ldpos = self._pos(pos, tokens)
        _check(self.lib.tr_rotate_backward(self._ctx, tokens, g[0], g[1], x[0], x[1], self._weight("wq", wq),
                                           self._weight("wk", wk), at, ldpos, d[0], d[1], _ptr(dw[0]), _ptr(dw[1]),
                                           self._stream(stream)), "tr_rotate_backward")
        return outs[0], outs[1], dw[0], dw[1]

    def append(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, pos: torch.Tensor, cache: KVCache,
               step: Step, *, wq: Optional[torch.Tensor] = None, wk: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
        """rotate for the new tokens of a step: their keys go to their place in
        the cache, their values (as they are) beside them; returns q_out (None
        where q is).  Slices of one projection's output are fine.  Passes no
        gradient."""
        tokens = k.shape[0]
        hk, hv = self._heads("k", k, self.kv_heads, tokens), self._heads("v", v, self.kv_heads, tokens)
        hq = oq = _NONE
        if q is not None:
            hq = self._heads("q", q, self.heads, tokens)
            q_out, oq = self._out("q_out", q_out, tokens, self.heads, stream)
        at, ldpos = self._pos(pos, tokens)
        status = self.lib.tr_append(self._ctx, tokens, hq, hk, hv, self._weight("wq", wq), self._weight("wk", wk), at,
                                    ldpos, oq, self._cache(cache), self._step(step), self._stream(stream))
        _check(status, "tr_append")
        return q_out if q is not None else None

    def attend(self, q: torch.Tensor, cache: KVCache, step: Step, *, scale: Optional[float] = None,
               causal: bool = True, window: int = 0, out: Optional[torch.Tensor] = None, want_lse: bool = False,
               stream=None):
        """(out, lse): attention of the new tokens' queries q [tokens, heads,
        head_dim] over their sequences' tokens in the cache (bf16).

        causal: a token sees itself and those before it, with window > 0 the last
        `window` of them; otherwise all kv_len tokens of its sequence.  A row
        that sees none is 0 with lse = -inf.  scale is 1 / sqrt(head_dim) unless
        given.  lse (float32 [tokens, heads], natural logarithm) is None unless
        wanted.  Passes no gradient.
        """
        tokens = q.shape[0]
        hq = self._heads("q", q, self.heads, tokens)
        out, ho = self._out("out", out, tokens, self.heads, stream)
        lse = _empty((tokens, self.heads), torch.float32, self.device, stream) if want_lse else None
        status = self.lib.tr_attend(self._ctx, tokens, hq, self._cache(cache), self._step(step),
                                    1.0 / math.sqrt(self.head_dim) if scale is None else float(scale), 1 if causal else 0,
                                    int(window), ho, _ptr(lse), self._stream(stream))
        _check(status, "tr_attend")
        return out, lse

    def close(self):
        if getattr(self, "_ctx", None):
            self.lib.tr_attn_destroy(self._ctx)
            self._ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
