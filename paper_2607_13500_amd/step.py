"""What goes on around the attention of a step (tr_update_pages and tr_verify_drafts of
include/tr.h):

* update_pages   - page tables, row starts, slots and positions from the sequences'
                   lengths and what they gain or lose;
* verify_drafts  - how many drafted tokens the target's probabilities accept, and the
                   token drawn behind them, from given random numbers.

A decoding step with drafts is update_pages, the model (Attention.append and attend
in each layer), verify_drafts, and update_pages with its `change`, by which the rejected
drafts leave before the next step adds tokens.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from . import _lib
from ._lib import Pool
from .attention import _DTYPES, Step, _check, _empty, _raw_stream


class PagePool(NamedTuple):
    """Free pages of a cache: a ring int32 [pages] of page numbers, state[1] of them
    from index state[0] on.  A new cache's: arange(pages) and [0, pages]."""
    ring: torch.Tensor
    state: torch.Tensor            # int32 [2]


class PageUpdate(NamedTuple):
    step: Step                     # q_start, the new lengths, the table
    slots: torch.Tensor            # int64 [rows] page * page_size + row of each new token, -1 behind them
    pos: torch.Tensor              # int32 [rows] its place in its sequence (tokens before it), 0 behind them
    pool: PagePool                 # the ring and its new state
    short: torch.Tensor            # int32 [1]: 0, or the pages that are lacking (then nothing has changed)


class Verified(NamedTuple):
    tokens: torch.Tensor           # int32 [seqs, width]: accepted drafts, the drawn token, then -1
    accepted: torch.Tensor         # int32 [seqs] accepted drafts
    change: torch.Tensor           # int32 [seqs] accepted minus drafted: what the sequence's length changes by, for update_pages


# Small calls are bound by this module's own work (64 requests' tables: 11 us a call
# against 4 on the device), so a call's results share one allocation where they can,
# and each tensor is looked at once.
_I32, _I64, _F32 = torch.int32, torch.int64, torch.float32


def _vector(name, t, index, dtype, size):
    if not isinstance(t, torch.Tensor) or t.get_device() != index or t.dtype is not dtype or t.shape != (size,) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s [%d] tensor on cuda:%d" % (name, dtype, size, index))
    return t.data_ptr()


def _matrix(name, t, index, dtype, rows):
    """Address, row stride and columns of a tensor with rows contiguous."""
    if isinstance(t, torch.Tensor) and t.get_device() == index and t.dtype is dtype and t.dim() == 2:
        (n, columns), (row, unit) = t.shape, t.stride()
        if n == rows and (unit == 1 or columns <= 1):
            return t.data_ptr(), row, columns
    raise ValueError("%s must be a %s [%d, columns] tensor with rows contiguous on cuda:%d" % (name, dtype, rows, index))


def _run(call, name, index, stream, *args):
    handle = _raw_stream(index) if stream is None else stream.cuda_stream
    if index == torch.cuda.current_device():
        status = call(*args, handle)
    else:
        with torch.cuda.device(index):
            status = call(*args, handle)
    _check(status, name)


def update_pages(change: torch.Tensor, kv_len: torch.Tensor, table: torch.Tensor, pool: PagePool, page_size: int, rows: int, *,
                 in_place: bool = False, stream=None) -> PageUpdate:
    """The next step of sequences of kv_len tokens: sequence b gains change[b] new
    tokens, or loses its last -change[b] (all, if it has fewer).

    Each holds ceil(length / page_size) pages in its row of `table`, which is updated
    in place as the pool's ring is: pages are taken from the ring's front, and those of
    lost tokens go to its end, where the same call does not take them.  `rows` is the
    room for new tokens' slots and positions (packed as step.q_start says).  If the
    pool lacks pages, a sequence outgrows its row of the table or the new tokens the
    rows, nothing changes, no row belongs to any sequence, and `short` is the number of
    lacking pages, in the last two cases 2^31 - 1.

    A sequence gains or loses tokens in one call, not both: what Verified.change takes
    away goes in a call of its own (of no rows) before the one that adds the next tokens.
    The sum of the two in one call would add too few rows, at later places.

    `pos` is a token's position in a context of one axis whose tokens count as one each;
    append takes it as it is then.  Contexts of several axes take int32 [axes, rows], and
    text behind an image's kept tokens, which have their grid's positions, is a number
    of positions ahead of its places that the caller knows for each sequence.

    in_place: the new lengths and the pool's new state are written to kv_len and
    pool.state themselves, as a recorded graph that is replayed needs it.
    """
    if not isinstance(kv_len, torch.Tensor) or not kv_len.is_cuda or kv_len.dim() != 1:
        raise ValueError("kv_len must be an int32 [seqs] tensor on a ROCm device")
    index, seqs, rows = kv_len.get_device(), kv_len.shape[0], int(rows)
    at_kv = _vector("kv_len", kv_len, index, _I32, seqs)
    at_change = _vector("change", change, index, _I32, seqs)
    at_table, row, width = _matrix("table", table, index, _I32, seqs)
    ring, state = pool
    if not isinstance(ring, torch.Tensor) or ring.dim() != 1:
        raise ValueError("pool.ring must be an int32 [pages] tensor on cuda:%d" % index)
    pages = ring.shape[0]
    at_ring, at_state = _vector("pool.ring", ring, index, _I32, pages), _vector("pool.state", state, index, _I32, 2)
    page_size = int(page_size)
    if rows < 0 or not 0 < page_size < 1 << 31:
        raise ValueError("rows must be >= 0 (got %d) and page_size in [1, 2^31 - 1] (got %d)" % (rows, page_size))
    sizes = [seqs + 1, rows, 1] if in_place else [seqs + 1, rows, 1, seqs, 2]
    parts = _empty((sum(sizes),), _I32, kv_len.device, stream).unsafe_split_with_sizes(sizes)
    q_start, pos, short = parts[:3]
    kv_out, state_out = (kv_len, state) if in_place else parts[3:]
    slots = _empty((rows,), _I64, kv_len.device, stream)
    p = Pool(pages, at_ring, at_state, state_out.data_ptr())
    _run(_lib.load().tr_update_pages, "tr_update_pages", index, stream, seqs, at_change, at_kv, kv_out.data_ptr(), at_table, width, row,
         page_size, ctypes.byref(p), q_start.data_ptr(), rows, slots.data_ptr(), pos.data_ptr(), short.data_ptr())
    return PageUpdate(Step(q_start, kv_out, table), slots, pos, PagePool(ring, state_out), short)


def verify_drafts(target: torch.Tensor, ids: torch.Tensor, q_start: torch.Tensor, accept: torch.Tensor, draw: torch.Tensor,
                  width: int, *, draft: Optional[torch.Tensor] = None, stream=None) -> Verified:
    """Drafted tokens against the target's probabilities.

    Rows are packed as in a Step: sequence b's rows q_start[b] .. q_start[b + 1] - 1 are
    its last accepted token and its drafts, ids int32 [tokens].  Row i of target
    (float32 or bfloat16 [tokens, vocab]) is the distribution of the token behind it,
    that of draft the one from which ids[i + 1] was drawn (None: drafts were certain).

    A draft x of row i is accepted while accept[i] * draft[i, x] < target[i, x].
    Behind the accepted ones a token is drawn with draw[b]: from max(target - draft, 0)
    of the first rejected draft's row, from the last row's target where all were
    accepted; it is the lowest token at which the weights' sum exceeds draw[b] times
    the whole.  At most width - 1 drafts of a sequence are looked at.  accept (float32
    [tokens]) and draw (float32 [seqs]) lie in [0, 1).  Exact in 64 bits for the given
    numbers: the same ones give the same tokens.
    """
    if not isinstance(target, torch.Tensor) or not target.is_cuda or target.dim() != 2 or target.dtype not in _DTYPES:
        raise ValueError("target must be a float32 or bfloat16 [tokens, vocab] tensor on a ROCm device")
    index, dtype, (tokens, vocab), width = target.get_device(), target.dtype, target.shape, int(width)
    if not isinstance(q_start, torch.Tensor) or q_start.dim() != 1 or q_start.shape[0] < 1:
        raise ValueError("q_start must be an int32 [seqs + 1] tensor on cuda:%d" % index)
    seqs = q_start.shape[0] - 1
    if not 0 < width < 1 << 31:
        raise ValueError("width must be in [1, 2^31 - 1] (got %d)" % width)
    p, ld, _ = _matrix("target", target, index, dtype, tokens)
    q, ld_draft = None, 0
    if draft is not None:
        q, ld_draft, columns = _matrix("draft", draft, index, dtype, tokens)
        if columns != vocab:
            raise ValueError("draft must have target's %d columns (got %d)" % (vocab, columns))
    lib = _lib.load()
    said, accepted, change = _empty((seqs * (width + 2),), _I32, target.device, stream).unsafe_split_with_sizes([seqs * width, seqs, seqs])
    scratch = _empty((lib.tr_verify_scratch(seqs),), torch.uint8, target.device, stream)    # 4 KB a sequence, not kept with the results
    _run(lib.tr_verify_drafts, "tr_verify_drafts", index, stream, tokens, vocab, _DTYPES[dtype], p, ld, q, ld_draft,
         _vector("ids", ids, index, _I32, tokens), seqs, _vector("q_start", q_start, index, _I32, seqs + 1),
         _vector("accept", accept, index, _F32, tokens), _vector("draw", draw, index, _F32, seqs), width,
         said.data_ptr(), accepted.data_ptr(), change.data_ptr(), scratch.data_ptr())
    return Verified(said.view(seqs, width), accepted, change)
