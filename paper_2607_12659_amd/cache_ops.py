"""Operators of a paged 8-bit KV cache on torch tensors (include/jpi_cache.h).

As in ``prefix_ops``, PyTorch provides device memory and streams only: every
function checks its tensors, fills in the C arguments and enqueues libjpi's
kernels on the current stream of the tensors' device, which may be capturing a
graph.  Outputs and workspaces are allocated by torch on that stream unless they
are given.  Queries, keys, values and outputs are bfloat16 or float32, codes int8
or float8_e4m3fn, scales float32, lengths, tables and counts int32.  No gradients
are recorded: tensors that require them are refused while torch records them.
Tensors that a call writes into count as changed in place.  Errors are raised as
``jpi.JpiError`` (the library's checks), ``ValueError`` or ``TypeError`` (shapes,
devices and types).

Sequence s holds slots 0 .. lens[s] - 1, slot j in the page that table[s][j //
page] names; refs counts the sequences that hold each page, and a page that none
holds is free.  Where pages are lacking, sequences keep the length that they had,
and their last page may still be another's too: what resize gave is the growth of
lens, and that is what a step may write.  A step of a program that samples texts::

    starts = lens.clone()
    resize(table, lens, refs, lens + n, pool)         # room, in all layers
    n_new = lens - starts                             # 0 for who was not served: nothing of it is written or attends
    for each layer:
        q, k = norm_rope(q, k, positions, q_weight=..., k_weight=...)
        append(pool.layer(i), table, starts, k, v, n_new=n_new)
        out, lse = attention(q, pool.layer(i), table, lens, q_lens=n_new)
    reorder(table, lens, refs, parents, page)         # fork, free, reorder
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple

import torch

from . import jpi as _j
from .prefix_ops import (_DTYPE, _F32, _I32, _INT_MAX, _LAST_ERROR, _V, _VIEW, _dense, _dtype, _launch, _lib, _no_gradients, _pack,
                         _recording, _turned, _view, _want, _written)

_CODE = {torch.int8: _j.JPI_INT8, torch.float8_e4m3fn: _j.JPI_E4M3}
_LAST_ERROR.update(dict.fromkeys(("jpi_norm_rope", "jpi_cache_append", "jpi_cache_attention", "jpi_cache_resize", "jpi_cache_reorder",
                                  "jpi_cache_compact"), _j.jpi_cache_last_error))

_NORM = struct.Struct("@PP2iqd")
_POOL = struct.Struct("@5iPPPP")
_SEQS = struct.Struct("@2iqPP")
_ATTN = struct.Struct("@6if" + _V + "P" + _V + "P")
_MOVES = struct.Struct("@2iqPPPPqPP2i")
assert (_NORM.size, _POOL.size, _SEQS.size, _ATTN.size, _MOVES.size) == tuple(
    ctypes.sizeof(c) for c in (_j.jpi_head_norm, _j.jpi_cache_pool, _j.jpi_cache_seqs, _j.jpi_cache_attn, _j.jpi_cache_moves))


class Pool(NamedTuple):
    """The pages of one layer, or of several in a leading dimension: codes k [pages][kv_heads][head_dim / 16][page][16] and
    v [pages][kv_heads][page / 16][head_dim][16], scales [pages][kv_heads]; all contiguous."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    @classmethod
    def zeros(cls, n_pages, kv_heads, head_dim, page, *, code=torch.float8_e4m3fn, layers=None, device="cuda"):
        """A new pool; without `layers` of one layer."""
        if code not in _CODE:
            raise TypeError("codes must be int8 or float8_e4m3fn, got %s" % code)
        if head_dim % 16 or page % 16:
            raise ValueError("head_dim and page must be multiples of 16")
        lead = (n_pages, kv_heads) if layers is None else (layers, n_pages, kv_heads)
        shapes = ((head_dim // 16, page, 16), (page // 16, head_dim, 16))
        return cls(*(torch.zeros(lead + s, dtype=torch.uint8, device=device).view(code) for s in shapes),
                   *(torch.zeros(lead, dtype=_F32, device=device) for _ in shapes))

    def layer(self, i):
        return Pool(self.k[i], self.v[i], self.k_scale[i], self.v_scale[i])


# The checks below first ask in one expression whether all is well, and look for what is wrong only if not: a call's host time
# is mostly its checks.
def _pool(pool, layers):
    """The C structure, layers, pages, slots of a page, KV heads, head_dim and device of a pool, of one layer unless `layers`."""
    k, v, ks, vs = pool
    shape, dtype, dev = k.shape, k.dtype, k.get_device()
    if len(shape) == 5:
        n_pages, kv, pieces, page, width = shape
        n_layers, lead = 1, (n_pages, kv)
    elif layers and len(shape) == 6:
        n_layers, n_pages, kv, pieces, page, width = shape
        lead = (n_layers, n_pages, kv)
    else:
        raise ValueError("codes of K must be %s[pages][kv_heads][head_dim / 16][page][16]" % ("[layers]" if layers else ""))
    code, v_shape = _CODE.get(dtype), (*lead, page // 16, pieces * 16, 16)
    if not (code is not None and width == 16 and page % 16 == 0 and v.shape == v_shape and v.dtype is dtype and v.get_device() == dev
            and ks.shape == lead and ks.dtype is _F32 and ks.get_device() == dev and vs.shape == lead and vs.dtype is _F32
            and vs.get_device() == dev and k.is_contiguous() and v.is_contiguous() and ks.is_contiguous() and vs.is_contiguous()
            and n_pages <= _INT_MAX and kv <= _INT_MAX and pieces <= _INT_MAX >> 4 and page <= _INT_MAX):
        if code is None:
            raise TypeError("codes must be int8 or float8_e4m3fn, got %s" % dtype)
        if width != 16 or page % 16 or max(n_pages, kv, pieces * 16, page) > _INT_MAX:
            raise ValueError("codes of K must be [pages][kv_heads][head_dim / 16][page][16], got %s" % list(shape))
        _want("codes of V", v, v_shape, dtype, dev)
        _want("k_scale", ks, lead, _F32, dev)
        _want("v_scale", vs, lead, _F32, dev)
        for name, t in zip(("codes of K", "codes of V", "k_scale", "v_scale"), pool):
            _dense(name, t)
    packed = _POOL.pack(code, kv, pieces * 16, n_pages, page, k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr())
    return packed, n_layers, n_pages, page, kv, pieces * 16, dev


def _rows(name, table, n, dev):
    """n_seqs, max_pages and the row stride of a table of int32, with n rows unless that is None."""
    shape = table.shape
    if len(shape) != 2:
        raise ValueError("%s must be [sequences][pages]" % name)
    rows, width = shape
    stride, one = table.stride()
    if not (table.dtype is _I32 and table.get_device() == dev and (n is None or rows == n) and rows <= _INT_MAX and width <= _INT_MAX
            and (one == 1 or width <= 1)):
        _want(name, table, shape if n is None else (n, width), _I32, dev)
        if max(shape) > _INT_MAX:
            raise ValueError("%s is larger than 2^31 - 1 in a dimension" % name)
        raise ValueError("the entries of a row of %s must be contiguous" % name)
    return rows, width, stride if rows > 1 else width


def _ints(name, t, n, dev):
    """The address of n int32."""
    if not (t.shape == (n,) and t.dtype is _I32 and t.get_device() == dev and t.is_contiguous()):
        _want(name, t, (n,), _I32, dev)
        _dense(name, t)
    return t.data_ptr()


def _workspace(size_of, like, *args):
    n = ctypes.c_size_t()
    status = size_of(*args, ctypes.byref(n))
    if status != _j.JPI_OK:
        raise _j.JpiError(status, _j.jpi_cache_last_error())
    n = n.value
    return (torch.empty(n, dtype=torch.uint8, device=like.device), n) if n else (None, 0)


def norm_rope(q, k=None, positions=None, *, q_weight=None, k_weight=None, eps=1e-6, unit_offset=False, rot_dim=None, layout="half",
              base=1e4, scaling="none", factor=1.0, trained=0, beta_fast=32.0, beta_slow=1.0, amplitude=1.0, inverse=False,
              q_out=None, k_out=None):
    """Norms of the heads of q and k, then their rotary positions, in one pass: ``jpi_norm_rope``.

    q_weight, k_weight: [head_dim], or [heads][head_dim] of each tensor, both of one type (bfloat16 or float32); None: the
    norm alone.  unit_offset: the factor is 1 + weight.  Everything else as ``prefix_ops.rope``.  Returns (q_out, k_out).
    """
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError("q and k must be [batch][tokens][heads][head_dim]")
    if _recording():
        _no_gradients(q_weight, k_weight)
    if k is None and k_weight is not None:
        raise ValueError("k_weight without k")
    dh, dev, given = q.shape[3], q.get_device(), [(x, w) for x, w in ((q, q_weight), (k, k_weight)) if w is not None]
    dtype = given[0][1].dtype if given else _F32
    if dtype not in _DTYPE:
        raise TypeError("weights must be bfloat16 or float32, got %s" % dtype)
    stride = 0
    for x, w in given:
        _want("a weight", w, (dh,) if w.dim() == 1 else (x.shape[2], dh), dtype, dev)
        if w.dim() == 2:
            stride = dh
        _dense("a weight", w)
    if stride and any(w.dim() == 1 for _, w in given):
        raise ValueError("weights are [head_dim] for both tensors or [heads][head_dim] for both")
    norm = _pack(_NORM, 0 if q_weight is None else q_weight.data_ptr(), 0 if k_weight is None else k_weight.data_ptr(), _DTYPE[dtype],
                 int(bool(unit_offset)), stride, eps)
    return _turned(norm, q, k, positions, rot_dim, layout, base, scaling, factor, trained, beta_fast, beta_slow, amplitude, inverse,
                   q_out, k_out)


def append(pool, table, starts, k, v, *, n_new=None):
    """Write token t of k and v [sequences][tokens][kv_heads][head_dim] as slot starts[s] + t of sequence s into the pages of
    its row of table: ``jpi_cache_append``.  n_new: int32 [sequences], how many of its tokens are new, None for all; no more
    than resize gave room for, since a page that is written to may be no other sequence's as well.
    """
    packed, _, _, _, kv, dh, dev = _pool(pool, False)
    if k.dim() != 4:
        raise ValueError("k must be [sequences][tokens][kv_heads][head_dim]")
    if _recording():
        _no_gradients(k, v, *pool)
    n, width, stride = _rows("table", table, None, dev)
    seqs = _SEQS.pack(n, width, stride, table.data_ptr(), _ints("starts", starts, n, dev))
    tokens = k.shape[1]
    if tokens > _INT_MAX:
        raise ValueError("k has more than 2^31 - 1 tokens")
    dt, shape = _dtype(k), (n, tokens, kv, dh)
    _want("k", k, shape, k.dtype, dev)
    _want("v", v, shape, k.dtype, dev)
    _launch(dev, _lib.jpi_cache_append, packed, seqs, dt, tokens, _VIEW.pack(*_view("k", k)), _VIEW.pack(*_view("v", v)),
            None if n_new is None else _ints("n_new", n_new, n, dev))
    _written(pool)


def attention(q, pool, table, lens, *, q_lens=None, causal=True, window=0, sinks=0, scale=None, out=None, lse=None):
    """Attention of q [sequences][rows][heads][head_dim] to the slots of each sequence: ``jpi_cache_attention``.

    causal: the last q_lens[s] slots are the queries' own, and a row sees no later ones; window: it sees the last `window`
    of those only, and the first `sinks` of the sequence.  q_lens: int32 [sequences], rows of each, None for all; rows past
    them are left as they were.  scale: head_dim^-1/2 unless given.  Returns (out, lse): out like q, lse float32
    [sequences][rows][heads].
    """
    packed, _, _, _, kv, dh, dev = _pool(pool, False)
    if q.dim() != 4:
        raise ValueError("q must be [sequences][rows][heads][head_dim]")
    if _recording():
        _no_gradients(q, out, lse, *pool)
    given = [t for t in (out, lse) if t is not None]
    n, width, stride = _rows("table", table, None, dev)
    seqs = _SEQS.pack(n, width, stride, table.data_ptr(), _ints("lens", lens, n, dev))
    dt = _dtype(q)
    _, rows, heads, _ = q.shape
    _want("q", q, (n, rows, heads, dh), q.dtype, dev)
    if max(rows, heads) > _INT_MAX:
        raise ValueError("q is larger than 2^31 - 1 in a dimension")
    ql = 0 if q_lens is None else _ints("q_lens", q_lens, n, dev)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        _want("out", out, q.shape, q.dtype, dev)
    if lse is None:
        lse = q.new_empty((n, rows, heads), dtype=_F32)
    else:
        _want("lse", lse, (n, rows, heads), _F32, dev)
    args = _pack(_ATTN, dt, rows, heads, int(bool(causal)), window, sinks, dh ** -0.5 if scale is None else scale, *_view("q", q), ql,
                 *_view("out", out), _dense("lse", lse))
    ws, size = _workspace(_lib.jpi_cache_attention_workspace, q, args, packed, seqs)
    _launch(dev, _lib.jpi_cache_attention, args, packed, seqs, ws.data_ptr() if size else None, size)
    if given:
        _written(given)
    return out, lse


def _moves(table, lens, refs, pool, page, table_out, lens_out, refs_out):
    """The C structures of a move and its pool, layers, the workspace, the device, the number of sequences, and what changes."""
    if pool is not None:
        if _recording():
            _no_gradients(*pool)
        packed, layers, n_pages, slots, _, _, dev = _pool(pool, True)
        if page not in (None, slots):
            raise ValueError("page is %s, that of the pool %d" % (page, slots))
    else:
        packed, layers, n_pages, slots, dev = None, 0, refs.shape[0] if refs.dim() == 1 else 0, page, refs.get_device()
        if n_pages > _INT_MAX:
            raise ValueError("refs has more than 2^31 - 1 pages")
    n, width, stride = _rows("table", table, None, dev)
    if table_out is None:
        table_out, out_stride = table, stride
    else:
        _want("table_out", table_out, table.shape, _I32, dev)
        out_stride = _rows("table_out", table_out, n, dev)[2]
    at = out = 0
    changed = [table_out, refs if refs_out is None else refs_out]
    if lens is not None:
        at = out = _ints("lens", lens, n, dev)
        if lens_out is not None:
            out = _ints("lens_out", lens_out, n, dev)
        changed.append(lens if lens_out is None else lens_out)
    refs_at = _ints("refs", refs, n_pages, dev)
    refs_to = refs_at if refs_out is None else _ints("refs_out", refs_out, n_pages, dev)
    m = _pack(_MOVES, n, width, stride, table.data_ptr(), at, refs_at, table_out.data_ptr(), out_stride, out, refs_to, n_pages, slots)
    ws, size = _workspace(_lib.jpi_cache_moves_workspace, table, m)
    return m, packed, layers, ws, size, dev, n, changed


def _one(name, t, like, dev):
    if t is None:
        return torch.empty(1, dtype=_I32, device=like.device)
    _want(name, t, (1,), _I32, dev)
    return t


def resize(table, lens, refs, new_lens, pool=None, *, page=None, short=None, table_out=None, lens_out=None, refs_out=None):
    """Give sequence s room for new_lens[s] slots, or take what lies behind them back; a partly filled last page that others
    hold too is copied before it grows: ``jpi_cache_resize``.

    table int32 [sequences][pages], lens and new_lens int32 [sequences] (negative: as it is), refs int32 [pages]; each is
    changed in place unless it has an output of its own.  pool: all layers whose pages are copied; None for tables alone,
    with `page` slots of a page.  Returns (lens_out, short), short int32 [1]: pages that were lacking.
    """
    m, packed, layers, ws, size, dev, n, changed = _moves(table, lens, refs, pool, page, table_out, lens_out, refs_out)
    new = _ints("new_lens", new_lens, n, dev)
    short = _one("short", short, table, dev)
    _launch(dev, _lib.jpi_cache_resize, m, packed, layers, new, short.data_ptr(), ws.data_ptr(), size)
    _written([*changed, short, *(pool or ())])
    return changed[2], short


def reorder(table, lens, refs, parents, page, *, table_out=None, lens_out=None, refs_out=None):
    """Sequence s takes over what sequence parents[s] holds, nothing where there is no such sequence: ``jpi_cache_reorder``.
    Forks share their pages until they grow.  Arguments as resize; returns lens_out.
    """
    m, _, _, ws, size, dev, n, changed = _moves(table, lens, refs, None, page, table_out, lens_out, refs_out)
    _launch(dev, _lib.jpi_cache_reorder, m, _ints("parents", parents, n, dev), ws.data_ptr(), size)
    _written(changed)
    return changed[2]


def compact(table, refs, pool=None, *, page=None, n_live=None, table_out=None, refs_out=None):
    """Move the pages in use to the lowest numbers: ``jpi_cache_compact``.  Arguments as resize; returns n_live, int32 [1]:
    pages in use.
    """
    if pool is None and page is None:
        page = 16  # tables alone: of no consequence
    m, packed, layers, ws, size, dev, _, changed = _moves(table, None, refs, pool, page, table_out, None, refs_out)
    n_live = _one("n_live", n_live, table, dev)
    _launch(dev, _lib.jpi_cache_compact, m, packed, layers, n_live.data_ptr(), ws.data_ptr(), size)
    _written([*changed, n_live, *(pool or ())])
    return n_live
