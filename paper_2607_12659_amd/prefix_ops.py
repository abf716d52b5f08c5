"""Operators of a prefix cache on torch tensors (include/jpi_prefix.h).

PyTorch provides device memory and streams only: every function checks its
tensors, fills in the C arguments and enqueues libjpi's kernels on the current
stream of the tensors' device, which may be capturing a graph.  Outputs and
workspaces are allocated by torch on that stream unless they are given.
Floating tensors are bfloat16 or float32, lengths and positions int32; tensors
may be strided as long as the elements of a head are contiguous (attention and
slot weights want 16-byte aligned rows as well).  No gradients are recorded
(that of a rotation is the rotation with inverse=True), so tensors that require
them are refused while torch records gradients, as torch refuses them for its
own out= arguments; tensors that a call writes into count as changed in place.
Errors are raised as ``jpi.JpiError`` (the library's checks), ``ValueError`` or
``TypeError`` (shapes, devices and types).
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import jpi as _j

_LAYOUT = {"half": _j.JPI_ROPE_HALF, "interleaved": _j.JPI_ROPE_INTERLEAVED}
_SCALING = {"none": _j.JPI_ROPE_PLAIN, "linear": _j.JPI_ROPE_LINEAR, "base": _j.JPI_ROPE_BASE, "parts": _j.JPI_ROPE_PARTS}
_DTYPE = {torch.bfloat16: _j.JPI_BF16, torch.float32: _j.JPI_F32}
_I32, _F32 = torch.int32, torch.float32
_lib = _j._lib

# The C structures as bytes, which cost a small call a third of what a ctypes structure filled field by field does
_V = "Pqqq"
_VIEW = struct.Struct("@" + _V)
_ROPE = struct.Struct("@5i6d")
_ATTN = struct.Struct("@10if" + _V * 5 + "PP" + _V + "P")
_EVICT = struct.Struct("@8iPqP" + _V * 4 + "PqPP")
assert (_ROPE.size, _VIEW.size, _ATTN.size, _EVICT.size) == tuple(
    ctypes.sizeof(c) for c in (_j.jpi_rope_config, _j.jpi_view, _j.jpi_shared_attn, _j.jpi_evict_args))
_NONE = (0, 0, 0, 0)
_INT_MAX = 2 ** 31 - 1  # C's int, to which ctypes would cut a larger one without a word


def _pack(structure, *values):
    try:
        return structure.pack(*values)
    except (struct.error, OverflowError) as e:
        raise ValueError("an argument is no number or out of its C type's range: %s" % e) from None


def _dtype(t):
    dt = _DTYPE.get(t.dtype)
    if dt is None:
        raise TypeError("tensors must be bfloat16 or float32, got %s" % t.dtype)
    return dt


def _want(name, t, shape, dtype, dev):
    """t has this shape and type, and is on GPU number `dev`."""
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, list(shape), list(t.shape)))
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.get_device() != dev:
        raise ValueError("%s is on %s, other tensors on GPU %d" % (name, t.device, dev) if dev >= 0 else
                         "tensors must be on the GPU")


def _view(name, t):
    """data, and the strides of [outer][row][head][head_dim]; those of dimensions of size 1 do not count."""
    n, s = t.shape, t.stride()
    if s[3] != 1 and n[3] != 1:
        raise ValueError("the elements of a head of %s must be contiguous" % name)
    return t.data_ptr(), s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else 0, s[2] if n[2] > 1 else 0


def _dense(name, t):
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


_current_device, _raw_stream = getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None)


_recording, _written = torch.is_grad_enabled, torch.autograd.graph.increment_version


def _no_gradients(*tensors):
    """None of the tensors wants a gradient that the call would not record; asked for while torch records them."""
    for t in tensors:
        if t is not None and t.requires_grad:
            raise ValueError("no gradients are recorded through this call: detach its tensors, or call it under torch.no_grad()")


def _launch(dev, f, *args):
    """f of the library on the current stream of GPU `dev`, which is made current for the call where it is not."""
    if dev < 0:
        raise ValueError("tensors must be on the GPU")
    if dev == _current_device():
        status = f(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            status = f(*args, _raw_stream(dev))
    if status != _j.JPI_OK:
        raise _j.JpiError(status, _LAST_ERROR.get(f.__name__, _j.jpi_prefix_last_error)())


_LAST_ERROR = {}  # of functions of another header than include/jpi_prefix.h


def rope(q, k=None, positions=None, *, rot_dim=None, layout="half", base=1e4, scaling="none", factor=1.0, trained=0,
         beta_fast=32.0, beta_slow=1.0, amplitude=1.0, inverse=False, q_out=None, k_out=None):
    """Rotary positions of q [batch][tokens][heads][head_dim] and k (the same with its own heads): ``jpi_rope``.

    positions: int32 [batch][tokens] or [tokens], None for 0, 1, 2 ...  q_out, k_out: None for new tensors; q and k
    themselves to turn them in place.  Returns (q_out, k_out), k_out None without k.
    """
    return _turned(None, q, k, positions, rot_dim, layout, base, scaling, factor, trained, beta_fast, beta_slow, amplitude, inverse,
                   q_out, k_out)


def _turned(norm, q, k, positions, rot_dim, layout, base, scaling, factor, trained, beta_fast, beta_slow, amplitude, inverse, q_out,
            k_out):
    """jpi_rope, or jpi_norm_rope with the norm's arguments."""
    if q.dim() != 4:
        raise ValueError("q must be [batch][tokens][heads][head_dim]")
    if _recording():
        _no_gradients(q, k, q_out, k_out)
    given = [t for t in (q_out, k_out) if t is not None]
    b, n, heads, dh = q.shape
    dt, dev = _dtype(q), q.get_device()
    if layout not in _LAYOUT or scaling not in _SCALING:
        raise ValueError("unknown layout %r or scaling %r" % (layout, scaling))
    cfg = _pack(_ROPE, dh, dh if rot_dim is None else rot_dim, _LAYOUT[layout], _SCALING[scaling], int(bool(inverse)), base,
                factor, trained, beta_fast, beta_slow, amplitude)
    if b > _INT_MAX or n > _INT_MAX or heads > _INT_MAX:
        raise ValueError("q is larger than 2^31 - 1 in a dimension")
    if q_out is None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif q_out is not q:
        _want("q_out", q_out, q.shape, q.dtype, dev)
    if k is None:
        kv = ko = k_out = None
        k_heads = 0
    else:
        k_heads = k.shape[2] if k.dim() == 4 else 0
        _want("k", k, (b, n, k_heads, dh), q.dtype, dev)
        if k_heads > _INT_MAX:
            raise ValueError("k has more than 2^31 - 1 heads")
        if k_out is None:
            k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
        elif k_out is not k:
            _want("k_out", k_out, k.shape, q.dtype, dev)
        if k_heads:
            kv, ko = _VIEW.pack(*_view("k", k)), _VIEW.pack(*_view("k_out", k_out))
        else:
            kv = ko = None
    pos, pos_stride = None, 0
    if positions is not None:
        if positions.dim() == 2:
            _want("positions", positions, (b, n), _I32, dev)
            pos_stride = positions.stride(0) if b > 1 else 0
        else:
            _want("positions", positions, (n,), _I32, dev)
        if n > 1 and positions.stride(-1) != 1:
            raise ValueError("positions of a batch row must be contiguous")
        pos = positions.data_ptr()
    pack = _VIEW.pack
    args = (cfg, dt, b, n, pos, pos_stride, pack(*_view("q", q)), pack(*_view("q_out", q_out)), heads, kv, ko, k_heads)
    if norm is None:
        _launch(dev, _lib.jpi_rope, *args)
    else:
        _launch(dev, _lib.jpi_norm_rope, norm, *args)
    if given:
        _written(given)
    return q_out, k_out


def _shapes(q, k_prefix):
    if q.dim() != 4 or k_prefix.dim() != 4:
        raise ValueError("q and k_prefix must have four dimensions")
    b, rows, heads, dh = q.shape
    g, p, kv, _ = k_prefix.shape
    dev = q.get_device()
    _want("k_prefix", k_prefix, (g, p, kv, dh), q.dtype, dev)
    if g < 1 or b < 1 or b % g:
        raise ValueError("the batch of %d must be a multiple of the %d prefixes" % (b, g))
    return b, rows, heads, dh, g, p, kv, dev


def _lens(name, t, n, dev):
    if t is None:
        return 0
    _want(name, t, (n,), _I32, dev)
    return _dense(name, t)


def _workspace(size_of, args, q):
    n = ctypes.c_size_t()
    status = size_of(args, ctypes.byref(n))
    if status != _j.JPI_OK:
        raise _j.JpiError(status, _j.jpi_prefix_last_error())
    n = n.value
    return (q.new_empty(n, dtype=torch.uint8), n) if n else (None, 0)


def shared_attention(q, k_prefix, v_prefix, k_suffix=None, v_suffix=None, *, prefix_len=None, suffix_len=None, causal=False,
                     scale=None, out=None, lse=None):
    """Attention of a batch to a prefix shared by each group of rollouts, and to each rollout's own tail:
    ``jpi_shared_attention``.

    q [batch][rows][heads][head_dim]; k_prefix, v_prefix [groups][prefix][kv_heads][head_dim] (batch a multiple of
    groups, rollouts of a group next to each other); k_suffix, v_suffix [batch][suffix][kv_heads][head_dim] or None;
    prefix_len int32 [groups], suffix_len int32 [batch], None for all slots.  scale: head_dim^-1/2 unless given.
    Returns (out, lse): out like q, lse float32 [batch][rows][heads].
    """
    b, rows, heads, dh, g, p, kv, dev = _shapes(q, k_prefix)
    if _recording():
        _no_gradients(q, k_prefix, v_prefix, k_suffix, v_suffix, out, lse)
    given = [t for t in (out, lse) if t is not None]
    dt = _dtype(q)
    _want("v_prefix", v_prefix, k_prefix.shape, q.dtype, dev)
    if (k_suffix is None) != (v_suffix is None):
        raise ValueError("k_suffix and v_suffix go together")
    if k_suffix is None:
        if suffix_len is not None:
            raise ValueError("suffix_len without k_suffix")
        s, ks, vs = 0, _NONE, _NONE
    else:
        s = k_suffix.shape[1] if k_suffix.dim() == 4 else -1
        _want("k_suffix", k_suffix, (b, s, kv, dh), q.dtype, dev)
        _want("v_suffix", v_suffix, k_suffix.shape, q.dtype, dev)
        ks, vs = _view("k_suffix", k_suffix), _view("v_suffix", v_suffix)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        _want("out", out, q.shape, q.dtype, dev)
    if lse is None:
        lse = q.new_empty((b, rows, heads), dtype=_F32)
    else:
        _want("lse", lse, (b, rows, heads), _F32, dev)
    args = _pack(_ATTN, dt, g, b // g, rows, heads, kv, dh, p, s, int(bool(causal)), dh ** -0.5 if scale is None else scale,
                 *_view("q", q), *_view("k_prefix", k_prefix), *_view("v_prefix", v_prefix), *ks, *vs,
                 _lens("prefix_len", prefix_len, g, dev), _lens("suffix_len", suffix_len, b, dev), *_view("out", out),
                 _dense("lse", lse))
    ws, n = _workspace(_lib.jpi_shared_attention_workspace, args, q)
    _launch(dev, _lib.jpi_shared_attention, args, ws.data_ptr() if n else None, n)
    if given:
        _written(given)
    return out, lse


def prefix_weight(q, k_prefix, lse, weight=None, *, prefix_len=None, decay=1.0, scale=None, out=None):
    """decay * weight + the softmax weight that the rows of q lay on each prefix slot: ``jpi_prefix_weight``.

    q, k_prefix, prefix_len, scale as for shared_attention, whose lse is taken; weight: float32
    [groups][kv_heads][prefix] or None for zero.  out: None for a new tensor (slots past prefix_len are 0 in it), weight
    itself to accumulate in place.  Returns out.
    """
    b, rows, heads, dh, g, p, kv, dev = _shapes(q, k_prefix)
    if _recording():
        _no_gradients(q, k_prefix, lse, weight, out)
    dt, shape = _dtype(q), (g, kv, p)
    _want("lse", lse, (b, rows, heads), _F32, dev)
    w = None
    if weight is not None:
        _want("weight", weight, shape, _F32, dev)
        w = _dense("weight", weight)
    given = out is not None
    if not given:
        out = (q.new_empty if prefix_len is None else q.new_zeros)(shape, dtype=_F32)
    else:
        _want("out", out, shape, _F32, dev)
    args = _pack(_ATTN, dt, g, b // g, rows, heads, kv, dh, p, 0, 0, dh ** -0.5 if scale is None else scale, *_view("q", q),
                 *_view("k_prefix", k_prefix), *_NONE, *_NONE, *_NONE, _lens("prefix_len", prefix_len, g, dev), 0, *_NONE,
                 _dense("lse", lse))
    ws, n = _workspace(_lib.jpi_prefix_weight_workspace, args, q)
    _launch(dev, _lib.jpi_prefix_weight, args, w, float(decay), _dense("out", out), ws.data_ptr() if n else None, n)
    if given:
        _written(out)
    return out


def _room(name, t, own, dtype, dim, most, dev):
    """t, or `own` where it is None: like `own` but for dimension `dim`, which has room for `most`."""
    if t is None or t is own:
        return own
    if t.dim() <= dim or t.shape[dim] < most:
        raise ValueError("%s must have room for %d slots" % (name, most))
    n = own.shape
    _want(name, t, n[:dim] + t.shape[dim:dim + 1] + n[dim + 1:], dtype, dev)
    return t


def evict(k, v, weight, keep, *, lens=None, n_first=0, n_last=0, k_out=None, v_out=None, weight_out=None, index=None,
          lens_out=None):
    """Keep the `keep` heaviest slots of each cached sequence, in their order: ``jpi_evict``.

    k, v [outer][slots][heads][head_dim]; weight float32 [outer][heads][slots]; lens int32 [outer] or None for all slots.
    k_out, v_out [outer][min(keep, slots) or more][heads][head_dim], weight_out [outer][heads][min(keep, slots) or
    more]: where the kept slots go; None compacts k, v and weight themselves.  index: int32 [outer][heads][keep] for the
    old slots, None for a new tensor (-1 past the kept ones).  Returns (index, lens_out).
    """
    if k.dim() != 4:
        raise ValueError("k must be [outer][slots][heads][head_dim]")
    if _recording():
        _no_gradients(k, v, weight, k_out, v_out, weight_out)
    given = [t for t in (index, lens_out) if t is not None]
    n, slots, heads, dh = k.shape
    dt, dev = _dtype(k), k.get_device()
    _want("v", v, k.shape, k.dtype, dev)
    _want("weight", weight, (n, heads, slots), _F32, dev)
    keep = int(keep)
    if keep > _INT_MAX:
        raise ValueError("keep is larger than 2^31 - 1")
    most = min(keep, slots)
    k_out, v_out = _room("k_out", k_out, k, k.dtype, 1, most, dev), _room("v_out", v_out, v, k.dtype, 1, most, dev)
    weight_out = _room("weight_out", weight_out, weight, _F32, 2, most, dev)
    if index is None:
        index = torch.full((n, heads, max(keep, 0)), -1, dtype=_I32, device=k.device)
    else:
        _want("index", index, (n, heads, keep), _I32, dev)
    if lens_out is None:
        lens_out = torch.empty((n,), dtype=_I32, device=k.device)
    else:
        _want("lens_out", lens_out, (n,), _I32, dev)
    args = _pack(_EVICT, dt, n, heads, dh, slots, keep, n_first, n_last, _dense("weight", weight), slots,
                 _lens("lens", lens, n, dev), *_view("k", k), *_view("v", v), *_view("k_out", k_out), *_view("v_out", v_out),
                 _dense("weight_out", weight_out), weight_out.shape[2], _dense("index", index), _dense("lens_out", lens_out))
    _launch(dev, _lib.jpi_evict, args)
    _written([k_out, v_out, weight_out, *given])
    return index, lens_out
