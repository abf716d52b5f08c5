"""Operators of a prefix cache on torch tensors (include/jpi_prefix.h).

PyTorch provides device memory and streams only: every function checks its
tensors, fills in the C arguments and enqueues libjpi's kernels on the current
stream of the tensors' device, which may be capturing a graph.  Outputs and
workspaces are allocated by torch on that stream unless they are given.
Floating tensors are bfloat16 or float32, lengths and positions int32; tensors
may be strided as long as the elements of a head are contiguous.  Errors are
raised as ``jpi.JpiError`` (the library's checks), ``ValueError`` or
``TypeError`` (shapes, devices and types).
"""
from __future__ import annotations

import ctypes

import torch

from . import jpi as _j

_LAYOUT = {"half": _j.JPI_ROPE_HALF, "interleaved": _j.JPI_ROPE_INTERLEAVED}
_SCALING = {"none": _j.JPI_ROPE_PLAIN, "linear": _j.JPI_ROPE_LINEAR, "base": _j.JPI_ROPE_BASE, "parts": _j.JPI_ROPE_PARTS}
_DTYPE = {torch.bfloat16: _j.JPI_BF16, torch.float32: _j.JPI_F32}


def _check(status):
    if status != _j.JPI_OK:
        raise _j.JpiError(status, _j.jpi_prefix_last_error())


def _dtype(t):
    dt = _DTYPE.get(t.dtype)
    if dt is None:
        raise TypeError("tensors must be bfloat16 or float32, got %s" % t.dtype)
    return dt


def _want(name, t, shape, dtype, device):
    """t has this shape, type and device; a size of None in `shape` fits any."""
    if tuple(t.shape) != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, list(shape), list(t.shape)))
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.device != device:
        raise ValueError("%s is on %s, other tensors on %s" % (name, t.device, device))


def _view(name, t):
    """[outer][row][head][head_dim]; strides of dimensions of size 1 do not count."""
    n, s = t.shape, t.stride()
    if s[3] != 1 and n[3] != 1:
        raise ValueError("the elements of a head of %s must be contiguous" % name)
    inner = n[3]
    return _j.jpi_view(t.data_ptr() or None, s[0] if n[0] > 1 else inner, s[1] if n[1] > 1 else inner, s[2] if n[2] > 1 else inner)


def _dense(name, t):
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr() or None


class _On:
    """The tensors' device made current for a call, where it is not (None: nothing to do)."""
    __slots__ = ("guard",)

    def __init__(self, device):
        if device.type != "cuda":
            raise ValueError("tensors must be on the GPU, got %s" % device)
        self.guard = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *e):
        if self.guard is not None:
            self.guard.__exit__(*e)


def rope(q, k=None, positions=None, *, rot_dim=None, layout="half", base=1e4, scaling="none", factor=1.0, trained=0,
         beta_fast=32.0, beta_slow=1.0, amplitude=1.0, inverse=False, q_out=None, k_out=None):
    """Rotary positions of q [batch][tokens][heads][head_dim] and k (the same with its own heads): ``jpi_rope``.

    positions: int32 [batch][tokens] or [tokens], None for 0, 1, 2 ...  q_out, k_out: None for new tensors; q and k
    themselves to turn them in place.  Returns (q_out, k_out), k_out None without k.
    """
    if q.dim() != 4:
        raise ValueError("q must be [batch][tokens][heads][head_dim]")
    b, n, heads, dh = q.shape
    dt, dev = _dtype(q), q.device
    try:
        cfg = _j.jpi_rope_config(dh, dh if rot_dim is None else rot_dim, _LAYOUT[layout], _SCALING[scaling], int(bool(inverse)),
                                 base, factor, trained, beta_fast, beta_slow, amplitude)
    except KeyError as e:
        raise ValueError("unknown layout or scaling %s" % e) from None
    if k is None:
        kv = ko = None
        k_heads = 0
    else:
        k_heads = k.shape[2] if k.dim() == 4 else 0
        _want("k", k, (b, n, k_heads, dh), q.dtype, dev)
        if k_out is None:
            k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
        elif k_out is not k:
            _want("k_out", k_out, tuple(k.shape), q.dtype, dev)
        kv, ko = ctypes.byref(_view("k", k)), ctypes.byref(_view("k_out", k_out))
    if q_out is None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif q_out is not q:
        _want("q_out", q_out, tuple(q.shape), q.dtype, dev)
    pos, pos_stride = None, 0
    if positions is not None:
        if positions.dim() == 2:
            _want("positions", positions, (b, n), torch.int32, dev)
            pos_stride = positions.stride(0)
        else:
            _want("positions", positions, (n,), torch.int32, dev)
        if n > 1 and positions.stride(-1) != 1:
            raise ValueError("positions of a batch row must be contiguous")
        pos = positions.data_ptr() or None
    qv, qo = ctypes.byref(_view("q", q)), ctypes.byref(_view("q_out", q_out))
    with _On(dev) as stream:
        _check(_j.jpi_rope(cfg, dt, b, n, pos, pos_stride, qv, qo, heads, kv, ko, k_heads, stream))
    return q_out, k_out if k is not None else None


def _attn_args(q, k_prefix, scale, prefix_len):
    if q.dim() != 4 or k_prefix.dim() != 4:
        raise ValueError("q and k_prefix must have four dimensions")
    b, rows, heads, dh = q.shape
    g, p, kv, _ = k_prefix.shape
    _want("k_prefix", k_prefix, (g, p, kv, dh), q.dtype, q.device)
    if g < 1 or b < 1 or b % g:
        raise ValueError("the batch of %d must be a multiple of the %d prefixes" % (b, g))
    a = _j.jpi_shared_attn(_dtype(q), g, b // g, rows, heads, kv, dh, p, 0, 0, dh ** -0.5 if scale is None else scale)
    a.q = _view("q", q)
    a.k_prefix = _view("k_prefix", k_prefix)
    if prefix_len is not None:
        _want("prefix_len", prefix_len, (g,), torch.int32, q.device)
        a.prefix_len = _dense("prefix_len", prefix_len)
    return a


def _workspace(a, size_of, device):
    need = size_of(a)
    if not need:
        return None, 0
    return torch.empty(need, dtype=torch.uint8, device=device), need


def shared_attention(q, k_prefix, v_prefix, k_suffix=None, v_suffix=None, *, prefix_len=None, suffix_len=None, causal=False,
                     scale=None, out=None, lse=None):
    """Attention of a batch to a prefix shared by each group of rollouts, and to each rollout's own tail:
    ``jpi_shared_attention``.

    q [batch][rows][heads][head_dim]; k_prefix, v_prefix [groups][prefix][kv_heads][head_dim] (batch a multiple of
    groups, rollouts of a group next to each other); k_suffix, v_suffix [batch][suffix][kv_heads][head_dim] or None;
    prefix_len int32 [groups], suffix_len int32 [batch], None for all slots.  scale: head_dim^-1/2 unless given.
    Returns (out, lse): out like q, lse float32 [batch][rows][heads].
    """
    a = _attn_args(q, k_prefix, scale, prefix_len)
    b, rows, heads, dh = q.shape
    dev = q.device
    _want("v_prefix", v_prefix, tuple(k_prefix.shape), q.dtype, dev)
    a.v_prefix = _view("v_prefix", v_prefix)
    if (k_suffix is None) != (v_suffix is None):
        raise ValueError("k_suffix and v_suffix go together")
    if k_suffix is not None:
        s = k_suffix.shape[1] if k_suffix.dim() == 4 else -1
        shape = (b, s, a.n_kv_heads, dh)
        _want("k_suffix", k_suffix, shape, q.dtype, dev)
        _want("v_suffix", v_suffix, shape, q.dtype, dev)
        a.suffix = s
        a.k_suffix, a.v_suffix = _view("k_suffix", k_suffix), _view("v_suffix", v_suffix)
        if suffix_len is not None:
            _want("suffix_len", suffix_len, (b,), torch.int32, dev)
            a.suffix_len = _dense("suffix_len", suffix_len)
    elif suffix_len is not None:
        raise ValueError("suffix_len without k_suffix")
    a.causal = int(bool(causal))
    if out is None:
        out = torch.empty((b, rows, heads, dh), dtype=q.dtype, device=dev)
    else:
        _want("out", out, (b, rows, heads, dh), q.dtype, dev)
    a.out = _view("out", out)
    if lse is None:
        lse = torch.empty((b, rows, heads), dtype=torch.float32, device=dev)
    else:
        _want("lse", lse, (b, rows, heads), torch.float32, dev)
    a.lse = _dense("lse", lse)
    with _On(dev) as stream:
        ws, n = _workspace(a, _attention_bytes, dev)
        _check(_j.jpi_shared_attention(a, ws, n, stream))
    return out, lse


def _attention_bytes(a):
    st, n = _j.jpi_shared_attention_workspace(a)
    _check(st)
    return n


def _weight_bytes(a):
    st, n = _j.jpi_prefix_weight_workspace(a)
    _check(st)
    return n


def prefix_weight(q, k_prefix, lse, weight=None, *, prefix_len=None, decay=1.0, scale=None, out=None):
    """decay * weight + the softmax weight that the rows of q lay on each prefix slot: ``jpi_prefix_weight``.

    q, k_prefix, prefix_len, scale as for shared_attention, whose lse is taken; weight: float32
    [groups][kv_heads][prefix] or None for zero.  out: None for a new tensor (slots past prefix_len are 0 in it), weight
    itself to accumulate in place.  Returns out.
    """
    a = _attn_args(q, k_prefix, scale, prefix_len)
    dev = q.device
    shape = (a.n_groups, a.n_kv_heads, a.prefix)
    _want("lse", lse, tuple(q.shape[:3]), torch.float32, dev)
    a.lse = _dense("lse", lse)
    w = None
    if weight is not None:
        _want("weight", weight, shape, torch.float32, dev)
        w = _dense("weight", weight)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=dev) if prefix_len is None else torch.zeros(shape, device=dev)
    else:
        _want("out", out, shape, torch.float32, dev)
    with _On(dev) as stream:
        ws, n = _workspace(a, _weight_bytes, dev)
        _check(_j.jpi_prefix_weight(a, w, decay, _dense("out", out), ws, n, stream))
    return out


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
    n, slots, heads, dh = k.shape
    dev = k.device
    _want("v", v, tuple(k.shape), k.dtype, dev)
    _want("weight", weight, (n, heads, slots), torch.float32, dev)
    keep = int(keep)
    most = min(keep, slots)

    def like(name, t, own, dtype, dim):
        if t is None:
            return own
        if t is not own:
            if t.dim() <= dim or t.shape[dim] < most:
                raise ValueError("%s must have room for %d slots" % (name, most))
            shape = list(own.shape)
            shape[dim] = t.shape[dim]
            _want(name, t, tuple(shape), dtype, dev)
        return t

    k_out, v_out = like("k_out", k_out, k, k.dtype, 1), like("v_out", v_out, v, k.dtype, 1)
    weight_out = like("weight_out", weight_out, weight, torch.float32, 2)
    if index is None:
        index = torch.full((n, heads, max(keep, 0)), -1, dtype=torch.int32, device=dev)
    else:
        _want("index", index, (n, heads, keep), torch.int32, dev)
    if lens_out is None:
        lens_out = torch.empty((n,), dtype=torch.int32, device=dev)
    else:
        _want("lens_out", lens_out, (n,), torch.int32, dev)
    a = _j.jpi_evict_args(_dtype(k), n, heads, dh, slots, keep, n_first, n_last, _dense("weight", weight), slots)
    if lens is not None:
        _want("lens", lens, (n,), torch.int32, dev)
        a.len = _dense("lens", lens)
    a.k, a.v, a.k_out, a.v_out = _view("k", k), _view("v", v), _view("k_out", k_out), _view("v_out", v_out)
    a.weight_out, a.weight_out_stride = _dense("weight_out", weight_out), weight_out.shape[2]
    a.index, a.len_out = _dense("index", index), _dense("lens_out", lens_out)
    with _On(dev) as stream:
        _check(_j.jpi_evict(a, stream))
    return index, lens_out
