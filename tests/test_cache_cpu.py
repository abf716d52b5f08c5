"""Refusals of the operators of a paged 8-bit cache (include/jpi_cache.h) that need no GPU: every check is made on the host,
before anything is enqueued, so no pointer here is ever used."""
import ctypes
import math

import pytest

from paper_2607_12659_amd import jpi as j

FAKE = 0x10000


def view(data=FAKE, outer=0, row=256, head=256):
    return j.jpi_view(data, outer, row, head)


def put(structure, kw):
    for n, v in kw.items():
        setattr(structure, n, v)
    return structure


def pool(**kw):
    return put(j.jpi_cache_pool(j.JPI_E4M3, 2, 128, 100, 64, FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE), kw)


def seqs(**kw):
    return put(j.jpi_cache_seqs(3, 8, 8, FAKE, FAKE), kw)


BAD_POOL = [dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=96), dict(head_dim=512), dict(n_pages=0),
            dict(n_pages=(1 << 24) + 1), dict(page=0), dict(page=8), dict(page=48), dict(page=256)]
BAD_DATA = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=FAKE + 8), dict(v=FAKE + 1), dict(v=FAKE),
            dict(v_scale=3 * FAKE)]
BAD_SEQS = [dict(n_seqs=0), dict(n_seqs=65537), dict(max_pages=0), dict(max_pages=(1 << 22) + 1, table_stride=1 << 23),
            dict(table_stride=7)]


# ---- norms with rotation -------------------------------------------------------------------------------------------------
def norm_call(q=None, k=None, k_out=None, dtype=j.JPI_BF16, batch=1, tokens=4, heads=2, k_heads=0, pos_stride=0, q_out=None, norm=None,
              **kw):
    cfg = dict(head_dim=64, rot_dim=64, layout=0, scaling=0, inverse=0, base=1e4, factor=1.0, trained=0.0, beta_fast=32.0,
               beta_slow=1.0, amplitude=1.0)
    cfg.update(kw)
    n = put(j.jpi_head_norm(FAKE, FAKE, j.JPI_BF16, 0, 0, 1e-6), norm or {})
    return j.jpi_norm_rope(n, j.jpi_rope_config(**cfg), dtype, batch, tokens, None, pos_stride, q or view(), q_out or view(2 * FAKE),
                           heads, k, k_out, k_heads)


@pytest.mark.parametrize("bad", [dict(norm=dict(eps=0.0)), dict(norm=dict(eps=-1.0)), dict(norm=dict(eps=1e-60)),
                                 dict(norm=dict(eps=math.inf)), dict(norm=dict(eps=math.nan)), dict(norm=dict(weight_stride=-1)),
                                 dict(head_dim=65), dict(rot_dim=66), dict(layout=2), dict(scaling=4), dict(base=1.0),
                                 dict(amplitude=1e39), dict(batch=-1), dict(heads=0), dict(k=view()), dict(q=view(None)),
                                 dict(q=view(), q_out=view(row=512)), dict(q_out=view(2 * FAKE, row=0)),
                                 dict(q=view(), k=view(3 * FAKE), q_out=view(2 * FAKE), k_out=view(2 * FAKE), k_heads=2)])
def test_norm_rope_refuses(bad):
    assert norm_call(**bad) == j.JPI_ERR_ARG
    assert j.jpi_cache_last_error().startswith("jpi_norm_rope: ")


def test_norm_rope_refuses_types_and_sizes():
    assert norm_call(dtype=2) == j.JPI_ERR_DTYPE
    assert norm_call(norm=dict(weight_dtype=2)) == j.JPI_ERR_DTYPE
    assert norm_call(batch=1 << 16, tokens=1 << 15) == j.JPI_ERR_SHAPE
    assert j._lib.jpi_norm_rope(None, None, 1, 1, 1, None, 0, None, None, 1, None, None, 0, None) == j.JPI_ERR_ARG
    assert norm_call(tokens=0, q=view(None)) == j.JPI_OK


# ---- append --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("bad", BAD_POOL + BAD_DATA)
def test_append_refuses_pools(bad):
    assert j.jpi_cache_append(pool(**bad), seqs(), j.JPI_BF16, 4, view(), view()) == j.JPI_ERR_ARG
    assert j.jpi_cache_last_error().startswith("jpi_cache_append: ")


@pytest.mark.parametrize("bad", BAD_SEQS + [dict(table=None), dict(len=None)])
def test_append_refuses_sequences(bad):
    assert j.jpi_cache_append(pool(), seqs(**bad), j.JPI_BF16, 4, view(), view()) == j.JPI_ERR_ARG


def test_append_refuses_the_rest():
    def call(tokens=4, k=view(), v=view(), dt=j.JPI_BF16, p=None, q=None):
        return j.jpi_cache_append(p or pool(), q or seqs(), dt, tokens, k, v)
    assert call(tokens=-1) == j.JPI_ERR_ARG
    for bad in (None, view(None), view(row=-1), view(outer=-1), view(head=-8)):
        assert call(k=bad) == j.JPI_ERR_ARG and call(v=bad) == j.JPI_ERR_ARG
    assert call(dt=2) == j.JPI_ERR_DTYPE and call(p=pool(code=2)) == j.JPI_ERR_DTYPE and call(p=pool(code=-1)) == j.JPI_ERR_DTYPE
    assert call(tokens=1 << 30, q=seqs(n_seqs=4)) == j.JPI_ERR_SHAPE
    assert call(tokens=1 << 20, q=seqs(n_seqs=1024), p=pool(page=16)) == j.JPI_ERR_SHAPE and "workgroups" in j.jpi_cache_last_error()
    assert j._lib.jpi_cache_append(None, None, 1, 1, None, None, None, None) == j.JPI_ERR_ARG
    assert j.jpi_cache_append(pool(), None, j.JPI_BF16, 4, view(), view()) == j.JPI_ERR_ARG
    assert call(tokens=0, p=pool(k=None), k=None) == j.JPI_OK


# ---- attention -----------------------------------------------------------------------------------------------------------
def attn(**kw):
    return put(j.jpi_cache_attn(j.JPI_BF16, 5, 8, 1, 0, 0, 0.125, view(), None, view(2 * FAKE, 2048), None), kw)


def attend(a=None, p=None, q=None, ws=FAKE, size=1 << 40):
    return j.jpi_cache_attention(a or attn(), p or pool(), q or seqs(), ws, size)


@pytest.mark.parametrize("bad", [dict(q_rows=0), dict(n_heads=0), dict(n_heads=3), dict(window=-1), dict(sinks=-1),
                                 dict(window=5, causal=0), dict(sinks=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
                                 dict(scale=3e38), dict(q=view(None)), dict(out=view(None)), dict(q=view(FAKE + 8)),
                                 dict(q=view(row=12)), dict(out=view(2 * FAKE, row=-8)), dict(out=view()),
                                 dict(out=view(2 * FAKE, outer=0)), dict(out=view(2 * FAKE, outer=2048, row=0)),
                                 dict(out=view(2 * FAKE, outer=2048, head=0))])
def test_attention_refuses(bad):
    assert attend(attn(**bad)) == j.JPI_ERR_ARG
    assert j.jpi_cache_last_error().startswith("jpi_cache_attention: ")


@pytest.mark.parametrize("bad", BAD_POOL + BAD_DATA)
def test_attention_refuses_pools(bad):
    assert attend(p=pool(**bad)) == j.JPI_ERR_ARG


@pytest.mark.parametrize("bad", BAD_SEQS + [dict(table=None), dict(len=None)])
def test_attention_refuses_sequences(bad):
    assert attend(q=seqs(**bad)) == j.JPI_ERR_ARG


def test_attention_refuses_types_sizes_and_workspaces():
    assert attend(attn(dtype=2)) == j.JPI_ERR_DTYPE and attend(p=pool(code=2)) == j.JPI_ERR_DTYPE
    assert attend(attn(q_rows=1 << 28)) == j.JPI_ERR_SHAPE
    assert attend(attn(dtype=j.JPI_F32, q_rows=1 << 22, n_heads=2), pool(), seqs(n_seqs=128)) == j.JPI_ERR_SHAPE  # a workgroup for each 16 rows
    assert "workgroups" in j.jpi_cache_last_error()
    long = seqs(max_pages=1024, table_stride=1024)
    st, n = j.jpi_cache_attention_workspace(attn(), pool(), long)
    st2, groups, tiles, ranges = j.jpi_debug_cache_plan(attn(), pool(), long)
    assert st == st2 == j.JPI_OK and groups == 0 and tiles == 2 and ranges > 1
    assert n == 3 * 2 * tiles * ranges * 16 * (128 * 4 + 8)  # a sum and two statistics of each row in each range
    assert attend(q=long, ws=None) == j.JPI_ERR_ARG and "workspace" in j.jpi_cache_last_error()
    assert attend(q=long, size=n - 1) == j.JPI_ERR_ARG and attend(q=long, ws=FAKE + 4, size=n) == j.JPI_ERR_ARG
    assert j.jpi_cache_attention_workspace(attn(scale=0.0), pool(), long) == (j.JPI_ERR_ARG, 0)
    assert j._lib.jpi_cache_attention_workspace(None, None, None, None) == j.JPI_ERR_ARG
    assert j._lib.jpi_cache_attention(None, None, None, None, 0, None) == j.JPI_ERR_ARG
    assert j._lib.jpi_debug_cache_plan(None, None, None, None, None, None) == j.JPI_ERR_ARG


def test_how_a_call_is_cut():
    """Waves, groups and ranges by sizes: a row before a short table, a chunk, a long table, many rows, and fp32."""
    def plan(rows, heads, kv, dim, width, n=1, **kw):
        a, p, q = attn(q_rows=rows, n_heads=heads, **kw), pool(n_kv_heads=kv, head_dim=dim), seqs(n_seqs=n, max_pages=width, table_stride=width)
        (st, groups, _, ranges), (st2, waves) = j.jpi_debug_cache_plan(a, p, q), j.jpi_debug_cache_waves(a, p, q)
        assert st == st2 == j.JPI_OK
        return waves, groups > 0, ranges > 1
    assert plan(1, 8, 1, 256, 13) == (8, False, False) and plan(1, 8, 1, 256, 13, dtype=j.JPI_F32) == (4, False, True)
    assert plan(50, 8, 1, 256, 14, n=8) == (8, False, False) and plan(50, 8, 1, 256, 64) == (8, False, True)
    assert plan(1, 32, 8, 128, 64) == (4, False, True) and plan(1, 32, 8, 128, 7) == (4, False, False)
    assert plan(1, 32, 8, 128, 128, n=64) == (4, False, False) and plan(4096, 32, 8, 128, 64)[1:] == (True, False)
    assert plan(512, 32, 8, 128, 128)[1:] == (True, True)
    assert j.jpi_debug_cache_waves(attn(q_rows=0), pool(), seqs()) == (j.JPI_ERR_ARG, 0)
    assert j.jpi_cache_last_error().startswith("jpi_debug_cache_waves: ")
    assert j._lib.jpi_debug_cache_waves(None, None, None, None) == j.JPI_ERR_ARG


# ---- moves of pages ------------------------------------------------------------------------------------------------------
def moves(**kw):
    m = j.jpi_cache_moves(seqs(table=FAKE, len=2 * FAKE), 3 * FAKE, 4 * FAKE, 8, 5 * FAKE, 6 * FAKE, 100, 64)
    return put(m, kw)


CALLS = {"resize": lambda m, ws=FAKE, n=1 << 40, p=None, layers=0: j.jpi_cache_resize(m, p, layers, 7 * FAKE, None, ws, n),
         "reorder": lambda m, ws=FAKE, n=1 << 40: j.jpi_cache_reorder(m, 7 * FAKE, ws, n),
         "compact": lambda m, ws=FAKE, n=1 << 40, p=None, layers=0: j.jpi_cache_compact(m, p, layers, None, ws, n)}


@pytest.mark.parametrize("name", CALLS)
def test_moves_refuse(name):
    call = CALLS[name]
    bad = [dict(refs=None), dict(table_out=None), dict(refs_out=None), dict(table_out_stride=7), dict(n_pages=0),
           dict(n_pages=(1 << 24) + 1), dict(page=8), dict(page=65), dict(seqs=seqs(table=None)),
           dict(table_out=3 * FAKE), dict(refs_out=FAKE), dict(refs_out=4 * FAKE), dict(table_out=FAKE, table_out_stride=9)]
    bad += [dict(seqs=seqs(**b)) for b in BAD_SEQS]
    if name != "compact":
        bad += [dict(seqs=seqs(len=None)), dict(len_out=None), dict(len_out=FAKE), dict(len_out=4 * FAKE), dict(refs_out=2 * FAKE)]
    for b in bad:
        assert call(moves(**b)) == j.JPI_ERR_ARG, b
        assert j.jpi_cache_last_error().startswith("jpi_cache_%s: " % name)
    if name != "reorder":
        for b in BAD_POOL + BAD_DATA + [dict(n_pages=99), dict(page=32)]:
            assert call(moves(), p=pool(**b), layers=1) == j.JPI_ERR_ARG, b
        for layers in (0, -1, 65537):
            assert call(moves(), p=pool(), layers=layers) == j.JPI_ERR_ARG
        assert call(moves(), p=pool(code=7), layers=1) == j.JPI_ERR_DTYPE
    many = seqs(n_seqs=65536, max_pages=1 << 15, table_stride=1 << 15, len=2 * FAKE)
    assert call(moves(seqs=many, table_out_stride=1 << 15)) == j.JPI_ERR_SHAPE
    st, n = j.jpi_cache_moves_workspace(moves())
    assert st == j.JPI_OK and n > 0
    assert call(moves(), None) == j.JPI_ERR_ARG and call(moves(), FAKE, n - 1) == j.JPI_ERR_ARG
    assert call(moves(), FAKE + 4, n) == j.JPI_ERR_ARG and "workspace" in j.jpi_cache_last_error()
    assert j.jpi_cache_moves_workspace(moves(page=5)) == (j.JPI_ERR_ARG, 0)


def test_moves_refuse_null():
    assert j.jpi_cache_resize(moves(), None, 0, None, None, FAKE, 1 << 40) == j.JPI_ERR_ARG
    assert j.jpi_cache_reorder(moves(), None, FAKE, 1 << 40) == j.JPI_ERR_ARG
    assert j.jpi_cache_reorder(moves(), 5 * FAKE, FAKE, 1 << 40) == j.JPI_ERR_ARG  # len_out
    assert j._lib.jpi_cache_compact(None, None, 0, None, None, 0, None) == j.JPI_ERR_ARG
    assert j._lib.jpi_cache_moves_workspace(None, None) == j.JPI_ERR_ARG


def test_structures_have_the_headers_sizes():
    """Field by field the header's types: 8-byte members aligned, ints of 4 bytes."""
    assert ctypes.sizeof(j.jpi_cache_pool) == 24 + 4 * 8
    assert ctypes.sizeof(j.jpi_cache_seqs) == 8 + 3 * 8
    assert ctypes.sizeof(j.jpi_head_norm) == 16 + 8 + 16
    assert ctypes.sizeof(j.jpi_cache_attn) == 32 + 32 + 8 + 32 + 8
    assert ctypes.sizeof(j.jpi_cache_moves) == 32 + 8 + 8 + 8 + 16 + 8


# ---- the same on tensors ---------------------------------------------------------------------------------------------------
@pytest.fixture
def ops():
    pytest.importorskip("torch")
    from paper_2607_12659_amd import cache_ops
    return cache_ops


def tensors(ops):
    import torch
    p = ops.Pool.zeros(10, 2, 64, 32, device="cpu")
    i32 = dict(dtype=torch.int32)
    return p, torch.zeros(3, 4, **i32), torch.zeros(3, **i32), torch.zeros(10, **i32), torch.zeros(3, 5, 4, 64), torch.zeros(3, 5, 2, 64)


def test_tensors_on_the_cpu_are_refused(ops):
    p, table, lens, refs, q, k = tensors(ops)
    for call in (lambda: ops.norm_rope(q, k), lambda: ops.append(p, table, lens, k, k), lambda: ops.attention(q, p, table, lens),
                 lambda: ops.resize(table, lens, refs, lens.clone(), p), lambda: ops.reorder(table, lens, refs, lens.clone(), 32),
                 lambda: ops.compact(table, refs, p)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_tensors_of_other_shapes_and_types_are_refused(ops):
    import torch
    p, table, lens, refs, q, k = tensors(ops)
    w = torch.zeros(64)
    shape = [lambda: ops.attention(q[0], p, table, lens), lambda: ops.attention(q[:2], p, table, lens),
             lambda: ops.attention(q, p, table[0], lens), lambda: ops.attention(q, p, table, lens[:2]),
             lambda: ops.attention(q, p, table, lens, q_lens=lens[:1]), lambda: ops.attention(q, p, table, lens, out=q[:1]),
             lambda: ops.attention(q, p, table, lens, lse=w), lambda: ops.attention(q, p._replace(k=p.k[0]), table, lens),
             lambda: ops.attention(q, p._replace(v=p.v[:5]), table, lens), lambda: ops.attention(q, p._replace(v_scale=w), table, lens),
             lambda: ops.attention(q, ops.Pool(*(x[None] for x in p)), table, lens),
             lambda: ops.attention(q, p, table.t().contiguous().t(), lens),
             lambda: ops.append(p, table, lens, q, q), lambda: ops.append(p, table, lens, k, k[:, :1]),
             lambda: ops.append(p, table, lens, k, k, n_new=refs), lambda: ops.append(p, table, lens[:1], k, k),
             lambda: ops.norm_rope(q[0]), lambda: ops.norm_rope(q, k_weight=w), lambda: ops.norm_rope(q, q_weight=w[:5]),
             lambda: ops.norm_rope(q, k, q_weight=w, k_weight=torch.zeros(2, 64)),
             lambda: ops.resize(table, lens, refs[:3], lens, p), lambda: ops.resize(table, lens, refs, refs, p),
             lambda: ops.resize(table, lens, refs, lens, p, page=64), lambda: ops.resize(table, lens, refs, lens, p, short=refs),
             lambda: ops.reorder(table, lens, refs, refs, 32), lambda: ops.reorder(table, lens, refs, lens, 32, table_out=table[:1]),
             lambda: ops.compact(table, refs, p, n_live=lens), lambda: ops.compact(table, refs, p, refs_out=lens),
             lambda: ops.Pool.zeros(3, 1, 72, 16, device="cpu"), lambda: ops.Pool.zeros(3, 1, 64, 24, device="cpu")]
    for i, call in enumerate(shape):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d" % i)
    types = [lambda: ops.attention(q.half(), p, table, lens), lambda: ops.attention(q, p, table.long(), lens),
             lambda: ops.attention(q, p._replace(k=p.k.view(torch.uint8)), table, lens),
             lambda: ops.attention(q, p._replace(v=p.v.view(torch.int8)), table, lens),
             lambda: ops.append(p, table, lens, k.half(), k.half()), lambda: ops.append(p, table, lens, k, k.bfloat16()),
             lambda: ops.norm_rope(q, q_weight=w.half()), lambda: ops.norm_rope(q, k, q_weight=w, k_weight=w.bfloat16()),
             lambda: ops.Pool.zeros(3, 1, 64, 16, code=torch.uint8, device="cpu"), lambda: ops.resize(table, lens, refs, lens.long(), p)]
    for i, call in enumerate(types):
        with pytest.raises(TypeError):
            call()
            pytest.fail("call %d" % i)
    numbers = [lambda: ops.attention(q, p, table, lens, window=2 ** 31), lambda: ops.attention(q, p, table, lens, scale="one"),
               lambda: ops.attention(q, p, table, lens, sinks=0.5), lambda: ops.norm_rope(q, eps="small"),
               lambda: ops.reorder(table, lens, refs, lens, 2 ** 31)]
    for call in numbers:
        with pytest.raises(ValueError, match="range|could not convert"):
            call()


def test_tensors_that_want_gradients_are_refused(ops):
    import torch
    p, table, lens, refs, q, k = tensors(ops)
    leaf, leaf_k, w = q.clone().requires_grad_(), k.clone().requires_grad_(), torch.zeros(64, requires_grad=True)
    for call in (lambda: ops.norm_rope(leaf), lambda: ops.norm_rope(q, leaf_k), lambda: ops.norm_rope(q, q_weight=w),
                 lambda: ops.append(p, table, lens, leaf_k, k), lambda: ops.append(p, table, lens, k, leaf_k),
                 lambda: ops.attention(leaf, p, table, lens), lambda: ops.attention(q, p, table, lens, out=leaf)):
        with pytest.raises(ValueError, match="gradients"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call()


def test_pools_that_want_gradients_are_refused_by_moves(ops):
    import torch
    p, table, lens, refs, _, _ = tensors(ops)
    for i in (2, 3):
        leaf = p._replace(**{p._fields[i]: p[i].clone().requires_grad_()})
        for call in (lambda: ops.resize(table, lens, refs, lens.clone(), leaf), lambda: ops.compact(table, refs, leaf)):
            with pytest.raises(ValueError, match="gradients"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
                call()


# ---- the step that the module describes, in a pool that runs out -------------------------------------------------------------
def test_the_described_step_leaves_alone_who_was_not_served(ops):
    """The step of the module's docstring, run over the plain forms: two forks that share their last page want to grow, and the
    pool has a page for neither or for one; a third one has room in its own page."""
    import re
    import textwrap

    import numpy as np

    import cache_reference as ref

    text = re.search(r"::\n\n(.*?)\n\n?\Z", ops.__doc__ + "\n", re.S).group(1)
    code = textwrap.dedent(text).replace("for each layer:", "for i in range(layers):")
    page, layers, kv, dh = 16, 2, 1, 64

    class Layers(list):
        layer = list.__getitem__

    for free in (0, 1):
        n_pages = 3 + free
        r = np.random.RandomState(free)
        pool = Layers([[r.randint(0, 64, (n_pages, kv, dh // 16, page, 16)).astype(np.uint8),
                        r.randint(0, 64, (n_pages, kv, page // 16, dh, 16)).astype(np.uint8),
                        np.ones((n_pages, kv), np.float32), np.ones((n_pages, kv), np.float32)] for _ in range(layers)])
        table, lens = np.array([[1, -1], [1, -1], [2, -1]], np.int32), np.array([5, 5, 7], np.int32)
        refs = np.array([1, 2, 1] + [0] * free, np.int32)
        shared = [[x[1].copy() for x in p] for p in pool]
        rows = []

        class Lens(np.ndarray):
            clone = np.ndarray.copy

        def resize(table, lens, refs, new, pool):
            *state, short, copies = ref.resize(table, np.asarray(lens), refs, np.asarray(new), page)
            for x, y in zip((table, lens, refs), state):
                x[...] = y
            for p in pool:
                for x in p:
                    for a, b in copies:
                        x[b] = x[a]
            return lens, short

        def append(p, table, starts, k, v, n_new=None):
            n = np.full(3, k.shape[1]) if n_new is None else np.asarray(n_new)
            for x, of in ((0, k), (1, v)):
                ref.append_one(p[x], p[2 + x], x == 0, "int8", page, table, starts, of, n)

        def attention(q, p, table, lens, q_lens=None, **kw):
            rows.append(np.full(3, q.shape[1]) if q_lens is None else np.asarray(q_lens))
            return q, None

        x = r.randn(3, 1, kv, dh).astype(np.float32)
        exec(code, dict(resize=resize, append=append, attention=attention, norm_rope=lambda q, k, *a, **kw: (q, k),
                        reorder=lambda *a: None, table=table, lens=lens.view(Lens), refs=refs, pool=pool, layers=layers, page=page,
                        n=1, q=x, k=x, v=x, positions=None, parents=None))
        assert lens.tolist() == [5 + free, 5, 8]
        assert [n.tolist() for n in rows] == [[free, 0, 1]] * layers
        for p, before in zip(pool, shared):
            for y, b in zip(p, before):
                assert np.array_equal(y[1], b), "a shared page changed"
