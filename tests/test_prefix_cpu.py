"""Refusals of the prefix-cache operators (include/jpi_prefix.h) that need no GPU: every check is made on the host,
before anything is enqueued, so no pointer here is ever used."""
import ctypes

import pytest

from paper_2607_12659_amd import jpi as j

FAKE = 0x10000


def view(data=FAKE, outer=0, row=256, head=256):
    return j.jpi_view(data, outer, row, head)


def rope_call(q=None, k=None, k_out=None, dtype=j.JPI_BF16, batch=1, tokens=4, heads=2, k_heads=0, pos_stride=0, q_out=None, **kw):
    cfg = dict(head_dim=64, rot_dim=64, layout=0, scaling=0, inverse=0, base=1e4, factor=1.0, trained=0.0, beta_fast=32.0,
               beta_slow=1.0, amplitude=1.0)
    cfg.update(kw)
    return j.jpi_rope(j.jpi_rope_config(**cfg), dtype, batch, tokens, None, pos_stride, q or view(), q_out or view(2 * FAKE), heads,
                      k, k_out, k_heads)


@pytest.mark.parametrize("bad", [dict(head_dim=0), dict(head_dim=65), dict(head_dim=514), dict(rot_dim=0), dict(rot_dim=7),
                                 dict(rot_dim=66), dict(layout=2), dict(scaling=4), dict(scaling=-1), dict(base=1.0),
                                 dict(base=float("nan")), dict(amplitude=float("inf")), dict(scaling=1, factor=0.5),
                                 dict(scaling=2, factor=2.0, rot_dim=2), dict(scaling=3, factor=2.0),
                                 dict(scaling=3, factor=2.0, trained=4096.0, beta_fast=1.0), dict(batch=-1), dict(tokens=-1),
                                 dict(pos_stride=-1), dict(heads=0), dict(k=view(), k_out=view(), k_heads=0), dict(k=view()),
                                 dict(q=view(None)), dict(q_out=view(None)), dict(q=view(row=-1)),
                                 dict(q=view(), q_out=view(row=512))])
def test_rope_refuses(bad):
    assert rope_call(**bad) == j.JPI_ERR_ARG
    assert j.jpi_prefix_last_error().startswith("jpi_rope: ")


def test_rope_refuses_types_and_sizes():
    assert rope_call(dtype=2) == j.JPI_ERR_DTYPE
    assert rope_call(batch=1 << 16, tokens=1 << 15) == j.JPI_ERR_SHAPE
    assert j._lib.jpi_rope(None, 1, 1, 1, None, 0, None, None, 1, None, None, 0, None) == j.JPI_ERR_ARG


def test_rope_of_nothing_is_no_call():
    assert rope_call(tokens=0, q=view(None), q_out=view(None)) == j.JPI_OK


def attn_args(**kw):
    a = j.jpi_shared_attn(j.JPI_BF16, 2, 3, 5, 8, 1, 64, 100, 7, 0, 0.125)
    for n in ("q", "k_prefix", "v_prefix", "k_suffix", "v_suffix", "out"):
        setattr(a, n, view())
    for n, v in kw.items():
        setattr(a, n, v)
    return a


@pytest.mark.parametrize("bad", [dict(n_groups=0), dict(group=0), dict(q_rows=0), dict(n_heads=0), dict(n_kv_heads=0),
                                 dict(n_kv_heads=3), dict(head_dim=96), dict(prefix=-1), dict(suffix=-1), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=float("nan")), dict(q=view(None)), dict(out=view(None)),
                                 dict(k_prefix=view(None)), dict(v_prefix=view(None)), dict(k_suffix=view(None)),
                                 dict(v_suffix=view(None)), dict(q=view(FAKE + 8)), dict(out=view(row=-8)),
                                 dict(k_prefix=view(row=12)), dict(v_suffix=view(head=4)), dict(k_prefix=view(row=(1 << 24) + 8)),
                                 dict(k_suffix=view(row=1 << 25))])
def test_shared_attention_refuses(bad):
    a = attn_args(**bad)
    assert j.jpi_shared_attention(a, FAKE, 1 << 40) == j.JPI_ERR_ARG
    assert j.jpi_prefix_last_error().startswith("jpi_shared_attention: ")


def test_shared_attention_refuses_types_and_sizes():
    assert j.jpi_shared_attention(attn_args(dtype=2)) == j.JPI_ERR_DTYPE
    assert j.jpi_shared_attention(attn_args(group=1 << 27)) == j.JPI_ERR_SHAPE
    assert j.jpi_shared_attention(attn_args(prefix=1 << 28)) == j.JPI_ERR_SHAPE
    assert j._lib.jpi_shared_attention(None, None, 0, None) == j.JPI_ERR_ARG
    assert j._lib.jpi_shared_attention_workspace(None, None) == j.JPI_ERR_ARG
    st, n = j.jpi_shared_attention_workspace(attn_args(head_dim=32))
    assert st == j.JPI_ERR_ARG and n == 0


def test_workspaces_are_checked():
    a = attn_args(prefix=5000, lse=FAKE)
    st, n = j.jpi_shared_attention_workspace(a)
    assert st == j.JPI_OK and n > 0
    assert j.jpi_shared_attention(a) == j.JPI_ERR_ARG and "workspace" in j.jpi_prefix_last_error()
    assert j.jpi_shared_attention(a, FAKE, n - 1) == j.JPI_ERR_ARG
    assert j.jpi_shared_attention(a, FAKE + 4, n) == j.JPI_ERR_ARG
    a = attn_args(n_groups=1, prefix=100, group=400, lse=FAKE)
    st, n = j.jpi_prefix_weight_workspace(a)
    assert st == j.JPI_OK and n > 0
    assert j.jpi_prefix_weight(a, None, 1.0, FAKE) == j.JPI_ERR_ARG and "workspace" in j.jpi_prefix_last_error()
    assert j.jpi_prefix_weight(a, None, 1.0, FAKE, FAKE, n - 1) == j.JPI_ERR_ARG


@pytest.mark.parametrize("bad", [dict(lse=None), dict(q=view(None)), dict(k_prefix=view(None)), dict(scale=0.0)])
def test_prefix_weight_refuses(bad):
    a = attn_args(**{"lse": FAKE, **bad})
    assert j.jpi_prefix_weight(a, None, 1.0, FAKE, FAKE, 1 << 40) == j.JPI_ERR_ARG
    assert j.jpi_prefix_last_error().startswith("jpi_prefix_weight: ")


def test_prefix_weight_refuses_decay_and_output():
    a = attn_args(lse=FAKE)
    assert j.jpi_prefix_weight(a, None, float("nan"), FAKE, FAKE, 1 << 40) == j.JPI_ERR_ARG
    assert j.jpi_prefix_weight(a, None, 1.0, None, FAKE, 1 << 40) == j.JPI_ERR_ARG
    assert j.jpi_prefix_weight(attn_args(prefix=0), None, 1.0, None) == j.JPI_OK  # no slots: nothing to do


def evict_args(**kw):
    a = j.jpi_evict_args(j.JPI_BF16, 2, 1, 64, 100, 40, 4, 8, FAKE, 100)
    a.k, a.v, a.k_out, a.v_out = view(), view(2 * FAKE), view(3 * FAKE), view(4 * FAKE)
    a.index = FAKE
    for n, v in kw.items():
        setattr(a, n, v)
    return a


@pytest.mark.parametrize("bad", [dict(n_outer=-1), dict(n_heads=0), dict(head_dim=0), dict(head_dim=4097), dict(slots=-1),
                                 dict(keep=0), dict(n_first=-1), dict(n_last=-1), dict(n_first=30, n_last=11),
                                 dict(n_first=2 ** 31 - 1, n_last=2 ** 31 - 1), dict(weight=None), dict(index=None),
                                 dict(weight_stride=99), dict(weight_out=FAKE + 64, weight_out_stride=39),
                                 dict(weight_out=FAKE, weight_out_stride=101), dict(k=view(None)), dict(v_out=view(None)),
                                 dict(k=view(row=-1)), dict(k_out=view(row=512))])
def test_evict_refuses(bad):
    assert j.jpi_evict(evict_args(**bad)) == j.JPI_ERR_ARG
    assert j.jpi_prefix_last_error().startswith("jpi_evict: ")


def test_evict_refuses_types_and_sizes():
    assert j.jpi_evict(evict_args(dtype=3)) == j.JPI_ERR_DTYPE
    assert j.jpi_evict(evict_args(slots=(1 << 26) + 1, weight_stride=1 << 27)) == j.JPI_ERR_SHAPE
    assert j.jpi_evict(evict_args(n_outer=1 << 20, n_heads=17)) == j.JPI_ERR_SHAPE
    assert j._lib.jpi_evict(None, None) == j.JPI_ERR_ARG
    assert j.jpi_evict(evict_args(n_outer=0, weight=None)) == j.JPI_OK


def test_structures_have_the_headers_sizes():
    """Field by field the header's types: 8-byte members aligned, ints of 4 bytes."""
    assert ctypes.sizeof(j.jpi_view) == 32
    assert ctypes.sizeof(j.jpi_rope_config) == 24 + 6 * 8
    assert ctypes.sizeof(j.jpi_shared_attn) == 48 + 5 * 32 + 16 + 32 + 8
    assert ctypes.sizeof(j.jpi_evict_args) == 32 + 24 + 4 * 32 + 32


def test_tensors_on_the_cpu_are_refused():
    torch = pytest.importorskip("torch")
    from paper_2607_12659_amd import prefix_ops as ops
    q = torch.zeros(2, 3, 4, 64)
    with pytest.raises(ValueError, match="GPU"):
        ops.rope(q)
    with pytest.raises(ValueError, match="GPU"):
        ops.shared_attention(q, q[:1], q[:1])
    with pytest.raises(ValueError, match="GPU"):
        ops.evict(q, q.clone(), torch.zeros(2, 4, 3), 2)
    with pytest.raises(TypeError):
        ops.rope(q.half())
    with pytest.raises(ValueError, match="shape"):
        ops.rope(q, torch.zeros(2, 3, 4, 32))
    with pytest.raises(ValueError, match="multiple"):
        ops.shared_attention(torch.zeros(3, 1, 4, 64), q, q)
    with pytest.raises(ValueError, match="layout"):
        ops.rope(q, layout="other")
    with pytest.raises(ValueError, match="contiguous"):
        ops.rope(torch.zeros(2, 3, 4, 128)[..., ::2])


def test_shared_attention_refuses_more_than_a_launch_holds_and_overlap():
    assert j.jpi_shared_attention(attn_args(n_groups=(1 << 22) + 1, group=1, q_rows=1, prefix=1)) == j.JPI_ERR_SHAPE
    assert j.jpi_shared_attention(attn_args(n_groups=17, prefix=1 << 26)) == j.JPI_ERR_SHAPE
    a = attn_args(prefix=0, suffix=0, q=view(2 * FAKE), out=view(2 * FAKE))
    assert j.jpi_shared_attention(a, FAKE, 1 << 40) == j.JPI_ERR_ARG and "may not be an input" in j.jpi_prefix_last_error()


@pytest.mark.parametrize("of_weight,sizes", [
    (False, dict(dtype=j.JPI_F32, n_groups=1, group=(1 << 22) + 1, q_rows=1, n_heads=1, prefix=1 << 27, suffix=0)),  # the join
    (False, dict(dtype=j.JPI_F32, n_groups=(1 << 21) + 1, group=5, q_rows=1, n_heads=1, head_dim=256, prefix=1, suffix=1 << 27)),
    (True, dict(n_groups=1, group=1 << 13, q_rows=1, n_heads=8, n_kv_heads=8, prefix=1 << 27, suffix=0)),            # slots x rows
])
def test_calls_that_no_launch_holds_are_refused_before_anything_is_enqueued(of_weight, sizes):
    """Sizes that pass every limit by themselves, but make 2^32 threads or more."""
    a = attn_args(lse=FAKE, **sizes)
    if of_weight:
        assert j.jpi_prefix_weight_workspace(a) == (j.JPI_ERR_SHAPE, 0)
        assert j.jpi_prefix_weight(a, None, 1.0, FAKE, FAKE, 1 << 50) == j.JPI_ERR_SHAPE
    else:
        assert j.jpi_shared_attention_workspace(a) == (j.JPI_ERR_SHAPE, 0)
        assert j.jpi_shared_attention(a, FAKE, 1 << 50) == j.JPI_ERR_SHAPE
    assert "workgroups" in j.jpi_prefix_last_error()


def test_strides_in_place_count_where_there_are_several():
    """Two kept slots in place want the inputs' row stride, two sequences their weights' stride."""
    def call(most, n_outer=1, outer=0):
        a = evict_args(n_outer=n_outer, slots=100, keep=most, n_first=0, n_last=0, weight_out=FAKE, weight_out_stride=50)
        a.k = j.jpi_view(FAKE, 25600, 256, 256)
        a.k_out = j.jpi_view(FAKE, outer, 0, 0)
        return j.jpi_evict(a), j.jpi_prefix_last_error()
    assert call(2)[0] == j.JPI_ERR_ARG and "same strides" in call(2)[1]
    assert call(1, n_outer=2, outer=25600)[0] == j.JPI_ERR_ARG and "same stride" in call(1, n_outer=2, outer=25600)[1]


def test_tensors_that_want_gradients_are_refused():
    torch = pytest.importorskip("torch")
    from paper_2607_12659_amd import prefix_ops as ops
    q, lse = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 4)
    w, leaf = torch.zeros(2, 4, 3), torch.zeros(2, 3, 4, 64, requires_grad=True)
    calls = [lambda t: ops.rope(t), lambda t: ops.rope(q, t), lambda t: ops.rope(q, q_out=t),
             lambda t: ops.shared_attention(t, q, q), lambda t: ops.shared_attention(q, q, t),
             lambda t: ops.shared_attention(q, q, q, q, t), lambda t: ops.prefix_weight(q, t, lse),
             lambda t: ops.evict(q, t, w, 2), lambda t: ops.evict(t, q, w, 2)]
    for call in calls:
        with pytest.raises(ValueError, match="gradients"):
            call(leaf)
        for off in (torch.no_grad, torch.inference_mode):  # taken, up to the next check
            with off(), pytest.raises(ValueError, match="GPU"):
                call(leaf)
        with pytest.raises(ValueError, match="GPU"):
            call(leaf.detach())


def test_sizes_past_c_ints_and_numbers_that_are_none_are_refused():
    """2^32 + 5 tokens are not five of them; what does not fit the C structures raises what the module documents."""
    torch = pytest.importorskip("torch")
    from paper_2607_12659_amd import prefix_ops as ops
    many = torch.zeros(1, 1, 1, 2).expand(1, 2 ** 32 + 5, 1, 2)
    for x in (many, many.transpose(0, 1), many.transpose(1, 2)):
        with pytest.raises(ValueError, match="2\\^31"):
            ops.rope(x, q_out=x)
    few = torch.zeros(1, 1, 1, 2)
    with pytest.raises(ValueError, match="2\\^31"):
        ops.rope(few, many.transpose(1, 2), k_out=many.transpose(1, 2))
    q, w = torch.zeros(2, 3, 4, 64), torch.zeros(2, 4, 3)
    with pytest.raises(ValueError, match="2\\^31"):
        ops.evict(q, q.clone(), w, 2 ** 40)
    for call in (lambda: ops.rope(q, rot_dim=2.5), lambda: ops.rope(q, base="ten"), lambda: ops.rope(q, rot_dim=2 ** 31),
                 lambda: ops.rope(q, factor=10 ** 400), lambda: ops.shared_attention(q, q, q, scale="one"),
                 lambda: ops.evict(q, q.clone(), w, 2, n_first=2 ** 31), lambda: ops.evict(q, q.clone(), w, 2, n_last=0.5),
                 lambda: ops.prefix_weight(q, q, torch.zeros(2, 3, 4), decay="half")):
        with pytest.raises(ValueError, match="range|could not convert"):
            call()


def test_numbers_that_are_infinite_in_fp32_are_refused():
    """An amplitude past fp32, and a scale whose scores in powers of two would be 0 * inf."""
    assert rope_call(amplitude=1e39) == j.JPI_ERR_ARG and rope_call(amplitude=-1e300) == j.JPI_ERR_ARG
    for call in (lambda a: j.jpi_shared_attention(a, FAKE, 1 << 40), lambda a: j.jpi_prefix_weight(a, None, 1.0, FAKE, FAKE, 1 << 40)):
        assert call(attn_args(lse=FAKE, scale=3e38)) == j.JPI_ERR_ARG
        assert "scale" in j.jpi_prefix_last_error()


def test_outputs_that_overlap_at_first_sight_are_refused():
    """Outputs at each other's address or at the other tensor's, and outputs whose elements are one."""
    at = [view(i * FAKE, outer=1024) for i in range(1, 5)]
    for q_out, k_out in ((at[2], at[2]), (at[1], at[2]), (at[2], at[0]), (at[1], at[0])):
        assert rope_call(q=at[0], k=at[1], q_out=q_out, k_out=k_out, k_heads=2) == j.JPI_ERR_ARG
        assert "another tensor" in j.jpi_prefix_last_error()
        assert j.jpi_evict(evict_args(k=at[0], v=at[1], k_out=q_out, v_out=k_out)) == j.JPI_ERR_ARG
        assert "another tensor" in j.jpi_prefix_last_error()
    for fold in (dict(outer=0), dict(outer=1024, row=0), dict(outer=1024, head=0)):
        out = view(3 * FAKE, **fold)
        assert rope_call(q=at[0], q_out=out, batch=2) == j.JPI_ERR_ARG and "stride of 0" in j.jpi_prefix_last_error()
        assert rope_call(q=out, q_out=out, batch=2) == j.JPI_ERR_ARG and "stride of 0" in j.jpi_prefix_last_error()
        a = attn_args(out=out, lse=FAKE)
        assert j.jpi_shared_attention(a, FAKE, 1 << 40) == j.JPI_ERR_ARG and "stride of 0" in j.jpi_prefix_last_error()
        a = evict_args(n_heads=2, k=at[0], v=at[1], k_out=out, v_out=at[3])
        assert j.jpi_evict(a) == j.JPI_ERR_ARG and "stride of 0" in j.jpi_prefix_last_error()


def test_the_plan_of_a_call():
    a = attn_args(prefix=5000)
    st, waves, tiles, ranges = j.jpi_debug_prefix_plan(a, 0)
    assert st == j.JPI_OK and waves in (1, 2, 4) and tiles == -(-3 * 5 * 8 // (32 * waves)) and ranges > 1
    _, n = j.jpi_shared_attention_workspace(a)
    assert n == ranges * 2 * 3 * 5 * 8 * (64 * 4 + 8)  # a sum and two statistics of each row in each range
    st, waves, tiles, ranges = j.jpi_debug_prefix_plan(a, 1)
    assert st == j.JPI_OK and waves == 4 and tiles == -(-5000 // 256)
    assert j._lib.jpi_debug_prefix_plan(ctypes.byref(a), 0, None, None, None) == j.JPI_ERR_ARG
    assert j.jpi_debug_prefix_plan(attn_args(head_dim=32), 0)[0] == j.JPI_ERR_ARG
