"""The operators of a paged 8-bit cache (include/jpi_cache.h) against plain implementations in 64 bits on the CPU.

Codes, scales, tables and counts have to be equal.  Tolerances of the others come from the formats: h is half a step of the
output type relative to the value (bf16 2^-8, fp32 2^-24), u = 2^-24 a rounding in fp32.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
TYPES = [torch.bfloat16, torch.float32]
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
INF = float("inf")


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_12659_amd import cache_ops
    return cache_ops


def rand(seed, *shape, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype)


def dev(t):
    return None if t is None else t.cuda() if torch.is_tensor(t) else torch.from_numpy(np.ascontiguousarray(t)).cuda()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def within(got, want, tol):
    """Every element within its own tolerance; non-finite ones equal."""
    got, want = got.double().cpu(), torch.as_tensor(want, dtype=torch.float64)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fin)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)])
    tol = torch.as_tensor(tol, dtype=torch.float64).expand_as(want)
    over = ((got - want).abs() - tol)[fin]
    assert over.numel() == 0 or over.max() <= 0, "off by %g past the tolerance" % over.max()


# ---------------------------------------------------------------------------
# norms with rotation
# ---------------------------------------------------------------------------
def norm64(x, w, offset, eps, pos, rot, layout="half", base=1e4, scaling="none", factor=1.0, trained=0, beta_fast=32.0, beta_slow=1.0,
           amplitude=1.0, inverse=False):
    """The result, and the size of each element's pair, the scale of its errors."""
    x = x.double()
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * (w.double() + offset)
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    f = torch.tensor([base ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        keep = ((trained * f / (2 * math.pi) - beta_slow) / (beta_fast - beta_slow)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    ang = pos.double()[..., None, None] * f * (-1 if inverse else 1)
    c, s = amplitude * torch.cos(ang), amplitude * torch.sin(ang)
    out, size = y.clone(), y.abs()
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = y[..., lo], y[..., hi]
    out[..., lo], out[..., hi] = a * c - b * s, a * s + b * c
    size[..., lo] = size[..., hi] = amplitude * (a.abs() + b.abs())
    return out, size


def norm_close(got, x, w, offset, eps, pos, rot, **kw):
    """Squares are summed in fp32: D / 2 u of the factor at most (it is a root), and a few u for the mean, the root, the
    division and the products; the rotation as jpi_rope's (8 u of the pair's size); then the output's rounding."""
    want, size = norm64(x, w, offset, eps, pos, rot, **kw)
    within(got, want, H[x.dtype] * want.abs() + (x.shape[-1] / 2 + 16) * U * size * 1.01)


NORM = [
    # batch, tokens, heads, kv heads, head dim, rot, weights (0 none, 1 shared, 2 of each head), offset, what else
    (1, 1, 8, 1, 256, 256, 1, 1, {}),
    (2, 7, 3, 2, 64, 32, 1, 0, dict(layout="interleaved")),
    (3, 1030, 2, 0, 128, 128, 2, 0, dict(scaling="linear", factor=4.0)),
    (2, 513, 4, 1, 64, 64, 2, 1, dict(layout="interleaved", scaling="base", factor=8.0)),
    (1, 90, 2, 1, 128, 64, 0, 0, dict(scaling="parts", factor=5.5, trained=4096, amplitude=1.125)),
    (2, 5, 3, 1, 10, 6, 1, 0, {}),                           # pieces of single elements
    (2, 5, 3, 1, 10, 6, 2, 1, dict(layout="interleaved")),
    (2, 3, 2, 1, 512, 2, 1, 0, {}),                          # nearly all of it passes by, element by element
    (1, 3, 1, 1, 512, 512, 1, 0, dict(inverse=True, amplitude=0.5)),
    (1, 3, 1, 1, 512, 512, 0, 1, dict(layout="interleaved")),
    (1, 3, 2, 1, 2, 2, 1, 0, dict(base=500.0)),
    (1, 2, 3, 3, 96, 48, 1, 0, {}),                          # a head that is no power of two
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("wtype", TYPES)
@pytest.mark.parametrize("case", NORM, ids=lambda c: "b%d-n%d-h%d+%d-d%d-r%d-w%d%d" % c[:8])
def test_norm_rope(ops, case, dtype, wtype):
    b, n, heads, kv, dh, rot, kind, offset, kw = case
    q, k = 3 * rand(1, b, n, heads, dh), 3 * rand(2, b, n, kv, dh) if kv else None
    q, k = q.to(dtype), None if k is None else k.to(dtype)
    shape = lambda h: () if kind == 0 else (dh,) if kind == 1 else (h, dh)  # noqa: E731
    qw = (1 - offset + 0.3 * rand(3, *shape(heads))).to(wtype) if kind else None
    kw_ = (1 - offset + 0.3 * rand(4, *shape(kv))).to(wtype) if kind and kv else None
    pos = torch.randint(0, 1 << 20, (b, n), generator=torch.Generator().manual_seed(3)).int()
    qo, ko = ops.norm_rope(dev(q), dev(k), dev(pos), q_weight=dev(qw), k_weight=dev(kw_), unit_offset=bool(offset), eps=1e-3,
                           rot_dim=rot, **kw)
    norm_close(qo, q, qw, offset, 1e-3, pos, rot, **kw)
    if kv:
        norm_close(ko, k, kw_, offset, 1e-3, pos, rot, **kw)
    else:
        assert ko is None


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_rope_positions_strides_and_in_place(ops, dtype):
    # q and k as slices of one projection whose rows start off 16-byte boundaries, k_out a longer tensor's middle
    b, n, dh = 2, 9, 64
    both = rand(5, b, n, 6, dh + 3, dtype=dtype)
    d = dev(both)
    q, k = d[:, :, :4, :dh], d[:, :, 4:, :dh]
    longer = torch.full((b, 20, 2, dh), 7.0, dtype=dtype, device="cuda")
    w = rand(6, dh)
    pos = torch.tensor([3, -5, 0, 100000, 2, 2, 1 << 24, -(1 << 24), 8]).int()
    qo, ko = ops.norm_rope(q, k, dev(pos), q_weight=dev(w), q_out=q, k_out=longer[:, 5:14])  # k: the norm alone
    assert qo is q
    norm_close(qo, both[:, :, :4, :dh], w, 0, 1e-6, pos.expand(b, n), dh)
    norm_close(ko, both[:, :, 4:, :dh], None, 0, 1e-6, pos.expand(b, n), dh)
    assert torch.equal(d[:, :, 4:].cpu(), both[:, :, 4:]) and torch.equal(d[..., dh:].cpu(), both[..., dh:])
    assert (longer[:, :5] == 7).all() and (longer[:, 14:] == 7).all()
    # weights of each head of k alone; consecutive positions; one head read by all (stride 0)
    x, one, kw = rand(7, 2, 5, 2, dh, dtype=dtype), rand(8, 2, 5, 1, dh, dtype=dtype), rand(9, 3, dh)
    qo, ko = ops.norm_rope(dev(x), dev(one).expand(2, 5, 3, dh), k_weight=dev(kw), unit_offset=True)
    at = torch.arange(5).expand(2, 5)
    norm_close(qo, x, None, 0, 1e-6, at, dh)
    norm_close(ko, one.expand(2, 5, 3, dh), kw, 1, 1e-6, at, dh)


def test_norm_rope_zero_and_spoilt_heads(ops):
    """A head of zeros stays zero; NaN and infinity spoil their own head only."""
    x = rand(10, 1, 6, 2, 64)
    x[0, 1, 0], x[0, 2, 1, 5], x[0, 3, 0, 7] = 0, float("nan"), INF
    got = ops.norm_rope(dev(x))[0].cpu()
    want, _ = norm64(x, None, 0, 1e-6, torch.arange(6)[None], 64)
    assert torch.equal(got[0, 1, 0], torch.zeros(64)) and torch.isnan(got[0, 2, 1]).any() and torch.isnan(got[0, 3, 0]).any()
    fine = torch.ones(1, 6, 2, dtype=torch.bool)
    fine[0, 2, 1] = fine[0, 3, 0] = False
    within(got[fine], want[fine], (32 + 16) * U * 8)


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
def filled(seed, n_pages, kv, dh, page, code, scales=True):
    """A pool of coded normal values as numpy: (k bytes, v bytes, k scales, v scales)."""
    r = np.random.RandomState(seed)
    out = []
    for shape in ((dh // 16, page, 16), (page // 16, dh, 16)):
        x = r.randn(n_pages, kv, *shape).astype(np.float32) * np.exp(0.7 * r.randn(n_pages, kv, 1, 1, 1)).astype(np.float32)
        s = np.array([[ref.scale_for(float(np.abs(x[p, h]).max()), code) for h in range(kv)] for p in range(n_pages)], np.float32)
        out.append((ref.encode(x / s[..., None, None, None], code), s))
    return [out[0][0], out[1][0], out[0][1], out[1][1]]


def on_gpu(ops, pool, code):
    return ops.Pool(dev(pool[0]).view(CODES[code]), dev(pool[1]).view(CODES[code]), dev(pool[2]), dev(pool[3]))


def same_pool(got, want):
    for g, w, name in zip(got, want, ("k", "v", "k_scale", "v_scale")):
        g = g.cpu()
        g = g.numpy() if g.dtype == torch.float32 else g.view(torch.uint8).numpy()
        if g.dtype == np.float32:
            np.testing.assert_array_equal(g, w, err_msg=name)  # NaN equals NaN
        else:
            assert np.array_equal(g, w), "%s: %d of %d bytes differ" % (name, (g != w).sum(), g.size)


def numbered(seed, counts, width, n_pages):
    """A table whose rows take shuffled page numbers, garbage behind them."""
    order = np.random.RandomState(seed).permutation(n_pages)
    table, at = np.full((len(counts), width), -7, np.int32), 0
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    assert at <= n_pages
    return table


def append_both(ops, pool, code, page, table, starts, k, v, n_new=None):
    """Append on the GPU and in numpy, and compare; the pool in numpy changes."""
    n = np.full(len(starts), k.shape[1]) if n_new is None else np.asarray(n_new)
    d = on_gpu(ops, pool, code)
    ops.append(d, dev(table), i32(starts), dev(k), dev(v), n_new=None if n_new is None else i32(n_new))
    for i, x in ((0, k), (1, v)):
        ref.append_one(pool[i], pool[2 + i], i == 0, code, page, table, starts, x.float().numpy(), n)
    same_pool(d, pool)
    return d


APPEND = [
    # sequences' slots before, tokens, tokens that are new (None: all), kv heads, dim, page
    ([0], 1, None, 1, 64, 16),
    ([0, 15, 16, 17, 31], 1, None, 2, 64, 16),
    ([5, 0, 90, 63, 64], 70, [70, 0, 1, 33, 69], 2, 128, 64),
    ([1, 127, 128, 300], 260, [260, 1, 129, 0], 1, 256, 128),
    ([0, 3], 816, [816, 500], 1, 256, 32),
    ([7, 8, 9], 3, None, 8, 128, 16),
    ([40], 1000, [2000], 1, 64, 128),      # more than there are: all
    ([-3, 2], 5, [-1, 5], 1, 64, 16),      # lengths and counts below 0: 0
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(ops, case, code, dtype):
    starts, tokens, n_new, kv, dh, page = APPEND[case]
    n = [tokens] * len(starts) if n_new is None else n_new
    counts = [-(-(max(s, 0) + min(max(t, 0), tokens)) // page) for s, t in zip(starts, n)]
    n_pages = sum(counts) + 2
    pool = filled(case, n_pages, kv, dh, page, code)
    table = numbered(case, counts, max(counts) + 1, n_pages)
    k = rand(20 + case, len(starts), tokens, kv, dh) * torch.exp(0.8 * rand(30 + case, len(starts), tokens, 1, 1))
    v = rand(40 + case, len(starts), tokens, kv, dh) * torch.exp(0.8 * rand(50 + case, len(starts), tokens, 1, 1))
    append_both(ops, pool, code, page, table, starts, k.to(dtype), v.to(dtype), n_new)


@pytest.mark.parametrize("code", CODES)
def test_append_token_by_token(ops, code):
    """Scales that grow again and again, and values that fall on ties and on the largest code."""
    kv, dh, page = 1, 64, 16
    pool = filled(3, 4, kv, dh, page, code)
    table = numbered(3, [3], 3, 4)
    top = ref.TOP[code]
    for t in range(40):
        x = rand(100 + t, 1, 1, kv, dh) * 1.3 ** t
        if t % 4 == 1:
            x = torch.round(x * 4) / 8  # halves: ties of int8
        if t % 4 == 2:
            x[..., 0] = top * 2.0 ** (t // 4)  # the largest code exactly
        if t % 4 == 3:
            x[..., 0] = top * 2.0 ** (t // 4) * (1 + 2.0 ** -22)  # just above it
        append_both(ops, pool, code, page, table, [t], x, -x)


@pytest.mark.parametrize("code", CODES)
def test_append_odd_values(ops, code):
    """Zeros, subnormals, the largest numbers, NaN and infinities, and scales that no append would have set."""
    kv, dh, page = 2, 64, 16
    pool = filled(4, 12, kv, dh, page, code)
    table = numbered(4, [1] * 12, 2, 12)
    pool[2][table[8, 0]], pool[2][table[9, 0]], pool[3][table[9, 0]] = 0.0, 0.3, 0.01
    pool[2][table[10, 0], 0] = np.nan
    k, v = rand(60, 12, 2, kv, dh), rand(61, 12, 2, kv, dh)
    k[0], v[0] = 0, 0
    k[1] *= 2.0 ** -130
    v[1] *= 2.0 ** -148
    k[2] *= 2.0 ** 124
    k[3, 1, 0, 5], v[3, 0, 1, 6] = float("nan"), INF
    k[4, 0, 1, 0], v[4, 0, 0, 0] = -INF, -float("nan")
    k[5] = 3.3e38
    k[6], v[7] = -3.4e38, 1.5e-45
    k[8] = 0
    starts = [0, 0, 0, 0, 3, 2, 3, 0, 4, 4, 4, 14]
    append_both(ops, pool, code, page, table, starts, k, v)
    # what was spoilt stays so, until the page is begun anew
    append_both(ops, pool, code, page, table, [2, 2, 2, 2, 5, 4, 5, 2, 6, 6, 6, 15], rand(62, 12, 1, kv, dh), rand(63, 12, 1, kv, dh))
    append_both(ops, pool, code, page, table, [0] * 12, rand(64, 12, 16, kv, dh), rand(65, 12, 16, kv, dh))
    assert np.isfinite(pool[2]).all() and np.isfinite(pool[3]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_append_strides_and_numbers_that_name_no_page(ops, dtype):
    kv, dh, page, code = 2, 128, 32, "e4m3"
    pool = filled(5, 9, kv, dh, page, code)
    table = numbered(5, [3, 3, 3], 3, 9)
    table[0, 1], table[1, 0], table[2, 2] = -1, 9, 1 << 30
    qkv = rand(66, 3, 100, 4 * kv, dh + 1, dtype=dtype)  # rows off 16-byte boundaries
    k, v = qkv[:, :, kv:2 * kv, :dh], qkv[:, :, 2 * kv:3 * kv, 1:]
    before = [x.copy() for x in pool]
    d = on_gpu(ops, pool, code)
    g = dev(qkv)
    ops.append(d, dev(np.hstack([table, table]))[:, :3], i32([0, 10, 20]), g[:, :, kv:2 * kv, :dh], g[:, :, 2 * kv:3 * kv, 1:])
    for i, x in ((0, k), (1, v)):  # tokens past the table's three pages are dropped
        ref.append_one(pool[i], pool[2 + i], i == 0, code, page, table, [0, 10, 20], x.float().numpy(), [100] * 3)
    same_pool(d, pool)
    assert sum((a != b).any() for a, b in zip(pool, before)) == 4
    # a token of all sequences (stride 0 along them), aligned rows
    one = rand(67, 1, 4, kv, dh, dtype=dtype)
    d = on_gpu(ops, pool, code)
    table = numbered(6, [3, 3, 3], 3, 9)
    ops.append(d, dev(table), i32([30, 0, 64]), dev(one).expand(3, 4, kv, dh), dev(one).expand(3, 4, kv, dh))
    for i in (0, 1):
        ref.append_one(pool[i], pool[2 + i], i == 0, code, page, table, [30, 0, 64], one.float().expand(3, 4, kv, dh).numpy(), [4] * 3)
    same_pool(d, pool)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def attn64(q, pool, code, page, table, lens, q_lens, causal, window, sinks, scale):
    """out, lse; per element the sum of p |v|; per row the scale of its scores' errors; rows that exist."""
    S, R, nh, D = q.shape
    kv = pool[2].shape[1]
    q = q.double().numpy()
    out, mag = np.zeros((S, R, nh, D)), np.zeros((S, R, nh, D))
    lse, err, there = np.full((S, R, nh), -INF), np.zeros((S, R, nh)), np.zeros((S, R), bool)
    for s in range(S):
        n, nq = min(max(lens[s], 0), table.shape[1] * page), min(max(q_lens[s], 0), R)
        there[s, :nq] = True
        K, V = (ref.slots(pool[i], pool[2 + i], i == 0, code, page, table[s], n) for i in (0, 1))
        see = ref.seen(n, nq, causal, window, sinks)
        any_row = see.any(1)
        for h in range(nh):
            k, v = K[h // (nh // kv)], V[h // (nh // kv)]
            x = np.where(see, scale * (q[s, :nq, h] @ k.T), -INF)[any_row]
            if not x.size:
                continue
            m = x.max(1, keepdims=True)
            e = np.exp(x - m)
            total = e.sum(1, keepdims=True)
            lse[s, :nq, h][any_row] = (m + np.log(total))[:, 0]
            bad = np.isnan(v).any(1)  # slots that hold NaN: 0 * NaN where they are not seen
            e, v = e / total, np.where(bad[:, None], 0, v)
            spoilt = (see[any_row] & bad).any(1)[:, None]
            out[s, :nq, h][any_row], mag[s, :nq, h][any_row] = np.where(spoilt, np.nan, e @ v), np.where(spoilt, np.nan, e @ np.abs(v))
            err[s, :nq, h][any_row] = scale * np.where(see, np.abs(q[s, :nq, h]) @ np.abs(k).T, 0)[any_row].max(1)
    return out, lse, mag, err, there


def attn_tolerance(dtype, out, lse, mag, err, keys, D):
    """Codes are exact.  Scores: products summed in fp32, D u of the sum of magnitudes (3 D in the parts of fp32 queries, whose
    smaller ones add next to nothing), and 8 u for scale, page scale and reference; exp2, sums and joins (keys + 40) u; the
    probability times the page's scale is rounded to bf16 or to 24 bits in parts; then the output's rounding."""
    ds = ((1 if dtype == torch.bfloat16 else 3) * D + 8) * U * err + 8 * U * (np.nan_to_num(np.abs(lse), posinf=0) + 1)
    soft = 2 * ds + (keys + 40) * U
    p = H[dtype] if dtype == torch.bfloat16 else 4 * U
    return H[dtype] * np.abs(out) + mag * (soft[..., None] + p) * 1.01 + 1e-30, np.where(lse == -INF, 0, soft + 1e-30)


def attend_both(ops, q, pool, code, page, table, lens, q_lens=None, causal=True, window=0, sinks=0, scale=None):
    S, R, nh, D = q.shape
    ql = [R] * S if q_lens is None else q_lens
    marker = -77.0
    out = torch.full(q.shape, marker, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:3], marker, device="cuda")
    got = ops.attention(dev(q), on_gpu(ops, pool, code), dev(table), i32(lens), q_lens=None if q_lens is None else i32(q_lens),
                        causal=causal, window=window, sinks=sinks, scale=scale, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    o, l, mag, err, there = attn64(q, pool, code, page, table, lens, ql, causal, window, sinks, D ** -0.5 if scale is None else scale)
    tol_o, tol_l = attn_tolerance(q.dtype, o, l, mag, err, max([1] + list(lens)), D)
    there = torch.from_numpy(there)
    within(out.cpu()[there], o[there.numpy()], tol_o[there.numpy()])
    within(lse.cpu()[there], l[there.numpy()], tol_l[there.numpy()])
    assert (out.cpu()[~there] == marker).all() and (lse.cpu()[~there] == marker).all()
    return out, lse


def plan_of(n, rows, heads, kv, dh, page, causal, window, sinks, width, code):
    """(groups, tiles, ranges) of a bf16 call."""
    from paper_2607_12659_amd import jpi as j
    a = j.jpi_cache_attn(j.JPI_BF16, rows, heads, int(causal), window, sinks, dh ** -0.5)
    st, *plan = j.jpi_debug_cache_plan(a, j.jpi_cache_pool(getattr(j, "JPI_" + code.upper()), kv, dh, 1, page), j.jpi_cache_seqs(n, width, width))
    assert st == j.JPI_OK
    return plan


ATTN = [
    # rows, heads, kv heads, dim, page, lengths, rows of each (None: all), causal, window, sinks, pages in the table
    (1, 1, 1, 64, 16, [1], None, True, 0, 0, 1),
    (1, 8, 1, 256, 64, [817], None, True, 0, 0, 13),
    (1, 8, 1, 256, 64, [817], None, True, 0, 0, 600),                       # a table for far more
    (1, 32, 8, 128, 64, [300, 1, 0, 129, 64, 65], None, True, 0, 0, 8),
    (5, 8, 1, 64, 16, [3, 5, 17, 100], None, True, 0, 0, 8),                # shorter than its rows
    (7, 4, 2, 64, 16, [333, 113, 223], None, True, 100, 3, 21),
    (7, 4, 2, 128, 32, [333, 0, 7, 223], [7, 3, 0, 1], True, 0, 0, 11),     # ragged rows
    (50, 8, 1, 256, 32, [866, 50, 31], None, False, 0, 0, 28),
    (33, 6, 6, 128, 128, [200, 40], None, True, 1, 0, 2),                   # a window of a row itself
    (33, 6, 3, 64, 16, [200, 40], [20, 33], True, 5, 40, 13),               # more sinks than window
    (65, 3, 1, 128, 64, [65, 300], None, True, 64, 64, 5),
    (2, 16, 1, 64, 32, [5000, 4999, 31], None, True, 1000, 4, 157),
    (1, 5, 5, 128, 16, [2049, 700], None, True, 37, 1, 129),
    (3, 40, 1, 128, 16, [75, 64], None, True, 0, 0, 5),                     # 40 heads: rows of a token in two tiles
    (300, 2, 2, 64, 128, [300], [299], True, 0, 0, 3),
    (1, 4, 4, 256, 128, [9000], None, True, 0, 0, 71),
    # 256 dims, tiles for half of the card: eight waves share out a tile's keys
    (50, 8, 1, 256, 32, [866, 50, 31, 0, 513, 70], [50, 50, 31, 7, 49, 1], False, 0, 0, 28),
    (816, 8, 1, 256, 64, [816], None, True, 0, 0, 13),
    (35, 16, 4, 256, 16, [700, 36, 513, 1], [35, 35, 0, 1], True, 300, 3, 44),
    # tables for so few slots that eight waves need no ranges
    (2, 8, 2, 64, 64, [1024, 513, 1], None, True, 0, 0, 16),
    (9, 4, 4, 128, 32, [500, 0, 31, 544], [9, 9, 3, 0], False, 0, 0, 17),
    (1, 8, 1, 256, 16, [1000, 64, 129], None, True, 500, 2, 64),
]


# many rows: the kernel that passes the keys through LDS
RING = [
    (70, 32, 32, 64, 16, [333, 0, 70, 69, 1, 200, 64, 65], None, True, 0, 0, 21),
    (9, 128, 16, 128, 64, [300, 64, 9, 1, 128, 70, 0, 63] * 2, [9, 0, 9, 4, 1, 8, 9, 3] * 2, True, 0, 0, 5),
    (50, 8, 1, 256, 32, [116] * 28 + [866, 50, 31, 115], None, False, 0, 0, 28),
    (130, 16, 16, 64, 32, [3000, 130, 1100, 131] * 2, [130, 129, 128, 7] * 2, True, 700, 5, 94),
    (100, 32, 32, 128, 128, [2500, 100, 40, 130, 260, 129, 99, 0], None, True, 1, 0, 20),
    (40, 64, 16, 128, 16, [2200, 40, 39, 41, 55, 64, 80, 100, 7, 1], None, True, 33, 70, 138),
    (64, 32, 32, 64, 64, [64, 300, 20, 5, 1, 0, 64, 128], [64, 1, 20, 64, 64, 64, 0, 63], False, 0, 0, 5),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("case", range(len(ATTN) + len(RING)))
def test_attention(ops, case, code, dtype):
    rows, heads, kv, dh, page, lens, q_lens, causal, window, sinks, width = (ATTN + RING)[case]
    if case >= len(ATTN) and dtype == torch.bfloat16:
        assert plan_of(len(lens), rows, heads, kv, dh, page, causal, window, sinks, width, code)[0] > 0
    counts = [-(-n // page) for n in lens]
    n_pages = sum(counts) + 1
    pool = filled(case, n_pages, kv, dh, page, code)
    table = numbered(case, counts, width, n_pages)
    # what lies behind a length may be anything: NaN codes of e4m3 among it
    for s, n in enumerate(lens):
        if n % page:
            for i in (0, 1):
                x = ref.natural(pool[i][table[s, n // page]], i == 0).copy()
                x[:, n % page:] = 0x7f
                pool[i][table[s, n // page]] = ref.in_pieces(x, i == 0)
    q = rand(70 + case, len(lens), rows, heads, dh, dtype=dtype)
    attend_both(ops, q, pool, code, page, table, lens, q_lens, causal, window, sinks)


# few rows whose keys are cut into ranges; the last two entries: waves of a workgroup, and whether they are cut
SPLIT = [
    (1, 32, 8, 128, 64, [4000, 70], None, True, 0, 0, 64, 4, True),
    (5, 16, 2, 128, 16, [1700, 3, 900], [5, 3, 0], True, 1200, 7, 300, 4, True),
    (3, 4, 4, 64, 32, [3000, 64, 1], None, False, 0, 0, 100, 4, True),
    (1, 8, 1, 256, 64, [5000, 817], None, True, 0, 0, 80, 4, True),
    (50, 8, 1, 256, 64, [4000, 50], None, True, 0, 0, 64, 8, True),
    (40, 16, 2, 256, 32, [2000, 700], [40, 33], True, 1500, 3, 64, 8, True),
    (33, 4, 1, 256, 16, [1500, 33, 0, 64], [33, 1, 33, 30], False, 0, 0, 128, 8, True),
    (130, 1, 1, 256, 128, [3000], [129], True, 0, 0, 30, 8, True),
    (2, 8, 1, 256, 64, [300, 65], None, True, 0, 0, 5, 4, False),
]


def waves_of(n, rows, heads, kv, dh, page, causal, window, sinks, width, code, dtype=torch.bfloat16):
    from paper_2607_12659_amd import jpi as j
    a = j.jpi_cache_attn(j.JPI_BF16 if dtype == torch.bfloat16 else j.JPI_F32, rows, heads, int(causal), window, sinks, dh ** -0.5)
    st, waves = j.jpi_debug_cache_waves(a, j.jpi_cache_pool(getattr(j, "JPI_" + code.upper()), kv, dh, 1, page), j.jpi_cache_seqs(n, width, width))
    assert st == j.JPI_OK
    return waves


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("case", range(len(SPLIT)))
def test_attention_ranges_of_few_rows(ops, case, code, dtype):
    rows, heads, kv, dh, page, lens, q_lens, causal, window, sinks, width, waves, cut = SPLIT[case]
    sizes = (len(lens), rows, heads, kv, dh, page, causal, window, sinks, width, code)
    if dtype == torch.bfloat16:
        groups, _, ranges = plan_of(*sizes)
        assert groups == 0 and (ranges > 1) == cut and waves_of(*sizes) == waves
    counts = [-(-n // page) for n in lens]
    pool = filled(30 + case, sum(counts) + 1, kv, dh, page, code)
    table = numbered(30 + case, counts, width, sum(counts) + 1)
    q = rand(130 + case, len(lens), rows, heads, dh, dtype=dtype)
    first = attend_both(ops, q, pool, code, page, table, lens, q_lens, causal, window, sinks)
    same_bits(first, attend_both(ops, q, pool, code, page, table, lens, q_lens, causal, window, sinks))


@pytest.mark.parametrize("code", CODES)
def test_every_form_of_few_rows_is_compared(ops, code):
    """The entries above reach each number of waves of each dim, with ranges and without, that a rule sends calls to: if a limit
    between them moves, their sizes have to move too."""
    reached = set()
    for entry in ATTN + SPLIT:
        rows, heads, kv, dh, page, lens, _, causal, window, sinks, width = entry[:11]
        for dtype in TYPES:
            sizes = (len(lens), rows, heads, kv, dh, page, causal, window, sinks, width, code)
            groups, _, ranges = plan_of(*sizes)
            if dtype == torch.bfloat16 and groups == 0:
                reached.add((dh, waves_of(*sizes), ranges > 1))
            assert dtype == torch.bfloat16 or waves_of(*sizes, dtype) == 4
    assert reached == {(64, 4, False), (64, 4, True), (64, 8, False), (128, 4, False), (128, 4, True), (128, 8, False), (256, 4, False),
                       (256, 4, True), (256, 8, False), (256, 8, True)}


# many rows whose keys are cut into ranges: mostly tables for far more slots than there are; the last entry: 8192 rows and more
RANGES = [
    (100, 4, 1, 64, 128, [1500, 100, 0, 257, 256], None, True, 0, 0, 1400, False),
    (64, 2, 2, 128, 64, [1025, 64, 1, 640], [64, 1, 64, 63], False, 0, 0, 5000, False),
    (200, 16, 16, 128, 16, [2700, 200, 515, 199, 0], [200, 200, 131, 7, 3], True, 0, 0, 550, True),
    (70, 64, 8, 64, 64, [9300, 70], None, True, 9000, 70, 10000, True),           # ranges of a window's keys
    (50, 8, 1, 256, 32, [866, 50, 31, 116, 1100, 0, 600, 64], None, False, 0, 0, 200, False),
    (50, 16, 2, 256, 64, [300, 50, 49, 1] * 3, [50, 49, 50, 0] * 3, True, 0, 0, 64, True),
]


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("case", range(len(RANGES)))
def test_attention_ranges_of_many_rows(ops, case, code):
    rows, heads, kv, dh, page, lens, q_lens, causal, window, sinks, width, large = RANGES[case]
    groups, _, ranges = plan_of(len(lens), rows, heads, kv, dh, page, causal, window, sinks, width, code)
    assert groups > 0 and ranges > 1
    assert large == (len(lens) * kv * groups * 128 >= 8192)
    counts = [-(-n // page) for n in lens]
    pool = filled(40 + case, sum(counts) + 1, kv, dh, page, code)
    table = numbered(40 + case, counts, width, sum(counts) + 1)
    if page > 16 and lens[0] % page:  # codes behind a length
        for i in (0, 1):
            x = ref.natural(pool[i][table[0, lens[0] // page]], i == 0).copy()
            x[:, lens[0] % page:] = 0x7f
            pool[i][table[0, lens[0] // page]] = ref.in_pieces(x, i == 0)
    q = rand(140 + case, len(lens), rows, heads, dh, dtype=torch.bfloat16)
    first = attend_both(ops, q, pool, code, page, table, lens, q_lens, causal, window, sinks)
    same_bits(first, attend_both(ops, q, pool, code, page, table, lens, q_lens, causal, window, sinks))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_spoilt_pages(ops, dtype):
    """A page that holds NaN, and a number that names none, spoil the rows that see them, and no others."""
    kv, dh, page, code = 2, 64, 16, "e4m3"
    lens = [200, 200, 200, 100]
    pool = filled(7, 60, kv, dh, page, code)
    table = numbered(7, [13, 13, 13, 7], 13, 60)
    pool[2][table[0, 3], 1] = np.nan  # K of the second KV head
    pool[3][table[1, 12], 0] = np.nan  # V of the last slots
    table[2, 0] = 60
    table[3, 5] = -1
    q = rand(80, 4, 120, 4, dh, dtype=dtype)
    out, lse = attend_both(ops, q, pool, code, page, table, lens, causal=True, window=20, sinks=2)
    assert torch.isnan(out[0, :, 2:]).any() and not torch.isnan(out[0, :, :2]).any() and not torch.isnan(lse[1]).any()
    assert torch.isnan(out[2]).all()
    attend_both(ops, q[:, :1], pool, code, page, table, lens)
    # the same pages for sixteen times as many heads' rows: through LDS
    many = rand(84, 4, 120, 64, dh, dtype=dtype)
    wide = [np.repeat(x, 16, 1) for x in pool]
    out, lse = attend_both(ops, many, wide, code, page, table, lens, causal=True, window=20, sinks=2)
    assert torch.isnan(out[2]).all() and not torch.isnan(out[0, :, :32]).any()


NO_PAGE_CALLS = [(5, 4, 64, torch.float32), (5, 4, 64, torch.bfloat16), (5, 4, 256, torch.bfloat16), (200, 256, 64, torch.bfloat16),
                 (200, 128, 256, torch.bfloat16)]  # rows, heads, dim, type: few rows of four and eight waves, and many


@pytest.mark.parametrize("number", [-1, -2, -3, -(1 << 31), (1 << 31) - 1, 40])
@pytest.mark.parametrize("case", range(len(NO_PAGE_CALLS)))
def test_attention_takes_any_number_that_names_no_page_for_nan(ops, case, number):
    """Each number outside [0, n_pages), in the middle of what all rows see and in the last page."""
    rows, heads, dh, dtype = NO_PAGE_CALLS[case]
    kv, page, code, lens = heads // 4, 16, "e4m3", [300, 296, 300]
    pool = filled(11, 40, kv, dh, page, code)
    table = numbered(11, [13] * 3, 19, 40)
    table[:, 13:] = table[:, :6]
    table[0, 4], table[1, 18] = number, number
    q = rand(85 + case, 3, rows, heads, dh, dtype=dtype)
    out, _ = attend_both(ops, q, pool, code, page, table, lens)
    assert torch.isnan(out[0]).all() and torch.isnan(out[1, -1]).all() and not torch.isnan(out[2]).any()


@pytest.mark.parametrize("case", range(len(NO_PAGE_CALLS)))
def test_attention_reads_nothing_out_of_pages_that_are_none(ops, case):
    """Entries that name no page, behind a window: rows that do not see them are as without them, whatever free pages hold."""
    rows, heads, dh, dtype = NO_PAGE_CALLS[case]
    kv, page, code, lens, window = heads // 4, 16, "e4m3", [300, 296, 301], 53
    pool = filled(12, 40, kv, dh, page, code)
    table = numbered(12, [13] * 3, 19, 40)
    table[:, 13:] = table[:, :6]
    used = set(table.ravel().tolist())
    free = [p for p in range(40) if p not in used]
    pool[0][free], pool[1][free] = 0x7f, 0x7f  # NaN codes
    order = np.arange(40)  # page 0 is free
    order[[0, free[0]]] = free[0], 0
    pool, table = [x[order] for x in pool], np.argsort(order)[table].astype(np.int32)
    q = rand(86 + case, 3, rows, heads, dh, dtype=dtype)
    attend_both(ops, q, pool, code, page, table, lens, causal=True, window=window)
    # pages that lie before all windows go, those of their tiles of 64 slots among them
    for s, n in enumerate(lens):
        gone = max(0, n - rows - window + 1) // page
        assert gone * page % 64 != 0
        table[s, :gone] = -1
    out, _ = attend_both(ops, q, pool, code, page, table, lens, causal=True, window=window)
    assert torch.isfinite(out).all()
    table[1, 17] = 1 << 20  # among what some rows see
    out, _ = attend_both(ops, q, pool, code, page, table, lens, causal=True, window=window)
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1, -1]).all() and torch.isfinite(out[2]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_spoilt_queries_and_sizes_of_values(ops, dtype):
    """NaN and infinity of a query stay in its row; scales of pages far apart; scores that differ by hundreds."""
    kv, dh, page, code = 1, 128, 32, "int8"
    pool = filled(8, 12, kv, dh, page, code)
    table = numbered(8, [6, 6], 6, 12)
    for i, p in enumerate(table[0]):
        pool[3][p] = 2.0 ** (6 * i - 40)
    for i, p in enumerate(table[1]):
        pool[2][p] *= 2.0 ** (i - 2)
    q = rand(81, 2, 9, 4, dh, dtype=dtype)
    q[1] *= 8
    attend_both(ops, q, pool, code, page, table, [190, 192])
    bad = q.clone()
    bad[0, 3, 1, 7], bad[1, 4, 2, 100] = float("nan"), INF
    args = (on_gpu(ops, pool, code), dev(table), i32([190, 192]))
    good, got = ops.attention(dev(q), *args), ops.attention(dev(bad), *args)
    for g, w in zip(got, good):
        keep = torch.ones(2, 9, 4, dtype=torch.bool)
        keep[0, 3, 1] = keep[1, 4, 2] = False
        assert torch.equal(g.cpu()[keep], w.cpu()[keep]) and torch.isnan(g.cpu()[~keep]).any(-1).all()


MANY = [(9, 4, 1, 64), (70, 64, 32, 64), (70, 32, 4, 256)]  # rows, heads, KV heads, dim: few rows, and many


@pytest.mark.parametrize("case", MANY)
def test_attention_counts_out_of_range_and_a_broadcast_query(ops, case):
    """Lengths and counts of rows outside their ranges count as the nearer end; a query of all heads has a stride of 0."""
    rows, heads, kv, dh = case
    page, width, code = 16, 10, "e4m3"
    lens, q_lens = [-5, 1 << 30, 161, 100, 160, 7, 90, -(1 << 31)], [rows, 1 << 30, rows, -1, rows - 1, 1 << 30, -(1 << 31), 3]
    assert (plan_of(8, rows, heads, kv, dh, page, True, 0, 0, width, code)[0] > 0) == (rows == 70)
    pool = filled(60, 81, kv, dh, page, code)
    table = numbered(60, [10] * 8, width, 81)
    q = rand(160, 8, rows, 1, dh, dtype=torch.bfloat16).expand(8, rows, heads, dh)
    out, lse = torch.full((2, 8, rows, heads, dh), -77.0, dtype=q.dtype, device="cuda"), torch.full((8, rows, heads), -77.0, device="cuda")
    g = dev(q[:, :, :1]).expand(8, rows, heads, dh)
    ops.attention(g, on_gpu(ops, pool, code), dev(table), i32(lens), q_lens=i32(q_lens), out=out[1], lse=lse)
    o, l, mag, err, there = attn64(q, pool, code, page, table, lens, q_lens, True, 0, 0, dh ** -0.5)
    tol_o, tol_l = attn_tolerance(q.dtype, o, l, mag, err, 160, dh)
    within(out[1].cpu()[torch.from_numpy(there)], o[there], tol_o[there])
    within(lse.cpu()[torch.from_numpy(there)], l[there], tol_l[there])
    assert (out[1].cpu()[torch.from_numpy(~there)] == -77).all() and (out[0] == -77).all()
    assert (lse.cpu()[torch.from_numpy(~there)] == -77).all()


@pytest.mark.parametrize("case", MANY[1:])
@pytest.mark.parametrize("code", CODES)
def test_attention_many_rows_spoilt_queries_and_sizes_of_values(ops, case, code):
    """As for few rows: NaN and infinity stay in their rows; scales of pages far apart, and none of a power of two; scores that
    differ by hundreds; scales of 0."""
    rows, heads, kv, dh = case
    page = 32
    pool = filled(61, 50, kv, dh, page, code)
    table = numbered(61, [6] * 8, 6, 50)
    for i in range(6):
        pool[3][table[0, i]] = 2.0 ** (6 * i - 20)
        pool[3][table[1, i]] = 1.3 * 2.0 ** (i - 3)
        pool[2][table[2, i]] *= 2.0 ** (i - 2)
        pool[3][table[4, i]] = 2.0 ** (90 * (i % 2) - 45 + i)
    pool[2][table[3, 2]], pool[3][table[3, 3]], pool[2][table[3, 5]], pool[3][table[3, 5]] = 0, 0, 0, 0
    q = rand(161, 8, rows, heads, dh, dtype=torch.bfloat16)
    q[2] *= 8
    lens = [190, 192, 180, 192, 150, 70, 64, 33]
    assert plan_of(8, rows, heads, kv, dh, page, True, 0, 0, 6, code)[0] > 0
    attend_both(ops, q, pool, code, page, table, lens)
    bad = q.clone()
    bad[0, 3, 1, 7], bad[1, 4, 2, 60] = float("nan"), INF
    args = (on_gpu(ops, pool, code), dev(table), i32(lens))
    good, got = ops.attention(dev(q), *args), ops.attention(dev(bad), *args)
    keep = torch.ones(8, rows, heads, dtype=torch.bool)
    keep[0, 3, 1] = keep[1, 4, 2] = False
    for g, w in zip(got, good):
        assert torch.equal(g.cpu()[keep], w.cpu()[keep]) and torch.isnan(g.cpu()[~keep].reshape(2, -1)).any(-1).all()


# rows, heads, KV heads, dim of eight sequences: few rows in four and in eight waves, and many
PRECISE = [(9, 4, 1, 64), (1, 8, 2, 128), (20, 8, 1, 256), (70, 64, 32, 64), (70, 64, 16, 128), (70, 32, 4, 256)]


@pytest.mark.parametrize("case", range(len(PRECISE)))
@pytest.mark.parametrize("code", CODES)
def test_attention_of_few_slots_is_as_good_as_its_parts(ops, case, code):
    """Two bf16 parts of a probability leave 2^-16 of it (half a step, 2^-8, of the remainder, itself 2^-8 at most), one part
    2^-8.  The output's own half step shrinks with values that cancel, and slots are few, so that one part where there should be
    two shows.  Scores and sums as in attn_tolerance."""
    rows, heads, kv, dh = PRECISE[case]
    page, width, many = 16, 10, rows == 70
    assert (plan_of(8, rows, heads, kv, dh, page, False, 0, 0, width, code)[0] > 0) == many
    lens = [1, 2, 3, 4, 5, 7, 17, 40]
    pool = filled(62, 12, kv, dh, page, code)
    table = numbered(62, [-(-n // page) for n in lens], width, 12)
    q = (0.5 * rand(162 + case, 8, rows, heads, dh)).to(torch.bfloat16)
    out, lse = ops.attention(dev(q), on_gpu(ops, pool, code), dev(table), i32(lens), causal=False)
    o, l, mag, err, _ = attn64(q, pool, code, page, table, lens, [rows] * 8, False, 0, 0, dh ** -0.5)
    ds = (dh + 8) * U * err + 8 * U * (np.abs(l) + 1)
    soft = 2 * ds + (40 + 40) * U
    within(lse, l, soft)
    within(out, o, 2.0 ** -8 * np.abs(o) + mag * (soft[..., None] + (2.0 ** -8 if many else 2.0 ** -16)) * 1.01)
    # all of a row on one slot: its value, which bf16 holds
    out, _ = ops.attention(dev(q), on_gpu(ops, pool, code), dev(table), i32([1] * 8), causal=False)
    for s in range(8):
        v = torch.from_numpy(ref.slots(pool[1], pool[3], False, code, page, table[s], 1)[:, 0])
        assert torch.equal(out[s].cpu().double(), v.repeat_interleave(heads // kv, 0).expand(rows, heads, dh))


@pytest.mark.parametrize("code", CODES)
def test_attention_takes_fp32_queries_whole(ops, code):
    """Slots with one element that is not 0: a row's score is the product of two numbers, 24 bits of them the query's.  fp32
    rounds the sum of the three parts' products, the scale, the product with it, the reference, the power and the logarithm,
    once each or twice: 8 u of the score, and 8 u of a number below 2.  Without the third part 128 u of it would be missing."""
    kv, dh, page = 1, 64, 16
    codes = np.zeros((1, kv, page, dh), np.uint8)
    pool = filled(63, 1, kv, dh, page, code)
    codes[0, 0, 0, 37] = ref.encode(96.0, code)
    pool[0] = ref.in_pieces(codes, True)
    pool[2][:] = 0.25
    q = rand(163, 1, 500, 2, dh)
    _, lse = ops.attention(dev(q), on_gpu(ops, pool, code), dev(np.zeros((1, 1), np.int32)), i32([1]), causal=False)
    want = q[..., 37].double() * 24 / 8
    within(lse, want, 8 * U * (want.abs() + 1))


@pytest.mark.parametrize("case", range(len(PRECISE)))
@pytest.mark.parametrize("code", CODES)
def test_attention_scales_of_values_from_end_to_end(ops, case, code):
    """Pages of zeros as append writes them (a scale of 2^-126), scales from 2^-90 to 2^100, 0 and odd ones, one of them in a
    sequence and several: out and lse as ever, in the scale of what a row sees."""
    rows, heads, kv, dh = PRECISE[case]
    page, width = 16, 10
    pool = filled(64, 60, kv, dh, page, code)
    scales = [[2.0 ** -126] * 6, [2.0 ** -126, 1, 2.0 ** -126, 0.5, 1, 1], [2.0 ** 100] * 6, [2.0 ** -90] * 6,
              [2.0 ** -60, 2.0 ** -70, 2.0 ** -80, 2.0 ** -79, 2.0 ** -62, 2.0 ** -66], [2.0 ** 60, 2.0 ** 66, 2.0 ** 64, 2.0 ** 65, 2.0 ** 63, 2.0 ** 70],
              [0, 0, 2.0 ** -6, 0, 2.0 ** -6, 0], [1.7 * 2.0 ** 30, 1.999 * 2.0 ** -3, 2.0 ** -3, 1.2 * 2.0 ** 30, 2.0 ** 29, 1]]
    table = numbered(64, [6] * 8, width, 60)
    for s in range(8):
        for i in range(6):
            pool[3][table[s, i]] = scales[s][i]
            if scales[s][i] == 2.0 ** -126:
                pool[1][table[s, i]] = 0
    lens = [96, 95, 80, 96, 90, 96, 33, 96]
    q = rand(164 + case, 8, rows, heads, dh).to(torch.bfloat16)
    q[1] *= 4
    out, lse = ops.attention(dev(q), on_gpu(ops, pool, code), dev(table), i32(lens))
    o, l, mag, err, _ = attn64(q, pool, code, page, table, lens, [rows] * 8, True, 0, 0, dh ** -0.5)
    tol_o, tol_l = attn_tolerance(q.dtype, o, l, mag, err, 96, dh)
    # instead of 1e-30: nothing below 2^-126, fp32's and bf16's least normal number, need be held
    tol_o = np.where(mag > 0, tol_o - 1e-30 + 2.0 ** -126, 0)
    within(lse, l, tol_l)
    within(out, o, tol_o)


def test_attention_strides_shared_pages_and_a_single_slot(ops):
    """q as a part of a projection, out as heads of another tensor, a table with a longer row; sequences that share pages; all
    probability on one slot gives its value."""
    kv, dh, page, code = 2, 128, 64, "e4m3"
    pool = filled(9, 5, kv, dh, page, code)
    table = np.array([[3, 1, 0], [3, 1, 2], [4, 4, 4]], np.int32)
    qkv = rand(82, 3, 6, 10, dh, dtype=torch.bfloat16)
    g, wide = dev(qkv), torch.zeros(3, 4, 6, 16, dh, dtype=torch.bfloat16, device="cuda")
    lens = [150, 180, 130]
    d = on_gpu(ops, pool, code)
    t = torch.full((3, 9), -1, dtype=torch.int32, device="cuda")
    t[:, :3] = dev(table)
    out, lse = ops.attention(g[:, 1:5, :6], d, t[:, :3], i32(lens), out=wide[:, :, :, 3])
    o, l, mag, err, _ = attn64(qkv[:, 1:5, :6], pool, code, page, table, lens, [4] * 3, True, 0, 0, dh ** -0.5)
    tol_o, tol_l = attn_tolerance(torch.bfloat16, o, l, mag, err, 180, dh)
    within(out, o, tol_o)
    within(lse, l, tol_l)
    assert (wide[:, :, :, :3] == 0).all() and (wide[:, :, :, 4:] == 0).all()
    q = rand(83, 3, 1, 2, dh)
    one, lse = ops.attention(dev(q), d, dev(table), i32([1, 1, 1]))
    for s in range(3):
        v = ref.slots(pool[1], pool[3], False, code, page, table[s], 1)[:, 0]
        # p v / p with p = exp2(a rounding of the score) near 1: p v is exact in its three parts but for one rounding, 1 / p
        # and the product with it are one each
        within(one[s, 0], v, 3 * U * np.abs(v))


# ---------------------------------------------------------------------------
# moves of pages
# ---------------------------------------------------------------------------
def scattered(seed, lens, page, width, n_pages, shared=0.0):
    """Tables of sequences over a shuffled pool, some of whose pages are held twice, and the counts."""
    r = np.random.RandomState(seed)
    counts = [-(-n // page) for n in lens]
    table = numbered(seed, counts, width, n_pages)
    for s, c in enumerate(counts):
        table[s, c:] = -1
        if s and shared and r.rand() < shared:
            m = min(c, counts[s - 1])
            table[s, :m] = table[s - 1, :m]
    refs = np.zeros(n_pages, np.int32)
    for s, c in enumerate(counts):
        for e in table[s, :c]:
            refs[e] += 1
    return table, np.array(lens, np.int32), refs


def layered(seed, layers, n_pages, kv, dh, page):
    r = np.random.RandomState(seed)
    k = r.randint(0, 256, (layers, n_pages, kv, dh // 16, page, 16)).astype(np.uint8)
    v = r.randint(0, 256, (layers, n_pages, kv, page // 16, dh, 16)).astype(np.uint8)
    return [k, v, r.rand(layers, n_pages, kv).astype(np.float32), r.rand(layers, n_pages, kv).astype(np.float32)]


def moved(pool, moves):
    pool = [x.copy() for x in pool]
    for a, b in moves:
        for x in pool:
            x[:, b] = x[:, a]
    return pool


def equal(got, want, name):
    assert np.array_equal(got.cpu().numpy(), want), (name, got.cpu().numpy(), want)


RESIZE = [
    # lengths, new lengths, page, entries of a row, pages, how many share
    ([0], [1], 16, 1, 1, 0),
    ([5, 16, 0, 33], [6, 17, 40, 0], 16, 4, 12, 0),
    ([5, 16, 0, 33], [60, -1, 64, 100], 16, 4, 12, 0),             # more than a row holds; more than there are
    ([70, 70, 71, 70], [71, 75, -5, 128], 64, 2, 12, 1.0),         # copies
    ([70, 70, 71, 70], [71, 75, 150, 128], 64, 3, 9, 1.0),         # some are not served
    ([100] * 20, [101 + 7 * i for i in range(20)], 32, 9, 90, 0.7),
    ([i % 50 for i in range(1500)], [(i * 7) % 60 for i in range(1500)], 16, 4, 6200, 0.5),
    ([40] * 1030, [41] * 1030, 32, 2100, 9000, 0.9),               # rows of several workgroups
    ([64, 64], [10, 65], 32, 4, 4, 1.0),                           # pages that a shorter one leaves serve from the next call on
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("case", range(len(RESIZE)))
def test_resize(ops, case, in_place):
    lens, new, page, width, n_pages, share = RESIZE[case]
    table, lens, refs = scattered(case, lens, page, width, n_pages, share)
    layers, kv, dh = 3, 1, 64
    pool = layered(case, layers, n_pages, kv, dh, page) if n_pages < 5000 else None
    want_t, want_l, want_r, want_short, copies = ref.resize(table, lens, refs, new, page)
    t, l, r = dev(table), dev(lens), dev(refs)
    outs = {} if in_place else dict(table_out=torch.full_like(t, 9), lens_out=torch.full_like(l, 9), refs_out=torch.full_like(r, 9))
    d = ops.Pool(dev(pool[0]).view(torch.int8), dev(pool[1]).view(torch.int8), dev(pool[2]), dev(pool[3])) if pool else None
    got_l, short = ops.resize(t, l, r, i32(new), d, page=page, **outs)
    equal(outs.get("table_out", t), want_t, "table")
    equal(got_l, want_l, "lens")
    equal(outs.get("refs_out", r), want_r, "refs")
    assert short.item() == want_short
    if pool:
        same_pool(d, moved(pool, copies))
    if not in_place:
        equal(t, table, "table")
        equal(l, lens, "lens")
        equal(r, refs, "refs")


REORDER = [
    # lengths, parents, page, entries of a row
    ([5], [0], 16, 1),
    ([5], [-1], 16, 1),
    ([40, 3, 0, 64], [0, 0, 0, 0], 16, 4),          # forks
    ([40, 3, 0, 64], [1, 2, 3, 0], 16, 4),          # a turn
    ([40, 3, 0, 64], [0, -1, 7, 3], 16, 4),         # freed
    ([7 * i % 90 for i in range(300)], [(i * i + 3) % 310 for i in range(300)], 32, 3),
    ([3000, 2000, 2999], [2, 2, 0], 16, 2500),
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("case", range(len(REORDER)))
def test_reorder(ops, case, in_place):
    lens, parents, page, width = REORDER[case]
    table, lens, refs = scattered(case, lens, page, width, sum(-(-n // page) for n in lens) + 3, 0.5)
    want_t, want_l, want_r = ref.reorder(table, lens, refs, parents, page)
    t, l, r = dev(table), dev(lens), dev(refs)
    outs = {} if in_place else dict(table_out=torch.full_like(t, 9), lens_out=torch.full_like(l, 9), refs_out=torch.full_like(r, 9))
    got_l = ops.reorder(t, l, r, i32(parents), page, **outs)
    equal(outs.get("table_out", t), want_t, "table")
    equal(got_l, want_l, "lens")
    equal(outs.get("refs_out", r), want_r, "refs")


COMPACT = [
    # lengths, page, entries of a row, free pages, how many share
    ([1], 16, 1, 0, 0),
    ([1], 16, 3, 5, 0),
    ([0, 0], 16, 3, 5, 0),                        # nothing in use
    ([100, 50, 0, 64, 33], 16, 7, 40, 0.5),
    ([16 * 7] * 9, 16, 7, 1, 0),                  # one hole
    ([64 * (i % 5) + 1 for i in range(200)], 64, 5, 4200, 0.3),
    ([500] * 100, 32, 1100, 9000, 0),
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("case", range(len(COMPACT)))
def test_compact(ops, case, in_place):
    lens, page, width, spare, share = COMPACT[case]
    n_pages = sum(-(-n // page) for n in lens) + spare
    table, lens, refs = scattered(case, lens, page, width, n_pages, share)
    if n_pages > 20:
        refs[np.flatnonzero(refs == 0)[:2]] = -1  # free is free
    pool = layered(case, 2, n_pages, 2, 64, page) if n_pages < 6000 else None
    want_t, want_r, n_live, moves = ref.compact(table, refs)
    t, r = dev(table), dev(refs)
    outs = {} if in_place else dict(table_out=torch.full_like(t, 9), refs_out=torch.full_like(r, 9))
    d = ops.Pool(dev(pool[0]).view(torch.int8), dev(pool[1]).view(torch.int8), dev(pool[2]), dev(pool[3])) if pool else None
    assert ops.compact(t, r, d, **outs).item() == n_live
    equal(outs.get("table_out", t), want_t, "table")
    equal(outs.get("refs_out", r), want_r, "refs")
    if pool:
        same_pool(d, moved(pool, moves))


def test_moves_pass_by_numbers_that_name_no_page(ops):
    table = np.array([[0, -3, 5, -1], [99, 1, 2, -1], [3, 1 << 30, -1, -1]], np.int32)
    lens, refs, page = np.array([40, 48, 20], np.int32), np.array([1, 1, 1, 1, 0, 1, 0, 0], np.int32), 16
    for new in ([50, 10, 0], [16, 49, 21], [0, 0, 0]):
        t, l, r = dev(table), dev(lens), dev(refs)
        want = ref.resize(table, lens, refs, new, page)
        _, short = ops.resize(t, l, r, i32(new), page=page)
        for got, w in zip((t, l, r), want):
            equal(got, w, "resize")
        assert short.item() == want[3]
    t, l, r = dev(table), dev(lens), dev(refs)
    ops.reorder(t, l, r, i32([1, 1, -1]), page)
    for got, w in zip((t, l, r), ref.reorder(table, lens, refs, [1, 1, -1], page)):
        equal(got, w, "reorder")
    t, r = dev(table), dev(refs)
    assert ops.compact(t, r).item() == 5
    for got, w in zip((t, r), ref.compact(table, refs)):
        equal(got, w, "compact")


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("code,dtype", [("e4m3", torch.bfloat16), ("int8", torch.float32)])
def test_a_run_of_them_together(ops, code, dtype):
    """A prefix is read, forked into candidates, each grows by tokens of its own, the lighter ones are dropped for copies of
    the others, and the pool is moved together; after each step everything is as the plain forms have it."""
    layers, kv, heads, dh, page, S, width, n_pages = 2, 1, 4, 64, 16, 4, 6, 24
    pool = [np.zeros_like(x) for x in layered(0, layers, n_pages, kv, dh, page)]
    d = ops.Pool(dev(pool[0]).view(CODES[code]), dev(pool[1]).view(CODES[code]), dev(pool[2]), dev(pool[3]))
    table, lens, refs = np.full((S, width), -1, np.int32), np.zeros(S, np.int32), np.zeros(n_pages, np.int32)
    t, l, r = dev(table), dev(lens), dev(refs)
    qw, kw = 1 + 0.2 * rand(1, dh), 1 + 0.2 * rand(2, dh)
    seed = 100

    def step(n_new, window):
        nonlocal table, lens, refs, pool, seed
        tokens = max(n_new)
        starts, want = lens.copy(), lens + np.array(n_new, np.int32)
        before = l.clone()
        got_l, short = ops.resize(t, l, r, l + i32(n_new), d)
        table, lens, refs, lack, copies = ref.resize(table, lens, refs, want, page)
        pool = moved(pool, copies)
        assert lack == 0 and short.item() == 0
        pos = torch.from_numpy(starts)[:, None] + torch.arange(tokens)
        for layer in range(layers):
            seed += 3
            q, k, v = (rand(seed + i, S, tokens, heads if i == 0 else kv, dh, dtype=dtype) for i in range(3))
            qo, ko = ops.norm_rope(dev(q), dev(k), dev(pos.int()), q_weight=dev(qw), k_weight=dev(kw))
            norm_close(qo, q, qw, 0, 1e-6, pos, dh)
            norm_close(ko, k, kw, 0, 1e-6, pos, dh)
            ops.append(d.layer(layer), t, before, ko, dev(v), n_new=i32(n_new))
            mine = [x[layer] for x in pool]
            for i, x in ((0, ko), (1, v)):
                ref.append_one(mine[i], mine[2 + i], i == 0, code, page, table, starts, x.cpu().float().numpy(), n_new)
            same_pool(d.layer(layer), mine)
            out, lse = ops.attention(qo, d.layer(layer), t, l, q_lens=i32(n_new), window=window, sinks=2 if window else 0)
            o, ls, mag, err, there = attn64(qo.cpu(), mine, code, page, table, lens, n_new, True, window, 2 if window else 0, dh ** -0.5)
            tol_o, tol_l = attn_tolerance(dtype, o, ls, mag, err, lens.max(), dh)
            within(out.cpu()[torch.from_numpy(there)], o[there], tol_o[there])
            within(lse.cpu()[torch.from_numpy(there)], ls[there], tol_l[there])

    def reordered(parents):
        nonlocal table, lens, refs
        ops.reorder(t, l, r, i32(parents), page)
        table, lens, refs = ref.reorder(table, lens, refs, parents, page)

    step([37, 0, 0, 0], 0)
    reordered([0, 0, 0, 0])
    step([1, 1, 1, 1], 0)
    step([3, 1, 12, 0], 10)
    reordered([2, 1, 2, -1])
    table, refs, n_live, moves = ref.compact(table, refs)
    pool = moved(pool, moves)
    assert ops.compact(t, r, d).item() == n_live
    step([1, 1, 1, 20], 10)
    step([1, 1, 1, 1], 0)
    for got, want, name in ((t, table, "table"), (l, lens, "lens"), (r, refs, "refs")):
        equal(got, want, name)
    reordered([-1] * 4)
    assert (r.cpu() == 0).all()


@pytest.mark.parametrize("code,dtype", [("e4m3", torch.bfloat16), ("int8", torch.float32)])
def test_a_step_in_a_pool_that_runs_out(ops, code, dtype):
    """Three forks of 21 slots and a sequence of 26 want three tokens each, and there is one page: it goes to the first fork;
    the two others' shared page, their rows of the outputs and their lengths stay as they were, until pages are free again."""
    kv, heads, dh, page, S, tokens = 2, 4, 64, 16, 4, 3
    pool = filled(13, 6, kv, dh, page, code)
    d = on_gpu(ops, pool, code)
    table = np.array([[0, 1, -1], [0, 1, -1], [0, 1, -1], [2, 3, -1]], np.int32)
    lens, refs = np.array([21, 21, 21, 26], np.int32), np.array([3, 3, 1, 1, 1, 0], np.int32)  # page 4 is somebody else's
    t, l, r = dev(table), dev(lens), dev(refs)
    for step, given in enumerate(([3, 0, 0, 3], [0, 0, 3, 3])):
        if step:  # the first two forks give their pages back; the third has its last page for itself
            ops.reorder(t, l, r, i32([-1, -1, 2, 3]), page)
            table, lens, refs = ref.reorder(table, lens, refs, [-1, -1, 2, 3], page)
            want = np.array([0, 0, 24, 32], np.int32)
        else:
            want = lens + 3
        starts, before = l.clone(), [x.copy() for x in pool]
        _, short = ops.resize(t, l, r, i32(want), ops.Pool(*(x[None] for x in d)))
        table, lens, refs, lack, copies = ref.resize(table, lens, refs, want, page)
        assert short.item() == lack == (0 if step else 2)
        pool = [x.copy() for x in pool]
        for a, b in copies:
            for x in pool:
                x[b] = x[a]
        n_new = l - starts
        assert n_new.tolist() == given
        q, k, v = (dev(rand(270 + 3 * step + i, S, tokens, heads if i == 0 else kv, dh, dtype=dtype)) for i in range(3))
        ops.append(d, t, starts, k, v, n_new=n_new)
        for i, x in ((0, k), (1, v)):
            ref.append_one(pool[i], pool[2 + i], i == 0, code, page, table, starts.tolist(), x.cpu().float().numpy(), given)
        same_pool(d, pool)
        if not step:
            assert all(np.array_equal(x[1], b[1]) for x, b in zip(pool, before))  # the shared page
        out = torch.full(q.shape, -77.0, dtype=dtype, device="cuda")
        lse = torch.full(q.shape[:3], -77.0, device="cuda")
        ops.attention(q, d, t, l, q_lens=n_new, out=out, lse=lse)
        o, ls, mag, err, there = attn64(q.cpu(), pool, code, page, table, lens, given, True, 0, 0, dh ** -0.5)
        tol_o, tol_l = attn_tolerance(dtype, o, ls, mag, err, 32, dh)
        there = torch.from_numpy(there)
        within(out.cpu()[there], o[there.numpy()], tol_o[there.numpy()])
        within(lse.cpu()[there], ls[there.numpy()], tol_l[there.numpy()])
        assert (out.cpu()[~there] == -77).all() and (lse.cpu()[~there] == -77).all()


# ---------------------------------------------------------------------------
# as programs call them
# ---------------------------------------------------------------------------
def decode_state(ops, code="e4m3", S=5, kv=2, heads=4, dh=64, page=16, width=8, n_pages=64, layers=1):
    """Sequences of a few slots each, room for more, and everything on the GPU."""
    pool = filled(1, n_pages, kv, dh, page, code)
    lens = [37, 0, 16, 90, 5][:S]
    table, lens, refs = scattered(1, lens, page, width, n_pages)
    return dict(pool=on_gpu(ops, pool, code), table=dev(table), lens=dev(lens), refs=dev(refs), page=page,
                qw=dev(1 + 0.1 * rand(1, dh)), kw=dev(1 + 0.1 * rand(2, dh)))


def decode_step(ops, st, q, k, v, window=0):
    """One token for each sequence, as a sampling program does it."""
    starts = st["lens"].clone()
    new = st["lens"] + 1
    ops.resize(st["table"], st["lens"], st["refs"], new, st["pool"])
    qo, ko = ops.norm_rope(q, k, starts[:, None], q_weight=st["qw"], k_weight=st["kw"])
    ops.append(st["pool"], st["table"], starts, ko, v)
    return ops.attention(qo, st["pool"], st["table"], st["lens"], window=window, sinks=2 if window else 0)


def everything(st):
    return [t.clone() for t in (*st["pool"], st["table"], st["lens"], st["refs"])]


def same_bits(a, b):
    for x, y in zip(a, b):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


def copied(st):
    return {k: type(v)(*(t.clone() for t in v)) if isinstance(v, tuple) else v.clone() if torch.is_tensor(v) else v for k, v in st.items()}


@pytest.mark.parametrize("dtype", TYPES)
def test_a_captured_step_replays_as_the_eager_one_runs(ops, dtype):
    """The graph advances its own state; each replay is compared with an eager step on a copy, with eager work between."""
    st = decode_state(ops)
    inputs = [[rand(200 + 3 * i + j, 5, 1, 4 if j == 0 else 2, 64, dtype=dtype).cuda() for j in range(3)] for i in range(7)]
    hold = [x.clone() for x in inputs[0]]
    other = copied(st)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = decode_step(ops, other, *inputs[0], window=30)  # also the call before the capture
        warm = copied(st)
        decode_step(ops, warm, *hold, window=30)
    torch.cuda.synchronize()
    other = copied(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = decode_step(ops, st, *hold, window=30)
    same_bits(everything(st), everything(other))  # capturing runs nothing
    for i in range(7):
        for h, x in zip(hold, inputs[i]):
            h.copy_(x)
        graph.replay()
        want = decode_step(ops, other, *inputs[i], window=30)
        torch.cuda.synchronize()
        same_bits(got, want)
        same_bits(everything(st), everything(other))
        if i % 2:
            rand(1, 100).cuda().sum().item()


def test_two_graphs_in_turn(ops):
    """Two captured calls that want workspaces, replayed one after the other, over and over."""
    pool = on_gpu(ops, filled(2, 300, 1, 64, 16, "int8"), "int8")
    table = dev(numbered(2, [140, 140], 140, 300))
    lens = i32([2200, 1999])
    q = [dev(rand(210 + i, 2, 1, 8, 64)) for i in range(2)]
    want = [[t.clone() for t in ops.attention(x, pool, table, lens)] for x in q]
    graphs, got = [], []
    for x in q:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(ops.attention(x, pool, table, lens))
        graphs.append(g)
    for _ in range(4):
        for g in graphs:
            g.replay()
        for t in (*got[0], *got[1]):
            assert torch.isfinite(t).all()
        for w, y in zip(want, got):
            same_bits(w, y)
        for y in got:
            for t in y:
                t.fill_(float("nan"))


def test_streams(ops):
    """On a stream of the caller's, whose earlier work makes the inputs; and two calls at once on two streams."""
    pool = on_gpu(ops, filled(3, 300, 2, 128, 16, "e4m3"), "e4m3")
    table, lens = dev(numbered(3, [140, 140], 140, 300)), i32([2200, 1500])
    qs = [dev(rand(220 + i, 2, 3, 4, 128, dtype=torch.bfloat16)) for i in range(2)]
    want = [[t.clone() for t in ops.attention(x, pool, table, lens)] for x in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, x in zip(streams, qs):
            with torch.cuda.stream(s):
                late = torch.zeros(1 << 24, device="cuda").add_(1).sum() * 0  # work before the input is there
                got.append(ops.attention((x.float() + late).to(x.dtype), pool, table, lens))
        torch.cuda.synchronize()
        for w, y in zip(want, got):
            same_bits(w, y)


@pytest.mark.parametrize("code", CODES)
def test_a_pool_past_4_gib(ops, code):
    """Pages whose codes lie past 2^32 bytes, and past 2^31 elements, act as low ones do."""
    kv, dh, page, n_pages = 8, 128, 128, 33500
    pool = ops.Pool(*(torch.empty((n_pages, kv, *s), dtype=torch.uint8, device="cuda").view(CODES[code]) for s in ((dh // 16, page, 16), (page // 16, dh, 16))),
                    *(torch.zeros((n_pages, kv), device="cuda") for _ in range(2)))
    assert pool.k.numel() > 1 << 32
    tables = [dev(np.array([[0, 1, 2], [3, 4, 5]], np.int32)), dev(np.array([[33499, 33000, 16500], [33498, 16384, 32768]], np.int32))]
    k, v = dev(rand(230, 2, 300, kv, dh)), dev(rand(231, 2, 300, kv, dh))
    got = []
    for t in tables:
        for start, n in ((0, 200), (200, 100)):
            ops.append(pool, t, i32([start, start]), k[:, start:start + n], v[:, start:start + n])
        few = ops.attention(dev(rand(232, 2, 1, 32, dh)), pool, t, i32([300, 299]))
        many = ops.attention(dev(rand(233, 2, 600, 64, dh, dtype=torch.bfloat16)), pool, t, i32([300, 299]), causal=False)
        got.append([*few, *many])
    same_bits(*got)
    # and moved: pages in use are the three highest
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    t = dev(np.array([[33499, 33000, 16500]], np.int32))
    refs[t[0].long()] = 1
    before = [x[t[0].long()].view(torch.uint8) for x in pool]
    lead = ops.Pool(*(x[None] for x in pool))
    assert ops.compact(t, refs, lead).item() == 3
    assert sorted(t[0].tolist()) == [0, 1, 2]
    same_bits(before, [x[t[0].long()] for x in pool])


@pytest.mark.parametrize("rows,heads,dh,dtype", [(1, 4, 128, torch.float32), (3, 4, 64, torch.bfloat16), (150, 256, 64, torch.bfloat16),
                                                 (100, 128, 256, torch.bfloat16)])
def test_the_longest_sequence(ops, rows, heads, dh, dtype):
    """2^29 slots in 2^22 pages, most of them the same few: a window at its end sees what the end of a short sequence does."""
    kv, page, code, window, sinks, width = heads // 4, 128, "int8", 700, 5, 1 << 22
    assert (plan_of(1, rows, heads, kv, dh, page, True, window, sinks, width, code)[0] > 0) == (rows >= 100)
    pool = filled(70, 12, kv, dh, page, code)
    behind = 37  # slots of the last page that are not there
    few = np.array([[3, 7, 0, 9, 4, 1, 5, 8]], np.int32)  # the first page, and the last ones
    table = torch.full((1, width), 11, dtype=torch.int32)
    table[0, 0], table[0, -7:] = 3, torch.from_numpy(few[0, 1:])
    q = rand(250, 1, rows, heads, dh, dtype=dtype)
    o, l, mag, err, _ = attn64(q, pool, code, page, few, [8 * page - behind], [rows], True, window, sinks, dh ** -0.5)
    tol_o, tol_l = attn_tolerance(dtype, o, l, mag, err, window + sinks, dh)
    d = on_gpu(ops, pool, code)
    out, lse = ops.attention(dev(q), d, dev(table), i32([(1 << 29) - behind]), window=window, sinks=sinks)
    within(out, o, tol_o)
    within(lse, l, tol_l)
    # tokens at its end; those past it are dropped
    k, v = rand(251, 1, 41, kv, dh), rand(252, 1, 41, kv, dh)
    ops.append(d, dev(table), i32([(1 << 29) - behind]), dev(k), dev(v))
    for i, x in ((0, k), (1, v)):
        ref.append_one(pool[i], pool[2 + i], i == 0, code, page, few, [8 * page - behind], x.numpy(), [41])
    same_pool(d, pool)


def test_moves_of_the_longest_sequence(ops):
    width, n_pages, page = 1 << 22, (1 << 22) + 3, 128
    table, lens = torch.full((1, width), -1, dtype=torch.int32, device="cuda"), i32([0])
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[1::1 << 21] = 1  # three pages of others
    others = refs.clone()
    free = (others == 0).nonzero()[:width, 0].int()
    _, short = ops.resize(table, lens, refs, i32([1 << 29]), page=page)
    assert short.item() == 0 and lens.item() == 1 << 29 and torch.equal(table[0], free)
    assert (refs == 1).all()
    ops.resize(table, lens, refs, i32([(1 << 28) + 1]), page=page)
    has = (1 << 21) + 1
    assert torch.equal(table[0, :has], free[:has]) and (table[0, has:] == -1).all()
    assert torch.equal((refs == 0).nonzero()[:, 0], free[has:].long())
    both = torch.cat([table, table])
    other = torch.tensor([(1 << 28) + 1, 0], dtype=torch.int32, device="cuda")
    ops.reorder(both, other, refs, i32([1, 0]), page)
    assert (both[0] == -1).all() and torch.equal(both[1], table[0]) and other.tolist() == [0, (1 << 28) + 1]
    ops.reorder(both, other, refs, i32([-1, 1]), page)
    assert torch.equal((refs != 0).nonzero()[:, 0], torch.cat([free[:has].long(), (others != 0).nonzero()[:, 0]]).sort().values)
    n_live = ops.compact(both, refs)
    assert n_live.item() == has + 3 and (refs[:has + 3] == 1).all() and (refs[has + 3:] == 0).all()


@pytest.mark.parametrize("rows,heads", [(3, 8), (3, 160)])
def test_strides_past_2_to_the_31(ops, rows, heads):
    """Rows 2^31 elements apart give what neighbouring ones give."""
    kv, dh, page, code = heads // 4, 128, 32, "e4m3"
    far = torch.empty((2 << 31) + heads * dh, dtype=torch.bfloat16, device="cuda")
    wide = far.as_strided((1, rows, heads, dh), (far.numel(), 1 << 31, dh, 1))
    q = dev(rand(260, 1, rows, heads, dh, dtype=torch.bfloat16))
    w = dev(rand(261, dh))
    wide.copy_(q)
    near, _ = ops.norm_rope(q, q_weight=w)
    ops.norm_rope(wide, q_weight=w, q_out=wide)
    same_bits([wide], [near])
    d, other = (on_gpu(ops, filled(71, 4, kv, dh, page, code), code) for _ in range(2))
    table = dev(np.array([[2, 0, 3]], np.int32))
    ops.append(d, table, i32([60]), near[:, :, :kv], near[:, :, kv:2 * kv])
    ops.append(other, table, i32([60]), wide[:, :, :kv], wide[:, :, kv:2 * kv])
    same_bits(d, other)
    want, lse = ops.attention(near, d, table, i32([63]))
    got, lse_far = ops.attention(wide, d, table, i32([63]))
    same_bits([want, lse], [got, lse_far])
    ops.attention(near, d, table, i32([63]), out=wide)
    same_bits([want], [wide])


def test_equal_calls_give_equal_bits_and_writes_count(ops):
    pool = on_gpu(ops, filled(4, 300, 2, 128, 16, "e4m3"), "e4m3")
    table, lens = dev(numbered(4, [140, 140], 140, 300)), i32([2200, 1500])
    q = dev(rand(240, 2, 3, 8, 128, dtype=torch.bfloat16))
    first = [t.clone() for t in ops.attention(q, pool, table, lens)]
    for _ in range(3):
        same_bits(first, ops.attention(q, pool, table, lens))
    out, lse = torch.empty_like(q), torch.empty(2, 3, 8, device="cuda")
    refs = torch.ones(300, dtype=torch.int32, device="cuda")
    k = dev(rand(241, 2, 1, 2, 128))

    def moved_on(call, *tensors):
        before = [t._version for t in tensors]
        call()
        assert all(t._version > b for t, b in zip(tensors, before))

    moved_on(lambda: ops.attention(q, pool, table, lens, out=out, lse=lse), out, lse)
    moved_on(lambda: ops.append(pool, table, lens, k, k), *pool)
    moved_on(lambda: ops.resize(table, lens, refs, lens - 1, pool), table, lens, refs, *pool)
    moved_on(lambda: ops.reorder(table, lens, refs, i32([1, 0]), 16), table, lens, refs)
    moved_on(lambda: ops.compact(table, refs, pool), table, refs, *pool)
    x = q.clone()
    moved_on(lambda: ops.norm_rope(x, q_out=x), x)
    with torch.inference_mode():
        same_bits([ops.norm_rope(q)[0]], [ops.norm_rope(q.clone())[0]])
