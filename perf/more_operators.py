"""Operators of a paged 8-bit KV cache that are timed and compared: norms of
queries and keys with their rotation, writing tokens into the cache, attention
over it (whole, causal, or with a sliding window and a few first slots), and
the moves of its pages (fork, growth with copy on write, compaction).

Shapes are the repository's own (the pi0.5 expert's eight heads of 256 over one
KV head, prefixes of 816 tokens, chunks of 50 actions, eighteen layers, the
tiny fp32 expert's heads of 64) and generic ones (32 heads over 8 KV heads of
128, long caches).  ``run`` computes the operators in elementary torch
operations, or through ``paper_2607_12659_amd.cache_ops`` where ``own`` is true.

A pool of pages holds K as [pages][kv][D / 16][slots][16 dims] and V as
[pages][kv][slots / 16][D][16 slots] in codes of 8 bits, each (page, kv head)
with a scale.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
NEG_INF = float("-inf")
EPS = 1e-6
CODES = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _norm(name, batch, tokens, heads, kv, dh, rot, layout="half", offset=False, far=0, dtype="bf16"):
    """far: positions are drawn below it (0: consecutive ones).  offset: the norm's factor is 1 + weight."""
    return {"name": name, "kind": "norm", "batch": batch, "tokens": tokens, "heads": heads, "kv": kv, "dh": dh, "rot": rot,
            "layout": layout, "offset": offset, "far": far, "dtype": dtype}


def _append(name, batch, tokens, kv, dh, page, start, ragged=False, code="e4m3", dtype="bf16"):
    """start: slots that the longest sequence holds before the call."""
    return {"name": name, "kind": "append", "batch": batch, "tokens": tokens, "kv": kv, "dh": dh, "page": page, "start": start,
            "ragged": ragged, "code": code, "dtype": dtype}


def _attn(name, batch, rows, heads, kv, dh, page, length, causal=True, window=0, sinks=0, shared=0, ragged=False, code="e4m3",
          dtype="bf16"):
    """shared: the first slots that all sequences have in the same pages."""
    return {"name": name, "kind": "attn", "batch": batch, "rows": rows, "heads": heads, "kv": kv, "dh": dh, "page": page,
            "length": length, "causal": causal, "window": window, "sinks": sinks, "shared": shared, "ragged": ragged, "code": code,
            "dtype": dtype}


def _pages(name, op, layers, seqs, length, grow, kv, dh, page, spare, beams=False, code="int8"):
    """spare: pages of the pool that no sequence holds at first.  beams: parents spread over the sequences, else all are sequence 0."""
    return {"name": name, "kind": op, "layers": layers, "seqs": seqs, "length": length, "grow": grow, "kv": kv, "dh": dh, "page": page,
            "spare": spare, "beams": beams, "code": code}


def listed():
    return [
        # queries and key of one new token of one sequence in one layer, latency-bound
        _norm("norm-token", 1, 1, 8, 1, 256, 256, offset=True, far=4096),
        # the queries and keys of one layer for two long texts, fp32, half of each head turned in neighbouring pairs
        _norm("norm-far-f32", 2, 4099, 32, 8, 128, 64, "interleaved", far=131072, dtype="f32"),
        # one decoded token of each of sixty-four rollouts, somewhere inside their last pages
        _append("append-token-b64", 64, 1, 8, 128, 64, 2050, ragged=True),
        # the prefix of eight observations behind a short text each, pages of 32 slots
        _append("append-prefix-b8", 8, 816, 1, 256, 32, 51, code="int8"),
        # one decoded token of one rollout behind its prefix, latency-bound
        _attn("attn8-token", 1, 1, 8, 1, 256, 64, 817),
        # eight candidate action chunks denoised against one observation whose pages they share
        _attn("attn8-chunk-b8", 8, 50, 8, 1, 256, 32, 866, causal=False, shared=816),
        # one token of each of sixty-four sampled texts of unequal lengths
        _attn("attn8-decode-b64", 64, 1, 32, 8, 128, 64, 8192, ragged=True, code="int8"),
        # a long text read in one call, each token seeing the last 1024 and the first four
        _attn("attn8-window-4099", 1, 4099, 32, 8, 128, 16, 4099, window=1024, sinks=4),
        # the tiny fp32 expert's heads: a few rows of three short texts of unequal lengths
        _attn("attn8-f32-odd", 3, 7, 4, 2, 64, 16, 333, window=100, sinks=3, ragged=True, code="int8", dtype="f32"),
        # one observation's cache in all layers forked into eight candidates, each with room for a chunk
        _pages("fork-l18-g8", "fork", 18, 8, 816, 50, 1, 256, 64, 80),
        # one step of a search over sixty-four beams: reordered by their parents, a token of room for each
        _pages("fork-beams-b64", "fork", 1, 64, 4000, 1, 8, 128, 64, 128, beams=True),
        # a pool half of whose pages went free, moved together
        _pages("compact-b32", "compact", 2, 32, 4000, 0, 8, 128, 64, 2000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# what the listed cases of each kind cost at most; a drawn case is cut until it costs no more
_MOST_BYTES = {"norm": 335e6, "append": 10e6, "attn": 545e6, "fork": 16e6, "compact": 450e6}
_MOST_FLOPS = {"bf16": 6e10, "f32": 1e10}


def draw(rng):
    kind = rng.choice(["norm", "append", "attn", "attn", "attn", "fork", "compact"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    code = rng.choice(["e4m3", "int8"])
    dh, page = rng.choice([64, 128, 256]), rng.choice([16, 32, 64, 128])
    if kind == "norm":
        heads, kv = rng.choice([(8, 1), (4, 2), (32, 8), (7, 0)])
        c = _norm("", _log(rng, 1, 16), _log(rng, 1, 8192), heads, kv, dh, dh // rng.choice([1, 1, 2, 4]),
                  rng.choice(["half", "interleaved"]), rng.random() < 0.5, rng.choice([0, _log(rng, 1000, 1000000)]), dtype)
        cut = "tokens"
    elif kind == "append":
        c = _append("", _log(rng, 1, 128), rng.choice([1, 1, _log(rng, 1, 2048)]), rng.choice([1, 2, 8]), dh, page,
                    _log(rng, 1, 4096) - 1, rng.random() < 0.5, code, dtype)
        cut = "tokens" if c["tokens"] > 1 else "batch"
    elif kind == "attn":
        heads, kv = rng.choice([(8, 1), (8, 1), (4, 2), (32, 8), (6, 6)])
        rows = rng.choice([1, 1, _log(rng, 1, 64), _log(rng, 64, 2048)])
        length = rows + _log(rng, 1, 32768) - 1
        causal = rng.random() < 0.75
        window = _log(rng, 1, 4096) if causal and rng.random() < 0.5 else 0
        c = _attn("", _log(rng, 1, 64), rows, heads, kv, dh, page, length, causal, window, rng.randint(0, 8) if window else 0,
                  rng.choice([0, length // 2]), rng.random() < 0.5, code, dtype)
        cut = "batch"
    else:
        c = _pages("", kind, _log(rng, 1, 18), _log(rng, 1, 128), _log(rng, 1, 8192), rng.choice([1, _log(rng, 1, 200)]) * (kind == "fork"),
                   rng.choice([1, 2, 8]), dh, page, 0, rng.random() < 0.5, code)
        c["spare"] = _pages_of(c["length"] + c["grow"], page) * (1 + c["seqs"] // rng.choice([1, 2, 4]))
        cut = "layers"
    while work(c)["bytes"] > _MOST_BYTES[kind] or (kind == "attn" and _plain_flops(c) > _MOST_FLOPS[dtype]) or (
            kind in ("fork", "compact") and _pool_bytes(c) > 1.3e9):
        if c[cut] == 1:
            cut = {"batch": "length", "layers": "seqs"}[cut]
        c[cut] = max(1, c[cut] * 2 // 3)
        if kind == "attn":
            c["rows"], c["shared"] = min(c["rows"], c["length"]), min(c["shared"], c["length"])
    c.pop("name")
    return c


# ---------------------------------------------------------------------------
# lengths and parents, the same for every seed
# ---------------------------------------------------------------------------
def _pages_of(n, page):
    return -(-n // page)


def _starts(c):
    """Slots before the new tokens: ragged ones are spread between none and all."""
    b, s = c["batch"], c["start"]
    return [s - (s * ((i * 7) % b)) // b for i in range(b)] if c["ragged"] else [s] * b


def _new(c):
    """Tokens that are new: ragged ones fall from all to one."""
    b, t = c["batch"], c["tokens"]
    return [t - ((t - 1) * i) // b for i in range(b)] if c["ragged"] else [t] * b


def _lengths(c):
    """Slots of each sequence: ragged ones are spread between two and all, but never below the shared ones."""
    b, n = c["batch"], c["length"]
    return [max(c["shared"], n - ((n - 2) * ((i * 5) % b)) // b) for i in range(b)] if c["ragged"] and n > 2 else [n] * b


def _held(c):
    """Slots of each sequence of a pool before the pages move: spread between a little over half and all."""
    s, n = c["seqs"], c["length"]
    return [n - (n * ((i * 3) % s)) // (2 * s) for i in range(s)]


def _parents(c):
    return [((i * 7) % c["seqs"]) // 2 for i in range(c["seqs"])] if c["beams"] else [0] * c["seqs"]


def _copies(c):
    """Sequences of a fork whose last page is a shared, partial one."""
    held, parents = _held(c), _parents(c)
    return sum(held[p] % c["page"] != 0 and parents.count(p) > 1 for p in parents)


def _table_pages(c):
    return _pages_of(c["length"] + c["grow"], c["page"]) + 1


def _pool_pages(c):
    return sum(_pages_of(n, c["page"]) for n in _held(c)) + c["spare"]


def _page_bytes(c):
    return 2 * c["kv"] * (c["page"] * c["dh"] + 4) * c["layers"]


def _pool_bytes(c):
    return _pool_pages(c) * _page_bytes(c)


def _seen(c, n):
    """Slots that row i of a sequence of n sees, summed over the rows, and those that any row sees."""
    rows, total, low = c["rows"], 0, n
    if not c["causal"]:
        return rows * n, n
    for i in range(rows):
        p = n - rows + i
        if p < 0:
            continue
        first = max(0, p - c["window"] + 1) if c["window"] else 0
        total += p + 1 - first + min(first, c["sinks"])
        low = min(low, first)
    return total, n - low + min(low, c["sinks"])


def _plain_flops(c):
    """What the plain form, which knows no window, multiplies."""
    return 4 * c["dh"] * c["rows"] * c["heads"] * c["batch"] * c["length"]


def work(c):
    es = 2 if c.get("dtype") == "bf16" else 4
    k = c["kind"]
    if k == "norm":
        n = c["batch"] * c["tokens"]
        return {"bytes": 2 * n * (c["heads"] + c["kv"]) * c["dh"] * es + 4 * n, "flops": n * (c["heads"] + c["kv"]) * (4 * c["dh"] + 3 * c["rot"])}
    if k == "append":
        n = 2 * sum(_new(c)) * c["kv"] * c["dh"]
        return {"bytes": n * (es + 1) + 8 * c["batch"], "flops": 2 * n}
    if k == "attn":
        pairs, slots = 0, -c["shared"] * (c["batch"] - 1) if not c["window"] else 0
        for n in _lengths(c):
            p, any_row = _seen(c, n)
            pairs, slots = pairs + p, slots + any_row
        rows = c["batch"] * c["rows"] * c["heads"]
        return {"bytes": max(slots, 1) * c["kv"] * (2 * c["dh"] + 8 / c["page"]) + 2 * rows * c["dh"] * es + 4 * rows, "flops": 4 * c["dh"] * c["heads"] * pairs}
    meta = 8 * c["seqs"] * _table_pages(c) + 8 * _pool_pages(c)
    if k == "fork":
        return {"bytes": 2 * meta + 2 * _copies(c) * _page_bytes(c), "flops": 0}
    live = sum(_pages_of(n, c["page"]) for n in _held(c))  # of its pages a share as large as the free one's lies behind them
    return {"bytes": meta + 2 * live * c["spare"] // (live + c["spare"]) * _page_bytes(c), "flops": 0}


# ---------------------------------------------------------------------------
# inputs from the seed
# ---------------------------------------------------------------------------
def _scale_of(amax, code):
    """The least power of two, from 2^-126 on, whose multiple by the largest code reaches amax; NaN where amax is not finite."""
    m, e = torch.frexp(amax)
    e = e - 7 + (m > 127 / 128).int() if code == "int8" else e - 9 + (m > 0.875).int()
    s = ((torch.where(amax > 0, e, -126).clamp(min=-126) + 127).int() << 23).view(torch.float32)
    return torch.where(torch.isfinite(amax), s, float("nan"))


def _coded(y, code):
    return y.round().to(torch.int8) if code == "int8" else y.to(torch.float8_e4m3fn)


def _filled(c, normal, *pages):
    """Codes and scales of pages of normal values, their sizes spread as those of heads and texts are."""
    kv, dh, page = c["kv"], c["dh"], c["page"]
    got = []
    for shape in ((dh // 16, page, 16), (page // 16, dh, 16)):
        x = normal(*pages, kv, *shape).mul_(torch.exp(0.5 * normal(*pages, kv, 1, 1, 1)))
        s = _scale_of(x.abs().amax((-3, -2, -1)), c["code"])
        got.append((_coded(x / s[..., None, None, None], c["code"]), s))
    return got[0][0], got[1][0], got[0][1], got[1][1]


def _numbered(pages, counts, width, shared=0):
    """A table of rows that take the page numbers in order, -1 behind them; the first `shared` entries are row 0's in all rows."""
    rows, at = [], 0
    for i, n in enumerate(counts):
        head = rows[0][:shared] if i else []
        rows.append(head + pages[at:at + n - len(head)] + [-1] * (width - n))
        at += n - len(head)
    return rows


def prepare(c, seed):
    """Inputs, the cache, and the buffers that a serving program keeps for the outputs."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + 41)
    cpu = torch.Generator()
    cpu.manual_seed(1000003 * int(seed) + 43)
    dt = torch.bfloat16 if c.get("dtype") == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=DEV)

    st, k = {"case": c}, c["kind"]
    if k == "norm":
        b, n, dh = c["batch"], c["tokens"], c["dh"]
        st["q"] = (3 * normal(b, n, c["heads"], dh)).to(dt)
        st["k"] = (3 * normal(b, n, c["kv"], dh)).to(dt) if c["kv"] else None
        shift = 0.0 if c["offset"] else 1.0
        st["qw"], st["kw"] = (shift + 0.2 * normal(dh)).to(dt), (shift + 0.2 * normal(dh)).to(dt)
        if c["far"]:
            st["pos"] = torch.randint(0, c["far"], (b, n), generator=g, device=DEV).to(torch.int32)
        else:
            st["pos"] = torch.arange(n, device=DEV, dtype=torch.int32).expand(b, n).contiguous()
        st["q_out"] = torch.empty_like(st["q"])
        st["k_out"] = torch.empty_like(st["k"]) if c["kv"] else None
        return st
    page = c["page"]
    if k == "append":
        b, t, starts, new = c["batch"], c["tokens"], _starts(c), _new(c)
        # the sizes of tokens differ, so that some pages get a larger scale
        for x in ("k", "v"):
            st[x] = (normal(b, t, c["kv"], c["dh"]) * torch.exp(0.5 * normal(b, t, 1, 1))).to(dt)
        counts = [_pages_of(s + n, page) for s, n in zip(starts, new)]
        n_pages, width = sum(counts) + 3, max(counts) + 1
        st["pool"] = _filled(c, normal, n_pages)
        st["table"] = ints(_numbered(torch.randperm(n_pages, generator=cpu).tolist(), counts, width))
        st["starts"], st["new"] = ints(starts), ints(new)
        return st
    if k == "attn":
        lens = _lengths(c)
        counts, shared = [_pages_of(n, page) for n in lens], c["shared"] // page
        n_pages = sum(counts) - shared * (c["batch"] - 1) + 2
        st["pool"] = _filled(c, normal, n_pages)
        st["table"] = ints(_numbered(torch.randperm(n_pages, generator=cpu).tolist(), counts, max(counts), shared))
        st["lens"] = ints(lens)
        st["q"] = normal(c["batch"], c["rows"], c["heads"], c["dh"]).to(dt)
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:3], device=DEV)
        return st
    held, n_pages = _held(c), _pool_pages(c)
    counts = [_pages_of(n, page) for n in held]
    st["pool"] = _filled(c, normal, c["layers"], n_pages)
    order = torch.randperm(n_pages, generator=cpu).tolist()
    st["table"], st["lens"] = ints(_numbered(order, counts, _table_pages(c))), ints(held)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[order[:sum(counts)]] = 1
    st["refs"] = refs.to(DEV)
    if k == "fork":
        parents = _parents(c)
        st["parents"] = ints(parents)
        st["new_lens"] = ints([held[p] + c["grow"] for p in parents])
    for x in ("table", "lens", "refs"):
        st[x + "_out"] = torch.empty_like(st[x])
    st["count"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_norm(c, x, w, cos, sin):
    rot = c["rot"]
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * (w.float() + 1 if c["offset"] else w.float())
    r = y[..., :rot]
    if c["layout"] == "half":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([r, y[..., rot:]], -1).to(x.dtype)


def _run_norm(st):
    c = st["case"]
    f = 1e4 ** (-torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64) / c["rot"])
    angle = st["pos"].double()[..., None, None] * f
    cos, sin = angle.cos().float(), angle.sin().float()
    out = {"q": _plain_norm(c, st["q"], st["qw"], cos, sin)}
    if st["k"] is not None:
        out["k"] = _plain_norm(c, st["k"], st["kw"], cos, sin)
    return out


def _natural(codes, of_keys):
    """[...][kv][D / 16][slots][16] or [...][kv][slots / 16][D][16] -> [...][kv][slots][D]"""
    x = codes.transpose(-3, -2) if of_keys else codes.transpose(-2, -1)
    return x.flatten(-2) if of_keys else x.flatten(-3, -2)


def _in_pieces(x, of_keys):
    """The way back."""
    return x.unflatten(-1, (-1, 16)).transpose(-3, -2) if of_keys else x.unflatten(-2, (-1, 16)).transpose(-2, -1)


def _append_one(st, x, codes, scale, of_keys):
    c = st["case"]
    page, code = c["page"], c["code"]
    top = CODES[code][1]
    start, n = st["starts"].long(), st["new"].long()
    count = (c["tokens"] + page - 2) // page + 1  # pages that a sequence's new tokens touch at most
    first = start // page
    number = first[:, None] + torch.arange(count, device=DEV)  # [B][count] in the table
    touched = (number * page < (start + n)[:, None]) & (n > 0)[:, None]
    at = st["table"].gather(1, number.clamp(max=st["table"].shape[1] - 1)).long()[touched]  # pages, one after the other
    slot = (number * page)[..., None] + torch.arange(page, device=DEV)  # [B][count][page]
    token = slot - start[:, None, None]
    fresh = ((token >= 0) & (token < n[:, None, None]))[touched][:, None, :, None]  # [m][1][page][1]
    older = (token < 0)[touched][:, None, :, None]
    row = torch.arange(c["batch"], device=DEV)[:, None].expand(-1, count)[touched]
    y = x[row[:, None], token[touched].clamp(0, c["tokens"] - 1)].float().transpose(1, 2)  # [m][kv][page][D]
    amax = torch.where(fresh, y, 0.0).abs().amax((-2, -1))
    had = older.any(-2)[:, :, 0]
    old = scale[at]
    new = torch.where(had & (amax <= top * old), old, _scale_of(amax, code))
    new = torch.where(had & torch.isnan(old), old, new)
    was = _natural(codes.view(torch.uint8)[at].view(codes.dtype), of_keys)
    kept = torch.where((new == old)[..., None, None], was.float(), was.float() * (old / new)[..., None, None])
    fine = ~torch.isnan(new)[..., None, None]
    got = _coded(torch.where(fresh, torch.where(fine, y / new[..., None, None], 0.0), kept), code)
    got = torch.where(fresh | (older & fine), got.view(torch.uint8), was.contiguous().view(torch.uint8))
    codes.view(torch.uint8)[at] = _in_pieces(got, of_keys)
    scale[at] = new


def _run_append(st):
    ck, cv, sk, sv = st["pool"]
    _append_one(st, st["k"], ck, sk, True)
    _append_one(st, st["v"], cv, sv, False)
    return {"k": ck, "v": cv, "k_scale": sk, "v_scale": sv}


def _values(codes, scale, table, of_keys):
    """The values of the pages of each table row: [B][kv][slots][D]"""
    at = table.clamp(min=0).long()
    x = codes.view(torch.uint8)[at].view(codes.dtype).float() * scale[at][..., None, None, None]
    return _natural(x, of_keys).transpose(1, 2).flatten(2, 3)


def _run_attn(st):
    c = st["case"]
    B, R, nh, kv, dh = (c[x] for x in ("batch", "rows", "heads", "kv", "dh"))
    ck, cv, sk, sv = st["pool"]
    q = st["q"].float() * dh ** -0.5
    q = q.view(B, R, kv, nh // kv, dh).permute(0, 2, 1, 3, 4).reshape(B, kv, -1, dh)  # rows of one KV head side by side
    s = q @ _values(ck, sk, st["table"], True).transpose(2, 3)
    j, n = torch.arange(s.shape[-1], device=DEV), st["lens"].view(B, 1, 1, 1)
    see = j < n
    if c["causal"]:
        p = n - R + (torch.arange(s.shape[2], device=DEV) // (nh // kv)).view(1, 1, -1, 1)
        see = see & (j <= p)
        if c["window"]:
            see = see & ((j > p - c["window"]) | (j < c["sinks"]))
    s = s.masked_fill(~see, NEG_INF)
    m = s.amax(-1, keepdim=True)
    m = m.masked_fill(m == NEG_INF, 0.0)  # a row that sees nothing
    s = torch.exp(s - m)
    total = s.sum(-1, keepdim=True)
    v = torch.where((j < n).transpose(2, 3), _values(cv, sv, st["table"], False), 0.0)
    o = torch.where(total > 0, (s @ v) / total, 0.0)
    lse = m + torch.log(total)
    rows = lambda x: x.view(B, kv, R, nh // kv, -1).permute(0, 2, 1, 3, 4).reshape(B, R, nh, -1)  # noqa: E731
    return {"out": rows(o).to(st["q"].dtype), "lse": rows(lse)[..., 0]}


def _counted(refs, table, lens, page, by):
    """refs with `by` added for each page that the rows hold."""
    n = refs.shape[0]
    held = torch.arange(table.shape[1], device=DEV) < ((lens + page - 1) // page)[:, None]
    at = torch.where(held, table, n).long().flatten()
    return torch.cat([refs, refs.new_zeros(1)]).index_add(0, at, torch.full_like(at, by, dtype=torch.int32))[:n]


def _plain_resize(c, st, table, lens, refs):
    page, n_pages = c["page"], refs.shape[0]
    new = st["new_lens"]
    a, b = (lens + page - 1) // page, (new + page - 1) // page
    grows = new > lens
    last = table.gather(1, (a - 1).clamp(min=0)[:, None].long())[:, 0]
    copied = grows & (lens % page != 0) & (refs[last.clamp(min=0).long()] > 1)
    need = torch.where(grows, b - a, 0) + copied.int()
    upto = need.cumsum(0)
    free = torch.sort((refs > 0).int(), stable=True).indices  # free pages first, in ascending order
    n_free = (refs <= 0).sum()
    served = (need == 0) | (upto <= n_free)
    first = upto - need
    e = torch.arange(table.shape[1], device=DEV)
    nth = torch.where(copied[:, None] & (e == (a - 1)[:, None]), first[:, None], (first + copied.int() - a)[:, None] + e)
    fresh = ((e >= a[:, None]) & (e < b[:, None])) | (copied[:, None] & (e == (a - 1)[:, None]))
    fresh = fresh & grows[:, None] & served[:, None]
    taken = torch.where(fresh, free[nth.clamp(0, n_pages - 1)].int(), table)
    taken = torch.where((e >= b[:, None]) & (e < a[:, None]), -1, taken)
    now = torch.where(served, new, lens)
    moved = copied & served
    src, dst = last[moved].long(), taken.gather(1, (a - 1).clamp(min=0)[:, None].long())[:, 0][moved].long()
    _move(st, src, dst)
    refs = _counted(_counted(refs, table, lens, page, -1), taken, now, page, 1)
    return taken, now, refs, (upto[-1:] - n_free).clamp(min=0).int()


def _move(st, src, dst):
    codes, scales = [x.view(torch.uint8) for x in st["pool"][:2]], st["pool"][2:]
    codes[0][:, dst], codes[1][:, dst] = codes[0][:, src], codes[1][:, src]
    scales[0][:, dst], scales[1][:, dst] = scales[0][:, src], scales[1][:, src]


def _pool_out(st):
    return dict(zip(("k", "v", "k_scale", "v_scale"), st["pool"]))


def _run_fork(st):
    c = st["case"]
    page, parents = c["page"], st["parents"].long()
    table, lens = st["table"][parents], st["lens"][parents]
    refs = _counted(_counted(st["refs"], st["table"], st["lens"], page, -1), table, lens, page, 1)
    table, lens, refs, short = _plain_resize(c, st, table, lens, refs)
    return {"table": table, "lens": lens, "refs": refs, "count": short, **_pool_out(st)}


def _run_compact(st):
    refs = st["refs"]
    n = refs.shape[0]
    live = refs > 0
    n_live = live.sum()
    at = torch.arange(n, device=DEV)
    src, dst = (live & (at >= n_live)).nonzero()[:, 0], (~live & (at < n_live)).nonzero()[:, 0]
    to = at.clone()
    to[src] = dst
    table = torch.where(st["table"] >= 0, to[st["table"].clamp(min=0).long()].int(), st["table"])
    out = refs.clone()
    out[dst], out[src] = refs[src], 0
    _move(st, src, dst)
    return {"table": table, "refs": out, "count": n_live.view(1).int(), **_pool_out(st)}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own(st):
    from paper_2607_12659_amd import cache_ops as ops
    c, k = st["case"], st["case"]["kind"]
    if k == "norm":
        q, kk = ops.norm_rope(st["q"], st["k"], st["pos"], q_weight=st["qw"], k_weight=st["kw"] if c["kv"] else None, eps=EPS,
                              unit_offset=c["offset"], rot_dim=c["rot"], layout=c["layout"], base=1e4, q_out=st["q_out"],
                              k_out=st["k_out"])
        return {"q": q} if kk is None else {"q": q, "k": kk}
    pool = ops.Pool(*st["pool"])
    if k == "append":
        ops.append(pool, st["table"], st["starts"], st["k"], st["v"], n_new=st["new"])
        return _pool_out(st)
    if k == "attn":
        out, lse = ops.attention(st["q"], pool, st["table"], st["lens"], causal=c["causal"], window=c["window"], sinks=c["sinks"],
                                 out=st["out"], lse=st["lse"])
        return {"out": out, "lse": lse}
    out = {"table_out": st["table_out"], "refs_out": st["refs_out"]}
    if k == "compact":
        ops.compact(st["table"], st["refs"], pool, n_live=st["count"], **out)
        return {"table": st["table_out"], "refs": st["refs_out"], "count": st["count"], **_pool_out(st)}
    ops.reorder(st["table"], st["lens"], st["refs"], st["parents"], c["page"], lens_out=st["lens_out"], **out)
    ops.resize(st["table_out"], st["lens_out"], st["refs_out"], st["new_lens"], pool, short=st["count"])
    return {"table": st["table_out"], "lens": st["lens_out"], "refs": st["refs_out"], "count": st["count"], **_pool_out(st)}


_PLAIN = {"norm": _run_norm, "append": _run_append, "attn": _run_attn, "fork": _run_fork, "compact": _run_compact}


@torch.no_grad()
def run(st):
    if own:
        return _own(st)
    return _PLAIN[st["case"]["kind"]](st)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_norm(c, x, w, pos):
    """Pairs of the normed head as complex numbers, turned by the position's angle."""
    rot = c["rot"]
    y = x.double()
    y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / c["dh"] + EPS) * (w.double() + (1.0 if c["offset"] else 0.0))
    f = torch.tensor([math.pow(1e4, -2 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device=DEV)
    angle = pos.double()[:, :, None, None] * f
    turn = torch.polar(torch.ones_like(angle), angle)
    if c["layout"] == "half":
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * turn
        head = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.complex(y[..., 0:rot:2].contiguous(), y[..., 1:rot:2].contiguous()) * turn
        head = torch.view_as_real(z).flatten(-2)
    return torch.cat([head, y[..., rot:]], -1)


def _exact_codes(y, code):
    """Nearest codes, ties to even."""
    if code == "int8":
        return torch.round(y)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _exact_append(st, x, codes, scale, of_keys):
    c = st["case"]
    page, code, top = c["page"], c["code"], CODES[c["code"]][1]
    out, s_out = codes.to(torch.float32).double(), scale.double()
    table = st["table"].tolist()
    for b, (start, n) in enumerate(zip(_starts(c), _new(c))):
        for number in range(start // page, _pages_of(start + n, page)):
            at, lo, hi = table[b][number], max(start, number * page), min(start + n, (number + 1) * page)
            y = x[b, lo - start:hi - start].double().transpose(0, 1)  # [kv][slots][D]
            plain = out[at].permute((0, 2, 1, 3) if of_keys else (0, 1, 3, 2)).reshape(c["kv"], page, -1).clone()
            older = lo - number * page
            for h in range(c["kv"]):
                a, s = float(y[h].abs().max()), float(s_out[at, h])
                if older == 0 or a > top * s:
                    t = 2.0 ** max(-126, math.ceil(math.log2(a / top)) if a else -126)
                    if older:
                        plain[h, :older] = _exact_codes(plain[h, :older] * (s / t), code)
                    s = t
                plain[h, older:older + hi - lo] = _exact_codes(y[h] / s, code)
                s_out[at, h] = s
            if of_keys:
                out[at] = plain.reshape(c["kv"], page, -1, 16).permute(0, 2, 1, 3)
            else:
                out[at] = plain.reshape(c["kv"], page // 16, 16, -1).permute(0, 1, 3, 2)
    return out, s_out


def _exact_attn(st):
    c = st["case"]
    R, nh, kv, dh, page = (c[x] for x in ("rows", "heads", "kv", "dh", "page"))
    per = nh // kv
    ck, cv, sk, sv = st["pool"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(out.shape[:3], NEG_INF, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(c)):
        at = st["table"][b, :_pages_of(n, page)].tolist()
        at = torch.tensor(at, device=DEV)
        j = torch.arange(n, device=DEV)[None, :]
        p = n - R + torch.arange(R, device=DEV)[:, None]
        hide = torch.zeros((R, n), dtype=torch.bool, device=DEV)
        if c["causal"]:
            hide = j > p
            if c["window"]:
                hide = hide | ((j <= p - c["window"]) & (j >= c["sinks"]))
        for h in range(kv):
            K = ck.view(torch.uint8)[at, h].view(ck.dtype).to(torch.float32).double() * sk[at, h].double()[:, None, None, None]
            V = cv.view(torch.uint8)[at, h].view(cv.dtype).to(torch.float32).double() * sv[at, h].double()[:, None, None, None]
            K = K.permute(0, 2, 1, 3).reshape(-1, dh)[:n]  # [slots][D]
            V = V.permute(0, 1, 3, 2).reshape(-1, dh)[:n]
            for r in range(h * per, (h + 1) * per):
                s = st["q"][b, :, r].double() @ K.T / math.sqrt(dh)
                s = s.masked_fill(hide, NEG_INF)
                lse[b, :, r] = torch.logsumexp(s, -1)
                out[b, :, r] = torch.nan_to_num(torch.softmax(s, -1), nan=0.0) @ V
    return {"out": out, "lse": lse}


def _exact_pages(st):
    """Sequence by sequence, page by page."""
    c = st["case"]
    page, moves = c["page"], []
    table, lens, refs = st["table"].tolist(), st["lens"].tolist(), st["refs"].tolist()
    n_pages = len(refs)
    if c["kind"] == "compact":
        n_live = sum(r > 0 for r in refs)
        holes = [p for p in range(n_live) if refs[p] <= 0]
        for p in range(n_live, n_pages):
            if refs[p] > 0:
                to = holes.pop(0)
                moves.append((p, to))
                refs[to], refs[p] = refs[p], 0
        new = dict(moves)
        out = {"table": [[new.get(p, p) for p in row] for row in table], "refs": refs, "count": [n_live]}
    else:
        old = [row[:_pages_of(n, page)] for row, n in zip(table, lens)]
        rows = [list(old[p]) for p in _parents(c)]
        refs = [0] * n_pages
        for row in rows:
            for p in row:
                refs[p] += 1
        lens, before = [lens[p] for p in _parents(c)], list(refs)
        free, missing, wanted = [p for p in range(n_pages) if refs[p] == 0], 0, 0
        n_free = len(free)
        for i, n in enumerate(lens):
            m = n + c["grow"]
            copy = m > n and n % page != 0 and before[rows[i][-1]] > 1
            need = _pages_of(m, page) - len(rows[i]) + copy
            wanted += need
            if need and wanted > n_free:
                missing = wanted - n_free
                continue
            if copy:
                moves.append((rows[i][-1], free[0]))
                refs[rows[i][-1]] -= 1
                rows[i][-1] = free.pop(0)
                refs[rows[i][-1]] += 1
            while len(rows[i]) < _pages_of(m, page):
                rows[i].append(free.pop(0))
                refs[rows[i][-1]] += 1
            lens[i] = m
        out = {"table": [r + [-1] * (_table_pages(c) - len(r)) for r in rows], "lens": lens, "refs": refs, "count": [missing]}
    out = {k: torch.tensor(v, dtype=torch.int32) for k, v in out.items()}
    pool = [x.view(torch.uint8) if x.dtype != torch.float32 else x for x in st["pool"]]
    for src, dst in moves:
        for x in pool:
            x[:, dst] = x[:, src]
    out["k_scale"], out["v_scale"] = st["pool"][2].double(), st["pool"][3].double()
    out["k"], out["v"] = (None, None) if c["code"] == "int8" else (x.to(torch.float32).double() for x in st["pool"][:2])
    return out


@torch.no_grad()
def exact(c, seed):
    st, k = prepare(c, seed), c["kind"]
    if k == "norm":
        out = {"q": _exact_norm(c, st["q"], st["qw"], st["pos"])}
        if st["k"] is not None:
            out["k"] = _exact_norm(c, st["k"], st["kw"], st["pos"])
        return out
    if k == "append":
        (ck, cv, sk, sv) = st["pool"]
        if c["batch"] * c["kv"] * _pages_of(c["tokens"], c["page"]) > 20000:
            return None
        (K, Ks), (V, Vs) = _exact_append(st, st["k"], ck, sk, True), _exact_append(st, st["v"], cv, sv, False)
        return {"k": K, "v": V, "k_scale": Ks, "v_scale": Vs}
    return _exact_attn(st) if k == "attn" else _exact_pages(st)
