"""Operators of a prefix cache that are timed and compared: rotary positions,
attention of a batch that shares one prefix, the weight that its queries lay
on each prefix slot, and eviction of the lightest slots.

Shapes are the repository's own (the pi0.5 expert's eight heads of 256 over one
KV head, prefixes of 816 and 1600 tokens, chunks of 50 actions, the tiny fp32
expert) and generic ones (32 heads over 8 KV heads of 128, long caches).
``run`` computes the operators in elementary torch operations, or through
``paper_2607_12659_amd.prefix_ops`` where ``own`` is true.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
NEG_INF = float("-inf")


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _rope(name, batch, tokens, heads, kv, dh, rot, layout="half", scaling="none", factor=1.0, far=0, dtype="bf16"):
    """far: positions are drawn below it (0: consecutive ones)."""
    return {"name": name, "kind": "rope", "batch": batch, "tokens": tokens, "heads": heads, "kv": kv, "dh": dh, "rot": rot,
            "layout": layout, "scaling": scaling, "factor": factor, "far": far, "dtype": dtype}


def _attn(name, groups, group, rows, heads, kv, dh, prefix, suffix, causal=False, ragged=False, dtype="bf16"):
    return {"name": name, "kind": "attn", "groups": groups, "group": group, "rows": rows, "heads": heads, "kv": kv, "dh": dh,
            "prefix": prefix, "suffix": suffix, "causal": causal, "ragged": ragged, "dtype": dtype}


def _weight(name, groups, group, rows, heads, kv, dh, prefix, ragged=False, dtype="bf16"):
    return {"name": name, "kind": "weight", "groups": groups, "group": group, "rows": rows, "heads": heads, "kv": kv, "dh": dh,
            "prefix": prefix, "suffix": rows, "ragged": ragged, "dtype": dtype}


def _evict(name, seqs, kv, dh, slots, keep, first=0, last=0, ragged=False, dtype="bf16"):
    return {"name": name, "kind": "evict", "seqs": seqs, "kv": kv, "dh": dh, "slots": slots, "keep": keep, "first": first,
            "last": last, "ragged": ragged, "dtype": dtype}


def listed():
    return [
        # one new token of one sequence behind its prefix: queries and key of one layer, latency-bound
        _rope("rope-token", 1, 1, 8, 1, 256, 256, far=4096),
        # the queries and keys of one layer of an eight-rollout prefill
        _rope("rope-prefill-b8", 8, 816, 8, 1, 256, 256),
        # a long context past the trained one: half of each head rotated in neighbouring pairs, fp32, positions far out
        _rope("rope-far-f32", 2, 4099, 32, 8, 128, 64, "interleaved", "parts", 8.0, 131072, "f32"),
        # one decoded token of each of four candidates of one observation
        _attn("attn-token-g4", 1, 4, 1, 8, 1, 256, 816, 51, ragged=True),
        # eight candidate action chunks denoised against one observation
        _attn("attn-chunk-g8", 1, 8, 50, 8, 1, 256, 816, 50),
        # an evaluation batch: four observations of six images, sixteen candidates of each
        _attn("attn-chunk-g64-p1600", 4, 16, 50, 8, 1, 256, 1600, 50, ragged=True),
        # sixty-four samples decoded from one very long prompt, each with its own tail of up to 512 tokens
        _attn("attn-decode-p65536", 1, 64, 1, 32, 8, 128, 65536, 512, ragged=True),
        # the tiny fp32 expert's head size: short causal tails behind prefixes of odd lengths, one of them empty
        _attn("attn-f32-odd", 3, 5, 7, 4, 2, 64, 333, 13, causal=True, ragged=True, dtype="f32"),
        # what the chunks of eight candidates look at, slot by slot
        _weight("weight-chunk-g8", 1, 8, 50, 8, 1, 256, 816),
        # the same for sixty-four samples of one very long prompt
        _weight("weight-decode-p65536", 1, 64, 1, 32, 8, 128, 65536),
        # every layer's prefix of one rollout cut to half, the first and last tokens protected
        _evict("evict-l18-p816", 18, 1, 256, 816, 408, 4, 48),
        # eight rollouts' long prefixes of unequal lengths, in all layers, cut to a quarter
        _evict("evict-l18-b8-p4096", 144, 1, 256, 4096, 1024, 4, 64, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# what the listed cases of each kind cost at most; a drawn case is cut until it costs no more
_MOST_BYTES = {"rope": 335e6, "evict": 300e6}
_MOST_FLOPS = {("attn", "bf16"): 6e10, ("attn", "f32"): 1e10, ("weight", "bf16"): 3e10, ("weight", "f32"): 1e10}


def draw(rng):
    kind = rng.choice(["rope", "attn", "attn", "weight", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "rope":
        heads, kv = rng.choice([(8, 1), (4, 2), (32, 8), (7, 0)])
        dh = rng.choice([64, 128, 256])
        c = _rope("", _log(rng, 1, 16), _log(rng, 1, 8192), heads, kv, dh, dh // rng.choice([1, 1, 2, 4]),
                  rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "base", "parts"]), rng.choice([2.0, 5.5, 32.0]),
                  rng.choice([0, _log(rng, 1000, 1000000)]), dtype)
        while work(c)["bytes"] > _MOST_BYTES[kind]:
            c["tokens"] = c["tokens"] * 2 // 3
    elif kind == "evict":
        slots = _log(rng, 16, 16384)
        keep = max(1, int(slots * rng.uniform(0.05, 0.95)))
        first = rng.randint(0, min(8, keep // 2))
        c = _evict("", _log(rng, 1, 160), rng.choice([1, 1, 2, 8]), rng.choice([64, 128, 256]), slots, keep, first,
                   rng.randint(0, min(64, keep - first)), rng.random() < 0.5, dtype)
        while work(c)["bytes"] > _MOST_BYTES[kind]:
            c["seqs"] = c["seqs"] * 2 // 3
    else:
        heads, kv = rng.choice([(8, 1), (8, 1), (4, 2), (32, 8), (6, 6)])
        args = (_log(rng, 1, 6), _log(rng, 1, 64), rng.choice([1, 1, _log(rng, 1, 64)]), heads, kv, rng.choice([64, 128, 256]),
                _log(rng, 1, 65536))
        ragged = rng.random() < 0.5
        if kind == "attn":
            suffix = rng.choice([0, args[2], _log(rng, 1, 512)])
            c = _attn("", *args, suffix, suffix > 0 and rng.random() < 0.5, ragged, dtype)
        else:
            c = _weight("", *args, ragged, dtype)
        while work(c)["flops"] > _MOST_FLOPS[kind, dtype]:
            cut = "group" if c["group"] > 1 else "prefix"
            c[cut] = c[cut] * 2 // 3
    c.pop("name")
    return c


# ---------------------------------------------------------------------------
# lengths, the same for every seed
# ---------------------------------------------------------------------------
def _prefix_lens(c):
    """Valid prefix slots of each group: ragged ones fall from all to none in equal steps."""
    g, p = c["groups"], c["prefix"]
    return [p - (p * i) // max(1, g - 1) if i else p for i in range(g)] if c["ragged"] else [p] * g


def _suffix_lens(c):
    """Valid keys of each rollout's own tail: ragged ones are spread between one and all."""
    b, s = c["groups"] * c["group"], c["suffix"]
    return [s - (s * ((i * 7) % b)) // b for i in range(b)] if c["ragged"] else [s] * b


def _evict_lens(c):
    """Valid slots of each sequence: ragged ones reach from a little under `keep` to all."""
    n, p = c["seqs"], c["slots"]
    lo = max(0, c["keep"] - 3)
    return [p - ((p - lo) * ((i * 5) % n)) // n for i in range(n)] if c["ragged"] else [p] * n


def work(c):
    es = 2 if c["dtype"] == "bf16" else 4
    k = c["kind"]
    if k == "rope":
        n = c["batch"] * c["tokens"]
        return {"bytes": 2 * n * (c["heads"] + c["kv"]) * c["dh"] * es + 4 * n, "flops": 3 * n * (c["heads"] + c["kv"]) * c["rot"]}
    if k == "evict":
        lens = _evict_lens(c)
        kept = sum(min(n, c["keep"]) for n in lens) * c["kv"]
        return {"bytes": kept * (4 * c["dh"] * es + 8) + 4 * c["kv"] * sum(lens), "flops": 0}
    rows = c["group"] * c["rows"] * c["heads"]  # of one group
    pre, suf = _prefix_lens(c), _suffix_lens(c) if k == "attn" else []
    once = sum(pre) * c["kv"] * c["dh"] * es
    q = c["groups"] * rows * c["dh"] * es
    if k == "weight":
        return {"bytes": once + q + 4 * c["groups"] * rows + 8 * sum(pre) * c["kv"], "flops": 2 * rows * sum(pre) * c["dh"]}
    return {"bytes": 2 * once + 2 * sum(suf) * c["kv"] * c["dh"] * es + 2 * q + 4 * c["groups"] * rows,
            "flops": 4 * c["dh"] * (rows * sum(pre) + c["rows"] * c["heads"] * sum(suf))}


# ---------------------------------------------------------------------------
# inputs from the seed
# ---------------------------------------------------------------------------
def prepare(c, seed):
    """Inputs and the buffers that a serving program keeps for the outputs (caches and weights start at zero)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + 29)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV).to(dt)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=DEV)

    st, k = {"case": c}, c["kind"]
    if k == "rope":
        b, n = c["batch"], c["tokens"]
        st["q"] = normal(b, n, c["heads"], c["dh"])
        st["k"] = normal(b, n, c["kv"], c["dh"]) if c["kv"] else None
        if c["far"]:
            st["pos"] = torch.randint(0, c["far"], (b, n), generator=g, device=DEV).to(torch.int32)
        else:
            st["pos"] = torch.arange(n, device=DEV, dtype=torch.int32).expand(b, n).contiguous()
        st["q_out"] = torch.empty_like(st["q"])
        st["k_out"] = torch.empty_like(st["k"]) if c["kv"] else None
        return st
    if k == "evict":
        n, p, kv, dh = c["seqs"], c["slots"], c["kv"], c["dh"]
        st["k"], st["v"] = normal(n, p, kv, dh), normal(n, p, kv, dh)
        # accumulated weights: a few heavy slots, most light, many of them equal
        st["w"] = torch.round(torch.exp(1.5 * torch.randn((n, kv, p), generator=g, device=DEV)) * 16) / 16
        st["lens"] = ints(_evict_lens(c))
        st["k_out"] = torch.zeros((n, c["keep"], kv, dh), dtype=dt, device=DEV)
        st["v_out"] = torch.zeros_like(st["k_out"])
        st["w_out"] = torch.zeros((n, kv, c["keep"]), device=DEV)
        st["index"] = torch.zeros((n, kv, c["keep"]), dtype=torch.int32, device=DEV)
        return st
    G, R, H, nh, kv, dh, P, S = (c[x] for x in ("groups", "group", "rows", "heads", "kv", "dh", "prefix", "suffix"))
    st["q"] = normal(G * R, H, nh, dh)
    st["kp"] = normal(G, P, kv, dh)
    st["plen"] = ints(_prefix_lens(c))
    if k == "weight":
        # the log-sum of a row's scores, as the attention hands it over: unit normal scores over prefix and tail
        keys = st["plen"].float().repeat_interleave(R).view(-1, 1, 1) + S
        st["lse"] = torch.log(keys) + 0.5 + 0.05 * torch.randn((G * R, H, nh), generator=g, device=DEV)
        st["w"] = torch.rand((G, kv, P), generator=g, device=DEV)
        st["w_out"] = torch.zeros((G, kv, P), device=DEV)
        return st
    st["vp"] = normal(G, P, kv, dh)
    st["ks"], st["vs"] = (normal(G * R, S, kv, dh), normal(G * R, S, kv, dh)) if S else (None, None)
    st["slen"] = ints(_suffix_lens(c)) if S else None
    st["out"] = torch.empty_like(st["q"])
    st["lse"] = torch.empty((G * R, H, nh), device=DEV)
    return st


DECAY = 0.75
BETA_FAST, BETA_SLOW, TRAINED, AMPLITUDE = 32.0, 1.0, 4096, 1.125


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _inverse_periods(c):
    """Angle per position of each pair, in 64 bits."""
    rot, s = c["rot"], c["factor"]
    base = 1e4 * s ** (rot / (rot - 2)) if c["scaling"] == "base" else 1e4
    f = base ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    if c["scaling"] == "linear":
        return f / s
    if c["scaling"] == "parts":
        turns = TRAINED * f / (2 * math.pi)
        keep = ((turns - BETA_SLOW) / (BETA_FAST - BETA_SLOW)).clamp(0, 1)
        return f * (keep + (1 - keep) / s)
    return f


def _plain_rope(c, x, cos, sin):
    rot = c["rot"]
    r = x[..., :rot].float()
    if c["layout"] == "half":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([y.to(x.dtype), x[..., rot:]], -1)


def _run_rope(st):
    c = st["case"]
    amp = AMPLITUDE if c["scaling"] == "parts" else 1.0
    angle = st["pos"].double()[..., None, None] * _inverse_periods(c)
    cos, sin = (amp * angle.cos()).float(), (amp * angle.sin()).float()
    out = {"q": _plain_rope(c, st["q"], cos, sin)}
    if st["k"] is not None:
        out["k"] = _plain_rope(c, st["k"], cos, sin)
    return out


def _grouped(q, n, kv):
    """[n * r][H][heads][D] -> [n][kv][r * H * heads / kv][D]: the rows of one KV head side by side."""
    b, h, nh, d = q.shape
    return q.view(n, b // n * h, kv, nh // kv, d).permute(0, 2, 1, 3, 4).reshape(n, kv, -1, d)


def _run_attn(st):
    c = st["case"]
    G, R, H, nh, kv, dh, P, S = (c[x] for x in ("groups", "group", "rows", "heads", "kv", "dh", "prefix", "suffix"))
    B, g = G * R, nh // kv
    q = st["q"].float() * dh ** -0.5
    kp, vp = (st[x].float().transpose(1, 2) for x in ("kp", "vp"))  # [G][kv][P][D]
    sp = _grouped(q, G, kv) @ kp.transpose(2, 3)
    valid = torch.arange(P, device=DEV) < st["plen"].view(G, 1, 1, 1)
    sp = sp.masked_fill(~valid, NEG_INF)
    m = sp.amax(-1, keepdim=True)  # [G][kv][R * H * g][1]
    if S:
        ks, vs = (st[x].float().transpose(1, 2) for x in ("ks", "vs"))
        ss = _grouped(q, B, kv) @ ks.transpose(2, 3)  # [B][kv][H * g][S]
        last = st["slen"].view(B, 1, 1, 1) - 1
        if c["causal"]:
            last = last - (H - 1) + (torch.arange(H * g, device=DEV) // g).view(1, 1, -1, 1)
        ss = ss.masked_fill(torch.arange(S, device=DEV) > last, NEG_INF)
        # the rollouts' rows in the order of the group's
        ms = ss.amax(-1, keepdim=True).view(G, R, kv, H * g, 1).transpose(1, 2).reshape(G, kv, -1, 1)
        m = torch.maximum(m, ms)
    m = m.masked_fill(m == NEG_INF, 0.0)  # a row that sees nothing
    ep = torch.exp(sp - m)
    total, o = ep.sum(-1, keepdim=True), ep @ vp
    if S:
        mb = m.view(G, kv, R, H * g, 1).transpose(1, 2).reshape(B, kv, H * g, 1)
        es = torch.exp(ss - mb)
        back = lambda x: x.view(G, R, kv, H * g, -1).transpose(1, 2).reshape(G, kv, R * H * g, -1)  # noqa: E731
        total, o = total + back(es.sum(-1, keepdim=True)), o + back(es @ vs)
    o = torch.where(total > 0, o / total, 0.0)
    lse = m + torch.log(total)
    rows = lambda x: x.view(G, kv, R * H, g, -1).permute(0, 2, 1, 3, 4).reshape(B, H, nh, -1)  # noqa: E731
    return {"out": rows(o).to(st["q"].dtype), "lse": rows(lse)[..., 0]}


def _run_weight(st):
    c = st["case"]
    G, kv, P = c["groups"], c["kv"], c["prefix"]
    q = _grouped(st["q"].float() * c["dh"] ** -0.5, G, kv)
    lse = _grouped(st["lse"][..., None], G, kv)
    p = torch.exp(q @ st["kp"].float().permute(0, 2, 3, 1) - lse)
    w = DECAY * st["w"] + p.sum(2)
    return {"weight": torch.where(torch.arange(P, device=DEV) < st["plen"].view(G, 1, 1), w, st["w_out"])}


def _run_evict(st):
    c = st["case"]
    keep = c["keep"]
    w, lens = st["w"], st["lens"].view(-1, 1, 1)
    at = torch.arange(c["slots"], device=DEV)
    level = (at < lens).int() + ((at < lens) & ((at < c["first"]) | (at >= lens - c["last"]))).int()
    # by weight, then by level, the earlier order kept among equals: protected slots, valid ones, the rest
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    rank = torch.sort(level.expand_as(w).gather(-1, order), dim=-1, descending=True, stable=True).indices
    chosen = order.gather(-1, rank)[..., :keep]
    chosen = torch.where(chosen < lens, chosen, c["slots"]).sort(-1).values
    n_new = st["lens"].clamp(max=keep)
    there = chosen < c["slots"]
    src = chosen.clamp(max=c["slots"] - 1)
    rows = src.transpose(1, 2)[..., None].expand(-1, -1, -1, c["dh"])
    mask = there.transpose(1, 2)[..., None]
    return {"k": torch.where(mask, st["k"].gather(1, rows), st["k_out"]), "v": torch.where(mask, st["v"].gather(1, rows), st["v_out"]),
            "weight": torch.where(there, w.gather(-1, src), st["w_out"]),
            "index": torch.where(there, chosen.int(), st["index"]), "lens": n_new}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own(st):
    from paper_2607_12659_amd import prefix_ops as ops
    c, k = st["case"], st["case"]["kind"]
    if k == "rope":
        parts = c["scaling"] == "parts"
        q, kk = ops.rope(st["q"], st["k"], st["pos"], rot_dim=c["rot"], layout=c["layout"], base=1e4, scaling=c["scaling"],
                         factor=c["factor"], trained=TRAINED, beta_fast=BETA_FAST, beta_slow=BETA_SLOW,
                         amplitude=AMPLITUDE if parts else 1.0, q_out=st["q_out"], k_out=st["k_out"])
        return {"q": q} if kk is None else {"q": q, "k": kk}
    if k == "attn":
        out, lse = ops.shared_attention(st["q"], st["kp"], st["vp"], st["ks"], st["vs"], prefix_len=st["plen"],
                                        suffix_len=st["slen"], causal=c["causal"], out=st["out"], lse=st["lse"])
        return {"out": out, "lse": lse}
    if k == "weight":
        return {"weight": ops.prefix_weight(st["q"], st["kp"], st["lse"], st["w"], prefix_len=st["plen"], decay=DECAY,
                                            out=st["w_out"])}
    index, lens = ops.evict(st["k"], st["v"], st["w"], c["keep"], lens=st["lens"], n_first=c["first"], n_last=c["last"],
                            k_out=st["k_out"], v_out=st["v_out"], weight_out=st["w_out"], index=st["index"])
    return {"k": st["k_out"], "v": st["v_out"], "weight": st["w_out"], "index": index, "lens": lens}


_PLAIN = {"rope": _run_rope, "attn": _run_attn, "weight": _run_weight, "evict": _run_evict}


@torch.no_grad()
def run(st):
    if own:
        return _own(st)
    return _PLAIN[st["case"]["kind"]](st)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _rotated64(c, x, pos):
    """Pairs as complex numbers, turned by the position's angle."""
    rot, s = c["rot"], c["factor"]
    f = []
    for i in range(rot // 2):
        if c["scaling"] == "base":
            fi = math.pow(1e4 * math.pow(s, rot / (rot - 2)), -2 * i / rot)
        else:
            fi = math.pow(1e4, -2 * i / rot)
        if c["scaling"] == "linear":
            fi /= s
        elif c["scaling"] == "parts":
            r = TRAINED * fi / (2 * math.pi)
            k = min(1.0, max(0.0, (r - BETA_SLOW) / (BETA_FAST - BETA_SLOW)))
            fi = fi * k + fi / s * (1 - k)
        f.append(fi)
    angle = pos.double()[:, :, None, None] * torch.tensor(f, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(angle, AMPLITUDE if c["scaling"] == "parts" else 1.0), angle)
    y = x.double()
    if c["layout"] == "half":
        z = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * turn
        head = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.complex(y[..., 0:rot:2], y[..., 1:rot:2]) * turn
        head = torch.view_as_real(z).flatten(-2)
    return torch.cat([head, y[..., rot:]], -1)


@torch.no_grad()
def exact(c, seed):
    st, k = prepare(c, seed), c["kind"]
    if k == "rope":
        out = {"q": _rotated64(c, st["q"], st["pos"])}
        if st["k"] is not None:
            out["k"] = _rotated64(c, st["k"], st["pos"])
        return out
    if k == "evict":
        keep, first, last = c["keep"], c["first"], c["last"]
        K, V, W, index = (st[x].double() for x in ("k_out", "v_out", "w_out", "index"))
        lens = _evict_lens(c)
        ranked = st["w"].cpu()
        for i, n in enumerate(lens):
            for h in range(c["kv"]):
                kept = list(range(n))
                if n > keep:
                    w = ranked[i, h, :n].tolist()
                    middle = sorted(range(first, n - last), key=lambda j: (-w[j], j))[:keep - first - last]
                    kept = list(range(first)) + sorted(middle) + list(range(n - last, n))
                at, m = torch.tensor(kept, dtype=torch.int64, device=DEV), len(kept)
                K[i, :m, h], V[i, :m, h] = st["k"][i, at, h].double(), st["v"][i, at, h].double()
                W[i, h, :m], index[i, h, :m] = st["w"][i, h, at].double(), at.double()
        return {"k": K, "v": V, "weight": W, "index": index.int(), "lens": torch.tensor([min(n, keep) for n in lens], dtype=torch.int32)}
    G, R, H, nh, kv, P = (c[x] for x in ("groups", "group", "rows", "heads", "kv", "prefix"))
    pre, per = _prefix_lens(c), nh // kv
    if k == "weight":
        W = st["w_out"].double()
        for g in range(G):
            for h in range(kv):
                q = st["q"][g * R:(g + 1) * R, :, h * per:(h + 1) * per].double().reshape(-1, c["dh"])
                lse = st["lse"][g * R:(g + 1) * R, :, h * per:(h + 1) * per].double().reshape(-1, 1)
                s = q @ st["kp"][g, :pre[g], h].double().T / math.sqrt(c["dh"])
                W[g, h, :pre[g]] = DECAY * st["w"][g, h, :pre[g]].double() + torch.exp(s - lse).sum(0)
        return {"weight": W}
    suf = _suffix_lens(c)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(out.shape[:3], dtype=torch.float64, device=DEV)
    for g in range(G):
        for h in range(kv):
            kp, vp = st["kp"][g, :pre[g], h].double(), st["vp"][g, :pre[g], h].double()
            for b in range(g * R, (g + 1) * R):
                keys, values, n = kp, vp, suf[b]
                if c["suffix"]:
                    keys, values = torch.cat([kp, st["ks"][b, :n, h].double()]), torch.cat([vp, st["vs"][b, :n, h].double()])
                q = st["q"][b, :, h * per:(h + 1) * per].double()
                s = torch.einsum("ihd,jd->ihj", q, keys) / math.sqrt(c["dh"])
                if c["causal"]:
                    i, j = torch.arange(H, device=DEV)[:, None, None], torch.arange(len(keys), device=DEV) - pre[g]
                    s = s.masked_fill((j >= 0) & (j > n - H + i), NEG_INF)
                if s.shape[-1]:
                    p = torch.nan_to_num(torch.softmax(s, -1), nan=0.0)
                    out[b, :, h * per:(h + 1) * per] = torch.einsum("ihj,jd->ihd", p, values)
                lse[b, :, h * per:(h + 1) * per] = torch.logsumexp(s, -1)
    return {"out": out, "lse": lse}
