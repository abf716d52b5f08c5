"""The operators of a paged 8-bit cache (include/jpi_cache.h) in plain Python and numpy, for their tests."""
import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}
E4M3 = None


def e4m3_values():
    """The value of each code: 1 sign, 4 exponent (bias 7) and 3 fraction bits, NaN where exponent and fraction are all ones."""
    global E4M3
    if E4M3 is None:
        c = np.arange(256)
        sign, e, f = np.where(c & 128, -1.0, 1.0), c >> 3 & 15, c & 7
        E4M3 = sign * np.where(e > 0, 2.0 ** (e - 7.0) * (1 + f / 8), 2.0 ** -6 * f / 8)
        E4M3[(c & 127) == 127] = np.nan
    return E4M3


def decode(codes, code):
    return codes.view(np.int8).astype(np.float64) if code == "int8" else e4m3_values()[codes.view(np.uint8)]


def encode(y, code):
    """Nearest codes of float32 values within the codes' range, ties to even; as bytes."""
    y = np.asarray(y, np.float32).astype(np.float64)
    if code == "int8":
        return np.rint(y).astype(np.int8).view(np.uint8)
    a = np.abs(y)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    a = np.rint(a / step) * step  # may be the next power of two
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    f = np.where(a < 2.0 ** -6, a * 2.0 ** 9, (e + 7) * 8 + (a / 2.0 ** e - 1) * 8)
    return (f.astype(np.int64) | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def natural(codes, of_keys):
    """[...][kv][D / 16][slots][16] or [...][kv][slots / 16][D][16] -> [...][kv][slots][D]"""
    x = np.swapaxes(codes, -3, -2) if of_keys else np.swapaxes(codes, -2, -1)
    return x.reshape(*x.shape[:-2], -1) if of_keys else x.reshape(*x.shape[:-3], -1, x.shape[-1])


def in_pieces(x, of_keys):
    if of_keys:
        return np.swapaxes(x.reshape(*x.shape[:-1], -1, 16), -3, -2)
    return np.swapaxes(x.reshape(*x.shape[:-2], -1, 16, x.shape[-1]), -2, -1)


def scale_for(a, code):
    """The least power of two, from 2^-126 on, whose multiple by the largest code reaches a."""
    e = -126
    while TOP[code] * 2.0 ** e < a:
        e += 1
    return np.float32(2.0 ** e)


def append_one(codes, scales, of_keys, code, page, table, starts, x, n_new):
    """codes (bytes) and scales of K or V change in place; x [sequences][tokens][kv][D] in float32."""
    n_pages, kv = scales.shape
    cap = table.shape[1] * page
    for s in range(len(starts)):
        start = min(max(int(starts[s]), 0), cap)
        end = min(start + min(max(int(n_new[s]), 0), x.shape[1]), cap)
        for number in range(start // page, -(-end // page)):
            lo, hi, at = max(start, number * page) - number * page, min(end, (number + 1) * page) - number * page, int(table[s, number])
            if hi <= lo or not 0 <= at < n_pages:
                continue
            t0 = number * page + lo - start
            plain = natural(codes[at], of_keys).copy()
            for h in range(kv):
                y = x[s, t0:t0 + hi - lo, h]
                old = scales[at, h]
                if not np.isfinite(y).all() or (lo > 0 and np.isnan(old)):
                    scales[at, h] = np.nan
                    plain[h, lo:hi] = 0
                    continue
                a = np.abs(y).max()
                with np.errstate(over="ignore"):
                    now = old if lo > 0 and a <= np.float32(TOP[code]) * old else scale_for(float(a), code)
                if lo > 0 and now != old:
                    plain[h, :lo] = encode(decode(plain[h, :lo], code).astype(np.float32) * (old / now), code)
                plain[h, lo:hi] = encode(y / now, code) if now != 0 else 0
                scales[at, h] = now
            codes[at] = in_pieces(plain, of_keys)


def slots(codes, scales, of_keys, code, page, row, n):
    """[kv][n][D] in 64 bits: the values of the first n slots of a table row; NaN where a number names no page."""
    kv, dim = codes.shape[1], codes.shape[2] * 16 if of_keys else codes.shape[3]
    if n == 0:
        return np.zeros((kv, 0, dim))
    at = np.asarray(row[:-(-n // page)], np.int64)
    bad = (at < 0) | (at >= len(scales))
    at = np.where(bad, 0, at)
    x = natural(decode(codes[at], code), of_keys) * np.where(bad[:, None], np.nan, scales[at].astype(np.float64))[..., None, None]
    return np.moveaxis(x, 0, 1).reshape(kv, -1, dim)[:, :n]


def seen(n, nq, causal, window, sinks):
    """[nq][n]: whether row i sees slot j."""
    j, p = np.arange(n)[None], (n - nq + np.arange(nq))[:, None]
    see = np.ones((nq, n), bool)
    if causal:
        see = j <= p
        if window:
            see = see & ((j > p - window) | (j < sinks))
    return see


def resize(table, lens, refs, new_lens, page):
    """New table, lens, refs, the pages lacking, and the copies as (from, to)."""
    table, lens, refs = table.copy(), lens.copy(), refs.copy()
    cap, n_pages, before = table.shape[1] * page, len(refs), refs.copy()
    free = [p for p in range(n_pages) if before[p] <= 0]
    wanted, copies, n_free, taken = 0, [], len(free), 0
    for s in range(len(lens)):
        old = min(max(int(lens[s]), 0), cap)
        new = old if new_lens[s] < 0 else min(int(new_lens[s]), cap)
        had, has = -(-old // page), -(-new // page)
        last = int(table[s, had - 1]) if had else -1
        copy = new > old and old % page != 0 and 0 <= last < n_pages and before[last] > 1
        need = (has - had + copy) if new > old else 0
        wanted += need
        if need and wanted > n_free:
            new, has = old, had
        else:
            got = free[taken:taken + need]
            taken += need
            if copy:
                copies.append((last, got[0]))
                refs[last] -= 1
                table[s, had - 1] = got[0]
            for i, p in enumerate(got[int(copy):]):
                table[s, had + i] = p
            for p in got:
                refs[p] = 1
            for e in range(has, had):
                if 0 <= table[s, e] < n_pages:
                    refs[table[s, e]] -= 1
        table[s, has:] = -1
        lens[s] = new
    return table, lens, refs, max(0, wanted - n_free), copies


def reorder(table, lens, refs, parents, page):
    new, out_lens, refs = np.full_like(table, -1), np.zeros_like(lens), refs.copy()
    cap, n_pages = table.shape[1] * page, len(refs)
    held = [min(max(int(n), 0), cap) for n in lens]
    for s, p in enumerate(parents):
        n = held[p] if 0 <= p < len(lens) else 0
        if n:
            new[s, :-(-n // page)] = table[p, :-(-n // page)]
        out_lens[s] = n
        if p != s:
            for e in table[s, :-(-held[s] // page)]:
                if 0 <= e < n_pages:
                    refs[e] -= 1
            for e in new[s]:
                if 0 <= e < n_pages:
                    refs[e] += 1
    return new, out_lens, refs


def compact(table, refs):
    """New table and refs, pages in use, and the moves as (from, to)."""
    live = [p for p in range(len(refs)) if refs[p] > 0]
    n_live = len(live)
    holes = [p for p in range(n_live) if refs[p] <= 0]
    moves = list(zip([p for p in live if p >= n_live], holes))
    new, table, out = dict(moves), table.copy(), refs.copy()
    for s in range(table.shape[0]):
        for e in range(table.shape[1]):
            table[s, e] = new.get(int(table[s, e]), table[s, e])
    for a, b in moves:
        out[b], out[a] = refs[a], 0
    return table, out, n_live, moves
