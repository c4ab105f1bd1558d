"""Plain forms of the key-value cache's operators in numpy, in 64 bits (codes
and scales in float32, as their definition has them)."""
import math

import numpy as np

BLOCK = 16
QMAX = {"int8": np.float32(127), "e4m3": np.float32(448)}


def e4m3_table():
    """Values of the 256 e4m3 codes (NaN for 0x7f and 0xff)."""
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[b] = math.nan if b & 127 == 127 else -v if b & 128 else v
    return out


E4M3 = e4m3_table()
_POS = np.append(E4M3[:127], 480.0)  # ascending


def values(codes, kind):
    return codes.view(np.int8).astype(np.float64) if kind == "int8" else E4M3[codes]


def to_codes(y, kind):
    """float32 values within the codes' range to codes, to nearest, ties to even."""
    y = np.asarray(y, np.float32).astype(np.float64)
    if kind == "int8":
        return np.rint(y).astype(np.int8).view(np.uint8)
    a = np.abs(y)
    hi = np.searchsorted(_POS, a)  # _POS[hi - 1] < a <= _POS[hi]
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.minimum(code, 126).astype(np.uint8)
    return np.where(np.signbit(y), code | 128, code).astype(np.uint8)


def append(pool, scale, table, lens, slots, starts, x, kind):
    """pool uint8 [pages, heads, page, dim], scale [pages, heads, page / 16], x
    float32 [tokens, heads, dim]; in place, as tq_kv_append defines it."""
    page = pool.shape[2]
    for i, slot in enumerate(slots):
        new = x[starts[i]: starts[i + 1]]
        begin = lens[slot] - len(new)
        at = begin
        while at < lens[slot]:
            end = min(lens[slot], (at // BLOCK + 1) * BLOCK)
            p, b, first = table[slot, at // page], at % page // BLOCK, at % BLOCK
            part = new[at - begin: end - begin]
            size = np.where(np.isfinite(part), np.abs(part), np.float32(0))
            s = (size.max((0, 2)) / QMAX[kind]).astype(np.float32)
            line = pool[p, :, b * BLOCK: (b + 1) * BLOCK]
            if first:
                old = scale[p, :, b]
                grown = s > old
                s = np.maximum(s, old)
                ratio = np.where(grown, old / np.where(grown, s, 1), np.float32(1)).astype(np.float32)
                held = values(line[:, :first], kind).astype(np.float32) * ratio[:, None, None]
                line[:, :first] = np.where(grown[:, None, None], to_codes(held, kind), line[:, :first])
            with np.errstate(invalid="ignore", divide="ignore"):
                y = (part / s[None, :, None]).astype(np.float32)
            y = np.where((s > 0)[None, :, None] & ~np.isnan(part), y, np.float32(0))
            y = np.clip(y, -QMAX[kind], QMAX[kind])
            line[:, first: first + end - at] = to_codes(y, kind).transpose(1, 0, 2)
            scale[p, :, b] = s
            at = end


def read(pool, scale, table, slot, n, kind):
    """Values of the first n tokens of a slot, float64 [n, heads, dim]."""
    page = pool.shape[2]
    out = np.zeros((n, pool.shape[1], pool.shape[3]))
    for t in range(n):
        p, inside = table[slot, t // page], t % page
        out[t] = values(pool[p, :, inside], kind) * scale[p, :, inside // BLOCK].astype(np.float64)[:, None]
    return out


def attention(k, v, q, scale, window):
    """One sequence: k, v float64 [len, kv_heads, dim], q float64 [m, heads, dim]:
    (out, lse, size, error): size = sum p |v|, error = how far a float32 sum of
    the scores may be off."""
    n, kv_heads, dim = k.shape
    m, heads, _ = q.shape
    out, lse = np.zeros((m, heads, dim)), np.full((m, heads), -np.inf)
    size, error = np.zeros((m, heads, dim)), np.zeros((m, heads))
    for r in range(m):
        place = n - m + r
        lo = max(0, place - window + 1) if window else 0
        if place < 0:
            continue
        for h in range(heads):
            kk, vv = k[lo: place + 1, h * kv_heads // heads], v[lo: place + 1, h * kv_heads // heads]
            s = kk @ q[r, h] * scale
            top = s.max()
            p = np.exp(s - top)
            lse[r, h] = top + math.log(p.sum())
            p /= p.sum()
            out[r, h], size[r, h] = p @ vv, p @ np.abs(vv)
            error[r, h] = dim * 2.0 ** -23 * abs(scale) * (np.abs(kk) @ np.abs(q[r, h])).max()
    return out, lse, size, error


def verify(target, drafts, uniforms, noise, draft=None, lens=None):
    n, t1, vocab = target.shape
    tokens, accepted = np.full((n, t1), -1, np.int32), np.zeros(n, np.int32)
    for i in range(n):
        m = t1 - 1 if lens is None else lens[i]
        a = 0
        while a < m:
            x = drafts[i, a]
            if not 0 <= x < vocab:
                break
            q = np.float32(1) if draft is None else np.float32(draft[i, a, x])
            if not np.float32(uniforms[i, a]) * q < np.float32(target[i, a, x]):
                break
            a += 1
        p = target[i, a].astype(np.float32)
        w = p
        if a < m:
            if draft is not None:
                w = np.maximum(p - draft[i, a].astype(np.float32), np.float32(0))
            else:
                w = p.copy()
                if 0 <= drafts[i, a] < vocab:
                    w[drafts[i, a]] = 0
            if not (w > 0).any():
                w = p
        tokens[i, :a] = drafts[i, :a]
        tokens[i, a] = np.argmax(w / noise[i])
        accepted[i] = a
    return tokens, accepted
