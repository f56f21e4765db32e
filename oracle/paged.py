"""Float64 oracle of the paged 8-bit K/V cache, written from the definitions in
include/fkv.h: plain numpy, one request, page and row at a time."""
from __future__ import annotations

import math

import numpy as np

E4M3, INT8 = "e4m3", "int8"
FLOOR, CEILING = 2.0 ** -100, 2.0 ** 100


def _e4m3_table():
    """What each of the 256 codes stands for: sign, 4 exponent bits of bias 7, 3 fraction bits."""
    out = np.empty(256)
    for c in range(256):
        s, e, f = c >> 7, c >> 3 & 15, c & 7
        v = math.ldexp(f, -9) if e == 0 else math.ldexp(8 + f, e - 10)
        out[c] = math.nan if e == 15 and f == 7 else (-v if s else v)
    return out


E4M3_VALUES = _e4m3_table()


def values(codes, fmt):
    """uint8 codes -> float64 (NaN codes of slots never written included)."""
    codes = np.asarray(codes, np.uint8)
    return E4M3_VALUES[codes] if fmt == E4M3 else codes.view(np.int8).astype(np.float64)


def to_codes(y, fmt):
    """The nearest codes of float64 values (ties to even), beyond the largest as the largest."""
    y = np.asarray(y, np.float64)
    if fmt == INT8:
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    mag = np.minimum(np.abs(y), 448.0)
    pos = E4M3_VALUES[:127]                                # increasing; codes of even fraction are even numbers
    hi = np.searchsorted(pos, mag)                         # the first code not below mag
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = mag - pos[lo], pos[hi] - mag
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    pick = np.where(pos[hi] == mag, hi, pick)
    return (pick | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def scale_of(amax, fmt):
    """float32 scale of a run whose largest finite magnitude is amax."""
    if amax == 0:
        return np.float32(FLOOR)
    if fmt == INT8:
        return np.float32(min(max(np.float32(np.float32(amax) / np.float32(127)), FLOOR), CEILING))
    m, e = math.frexp(amax / 448.0)
    return np.float32(min(max(math.ldexp(1.0, e - 1 if m == 0.5 else e), FLOOR), CEILING))


def write(codes, scale, x, slots, fmt):
    """codes uint8 [n_blocks, H, B, D] and scale float32 [n_blocks, H] updated in place; x float64 [T, H, D].
    The rounding steps that fkv.h names in float32 are float32 here."""
    B = codes.shape[2]
    t, T = 0, len(slots)
    while t < T:
        s = int(slots[t])
        if s < 0 or s // B >= codes.shape[0]:
            t += 1
            continue
        blk, off, n = s // B, s % B, 1
        while t + n < T and off + n < B and slots[t + n] == s + n:
            n += 1
        for h in range(codes.shape[1]):
            run = x[t:t + n, h]
            fin = np.abs(run[np.isfinite(run)])
            want = scale_of(fin.max() if fin.size else 0.0, fmt)
            was = scale[blk, h] if off else np.float32(0)
            now = was if was >= want else want
            inv = np.float32(1) / now
            if off and now != was:
                old = values(codes[blk, h, :off], fmt).astype(np.float32) * np.float32(was * inv)
                codes[blk, h, :off] = to_codes(old, fmt)
            with np.errstate(over="ignore", invalid="ignore"):
                y = np.where(np.isnan(run), 0.0, run).astype(np.float32) * inv
            codes[blk, h, off:off + n] = to_codes(np.clip(y, -1e30, 1e30), fmt)
            scale[blk, h] = now
        t += n


def plan(n_new, kv_len, table, free, taken, block, rows):
    """(cu, slots, positions, kv_len, taken, table, free, fits) after the call; the inputs are not changed."""
    n_new, kv_len = np.asarray(n_new, np.int64), np.asarray(kv_len, np.int64)
    table, free = table.copy(), free.copy()
    n, width = len(n_new), table.shape[1]
    b = lambda tokens: -(-int(tokens) // block)
    cu, slots, pos = np.zeros(n + 1, np.int64), np.full(rows, -1, np.int64), np.full(rows, -1, np.int64)
    back = sum(b(kv_len[r]) for r in range(n) if n_new[r] < 0 and kv_len[r] >= 0)
    need = sum(b(kv_len[r] + n_new[r]) - b(kv_len[r]) for r in range(n) if n_new[r] >= 0 and kv_len[r] >= 0)
    tokens = int(np.maximum(n_new, 0).sum())
    fits = (all(0 <= kv_len[r] <= 1 << 30 and n_new[r] <= 1 << 30 and b(kv_len[r] + max(n_new[r], 0)) <= width
                for r in range(n)) and 0 <= taken <= len(free) and back <= taken and
            taken - back + need <= len(free) and tokens <= rows)
    if not fits:
        return cu, slots, pos, kv_len, taken, table, free, False
    at = top = taken - back
    for r in range(n):
        if n_new[r] < 0:
            for j in range(b(kv_len[r])):
                free[at] = table[r, j]
                at += 1
    after = kv_len.copy()
    for r in range(n):
        cu[r + 1] = cu[r] + max(n_new[r], 0)
        if n_new[r] < 0:
            after[r] = 0
            continue
        after[r] += n_new[r]
        for j in range(b(kv_len[r]), b(after[r])):
            table[r, j] = free[top]
            top += 1
        for i in range(n_new[r]):
            p = kv_len[r] + i
            slots[cu[r] + i] = table[r, p // block] * block + p % block
            pos[cu[r] + i] = p
    return cu, slots, pos, after, top, table, free, True


def gather(codes, scale, table_row, tokens, fmt):
    """float64 values [H, tokens, D] of one request's first positions."""
    B = codes.shape[2]
    ids = [int(i) for i in table_row[:-(-tokens // B)]]
    if not ids:
        return np.zeros((codes.shape[1], 0, codes.shape[3]))
    v = [values(codes[i], fmt) * scale[i].astype(np.float64)[:, None, None] for i in ids]
    return np.concatenate(v, 1)[:, :tokens]


def visible(n_new, length, causal=True, window=0, sinks=0, prefix=None):
    """bool [n_new, length]"""
    p = (length - n_new + np.arange(n_new))[:, None]
    j = np.arange(length)[None, :]
    near = (j <= p) if causal else np.ones((n_new, length), bool)
    if window:
        near = near & ((j > p - window) | (j < sinks))
    if prefix is not None:
        near = near | (j < prefix)
    return near & (p >= 0)


def attend(q, k, v, scale, seen, softcap=0.0, slopes=None, p0=0):
    """One request: q [n_new, Hq, D], k and v [H, length, D] float64 -> (out, lse,
    sum of weight x |v|, largest scale sum |q||k| of a visible score)."""
    n, Hq, D = q.shape
    G = Hq // k.shape[0]
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    mass, size = np.zeros((n, Hq, D)), np.zeros((n, Hq))
    j = np.arange(k.shape[1])
    for u in range(Hq):
        kk, vv = k[u // G], v[u // G]
        for i in range(n):
            on = seen[i]
            if not on.any():
                continue
            x = scale * (kk[on] @ q[i, u])
            size[i, u] = abs(scale) * (np.abs(kk[on]) @ np.abs(q[i, u])).max()
            if softcap:
                x = softcap * np.tanh(x / softcap)
            if slopes is not None:
                x = x + float(slopes[u]) * (j[on] - (p0 + i))
            m = x.max()
            w = np.exp(x - m)
            out[i, u] = w @ vv[on] / w.sum()
            mass[i, u] = w @ np.abs(vv[on]) / w.sum()
            lse[i, u] = m + math.log(w.sum())
    return out, lse, mass, size
