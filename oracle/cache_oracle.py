"""CPU oracle for rotary positions with several axes and the paged 8-bit KV cache (TEST INFRASTRUCTURE).

Definitions written out in float64 and Python integers, one sequence, block or row at a time; shares no code with the
CUDA library.  Caches are arrays of codes (bytes) with float scales; code tables are built from the formats' definitions.
"""
from __future__ import annotations

import numpy as np

E4M3, I8 = 0, 1
Q_MAX = {E4M3: 448.0, I8: 127.0}
E_MIN, E_MAX = -48, 48
HALVES, ADJACENT = 0, 1


# --------------------------------------------------------------------------- rotary positions
def rope(x, pos, inv_freq, axis, pairing=HALVES, inverse=False):
    """x [H, S, d], pos [P, S] integers, inv_freq and axis [rot / 2] -> [H, S, d] float64."""
    y = np.array(x, dtype=np.float64)
    x = y.copy()
    n = len(inv_freq)
    for i in range(n):
        angle = pos[axis[i]].astype(np.float64) * float(inv_freq[i])
        c, s = np.cos(angle), np.sin(-angle if inverse else angle)
        a, b = (i, i + n) if pairing == HALVES else (2 * i, 2 * i + 1)
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y


# --------------------------------------------------------------------------- block tables
def plan(past, new, table, ring, state, block_size, rows):
    """Integers and lists in, a dict of new values out; slots and positions of the new rows only."""
    past, new = [int(v) for v in past], [int(v) for v in new]
    table, ring = [list(map(int, r)) for r in table], [int(v) for v in ring]
    head, tail = int(state[0]), int(state[1])
    n, columns = len(ring), len(table[0]) if table else 0
    room = columns * block_size
    blocks = lambda t: -(-t // block_size)  # noqa: E731
    code = taken = given = total = 0
    for p, g in zip(past, new):
        if p < 0 or p + g < 0:
            code |= 8
            continue
        if max(p, p + g) > room:
            code |= 2
        taken += max(blocks(p + g) - blocks(p), 0)
        given += max(blocks(p) - blocks(p + g), 0)
        total += max(g, 0)
    if total > rows:
        code |= 4
    if head < 0 or not 0 <= tail - head <= n or tail - head + given > n:
        code |= 16
    if taken > tail - head:
        code |= 1
    top = 2 ** 31 - 1      # the report is 32 bits wide
    out = {"report": [code, min(taken, top), min(given, top), min(total, top)], "table": table, "ring": ring, "slots": [], "positions": []}
    if code:
        out.update(kv_len=[min(max(p, 0), room) for p in past], row_offset=[0] * (len(past) + 1), state=[head, tail])
        return out
    source = list(ring)
    out.update(kv_len=[p + g for p, g in zip(past, new)], row_offset=[0], state=[head + taken, tail + given])
    for b, (p, g) in enumerate(zip(past, new)):
        for j in range(blocks(p), blocks(p + g)):
            table[b][j] = source[head % n]
            head += 1
        for j in range(blocks(p + g), blocks(p)):
            ring[tail % n] = table[b][j]
            tail += 1
        for t in range(p, p + g):
            out["slots"].append(table[b][t // block_size] * block_size + t % block_size)
            out["positions"].append(t)
        out["row_offset"].append(len(out["positions"]))
    return out


# --------------------------------------------------------------------------- codes
def code_values(kind):
    """The value of each of the 256 codes."""
    v = np.arange(256)
    if kind == I8:
        return np.where(v < 128, v, v - 256).astype(np.float64)
    sign, e, m = np.where(v & 0x80, -1.0, 1.0), (v >> 3) & 15, v & 7
    out = sign * np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    out[[0x7F, 0xFF]] = np.nan
    return out


def encode(x, kind):
    """Nearest code of each value, ties to the code whose last bit is 0, beyond the largest the largest; NaN: the code of 0."""
    x = np.where(np.isnan(x), 0.0, np.asarray(x, dtype=np.float64))
    if kind == I8:
        return np.clip(np.rint(x), -127, 127).astype(np.int64).astype(np.uint8)
    positive = code_values(E4M3)[:0x7F]
    mag = np.minimum(np.abs(x), 448.0)
    hi = np.searchsorted(positive, mag).clip(0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    near = np.where(mag - positive[lo] < positive[hi] - mag, lo, np.where(mag - positive[lo] > positive[hi] - mag, hi, np.where(lo % 2 == 0, lo, hi)))
    return (near + np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def least_scale(amax, kind):
    for e in range(E_MIN, E_MAX + 1):
        if amax <= Q_MAX[kind] * 2.0 ** e:
            return 2.0 ** e
    return 2.0 ** E_MAX


# --------------------------------------------------------------------------- the cache
def write(codes, scale, rows, kv_len, table, block_size, kind):
    """codes [blocks, H, bs, d] uint8 and scale [blocks, H], changed in place; rows: per sequence [n, H, d] float64."""
    values = code_values(kind)
    nb, H = scale.shape
    for b, x in enumerate(rows):
        n = len(x)
        start = int(kv_len[b]) - n
        if start < 0 or n == 0:
            continue
        for j in range(start // block_size, -(-(start + n) // block_size)):
            if j >= len(table[b]) or not 0 <= table[b][j] < nb:
                continue
            blk, lo = int(table[b][j]), max(start, j * block_size)
            part = x[lo - start:min((j + 1) * block_size, start + n) - start]
            off = lo - j * block_size
            for h in range(H):
                p = part[:, h]
                s = least_scale(np.abs(p).max(), kind) if np.isfinite(p).all() else np.nan
                if off:
                    old = scale[blk, h]
                    s = np.nan if np.isnan(s) or np.isnan(old) else max(s, old)
                    if s != old:
                        codes[blk, h, :off] = encode(values[codes[blk, h, :off]] * (old / s), kind)
                codes[blk, h, off:off + len(p)] = encode(p / s, kind)
                scale[blk, h] = s


def gather(codes, scale, table_row, length, block_size, kind):
    """[T, H, d] values that a sequence's tokens stand for, and which of them are there at all."""
    values = code_values(kind)
    nb, H, _, d = codes.shape
    length = min(max(int(length), 0), len(table_row) * block_size)
    out, there = np.zeros((length, H, d)), np.zeros(length, dtype=bool)
    for t in range(length):
        blk = int(table_row[t // block_size])
        if 0 <= blk < nb:
            out[t] = values[codes[blk, :, t % block_size]] * scale[blk][:, None]
            there[t] = True
    return out, there


def attention(q, k, v, there, scale, causal, start):
    """q [n, Hq, d], k and v [T, Hkv, d]; row i stands at start + i.  -> out [n, Hq, d], lse [n, Hq], and two sizes that the
    tolerances of the tests are made of: sum of p |v| like out, and the largest scale * sum |q| |k| like lse."""
    n, Hq, d = q.shape
    group = Hq // k.shape[1]
    out, lse = np.zeros((n, Hq, d)), np.full((n, Hq), -np.inf)
    weight, reach = np.zeros((n, Hq, d)), np.zeros((n, Hq))
    for i in range(n):
        seen = there & (np.arange(len(there)) <= start + i) if causal else there
        if not seen.any():
            continue
        for h in range(Hq):
            kk, vv = k[seen, h // group], v[seen, h // group]
            s = scale * (kk @ q[i, h])
            top = s.max()
            e = np.exp(s - top)
            out[i, h] = e @ vv / e.sum()
            weight[i, h] = e @ np.abs(vv) / e.sum()
            lse[i, h] = top + np.log(e.sum())
            reach[i, h] = abs(scale) * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, lse, weight, reach
