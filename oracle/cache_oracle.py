"""Plain CPU oracle of the serving operators (include/tsq_cache.h), written from their formulas in numpy: schedules in
whole numbers, norm, rotation and attention in binary64, the cache's codes and scales in the binary32 steps that define
them.  Shares no code with the GPU path.

A cache here: k [blocks, kv_heads, block_tokens, head_dim] int8, v [blocks, kv_heads, head_dim, block_tokens] int8,
k_scale and v_scale [blocks, kv_heads] float32, as the header lays them out.
"""
from __future__ import annotations

import numpy as np

OK, INVALID, CAPACITY = 0, 1, 3


def schedule(new, lengths, table, ring, counters, block, max_blocks, capacity):
    """-> dict of what the call leaves; table and ring are copied."""
    blocks, n = len(ring), len(new)
    table, ring = table.copy(), ring.copy()
    taken, returned = int(counters[0]), int(counters[1])
    held = lambda t: -(-t // block)                                            # noqa: E731
    bad = not (0 <= taken <= returned and returned - taken <= blocks)
    full, rows, want, back = False, 0, 0, 0
    for m, t in zip(new.tolist(), lengths.tolist()):
        if t < 0 or t > max_blocks * block or m < -1:
            bad = True
        elif m < 0:
            back += held(t)
        elif t + m > max_blocks * block or m > capacity:
            full = True
        else:
            rows += m
            want += held(t + m) - held(t)
    full |= rows > capacity or want > returned - taken
    bad |= returned - taken + back > blocks
    positions, slots = np.full(capacity, -1, np.int32), np.full(capacity, -1, np.int32)
    if bad or full:
        return dict(status=INVALID if bad else CAPACITY, lengths=lengths.copy(), counters=counters.copy(),
                    starts=np.zeros(n + 1, np.int32), positions=positions, slots=slots, table=table, ring=ring)
    starts, out = [0], []
    for r, (m, t) in enumerate(zip(new.tolist(), lengths.tolist())):
        if m < 0:
            for j in range(held(t)):
                ring[returned % blocks] = table[r, j]
                returned += 1
            out.append(0)
            starts.append(starts[-1])
            continue
        for j in range(held(t), held(t + m)):
            table[r, j] = ring[taken % blocks]
            taken += 1
        for i in range(m):
            positions[starts[-1] + i] = t + i
            b = int(table[r, (t + i) // block])
            slots[starts[-1] + i] = b * block + (t + i) % block if 0 <= b < blocks else -1
        out.append(t + m)
        starts.append(starts[-1] + m)
    return dict(status=OK, lengths=np.array(out, np.int32), counters=np.array([taken, returned], np.int64),
                starts=np.array(starts, np.int32), positions=positions, slots=slots, table=table, ring=ring)


def norm_rotate(x, weight, eps, angles, positions, rotary, neighbours):
    """x [tokens, heads, dim] float64 -> the same, binary64.  Rows of a position past the angles are NaN."""
    y = x.astype(np.float64).copy()
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    half = rotary // 2
    known = positions < len(angles)
    at = np.where(known, positions, 0)
    c, s = angles[at, :half].astype(np.float64)[:, None], angles[at, half:].astype(np.float64)[:, None]
    first, second = (slice(0, rotary, 2), slice(1, rotary, 2)) if neighbours else (slice(0, half), slice(half, rotary))
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    y[~known] = np.nan
    return y


def _append_one(codes, scale, x, slots, block):
    """codes [blocks, heads, block tokens, dim] (a view is fine), x [tokens, heads, dim] float32; in place."""
    tokens, i = len(slots), 0
    blocks = codes.shape[0]
    one = np.float32(1)
    while i < tokens:
        slot = int(slots[i])
        if slot < 0 or slot // block >= blocks:
            i += 1
            continue
        b, o, n = slot // block, slot % block, 1
        while i + n < tokens and o + n < block and int(slots[i + n]) == slot + n:
            n += 1
        rows = x[i:i + n]                                                       # [n, heads, dim]
        for h in range(x.shape[1]):
            part = rows[:, h]
            before = scale[b, h] if o else np.float32(0)
            most = np.abs(part).max()
            now = np.float32(most / np.float32(127))
            if now < np.float32(2.0 ** -126):
                now = np.float32(0)
            if not np.isfinite(part).all() or np.isnan(before):
                now = np.float32(np.nan)
            else:
                now = max(before, now)
            scale[b, h] = now
            if not now > 0:
                codes[b, h, o:o + n] = 0
                continue
            if o and now != before:
                codes[b, h, :o] = np.rint(codes[b, h, :o].astype(np.float32) * np.float32(before / now))
            inverse = one / now
            codes[b, h, o:o + n] = np.clip(np.rint(part * inverse), -127, 127)
        i += n


def append(k, v, k_scale, v_scale, new_k, new_v, slots, block):
    with np.errstate(all="ignore"):
        _append_one(k, k_scale, new_k, slots, block)
        _append_one(v.swapaxes(2, 3), v_scale, new_v, slots, block)


def tokens_of(codes, scale, row, length, block, max_blocks):
    """[length, heads, dim] float64 of a request; what the table does not hold is NaN."""
    blocks = codes.shape[0]
    out = np.full((length, codes.shape[1], codes.shape[3]), np.nan)
    for j in range(-(-length // block)):
        here = out[j * block:(j + 1) * block]
        if j < max_blocks and 0 <= row[j] < blocks:
            here[:] = (codes[row[j]].astype(np.float64) * scale[row[j]].astype(np.float64)[:, None, None]).swapaxes(0, 1)[:len(here)]
    return out


def attend(k, v, k_scale, v_scale, block, max_blocks, table, starts, lengths, q, scale, causal, window):
    """q [tokens, q_heads, dim] -> out, lse and the sum of weight * |value| (what a relative error of the weights
    can do to out), all binary64."""
    tokens, heads, dim = q.shape
    kv_heads = k.shape[1]
    out, lse, spread = np.zeros((tokens, heads, dim)), np.full((tokens, heads), -np.inf), np.zeros((tokens, heads, dim))
    for r, length in enumerate(lengths.tolist()):
        n, first = int(starts[r + 1] - starts[r]), int(starts[r])
        if n <= 0:
            continue
        whole = length <= max_blocks * block
        keys = tokens_of(k, k_scale, table[r], length, block, max_blocks)
        values = tokens_of(v.swapaxes(2, 3), v_scale, table[r], length, block, max_blocks)
        if not whole:
            keys[:] = np.nan
        t = np.arange(length)
        for i in range(n):
            p = length - n + i
            seen = np.ones(length, bool)
            if causal:
                seen &= t <= p
            if window:
                seen &= t > p - window
            if not seen.any():
                continue
            for h in range(heads):
                g = h // (heads // kv_heads)
                s = keys[seen, g] @ q[first + i, h].astype(np.float64) * scale
                top = s.max()
                w = np.exp(s - top)
                # (a block that is marked spoils both, whether it is its keys or its values that are)
                lse[first + i, h] = np.nan if np.isnan(values[seen, g]).any() else top + np.log(w.sum())
                w /= w.sum()
                out[first + i, h] = w @ values[seen, g]
                spread[first + i, h] = w @ np.abs(values[seen, g])
    return out, lse, spread
