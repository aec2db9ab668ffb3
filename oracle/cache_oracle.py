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
    def held(r, length):
        return (tokens_of(k, k_scale, table[r], length, block, max_blocks),
                tokens_of(v.swapaxes(2, 3), v_scale, table[r], length, block, max_blocks))
    return _attend(held, k.shape[1], block, max_blocks, starts, lengths, q, scale, causal, window)


def _attend(held, kv_heads, block, max_blocks, starts, lengths, q, scale, causal, window):
    """held(r, length) -> keys, values [length, kv_heads, dim] of a request."""
    tokens, heads, dim = q.shape
    out, lse, spread = np.zeros((tokens, heads, dim)), np.full((tokens, heads), -np.inf), np.zeros((tokens, heads, dim))
    for r, length in enumerate(lengths.tolist()):
        n, first = int(starts[r + 1] - starts[r]), int(starts[r])
        if n <= 0:
            continue
        whole = length <= max_blocks * block
        keys, values = held(r, length)
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


# ------------------------------------------------------------------ a cache in 4 bits
#
# k, v [blocks, kv_heads, block_tokens, head_dim / 2] uint8, scales [blocks, kv_heads, head_dim / 32, block_tokens] uint8.

FOUR = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def four_scale(x, dtype):
    """x [..., 32] float64, finite -> byte of the scale: the least of the type's powers of two with max|x| <= 7 of it."""
    lowest, highest = (-23, 13) if dtype == "f16" else (-120, 125)
    most = np.abs(x).max(-1)
    e = np.full(most.shape, highest)
    for at in range(highest - 1, lowest - 1, -1):
        e = np.where(most <= 7 * 2.0 ** at, at, e)
    return np.where(most == 0, 0, e) + 127


def four_code(x, byte):
    """x [..., 32] float64 -> codes of the nearest values, of two the even one; 6 for what is larger."""
    a = np.minimum(np.abs(x) * 2.0 ** (127.0 - byte)[..., None], 6.0)
    off = np.abs(a[..., None] - FOUR[:8])
    near = off == off.min(-1, keepdims=True)
    first = near.argmax(-1)
    second = 7 - near[..., ::-1].argmax(-1)
    return np.where(first % 2 == 0, first, second) + 8 * np.signbit(x)


def four_append(k, v, k_scale, v_scale, new_k, new_v, slots, block, dtype):
    """new_k, new_v [tokens, heads, dim]; in place."""
    for token, slot in enumerate(slots.tolist()):
        b, o = slot // block, slot % block
        if slot < 0 or b >= k.shape[0]:
            continue
        for h in range(k.shape[1]):
            odd = not (np.isfinite(new_k[token, h]).all() and np.isfinite(new_v[token, h]).all())
            for codes, scale, x in ((k, k_scale, new_k), (v, v_scale, new_v)):
                if odd:                          # (the codes of a token that is marked are not looked at)
                    scale[b, h, :, o] = 255
                    continue
                x = x[token, h].astype(np.float64).reshape(-1, 32)
                byte = four_scale(x, dtype)
                c = four_code(x, byte.astype(np.float64)).reshape(-1)
                codes[b, h, o] = c[0::2] + 16 * c[1::2]
                scale[b, h, :, o] = byte


def four_values(codes, scale):
    """[blocks, heads, block tokens, dim] float64."""
    x = np.stack((FOUR[codes & 15], FOUR[codes >> 4]), -1).reshape(codes.shape[:3] + (codes.shape[3] // 16, 32))
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (x * s.swapaxes(2, 3)[..., None]).reshape(codes.shape[:3] + (2 * codes.shape[3],))


def four_tokens_of(codes, scale, row, length, block, max_blocks):
    """[length, heads, dim] float64 of a request; what the table does not hold is NaN."""
    out = np.full((length, codes.shape[1], 2 * codes.shape[3]), np.nan)
    for j in range(min(-(-length // block), max_blocks)):
        here = out[j * block:(j + 1) * block]
        if 0 <= row[j] < codes.shape[0]:
            one = slice(row[j], row[j] + 1)
            here[:] = four_values(codes[one], scale[one])[0].swapaxes(0, 1)[:len(here)]
    return out


def four_attend(k, v, k_scale, v_scale, block, max_blocks, table, starts, lengths, q, scale, causal, window):
    """As attend."""
    def held(r, length):
        return (four_tokens_of(k, k_scale, table[r], length, block, max_blocks), four_tokens_of(v, v_scale, table[r], length, block, max_blocks))
    return _attend(held, k.shape[1], block, max_blocks, starts, lengths, q, scale, causal, window)


def norm_rotate_axes(x, weight, eps, angles, positions, axis, rotary, neighbours):
    """As norm_rotate, with positions [axes, tokens] and the axis that each pair turns by.  Rows with a position past the
    angles are NaN, and so are pairs of an axis that there is not."""
    half = rotary // 2
    known = (positions < len(angles)).all(0)
    own = np.zeros((x.shape[0], rotary), angles.dtype)
    for i in range(half):
        for part in (i, half + i):
            own[:, part] = np.nan if axis[i] >= len(positions) else angles[np.where(known, positions[axis[i]], 0), part]
    y = norm_rotate(x, weight, eps, own, np.arange(x.shape[0]), rotary, neighbours)
    y[~known] = np.nan
    return y
