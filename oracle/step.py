"""A serving step around the paged cache, stated plainly on the CPU (test infrastructure): where new tokens go, the pages taken
and given back, and the norms and the rotation of heads in fp64.
"""
from __future__ import annotations

import numpy as np


def plan(lens, counts, table, free, depth, page, rows):
    """(starts, lens, table, slots, positions, depth, bad) of a step, one sequence after another.  bad: something was out of
    its range or left out."""
    B, width = table.shape
    room, table = width * page, table.copy()
    starts, lens_out = np.zeros(B + 1, np.int32), np.zeros(B, np.int32)
    slots, positions = np.full(rows, -1, np.int32), np.full(rows, -1, np.int32)
    bad = not 0 <= depth <= len(free)
    depth = min(max(depth, 0), len(free))
    start = base = taken = 0
    for b in range(B):
        n, have = max(int(counts[b]), 0), min(max(int(lens[b]), 0), room)
        bad |= counts[b] < 0 or have != lens[b]
        starts[b], lens_out[b] = min(start, rows), have
        held = -(-have // page)
        fits = have == lens[b] and have + n <= room
        need = -(-(have + n) // page) - held if fits else 0
        if n > 0 and fits and start + n <= rows and (need == 0 or base + need <= depth):
            for i in range(need):
                table[b, held + i] = free[depth - 1 - base - i]
                bad |= table[b, held + i] < 0
            for i in range(n):
                p = have + i
                entry = int(table[b, p // page])
                slot = entry * page + p % page
                positions[start + i] = p
                slots[start + i] = slot if entry >= 0 and slot < 2 ** 31 else -1
                bad |= slots[start + i] < 0
            lens_out[b] = have + n
            taken = base + need if need else taken
        else:
            bad |= n > 0
        start += n
        base += need
    starts[B] = min(start, rows)
    return starts, lens_out, table, slots, positions, depth - taken, bool(bad)


def release(lens, done, table, free, depth, page):
    """(lens, free, depth, bad) after the finished sequences' pages are back on the stack."""
    B, width = table.shape
    free, out = free.copy(), np.zeros(B, np.int32)
    bad = not 0 <= depth <= len(free)
    depth = min(max(depth, 0), len(free))
    for b in range(B):
        have = min(max(int(lens[b]), 0), width * page)
        bad |= have != lens[b]
        out[b] = 0 if done[b] else have
        for i in range(-(-have // page) if done[b] else 0):
            bad |= table[b, i] < 0 or depth >= len(free)
            if depth < len(free):
                free[depth] = table[b, i]
                depth += 1
    return out, free, depth, bool(bad)


def head_norm_rope(x, weight, eps, freq, positions, rot, pairs):
    """Norm and rotation of heads x [rows, heads, 128] in fp64: (y, scale) with scale the |a| + |b| of each value's pair (of the
    value itself where it is not rotated), the measure of fp32's errors.  A negative position gives zeros."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + float(np.float32(eps))) * np.asarray(weight, np.float64)
    # (64 bits of mantissa hold the product of a position and an fp32 frequency)
    angle = np.asarray(positions, np.longdouble)[:, None] * np.asarray(freq, np.float32).astype(np.longdouble)[None, :]
    cos, sin = (f(angle).astype(np.float64)[:, None, :] for f in (np.cos, np.sin))
    half = rot // 2
    i = np.arange(half)
    first, second = (2 * i, 2 * i + 1) if pairs else (i, i + half)
    a, b = x[..., first], x[..., second]
    y, scale = x.copy(), np.abs(x)
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    scale[..., first] = scale[..., second] = np.abs(a) + np.abs(b)
    y[np.asarray(positions) < 0] = 0.0
    scale[np.asarray(positions) < 0] = 0.0
    return y, scale
