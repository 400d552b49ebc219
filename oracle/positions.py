"""Oracle of the steps in front of the append: pages out of a list of free ones, and rotary positions.

TEST INFRASTRUCTURE ONLY: plain numpy and Python integers; shares no code with the library.
"""
import math

import numpy as np


def assign(prefix, chunks, free, taken, tables, page_size, num_pages, capacity):
    """Returns (tables, row_offsets, positions, slots, taken, error): error 0, 3 (out of bounds) or 1 (a negative length)."""
    tables, B, error = tables.copy(), page_size, 0
    if not 0 <= taken <= len(free):
        taken, error = min(max(taken, 0), len(free)), 3
    most = tables.shape[1]
    positions, slots = np.zeros(capacity, np.int32), np.full(capacity, -1, np.int64)
    rows = [0]
    for i, (P, C) in enumerate(zip((int(x) for x in prefix), (int(x) for x in chunks))):
        if P < 0 or C < 0:
            P, C, error = 0, 0, error or 1
        for blk in range(-(-P // B), min(-(-(P + C) // B), most)):
            page = int(free[taken]) if taken < len(free) else -1
            taken = min(taken + 1, len(free))
            if not 0 <= page < num_pages:
                page, error = -1, error or 3
            tables[i, blk] = page
        for j in range(C):
            t, pos = rows[-1] + j, P + j
            if t >= capacity:
                error = error or 3
                break
            page = int(tables[i, pos // B]) if pos // B < most else -1
            if not 0 <= page < num_pages:
                page, error = -1, error or 3
            positions[t], slots[t] = pos, page * B + pos % B if page >= 0 else -1
        rows.append(rows[-1] + C)
    return tables, np.array(rows, np.int64), positions, slots, taken, error


def frequencies(rot_dim, base=10000.0, scaling="none", factor=1.0, original_context=0, low=0.0, high=0.0):
    """(radians per position of every pair, magnitude) from the definitions."""
    n = rot_dim
    low, high = low or 1.0, high or (32.0 if scaling == "turns" else 4.0)
    out = []
    for i in range(n // 2):
        f = base ** (-2.0 * i / n)
        if scaling == "linear":
            f /= factor
        elif scaling == "base":
            f = (base * factor ** (n / (n - 2.0))) ** (-2.0 * i / n)
        elif scaling == "wavelength":
            turns = original_context * f / (2 * math.pi)
            if turns < low:
                f /= factor
            elif turns <= high:
                share = (turns - low) / (high - low)
                f = (1 - share) * f / factor + share * f
        elif scaling == "turns":
            def pair(turns):
                return n * math.log(original_context / (turns * 2 * math.pi)) / (2 * math.log(base))
            lo, hi = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), n - 1)
            ramp = min(max((i - lo) / (hi - lo if hi != lo else 0.001), 0.0), 1.0)
            f = f / factor * ramp + f * (1 - ramp)
        out.append(f)
    return np.array(out), 0.1 * math.log(factor) + 1.0 if scaling == "turns" else 1.0


def rotate(x, turns, positions, interleaved, magnitude):
    """x: float64 [T, H, d]; turns: integers [rot_dim / 2], of a turn per position in 2^-64.  Returns (rotated, |a| + |b| of each
    element's pair, 0 behind rot_dim)."""
    n = 2 * len(turns)
    at = np.array([[((int(p) * int(f)) % (1 << 64)) / 2.0 ** 64 for f in turns] for p in positions]).reshape(len(positions), n // 2)
    c, s = np.cos(2 * np.pi * at)[:, None] * magnitude, np.sin(2 * np.pi * at)[:, None] * magnitude
    a, b = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    y, size = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size
