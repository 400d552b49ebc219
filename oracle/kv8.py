"""Oracle of the cache held in 8 bits: e4m3 codes with a scale per page and head, the append, and attention over what they stand for.

A code is an 8-bit floating-point number: sign, four bits of exponent (bias 7), three of mantissa; S.1111.111 is NaN, there are no
infinities, the largest number is 448.  A block (page, KV head) is page_size rows of d codes and, behind them, 16 bytes of which the
first four are its scale, an fp32 power of two from 2^-56 to 2^40.  Element = scale * code.

The rows that a chunk has in a page share the scale: the least 2^e with which their largest finite absolute value is within 448, and no
less than the scale of prefix rows that stand in the page, whose codes are scaled down and rounded again where it rises.

TEST INFRASTRUCTURE ONLY: plain numpy; shares no code with the library.
"""
import numpy as np

from .kv4 import bf16_bits, bf16_values  # noqa: F401

LEAST_EXP, MOST_EXP = -56, 40


def _numbers():
    byte = np.arange(256)
    e, m = byte // 8 % 16, byte % 8
    x = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7.0)) * np.where(byte < 128, 1.0, -1.0)
    x[byte % 128 == 127] = np.nan
    return x


NUMBERS = _numbers()


def encode(x):
    """Codes of float64 values: nearest, halves to the even code, beyond +-448: +-448; NaN and infinities 0x7f."""
    x = np.asarray(x, np.float64)
    a, grid = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), 448.0), NUMBERS[:127]
    above = np.clip(np.searchsorted(grid, a), 1, 126)
    mid = (grid[above - 1] + grid[above]) / 2
    code = np.where((a > mid) | ((a == mid) & (above % 2 == 0)), above, above - 1)
    return np.where(np.isfinite(x), code | np.where(np.signbit(x), 0x80, 0), 0x7F).astype(np.uint8)


def scale_exp(x):
    """Exponent of the least scale for these values."""
    a = np.abs(np.asarray(x, np.float64))
    top = a[np.isfinite(a)].max(initial=0.0)
    e = LEAST_EXP
    while e < MOST_EXP and top > 448.0 * 2.0 ** e:
        e += 1
    return e


def block_scale(block, page_size, d):
    return np.ascontiguousarray(block[page_size * d:page_size * d + 4]).view(np.float32)[0]


def append(k_new, v_new, k_pool, v_pool, block_tables, prefix_lens, chunk_lens, page_size):
    """bf16 bit patterns [T, Hkv, d] into copies of the pools (uint8 [pages, Hkv, bytes]); returns (k_pool, v_pool)."""
    out = []
    B, d = page_size, k_new.shape[2]
    for new, pool in ((k_new, k_pool), (v_new, v_pool)):
        pool, x = pool.copy(), bf16_values(new).astype(np.float64)
        row = 0
        for i, C in enumerate(int(c) for c in chunk_lens):
            P = int(prefix_lens[i])
            for first in range(P // B * B, P + C if C else 0, B):
                lo, hi = max(P, first), min(P + C, first + B)
                for h in range(new.shape[1]):
                    block = pool[int(block_tables[i, first // B]), h]
                    rows = x[row + lo - P:row + hi - P, h]
                    e = scale_exp(rows)
                    if lo > first:
                        old = int(np.log2(block_scale(block, B, d)))
                        if e > old:
                            stand = NUMBERS[block[:(lo - first) * d]] * 2.0 ** (old - e)
                            block[:(lo - first) * d] = encode(stand)
                        e = max(e, old)
                    block[(lo - first) * d:(hi - first) * d] = encode(rows * 2.0 ** -e).reshape(-1)
                    block[B * d:B * d + 4] = np.array([2.0 ** e], np.float32).view(np.uint8)
            row += C
        out.append(pool)
    return tuple(out)


def rows_of(pool, table_row, n, page_size, d, head):
    """(float64 values [n, d], scales [n]) of positions 0 .. n - 1 of a request."""
    pages = [int(p) for p in table_row[:(n + page_size - 1) // page_size]]
    x = np.concatenate([NUMBERS[pool[p, head, :page_size * d]].reshape(page_size, d) for p in pages])
    s = np.repeat([float(block_scale(pool[p, head], page_size, d)) for p in pages], page_size)
    return (x * s[:, None])[:n], s[:n]


def attention(q, k_pool, v_pool, block_tables, prefix_lens, chunk_lens, page_size, num_kv_heads, sm_scale=0.0):
    """q: float64 [T, Hq, d].  Returns (out float64 [T, Hq, d], lse float64 [T, Hq], spread, even: float64 [T, Hq, d]): spread is
    sum_j p_j |v_j| per element, what roundings of the p_j are relative to; even is max_j p_j sum_j |v_j|, what errors of the p_j
    relative to the row's largest are relative to."""
    T, Hq, d = q.shape
    G = Hq // num_kv_heads
    scale = sm_scale if sm_scale > 0 else d ** -0.5
    out, lse, spread, even = np.zeros((T, Hq, d)), np.zeros((T, Hq)), np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    row = 0
    for i, C in enumerate(int(c) for c in chunk_lens):
        P = int(prefix_lens[i])
        for g in range(num_kv_heads if C else 0):
            K, _ = rows_of(k_pool, block_tables[i], P + C, page_size, d, g)
            V, _ = rows_of(v_pool, block_tables[i], P + C, page_size, d, g)
            for t in range(C):
                n = P + t + 1
                s = scale * (K[:n] @ q[row + t, g * G:(g + 1) * G].T)               # [keys, heads]
                m = s.max(0)
                e = np.exp(s - m)
                z = e.sum(0)
                out[row + t, g * G:(g + 1) * G] = e.T @ V[:n] / z[:, None]
                spread[row + t, g * G:(g + 1) * G] = e.T @ np.abs(V[:n]) / z[:, None]
                even[row + t, g * G:(g + 1) * G] = np.abs(V[:n]).sum(0) / z[:, None]
                lse[row + t, g * G:(g + 1) * G] = m + np.log(z)
        row += C
    return out, lse, spread, even
