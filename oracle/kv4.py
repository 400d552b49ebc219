"""Oracle of the cache held in 4 bits: rows as codes and two bf16 numbers, the append, and attention over what they stand for.

A row x of d bf16 values (one token, KV head, K or V) is kept as
    least = min x (+0 where that is -0),    scale = bf16((max x - least) / 15)  (difference and quotient in fp32),
    c_e   = (x_e - least) / scale, difference and quotient in fp32, to the nearest integer, halves to the even one,
and stands for least + scale * c_e.  scale < 2^-100: scale and codes 0.  A row with a NaN or an infinity, or whose extent is not a
finite fp32 number: least = NaN (0x7fc0), scale and codes 0.  A block (page, KV head) is page_size rows of d / 2 bytes (element
2 i in the low half of byte i) and, behind them, page_size pairs (least, scale).

TEST INFRASTRUCTURE ONLY: plain numpy; shares no code with the library.
"""
import numpy as np


def bf16_values(bits):
    """float32 values of bf16 bit patterns (uint16)."""
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32)


def bf16_bits(x):
    """bf16 bit patterns of finite float32 values, rounded to nearest even."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def pack_rows(bits):
    """[..., d] bf16 bit patterns -> (codes uint8 [..., d], pairs uint16 [..., 2])."""
    x = bf16_values(bits)
    with np.errstate(all="ignore"):
        least = np.min(x, -1, keepdims=True) + np.float32(0)
        extent = np.max(x, -1, keepdims=True) - least
        fine = np.isfinite(extent)
        scale = bf16_values(bf16_bits(np.where(fine, extent, 0) / np.float32(15)))
        scale = np.where(fine & (scale >= 2.0 ** -100), scale, np.float32(0))
        quotient = (x - least) / np.where(scale > 0, scale, np.float32(1))
        codes = np.where(scale > 0, np.rint(quotient), 0).astype(np.uint8)
    pairs = np.concatenate([np.where(fine, bf16_bits(np.where(fine, least, 0)), 0x7FC0), bf16_bits(scale)], -1).astype(np.uint16)
    return codes, pairs


def write_row(pool, page, head, slot, page_size, codes, pairs):
    """One packed row into pool [pages, heads, bytes] (uint8)."""
    d = codes.shape[-1]
    pool[page, head, slot * (d // 2):(slot + 1) * (d // 2)] = codes[0::2] | codes[1::2] << 4
    at = page_size * (d // 2) + slot * 4
    pool[page, head, at:at + 4] = np.ascontiguousarray(pairs).view(np.uint8)


def read_row(pool, page, head, slot, page_size, d):
    """The float64 values that a row of the pool stands for."""
    b = pool[page, head, slot * (d // 2):(slot + 1) * (d // 2)]
    c = np.empty(d)
    c[0::2], c[1::2] = b & 15, b >> 4
    at = page_size * (d // 2) + slot * 4
    least, scale = bf16_values(np.ascontiguousarray(pool[page, head, at:at + 4]).view(np.uint16)).astype(np.float64)
    return least + scale * c


def append(k_new, v_new, k_pool, v_pool, block_tables, prefix_lens, chunk_lens, page_size):
    """bf16 bit patterns [T, Hkv, d] into copies of the pools; returns (k_pool, v_pool)."""
    out = []
    for new, pool in ((k_new, k_pool), (v_new, v_pool)):
        pool = pool.copy()
        codes, pairs = pack_rows(new)
        row = 0
        for i, C in enumerate(int(c) for c in chunk_lens):
            for t in range(C):
                pos = int(prefix_lens[i]) + t
                page = int(block_tables[i, pos // page_size])
                for h in range(new.shape[1]):
                    write_row(pool, page, h, pos % page_size, page_size, codes[row, h], pairs[row, h])
                row += 1
        out.append(pool)
    return tuple(out)


def attention(q, k_pool, v_pool, block_tables, prefix_lens, chunk_lens, page_size, num_kv_heads, sm_scale=0.0):
    """q: float64 [T, Hq, d].  Returns (out float64 [T, Hq, d], lse float64 [T, Hq], spread float64 [T, Hq, d]); spread is
    sum_j p_j max(|v_j|, |8 scale_j|) per element: what roundings of the p_j and v_j are relative to."""
    T, Hq, d = q.shape
    G = Hq // num_kv_heads
    scale = sm_scale if sm_scale > 0 else d ** -0.5
    out, lse, spread = np.zeros((T, Hq, d)), np.zeros((T, Hq)), np.zeros((T, Hq, d))
    row = 0
    for i, C in enumerate(int(c) for c in chunk_lens):
        P = int(prefix_lens[i])
        for g in range(num_kv_heads):
            if C == 0:
                continue
            where = [(int(block_tables[i, j // page_size]), g, j % page_size) for j in range(P + C)]
            K = np.array([read_row(k_pool, *w, page_size, d) for w in where])
            V = np.array([read_row(v_pool, *w, page_size, d) for w in where])
            at = [page_size * (d // 2) + w[2] * 4 + 2 for w in where]
            vs = np.array([bf16_values(np.ascontiguousarray(v_pool[w[0], w[1], a:a + 2]).view(np.uint16))[0] for w, a in zip(where, at)])
            big = np.maximum(np.abs(V), np.abs(8.0 * vs)[:, None])
            for t in range(C):
                n = P + t + 1
                s = scale * (K[:n] @ q[row + t, g * G:(g + 1) * G].T)               # [keys, heads]
                m = s.max(0)
                e = np.exp(s - m)
                out[row + t, g * G:(g + 1) * G] = e.T @ V[:n] / e.sum(0)[:, None]
                spread[row + t, g * G:(g + 1) * G] = e.T @ big[:n] / e.sum(0)[:, None]
                lse[row + t, g * G:(g + 1) * G] = m + np.log(e.sum(0))
        row += C
    return out, lse, spread
