"""Oracle of linear attention with a decay per head, token by token in fp64:

    S_t = exp(g_t) S_{t-1} + k_t v_t^T,      o_t = scale S_t^T q_t,

per request and head, resumed from and stored to slots of a pool, snapshotted at the multiples p of an interval with
prefix < p <= prefix + chunk.

TEST INFRASTRUCTURE ONLY: plain numpy; shares no code with the library.
"""
import numpy as np


def linear_chunk(q, k, v, log_decay, chunk_lens, state_pool, state_in, state_out, prefix_lens=None, snap_interval=0, snap_slots=None,
                 scale=1.0):
    """q, k, v: [T, H, d]; log_decay: [H] or [T, H]; state_pool: float64 [slots, H, d, d], updated in place.  Returns
    (o, size): size is what o's terms add up to without their signs, which roundings of them are relative to."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    T, H, d = q.shape
    with np.errstate(under="ignore"):
        a = np.exp(np.broadcast_to(np.asarray(log_decay, np.float64), (T, H)))
    o, size = np.zeros((T, H, d)), np.zeros((T, H, d))
    row = 0
    for i, C in enumerate(int(c) for c in chunk_lens):
        P = 0 if prefix_lens is None else int(prefix_lens[i])
        S = np.zeros((H, d, d)) if state_in[i] < 0 else state_pool[state_in[i]].copy()
        A = np.abs(S)
        n = 0
        for t in range(row, row + C):
            S = a[t][:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
            A = a[t][:, None, None] * A + np.abs(k[t])[:, :, None] * np.abs(v[t])[:, None, :]
            o[t] = scale * np.einsum("hkv,hk->hv", S, q[t])
            size[t] = abs(scale) * np.einsum("hkv,hk->hv", A, np.abs(q[t]))
            if snap_interval > 0 and (P + t - row + 1) % snap_interval == 0:
                if snap_slots is not None and n < snap_slots.shape[1] and snap_slots[i, n] >= 0:
                    state_pool[snap_slots[i, n]] = S
                n += 1
        if state_out[i] >= 0:
            state_pool[state_out[i]] = S
        row += C
    return o, size
