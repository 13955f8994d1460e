"""Oracle of attention over a latent cache in 64 bits, absorbed and expanded forms."""
import numpy as np


def rows_of(cache, b, n, table=None):
    """The n rows of sequence b from [blk, tok, Dk] storage."""
    if table is None:
        return cache[b, :n]
    ps = cache.shape[1]
    ids = np.clip(table[b, :-(-n // ps)], 0, cache.shape[0] - 1)
    return cache[ids].reshape(-1, cache.shape[2])[:n]


def verify(q, cache, lens, k, sm_scale, Dc, table=None):
    """q [B, k+1, Hq, Dk], cache as values (fp64): (out, lse, sum_j p_j |c_j|)."""
    B, _, Hq, _ = q.shape
    cap = cache.shape[1] * (1 if table is None else table.shape[1])
    out, lse = np.zeros((B, k + 1, Hq, Dc)), np.full((B, k + 1, Hq), -np.inf)
    size = np.zeros_like(out)
    for b in range(B):
        n = min(max(int(lens[b]), 0), cap)
        rows = rows_of(cache, b, n, table)
        for i in range(k + 1):
            seen = rows[:max(0, n - k + i)]
            if len(seen) == 0:
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                s = q[b, i] @ seen.T * sm_scale
                m = s.max(1, keepdims=True)
                p = np.exp(s - np.where(np.isneginf(m), 0, m))
                l = p.sum(1, keepdims=True)
                some = l[:, 0] != 0
                lse[b, i, some] = (m + np.log(l))[some, 0]
                out[b, i, some] = (p / l @ seen[:, :Dc])[some]
                size[b, i, some] = (p / l @ np.abs(seen[:, :Dc]))[some]
    return out, lse, size


def expanded(q_nope, q_rope, rows, visible, w_k, w_v, sm_scale):
    """Ordinary attention of one token's heads: keys [W_k c, r], values W_v c.
    q_nope [Hq, Dn], q_rope [Hq, Dr], rows [n, Dc + Dr], w_k [Hq, Dn, Dc], w_v [Hq, Dv, Dc]."""
    Dc = w_k.shape[2]
    out = []
    for h in range(q_nope.shape[0]):
        keys = np.concatenate([rows[:visible, :Dc] @ w_k[h].T, rows[:visible, Dc:]], 1)
        s = keys @ np.concatenate([q_nope[h], q_rope[h]]) * sm_scale
        p = np.exp(s - s.max())
        out.append(p / p.sum() @ (rows[:visible, :Dc] @ w_v[h].T))
    return np.stack(out)
