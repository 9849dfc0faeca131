"""Float64 definitions of the operators on a caller's own tensors: rotary
positions and attention of one sequence's rows under the three masks."""
from __future__ import annotations

import numpy as np

MASKS = ("full", "causal", "shadow")


def rope(x, pos, freq, rotary_dim, interleaved=False, magnitude=1.0, inverse=False):
    """x [tokens, heads, head_dim] turned by pos[t] * freq[j]; float64."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    ang = np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64)[None, :]
    c, s = (magnitude * np.cos(ang))[:, None, :], (magnitude * np.sin(ang))[:, None, :]
    if inverse:
        s = -s
    r = rotary_dim
    ia, ib = (np.arange(0, r, 2), np.arange(1, r, 2)) if interleaved else (np.arange(r // 2), np.arange(r // 2, r))
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def sees(mask, n_q, n_kv, block_len=0, cur_start=0):
    """bool [n_q, n_kv]: which keys each row sees."""
    i, j = np.arange(n_q)[:, None], np.arange(n_kv)[None, :]
    if mask == "full":
        return np.ones((n_q, n_kv), bool)
    if mask == "causal":
        return j <= n_kv - n_q + i
    s = i - (n_q - block_len)
    return np.where(s < 0, j < n_kv - block_len, j != cur_start + s)


def attention(q, k, v, scale, visible):
    """One sequence: q [n_q, Hq, hd], k and v [n_kv, Hk, hd], visible [n_q, n_kv].  Returns (o, lse, a, d): a is the
    softmax-weighted mean of |v| and d the largest sum of |q_e k_e| * scale over a row's keys, which size the
    tolerances.  Values at keys a row does not see do not enter."""
    n_q, hq, hd = q.shape
    hk = k.shape[1]
    o, a = np.zeros((n_q, hq, hd)), np.zeros((n_q, hq, hd))
    lse, d = np.full((n_q, hq), -np.inf), np.zeros((n_q, hq))
    for h in range(hq):
        kk, vv = k[:, h // (hq // hk)], v[:, h // (hq // hk)]
        for i in range(n_q):
            w = visible[i]
            if not w.any():
                continue
            z = (kk[w] @ q[i, h]) * scale
            m = z.max()
            p = np.exp(z - m)
            lse[i, h] = m + np.log(p.sum())
            p = p / p.sum()
            with np.errstate(invalid="ignore"):
                o[i, h] = p @ vv[w]
                a[i, h] = p @ np.abs(vv[w])
            d[i, h] = (np.abs(kk[w]) @ np.abs(q[i, h])).max() * scale
    return o, lse, a, d
