"""Attention of new tokens behind a cached prefix, in float64, from the logical sequence (never a cache)."""
import numpy as np

from oracle.attention import group_of


def visible(start, t, streaming, n_sink, window, evict):
    """Boolean [len(t), start + max(t) + 1]: positions that new tokens t, at start + t, see.

    evict: streaming heads see the sinks, the window before the new tokens and the new tokens, as after the eviction that
    follows each chunk; else the sinks and the window of the token itself."""
    p = start + np.asarray(t, dtype=np.int64)[:, None]
    j = np.arange(int(p.max()) + 1, dtype=np.int64)[None, :]
    on = j <= p
    if streaming:
        on &= (j < n_sink) | (j >= (start - window if evict else p - window + 1))
    return on


def extend(q, k, v, start, streaming, n_sink, window, evict, rows=None):
    """q [n, Hq, D] new queries, k, v [start + n, Hkv, D] the whole sequence, streaming [Hkv] -> out [rows, Hq, D], and
    sum_j w_j |v_j| and max_j sum_d |q_d k_jd| / sqrt(D) of every row, which error bounds need."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    rows = np.arange(q.shape[0]) if rows is None else np.asarray(rows)
    n, hq, d = len(rows), q.shape[1], q.shape[2]
    out, mass, size = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq, 1))
    for g in range(k.shape[1]):
        on = visible(start, rows, streaming[g], n_sink, window, evict)
        kk, vv = k[:on.shape[1], g], v[:on.shape[1], g]
        for h in [h for h in range(hq) if group_of(h, hq, k.shape[1]) == g]:
            s = np.where(on, q[rows, h] @ kk.T / np.sqrt(d), -np.inf)
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            out[:, h], mass[:, h] = w @ vv, w @ np.abs(vv)
            size[:, h, 0] = np.where(on, np.abs(q[rows, h]) @ np.abs(kk).T, 0).max(1) / np.sqrt(d)
    return out, mass, size
