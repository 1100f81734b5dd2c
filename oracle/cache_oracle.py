"""Float64 restatement of the attention of newly appended tokens (sliding
window, sinks, accumulated weights) and of the eviction by accumulated weight.
Plain numpy, written from the definitions; shares no code with the CUDA path.
"""

from __future__ import annotations

import numpy as np


def seen_mask(length: int, n: int, window: int, sinks: int) -> np.ndarray:
    """[n, length] truth values: which cached tokens the n newest ones see."""
    t = np.arange(length - n, length)[:, None]
    j = np.arange(length)[None, :]
    m = j <= t
    if window >= 0:
        m &= (j > t - window) | (j < sinks)
    return m


def attend_new(q, k, v, length, n, window=-1, sinks=0, scale=None):
    """One sequence.  q [n_new, H, D] (rows past n are padding), k and v
    [Hkv, T, D], all float64.  Returns a dict:
      out [n_new, H, D], lse [n_new, H], weight [Hkv, length],
      absout  sum_j p_j |v_j| per element (what rounding errors scale with),
      zmag    max over visible j of scale * sum_d |q_d k_jd| per row.
    """
    n_new, H, D = q.shape
    Hkv = k.shape[0]
    G = H // Hkv
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out = np.zeros((n_new, H, D))
    absout = np.zeros((n_new, H, D))
    lse = np.full((n_new, H), -np.inf)
    zmag = np.zeros((n_new, H))
    weight = np.zeros((Hkv, length))
    mask = seen_mask(length, n, window, sinks)
    for i in range(n):
        js = np.nonzero(mask[i])[0]
        if not js.size:
            continue
        for h in range(H):
            g = h // G
            kk, vv = k[g, js], v[g, js]
            z = scale * (kk @ q[i, h])
            m = z.max()
            e = np.exp(z - m)
            s = e.sum()
            p = e / s
            out[i, h] = p @ vv
            absout[i, h] = p @ np.abs(vv)
            lse[i, h] = m + np.log(s)
            zmag[i, h] = (scale * (np.abs(kk) @ np.abs(q[i, h]))).max()
            weight[g, js] += p
    return dict(out=out, lse=lse, weight=weight, absout=absout, zmag=zmag, mask=mask)


def evict(weight, length: int, keep: int, sinks: int, recent: int) -> np.ndarray:
    """Kept positions (ascending) of one kept set; weight [length] float32."""
    if length <= keep:
        return np.arange(length)
    w = np.asarray(weight[:length], dtype=np.float32)
    middle = np.arange(sinks, length - recent)
    rank = np.where(np.isnan(w[middle]), -np.inf, w[middle].astype(np.float64))
    nan = np.isnan(w[middle])
    order = np.lexsort((middle, nan, -rank))  # by weight, then NaN last, then position
    chosen = middle[order[: keep - sinks - recent]]
    return np.sort(np.concatenate([np.arange(sinks), chosen, np.arange(length - recent, length)]))
