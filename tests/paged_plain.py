"""Scored attention over a paged cache from its definition, in binary64."""
import numpy as np

from paged_cases import attention_tolerance


def seen(p, t, total, window=0, sinks=0, begin=None, end=None):
    """Which tokens t the queries at positions p see ([n, 1] and [1, total])."""
    high = p + 1 if end is None else np.minimum(end[:, None].astype(np.int64), total)
    see = (t < high)
    near = np.ones_like(see)
    if begin is not None:
        near &= t >= begin[:, None].astype(np.int64)
    if window:
        near &= t > p - window
    return see & (near | (t < sinks))


def scored_attention(batch, q, window=0, sinks=0, cap=0.0, slopes=None, begin=None, end=None,
                     sm_scale=None, out=None):
    """[T, H, D] binary64 over a paged_cases.Batch; rows of no sequence as in `out`."""
    out = np.zeros(q.shape) if out is None else out
    H, rep, sm = q.shape[1], q.shape[1] // batch.hkv, batch.D ** -0.5 if sm_scale is None else sm_scale
    K, V = batch.values(batch.k), batch.values(batch.v)
    for b in range(len(batch.new)):
        n, total = batch.new[b], batch.total[b]
        if n == 0:
            continue
        rows = slice(batch.cu[b], batch.cu[b + 1])
        t = np.arange(max(total, 0))[None]
        p = np.arange(total - n, total)[:, None]
        page = batch.table[b, t[0] // batch.page] if total > 0 else t[0]
        held = page >= 0
        k, v = (x[np.maximum(page, 0), :, t[0] % batch.page] for x in (K, V))  # [total, hkv, D]
        see = seen(p, t, total, window, sinks, None if begin is None else begin[rows],
                   None if end is None else end[rows]) & held[None]
        for h in range(H):
            kk = np.where(see.any(0)[:, None], k[:, h // rep], 0.0)
            x = sm * (q[rows, h].astype(np.float64) @ kk.T)
            if cap:
                x = cap * np.tanh(x / cap)
            if slopes is not None:
                x = x - float(slopes[h]) * np.abs(p - t)
            x = np.where(see, x, -np.inf)
            m = x.max(-1, keepdims=True, initial=-np.inf)
            w = np.exp(x - np.where(np.isfinite(m), m, 0.0))
            w = np.where(see, w, 0.0)
            s = w.sum(-1, keepdims=True)
            vv = v[:, h // rep]
            odd = ~np.isfinite(vv).all(-1)
            o = w @ np.where(odd[:, None], 0.0, vv)
            for j in np.nonzero(odd)[0]:  # reaches only the queries that see it
                o += np.where(see[:, j:j + 1], w[:, j:j + 1] * vv[j], 0.0)
            out[rows, h] = np.where(s > 0, o / np.where(s > 0, s, 1.0), 0.0)
    return out


def scored_tolerance(batch, q, exact, cap=0.0, sm_scale=None):
    """attention_tolerance (a cap's slope is 1 at most, so no error grows by it) and what
    the form adds to a score, in binary32: the cap's c - 2 c / (1 + e) some roundings of c,
    2^-22 of it with those of the exponential and the reciprocal; distances a rounding of
    what is added to scores that have any weight, 64 at most.  A score off by d changes an
    output by 2 d V at most."""
    V = np.nan_to_num(np.abs(batch.values(batch.v)), nan=0.0, posinf=0.0).max()
    return attention_tolerance(batch, q, exact, sm_scale) + V * 2 * (min(cap, 128.0) + 64) * 2.0 ** -22
