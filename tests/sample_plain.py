"""Sampling from its definition: binary64 exponentials, whole numbers of Python."""
import numpy as np


def one_of(vocab):
    bits = (vocab - 1).bit_length()
    return min(51, 62 - bits)


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    rows, V = logits.shape
    out = []
    for r in range(rows):
        x = logits[r].astype(np.float64)
        x = np.where(np.isnan(x), -np.inf, x)
        best = int(np.argmax(x))
        order = np.argsort(-x, kind="stable")
        x = np.minimum(x, float(np.finfo(np.float32).max))
        m = x[best]
        if m == -np.inf:
            out.append(-1)
            continue
        t = 1.0 if temperature is None else float(temperature[r])
        if not t > 0:
            out.append(best)
            continue
        order = order[x[order] > -np.inf]
        k = 0 if top_k is None else int(top_k[r])
        if k > 0:
            order = order[:k]
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.exp(np.where(x > -np.inf, (x - m) / t, -np.inf))
        whole = np.rint(w * 2.0 ** one_of(V)).astype(np.int64)  # below 2^52 each
        p = 1.0 if top_p is None else float(top_p[r])
        if p < 1:
            upto = np.cumsum(whole[order])  # below 2^63
            target = int(np.ceil(max(1.0, p * float(upto[-1]))))
            order = order[:int(np.searchsorted(upto, min(target, int(upto[-1])))) + 1]
        least = 0.0 if min_p is None else float(min_p[r])
        if least > 0:
            order = order[w[order] >= min(least, 1.0)]
        order = np.sort(order)
        upto = np.cumsum(whole[order])
        uu = float(u[r])
        share = int(min(uu, 1.0) * float(upto[-1])) if uu > 0 else 0
        share = min(share, int(upto[-1]) - 1)
        out.append(int(order[int(np.searchsorted(upto, share, side="right"))]))
    return np.array(out, np.int32)
