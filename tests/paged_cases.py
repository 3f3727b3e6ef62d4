"""Batches over a paged 4-bit cache for the tests: pools with their pages dealt
out in random order, as numpy arrays."""
import numpy as np


class Batch:
    """new[b] new tokens of sequence b whose cache holds total[b] tokens with
    them; `behind` rows of no sequence follow.  The cache's rows are random codes
    with a power of two for a scale (exact), or whatever the quantizer gives for
    normal rows; what no sequence holds is NaN where `nan` is set."""

    def __init__(self, seed, new, total, hkv, D, G, page, behind=0, exact=True, nan=True, spare=2):
        rng = np.random.default_rng(seed)
        self.rng, self.hkv, self.D, self.G, self.page = rng, hkv, D, G, page
        self.new, self.total = list(new), list(total)
        self.cu = np.cumsum([0] + self.new).astype(np.int32)
        self.lens = np.array(self.total, np.int32)
        self.T = int(self.cu[-1]) + behind
        need = [max(0, -(-t // page)) for t in self.total]
        self.pages = sum(need) + spare
        order = rng.permutation(self.pages)
        self.table = np.full((len(need), max(need + [1])), -1, np.int32)
        held = np.zeros((self.pages, page), bool)
        at = 0
        for b, x in enumerate(need):
            self.table[b, :x] = order[at:at + x]
            for i in range(x):
                held[self.table[b, i], :min(page, self.total[b] - i * page)] = True
            at += x
        self.held = held
        self.k = self._pool(exact, nan)
        self.v = self._pool(exact, nan)

    def _pool(self, exact, nan):
        import oracle
        rng, D, G = self.rng, self.D, self.G
        lead = (self.pages, self.hkv, self.page)
        if exact:
            c = rng.integers(0, 256, lead + (D // 2,), dtype=np.uint8)
            s = 2.0 ** rng.integers(-3, 0, lead + (D // G,))
            z = -s * rng.integers(4, 12, lead + (D // G,))
            s, z = s.astype(np.float16), z.astype(np.float16)
        else:
            x = rng.standard_normal((int(np.prod(lead)), D), dtype=np.float32)
            c, s, z = oracle.kv_quant_f32(x, G, 0.95)
            c, s, z = (a.reshape(lead + (-1,)) for a in (c, s, z))
        if nan:
            free = np.broadcast_to(~self.held[:, None], lead)
            s[free], z[free] = np.nan, np.inf
        return c, s, z

    def queries(self, H, sigma=1.0):
        return (self.rng.standard_normal((self.T, H, self.D)) * sigma).astype(np.float16)

    def values(self, pool):
        """Dequantized pool in binary64."""
        c, s, z = pool
        x = np.empty(c.shape[:-1] + (self.D,), np.float64)
        x[..., 0::2], x[..., 1::2] = c & 15, c >> 4
        return x * np.repeat(s.astype(np.float64), self.G, -1) + \
            np.repeat(z.astype(np.float64), self.G, -1)


def half_step():
    return 2.0 ** -11  # fp16: half a step, relative


def attention_tolerance(batch, q, exact, sm_scale=None):
    """How far an output may be from the exact one: with V the largest |vhat|,
    n the tokens and S the largest sm_scale sum_d |q_d| |khat_d|,
      V (1 + 1) 2^-11   a weight's and the output's rounding to fp16
      V n 2^-25         weights that are fp16 subnormals (the largest is 1, so
                        their sum is 1 at least)
      V (S + 2) 2^-18   binary32: sums of 256 products, exp2's argument and
                        value, sums of weights
      V (2 S + 1) 2^-11 keys and values rounded to fp16, where that is not exact
                        (a score off by d changes an output by 2 d V at most)."""
    n = max(batch.total + [1])
    kv, vv = (np.nan_to_num(np.abs(batch.values(p)), nan=0.0, posinf=0.0) for p in (batch.k, batch.v))
    V = vv.max()
    sm = batch.D ** -0.5 if sm_scale is None else sm_scale
    S = sm * np.abs(q.astype(np.float64)).sum(-1).max() * kv.max()
    S = min(S, sm * np.sqrt((q.astype(np.float64) ** 2).sum(-1).max() * (kv ** 2).sum(-1).max()))
    tol = 2 * half_step() + n * 2.0 ** -25 + (S + 2) * 2.0 ** -18
    if not exact:
        tol += (2 * S + 1) * half_step()
    return V * tol


# How far outputs may be off on average, relative to their own size.  A rounding to
# fp16 is off by 2^-10 / sqrt(12) = 2.8e-4 of a value at most as a root mean square
# (just above a power of two).  Few rows of one group: the output's alone.  Otherwise
# the weights' as well, and where they are not exact the values' and, through scores
# of about standard size, the keys': four alike, 5.6e-4.
ONE_ROUNDING, FOUR_ROUNDINGS = 4e-4, 1e-3


def few_rows(batch, H):
    """Whether the plan takes codes and weights unrounded (16 query rows of a
    sequence at most, one group a row)."""
    rep = H // batch.hkv
    rows = max(batch.new) * rep if len(batch.new) > 1 else batch.T * rep
    return batch.G == batch.D and rows <= 16


def relative_rms(batch, got, ref):
    """Largest root mean square error of a sequence's queries of one head, relative
    to that of the outputs themselves (an output of zeros has to be that)."""
    worst = 0.0
    for b in range(len(batch.new)):
        rows = slice(batch.cu[b], batch.cu[b + 1])
        e = np.sqrt(((got[rows].astype(np.float64) - ref[rows]) ** 2).sum((0, 2)))
        r = np.sqrt((ref[rows] ** 2).sum((0, 2)))
        assert (e[r == 0] == 0).all()
        worst = max(worst, (e[r > 0] / r[r > 0]).max(initial=0.0))
    return worst
