"""What one query of a chunk may not see has no influence on its output, whatever
it holds: cached rows that are not finite, seen by some queries of a block and not
by others."""
import numpy as np
import pytest

from paged_cases import Batch, attention_tolerance
from test_gpu_paged import attend, dev  # noqa: F401

pytestmark = pytest.mark.gpu


def sees(total, new, t, window, sinks):
    """Which of the new queries of a sequence see token t."""
    p = np.arange(total - new, total)
    return (t <= p) & ((window == 0) | (t > p - window) | (t < sinks))


FORMS = [
    # new, total, H, hkv, D, G, page, window, sinks: tiles of 64, 128 and 256 rows,
    # few rows in groups and in one, long and short sequences apart
    ([8], [100], 8, 1, 128, 128, 16, 0, 0),
    ([16], [100], 8, 1, 128, 32, 16, 0, 0),
    ([64], [300], 16, 2, 128, 128, 64, 0, 0),
    ([300], [300], 2, 2, 128, 64, 16, 0, 0),
    ([70], [200], 8, 2, 64, 32, 16, 40, 3),
    ([9], [80], 4, 1, 64, 64, 16, 0, 0),
    ([40], [90], 2, 1, 256, 64, 32, 0, 0),
    ([90], [200], 5, 1, 256, 256, 16, 33, 1),
    ([5, 4], [70, 40], 4, 2, 128, 32, 16, 0, 0),
    ([4, 12], [90, 140], 2, 2, 128, 64, 16, 7, 2),
    ([6, 3], [70, 9], 2, 1, 256, 32, 16, 0, 0),
    ([7], [100], 4, 2, 64, 32, 16, 5, 0),
    ([7, 2], [100, 30], 8, 4, 128, 128, 16, 0, 0),
    ([1, 60, 4, 2], [30, 90, 100, 20], 16, 4, 128, 64, 16, 0, 0),
]
KINDS = {"scale inf": ("s", np.inf), "zero -inf": ("z", -np.inf), "scale nan": ("s", np.nan),
         "zero nan": ("z", np.nan), "past fp16": ("s", 6000.0)}


@pytest.mark.parametrize("most", [None, 1 << 16])
@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("new,total,H,hkv,D,G,page,window,sinks", FORMS)
def test_values_of_unseen_tokens(dev, orc, new, total, H, hkv, D, G, page, window, sinks, kind, most):
    """Values that are not finite (an infinite or undefined constant of a group, or
    code 15 of a scale that passes what fp16 holds), in some new tokens of each
    sequence and one older one: elements that the definition leaves finite are
    right, the others are not finite."""
    bt = Batch(7 * D + G + H, new, total, hkv, D, G, page, behind=1)
    qh = bt.queries(H)
    tol = attention_tolerance(bt, qh, True)
    c, s, z = bt.v
    hidden = np.ones((bt.T, H), bool)  # queries that see none of these tokens
    for b, (n, end) in enumerate(zip(new, total)):
        for i, t in enumerate(sorted({end - 1, end - (n + 1) // 2, max(0, end - n - 1)})):
            if i == 0 and window == 0:
                continue  # every query would see it
            h, g = (b + i) % hkv, i % (D // G)
            pg, slot = bt.table[b, t // page], t % page
            field, value = KINDS[kind]
            (s if field == "s" else z)[pg, h, slot, g] = value
            if kind == "past fp16":
                c[pg, h, slot] = 0xFF
            rows = bt.cu[b] + np.flatnonzero(sees(end, n, t, window, sinks))
            hidden[rows[:, None], np.arange(H) // (H // hkv) == h] = False
    ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, G, window, sinks,
                              out=np.full(qh.shape, 9.0))
    got = attend(dev, bt, qh, window=window, n_sinks=sinks,
                 **({} if most is None else dict(max_seq_len=most))).astype(np.float64)
    live = hidden[:bt.cu[-1]]
    assert live.any() and not live.all()
    assert np.isfinite(got[hidden]).all(), "a value reaches a query that may not see it"
    assert np.abs(got[hidden] - ref[hidden]).max() <= tol
    if kind != "past fp16":  # (one past fp16 may be taken as infinite)
        fin = np.isfinite(ref)
        assert not np.isfinite(got[~fin]).any() and np.isfinite(got[fin]).all()
        assert np.abs(got[fin] - ref[fin]).max() <= tol


@pytest.mark.parametrize("new,total,H,hkv,D,G,page,window,sinks", FORMS)
def test_keys_of_unseen_tokens(dev, orc, new, total, H, hkv, D, G, page, window, sinks):
    """The same for keys: a query that sees one has no finite output."""
    bt = Batch(5 * D + G + H, new, total, hkv, D, G, page, behind=1)
    qh = bt.queries(H)
    tol = attention_tolerance(bt, qh, True)
    hidden = np.ones((bt.T, H), bool)
    for b, (n, end) in enumerate(zip(new, total)):
        t, h = end - (n + 1) // 2, b % hkv
        bt.k[1][bt.table[b, t // page], h, t % page] = np.nan
        rows = bt.cu[b] + np.flatnonzero(sees(end, n, t, window, sinks))
        hidden[rows[:, None], np.arange(H) // (H // hkv) == h] = False
    ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, G, window, sinks,
                              out=np.full(qh.shape, 9.0))
    got = attend(dev, bt, qh, window=window, n_sinks=sinks).astype(np.float64)
    assert np.isfinite(got[hidden]).all() and not np.isfinite(got[~hidden]).any()
    assert np.abs(got[hidden] - ref[hidden]).max() <= tol


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("new,total,H,hkv,D,G,page,window,sinks", FORMS)
def test_queries_that_are_not_finite(dev, orc, new, total, H, hkv, D, G, page, window, sinks, bad):
    """One element of some queries that is not finite: their outputs are not, and no
    other query's changes."""
    bt = Batch(11 * D + G + H, new, total, hkv, D, G, page, behind=1)
    qh = bt.queries(H)
    tol = attention_tolerance(bt, qh, True)
    ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, G, window, sinks,
                              out=np.full(qh.shape, 9.0))
    hit = np.zeros((bt.T, H), bool)
    for b, n in enumerate(new):
        hit[bt.cu[b] + n // 2, b % H] = hit[bt.cu[b + 1] - 1, H - 1] = True
    qh[hit, D // 3] = bad
    got = attend(dev, bt, qh, window=window, n_sinks=sinks).astype(np.float64)
    assert not np.isfinite(got[hit]).any() and np.isfinite(got[~hit]).all()
    assert np.abs(got[~hit] - ref[~hit]).max() <= tol
