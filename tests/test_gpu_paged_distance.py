"""Slopes whose heaviest tokens are far from the query (negative slopes, sinks nearer than
a span): scores of hundreds of thousands between them must not cost the weights their last
bits."""
import numpy as np
import pytest

from paged_cases import Batch
from paged_plain import scored_tolerance
from test_gpu_paged_scored import check, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2404_00456_amd as q
    q.lib()
    return torch.device("cuda:0")


SLOPES = np.array([-8.0, 0.25, -0.3, 0.0], np.float32)


@pytest.mark.parametrize("new,total,D,G", [([1, 3], [30000, 700], 64, 64), ([2], [30000], 128, 32),
                                           ([4, 1], [20000, 64], 128, 128), ([40], [30000], 64, 64),
                                           ([30, 2], [20000, 3000], 128, 32), ([33], [9000], 256, 256)])
@pytest.mark.parametrize("form", [{}, dict(cap=6.0), dict(cap=3000.0), dict(sinks=5, window=4000),
                                  dict(spans=True)])
def test_negative_slopes(dev, new, total, D, G, form):
    """The farthest token weighs most."""
    bt = Batch(21, new, total, 1, D, G, 64, spare=1)
    kw = dict(form)
    if kw.pop("spans", False):
        rng = np.random.default_rng(3)
        p = np.concatenate([np.arange(t - n, t) for n, t in zip(new, total)])
        kw.update(begin=(p * rng.random(len(p)) * 0.5).astype(np.int32),
                  end=np.maximum((p * (0.6 + 0.6 * rng.random(len(p)))).astype(np.int32), 1), sinks=3)
    check(dev, bt, bt.queries(4, 8.0), slopes=SLOPES, **kw)


@pytest.mark.parametrize("D,G", [(64, 64), (128, 32), (256, 256)])
@pytest.mark.parametrize("slope", [8.0, -8.0, 0.3])
@pytest.mark.parametrize("cap", [0.0, 4000.0])
def test_sinks_nearer_than_the_span(dev, D, G, slope, cap):
    """The first queries of a prompt see its last tokens and a few sinks around them."""
    n, some, sinks = 24000, 40, 6
    bt = Batch(22, [n], [n], 1, D, G, 64, spare=1)
    qh = bt.queries(1, 8.0)
    begin, end = np.zeros(n, np.int32), np.zeros(n, np.int32)
    begin[:some], end[:some] = n - 700 + np.arange(some), n - np.arange(some) // 8
    got = run(dev, bt, qh, G, begin=begin, end=end, sinks=sinks, cap=cap, slopes=np.array([slope], np.float32))
    assert (got[some:] == 0).all()
    t, p = np.arange(n)[None], np.arange(some)[:, None]
    at = bt.table[0, t[0] // 64], 0, t[0] % 64
    K, V = bt.values(bt.k)[at], bt.values(bt.v)[at]
    see = (t < end[:some, None]) & ((t >= begin[:some, None]) | (t < sinks))
    x = D ** -0.5 * (qh[:some, 0].astype(np.float64) @ K.T)
    x = cap * np.tanh(x / cap) if cap else x
    x = np.where(see, x - float(np.float32(slope)) * np.abs(p - t), -np.inf)
    w = np.exp(x - x.max(-1, keepdims=True))
    ref = w @ V / w.sum(-1, keepdims=True)
    assert np.abs(got[:some, 0] - ref).max() <= scored_tolerance(bt, qh, True, cap)
