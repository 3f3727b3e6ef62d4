"""Spans of scored attention that end before they begin, beside values that are not finite,
and slopes whose heaviest tokens are far away: in the kernels for few rows and in the
tiles, whole and split."""
import numpy as np
import pytest

from paged_cases import Batch
from paged_plain import scored_attention, scored_tolerance
from test_gpu_paged_scored import run

pytestmark = pytest.mark.gpu

LARGEST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2404_00456_amd as q
    q.lib()
    return torch.device("cuda:0")


def compare(bt, got, ref, tol, nothing):
    """Finite where the definition is, within tol there, and 0 in rows `nothing` [T]."""
    fine = np.isfinite(ref)
    assert fine.any()
    assert np.array_equal(fine, np.isfinite(got))
    assert np.abs(got[fine].astype(np.float64) - ref[fine]).max() <= tol
    assert (got[nothing] == 0).all()


# spans of a block's rows in turn, over a context of 160 (times `far`)
TURNS = {
    "begin_past_the_end": [(0, 100), (120, 100)],
    "begin_far_past": [(0, 100), (10000, 101)],
    "begin_at_the_largest": [(0, 100), (LARGEST, 100)],
    "end_at_0": [(0, 100), (0, 0)],
    "end_before_0": [(30, 100), (0, -5)],
    "third_row": [(0, 50), (1000, 50), (20, 50)],
    "third_row_largest": [(0, 50), (LARGEST, LARGEST), (20, 50)],
    "first_of_all": [(LARGEST, LARGEST), (0, 100)],
}


@pytest.mark.parametrize("turns", TURNS)
@pytest.mark.parametrize("sinks", [0, 3])
@pytest.mark.parametrize("far", [1, 20])  # 20: the block's tokens are split
@pytest.mark.parametrize("new,D,G", [(2, 128, 32), (3, 128, 64), (4, 128, 32), (4, 64, 32), (3, 256, 32),
                                     (2, 128, 128), (40, 128, 128), (40, 64, 32)])
def test_spans_that_see_nothing_beside_values_that_are_not_finite(dev, new, D, G, far, sinks, turns):
    """An undefined value at the first token of the first span that has any (in one cache
    head) and an infinite one at its last (in another) reach the rows that see them, and no
    other row of their blocks."""
    total = 160 * far
    bt = Batch(17, [new, 1], [total, 50], 3, D, G, 16)
    scaled = [tuple(int(x) if abs(x) > 10 ** 6 else int(x) * far for x in s) for s in TURNS[turns]]
    begin = np.array([scaled[i % len(scaled)][0] for i in range(new)] + [0], np.int64).astype(np.int32)
    end = np.array([scaled[i % len(scaled)][1] for i in range(new)] + [50], np.int64).astype(np.int32)
    first, last = next((max(b, sinks), e - 1) for b, e in scaled if b < e)
    for x, (t, value) in enumerate(((first, np.nan), (last, np.inf))):
        bt.v[1 + x][bt.table[0, t // 16], x, t % 16, -x] = value
    qh = bt.queries(12)
    kw = dict(begin=begin, end=end, sinks=sinks)
    got = run(dev, bt, qh, G, **kw)
    with np.errstate(invalid="ignore"):
        ref = scored_attention(bt, qh, begin=begin, end=end, sinks=sinks)
        tol = scored_tolerance(bt, qh, True)
    assert not np.isfinite(ref).all()
    high = np.minimum(end.astype(np.int64), np.repeat(bt.lens, bt.new))
    nothing = (begin >= high) & (np.minimum(high, sinks) <= 0)
    assert nothing[:new].any() or sinks
    compare(bt, got, ref, tol, nothing)
    # the third cache head holds no such value
    assert np.isfinite(got[:, 8:]).all()


@pytest.mark.parametrize("G", [32, 128])
@pytest.mark.parametrize("sinks", [0, 2])
def test_guessed_tokens_on_both_sides_of_a_document(dev, G, sinks):
    """Begins that lie 30000 tokens apart, with a value that is not finite in each part."""
    total = 30100
    bt = Batch(18, [4], [total], 1, 128, G, 64, spare=1)
    begin = np.array([0, 0, total - 2, total - 2], np.int32)
    end = np.arange(total - 3, total + 1).astype(np.int32)
    for t in (20000, total - 1):
        bt.v[2][bt.table[0, t // 64], 0, t % 64, 0] = np.nan
    qh = bt.queries(4)
    got = run(dev, bt, qh, G, begin=begin, end=end, sinks=sinks)
    with np.errstate(invalid="ignore"):
        ref = scored_attention(bt, qh, begin=begin, end=end, sinks=sinks)
        tol = scored_tolerance(bt, qh, True)
    assert np.isnan(ref[:2, :, 0]).all() and np.isnan(ref[3, :, 0]).all() and np.isfinite(ref[2]).all()
    compare(bt, got, ref, tol, np.zeros(4, bool))


@pytest.mark.parametrize("D,G,rep", [(64, 32, 4), (128, 32, 2), (128, 64, 5), (256, 32, 4), (256, 64, 3)])
@pytest.mark.parametrize("seed", range(6))
def test_any_spans_among_values_that_are_not_finite(dev, D, G, rep, seed):
    """A value in twenty is not finite; spans, windows and sinks of any kind."""
    rng = np.random.default_rng(seed)
    new, total = [1 + 15 // rep, 2, 1], [int(rng.integers(40, 2500)), int(rng.integers(5, 300)), 77]
    bt = Batch(30 + seed, new, total, 2, D, G, 16, behind=1)
    held = np.argwhere(bt.held)
    for page, at in held[rng.random(len(held)) < 0.05]:
        bt.v[1 + rng.integers(2)][page, rng.integers(2), at, rng.integers(D // G)] = rng.choice([np.nan, np.inf, -np.inf])
    begin, end = np.zeros(bt.T, np.int32), np.zeros(bt.T, np.int32)
    for b in range(len(new)):
        for i in range(bt.cu[b], bt.cu[b + 1]):
            # mostly near one another, so that there are rows that see none of these values
            begin[i] = rng.choice([rng.integers(0, total[b]), total[b] - 9, LARGEST, -7])
            end[i] = rng.choice([begin[i] % 2 ** 30 + rng.integers(0, 12), total[b], 0, LARGEST])
    qh = bt.queries(2 * rep)
    kw = dict(begin=begin, end=end, sinks=int(rng.choice([0, 2])), window=int(rng.choice([0, 0, 20])))
    got = run(dev, bt, qh, G, **kw)[:bt.cu[-1]]
    with np.errstate(invalid="ignore"):
        ref = scored_attention(bt, qh, **kw)[:bt.cu[-1]]
        tol = scored_tolerance(bt, qh, True)
    p = np.concatenate([np.arange(t - n, t) for n, t in zip(new, total)])
    low = np.maximum(begin[:len(p)], p - kw["window"] + 1 if kw["window"] else 0)
    high = np.minimum(end[:len(p)].astype(np.int64), np.repeat(bt.lens, new))
    compare(bt, got, ref, tol, (low >= high) & (np.minimum(high, kw["sinks"]) <= 0))
