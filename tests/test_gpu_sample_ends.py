"""Sampling on the GPU at temperatures near the ends of binary32, where a step of a histogram
or a difference of logits is no binary32 number any more."""
import numpy as np
import pytest

from test_gpu_sample import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2404_00456_amd as q
    q.lib()
    return torch.device("cuda:0")


@pytest.mark.parametrize("V", [3001, 30000])
@pytest.mark.parametrize("T", [1e-36, 2e-37, 1e-37, 1e-38, 3e-40])
def test_temperatures_as_small_as_the_logits_differ(dev, V, T):
    """Cut to k, a list of them and too many for a list."""
    rng = np.random.default_rng(V)
    rows = 16
    x = (rng.standard_normal((rows, V)) * 2 * T).astype(np.float32)
    kw = dict(temperature=[T] * rows)
    for k in (2, 50, 1500, V // 2, V - 1):
        check(dev, x, rng.random(rows), top_k=[k] * rows, **kw)
    check(dev, x, rng.random(rows), top_k=[V // 2] * rows, top_p=[0.8] * rows, min_p=[0.01] * rows, **kw)
    check(dev, x, rng.random(rows), top_p=[0.8] * rows, **kw)
    # beside logits of ordinary size, which weigh nothing
    x[:, ::3] = rng.standard_normal((rows, len(x[0, ::3]))) - 9
    for k in (2, 50, V // 2, V - 1):
        check(dev, x, rng.random(rows), top_k=[k] * rows, **kw)


@pytest.mark.parametrize("V", [3001, 30000])
@pytest.mark.parametrize("T", [1e37, 1e38, 3e38])
def test_logits_further_apart_than_the_largest_number(dev, V, T):
    rng = np.random.default_rng(V)
    rows = 16
    x = (rng.uniform(-3.3e38, 3.3e38, (rows, V))).astype(np.float32)
    x[:, ::7] = -np.inf
    x[:, 1::50] = np.nan
    kw = dict(temperature=[T] * rows)
    for k in (2, 50, 1500, V // 2, V - 1):
        check(dev, x, rng.random(rows), top_k=[k] * rows, **kw)
        check(dev, x, rng.random(rows), top_k=[k] * rows, top_p=[0.7] * rows, **kw)
    # one far above all others
    x[:, 5] = 3.4e38
    x[:, 6:] = np.minimum(x[:, 6:], -3e38)
    x[:, :5] = -3e38
    for k in (2, 50, 1500, V // 2):
        check(dev, x, rng.random(rows), top_k=[k] * rows, **kw)


@pytest.mark.parametrize("V", [3001, 30000])
def test_an_infinite_temperature(dev, V):
    """Every finite logit weighs the same, whatever their size."""
    rng = np.random.default_rng(V)
    rows = 16
    x = (rng.uniform(-3.3e38, 3.3e38, (rows, V))).astype(np.float32)
    x[:, ::7] = -np.inf
    x[:, 1::50] = np.nan
    kw = dict(temperature=[np.inf] * rows)
    check(dev, x, rng.random(rows), **kw)
    for k in (2, 1500, V // 2):
        check(dev, x, rng.random(rows), top_k=[k] * rows, **kw)
    check(dev, x, rng.random(rows), top_p=[0.7] * rows, **kw)
    for p in (0.5, 1.0):
        check(dev, x, rng.random(rows), min_p=[p] * rows, **kw)
    # two infinite ones weigh as the others
    x[:, [3, V - 2]] = np.inf
    for k in (0, 1, 2, 3, V // 2):
        check(dev, x, rng.random(rows), top_k=[k] * rows, **kw)


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("V", [600, 11505, 60000])
@pytest.mark.parametrize("T", [1e-40, 1e-30, 1e-20, 1.0])
def test_the_largest_logits_are_zeros(dev, V, T, dtype):
    """More equal ones than a list holds, where the next logit below is a subnormal number."""
    rng = np.random.default_rng(V)
    rows = 8
    x = np.zeros((rows, V), dtype)
    x[::2, ::3] = -0.0
    x[4:, 1::2] = -np.inf
    x[6:, ::5] = -rng.integers(1, 9, x[6:, ::5].shape) * float(np.finfo(dtype).smallest_subnormal)
    kw = dict(temperature=[T] * rows)
    for mp in (1.0, 0.9, 1e-9):
        check(dev, x, rng.random(rows), min_p=[mp] * rows, **kw)
        check(dev, x, rng.random(rows), min_p=[mp] * rows, top_k=[V // 3] * rows, **kw)
    for p in (0.1, 0.9):
        check(dev, x, rng.random(rows), top_p=[p] * rows, **kw)
        check(dev, x, rng.random(rows), top_p=[p] * rows, top_k=[V // 3] * rows, **kw)


@pytest.mark.parametrize("few", [False, True])
def test_a_step_of_the_histogram_ends_at_zero(dev, few):
    """At this temperature a step of the first histogram reaches from the largest logit down
    to 0, and the next one begins at the number below it."""
    least, V, rows = 2.0 ** -149, 60000, 8
    rng = np.random.default_rng(7)
    x = np.full((rows, V), -np.inf, np.float32)
    for r in range(rows):
        at = rng.permutation(V)[:V // 6 if few else V]
        n = len(at) // 3
        x[r, at[:n]] = rng.choice([0.0, -0.0], n)
        x[r, at[n:]] = -least * rng.integers(1, 1000, len(at) - n)
        x[r, at[-1]] = 4445110 * least
    T = [3.874576352977353e-37] * rows
    n = np.isfinite(x[0]).sum()
    for k in (n // 3, n // 3 + 1, n // 3 + 2, n // 2, n - 1):
        check(dev, x, rng.random(rows), temperature=T, top_k=[k] * rows)
        check(dev, x, rng.random(rows), temperature=T, top_k=[k] * rows, top_p=[0.8] * rows)
