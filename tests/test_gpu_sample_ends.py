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
