"""Sampling on the GPU against its definition (tests/sample_plain.py): tokens are whole
numbers and have to be equal.  (The exponentials of both sides are off by some 1e-13 of a
weight; that decides a token once in 10^7 rows.)"""
import numpy as np
import pytest

from sample_plain import sample

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2404_00456_amd as q
    q.lib()
    return torch.device("cuda:0")


def D_(a, dev):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dev)


def check(dev, logits, u, lead=0, **kw):
    """`lead`: elements before the first row and between the rows."""
    import torch
    import paper_2404_00456_amd as q
    f = {"temperature": np.float32, "top_k": np.int32, "top_p": np.float32, "min_p": np.float32}
    kw = {n: np.asarray(v, f[n]) for n, v in kw.items()}
    rows, V = logits.shape
    wide = torch.full((rows * (V + lead) + lead,), float("inf"), device=dev,
                      dtype=torch.float16 if logits.dtype == np.float16 else torch.float32)
    x = wide[lead:].view(rows, V + lead)[:, :V]
    x.copy_(D_(logits, dev))
    got = q.quarot_sample(x, D_(np.asarray(u, np.float32), dev), **{n: D_(v, dev) for n, v in kw.items()})
    with np.errstate(all="ignore"):
        ref = sample(logits, np.asarray(u, np.float32), **kw)
    assert np.array_equal(got.cpu().numpy(), ref), (got.cpu().numpy()[got.cpu().numpy() != ref],
                                                    ref[got.cpu().numpy() != ref])
    return ref


def likely(rng, rows, V, sigma, dtype=np.float16):
    x = rng.standard_normal((rows, V)) * sigma
    for r in range(rows):
        x[r, rng.integers(0, V, 10)] = 4 * sigma + rng.standard_normal(10) * 2
    return x.astype(dtype)


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("rows,V,lead", [(40, 1, 0), (40, 2, 1), (50, 7, 0), (50, 511, 3), (40, 513, 0),
                                         (40, 1000, 1), (30, 8191, 5), (20, 32000, 0), (12, 50003, 0),
                                         (9, 131072, 0)])
def test_limits_alone_and_together(dev, rows, V, lead, dtype):
    rng = np.random.default_rng(V)
    x = likely(rng, rows, V, 2.0, dtype)
    u = rng.random(rows)
    check(dev, x, u, lead)
    for T in (0.3, 1.0, 3.0):
        t = np.full(rows, T)
        k = rng.integers(-1, min(V, 60) + 2, rows)
        p = rng.choice([0.1, 0.5, 0.9, 0.99, 1.0], rows)
        mp = rng.choice([0.0, 0.01, 0.3, 1.0], rows)
        check(dev, x, u, lead, temperature=t, top_k=k)
        check(dev, x, u, lead, temperature=t, top_p=p)
        check(dev, x, u, lead, temperature=t, min_p=mp)
        check(dev, x, u, lead, temperature=t, top_k=k * 40, top_p=p, min_p=mp)


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_equal_logits(dev, dtype):
    """Few values, so that every cut falls among equal ones; rows of one value."""
    rng = np.random.default_rng(1)
    rows, V = 24, 30011
    x = rng.choice([-3.0, -1.0, 0.0, -0.0, 0.5, 1.0], (rows, V)).astype(dtype)
    x[:6] = 2.5
    u = rng.random(rows)
    k = np.array([1, 2, 100, 1000, 20000, V] * 4)
    p = np.tile(np.repeat([0.0, 1e-6, 0.25, 0.75], 3), 2)
    check(dev, x, u, top_k=k)
    check(dev, x, u, top_p=p)
    check(dev, x, u, top_k=k, top_p=p, min_p=np.full(rows, 0.05), temperature=np.full(rows, 0.8))
    check(dev, x, u, temperature=np.zeros(rows))
    # zeros of either sign are equal: the lowest index is the largest logit's
    z = np.full((2, 600), -0.0, dtype)
    z[0, 5] = 0.0
    assert check(dev, z, [0.0, 0.5], temperature=[0, 0]).tolist() == [0, 0]
    assert check(dev, z, [0.0, 0.0], top_k=[1, 1]).tolist() == [0, 0]


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_masks_and_what_is_no_number(dev, dtype):
    rng = np.random.default_rng(2)
    rows, V = 16, 5003
    x = likely(rng, rows, V, 3.0, dtype)
    x[rng.random((rows, V)) < 0.9] = -np.inf
    x[0] = -np.inf
    x[1] = np.nan
    x[2] = -np.inf
    x[2, 4000] = -60000.0
    x[3, ::7] = np.nan
    x[4, 77] = np.inf
    x[5, 30:2000:3] = np.inf
    x[6] = -np.inf
    x[6, V - 1] = 1.0
    x[7] = np.finfo(dtype).min
    x[8, 0] = np.finfo(dtype).max
    u = rng.random(rows)
    for kw in ({}, dict(temperature=np.full(rows, 0.0)), dict(top_k=np.full(rows, 5)),
               dict(top_p=np.full(rows, 0.9)), dict(min_p=np.full(rows, 0.5)),
               dict(top_k=np.full(rows, 300), top_p=np.full(rows, 0.8), temperature=np.full(rows, 5.0))):
        ref = check(dev, x, u, 1, **kw)
        assert ref[0] == ref[1] == -1 and ref[2] == 4000 and ref[4] == 77 and ref[6] == V - 1


def test_numbers_at_their_ends(dev):
    rng = np.random.default_rng(3)
    inf, nan = np.inf, np.nan
    ends = [0.0, -1.0, nan, 1e-45, 1e-38, 1e-3, 1.0, 1e4, 3e38, inf]
    x = likely(rng, len(ends), 3001, 2.0)
    for u in (0.0, 2.0 ** -24, 0.5, 1 - 2.0 ** -24, 1.0, 7.0, -1.0, nan, inf):
        check(dev, x, [u] * len(ends), temperature=ends)
        check(dev, x, [u] * len(ends), temperature=ends, top_p=[0.7] * len(ends))
    p = [0.0, -3.0, 1e-30, 0.5, 1 - 2.0 ** -24, 1.0, 2.0, nan, inf, -inf]
    for mp in (0.0, -1.0, 1e-30, 1.0, 2.0, nan, inf):
        check(dev, x, rng.random(10), top_p=p, min_p=[mp] * 10)
    check(dev, x, rng.random(10), top_k=[0, -1, -2 ** 31, 2 ** 31 - 1, 3001, 3000, 1, 2, 3002, 7])


def test_flat_rows_use_every_level(dev):
    """Far more tokens in a step of the first histogram than are ranked together."""
    rng = np.random.default_rng(4)
    for V, dtype in ((131072, np.float16), (60001, np.float32), (1 << 20, np.float32)):
        rows = 3 if V < 1 << 20 else 1
        x = (rng.standard_normal((rows, V)) * 0.01 + 5).astype(dtype)
        for T in (1.0, 50.0):
            kw = dict(temperature=[T] * rows)
            check(dev, x, rng.random(rows), **kw)
            check(dev, x, rng.random(rows), top_k=[V // 3] * rows, **kw)
            check(dev, x, rng.random(rows), top_p=[0.6] * rows, **kw)
            check(dev, x, rng.random(rows), top_k=[V // 2] * rows, top_p=[0.9] * rows, min_p=[0.9] * rows, **kw)


def test_infinite_beside_the_largest_number(dev):
    """They weigh the same, and the infinite ones come first."""
    inf, big = np.float32(np.inf), np.finfo(np.float32).max
    x = np.tile(np.array([1.0, big, inf, big, inf, -inf, big], np.float32), (8, 300))
    u = (np.arange(8) + 0.5) / 8
    for kw in ({}, dict(temperature=[0.0] * 8), dict(top_k=[1, 2, 3, 599, 600, 601, 1500, 0]),
               dict(top_p=[1e-6, 0.1, 0.3, 0.4, 0.41, 0.7, 0.99, 1.0]), dict(min_p=[0.5] * 8)):
        check(dev, x, u, **kw)


@pytest.mark.parametrize("V", [600, 30000])
def test_cuts_at_logits_near_zero(dev, V):
    """Where the least logit of a step of the exponent is next to 0 a rounding of the largest
    logit is billions of numbers there."""
    rng = np.random.default_rng(V)
    rows, steps = 12, 8 * 40 + 7.5
    x = (rng.standard_normal((rows, V)) * 10.0 ** rng.integers(-30, -6, (rows, V))).astype(np.float32)
    x[:, V // 2] = 1.0
    T = 256 / np.log(2) / steps
    share = 1 / (1 + V * np.exp(-1 / T))  # of the one token
    p = share + (1 - share) * rng.random(rows)
    for t in (T, T * (1 + 1e-6), T * (1 - 1e-6)):
        kw = dict(temperature=[t] * rows)
        check(dev, x, rng.random(rows), top_p=p, **kw)
        check(dev, x, rng.random(rows), min_p=np.exp(-1 / t) * (1 + rng.standard_normal(rows) * 1e-7), **kw)
        check(dev, x, rng.random(rows), top_p=p, top_k=rng.integers(1, V, rows), **kw)


def test_frequencies(dev):
    """Evenly spaced random numbers give each token its share of them, to one."""
    import torch
    import paper_2404_00456_amd as q
    n = 4096
    x = torch.tensor([0.0, 1.0, -2.0, 0.5, -np.inf, 1.0], device=dev).half()
    u = (torch.arange(n, device=dev) + 0.5) / n
    got = torch.bincount(q.quarot_sample(x.expand(n, 6).contiguous(), u).long(), minlength=6)
    p = torch.softmax(x.double(), 0)
    assert ((got - n * p).abs() <= 1.0).all()


def test_graph_and_stream(dev):
    import torch
    import paper_2404_00456_amd as q
    rng = np.random.default_rng(6)
    rows, V = 5, 9001
    x = torch.zeros((rows, V), dtype=torch.float16, device=dev)
    u, t, p = (torch.zeros(rows, device=dev) for _ in range(3))
    k = torch.zeros(rows, dtype=torch.int32, device=dev)
    out = torch.zeros(rows, dtype=torch.int32, device=dev)
    g = torch.cuda.CUDAGraph()
    q.quarot_sample(x, u, t, k, p, tokens=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        q.quarot_sample(x, u, t, k, p, tokens=out)
    s = torch.cuda.Stream()
    for _ in range(4):
        a = likely(rng, rows, V, 2.0)
        v = dict(temperature=rng.choice([0.0, 0.7, 1.0], rows).astype(np.float32),
                 top_k=rng.integers(0, 50, rows).astype(np.int32),
                 top_p=rng.choice([0.6, 1.0], rows).astype(np.float32))
        uu = rng.random(rows).astype(np.float32)
        for d, h in ((x, a), (u, uu), (t, v["temperature"]), (k, v["top_k"]), (p, v["top_p"])):
            d.copy_(D_(h, dev))
        out.fill_(-5)
        g.replay()
        torch.cuda.synchronize()
        ref = sample(a, uu, **v)
        assert np.array_equal(out.cpu().numpy(), ref)
        got = q.quarot_sample(x, u, t, k, p, stream=s)
        s.synchronize()
        assert np.array_equal(got.cpu().numpy(), ref)
