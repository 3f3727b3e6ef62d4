"""Weights that are small beside one large weight: thousands of tokens behind one
that takes nearly all of the softmax, unsplit, so that one reference has to do."""
import numpy as np
import pytest

from paged_cases import Batch
from test_gpu_paged import attend, dev  # noqa: F401

pytestmark = pytest.mark.gpu


def one_large(seed, n, new, H, hkv, D, G, bits, spread):
    """A sequence of n tokens whose first one has a score `bits` log2 units above
    the others (give or take a tenth for each query, and `spread` for each token) and
    a value of 0; all of its values are 0 or more."""
    bt = Batch(seed, [new], [n], hkv, D, G, 64)
    rng = bt.rng
    qh = np.broadcast_to(rng.uniform(0.9, 1.1, (bt.T, H, 1)), (bt.T, H, D)).astype(np.float16)
    score = np.zeros(n)
    score[1:] = rng.uniform(-spread, spread, n - 1)
    score[0] = bits
    at = bt.table[0, np.arange(n) // 64], slice(None), np.arange(n) % 64
    # keys of equal elements: the score is sqrt(D) times the element and the query's
    bt.k[1][at] = 0
    bt.k[2][at] = (score * np.log(2) / np.sqrt(D)).astype(np.float16)[:, None, None]
    first = bt.table[0, 0], slice(None), 0
    return bt, qh, at, first


def weights(bt, qh, n):
    """Softmax numerators [T, H, n] (the largest is 1) in binary64, masked causally."""
    z = bt.k[2][bt.table[0, np.arange(n) // 64], 0, np.arange(n) % 64, 0].astype(np.float64)
    s = qh[..., :1].astype(np.float64) * z * np.sqrt(bt.D)
    p = np.arange(n - bt.T, n)[:, None, None]
    s = np.where(np.arange(n) <= p, s, -np.inf)
    return np.exp(s - s.max(-1, keepdims=True))


def binary32(n, bits):
    """Relative error of the sums over n tokens: adds of 32 at a time and a wave's
    end, and of the weights (paged_cases: S = scores in nats)."""
    return (n / 32 + 16) * 2.0 ** -24 + (bits * np.log(2) * 1.1 + 2) * 2.0 ** -18


@pytest.mark.parametrize("bits", [20, 16])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_two_part_weights(dev, orc, D, bits):
    """Few rows, one group a row: weights times scales are two fp16 parts, the second
    rounded to nearest: off by 2^-21 of themselves (the first part leaves 2^-10, the
    second half a step of that), or by half of fp16's smallest number, 2^-25, where that
    is more: the largest starts at 2^8 or more, of which it is 2^-33."""
    n, H = 8000, 4
    bt, qh, at, first = one_large(D + bits, n, 1, H, 1, D, D, bits, 0.5)
    c, s, z = bt.v
    s[first], z[first], c[first] = 0.5, 0.0, 0  # (nothing of it in any sum)
    got = attend(dev, bt, qh, max_seq_len=1)
    ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, D)
    w = weights(bt, qh, n)
    most = (15 * s[at] + np.abs(z[at])).astype(np.float64)[:, 0, 0]
    mass = (w * most)[..., 1:].sum(-1)[..., None]
    tol = np.abs(ref) * 2.0 ** -11 + 2.0 ** -25 + \
        mass * (2.0 ** -21 + binary32(n, bits)) + n * 15 * 2.0 ** -33
    assert (np.abs(got - ref) / tol).max() <= 1


@pytest.mark.parametrize("bits", [19, 16])
@pytest.mark.parametrize("new,H,hkv,D,G", [
    (2, 8, 1, 128, 32), (4, 4, 1, 64, 32), (3, 4, 1, 256, 64),                    # few rows, groups
    (40, 1, 1, 128, 128), (30, 4, 1, 128, 64), (64, 8, 2, 128, 128),              # tiles
    (50, 1, 1, 64, 64), (100, 4, 1, 64, 32), (60, 2, 1, 256, 256), (70, 1, 1, 256, 128)])
def test_one_part_weights(dev, orc, new, H, hkv, D, G, bits):
    """Weights rounded to fp16 are off by half a step, 2^-11 of themselves, or by half of
    fp16's smallest number, 2^-25, where that is more: the largest starts at 2^6 or more,
    of which it is 2^-31."""
    n = 6000
    bt, qh, at, first = one_large(new + D + bits, n, new, H, hkv, D, G, bits, 0.0)
    c, s, z = bt.v
    z[at], c[first], s[at] = 0, 0, 0.5
    got = attend(dev, bt, qh, max_seq_len=1)
    ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, G)
    # all values are 0 or more, so the sums are the outputs
    tol = np.abs(ref) * (2 * 2.0 ** -11 + binary32(n, bits)) + 2.0 ** -25 + n * 7.5 * 2.0 ** -31
    assert (np.abs(got - ref) / tol).max() <= 1
