"""Paged attention: the average error of each sequence's queries of a head, relative to
the outputs' size (limits and what they find: paged_cases, test_paged_limits)."""
import numpy as np
import pytest

from paged_cases import FOUR_ROUNDINGS, ONE_ROUNDING, Batch, few_rows, relative_rms
from test_gpu_paged import D_, SHAPES, attend, dev  # noqa: F401

pytestmark = pytest.mark.gpu

MORE = [
    # long caches, many sequences, batches of long and short ones
    ([1], [9001], 1, 1, 128, 128, 64), ([1], [9001], 16, 2, 64, 64, 64), ([1], [4100], 8, 2, 256, 256, 64),
    ([3], [6001], 5, 1, 128, 64, 64), ([90], [5000], 4, 1, 128, 128, 64), ([1] * 40, [97] * 40, 8, 2, 128, 128, 16),
    ([1, 40, 2, 16, 17, 0, 3], [900, 40, 333, 700, 17, 5, 64], 16, 2, 128, 128, 64),
    ([4] * 6, [500, 4, 64, 333, 1000, 77], 16, 2, 128, 128, 16), ([1, 1], [700, 90], 24, 1, 128, 128, 16),
    ([2, 3], [700, 90], 8, 2, 128, 32, 16), ([1, 2], [900, 33], 8, 2, 256, 64, 32),
]


def check(dev, orc, bt, H, **kw):
    qh = bt.queries(H)
    got = attend(dev, bt, qh, **kw)
    ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, bt.G, kw.get("window", 0),
                              kw.get("n_sinks", 0))
    limit = ONE_ROUNDING if few_rows(bt, H) else FOUR_ROUNDINGS
    found = relative_rms(bt, got, ref)
    print(f"average error {found:.3g}, limit {limit:.3g}", flush=True)
    assert found <= limit


@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("new,total,H,hkv,D,G,page", SHAPES + MORE)
def test_average_error(dev, orc, new, total, H, hkv, D, G, page, exact):
    bt = Batch(3 * len(new) + D + page, new, total, hkv, D, G, page, behind=1, exact=exact)
    check(dev, orc, bt, H)
    check(dev, orc, bt, H, window=70, n_sinks=5)
    check(dev, orc, bt, H, max_seq_len=1 << 16)
    check(dev, orc, bt, H, max_seq_len=1)


def test_average_error_of_dense_caches(dev, orc):
    """Caches that quarot_kv_quant filled, [batch, heads, s_max, ..], as one page per
    sequence; and the dense decode attention of the same."""
    import torch
    import paper_2404_00456_amd as q
    B, H, hkv, S, D = 3, 8, 2, 96, 128
    torch.manual_seed(0)
    pools = [q.quarot_kv_quant(torch.randn(B, hkv, S, D, device=dev).half()) for _ in range(2)]
    x = torch.randn(B, H, D, device=dev).half()
    bt = Batch(0, [1] * B, [77] * B, hkv, D, D, S)
    bt.table[:] = np.arange(B)[:, None]
    ref = orc.paged_attention(x.cpu().numpy(), *[tuple(t.cpu().numpy() for t in p) for p in pools],
                              bt.table, bt.lens, bt.cu)
    paged = q.quarot_kv_paged_attention(x, *pools, *[D_(a, dev) for a in (bt.table, bt.lens, bt.cu)])
    dense = q.quarot_kv_decode_attention(x.view(B * H, D), *[tuple(t.view(B * hkv, S, -1) for t in p)
                                                            for p in pools], 77).view(B, H, D)
    for got in (paged, dense):
        assert relative_rms(bt, got.cpu().numpy(), ref) <= ONE_ROUNDING
