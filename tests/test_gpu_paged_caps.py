"""Caps at the ends of what is accepted, beside scales of the scores that are large or small."""
import numpy as np
import pytest

from paged_cases import Batch
from paged_plain import scored_attention, scored_tolerance
from test_gpu_paged_scored import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2404_00456_amd as q
    q.lib()
    return torch.device("cuda:0")


@pytest.mark.parametrize("cap,sm_scale", [(2.0 ** -64, 2.0 ** 100), (2.0 ** -64, 2.0 ** 63), (2.0 ** -64, 2.0 ** -100),
                                          (2.0 ** -30, 1.0), (2.0 ** 64, 2.0 ** -100), (2.0 ** 64, 0.01)])
@pytest.mark.parametrize("new,total,D,G", [([2, 1], [90, 300], 128, 128), ([3], [200], 64, 32), ([40], [130], 128, 64),
                                           ([33, 50], [33, 500], 64, 64), ([40], [100], 256, 256)])
def test_queries_of_zeros_see_all_alike(dev, new, total, D, G, cap, sm_scale):
    """Scores of 0 stay 0 under any cap, beside others at its ends."""
    bt = Batch(41, new, total, 1, D, G, 16)
    qh = bt.queries(4)
    qh[::2] = 0
    qh[:, 1] = 0
    got = run(dev, bt, qh, G, cap=cap, sm_scale=sm_scale)
    ref = scored_attention(bt, qh, cap=cap, sm_scale=sm_scale)
    zero = ~qh.any(-1)
    tol = scored_tolerance(bt, np.zeros_like(qh), True, cap)
    assert np.isfinite(got.astype(np.float64)).all()
    assert np.abs(got[zero].astype(np.float64) - ref[zero]).max() <= tol
    if cap < 1:  # capped scores are 0 as well, as far as weights can tell
        assert np.abs(got.astype(np.float64) - ref).max() <= tol
