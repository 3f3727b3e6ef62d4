"""What the average error's limits (paged_cases) find, with mistakes planted in the
oracle: none of these passes."""
import numpy as np
import pytest

from paged_cases import FOUR_ROUNDINGS, ONE_ROUNDING, Batch, few_rows, relative_rms

CASES = [([300], [700], 12, 4, 128, 64, 128), ([1, 1, 1], [500, 17, 333], 16, 2, 128, 128, 64),
         ([1], [9001], 1, 1, 128, 128, 64), ([3, 70, 1], [450, 70, 2], 8, 2, 128, 128, 32)]


def run(orc, bt, qh, k=None, v=None, table=None, lens=None):
    return orc.paged_attention(qh, k or bt.k, v or bt.v, bt.table if table is None else table,
                               bt.lens if lens is None else lens, bt.cu, bt.G)


@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("new,total,H,hkv,D,G,page", CASES)
def test_mistakes_are_found(orc, new, total, H, hkv, D, G, page, exact):
    bt = Batch(len(new) * D + page, new, total, hkv, D, G, page, exact=exact, nan=False)
    qh = bt.queries(H)
    ref = run(orc, bt, qh)
    limit = ONE_ROUNDING if few_rows(bt, H) else FOUR_ROUNDINGS
    assert relative_rms(bt, ref.astype(np.float16), ref) < ONE_ROUNDING  # the output's rounding

    def times(pool, f):
        return pool[0], (pool[1] * np.float16(f)).astype(np.float16), (pool[2] * np.float16(f)).astype(np.float16)

    table = bt.table.copy()
    b = int(np.argmax(bt.total))
    table[b, (bt.total[b] - 1) // page // 2] = -1  # a page in the middle
    for name, wrong in (("values", run(orc, bt, qh, v=times(bt.v, 1.01))),
                        ("keys", run(orc, bt, qh, k=times(bt.k, 1.01))),
                        ("page", run(orc, bt, qh, table=table)),
                        ("zero", run(orc, bt, qh, v=(bt.v[0], bt.v[1], bt.v[2] * np.float16(1.01)))),
                        ("scale", orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, bt.G,
                                                      sm_scale=1.01 * D ** -0.5))):
        found = relative_rms(bt, wrong, ref)
        assert found > 2 * limit, (name, found)


def test_missing_newest_tokens_are_found(orc):
    """Dense caches as pools: the 13 newest of 77 tokens left out."""
    bt = Batch(5, [1, 1, 1], [77, 77, 77], 2, 128, 128, 96, exact=False, nan=False)
    qh = bt.queries(8)
    assert few_rows(bt, 8)
    ref = run(orc, bt, qh)
    assert relative_rms(bt, run(orc, bt, qh, lens=bt.lens - 13), ref) > 2 * ONE_ROUNDING
