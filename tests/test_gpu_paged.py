"""Rotary positions, the paged append and the paged attention on the GPU against
the CPU oracle: rotary results, codes, scales and zeros bit for bit, attention
within tolerances that count the roundings (paged_cases)."""
import numpy as np
import pytest

from paged_cases import Batch, attention_tolerance

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
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev)


def bits(a):
    return np.ascontiguousarray(a).view(np.uint16)


def freq(rot, base=10000.0):
    return (base ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)


def sections_of(half, axes):
    cut = [half // axes] * axes
    cut[0] += half - sum(cut)
    return cut


def axis_of(sections):
    return np.repeat(np.arange(len(sections)), sections).astype(np.uint8)


# ---------------------------------------------------------------- rotary ----

@pytest.mark.parametrize("T,H,D,rot,axes,inter,rotate", [
    (1, 1, 64, 64, 1, False, False),
    (1, 64, 128, 128, 1, False, True),
    (5, 3, 128, 32, 2, False, True),
    (33, 7, 128, 128, 3, True, True),
    (300, 2, 256, 256, 4, False, True),
    (17, 5, 256, 64, 3, True, False),
    (9, 40, 64, 16, 1, False, True),
    (2100, 9, 128, 96, 3, False, True),
    (40, 1, 64, 48, 2, True, True),
])
def test_rope_matches_oracle(dev, orc, T, H, D, rot, axes, inter, rotate):
    import torch
    import paper_2404_00456_amd as q
    rng = np.random.default_rng(T * 1000 + D + rot)
    x = (rng.standard_normal((T, H + 2, D)) * 3).astype(np.float16)
    pos = rng.integers(-2 ** 31, 2 ** 31, (axes, T)).astype(np.int32)
    pos[:, :1] = 2 ** 31 - 1
    pos[:, T // 2:] = rng.integers(0, 5000, (axes, T - T // 2))
    sec = sections_of(rot // 2, axes)
    wide = D_(x, dev)
    part = wide[:, 1:1 + H]  # the heads in the middle of a wider tensor
    y = q.quarot_rope(part, D_(pos, dev), D_(freq(rot), dev), sections=sec, interleaved=inter,
                      rotate=rotate)
    ref = orc.rope(x[:, 1:1 + H], pos, freq(rot), axis_of(sec), inter)
    ref = orc.f32_to_f16(orc.rotate_rows(ref) if rotate else ref)
    assert np.array_equal(bits(y.cpu().numpy()), bits(ref))
    # in place, and the heads beside it untouched
    assert q.quarot_rope(part, D_(pos, dev), D_(freq(rot), dev), sections=bytes(axis_of(sec)),
                         interleaved=inter, rotate=rotate, y=part) is part
    x[:, 1:1 + H] = ref
    assert np.array_equal(bits(wide.cpu().numpy()), bits(x))


def test_rope_axes_in_any_order(dev, orc):
    import paper_2404_00456_amd as q
    rng = np.random.default_rng(4)
    x = rng.standard_normal((11, 4, 128)).astype(np.float16)
    pos = rng.integers(0, 1 << 20, (4, 11)).astype(np.int32)
    axis = rng.integers(0, 4, 64).astype(np.uint8)
    y = q.quarot_rope(D_(x, dev), D_(pos, dev), D_(freq(128), dev), sections=bytes(axis))
    assert np.array_equal(bits(y.cpu().numpy()),
                          bits(orc.f32_to_f16(orc.rope(x, pos, freq(128), axis))))


# ---------------------------------------------------------------- append ----

APPEND = [
    # new, total, H, hkv, D, G, page, rot, axes, rotate_k, rotate_v
    ([1], [1], 4, 4, 128, 128, 16, 128, 1, True, False),
    ([1, 1, 1], [7, 64, 65], 8, 1, 128, 128, 64, 128, 1, True, False),
    ([3, 0, 70, 1], [3, 0, 90, 17], 16, 4, 128, 32, 16, 64, 3, True, True),
    ([33, 2], [40, 100], 5, 5, 64, 64, 48, 64, 2, False, True),
    ([5, 9], [300, 9], 2, 1, 256, 256, 32, 256, 1, True, False),
    ([5, 9], [30, 9], 0, 3, 256, 64, 128, 32, 4, True, True),
    ([2500], [2611], 3, 2, 64, 32, 16, 16, 1, True, False),
]


@pytest.mark.parametrize("new,total,H,hkv,D,G,page,rot,axes,rot_k,rot_v", APPEND)
def test_append_matches_oracle(dev, orc, new, total, H, hkv, D, G, page, rot, axes, rot_k, rot_v):
    import torch
    import paper_2404_00456_amd as q
    bt = Batch(1, new, total, hkv, D, G, page, behind=3)
    x = (bt.rng.standard_normal((bt.T, H + 2 * hkv, D)) * 2).astype(np.float16)
    x[0, H] = 0  # a key of zeros: scale 0
    pos = bt.rng.integers(0, 1 << 18, (axes, bt.T)).astype(np.int32)
    sec = sections_of(rot // 2, axes)
    fr = freq(rot)
    wide = D_(x, dev)
    kp, vp = (tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v))
    qo = torch.full((bt.T, H, D), 7.0, dtype=torch.float16, device=dev) if H else None
    got = q.quarot_kv_append_paged(
        wide[:, H:H + hkv], wide[:, H + hkv:], kp, vp, D_(bt.table, dev), D_(bt.lens, dev),
        D_(bt.cu, dev), group=G, q=wide[:, :H] if H else None, positions=D_(pos, dev),
        inv_freq=D_(fr, dev), sections=sec, rotate_k=rot_k, rotate_v=rot_v, clip_ratio=0.95,
        q_out=qo)
    assert got is qo

    def ready(part, turn, rotate):
        y = orc.rope(part, pos, fr, axis_of(sec)) if turn else part.astype(np.float32)
        return orc.rotate_rows(y) if rotate else y

    rk = orc.kv_append_paged(ready(x[:, H:H + hkv], True, rot_k), bt.k, bt.table, bt.lens, bt.cu, G)
    rv = orc.kv_append_paged(ready(x[:, H + hkv:], False, rot_v), bt.v, bt.table, bt.lens, bt.cu, G)
    for pool, ref in ((kp, rk), (vp, rv)):  # whole pools: nothing else was written
        assert np.array_equal(pool[0].cpu().numpy(), ref[0])
        assert np.array_equal(bits(pool[1].cpu().numpy()), bits(ref[1]))
        assert np.array_equal(bits(pool[2].cpu().numpy()), bits(ref[2]))
    if H:
        ref = np.full((bt.T, H, D), 7.0, np.float16)
        ref[:bt.cu[-1]] = orc.f32_to_f16(ready(x[:, :H], True, rot_k))[:bt.cu[-1]]
        assert np.array_equal(bits(qo.cpu().numpy()), bits(ref))


def test_append_positions_of_the_cache_and_no_rotary(dev, orc):
    """positions None takes each token's position in its sequence; without
    inv_freq nothing turns."""
    import paper_2404_00456_amd as q
    bt = Batch(2, [4, 1, 7], [20, 55, 7], 2, 128, 128, 16)
    x = bt.rng.standard_normal((bt.T, 2, 128)).astype(np.float16)
    at = np.array([t for _, _, t, _, _ in orc.paged_place(bt.table, bt.pages, 16, bt.lens, bt.cu)],
                  np.int32)
    for fr in (freq(128), None):
        kp, vp = (tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v))
        args = (D_(x, dev), D_(x, dev), kp, vp, D_(bt.table, dev), D_(bt.lens, dev), D_(bt.cu, dev))
        assert q.quarot_kv_append_paged(*args, inv_freq=None if fr is None else D_(fr, dev)) is None
        y = orc.rope(x, at, fr) if fr is not None else x.astype(np.float32)
        rk = orc.kv_append_paged(orc.rotate_rows(y), bt.k, bt.table, bt.lens, bt.cu)
        rv = orc.kv_append_paged(x.astype(np.float32), bt.v, bt.table, bt.lens, bt.cu)
        for pool, ref in ((kp, rk), (vp, rv)):
            assert np.array_equal(pool[0].cpu().numpy(), ref[0])
            assert np.array_equal(bits(pool[1].cpu().numpy()), bits(ref[1]))
            assert np.array_equal(bits(pool[2].cpu().numpy()), bits(ref[2]))


def test_append_leaves_what_has_no_page(dev, orc):
    """Pages outside the pool, positions past the table and before 0: not
    stored, nothing else touched; the queries are still made ready."""
    import torch
    import paper_2404_00456_amd as q
    bt = Batch(3, [20, 6, 5], [40, 6, 33], 2, 64, 64, 16)
    bt.table[0, 1] = -5               # positions 16 .. 31 of sequence 0
    bt.table[0, 2] = bt.pages         # and 32 ..
    bt.lens[1] = 4                    # two tokens before position 0
    bt.lens[2] = bt.table.shape[1] * 16 + 2  # two tokens past the table
    x = bt.rng.standard_normal((bt.T, 2, 64)).astype(np.float16)
    kp, vp = (tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v))
    qo = q.quarot_kv_append_paged(D_(x, dev), D_(x, dev), kp, vp, D_(bt.table, dev),
                                  D_(bt.lens, dev), D_(bt.cu, dev), group=64, q=D_(x, dev),
                                  rotate_k=False)
    rk = orc.kv_append_paged(x.astype(np.float32), bt.k, bt.table, bt.lens, bt.cu, 64)
    for a, b in zip(kp, rk):
        assert np.array_equal(a.cpu().numpy().view(np.uint8), b.view(np.uint8))
    assert np.array_equal(bits(qo.cpu().numpy()), bits(x))


# ------------------------------------------------------------- attention ----

def attend(dev, bt, qh, **kw):
    import torch
    import paper_2404_00456_amd as q
    out = torch.full(qh.shape, 9.0, dtype=torch.float16, device=dev)
    q.quarot_kv_paged_attention(D_(qh, dev), tuple(D_(a, dev) for a in bt.k),
                                tuple(D_(a, dev) for a in bt.v), D_(bt.table, dev),
                                D_(bt.lens, dev), D_(bt.cu, dev), group=bt.G, out=out, **kw)
    return out.cpu().numpy()


def check(dev, orc, bt, H, window=0, sinks=0, exact=True, sigma=1.0, **kw):
    qh = bt.queries(H, sigma)
    got = attend(dev, bt, qh, window=window, n_sinks=sinks, **kw)
    ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu, bt.G, window, sinks,
                              out=np.full(qh.shape, 9.0))
    assert np.isfinite(got).all()
    assert (got[bt.cu[-1]:] == 9.0).all()  # rows of no sequence
    err, tol = np.abs(got - ref).max(initial=0), attention_tolerance(bt, qh, exact)
    print(f"max error {err:.3g}, tolerance {tol:.3g}", flush=True)
    assert err <= tol


SHAPES = [
    # new, total, H, hkv, D, G, page
    ([1], [1], 1, 1, 128, 128, 16),
    ([1], [2], 8, 1, 128, 128, 16),
    ([1, 1, 1, 1], [1, 63, 64, 65], 8, 2, 128, 128, 16),
    ([1, 1, 1], [500, 17, 333], 16, 2, 128, 128, 64),
    ([1, 1], [129, 300], 7, 7, 128, 128, 48),
    ([1, 1], [129, 300], 10, 2, 64, 64, 32),
    ([1, 1], [129, 300], 6, 2, 256, 256, 16),
    ([1, 1, 1], [40, 77, 130], 20, 1, 128, 32, 16),
    ([1, 1, 1], [40, 77, 130], 17, 1, 128, 64, 16),
    ([2, 4, 3], [70, 4, 200], 8, 2, 128, 128, 16),
    ([2, 4, 3], [70, 4, 200], 8, 2, 64, 32, 16),
    ([3, 5], [70, 100], 4, 1, 256, 64, 32),
    ([0, 0, 3, 0], [5, 0, 9, 2], 4, 2, 128, 128, 16),
    ([64], [64], 1, 1, 128, 128, 64),
    ([65], [65], 1, 1, 128, 128, 16),
    ([33], [97], 5, 1, 128, 128, 48),
    ([100, 1, 37], [100, 250, 90], 8, 2, 128, 128, 32),
    ([129, 250], [400, 250], 4, 4, 128, 128, 16),
    ([257, 3], [300, 300], 6, 2, 64, 64, 16),
    ([130, 20], [131, 333], 3, 1, 256, 32, 16),
    ([300], [700], 12, 4, 128, 64, 128),
]


@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("new,total,H,hkv,D,G,page", SHAPES)
def test_attention_matches_oracle(dev, orc, new, total, H, hkv, D, G, page, exact):
    check(dev, orc, Batch(len(new) * D + page, new, total, hkv, D, G, page, behind=2, exact=exact), H,
          exact=exact)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (63, 0), (64, 64), (65, 1),
                                          (200, 17), (5000, 3), (2 ** 40, 2 ** 40)])
@pytest.mark.parametrize("new,total,H,hkv,D,G,page", [
    ([1, 1, 1], [500, 17, 333], 8, 2, 128, 128, 16),
    ([3, 70, 1], [450, 70, 2], 8, 2, 128, 128, 32),
    ([140], [600], 2, 1, 64, 32, 16),
    ([20, 33], [300, 200], 4, 1, 256, 256, 16),
    ([300], [900], 8, 8, 128, 128, 64),
])
def test_window_and_sinks(dev, orc, new, total, H, hkv, D, G, page, window, sinks):
    check(dev, orc, Batch(window % 97 + D, new, total, hkv, D, G, page, behind=1), H, window, sinks)


@pytest.mark.parametrize("new,total,H,hkv,D,G", [
    ([1], [9001], 8, 1, 128, 128),
    ([1], [9001], 1, 1, 128, 128),
    ([1, 1], [5000, 3], 16, 2, 64, 64),
    ([1], [4100], 8, 2, 256, 256),
    ([3], [6001], 5, 1, 128, 64),
    ([90], [5000], 4, 1, 128, 128),
    ([1, 300], [3000, 2500], 2, 2, 128, 128),
])
def test_long_sequences_are_split(dev, orc, new, total, H, hkv, D, G):
    """Few rows over long caches: the split of the tokens and its joining; the
    plan of a much longer table is right as well."""
    import paper_2404_00456_amd as q
    bt = Batch(7, new, total, hkv, D, G, 64)
    assert q.quarot_kv_paged_attention_workspace_size(bt.T, len(new), H, hkv, D, max(total)) > 0
    check(dev, orc, bt, H, max_seq_len=max(total))
    check(dev, orc, bt, H, max_seq_len=1 << 20)
    check(dev, orc, bt, H, max_seq_len=1)


@pytest.mark.parametrize("D,G,H,hkv,page", [(64, 64, 8, 8, 16), (128, 128, 16, 2, 64),
                                            (128, 128, 5, 5, 48), (256, 256, 16, 1, 32)])
@pytest.mark.parametrize("new", [[1, 40, 2, 16, 17, 0, 3], [64, 1, 1], [1, 1, 1, 1, 300],
                                 [1] * 70 + [90] + [2] * 70, [0, 0, 33, 0, 0], [1] * 130 + [500]])
def test_mixed_batches(dev, orc, D, G, H, hkv, page, new):
    """Long and short sequences of a batch go through kernels of their own."""
    total = [n + (37 * i) % 90 + (3 * (len(new) < 10) << (i % 9)) for i, n in enumerate(new)]
    bt = Batch(11, new, total, hkv, D, G, page)
    check(dev, orc, bt, H)
    check(dev, orc, bt, H, window=50, sinks=5)
    if len(new) < 10:  # both of their sums over splits
        check(dev, orc, bt, H, max_seq_len=30000)


@pytest.mark.parametrize("D,G", [(64, 32), (128, 32), (128, 64), (256, 32), (256, 64), (256, 128)])
@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("new,total,page", [([1, 1, 1, 1], [1, 33, 700, 128], 16),
                                            ([2, 1, 0, 4], [65, 1, 9, 515], 48),
                                            ([1] * 9 + [9], [40 * i + 1 for i in range(9)] + [333], 64)])
def test_few_rows_in_groups(dev, orc, D, G, exact, new, total, page):
    """Few rows whose cached rows are several groups, with and without a window,
    whole and in splits."""
    bt = Batch(70 + D, new, total, 2, D, G, page, behind=1, exact=exact)
    check(dev, orc, bt, 8, exact=exact)
    check(dev, orc, bt, 2, window=70, sinks=3, exact=exact)
    check(dev, orc, bt, 8, max_seq_len=1 << 16, exact=exact)
    for pool in (bt.k, bt.v):  # groups of equal values
        pool[1][..., ::2][np.broadcast_to(bt.held[:, None, :, None], pool[1][..., ::2].shape)] = 0
    check(dev, orc, bt, 8, exact=exact)


@pytest.mark.parametrize("D,G", [(128, 128), (64, 32)])
@pytest.mark.parametrize("new,first", [([1, 1, 40], 2), ([20, 1, 1], 33), ([1, 1, 1, 1], 100),
                                       ([300], 19)])
def test_rows_before_the_first_sequence(dev, orc, D, G, new, first):
    """cu_new need not begin at 0: rows in front belong to nobody as well."""
    import torch
    import paper_2404_00456_amd as q
    bt = Batch(90, new, [n + 70 for n in new], 2, D, G, 16, behind=first + 1)
    bt.cu += first
    check(dev, orc, bt, 4)
    check(dev, orc, bt, 16, max_seq_len=1 << 15)
    k, v = (torch.randn(bt.T, 2, D, device=dev).half() for _ in range(2))
    x = torch.randn(bt.T, 4, D, device=dev).half()
    pools = [tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v)]
    out = torch.full_like(x, 9.0)
    q.quarot_kv_append_paged(k, v, *pools, D_(bt.table, dev), D_(bt.lens, dev), D_(bt.cu, dev),
                             group=G, q=x, q_out=out)
    assert (out[:first] == 9.0).all() and (out[bt.cu[-1]:] == 9.0).all()
    for pool, host, rows in ((pools[0], bt.k, orc.rotate_rows(k.cpu().numpy().astype(np.float32))),
                             (pools[1], bt.v, v.cpu().numpy().astype(np.float32))):
        ref = orc.kv_append_paged(rows, host, bt.table, bt.lens, bt.cu, G)
        for a, b in zip(pool, ref):
            assert np.array_equal(a.cpu().numpy().view(np.uint8), b.view(np.uint8))


def test_large_scores(dev, orc):
    """Queries whose scores reach hundreds: one token takes all the weight."""
    check(dev, orc, Batch(9, [1, 40], [300, 300], 2, 128, 128, 16), 8, sigma=60.0)


def test_pages_that_do_not_exist(dev, orc):
    """Entries outside the pool hide their tokens; where they hide everything the
    output is zero.  A sequence longer than its table sees what the table has."""
    bt = Batch(11, [1, 2, 80, 1, 5], [100, 64, 200, 48, 48], 2, 128, 128, 16, behind=1)
    bt.table[0, 2], bt.table[0, 5] = -1, bt.pages + 3
    bt.table[1, :] = -1
    bt.table[2, 0], bt.table[2, 7] = 2 ** 30, -2 ** 31
    bt.lens[3] = 10 ** 6
    bt.lens[4] = 3  # two queries before position 0
    qh = bt.queries(8)
    got = attend(dev, bt, qh)
    ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, np.where(bt.lens > 10 ** 5, 208, bt.lens),
                              bt.cu, 128, out=np.full(qh.shape, 9.0))
    assert (got[1:3] == 0).all() and (got[84:86] == 0).all()
    err, tol = np.abs(got - ref).max(), attention_tolerance(bt, qh, True)
    assert err <= tol


def test_bad_batch_stays_in_its_buffers(dev):
    """Contents of cu_new and seq_lens that break the rules give no results
    worth having, but nothing outside the rows of the batch is written."""
    import torch
    import paper_2404_00456_amd as q
    bt = Batch(12, [4, 4, 4], [50, 50, 50], 2, 128, 128, 16, nan=False)
    buf = torch.full((bt.T + 64, 8, 128), 5.0, dtype=torch.float16, device=dev)
    kp, vp = (tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v))
    x = D_(bt.queries(8), dev)
    for cu in ([0, 4, 8, 500], [-7, 4, 8, 12], [12, 8, 4, 0], [0, 2 ** 31 - 1, 3, 12]):
        for lens in ([50, 2 ** 31 - 1, 50], [-2 ** 31, -1, 0]):
            c, ln = D_(np.array(cu, np.int32), dev), D_(np.array(lens, np.int32), dev)
            q.quarot_kv_append_paged(x[:, :2], x[:, 2:4], kp, vp, D_(bt.table, dev), ln, c, q=x,
                                     q_out=buf[:bt.T])
            q.quarot_kv_paged_attention(x, kp, vp, D_(bt.table, dev), ln, c, out=buf[:bt.T])
            torch.cuda.synchronize()
    assert (buf[bt.T:] == 5.0).all()


def test_dense_caches_are_pools(dev, orc):
    """Caches that quarot_kv_append filled, [batch, heads, s_max, ..], are read as
    one page per sequence, with the result of quarot_kv_decode_attention."""
    import torch
    import paper_2404_00456_amd as q
    B, H, hkv, S, D = 3, 8, 2, 96, 128
    torch.manual_seed(0)
    pools = []
    for _ in range(2):
        pools.append(q.quarot_kv_quant(torch.randn(B, hkv, S, D, device=dev).half()))
    x = torch.randn(B, H, D, device=dev).half()
    table = torch.arange(B, dtype=torch.int32, device=dev)[:, None].contiguous()
    cu = torch.arange(B + 1, dtype=torch.int32, device=dev)
    lens = torch.full((B,), 77, dtype=torch.int32, device=dev)
    got = q.quarot_kv_paged_attention(x, *pools, table, lens, cu)
    ref = q.quarot_kv_decode_attention(x.view(B * H, D), *[tuple(t.view(B * hkv, S, -1) for t in p)
                                                          for p in pools], 77)
    ref = ref.view(B, H, D)
    vmax = q.quarot_kv_dequant(*pools[1]).abs().max().item()
    # both are within the tolerance of paged_cases of the exact value (scores
    # below 2 sqrt(128) |q| |k| / .. <= 60 here)
    assert (got.float() - ref.float()).abs().max().item() <= 2 * vmax * (2 * 60 + 3) * 2.0 ** -11


def test_a_server_run(dev, orc):
    """Prompts in chunks, then single tokens, through both calls from a captured
    graph that is replayed for other lengths: every step against the oracle."""
    import torch
    import paper_2404_00456_amd as q
    H, hkv, D, page, cap = 8, 2, 128, 16, 24
    rng = np.random.default_rng(5)
    pages, P = 64, 12
    pools = [tuple(t.to(dev) for t in (torch.zeros(pages, hkv, page, D // 2, dtype=torch.uint8),
                                       torch.full((pages, hkv, page, 1), float("nan")).half(),
                                       torch.zeros(pages, hkv, page, 1).half())) for _ in range(2)]
    host = [tuple(t.cpu().numpy().copy() for t in p) for p in pools]
    table = rng.permutation(pages)[:3 * P].reshape(3, P).astype(np.int32)
    fr = freq(D)
    st = dict(x=torch.zeros(cap, H + 2 * hkv, D, dtype=torch.float16, device=dev),
              cu=torch.zeros(4, dtype=torch.int32, device=dev),
              lens=torch.zeros(3, dtype=torch.int32, device=dev), table=D_(table, dev),
              fr=D_(fr, dev),
              ready=torch.zeros(cap, H, D, dtype=torch.float16, device=dev),
              out=torch.zeros(cap, H, D, dtype=torch.float16, device=dev))
    need = q.quarot_kv_paged_attention_workspace_size(cap, 3, H, hkv, D, P * page, 40, 4)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)

    def step():
        x = st["x"]
        q.quarot_kv_append_paged(x[:, H:H + hkv], x[:, H + hkv:], *pools, st["table"], st["lens"],
                                 st["cu"], q=x[:, :H], inv_freq=st["fr"], q_out=st["ready"])
        q.quarot_kv_paged_attention(st["ready"], *pools, st["table"], st["lens"], st["cu"],
                                    window=40, n_sinks=4, out=st["out"], workspace=ws)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()  # an empty batch: nothing happens
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    lens = np.zeros(3, np.int64)
    for new in ([20, 4, 0], [10, 10, 3], [1, 1, 1], [1, 0, 1], [1, 1, 20], [1, 1, 1], [0, 24, 0],
                [1, 1, 1]):
        cu = np.cumsum([0] + new).astype(np.int32)
        lens += new
        x = rng.standard_normal((cap, H + 2 * hkv, D)).astype(np.float16)
        st["x"].copy_(D_(x, dev))
        st["cu"].copy_(D_(cu, dev))
        st["lens"].copy_(D_(lens.astype(np.int32), dev))
        st["out"].fill_(3.0)
        (st["x"].float() @ st["x"].float().transpose(1, 2)).sum().item()  # other work between
        graph.replay()
        torch.cuda.synchronize()
        at = np.zeros(cap, np.int32)
        for r, _, t, _, _ in orc.paged_place(table, pages, page, lens, cu):
            at[r] = t
        turned = orc.rope(x[:, :H + hkv], at, fr)
        turned = orc.rotate_rows(turned)
        host[0] = orc.kv_append_paged(turned[:, H:], host[0], table, lens, cu)
        host[1] = orc.kv_append_paged(x[:, H + hkv:].astype(np.float32), host[1], table, lens, cu)
        for pool, ref in zip(pools, host):
            for a, b in zip(pool, ref):
                assert np.array_equal(a.cpu().numpy().view(np.uint8), b.view(np.uint8))
        qh = orc.f32_to_f16(turned[:, :H])
        ref = orc.paged_attention(qh, host[0], host[1], table, lens, cu, 128, 40, 4,
                                  out=np.full((cap, H, D), 3.0))
        got = st["out"].cpu().numpy()
        # paged_cases' tolerance with V = 5, S = |q| |k| / sqrt(D) <= 20
        err = np.abs(got - ref).max()
        assert err <= 5 * (2 * 20 + 3.2) * 2.0 ** -11
        assert (got[cu[-1]:] == 3.0).all()


def test_two_streams_at_once(dev, orc):
    """Calls on two streams with a workspace each."""
    import torch
    import paper_2404_00456_amd as q
    runs = []
    for s in range(2):
        bt = Batch(20 + s, [1, 1], [6000 + s, 3000], 2, 128, 128, 64)
        qh = bt.queries(16)
        need = q.quarot_kv_paged_attention_workspace_size(bt.T, 2, 16, 2, 128, 6001)
        runs.append((bt, qh, torch.cuda.Stream(), torch.empty(need, dtype=torch.uint8, device=dev),
                     [D_(a, dev) for a in (qh, *bt.k, *bt.v, bt.table, bt.lens, bt.cu)], []))
    torch.cuda.synchronize()
    for _ in range(10):
        for bt, qh, stream, ws, d, outs in runs:
            with torch.cuda.stream(stream):
                outs.append(q.quarot_kv_paged_attention(d[0], d[1:4], d[4:7], *d[7:],
                                                        max_seq_len=6001, workspace=ws))
    torch.cuda.synchronize()
    for bt, qh, _, _, _, outs in runs:
        ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, bt.lens, bt.cu)
        err, tol = np.abs(outs[0].cpu().numpy() - ref).max(), attention_tolerance(bt, qh, True)
        assert err <= tol
        for o in outs[1:]:
            assert torch.equal(o, outs[0])


@pytest.mark.parametrize("new", [[1, 1, 1], [1, 30, 17]])
@pytest.mark.parametrize("D,hkv", [(128, 2), (64, 4), (256, 1)])
def test_zero_scales(dev, orc, new, D, hkv):
    """Rows of equal values have a scale of 0 and are their zero: some tokens of
    each sequence, all of the last."""
    bt = Batch(31, new, [200, 130, 77], hkv, D, D, 16)
    for pool in (bt.k, bt.v):
        for b, page in enumerate(bt.table):
            for i, pg in enumerate(page):
                if pg >= 0:
                    held = bt.held[pg] & (np.arange(16) % 3 == 0 if b < 2 else True)
                    pool[1][pg][:, held] = 0
    check(dev, orc, bt, 4 * hkv)


def test_two_graphs_share_a_workspace(dev, orc):
    """A decode step and a mixed batch, captured with the same workspace and
    replayed in turn for other lengths."""
    import torch
    import paper_2404_00456_amd as q
    H, hkv, D = 16, 2, 128
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=dev)
    stream, runs = torch.cuda.Stream(), []
    for new, total in (([1, 1, 1], [5000, 3001, 64]), ([1, 70, 0, 2], [4100, 3000, 9, 2222])):
        bt = Batch(40 + len(new), new, total, hkv, D, D, 64, behind=3)
        qh = bt.queries(H)
        assert 0 < q.quarot_kv_paged_attention_workspace_size(bt.T, len(new), H, hkv, D, 5000) <= 1 << 24
        d = [D_(a, dev) for a in (qh, *bt.k, *bt.v, bt.table, bt.lens, bt.cu)]
        out = torch.zeros(qh.shape, dtype=torch.float16, device=dev)

        def step(d=d, out=out):
            q.quarot_kv_paged_attention(d[0], d[1:4], d[4:7], *d[7:], max_seq_len=5000, out=out,
                                        workspace=ws)
        with torch.cuda.stream(stream):
            step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        runs.append((bt, qh, d, out, graph))
    for k in range(4):
        for bt, qh, d, out, graph in runs:
            lens = np.maximum(bt.lens - 37 * k, np.diff(bt.cu)).astype(np.int32)
            d[8].copy_(D_(lens, dev))
            out.fill_(9.0)
            (d[0].float() @ d[0].float().transpose(1, 2)).sum().item()  # other work between
            graph.replay()
            torch.cuda.synchronize()
            got = out.cpu().numpy()
            ref = orc.paged_attention(qh, bt.k, bt.v, bt.table, lens, bt.cu, D,
                                      out=np.full(qh.shape, 9.0))
            assert (got[bt.cu[-1]:] == 9.0).all()
            assert np.abs(got - ref).max() <= attention_tolerance(bt, qh, True)


def test_pools_past_32_bits(dev, orc):
    """Pages whose offsets pass 2^32 bytes hold and give what the same pages do at
    the front of a small pool."""
    import torch
    import paper_2404_00456_amd as q
    hkv, D, G, page = 2, 256, 32, 64
    bt = Batch(50, [1, 40], [150, 300], hkv, D, G, page, exact=False)
    per = hkv * page * D // 2
    shift = (1 << 32) // per + 3
    far = bt.table + np.where(bt.table >= 0, shift, 0).astype(np.int32)
    x = torch.randn(bt.T, 4 * hkv, D, device=dev).half()
    results = []
    for table, pages in ((bt.table, bt.pages), (far, bt.pages + shift)):
        pools = []
        for pool in (bt.k, bt.v):
            big = [torch.empty((pages,) + a.shape[1:], dtype=torch.from_numpy(a).dtype, device=dev)
                   for a in pool]
            for t, a in zip(big, pool):
                t[pages - bt.pages:] = D_(a, dev)
            pools.append(tuple(big))
        rest = (D_(table, dev), D_(bt.lens, dev), D_(bt.cu, dev))
        q.quarot_kv_append_paged(x[:, :hkv], x[:, hkv:2 * hkv], *pools, *rest, group=G)
        results.append([t[pages - bt.pages:].clone() for p in pools for t in p] +
                       [q.quarot_kv_paged_attention(x, *pools, *rest, group=G),
                        q.quarot_kv_paged_attention(x[:1], *pools, *(t[:1] for t in rest[:2]),
                                                    rest[2][:2], group=G)])
        del pools, big
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert not torch.equal(results[0][0], D_(bt.k[0], dev))  # the new tokens were stored


@pytest.mark.parametrize("G", [128, 32])
def test_one_group_pools_past_32_bits(dev, orc, G):
    """The same for the kernel of single tokens (one group a row)."""
    import torch
    import paper_2404_00456_amd as q
    hkv, D, page = 1, 128, 16
    bt = Batch(51, [1, 1], [100, 37], hkv, D, G, page)
    shift = (1 << 32) // (hkv * page * D // 2) + 1
    qh = D_(bt.queries(8), dev)
    outs = []
    for off in (0, shift):
        pools = []
        for pool in (bt.k, bt.v):
            big = [torch.empty((bt.pages + off,) + a.shape[1:], dtype=torch.from_numpy(a).dtype,
                               device=dev) for a in pool]
            for t, a in zip(big, pool):
                t[off:] = D_(a, dev)
            pools.append(tuple(big))
        table = bt.table + np.where(bt.table >= 0, off, 0).astype(np.int32)
        outs.append(q.quarot_kv_paged_attention(qh, *pools, D_(table, dev), D_(bt.lens, dev),
                                                D_(bt.cu, dev), group=G))
        del pools, big
    assert torch.equal(outs[0], outs[1])


def test_memory_of_a_call_on_another_stream(dev, orc, monkeypatch):
    """What a call on `stream` allocates is that stream's, not the current one's,
    whose work may still use it or reuse it too soon."""
    import torch
    import paper_2404_00456_amd as q
    bt = Batch(60, [1, 1], [3000, 500], 2, 128, 128, 64)
    qh = D_(bt.queries(16), dev)
    args = [D_(a, dev) for a in (*bt.k, *bt.v, bt.table, bt.lens, bt.cu)]
    pos, fr = torch.zeros(2, dtype=torch.int32, device=dev), D_(freq(128), dev)
    kv = torch.zeros(2, 2, 128, dtype=torch.float16, device=dev)
    want = q.quarot_kv_paged_attention(qh, args[:3], args[3:6], *args[6:])
    turned = q.quarot_rope(qh, pos, fr)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on, empty = [], torch.empty

    def spy(*a, **kw):
        on.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **kw)

    with monkeypatch.context() as m:
        m.setattr(torch, "empty", spy)
        outs = [q.quarot_kv_paged_attention(qh, args[:3], args[3:6], *args[6:], stream=side),
                q.quarot_rope(qh, pos, fr, stream=side)]
        q.quarot_kv_append_paged(kv, kv, args[:3], args[3:6], *args[6:], q=qh, stream=side)
    assert len(on) == 4 and set(on) == {side.cuda_stream}
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], turned)


def test_no_tokens(dev):
    """A batch without new tokens: nothing is done, and nothing refused."""
    import torch
    import paper_2404_00456_amd as q
    bt = Batch(61, [0, 0], [40, 0], 2, 64, 32, 16)
    args = [D_(a, dev) for a in (*bt.k, *bt.v, bt.table, bt.lens, bt.cu)]
    before = [a.clone() for a in args]
    x, kv = (torch.zeros(0, h, 64, dtype=torch.float16, device=dev) for h in (6, 2))
    pos = torch.zeros(3, 0, dtype=torch.int32, device=dev)
    fr = D_(freq(64), dev)
    assert q.quarot_rope(x, pos[0], fr).shape == x.shape
    assert q.quarot_rope(x, pos, fr, sections=[2, 15, 15], rotate=True).shape == x.shape
    assert q.quarot_kv_append_paged(kv, kv, args[:3], args[3:6], *args[6:], group=32, q=x,
                                    positions=pos, inv_freq=fr, sections=[2, 15, 15]).shape == x.shape
    assert q.quarot_kv_paged_attention(x, args[:3], args[3:6], *args[6:], group=32).shape == x.shape
    for a, b in zip(args, before):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
