"""Scored attention over the paged cache on the GPU against its definition in
binary64: caps, slopes, spans, alone and together, in the kernels for few rows and in
the tiles of every head width."""
import numpy as np
import pytest

from paged_cases import FOUR_ROUNDINGS, ONE_ROUNDING, Batch, few_rows, relative_rms
from paged_plain import scored_attention, scored_tolerance

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


def run(dev, bt, qh, G, fill=7.0, out=None, **kw):
    import torch
    import paper_2404_00456_amd as q
    kp, vp = (tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v))
    form = {n: D_(kw.pop(n, None), dev) for n in ("slopes", "begin", "end")}
    if out is None:
        out = torch.full(qh.shape, fill, dtype=torch.float16, device=dev)
    got = q.quarot_kv_paged_attention_scored(
        D_(qh, dev), kp, vp, D_(bt.table, dev), D_(bt.lens, dev), D_(bt.cu, dev), group=G, out=out,
        window=kw.pop("window", 0), n_sinks=kw.pop("sinks", 0), **form, **kw)
    assert got is out
    return got.cpu().numpy()


def check(dev, bt, qh, exact=True, cap=0.0, sm_scale=None, max_seq_len=None, **kw):
    got = run(dev, bt, qh, bt.G, cap=cap, sm_scale=sm_scale, max_seq_len=max_seq_len, **kw)
    ref = scored_attention(bt, qh, cap=cap, sm_scale=sm_scale, out=np.full(qh.shape, 7.0), **kw)
    tol = scored_tolerance(bt, qh, exact, cap, sm_scale)
    assert np.abs(got.astype(np.float64) - ref).max() <= tol
    assert (got[bt.cu[-1]:] == 7.0).all()
    # what the form adds to a score is too little to show on average
    assert relative_rms(bt, got, ref) < (ONE_ROUNDING if few_rows(bt, qh.shape[1]) else FOUR_ROUNDINGS)
    return got, ref


def spans(bt, kind, seed=3):
    """begin, end [T] of documents, prefixes, any spans, or such that see nothing."""
    rng = np.random.default_rng(seed)
    begin, end = np.zeros(bt.T, np.int32), np.zeros(bt.T, np.int32)
    for b, (n, total) in enumerate(zip(bt.new, bt.total)):
        p = np.arange(total - n, total)
        r = slice(bt.cu[b], bt.cu[b + 1])
        cut = np.sort(rng.integers(0, total + 1, 1 + total // 40))
        cut = np.concatenate([[0], cut])
        if kind == "documents":
            begin[r], end[r] = cut[np.searchsorted(cut, p, side="right") - 1], p + 1
        elif kind == "prefix":
            begin[r], end[r] = 0, np.maximum(p + 1, rng.integers(0, total + 1))
        else:  # any: before, behind, outside, empty
            begin[r] = rng.integers(-50, total + 50, n)
            end[r] = rng.integers(-50, total + 80, n)
            far = rng.random(n) < 0.1
            begin[r] = np.where(far, rng.choice([-2 ** 31, 2 ** 31 - 1], n), begin[r])
            end[r] = np.where(rng.random(n) < 0.1, rng.choice([-2 ** 31, 2 ** 31 - 1], n), end[r])
    return begin, end


FORMS = {
    "cap": dict(cap=5.0),
    "slopes": dict(slopes=True),
    "both": dict(cap=30.0, slopes=True),
    "documents": dict(spans="documents"),
    "prefix": dict(spans="prefix", cap=8.0),
    "prefix_slopes": dict(spans="prefix", slopes=True),
    "any": dict(spans="any", slopes=True, cap=20.0),
    "any_sinks": dict(spans="any", sinks=5),
    "window": dict(window=37, sinks=3, slopes=True),
    "window_documents": dict(window=70, sinks=9, spans="documents", cap=3.0),
    "large_cap": dict(cap=3000.0, slopes=True),
}

SHAPES = [
    # new, total, H, hkv, D, G, page
    ([1], [1], 4, 4, 128, 128, 16),
    ([1], [700], 16, 2, 128, 128, 64),
    ([1, 1, 1], [7, 64, 65], 8, 1, 128, 128, 64),
    ([1, 2, 1, 0], [300, 90, 1, 5], 8, 2, 64, 64, 16),
    ([2, 1, 3], [130, 77, 40], 4, 1, 128, 32, 48),
    ([1, 4], [200, 333], 3, 3, 256, 64, 32),
    ([1, 1], [3, 257], 5, 5, 256, 256, 16),
    ([33, 2], [40, 100], 5, 5, 64, 64, 48),
    ([100, 1, 29], [230, 300, 29], 8, 2, 128, 128, 64),
    ([65, 1], [65, 9], 40, 2, 128, 64, 32),
    ([40, 7], [300, 90], 2, 1, 256, 128, 128),
    ([150], [400], 6, 3, 64, 32, 16),
]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("new,total,H,hkv,D,G,page", SHAPES)
def test_forms_match_definition(dev, new, total, H, hkv, D, G, page, form):
    f = dict(FORMS[form])
    bt = Batch(len(form) + sum(total), new, total, hkv, D, G, page, behind=2)
    kw = dict(cap=f.get("cap", 0.0), window=f.get("window", 0), sinks=f.get("sinks", 0))
    if f.get("slopes"):
        s = 2.0 ** (-8.0 * np.arange(1, H + 1) / H)
        s[H // 2] = 0.0
        kw["slopes"] = s.astype(np.float32)
    if "spans" in f:
        kw["begin"], kw["end"] = spans(bt, f["spans"])
    check(dev, bt, bt.queries(H), **kw)


@pytest.mark.parametrize("D,G,new,total", [(128, 128, [520, 1], [1100, 1500]),
                                           (64, 32, [700], [900]), (256, 256, [150], [600])])
@pytest.mark.parametrize("form", ["cap", "both", "prefix_slopes", "any"])
def test_longer_ones_of_normal_rows(dev, D, G, new, total, form):
    """Rows as the quantizer leaves them, split over blocks (one cache head)."""
    f = dict(FORMS[form])
    bt = Batch(5, new, total, 1, D, G, 32, behind=1, exact=False)
    kw = dict(cap=f.get("cap", 0.0), sinks=4)
    if f.get("slopes"):
        kw["slopes"] = np.array([0.5, 0.004], np.float32)
    if "spans" in f:
        kw["begin"], kw["end"] = spans(bt, f["spans"])
    check(dev, bt, bt.queries(2, 2.0), exact=False, max_seq_len=max(total), **kw)


@pytest.mark.parametrize("hkv,rep,D,G", [(1, 1, 128, 128), (2, 1, 64, 32), (1, 3, 256, 256), (3, 2, 128, 32)])
@pytest.mark.parametrize("form", ["cap", "any"])
def test_many_splits_of_few_heads(dev, hkv, rep, D, G, form):
    """Rows of a tile whose splits are joined by blocks of a few rows each; the last tile
    of a sequence is partly rows of nobody."""
    f = dict(FORMS[form])
    new, total = [300, 33, 1, 129], [2900, 700, 500, 1600]
    bt = Batch(11, new, total, hkv, D, G, 16, behind=2, exact=False)
    kw = dict(cap=f.get("cap", 0.0), sinks=3)
    if "spans" in f:
        kw["begin"], kw["end"] = spans(bt, f["spans"])
    check(dev, bt, bt.queries(hkv * rep, 2.0), exact=False, max_seq_len=max(total), **kw)


def test_no_form_is_the_plain_attention(dev):
    """No cap, no slopes, no spans: few rows bit for bit, tiles within their roundings;
    slopes of 0 and spans of the causal order change nothing."""
    import paper_2404_00456_amd as q
    for new, total, H in (([1, 1], [300, 40], 8), ([90, 3], [200, 50], 8)):
        bt = Batch(8, new, total, 2, 128, 128, 16)
        qh = bt.queries(H)
        kp, vp = (tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v))
        ref = q.quarot_kv_paged_attention(D_(qh, dev), kp, vp, D_(bt.table, dev), D_(bt.lens, dev),
                                          D_(bt.cu, dev), window=50, n_sinks=2).cpu().numpy()
        p = np.concatenate([np.arange(t - n, t) for n, t in zip(new, total)]).astype(np.int32)
        for kw in ({}, dict(slopes=np.zeros(H, np.float32)), dict(end=p + 1),
                   dict(begin=np.zeros_like(p), end=p + 1)):
            got = run(dev, bt, qh, 128, window=50, sinks=2, **kw)
            assert np.abs(got.astype(np.float64) - ref).max() <= \
                scored_tolerance(bt, qh, True) + np.abs(ref.astype(np.float64)).max() * 2.0 ** -11
            if not kw:
                assert np.array_equal(got.view(np.uint16), ref.view(np.uint16))


def test_distance_of_far_spans(dev):
    """A query whose span ends far before it: its weights among those tokens are as exact
    as nearby (slope 1/2 over 30000 positions is 15000)."""
    bt = Batch(9, [1, 40], [30000, 20000], 1, 64, 64, 64, spare=1)
    qh = bt.queries(4)
    begin = np.full(bt.T, 30, np.int32)
    end = np.full(bt.T, 64, np.int32)
    begin[0], end[0] = 100, 131
    check(dev, bt, qh, slopes=np.array([0.5, 0.1, 0.0, 1.5], np.float32), begin=begin, end=end, sinks=1)


@pytest.mark.parametrize("new,G", [([1, 2], 128), ([1, 2], 32), ([70, 9], 128), ([70, 9], 64)])
def test_values_that_are_not_finite_reach_who_sees_them(dev, new, G):
    """Infinite and undefined values in a document reach its queries alone."""
    total = [200, 160]
    bt = Batch(11, new, total, 1, 128, G, 16)
    qh = bt.queries(4)
    begin, end = spans(bt, "documents", 5)
    # before the last row's document, and the last token (its own row alone sees it)
    assert begin[bt.cu[1] - 1] > 0
    for b, at in ((0, begin[bt.cu[1] - 1] - 1), (1, 3), (1, total[1] - 1)):
        bt.v[1][bt.table[b, at // 16], 0, at % 16, 0] = np.inf if b else np.nan
    got = run(dev, bt, qh, G, begin=begin, end=end, cap=9.0, slopes=np.full(4, 0.01, np.float32))
    with np.errstate(invalid="ignore"):
        ref = scored_attention(bt, qh, begin=begin, end=end, cap=9.0, slopes=np.full(4, 0.01))
        tol = scored_tolerance(bt, qh, True, 9.0)
    fine = np.isfinite(ref)
    assert not fine.all() and fine.any()
    assert np.array_equal(fine, np.isfinite(got[:len(ref)]))
    assert np.abs(got[fine].astype(np.float64) - ref[fine]).max() <= tol


@pytest.mark.parametrize("D,G", [(128, 128), (64, 32)])
@pytest.mark.parametrize("new,total", [([9, 2, 5], [4, 1, 0]), ([60, 40], [33, 0]), ([50, 3], [49, 300])])
def test_positions_before_the_first(dev, new, total, D, G):
    """More new tokens than cached ones: those before position 0 see what their spans say,
    the others what they see at all; spans and windows that begin before 0."""
    bt = Batch(14, new, total, 2, D, G, 16, behind=1)
    qh = bt.queries(6)
    n = len(qh)
    rng = np.random.default_rng(2)
    begin = rng.integers(-90, 20, n).astype(np.int32)
    end = rng.integers(-20, 90, n).astype(np.int32)
    for kw in (dict(slopes=np.full(6, 0.05, np.float32)), dict(begin=begin), dict(end=end, cap=4.0),
               dict(begin=begin, end=end, window=12, sinks=2), dict(begin=begin, window=30),
               dict(begin=np.full(n, -2 ** 31, np.int32), window=5, sinks=1)):
        check(dev, bt, qh, **kw)


def test_heads_beside_and_another_stream(dev):
    """Queries and outputs as slices of wider tensors, on a stream of their own."""
    import torch
    import paper_2404_00456_amd as q
    bt = Batch(12, [30, 1], [80, 400], 2, 128, 128, 32)
    qh = bt.queries(8)
    wide = torch.zeros((bt.T, 12, 128), dtype=torch.float16, device=dev)
    wide[:, 2:10] = D_(qh, dev)
    out = torch.full((bt.T, 11, 128), 3.0, dtype=torch.float16, device=dev)
    kp, vp = (tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v))
    args = (kp, vp, D_(bt.table, dev), D_(bt.lens, dev), D_(bt.cu, dev))
    slopes = D_(np.full(8, 0.02, np.float32), dev)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    q.quarot_kv_paged_attention_scored(wide[:, 2:10], *args, cap=6.0, slopes=slopes, out=out[:, 1:9],
                                       stream=s)
    s.synchronize()
    got = out.cpu().numpy()
    ref = scored_attention(bt, qh, cap=6.0, slopes=np.full(8, 0.02))
    assert np.abs(got[:, 1:9] - ref).max() <= scored_tolerance(bt, qh, True, 6.0)
    assert (got[:, :1] == 3.0).all() and (got[:, 9:] == 3.0).all()


def test_graph_replays_other_spans(dev):
    """A captured call reads lengths, spans and slopes when it runs."""
    import torch
    import paper_2404_00456_amd as q
    bt = Batch(13, [40, 1, 3], [90, 300, 70], 2, 128, 128, 16)
    qh = bt.queries(4)
    kp, vp = (tuple(D_(a, dev) for a in p) for p in (bt.k, bt.v))
    table, lens, cu, qd = D_(bt.table, dev), D_(bt.lens, dev), D_(bt.cu, dev), D_(qh, dev)
    begin, end = torch.zeros(bt.T, dtype=torch.int32, device=dev), torch.zeros(bt.T, dtype=torch.int32, device=dev)
    slopes, out = torch.zeros(4, device=dev), torch.zeros_like(qd)
    need = q.quarot_kv_paged_attention_workspace_size(bt.T, 3, 4, 2, 128, 304)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)

    def call():
        q.quarot_kv_paged_attention_scored(qd, kp, vp, table, lens, cu, cap=7.0, slopes=slopes,
                                           begin=begin, end=end, max_seq_len=304, out=out, workspace=ws)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed, kind in ((1, "documents"), (2, "any"), (3, "prefix"), (4, "any")):
        b_, e_ = spans(bt, kind, seed)
        s_ = np.array([0.0, 0.3, 0.01, 1.0], np.float32) / seed
        begin.copy_(D_(b_, dev))
        end.copy_(D_(e_, dev))
        slopes.copy_(D_(s_, dev))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        ref = scored_attention(bt, qh, cap=7.0, slopes=s_, begin=b_, end=e_)
        assert np.abs(out.cpu().numpy() - ref).max() <= scored_tolerance(bt, qh, True, 7.0)
