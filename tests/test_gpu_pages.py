"""The cache's pages on the GPU against the plain ones (tests/pages_plain.py): tables,
lengths, references, lists and copies, whole numbers all of them."""
import random

import numpy as np
import pytest

from pages_plain import Pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2404_00456_amd as q
    q.lib()
    return torch.device("cuda:0")


def ints(x, dev):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=dev)


class Both:
    """The plain pages and the device's, on which every call is made and compared."""

    def __init__(self, dev, *sizes):
        self.p, self.dev = Pages(*sizes), dev
        self.put()

    def put(self):
        # views at odd offsets of a wider buffer: 4-byte alignment is all that is asked
        import torch
        wide = torch.full((len(self.p.refs) + 1,), -7, dtype=torch.int32, device=self.dev)
        wide[1:] = ints(self.p.refs, self.dev)
        self.refs = wide[1:]
        self.table, self.lens = ints(self.p.table, self.dev), ints(self.p.lens, self.dev)

    def same(self):
        assert self.table.tolist() == self.p.table
        assert self.lens.tolist() == self.p.lens
        assert self.refs.tolist() == self.p.refs

    def fork(self, parent):
        import paper_2404_00456_amd as q
        self.p.fork(parent)
        q.quarot_kv_pages_fork(self.table, self.lens, self.refs, ints(parent, self.dev))
        self.same()

    def reserve(self, new):
        import paper_2404_00456_amd as q
        ref = self.p.reserve(new)
        got = q.quarot_kv_pages_reserve(self.table, self.lens, self.refs, ints(new, self.dev), self.p.page)
        for g, r in zip(got, ref):
            assert g.tolist() == (r if isinstance(r, list) else [r])
        self.same()
        return ref

    def compact(self):
        import paper_2404_00456_amd as q
        ref = self.p.compact()
        got = q.quarot_kv_pages_compact(self.table, self.refs)
        for g, r in zip(got, ref):
            assert g.tolist() == (r if isinstance(r, list) else [r])
        self.same()


@pytest.mark.parametrize("B,most,n,page", [
    (1, 1, 1, 16), (1, 9, 3, 16), (3, 5, 40, 32), (64, 20, 700, 16), (257, 70, 9000, 48),
    (1100, 6, 20000, 16), (5, 1100, 3000, 64), (4097, 3, 17000, 16),
])
def test_calls_in_any_order(dev, B, most, n, page):
    rng = random.Random(B * 1000 + n)
    x = Both(dev, B, most, n, page)
    for step in range(24):
        op = rng.choice(["grow", "grow", "grow", "shrink", "fork", "reorder", "compact"])
        if op in ("grow", "shrink"):
            big = rng.random() < 0.3
            room = [most * page - t for t in x.p.lens]
            new = [min(r, rng.choice([0, 1, 1, 2, page, rng.randint(0, 3 * page) if big else 1])) for r in room]
            if op == "shrink":
                new = [-rng.randint(0, 2 * page) if rng.random() < 0.5 else v for v in new]
            missing = x.reserve(new)[3]
            if missing:
                x.fork([b if rng.random() < 0.5 else -1 for b in range(B)])
        elif op == "fork":
            x.fork([rng.choice([b, b, b, rng.randrange(B), -1]) for b in range(B)])
        elif op == "reorder":
            order = list(range(B))
            rng.shuffle(order)
            x.fork(order)
        else:
            x.compact()
        assert x.p.consistent()


def test_forked_prompts_write_apart(dev):
    """Four beams of each prompt grow from a page that all of them hold: the lowest keeps
    it, the others copy it; where one of them waits, all that grow copy."""
    x = Both(dev, 12, 8, 64, 16)
    x.reserve([20, 0, 0, 0, 33, 0, 0, 0, 32, 0, 0, 0])
    x.fork([0, 0, 0, 0, 4, 4, 4, 4, 8, 8, 8, 8])
    cu, src, dst, missing = x.reserve([1, 1, 1, 1, 1, 0, 1, 1, 1, 1, 1, 1])
    assert src[:8] == [-1, 1, 1, 1, 4, -1, 4, 4] and src[8:] == [-1] * 4 and missing == 0
    assert cu == [0, 1, 2, 3, 4, 5, 5, 6, 7, 8, 9, 10, 11]


def test_limits(dev):
    """Positions past the table, too few pages, lengths and numbers at their ends."""
    x = Both(dev, 3, 4, 6, 16)
    assert x.reserve([64, 0, 1])[3] == 0
    assert x.reserve([1, 0, 0])[3] == -1
    assert x.reserve([0, 17, 0])[3] == 1 and x.reserve([0, 64, 49])[3] == 6
    assert x.reserve([2 ** 31 - 1, 1, 1])[3] == -1
    assert x.reserve([-2 ** 31, 1, 1])[3] == 0 and x.p.lens[0] == 0
    x.fork([2 ** 31 - 1, -2 ** 31, 2])
    assert x.p.lens == [0, 0, 2]


def test_tables_of_any_content(dev):
    """Entries outside the pool are no page; pages held without a reference stay whose
    they are.  (Nothing else is said of such tables but what the plain ones do.)"""
    x = Both(dev, 4, 6, 10, 16)
    x.reserve([30, 10, 0, 50])
    x.p.table[0][3] = 10
    x.p.table[1][1] = -2 ** 31
    x.p.table[2] = [2 ** 31 - 1, 55, -9, -1, -1, 12]
    x.p.table[3][0] = 77  # a page that held older tokens is given back by its owner
    x.p.refs[3] = 0
    x.p.lens[3] = 20
    x.put()
    x.reserve([2, 3, 1, 1])
    x.fork([1, 0, 3, 2])
    x.compact()
    x.reserve([5, -3, 1, -30])


@pytest.mark.parametrize("hkv,page,D,G,pages", [(1, 16, 64, 64, 7), (8, 64, 128, 128, 40),
                                                (3, 48, 128, 32, 33), (5, 128, 256, 32, 9)])
def test_copies_move_bytes(dev, hkv, page, D, G, pages):
    import torch
    import paper_2404_00456_amd as q
    rng = np.random.default_rng(pages)
    lead = (pages, hkv, page)
    pools = [rng.integers(0, 256, lead + (w,), dtype=np.uint8)
             for w in (D // 2, 2 * D // G, 2 * D // G) * 2]
    ref = [x.copy() for x in pools]
    order = rng.permutation(pages)
    src, dst = order[:pages // 2].copy(), order[pages // 2:][:pages // 2].copy()
    for x in ref:
        x[dst] = x[src]
    # pairs that are left out, at every place
    s = np.array([-1, *src, pages, -2 ** 31, int(src[0]), 2 ** 31 - 1, int(dst[0])], np.int32)
    d = np.array([int(dst[0]), *dst, int(dst[0]), int(dst[0]), -1, int(dst[0]), int(dst[0])], np.int32)
    kind = [torch.uint8, torch.float16, torch.float16] * 2
    dv = [torch.from_numpy(x).to(dev).view(t) for x, t in zip(pools, kind)]
    q.quarot_kv_pages_copy(tuple(dv[:3]), tuple(dv[3:]), ints(s, dev), ints(d, dev))
    for x, y in zip(dv, ref):
        assert np.array_equal(x.view(torch.uint8).cpu().numpy(), y)
    q.quarot_kv_pages_copy(tuple(dv[:3]), tuple(dv[3:]), ints([], dev), ints([], dev))


def test_large_pool_past_32_bits(dev):
    """Pages that begin behind 2^32 bytes of their pool."""
    import torch
    import paper_2404_00456_amd as q
    n = 2 ** 32 // (8 * 128 * 64) + 5
    kc = torch.zeros((n, 8, 128, 64), dtype=torch.uint8, device=dev)
    ks, kz = (torch.zeros((n, 8, 128, 1), dtype=torch.float16, device=dev) for _ in range(2))
    kc[n - 1], ks[n - 1], kz[0] = 7, 2.0, 3.0
    kc[1] = 9
    q.quarot_kv_pages_copy((kc, ks, kz), (kc.clone(), ks.clone(), kz.clone()), ints([n - 1, 1, 0], dev),
                           ints([3, n - 2, n - 3], dev))
    assert (kc[3] == 7).all() and (kc[n - 2] == 9).all() and (ks[3] == 2).all() and (kz[n - 3] == 3).all()
    assert (kc[4] == 0).all() and (kc[n - 3] == 0).all()


def test_step_in_a_graph(dev):
    """A captured step (fork, reserve, copy) goes on from its own results."""
    import torch
    import paper_2404_00456_amd as q
    B, page, most, n = 8, 16, 12, 120
    p = Pages(B, most, n, page)
    p.reserve([40] * B)
    table, lens, refs = ints(p.table, dev), ints(p.lens, dev), ints(p.refs, dev)
    parent, new = ints(list(range(B)), dev), ints([0] * B, dev)
    kc = torch.randint(0, 256, (n, 1, page, 32), dtype=torch.uint8, device=dev)
    ks = torch.randn((n, 1, page, 1), device=dev).half()
    k, v = (kc, ks, ks.clone()), (kc.clone(), ks.clone(), ks.clone())
    ref = kc.cpu().numpy().copy()
    ws = torch.empty(q.quarot_kv_pages_workspace_size(n), dtype=torch.uint8, device=dev)
    out = [ints([0] * m, dev) for m in (B + 1, B, B, 1)]

    def step():
        q.quarot_kv_pages_fork(table, lens, refs, parent)
        q.quarot_kv_pages_reserve(table, lens, refs, new, page, *out, workspace=ws)
        q.quarot_kv_pages_copy(k, v, out[1], out[2])

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    rng = random.Random(1)
    for _ in range(12):
        pa = [rng.randrange(B) for _ in range(B)]
        nn = [rng.choice([1, 1, 5, -2, 0]) for _ in range(B)]
        parent.copy_(ints(pa, dev))
        new.copy_(ints(nn, dev))
        g.replay()
        torch.cuda.synchronize()
        p.fork(pa)
        cu, src, dst, missing = p.reserve(nn)
        for s, d in zip(src, dst):
            if s >= 0:
                ref[d] = ref[s]
        assert [o.tolist() for o in out] == [cu, src, dst, [missing]]
        assert table.tolist() == p.table and lens.tolist() == p.lens and refs.tolist() == p.refs
        assert np.array_equal(kc.cpu().numpy(), ref) and np.array_equal(v[0].cpu().numpy(), ref)


def test_another_stream(dev):
    import torch
    import paper_2404_00456_amd as q
    x = Both(dev, 3, 4, 20, 16)
    new = ints([17, 5, 0], dev)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = q.quarot_kv_pages_reserve(x.table, x.lens, x.refs, new, 16, stream=s)
    q.quarot_kv_pages_fork(x.table, x.lens, x.refs, ints([0, 0, 1], dev), stream=s)
    s.synchronize()
    x.p.reserve([17, 5, 0])
    x.p.fork([0, 0, 1])
    x.same()
    assert got[0].tolist() == [0, 17, 22, 22]


@pytest.mark.parametrize("B", [3, 1500])
def test_new_tokens_of_a_batch(dev, B):
    """More than 2^30 new tokens are refused, however few each sequence has."""
    import torch
    import paper_2404_00456_amd as q
    table = torch.full((B, 1), -1, dtype=torch.int32, device=dev)
    lens, refs = ints([0] * B, dev), ints([0] * 8, dev)
    page = 1 << 29
    new = ints([page] * 3 + [0] * (B - 3), dev)
    cu, src, dst, missing = q.quarot_kv_pages_reserve(table, lens, refs, new, page)
    assert missing.item() == -1 and not cu.any() and not lens.any() and (table == -1).all()
    new[0] = 0
    cu, src, dst, missing = q.quarot_kv_pages_reserve(table, lens, refs, new, page)
    assert missing.item() == 0 and cu[-1].item() == 2 * page and lens.tolist()[:4] == [0, page, page, 0][:min(4, B)]
