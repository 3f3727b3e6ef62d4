"""The serving calls as they are used together: prompts of a small attention layer with a
prefix that sees itself, forked into beams, sampled, grown, forked again and compacted,
against the same steps in plain numpy with a cache of its own."""
import random

import numpy as np
import pytest

from pages_plain import Pages
from sample_plain import sample

pytestmark = pytest.mark.gpu

H, HKV, D, G, PAGE, VOCAB = 8, 2, 128, 128, 16, 1000
CAP = 12.0
SLOPES = (2.0 ** -np.arange(1, H + 1)).astype(np.float32)


@pytest.fixture(scope="module")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2404_00456_amd as q
    q.lib()
    return torch.device("cuda:0")


class Layer:
    """One attention layer with random weights: tokens to queries, keys and values, and the
    attention's output to logits."""

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.qkv = (rng.standard_normal((VOCAB, H + 2 * HKV, D)) * 1.5).astype(np.float16)
        self.out = (rng.standard_normal((H * D, VOCAB)) * 0.15).astype(np.float32)


class Plain:
    """Each sequence's tokens in lists, its keys and values as the quantizer leaves them."""

    def __init__(self, orc, layer, B):
        self.orc, self.layer = orc, layer
        self.tokens = [[] for _ in range(B)]
        self.prefix = [0] * B

    def fork(self, parent):
        self.tokens = [list(self.tokens[p]) if p >= 0 else [] for p in parent]
        self.prefix = [self.prefix[p] if p >= 0 else 0 for p in parent]

    def values(self, rows):
        c, s, z = self.orc.kv_quant_f32(np.ascontiguousarray(rows, np.float32), G, 0.95)
        x = np.empty(rows.shape)
        x[:, 0::2], x[:, 1::2] = c & 15, c >> 4
        return x * s.astype(np.float64) + z.astype(np.float64)

    def attend(self, b, n):
        """Outputs [n, H, D] of the last n tokens, which are in the cache."""
        t = np.array(self.tokens[b])
        total = len(t)
        rows = self.layer.qkv[t]
        out = np.zeros((n, H, D))
        p, at = np.arange(total - n, total)[:, None], np.arange(total)[None]
        see = (at <= p) | (at < self.prefix[b])
        for h in range(HKV):
            k = self.values(self.orc.rotate_rows(np.ascontiguousarray(rows[:, H + h])))
            v = self.values(rows[:, H + HKV + h].astype(np.float32))
            for r in range(h * H // HKV, (h + 1) * H // HKV):
                qr = self.orc.f32_to_f16(self.orc.rotate_rows(np.ascontiguousarray(rows[total - n:, r])))
                x = CAP * np.tanh(qr.astype(np.float64) @ k.T / D ** 0.5 / CAP) - SLOPES[r] * abs(p - at)
                w = np.exp(np.where(see, x, -np.inf))
                out[:, r] = w @ v / w.sum(-1, keepdims=True)
        return out


class Device:
    """The same on the GPU: pools, a table, lengths and references."""

    def __init__(self, dev, layer, B, most, pages):
        import torch
        self.dev, self.t = dev, torch
        i32 = dict(dtype=torch.int32, device=dev)
        self.table, self.lens = torch.full((B, most), -1, **i32), torch.zeros(B, **i32)
        self.refs = torch.zeros(pages, **i32)
        self.k, self.v = ((torch.zeros((pages, HKV, PAGE, D // 2), dtype=torch.uint8, device=dev),
                           *(torch.full((pages, HKV, PAGE, D // G), float("nan"), dtype=torch.float16, device=dev)
                             for _ in range(2))) for _ in range(2))
        self.qkv = torch.from_numpy(layer.qkv).to(dev)
        self.out = torch.from_numpy(layer.out).to(dev)
        self.slopes = torch.from_numpy(SLOPES).to(dev)

    def ints(self, x):
        return self.t.tensor(x, dtype=self.t.int32, device=self.dev)

    def step(self, new_tokens, counts, prefix):
        """The tokens of all sequences (rows behind cu's last belong to none): outputs, cu."""
        import paper_2404_00456_amd as q
        cu, src, dst, missing = q.quarot_kv_pages_reserve(self.table, self.lens, self.refs, counts, PAGE)
        q.quarot_kv_pages_copy(self.k, self.v, src, dst)
        x = self.qkv[new_tokens.long()]
        ready = q.quarot_kv_append_paged(x[:, H:H + HKV], x[:, H + HKV:], self.k, self.v, self.table, self.lens,
                                         cu, group=G, q=x[:, :H])
        n = cu.diff()
        T = new_tokens.shape[0]
        b = self.t.searchsorted(cu[1:].contiguous(), self.t.arange(T, device=self.dev, dtype=self.t.int32),
                                right=True).clamp(max=n.shape[0] - 1)
        p = (self.lens - n)[b] + self.t.arange(T, device=self.dev) - cu[b]
        end = self.t.maximum(p + 1, prefix[b]).to(self.t.int32)
        o = q.quarot_kv_paged_attention_scored(ready, self.k, self.v, self.table, self.lens, cu, group=G, cap=CAP,
                                               slopes=self.slopes, end=end)
        return o, cu, missing


@pytest.mark.parametrize("seed,graph", [(0, False), (1, True)])
def test_beams_from_prompts(dev, orc, seed, graph):
    import torch
    import paper_2404_00456_amd as q
    rng = random.Random(seed)
    layer = Layer(seed)
    B, most, pages = 8, 12, 60
    plain, d, book = Plain(orc, layer, B), Device(dev, layer, B, most, pages), Pages(B, most, pages, PAGE)

    # two prompts, whose first parts see each other
    prompts = {0: 37, 4: 70}
    new = [prompts.get(b, 0) for b in range(B)]
    for b, n in prompts.items():
        plain.tokens[b] = [rng.randrange(VOCAB) for _ in range(n)]
        plain.prefix[b] = rng.randint(1, n)
    flat = [x for b in range(B) for x in plain.tokens[b]] + [0, 0]  # and rows of no sequence
    prefix = d.ints(plain.prefix)
    o, cu, missing = d.step(d.ints(flat), d.ints(new), prefix)
    book.reserve(new)
    assert missing.item() == 0 and cu.tolist() == np.cumsum([0] + new).tolist()
    got = o.cpu().numpy().astype(np.float64)
    for b, n in prompts.items():
        check(got[cu[b]:cu[b + 1]], plain.attend(b, n), layer)

    # every prompt's four beams
    parent = [0, 0, 0, 0, 4, 4, 4, 4]
    q.quarot_kv_pages_fork(d.table, d.lens, d.refs, d.ints(parent))
    plain.fork(parent)
    book.fork(parent)
    prefix.copy_(d.ints(plain.prefix))
    last = torch.stack([o[cu[1] - 1]] * 4 + [o[cu[5] - 1]] * 4)

    tokens, counts, u, parents = d.ints([0] * B), d.ints([1] * B), torch.zeros(B, device=dev), d.ints(list(range(B)))
    temperature, top_p = torch.full((B,), 0.9, device=dev), torch.full((B,), 0.95, device=dev)
    top_k, logits = d.ints([40] * B), torch.zeros((B, VOCAB), device=dev)

    def one_step():
        """Beams chosen, their next tokens drawn, appended and attended to."""
        q.quarot_kv_pages_fork(d.table, d.lens, d.refs, parents)
        torch.mm(last.view(B, -1).float(), d.out, out=logits)
        q.quarot_sample(logits, u, temperature, top_k, top_p, tokens=tokens)
        o, cu, missing = d.step(tokens, counts, prefix)
        last.copy_(o)
        return missing

    run, state = one_step, (d.table, d.lens, d.refs, last, tokens, *d.k, *d.v)
    if graph:
        kept = [x.clone() for x in state]
        one_step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            missing = one_step()
        for x, y in zip(state, kept):
            x.copy_(y)
        run = lambda: (g.replay(), missing)[1]  # noqa: E731
    for step in range(24):
        # beams go on from some beam of their prompt, whose logits they take
        parent = [b // 4 * 4 + rng.randrange(4) if step % 3 == 0 else b for b in range(B)]
        us = [rng.random() for _ in range(B)]
        parents.copy_(d.ints(parent))
        u.copy_(torch.tensor(us))
        last.copy_(last[parents.long()])
        before = last.cpu()
        miss = run()
        torch.cuda.synchronize()
        assert miss.item() == 0
        # the drawn tokens are those of these logits
        seen = logits.cpu().numpy()
        assert np.abs(seen - before.view(B, -1).double().numpy() @ layer.out).max() < 1e-3
        drawn = tokens.tolist()
        assert drawn == sample(seen, np.array(us, np.float32), [np.float32(0.9)] * B, [40] * B,
                               [np.float32(0.95)] * B).tolist()
        plain.fork(parent)
        book.fork(parent)
        book.reserve([1] * B)
        for b, x in enumerate(drawn):
            plain.tokens[b].append(x)
        assert d.table.tolist() == book.table and d.lens.tolist() == book.lens and d.refs.tolist() == book.refs
        got = last.cpu().numpy().astype(np.float64)
        for b in range(B):
            check(got[b:b + 1], plain.attend(b, 1), layer)
        if step == 11:  # one prompt ends, the pool is compacted
            keep = [0, 1, 2, 3, -1, -1, -1, -1]
            q.quarot_kv_pages_fork(d.table, d.lens, d.refs, d.ints(keep))
            src, dst, live = q.quarot_kv_pages_compact(d.table, d.refs)
            q.quarot_kv_pages_copy(d.k, d.v, src, dst)
            book.fork(keep)
            assert (src.tolist(), dst.tolist(), live.item()) == book.compact()
            # and the other's beams take its places
            again = [0, 1, 2, 3, 0, 1, 2, 3]
            q.quarot_kv_pages_fork(d.table, d.lens, d.refs, d.ints(again))
            book.fork(again)
            plain.fork(again)
            prefix.copy_(d.ints(plain.prefix))
            last.copy_(last[d.ints(again).long()])
    assert book.consistent()


def check(got, ref, layer):
    """Values are below 6 (normal rows of 1.5, scales of a 15th of their range), weights and
    outputs are rounded to fp16 and, in tiles, keys and values too: with scores up to CAP a
    weight is off by exp(2 CAP 2^-11) - 1 at most, an output by twice that, and a value's
    own and the output's roundings."""
    tol = 6 * (2 * np.expm1(2 * CAP * 2.0 ** -11) + 3 * 2.0 ** -11)
    assert np.abs(got - ref).max() <= tol
