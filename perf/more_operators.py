"""Further calls of a server over the paged 4-bit KV cache, as measured cases:
attention whose scores are capped, lose by distance, or are limited to a span of
each query's own (packed documents, prefixes that see each other); the pages
themselves (sequences forked, freed, grown and shrunk, shared pages copied before
they are written, the pool compacted); and the sampling of the next tokens, by which
sequences are forked.

A case is a dict of plain values.  ``prepare`` makes its inputs on the GPU from
a seed, ``run`` is one pass: the library's calls where ``own`` is true, plain
torch otherwise.  ``exact`` is the same result in binary64.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"


# ---------------------------------------------------------------- cases ----

def _attend(name, batch, new, seq, heads, kv_heads, dim, group, page, lens, cap=0.0, slopes=False,
            docs=0, prefix=False, window=0, sinks=0):
    return dict(name=name, op="attend", batch=batch, new=new, seq=seq, heads=heads,
                kv_heads=kv_heads, dim=dim, group=group, page=page, lens=lens, cap=cap,
                slopes=slopes, docs=docs, prefix=prefix, window=window, sinks=sinks)


def _grow(name, batch, beams, seq, new, fork, kv_heads, dim, group, page, lens):
    return dict(name=name, op="grow", batch=batch, beams=beams, seq=seq, new=new, fork=fork,
                kv_heads=kv_heads, dim=dim, group=group, page=page, lens=lens)


def _compact(name, batch, seq, drop, kv_heads, dim, group, page, lens):
    return dict(name=name, op="compact", batch=batch, seq=seq, drop=drop, kv_heads=kv_heads,
                dim=dim, group=group, page=page, lens=lens)


def _sample(name, batch, vocab, dtype, sigma, temperature, top_k, top_p, min_p, masked):
    return dict(name=name, op="sample", batch=batch, vocab=vocab, dtype=dtype, sigma=sigma,
                temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, masked=masked)


def listed():
    return [
        # one chat of a model with capped scores, one new token
        _attend("cap_decode_1x2048", 1, 1, 2048, 16, 8, 128, 128, 64, 0, cap=50.0),
        # 64 chats of 1 .. 8192 tokens of a model whose scores fall with the distance
        _attend("slopes_decode_64x8192_ragged", 64, 1, 8192, 64, 8, 128, 128, 64, 11, slopes=True),
        # short documents packed into one prompt of 8192, 32 leading tokens seen by all
        _attend("documents_8192", 1, 8192, 8192, 64, 8, 128, 128, 64, 3, docs=700, sinks=32),
        # ragged prompts whose first parts (an image, a question) see each other,
        # small heads in groups of 32, capped
        _attend("prefix_6x2000_ragged", 6, 2000, 2000, 16, 4, 64, 32, 16, 5, cap=30.0, prefix=True),
        # a whole prompt with capped scores: the largest call
        _attend("cap_prefill_8192", 1, 8192, 8192, 64, 8, 128, 128, 64, 0, cap=50.0),
        # a step of 64 chats: each grows by a token, the table's pages dealt
        _grow("pages_step_64x1", 64, 1, 4096, 1, "none", 8, 128, 128, 64, 7),
        # a beam search step: 32 prompts with 8 beams each, every beam goes on from
        # some beam of its prompt, last pages are copied where they are shared
        _grow("pages_beam_32x8", 32, 8, 4096, 1, "random", 8, 128, 128, 64, 9),
        # a small pool after half of its 24 sequences ended
        _compact("pages_compact_24x500", 24, 500, 2, 4, 64, 32, 16, 13),
        # a large pool after every third of its 128 sequences ended
        _compact("pages_compact_128x8192", 128, 8192, 3, 8, 128, 128, 64, 15),
        # one chat's next token: vocabulary of 32000, k and p
        _sample("sample_1x32000", 1, 32000, "float16", 3.0, 0.7, 40, 0.95, 0.0, 0),
        # a batch of sequences over a large vocabulary, every limit on in some row
        _sample("sample_256x131072", 256, 131072, "float16", 2.5, 0.8, 1000, 0.9, 0.02, 0),
        # 32-bit logits of an odd vocabulary, a grammar masks most tokens, p alone
        _sample("sample_37x50003_masked", 37, 50003, "float32", 2.0, 1.0, 0, 0.98, 0.0, 3),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "grow", "compact", "sample", "sample"])
    if op == "sample":
        vocab = _log(rng, 1000, 131072)
        return dict(op=op, batch=_log(rng, 1, 256), vocab=vocab,
                    dtype=rng.choice(["float16", "float32"]), sigma=rng.choice([1.0, 2.0, 3.0]),
                    temperature=rng.choice([0.0, 0.6, 1.0, 1.3]),
                    top_k=rng.choice([0, 0, 1, 50, _log(rng, 2, vocab)]),
                    top_p=rng.choice([1.0, 0.9, 0.95, 0.5]),
                    min_p=rng.choice([0.0, 0.0, 0.05]), masked=rng.choice([0, 0, 2, 9]))
    dim = rng.choice([64, 128, 128, 128, 256])
    shape = dict(kv_heads=rng.choice([1, 2, 4, 8]), dim=dim, group=rng.choice([dim, dim, dim, 32]),
                 page=rng.choice([16, 32, 64, 128, 48]), lens=rng.randint(1, 10 ** 6))
    if op == "grow":
        beams = rng.choice([1, 2, 4, 8])
        return dict(op=op, batch=_log(rng, 1, 256 // beams), beams=beams, seq=_log(rng, 16, 4096),
                    new=rng.choice([1, 1, 1, 4, _log(rng, 2, 512)]),
                    fork="none" if beams == 1 else rng.choice(["first", "random"]), **shape)
    if op == "compact":
        return dict(op=op, batch=_log(rng, 2, 128), seq=_log(rng, 16, 8192),
                    drop=rng.choice([2, 3, 5]), **shape)
    heads = shape["kv_heads"] * rng.choice([1, 4, 5, 8])
    if rng.random() < 0.5:  # one new token, or a few that were guessed ahead
        new = rng.choice([1, 1, 1, 2, 4])
        batch = _log(rng, 1, 64)
        seq = max(new, _log(rng, 16, 32768 if batch <= 16 else 8192))
    else:
        batch = rng.randint(1, 8)
        new = _log(rng, 8, 2048)
        seq = max(new, _log(rng, 64, min(16384, 2 ** 32 // (batch * heads * new))))
    limit = rng.choice(["none", "docs", "prefix", "window"])
    return dict(op=op, batch=batch, new=new, seq=seq, heads=heads,
                cap=rng.choice([0.0, 30.0, 50.0]), slopes=rng.random() < 0.5,
                docs=_log(rng, 8, 4096) if limit == "docs" else 0, prefix=limit == "prefix",
                window=_log(rng, 16, 4096) if limit == "window" else 0,
                sinks=rng.choice([0, 1, 4, 64]) if limit in ("docs", "window") else 0, **shape)


def _lengths(case):
    """(new tokens, tokens with the new ones) of each sequence; the first has
    the case's own, the others are ragged where the case has a `lens`."""
    B, new, total = case["batch"], case["new"], case["seq"]
    rng = random.Random(case["lens"])
    n, length = [new], [total]
    for _ in range(B - 1):
        x = new
        if case["lens"] and new > 1:
            x = 1 if rng.random() < 0.3 else rng.randint(1, new)
        n.append(x)
        length.append(x + rng.randint(0, total - new) if case["lens"] else total)
    return n, length


def _spans(case):
    """First position that each new token sees (sinks apart) and the one after its
    last, [T] each: of its document, and to the end of the prefix that it is in."""
    rng = random.Random(case["lens"] + 1)
    begin, end = [], []
    for n, total in zip(*_lengths(case)):
        p = np.arange(total - n, total)
        first, last = np.zeros_like(p), p + 1
        if case["docs"]:
            starts = [0]
            while starts[-1] < total:
                starts.append(starts[-1] + rng.randint(1, 2 * case["docs"]))
            starts = np.array(starts)
            first = starts[np.searchsorted(starts, p, side="right") - 1]
        if case["prefix"]:
            last = np.maximum(last, rng.randint(0, total))
        begin.append(first)
        end.append(last)
    return np.concatenate(begin), np.concatenate(end)


# -------------------------------------------------------------- inputs ----

def _deal(rng, length, page, spare=0):
    """A table that deals the sequences' pages out in random order."""
    need = [(x + page - 1) // page for x in length]
    order = torch.randperm(sum(need) + spare, device=DEV, generator=rng).to(torch.int32)
    table = torch.full((len(length), max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, x in enumerate(need):
        table[b, :x] = order[at:at + x]
        at += x
    return table, sum(need) + spare


def _random_cache(rng, pages, kv_heads, page, dim, group):
    """Codes, scales and zeros of normal rows, as the cache's quantizer leaves
    them: groups whose range is a few sigma, codes around its middle."""
    lead = (pages, kv_heads, page)
    codes = torch.empty((*lead, dim // 2), dtype=torch.uint8, device=DEV)
    scale = torch.empty((*lead, dim // group), dtype=torch.float16, device=DEV)
    zero = torch.empty_like(scale)
    flat = [x.view(-1, x.shape[-1]) for x in (codes, scale, zero)]
    step = max(1, (1 << 26) // dim)
    for r in range(0, flat[0].shape[0], step):
        m = min(step, flat[0].shape[0] - r)
        x = torch.randn((m, dim // group, group), device=DEV, generator=rng)
        lo, hi = x.amin(-1, keepdim=True) * 0.95, x.amax(-1, keepdim=True) * 0.95
        s, z = ((hi - lo) / 15).half(), lo.half()
        c = ((x - z.float()) / s.float()).round_().clamp_(0, 15).to(torch.uint8)
        c = c.view(m, dim // 2, 2)
        flat[0][r:r + step] = c[:, :, 0] | (c[:, :, 1] << 4)
        flat[1][r:r + step], flat[2][r:r + step] = s[:, :, 0], z[:, :, 0]
    return codes, scale, zero


def _any_cache(rng, pages, kv_heads, page, dim, group):
    """Pools whose content only moves: any codes, scales and zeros."""
    lead = (pages, kv_heads, page)
    codes = torch.randint(0, 256, (*lead, dim // 2), dtype=torch.uint8, device=DEV, generator=rng)
    const = torch.randn((2, *lead, dim // group), device=DEV, generator=rng,
                        dtype=torch.float16)
    return codes, const[0].contiguous(), const[1].contiguous()


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _prepare_attend(case, rng, st):
    D, G, Hkv, page, H = (case[k] for k in ("dim", "group", "kv_heads", "page", "heads"))
    n, length = _lengths(case)
    st["n"], st["length"], st["max_len"] = n, length, case["seq"]
    st["cu"], st["lens"] = _int32(np.cumsum([0] + n)), _int32(length)
    st["table"], pages = _deal(rng, length, page)
    st["k_cache"] = _random_cache(rng, pages, Hkv, page, D, G)
    st["v_cache"] = _random_cache(rng, pages, Hkv, page, D, G)
    # scores of a few sigma, more where they are capped
    sigma = 5.0 if case["cap"] else 2.0
    st["q"] = (torch.randn((sum(n), H, D), device=DEV, generator=rng) * sigma).half()
    begin, end = _spans(case)
    st["begin"] = _int32(begin) if case["docs"] else None
    st["end"] = _int32(end) if case["prefix"] else None
    st["slopes"] = None
    if case["slopes"]:  # 2^(-8 (h + 1) / heads)
        h = torch.arange(1, H + 1, dtype=torch.float64, device=DEV)
        st["slopes"] = torch.exp2(-8.0 * h / H).float()


def _meta(st, table, lens, refs):
    """Table, lengths and references in one buffer, which a pass starts from again."""
    st["meta0"] = torch.cat([table.flatten(), lens, refs]).to(torch.int32)
    st["meta"] = st["meta0"].clone()
    a, b = table.numel(), table.numel() + lens.numel()
    st["table"] = st["meta"][:a].view(table.shape)
    st["lens"], st["refs"] = st["meta"][a:b], st["meta"][b:]


def _references(table, pages):
    t = table.flatten().long()
    one = torch.zeros(pages + 1, dtype=torch.int64, device=DEV)
    one.index_add_(0, torch.where(t < 0, pages, t), torch.ones_like(t))
    return one[:pages].to(torch.int32)


def _grow_lengths(case):
    """(tokens that a group's beams share, tokens, new tokens, parent) by sequence."""
    rng = random.Random(case["lens"])
    shared, length, new, parent = [], [], [], []
    beams = case["beams"]
    for g in range(case["batch"]):
        s = rng.randint(max(1, case["seq"] // 4), case["seq"])
        for k in range(beams):
            shared.append(s)
            # beams after the first few steps, all of one length
            length.append(s + (case["page"] // 2 if beams > 1 else 0))
            new.append(case["new"] if rng.random() < 0.7 else rng.randint(1, case["new"]))
            parent.append(g * beams + (k if case["fork"] == "none" else 0 if case["fork"] == "first"
                                       else rng.randrange(beams)))
    return shared, length, new, parent


def _prepare_grow(case, rng, st):
    page, beams = case["page"], case["beams"]
    shared, length, new, parent = _grow_lengths(case)
    most = (case["seq"] + page + case["new"]) // page + 2
    growth = sum((x + n + page - 1) // page for x, n in zip(length, new)) + len(length)
    table, pages = _deal(rng, length, page, spare=growth)
    wide = torch.full((len(length), most), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    whole = _int32([x // page for x in shared])  # pages that hold nothing but shared tokens
    first = torch.arange(len(length), device=DEV) // beams * beams
    own_page = torch.arange(most, device=DEV)[None] >= whole[:, None]
    wide = torch.where(own_page, wide, wide[first])
    _meta(st, wide, _int32(length), _references(wide, pages))
    st["parent"], st["new"] = _int32(parent), _int32(new)
    shape = (pages, case["kv_heads"], page, case["dim"], case["group"])
    st["k_cache"], st["v_cache"] = _any_cache(rng, *shape), _any_cache(rng, *shape)


def _compact_lengths(case):
    rng = random.Random(case["lens"])
    length = [rng.randint(max(1, case["seq"] // 4), case["seq"]) for _ in range(case["batch"])]
    return length, [-1 if b % case["drop"] == 0 else b for b in range(case["batch"])]


def _prepare_compact(case, rng, st):
    page = case["page"]
    length, parent = _compact_lengths(case)
    table, pages = _deal(rng, length, page, spare=len(length))
    _meta(st, table, _int32(length), _references(table, pages))
    st["parent"] = _int32(parent)
    shape = (pages, case["kv_heads"], page, case["dim"], case["group"])
    st["k_cache"], st["v_cache"] = _any_cache(rng, *shape), _any_cache(rng, *shape)


def _prepare_sample(case, rng, st):
    B, V = case["batch"], case["vocab"]
    x = torch.randn((B, V), device=DEV, generator=rng) * case["sigma"]
    # the few tokens that a model holds likely
    likely = torch.randint(0, V, (B, 24), device=DEV, generator=rng)
    x.scatter_(1, likely, 4 * case["sigma"] + torch.randn((B, 24), device=DEV, generator=rng) * 2)
    if case["masked"]:  # all but one token in so many are forbidden
        allowed = torch.randint(0, case["masked"], (B, V), device=DEV, generator=rng) == 0
        x.masked_fill_(~allowed, -math.inf)
    st["logits"] = x.to(getattr(torch, case["dtype"]))
    st["u"] = torch.rand(B, device=DEV, generator=rng)

    def rows(value, off, dtype):  # the case's value in most rows, off in some
        t = torch.full((B,), value, dtype=dtype, device=DEV)
        if B > 1:
            t[torch.rand(B, device=DEV, generator=rng) < 0.2] = off
        return t

    st["temperature"] = rows(case["temperature"], 0.0, torch.float32)
    st["top_k"] = rows(case["top_k"], 0, torch.int32) if case["top_k"] else None
    st["top_p"] = rows(case["top_p"], 1.0, torch.float32) if case["top_p"] < 1 else None
    st["min_p"] = rows(case["min_p"], 0.0, torch.float32) if case["min_p"] else None


def prepare(case, seed):
    rng = torch.Generator(device=DEV)
    rng.manual_seed(seed)
    st = dict(case=case)
    {"attend": _prepare_attend, "grow": _prepare_grow, "compact": _prepare_compact,
     "sample": _prepare_sample}[case["op"]](case, rng, st)
    return st


# ------------------------------------------------------------ plain form ----

def _unpack(cache, group):
    """A cache's values in binary32 [.., D]."""
    codes, scale, zero = cache
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    c = c.unflatten(-1, (-1, group))
    return (c * scale.float()[..., None] + zero.float()[..., None]).flatten(-2)


def _run_attend(st):
    case = st["case"]
    H, Hkv, D, G = (case[k] for k in ("heads", "kv_heads", "dim", "group"))
    B, rep, T, S = case["batch"], H // Hkv, st["q"].shape[0], st["max_len"]

    def dense(cache):  # the sequences' tokens in order: [B, Hkv, S, D]
        table = st["table"].clamp(min=0).long()
        x = _unpack(tuple(c[table] for c in cache), G)  # [B, P, Hkv, page, D]
        return x.transpose(1, 2).flatten(2, 3)[:, :, :S]

    # a padded batch of the queries: [B, Hkv, rep * new, D], and what they see
    n = st["cu"].diff()
    b = torch.repeat_interleave(torch.arange(B, device=DEV), n, output_size=T)
    i = torch.arange(T, device=DEV) - st["cu"][b]
    p = (st["lens"] - n)[b] + i
    q = torch.zeros((B, case["new"], H, D), device=DEV)
    q[b, i] = st["q"].float()
    q = q.view(B, -1, Hkv, rep, D).permute(0, 2, 3, 1, 4).flatten(2, 3)

    def padded(rows, fill):
        t = torch.full((B, case["new"], 1), fill, device=DEV)
        t[b, i, 0] = rows.long()
        return t

    at = padded(p, -1)
    end = at + 1 if st["end"] is None else torch.minimum(padded(st["end"], 0),
                                                         st["lens"][:, None, None])
    key = torch.arange(S, device=DEV)
    low = torch.zeros_like(at) if st["begin"] is None else padded(st["begin"], 0)
    if case["window"]:
        low = torch.maximum(low, at + 1 - case["window"])
    hidden = (key >= end) | ((key < low) & (key >= case["sinks"]))

    s = torch.matmul(q, dense(st["k_cache"]).transpose(-1, -2)).mul_(D ** -0.5)
    s = s.view(B, Hkv, rep, -1, S)
    if case["cap"]:
        s = s.div_(case["cap"]).tanh_().mul_(case["cap"])
    if st["slopes"] is not None:  # one head of each cache head at a time: [B, new, S] distances
        away = (key - at).abs().neg_().float()
        for r in range(rep):
            s[:, :, r].addcmul_(st["slopes"].view(Hkv, rep)[:, r][None, :, None, None],
                                away[:, None])
    s = s.masked_fill_(hidden[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True).clamp_(min=-3e38)
    e = s.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.flatten(2, 3), dense(st["v_cache"])).view(B, Hkv, rep, -1, D) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(B, -1, H, D)
    return o[b, i].half()


def _count(refs, pages, by):
    """refs + by for every entry of `pages` that is a page."""
    n = refs.shape[0]
    wide = torch.cat([refs, refs.new_zeros(1)])
    pages = pages.flatten().long()
    wide.index_add_(0, torch.where((pages < 0) | (pages >= n), n, pages),
                    torch.full_like(pages, by, dtype=torch.int32))
    refs.copy_(wide[:n])


def _fork(st):
    table, lens, refs, parent = st["table"], st["lens"], st["refs"], st["parent"].long()
    there = (parent >= 0) & (parent < table.shape[0])
    safe = torch.where(there, parent, 0)
    after = torch.where(there[:, None], table[safe], -1)
    length = torch.where(there, lens[safe], 0)
    _count(refs, table, -1)
    _count(refs, after, 1)
    table.copy_(after)
    lens.copy_(length)


def _reserve(st):
    table, lens, refs, new, page = st["table"], st["lens"], st["refs"], st["new"], st["case"]["page"]
    (B, P), n = table.shape, refs.shape[0]
    after = (lens + new).clamp(min=0)
    j = torch.arange(P, device=DEV)
    # entries on which new tokens fall, and the page that holds older ones as well
    touched = (new > 0)[:, None] & (j >= (lens // page)[:, None]) & (j * page < after[:, None])
    old = touched & (j * page < lens[:, None])
    entry = table.long()
    valid = (entry >= 0) & (entry < n)
    safe = torch.where(valid, entry, 0)
    shared = valid & (refs[safe] > 1)
    # the lowest of a shared page's sequences keeps it if all of them grow
    where = torch.where(old & shared, safe, n).flatten()
    growing = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    growing.index_add_(0, where, torch.ones_like(where, dtype=torch.int32))
    row = torch.arange(B, device=DEV)[:, None].expand(B, P).flatten()
    lowest = torch.full((n + 1,), B, device=DEV).scatter_reduce_(0, where, row, "amin")
    keeps = (growing[safe] == refs[safe]) & (lowest[safe] == row.view(B, P))
    need = touched & torch.where(old, shared & ~keeps, ~valid | shared)
    rank = need.flatten().cumsum(0).view(B, P)
    free = refs == 0
    at = free.cumsum(0)
    deal = torch.full((n + 1,), -1, dtype=torch.int32, device=DEV)
    deal.scatter_(0, torch.where(free, at - 1, n), torch.arange(n, dtype=torch.int32, device=DEV))
    lacking = rank[-1, -1] - at[-1]
    past = (after > P * page).any()
    done = (lacking <= 0) & ~past
    fresh = torch.where(need, deal[(rank - 1).clamp(0, n - 1)], -1)
    out = (new < 0)[:, None] & (j >= ((after + page - 1) // page)[:, None]) & \
        (j < ((lens + page - 1) // page)[:, None])
    mended = torch.where(need, fresh, torch.where(out, -1, table))
    mended = torch.where(done, mended, table)
    moved = done & need & old
    src = torch.where(moved, table, -1).amax(1)
    dst = torch.where(moved, fresh, -1).amax(1)
    _count(refs, torch.where(done & (need | out), table, -1), -1)
    _count(refs, torch.where(done & need, fresh, -1), 1)
    table.copy_(mended)
    lens.copy_(torch.where(done, after, lens))
    cu = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    cu[1:] = torch.where(done, new.clamp(min=0), 0).cumsum(0)
    missing = torch.where(past, -1, lacking.clamp(min=0)).to(torch.int32).view(1)
    return cu, src, dst, missing


def _copy_pages(st, src, dst):
    move = src >= 0
    src, dst = src[move].long(), dst[move].long()
    for cache in (st["k_cache"], st["v_cache"]):
        for x in cache:
            x[dst] = x[src]


def _squeeze(st):
    """The live pages past the number of them, onto the free ones before it."""
    table, refs = st["table"], st["refs"]
    n = refs.shape[0]
    live = refs > 0
    count = live.sum()
    at = torch.arange(n, dtype=torch.int32, device=DEV)
    high, low = live & (at >= count), ~live & (at < count)
    src = torch.full((n + 1,), -1, dtype=torch.int32, device=DEV)
    dst = src.clone()
    src.scatter_(0, torch.where(high, high.cumsum(0) - 1, n), at)
    dst.scatter_(0, torch.where(low, low.cumsum(0) - 1, n), at)
    src, dst = src[:n // 2], dst[:n // 2]
    to = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    to.scatter_(0, torch.where(src < 0, n, src).long(), dst)
    entry = table.long()
    valid = (entry >= 0) & (entry < n)
    table.copy_(torch.where(valid, to[torch.where(valid, entry, 0)], table))
    wide = torch.cat([refs, refs.new_zeros(1)])
    wide.scatter_(0, torch.where(src < 0, n, dst).long(), refs[src.clamp(min=0).long()])
    wide.scatter_(0, torch.where(src < 0, n, src).long(), torch.zeros_like(src))
    refs.copy_(wide[:n])
    return src, dst, count.to(torch.int32).view(1)


def _run_sample(st):
    x = st["logits"].double()
    B, V = x.shape
    order, index = torch.sort(x, dim=1, descending=True, stable=True)
    t = st["temperature"].double()[:, None]
    greedy = ~(t > 0)
    w = ((order - order[:, :1]) / torch.where(greedy, 1.0, t)).exp()
    keep = torch.ones_like(w, dtype=torch.bool)
    rank = torch.arange(V, device=DEV)
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        keep &= (rank < k) | (k <= 0)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        upto = torch.where(keep, w, 0.0).cumsum(1)
        # those before which the sum has not reached its share yet
        keep &= ((upto - w) < p * upto[:, -1:]) | (p >= 1)
        keep[:, 0] = True
    if st["min_p"] is not None:
        keep &= w >= st["min_p"].double()[:, None]
    w = torch.zeros_like(w).scatter_(1, index, torch.where(keep, w, 0.0))
    upto = w.cumsum(1)
    token = (upto <= st["u"].double()[:, None] * upto[:, -1:]).sum(1).clamp(max=V - 1)
    return torch.where(greedy[:, 0], index[:, 0], token).to(torch.int32)


# --------------------------------------------------- the library's calls ----

def _own_attend(st):
    import paper_2404_00456_amd as quarot
    case = st["case"]
    return quarot.quarot_kv_paged_attention_scored(
        st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], st["cu"],
        group=case["group"], window=case["window"], n_sinks=case["sinks"],
        max_seq_len=st["max_len"], cap=case["cap"], slopes=st["slopes"], begin=st["begin"],
        end=st["end"])


def _own_sample(st):
    import paper_2404_00456_amd as quarot
    return quarot.quarot_sample(st["logits"], st["u"], temperature=st["temperature"],
                                top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])


def _pages(st):
    """What a pass over the pages leaves: the pools as they are stored (codes are
    whole numbers here, which move and stand for nothing else)."""
    return [st["table"], st["lens"], st["refs"], *st["k_cache"], *st["v_cache"]]


def _run_grow(st):
    st["meta"].copy_(st["meta0"])  # as a scheduler's own copy has it
    fork = st["case"]["fork"] != "none"
    if own:
        import paper_2404_00456_amd as quarot
        if fork:
            quarot.quarot_kv_pages_fork(st["table"], st["lens"], st["refs"], st["parent"])
        cu, src, dst, missing = quarot.quarot_kv_pages_reserve(
            st["table"], st["lens"], st["refs"], st["new"], st["case"]["page"])
        quarot.quarot_kv_pages_copy(st["k_cache"], st["v_cache"], src, dst)
    else:
        if fork:
            _fork(st)
        cu, src, dst, missing = _reserve(st)
        _copy_pages(st, src, dst)
    return _pages(st) + [cu, src, dst, missing]


def _run_compact(st):
    st["meta"].copy_(st["meta0"])
    if own:
        import paper_2404_00456_amd as quarot
        quarot.quarot_kv_pages_fork(st["table"], st["lens"], st["refs"], st["parent"])
        src, dst, live = quarot.quarot_kv_pages_compact(st["table"], st["refs"])
        quarot.quarot_kv_pages_copy(st["k_cache"], st["v_cache"], src, dst)
    else:
        _fork(st)
        src, dst, live = _squeeze(st)
        _copy_pages(st, src, dst)
    return _pages(st) + [src, dst, live]


def run(st):
    op = st["case"]["op"]
    if op == "grow":
        return _run_grow(st)
    if op == "compact":
        return _run_compact(st)
    if op == "attend":
        return _own_attend(st) if own else _run_attend(st)
    return _own_sample(st) if own else _run_sample(st)


# ------------------------------------------------------------------ work ----

def _page_bytes(case):
    rows = case["kv_heads"] * case["page"]
    return 2 * rows * (case["dim"] // 2 + 4 * (case["dim"] // case["group"]))


def _pages_of(x, page):
    return (x + page - 1) // page


def work(case):
    if case["op"] == "sample":
        size = 2 if case["dtype"] == "float16" else 4
        # a comparison, and where it counts a weight and its sum, of each logit
        return {"bytes": case["batch"] * (case["vocab"] * size + 24),
                "flops": 4 * case["batch"] * case["vocab"]}
    if case["op"] == "grow":
        page = case["page"]
        shared, length, new, parent = _grow_lengths(case)
        # entries read, and written where they change; pages that several go on from
        entries = 2 * sum(_pages_of(x, page) for x in length) if case["fork"] != "none" else 0
        followers, whole = {}, 0
        for b, p in enumerate(parent):
            followers[p] = followers.get(p, 0) + 1
        for p, k in followers.items():
            whole += (k - 1) if length[p] % page else 0
        grown = sum(_pages_of(length[p] + n, page) - _pages_of(length[p], page)
                    for p, n in zip(parent, new))
        return {"bytes": 2 * whole * _page_bytes(case) + 4 * (entries + 2 * grown + 6 * len(new)),
                "flops": len(new)}
    if case["op"] == "compact":
        length, parent = _compact_lengths(case)
        each = [_pages_of(x, case["page"]) for x in length]
        n = sum(each) + len(each)
        live = sum(x for x, p in zip(each, parent) if p >= 0)
        moved = live * (n - live) / n  # of pages dealt out at random
        return {"bytes": 2 * moved * _page_bytes(case) + 4 * (2 * sum(each) + 2 * n), "flops": n}
    n, length = _lengths(case)
    D, G, Hkv, H = case["dim"], case["group"], case["kv_heads"], case["heads"]
    begin, end = _spans(case)
    pairs = seen = row = 0
    for x, total in zip(n, length):
        p = np.arange(total - x, total, dtype=np.int64)
        low, high = begin[row:row + x].astype(np.int64), end[row:row + x].astype(np.int64)
        if case["window"]:
            low = np.maximum(low, p + 1 - case["window"])
        low = np.minimum(np.maximum(low, 0), high)
        pairs += int((high - low + np.minimum(low, case["sinks"])).sum())
        first = int(low.min())
        seen += int(high.max()) - first + min(first, case["sinks"])
        row += x
    packed = D // 2 + 4 * (D // G)  # bytes of a cached row
    return {"bytes": 2 * seen * Hkv * packed + 4 * sum(n) * H * D, "flops": 4 * D * H * pairs}


# ----------------------------------------------------------------- exact ----

def _exact_values(cache, group):
    codes, scale, zero = cache
    x = torch.empty((*codes.shape[:-1], codes.shape[-1] * 2), dtype=torch.float64, device=DEV)
    x[..., 0::2], x[..., 1::2] = (codes % 16).double(), (codes // 16).double()
    x *= scale.double().repeat_interleave(group, -1)
    return x + zero.double().repeat_interleave(group, -1)


def _exact_attend(case, st):
    page, D, rep = case["page"], case["dim"], case["heads"] // case["kv_heads"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    begin, end = (torch.tensor(x, device=DEV) for x in _spans(case))
    row = 0
    for b, (n, total) in enumerate(zip(st["n"], st["length"])):
        pages = st["table"][b, :_pages_of(total, page)].long()
        t = torch.arange(total, device=DEV)[None]
        for h in range(case["kv_heads"]):
            k, v = (_exact_values(tuple(c[pages, h] for c in cache), case["group"])
                    .reshape(-1, D)[:total] for cache in (st["k_cache"], st["v_cache"]))
            for at in range(0, n, 1024):  # so many queries at a time
                m = min(1024, n - at)
                q = st["q"][row + at:row + at + m, h * rep:(h + 1) * rep].double()
                s = torch.matmul(q.reshape(m * rep, -1), k.T).view(m, rep, -1) / math.sqrt(D)
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                p = torch.arange(total - n + at, total - n + at + m, device=DEV)[:, None]
                if st["slopes"] is not None:
                    slope = st["slopes"][h * rep:(h + 1) * rep].double()
                    s -= slope[None, :, None] * (p - t).abs()[:, None]
                see = t >= begin[row + at:row + at + m, None]
                if case["window"]:
                    see &= p - t < case["window"]
                see |= t < case["sinks"]
                see &= t < end[row + at:row + at + m, None]
                s = s.masked_fill(~see[:, None], -math.inf).softmax(-1)
                out[row + at:row + at + m, h * rep:(h + 1) * rep] = \
                    torch.matmul(s.view(m * rep, -1), v).view(m, rep, -1)
        row += n
    return out


class _Book:
    """Tables and references by lists and loops."""

    def __init__(self, st):
        self.table = st["table"].tolist()
        self.lens, self.refs = st["lens"].tolist(), st["refs"].tolist()

    def fork(self, parent):
        old, lens = [list(r) for r in self.table], list(self.lens)
        for b, p in enumerate(parent):
            for e in old[b]:
                if e >= 0:
                    self.refs[e] -= 1
            self.table[b] = list(old[p]) if p >= 0 else [-1] * len(old[b])
            self.lens[b] = lens[p] if p >= 0 else 0
            for e in self.table[b]:
                if e >= 0:
                    self.refs[e] += 1

    def reserve(self, new, page):
        free = [i for i, r in enumerate(self.refs) if r == 0]
        start = list(self.refs)
        users = {}
        for b, n in enumerate(new):  # who writes on a page that holds older tokens
            if n > 0 and self.lens[b] % page:
                users.setdefault(self.table[b][self.lens[b] // page], []).append(b)
        src, dst, cu, used = [-1] * len(new), [-1] * len(new), [0], 0
        for b, n in enumerate(new):
            x = self.lens[b]
            for j in range(x // page, _pages_of(x + n, page)):
                e = self.table[b][j]
                if e >= 0 and start[e] == 1:
                    continue
                if e >= 0 and j * page < x and len(users[e]) == start[e] and users[e][0] == b:
                    continue
                y = free[used]
                used += 1
                self.table[b][j] = y
                self.refs[y] += 1
                if e >= 0:
                    self.refs[e] -= 1
                    if j * page < x:
                        src[b], dst[b] = e, y
            self.lens[b] = x + n
            cu.append(cu[-1] + n)
        return cu, src, dst

    def compact(self):
        n, live = len(self.refs), sum(r > 0 for r in self.refs)
        src = [i for i in range(live, n) if self.refs[i] > 0]
        dst = [i for i in range(live) if self.refs[i] == 0]
        to = dict(zip(src, dst))
        self.table = [[to.get(e, e) for e in r] for r in self.table]
        for s, d in to.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
        pad = [-1] * (n // 2 - len(src))
        return src + pad, dst + pad, live


def _exact_pages(case, st):
    book = _Book(st)
    if case["op"] == "grow":
        if case["fork"] != "none":
            book.fork(st["parent"].tolist())
        cu, src, dst = book.reserve(st["new"].tolist(), case["page"])
        tail = [_int32(cu), _int32(src), _int32(dst), _int32([0])]
    else:
        book.fork(st["parent"].tolist())
        src, dst, live = book.compact()
        tail = [_int32(src), _int32(dst), _int32([live])]
    pools = []
    for x in (*st["k_cache"], *st["v_cache"]):
        y = x.clone()
        for s, d in zip(src, dst):
            if s >= 0:
                y[d] = x[s]
        pools.append(y.double() if y.is_floating_point() else y)
    return [_int32(book.table), _int32(book.lens), _int32(book.refs), *pools, *tail]


def _exact_sample(st):
    logits = st["logits"].double().cpu().numpy()
    t, u = st["temperature"].double().tolist(), st["u"].double().tolist()

    def limit(name, off):
        return st[name].tolist() if st[name] is not None else [off] * len(t)

    limits = zip(limit("top_k", 0), limit("top_p", 1.0), limit("min_p", 0.0))
    out = []
    for x, tt, uu, (k, p, mp) in zip(logits, t, u, limits):
        best = int(np.argmax(x))
        if not tt > 0:
            out.append(best)
            continue
        order = np.argsort(-x, kind="stable")
        order = order[:k] if k > 0 else order
        w = np.exp((x[order] - x[best]) / tt)
        if p < 1:
            upto = np.cumsum(w)
            order = order[:max(1, int(np.searchsorted(upto, p * upto[-1])) + 1)]
            w = w[:len(order)]
        order = np.sort(order[w >= mp])
        upto = np.cumsum(np.exp((x[order] - x[best]) / tt))
        i = int(np.searchsorted(upto, uu * upto[-1], side="right"))
        out.append(int(order[min(i, len(order) - 1)]))
    return _int32(out)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(case, st)
    return _exact_sample(st) if case["op"] == "sample" else _exact_pages(case, st)
