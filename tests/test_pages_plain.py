"""The plain pages themselves (tests/pages_plain.py): what a server relies on."""
import random

import pytest

from pages_plain import Pages


@pytest.mark.parametrize("seed", range(6))
def test_sequences_keep_their_tokens(seed):
    """Tokens written through the tables, as the append does it, are what each sequence
    reads again, however it was forked, grown, shrunk and moved."""
    rng = random.Random(seed)
    B, page = 6, 4
    p = Pages(B, 9, 40, page)
    data = [[None] * page for _ in range(p.n)]
    said = [[] for _ in range(B)]
    for step in range(200):
        op = rng.choice(["grow", "grow", "grow", "fork", "compact"])
        if op == "fork":
            parent = [rng.choice([b, b, rng.randrange(-1, B + 1)]) for b in range(B)]
            p.fork(parent)
            said = [list(said[x]) if 0 <= x < B else [] for x in parent]
        elif op == "compact":
            src, dst, live = p.compact()
            assert not set(x for x in src if x >= 0) & set(x for x in dst if x >= 0)
            for s, d in zip(src, dst):
                if s >= 0:
                    data[d] = list(data[s])
            assert all(r > 0 for r in p.refs[:live]) and not any(p.refs[live:])
        else:
            new = [rng.choice([0, 1, 1, 3, 7, -2, -5]) for _ in range(B)]
            cu, src, dst, missing = p.reserve(new)
            if missing:
                assert not any(cu) and set(src) == {-1}
                p.fork([b if rng.random() < 0.6 else -1 for b in range(B)])
                said = [x if p.lens[b] else [] for b, x in enumerate(said)]
                continue
            for s, d in zip(src, dst):
                if s >= 0:
                    data[d] = list(data[s])
            for b, n in enumerate(new):
                said[b] = said[b][:max(0, len(said[b]) + min(n, 0))]
                for i in range(max(n, 0)):
                    t = len(said[b])
                    said[b].append((step, b, i))
                    data[p.table[b][t // page]][t % page] = said[b][-1]
        assert p.consistent()
        for b in range(B):
            assert len(said[b]) == p.lens[b]
            assert [data[p.table[b][t // page]][t % page] for t in range(p.lens[b])] == said[b]
