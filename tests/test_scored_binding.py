"""What the binding of the scored attention says of its queries, before it looks at what has
to fit them."""
import pytest
import torch

import paper_2404_00456_amd as q


def call(x, **kw):
    pool = (torch.zeros(5, 2, 16, 64, dtype=torch.uint8),) + (torch.zeros(5, 2, 16, 1, dtype=torch.float16),) * 2
    ints = [torch.zeros(*n, dtype=torch.int32) for n in ((3, 4), (3,), (4,))]
    return q.quarot_kv_paged_attention_scored(x, pool, pool, *ints, **kw)


@pytest.mark.parametrize("kw", [{}, dict(cap=3.0), dict(slopes=torch.zeros(4)), dict(end=torch.zeros(8, dtype=torch.int32))])
def test_queries_are_looked_at_first(kw):
    for shape in ((), (8,), (8, 512), (8, 4, 128, 1)):
        with pytest.raises(ValueError, match="q must be 3-D"):
            call(torch.zeros(shape, dtype=torch.float16), **kw)
    with pytest.raises(TypeError, match="q must be torch.float16"):
        call(torch.zeros(8, 4, 128), **kw)
    for x in (None, [1.0]):
        with pytest.raises(TypeError, match="q must be a torch.Tensor"):
            call(x, **kw)
