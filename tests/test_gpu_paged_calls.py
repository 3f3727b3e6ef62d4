"""Refusals of the rotary and paged calls that need device tensors."""
import pytest

pytestmark = pytest.mark.gpu


def test_stream_of_another_device():
    """A stream whose device is not the tensors' is refused before anything is
    allocated or launched (a stand-in for one: there may be only one device)."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2404_00456_amd as q

    class Other:
        device = torch.device("cuda", 1)
        cuda_stream = torch.cuda.current_stream().cuda_stream

    dev = torch.device("cuda:0")
    pool = [torch.zeros(2, 1, 16, 32, dtype=torch.uint8, device=dev)] + \
        [torch.zeros(2, 1, 16, 1, dtype=torch.float16, device=dev) for _ in range(2)]
    batch = [torch.tensor(x, dtype=torch.int32, device=dev) for x in ([[0]], [1], [0, 1])]
    x = torch.ones(1, 1, 64, dtype=torch.float16, device=dev)
    out = torch.full_like(x, 7.0)
    fr, pos = torch.ones(32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    for call in (lambda s: q.quarot_rope(x, pos, fr, y=out, stream=s),
                 lambda s: q.quarot_kv_append_paged(x, x, pool, pool, *batch, group=64, q=x, q_out=out,
                                                    stream=s),
                 lambda s: q.quarot_kv_paged_attention(x, pool, pool, *batch, group=64, out=out, stream=s)):
        with pytest.raises(ValueError, match="stream must be on cuda:0"):
            call(Other())
        torch.cuda.synchronize()
        assert (out == 7.0).all() and (pool[0] == 0).all()
        call(torch.cuda.Stream())
        torch.cuda.synchronize()
        out.fill_(7.0)
        for t in pool:
            t.zero_()
