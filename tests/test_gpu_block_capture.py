"""Block-cache calls that are captured before any other call of their context has been made: the scratch hint has to be enough."""
import pytest
import torch

from block_reference import BlockState
from helpers import gpu_context

pytestmark = pytest.mark.gpu


def test_first_calls_are_captured():
    from paper_2511_06029_b200 import binding
    gpu_context().close()                            # the library is built
    st = BlockState(2, 3, 8, 2, 128, 32, 20, 32 * 17 + 5, True, seed=1)
    g = torch.Generator().manual_seed(1)
    q = torch.randn((2, 3, 8, 128), generator=g).to(torch.bfloat16)
    cache, qd = st.device_cache(), q.cuda()
    sel, out = torch.empty((2, 3, 2, 5), dtype=torch.int32, device="cuda"), torch.empty_like(qd)
    ctx = binding.Context(0, scratch_bytes_hint=4 << 20)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx.block_select(cache, 0, 2, qd, 1, 1, sel)
        ctx.block_attend(cache, 0, 2, qd, [0.1, 0.08], out, selected=sel)
    for _ in range(3):
        sel.fill_(-9)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(sel.cpu(), st.select(0, q, 5, 1, 1))
        want, _, bound, _ = st.attend(0, q, [0.1, 0.08], sel.cpu())
        assert bool(((out.cpu().double() - want).abs() <= bound).all())
    assert ctx.poll_status()[0] == 0
    del graph
    ctx.close()


def test_without_a_hint_the_capture_is_refused():
    from paper_2511_06029_b200 import binding
    st = BlockState(1, 1, 4, 1, 64, 16, 4, 50, False, seed=2)
    cache = st.device_cache()
    q = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    ctx = binding.Context(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(binding.LetheError) as e:
            ctx.block_attend(cache, 0, 1, q, [0.1], out)
        q.add_(0)
    assert e.value.status == binding.ERR_UNSUPPORTED
    ctx.block_attend(cache, 0, 1, q, [0.1], out)
    assert ctx.poll_status()[0] == 0
    del graph
    ctx.close()
