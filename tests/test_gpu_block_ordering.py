"""Block caches: results that cross thread blocks or launches are the newest ones.  Neither property can be provoked to fail from
outside; the tests run the paths with data that changes from call to call, so that anything left from before would show."""
import pytest
import torch

from block_reference import BlockState
from helpers import gpu_context

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_context()
    yield c
    assert c.poll_status()[0] == 0
    c.close()


def test_parts_of_shared_items_are_this_calls(ctx):
    """Two items that all CTAs share, two caches and two queries in turn: every merge reads parts that the call before filled with
    something else."""
    states = [BlockState(1, 2, 8, 1, 128, 32, 300, 9000 + 13 * i, False, seed=40 + i) for i in range(2)]
    caches = [s.device_cache(with_range=False) for s in states]
    g = torch.Generator().manual_seed(5)
    q = [torch.randn((1, 2, 8, 128), generator=g).to(torch.bfloat16) for _ in range(2)]
    qd = [x.cuda() for x in q]
    want = [s.attend(0, x, [0.1]) for s, x in zip(states, q)]
    first = None
    for turn in range(50):
        outs = [torch.empty_like(x) for x in qd]
        for i in range(2):
            ctx.block_attend(caches[i], 0, 1, qd[i], [0.1], outs[i])
        if first is None:
            first = outs
            for o, (w, _, bound, _) in zip(outs, want):
                assert bool(((o.cpu().double() - w).abs() <= bound).all())
        assert all(torch.equal(a, b) for a, b in zip(outs, first)), turn


def test_selection_sees_the_append_before_it(ctx):
    """Appends that fill blocks and selections one right after the other, no synchronisation between them: the newest blocks are
    scored with the ranges and scales that the append has just written."""
    from block_reference import starts
    T, B = 16, 4
    st = BlockState(1, B, 8, 2, 128, T, 64, 16 * 20, False, seed=50)
    cache = st.device_cache()
    g = torch.Generator().manual_seed(6)
    n, calls = 32, 20
    rows = [[(torch.randn((1, B * n, 2, 128), generator=g) * (1 + i)).to(torch.bfloat16) for _ in range(2)] for i in range(calls)]
    q = torch.randn((1, B, 8, 128), generator=g).to(torch.bfloat16)
    dev = [[x.cuda() for x in r] for r in rows]
    qd, start = q.cuda(), starts([n] * B)
    sd = start.cuda()
    got = torch.empty((calls, 1, B, 2, 7), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    for i in range(calls):
        ctx.block_append(cache, 0, 1, sd, n, *dev[i])
        ctx.block_select(cache, 0, 1, qd, 1, 0, got[i])
    for i in range(calls):
        st.append(0, start, *rows[i])
        assert torch.equal(got[i].cpu(), st.select(0, q, 7, 1, 0)), i
