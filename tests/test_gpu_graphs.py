"""Decode calls and prune rounds captured into CUDA graphs: what a graph was given stays valid whatever the context is used for
between capture and replay.  A replay has to give the same bits as the eager call."""
import pytest
import torch

from helpers import gpu_context, random_cache, to_device

pytestmark = pytest.mark.gpu

HQ, HKV, D, CAP = 16, 8, 64, 96
SCALE, GAMMA = 0.11, 0.97


def cache(L, B, seed, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(20, CAP - 8, (L, B, HKV), generator=g)
    return to_device(random_cache(L, B, HQ, HKV, D, CAP, lens, dtype=dtype, seed=seed, rel_init="rand"))


def prune(ctx, gc, keep):
    L, B = gc.len.shape[:2]
    ctx.rasr_prune(gc, torch.full((L, B), keep, dtype=torch.int32, device="cuda"), 4, 2)


def step_inputs(gc, seed):
    L, B = gc.len.shape[:2]
    g = torch.Generator().manual_seed(seed)
    rn = lambda h: torch.randn((L, B, h, D), generator=g).to(torch.bfloat16).cuda()  # noqa: E731
    return rn(HQ), rn(HKV), rn(HKV), torch.full((B,), 500, dtype=torch.int32, device="cuda")


def decode(ctx, gc, x, out):
    L = gc.len.shape[0]
    ctx.decode_attend(gc, 0, L, *x, [SCALE] * L, GAMMA, out)


def state(gc):
    return [t.clone() for t in (gc.k, gc.v, gc.rel, gc.pos, gc.len)]


def restore(gc, s):
    for t, old in zip((gc.k, gc.v, gc.rel, gc.pos, gc.len), s):
        t.copy_(old)


def same_state(gc, s):
    live = torch.arange(CAP, device="cuda") < gc.len[..., None]
    return torch.equal(gc.len, s[4]) and torch.equal(gc.rel[live], s[2][live]) and torch.equal(gc.pos[live], s[3][live]) and \
        torch.equal(gc.k[live], s[0][live]) and torch.equal(gc.v[live], s[1][live])


def test_captured_decode_outlives_prunes_of_other_caches():
    """The order of the items that a prune round leaves for the decode calls: other caches with more, fewer and as many items are
    pruned between capture and replay."""
    own = gpu_context()
    a = cache(10, 4, seed=1)                                         # 320 items: enough for the queue of the persistent kernels
    prune(own, a, 40)
    begin, x = state(a), step_inputs(a, 2)
    out = torch.zeros_like(x[0])
    decode(own, a, x, out)
    want, end = out.clone(), state(a)
    restore(a, begin)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode(own, a, x, out)
    others = [cache(20, 4, seed=3), cache(37, 1, seed=4), cache(5, 8, seed=5)]  # 640, 296, 320 items
    for c in others:
        prune(own, c, 30)
    filler = torch.full((16 << 20,), 255, dtype=torch.uint8, device="cuda")     # what a freed buffer could have become
    for _ in range(2):
        restore(a, begin)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert own.poll_status()[0] == 0
        assert torch.equal(out, want) and same_state(a, end)
    assert bool((filler == 255).all())
    del graph
    own.close()


@pytest.mark.parametrize("known", [False, True])
def test_captured_prune_round(known):
    """A prune round captured before any other of that number of items, or after one of another cache; eager decode calls of both
    caches before and after the replay."""
    own, plain = gpu_context(), gpu_context()
    a, b = cache(10, 4, seed=6), cache(5, 8, seed=7)                 # 320 items each
    x, y = step_inputs(a, 8), step_inputs(b, 9)
    if known:
        prune(own, b, 50)
    begin_a, begin_b = state(a), state(b)

    def both(ctx, c, s, inputs):
        restore(c, s)
        out = torch.zeros_like(inputs[0])
        decode(ctx, c, inputs, out)
        end = state(c)
        restore(c, s)
        return out, end

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        prune(own, a, 40)
    assert torch.equal(a.len, begin_a[4])
    for c, s, inputs in ((a, begin_a, x), (b, begin_b, y)):          # nothing has run yet
        got, want = both(own, c, s, inputs), both(plain, c, s, inputs)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1][2].nan_to_num(), want[1][2].nan_to_num())
    graph.replay()
    pruned = state(a)
    restore(a, begin_a)
    prune(plain, a, 40)
    assert same_state(a, pruned)
    for c, s, inputs in ((a, pruned, x), (b, begin_b, y)):
        got, want = both(own, c, s, inputs), both(plain, c, s, inputs)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1][2].nan_to_num(), want[1][2].nan_to_num())
    assert own.poll_status()[0] == 0 and plain.poll_status()[0] == 0
    del graph
    own.close()
    plain.close()
