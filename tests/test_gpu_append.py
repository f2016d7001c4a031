"""lethe_append (new rows into a cache without attending, rotated on the way) against its definition and against the calls that it
stands for."""
import ctypes

import pytest
import torch

import chunk_reference as ref
from block_reference import starts
from helpers import gpu_context

pytestmark = pytest.mark.gpu
F32, BF16, E4M3, E5M2 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def ctx():
    c = gpu_context()
    yield c
    assert c.poll_status()[0] == 0
    c.close()


def rows(L, n, Hq, Hkv, D, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    act = F32 if dtype == F32 else BF16
    return [(torch.randn((L, n, h, D), generator=g) * 3).to(act) for h in (Hq, Hkv, Hkv)]


def raw(x):
    return x.cpu().flatten().clone(memory_format=torch.contiguous_format).view(torch.uint8)


def state_and_cache(L, B, Hq, Hkv, D, cap, lens, dtype, page, seed=0):
    st = ref.State(L, B, Hq, Hkv, D, cap, lens, dtype, page=page, seed=seed, junk=5.0)
    return st, st.device_cache()


def expected(st, cache, l0, start, k, v, pos):
    """The cache after the call, by plain indexing on the CPU; returns (k, v, rel, pos, len) as the device would hold them."""
    K, V, rel, ps, ln = (x.cpu().clone() for x in (cache.k, cache.v, cache.rel, cache.pos, cache.len))
    r = st.raw
    for li in range(k.shape[0]):
        l = l0 + li
        for b in range(st.B):
            t0, t1 = int(start[b]), int(start[b + 1])
            for h in range(st.Hkv):
                n = int(ln[l, b, h])
                if n + t1 - t0 > st.cap:
                    continue
                for pool, x, sc in ((K, k, st.k_scale), (V, v, st.v_scale)):
                    y = ref.stored(x[li, t0:t1, h], st.dtype, (sc or [1.0] * st.L)[l])
                    for i in range(t1 - t0):
                        at = (int(st.table[l, b, h, (n + i) // st.page]), (n + i) % st.page) if st.page else (l, b, h, n + i)
                        pool.view(r)[at] = y.view(r)[i]
                rel[l, b, h, n:n + t1 - t0] = 0
                ps[l, b, h, n:n + t1 - t0] = pos[t0:t1]
                ln[l, b, h] = n + t1 - t0
    return K, V, rel, ps, ln


def same(cache, want):
    for x, y in zip((cache.k, cache.v, cache.rel, cache.pos, cache.len), want):
        assert torch.equal(raw(x), raw(y))


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3, E5M2])
@pytest.mark.parametrize("L,B,Hq,Hkv,D,page,lens,chunks", [
    (1, 1, 1, 1, 64, 0, 0, [1]), (3, 2, 8, 2, 128, 16, 30, [1, 1]), (2, 3, 5, 5, 64, 16, 15, [17, 0, 2]), (1, 2, 7, 1, 128, 0, 9, [40, 33]), (2, 1, 6, 3, 128, 16, 0, [1100])])
def test_append(ctx, dtype, L, B, Hq, Hkv, D, page, lens, chunks):
    cap = -(-(lens + max(chunks) + 5) // 16) * 16
    st, cache = state_and_cache(L, B, Hq, Hkv, D, cap, lens, dtype, page)
    n = sum(chunks)
    _, k, v = rows(L, n, Hq, Hkv, D, dtype, seed=n)
    pos = torch.arange(n, dtype=torch.int32) * 3 + 1
    start = starts(chunks)
    want = expected(st, cache, 0, start, k, v, pos)
    ctx.append(cache, 0, L, start.cuda(), max(chunks), k.cuda(), v.cuda(), pos.cuda())
    same(cache, want)
    assert ctx.poll_status()[0] == 0


def rotated(ctx, r, k):
    """Keys [L][n][Hkv][D] as the call rotates them: appended to an empty cache of their own type."""
    from paper_2511_06029_b200 import binding
    L, n, H, D = k.shape
    x = torch.empty((L, 1, H, n, D), dtype=k.dtype, device="cuda")
    c = binding.Cache(H, x, torch.empty_like(x), torch.zeros((L, 1, H, n), device="cuda"), torch.zeros((L, 1, H, n), dtype=torch.int32, device="cuda"),
                      torch.zeros((L, 1, H), dtype=torch.int32, device="cuda"))
    ctx.append(c, 0, L, starts([n]).cuda(), n, k.cuda(), k.cuda(), torch.zeros(n, dtype=torch.int32, device="cuda"), rotary=r)
    return x[:, 0].transpose(1, 2).contiguous()


def angles(rot, axes, n, far=10 ** 6):
    half = rot // 2
    pos = torch.randint(-far, far, (axes, n), dtype=torch.int32)
    return [p % axes for p in range(half)], [10000.0 ** (-p / half) for p in range(half)], pos


def off_by(want, size, dtype):
    """Cosines and sines are off by 2^-23 at most (and the angle by half of 2^-32 turn), one product and the sum round, then the output
    by half a step of its type."""
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    return size * (2.0 ** -23 + 2.0 ** -30 + 2 * 2.0 ** -24) + want.abs() * half + 1e-30


@pytest.mark.parametrize("rot", [0, 64, 42])
def test_single_tokens_of_many_sequences(ctx, rot):
    """More sequences than a block keeps the starts of, one token each (some none)."""
    from paper_2511_06029_b200 import binding
    B, Hkv, D = 1500, 1, 64
    st, cache = state_and_cache(1, B, 2, Hkv, D, 16, 3, BF16, 0)
    chunks = [0 if b % 7 == 3 else 1 for b in range(B)]
    n = sum(chunks)
    _, k, v = rows(1, n, 2, Hkv, D, BF16)
    pos = torch.arange(n, dtype=torch.int32)
    r, kr = None, k
    if rot:
        r = binding.Rotary([0] * (rot // 2), [0.01 * p for p in range(rot // 2)], pos[None].contiguous().cuda())
        kr = rotated(ctx, r, k)
    start = starts(chunks)
    want = expected(st, cache, 0, start, kr.cpu(), v, pos)
    ctx.append(cache, 0, 1, start.cuda(), 1, k.cuda(), v.cuda(), pos.cuda(), rotary=r)
    same(cache, want)
    assert ctx.poll_status()[0] == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,rot,pairs,axes,far", [(64, 64, False, 1, 5000), (128, 128, True, 3, 10 ** 6), (64, 32, False, 2, 2 ** 31 - 1), (128, 42, False, 4, 100),
                                                  (64, 6, True, 2, 10 ** 9), (128, 96, True, 1, 3)])
@pytest.mark.parametrize("n", [7, 1500])
def test_rotation_against_definition(ctx, dtype, D, rot, pairs, axes, far, n):
    from paper_2511_06029_b200 import binding
    q, k, v = rows(1, n, 4, 2, D, dtype, seed=rot)
    axis, freq, pos = angles(rot, axes, n, far)
    r = binding.Rotary(axis, freq, pos.cuda(), style=binding.ROT_PAIRS if pairs else binding.ROT_HALVES)
    st, cache = state_and_cache(1, 1, 4, 2, D, n + 3, 2, dtype, 0)
    q_out = torch.empty_like(q, device="cuda")
    ctx.append(cache, 0, 1, starts([n]).cuda(), n, k.cuda(), v.cuda(), pos[0].cuda(), rotary=r, q=q.cuda(), q_out=q_out)
    for x, y in ((q, q_out), (k, cache.k[:, 0, :, 2:2 + n].transpose(1, 2))):
        want, size = ref.rotate(x, axis, freq, pos, pairs, False)
        d = (y.cpu().double() - want).abs()
        assert bool((d <= off_by(want, size, dtype)).all()), f"worst {float((d / off_by(want, size, dtype)).max()):.3g}"
        assert torch.equal(y.cpu()[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", [F32, BF16, E4M3])
@pytest.mark.parametrize("rot,pairs,axes", [(64, False, 1), (64, True, 3), (32, False, 2), (42, False, 4), (6, True, 2)])
@pytest.mark.parametrize("chunks", [[1, 1], [600, 700]])
def test_rotated_on_the_way_is_rotated_before(ctx, dtype, rot, pairs, axes, chunks):
    from paper_2511_06029_b200 import binding
    L, B, Hq, Hkv, D = 2, 2, 6, 2, 64
    st, ca = state_and_cache(L, B, Hq, Hkv, D, 800, 20, dtype, 16)
    cb = st.device_cache()
    n = sum(chunks)
    q, k, v = (x.cuda() for x in rows(L, n, Hq, Hkv, D, dtype))
    axis, freq, pos = angles(rot, axes, n)
    pos = pos.cuda()
    r = binding.Rotary(axis, freq, pos, style=binding.ROT_PAIRS if pairs else binding.ROT_HALVES)
    q_out, start = torch.empty_like(q), starts(chunks).cuda()
    ctx.append(ca, 0, L, start, max(chunks), k, v, pos[0], rotary=r, q=q, q_out=q_out)
    ctx.append(cb, 0, L, start, max(chunks), rotated(ctx, r, k), v, pos[0])
    assert torch.equal(q_out, rotated(ctx, r, q))
    for name in ("k", "v", "rel", "pos", "len"):
        assert torch.equal(raw(getattr(ca, name)), raw(getattr(cb, name))), name
    cc = st.device_cache()
    keep = q.clone()
    ctx.append(cc, 0, L, start, max(chunks), k, v, pos[0], rotary=r, q=keep, q_out=keep)    # in place
    assert torch.equal(keep, q_out) and torch.equal(raw(cc.k), raw(ca.k))


def test_prompt_then_relevance(ctx):
    """What the call is there for: a prompt's keys into the cache, then lethe_prefill_seed; as with keys put there by hand."""
    L, B, Hq, Hkv, D, P = 1, 2, 8, 2, 128, 96
    st, cache = state_and_cache(L, B, Hq, Hkv, D, 128, 0, BF16, 16)
    q, k, v = (x.cuda() for x in rows(L, B * P, Hq, Hkv, D, BF16))
    pos = torch.arange(P, dtype=torch.int32).repeat(B).cuda()
    ctx.append(cache, 0, L, starts([P, P]).cuda(), P, k, v, pos)
    by_hand = st.device_cache()
    for b in range(B):
        for h in range(Hkv):
            pages = st.table[0, b, h, :P // 16].long().cuda()
            by_hand.k[pages] = k[0, b * P:(b + 1) * P, h].view(P // 16, 16, D)
    by_hand.len[:] = P
    for c in (cache, by_hand):
        ctx.prefill_seed(c, q.view(L, B, P, Hq, D), [0.09], 0.99)
    assert torch.equal(cache.rel[..., :P], by_hand.rel[..., :P]) and float(cache.rel[..., :P].min()) > 0


def test_refusals_on_the_device(ctx):
    from paper_2511_06029_b200 import binding
    st, cache = state_and_cache(1, 3, 2, 1, 64, 32, [[[30], [4], [32]]], BF16, 16)
    _, k, v = rows(1, 14, 2, 1, 64, BF16)
    pos = torch.arange(14, dtype=torch.int32)
    start = starts([3, 10, 1])
    want = expected(st, cache, 0, start, k, v, pos)
    ctx.append(cache, 0, 1, start.cuda(), 10, k.cuda(), v.cuda(), pos.cuda())
    same(cache, want)
    assert ctx.poll_status()[0] == binding.ERR_CAPACITY
    for bad in ([0, 5, 3, 9], [-1, 2, 3, 4], [0, 5, 9, 15], [0, 11, 12, 13]):
        ctx.append(cache, 0, 1, torch.tensor(bad, dtype=torch.int32, device="cuda"), 10, k.cuda(), v.cuda(), pos.cuda())
        assert ctx.poll_status()[0] == binding.ERR_INVALID_ARG
        same(cache, want)
    cache.page_table[0, 1, 0, 1] = -1
    before = cache.k.clone()
    ctx.append(cache, 0, 1, starts([0, 4, 0]).cuda(), 10, k[:, :4].contiguous().cuda(), v[:, :4].contiguous().cuda(), pos[:4].cuda())
    assert ctx.poll_status()[0] == binding.ERR_PAGE and int(cache.len[0, 1, 0]) == 18
    changed = (cache.k != before).view(-1, 64).any(1).sum()
    assert int(changed) == 2          # slots 14 and 15; the other two have no page


def test_captured_and_replayed(ctx):
    st, ca = state_and_cache(2, 2, 4, 2, 128, 64, 5, BF16, 16)
    cb = st.device_cache()
    _, k, v = (x.cuda() for x in rows(2, 4, 4, 2, 128, BF16))
    pos = torch.tensor([5, 6, 5, 6], dtype=torch.int32, device="cuda")
    start = starts([2, 2]).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.append(cb, 0, 2, start, 2, k, v, pos)
    for _ in range(9):
        k.mul_(-1.5)
        ctx.append(ca, 0, 2, start, 2, k, v, pos)
        graph.replay()
    torch.cuda.synchronize()
    for name in ("k", "v", "rel", "pos", "len"):
        assert torch.equal(raw(getattr(ca, name)), raw(getattr(cb, name))), name


def test_refusals(ctx):
    from paper_2511_06029_b200 import binding
    lib, INV = ctx.lib, binding.ERR_INVALID_ARG
    st, cache = state_and_cache(2, 1, 4, 2, 64, 32, 3, BF16, 16)
    q, k, v = (x.cuda() for x in rows(2, 2, 4, 2, 64, BF16))
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    start = starts([2]).cuda()
    r = binding.Rotary([0], [1.0], torch.zeros((1, 2), dtype=torch.int32, device="cuda"))

    def call(c=ctypes.byref(cache.c), l0=0, l1=2, s=start.data_ptr(), n=2, m=2, qq=None, kk=k.data_ptr(), vv=v.data_ptr(), p=pos.data_ptr(), rot=None, qo=None):
        return lib.lethe_append(ctx.h, c, l0, l1, s, n, m, qq, kk, vv, p, rot, qo, None)

    assert lib.lethe_append(None, ctypes.byref(cache.c), 0, 2, None, 1, 1, None, None, None, None, None, None, None) == INV
    assert call(c=None) == INV and call(l0=2) == INV and call(l1=3) == INV and call(s=None) == INV and call(n=-1) == INV and call(m=0) == INV
    assert call(kk=None) == INV and call(vv=None) == INV and call(p=None) == INV and call(kk=k.data_ptr() + 4) == INV
    assert call(qq=q.data_ptr()) == INV and call(qo=q.data_ptr()) == INV and call(qq=q.data_ptr(), qo=q.data_ptr()) == INV
    assert call(qq=q.data_ptr(), qo=q.data_ptr() + 16, rot=r.ref) == INV and call(qq=q.data_ptr(), qo=v.data_ptr(), rot=r.ref) == INV
    assert call(n=0) == 0
    torch.cuda.synchronize()
    assert int(cache.len.max()) == 3 and ctx.poll_status()[0] == 0
