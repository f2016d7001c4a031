"""Paths of the appends and of the block attention that calls of real sizes take and small ones do not: two KV heads to a block of
threads, every head dimension and block size with a rotation, many rows to a token, the line of more items than the table holds with
lists and large blocks."""
import pytest
import torch

import chunk_reference as ref
from block_reference import BlockState, starts
from helpers import gpu_context
from test_gpu_append import angles, expected, off_by, raw, rotated, rows, same, state_and_cache

pytestmark = pytest.mark.gpu
E4M3, BF16 = torch.float8_e4m3fn, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = gpu_context()
    yield c
    assert c.poll_status()[0] == 0
    c.close()


def rotary(rot, axes, n, pairs, seed=0):
    from paper_2511_06029_b200 import binding
    torch.manual_seed(seed)
    axis, freq, pos = angles(rot, axes, n)
    return binding.Rotary(axis, freq, pos.cuda(), style=binding.ROT_PAIRS if pairs else binding.ROT_HALVES), (axis, freq, pos)


def block_rows(st, nl, n, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((nl, n, h, st.D), generator=g).to(BF16) for h in (st.Hq, st.Hkv, st.Hkv)]


def same_blocks(st, cache):
    assert torch.equal(cache.len.cpu(), st.len)
    kept = torch.arange(st.capacity) < (st.len // st.T)[..., None]
    for name in ("k", "v", "k_scale", "v_scale", "k_range"):
        assert torch.equal(st.back(getattr(cache, name))[kept], getattr(st, name)[kept]), name
    for name in ("k_open", "v_open"):
        assert torch.equal(getattr(cache, name).cpu().view(torch.int16), getattr(st, name).view(torch.int16)), name


def block_append_and_compare(ctx, st, chunks, rot, pairs, axes, with_q=True, seed=0):
    """The rotated append against the plain statement on keys that lethe_append rotated (itself compared with the definition), bit for
    bit, and the keys that stay open against the definition."""
    L, n = st.L, sum(chunks)
    cache = st.device_cache()
    q, k, v = block_rows(st, L, n, seed)
    r, how = rotary(rot, axes, n, pairs, seed)
    kr = rotated(ctx, r, k.cuda()).cpu()
    want, size = ref.rotate(k, *how, pairs, False)
    assert bool(((kr.double() - want).abs() <= off_by(want, size, BF16)).all())
    q_out = torch.empty_like(q, device="cuda") if with_q else None
    ctx.block_append(cache, 0, L, starts(chunks).cuda(), max(chunks), k.cuda(), v.cuda(), rotary=r, q=q.cuda() if with_q else None, q_out=q_out)
    st.append(0, starts(chunks), kr, v)
    same_blocks(st, cache)
    if with_q:
        assert torch.equal(q_out, rotated(ctx, r, q.cuda()))


# rot_dim: the whole row; whole pieces of 16 elements; not whole pieces
@pytest.mark.parametrize("D,T", [(64, 16), (64, 32), (64, 64), (64, 128), (128, 16), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("rot,pairs,axes", [(64, False, 1), (32, True, 3), (50, False, 2), (6, True, 1)])
def test_rotation_at_every_block_size(ctx, D, T, rot, pairs, axes):
    rot = rot * D // 64
    lens = [[[T - 1, 2 * T - 1], [3, 3], [T + 5, 0]]] * 2
    for i, chunks in enumerate(([1, 1, 1], [2, 4, 3], [T + 3, 1, 2 * T], [5 * T, 7, T])):
        st = BlockState(2, 3, 6, 2, D, T, 12, lens, True, seed=T + i)
        block_append_and_compare(ctx, st, chunks, rot, pairs, axes, with_q=i % 2 == 0, seed=i)
    assert ctx.poll_status()[0] == 0


@pytest.mark.parametrize("D,T,L,Hkv,chunks", [(64, 16, 1, 8, [1300, 1101]), (64, 16, 1, 7, [2900]), (128, 16, 3, 3, [700, 1500, 9]), (128, 32, 5, 4, [1990]), (64, 64, 8, 5, [2001]),
                                              (128, 64, 8, 4, [1200, 1300]), (64, 128, 10, 8, [1800])])
@pytest.mark.parametrize("rot,pairs", [(64, False), (50, False), (0, False)])
@pytest.mark.parametrize("uneven", [False, True])
def test_two_heads_to_a_block_of_threads(ctx, D, T, L, Hkv, chunks, rot, pairs, uneven):
    """1184 blocks to fill and more.  Heads of equal length share the cosines and sines of their tokens, heads of unequal length and a last
    one without a partner do not; one head has no room, and rows are left for the open block."""
    from paper_2511_06029_b200 import binding
    B, n = len(chunks), sum(chunks)
    assert L * Hkv * (n // T + B) >= 1184
    g = torch.Generator().manual_seed(T)
    lens = torch.randint(0, 2 * T, (L, B, 1), generator=g).expand(L, B, Hkv).clone()
    capacity = max(chunks) // T + 3
    if uneven:
        lens = torch.randint(0, 2 * T, (L, B, Hkv), generator=g)
        lens[:, 0, Hkv - 2] = lens[:, 0, Hkv - 1]
        lens[L - 1, 0, 1] = capacity * T - 5            # no room
    st = BlockState(L, B, Hkv, Hkv, D, T, capacity, lens, uneven, seed=D)
    if rot:
        block_append_and_compare(ctx, st, chunks, rot, pairs, 2, with_q=uneven, seed=T)
    else:
        cache = st.device_cache()
        _, k, v = block_rows(st, L, n, T)
        ctx.block_append(cache, 0, L, starts(chunks).cuda(), max(chunks), k.cuda(), v.cuda())
        st.append(0, starts(chunks), k, v)
        same_blocks(st, cache)
    assert ctx.poll_status()[0] == (binding.ERR_CAPACITY if uneven else 0)


@pytest.mark.parametrize("dtype", [BF16, E4M3, torch.float32])
@pytest.mark.parametrize("L,Hq,Hkv,chunks", [(2, 32, 8, [1025]), (1, 64, 8, [1000, 1, 500]), (3, 5, 5, [1024, 3]), (5, 7, 1, [2047])])
@pytest.mark.parametrize("rot", [64, 42, 0])
def test_append_many_tokens_of_many_rows(ctx, dtype, L, Hq, Hkv, chunks, rot):
    """1024 tokens and more (two to a block of threads), more rows to a token than a block takes, an odd token left over."""
    n, B = sum(chunks), len(chunks)
    st, cache = state_and_cache(L, B, Hq, Hkv, 64, -(-(max(chunks) + 9) // 16) * 16, 7, dtype, 16, seed=n)
    q, k, v = rows(L, n, Hq, Hkv, 64, dtype, seed=n)
    pos = torch.arange(n, dtype=torch.int32)
    r, kr, q_out = None, k, None
    if rot:
        r, how = rotary(rot, 3, n, False)
        kr = rotated(ctx, r, k.cuda()).cpu()
        want, size = ref.rotate(k, *how, False, False)
        assert bool(((kr.double() - want).abs() <= off_by(want, size, k.dtype)).all())
        q_out = torch.empty_like(q, device="cuda")
    start = starts(chunks)
    want = expected(st, cache, 0, start, kr, v, pos)
    ctx.append(cache, 0, L, start.cuda(), max(chunks), k.cuda(), v.cuda(), pos.cuda(), rotary=r, q=q.cuda() if rot else None, q_out=q_out)
    same(cache, want)
    if rot:
        assert torch.equal(raw(q_out), raw(rotated(ctx, r, q.cuda())))
    assert ctx.poll_status()[0] == 0


@pytest.mark.parametrize("D,T,lists", [(128, 32, False), (64, 64, True), (64, 16, True), (128, 128, True)])
def test_more_items_than_the_table_of_places(ctx, D, T, lists):
    """Beyond 2048 items a CTA keeps the places of every so many-th only: with blocks of 32 and more, and with lists."""
    g = torch.Generator().manual_seed(T)
    L, B, Hkv, n = 4, 75, 7, 3
    lens = torch.randint(0, 6 * T, (L, B, Hkv), generator=g)
    lens[1, 20:40] = 0
    st = BlockState(L, B, 2 * Hkv, Hkv, D, T, 6, lens, False, seed=T)
    q = torch.randn((L, B, 2 * Hkv, D), generator=g).to(BF16)
    scale = [0.1, 0.05, 0.125, 0.09]
    cache = st.device_cache()
    sel = None
    if lists:
        sel = torch.empty((L, B, Hkv, n), dtype=torch.int32, device="cuda")
        ctx.block_select(cache, 0, L, q.cuda(), 1, 1, sel)
        assert torch.equal(sel.cpu(), st.select(0, q, n, 1, 1))
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(q.shape[:3], device="cuda")
    ctx.block_attend(cache, 0, L, q.cuda(), scale, out, lse=lse, selected=sel)
    want, z, b_out, b_lse = st.attend(0, q, scale, None if sel is None else sel.cpu())
    assert bool(((out.cpu().double() - want).abs() <= b_out).all())
    none = torch.isinf(z)
    assert torch.equal(torch.isinf(lse.cpu()), none) and bool(((lse.cpu().double() - z)[~none].abs() <= b_lse[~none]).all())
    assert ctx.poll_status()[0] == 0


@pytest.mark.parametrize("D,T,rot,pairs", [(64, 16, 64, False), (64, 16, 50, True), (128, 32, 128, False), (128, 32, 0, False), (64, 128, 32, True), (128, 16, 42, False), (64, 64, 64, True)])
@pytest.mark.parametrize("with_q", [False, True])
def test_single_tokens_of_many_items(ctx, D, T, rot, pairs, with_q):
    """2048 items and more, one token each or none: a warp to an item.  Some items fill a block, some have no room, heads of a sequence
    differ in length; and the same of fewer items, a block of threads each, leaves the same."""
    from paper_2511_06029_b200 import binding
    g = torch.Generator().manual_seed(D + T)
    L, B, Hkv = 2, 147, 7
    lens = torch.randint(0, 2 * T, (L, B, Hkv), generator=g)
    lens[:, ::3] = lens[:, ::3, :1]
    lens[:, 5:20] = T - 1
    lens[1, 30, 2] = lens[0, 3, 0] = 2 * T
    chunks = [0 if b % 11 == 4 else 1 for b in range(B)]
    chunks[3] = chunks[30] = 1
    n = sum(chunks)
    st = BlockState(L, B, 2 * Hkv, Hkv, D, T, 2, lens, True, seed=T)
    caches = [st.device_cache() for _ in range(2)]
    q, k, v = block_rows(st, L, n, T)
    r, kr, qr = None, k, None
    if rot:
        r, _ = rotary(rot, 2, n, pairs, T)
        kr, qr = rotated(ctx, r, k.cuda()).cpu(), rotated(ctx, r, q.cuda())
    with_q = with_q and rot > 0
    start = starts(chunks).cuda()
    outs = [torch.empty_like(q, device="cuda") if with_q else None for _ in range(2)]
    ctx.block_append(caches[0], 0, L, start, 1, k.cuda(), v.cuda(), rotary=r, q=q.cuda() if with_q else None, q_out=outs[0])
    for l in range(L):
        ctx.block_append(caches[1], l, l + 1, start, 1, k[l:l + 1].cuda(), v[l:l + 1].cuda(), rotary=r, q=q[l:l + 1].cuda() if with_q else None,
                         q_out=outs[1][l:l + 1] if with_q else None)
    st.append(0, starts(chunks), kr, v)
    for c, o in zip(caches, outs):
        same_blocks(st, c)
        assert o is None or torch.equal(o, qr)
    assert ctx.poll_status()[0] == binding.ERR_CAPACITY
    # the same without a page for the blocks that are filled next
    caches[0].len[:] = T - 1
    caches[0].page_table[0, :9, :, 0] = -1
    ctx.block_append(caches[0], 0, L, start, 1, k.cuda(), v.cuda(), rotary=r)
    assert ctx.poll_status()[0] == binding.ERR_PAGE
    assert torch.equal(caches[0].len.cpu(), T - 1 + torch.tensor(chunks, dtype=torch.int32).view(1, B, 1).expand(L, B, Hkv))


@pytest.mark.parametrize("dtype", [BF16, E4M3, torch.float32])
@pytest.mark.parametrize("L,B,Hq,Hkv,rot", [(9, 40, 6, 3, 64), (20, 17, 1, 1, 0), (3, 600, 2, 1, 32), (16, 33, 5, 5, 42)])
def test_append_single_tokens_of_many_rows(ctx, dtype, L, B, Hq, Hkv, rot):
    """One token to a sequence (or none, or no room), more rows than small blocks are taken for: two tokens to a block, which sets the
    lengths; an odd number of tokens."""
    from paper_2511_06029_b200 import binding
    st, cache = state_and_cache(L, B, Hq, Hkv, 64, 16, 6, dtype, 16, seed=B)
    cache.len[L - 1, 1, 0] = 16
    chunks = [0 if b % 5 == 2 else 1 for b in range(B)]
    chunks[0] += (sum(chunks) + 1) % 2 and -1
    n = sum(chunks)
    assert n % 2
    q, k, v = rows(L, n, Hq, Hkv, 64, dtype, seed=n)
    pos = torch.arange(n, dtype=torch.int32)
    r, kr = None, k
    if rot:
        r, _ = rotary(rot, 2, n, True)
        kr = rotated(ctx, r, k.cuda()).cpu()
    start = starts(chunks)
    want = expected(st, cache, 0, start, kr, v, pos)
    q_out = torch.empty_like(q, device="cuda") if rot else None
    ctx.append(cache, 0, L, start.cuda(), 1, k.cuda(), v.cuda(), pos.cuda(), rotary=r, q=q.cuda() if rot else None, q_out=q_out)
    same(cache, want)
    if rot:
        assert torch.equal(raw(q_out), raw(rotated(ctx, r, q.cuda())))
    assert ctx.poll_status()[0] == binding.ERR_CAPACITY


def test_attend_takes_what_its_line_holds(ctx):
    """Long page tables of empty items: refused where the line of 32-token steps no longer fits 32 bits, not before.  (Nothing is read of
    the tables: all lengths are zero.)"""
    import ctypes
    from paper_2511_06029_b200 import binding
    st = BlockState(3, 2, 2, 2, 64, 128, 1, 0, True, seed=1)
    cache = st.device_cache(with_range=False)
    q = torch.ones((3, 6, 2, 64), dtype=torch.bfloat16, device="cuda")     # room for six sequences
    out = torch.ones_like(q)
    scale = (ctypes.c_float * 3)(0.1, 0.1, 0.1)
    c = binding.lethe_block_cache.from_buffer_copy(cache.c)

    def attend():
        return ctx.lib.lethe_block_attend(ctx.h, ctypes.byref(c), 0, 3, q.data_ptr(), scale, None, 0, out.data_ptr(), None, None)

    c.capacity = 2 ** 24 - 1                                   # 12 items: 12 x (2^24 x 4 + ..) < 2^30
    assert attend() == 0
    torch.cuda.synchronize()
    assert not bool(out.view(-1)[:3 * 2 * 2 * 64].any()) and ctx.poll_status()[0] == 0
    wide = torch.zeros((3, 6, 2), dtype=torch.int32, device="cuda")
    c.batch, c.len = 6, wide.data_ptr()                        # 36 items
    assert attend() == binding.ERR_UNSUPPORTED


@pytest.mark.parametrize("B,chunk", [(3, 45), (300, 1), (40, 2)])
def test_appends_without_ranges_and_in_place(ctx, B, chunk):
    """A cache from which nothing is selected has no ranges; queries rotated where they lie.  As with ranges and apart."""
    L, Hkv, D, T = 2, 4, 64, 16
    st = BlockState(L, B, 2 * Hkv, Hkv, D, T, chunk // T + 3, torch.randint(0, 2 * T, (L, B, Hkv), generator=torch.Generator().manual_seed(B)), False, seed=B)
    n = B * chunk
    q, k, v = (x.cuda() for x in block_rows(st, L, n, B))
    r, _ = rotary(64, 2, n, False, B)
    kr, qr = rotated(ctx, r, k).cpu(), rotated(ctx, r, q)
    cache = st.device_cache(with_range=False)
    ctx.block_append(cache, 0, L, starts([chunk] * B).cuda(), chunk, k, v, rotary=r, q=q, q_out=q)
    st.append(0, starts([chunk] * B), kr, v.cpu())
    cache.k_range = st.k_range.cuda()     # not the call's business
    same_blocks(st, cache)
    assert torch.equal(q, qr) and ctx.poll_status()[0] == 0
