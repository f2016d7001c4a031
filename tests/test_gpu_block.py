"""Block caches (8 bits, one scale for each block of tokens): filling, reading back, selecting blocks, attending, against plain
statements."""
import ctypes
import math

import numpy as np
import pytest
import torch

from block_reference import BlockState, quantise, starts
from helpers import gpu_context

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_context()
    yield c
    assert c.poll_status()[0] == 0
    c.close()


def new_rows(st, nl, n, seed=0, gain=1.0):
    g = torch.Generator().manual_seed(1000 + seed)
    return [(torch.randn((nl, n, h, st.D), generator=g) * gain).to(torch.bfloat16) for h in (st.Hq, st.Hkv, st.Hkv)]


def same_cache(st, cache):
    """The device's cache is the reference's, bit for bit, wherever it means something."""
    assert torch.equal(cache.len.cpu(), st.len)
    full = st.len // st.T
    kept = torch.arange(st.capacity) < full[..., None]
    for name in ("k", "v", "k_scale", "v_scale", "k_range"):
        assert torch.equal(st.back(getattr(cache, name))[kept], getattr(st, name)[kept]), name
    for name in ("k_open", "v_open"):   # all rows: those behind the last one stay as they were
        assert torch.equal(getattr(cache, name).cpu().view(torch.int16), getattr(st, name).view(torch.int16)), name


# ------------------------------------------------------------------------------------------------------------- filling

@pytest.mark.parametrize("L,B,Hq,Hkv,D,T,paged,lens,chunks", [
    (1, 1, 4, 1, 128, 32, False, 0, [1]), (2, 3, 8, 2, 128, 32, True, 31, [1, 0, 1]), (1, 2, 5, 5, 64, 16, True, 0, [16, 15]),
    (1, 2, 16, 2, 128, 64, False, 63, [1, 66]), (2, 1, 8, 1, 64, 128, True, 100, [29]), (1, 3, 7, 1, 128, 128, False, 127, [258, 1, 130]),
    (1, 4, 6, 2, 64, 32, True, 5, [200, 27, 26, 64]), (1, 1, 2, 2, 128, 16, True, 3, [1000]), (1, 2, 4, 4, 64, 64, False, 64, [63, 64])])
def test_append_without_rotation_is_exact(ctx, L, B, Hq, Hkv, D, T, paged, lens, chunks):
    cap = -(-(lens + max(chunks)) // T) + 1
    st = BlockState(L, B, Hq, Hkv, D, T, cap, lens, paged, seed=D + T)
    cache = st.device_cache()
    n = sum(chunks)
    _, k, v = new_rows(st, L, n, seed=n)
    start = starts(chunks)
    ctx.block_append(cache, 0, L, start.cuda(), max(chunks), k.cuda(), v.cuda())
    st.append(0, start, k, v)
    same_cache(st, cache)
    assert ctx.poll_status()[0] == 0


def test_append_token_by_token_is_append_at_once(ctx):
    a, b = (BlockState(2, 2, 4, 2, 128, 32, 5, 0, True, seed=3) for _ in range(2))
    ca, cb = a.device_cache(), b.device_cache()
    n = 75
    _, k, v = new_rows(a, 2, 2 * n)
    start = starts([n, n])
    ctx.block_append(ca, 0, 2, start.cuda(), n, k.cuda(), v.cuda())
    for i in range(n):
        pick = [i, n + i]
        ctx.block_append(cb, 0, 2, starts([1, 1]).cuda(), 1, k[:, pick].contiguous().cuda(), v[:, pick].contiguous().cuda())
    a.append(0, start, k, v)
    same_cache(a, ca)
    kept = torch.arange(5) < 2
    for name in ("k", "v", "k_scale", "v_scale", "k_range"):
        assert torch.equal(a.back(getattr(ca, name))[:, :, :, kept], a.back(getattr(cb, name))[:, :, :, kept]), name
    rows = torch.arange(32) < n % 32
    assert torch.equal(ca.k_open.cpu()[..., rows, :], cb.k_open.cpu()[..., rows, :]) and torch.equal(ca.len, cb.len)


def test_append_extreme_values(ctx):
    """Zeros, values below the threshold, infinities, NaN, the largest magnitudes."""
    st = BlockState(1, 1, 1, 1, 64, 16, 8, 0, seed=1)
    _, k, v = new_rows(st, 1, 96)
    k[0, :16] = 0
    k[0, 16:32] *= 2.0 ** -120
    k[0, 32, 0, :5] = torch.tensor([float("inf"), -float("inf"), float("nan"), 3.0, -0.0])
    k[0, 48:64] *= 3.3e38 / k[0, 48:64].abs().max()
    v[0, 64:80] = float("nan")
    v[0, 80:96, 0, 3] = 1e-30
    cache = st.device_cache()
    ctx.block_append(cache, 0, 1, starts([96]).cuda(), 96, k.cuda(), v.cuda())
    st.append(0, starts([96]), k, v)
    same_cache(st, cache)
    assert float(st.k_scale[0, 0, 0, 0]) == float(st.k_scale[0, 0, 0, 1]) == 0.0


@pytest.mark.parametrize("rot,pairs,axes", [(128, False, 1), (128, True, 3), (64, False, 2), (90, False, 4), (34, True, 2), (2, False, 1)])
@pytest.mark.parametrize("chunks", [[1, 1, 0], [70, 3, 33], [2, 4, 3], [500, 900, 1]])
def test_append_rotated_on_the_way_is_rotated_before(ctx, rot, pairs, axes, chunks):
    from paper_2511_06029_b200 import binding
    from test_gpu_append import angles, rotated
    lens = [[[31, 31], [40, 39], [0, 5]]] * 2       # heads of a sequence may differ in length
    a = BlockState(2, 3, 8, 2, 128, 32, 32, lens, True, seed=7)
    ca, cb, cc = (a.device_cache() for _ in range(3))
    n = sum(chunks)
    q, k, v = (x.cuda() for x in new_rows(a, 2, n, seed=rot))
    start = starts(chunks).cuda()
    axis, freq, pos = angles(rot, axes, n)
    r = binding.Rotary(axis, freq, pos.cuda(), style=binding.ROT_PAIRS if pairs else binding.ROT_HALVES)
    q_out, kr = torch.empty_like(q), rotated(ctx, r, k)
    ctx.block_append(ca, 0, 2, start, max(chunks), k, v, rotary=r, q=q, q_out=q_out)
    ctx.block_append(cb, 0, 2, start, max(chunks), kr, v)
    assert torch.equal(q_out, rotated(ctx, r, q))
    for name in ("k", "v", "k_scale", "v_scale", "k_range", "k_open", "v_open", "len"):
        x, y = getattr(ca, name), getattr(cb, name)
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), name
    a.append(0, starts(chunks), kr.cpu(), v.cpu())
    same_cache(a, ca)
    keep = q.clone()                                                       # in place
    ctx.block_append(cc, 0, 2, start, max(chunks), k, v, rotary=r, q=keep, q_out=keep)
    assert torch.equal(keep, q_out)


def test_append_layers_and_rows_outside(ctx):
    """Only the layers of the call change; packed rows before the first and behind the last sequence's are not used."""
    st = BlockState(3, 2, 4, 2, 64, 16, 4, 7, False, seed=11)
    cache = st.device_cache()
    _, k, v = new_rows(st, 1, 40)
    start = torch.tensor([5, 17, 30], dtype=torch.int32)
    q = torch.full((1, 40, 4, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    from paper_2511_06029_b200 import binding
    r = binding.Rotary([0], [0.0], torch.zeros((1, 40), dtype=torch.int32, device="cuda"))
    q_out = torch.full_like(q, 9.0)
    ctx.block_append(cache, 1, 2, start.cuda(), 13, k.cuda(), v.cuda(), rotary=r, q=q, q_out=q_out)
    st.append(1, start, k, v)
    same_cache(st, cache)
    assert bool((q_out[:, :5] == 9).all()) and bool((q_out[:, 30:] == 9).all()) and bool((q_out[:, 5:30] == 2).all())


def test_append_refusals_on_the_device(ctx):
    from paper_2511_06029_b200 import binding
    st = BlockState(1, 3, 2, 1, 64, 16, 3, [[[40], [10], [48]]], True, seed=5)
    cache = st.device_cache()
    _, k, v = new_rows(st, 1, 30)
    start = starts([9, 20, 1])                     # 40 + 9 > 48 and 48 + 1 > 48: both stay as they are
    ctx.block_append(cache, 0, 1, start.cuda(), 20, k.cuda(), v.cuda())
    st.append(0, start, k, v)
    same_cache(st, cache)
    assert ctx.poll_status() [0] == binding.ERR_CAPACITY
    for bad in ([0, 5, 3, 9], [-1, 2, 3, 4], [0, 10, 20, 31], [0, 21, 22, 23]):
        before = cache.len.clone()
        ctx.block_append(cache, 0, 1, torch.tensor(bad, dtype=torch.int32, device="cuda"), 20, k.cuda(), v.cuda())
        assert ctx.poll_status()[0] == binding.ERR_INVALID_ARG and torch.equal(before, cache.len)
    cache.page_table[0, 1, 0, 2] = st.n_pages      # sequence 1 has 30 tokens now: its third block gets no page
    ctx.block_append(cache, 0, 1, starts([0, 4, 0]).cuda(), 20, k.cuda()[:, :4].contiguous(), v.cuda()[:, :4].contiguous())
    assert ctx.poll_status()[0] == 0               # still open
    cache.page_table[0, 1, 0, 2] = -1
    ctx.block_append(cache, 0, 1, starts([0, 14, 0]).cuda(), 20, k.cuda()[:, :14].contiguous(), v.cuda()[:, :14].contiguous())
    assert ctx.poll_status()[0] == binding.ERR_PAGE and int(cache.len[0, 1, 0]) == 48


# -------------------------------------------------------------------------------------------------------- reading back

@pytest.mark.parametrize("D,T,paged", [(128, 32, True), (64, 16, False), (128, 128, False)])
def test_read(ctx, D, T, paged):
    st = BlockState(2, 3, 4, 2, D, T, 6, [[[0], [5 * T + 3], [2 * T]]] * 2, paged, seed=2)
    cache = st.device_cache()
    begin = torch.tensor([0, -2, T + 1], dtype=torch.int32)
    for li0, li1, sb in ((0, 2, begin), (1, 2, None)):
        n = 3 * T + 5
        ko = torch.full((li1 - li0, 3, 2, n, D), 7.0, dtype=torch.bfloat16, device="cuda")
        vo = torch.full_like(ko, 7.0)
        ctx.block_read(cache, li0, li1, None if sb is None else sb.cuda(), ko, vo)
        for li in range(li0, li1):
            for b in range(3):
                for h in range(2):
                    s0 = 0 if sb is None else int(sb[b])
                    for rows, got in zip(st.rows((li, b, h)), (ko, vo)):
                        want = torch.zeros((n, D), dtype=torch.float64)
                        for i in range(n):
                            if 0 <= s0 + i < len(rows):
                                want[i] = rows[s0 + i]
                        # a product rounded to fp32, then to bf16
                        assert bool(((got[li - li0, b, h].cpu().double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -24)).all())
    assert ctx.poll_status()[0] == 0


# ----------------------------------------------------------------------------------------------------------- selecting

@pytest.mark.parametrize("L,B,Hq,Hkv,D,T,paged,lens,n,sink,recent", [
    (1, 1, 4, 1, 128, 32, False, 33, 1, 0, 0), (1, 2, 8, 2, 128, 32, True, 32 * 70 + 5, 9, 1, 2), (2, 2, 16, 2, 64, 16, True, 16 * 300, 40, 0, 0),
    (1, 1, 7, 1, 128, 64, False, 64 * 20 + 63, 20, 3, 4), (1, 1, 7, 1, 128, 64, False, 64 * 20 + 63, 19, 10, 9), (1, 3, 3, 3, 64, 128, True, 128 * 5, 4, 4, 0),
    (1, 1, 8, 1, 128, 16, True, 16 * 5000 + 1, 777, 2, 2), (1, 1, 1, 1, 64, 16, False, 16 * 9000, 300, 0, 1), (1, 2, 2, 1, 128, 32, False, 0, 5, 1, 1)])
def test_select(ctx, L, B, Hq, Hkv, D, T, paged, lens, n, sink, recent):
    st = BlockState(L, B, Hq, Hkv, D, T, lens // T + 1, lens, paged, seed=n)
    cache = st.device_cache()
    q, _, _ = new_rows(st, L, B, seed=n)
    got = torch.full((L, B, Hkv, n), 99, dtype=torch.int32, device="cuda")
    for _ in range(2):   # the counters are left as they were found
        ctx.block_select(cache, 0, L, q.cuda(), sink, recent, got)
        assert torch.equal(got.cpu(), st.select(0, q, n, sink, recent))
    assert ctx.poll_status()[0] == 0


def test_select_ties_and_extremes(ctx):
    st = BlockState(1, 4, 8, 1, 128, 16, 400, 6400, seed=4)
    q, _, _ = new_rows(st, 1, 4)
    q[0, 0] = 0                                       # every score is zero
    st.k_range[0, 1] = st.k_range[0, 1, :, :1]         # two kinds of blocks
    st.k_scale[0, 1] = st.k_scale[0, 1, 0, 0]
    st.k_scale[0, 1, 0, 100:300] *= 1.5
    st.k_range[0, 2] = torch.tensor([-127, 127]).view(1, 1, 2, 1).to(torch.int8)   # the largest sums there are
    q[0, 2] = 5.0
    q[0, 3, 0, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
    st.k_scale[0, 3, 0, ::3] = 0.0
    cache = st.device_cache()
    for n, sink, recent in ((37, 0, 0), (210, 2, 3), (399, 1, 0), (5, 2, 3)):
        got = torch.empty((1, 4, 1, n), dtype=torch.int32, device="cuda")
        ctx.block_select(cache, 0, 1, q.cuda(), sink, recent, got)
        assert torch.equal(got.cpu(), st.select(0, q, n, sink, recent))
    assert ctx.poll_status()[0] == 0


# ----------------------------------------------------------------------------------------------------------- attending

def check_attend(ctx, st, cache, l0, q, scale, selected=None, with_lse=True):
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda") if with_lse else None
    ctx.block_attend(cache, l0, l0 + q.shape[0], q.cuda(), scale, out, lse=lse, selected=None if selected is None else selected.cuda())
    want, z, b_out, b_lse = st.attend(l0, q, scale, selected)
    d = (out.cpu().double() - want).abs()
    assert bool((d <= b_out).all()), f"out: {float((d / b_out.clamp(min=1e-38)).max()):.3g} of the bound"
    if with_lse:
        none = torch.isinf(z)
        assert torch.equal(torch.isinf(lse.cpu()), none) and bool((out.cpu()[none] == 0).all())
        d = (lse.cpu().double() - z)[~none].abs()
        assert bool((d <= b_lse[~none]).all()), f"lse: {float((d / b_lse[~none]).max()):.3g} of the bound"
    return out, lse


SHAPES = [  # L, B, Hq, Hkv, D, T, paged, lens
    (1, 1, 1, 1, 128, 16, False, 1), (1, 1, 8, 1, 64, 16, True, 15), (1, 1, 4, 1, 128, 16, False, 16), (1, 2, 7, 1, 128, 32, True, 33), (2, 2, 8, 2, 64, 64, False, 127),
    (1, 3, 6, 3, 128, 128, True, 128 * 3 + 127), (1, 1, 5, 1, 128, 32, False, 3000), (3, 8, 32, 8, 128, 32, True, 200), (1, 1, 8, 1, 128, 16, True, 40000),
    (1, 1, 3, 3, 64, 128, False, 20011), (2, 5, 16, 8, 64, 32, True, 700)]


@pytest.mark.parametrize("L,B,Hq,Hkv,D,T,paged,lens", SHAPES)
def test_attend(ctx, L, B, Hq, Hkv, D, T, paged, lens):
    st = BlockState(L, B, Hq, Hkv, D, T, lens // T + 1, lens, paged, seed=lens)
    q, _, _ = new_rows(st, L, B, seed=lens, gain=1.5)
    scale = [1 / math.sqrt(D) * (1 + 0.3 * i) for i in range(L)]
    cache = st.device_cache(with_range=False)
    a = check_attend(ctx, st, cache, 0, q, scale)
    b = check_attend(ctx, st, cache, 0, q, scale)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])       # bit for bit
    check_attend(ctx, st, cache, L - 1, q[:1], scale, with_lse=False)
    assert ctx.poll_status()[0] == 0


def test_attend_ragged_with_empty_items(ctx):
    g = torch.Generator().manual_seed(0)
    lens = torch.randint(0, 700, (3, 7, 2), generator=g)
    lens[0, 0] = 0
    lens[1, 3, 1] = 0
    lens[2, 6] = torch.tensor([9000, 0])
    st = BlockState(3, 7, 10, 2, 128, 32, 300, lens, True, seed=1)
    q, _, _ = new_rows(st, 3, 7)
    check_attend(ctx, st, st.device_cache(), 0, q, [0.1, 0.09, 0.2])
    st.len[:] = 0
    check_attend(ctx, st, st.device_cache(), 0, q, [0.1, 0.09, 0.2])


def test_attend_more_items_than_the_table_of_places(ctx):
    """Beyond 2048 items a CTA keeps the places of every so many-th only."""
    g = torch.Generator().manual_seed(2)
    lens = torch.randint(0, 70, (5, 60, 8), generator=g)
    st = BlockState(5, 60, 8, 8, 64, 16, 5, lens, True, seed=3)
    q, _, _ = new_rows(st, 5, 60)
    check_attend(ctx, st, st.device_cache(), 0, q, [0.1, 0.2, 0.125, 0.09, 0.3])
    assert ctx.poll_status()[0] == 0


def test_attend_queries_that_are_not_finite(ctx):
    """A head's NaN or infinity stays with that head; a zero query gives the mean of the values."""
    st = BlockState(1, 2, 8, 1, 128, 32, 8, [[[200], [9]]], False, seed=14)
    q, _, _ = new_rows(st, 1, 2)
    cache = st.device_cache()
    plain = check_attend(ctx, st, cache, 0, q, [0.1])[0]
    bad = q.clone()
    bad[0, :, 2, 5] = float("nan")
    bad[0, :, 6, 100] = -float("inf")
    bad[0, :, 3] = 0
    out = torch.empty_like(q, device="cuda")
    ctx.block_attend(cache, 0, 1, bad.cuda(), [0.1], out)
    assert bool(out[0, :, [2, 6]].isnan().all())
    keep = [0, 1, 4, 5, 7]
    assert torch.equal(out[0, :, keep], plain[0, :, keep])
    want, _, bound, _ = st.attend(0, torch.where(bad.isfinite(), bad, 0), [0.1])
    assert bool(((out[0, :, 3].cpu().double() - want[0, :, 3]).abs() <= bound[0, :, 3]).all())


@pytest.mark.parametrize("D", [64, 128])
def test_attend_wide_ranges(ctx, D):
    """Scales of blocks far apart, large and small queries, blocks of zeros, logits that rise along the cache."""
    T, lens = 16, 16 * 50 + 9
    st = BlockState(1, 6, 8, 1, D, T, 60, lens, False, seed=D)
    f = torch.arange(60).float()
    st.v_scale[0, 0, 0] *= 10.0 ** (f % 7 - 3)
    st.v_scale[0, 1, 0, :50:2] = 0.0
    st.v[0, 1, 0, ::2] = 0
    st.v_scale[0, 2, 0] *= 1e-18
    st.v_open[0, 2] = (st.v_open[0, 2].float() * 1e-18).to(torch.bfloat16)
    st.k_scale[0, 3, 0] *= 1 + f / 4          # the largest logit keeps moving
    st.k_scale[0, 4, 0] = 1e-3
    q, _, _ = new_rows(st, 1, 6)
    q[0, 4] = (q[0, 4].float() * 1e4).to(torch.bfloat16)
    q[0, 5] = (q[0, 5].float() * 1e-20).to(torch.bfloat16)
    check_attend(ctx, st, st.device_cache(), 0, q, [1 / math.sqrt(D)])


@pytest.mark.parametrize("L,B,Hq,Hkv,D,T,paged,lens,n", [
    (1, 1, 4, 1, 128, 32, True, 3205, 10), (2, 3, 8, 2, 64, 16, False, 999, 17), (1, 8, 32, 8, 128, 64, True, 6000, 16), (1, 2, 7, 1, 128, 16, True, 40, 8)])
def test_select_and_attend(ctx, L, B, Hq, Hkv, D, T, paged, lens, n):
    st = BlockState(L, B, Hq, Hkv, D, T, lens // T + 1, lens, paged, seed=lens)
    q, _, _ = new_rows(st, L, B, seed=lens)
    cache = st.device_cache()
    sel = torch.empty((L, B, Hkv, n), dtype=torch.int32, device="cuda")
    ctx.block_select(cache, 0, L, q.cuda(), 1, 2, sel)
    scale = [1 / math.sqrt(D)] * L
    check_attend(ctx, st, cache, 0, q, scale, sel.cpu())
    if lens // T <= n:   # everything is selected
        out, all_ = torch.empty_like(q, device="cuda"), torch.empty_like(q, device="cuda")
        ctx.block_attend(cache, 0, L, q.cuda(), scale, out, selected=sel)
        ctx.block_attend(cache, 0, L, q.cuda(), scale, all_)
        assert torch.equal(out, all_)


def test_attend_lists_of_the_callers_own(ctx):
    from paper_2511_06029_b200 import binding
    st = BlockState(1, 3, 4, 1, 128, 32, 20, [[[640], [100], [35]]], True, seed=8)
    q, _, _ = new_rows(st, 1, 3)
    cache = st.device_cache()
    sel = torch.tensor([[3, -1, 3, 19, -7, 0], [2, 0, -1, 1, 5, 5], [-1, -1, -1, -1, -1, -1]], dtype=torch.int32).view(1, 3, 1, 6)
    check_attend(ctx, st, cache, 0, q, [0.1], sel)        # a repeated block counts twice, entries behind the full blocks are not read
    assert ctx.poll_status()[0] == 0
    sel[0, 1, 0, 0] = 3                                   # 100 tokens: three full blocks
    check_attend(ctx, st, cache, 0, q, [0.1], sel)
    st, _ = ctx.poll_status()
    assert st == binding.ERR_INVALID_ARG


def test_bad_pages_are_left_out(ctx):
    from paper_2511_06029_b200 import binding
    st = BlockState(1, 2, 4, 1, 64, 16, 12, 190, True, seed=9)
    q, _, _ = new_rows(st, 1, 2)
    cache = st.device_cache()
    cache.page_table[0, 0, 0, 4] = -5
    cache.page_table[0, 1, 0, 2] = st.n_pages
    out = torch.empty_like(q, device="cuda")
    ctx.block_attend(cache, 0, 1, q.cuda(), [0.2], out)
    assert ctx.poll_status()[0] == binding.ERR_PAGE
    keep = torch.tensor([[b for b in range(11) if b != 4] + [-1], [b for b in range(11) if b != 2] + [-1]], dtype=torch.int32).view(1, 2, 1, 11)
    want, _, bound, _ = st.attend(0, q, [0.2], keep)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())
    sel = torch.empty((1, 2, 1, 3), dtype=torch.int32, device="cuda")
    st.k_scale[0, 0, 0, 4] = st.k_scale[0, 1, 0, 2] = 0.0     # scores as zero
    ctx.block_select(cache, 0, 1, q.cuda(), 0, 0, sel)
    assert ctx.poll_status()[0] == binding.ERR_PAGE and torch.equal(sel.cpu(), st.select(0, q, 3, 0, 0))
    ko = torch.empty((1, 2, 1, 192, 64), dtype=torch.bfloat16, device="cuda")
    vo = torch.empty_like(ko)
    ctx.block_read(cache, 0, 1, None, ko, vo)
    assert ctx.poll_status()[0] == binding.ERR_PAGE and not bool(ko[0, 0, 0, 64:80].any()) and not bool(vo[0, 1, 0, 32:48].any())
    short = torch.full((1, 2, 1, 5, 64), 3.0, dtype=torch.bfloat16, device="cuda")     # from inside the block without a page
    ctx.block_read(cache, 0, 1, torch.tensor([70, 0], dtype=torch.int32, device="cuda"), short, torch.empty_like(short))
    assert ctx.poll_status()[0] == binding.ERR_PAGE and not bool(short[0, 0].any()) and bool(short[0, 1].any())


def test_captured_and_replayed(ctx):
    """Append, select and attend of decode steps as one graph, replayed, against calls one by one."""
    from paper_2511_06029_b200 import binding
    a, b = (BlockState(2, 3, 8, 2, 128, 16, 30, [[[45], [300], [7]]] * 2, True, seed=13) for _ in range(2))
    ca, cb = a.device_cache(), b.device_cache()
    q, k, v = (x.cuda() for x in new_rows(a, 2, 3))
    start = starts([1, 1, 1]).cuda()
    pos = torch.tensor([[45, 300, 7]], dtype=torch.int32, device="cuda")
    r = binding.Rotary([0] * 64, [10000.0 ** (-p / 64) for p in range(64)], pos)
    scale = [0.09, 0.08]

    def step(cache, qr, sel, out, lse):
        ctx.block_append(cache, 0, 2, start, 1, k, v, rotary=r, q=q, q_out=qr)
        ctx.block_select(cache, 0, 2, qr, 1, 1, sel)
        ctx.block_attend(cache, 0, 2, qr, scale, out, lse=lse, selected=sel)

    def outs():
        return torch.empty_like(q), torch.empty((2, 3, 2, 6), dtype=torch.int32, device="cuda"), torch.empty_like(q), torch.empty((2, 3, 8), device="cuda")

    one, two = outs(), outs()
    step(ca, *one)       # scratch has its size
    step(cb, *two)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(cb, *two)
    for i in range(20):
        q.mul_(-1.01)
        k.add_(0.25)
        pos.add_(1)
        step(ca, *one)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(one, two):
            assert torch.equal(x, y), i
    for name in ("k", "v", "k_scale", "v_scale", "k_range", "k_open", "v_open", "len"):
        assert torch.equal(getattr(ca, name).view(torch.uint8), getattr(cb, name).view(torch.uint8)), name
    assert ctx.poll_status()[0] == 0


def test_graph_outlives_growing_scratch(ctx):
    """A graph captured before a larger call is replayed after it: the scratch and the counters it names are still its own."""
    from paper_2511_06029_b200 import binding
    own = binding.Context(0)
    small = BlockState(1, 2, 4, 1, 64, 16, 20, 300, False, seed=31)
    large = BlockState(2, 12, 16, 8, 64, 16, 40, 600, True, seed=32)
    cs, cl = small.device_cache(), large.device_cache()
    qs, ql = new_rows(small, 1, 2)[0], new_rows(large, 2, 12)[0]
    q = qs.cuda()
    sel, out = torch.empty((1, 2, 1, 5), dtype=torch.int32, device="cuda"), torch.empty_like(q)

    def step():
        own.block_select(cs, 0, 1, q, 1, 1, sel)
        own.block_attend(cs, 0, 1, q, [0.125], out, selected=sel)

    step()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        got = torch.empty((2, 12, 8, 7), dtype=torch.int32, device="cuda")
        own.block_select(cl, 0, 2, ql.cuda(), 1, 0, got)
        assert torch.equal(got.cpu(), large.select(0, ql, 7, 1, 0))
        check_attend(own, large, cl, 0, ql, [0.1, 0.2], got.cpu())
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert own.poll_status()[0] == 0
    del graph
    own.close()


def test_other_stream_and_read_into_a_chunk(ctx):
    """A run of the operators on a side stream: a prompt is appended, read back as a contiguous cache, and drafted tokens attend over
    that with lethe_chunk_attend; single tokens attend over the block cache itself."""
    from paper_2511_06029_b200 import binding
    st = BlockState(1, 2, 8, 2, 128, 32, 8, 0, True, seed=21)
    cache = st.device_cache()
    q, k, v = new_rows(st, 1, 330)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        start = starts([130, 200]).cuda()
        kc, vc = k.cuda(), v.cuda()
        ctx.block_append(cache, 0, 1, start, 200, kc, vc)
        st.append(0, starts([130, 200]), k, v)
        ko = torch.empty((1, 2, 2, 208, 128), dtype=torch.bfloat16, device="cuda")
        vo = torch.empty_like(ko)
        ctx.block_read(cache, 0, 1, None, ko, vo)
        plain = binding.Cache(8, ko, vo, torch.zeros((1, 2, 2, 208), device="cuda"), torch.zeros((1, 2, 2, 208), dtype=torch.int32, device="cuda"), cache.len.clone())
        qs = q[:, :4].contiguous().cuda()
        out4, out1 = torch.empty_like(qs), torch.empty_like(qs[:, ::2].contiguous())
        ctx.chunk_attend(plain, 0, 1, starts([2, 2]).cuda(), 2, qs, None, None, None, [0.08], 0.99, out4)
        ctx.block_attend(cache, 0, 1, qs[:, ::2].contiguous(), [0.08], out1)
    side.synchronize()
    want, _, bound, _ = st.attend(0, q[:, :4:2], [0.08])
    assert bool(((out1.cpu().double() - want).abs() <= bound).all())
    # the chunk kernel on the rows that came back: probabilities in bf16 (half a step, 2^-8), logits summed in fp32 over D products
    qd = q[0, :4].double().view(4, 2, 4, 128)
    for i in range(4):
        b, n = i // 2, (130, 200)[i // 2]
        for h in range(2):
            K, V = ko[0, b, h, :n].cpu().double(), vo[0, b, h, :n].cpu().double()
            e = qd[i, h] @ K.T * float(np.float32(0.08))
            p = torch.softmax(e, 1)
            err = float((qd[i, h].abs() @ K.abs().T).max()) * 0.08 * (128 + 8) * 2.0 ** -23
            room = (p @ V.abs()) * (2.0 ** -8 + 2 * err + 2.0 ** -18) + (p @ V).abs() * 2.0 ** -8
            assert bool(((out4[0, i, 4 * h:4 * h + 4].cpu().double() - p @ V).abs() <= room).all())
    assert ctx.poll_status()[0] == 0


def test_waits_that_run_out(ctx):
    """With a limit of one look not all tiles of a cache far larger than L2 can be there in time: an error status, no hang, and the
    next call is right."""
    from paper_2511_06029_b200 import binding
    lead = (1, 8, 2, 2048)
    codes = [torch.randint(-127, 128, lead + (32, 128), dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.full(lead, 0.02, device="cuda") for _ in range(2)]
    still = torch.zeros((1, 8, 2, 32, 128), dtype=torch.bfloat16, device="cuda")
    large = binding.BlockCache(8, *codes, *scales, None, still, still, torch.full((1, 8, 2), 65536, dtype=torch.int32, device="cuda"))
    q = torch.randn((1, 8, 8, 128), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    ctx.set_wait_limit(1)
    ctx.block_attend(large, 0, 1, q, [0.1], out)
    status, _ = ctx.poll_status()
    ctx.set_wait_limit(0)
    assert status == binding.ERR_TIMEOUT
    first = out.clone()
    ctx.block_attend(large, 0, 1, q, [0.1], out)
    ctx.block_attend(large, 0, 1, q, [0.1], first)
    assert ctx.poll_status()[0] == 0 and torch.equal(out, first)
    st = BlockState(1, 4, 8, 2, 128, 32, 60, 1900, True, seed=6)
    q, _, _ = new_rows(st, 1, 4)
    check_attend(ctx, st, st.device_cache(), 0, q, [0.1])
    assert ctx.poll_status()[0] == 0


def test_refusals(ctx):
    from paper_2511_06029_b200 import binding
    lib, INV, UNS = ctx.lib, binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    st = BlockState(2, 1, 4, 2, 64, 16, 4, 20, True, seed=1)
    cache = st.device_cache()
    q, k, v = (x.cuda() for x in new_rows(st, 2, 2))
    start = starts([2]).cuda()
    scale = (ctypes.c_float * 2)(0.1, 0.1)
    qd = q[:, :1].contiguous()
    out, sel = torch.empty_like(qd), torch.empty((2, 1, 2, 3), dtype=torch.int32, device="cuda")

    def changed(**kw):
        c = binding.lethe_block_cache.from_buffer_copy(cache.c)
        for name, x in kw.items():
            setattr(c, name, x)
        return ctypes.byref(c)

    def append(c=cache.ref, l0=0, l1=2, s=start.data_ptr(), n=2, m=2, qq=None, kk=k.data_ptr(), vv=v.data_ptr(), rot=None, qo=None):
        return lib.lethe_block_append(ctx.h, c, l0, l1, s, n, m, qq, kk, vv, rot, qo, None)

    def attend(c=cache.ref, l0=0, l1=2, qq=qd.data_ptr(), sc=scale, s=None, n=0, o=out.data_ptr()):
        return lib.lethe_block_attend(ctx.h, c, l0, l1, qq, sc, s, n, o, None, None)

    def select(c=cache.ref, qq=qd.data_ptr(), n=3, a=0, b=0, s=sel.data_ptr()):
        return lib.lethe_block_select(ctx.h, c, 0, 2, qq, n, a, b, s, None)

    def read(c=cache.ref, n=4, kk=k.data_ptr(), vv=v.data_ptr()):
        return lib.lethe_block_read(ctx.h, c, 0, 2, None, n, kk, vv, None)

    for call in (append, attend, select, read):
        assert call(c=None) == INV and call(c=changed(len=None)) == INV and call(c=changed(k=cache.k.data_ptr() + 8)) == INV
        assert call(c=changed(head_dim=96)) == UNS and call(c=changed(block_tokens=48)) == UNS and call(c=changed(n_kv_heads=3)) == INV
        assert call(c=changed(capacity=0)) == INV and call(c=changed(layout=7)) == INV and call(c=changed(page_table=None)) == INV
        assert call(c=changed(n_pages=1 << 40)) == UNS and call(c=changed(batch=1 << 30, n_kv_heads=2)) == UNS and call(c=changed(n_layers=129)) == UNS
    assert append(l0=1, l1=1) == INV and append(l0=-1) == INV and append(l1=3) == INV
    assert append(s=None) == INV and append(kk=None) == INV and append(n=-1) == INV and append(m=0) == INV and append(kk=k.data_ptr() + 2) == INV
    assert append(qq=q.data_ptr()) == INV and append(qq=q.data_ptr(), qo=q.data_ptr()) == INV      # no rotary
    r = binding.Rotary([0], [1.0], torch.zeros((1, 2), dtype=torch.int32, device="cuda"))
    assert append(qq=q.data_ptr(), qo=q.data_ptr() + 64, rot=r.ref) == INV and append(qq=q.data_ptr(), qo=k.data_ptr(), rot=r.ref) == INV
    assert append(n=0) == 0 and read(n=0) == 0
    assert attend(qq=None) == INV and attend(sc=None) == INV and attend(o=None) == INV and attend(o=qd.data_ptr()) == INV and attend(s=sel.data_ptr(), n=0) == INV
    assert attend(sc=(ctypes.c_float * 2)(0.1, float("nan"))) == INV and attend(c=changed(n_q_heads=18)) == UNS and attend(qq=qd.data_ptr() + 2) == INV
    assert select(n=0) == INV and select(a=2, b=2) == INV and select(a=-1) == INV and select(s=None) == INV and select(c=changed(k_range=None)) == INV
    assert select(c=changed(n_q_heads=18)) == UNS and read(kk=None) == INV and read(n=-1) == INV and read(n=1 << 30) == UNS
    before = cache.len.clone()
    torch.cuda.synchronize()
    assert torch.equal(before, cache.len) and ctx.poll_status()[0] == 0
