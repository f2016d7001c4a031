"""Attention over block caches whose values lie anywhere in the range that a block cache holds (2^-100 to the largest bf16), alone and
next to one another in one item, against the 64-bit statement.  Every case runs as one long sequence (an item that all CTAs
share), as sequences of a few hundred tokens (an item for some warps), and as many short ones (an item for one warp)."""
import math

import pytest
import torch

from block_reference import BlockState
from helpers import gpu_context

pytestmark = pytest.mark.gpu
LENS = [(1, 1, 5003), (1, 4, 777), (4, 300, 75)]   # layers, sequences, tokens


@pytest.fixture(scope="module")
def ctx():
    c = gpu_context()
    yield c
    assert c.poll_status()[0] == 0
    c.close()


def state(L, B, lens, D, T, seed):
    return BlockState(L, B, 8, 1, D, T, lens // T + 1, lens, False, seed=seed)


def queries(st, L, gain=1.0, seed=1):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((L, st.B, st.Hq, st.D), generator=g) * gain).to(torch.bfloat16)


def scale_open(st, by):
    """Open rows times a factor [..] in range of bf16; rows that are not there stay as they are (NaN)."""
    st.v_open = (st.v_open.double() * by).to(torch.bfloat16)


def check(ctx, st, q, scale, room=0.0):
    """`room`: what is added to the relative error of a share (a logarithm that is larger than ordinary ones rounds more coarsely)."""
    L = q.shape[0]
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    ctx.block_attend(st.device_cache(with_range=False), 0, L, q.cuda(), [scale] * L, out, lse=lse)
    want, z, b_out, b_lse = st.attend(0, q, [scale] * L)
    if room:
        st.v_scale, st.v_open = st.v_scale.abs(), st.v_open.abs()
        st.v = st.v.abs()
        b_out = b_out + room * st.attend(0, q, [scale] * L)[0] + unseen(st, q, scale)
        b_lse = b_lse + room
    # the smallest normal number is 2^-126; steps below it are 2^-133 for bf16
    d = (out.cpu().double() - want).abs()
    assert bool((d <= b_out - 1e-30 + 2.0 ** -126).all()), f"out: {float((d / b_out).nan_to_num(1e9).max()):.3g} of the bound"
    d = (lse.cpu().double() - z).abs()
    assert bool((d <= b_lse).all()), f"lse: {float((d / b_lse).nan_to_num(1e9).max()):.3g} of the bound"


# ------------------------------------------------------------------------------------------ parts of an item

@pytest.mark.parametrize("L,B,lens", LENS)
@pytest.mark.parametrize("D,T", [(128, 32), (64, 16)])
@pytest.mark.parametrize("by", [1e36, 1e-27, 1e-30])
def test_values_of_one_size(ctx, L, B, lens, D, T, by):
    """All values large or all small: what a warp or a CTA leaves of an item is finite and not zero."""
    st = state(L, B, lens - lens % T if by > 1 else lens, D, T, seed=D)    # large: full blocks alone
    st.v_scale *= by
    scale_open(st, by)
    check(ctx, st, queries(st, L), 1 / math.sqrt(D))


# ------------------------------------------------------------------------------------------------- open rows

@pytest.mark.parametrize("L,B,lens", LENS + [(1, 3, 31)])
@pytest.mark.parametrize("D,T", [(128, 32), (64, 128)])
@pytest.mark.parametrize("by", [1e37, 2.0 ** 100, 2.0 ** -35, 2.0 ** -99])
def test_open_rows_of_any_size(ctx, L, B, lens, D, T, by):
    """Open rows far larger or smaller than the full blocks (which are as large where that fits the sums of the full blocks)."""
    st = state(L, B, lens, D, T, seed=D + 1)
    scale_open(st, by)
    st.v_scale *= min(max(by, 2.0 ** -30), 2.0 ** 60) if by > 1 else by
    check(ctx, st, queries(st, L), 1 / math.sqrt(D))


@pytest.mark.parametrize("rows", [1, 33, 127])
def test_open_rows_with_zeros_and_infinities(ctx, rows):
    """Rows of zeros have their share of the sum; a value that is not finite makes its element of out not finite, and only that."""
    st = state(1, 2, 128 + rows, 64, 128, seed=rows)
    st.v_open[0, 0, 0, :rows] = 0
    check(ctx, st, queries(st, 1), 0.125)
    st.v_open[0, 1, 0, 0, 3], st.v_open[0, 1, 0, 0, 9], st.v_open[0, 1, 0, 0, 60] = float("inf"), -float("inf"), float("nan")
    q = queries(st, 1)
    out = torch.empty_like(q, device="cuda")
    ctx.block_attend(st.device_cache(with_range=False), 0, 1, q.cuda(), [0.125], out)
    want, _, bound, _ = st.attend(0, q, [0.125])
    bad = torch.zeros(64, dtype=torch.bool)
    bad[[3, 9, 60]] = True
    assert not bool(out[0, 1][:, bad.cuda()].isfinite().any())
    d = (out.cpu().double() - want).abs()
    assert bool((d[0, 0] <= bound[0, 0]).all()) and bool((d[0, 1][:, ~bad] <= bound[0, 1][:, ~bad]).all())


# ------------------------------------------------------------------------------- blocks far apart in one item

APART = 2.0 ** -14
"""Where scales lie far apart a share is formed from logits with the scale's logarithm added: numbers below 2^9, in fp32 a rounding of
2^-16 each for the sum, for taking the logarithm off again and, below 2^8, three times 2^-17 for the logarithm and the two halves of
the factor that joins O and the sum: 3.5 x 2^-16 in the exponent of 2, times log 2."""


def unseen(st, q, scale):
    """What f16 does not hold of small shares: a share times its scale is kept 2^9 times as large as the largest of them at least, and
    below 2^-14 it is off by half of f16's smallest number, 2^-25.  So 2^-34 of the largest for each token and unit of its code, which
    counts where the tokens of the largest shares have small codes in an element.  Open rows have two bf16 terms in its place: below 2^-126
    a share vanishes, below 2^-117 its second term, half a step of 2^-9, does: 2 x 2^-135 of the largest share of a full block times its
    scale, for each token and |x|, the largest open value.

    Values of zero have a share but no size, and nothing says against what they should be held.  Full blocks of zeros count among the
    shares like blocks of 2^-40 of the reference r, the first scale (1 where there is none, 2^90 at most), open rows of zeros like others,
    that is like blocks of scale 1; a factor of 2^6 is how far m may lag.  What they outweigh so far that it leaves fp32 vanishes:
        full blocks before open zeros, rescaled:  p vs < p0 2^-126 2^6, times 127            -> p0 2^-113
        full blocks before full zeros, rescaled:  p vs < p0 2^-126 2^6 2^-40 r, times 127    -> p0 2^-153 r
        full blocks behind full zeros:            p vs < p0 2^-126 2^-9 2^-40 r, times 127   -> less than the line above
        open rows behind full zeros:              p < p0 2^-126 2^-9 2^-40 r, times |x|      -> p0 2^-175 r |x|
    for each token.  [nl][B][Hq][1]"""
    room = torch.zeros(q.shape[:3] + (1,), dtype=torch.float64)
    for li in range(q.shape[0]):
        for b in range(st.B):
            for h in range(st.Hkv):
                K, V = st.rows((li, b, h))
                n, hs = int(st.len[li, b, h]) // st.T, slice(h * st.G, (h + 1) * st.G)
                p = torch.softmax(q[li, b, hs].double() @ K.T * scale, 1)
                scales, largest = st.v_scale[li, b, h, :n].double(), V[n * st.T:].abs().amax(1)
                r = max([1.0] + [min(float(x), 2.0 ** 90) for x in scales])
                size = torch.cat([torch.where(scales == 0, r * 2.0 ** -40, scales).repeat_interleave(st.T), largest / 64])
                room[li, b, hs, 0] = (p * size).amax(1) * 127 * n * st.T * 2.0 ** -34
                if len(largest) and n:
                    full = (p[:, :n * st.T] * size[:n * st.T]).amax(1)
                    room[li, b, hs, 0] += full * float(largest.max()) * len(largest) * 2.0 ** -134
                zero = V.abs().amax(1) == 0
                if bool(zero.any()):
                    gone = 2.0 ** -113 + 2.0 ** -153 * r + 2.0 ** -175 * r * float(largest.max() if len(largest) else 0)
                    room[li, b, hs, 0] += p[:, zero].amax(1) * gone * len(V)
    return room


@pytest.mark.parametrize("L,B,lens", LENS)
@pytest.mark.parametrize("D,T", [(128, 32), (128, 16), (64, 64)])
@pytest.mark.parametrize("sizes", [(1e-30, 1e9), (1e9, 1e-30), (1.0, 2.0 ** 119), (2.0 ** 119, 1.0, 2.0 ** -99), (1.0, 2.0 ** 45), (1e30, 1e30, 1e-30)])
@pytest.mark.parametrize("spread", [1.0, 40.0])
def test_value_blocks_far_apart(ctx, L, B, lens, D, T, sizes, spread):
    """Blocks of very different size in turn.  With a wide spread of logits the small ones may outweigh the others, and do in some heads."""
    blocks_in_turn(ctx, L, B, lens, D, T, sizes, spread)


def blocks_in_turn(ctx, L, B, lens, D, T, sizes, spread):
    st = state(L, B, lens, D, T, seed=D + T)
    by = torch.tensor(sizes, dtype=torch.float64)[torch.arange(st.capacity) % len(sizes)]
    top = st.v_scale.nan_to_num(1).max()
    st.v_scale = (st.v_scale.double() / top * by / 127).float()        # the largest value of a block is at most its size
    scale_open(st, sizes[-1] / 8)
    check(ctx, st, queries(st, L, spread), 1 / math.sqrt(D), APART)


@pytest.mark.parametrize("small,large", [(2.0 ** -90, 2.0 ** 100), (1.0, 2.0 ** 60)])
def test_small_blocks_that_outweigh_large_ones(ctx, small, large):
    """One key direction: the blocks' logits are known.  Large values at logits lower by the ratio of the sizes: both matter in out, only
    the small ones in the sum; then the other way round."""
    T, D = 32, 128
    for up in (1, -1):
        st = state(1, 2, 32 * 60 + 9, D, T, seed=3)
        st.k.zero_()
        st.k[..., 0] = 100
        gap = math.log(large / small) * up / 2
        odd = torch.arange(61) % 2 == 1
        st.k_scale[:] = torch.where(odd, gap / 100, -gap / 100).float()      # logits gap and -gap
        st.v_scale[:] = torch.where(odd, small / 127, large / 127).float()
        st.k_open.zero_()
        scale_open(st, small)
        q = torch.zeros((1, 2, 8, D), dtype=torch.bfloat16)
        q[..., 0] = 1.0
        check(ctx, st, q, 1.0, APART)


def test_appended_values_far_apart(ctx):
    """Rows that the append takes, of all sizes that it holds, block by block."""
    from block_reference import starts
    st = BlockState(1, 2, 8, 2, 128, 16, 40, 0, True, seed=9)
    cache = st.device_cache()
    n = 16 * 37 + 5
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((1, 2 * n, 2, 128), generator=g) for _ in range(2))
    exponent = torch.randint(-96, 120, (2 * n // 16 + 1,), generator=g).double().repeat_interleave(16)[:2 * n]
    v = (v.double() * 2.0 ** exponent[None, :, None, None]).to(torch.bfloat16)
    k = k.to(torch.bfloat16)
    ctx.block_append(cache, 0, 1, starts([n, n]).cuda(), n, k.cuda(), v.cuda())
    st.append(0, starts([n, n]), k, v)
    q = queries(st, 1, 20.0)
    out = torch.empty_like(q, device="cuda")
    ctx.block_attend(cache, 0, 1, q.cuda(), [0.1], out)
    want, _, bound, _ = st.attend(0, q, [0.1])
    st.v, st.v_open = st.v.abs(), st.v_open.abs()
    bound = bound + APART * st.attend(0, q, [0.1])[0] + unseen(st, q, 0.1)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())


# ----------------------------------------------------------------------------------------------- blocks of zeros

@pytest.mark.parametrize("L,B,lens", LENS)
@pytest.mark.parametrize("T", [16, 32])
def test_blocks_of_zeros_among_small_ones(ctx, L, B, lens, T):
    """A large block that no query looks at, then blocks of zeros, then small ones at the same logits as the zeros: out is the small ones'
    share, to the precision that it has without the others."""
    D = 128
    st = state(L, B, lens, D, T, seed=T)
    n = st.capacity
    st.k.zero_()
    st.k[..., 0] = 127
    odd = torch.arange(n) % 2 == 1
    st.v_scale[:] = torch.where(odd, 2.0 ** -37 / 127, 0.0).float()
    st.v_scale[..., 0] = 1 / 127
    st.k_scale[..., 0] = 200 / 127     # logit -200 with a query of -1
    st.k_scale[..., 1:] = 1e-3
    st.k_open.zero_()
    scale_open(st, 2.0 ** -37)
    q = torch.zeros((L, B, 8, D), dtype=torch.bfloat16)
    q[..., 0] = -1.0
    check(ctx, st, q, 1.0)


@pytest.mark.parametrize("L,B,lens", LENS)
@pytest.mark.parametrize("D,T", [(128, 16), (64, 64)])
@pytest.mark.parametrize("sizes", [(2.0 ** 119, 1.0, 0.0, 2.0 ** -99), (0.0, 2.0 ** -99, 2.0 ** 119), (0.0, 1.0), (0.0,), (1.0, 0.0, 0.0)])
@pytest.mark.parametrize("spread", [1.0, 40.0])
def test_blocks_of_zeros_and_others_in_turn(ctx, L, B, lens, D, T, sizes, spread):
    blocks_in_turn(ctx, L, B, lens, D, T, sizes, spread)


# ------------------------------------------------------------------- what the device refuses, among such values

def test_bad_pages_and_entries_among_values_far_apart(ctx):
    """A page outside the pool and an entry that is no full block are left out and recorded wherever in the list they stand.  As many
    items of one length as the GPU has warps: each warp has one from end to end, and comes to the scales of a run of 32 blocks first."""
    from paper_2511_06029_b200 import binding
    T, B, bad = 16, torch.cuda.get_device_properties(0).multi_processor_count * 8, 39
    st = BlockState(1, B, 1, 1, 64, T, 41, T * 41, True, seed=4)
    st.v_scale *= torch.where(torch.arange(41) % 2 == 1, 1e-20, 1e20).float()
    q = queries(st, 1)
    cache = st.device_cache(with_range=False)
    out = torch.empty_like(q, device="cuda")
    full = torch.arange(41, dtype=torch.int32).expand(1, B, 1, 41).clone()
    few = BlockState.__new__(BlockState)               # the statement for the items that are looked at
    few.__dict__.update(st.__dict__)
    few.B = 9

    def check_first(lists):
        want, _, bound, _ = few.attend(0, q[:, :9], [0.1], lists[:, :9])
        few.v = st.v.abs()
        bound = bound + APART * few.attend(0, q[:, :9], [0.1], lists[:, :9])[0] + unseen(few, q[:, :9], 0.1)
        few.v = st.v
        assert bool(((out[:, :9].cpu().double() - want).abs() <= bound).all())

    page = cache.page_table[0, 7, 0, bad].clone()
    cache.page_table[0, 7, 0, bad] = st.n_pages
    ctx.block_attend(cache, 0, 1, q.cuda(), [0.1], out)
    assert ctx.poll_status() == (binding.ERR_PAGE, 7)
    cache.page_table[0, 7, 0, bad] = page
    lists = full.clone()
    lists[0, 7, 0, bad] = -1
    check_first(lists)
    given = lists.clone()
    given[0, 7, 0, bad] = 41
    ctx.block_attend(cache, 0, 1, q.cuda(), [0.1], out, selected=given.cuda())
    assert ctx.poll_status() == (binding.ERR_INVALID_ARG, 7)
    check_first(lists)
