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
        b_out = b_out + room * st.attend(0, q, [scale] * L)[0]
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
