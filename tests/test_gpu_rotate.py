"""lethe_rotate (rotary positions with several axes) against its 64-bit definition, its inverse, and its gradient."""
import ctypes
import math

import pytest
import torch

import chunk_reference as ref
from helpers import gpu_context

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_context()
    yield c
    c.close()


def inputs(nl, n, Hq, Hkv, D, dtype, axes, far, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k = torch.randn((nl, n, Hq, D), generator=g).to(dtype), torch.randn((nl, n, Hkv, D), generator=g).to(dtype)
    pos = torch.randint(-50, 50, (axes, n), generator=g, dtype=torch.int32) + far
    return q, k, pos.to(torch.int32)


def bound(want, size, dtype):
    """An angle is off by 2^-23 radians at most; two products, a sum and cos / sin round to fp32 (2 steps each at most), then the
    output rounds by half a step of its type."""
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    return size * (2.0 ** -23 + 6 * 2.0 ** -23) + want.abs() * half + 1e-30


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("nl,n,Hq,Hkv,D,rot,axes,far", [
    (1, 1, 8, 2, 64, 64, 1, 0), (1, 8, 32, 8, 128, 128, 3, 0), (2, 37, 28, 4, 128, 128, 3, 1000), (1, 5, 5, 1, 64, 48, 2, 10 ** 6),
    (1, 19, 6, 2, 128, 2, 1, 5), (1, 9, 3, 3, 128, 90, 4, 2 ** 31 - 100), (3, 4, 4, 1, 64, 14, 2, -2 ** 31 + 60), (1, 2000, 8, 2, 128, 96, 3, 12345)])
def test_against_definition(ctx, dtype, pairs, nl, n, Hq, Hkv, D, rot, axes, far):
    from paper_2511_06029_b200 import binding
    q, k, pos = inputs(nl, n, Hq, Hkv, D, dtype, axes, far, seed=n)
    half = rot // 2
    axis = [p % axes for p in range(half)]
    freq = [(-1) ** p * 10000.0 ** (-p / max(1, half)) * (2 * math.pi if p == 0 else 1.0) for p in range(half)]
    r = binding.Rotary(axis, freq, pos.cuda(), style=binding.ROT_PAIRS if pairs else binding.ROT_HALVES)
    for inverse in (False, True):
        qo, ko = torch.full_like(q, 9.0, device="cuda"), torch.full_like(k, 9.0, device="cuda")
        ctx.rotate(r, q.cuda(), k.cuda(), qo, ko, inverse=inverse)
        q_in, only = q.cuda(), torch.empty_like(q, device="cuda")
        ctx.rotate(r, q_in, None, only, None, inverse=inverse)          # queries alone
        assert torch.equal(only, qo)
        ctx.rotate(r, q_in, None, q_in, None, inverse=inverse)          # in place
        assert torch.equal(q_in, qo)
        for x, y in ((q, qo), (k, ko)):
            want, size = ref.rotate(x, axis, freq, pos, pairs, inverse)
            d = (y.cpu().double() - want).abs()
            assert bool((d <= bound(want, size, dtype)).all()), f"worst {float((d / bound(want, size, dtype)).max()):.3g}"
            assert torch.equal(y.cpu()[..., rot:], x[..., rot:])
    assert ctx.poll_status()[0] == 0


@pytest.mark.parametrize("pairs", [False, True])
def test_gradient(ctx, pairs):
    """The gradient of f(x) = <w, rotate(x)> is the inverse rotation of w: against the formula and against differences (f is linear
    in x, so a difference of any width is exact up to the rounding of its two values)."""
    from paper_2511_06029_b200 import binding
    nl, n, H, D, rot, axes = 1, 3, 2, 64, 48, 3
    x, w, pos = inputs(nl, n, H, H, D, torch.float32, axes, 700, seed=2)
    axis, freq = [p * axes // 24 for p in range(24)], [10000.0 ** (-p / 24) for p in range(24)]
    r = binding.Rotary(axis, freq, pos.cuda(), style=binding.ROT_PAIRS if pairs else binding.ROT_HALVES)
    grad = torch.empty_like(w, device="cuda")
    ctx.rotate(r, w.cuda(), None, grad, None, inverse=True)
    want, size = ref.rotate(w, axis, freq, pos, pairs, True)
    assert bool(((grad.cpu().double() - want).abs() <= bound(want, size, torch.float32)).all())

    def f(z):
        y = torch.empty_like(z, device="cuda")
        ctx.rotate(r, z.cuda(), None, y, None)
        return y.cpu().double()

    y0 = f(x)
    for at in ((0, 0, 0, 0), (0, 1, 1, 23), (0, 2, 0, 30), (0, 2, 1, 47), (0, 1, 0, 63)):
        z = x.clone()
        z[at] += 4.0
        got = float(((f(z) - y0) * w.double()).sum()) / float(z[at].double() - x[at].double())
        # two values of the pair, each off by at most 14 * 2^-23 of the operands' size (bound above, twice), times w, over 4
        slack = 2 * 14 * 2.0 ** -23 * float(w.abs().max()) * (2 * float(x.abs().max()) + 4.0) / 4.0 + float(size.max()) * 7 * 2.0 ** -23
        assert abs(got - float(want[at])) <= slack


def test_refusals(ctx):
    from paper_2511_06029_b200 import binding
    q, k, pos = inputs(1, 6, 4, 2, 64, torch.bfloat16, 2, 0)
    q, k, pos = q.cuda(), k.cuda(), pos.cuda()
    r = binding.Rotary([0, 1] * 16, [0.1] * 32, pos)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    p = binding._dp

    def call(rot=r.c, dtype=binding.BF16, D=64, nl=1, n=6, Hq=4, Hkv=2, q=q, k=k, qo=qo, ko=ko):
        return ctx.lib.lethe_rotate(ctx.h, ctypes.byref(rot) if rot is not None else None, dtype, D, nl, n, Hq, Hkv, p(q), p(k), 0, p(qo), p(ko), binding._stream(0))

    I = binding.ERR_INVALID_ARG
    assert call(rot=None) == I and call(q=None) == I and call(qo=None) == I and call(k=None) == I and call(ko=None) == I
    assert call(dtype=binding.FP8_E4M3) == I and call(D=96) == binding.ERR_UNSUPPORTED and call(nl=0) == I and call(n=-1) == I and call(Hkv=0) == I
    flat = torch.zeros(6 * 4 * 64 + 6 * 2 * 64, dtype=torch.bfloat16, device="cuda")
    assert call(q=flat, qo=flat[64:]) == I                              # overlaps its input without being it
    assert call(q=flat[1:]) == I                                        # not 16-byte aligned
    assert call(qo=flat, ko=flat[64:]) == I and call(qo=k, k=k) == I
    assert call(n=0) == binding.OK and call() == binding.OK
    assert ctx.poll_status()[0] == 0
