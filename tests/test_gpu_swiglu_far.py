"""The gate with its 8-bit checkpoint where sigmoid(g) is far from one: g from -20 down to -200 and of
either sign up to bf16's largest, beside u of any size, against the definition in fp64.

Tolerances.  sigmoid: x log2 e in fp32, with |x log2 e| < 2^7, is off by 2^-18 for its rounding and 2^-17.6 for
the constant's, and so the exponential by 2^-17.3 relative; with the other roundings 2^-17.  One
rounding to bf16 (2^-8), and half of bf16's smallest step, 2^-134, where the result is that small.
dg has the terms dh u s and dh u s g (1 - s), each off by that much."""
import math

import pytest
import torch

from paper_2412_04787_gb300 import dqt

pytestmark = pytest.mark.gpu

REL, TINY = 2.0 ** -8 + 2.0 ** -17, 2.0 ** -134


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2412_04787_gb300 import build
    build.build()
    dqt.lib()
    yield
    torch.cuda.synchronize()


def _values(codes, scales):
    F = codes.shape[-1]
    return codes.double() * scales.double().repeat_interleave(128, -1)[..., :F]


def _sig(x):
    """sigmoid(x) and sigmoid(-x) in fp64 without overflow."""
    e = torch.exp(-x.abs())
    a, b = 1 / (1 + e), e / (1 + e)
    return torch.where(x >= 0, a, b), torch.where(x >= 0, b, a)


def _check(g, u, dh):
    h, codes, scales = dqt.dqt_swiglu_ckpt_bf16(g, u)
    s, _ = _sig(g.double())
    want = g.double() * s * u.double()
    assert ((h.double() - want).abs() <= REL * want.abs() + TINY).all()
    dg, du = dqt.dqt_swiglu_ckpt_bwd_bf16(dh, codes, scales)
    v = _values(codes, scales)
    g, u, d = v[:, 0], v[:, 1], dh.double()
    s, t = _sig(g)
    wu = d * g * s
    assert ((du.double() - wu).abs() <= REL * wu.abs() + TINY).all()
    wg = d * u * s * (1 + g * t)
    room = 2.0 ** -16 * (d * u * s).abs() * (1 + g.abs() * t)
    assert ((dg.double() - wg).abs() <= 2.0 ** -8 * wg.abs() + room + TINY).all()


@pytest.mark.parametrize("size", [1.0, 1e-3, 1e15, 1e30])
@pytest.mark.parametrize("lo,hi", [(20, 79), (60, 90), (79, 81), (86, 100), (95, 200)])
def test_far_below_zero(lo, hi, size):
    """A block's whole range, and (rows 2, 3) one far value among ordinary ones."""
    gen = torch.Generator().manual_seed(lo + hi)
    g = -torch.linspace(lo, hi, 264).repeat(4, 1)
    g[2:] = torch.randn(2, 264, generator=gen)
    g[2:, ::40] = -float(hi)
    u, d = torch.randn(4, 264, generator=gen) * size, torch.randn(4, 264, generator=gen)
    _check(*(x.to(torch.bfloat16).cuda() for x in (g, u, d)))


@pytest.mark.parametrize("sign", [1, -1])
def test_up_to_the_largest(sign):
    gen = torch.Generator().manual_seed(3)
    g = sign * torch.logspace(1, 38, 512).repeat(3, 1)
    u, d = torch.randn(3, 512, generator=gen) * 0.1, torch.randn(3, 512, generator=gen) * 0.1
    _check(*(x.to(torch.bfloat16).cuda() for x in (g, u, d)))


def test_what_is_not_finite():
    """+inf and -inf have the values of x / (1 + exp(-x)): inf and NaN; NaN stays in its element."""
    g = torch.zeros(3, 128, dtype=torch.bfloat16, device="cuda")
    u = torch.ones_like(g)
    g[0, 5], g[1, 6], g[2, 7] = math.inf, -math.inf, math.nan
    h = dqt.dqt_swiglu_ckpt_bf16(g, u)[0]
    assert h[0, 5] == math.inf and h[1, 6].isnan() and h[2, 7].isnan()
    assert (h == 0).sum() == 3 * 128 - 3
