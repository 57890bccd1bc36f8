"""The logits' gradient where the logits are so large that lse = max + log S in fp32 loses log S: rows
of the type's lowest value alone (a mask that leaves nothing), and rows around some large value.
Against the definition in fp64.

Tolerances.  x - max is exact in fp32 or far below the largest, and p is formed from it: off by 2^-15
relative with |x - max| and log S up to 2^8 (2^-17 each from two subtractions, the product with
log2 e and the constant).  The entropy is within 4e-6 of sums of at most log V.  One rounding to bf16, 2^-8.  Up to |lse| =
1024 the probabilities are formed from lse, half a step of which is 2^-15: 2^-13 in all."""
import math

import pytest
import torch

from paper_2412_04787_gb300 import dqt

pytestmark = pytest.mark.gpu

LOWEST = torch.finfo(torch.bfloat16).min


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2412_04787_gb300 import build
    build.build()
    dqt.lib()
    yield
    torch.cuda.synchronize()


def _check(x, t):
    M, V = x.shape
    logp, H, lse, _, _ = dqt.dqt_token_logprob_bf16(x, t)
    g = torch.Generator().manual_seed(5)
    dl, de = torch.randn(M, generator=g).cuda(), torch.randn(M, generator=g).cuda()
    dx = dqt.dqt_token_logprob_bwd_bf16(x, t, lse, H, dl, de)
    z = x.double()
    z = z - z.max(1, keepdim=True).values
    rlogp = z - torch.logsumexp(z, 1, keepdim=True)
    p = rlogp.exp()
    lp = torch.where(p > 0, rlogp, 0.0)
    rH = -(p * lp).sum(1, keepdim=True)
    want_logp = rlogp.gather(1, t[:, None])[:, 0]
    assert ((logp - want_logp).abs() <= 2e-5 + 2e-6 * want_logp.abs()).all()
    assert ((H - rH[:, 0]).abs() <= 2e-5).all()
    a, b = dl.double()[:, None], de.double()[:, None]
    grad = -p * (a + b * (lp + rH))
    size = p * (a.abs() + b.abs() * (lp.abs() + rH + 1))
    grad.scatter_add_(1, t[:, None], a)
    size.scatter_add_(1, t[:, None], a.abs())
    assert ((dx.double() - grad).abs() <= 2.0 ** -8 * grad.abs() + 2.0 ** -13 * size + 1e-30).all()


@pytest.mark.parametrize("M", [3, 200])
@pytest.mark.parametrize("V", [1, 7, 1000, 9001, 40001])
def test_rows_of_the_lowest_value(V, M):
    """Every probability is 1 / V, not 1; then one row with a single logit left, and one with two."""
    x = torch.full((M, V), LOWEST, dtype=torch.bfloat16)
    x[1, V // 2] = 0.0
    x[2, ::max(1, V // 2)] = 3.0
    t = torch.arange(M) % V
    _check(x.cuda(), t.cuda())


@pytest.mark.parametrize("middle", [500.0, 1000.0, 1023.0, 1030.0, 2000.0, 3e4, 1e6, 1e30, 3e38])
@pytest.mark.parametrize("sign", [1, -1])
def test_rows_around_a_large_value(sign, middle):
    """Values a few steps of bf16 apart (512 and more apart beyond 65536: one probability a row, or
    equal ones)."""
    g = torch.Generator().manual_seed(int(math.log(middle) * 10))
    x = torch.full((5, 5003), sign * middle).to(torch.bfloat16)
    step = 2.0 ** (math.frexp(middle)[1] - 8)
    x = (x.double() - step * torch.randint(0, 4, x.shape, generator=g)).to(torch.bfloat16)
    x[4] = sign * middle
    _check(x.cuda(), torch.tensor([0, 9, 77, 5002, 1]).cuda())


def test_rows_apart_and_at_any_alignment():
    g = torch.Generator().manual_seed(2)
    wide = (torch.randint(-3, 1, (6, 3010), generator=g) * 16.0 + 4000.0).to(torch.bfloat16).cuda()
    for first in range(9):
        _check(wide[:, first:first + 3001], torch.arange(6).cuda() * 500)
