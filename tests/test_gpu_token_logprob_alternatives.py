"""The alternatives' ids and log probabilities, value by value, against the definition in fp64: few rows
(no more than there are SMs) and many, rows at any alignment and distance, masked and equal logits.

Tolerances.  fp32 throughout: a row's sum of V exponentials, each off by a few 2^-24 relative and added
in a tree or in steps of thousands, is within 2e-6 relative, so a log probability is within 4e-6 plus 2e-6 of
the magnitudes it is made of (|x|, |max|, log V).  Ids are exact; -inf is -inf."""
import math

import pytest
import torch

from paper_2412_04787_gb300 import dqt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2412_04787_gb300 import build
    build.build()
    dqt.lib()
    yield
    torch.cuda.synchronize()


def _check(x, top):
    M, V = x.shape
    _, _, _, ids, best = dqt.dqt_token_logprob_bf16(x, torch.zeros(M, dtype=torch.int64, device="cuda"), top)
    assert ids.shape == best.shape == (M, top)
    z = x.double()
    want = torch.sort(z, dim=-1, descending=True, stable=True)[1][:, :top]
    assert torch.equal(ids, want)
    logp = (z - torch.logsumexp(z, 1, keepdim=True)).gather(1, want)
    room = 4e-6 + 2e-6 * (z.max(1, keepdim=True).values.abs() + math.log(V) + 1 + logp.abs())
    off = (best.double() - logp).abs()
    assert ((off <= room) | (best == logp)).all()  # (equal: -inf)


def _logits(M, V, seed, std=2.0):
    return (torch.randn(M, V, generator=torch.Generator().manual_seed(seed)) * std).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("M", [1, 5, 140, 400])
@pytest.mark.parametrize("V", [1, 2, 31, 257, 1000, 5003, 32000, 50257])
def test_ordinary_rows(V, M):
    for top in sorted({1, min(V, 8), min(V, 32)}):
        _check(_logits(M, V, M + V), top)


@pytest.mark.parametrize("M", [6, 300])
@pytest.mark.parametrize("V,pitch", [(1000, 1037), (5001, 5004), (32001, 32004), (50257, 50304)])
def test_rows_apart_and_at_any_alignment(V, pitch, M):
    wide = _logits(M, pitch, V)
    for first in (0, 1, 3):
        _check(wide[:, first:first + V], 7)


@pytest.mark.parametrize("M", [5, 300])
@pytest.mark.parametrize("V", [40, 4099, 32000])
def test_equal_masked_and_large(V, M):
    x = torch.zeros(5, V)
    x[1] = torch.arange(V) % 3
    x[2] = -math.inf
    x[2, V // 3::7] = torch.arange(len(range(V // 3, V, 7))) % 5 + 1.0
    x[3] = 2000.0 - torch.arange(V) % 16 * 8
    x[4, V - 3:] = 80.0
    _check(x.repeat(M // 5, 1).to(torch.bfloat16).cuda(), 32 if V > 40 else 5)
