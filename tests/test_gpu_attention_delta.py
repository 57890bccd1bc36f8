"""Attention backward where delta_i = do_i . o_i is not finite: dq_i and the dk_j of the rows that i sees are
not, and nothing else.  dv_j = sum_i p_ij do_i has no delta in it and keeps its bits.

Each case changes a row of o, or values so large that the fp32 sum of delta overflows; do, q, k, v and lse
stay finite."""
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
    dqt.dqt_check_device_status()


def _inputs(lengths, H, KV, D, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(sum(lengths), h, D, generator=g).to(torch.bfloat16).cuda() for h in (H, KV, KV, H)]


@pytest.mark.parametrize("H,KV,D", [(2, 2, 64), (4, 1, 64), (2, 1, 128)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("row", [0, 70, 200, 330])
def test_a_delta_that_is_not_finite(row, bad, H, KV, D):
    lengths = (300, 129)
    q, k, v, do = _inputs(lengths, H, KV, D, seed=D + row)
    plan = dqt.attn_plan(lengths)
    o, lse = dqt.dqt_attn_fwd_bf16(q, k, v, plan)
    want = dqt.dqt_attn_bwd_bf16(do, q, k, v, o, lse, plan)
    o[row, 0, 3] = bad  # one q head's
    dq, dk, dv = dqt.dqt_attn_bwd_bf16(do, q, k, v, o, lse, plan)
    assert torch.equal(dv, want[2])
    other = torch.ones(sum(lengths), H, dtype=torch.bool, device="cuda")
    other[row, 0] = False
    assert torch.equal(dq[other], want[0][other]) and not dq[row, 0].isfinite().any()
    first = 0 if row < 300 else 300
    seen = torch.zeros(sum(lengths), KV, dtype=torch.bool, device="cuda")
    seen[first:row + 1, 0] = True
    assert torch.equal(dk[~seen], want[1][~seen]) and not dk[seen].isfinite().any()


@pytest.mark.parametrize("D", [64, 128])
def test_a_delta_beyond_fp32(D):
    """do . o of 1e39 and more from finite bf16: dv against the definition in fp64 (p and the result as
    bf16, 2^-8 each, of the sums of magnitudes, and 10 % for the fp32 sums)."""
    lengths = (150,)
    q, k, v, do = _inputs(lengths, 2, 1, D, seed=7)
    v, do = v.abs() * 1e19, do.abs() * 1e20
    plan = dqt.attn_plan(lengths)
    o, lse = dqt.dqt_attn_fwd_bf16(q, k, v, plan)
    assert o.isfinite().all()
    dq, dk, dv = dqt.dqt_attn_bwd_bf16(do, q, k, v, o, lse, plan)
    seen = torch.ones(150, 150, dtype=torch.bool, device="cuda").tril()
    want = torch.zeros(150, D, dtype=torch.float64, device="cuda")
    for h in range(2):
        x = (q[:, h].double() @ k[:, 0].double().T * D ** -0.5).masked_fill(~seen, -math.inf)
        want += torch.softmax(x, 1).T @ do[:, h].double()
    assert ((dv[:, 0].double() - want).abs() <= 1.1 * 2 * 2.0 ** -8 * want).all()  # (all terms are positive)
    assert not dq.isfinite().any() and not dk.isfinite().any()
