"""The attention backward on a given stream, with a workspace of its own: other tensors of the current
stream do not take its memory while the call is still running there."""
import ctypes as C

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


def test_the_workspace_is_kept_until_the_call_is_done():
    lengths = (2048,) * 4
    g = torch.Generator().manual_seed(1)
    q, k, v, do = (torch.randn(sum(lengths), 16, 64, generator=g).to(torch.bfloat16).cuda() for _ in range(4))
    plan = dqt.attn_plan(lengths)
    o, lse = dqt.dqt_attn_fwd_bf16(q, k, v, plan)
    want = dqt.dqt_attn_bwd_bf16(do, q, k, v, o, lse, plan)
    nbytes = dqt.lib().dqt_attn_bwd_workspace_size(C.byref(dqt._attn_layout(q, k, v, plan)))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            torch.cuda._sleep(2_000_000)  # about a millisecond
        got = dqt.dqt_attn_bwd_bf16(do, q, k, v, o, lse, plan, stream=side)
        junk = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        for _ in range(600):  # for as long as the call takes and more
            junk.fill_(0x3F)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        del junk, got
