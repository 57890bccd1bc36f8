"""A value that is not finite inside a document: the rows that see it are not finite, and what stands in other
tiles of 128 rows and does not see it keeps its bits, forward and backward."""
import math

import pytest
import torch

from paper_2412_04787_gb300 import dqt

pytestmark = pytest.mark.gpu

N, ROW = 500, 200  # the document, and its bad row: in the tile of rows 128 to 255


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


def _run(t, plan):
    o, lse = dqt.dqt_attn_fwd_bf16(t["q"], t["k"], t["v"], plan)
    dq, dk, dv = dqt.dqt_attn_bwd_bf16(t["do"], t["q"], t["k"], t["v"], o, lse, plan)
    return {"o": o, "lse": lse.t(), "dq": dq, "dk": dk, "dv": dv}


@pytest.mark.parametrize("H,KV,D", [(2, 2, 64), (4, 1, 64), (3, 1, 128)])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
def test_rows_that_do_not_see_it(name, bad, H, KV, D):
    g = torch.Generator().manual_seed(D)
    t = {n: torch.randn(N, h, D, generator=g).to(torch.bfloat16).cuda()
         for n, h in (("q", H), ("k", KV), ("v", KV), ("do", H))}
    plan = dqt.attn_plan((N,))
    want = _run(t, plan)
    t[name][ROW] = bad
    got = _run(t, plan)
    other = torch.ones(N, dtype=torch.bool, device="cuda")
    other[ROW] = False
    early, late = torch.arange(N, device="cuda") < 128, torch.arange(N, device="cuda") >= 256
    same = {"q": {"o": other, "lse": other, "dq": other, "dk": late, "dv": late},
            "k": {"o": early, "lse": early, "dq": early},
            "v": {"o": early, "lse": other | True, "dq": early, "dv": other | True},
            "do": {"o": other | True, "lse": other | True, "dq": other, "dk": late, "dv": late}}[name]
    for n, rows in same.items():
        assert torch.equal(got[n][rows], want[n][rows]), n
    reached = {"q": {"o": ROW, "dq": ROW, "dk": slice(0, ROW + 1), "dv": slice(0, ROW + 1)},
               "k": {"o": slice(ROW, N), "dq": slice(ROW, N)},
               "v": {"o": slice(ROW, N), "dq": slice(ROW, N)},
               "do": {"dq": ROW, "dk": slice(0, ROW + 1), "dv": slice(0, ROW + 1)}}[name]
    for n, rows in reached.items():
        assert not got[n][rows].isfinite().any(), n
