"""A table whose tiles do not start at multiples of 128 rows: such tiles are left out, forward and
backward, whatever the others are.  (The keys' kernel finds the statistics of a document's queries by
the tiles before; from another row it would look one tile past the workspace.)"""
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


@pytest.mark.parametrize("H,KV,D", [(2, 1, 64), (1, 1, 64), (16, 1, 64), (2, 1, 128), (3, 1, 128)])
def test_tiles_between_the_rows_are_left_out(H, KV, D):
    T = 300
    g = torch.Generator().manual_seed(H + D)
    q, k, v, do = (torch.randn(T, h, D, generator=g).to(torch.bfloat16).cuda() for h in (H, KV, KV, H))
    plan = dqt.attn_plan((T,))
    o, lse = dqt.dqt_attn_fwd_bf16(q, k, v, plan)
    dq, dk, dv = dqt.dqt_attn_bwd_bf16(do, q, k, v, o, lse, plan)
    table = plan.table.clone()
    table[:, 2] += (table[:, 2] == 256).int()  # the document's last tile, in each of the lists
    assert sorted(set(table[:, 2].tolist())) == [0, 128, 257]
    lay = dqt._attn_layout(q, k, v, plan)
    got = {n: torch.full_like(t, 7.0) for n, t in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv))}
    p = {n: t.data_ptr() for n, t in got.items()}
    ws = torch.zeros(dqt.lib().dqt_attn_bwd_workspace_size(C.byref(lay)), dtype=torch.uint8, device="cuda")
    assert dqt.lib().dqt_attn_fwd_bf16(q.data_ptr(), k.data_ptr(), v.data_ptr(), C.byref(lay), table.data_ptr(),
                                       D ** -0.5, p["o"], p["lse"], dqt._stream()) == dqt.DQT_OK
    assert dqt.lib().dqt_attn_bwd_bf16(do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                       lse.data_ptr(), C.byref(lay), table.data_ptr(), D ** -0.5, p["dq"],
                                       p["dk"], p["dv"], ws.data_ptr(), ws.numel(), dqt._stream()) == dqt.DQT_OK
    torch.cuda.synchronize()
    for n, t in got.items():
        t = t.transpose(0, 1) if n == "lse" else t
        assert (t[256:] == 7).all(), n
    for n, want in (("o", o), ("lse", lse.t()), ("dq", dq)):
        t = got[n].t() if n == "lse" else got[n]
        assert torch.equal(t[:256], want[:256]), n
