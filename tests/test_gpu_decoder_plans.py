"""Training steps of a decoder with shared k and v heads, captured in a CUDA graph, with calls at other
shapes and other tensors in freed memory between the replays: what eager steps leave, bit for bit."""
import pytest
import torch

from paper_2412_04787_gb300 import dqt
from paper_2412_04787_gb300.decoder import DecoderConfig, DQTDecoder

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


def _make():
    model = DQTDecoder(DecoderConfig(layers=2, hidden=256, heads=4, kv_heads=2, ffn=512, vocab=512, lr=2e-3,
                                     seed=9, ckpt8=True))
    model.enable_graph_updates()
    return model, torch.optim.AdamW(model.dense_parameters(), lr=2e-3, capturable=True)


def _step(model, opt, ids, targets, plan, slot):
    model.prepare_step(slot)
    model.upload_update_consts(slot)
    model(ids, targets, plan=plan).backward()
    opt.step()
    opt.zero_grad(set_to_none=True)


def _disturb(model, seed):
    """Calls at other shapes, and small tensors of arbitrary bits that take freed memory."""
    with torch.no_grad():
        for shape in ((2, 70), (1, 200 + seed), (7, 3)):
            model(torch.zeros(shape, dtype=torch.int64, device="cuda"))
    junk = [torch.full((64 * (1 + i % 8),), -1 - i, dtype=torch.int32, device="cuda") for i in range(256)]
    torch.cuda.synchronize()
    return junk


@pytest.mark.parametrize("packed", [False, True])
def test_replays_between_calls_at_other_shapes(packed):
    lengths = (130, 5, 65)
    shape = (sum(lengths),) if packed else (4, 64)
    g = torch.Generator().manual_seed(4)
    batches = [torch.randint(0, 512, shape, generator=g).cuda() for _ in range(6)]
    plan = dqt.attn_plan(lengths) if packed else None

    def targets(ids):
        return torch.roll(ids, -1)

    ea, oa = _make()
    for i, ids in enumerate(batches):
        _step(ea, oa, ids, targets(ids), plan, i % 2)

    gb, ob = _make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i, ids in enumerate(batches[:2]):
            _step(gb, ob, ids, targets(ids), plan, i % 2)
    torch.cuda.current_stream().wait_stream(side)
    at = batches[2].clone()
    graph = torch.cuda.CUDAGraph()
    ob.zero_grad(set_to_none=True)
    with torch.cuda.graph(graph):
        gb(at, targets(at), plan=plan).backward()
        ob.step()
    for i, ids in enumerate(batches[2:], start=2):
        junk = _disturb(gb, i)
        at.copy_(ids)
        gb.prepare_step(i % 2)
        gb.upload_update_consts(i % 2)
        graph.replay()
        torch.cuda.synchronize()
        del junk
    for la, lb in zip(ea.bitlinear_layers(), gb.bitlinear_layers()):
        assert la.step == lb.step == 6
        assert torch.equal(la.codes, lb.codes)
        assert torch.equal(la.m, lb.m) and torch.equal(la.v, lb.v)
    for a, b in zip(ea.dense_parameters(), gb.dense_parameters()):
        assert torch.equal(a, b)
