"""The plans that a decoder with shared k and v heads keeps for rectangular batches: their tables
stay in place as long as the model does (a captured CUDA graph reads them by address), each call
takes the plan of its own shape, also beside another thread's.  Host code: blocks that note the plan
stand in for the decoder's."""
import threading
import time
import weakref

import pytest
import torch

from paper_2412_04787_gb300 import build
from paper_2412_04787_gb300.decoder import DecoderConfig, DQTDecoder


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


class _Note(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.seen = threading.local()

    def forward(self, x, cos_sin, plan=None):
        self.seen.plan = plan
        return x


class _Yields(DQTDecoder):
    """Lets other threads run whenever an attribute has been set."""

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        time.sleep(1e-3)


def _model(cls=DQTDecoder):
    """No layers but a block that notes its plan; two heads over one."""
    model = cls(DecoderConfig(layers=0, hidden=128, heads=2, kv_heads=1, vocab=8), device="cpu")
    model.blocks.append(_Note())
    model.norm = torch.nn.Identity()
    return model


def _plan_of(model, B, S):
    with torch.no_grad():
        model(torch.zeros(B, S, dtype=torch.int64))
    return model.blocks[0].seen.plan


def test_a_table_outlives_calls_at_other_shapes():
    model = _model()
    table = weakref.ref(_plan_of(model, 2, 8).table)
    for shape in ((4, 4), (1, 300), (3, 1)):
        _plan_of(model, *shape)
    model.blocks[0].seen.plan = None
    assert table() is not None
    again = _plan_of(model, 2, 8)
    assert again.table is table() and again.lengths == (8, 8)


def test_threads_take_their_own_shapes_plan():
    """2 x 8 and 4 x 4 have the same tokens, so that no check of shapes would tell them apart."""
    model, wrong = _model(_Yields), []

    def work(B, S):
        for _ in range(50):
            if _plan_of(model, B, S).lengths != (S,) * B:
                wrong.append((B, S))
                return

    threads = [threading.Thread(target=work, args=a) for a in ((2, 8), (4, 4), (8, 2), (1, 16))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
