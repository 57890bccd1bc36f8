"""A plan's table and positions are copied from host memory, which cannot be part of a CUDA graph: refused
during a capture before anything is copied (where a capture does not check for it, the graph would read
freed host memory).  The capture is a stand-in; nothing here needs a GPU."""
import types

import pytest
import torch

from paper_2412_04787_gb300 import build, dqt


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


def test_refused_during_a_capture(monkeypatch):
    table = types.SimpleNamespace(device=torch.device("cuda", 0))
    plan = dqt.AttnPlan((3, 2), 2, 2, 3, table)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    monkeypatch.setattr(torch.Tensor, "to", lambda *a, **k: pytest.fail("copied during a capture"))
    for device in ("cuda", "cuda:0", torch.device("cuda")):
        with pytest.raises(RuntimeError, match="captur"):
            dqt.attn_plan((3, 2), device=device)
    with pytest.raises(RuntimeError, match="captur"):
        plan.positions()


def test_on_the_host_a_capture_does_not_matter(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    plan = dqt.attn_plan((3, 2), device="cpu")
    assert plan.positions().tolist() == [0, 1, 2, 0, 1]
