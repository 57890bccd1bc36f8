"""Head sizes that this library's attention does not have: refused by name where the decoder would need it,
accepted where it does not."""
import pytest
import torch

from paper_2412_04787_gb300 import build, dqt
from paper_2412_04787_gb300.decoder import DecoderConfig, DQTDecoder


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


@pytest.mark.parametrize("hidden,heads", [(128, 4), (192, 2), (512, 2), (80, 1)])
def test_other_sizes(hidden, heads):
    cfg = DecoderConfig(layers=0, hidden=hidden, heads=heads, vocab=8)  # rectangular batches, a head to a head
    if heads > 1:
        with pytest.raises(ValueError, match="head size"):
            DecoderConfig(hidden=hidden, heads=heads, kv_heads=heads // 2)
    model = DQTDecoder(cfg, device="cpu")
    with pytest.raises(ValueError, match="head size"):
        model(torch.zeros(5, dtype=torch.int64), plan=dqt.attn_plan((2, 3), device="cpu"))


@pytest.mark.parametrize("hidden,heads", [(128, 2), (256, 2), (768, 12), (2048, 32)])
def test_sizes_that_are_there(hidden, heads):
    assert DecoderConfig(hidden=hidden, heads=heads, kv_heads=heads // 2).kv_heads == heads // 2
