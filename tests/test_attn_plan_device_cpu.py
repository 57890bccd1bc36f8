"""A plan whose table is not on the operands' device is refused before its address reaches a kernel.  Host
code: stand-ins that answer like CUDA tensors (the entries that launch are not called)."""
import pytest
import torch

from paper_2412_04787_gb300 import build, dqt


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


class _OnCuda:
    """A contiguous bf16 tensor of this shape on a CUDA device, as far as the checks look."""
    is_cuda, dtype = True, torch.bfloat16

    def __init__(self, shape, index=0):
        self.shape, self.device = torch.Size(shape), torch.device("cuda", index)

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self.shape[1] * self.shape[2], self.shape[2], 1


def _operands(*index):
    return [_OnCuda((200, h, 64), i) for h, i in zip((4, 2, 2), index)]


def _plan(device):
    plan = dqt.attn_plan((130, 70), device="cpu")
    table = torch.empty(0) if device == "cpu" else _OnCuda((plan.table.shape[0], 4, 1), device)
    return dqt.AttnPlan(plan.lengths, plan.tiles, plan.tiles256, plan.longest, table)


def test_one_device_is_taken():
    for i in (0, 1):
        lay = dqt._attn_layout(*_operands(i, i, i), _plan(i))
        assert (lay.tokens, lay.heads, lay.kv_heads, lay.dim, lay.tiles) == (200, 4, 2, 64, 3)


@pytest.mark.parametrize("index,table", [((0, 0, 0), "cpu"), ((0, 0, 0), 1), ((1, 1, 1), 0), ((0, 1, 0), 0),
                                         ((0, 0, 1), 0), ((1, 0, 0), 0)])
def test_other_devices_are_refused(index, table):
    with pytest.raises(ValueError, match="one device"):
        dqt._attn_layout(*_operands(*index), _plan(table))


@pytest.mark.parametrize("table", ["cpu", 1])
def test_refused_by_both_calls(table):
    q, k, v = _operands(0, 0, 0)
    with pytest.raises(ValueError, match="one device"):
        dqt.dqt_attn_fwd_bf16(q, k, v, _plan(table))
    with pytest.raises(ValueError, match="one device"):
        dqt.dqt_attn_bwd_bf16(q, q, k, v, q, None, _plan(table))
