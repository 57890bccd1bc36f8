"""The autograd functions for packed documents have first derivatives only: differentiating their gradients
again is an error, not a gradient that leaves their part out."""
import pytest
import torch

from paper_2412_04787_gb300 import dqt
from paper_2412_04787_gb300.decoder import _PackedAttention, _SwiGLUCkpt, _TokenLogprob

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


def _calls():
    g = torch.Generator().manual_seed(1)

    def rand(*shape):
        return torch.randn(*shape, generator=g).to(torch.bfloat16).cuda().requires_grad_()

    plan = dqt.attn_plan((30, 40))
    t = torch.arange(70).cuda()
    return {"attention": (lambda q, k, v: _PackedAttention.apply(q, k, v, plan),
                          (rand(70, 4, 64), rand(70, 2, 64), rand(70, 2, 64))),
            "logprob": (lambda x: _TokenLogprob.apply(x, t, 3)[0], (rand(70, 100),)),
            "entropy": (lambda x: _TokenLogprob.apply(x, t, 0)[1], (rand(70, 100),)),
            "gate": (_SwiGLUCkpt.apply, (rand(70, 264), rand(70, 264)))}


@pytest.mark.parametrize("name", ["attention", "logprob", "entropy", "gate"])
def test_a_second_derivative_is_refused(name):
    f, x = _calls()[name]
    first = torch.autograd.grad(f(*x).float().square().sum(), x)
    again = torch.autograd.grad(f(*x).float().square().sum(), x, create_graph=True)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    # a penalty on the gradient, beside a term of the inputs themselves
    loss = sum(b.float().square().sum() + t.float().sum() for b, t in zip(again, x))
    with pytest.raises(RuntimeError, match="once_differentiable"):
        loss.backward()
