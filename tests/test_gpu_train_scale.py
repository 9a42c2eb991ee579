"""The training loop's gradients with every kind of residual scale: the norm in front of the feed-forward block is that of its input,
whatever the scale.  Needs a GPU."""
import pytest

from test_gpu_train import torch  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.5, -0.5, 0.01, 0.0])
def test_gradients_of_any_residual_scale(torch, scale):  # noqa: F811
    """Every parameter's gradient against autograd of the loss in 64 bits, parameter by parameter, with the 6e-4 of the norm that 32 bits
    carry here (test_gpu_train.py).  Inputs of a thousandth, so that eps counts in x's norm."""
    from paper_1805_01993_amd.train import Trainer
    t = Trainer(4, 2, 72, 136, 50, "f32", dropout=0.0, residual_scale=scale)
    t.x *= 1e-3
    p = {k: v.double().detach().requires_grad_() for k, v in t.parameters().items()}
    norm = lambda v, w: v / torch.sqrt(v.square().mean(1, keepdim=True) + 1e-6) * w  # noqa: E731
    x, target = t.x.double(), t.target.double()
    a = norm(x, p["w_pre"]) @ p["W_in"].t().contiguous()
    f = (torch.nn.functional.silu(a[:, :136]) * a[:, 136:]) @ p["W_out"].t().contiguous()
    y = scale * x + p["gate"] * norm(f, p["w_post"])
    ((y - target).square().sum() / 2).backward()
    t.step(0, rate=0.0)
    got, at = t.Phi.view(-1).double(), 0
    for name, v in p.items():
        part = got[at:at + v.numel()].view(v.shape)
        at += v.numel()
        assert (part - v.grad).norm() <= 6e-4 * v.grad.norm(), name
