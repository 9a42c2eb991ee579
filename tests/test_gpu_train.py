"""The training loop on the emulated cluster: the loss falls, the summed gradients are the gradient of the whole data set by
automatic differentiation of the definition, and every node maps its files to the same bits.  Needs a GPU."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    torch.cuda.set_device(0)
    return torch


@pytest.mark.parametrize("mode", ["bf16", "f16", "f32", "h32"])
def test_every_node_maps_its_files_to_the_same_bits(torch, mode):
    from paper_1805_01993_amd.train import Trainer
    t = Trainer(4, 2, 72, 136, [40, 0, 1, 77, 33, 64], mode, dropout=0.2)
    t.map(t.every, t.x, t.target, t.V, seed=5)
    for node in range(4):
        files, V = t.own_rows(node, 5)
        assert len(files) == 3
        assert torch.equal(V, t.V[0, files])


def test_the_loss_falls(torch):
    from paper_1805_01993_amd.train import Trainer
    t = Trainer(5, 2, 128, 256, 48, "bf16", dropout=0.05)
    losses = [float(t.step(n)) for n in range(30)]
    assert all(math.isfinite(v) for v in losses) and losses[-1] < 0.7 * losses[0], losses


def test_the_sum_is_the_gradient_of_the_whole(torch):
    """Phi against autograd of the loss over all tokens, in 64 bits; fp32 carries sums of 300 tokens and 136 products, each at
    most (300 + 136 + 64) 2^-23 = 6e-5 of its terms off, and the terms of these gradients cancel to no less than a tenth."""
    from paper_1805_01993_amd.train import Trainer
    t = Trainer(4, 2, 72, 136, 50, "f32", dropout=0.0)
    p = {k: v.double().detach().requires_grad_() for k, v in t.parameters().items()}
    norm = lambda v, w: v / torch.sqrt(v.square().mean(1, keepdim=True) + 1e-6) * w  # noqa: E731
    x, target = t.x.double(), t.target.double()
    a = norm(x, p["w_pre"]) @ p["W_in"].t().contiguous()
    f = (torch.nn.functional.silu(a[:, :136]) * a[:, 136:]) @ p["W_out"].t().contiguous()
    y = t.scale * x + p["gate"] * norm(f, p["w_post"])
    ((y - target).square().sum() / 2).backward()
    t.step(0, rate=0.0)
    want = torch.cat([p[k].grad.reshape(-1) for k in t.sizes])
    got = t.Phi.view(-1)[:want.numel()].double()
    assert (got - want).norm() <= 6e-4 * want.norm()
    assert (t.Phi.view(-1)[want.numel():] == 0).all()


def test_the_command(torch, capsys):
    from paper_1805_01993_amd.train import main
    assert main(["--nodes", "4", "--width", "64", "--hidden", "96", "--tokens", "16", "--steps", "3", "--mode", "f16"]) == 0
    assert "the same bits: True" in capsys.readouterr().out
