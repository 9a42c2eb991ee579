"""The training loop with a teacher: gradients against automatic differentiation of the definition, the same bits on every node, the
command.  Needs a GPU."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def trainer(*args, **more):
    from paper_1805_01993_amd.train import Trainer
    torch.cuda.set_device(0)
    return Trainer(*args, **more)


@pytest.mark.parametrize("mode", ["bf16", "f16", "f32", "h32"])
@pytest.mark.parametrize("width,tokens", [(72, [40, 0, 1, 77, 33, 64]), (72, [5, 0, 1, 9, 3, 6]), (1032, [20, 0, 1, 7, 33, 14])])
def test_every_node_maps_its_files_to_the_same_bits(mode, width, tokens):
    """Also nodes with so few rows that a product of them alone would take another kernel."""
    t = trainer(4, 2, width, 136, tokens, mode, dropout=0.2, teacher=9)
    t.map(t.every, t.x, t.target, t.V, seed=5)
    assert bool((t.V != 0).any())
    for node in range(4):
        files, V = t.own_rows(node, 5)
        assert torch.equal(V, t.V[0, files])


def test_the_sum_is_the_gradient_of_the_whole():
    """Phi against autograd of the loss over all tokens, in 64 bits, from the teacher's answers as they are; the bound as without a teacher
    (test_gpu_train.py), the loss's own gradient adds some 400 roundings of 2^-24, 2.4e-5."""
    from paper_1805_01993_amd.train import TEMPERATURE as T
    t = trainer(4, 2, 72, 136, 50, "f32", dropout=0.0, teacher=10)
    t.step(0, rate=0.0)
    p = {k: v.double().detach().requires_grad_() for k, v in t.parameters().items()}
    norm = lambda v, w: v / torch.sqrt(v.square().mean(1, keepdim=True) + 1e-6) * w  # noqa: E731
    x, s = t.x.double(), t.every
    a = norm(x, p["w_pre"]) @ p["W_in"].t().contiguous()
    f = (torch.nn.functional.silu(a[:, :136]) * a[:, 136:]) @ p["W_out"].t().contiguous()
    y = t.scale * x + p["gate"] * norm(f, p["w_post"])
    index = s["index"].long()
    teacher = torch.softmax(torch.cat((s["value"].double() / T, s["rest"].double()[:, None]), 1), 1)
    log_q = torch.log_softmax(y / T, 1)
    listed = torch.zeros_like(log_q, dtype=torch.bool).scatter_(1, index, True)
    rest = torch.logsumexp(log_q.masked_fill(listed, -math.inf), 1)
    student = torch.cat((log_q.gather(1, index), rest[:, None]), 1)
    loss = T * T * (teacher * (teacher.log() - student)).sum(1)
    loss.sum().backward()
    assert torch.allclose(s["loss"].double(), loss.detach(), rtol=1e-4, atol=1e-5)
    want = torch.cat([p[k].grad.reshape(-1) for k in t.sizes])
    got = t.Phi.view(-1)[:want.numel()].double()
    assert (got - want).norm() <= 6.3e-4 * want.norm()


def test_the_teachers_answers_are_its_packed_products():
    import teacher_reference as R
    t = trainer(4, 2, 72, 136, 50, "bf16", teacher=10)
    t.step(0)
    s, rows = t.every, t.x.shape[0]
    q, scale = R.quantise(t.x.double())
    assert torch.equal(s["q"][:rows].cpu(), q) and torch.equal(s["scale"][:rows].cpu(), scale)
    want, off = R.product(R.values(q, scale), R.values(*t.packed), "bf16")
    assert bool(((s["logits"][:rows, :].double().cpu() - want).abs() <= off).all())
    index, value, _ = R.top(s["logits"][:rows], 10, 2.0)
    assert torch.equal(s["index"].cpu(), index) and torch.equal(s["value"].double().cpu(), value)


def test_the_command(capsys):
    from paper_1805_01993_amd.train import main
    assert main(["--nodes", "4", "--width", "64", "--hidden", "96", "--tokens", "16", "--steps", "3", "--mode", "f16", "--teacher", "8"]) == 0
    assert "the same bits: True" in capsys.readouterr().out
