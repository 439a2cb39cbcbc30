"""The example that trains a small network through the masked products and the calls around them: its loss falls, and
one step's gradients agree with float64 autograd of the unmasked network (2-norm; the masking noise at 100 times the
inputs leaves the products' 1e-3 class, as in the chain test)."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("masked_training", os.path.join(ROOT, "examples", "masked_training.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_loss_falls(example):
    losses = example.main(steps=25)
    assert losses[0] > 4.0 and losses[-1] < 0.5 * losses[0]


def test_gradients_of_a_step(example):
    net = example.Network(seed=3)
    x, target = next(example.images(net.n, seed=4))
    loss, grads, verdicts = net.gradients(x, target)
    assert all(v["ok"] == 1 and v["n_flagged"] == 0 for v in verdicts)
    params = {"V": net.V, **{f"{k}{i}": getattr(net, k)[i] for i in range(2) for k in ("W", "gamma", "beta")}}
    leaves = {k: v.detach().double().cpu().requires_grad_(True) for k, v in params.items()}
    a = x.double().cpu().permute(0, 3, 1, 2)
    for i in range(2):
        z = torch.nn.functional.conv2d(a, leaves[f"W{i}"].permute(0, 3, 1, 2), padding=1)
        z = torch.nn.functional.group_norm(z, example.GROUPS, leaves[f"gamma{i}"], leaves[f"beta{i}"], example.EPS)
        a = torch.nn.functional.silu(z)
    logits = a.permute(0, 2, 3, 1).reshape(net.n, -1) @ leaves["V"].T
    want = torch.nn.functional.cross_entropy(logits, target.cpu())
    want.backward()
    assert abs(float(loss) - float(want)) <= 1e-3 * float(want)
    for k, leaf in leaves.items():
        got = grads[k].double().cpu()
        assert float((got - leaf.grad).norm()) <= 5e-3 * float(leaf.grad.norm()), k
    net.ctx.close()


def test_every_step_trains(example):
    """The loss falls over the whole run and never reaches zero, where the gradients would be rounding noise."""
    losses = example.main(steps=25)
    fives = [sum(losses[i:i + 5]) / 5 for i in range(0, 25, 5)]
    assert all(b < a for a, b in zip(fives, fives[1:])) and min(losses) > 0.1
