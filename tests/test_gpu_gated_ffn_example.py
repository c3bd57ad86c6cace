"""GPU: the example training step -- feed-forward block, dropout, compressed offload of the hidden map -- against torch's
autograd with the same dropout masks, and that training lowers the loss."""
import importlib.util
import os

import pytest
import torch

from oracle import dropout_numpy as dn

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_ffn_training_step.py")


def example():
    spec = importlib.util.spec_from_file_location("gated_ffn_training_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_of_a_step_are_those_of_autograd():
    m, k, f, p, step = 300, 256, 712, 0.2, 3
    block = example().GatedFfn(m, k, f, p, seed=9, dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn(m, k, generator=g, device="cuda") for _ in range(2))
    y, ticket = block.forward(x, step)
    grads = block.backward(x, dy, ticket, step)
    block.close()

    mask = lambda cols, seq: torch.from_numpy(dn.keep_mask(m, cols, p, 9, seq)).cuda().double() * dn.scale(p)
    leaves = [t.double().clone().requires_grad_() for t in (x, block.wg, block.wu, block.wd)]
    xx, wg, wu, wd = leaves
    h = torch.relu(xx @ wg.t()) * (xx @ wu.t()) * mask(f, 2 * step)
    want = xx + (h @ wd.t()) * mask(k, 2 * step + 1)
    want.backward(dy.double())
    # torch's own products here run in 32 bits (sums of up to 712 terms): 2^-16 of the whole is far above both sides' losses
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    assert rel(y, want.detach()) < 2.0 ** -16
    for got, leaf in zip(grads, leaves):
        assert rel(got, leaf.grad) < 2.0 ** -14      # a gate at zero may fall on either side


def test_training_lowers_the_loss(capsys):
    losses = example().main(["--tokens", "512", "--width", "256", "--hidden", "712", "--steps", "6"])
    assert losses[-1] < losses[0]
    assert "over the host link" in capsys.readouterr().out
