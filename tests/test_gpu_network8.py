"""The example of a network in eight bits: its gradients are those of the network, and it learns."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("network_in_eight_bits", os.path.join(ROOT, "examples", "network_in_eight_bits.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _data(network):
    torch.manual_seed(2)
    return torch.randn(network.T, network.D, device="cuda").bfloat16(), torch.randint(0, network.V, (network.T,), device="cuda")


def test_gradients_are_those_of_the_network(example):
    # Entries of 8-bit operands are off by 2.6 % (three bits of mantissa) and 5.2 % (two) in the mean, a product by the root of the squares: 4 % forward, 6 % backward; two products
    # forward and two backward make 11 % in the gradient of the first layer, and ReLUs whose sign differs add some.  The dropped entries are the same: a wrong mask,
    # scale or operand gives errors of 40 % and more.
    network = example.Network(tokens=333, width=136, hidden=520, vocabulary=1003)
    x, target = _data(network)
    loss = network.step(x, target, 3).clone()
    kept = network.h.float() - x.float()
    ones, mask = torch.ones_like(network.h), torch.empty_like(network.h)
    example.cdl.cdl_dropout(ones, ones.numel(), network.p, network.seed, 3 * ((ones.numel() + 7) // 8), mask)
    assert ((mask == 0) <= (kept == 0)).all()
    w1, w2, E = (w.double().cpu().requires_grad_() for w in (network.up.w, network.down.w, network.E))
    X = x.double().cpu()
    h = mask.double().cpu() * (torch.relu(X @ w1.T) @ w2.T) + X
    plain = torch.nn.functional.cross_entropy(h @ E.T, target.cpu(), reduction="none")
    plain.mean().backward()
    for own, want in ((loss, plain.detach()), (network.down.d_w, w2.grad), (network.up.d_w, w1.grad), (network.d_E, E.grad)):
        assert (own.double().cpu() - want).norm() <= 0.2 * want.norm()


def test_it_learns(example):
    network = example.Network(tokens=256, width=128, hidden=256, vocabulary=1000)
    x, target = _data(network)
    losses = []
    for number in range(30):
        losses.append(network.step(x, target, number).mean().item())
        network.update(0.5)
    assert losses[0] > 6.0 and losses[-1] < 0.5 * losses[0]
