"""examples/train_experts.py: sorting, lookups, products per group, dropout, the kept tensors and the page update together."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle.tokens as T

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def reference(net, words, dy):
    """Output and gradients by torch's differentiation in 64 bits, of the same parameters, experts and masks; nothing in 8 bits, nothing rounded."""
    p = {k: v.detach().double().requires_grad_() for k, v in net.p.value.items()}
    shape, seed = (net.tokens, net.width), net.seed + int(net.step_word)
    bound = round(net.drop * 65536)
    masks = [torch.from_numpy((T.dropout_bits(*shape, seed, layer) >= bound) * (65536 / (65536 - bound))).to(dy.device) for layer in (0, 1)]
    x = p["E"][words] * net.width ** 0.5 * masks[0]
    n = x / torch.sqrt(x.square().mean(dim=1, keepdim=True) + 1e-5) * p["norm"]
    picked = net.by_expert.ids.long()
    weights = torch.softmax((n @ p["R"].T).gather(1, picked), 1)
    branch = torch.zeros_like(n)
    for e in range(net.experts):
        at, j = (picked == e).nonzero(as_tuple=True)
        a = (n[at] @ p["W1"][e].T + p["b1"][e]).relu().square()
        branch = branch.index_add(0, at, weights[at, j, None] * (a @ p["W2"][e].T))
    y = x + branch * masks[1]
    (y * dy.double()).sum().backward()
    return y.detach(), {k: v.grad for k, v in p.items()}


def test_gradients_of_a_whole_network():
    """bf16 products are off by up to 2^-9 of their inputs, 8-bit tensors by about 0.6 % of their values, a few of which come together in one gradient and
    partly average out: a bound of five times that, in the 2-norm."""
    from train_experts import Network
    net = Network(300, 700, 72, 136, 5, seed=3)
    g = torch.Generator(device="cuda:0").manual_seed(5)
    words, dy = torch.randint(0, 700, (300,), device="cuda:0", generator=g) % 350, torch.randn(300, 72, device="cuda:0", generator=g)
    net.step_word.fill_(7)
    got = net.forward(words).clone()
    y, want = reference(net, words, dy)
    assert float((got.double() - y).norm() / y.norm()) < 0.01
    net.backward(dy)
    for name, grad in net.p.grad.items():
        assert float((grad.double() - want[name]).norm() / want[name].norm()) < 0.03, name
    assert bool((net.p.grad["E"][350:] == 0).all())


def test_a_step_runs_and_leaves_untouched_pages_alone():
    """A page of words that no token has keeps its bits; another step draws another mask."""
    from train_experts import Network
    net = Network(64, 4096, 64, 64, 4)
    words = torch.arange(64, device="cuda:0")
    before = net.p.value["E"].clone()
    first = net.forward(words).clone()
    net.backward(first)
    net.p.step(1e-2)
    after = net.p.value["E"]
    assert not torch.equal(after[:64], before[:64]) and torch.equal(after[64:], before[64:])
    assert int(net.p.skipped.sum()) >= 63
    net.step_word.fill_(1)
    net.p.value["E"].copy_(before)
    assert not torch.equal(net.forward(words) == 0, first == 0)


def test_the_example_runs():
    from train_experts import train
    losses = train(steps=3, tokens=512, words=900, width=64, hidden=128, experts=4, say=lambda *_: None)
    assert len(losses) == 3 and all(np.isfinite(losses))
