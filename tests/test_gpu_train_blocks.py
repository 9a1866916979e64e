"""examples/train_blocks.py: the activation calls and the page update together."""
import os
import sys

import pytest
import torch

import paper_2303_02868_amd as apm

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def reference(net, x, dn):
    """The network's output and gradients by torch's differentiation in 64 bits, of the same parameters; nothing kept in 8 bits, nothing rounded."""
    p = {k: v.detach().double().requires_grad_() for k, v in net.p.value.items()}
    rms = lambda v: v / torch.sqrt(v.square().mean(dim=1, keepdim=True) + 1e-5)
    y = x.double()
    n = rms(y) * p["0.pre"]
    for i in range(1, net.blocks + 1):
        a = (n @ p[f"{i}.w1"].T).relu().square()
        y = y + p[f"{i}.gate"] * rms(a @ p[f"{i}.w2"].T) * p[f"{i}.post"]
        n = rms(y) * p[f"{i}.pre"]
    (n * dn.double()).sum().backward()
    return n.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("form,worst", [(apm.APM_CKPT_I8, 0.03), (apm.APM_CKPT_F8, 0.08)])
def test_gradients_of_a_whole_network(form, worst):
    """bf16 products are off by up to 2^-9 of their inputs, 8-bit tensors by about 0.6 % (I8) and 2.6 % (F8) of their values, a few of which come
    together in one gradient and partly average out: bounds of five and three times that, in the 2-norm."""
    from train_blocks import Network
    net = Network(300, 200, 328, 2, form)
    g = torch.Generator(device="cuda:0").manual_seed(5)
    x, dn = torch.randn(300, 200, device="cuda:0", generator=g), torch.randn(300, 200, device="cuda:0", generator=g).bfloat16()
    n, want = reference(net, x, dn)
    got = net.forward(x)
    assert float((got.double() - n).norm() / n.norm()) < 0.01
    net.backward(dn)
    for name, grad in net.p.grad.items():
        assert float((grad.double() - want[name]).norm() / want[name].norm()) < worst, name


@pytest.mark.parametrize("form", [apm.APM_CKPT_I8, apm.APM_CKPT_F8])
def test_training_learns(form):
    from train_blocks import train
    losses = train(steps=60, tokens=512, width=128, hidden=256, blocks=2, form=form, say=lambda *_: None)
    assert losses[-1] < 0.6 * losses[0]
