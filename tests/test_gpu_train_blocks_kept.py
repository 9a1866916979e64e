"""examples/train_blocks.py: what it says that it keeps between the passes is all that it keeps."""
import os
import sys

import pytest
import torch

import paper_2303_02868_amd as apm

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_a_block_more_costs_what_is_counted():
    from train_blocks import Network

    def measured(blocks):
        """Bytes that a network of so many blocks holds beside its pages, what it says that it keeps, its parameters, and how many tensors these are."""
        before = torch.cuda.memory_allocated()
        net = Network(1024, 128, 256, blocks)
        return torch.cuda.memory_allocated() - before, net.kept()[1], sum(net.p.numels), 10 * blocks + 5 * blocks, net

    *few, first = measured(2)
    *many, second = measured(7)
    held, kept, parameters, tensors = (b - a for a, b in zip(few, many))
    # parameters and gradients in bf16; the allocator rounds each tensor up to 512 bytes
    assert kept + 4 * parameters <= held <= kept + 4 * parameters + 512 * tensors
    del first, second


def test_the_backward_pass_reads_nothing_else():
    from train_blocks import Network
    net = Network(300, 200, 328, 2, apm.APM_CKPT_I8)
    g = torch.Generator(device="cuda:0").manual_seed(5)
    x, dn = torch.randn(300, 200, device="cuda:0", generator=g), torch.randn(300, 200, device="cuda:0", generator=g).bfloat16()
    net.forward(x)
    net.backward(dn)
    want = {n: t.clone() for n, t in net.p.grad.items()}
    net.forward(x)
    for t in (net.y, net.n, net.branch, net.u_back, net.dy, net.dn, net.dbranch, net.room.view(torch.float32)):
        t.fill_(float("nan"))
    net.backward(dn)
    for name, t in net.p.grad.items():
        assert torch.equal(t, want[name]), name
