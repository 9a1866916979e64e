"""The activation calls where values leave the number range."""
from __future__ import annotations

import pytest
import torch

import oracle.activations as A
import paper_2303_02868_amd as apm
from test_gpu_activations import BF16, DEV, F32, random_kept

pytestmark = pytest.mark.gpu
INF = float("inf")


def same_bits(a, b):
    """NaNs of one bit pattern are the same here."""
    kind = torch.int16 if a.dtype == BF16 else torch.int32
    return torch.equal(a.view(kind), b.view(kind))


# ---- weight gradients: what is asked for beside dw ----------------------------------------------

def weight_grad(dy, kept, fmt, out_type=F32, **more):
    dw = torch.full((dy.shape[1], kept[0].shape[1]), 7.0, dtype=out_type, device=DEV)
    grad = apm.make_weight_grad(dy, apm.make_ckpt(*kept, fmt), dw, **more)
    size = apm.apm_ckpt_weight_grad_workspace_bytes(grad)
    apm.apm_ckpt_weight_grad(grad, torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if size else None)
    return dw, size > 0


@pytest.mark.parametrize("tokens,split", [(96, False), (2000, True)])
@pytest.mark.parametrize("fmt", [A.I8, A.F8])
@pytest.mark.parametrize("weight", [False, True])
def test_sums_of_dy_do_not_reach_dw_without_a_bias(tokens, split, fmt, weight):
    """dy's sum over the tokens overflows in output 3, and output 5 has an infinity: without a bias, or where it is zero, no sum of dy enters dw."""
    out, k = 70, 90
    kept, z = random_kept(tokens, k, fmt, 3)
    dy = torch.randn(tokens, out, device=DEV, generator=torch.Generator(device=DEV).manual_seed(tokens)).bfloat16()
    dy[:, 3] = 0
    dy[10, 3], dy[20, 3] = 3e38, 3e38                               # sums to 6e38, beyond fp32
    kept[0][[10, 20]] = 1 if fmt == A.I8 else 0x08                  # 2^-6, under a scale of 2^-7: products of 4e34
    kept[1][[10, 20]] = 120
    dy[30, 5] = INF
    w = torch.rand(k, device=DEV) + 0.5 if weight else None
    plain, splits = weight_grad(dy, kept, fmt, weight=w)
    assert splits == split and bool(torch.isfinite(plain[3]).all())
    db = torch.empty(out, device=DEV)
    with_sums, _ = weight_grad(dy, kept, fmt, weight=w, db=db)
    assert same_bits(plain, with_sums)
    assert torch.isinf(db[3]) and torch.isinf(db[5])
    zero = torch.zeros(k, device=DEV)
    for more in ({}, {"db": db}):
        with_zeros, _ = weight_grad(dy, kept, fmt, weight=w, bias=zero, **more)
        assert same_bits(plain, with_zeros)
    some = zero.clone()
    some[7] = 1.0
    with_one, _ = weight_grad(dy, kept, fmt, weight=w, bias=some)
    others = torch.arange(k, device=DEV) != 7
    assert same_bits(plain[:, others].contiguous(), with_one[:, others].contiguous()) and torch.isinf(with_one[3, 7])
