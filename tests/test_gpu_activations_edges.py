"""The activation calls where values leave the number range, where rows are very wide, and on every path of the weight gradients."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest
import torch

import oracle.activations as A
import paper_2303_02868_amd as apm
from test_gpu_activations import BF16, DEV, F32, Join, check_weight_grad, f64, kept_blank, random_kept, room_for

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


# ---- 8-bit matrices of very wide rows -----------------------------------------------------------

@pytest.mark.parametrize("fmt", [A.I8, A.F8])
def test_rows_of_fp32_beyond_4_gib(fmt):
    """A buffer flattened to one row: byte offsets of its columns pass 32 bits at column 2^30."""
    far = 2 ** 30
    cols = far + 1005
    x = torch.empty(1, cols, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(9)
    for at in range(0, cols, 1 << 28):
        x[:, at:at + (1 << 28)].normal_(generator=g)
    x[:, far:] *= 8.0                                               # no scale byte as at the row's beginning
    kept = kept_blank(1, cols)
    apm.apm_ckpt_write(x, apm.make_ckpt(*kept, fmt))
    whole = kept_blank(far >> 15, 1 << 15)                          # the same blocks, as rows of 2^15 columns
    apm.apm_ckpt_write(x[0, :far].view(far >> 15, 1 << 15), apm.make_ckpt(*whole, fmt))
    assert torch.equal(kept[0][0, :far], whole[0].view(-1)) and torch.equal(kept[1][0, :far // 32], whole[1].view(-1))
    q, s = A.encode(f64(x[:, far:]), fmt)
    assert np.array_equal(kept[0][:, far:].cpu().numpy(), q) and np.array_equal(kept[1][:, far // 32:].cpu().numpy(), s)
    first = x[:, :1000].clone()
    back = x.fill_(7.0)
    apm.apm_ckpt_read(apm.make_ckpt(*kept, fmt), back)
    assert np.array_equal(f64(back[:, far:]), A.decode(q, s, fmt))
    q, s = A.encode(f64(first)[:, :992], fmt)
    assert np.array_equal(f64(back[:, :992]), A.decode(q, s, fmt))
    again = torch.empty(far >> 15, 1 << 15, device=DEV)
    apm.apm_ckpt_read(apm.make_ckpt(*whole, fmt), again)
    assert torch.equal(back[0, :far], again.view(-1))


# ---- join gradients: values that are no numbers -------------------------------------------------

@pytest.mark.parametrize("rows,cols", [(6, 100), (400, 600), (5, 9000)])
@pytest.mark.parametrize("gate", [A.NO_GATE, A.CHANNEL, A.TOKEN, A.FULL])
def test_without_a_norm_the_gradient_of_the_branch_does_not_depend_on_what_was_kept(rows, cols, gate):
    """dbranch = gate D post.weight: a block of the branch that stands for NaN reaches the gradients of gate and weight alone."""
    J = Join(rows, cols, post=A.NONE, gate=gate)
    join = J.join()
    apm.apm_norm_join_forward(join)
    J.kept2[1][2, 1] = 255                                          # row 2, channels 32 .. 63
    apm.apm_norm_join_backward(join, J.grads(join, dgate=None, dpost_weight=None), room_for(rows, cols))
    alone = J.dbranch.clone()
    assert bool(torch.isfinite(alone).all())
    for more in ({}, {"dgate": None}, {"dpost_weight": None}):
        J.dbranch.fill_(7.0)
        apm.apm_norm_join_backward(join, J.grads(join, **more), room_for(rows, cols))
        assert torch.equal(J.dbranch, alone)
    apm.apm_norm_join_backward(join, J.grads(join), room_for(rows, cols))
    nan = torch.isnan(J.dw2)
    assert bool(nan[32:64].all()) and int(nan.sum()) == 32


@pytest.mark.parametrize("rows,cols", [(6, 100), (400, 600), (5, 9000)])
def test_a_gradient_that_is_missing_is_zero_whatever_it_would_be_multiplied_by(rows, cols):
    """Without dn nothing of the first norm is needed: neither an infinite weight nor what rstd holds reaches a result."""
    J = Join(rows, cols, gate=A.TOKEN)
    join = J.join()
    apm.apm_norm_join_forward(join)
    J.w1[3], J.w1[40] = INF, float("nan")
    J.r1.fill_(float("nan"))
    apm.apm_norm_join_backward(join, J.grads(join, dn=None), room_for(rows, cols))
    want = J.scale * J.dy.float()
    assert bool(((J.dx.float() - want).abs() <= 2.0 ** -8 * want.abs()).all())
    for t in (J.dbranch, J.dgate, J.dw2, J.db2):
        assert bool(torch.isfinite(t).all())
    assert bool((J.dw1 == 0).all()) and bool((J.db1 == 0).all())


@pytest.mark.parametrize("rows,cols", [(1, 100), (5, 100), (5, 700), (300, 100), (301, 700), (771, 2000), (3, 9000)])
@pytest.mark.parametrize("gate", [A.CHANNEL, A.TOKEN])
def test_rows_that_are_not_there_add_nothing_under_an_infinite_weight(rows, cols, gate):
    """Without a first norm D = dy + dn pre.weight: with a weight of +inf, and dn and hat2 positive, the sums over rows are +inf, whatever their number."""
    J = Join(rows, cols, F32, F32, F32, pre=A.NONE, gate=gate)
    J.branch.abs_().add_(0.1)
    J.dn.abs_().add_(0.1)
    J.gate.abs_().add_(0.1)
    join = J.join()
    apm.apm_norm_join_forward(join)
    J.w1[3] = INF
    J.w2[3] = 0.5
    J.kept2[0][:, 3] = 64                                           # in I8: 1 times the block's scale
    apm.apm_norm_join_backward(join, J.grads(join), room_for(rows, cols))
    for t in (J.dw2, J.db2):
        assert float(t[3]) == INF
    others = torch.arange(cols, device=DEV) != 3
    assert bool(torch.isfinite(J.dw2[others]).all()) and bool(torch.isfinite(J.db2[others]).all()) and bool((J.dx[:, 3] == INF).all())


# ---- weight gradients: every tile, with and without parts ---------------------------------------

def path(tokens, out, k, groups=0):
    """The tile that the rule takes for a shape, and into how many parts it splits the tokens."""
    g = apm.apm_weight_grad()
    g.tokens, g.out, g.n_groups, g.offsets, g.dw_group_stride = tokens, out, groups, 4096 if groups else None, out * k
    setattr(g, "in", k)
    g.dy, g.kept, g.dw = apm.apm_matrix(4096, out, apm.APM_BF16, 0), apm.apm_ckpt(4096, 4096, k, -(-k // 32), 0, 0), apm.apm_matrix(4096, k, apm.APM_F32, 0)
    size = apm.apm_ckpt_weight_grad_workspace_bytes(g)
    return apm.lib().apm_test_weight_grad_tile(C.byref(g)), max(1, size // (4 * max(1, groups) * out * (k + 1)))


def shares(tokens, groups):
    """Uneven groups, the second of them empty."""
    if not groups:
        return None
    cut = np.sort(np.random.default_rng(tokens).integers(0, tokens, groups - 1)).tolist()
    offsets = [0] + cut + [tokens]
    offsets[2] = offsets[1] if groups > 2 else offsets[2]
    return offsets if groups > 2 else [0, 0, tokens]


SHAPES = [  # tile, parts, tokens, out, in, groups
    (256, 1, 700, 2100, 4000, 0), (256, 1, 1500, 520, 2000, 8), (256, 3, 3000, 2100, 2100, 0), (256, 3, 6000, 1500, 1500, 2),
    (128, 1, 500, 1000, 4000, 0), (128, 1, 1500, 200, 4000, 4), (128, 4, 4000, 130, 4000, 0), (128, 4, 6000, 200, 2000, 2),
    (64, 1, 500, 130, 300, 0), (64, 1, 500, 130, 130, 3), (64, 6, 700, 130, 130, 0), (64, 6, 1500, 200, 130, 2),
]


@pytest.mark.parametrize("tile,parts,tokens,out,k,groups", SHAPES)
@pytest.mark.parametrize("fmt,dtype,weight,bias,db,accumulate", [(A.I8, F32, True, True, True, False), (A.F8, BF16, False, False, False, False),
                                                                  (A.F8, F32, True, False, True, True), (A.I8, BF16, True, False, False, True)])
def test_every_tile_with_and_without_parts(tile, parts, tokens, out, k, groups, fmt, dtype, weight, bias, db, accumulate):
    assert path(tokens, out, k, groups) == (tile, parts)
    check_weight_grad(tokens, out, k, fmt, dtype, weight, bias, db, offsets=shares(tokens, groups), accumulate=accumulate)


@pytest.mark.parametrize("tile,parts,tokens,out,k,groups", [s for s in SHAPES if s[5]])
@pytest.mark.parametrize("accumulate", [False, True])
def test_groups_without_tokens_take_no_weight_and_no_bias(tile, parts, tokens, out, k, groups, accumulate):
    assert path(tokens, out, k, groups) == (tile, parts)
    kept, _ = random_kept(tokens, k, A.I8, 2)
    dy = torch.randn(tokens, out, device=DEV).bfloat16()
    w = torch.full((k,), INF, device=DEV)
    old = 3.0 if accumulate else 0.0
    dw, db = torch.full((groups, out, k), 3.0, device=DEV), torch.full((groups, out), 3.0, device=DEV)
    grad = apm.make_weight_grad(dy, apm.make_ckpt(*kept, A.I8), dw, db=db, weight=w, bias=w, offsets=torch.tensor(shares(tokens, groups), device=DEV),
                                accumulate=accumulate)
    size = apm.apm_ckpt_weight_grad_workspace_bytes(grad)
    assert (size > 0) == (parts > 1)
    apm.apm_ckpt_weight_grad(grad, torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if size else None)
    empty = 1 if groups > 2 else 0
    assert bool((dw[empty] == old).all()) and bool((db[empty] == old).all())
    assert not bool(torch.isfinite(dw[-1]).any())


# ---- what the smallest and largest values become ------------------------------------------------

@pytest.mark.parametrize("fmt", [A.I8, A.F8])
def test_every_code_and_scale_read_to_bf16_is_the_nearest_bf16_number(fmt):
    """Nothing is rounded but what no bf16 number is: F8 values under the scale bytes 0 to 2, and 2^128."""
    q = torch.arange(256, device=DEV).to(torch.uint8).repeat(256, 1)
    q[:, [128] if fmt == A.I8 else [127, 255]] = 0
    s = torch.arange(256, device=DEV).to(torch.uint8)[:, None].repeat(1, 8).contiguous()
    out = torch.empty(256, 256, dtype=BF16, device=DEV)
    apm.apm_ckpt_read(apm.make_ckpt(q, s, fmt), out)
    exact = A.decode(q.cpu().numpy(), s.cpu().numpy(), fmt)
    with np.errstate(over="ignore"):
        nearest = torch.from_numpy(exact.astype(np.float32)).bfloat16().double().numpy()
    assert np.array_equal(f64(out), nearest, equal_nan=True)
    rounded = ~np.isnan(exact) & (nearest != exact)
    rows = np.unique(np.nonzero(rounded)[0]).tolist()
    if fmt == A.I8:
        assert rows == []
    else:
        assert rows[:3] == [0, 1, 2] and all(np.isinf(nearest[r][rounded[r]]).all() for r in rows[3:])


def test_accumulation_rounds_as_stated():
    """What is added to dw: v weight + bias (sum of dy) in one rounding to fp32, the sum with what is there in another, the type in a third."""
    dy = torch.full((1, 1), 1.0, device=DEV).bfloat16()
    kept = torch.full((1, 1), 64, dtype=torch.uint8, device=DEV), torch.full((1, 1), 127, dtype=torch.uint8, device=DEV)   # 1.0
    w = torch.full((1,), 1 + 2.0 ** -23, device=DEV)
    b = torch.full((1,), 2.0 ** -24, device=DEV)                   # w + b is a tie: 1 + 2^-22, the even one
    for dtype, old, want in ((F32, 4.0, 5.0), (F32, 2.0 ** -23, 1 + 3 * 2.0 ** -23), (BF16, 2.0 ** -7, 1 + 2.0 ** -7), (BF16, 2.0 ** -8, 1 + 2.0 ** -7)):
        dw, db = torch.full((1, 1), old, dtype=dtype, device=DEV), torch.full((1,), old, dtype=dtype, device=DEV)
        grad = apm.make_weight_grad(dy, apm.make_ckpt(*kept, A.I8), dw, db=db, weight=w, bias=b, accumulate=True)
        apm.apm_ckpt_weight_grad(grad)
        step = torch.tensor(1 + 2.0 ** -22, device=DEV) + torch.tensor(old, device=DEV)        # each in fp32
        assert float(dw) == float(step.to(dtype)) == want
        assert float(db) == float((torch.tensor(1.0, device=DEV) + old).to(dtype))
