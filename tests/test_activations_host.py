"""Refusals of the activation calls: they come from the arguments alone, before anything is launched, so they need no GPU."""
import ctypes as C

import pytest

import paper_2303_02868_amd as apm

PTR = 1 << 20          # an address that nothing may be read from here


def matrix(data=PTR, stride=64, dtype=apm.APM_BF16):
    return apm.apm_matrix(data, stride, dtype, 0)


def ckpt(q=PTR, scale=PTR, q_stride=64, scale_stride=2, format=apm.APM_CKPT_I8):
    return apm.apm_ckpt(q, scale, q_stride, scale_stride, format, 0)


def refused(rc, code, word):
    assert rc == code and word in apm.apm_last_error(), (rc, apm.apm_last_error())


@pytest.mark.parametrize("call", ["apm_ckpt_write", "apm_ckpt_read"])
def test_8_bit_matrices(call):
    def go(rows=4, cols=64, x=None, c=None):
        x, c = x or matrix(), c or ckpt()
        return getattr(apm.lib(), call)(rows, cols, *((x, c) if call.endswith("write") else (c, x)), None)

    refused(go(rows=-1), apm.APM_EINVAL, "bad size")
    refused(go(cols=0), apm.APM_EINVAL, "bad size")
    refused(go(cols=2 ** 31), apm.APM_EINVAL, "bad size")
    refused(go(x=matrix(None)), apm.APM_EINVAL, "x is missing")
    refused(go(x=matrix(dtype=2)), apm.APM_EINVAL, "dtype")
    refused(go(x=matrix(PTR + 1)), apm.APM_EINVAL, "aligned")
    refused(go(x=matrix(PTR + 2, dtype=apm.APM_F32)), apm.APM_EINVAL, "aligned")
    refused(go(x=matrix(stride=-64)), apm.APM_EINVAL, "stride")
    refused(go(c=ckpt(q=None)), apm.APM_EINVAL, "missing")
    refused(go(c=ckpt(scale=None)), apm.APM_EINVAL, "missing")
    refused(go(c=ckpt(format=2)), apm.APM_EINVAL, "format")
    if call.endswith("write"):
        refused(go(c=ckpt(q_stride=63)), apm.APM_EINVAL, "stride")
        refused(go(c=ckpt(scale_stride=1)), apm.APM_EINVAL, "stride")
    else:
        refused(go(x=matrix(stride=63)), apm.APM_EINVAL, "stride")
    refused(getattr(apm.lib(), call)(4, 64, None, None, None), apm.APM_EINVAL, "missing")
    assert go(rows=0) == apm.APM_OK


def join(rows=4, cols=64, **over):
    j = apm.apm_norm_join()
    j.rows, j.cols, j.residual_scale = rows, cols, 1.0
    j.x, j.branch, j.y, j.n, j.gate = matrix(), matrix(), matrix(), matrix(), matrix()
    j.gate_kind = apm.APM_GATE_FULL
    for m in (j.pre, j.post):
        m.kind, m.eps, m.ckpt, m.rstd = apm.APM_NORM_RMS, 1e-6, ckpt(), PTR
    for path, v in over.items():
        at, names = j, path.split("__")
        for n in names[:-1]:
            at = getattr(at, n)
        setattr(at, names[-1], v)
    return j


def test_join_forward():
    go = lambda **o: apm.lib().apm_norm_join_forward(join(**o), None)
    refused(go(rows=-1), apm.APM_EINVAL, "bad size")
    refused(go(cols=0), apm.APM_EINVAL, "bad size")
    refused(go(cols=apm.APM_JOIN_MAX_COLS + 1), apm.APM_EINVAL, "bad size")
    refused(go(x=matrix(None)), apm.APM_EINVAL, "x is missing")
    refused(go(y=matrix(stride=32)), apm.APM_EINVAL, "y: a row stride")
    refused(go(n=matrix(stride=32)), apm.APM_EINVAL, "n: a row stride")
    refused(go(gate_kind=4), apm.APM_EINVAL, "gate kind")
    refused(go(gate_kind=apm.APM_GATE_NONE), apm.APM_EINVAL, "contradict")
    refused(go(gate=matrix(None)), apm.APM_EINVAL, "contradict")
    refused(go(pre__kind=3), apm.APM_EINVAL, "norm kind")
    refused(go(post__kind=-1), apm.APM_EINVAL, "norm kind")
    refused(go(pre__eps=-1.0), apm.APM_EINVAL, "eps")
    refused(go(post__eps=float("nan")), apm.APM_EINVAL, "eps")
    refused(go(pre__weight=apm.apm_vector(PTR, 7, 0)), apm.APM_EINVAL, "dtype")
    refused(go(post__bias=apm.apm_vector(PTR + 1, apm.APM_BF16, 0)), apm.APM_EINVAL, "aligned")
    refused(go(pre__ckpt=ckpt(q_stride=1)), apm.APM_EINVAL, "pre.ckpt")
    refused(go(post__ckpt=ckpt(scale=None)), apm.APM_EINVAL, "post.ckpt")
    refused(go(pre__rstd=PTR + 2), apm.APM_EINVAL, "rstd")
    refused(go(branch=matrix(None)), apm.APM_EINVAL, "no branch")
    refused(go(y=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "different types")
    refused(go(n=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "different types")
    refused(go(branch=matrix(dtype=apm.APM_F32), n=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "not supported")
    refused(apm.lib().apm_norm_join_forward(None, None), apm.APM_EINVAL, "missing")
    assert go(rows=0) == apm.APM_OK


def test_join_backward():
    need = apm.apm_norm_join_workspace_bytes(4, 64)
    assert need > 0 and apm.apm_norm_join_workspace_bytes(-1, 64) == 0 and apm.apm_norm_join_workspace_bytes(4, 0) == 0

    def go(j=None, room=PTR, size=need, **over):
        g = apm.apm_norm_join_grads(*[matrix() for _ in range(5)], *[apm.apm_vector(PTR, apm.APM_F32, 0) for _ in range(4)])
        for k, v in over.items():
            setattr(g, k, v)
        return apm.lib().apm_norm_join_backward(j or join(), g, room, size, None)

    none = matrix(None)
    refused(go(dn=none, dy=none), apm.APM_EINVAL, "neither")
    refused(go(dx=matrix(stride=1)), apm.APM_EINVAL, "dx")
    refused(go(dbranch=matrix(stride=1)), apm.APM_EINVAL, "dbranch")
    refused(go(dgate=matrix(stride=1)), apm.APM_EINVAL, "dgate")
    refused(go(join(gate=none, gate_kind=apm.APM_GATE_NONE)), apm.APM_EINVAL, "dgate without a gate")
    refused(go(dx=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "different types")
    refused(go(dn=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "different types")
    refused(go(dn=matrix(dtype=apm.APM_F32), dbranch=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "not supported")
    refused(go(dpost_bias=apm.apm_vector(PTR + 1, apm.APM_BF16, 0)), apm.APM_EINVAL, "dpost_bias")
    refused(go(join(pre__ckpt=ckpt(q=None))), apm.APM_EINVAL, "pre.ckpt")
    refused(go(join(post__ckpt=ckpt(q=None))), apm.APM_EINVAL, "post.ckpt")
    refused(go(join(pre__rstd=None)), apm.APM_EINVAL, "pre.rstd")
    refused(go(join(post__rstd=None)), apm.APM_EINVAL, "post.rstd")
    refused(go(size=need - 1), apm.APM_ENOMEM, "workspace")
    refused(go(room=None), apm.APM_EINVAL, "workspace")
    refused(go(room=PTR + 8), apm.APM_EINVAL, "workspace")
    refused(go(join(cols=20000)), apm.APM_EINVAL, "bad size")
    refused(apm.lib().apm_norm_join_backward(None, None, None, 0, None), apm.APM_EINVAL, "missing")


def test_weight_gradient():
    def grad(**over):
        g = apm.apm_weight_grad()
        setattr(g, "in", 64)
        g.tokens, g.out, g.dy, g.kept, g.dw = 100, 64, matrix(), ckpt(), matrix()
        for k, v in over.items():
            setattr(g, k, v)
        return g

    def go(room=PTR, size=1 << 40, **over):
        return apm.lib().apm_ckpt_weight_grad(grad(**over), room, size, None)

    refused(go(tokens=-1), apm.APM_EINVAL, "bad size")
    refused(go(out=0), apm.APM_EINVAL, "bad size")
    refused(go(**{"in": 0}), apm.APM_EINVAL, "bad size")
    refused(go(n_groups=-1), apm.APM_EINVAL, "bad size")
    refused(go(n_groups=2), apm.APM_EINVAL, "offsets")
    refused(go(offsets=PTR), apm.APM_EINVAL, "offsets")
    refused(go(offsets=PTR + 4, n_groups=1), apm.APM_EINVAL, "offsets")
    refused(go(offsets=PTR, n_groups=2, dw_group_stride=64 * 64 - 1), apm.APM_EINVAL, "overlap")
    refused(go(dy=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "bf16")
    refused(go(dy=matrix(None)), apm.APM_EINVAL, "dy is missing")
    refused(go(kept=ckpt(q=None)), apm.APM_EINVAL, "kept")
    refused(go(dw=matrix(None)), apm.APM_EINVAL, "dw is missing")
    refused(go(dw=matrix(stride=63)), apm.APM_EINVAL, "dw")
    refused(go(weight=apm.apm_vector(PTR, 5, 0)), apm.APM_EINVAL, "weight")
    refused(go(db=apm.apm_vector(PTR + 1, apm.APM_BF16, 0)), apm.APM_EINVAL, "db")
    long = dict(tokens=100000)
    need = apm.apm_ckpt_weight_grad_workspace_bytes(grad(**long))
    assert need > 0
    refused(go(size=need - 1, **long), apm.APM_ENOMEM, "workspace")
    refused(go(room=None, **long), apm.APM_EINVAL, "workspace")
    refused(go(room=PTR + 4, **long), apm.APM_EINVAL, "workspace")
    refused(apm.lib().apm_ckpt_weight_grad(None, None, 0, None), apm.APM_EINVAL, "missing")
    assert apm.apm_ckpt_weight_grad_workspace_bytes(grad(out=0)) == 0


def test_rows_too_far_apart_for_an_address():
    far = 1 << 55
    refused(apm.lib().apm_ckpt_write(4, 64, matrix(stride=far), ckpt(), None), apm.APM_EINVAL, "stride")
    refused(apm.lib().apm_ckpt_read(4, 64, ckpt(q_stride=far), matrix(), None), apm.APM_EINVAL, "stride")
    refused(apm.lib().apm_norm_join_forward(join(x=matrix(stride=far)), None), apm.APM_EINVAL, "stride")
    g = apm.apm_weight_grad(100, 64, 64, 0, None, matrix(), ckpt(), apm.apm_vector(), apm.apm_vector(), matrix(stride=far))
    refused(apm.lib().apm_ckpt_weight_grad(g, None, 0, None), apm.APM_EINVAL, "stride")
    g = apm.apm_weight_grad(100, 64, 64, 9, PTR, matrix(), ckpt(), apm.apm_vector(), apm.apm_vector(), matrix(), 1 << 55)
    refused(apm.lib().apm_ckpt_weight_grad(g, None, 0, None), apm.APM_EINVAL, "apart")


def test_the_binding_looks_at_shapes_types_and_memory():
    torch = pytest.importorskip("torch")
    cpu = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        apm.make_matrix("x", cpu, 4, 64)
    with pytest.raises(ValueError, match="x"):
        apm.make_matrix("x", cpu, 4, 63)
    with pytest.raises(ValueError, match="strides"):
        apm.make_matrix("x", cpu.T, 64, 4)
    half = torch.zeros(4, 64, dtype=torch.float16)
    half.is_pinned = lambda: True                  # past the check of where it is
    with pytest.raises(ValueError, match="float16"):
        apm.make_matrix("x", half, 4, 64)
    with pytest.raises(ValueError, match="8-bit"):
        apm.make_ckpt(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 3, dtype=torch.uint8), 0)
    with pytest.raises(ValueError, match="w"):
        apm.make_vector("w", torch.zeros(5), 6)
    assert apm.make_matrix("x", None, 4, 64).data is None and apm.make_vector("w", None, 3).data is None


def test_structures_have_the_sizes_of_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ["apm_matrix", "apm_vector", "apm_ckpt", "apm_norm", "apm_norm_join", "apm_norm_join_grads", "apm_weight_grad"]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "apm.h"\nint main(void) {' + "".join(f'printf("%zu ", sizeof({n}));' for n in names) + "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    out = subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [C.sizeof(getattr(apm, n)) for n in names]
