"""The activation kernels against the 64-bit oracle, at the sizes and values where they can go wrong.

Tolerances.  u = 2^-24 is fp32's rounding; a sum of n fp32 terms in any order is off by at most n u times the sum of their sizes.
A bf16 result is rounded once more, by 2^-9 of itself; a bound of 2^-8 leaves that and the fp32 error of what is rounded.  Statistics of a row
(n terms, then a root and a division) are off by (n + 8) u relatively where all terms are positive.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.activations as A
import paper_2303_02868_amd as apm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def view(rows, cols, dtype, pad=0, shift=0, fill=None):
    """A rows x cols matrix inside a larger buffer of a known pattern: `pad` elements between rows, `shift` before the first."""
    flat = torch.full((shift + rows * (cols + pad) + 64,), 7.0 if fill is None else fill, dtype=dtype, device=DEV) if dtype != torch.uint8 else \
        torch.full((shift + rows * (cols + pad) + 64,), 0x55, dtype=dtype, device=DEV)
    return flat, torch.as_strided(flat, (rows, cols), (cols + pad, 1), shift)


def untouched(flat, m, value):
    """Everything of `flat` outside the matrix still holds `value`."""
    mask = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(mask, m.shape, m.stride(), m.storage_offset()).fill_(False)
    return bool((flat[mask] == value).all())


def kept_blank(rows, cols, pad=0):
    return torch.full((rows, cols + pad), 0x55, dtype=torch.uint8, device=DEV)[:, :cols], \
        torch.full((rows, -(-cols // 32) + pad), 0x55, dtype=torch.uint8, device=DEV)[:, :-(-cols // 32)]


def bytes_of(pair):
    return pair[0].cpu().numpy(), pair[1].cpu().numpy()


def random_kept(rows, cols, fmt, seed, pad=0):
    """An 8-bit matrix as the oracle encodes normal values, on the GPU, and its values in 64 bits."""
    x = np.random.default_rng(seed).standard_normal((rows, cols)) if rows else np.zeros((0, cols))
    if rows * cols > 20000:        # the oracle's encoder is slow: the same few rows again and again
        x = x[:max(1, 20000 // cols)]
    q, s = A.encode(x, fmt)
    if rows:
        again = -(-rows // len(x))
        q, s = np.tile(q, (again, 1))[:rows], np.tile(s, (again, 1))[:rows]
        if again > 1:              # of different sizes
            s = s + np.random.default_rng(seed + 1).integers(-2, 3, (rows, 1)).astype(np.uint8)
    out = kept_blank(rows, cols, pad)
    out[0].copy_(torch.from_numpy(q))
    out[1].copy_(torch.from_numpy(s))
    return out, A.decode(q, s, fmt)


# ---- 8-bit matrices -----------------------------------------------------------------------------

SIZES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 7), (17, 96), (4, 1001), (129, 264), (1, 5000), (300, 40), (2, 2049)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", [A.I8, A.F8])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 8), (5, 3)])
def test_write_and_read_bit_for_bit(rows, cols, dtype, fmt, pad, shift):
    g = torch.Generator(device=DEV).manual_seed(rows * 7 + cols)
    flat, x = view(rows, cols, dtype, pad, shift)
    x.copy_(torch.randn(rows, cols, device=DEV, generator=g) * torch.exp2(torch.randint(-20, 20, (rows, 1), device=DEV, generator=g).float()))
    kept = kept_blank(rows, cols, pad)
    apm.apm_ckpt_write(x, apm.make_ckpt(*kept, fmt))
    q, s = A.encode(f64(x), fmt)
    got = bytes_of(kept)
    assert np.array_equal(got[1], s) and np.array_equal(got[0], q)
    if pad and rows > 1:
        assert bool((torch.as_strided(kept[0], (rows - 1, pad), (cols + pad, 1), cols) == 0x55).all())
    want = A.decode(q, s, fmt)
    for back_type in (BF16, F32):
        flat, back = view(rows, cols, back_type, pad, shift)
        apm.apm_ckpt_read(apm.make_ckpt(*kept, fmt), back)
        assert np.array_equal(f64(back), want)          # values are bf16 numbers: nothing is rounded
        assert untouched(flat, back, 7.0)


@pytest.mark.parametrize("fmt", [A.I8, A.F8])
def test_write_at_the_ends_of_the_range(fmt):
    big = torch.finfo(F32).max
    x = torch.zeros(9, 64, device=DEV)
    x[0, :4] = torch.tensor([big, -big, big / 3, 1.0])
    x[1, :3] = torch.tensor([1e-45, -1e-44, 3e-39])             # fp32 subnormals
    x[2, 5], x[2, 40] = float("inf"), 2.0
    x[3, 5], x[3, 40] = 3.0, float("nan")
    x[4, 0], x[4, 33] = float("-inf"), float("nan")
    x[5, 0], x[5, 1] = 127.5 / 64, 1 / 64                        # ties that move the scale
    x[6, 0], x[6, 1] = 464.0, 463.9
    x[7, 0], x[7, 1] = 464.1, -0.0
    x[8] = -0.0
    kept = kept_blank(9, 64)
    apm.apm_ckpt_write(x, apm.make_ckpt(*kept, fmt))
    q, s = A.encode(f64(x), fmt)
    assert np.array_equal(bytes_of(kept)[1], s) and np.array_equal(bytes_of(kept)[0], q)
    back = torch.empty(9, 64, device=DEV)
    apm.apm_ckpt_read(apm.make_ckpt(*kept, fmt), back)
    with np.errstate(over="ignore"):                             # the largest fp32 numbers have no F8 neighbour below 2^128
        want = A.decode(q, s, fmt).astype(np.float32)
    assert np.array_equal(f64(back), want.astype(np.float64), equal_nan=True)
    assert np.isnan(f64(back)[2, :32]).all() and f64(back)[2, 40] == 2.0 and np.isnan(f64(back)[3, 32:]).all()


def test_every_code_and_scale_is_read():
    for fmt in (A.I8, A.F8):
        q = torch.arange(256, device=DEV).to(torch.uint8).repeat(256, 1)
        if fmt == A.I8:
            q[:, 128] = 0
        else:
            q[:, 127], q[:, 255] = 0, 0
        s = torch.arange(256, device=DEV).to(torch.uint8)[:, None].repeat(1, 8)
        out = torch.empty(256, 256, device=DEV)
        apm.apm_ckpt_read(apm.make_ckpt(q, s.contiguous(), fmt), out)
        want = A.decode(q.cpu().numpy(), s.cpu().numpy(), fmt)
        with np.errstate(over="ignore"):
            want = want.astype(np.float32).astype(np.float64)    # what no fp32 number is: infinite, or a rounded subnormal
        assert np.array_equal(f64(out), want, equal_nan=True)


def test_offsets_beyond_32_bits():
    cols, far = 96, 2 ** 31 + 24                                  # elements between rows
    buf = torch.zeros(far + cols, dtype=BF16, device=DEV)
    x = torch.as_strided(buf, (2, cols), (far, 1))
    x.copy_(torch.randn(2, cols, device=DEV))
    qbuf = torch.zeros(far + cols, dtype=torch.uint8, device=DEV)
    sbuf = torch.zeros(far + 3, dtype=torch.uint8, device=DEV)
    kept = torch.as_strided(qbuf, (2, cols), (far, 1)), torch.as_strided(sbuf, (2, 3), (far, 1))
    apm.apm_ckpt_write(x, apm.make_ckpt(*kept, A.I8))
    q, s = A.encode(f64(x), A.I8)
    assert np.array_equal(kept[0].cpu().numpy(), q) and np.array_equal(kept[1].cpu().numpy(), s)
    y, n = torch.as_strided(torch.empty_like(buf), (2, cols), (far, 1)), torch.empty(2, cols, dtype=BF16, device=DEV)
    apm.apm_norm_join_forward(apm.make_norm_join(2, cols, x=x, y=y, n=n, residual_scale=2.0, pre_norm=apm.APM_NORM_RMS, pre_eps=1e-6))
    assert torch.equal(y, (2.0 * x.float()).bfloat16())
    dw = torch.empty(cols, cols, device=DEV)
    apm.apm_ckpt_weight_grad(apm.make_weight_grad(x, apm.make_ckpt(*kept, A.I8), dw))
    want = A.weight_grad(f64(x), A.decode(q, s, A.I8), 1.0, 0.0)[0]
    assert np.all(np.abs(f64(dw) - want) <= 8 * U * (np.abs(f64(x)).T @ np.abs(A.decode(q, s, A.I8))))


def test_many_rows_and_rows_that_overlap():
    row = torch.randn(1, 70, device=DEV).bfloat16()
    kept = kept_blank(3000, 70)
    apm.apm_ckpt_write(row.expand(3000, 70), apm.make_ckpt(*kept, A.F8))     # stride 0: one row for all tokens
    q, s = A.encode(f64(row), A.F8)
    assert bool((kept[0].cpu() == torch.from_numpy(q)).all()) and bool((kept[1].cpu() == torch.from_numpy(s)).all())
    empty = torch.empty(0, 70, dtype=BF16, device=DEV)
    none = kept_blank(0, 70)
    apm.apm_ckpt_write(empty, apm.make_ckpt(*none, A.F8))
    apm.apm_ckpt_read(apm.make_ckpt(*none, A.F8), empty)


# ---- norm joins ---------------------------------------------------------------------------------

class Join:
    """One join's inputs, outputs and 64-bit values."""

    def __init__(self, rows, cols, res=BF16, act=BF16, par=F32, pre=A.RMS, post=A.RMS, gate=A.CHANNEL, affine=(True, True, True, True), scale=1.25,
                 fmt=A.I8, eps=1e-5, branch=True, pad=0, shift=0, seed=0):
        g = torch.Generator(device=DEV).manual_seed(rows * 31 + cols + seed)
        rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)
        self.rows, self.cols, self.fmt, self.scale, self.eps, self.pre, self.post, self.gate_kind = rows, cols, fmt, scale, eps, pre, post, gate
        self.res, self.act = res, act
        make = lambda t, v: view(v.shape[0], v.shape[1], t, pad, shift)[1].copy_(v)
        self.x = make(res, rnd(rows, cols) * 3 + 0.5)
        self.branch = make(act, rnd(rows, cols)) if branch else None
        self.w1, self.b1 = (rnd(cols).to(par) if affine[0] else None), (rnd(cols).to(par) if affine[1] else None)
        self.w2, self.b2 = (rnd(cols).to(par) if affine[2] else None), (rnd(cols).to(par) if affine[3] else None)
        shape = {A.NO_GATE: None, A.CHANNEL: (1, cols), A.TOKEN: (rows, 1), A.FULL: (rows, cols)}[gate]
        self.gate = rnd(*shape).to(par) if shape else None
        self.flat_y, self.y = view(rows, cols, res, pad, shift)
        self.flat_n, self.n = view(rows, cols, act, pad, shift)
        self.kept1, self.kept2 = kept_blank(rows, cols, pad), kept_blank(rows, cols, pad)
        self.r1, self.r2 = torch.full((rows,), 7.0, device=DEV), torch.full((rows,), 7.0, device=DEV)
        self.dn, self.dy = make(act, rnd(rows, cols)), make(res, rnd(rows, cols))
        self.flat_dx, self.dx = view(rows, cols, res, pad, shift)
        self.flat_db, self.dbranch = view(rows, cols, act, pad, shift)
        like = lambda t: None if t is None else torch.full_like(t, 7.0)
        self.dw1, self.db1, self.dw2, self.db2, self.dgate = (like(t) for t in (self.w1, self.b1, self.w2, self.b2, self.gate))
        if not branch:
            self.dw2 = self.db2 = None

    def join(self, **over):
        has = self.branch is not None
        args = dict(x=self.x, branch=self.branch, y=self.y, n=self.n, residual_scale=self.scale, gate_kind=self.gate_kind, gate=self.gate,
                    pre_norm=self.pre, pre_eps=self.eps, pre_weight=self.w1, pre_bias=self.b1, pre_ckpt=apm.make_ckpt(*self.kept1, self.fmt),
                    pre_rstd=self.r1, post_norm=self.post, post_eps=self.eps, post_weight=self.w2 if has else None, post_bias=self.b2 if has else None,
                    post_ckpt=apm.make_ckpt(*self.kept2, self.fmt) if has else None, post_rstd=self.r2 if has else None)
        return apm.make_norm_join(self.rows, self.cols, **dict(args, **over))

    def grads(self, join, **over):
        args = dict(dn=self.dn, dy=self.dy, dx=self.dx, dbranch=self.dbranch if self.branch is not None else None, dgate=self.dgate,
                    dpre_weight=self.dw1, dpre_bias=self.db1, dpost_weight=self.dw2, dpost_bias=self.db2)
        return apm.make_norm_join_grads(join, **dict(args, **over))

    def affine(self, which):
        w, b = (self.w1, self.b1) if which == 1 else (self.w2, self.b2)
        return (f64(w) if w is not None else 1.0), (f64(b) if b is not None else 0.0)

    def gate64(self):
        return f64(self.gate) if self.gate is not None else 1.0


def room_for(rows, cols):
    return torch.full((max(16, apm.apm_norm_join_workspace_bytes(rows, cols)),), 0xFF, dtype=torch.uint8, device=DEV)


def out_bound(t, want, error):
    """What an output of t's type may be off, where its fp32 value is off by `error`."""
    return error + (2.0 ** -8 if t.dtype == BF16 else 4 * U) * np.abs(want)


def check_kept(pair, fmt, want, error):
    """Codes are the nearest of a value that is off by `error`; scales are the oracle's, unless that error can move them."""
    q, s = bytes_of(pair)
    got = A.decode(q, s, fmt)
    unit = np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, axis=1)[:, :want.shape[1]]
    half = unit / 128 if fmt == A.I8 else np.maximum(np.abs(want) * 2.0 ** -4, unit * 2.0 ** -10)
    assert np.all(np.abs(got - want) <= half * (1 + 1e-9) + 2 * error)
    pad = -want.shape[1] % 32
    largest = lambda v: np.max(np.abs(np.pad(v, ((0, 0), (0, pad))).reshape(want.shape[0], -1, 32)), axis=2)
    top, err = largest(want), largest(np.broadcast_to(error, want.shape))
    limit = (127.5 / 64 if fmt == A.I8 else 464.0)
    assert np.all(top - err <= limit * 2.0 ** (s.astype(np.float64) - 127) * (1 + 1e-9))
    assert np.all((top + err >= limit * 2.0 ** (s.astype(np.float64) - 128) * (1 - 1e-9)) | (s == 0))


def check_forward(J):
    x, b = f64(J.x), f64(J.branch)
    w1, c1 = J.affine(1)
    w2, c2 = J.affine(2)
    y, n, h1, r1, h2, r2 = A.join_forward(x, b, J.scale, J.gate64(), (J.pre, J.eps, w1, c1), (J.post, J.eps, w2, c2))
    stat = (J.cols + 16) * U                                   # of a row's mean and root
    e2 = 0.0
    terms = np.abs(J.scale * x)
    if b is not None:
        lift = np.max(np.abs(b), axis=1, keepdims=True) * r2[:, None] if J.post else 0.0
        e2 = stat * (np.abs(h2) + lift)
        terms = terms + np.abs(J.gate64() * c2) + np.abs(J.gate64() * h2 * w2)
        if J.post:
            assert np.all(np.abs(f64(J.r2) - r2) <= 2 * stat * (1 + lift[:, 0]) * r2 + 1e-30)
        check_kept(J.kept2, J.fmt, h2, e2 + 4 * U * np.abs(h2))
    ey = 8 * U * terms + np.abs(J.gate64() * w2) * e2
    assert np.all(np.abs(f64(J.y) - y) <= out_bound(J.y, y, ey))
    if J.pre:
        lift = np.max(np.abs(y), axis=1, keepdims=True) * r1[:, None]
        worst = np.max(ey, axis=1, keepdims=True) * r1[:, None]
        e1 = stat * (np.abs(h1) + lift) + (2 + np.abs(h1)) * 2 * worst
        assert np.all(np.abs(f64(J.r1) - r1) <= (2 * stat * (1 + lift[:, 0]) + 4 * worst[:, 0]) * r1)
    else:
        e1 = ey
    check_kept(J.kept1, J.fmt, h1, e1 + 4 * U * np.abs(h1))
    assert np.all(np.abs(f64(J.n) - n) <= out_bound(J.n, n, np.abs(w1) * e1 + 8 * U * (np.abs(h1 * w1) + np.abs(c1))))


def check_backward(J, has_dn=True, has_dy=True):
    """Against the formulas at what was kept: the codes, and r as the forward pass stored it."""
    h1 = A.decode(*bytes_of(J.kept1), J.fmt)
    has = J.branch is not None
    h2 = A.decode(*bytes_of(J.kept2), J.fmt) if has else None
    w1, c1 = J.affine(1)
    w2, c2 = J.affine(2)
    one = np.ones(J.rows)
    r1, r2 = (f64(J.r1) if J.pre else one), (f64(J.r2) if J.post else one)
    dn, dy = (f64(J.dn) if has_dn else np.zeros((J.rows, J.cols))), (f64(J.dy) if has_dy else np.zeros((J.rows, J.cols)))
    gate = J.gate64()
    want = A.join_backward(dn, dy, J.scale, gate, J.gate_kind, (J.pre, J.eps, w1, c1), (J.post, J.eps, w2, c2), h1, r1, h2, r2)

    def through_error(t, et, h, r, kind):                      # of through(t): sums of cols terms, and what t brings
        if kind == A.NONE:
            return et
        mean = lambda v: np.mean(v, axis=1, keepdims=True)
        n = (J.cols + 8) * U
        size = np.abs(t) + np.abs(h) * mean(np.abs(t * h)) + mean(np.abs(t))
        return r[:, None] * (n * size + et + np.abs(h) * mean(et * np.abs(h)) + mean(et))

    t = dn * w1
    eD = through_error(t, 4 * U * np.abs(t), h1, r1, J.pre) + 4 * U * (np.abs(dy) + np.abs(want["D"]))
    D = np.abs(want["D"])
    assert np.all(np.abs(f64(J.dx) - want["dx"]) <= out_bound(J.dx, want["dx"], abs(J.scale) * (eD + 2 * U * D)))
    rows = (J.rows + 16) * U

    def sums(name, got, terms, errors):
        if got is not None:
            bound = out_bound(got, want[name].reshape(got.shape), (rows * terms + errors).reshape(got.shape))
            assert np.all(np.abs(f64(got) - want[name].reshape(got.shape)) <= bound), name

    sums("dpre_weight", J.dw1, np.abs(dn * h1).sum(0), 0.0 * np.abs(dn * h1).sum(0))
    sums("dpre_bias", J.db1, np.abs(dn).sum(0), 0.0 * np.abs(dn).sum(0))
    if not has:
        return
    inner, einner = np.abs(h2 * w2) + np.abs(c2), 0.0
    term, error = D * inner, (eD + 8 * U * D) * inner
    if J.gate_kind == A.CHANNEL:
        sums("dgate", J.dgate, term.sum(0, keepdims=True), error.sum(0, keepdims=True))
    elif J.gate_kind == A.TOKEN:
        cols = (J.cols + 16) * U
        bound = out_bound(J.dgate, want["dgate"], cols * term.sum(1, keepdims=True) + error.sum(1, keepdims=True))
        assert np.all(np.abs(f64(J.dgate) - want["dgate"]) <= bound)
    elif J.gate_kind == A.FULL:
        assert np.all(np.abs(f64(J.dgate) - want["dgate"]) <= out_bound(J.dgate, want["dgate"], error))
    u = gate * want["D"] * w2
    eu = np.abs(gate * w2) * (eD + 8 * U * D)
    eb = through_error(u, eu, h2, r2, J.post)
    assert np.all(np.abs(f64(J.dbranch) - want["dbranch"]) <= out_bound(J.dbranch, want["dbranch"], eb + 4 * U * np.abs(want["dbranch"])))
    shared = np.abs(gate) * D
    sums("dpost_weight", J.dw2, (shared * np.abs(h2)).sum(0), (np.abs(gate) * (eD + 8 * U * D) * np.abs(h2)).sum(0))
    sums("dpost_bias", J.db2, shared.sum(0), (np.abs(gate) * (eD + 8 * U * D)).sum(0))


def run_both(J):
    join = J.join()
    apm.apm_norm_join_forward(join)
    check_forward(J)
    apm.apm_norm_join_backward(join, J.grads(join), room_for(J.rows, J.cols))
    check_backward(J)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 32), (5, 33), (1, 512), (4, 513), (300, 264), (7, 1000), (3, 1024), (2, 1025), (33, 1537),
                                       (5, 2048), (600, 768), (2, 5120), (3, 8192), (2, 8193), (2, 12288), (1, 16384), (700, 48)])
@pytest.mark.parametrize("norm", [A.RMS, A.LAYER])
def test_join_sizes(rows, cols, norm):
    run_both(Join(rows, cols, pre=norm, post=norm, fmt=A.I8 if cols % 2 else A.F8))


@pytest.mark.parametrize("res,act,par", [(BF16, BF16, BF16), (F32, BF16, F32), (F32, F32, BF16), (F32, F32, F32)])
@pytest.mark.parametrize("gate", [A.NO_GATE, A.CHANNEL, A.TOKEN, A.FULL])
@pytest.mark.parametrize("pre,post", [(A.LAYER, A.RMS), (A.RMS, A.NONE), (A.NONE, A.LAYER), (A.NONE, A.NONE)])
def test_join_types_gates_and_norms(res, act, par, gate, pre, post):
    run_both(Join(9, 200, res, act, par, pre, post, gate))
    run_both(Join(4, 1100, res, act, par, pre, post, gate, fmt=A.F8))


@pytest.mark.parametrize("affine", [(True, False, True, False), (False, False, False, False), (True, False, False, True), (False, True, True, False)])
def test_join_without_some_vectors(affine):
    run_both(Join(40, 96, affine=affine, pre=A.LAYER, post=A.LAYER))
    run_both(Join(40, 96, affine=affine, gate=A.NO_GATE))


@pytest.mark.parametrize("cols", [50, 1030, 8200])
def test_join_rows_at_any_alignment(cols):
    J = Join(5, cols, pad=3, shift=1)
    run_both(J)
    for flat, m in ((J.flat_y, J.y), (J.flat_n, J.n), (J.flat_dx, J.dx), (J.flat_db, J.dbranch)):
        assert untouched(flat, m, 7.0)


@pytest.mark.parametrize("cols", list(range(1, 16)) + list(range(505, 513)) + list(range(1025, 1033)))
@pytest.mark.parametrize("res,act", [(BF16, BF16), (F32, BF16), (F32, F32)])
def test_join_rows_that_end_at_any_column(cols, res, act):
    J = Join(5 + 1300 // cols, cols, res, act, pre=A.LAYER, post=A.LAYER, gate=A.TOKEN, pad=3, shift=1)
    run_both(J)
    for flat, m in ((J.flat_y, J.y), (J.flat_n, J.n), (J.flat_dx, J.dx), (J.flat_db, J.dbranch)):
        assert untouched(flat, m, 7.0)


def test_join_without_a_branch_is_the_norm_of_the_stream():
    run_both(Join(20, 100, branch=False, gate=A.NO_GATE, post=A.NONE, pre=A.LAYER))


@pytest.mark.parametrize("cols", [100, 1500])
def test_join_backward_with_one_gradient_only(cols):
    J = Join(6, cols)
    join = J.join()
    apm.apm_norm_join_forward(join)
    for dn, dy in ((True, False), (False, True)):
        grads = J.grads(join, dn=J.dn if dn else None, dy=J.dy if dy else None)
        apm.apm_norm_join_backward(join, grads, room_for(J.rows, J.cols))
        check_backward(J, dn, dy)


def test_join_outputs_that_are_not_asked_for():
    J = Join(30, 700, pre=A.LAYER, gate=A.TOKEN)
    whole = J.join()
    apm.apm_norm_join_forward(whole)
    y, n, k1, k2 = J.y.clone(), J.n.clone(), J.kept1[0].clone(), J.kept2[0].clone()
    J.y.fill_(7.0)
    J.kept2[0].fill_(0)
    apm.apm_norm_join_forward(J.join(y=None, post_ckpt=None, post_rstd=None))
    assert torch.equal(J.n, n) and bool((J.y == 7.0).all()) and bool((J.kept2[0] == 0).all())
    J.n.fill_(7.0)
    apm.apm_norm_join_forward(J.join(n=None, pre_ckpt=None, pre_rstd=None))
    assert torch.equal(J.y, y) and bool((J.n == 7.0).all()) and torch.equal(J.kept2[0], k2)
    apm.apm_norm_join_backward(whole, J.grads(whole), room_for(30, 700))
    dx, db, dw2 = J.dx.clone(), J.dbranch.clone(), J.dw2.clone()
    for t in (J.dx, J.dbranch, J.dw2, J.dw1):
        t.fill_(7.0)
    apm.apm_norm_join_backward(whole, J.grads(whole, dbranch=None, dpre_weight=None, dpre_bias=None, dpost_bias=None), room_for(30, 700))
    assert torch.equal(J.dx, dx) and torch.equal(J.dw2, dw2) and bool((J.dbranch == 7.0).all()) and bool((J.dw1 == 7.0).all())
    apm.apm_norm_join_backward(whole, J.grads(whole, dx=None, dgate=None, dpre_weight=None, dpre_bias=None, dpost_bias=None, dpost_weight=None), room_for(30, 700))
    assert torch.equal(J.dbranch, db)


@pytest.mark.parametrize("cols", [64, 1100])
def test_join_in_place(cols):
    J = Join(11, cols, seed=3)
    join = J.join()
    apm.apm_norm_join_forward(join)
    y, n = J.y.clone(), J.n.clone()
    x, branch, dy, dn = J.x.clone(), J.branch.clone(), J.dy.clone(), J.dn.clone()
    apm.apm_norm_join_forward(J.join(x=x, y=x, branch=branch, n=branch))
    assert torch.equal(x, y) and torch.equal(branch, n)
    apm.apm_norm_join_backward(join, J.grads(join), room_for(11, cols))
    apm.apm_norm_join_backward(join, J.grads(join, dy=dy, dx=dy, dn=dn, dbranch=dn), room_for(11, cols))
    assert torch.equal(dy, J.dx) and torch.equal(dn, J.dbranch)


def test_join_of_no_tokens_writes_zero_sums():
    J = Join(0, 300)
    join = J.join()
    apm.apm_norm_join_forward(join)
    apm.apm_norm_join_backward(join, J.grads(join), room_for(0, 300))
    for t in (J.dw1, J.db1, J.dw2, J.db2, J.dgate):
        assert bool((t == 0).all())


@pytest.mark.parametrize("cols", [40, 2000])
def test_join_rows_do_not_touch_each_other(cols):
    """Rows of zeros, of one value, with an infinity or a NaN: their own outputs are what the formulas give, the others' are as without them."""
    J = Join(6, cols, pre=A.LAYER, post=A.LAYER, gate=A.TOKEN)
    plain = J.join()
    apm.apm_norm_join_forward(plain)
    y, n = J.y.clone(), J.n.clone()
    J.x[0], J.branch[0] = 0, 0
    J.x[1], J.branch[1] = 3.0, 5.0
    J.x[2, 5] = float("inf")
    J.branch[3, 7] = float("nan")
    apm.apm_norm_join_forward(plain)
    assert torch.equal(J.y[4:], y[4:]) and torch.equal(J.n[4:], n[4:])
    assert bool(torch.isfinite(J.n[:2]).all()) and bool(torch.isnan(J.n[2:4]).all())
    assert bool((J.kept1[1][2:4] == 255).all()) and bool((J.kept2[1][3] == 255).all()) and bool((J.kept2[1][2] != 255).all())
    apm.apm_norm_join_backward(plain, J.grads(plain), room_for(6, cols))
    assert bool(torch.isnan(J.dx[2:4]).all()) and bool(torch.isfinite(J.dx[[0, 1, 4, 5]]).all())
    assert bool(torch.isfinite(J.dbranch[[0, 1, 4, 5]]).all()) and bool(torch.isnan(J.dw1).all())


@pytest.mark.parametrize("rows,cols,gate", [(500, 300, A.CHANNEL), (500, 3000, A.TOKEN), (20, 9000, A.FULL)])
def test_join_gives_the_same_bits_again_whatever_the_workspace_held(rows, cols, gate):
    J = Join(rows, cols, gate=gate, pre=A.LAYER)
    join = J.join()
    apm.apm_norm_join_forward(join)
    seen = []
    for fill in (0, 0xFF, 0x7F):
        room = room_for(rows, cols).fill_(fill)
        apm.apm_norm_join_backward(join, J.grads(join), room)
        seen.append([t.clone() for t in (J.dx, J.dbranch, J.dgate, J.dw1, J.db1, J.dw2, J.db2)])
    for other in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], other))


def test_join_gradient_against_differences():
    """The kept tensors replace hat by what is up to 1/127 of a block's largest off (8 bits): a directional difference of the 32-bit forward pass
    agrees to that and no better.  Directions are the gradient's own, so that the derivative is a sum of squares and does not cancel."""
    J = Join(64, 256, F32, F32, F32, A.LAYER, A.LAYER, A.CHANNEL)
    join = J.join()
    apm.apm_norm_join_forward(join)
    apm.apm_norm_join_backward(join, J.grads(join), room_for(64, 256))

    def loss():
        apm.apm_norm_join_forward(J.join(pre_ckpt=None, post_ckpt=None))
        return float((J.y.double() * J.dy.double()).sum() + (J.n.double() * J.dn.double()).sum())

    for p, g in ((J.x, J.dx), (J.branch, J.dbranch), (J.gate, J.dgate), (J.w1, J.dw1), (J.b1, J.db1), (J.w2, J.dw2), (J.b2, J.db2)):
        keep, want = p.clone(), float(g.double().square().sum())
        h = 1e-2 / float(g.norm()) * float(p.norm())
        p.copy_(keep + h * g)
        hi = loss()
        p.copy_(keep - h * g)
        lo = loss()
        p.copy_(keep)
        assert abs((hi - lo) / (2 * h) - want) <= 0.02 * want


# ---- weight gradients ---------------------------------------------------------------------------

def check_weight_grad(tokens, out, k, fmt=A.I8, dtype=F32, weight=True, bias=True, db=True, offsets=None, accumulate=False, pad=0, shift=0, par=F32, seed=0):
    g = torch.Generator(device=DEV).manual_seed(tokens + out * 3 + k * 5 + seed)
    kept, z = random_kept(tokens, k, fmt, tokens + out + k + seed, pad)
    _, dy = view(tokens, out, BF16, pad, shift)
    dy.copy_(torch.randn(tokens, out, device=DEV, generator=g))
    w = torch.randn(k, device=DEV, generator=g).to(par) if weight else None
    b = torch.randn(k, device=DEV, generator=g).to(par) if bias else None
    groups = len(offsets) - 1 if offsets is not None else 0
    n = max(1, groups)
    flat = torch.full((shift + n * (out * (k + pad) + 64),), 7.0, dtype=dtype, device=DEV)
    dw = torch.as_strided(flat, (n, out, k), (out * (k + pad) + 64, k + pad, 1), shift)
    sums = torch.full((n, out), 7.0, dtype=dtype, device=DEV) if db else None
    if accumulate:
        dw.copy_(torch.randn(n, out, k, device=DEV, generator=g))
        if db:
            sums.copy_(torch.randn(n, out, device=DEV, generator=g))
    before, before_sums = f64(dw), f64(sums)
    offs = None if offsets is None else torch.tensor(offsets, dtype=torch.int64, device=DEV)
    grad = apm.make_weight_grad(dy, apm.make_ckpt(*kept, fmt), dw if groups else dw[0], db=sums, weight=w, bias=b, offsets=offs, accumulate=accumulate)
    size = apm.apm_ckpt_weight_grad_workspace_bytes(grad)
    apm.apm_ckpt_weight_grad(grad, torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if size else None)
    w64, b64 = (f64(w) if weight else 1.0), (f64(b) if bias else 0.0)
    want, want_sums = A.weight_grad(f64(dy), z, w64, b64, offsets)
    terms, term_sums = A.weight_grad(np.abs(f64(dy)), np.abs(z), np.abs(w64) if weight else 1.0, np.abs(b64) if bias else 0.0, offsets)
    if not groups:
        want, terms, want_sums, term_sums = want[None], terms[None], want_sums[None], term_sums[None]
    if accumulate:
        want, terms = want + before, terms + np.abs(before)
        if db:
            want_sums, term_sums = want_sums + before_sums, term_sums + np.abs(before_sums)
    # sums of `tokens` exact products in fp32, in any order, a matrix instruction's own additions truncated rather than rounded
    bound = 2 * (tokens + 16) * U
    assert np.all(np.abs(f64(dw) - want) <= out_bound(dw, want, bound * terms))
    if db:
        assert np.all(np.abs(f64(sums) - want_sums) <= out_bound(sums, want_sums, bound * term_sums))
    mask = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(mask, dw.shape, dw.stride(), shift).fill_(False)
    assert bool((flat[mask] == 7.0).all())
    return dw


@pytest.mark.parametrize("tokens", [0, 1, 5, 31, 32, 33, 64, 257, 1000])
@pytest.mark.parametrize("out,k", [(1, 1), (31, 33), (128, 128), (129, 40), (40, 260), (300, 513)])
def test_weight_gradient_sizes(tokens, out, k):
    check_weight_grad(tokens, out, k, fmt=A.I8 if tokens % 2 else A.F8)


@pytest.mark.parametrize("fmt", [A.I8, A.F8])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("weight,bias,db", [(False, False, False), (True, False, False), (False, True, False), (False, False, True), (True, True, True)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_gradient_forms(fmt, dtype, weight, bias, db, accumulate):
    check_weight_grad(300, 264, 136, fmt, dtype, weight, bias, db, accumulate=accumulate, par=dtype)
    check_weight_grad(70, 520, 520, fmt, dtype, weight, bias, db, accumulate=accumulate, par=dtype)


@pytest.mark.parametrize("tokens,out,k", [(200, 1024, 2048), (5000, 256, 256), (4100, 768, 130), (640, 2048, 1000)])
def test_weight_gradient_larger(tokens, out, k):
    check_weight_grad(tokens, out, k, dtype=BF16)


@pytest.mark.parametrize("pad,shift", [(8, 8), (16, 0), (3, 1), (0, 5)])
def test_weight_gradient_at_any_alignment(pad, shift):
    check_weight_grad(90, 200, 150, pad=pad, shift=shift)
    check_weight_grad(90, 256, 256, pad=pad, shift=shift, dtype=BF16)


@pytest.mark.parametrize("offsets", [[0, 100], [0, 0, 100, 100], [0, 33, 34, 34, 99, 100], [5, 20, 90], [-7, 40, 300], [0, 60, 30, 100], [0] * 9, [100] * 4])
@pytest.mark.parametrize("out,k", [(40, 50), (256, 300)])
def test_weight_gradient_of_groups(offsets, out, k):
    check_weight_grad(100, out, k, offsets=offsets, dtype=BF16)
    check_weight_grad(100, out, k, A.F8, offsets=offsets, bias=False, weight=False, accumulate=True, pad=1)


@pytest.mark.parametrize("tokens,out,k,pad,shift", [(130, 4096, 4096, 0, 0), (70, 4001, 4007, 1, 3), (300, 3900, 4100, 8, 8), (64, 4097, 4090, 0, 0)])
def test_weight_gradient_of_large_matrices(tokens, out, k, pad, shift):
    check_weight_grad(tokens, out, k, A.I8, BF16, pad=pad, shift=shift)
    check_weight_grad(tokens, out, k, A.F8, BF16, weight=False, bias=False, db=False, pad=pad, shift=shift)


@pytest.mark.parametrize("tokens,out,k,pad,shift", [(130, 4096, 2048, 0, 0), (70, 2048, 2304, 1, 3), (1500, 1024, 1100, 4, 0), (40, 1400, 700, 0, 1)])
def test_weight_gradient_in_fp32_of_large_matrices(tokens, out, k, pad, shift):
    check_weight_grad(tokens, out, k, A.F8, F32, pad=pad, shift=shift, accumulate=shift > 0)
    check_weight_grad(tokens, out, k, A.I8, F32, weight=False, bias=False, db=False, offsets=[0, 0, tokens // 2, tokens, tokens], pad=pad, shift=shift)


@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_gradient_of_groups_of_large_matrices(accumulate):
    check_weight_grad(300, 1100, 1030, A.F8, BF16, offsets=[0, 0, 129, 130, 130, 300, 300] + [300] * 10, accumulate=accumulate)
    check_weight_grad(2000, 1100, 1030, A.I8, F32, offsets=[0, 700, 700, 2000], accumulate=accumulate)


def test_weight_gradient_without_tokens_is_zero_whatever_the_weight():
    kept, _ = random_kept(600, 64, A.I8, 2)
    dy = torch.randn(600, 40, device=DEV).bfloat16()
    w = torch.full((64,), float("inf"), device=DEV)
    for offsets in ([0, 0, 600], [0] * 9 + [600]):
        n = len(offsets) - 1
        dw, db = torch.full((n, 40, 64), 7.0, device=DEV), torch.full((n, 40), 7.0, device=DEV)
        grad = apm.make_weight_grad(dy, apm.make_ckpt(*kept, A.I8), dw, db=db, weight=w, bias=w, offsets=torch.tensor(offsets, device=DEV))
        apm.apm_ckpt_weight_grad(grad, torch.empty(max(16, apm.apm_ckpt_weight_grad_workspace_bytes(grad)), dtype=torch.uint8, device=DEV))
        assert bool((dw[:-1] == 0).all()) and bool((db[:-1] == 0).all())


@pytest.mark.parametrize("fmt", [A.I8, A.F8])
def test_weight_gradient_reads_every_code_and_scale(fmt):
    """One token per scale: the product with a dy of one 1 per token and output is the kept value itself."""
    q = torch.arange(256, device=DEV).to(torch.uint8).repeat(255, 1)
    bad = [128] if fmt == A.I8 else [127, 255]
    q[:, bad] = 0
    s = torch.arange(255, device=DEV).to(torch.uint8)[:, None].repeat(1, 8).contiguous()
    dy = torch.eye(255, device=DEV).bfloat16()
    dw = torch.empty(255, 256, device=DEV)
    apm.apm_ckpt_weight_grad(apm.make_weight_grad(dy, apm.make_ckpt(q, s, fmt), dw), torch.empty(1 << 22, dtype=torch.uint8, device=DEV))
    want = A.decode(q.cpu().numpy(), s.cpu().numpy(), fmt)
    lost = (np.abs(want) >= 2.0 ** 128).any(axis=0)     # no bf16 number: infinite, and 0 times it is no number in the other tokens' rows
    assert np.isnan(f64(dw)[:-8, lost]).all() and lost.any() == (fmt == A.F8)
    normal = ~lost[None, :] & ((np.abs(want) >= 2.0 ** -126) | (want == 0))
    assert np.array_equal(f64(dw)[normal], want[normal])
    assert np.all(np.abs(f64(dw) - want)[:, ~lost] <= 2.0 ** -126)          # subnormals may be taken as zero


def test_weight_gradient_of_many_groups():
    check_weight_grad(2000, 64, 96, offsets=sorted(np.random.default_rng(3).integers(0, 2000, 201).tolist()))


def test_weight_gradient_keeps_a_nan_in_its_block_and_group():
    kept, _ = random_kept(64, 96, A.I8, 1)
    kept[1][40, 1] = 255                                            # token 40, channels 32 .. 63
    dy = torch.randn(64, 50, device=DEV).bfloat16()
    dy[3, 7] = float("inf")
    dw = torch.empty(2, 50, 96, device=DEV)
    apm.apm_ckpt_weight_grad(apm.make_weight_grad(dy, apm.make_ckpt(*kept, A.I8), dw, offsets=torch.tensor([0, 32, 64], device=DEV)))
    bad = ~torch.isfinite(dw)
    assert bool(bad[1, :, 32:64].all()) and not bool(bad[1, :, :32].any()) and not bool(bad[1, :, 64:].any())
    assert bool(bad[0, 7].all()) and int(bad[0].sum()) == 96


def test_weight_gradient_gives_the_same_bits_again():
    first = check_weight_grad(3000, 300, 300, seed=1).clone()
    assert torch.equal(first, check_weight_grad(3000, 300, 300, seed=1))


# ---- streams and graphs -------------------------------------------------------------------------

def test_all_of_it_on_another_stream_and_in_a_graph():
    """The calls go to the stream they are given; a captured sequence gives on every replay what the eager calls give on the same inputs."""
    J = Join(200, 600, seed=4)
    join = J.join()
    grads = J.grads(join)
    room = room_for(200, 600)
    dw, db = torch.empty(96, 600, dtype=BF16, device=DEV), torch.empty(96, device=DEV)
    dy = torch.randn(200, 96, device=DEV).bfloat16()
    grad = apm.make_weight_grad(dy, apm.make_ckpt(*J.kept1, J.fmt), dw, db=db, weight=J.w1, bias=J.b1)
    room2 = torch.empty(max(16, apm.apm_ckpt_weight_grad_workspace_bytes(grad)), dtype=torch.uint8, device=DEV)
    back = torch.empty(200, 600, device=DEV)
    outs = [J.y, J.n, J.dx, J.dbranch, J.dgate, J.dw1, J.db1, J.dw2, J.db2, dw, db, back]

    def all_of_it(stream):
        apm.apm_norm_join_forward(join, stream)
        apm.apm_ckpt_read(apm.make_ckpt(*J.kept1, J.fmt), back, stream)
        apm.apm_norm_join_backward(join, grads, room, stream)
        apm.apm_ckpt_weight_grad(grad, room2, stream)

    def clear():
        for t in outs:
            t.zero_()

    all_of_it(None)
    torch.cuda.synchronize()
    eager = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    clear()
    torch.cuda.synchronize()
    all_of_it(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        all_of_it(side)
    for seed in range(3):
        for t, s in ((J.x, 1), (J.branch, 2), (J.dn, 3), (J.dy, 4)):
            t.copy_(torch.randn(t.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(10 * seed + s)))
        torch.cuda.synchronize()
        clear()
        all_of_it(None)
        torch.cuda.synchronize()
        eager = [t.clone() for t in outs]
        clear()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
