"""Sorting, lookup, products per group and dropout on the GPU, against the oracle in 64 bits.

Bounds: one rounding to a result's type is half a step, eps / 2 of the value (and half the smallest subnormal of bf16, which has fp32's range:
2^-134); a sum of n terms in fp32, in any order, each of a product or two, is off by at most (n + 4) u of the sum of the terms' sizes, u = 2^-24.
A matrix instruction's own additions may be truncated, which doubles that.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.tokens as T
import paper_2303_02868_amd as apm
from test_gpu_activations import f64, untouched, view

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
BF16, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


def near(got, want, size, terms, roundings=1):
    """Whether each element is its exact value, but for a sum of `terms` terms in fp32 and so many roundings to the result's type."""
    slack = (terms + 4) * U * size
    half = roundings * torch.finfo(got.dtype).eps / 2 if got.dtype == BF16 else 0.0
    off = np.abs(f64(got) - want)
    ok = off <= slack + half * (np.abs(want) + slack) + 2.0 ** -133
    assert np.all(ok), (float(off[~ok].max()), int((~ok).sum()), np.argwhere(~ok)[:4].tolist())


def room(size):
    return torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if size else None


def rng(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


# ---- sorting ------------------------------------------------------------------------------------

def sort(ids, rows, offsets=True, more=True, workspace=None):
    n = ids.numel()
    out = [torch.full((n,), -77, dtype=I32, device=DEV) for _ in range(3)]
    offs = torch.full((rows + 1,), -77, dtype=I64, device=DEV) if offsets else None
    o = apm.make_token_order(ids, rows, out[0], offsets=offs, place=out[1] if more else None, token=out[2] if more else None)
    apm.apm_sort_tokens(o, room(apm.apm_sort_tokens_workspace_bytes(o)) if workspace is None else workspace)
    return o, (out[0], offs, out[1], out[2])


def check_sort(ids, rows):
    got = sort(ids, rows)[1]
    flat, per = ids.flatten().cpu().numpy().astype(np.int64), 1 if ids.dim() == 1 else ids.shape[1]
    if flat.size * rows < 1 << 22:
        want = T.sort_tokens(flat, rows, per)
    else:                       # the oracle keeps a list for each row
        key = np.where((flat >= 0) & (flat < rows), flat, rows)
        order = np.argsort(key, kind="stable")
        offsets = np.searchsorted(key[order], np.arange(rows + 1))
        place = np.full(flat.size, -1)
        place[order[:offsets[-1]]] = np.arange(offsets[-1])
        want = order, offsets, place, order // per
    for name, g, w in zip(("order", "offsets", "place", "token"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name


@pytest.mark.parametrize("rows", [1, 2, 64, 255, 256, 1000, 5000, 70000])
@pytest.mark.parametrize("n", [0, 1, 63, 64, 65, 1000, 1024, 1025, 4096, 4097, 16384, 16385, 50001])
def test_sort_sizes(n, rows):
    ids = torch.randint(-1, rows + 1, (n,), device=DEV, generator=rng(n + rows))   # some of them no rows
    check_sort(ids.to(I32) if n % 2 else ids, rows)


def test_sort_with_several_positions_of_a_token():
    for tokens, per, rows in ((5, 3, 4), (700, 8, 64), (3000, 8, 300), (9000, 7, 33)):
        check_sort(torch.randint(0, rows, (tokens, per), device=DEV, generator=rng(per)), rows)


def test_sort_where_all_are_equal_or_none_is_a_row():
    for n in (1, 70, 16384, 40000):
        check_sort(torch.full((n,), 3, device=DEV), 9)
        check_sort(torch.full((n,), -1, device=DEV), 9)
        check_sort(torch.full((n,), 8, dtype=I32, device=DEV), 9)


def test_sort_ids_far_outside():
    ids = torch.tensor([1 << 40, -(1 << 40), (1 << 32) + 1, 1, 0, (1 << 31), -(1 << 31), 2, 1], device=DEV)
    check_sort(ids, 2)
    big = apm.APM_MAX_POSITIONS
    ids = torch.tensor([big - 1, 5, big, 1 << 31, 5, -1, big - 1], device=DEV)       # the largest table there may be
    order = torch.empty(7, dtype=I32, device=DEV)
    place, token = torch.empty_like(order), torch.empty_like(order)
    o = apm.make_token_order(ids, 1, order, place=place, token=token)
    o.rows = big
    apm.apm_sort_tokens(o, room(apm.apm_sort_tokens_workspace_bytes(o)))
    assert order.tolist() == [1, 4, 0, 6, 2, 3, 5] and place.tolist() == [2, 0, -1, -1, 1, -1, 3] and token.tolist() == order.tolist()
    many = torch.randint(0, big, (20000,), device=DEV, generator=rng(1))
    order = torch.empty(20000, dtype=I32, device=DEV)
    o = apm.make_token_order(many, 1, order)
    o.rows = big
    apm.apm_sort_tokens(o, room(apm.apm_sort_tokens_workspace_bytes(o)))
    assert torch.equal(order.long(), torch.sort(many, stable=True).indices)


def test_sort_writes_what_is_asked_for():
    ids = torch.randint(0, 50, (20000,), device=DEV, generator=rng(0))
    whole = sort(ids, 50)[1]
    for n in (20000, 300):
        order = sort(ids[:n], 50, offsets=False, more=False)[1][0]
        assert torch.equal(order, sort(ids[:n], 50)[1][0])
    assert torch.equal(whole[0], sort(ids, 50, offsets=False)[1][0])


# ---- lookup -------------------------------------------------------------------------------------

def make_ids(tokens, per, rows, seed, dtype=I64, none=True):
    """Some rows often, and some ids that are no rows."""
    g = rng(seed)
    ids = torch.randint(0, rows, (tokens, per), device=DEV, generator=g)
    ids = torch.where(torch.rand(tokens, per, device=DEV, generator=g) < 0.4, ids % 3 % rows, ids)
    if none:
        ids = torch.where(torch.rand(tokens, per, device=DEV, generator=g) < 0.1, torch.where(ids % 2 == 0, -1 - ids, rows + ids), ids)
    return ids.to(dtype)


class Lookup:
    def __init__(self, tokens, per, rows, cols, table=BF16, y=BF16, weights=None, scale=1.0, pad=0, shift=0, seed=0, ids=I64):
        g = rng(seed)
        self.shape = tokens, per, rows, cols
        self.ids, self.scale, self.pad, self.shift = make_ids(tokens, per, rows, seed, ids), scale, pad, shift
        self.table = view(rows, cols, table, pad, shift)[1]
        self.table.copy_(torch.randn(rows, cols, device=DEV, generator=g))
        self.weights = None if weights is None else torch.randn(tokens, per, device=DEV, generator=g).to(weights)
        self.flat, self.y = view(tokens, cols, y, pad, shift)
        self.dy = view(tokens, cols, y, pad, shift)[1]
        self.dy.copy_(torch.randn(tokens, cols, device=DEV, generator=g))

    def forward(self, accumulate=False):
        tokens, per, rows, cols = self.shape
        u = apm.make_lookup(self.ids if per > 1 else self.ids[:, 0].contiguous(), self.table, self.y, scale=self.scale, weights=self.weights, accumulate=accumulate)
        want, size = T.lookup(self.ids.cpu().numpy(), f64(self.table), np.float32(self.scale), f64(self.weights))
        if accumulate:
            self.y.copy_(torch.randn(tokens, cols, device=DEV, generator=rng(5)))
            want, size = want + f64(self.y), size + np.abs(f64(self.y))
        apm.apm_lookup_forward(u)
        near(self.y, want, size, per + 2)
        assert untouched(self.flat, self.y, 7.0)

    def backward(self, dtype=F32, accumulate=False, weights=True):
        tokens, per, rows, cols = self.shape
        u = apm.make_lookup(self.ids, self.table, scale=self.scale, weights=self.weights)
        o = sort(self.ids, rows)[0]
        flat, dtable = view(rows, cols, dtype, self.pad, self.shift)
        dw = torch.full((tokens, per), 7.0, dtype=dtype, device=DEV) if weights else None
        want, size, want_w, size_w = T.lookup_gradients(self.ids.cpu().numpy(), f64(self.dy), rows, f64(self.table), np.float32(self.scale), f64(self.weights))
        if accumulate:
            dtable.copy_(torch.randn(rows, cols, device=DEV, generator=rng(6)))
            want, size = want + f64(dtable), size + np.abs(f64(dtable))
        g = apm.make_lookup_grads(u, self.dy, order=o, dtable=dtable, dweights=dw, accumulate=accumulate)
        apm.apm_lookup_backward(u, g, room(apm.apm_lookup_workspace_bytes(u)))
        near(dtable, want, size, np.bincount(np.clip(self.ids.cpu().numpy().ravel(), 0, rows - 1), minlength=rows)[:, None] + 2)
        assert untouched(flat, dtable, 7.0)
        if weights:
            near(dw, want_w, size_w, cols + 2)
        return dtable


@pytest.mark.parametrize("cols", [1, 7, 8, 9, 40, 511, 513, 1001, 2048])
@pytest.mark.parametrize("tokens,per,rows", [(1, 1, 1), (5, 1, 9), (130, 1, 40), (33, 2, 50), (17, 3, 5), (20, 9, 30)])
def test_lookup_sizes(tokens, per, rows, cols):
    case = Lookup(tokens, per, rows, cols, weights=F32 if per > 1 else None, seed=cols)
    case.forward()
    case.backward()


@pytest.mark.parametrize("table", [BF16, F32])
@pytest.mark.parametrize("y", [BF16, F32])
@pytest.mark.parametrize("weights", [None, BF16, F32])
def test_lookup_types(table, y, weights):
    for per, ids in ((1, I32), (3, I64)):
        case = Lookup(90, per, 23, 136, table, y, weights, 0.37, seed=per, ids=ids)
        case.forward()
        case.forward(accumulate=True)
        case.backward(table)
        case.backward(BF16, accumulate=True)


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8), (7, 2)])
def test_lookup_at_any_alignment(pad, shift):
    for y in (BF16, F32):
        case = Lookup(70, 2, 31, 200, y, y, pad=pad, shift=shift)
        case.forward()
        case.backward(y)


@pytest.mark.parametrize("tokens,rows", [(63, 1), (64, 1), (65, 1), (1000, 1), (4096, 2), (20000, 3), (777, 777), (640, 6000)])
def test_table_gradient_of_long_and_missing_rows(tokens, rows):
    """Rows that go over many chunks of sorted positions, end with one, begin with one; rows without positions."""
    case = Lookup(tokens, 1, rows, 24, seed=rows)
    case.backward(weights=False)
    case.ids = (torch.arange(tokens, device=DEV) * rows // tokens).view(-1, 1)      # runs of equal length
    case.backward(weights=False)


def test_table_gradient_gives_the_same_bits_again():
    case = Lookup(5000, 1, 40, 300, seed=2)
    assert torch.equal(case.backward(weights=False), case.backward(weights=False))


def test_table_gradient_leaves_rows_alone_where_it_adds():
    ids = torch.tensor([[4], [-1], [4]], device=DEV)
    dy = torch.ones(3, 16, dtype=BF16, device=DEV)
    dtable = torch.full((6, 16), float("nan"), device=DEV)
    dtable[4] = 1.5
    u = apm.make_lookup(ids, None, rows=6, cols=16)
    g = apm.make_lookup_grads(u, dy, order=sort(ids, 6)[0], dtable=dtable, accumulate=True)
    apm.apm_lookup_backward(u, g, room(apm.apm_lookup_workspace_bytes(u)))
    assert bool((dtable[4] == 3.5).all()) and bool(dtable[[0, 1, 2, 3, 5]].isnan().all())


def test_ids_that_are_no_rows_leave_no_trace():
    """Neither their weights nor what lies at the table's ends is looked at."""
    table = torch.full((3, 40), float("nan"), dtype=BF16, device=DEV)
    table[1] = 2.0
    ids = torch.tensor([[1, -1], [3, 1], [-5, 1 << 33]], device=DEV)
    weights = torch.tensor([[1.0, float("nan")], [float("inf"), 0.5], [float("nan"), float("nan")]], device=DEV)
    y = torch.empty(3, 40, device=DEV)
    apm.apm_lookup_forward(apm.make_lookup(ids, table, y, weights=weights))
    assert y[:, 0].tolist() == [2.0, 1.0, 0.0]
    dy, dtable, dw = torch.full((3, 40), 3.0, device=DEV), torch.full((3, 40), 7.0, device=DEV), torch.full((3, 2), 7.0, device=DEV)
    dy[2] = float("nan")
    u = apm.make_lookup(ids, table, weights=weights)
    g = apm.make_lookup_grads(u, dy, order=sort(ids, 3)[0], dtable=dtable, dweights=dw)
    apm.apm_lookup_backward(u, g, room(apm.apm_lookup_workspace_bytes(u)))
    assert dtable[:, 0].tolist() == [0.0, 4.5, 0.0]
    assert dw.tolist() == [[240.0, 0.0], [0.0, 240.0], [0.0, 0.0]]


def test_lookup_without_tokens():
    ids, dtable = torch.empty(0, 2, dtype=I64, device=DEV), torch.full((5, 24), 7.0, device=DEV)
    u = apm.make_lookup(ids, torch.ones(5, 24, device=DEV), torch.empty(0, 24, device=DEV))
    apm.apm_lookup_forward(u)
    g = apm.make_lookup_grads(u, torch.empty(0, 24, device=DEV), order=sort(ids, 5)[0], dtable=dtable, dweights=torch.empty(0, 2, device=DEV))
    apm.apm_lookup_backward(u, g, room(apm.apm_lookup_workspace_bytes(u)))
    assert bool((dtable == 0).all())


def test_an_order_of_something_else_stays_inside():
    """Contents that are no order of these ids give other values, and nothing outside dtable is written."""
    case = Lookup(500, 1, 50, 72)
    u = apm.make_lookup(case.ids, case.table)
    flat, dtable = view(50, 72, F32, 3, 5)
    order = torch.randint(-1000, 1000, (500,), dtype=I32, device=DEV, generator=rng(0))
    offsets = torch.randint(-1000, 1000, (51,), device=DEV, generator=rng(1))
    g = apm.make_lookup_grads(u, case.dy, dtable=dtable)
    g.order, g.offsets = order.data_ptr(), offsets.data_ptr()
    size = apm.apm_lookup_workspace_bytes(u)
    wide = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    apm.apm_lookup_backward(u, g, wide[2048:2048 + size])
    assert untouched(flat, dtable, 7.0) and bool((wide[:2048] == 0x5A).all()) and bool((wide[2048 + size:] == 0x5A).all())


def test_lookup_far_in_a_long_table():
    """Rows beyond 2^32 bytes."""
    rows, cols = 2 ** 21 + 3, 1200
    table = torch.empty(rows, cols, dtype=BF16, device=DEV)
    table[-3:] = torch.randn(3, cols, device=DEV, generator=rng(0)).to(BF16)
    ids = torch.tensor([rows - 1, rows - 3, rows - 2], device=DEV)
    y = torch.empty(3, cols, dtype=BF16, device=DEV)
    apm.apm_lookup_forward(apm.make_lookup(ids, table, y))
    assert torch.equal(y, table[ids])
    u = apm.make_lookup(ids, None, rows=rows, cols=cols)
    table.fill_(7.0)
    apm.apm_lookup_backward(u, apm.make_lookup_grads(u, y, order=sort(ids, rows)[0], dtable=table), room(apm.apm_lookup_workspace_bytes(u)))
    assert torch.equal(table[ids], y) and float(table[:-3].abs().max()) == 0.0


# ---- products -----------------------------------------------------------------------------------

def check_product(tokens, out, k, offsets=None, dtype=BF16, bias=None, transposed=False, accumulate=False, pad=0, shift=0, seed=0):
    g = rng(seed)
    groups = len(offsets) - 1 if offsets else 1
    x = view(tokens, k, BF16, pad, shift)[1]
    x.copy_(torch.randn(tokens, k, device=DEV, generator=g))
    w_shape = (k, out) if transposed else (out, k)
    w = view(groups * w_shape[0], w_shape[1], BF16, pad, shift)[1]
    w.copy_(torch.randn(w.shape, device=DEV, generator=g))
    w = torch.as_strided(w, (groups, *w_shape), (w_shape[0] * w.stride(0), w.stride(0), 1), w.storage_offset())
    b = None if bias is None else torch.randn(groups, out, device=DEV, generator=g).to(bias)
    flat, y = view(tokens, out, dtype, pad, shift)
    if accumulate:
        y.copy_(torch.randn(tokens, out, device=DEV, generator=g))
    before = f64(y)
    offs = torch.tensor(offsets, dtype=I64, device=DEV) if offsets else None
    p = apm.make_grouped_product(x, w if offsets else w[0], y, offsets=offs, bias=b, transposed=transposed, accumulate=accumulate)
    apm.apm_grouped_product(p, room(apm.apm_grouped_product_workspace_bytes(p)))
    want, size = T.grouped_product(f64(x), f64(w), offsets or [0, tokens], f64(b), transposed, before)
    if accumulate:
        inside = np.zeros(tokens, bool)
        for a, e in zip((offsets or [0, tokens])[:-1], (offsets or [0, tokens])[1:]):
            inside[max(a, 0):max(e, 0)] = True
        want[inside] += before[inside]
        size[inside] += np.abs(before[inside])
    near(y, want, size, 2 * (k + 16))
    assert untouched(flat, y, 7.0)
    return y


SIZES = [(1, 1, 1), (3, 8, 8), (33, 31, 33), (64, 64, 64), (70, 200, 40), (100, 129, 300), (129, 128, 512), (300, 264, 136), (257, 520, 1000), (1000, 72, 2048)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,out,k", SIZES)
def test_product_sizes(tokens, out, k, transposed):
    check_product(tokens, out, k, transposed=transposed, bias=F32)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("offsets", [[0, 0, 5, 5, 70], [3, 40, 41, 41, 200], [0, 300], [0] * 9 + [130, 290], [0, 1, 2, 3, 4, 5, 300], [100, 100, 100]])
def test_product_of_groups(offsets, transposed):
    for out, k in ((72, 96), (130, 257), (520, 64)):
        check_product(300, out, k, offsets, bias=BF16, transposed=transposed)


@pytest.mark.parametrize("groups", [63, 64, 65, 200, 1000])
def test_product_of_many_groups(groups):
    step = torch.randint(0, 9, (groups,), generator=torch.Generator().manual_seed(groups)).tolist()
    offsets = np.concatenate([[2], 2 + np.cumsum(step)]).tolist()
    check_product(offsets[-1] + 3, 40, 48, offsets, transposed=groups % 2 == 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bias", [None, BF16, F32])
@pytest.mark.parametrize("accumulate", [False, True])
def test_product_forms(dtype, bias, accumulate):
    for tokens, transposed in ((20, False), (150, True), (700, False)):
        check_product(tokens, 136, 264, [0, tokens // 3, tokens - 2], dtype, bias, transposed, accumulate)


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8), (8, 2), (2, 8)])
@pytest.mark.parametrize("transposed", [False, True])
def test_product_at_any_alignment(pad, shift, transposed):
    check_product(90, 200, 152, [0, 31, 90], pad=pad, shift=shift, transposed=transposed)
    check_product(600, 256, 256, [0, 290, 600], pad=pad, shift=shift, transposed=transposed, dtype=F32)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens", [30, 100, 200, 1500])
def test_product_lengths_of_the_sum(tokens, transposed):
    """Around what a stage takes, and fewer stages than are under way."""
    for k in (8, 24, 32, 40, 64, 72, 96, 128, 160, 192, 256, 328, 31, 65, 127, 129, 255):
        check_product(tokens, 136, k, transposed=transposed, seed=k)


def test_product_keeps_infinities_and_nans_in_their_place():
    """What stands behind a group's rows, behind the end of k and in other groups' weights is not mixed in."""
    for k in (40, 37):
        for transposed in (False, True):
            x = torch.randn(200, 64, device=DEV, generator=rng(k)).to(BF16)
            x[:, k:] = float("nan")
            x[50:], x[20, 3] = float("nan"), float("inf")
            w = torch.full((3, *((64, 48) if transposed else (48, 64))), float("nan"), dtype=BF16, device=DEV)
            inside = w[1, :k, :33] if transposed else w[1, :33, :k]
            inside.copy_(torch.randn(inside.shape, device=DEV, generator=rng(1)))
            y = torch.full((200, 33), 7.0, device=DEV)
            offs = torch.tensor([0, 0, 50, 50], device=DEV)
            wide = w[:, :k, :33] if transposed else w[:, :33, :k]
            apm.apm_grouped_product(apm.make_grouped_product(x[:, :k], wide, y, offsets=offs, transposed=transposed))
            got = y.cpu()
            rows = [r for r in range(50) if r != 20]
            assert bool(got[rows].isfinite().all()) and not bool(got[20].isfinite().any()) and bool((got[50:] == 7.0).all())


def test_product_offsets_outside_are_taken_as_the_end_next_to_them():
    x, w = torch.randn(90, 64, device=DEV, generator=rng(0)).to(BF16), torch.randn(3, 72, 64, device=DEV, generator=rng(1)).to(BF16)
    for offsets, same in (([-(1 << 40), 20, 70, 1 << 40], [0, 20, 70, 90]), ([0, 30, 10, 10], [0, 30, 30, 30]), ([95, 100, 200, 300], [90, 90, 90, 90])):
        y = [torch.full((90, 72), 7.0, device=DEV) for _ in range(2)]
        for out, offs in zip(y, (offsets, same)):
            apm.apm_grouped_product(apm.make_grouped_product(x, w, out, offsets=torch.tensor(offs, device=DEV)))
        assert torch.equal(*y)
    flat, y = view(90, 72, F32, 4, 4)            # groups that overlap: anything in y, nothing elsewhere
    apm.apm_grouped_product(apm.make_grouped_product(x, w, y, offsets=torch.tensor([0, 60, 30, 90], device=DEV)))
    assert untouched(flat, y, 7.0)


def test_product_gives_the_same_bits_again():
    a, b = (check_product(700, 264, 520, [0, 100, 101, 650], transposed=True) for _ in range(2))
    assert torch.equal(a, b)


def test_product_of_one_row_for_all_tokens():
    x = torch.randn(1, 64, device=DEV, generator=rng(0)).to(BF16).expand(40, 64)
    w, y = torch.randn(72, 64, device=DEV, generator=rng(1)).to(BF16), torch.empty(40, 72, device=DEV)
    apm.apm_grouped_product(apm.make_grouped_product(x, w, y))
    assert bool((y == y[0]).all())
    near(y, *T.grouped_product(f64(x), f64(w)[None], [0, 40]), 2 * 80)


def test_product_gradients_against_differences():
    """Both gradients of sum(y dy): the input's by this library's transposed product, the weights' as dy^T x."""
    x, w = torch.randn(40, 24, device=DEV, generator=rng(0)).to(BF16), torch.randn(2, 16, 24, device=DEV, generator=rng(1)).to(BF16)
    dy, offs = torch.randn(40, 16, device=DEV, generator=rng(2)).to(BF16), torch.tensor([0, 15, 40], device=DEV)
    dx = torch.empty(40, 24, device=DEV)
    apm.apm_grouped_product(apm.make_grouped_product(dy, w, dx, offsets=offs, transposed=True))
    loss = lambda v: np.sum(T.grouped_product(v, f64(w), [0, 15, 40])[0] * f64(dy))
    for at in ((0, 0), (14, 23), (15, 0), (39, 11)):
        step = np.zeros((40, 24))
        step[at] = 0.5
        want = loss(f64(x) + step) - loss(f64(x) - step)
        assert abs(float(dx[at]) - want) <= 2 * (16 + 20) * U * np.abs(f64(w)).max() * np.abs(f64(dy)).max() * 16


# ---- dropout ------------------------------------------------------------------------------------

def check_dropout(rows, cols, p, seed=0, x=BF16, y=BF16, residual=False, pad=0, shift=0, layer=0, first_row=0):
    g = rng(rows + cols)
    src = view(rows, cols, x, pad, shift)[1]
    src.copy_(torch.randn(rows, cols, device=DEV, generator=g))
    flat, out = view(rows, cols, y, pad, shift)
    r = None
    if residual:
        r = view(rows, cols, y, pad, shift)[1]
        r.copy_(torch.randn(rows, cols, device=DEV, generator=g))
    apm.apm_dropout_apply(apm.make_dropout(src, out, p=p, seed=seed, layer=layer, first_row=first_row, residual=r))
    want = T.dropout(f64(src), p, seed, layer, first_row, f64(r))
    near(out, want, 4 * np.abs(f64(src)) + (np.abs(f64(r)) if residual else 0.0), 1)       # 65536 / (65536 - T) is at most 4 here
    if not residual:
        assert np.array_equal(f64(out) == 0, want == 0)                                     # the mask to the bit
    assert untouched(flat, out, 7.0)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (1, 8), (40, 9), (33, 64), (5, 1001), (2, 4100), (300, 24)])
def test_dropout_sizes(rows, cols):
    check_dropout(rows, cols, 0.25, seed=(rows << 40) + cols)


@pytest.mark.parametrize("x", [BF16, F32])
@pytest.mark.parametrize("y", [BF16, F32])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_forms(x, y, residual):
    for pad, shift in ((0, 0), (3, 1), (8, 8), (1, 5)):
        check_dropout(20, 200, 0.5, 2 ** 64 - 1, x, y, residual, pad, shift, layer=2 ** 32 - 1, first_row=2 ** 40 + 3)


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.75])
def test_dropout_probabilities(p):
    check_dropout(20, 300, p, seed=4)


def test_dropout_of_everything_and_of_numbers_that_are_none():
    x = torch.full((4, 64), float("nan"), device=DEV)
    y = torch.full((4, 64), 7.0, device=DEV)
    apm.apm_dropout_apply(apm.make_dropout(x, y, p=1.0, seed=1))
    assert bool((y == 0).all())
    apm.apm_dropout_apply(apm.make_dropout(x, y, p=1.0, seed=1, residual=torch.ones_like(y)))
    assert bool((y == 1).all())
    apm.apm_dropout_apply(apm.make_dropout(x, y, p=0.5, seed=9))
    assert np.array_equal(np.isnan(f64(y)), T.dropout_bits(4, 64, 9) >= 32768)


def test_dropout_in_place_and_in_pieces():
    x = torch.randn(50, 333, device=DEV, generator=rng(0)).to(BF16)
    r = torch.randn(50, 333, device=DEV, generator=rng(1)).to(BF16)
    whole, into_r = torch.empty_like(x), r.clone()
    apm.apm_dropout_apply(apm.make_dropout(x, whole, p=0.3, seed=5, residual=r))
    apm.apm_dropout_apply(apm.make_dropout(x, into_r, p=0.3, seed=5, residual=into_r))
    pieces = x.clone()
    for a, b in ((0, 13), (13, 14), (14, 50)):
        apm.apm_dropout_apply(apm.make_dropout(pieces[a:b], pieces[a:b], p=0.3, seed=5, first_row=a, residual=r[a:b]))
    assert torch.equal(whole, into_r) and torch.equal(whole, pieces)


def test_dropout_seed_from_device_memory():
    x, y = torch.ones(8, 100, device=DEV), [torch.empty(8, 100, device=DEV) for _ in range(2)]
    word = torch.tensor([-3], device=DEV)
    apm.apm_dropout_apply(apm.make_dropout(x, y[0], p=0.5, seed=10, seed_at=word))
    apm.apm_dropout_apply(apm.make_dropout(x, y[1], p=0.5, seed=7))
    assert torch.equal(*y)


def test_dropout_gradient_is_the_same_call():
    """y is linear in x: the gradient of sum(y dy) is what the call makes of dy."""
    x, dy = torch.randn(6, 50, device=DEV, generator=rng(0)), torch.randn(6, 50, device=DEV, generator=rng(1))
    dx = torch.empty_like(x)
    apm.apm_dropout_apply(apm.make_dropout(dy, dx, p=0.4, seed=3, layer=2))
    loss = lambda v: np.sum(T.dropout(v, 0.4, 3, 2) * f64(dy))
    for at in ((0, 0), (3, 17), (5, 49), (2, 8)):
        step = np.zeros((6, 50))
        step[at] = 0.5
        assert abs(float(dx[at]) - (loss(f64(x) + step) - loss(f64(x) - step))) < 1e-6
