"""Calls on tokens where they are rarely made: every tile of the products, long sorts, streams, captured graphs, the widest rows."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle.tokens as T
import paper_2303_02868_amd as apm
from test_gpu_tokens import BF16, DEV, F32, I32, I64, Lookup, check_product, check_sort, rng, room, sort, untouched, view

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [3, 64, 300, 70000])
@pytest.mark.parametrize("n", [524288, 524289, 2000001])
def test_sort_of_many_positions(n, rows):
    ids = torch.randint(-1, rows + 1, (n,), device=DEV, generator=rng(rows))
    check_sort(torch.where(ids % 4 == 0, ids % 2, ids), rows)


@pytest.mark.parametrize("rows", [1, 5000, 70000])
def test_sort_where_a_row_has_nearly_all(rows):
    ids = torch.full((50001,), rows // 2, device=DEV)
    ids[::1000] = torch.arange(51, device=DEV) % rows
    check_sort(ids, rows)


def test_bags_of_many_rows():
    for per in (15, 16, 17, 40, 300):
        case = Lookup(9, per, 70, 72, weights=F32, seed=per)
        case.forward()
        case.backward()


def tile_of(tokens, out, k, groups, transposed, aligned):
    """Rows of the tile that such a product takes."""
    shift = 0 if aligned else 2
    at = lambda stride: apm.apm_matrix((1 << 30) + shift, stride, apm.APM_BF16, 0)
    w = k * out
    p = apm.apm_grouped_product_desc(tokens, out, k, groups, (1 << 30) if groups else None, at(k), at(out if transposed else k), at(out), w, apm.apm_vector(None, 0, 0),
                                     int(transposed), 0)
    return apm.lib().apm_test_grouped_product_tile(C.byref(p))


TILES = {256: (6100, 2056, 328), 128: (6850, 1032, 136), 64: (1300, 520, 136), 32: (40, 136, 1096)}


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("rows", sorted(TILES))
def test_products_on_every_tile(rows, aligned, transposed):
    tokens, out, k = TILES[rows]
    for groups in (0, 3):
        assert tile_of(tokens, out, k, groups, transposed, aligned) == rows
        offsets = [0, tokens // 5, tokens // 5 + 1, tokens - 7] if groups else None
        check_product(tokens, out, k, offsets, bias=F32, transposed=transposed, shift=0 if aligned else 1, seed=rows)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,tokens,k", [(192, 5100, 328), (192, 5100, 448), (-128, 7900, 1096), (-64, 255, 4168)])
def test_products_on_tiles_for_whole_vectors(rows, tokens, k, transposed):
    out = 2056
    for groups in (0, 3):
        assert tile_of(tokens, out, k, groups, transposed, True) == rows
        offsets = [0, tokens // 5, tokens // 5 + 1, tokens - 7] if groups else None
        check_product(tokens, out, k, offsets, bias=F32, transposed=transposed, accumulate=bool(groups), seed=k)
    assert tile_of(tokens, out, k, 0, transposed, False) != rows


@pytest.mark.parametrize("tokens,out,k", [(6100, 2056, 328), (5100, 2056, 328), (7900, 2056, 1096), (6850, 1032, 136), (1300, 520, 136), (255, 2056, 4168), (40, 136, 1096)])
def test_groups_that_overlap_write_inside_of_y(tokens, out, k):
    x, w = torch.randn(tokens, k, device=DEV, generator=rng(0)).to(BF16), torch.randn(3, out, k, device=DEV, generator=rng(1)).to(BF16)
    flat, y = view(tokens, out, F32, 4, 4)
    offsets = torch.tensor([0, tokens, tokens // 3, tokens + 9], device=DEV)
    apm.apm_grouped_product(apm.make_grouped_product(x, w, y, offsets=offsets))
    assert untouched(flat, y, 7.0)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("out,k", [(1024, 1024), (1032, 1088), (520, 1100)])
def test_products_of_groups_that_begin_at_different_k(out, k, transposed):
    """Groups of one row of tiles each, more of them than stages; whole and not."""
    sizes = [(37 * g) % 97 for g in range(40)]
    ends = [0]
    for s in sizes: ends.append(ends[-1] + s)
    check_product(ends[-1] + 3, out, k, ends, bias=F32, transposed=transposed, accumulate=True, seed=k)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows", sorted(TILES))
def test_products_of_odd_sizes_on_every_tile(rows, transposed):
    tokens, out, k = TILES[rows]
    tokens, out, k = tokens + 1, out - 3, k + 5
    assert tile_of(tokens, out, k, 0, transposed, False) == rows
    check_product(tokens, out, k, bias=BF16, dtype=F32, transposed=transposed, accumulate=True)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows,sizes", [(256, (6100, 2056, 1096)), (192, (5000, 2056, 1096)), (128, (2048, 2048, 1032)), (-128, (3000, 2048, 1032))])
def test_products_of_long_sums(rows, sizes, transposed):
    """More stages than are under way, again and again."""
    assert tile_of(*sizes, 0, transposed, True) == rows
    check_product(*sizes, transposed=transposed)


class Step:
    """The calls of a step with static buffers, on a stream."""

    def __init__(self, seed, tokens=700, per=2, rows=50, cols=136, out=72):
        g = rng(seed)
        self.ids = torch.randint(-1, rows, (tokens, per), device=DEV, generator=g)
        self.table, self.weights = torch.randn(rows, cols, device=DEV, generator=g).to(BF16), torch.rand(tokens, per, device=DEV, generator=g)
        self.w = torch.randn(rows, out, cols, device=DEV, generator=g).to(BF16)
        n = tokens * per
        self.order, self.place, self.token = (torch.empty(n, dtype=I32, device=DEV) for _ in range(3))
        self.offsets, self.word = torch.empty(rows + 1, dtype=I64, device=DEV), torch.zeros(1, dtype=I64, device=DEV)
        self.y, self.sorted, self.product = torch.empty(tokens, cols, dtype=BF16, device=DEV), torch.empty(n, cols, dtype=BF16, device=DEV), torch.zeros(n, out, device=DEV)
        self.dropped, self.dtable = torch.empty(n, out, device=DEV), torch.empty(rows, cols, device=DEV)
        self.dweights = torch.empty(tokens, per, device=DEV)
        self.sort = apm.make_token_order(self.ids, rows, self.order, offsets=self.offsets, place=self.place, token=self.token)
        self.lookup = apm.make_lookup(self.ids, self.table, self.y, weights=self.weights)
        self.dispatch = apm.make_lookup(self.token, self.y, self.sorted)
        self.experts = apm.make_grouped_product(self.sorted, self.w, self.product, offsets=self.offsets)
        self.dropout = apm.make_dropout(self.product, self.dropped, p=0.3, seed=5, seed_at=self.word)
        self.grads = apm.make_lookup_grads(self.lookup, self.y, order=self.sort, dtable=self.dtable, dweights=self.dweights)
        self.rooms = [room(max(16, b)) for b in (apm.apm_sort_tokens_workspace_bytes(self.sort), apm.apm_lookup_workspace_bytes(self.lookup),
                                                 apm.apm_grouped_product_workspace_bytes(self.experts))]

    def run(self, stream):
        apm.apm_sort_tokens(self.sort, self.rooms[0], stream)
        apm.apm_lookup_forward(self.lookup, stream)
        apm.apm_lookup_forward(self.dispatch, stream)
        apm.apm_grouped_product(self.experts, self.rooms[2], stream)
        apm.apm_dropout_apply(self.dropout, stream)
        apm.apm_lookup_backward(self.lookup, self.grads, self.rooms[1], stream)

    def outputs(self):
        return [t.clone() for t in (self.order, self.offsets, self.place, self.token, self.y, self.sorted, self.product, self.dropped, self.dtable, self.dweights)]


def test_captured_and_replayed():
    """Each replay reads what is in the buffers then, and gives the bits of the calls themselves, with other work and waits in between."""
    live, eager = Step(1), Step(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        live.run(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        live.run(side)
    masks = []
    for turn in range(5):
        for s in (live, eager):
            s.ids.copy_(torch.randint(-1, 50, s.ids.shape, device=DEV, generator=rng(turn)))
            s.table.copy_(torch.randn(s.table.shape, device=DEV, generator=rng(turn + 10)))
            s.word.fill_(turn)
            s.product.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager.run(None)
        torch.cuda.synchronize()
        for got, want in zip(live.outputs(), eager.outputs()):
            assert torch.equal(got, want)
        masks.append((live.dropped[:600] == 0) & (live.product[:600] != 0))
    assert not torch.equal(masks[0], masks[1])


def test_two_streams_at_once():
    steps, streams = [Step(3), Step(4)], [torch.cuda.Stream(), torch.cuda.Stream()]
    want = []
    for s in steps:
        s.run(None)
        torch.cuda.synchronize()
        want.append(s.outputs())
    torch.cuda.synchronize()
    for _ in range(20):
        for s, stream in zip(steps, streams):
            s.run(stream)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        for a, b in zip(s.outputs(), w):
            assert torch.equal(a, b)


def test_the_widest_rows():
    cols = 1 << 28
    x = torch.ones(1, cols, dtype=BF16, device=DEV)
    y = torch.empty_like(x)
    apm.apm_dropout_apply(apm.make_dropout(x, y, p=0.5, seed=3))
    words = [T.philox((cols // 8 - 1 - b, 0, 0, 0), (3, 0)) for b in (1, 0)]
    kept = np.array([(w[i // 2] >> (16 * (i % 2))) % 65536 >= 32768 for w in words for i in range(8)])
    assert np.array_equal(y[0, -16:].float().cpu().numpy(), np.where(kept, 2.0, 0.0))
    x[0, -3:] = torch.tensor([3.0, 4.0, 5.0])
    ids = torch.zeros(1, dtype=I64, device=DEV)
    apm.apm_lookup_forward(apm.make_lookup(ids, x, y, scale=2.0))
    assert y[0, -4:].tolist() == [2.0, 6.0, 8.0, 10.0] and float(y[0, :-3].float().sum(dtype=torch.float64)) == 2.0 * (cols - 3)


def test_rows_far_apart():
    """Distances between rows beyond 32 bits, where the products' loads do not go by 32-bit offsets."""
    far = (1 << 31) + 8
    buf = torch.zeros(far + 200, dtype=BF16, device=DEV)
    x = torch.as_strided(buf, (2, 96), (far, 1))
    x.copy_(torch.randn(2, 96, device=DEV, generator=rng(0)))
    w = torch.randn(40, 96, device=DEV, generator=rng(1)).to(BF16)
    got, want = torch.empty(2, 40, device=DEV), torch.empty(2, 40, device=DEV)
    apm.apm_grouped_product(apm.make_grouped_product(x, w, got))
    apm.apm_grouped_product(apm.make_grouped_product(x.contiguous(), w, want))
    near = (got - want).abs() <= 2 * 112 * 2.0 ** -24 * (x.float().abs() @ w.float().abs().T)      # another kernel: sums in another order
    assert bool(near.all())
    out = torch.as_strided(buf, (2, 96), (far, 1), 100)
    apm.apm_lookup_forward(apm.make_lookup(torch.tensor([1, 0], device=DEV), x, out))
    assert torch.equal(out, x.flip(0))
    apm.apm_dropout_apply(apm.make_dropout(x, out, p=0.0, seed=1))
    assert torch.equal(out, x)
