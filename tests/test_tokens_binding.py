"""What the binding of the calls on tokens takes for what: types of words, and structures laid out as the header has them."""
import pytest

import paper_2303_02868_amd as apm
from test_activations_arguments import OnGpu


def test_the_seed_is_a_whole_number(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2303_02868_amd import binding
    monkeypatch.setattr(binding, "_here", lambda: 0)
    on = lambda *s, dtype=torch.bfloat16: OnGpu(torch, 0, *s, dtype=dtype)
    make = lambda word: apm.make_dropout(on(4, 64), on(4, 64), p=0.5, seed=1, seed_at=word)
    for dtype in (torch.int64, torch.uint64):
        assert make(on(1, dtype=dtype)).seed_at
    for dtype in (torch.float64, torch.complex64, torch.int32, torch.uint32):
        with pytest.raises(ValueError, match="seed_at"):
            make(on(1, dtype=dtype))
    with pytest.raises(ValueError, match="seed_at"):
        make(on(2, dtype=torch.int64))


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    """Sizes, and where each field is: the binding fills them from packed words."""
    import ctypes as C
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structures = [apm.apm_indices, apm.apm_token_order, apm.apm_lookup, apm.apm_lookup_grads, apm.apm_grouped_product_desc, apm.apm_dropout]
    want, lines = [], []
    for s in structures:
        want.append(C.sizeof(s))
        lines.append(f'printf("%zu ", sizeof({s.__name__}));')
        for name, _ in s._fields_:
            want.append(getattr(s, name).offset)
            lines.append(f'printf("%zu ", offsetof({s.__name__}, {name}));')
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "apm.h"\nint main(void) {' + "".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    assert [int(v) for v in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split()] == want


def test_packed_words_are_the_fields(monkeypatch):
    """Each field of a structure that is made holds what it was given, and no other's."""
    torch = pytest.importorskip("torch")
    from paper_2303_02868_amd import binding
    monkeypatch.setattr(binding, "_here", lambda: 0)
    on = lambda *s, dtype=torch.bfloat16: OnGpu(torch, 0, *s, dtype=dtype)
    i32, i64, f32 = torch.int32, torch.int64, torch.float32

    def same(matrix, t, dtype):
        assert (matrix.data, matrix.stride, matrix.dtype) == (t.data_ptr(), t.stride()[0], dtype)

    ids, order, offsets, place, token = on(4, 2, dtype=i64), on(8, dtype=i32), on(4, dtype=i64), on(8, dtype=i32), on(8, dtype=i32)
    o = apm.make_token_order(ids, 3, order, offsets=offsets, place=place, token=token)
    assert (o.n, o.per_token, o.rows, o.ids.data, o.ids.type) == (8, 2, 3, ids.data_ptr(), apm.APM_I64)
    assert (o.order, o.offsets, o.place, o.token) == tuple(t.data_ptr() for t in (order, offsets, place, token))
    table, y, weights = on(3, 64), on(4, 64, dtype=f32), on(4, 2, dtype=f32)
    u = apm.make_lookup(ids, table, y, scale=0.25, weights=weights, accumulate=True)
    assert (u.tokens, u.per_token, u.rows, u.cols, u.scale, u.accumulate) == (4, 2, 3, 64, 0.25, 1)
    assert (u.ids.data, u.ids.type, u.weights.data, u.weights.dtype) == (ids.data_ptr(), apm.APM_I64, weights.data_ptr(), apm.APM_F32)
    same(u.table, table, apm.APM_BF16)
    same(u.y, y, apm.APM_F32)
    dy, dtable, dweights = on(4, 64), on(3, 64, dtype=f32), on(4, 2)
    g = apm.make_lookup_grads(u, dy, order=o, dtable=dtable, dweights=dweights, accumulate=True)
    same(g.dy, dy, apm.APM_BF16)
    same(g.dtable, dtable, apm.APM_F32)
    assert (g.dweights.data, g.dweights.dtype, g.order, g.offsets, g.accumulate) == (dweights.data_ptr(), apm.APM_BF16, order.data_ptr(), offsets.data_ptr(), 1)
    x, w, out, bias, ends = on(5, 64), on(2, 64, 40), on(5, 40, dtype=f32), on(2, 40), on(3, dtype=i64)
    p = apm.make_grouped_product(x, w, out, offsets=ends, bias=bias, transposed=True, accumulate=False)
    assert (p.tokens, p.out, getattr(p, "in"), p.n_groups, p.offsets, p.w_group_stride, p.transposed, p.accumulate) == (5, 40, 64, 2, ends.data_ptr(), 64 * 40, 1, 0)
    for m, t, dtype in ((p.x, x, apm.APM_BF16), (p.y, out, apm.APM_F32)):
        same(m, t, dtype)
    assert (p.w.data, p.w.stride, p.w.dtype, p.bias.data, p.bias.dtype) == (w.data_ptr(), 40, apm.APM_BF16, bias.data_ptr(), apm.APM_BF16)
    src, residual, dropped, word = on(6, 24), on(6, 24, dtype=f32), on(6, 24, dtype=f32), on(1, dtype=i64)
    d = apm.make_dropout(src, dropped, p=0.375, seed=-2, layer=9, first_row=1 << 40, residual=residual, seed_at=word)
    assert (d.rows, d.cols, d.p, d.seed, d.seed_at, d.first_row, d.layer) == (6, 24, 0.375, 2 ** 64 - 2, word.data_ptr(), 1 << 40, 9)
    for m, t, dtype in ((d.x, src, apm.APM_BF16), (d.residual, residual, apm.APM_F32), (d.y, dropped, apm.APM_F32)):
        same(m, t, dtype)
