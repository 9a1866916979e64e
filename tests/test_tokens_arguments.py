"""Refusals of the calls on tokens: they come from the arguments alone, before anything is launched, so they need no GPU."""
import pytest

import paper_2303_02868_amd as apm
from test_activations_arguments import OnGpu
from test_activations_host import PTR, matrix, refused


def indices(data=PTR, type=apm.APM_I64):
    return apm.apm_indices(data, type, 0)


def change(s, over):
    for k, v in over.items():
        setattr(s, k, v)
    return s


def order(**over):
    return change(apm.apm_token_order(8, 2, 10, indices(), PTR, PTR, PTR, PTR), over)


def test_sorting():
    need = apm.apm_sort_tokens_workspace_bytes(order(n=100000))
    go = lambda room=PTR, size=1 << 40, **o: apm.lib().apm_sort_tokens(order(**o), room, size, None)
    for bad in (dict(n=-1), dict(n=apm.APM_MAX_POSITIONS + 1), dict(rows=0), dict(rows=apm.APM_MAX_POSITIONS + 1), dict(per_token=0)):
        refused(go(**bad), apm.APM_EINVAL, "bad size")
        assert apm.apm_sort_tokens_workspace_bytes(order(**bad)) == 0
    refused(go(ids=indices(None)), apm.APM_EINVAL, "ids is missing")
    refused(go(ids=indices(type=2)), apm.APM_EINVAL, "ids: bad type")
    refused(go(ids=indices(PTR + 4)), apm.APM_EINVAL, "ids is not aligned")
    refused(go(order=None), apm.APM_EINVAL, "order is missing")
    for bad in (dict(order=PTR + 2), dict(place=PTR + 1), dict(token=PTR + 2), dict(offsets=PTR + 4)):
        refused(go(**bad), apm.APM_EINVAL, "not aligned")
    refused(go(n=100000, size=need - 1), apm.APM_ENOMEM, "workspace")
    refused(go(n=100000, room=None), apm.APM_EINVAL, "workspace")
    refused(go(n=100000, room=PTR + 8), apm.APM_EINVAL, "workspace")
    refused(apm.lib().apm_sort_tokens(None, None, 0, None), apm.APM_EINVAL, "missing")
    assert apm.apm_sort_tokens_workspace_bytes(None) == 0


def lookup(**over):
    u = apm.apm_lookup(4, 2, 10, 64, 1.0, indices(), apm.apm_vector(PTR, apm.APM_F32, 0), matrix(), matrix(), 0, 0)
    return change(u, over)


def test_lookup_forward():
    go = lambda **o: apm.lib().apm_lookup_forward(lookup(**o), None)
    for bad in (dict(tokens=-1), dict(per_token=0), dict(rows=0), dict(rows=apm.APM_MAX_POSITIONS + 1), dict(cols=0), dict(cols=2 ** 28 + 1),
                dict(tokens=2 ** 30, per_token=2), dict(tokens=2 ** 62, per_token=8), dict(tokens=1, per_token=2 ** 62)):
        refused(go(**bad), apm.APM_EINVAL, "bad size")
        assert apm.apm_lookup_workspace_bytes(lookup(**bad)) == 0
    refused(go(ids=indices(None)), apm.APM_EINVAL, "ids is missing")
    refused(go(weights=apm.apm_vector(PTR + 2, apm.APM_F32, 0)), apm.APM_EINVAL, "weights is not aligned")
    refused(go(weights=apm.apm_vector(PTR, 5, 0)), apm.APM_EINVAL, "weights: bad dtype")
    refused(go(table=matrix(None)), apm.APM_EINVAL, "table is missing")
    refused(go(table=matrix(dtype=3)), apm.APM_EINVAL, "table: bad dtype")
    refused(go(y=matrix(None)), apm.APM_EINVAL, "y is missing")
    refused(go(y=matrix(stride=63)), apm.APM_EINVAL, "y: a row stride")
    refused(apm.lib().apm_lookup_forward(None, None), apm.APM_EINVAL, "missing")
    assert go(tokens=0, y=matrix(None)) == apm.APM_OK


def test_lookup_backward():
    need = apm.apm_lookup_workspace_bytes(lookup())
    assert need > 0

    def go(u=None, room=PTR, size=need, **over):
        g = apm.apm_lookup_grads(matrix(), matrix(), apm.apm_vector(PTR, apm.APM_F32, 0), PTR, PTR, 0, 0)
        return apm.lib().apm_lookup_backward(u or lookup(), change(g, over), room, size, None)

    refused(go(lookup(cols=0)), apm.APM_EINVAL, "bad size")
    refused(go(lookup(ids=indices(None))), apm.APM_EINVAL, "ids is missing")
    refused(go(dy=matrix(None)), apm.APM_EINVAL, "dy is missing")
    refused(go(dtable=matrix(stride=1)), apm.APM_EINVAL, "dtable: a row stride")
    refused(go(order=None), apm.APM_EINVAL, "order and offsets")
    refused(go(offsets=None), apm.APM_EINVAL, "order and offsets")
    refused(go(order=PTR + 2), apm.APM_EINVAL, "not aligned")
    refused(go(offsets=PTR + 4), apm.APM_EINVAL, "not aligned")
    refused(go(size=need - 1), apm.APM_ENOMEM, "workspace")
    refused(go(room=None), apm.APM_EINVAL, "workspace")
    refused(go(dweights=apm.apm_vector(PTR + 1, apm.APM_BF16, 0)), apm.APM_EINVAL, "dweights")
    refused(go(lookup(table=matrix(None))), apm.APM_EINVAL, "table is missing")
    refused(go(lookup(tokens=2 ** 20, per_token=2 ** 10, cols=2 ** 20), dtable=matrix(stride=2 ** 20), dy=matrix(stride=2 ** 20), size=1 << 60), apm.APM_EINVAL, "too many")
    refused(apm.lib().apm_lookup_backward(None, None, None, 0, None), apm.APM_EINVAL, "missing")
    nothing = apm.apm_vector(None, 0, 0)
    assert go(dtable=matrix(None), dweights=nothing, order=None, offsets=None, room=None, size=0) == apm.APM_OK


def product(**over):
    p = apm.apm_grouped_product_desc(100, 64, 64, 4, PTR, matrix(), matrix(), matrix(), 4096, apm.apm_vector(PTR, apm.APM_F32, 0), 0, 0)
    return change(p, over)


def test_grouped_product():
    go = lambda room=PTR, size=1 << 40, **o: apm.lib().apm_grouped_product(product(**o), room, size, None)
    for bad in (dict(tokens=-1), dict(tokens=2 ** 41), dict(out=0), dict(out=2 ** 28 + 1), dict(n_groups=-1), dict(n_groups=apm.APM_MAX_GROUPS + 1), {"in": 0}, {"in": 2 ** 31}):
        refused(go(**bad), apm.APM_EINVAL, "bad size")
        assert apm.apm_grouped_product_workspace_bytes(product(**bad)) == 0
    refused(go(offsets=None), apm.APM_EINVAL, "contradict")
    refused(go(n_groups=0), apm.APM_EINVAL, "contradict")
    refused(go(offsets=PTR + 4), apm.APM_EINVAL, "offsets are not aligned")
    refused(go(x=matrix(None)), apm.APM_EINVAL, "x is missing")
    refused(go(x=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "x must be bf16")
    refused(go(w=matrix(None)), apm.APM_EINVAL, "w is missing")
    refused(go(w=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "w must be bf16")
    refused(go(w_group_stride=-1), apm.APM_EINVAL, "too far")
    refused(go(w_group_stride=1 << 56), apm.APM_EINVAL, "too far")
    refused(go(bias=apm.apm_vector(PTR + 1, apm.APM_BF16, 0)), apm.APM_EINVAL, "bias is not aligned")
    refused(go(y=matrix(None)), apm.APM_EINVAL, "y is missing")
    refused(go(y=matrix(stride=63)), apm.APM_EINVAL, "y: a row stride")
    refused(go(tokens=2 ** 40, out=2 ** 28, y=matrix(stride=2 ** 28), x=matrix(stride=0), size=1 << 62), apm.APM_EINVAL, "")
    refused(apm.lib().apm_grouped_product(None, None, 0, None), apm.APM_EINVAL, "missing")
    assert go(tokens=0) == apm.APM_OK


def dropout(**over):
    return change(apm.apm_dropout(4, 64, 0.5, 1, None, 0, 0, 0, matrix(), matrix(), matrix()), over)


def test_dropout():
    go = lambda **o: apm.lib().apm_dropout_apply(dropout(**o), None)
    for bad in (dict(rows=-1), dict(cols=0), dict(cols=2 ** 28 + 1), dict(first_row=-1)):
        refused(go(**bad), apm.APM_EINVAL, "bad size")
    for p in (-0.1, 1.1, float("nan")):
        refused(go(p=p), apm.APM_EINVAL, "no probability")
    refused(go(seed_at=PTR + 4), apm.APM_EINVAL, "seed_at is not aligned")
    refused(go(x=matrix(None)), apm.APM_EINVAL, "x is missing")
    refused(go(y=matrix(stride=32)), apm.APM_EINVAL, "y: a row stride")
    refused(go(residual=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "different types")
    refused(go(residual=matrix(PTR + 1)), apm.APM_EINVAL, "residual is not aligned")
    refused(go(x=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "in another form")
    refused(go(x=matrix(stride=128), rows=2), apm.APM_EINVAL, "in another form")
    refused(go(x=matrix(PTR + 16), residual=matrix(stride=128), rows=2), apm.APM_EINVAL, "in another form")
    refused(apm.lib().apm_dropout_apply(None, None), apm.APM_EINVAL, "missing")
    assert go(rows=0) == apm.APM_OK


def test_the_binding_looks_at_shapes_and_types(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2303_02868_amd import binding
    here = [0]
    monkeypatch.setattr(binding, "_here", lambda: here[0])

    class Here(OnGpu):
        def __getitem__(self, i):
            part = Here(torch, self.device, 1, dtype=self.t.dtype)
            part.t = self.t[i]
            return part

    on = lambda *s, dtype=torch.bfloat16, device=0: Here(torch, device, *s, dtype=dtype)
    i32, i64 = (lambda *s, **k: on(*s, dtype=torch.int32, **k)), (lambda *s, **k: on(*s, dtype=torch.int64, **k))
    wrong = [
        (lambda: apm.make_token_order(on(4), 3, i32(4)), "int32 or int64"),
        (lambda: apm.make_token_order(i64(4, 2, 2), 3, i32(16)), "ids of a token"),
        (lambda: apm.make_token_order(i64(4, 4)[(slice(None), slice(2))], 3, i32(8)), "contiguous"),
        (lambda: apm.make_token_order(i64(4, 2), 3, i32(4)), "order"),
        (lambda: apm.make_token_order(i64(4), 3, i64(4)), "order"),
        (lambda: apm.make_token_order(i64(4), 3, i32(4), offsets=i64(3)), "offsets"),
        (lambda: apm.make_token_order(i64(4), 3, i32(4), place=i32(5)), "place"),
        (lambda: apm.make_token_order(i64(4), 3, i32(4), token=i32(4, device=1)), "on GPU 1"),
        (lambda: apm.make_lookup(i64(4), on(3, 64), on(5, 64)), "y"),
        (lambda: apm.make_lookup(i64(4), on(3, 64), on(4, 64), weights=on(5)), "weights"),
        (lambda: apm.make_lookup(i64(4), None), "rows and cols"),
        (lambda: apm.make_grouped_product(on(4, 64), on(2, 32, 64), on(4, 32), offsets=i64(2)), "weights of"),
        (lambda: apm.make_grouped_product(on(4, 64), on(2, 32, 60), on(4, 32), offsets=i64(3)), "w"),
        (lambda: apm.make_grouped_product(on(4, 64), on(32, 64), on(4, 32), transposed=True), "w"),
        (lambda: apm.make_grouped_product(on(4, 64), on(2, 32, 64), on(4, 32), offsets=i64(3), bias=on(32)), "bias"),
        (lambda: apm.make_grouped_product(on(4, 64), on(2, 32, 64), on(4, 32), offsets=i32(3)), "offsets"),
        (lambda: apm.make_dropout(on(4, 64), on(4, 32), p=0.5, seed=1), "y"),
        (lambda: apm.make_dropout(on(4, 64), on(4, 64), p=0.5, seed=1, seed_at=i32(1)), "seed_at"),
        (lambda: apm.make_dropout(on(4, 64), on(4, 64), p=0.5, seed=1, residual=on(4, 64, device=1)), "on GPU 1"),
    ]
    for call, word in wrong:
        with pytest.raises(ValueError, match=word):
            call()
    made = apm.make_token_order(i64(4, 2), 3, i32(8), offsets=i64(4))
    u = apm.make_lookup(i64(4, 2), on(3, 64), on(4, 64))
    with pytest.raises(ValueError, match="order"):
        apm.make_lookup_grads(apm.make_lookup(i64(4), on(3, 64)), on(4, 64), order=made, dtable=on(3, 64))
    g = apm.make_lookup_grads(u, on(4, 64), order=made, dtable=on(3, 64))
    p, d = apm.make_grouped_product(on(4, 64), on(32, 64), on(4, 32)), apm.make_dropout(on(4, 64), on(4, 64), p=0.5, seed=1)
    here[0] = 1
    for call in (lambda: apm.apm_sort_tokens(made), lambda: apm.apm_lookup_forward(u), lambda: apm.apm_lookup_backward(u, g),
                 lambda: apm.apm_grouped_product(p), lambda: apm.apm_dropout_apply(d)):
        with pytest.raises(ValueError, match="looked at for GPU 0, the current one is 1"):
            call()
