"""Calls on tokens that take several launches: what a launch's last workgroup has to spare is no part of the next launch."""
from contextlib import contextmanager

import pytest
import torch

import paper_2303_02868_amd as apm
from test_gpu_tokens import BF16, DEV, F32, rng, room, sort

pytestmark = pytest.mark.gpu

# Slices of 512 columns, of which a launch has whole rows only: 1, 3, 5 and 7
COLS = [40, 1030, 2501, 3584]
WORKGROUPS = [1, 3, 5]      # of a launch, four wavefronts each


@contextmanager
def launches_of(workgroups):
    assert apm.lib().apm_test_set_launch_workgroups(workgroups) == apm.APM_OK
    try:
        yield
    finally:
        apm.lib().apm_test_set_launch_workgroups(0)


def randn(*shape, dtype=BF16, seed=0):
    return torch.randn(*shape, device=DEV, generator=rng(seed)).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("workgroups", WORKGROUPS)
def test_dropout_in_place(workgroups, cols, dtype):
    x, residual = randn(77, cols, dtype=dtype), randn(77, cols, dtype=dtype, seed=1)
    for r in (None, residual):
        want = torch.empty_like(x)
        apm.apm_dropout_apply(apm.make_dropout(x, want, p=0.25, seed=3, residual=r))
        in_x, in_r = x.clone(), residual.clone()
        with launches_of(workgroups):
            apm.apm_dropout_apply(apm.make_dropout(in_x, in_x, p=0.25, seed=3, residual=r))
            if r is not None:
                apm.apm_dropout_apply(apm.make_dropout(x, in_r, p=0.25, seed=3, residual=in_r))
                assert torch.equal(in_r, want)
        assert torch.equal(in_x, want)


@pytest.mark.parametrize("y", [BF16, F32])
@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("workgroups", WORKGROUPS)
def test_lookup_that_adds(workgroups, cols, y):
    ids = torch.randint(-1, 40, (101, 2), device=DEV, generator=rng(2))
    table, before = randn(40, cols), randn(101, cols, dtype=y, seed=1)
    want, got = before.clone(), before.clone()
    apm.apm_lookup_forward(apm.make_lookup(ids, table, want, accumulate=True))
    with launches_of(workgroups):
        apm.apm_lookup_forward(apm.make_lookup(ids, table, got, accumulate=True))
    assert torch.equal(got, want)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("workgroups", WORKGROUPS)
def test_gradients(workgroups, cols, dtype, accumulate):
    """Rows inside of a chunk of positions, rows that go over several, rows without any."""
    ids = torch.randint(-1, 300, (211, 2), device=DEV, generator=rng(2))
    ids[::5] = 7
    table, weights, dy, before = randn(300, cols), randn(211, 2, dtype=F32, seed=1), randn(211, cols, seed=3), randn(300, cols, dtype=dtype, seed=4)
    order = sort(ids, 300)[0]
    lookup = apm.make_lookup(ids, table, weights=weights)
    workspace = room(apm.apm_lookup_workspace_bytes(lookup))

    def gradients():
        dtable, dweights = before.clone(), torch.full((211, 2), 7.0, dtype=dtype, device=DEV)
        apm.apm_lookup_backward(lookup, apm.make_lookup_grads(lookup, dy, order=order, dtable=dtable, dweights=dweights, accumulate=accumulate), workspace)
        return dtable, dweights

    want = gradients()
    with launches_of(workgroups):
        got = gradients()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
