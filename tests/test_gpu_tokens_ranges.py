"""Calls on tokens at the ends of their ranges: weights whose rows overlap, as read-only matrices may, and are wider than they are apart; very many rows; probabilities between two."""
import numpy as np
import pytest
import torch

import oracle.tokens as T
import paper_2303_02868_amd as apm
from test_gpu_tokens import BF16, DEV, rng

pytestmark = pytest.mark.gpu


def test_what_is_behind_the_end_of_the_sum_stays_out_of_it():
    """The element 2^30 behind the first is one of the matrix here, as it is wide, and infinite: it is in the sums of its own columns and in no other."""
    k, out, apart = 4104, 1 << 26, 246264          # k ends inside a stage
    buf = torch.zeros((k - 1) * apart + out, dtype=BF16, device=DEV)
    buf[1 << 30:(1 << 30) + 8] = float("inf")
    w = torch.as_strided(buf, (k, out), (apart, 1))
    x, y = torch.ones(1, k, dtype=BF16, device=DEV), torch.full((1, out), 7.0, dtype=BF16, device=DEV)
    apm.apm_grouped_product(apm.make_grouped_product(x, w, y, transposed=True))
    want = torch.zeros(out, dtype=torch.bool, device=DEV)
    for r in range(((1 << 30) - out) // apart, k):
        for i in range(8):
            c = (1 << 30) + i - r * apart
            if 0 <= c < out:
                want[c] = True
    assert int(want.sum()) > 8 and not bool(want[:1 << 20].any())
    there, elsewhere = int(((y[0] == float("inf")) & want).sum()), int(((y[0] == 0) & ~want).sum())
    assert there == int(want.sum()) and elsewhere == out - there


@pytest.mark.parametrize("tokens", [(1 << 29) + 3, (1 << 30) + 70])
def test_more_rows_than_a_grid_of_the_smallest_tiles_holds(tokens):
    """w changes the order of the columns, so that y is x to the bit."""
    x = torch.empty(tokens, 8, dtype=BF16, device=DEV)
    x.view(torch.int16).random_(0, 0x4000, generator=rng(1))
    x.masked_fill_(x.abs() < 2.0 ** -100, 1.0)                 # the smallest may be taken as zero
    w = torch.eye(8, dtype=BF16, device=DEV).flip(0).contiguous()
    y = torch.empty_like(x)
    apm.apm_grouped_product(apm.make_grouped_product(x, w, y))
    step = 1 << 27
    for at in range(0, tokens, step):
        assert bool((y[at:at + step] == x[at:at + step].flip(1)).all()), at


@pytest.mark.parametrize("bound", [1, 3, 4, 16385, 32769, 65535, 65536])
def test_probabilities_between_two_bounds_take_the_upper_one(bound):
    """What is kept is multiplied by 65536 / (65536 - T), of which T can be told, in fp32 rounded twice at most."""
    x = torch.ones(8, 4096, device=DEV)
    y = torch.empty_like(x)
    p = (bound - 0.5) / 65536
    apm.apm_dropout_apply(apm.make_dropout(x, y, p=p, seed=4))
    kept = T.dropout_bits(8, 4096, 4) >= bound
    want = T.dropout(np.ones((8, 4096)), p, 4)
    got = y.double().cpu().numpy()
    assert np.array_equal(got != 0, kept) and np.array_equal(want != 0, kept)
    assert np.all(np.abs(got - want) <= 2.0 ** -23 * want)
