"""Products of weights whose rows overlap: read-only matrices may, and then they can be wider than their rows are apart."""
import pytest
import torch

import paper_2303_02868_amd as apm
from test_gpu_tokens import BF16, DEV

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
