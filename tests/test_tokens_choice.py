"""Which kernel a product takes, and which it refuses: decided on the host, from sizes and strides alone."""
import ctypes as C

import pytest

import paper_2303_02868_amd as apm
from test_activations_host import PTR


def product(tokens, out, k, *, x=None, w=None, transposed=False):
    """x and w: elements between rows, where rows do not follow each other."""
    at = lambda stride: apm.apm_matrix(PTR, stride, apm.APM_BF16, 0)
    return apm.apm_grouped_product_desc(tokens, out, k, 0, None, at(k if x is None else x), at((out if transposed else k) if w is None else w), at(out), 0,
                                        apm.apm_vector(None, 0, 0), int(transposed), 0)


def tile(*sizes, **strides):
    return apm.lib().apm_test_grouped_product_tile(C.byref(product(*sizes, **strides)))


@pytest.mark.parametrize("which", ["x", "w"])
def test_overlapping_rows_behind_the_reach_of_a_load_go_through_registers(which):
    """-128: a tile that goes straight into LDS, whose loads reach 2^30 elements from the first of 256 rows; 128: one that goes through registers."""
    apart, other = (1 << 22) - 8, "w" if which == "x" else "x"
    most = (1 << 30) - 255 * apart
    for k, rows in ((most - most % 8, -128), (most - most % 8 + 8, 128), (1 << 23, 128)):
        assert tile(7900, 2056, k, **{which: apart, other: 8}) == rows


def test_overlapping_rows_of_transposed_weights_behind_the_reach_of_a_load_go_through_registers():
    k, apart = 4104, 246264
    most = (1 << 30) - (k - 1) * apart
    assert tile(1, most - most % 8, k, w=apart, transposed=True) == 64
    assert tile(1, most - most % 8 + 8, k, w=apart, transposed=True) == 32
