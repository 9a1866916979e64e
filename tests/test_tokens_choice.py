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


def test_tiles_without_a_form_through_registers_are_not_taken_for_one():
    """Sizes at which whole vectors take those tiles (192, -128, -64), and around them; x is not aligned to a vector."""
    def through_registers(tokens, out, k, transposed):
        p = product(tokens, out, k, transposed=transposed)
        p.x.data += 2
        return apm.lib().apm_test_grouped_product_tile(C.byref(p))

    seen = set()
    for transposed in (False, True):
        for tokens in (1, 40, 255, 1300, 5100, 6100, 7900, 1 << 17):
            for out in (8, 136, 520, 1032, 2056, 8192):
                for k in (8, 328, 1096, 4168, 65536):
                    seen.add(tile(tokens, out, k, transposed=transposed))
                    assert through_registers(tokens, out, k, transposed) in (256, 128, 64, 32)
    assert {192, -128, -64} <= seen


def test_products_of_more_tiles_than_a_grid_holds_are_refused():
    """Rows that strides allow (2^56 elements), and too many of them for one launch; x is one row for all tokens."""
    for tokens, out in ((1 << 30, 1 << 20), (1 << 36, 1 << 10), (1 << 28, 1 << 28)):
        p = product(tokens, out, 64, x=0)
        assert tile(tokens, out, 64, x=0) == 0
        assert apm.lib().apm_grouped_product(C.byref(p), None, 0, None) == apm.APM_EINVAL
        assert "y is too large for one product" in apm.apm_last_error()


@pytest.mark.parametrize("tokens,out,k", [(1 << 29, 8, 8), (1 << 30, 32, 32), ((1 << 31) - 512, 136, 64), ((1 << 31) - 512, 8, 1), ((1 << 24) - 512, 1 << 15, 8)])
def test_products_that_a_grid_holds_with_another_tile_are_not_refused(tokens, out, k):
    for transposed in (False, True):
        assert tile(tokens, out, k, x=0, transposed=transposed) > 0
