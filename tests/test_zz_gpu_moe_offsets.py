"""The product's offsets that are not ascending from 0: negative ones, beyond the rows, and segments that end before
they begin. A whole sum to 32 bits and two products: 3 roundings, and one to the result's type."""
import numpy as np
import pytest

import paper_2608_00358_amd as H
from test_zz_gpu_moe import check_product

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def comm():
    with H.Comm(1, device=0) as c:
        yield c


@pytest.mark.parametrize("rows,inner,cols,experts", [(12, 200, 70, 4), (400, 130, 300, 6), (3000, 96, 1500, 12), (6000, 65, 2100, 8)])
def test_product_of_offsets_out_of_order(comm, rows, inner, cols, experts):
    """A segment that ends before it begins is empty; rows of the other segments, which do not overlap, are
    computed, and nothing else is written."""
    rng = np.random.default_rng(rows)
    third = rows // 3
    low = [-5 * rows] + [third] * (experts - 1) + [rows]                 # a negative first offset
    under = [-9, -7] + [-3] * (experts - 2) + [-1]                       # nothing but negative ones
    back = [third, 0] + [0] * (experts - 2) + [third]                    # back to 0, and rows up to a third at the end
    over = [2 * third] * (experts - 1) + [rows + 7, third]               # beyond the rows, then back
    far = [-(1 << 62)] + [0] * (experts - 1) + [1 << 62]                 # of any size
    for ends in (low, under, back, over, far):
        check_product(comm, rng, rows, inner, cols, experts, ends, "bf16")
        check_product(comm, rng, rows, inner, cols, experts, ends, "fp32", pad=3)
