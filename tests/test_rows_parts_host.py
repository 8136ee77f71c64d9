"""The numbers that the GPU tests of fp32 products use, without a GPU."""
import numpy as np

import rows_parts as parts
from rows_ref import U


def test_a_lost_product_of_parts_is_beyond_the_bound():
    """What the GPU tests of fp32 products compare with: each of the six products of bf16 parts is more than the
    bounds allow to be missing, and the three that are left out are within."""
    x, y = parts.three_parts()
    for a, more in ((x, 4), (np.float32(1) / np.float32(3), 6)):
        (pa, ra), (pb, rb) = parts.parts_of(a), parts.parts_of(y)
        assert ra == 0 and rb == 0 and pb[1] > 0 and pb[2] > 0
        exact, bound = float(a) * float(y), (parts.PARTS + more) * U * float(a) * float(y)
        taken = [(i, j) for i in range(3) for j in range(3) if i + j <= 2]
        total = sum(pa[i] * pb[j] for i, j in taken)
        assert abs(total - exact) <= 2 * U * exact
        for i, j in taken:
            assert abs(total - pa[i] * pb[j] - exact) > 2 * bound, (i, j)
