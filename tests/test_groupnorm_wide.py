"""Norms of wide rows: kernels with many threads to a CTA, one group or a few of more than 4096 bytes a row, against the formulas in 64 bits."""

import pytest

from tests.test_groupnorm import Norm


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("shape", [(4, 514, 2, 3, 1), (4, 514, 2, 2, 40), (12, 174, 2, 4, 3), (20, 206, 2, 2, 7), (4, 1026, 2, 2, 5), (2, 1028, 4, 3, 2),
                                   (6, 348, 4, 2, 9)], ids=lambda s: "T{}_C{}_g{}_B{}_S{}".format(*s))
def test_groups_that_end_inside_a_vector_of_a_wide_row(shape, dtype):
    """An odd number of channels a group, tuples of half a vector (of 16-bit types): what a thread keeps of its vector is of two groups."""
    n = Norm(*shape, dtype, "gelu", seed=sum(shape))
    n.fwd()
    n.check(("y", "stats"))
