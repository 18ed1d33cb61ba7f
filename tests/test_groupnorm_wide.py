"""Norms of wide rows: kernels with many threads to a CTA, one group or a few of more than 4096 bytes a row, against the formulas in 64 bits."""

import numpy as np
import pytest
import torch

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


def ids(s):
    return "T{}_C{}_g{}_B{}_S{}".format(*s)


# about the borders of the rules, 256 and 512 columns backward, 256 and 1024 forward: in 16 bits (8 elements a column), then in float (4)
WIDE16 = [(8, 256, 1, 5, 1), (8, 257, 1, 5, 1), (8, 320, 1, 2, 49), (8, 512, 1, 300, 1), (8, 513, 1, 3, 2), (8, 1024, 1, 3, 1), (8, 1025, 1, 3, 1),
          (16, 129, 1, 4, 1), (16, 256, 1, 2, 49), (16, 192, 1, 3, 7), (4, 514, 1, 5, 1), (4, 768, 1, 3, 64), (4, 1024, 1, 70, 1), (4, 1026, 1, 2, 3),
          (4, 514, 2, 3, 1), (4, 514, 2, 2, 40), (4, 516, 2, 2, 9), (12, 172, 1, 3, 3), (12, 174, 2, 2, 11), (12, 340, 1, 3, 1), (2, 1032, 1, 3, 5),
          (2, 1028, 4, 3, 2), (1, 2056, 1, 3, 5), (3, 688, 1, 3, 5), (6, 684, 2, 2, 3), (32, 65, 1, 3, 2), (64, 64, 1, 2, 9), (5, 824, 1, 2, 20)]
WIDE32 = [(8, 128, 1, 5, 1), (8, 129, 1, 5, 1), (8, 192, 1, 2, 49), (8, 256, 1, 300, 1), (8, 257, 1, 3, 2), (8, 512, 1, 3, 1), (8, 513, 1, 3, 1),
          (16, 65, 1, 4, 1), (16, 128, 1, 2, 49), (4, 257, 1, 5, 1), (4, 384, 1, 2, 49), (4, 512, 1, 70, 1), (12, 86, 1, 3, 3), (12, 170, 1, 3, 1),
          (2, 516, 1, 3, 5), (2, 514, 2, 3, 2), (1, 1028, 1, 3, 5), (3, 344, 1, 3, 5), (6, 342, 2, 2, 3), (32, 33, 1, 3, 2), (64, 32, 1, 2, 9)]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("dtype,shape", [(d, s) for d in ("fp16", "bf16") for s in WIDE16] + [("fp32", s) for s in WIDE32],
                         ids=lambda v: v if isinstance(v, str) else ids(v))
def test_wide_rows_against_the_formulas(shape, dtype, act):
    Norm(*shape, dtype, act, seed=sum(shape)).step()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,shape", [("fp16", (8, 512, 1, 9, 9)), ("bf16", (4, 768, 1, 7, 30)), ("fp16", (4, 514, 2, 6, 12)), ("fp32", (8, 192, 1, 8, 21)),
                                         ("fp32", (12, 86, 1, 7, 10))], ids=lambda v: v if isinstance(v, str) else ids(v))
def test_wide_rows_in_padded_batches_give_the_same_bits_again(shape, dtype):
    B, S = shape[3:]
    lengths = np.random.default_rng(3).integers(0, S + 1, B)
    lengths[:4] = (0, S, 1, 2)
    n = Norm(*shape, dtype, "silu", lengths=lengths, seed=4)
    n.step()
    first = n.outputs()
    n.x.masked_fill_(n.pad, float("nan"))
    n.dy.masked_fill_(n.pad, float("inf"))
    for _ in range(3):
        for k in ("stats", "dgamma", "dbeta"):
            getattr(n, k).fill_(float("nan"))
        n.fwd()
        n.bwd()
        again = n.outputs()
        assert all(torch.equal(first[k], again[k]) for k in first)
    n.guard.check()


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [False, True])
@pytest.mark.parametrize("shape", [(8, 80, 1, 5, 1), (8, 192, 1, 3, 1), (8, 256, 1, 3, 1), (8, 96, 1, 9, 40), (4, 8, 1, 9, 300), (1, 640, 1, 9, 8), (8, 160, 1, 6, 3),
                                   (4, 514, 2, 5, 2)], ids=ids)
def test_values_far_from_zero_where_warps_have_no_rows(shape, lengths):
    """One group a block whose columns leave warps idle, and instances shorter than a CTA has rows: the spread is a thousandth of the mean."""
    T, C, groups, B, S = shape
    rng = np.random.default_rng(5)
    n = Norm(*shape, "fp32", "none", seed=6, x=1000.0 + rng.standard_normal((B, S, C, T)),
             lengths=[(1, 2, 3, S, 0)[i % 5] for i in range(B)] if lengths else None)
    n.step()
