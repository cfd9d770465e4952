"""Routing of bf16 logits where more than k are equal and others, smaller, have the same 64-bit score at a lower index: sigmoid
near 1, logits near 0, softmax far below the largest.  Ids are compared as they are, weights by one fp32 rounding, as in
test_gpu_experts.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_experts import check_route, ctx, rk  # noqa: F401  (the fixtures)

pytestmark = pytest.mark.gpu

ROWS = {
    ("sigmoid", 38.0): 40.0,        # both score 1
    ("sigmoid", 0.0): 2.0 ** -60,   # both score 1/2
    ("sigmoid", -2.0 ** -70): 0.0,
    ("softmax", 0.0): 2.0 ** -60,
    ("softmax", -9000.0): -8000.0,  # both score 0 next to a logit of 1
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("score, low", sorted(ROWS))
def test_smaller_logits_of_the_same_score_come_by_index(ctx, score, low, dtype):  # noqa: F811
    high = ROWS[score, low]
    for e, k in ((8, 2), (64, 6), (256, 8), (1024, 16)):
        x = np.full((4, e), high)
        x[0, 0] = low                                    # one, in front of all
        x[1, : e // 2] = low                             # the first half
        x[2, 1::2] = low                                 # every other one
        x[3, e // 2] = low                               # too late to be chosen
        if low == -9000.0:
            x[:, e - 1] = 1.0
        for groups, top in ((1, 1), (4, 2)):
            ids, _ = check_route(ctx, x, k, None, dtype, score=score, n_groups=groups, top_groups=top)
            if groups == 1:
                first = [e - 1] if low == -9000.0 else []
                assert (ids.cpu() == torch.tensor((first + list(range(k)))[:k])).all()


def test_equal_rows_keep_the_lowest_indices(ctx):  # noqa: F811
    for value in (0.0, -0.0, -1e-30, 1.0, 20.0, -50.0, 2.0 ** -20, -(2.0 ** -21)):
        for score in ("softmax", "sigmoid"):
            ids, _ = check_route(ctx, np.full((5, 160), value), 6, None, torch.bfloat16, score=score, n_groups=8, top_groups=3, renorm=True)
            assert (ids.cpu() == torch.arange(6)).all()


def test_zeros_of_both_signs_and_tiny_neighbours(ctx):  # noqa: F811
    """+0 and -0 are one number; a row of zeros with one of 2^-133 (bf16's smallest) or -2^-133 among them is one of equal scores."""
    x = np.zeros((6, 64))
    x[0, :5] = -0.0
    x[1, ::2] = -0.0
    x[2, 40] = 2.0 ** -133
    x[3, 3] = -(2.0 ** -133)
    x[4, :32] = -(2.0 ** -133)
    x[5, :32], x[5, 32:] = 2.0 ** -19, 2.0 ** -19 + 2.0 ** -26           # neighbours whose scores differ
    for dtype in (torch.bfloat16, torch.float32):
        for score in ("softmax", "sigmoid"):
            for groups, top in ((1, 1), (8, 3)):
                check_route(ctx, x, 6, None, dtype, score=score, n_groups=groups, top_groups=top)
