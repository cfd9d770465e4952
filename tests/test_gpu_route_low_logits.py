"""Routing by sigmoid where the 64-bit scores of different logits are equal: exp(-x) is beyond double's range for logits below
-709.8, so that all of those score exactly 0 and their order is that of the indices.  Ids are compared as they are, weights by
one fp32 rounding, as in test_gpu_experts.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_experts import check_route, ctx, rk  # noqa: F401  (the fixtures)

pytestmark = pytest.mark.gpu


def test_a_few_logits_below_the_range(ctx):  # noqa: F811
    ids, w = check_route(ctx, [[-800.0, -750.0, -760.0, -790.0], [-800.0, -720.0, 2.0, 1.0]], 2, score="sigmoid")
    assert ids.tolist() == [[0, 1], [2, 3]] and (w[0] == 0).all()
    ids, _ = check_route(ctx, [[-800.0, -720.0, 2.0, 1.0]], 4, score="sigmoid", renorm=True)
    assert ids.tolist() == [[2, 3, 0, 1]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("e, groups, top, group_top, k", [
    (8, 1, 1, 1, 8), (64, 1, 1, 1, 6), (64, 8, 3, 1, 6), (64, 8, 3, 2, 6), (160, 8, 3, 1, 6), (256, 1, 1, 1, 16), (256, 8, 4, 1, 8), (1024, 32, 5, 1, 16),
])
def test_masks_of_large_finite_numbers(ctx, dtype, e, groups, top, group_top, k):  # noqa: F811
    rng = np.random.default_rng(e + 10 * groups + group_top)
    x = rng.standard_normal((12, e)) * 2
    order = np.argsort(rng.random((12, e)), axis=1)
    for t, left in enumerate((0, 1, 2, 3, 4, 5, 6, k, k + 1, e // 2, 1, 2)):        # experts that are not masked
        masked = order[t, left:]
        x[t, masked] = (-720.0, -1e4, -1e9, -3e38)[t % 4] * (0.9 + 0.1 * rng.random(len(masked)))
    x[10] = -705.0 - 10.0 * rng.random(e)                                          # on both sides of the border
    x[11] = -690.0 - 20.0 * rng.random(e)
    for bias in (None, np.zeros(e), rng.standard_normal(e) * 0.2):
        for renorm in (False, True):
            check_route(ctx, x, k, bias, dtype, score="sigmoid", n_groups=groups, top_groups=top, group_top=group_top, renorm=renorm)


def test_a_masked_group_is_ranked_by_its_index(ctx):  # noqa: F811
    """Two of four groups take part, three are masked by numbers that all score 0: the lowest of those three is the second."""
    x = np.full((1, 16), -800.0)
    x[0, 4:8] = [1.0, 2.0, 0.5, 0.0]
    x[0, 12:] = -720.0
    for group_top in (1, 2):
        ids, _ = check_route(ctx, x, 6, score="sigmoid", n_groups=4, top_groups=2, group_top=group_top)
        assert ids.tolist() == [[5, 4, 6, 7, 0, 1]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_group_ranks_of_equal_scores(ctx, score, dtype):  # noqa: F811
    """Groups of one expert: ranks that are equal, that differ where their scores do not (both ends, next to 0), and that differ."""
    pairs = {"sigmoid": [(40.0, 38.0), (-800.0, -1e4), (2.0 ** -60, 0.0), (0.0, -0.0), (1.0, 0.5), (-650.0, -655.0)],
             "softmax": [(-9000.0, -1e9), (2.0 ** -60, 0.0), (0.0, -0.0), (1.0, 0.5), (-500.0, -505.0)]}[score]
    for high, low in pairs:
        x = np.full((5, 16), high)
        x[0, 0] = low
        x[1, ::2] = low
        x[2, :12] = low
        x[3, 9] = low
        x[:4, 5] = 3.0 if abs(high) < 1e3 else 5.0
        for top in (1, 3, 6):
            check_route(ctx, x, top, None, dtype, score=score, n_groups=16, top_groups=top)
