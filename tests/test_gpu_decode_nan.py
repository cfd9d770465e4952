"""Cached rows that hold a NaN, wherever they stand among the keys that a query row sees: its output and its log-sum-exp
are NaN, and rows that do not see them are what they are without them."""
import numpy as np
import pytest
import torch

from tests.test_gpu_decode import SCALE, Pool, bf, check_attention, i32, make_ctx, plan_for

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


def rows_with_nan(case, rng):
    """(lengths of the segments, latents) of a request whose first segment holds the NaN rows."""
    if case == "one-row segment first":
        lens, bad = [1, 500], [0]
    elif case == "first tile all NaN":
        lens, bad = [128, 500], range(128)
    elif case == "whole segment NaN":
        lens, bad = [300, 500], range(300)
    else:  # "scores jump behind it": the second segment's lie more than 2^90 above the first's
        lens, bad = [128, 500], [5]
    c = rng.standard_normal((sum(lens), 512)) * 0.1
    c[:, 0] = 0.0
    if case == "scores jump behind it":
        c[lens[0]:, 0] = 7.0                                      # times q[0]: see below
    c[list(bad), 300] = np.nan
    return lens, c


# 160 requests: more tiles than thread blocks, so that a block meets the NaN rows and the clean ones in one run; 2 requests: one
# tile per block, joined afterwards
@pytest.mark.parametrize("requests", [160, 2])
@pytest.mark.parametrize("case", ["one-row segment first", "first tile all NaN", "whole segment NaN", "scores jump behind it"])
@pytest.mark.parametrize("heads", [16, 24, 64])
def test_nan_rows_before_clean_ones(rk, heads, case, requests):
    ctx = make_ctx(rk, heads)
    rng = np.random.default_rng(81)
    lens, c = rows_with_nan(case, rng)
    n = sum(lens)
    pool = Pool(rk, lens, seed=82)
    ctx.rk_cache4_append(pool.pages, pool.table, bf(c), bf(rng.standard_normal((n, 64))), i32([0, lens[0], n]))
    ctx.rk_poll_status()
    pool.from_device()
    # even requests see both segments, odd ones the second alone at the same offset
    both = [(0, 0), (1, lens[0])]
    items = [both if b % 2 == 0 else both[1:] for b in range(requests)]
    q_pos = np.full((requests, 1), n - 1)
    q = rng.standard_normal((requests, 1, heads, 576)) * 0.5
    q[..., 0] = 90.0 * np.log(2.0) / (7.0 * SCALE) * 1.25         # the jump: 112 in base-2 units
    q = bf(q)
    O, lse = ctx.rk_cache4_attn(pool.pages, plan_for(ctx, pool, items, q_pos), q)
    ctx.rk_poll_status()
    assert torch.isnan(O[0::2]).all()
    assert torch.isnan(lse[0::2]).all()
    clean = [1, requests - 1]
    check_attention(ctx, pool, [items[b] for b in clean], q_pos[clean], q[clean], O[clean], lse[clean], heads)
