"""Attention over the 4-bit cache with query positions at the ends of 32 bits: a padding token among drafted ones may
carry any negative position, and must neither see a key nor change what its neighbours see."""
import numpy as np
import pytest
import torch

from oracle import decode as D
from tests.test_gpu_decode import BASE, SCALE, Pool, bf, check_attention, fill_pool, i32, make_ctx, plan_for

pytestmark = pytest.mark.gpu

INT_MIN = -2 ** 31


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


# requests x tiles: at 160 x 2 most requests lie in one thread block, 30 x 10 and 1 x 600 are cut into runs of a few tiles
@pytest.mark.parametrize("requests, tiles", [(160, 2), (30, 10), (1, 600)])
@pytest.mark.parametrize("pad", [INT_MIN, INT_MIN + 1, -2 ** 30, -1])
def test_padding_tokens_at_the_lowest_positions(rk, requests, tiles, pad):
    """Tokens at n - 2 and n - 1 and a padding token.  The last key outweighs all others together, so a token that sees it
    without being allowed to is off by more than one in its log-sum-exp; all other keys score the same."""
    ctx = make_ctx(rk, 16)
    n = 128 * tiles
    pool = Pool(rk, [n], seed=71)
    c = np.zeros((n, 512))
    c[:, 1] = np.arange(n) % 5 - 2.0
    c[n - 1, 0] = 7.0
    fill_pool(ctx, pool, 71, c=c)
    want_gain = np.log(n) + 1.0                                   # logit of the last key over the others' zero
    q = np.zeros((requests, 3, 16, 576))
    q[..., 0] = want_gain / (7.0 * SCALE)
    q = bf(q)
    q_pos = np.tile(np.array([[n - 2, n - 1, pad]]), (requests, 1))
    items = [[(0, 0)] for _ in range(requests)]
    O, lse = ctx.rk_cache4_attn(pool.pages, plan_for(ctx, pool, items, q_pos), q)
    ctx.rk_poll_status()
    assert (O[:, 2] == 0).all() and torch.isneginf(lse[:, 2]).all()
    # n - 1 equal scores: log(n - 1), to fp32's rounding of the sum (at most tiles + 40 additions) and of the logarithm
    assert (lse[:, 0].double() - np.log(n - 1.0)).abs().max() <= (tiles + 48) * 2.0 ** -23 * np.log(n)
    first = [0, requests - 1]
    check_attention(ctx, pool, [items[b] for b in first], q_pos[first], q[first], O[first], lse[first], 16)


def test_padding_requests_at_the_lowest_position_beside_far_offsets(rk):
    """Whole padding requests, and a token at the largest position, with an item whose offset is close to 2^30."""
    ctx = make_ctx(rk, 16)
    n, far = 256, 2 ** 30 - 1000
    pool = Pool(rk, [n], seed=72)
    fill_pool(ctx, pool, 72)
    rng = np.random.default_rng(73)
    q = bf(rng.standard_normal((3, 2, 16, 576)))
    q_pos = np.array([[INT_MIN, INT_MIN], [INT_MIN, far + n - 1], [2 ** 31 - 1, INT_MIN]])
    items = [[(0, far)]] * 3
    O, lse = ctx.rk_cache4_attn(pool.pages, plan_for(ctx, pool, items, q_pos), q)
    ctx.rk_poll_status()
    check_attention(ctx, pool, items, q_pos, q, O, lse, 16)
