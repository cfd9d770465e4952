"""Device-side waits of the decode kernels that nothing satisfies: they expire after the configured limit, every role of the
kernel gives up and returns, the call is reported as timed out, and the context works on.  Nothing here faults the GPU: the
signal that a role waits for is withheld, and no memory access depends on it."""
import numpy as np
import pytest
import torch

from tests.test_gpu_decode import Pool, bf, check_attention, check_matvec, fill_pool, i32, make_ctx, plan_for
from oracle import decode as D
from oracle.harness import f64

pytestmark = pytest.mark.gpu

LOADS, QUERIES, QUERY_ROPE, KEYS, KEYS_FREE, SCORES, WEIGHTS, VALUES = range(1, 9)


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


def timed_out(rk, ctx):
    with pytest.raises(rk.RKError) as ei:
        ctx.rk_poll_status()
    assert ei.value.status == 9 and "wait expired" in str(ei.value)
    ctx.rk_poll_status()                                          # the status word was cleared


# heads x tokens: row tiles of 16, 32 and 64.  900 tiles: several per thread block, in one request (one group per block) and in 90
# (blocks that go from one request to the next).
@pytest.mark.parametrize("heads", [16, 32, 72])
@pytest.mark.parametrize("requests, tiles", [(1, 900), (90, 10)])
@pytest.mark.parametrize("withheld", [LOADS, QUERIES, QUERY_ROPE, KEYS, KEYS_FREE, SCORES, WEIGHTS, VALUES])
def test_attention_gives_up_and_the_context_works_on(rk, heads, requests, tiles, withheld):
    ctx = make_ctx(rk, heads)
    n = 128 * tiles - 5
    pool = Pool(rk, [n], seed=91)
    fill_pool(ctx, pool, 91)
    items, q_pos = [[(0, 0)]] * requests, np.full((requests, 1), n - 1)
    q = bf(np.random.default_rng(92).standard_normal((requests, 1, heads, 576)))
    plan = plan_for(ctx, pool, items, q_pos)
    O, lse = ctx.rk_cache4_attn(pool.pages, plan, q)
    ctx.rk_poll_status()
    ctx.rk_set_wait_limit_ms(20)
    ctx.rk_test_starve_loads(withheld)
    ctx.rk_cache4_attn(pool.pages, plan, q)
    timed_out(rk, ctx)
    ctx.rk_test_starve_loads(0)
    ctx.rk_set_wait_limit_ms(2000)
    again, lse_again = ctx.rk_cache4_attn(pool.pages, plan, q)
    ctx.rk_poll_status()
    assert torch.equal(O, again) and torch.equal(lse, lse_again)
    check_attention(ctx, pool, items[:1], q_pos[:1], q[:1], O[:1], lse[:1], heads)


# one thread block per run of rows, clusters of two to eight, and several rounds along k
@pytest.mark.parametrize("mats, n_out, k, group, tok", [(2, 256, 1024, 32, 1), (1, 512, 4096, 128, 9), (1, 512, 16384, 64, 3),
                                                        (1, 48, 33088, 64, 17)])
def test_products_give_up_and_the_context_works_on(rk, mats, n_out, k, group, tok):
    ctx = make_ctx(rk)
    rng = np.random.default_rng(93)
    w = bf(rng.standard_normal((mats, n_out, k)) * 0.02)
    x = bf(rng.standard_normal((tok, mats, k)))
    w4 = ctx.rk_quant4(w, group)
    ctx.rk_set_wait_limit_ms(20)
    ctx.rk_test_starve_loads(LOADS)
    ctx.rk_matvec4(w4, x)
    timed_out(rk, ctx)
    ctx.rk_test_starve_loads(0)
    ctx.rk_set_wait_limit_ms(2000)
    check_matvec(ctx.rk_matvec4(w4, x, out_dtype=torch.float32), f64(x), D.quantise_weights(f64(w), group), k, False)
    ctx.rk_poll_status()


@pytest.mark.parametrize("heads", [16, 32, 64])
@pytest.mark.parametrize("tiles", [1, 5])
def test_wait_that_runs_out_after_the_issuing_warp_has_left_is_reported(rk, heads, tiles):
    """One key tile per thread block: when the epilogue waits for the end of the value products, the warp that issued them has
    nothing left to do."""
    ctx = make_ctx(rk, heads)
    n = 128 * tiles
    pool = Pool(rk, [n], seed=94)
    fill_pool(ctx, pool, 94)
    plan = plan_for(ctx, pool, [[(0, 0)]], np.array([[n - 1]]))
    q = bf(np.random.default_rng(95).standard_normal((1, 1, heads, 576)))
    ctx.rk_set_wait_limit_ms(20)
    ctx.rk_test_starve_loads(VALUES)
    ctx.rk_cache4_attn(pool.pages, plan, q)
    timed_out(rk, ctx)
    ctx.rk_test_starve_loads(0)
    ctx.rk_set_wait_limit_ms(2000)
    O, lse = ctx.rk_cache4_attn(pool.pages, plan, q)
    ctx.rk_poll_status()
    check_attention(ctx, pool, [[(0, 0)]], np.array([[n - 1]]), q, O, lse, heads)
