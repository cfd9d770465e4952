"""Device-side waits of the 8-bit products that nothing satisfies: they expire after the configured limit, every role gives up and
returns, the call is reported as timed out, and the context works on.  The weights' copies are announced and not issued; no
memory access depends on them."""
import numpy as np
import pytest
import torch

from oracle import experts as X
from tests.test_gpu_matmul8 import bf, close, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


@pytest.fixture()
def ctx(rk):
    return rk.Context(16, 2, 256, 1024, [0, 8], 0.07)


def starve(rk, ctx, call):
    ctx.rk_set_wait_limit_ms(20)
    ctx.rk_test_starve_loads(1)
    call()
    with pytest.raises(rk.RKError) as ei:
        ctx.rk_poll_status()
    assert ei.value.status == 9 and "wait expired" in str(ei.value)
    ctx.rk_poll_status()                                          # the status word was cleared
    ctx.rk_test_starve_loads(0)
    ctx.rk_set_wait_limit_ms(2000)


# one pair per tile, several tiles per pair, k shared by two and four pairs of a cluster
@pytest.mark.parametrize("n, n_out, k", [(9, 300, 500), (3000, 2500, 300), (256, 1000, 2100), (3, 256, 8200)])
def test_dense_products_give_up_and_the_context_works_on(rk, ctx, n, n_out, k):
    rng = np.random.default_rng(n)
    w, wc, ws = weights(ctx, rng, 1, n_out, k)
    x = bf(rng.standard_normal((n, k)))
    q = ctx.rk_quant8(x)
    starve(rk, ctx, lambda: ctx.rk_matmul8(w, q))
    xc, xs = X.quant8(x.double().cpu().numpy())
    close(ctx.rk_matmul8(w, q, out_dtype=torch.float32), X.matmul8(wc[0], ws[0], xc, xs), torch.float32)
    ctx.rk_poll_status()


@pytest.mark.parametrize("n, n_e", [(7, 40), (3000, 5)])
def test_expert_products_give_up_and_the_context_works_on(rk, ctx, n, n_e):
    rng = np.random.default_rng(n)
    n_out, k = 300, 700
    w, wc, ws = weights(ctx, rng, n_e, n_out, k)
    ids = rng.integers(0, n_e, size=(n, 2))
    off, rows = ctx.rk_moe_group(torch.from_numpy(ids.astype(np.int32)).cuda(), n_e)
    x = bf(rng.standard_normal((n, k)))
    q = ctx.rk_quant8(x)
    starve(rk, ctx, lambda: ctx.rk_matmul8_experts(w, q, off, rows, 2))
    y = ctx.rk_matmul8_experts(w, q, off, rows, 2, out_dtype=torch.float32)
    ctx.rk_poll_status()
    xc, xs = X.quant8(x.double().cpu().numpy())
    want = np.zeros((2 * n, n_out))
    for p, e in enumerate(ids.reshape(-1)):
        want[p] = X.matmul8(wc[e], ws[e], xc[p // 2:p // 2 + 1], xs[p // 2:p // 2 + 1])[0]
    close(y, want, torch.float32)
