"""8-bit rows and their products against the float64 oracle.

Codes and scales are compared as they are.  Products: the integer sums are exact; converting one to fp32, and each of the two
products with a scale, rounds once (2^-24 each): |dy| <= 3.01 * 2^-24 |y| (u32), and one bf16 rounding more, 2^-8 |y| (u16)."""
import numpy as np
import pytest
import torch

from oracle import experts as X

pytestmark = pytest.mark.gpu

U32, U16 = 3.01 * 2.0 ** -24, 2.0 ** -8 * 1.0001


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ctx(rk):
    return rk.Context(16, 2, 256, 1024, [0, 8], 0.07)


def bf(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def special(rng, n, k):
    """Rows with the values quantisation can go wrong at: ties, zeros, tiny, huge, non-finite."""
    x = rng.standard_normal((n, k))
    for i in range(n):
        c = i % 10
        if c == 1:
            x[i] = 0.0
        elif c == 2:
            x[i] = rng.integers(-254, 255, size=k) * 0.5 * 2.0 ** rng.integers(-20, 20)    # halves of a power-of-two scale
            x[i, -1] = 127.0 * 2.0 ** rng.integers(-20, 20)
        elif c == 3:
            x[i] *= 10.0 ** rng.integers(-12, 6, size=k)
        elif c == 4:
            x[i] *= 1e-37                                                                 # scales below fp32's normal numbers
        elif c == 5:
            x[i] = rng.integers(-5, 6, size=k) * 9.2e-41                                  # bf16's smallest numbers
        elif c == 6:
            x[i, rng.integers(0, k)] = rng.choice([np.inf, -np.inf, np.nan])
        elif c == 7:
            x[i] *= 1e37
        elif c == 8:
            x[i, 1:] = 0.0
        elif c == 9:
            x[i] = 1.0 + rng.integers(0, 128, size=k) / 128.0
    return x


def check_rows(q8, x):
    codes, scales = X.quant8(x.double().cpu().numpy())
    got = q8.codes.reshape(len(x), -1).cpu().numpy().astype(np.int64)
    assert np.array_equal(got[:, :x.shape[1]], codes)
    assert (got[:, x.shape[1]:] == 0).all()
    assert np.array_equal(q8.scales.reshape(-1).double().cpu().numpy(), scales, equal_nan=True)
    return codes, scales


@pytest.mark.parametrize("n, k, stride, offset", [(1, 1, 1, 0), (10, 7, 7, 0), (10, 16, 16, 0), (20, 100, 104, 0), (13, 129, 131, 1), (20, 1024, 1024, 0),
                                                  (11, 4096, 4104, 8), (10, 4095, 4097, 3), (10, 16384, 16384, 0), (4, 20000, 20000, 0), (3, 131072, 131072, 0)])
def test_quant8_matches_oracle(ctx, n, k, stride, offset):
    rng = np.random.default_rng(n + k)
    raw = torch.full((offset + n * stride + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
    x = raw[offset:offset + n * stride].view(n, stride)[:, :k]
    x.copy_(bf(special(rng, n, k)))
    q = ctx.rk_quant8(x)
    ctx.rk_poll_status()
    check_rows(q, x)


def test_quant8_every_code_border(ctx):
    """One row per scale: x walks through all bf16 numbers near every border between two codes."""
    rng = np.random.default_rng(3)
    rows = []
    for top in list(rng.uniform(0.5, 2.0, size=40)) + [1.0, 1.9921875, 127.0, 254.0]:
        top = float(torch.tensor(top).to(torch.bfloat16))
        b = (np.arange(127) + 0.5) * top / 127.0
        near = bf(b).float().cpu().numpy()
        bits = near.view(np.uint32)
        rows.append(np.concatenate([near, (bits + 0x10000).view(np.float32), (bits - 0x10000).view(np.float32), -near, [top]]))
    x = bf(np.minimum(np.stack(rows), np.stack(rows)[:, -1:]))
    check_rows(ctx.rk_quant8(x), x)


def weights(ctx, rng, mats, n_out, k):
    w = bf(rng.standard_normal((mats, n_out, k)) * 0.02)
    q = ctx.rk_quant8(w)
    codes, scales = X.quant8(w.double().cpu().numpy().reshape(mats * n_out, k))
    return q, codes.reshape(mats, n_out, k), scales.reshape(mats, n_out)


def close(got, want, dtype):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    tol = U32 + (U16 if dtype == torch.bfloat16 else 0.0)
    err = np.abs(got - want)
    assert (err[~np.isnan(want)] <= tol * np.abs(want[~np.isnan(want)]) + 1e-38).all(), np.nanmax(err / np.maximum(np.abs(want), 1e-30))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n, n_out, k", [
    (1, 1, 1), (1, 16, 16), (2, 100, 33), (5, 256, 128), (16, 255, 127), (17, 257, 129), (31, 300, 1000), (33, 128, 512), (64, 512, 2048), (65, 384, 640),
    (128, 1000, 256), (200, 130, 4096), (255, 256, 777), (257, 511, 1024), (333, 1001, 777), (1, 4096, 8192), (7, 2050, 16384), (1500, 700, 300), (2500, 1300, 100),
])
def test_matmul8_matches_oracle(ctx, n, n_out, k, dtype):
    rng = np.random.default_rng(n + n_out + k)
    w, wc, ws = weights(ctx, rng, 1, n_out, k)
    x = bf(rng.standard_normal((n, k)) * (1.0 + 15.0 * (rng.random(k) < 0.02)))
    q = ctx.rk_quant8(x)
    xc, xs = X.quant8(x.double().cpu().numpy())
    y = ctx.rk_matmul8(w, q, out_dtype=dtype)
    ctx.rk_poll_status()
    close(y, X.matmul8(wc[0], ws[0], xc, xs), dtype)
    assert torch.equal(y, ctx.rk_matmul8(w, q, out_dtype=dtype))                       # and again the same bits


@pytest.mark.parametrize("n, n_out, k", [(3, 40, 131072), (300, 300, 131072)])
def test_matmul8_largest_sums(rk, ctx, n, n_out, k):
    """All codes +-127 at the longest k: the sums reach 127^2 * 131072 = 2114060288, just below 2^31."""
    w = torch.full((1, n_out, k), 127, dtype=torch.int8, device="cuda")
    x = torch.full((n, k), 127, dtype=torch.int8, device="cuda")
    x[1] = -127
    x[2, ::2] = -127
    q = rk.Q8(x, torch.full((n,), 2.0 ** -10, device="cuda"), k)
    y = ctx.rk_matmul8(rk.Q8(w, torch.ones((1, n_out), device="cuda"), k), q, out_dtype=torch.float32)
    ctx.rk_poll_status()
    want = np.zeros((n, n_out)) + 127.0 ** 2 * k * 2.0 ** -10
    want[1] *= -1
    want[2] = 0.0
    close(y, want, torch.float32)


def test_matmul8_strided_output_and_marked_rows(ctx):
    """Rows of y inside a wider tensor, at an odd offset; a token and a channel that are not numbers; a token of zeros."""
    rng = np.random.default_rng(11)
    n, n_out, k = 70, 190, 260
    wv = rng.standard_normal((1, n_out, k))
    wv[0, 5, 3] = np.inf
    w = ctx.rk_quant8(bf(wv))
    xv = rng.standard_normal((n, k))
    xv[4, 7] = np.nan
    xv[6] = 0.0
    q = ctx.rk_quant8(bf(xv))
    wc, ws = X.quant8(bf(wv).double().cpu().numpy()[0])
    xc, xs = X.quant8(bf(xv).double().cpu().numpy())
    want = X.matmul8(wc, ws, xc, xs)
    for dtype in (torch.bfloat16, torch.float32):
        for pad in (1, 3, 8):
            wide = torch.full((n, n_out + pad), 7.0, dtype=dtype, device="cuda")
            ctx.rk_matmul8(w, q, y=wide[:, 1:1 + n_out])
            ctx.rk_poll_status()
            close(wide[:, 1:1 + n_out], want, dtype)
            assert (wide[:, 0] == 7.0).all() and (wide[:, 1 + n_out:] == 7.0).all()


# ------------------------------------------------------------------------------------------------------------
# by expert
# ------------------------------------------------------------------------------------------------------------
def expert_case(rng, n, k_slots, n_e, skew, drop):
    pop = rng.standard_normal(n_e) * skew
    ids = np.argsort(-(rng.gumbel(size=(n, n_e)) + pop), axis=1)[:, :k_slots]
    ids[rng.random(ids.shape) < drop] = -1
    return ids


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n, slots, n_e, n_out, k, skew, drop", [
    (1, 1, 1, 16, 16, 0.0, 0.0), (1, 6, 64, 256, 128, 0.5, 0.0), (3, 2, 5, 100, 77, 1.0, 0.3), (64, 6, 128, 256, 512, 0.5, 0.2), (500, 4, 8, 300, 300, 2.0, 0.1),
    (700, 8, 40, 257, 129, 1.0, 0.5), (1100, 1, 3, 520, 256, 0.3, 0.0), (40, 16, 1024, 64, 64, 0.2, 0.1), (2000, 2, 2, 130, 200, 0.0, 0.0), (9, 6, 700, 24, 1000, 0.1, 0.9),
])
def test_experts_match_oracle(ctx, n, slots, n_e, n_out, k, skew, drop, dtype):
    rng = np.random.default_rng(n + slots + n_e)
    ids = expert_case(rng, n, slots, n_e, skew, drop)
    row_off, rows = ctx.rk_moe_group(torch.from_numpy(ids.astype(np.int32)).cuda(), n_e)
    w, wc, ws = weights(ctx, rng, n_e, n_out, k)
    for per in {slots, 1}:
        x = bf(rng.standard_normal((n * slots // per, k)))
        q = ctx.rk_quant8(x)
        xc, xs = X.quant8(x.double().cpu().numpy())
        y = torch.full((n * slots, n_out), 5.0, dtype=dtype, device="cuda")
        ctx.rk_matmul8_experts(w, q, row_off, rows, per, y=y)
        ctx.rk_poll_status()
        want = np.full((n * slots, n_out), 5.0)                    # rows of dropped pairs are left alone
        for p, e in enumerate(ids.reshape(-1)):
            if e >= 0:
                want[p] = X.matmul8(wc[e], ws[e], xc[p // per:p // per + 1], xs[p // per:p // per + 1])[0]
        close(y, want, dtype)


def test_experts_bad_tables_are_reported_and_skipped(rk, ctx):
    """Bounds that leave the list or fall, and pairs outside the pool: the rest is computed, the status says so."""
    rng = np.random.default_rng(5)
    n_e, n, n_out, k = 4, 12, 40, 64
    w, wc, ws = weights(ctx, rng, n_e, n_out, k)
    x = bf(rng.standard_normal((n, k)))
    q = ctx.rk_quant8(x)
    xc, xs = X.quant8(x.double().cpu().numpy())
    good = list(range(n))

    def run(off, rows):
        y = torch.full((n, n_out), 5.0, device="cuda")
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        ctx.rk_matmul8_experts(w, q, i32(off), i32(rows), 1, y=y)
        with pytest.raises(rk.RKError) as ei:
            ctx.rk_poll_status()
        assert ei.value.status == 4
        want = np.full((n, n_out), 5.0)
        for e in range(n_e):
            if 0 <= off[e] <= off[e + 1] <= n:
                for p in rows[off[e]:off[e + 1]]:
                    if 0 <= p < n:
                        mine = X.matmul8(wc[e], ws[e], xc[p:p + 1], xs[p:p + 1])[0]
                        # listed twice (bounds that fall): the product of either expert, element by element
                        got = y[p].double().cpu().numpy()
                        first = (want[p] != 5.0) & (np.abs(got - want[p]) < np.abs(got - mine))
                        want[p] = np.where(first, want[p], mine)
        close(y, want, torch.float32)

    run([0, 3, 6, 9, 13], good)
    run([0, 3, 2, 9, 12], good)
    run([-1, 3, 6, 9, 12], good)
    run([0, 3, 6, 9, 1 << 30], good)
    run([0, 3, 6, 9, 12], [0, 1, 2, 3, -5, 5, 6, 12, 8, 9, 1 << 30, 11])
    run([0, 3, 6, 9, 12], [-1] * 12)


def test_products_without_rows(rk, ctx):
    w = ctx.rk_quant8(torch.zeros((1, 32, 64), dtype=torch.bfloat16, device="cuda"))
    q = ctx.rk_quant8(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"))
    assert ctx.rk_matmul8(w, q).shape == (0, 32)
    off = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert ctx.rk_matmul8_experts(w, q, off, torch.empty(0, dtype=torch.int32, device="cuda"), 1).shape == (0, 32)


def test_product_refusals(rk, ctx):
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    w, x = ctx.rk_quant8(z(2, 32, 64)), ctx.rk_quant8(z(5, 64))
    w1 = ctx.rk_quant8(z(1, 32, 64))
    off, rows = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(10, dtype=torch.int32, device="cuda")
    for call, status in ((lambda: ctx.rk_matmul8(w, x), 3),                                      # two matrices, no lists
                         (lambda: ctx.rk_matmul8(w1, ctx.rk_quant8(z(5, 63))), 3),               # k differs
                         (lambda: ctx.rk_matmul8(w1, ctx.rk_quant8(z(2, 5, 64))), 3),            # tokens in two matrices
                         (lambda: ctx.rk_matmul8_experts(w, x, off, rows, 1), 3),                # ten pairs, five rows
                         (lambda: ctx.rk_matmul8_experts(w, x, off, rows, 0), 7),
                         (lambda: ctx.rk_matmul8_experts(w, x, off, rows, 17), 7),
                         (lambda: ctx.rk_quant8(z(1, 131073)), 7)):
        with pytest.raises(rk.RKError) as ei:
            call()
        assert ei.value.status == status
    with pytest.raises(TypeError):
        ctx.rk_matmul8(w1, x, out_dtype=torch.float16)
    with pytest.raises(TypeError):
        ctx.rk_quant8(z(5, 64).float())
    with pytest.raises(ValueError):
        ctx.rk_matmul8(w1, x, y=z(4, 32))
    with pytest.raises(ValueError):
        ctx.rk_matmul8(w1, x, y=z(5, 64)[:, ::2])
    with pytest.raises(ValueError):
        ctx.rk_matmul8_experts(w, x, off[:2], rows, 2)
    with pytest.raises(ValueError):
        rk.Q8(torch.zeros((4, 60), dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda"), 60)     # not padded to 64


def test_expert_layer_as_a_step_runs_it(ctx):
    """Route, fan-out, lists, first product, gate, second product, weighted sum; against the oracle's parts in 64 bits."""
    rng = np.random.default_rng(21)
    n, n_e, slots, d, inner = 50, 16, 6, 192, 80
    x = bf(rng.standard_normal((n, d)))
    logits = torch.from_numpy(rng.standard_normal((n, n_e)).astype(np.float32)).cuda()
    w1, c1, s1 = weights(ctx, rng, n_e, 2 * inner, d)
    w2, c2, s2 = weights(ctx, rng, n_e, d, inner)
    ids, wt = ctx.rk_moe_route(logits, slots, score="sigmoid", renorm=True)
    _, keep = ctx.rk_moe_fanout(wt, 0.7)
    off, rows = ctx.rk_moe_group(ids, n_e, keep)
    h = ctx.rk_matmul8_experts(w1, ctx.rk_quant8(x), off, rows, slots, y=torch.zeros((n * slots, 2 * inner), dtype=torch.bfloat16, device="cuda"))
    a = (torch.nn.functional.silu(h[:, :inner].float()) * h[:, inner:].float()).to(torch.bfloat16)
    y = ctx.rk_matmul8_experts(w2, ctx.rk_quant8(a), off, rows, 1, y=torch.zeros((n * slots, d), device="cuda"))
    ctx.rk_poll_status()
    got = (y.view(n, slots, d).double() * wt.double()[..., None]).sum(1).cpu().numpy()
    xc, xs = X.quant8(x.double().cpu().numpy())
    ac, as_ = X.quant8(a.double().cpu().numpy())
    hh = h.double().cpu().numpy()
    want, idh, kh, wh = np.zeros((n, d)), ids.cpu().numpy(), keep.cpu().numpy(), wt.double().cpu().numpy()
    for t in range(n):
        for s in range(slots):
            if (kh[t] >> s) & 1:
                e, p = idh[t, s], t * slots + s
                first = X.matmul8(c1[e], s1[e], xc[t:t + 1], xs[t:t + 1])[0]
                assert (np.abs(hh[p] - first) <= (U16 + U32) * np.abs(first)).all()
                want[t] += wh[t, s] * X.matmul8(c2[e], s2[e], ac[p:p + 1], as_[p:p + 1])[0]
    # every term is off by U32 of itself; the terms of a sum may cancel, so the bound is on the sum of their magnitudes
    assert np.abs(got - want).max() <= U32 * slots * np.abs(y.double().cpu().numpy()).max()
