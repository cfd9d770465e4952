"""Sampling against the float64 oracle.  Tokens are compared as they are; the random numbers of the tests lie between two
borders of the oracle's cumulated weights with a distance of at least 1e-9 of the sum (the kernel's weights are off by at most
2^-43 and 1.4e-13 of themselves each, and the sum is at least 1; the tests' 200003 of them would reach 2.3e-8 only if they
all erred to one side, and reach 5e-11 as roundings do), so that the token does not hang on a rounding.  Probabilities: one
fp32 rounding (2^-24) of a value whose own error is below 1e-9."""
import numpy as np
import pytest
import torch

from oracle import experts as X

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ctx(rk):
    return rk.Context(16, 2, 256, 1024, [0, 8], 0.07)


def dev(x, dtype=torch.float32):
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(dtype).cuda()


def clear_of_borders(x, u, temperature, top_k, top_p, min_p):
    """A number near u that is at least 1e-9 of the sum away from every border of the row's kept tokens."""
    if np.isnan(x).any() or not np.isfinite(x.max()) or not temperature > 0:
        return u
    _, p = X.kept(x, temperature, top_k, top_p, min_p)
    edges = np.concatenate([[0.0], np.cumsum(p)]) / p.sum()
    for _ in range(200):
        if np.abs(edges - float(np.float32(u))).min() > 1e-9:
            return u
        u = float(np.float32(u * 0.999 + 0.0003))
    raise AssertionError("no place between the borders")


def check(ctx, logits, u, dtype=torch.float32, temperature=None, top_k=None, top_p=None, min_p=None, strided=False, nudge=True):
    t = dev(logits, dtype)
    n = len(t)
    if strided:
        wide = torch.full((n, t.shape[1] + 5), float("nan"), dtype=dtype, device="cuda")
        wide[:, 3:-2] = t
        t = wide[:, 3:-2]
    x = t.double().cpu().numpy()
    f32 = lambda v, d: np.full(n, d) if v is None else np.float32(np.broadcast_to(np.asarray(v), (n,))).astype(np.float64)  # noqa: E731
    T, P, M = f32(temperature, 1.0), f32(top_p, 1.0), f32(min_p, 0.0)
    K = np.zeros(n, dtype=np.int64) if top_k is None else np.broadcast_to(np.asarray(top_k), (n,)).astype(np.int64)
    u = np.array([clear_of_borders(x[i], float(u[i]), T[i], int(K[i]), P[i], M[i]) if nudge else u[i] for i in range(n)])
    u = u.astype(np.float32)
    tokens, probs = ctx.rk_sample(t, dev(u), temperature=None if temperature is None else dev(T), top_k=None if top_k is None else dev(K, torch.int32),
                                  top_p=None if top_p is None else dev(P), min_p=None if min_p is None else dev(M))
    ctx.rk_poll_status()
    want = [X.sample(x[i], float(u[i]), T[i], int(K[i]), P[i], M[i]) for i in range(n)]
    assert tokens.cpu().tolist() == [w[0] for w in want]
    got, wp = probs.double().cpu().numpy(), np.array([w[1] for w in want])
    assert np.array_equal(np.isnan(got), np.isnan(wp))
    ok = ~np.isnan(wp)
    assert (np.abs(got - wp)[ok] <= 2.0 ** -24 * wp[ok] * 1.001 + 1e-9 * wp[ok]).all()
    return tokens, probs


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n, vocab", [(1, 1), (4, 2), (9, 33), (5, 1000), (3, 2049), (6, 4096), (3, 16385), (4, 32001), (2, 50000), (2, 131072), (1, 200003)])
def test_all_filters_match_oracle(ctx, n, vocab, dtype):
    rng = np.random.default_rng(vocab)
    x = rng.standard_normal((n, vocab)) * 2.5
    u = rng.random(n)
    check(ctx, x, u, dtype)                                                                # plain sampling
    check(ctx, x, u, dtype, temperature=0.7, strided=True)
    check(ctx, x, u, dtype, top_k=40)
    check(ctx, x, u, dtype, top_p=0.9)
    check(ctx, x, u, dtype, min_p=0.05)
    check(ctx, x, u, dtype, temperature=1.3, top_k=rng.integers(1, 100, size=n), top_p=rng.uniform(0.3, 1.0, size=n), min_p=rng.choice([0.0, 0.01], size=n))
    check(ctx, x, u, dtype, temperature=rng.choice([0.0, 0.5, 1.5], size=n), top_k=rng.integers(vocab // 2, 2 * vocab + 1, size=n), top_p=0.99, strided=True)


@pytest.mark.parametrize("vocab", [64, 5000, 70000])
def test_ties_and_equal_rows(ctx, vocab):
    """Equal logits: rank by index, in all three filters; a row of one value; few distinct values."""
    rng = np.random.default_rng(vocab)
    x = np.zeros((6, vocab))
    x[1] = -3.0
    x[2] = rng.integers(0, 3, size=vocab)
    x[3] = rng.integers(0, 3, size=vocab) * 1e-3
    x[4, ::2] = -0.0                                           # both zeros are one
    x[5] = np.where(rng.random(vocab) < 0.5, 1.0, -1.0)
    u = rng.random(6)
    for k in (1, 2, 7, vocab // 2, vocab - 1, vocab):
        check(ctx, x, u, top_k=k)
        check(ctx, x, u, top_k=k, top_p=0.5)
    for p in (1e-6, 0.25, 0.5, 0.75, 0.999):
        check(ctx, x, u, top_p=p)
        check(ctx, x, u, top_p=p, min_p=0.4)
    check(ctx, x, u, min_p=1.0)
    check(ctx, x, u, min_p=0.36788, temperature=1.0)


def test_masks_infinities_and_nan(ctx):
    rng = np.random.default_rng(2)
    v = 3001
    x = rng.standard_normal((12, v))
    x[0] = -np.inf                                              # nothing left
    x[1, 1:] = -np.inf                                          # the first only
    x[2, :-1] = -np.inf                                         # the last only
    x[3, 1234] = np.nan
    x[4, 77] = np.inf
    x[5, [5, 99, 2000]] = np.inf                                # three alike
    x[6, ::3] = -np.inf
    x[7] = np.finfo(np.float32).min                             # the type's lowest value is a number
    x[8, 10:] = np.finfo(np.float32).min
    x[9] *= 1e30
    x[10, :] = -np.inf
    x[10, 3] = np.nan
    x[11] = np.finfo(np.float32).max
    u = rng.random(12)
    for kw in ({}, dict(top_k=5), dict(top_p=0.8), dict(temperature=0.0), dict(temperature=0.8, top_k=50, top_p=0.9, min_p=0.1), dict(min_p=0.5)):
        check(ctx, x, u, **kw)


def test_parameters_out_of_their_range_are_off_or_greedy(ctx):
    rng = np.random.default_rng(4)
    x, u = rng.standard_normal((4, 500)), rng.random(4)
    base, _ = check(ctx, x, u)
    for kw in (dict(top_k=0), dict(top_k=-5), dict(top_k=500), dict(top_k=1 << 30), dict(top_p=1.0), dict(top_p=7.0), dict(min_p=0.0), dict(min_p=-1.0)):
        assert torch.equal(check(ctx, x, u, **kw)[0], base)
    t, one = dev(x), torch.ones(4, device="cuda")
    nan = one * float("nan")
    assert torch.equal(ctx.rk_sample(t, dev(u), top_p=nan)[0], ctx.rk_sample(t, dev(u))[0])
    assert torch.equal(ctx.rk_sample(t, dev(u), min_p=nan)[0], ctx.rk_sample(t, dev(u))[0])
    greedy = torch.argmax(t, 1).int()
    for kw in (dict(temperature=0 * one), dict(temperature=-one), dict(temperature=nan), dict(top_p=0 * one), dict(top_p=-one), dict(min_p=2 * one),
               dict(top_k=torch.ones(4, dtype=torch.int32, device="cuda")), dict(temperature=1e-38 * one)):
        tokens, probs = ctx.rk_sample(t, dev(u), **kw)
        assert torch.equal(tokens, greedy) and (probs == 1).all()
    check(ctx, x, u, temperature=float("inf"))                  # every token alike
    check(ctx, x, u, temperature=1e30)


def test_random_numbers_at_the_ends(ctx):
    x = np.array([[0.0, 1.0, -np.inf, 2.0, -np.inf]] * 6)
    u = np.array([0.0, 1.0, 2.0, -1.0, np.nan, 1 - 2.0 ** -24])
    tokens, _ = ctx.rk_sample(dev(x), dev(u))
    assert tokens.cpu().tolist() == [0, 3, 3, 0, 0, 3]
    tokens, _ = ctx.rk_sample(dev(np.zeros((4, 2))), dev([0.0, 0.49999997, 0.5, 0.9999999]))    # a border goes to the next token
    assert tokens.cpu().tolist() == [0, 0, 1, 1]


def test_frequencies(ctx):
    """4096 evenly spread numbers draw every token as often as its probability says, to within one draw per border."""
    x = np.array([0.3, -1.0, 2.0, 0.0, 1.0, -4.0])
    n = 4096
    tokens, probs = ctx.rk_sample(dev(x).repeat(n, 1), dev((np.arange(n) + 0.5) / n), temperature=dev(np.full(n, 0.9)))
    p = np.exp((x - 2.0) / float(np.float32(0.9)))
    p /= p.sum()
    count = np.bincount(tokens.cpu().numpy(), minlength=6)
    assert (np.abs(count - n * p) <= 1.0 + 1e-3).all()
    assert np.abs(probs.double().cpu().numpy() - p[tokens.cpu().numpy()]).max() <= 2.0 ** -23


def test_a_captured_step_follows_its_inputs(ctx):
    """The last calls of a generating step: the head's 4-bit product, then the token; replayed with other activations."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n, vocab, k = 5, 4000, 256
    head = ctx.rk_quant4((torch.randn((1, vocab, k), generator=g, device="cuda") * 0.2).to(torch.bfloat16), 128)
    x = torch.randn((n, 1, k), generator=g, device="cuda").to(torch.bfloat16)
    u, T = torch.rand(n, generator=g, device="cuda"), torch.full((n,), 0.8, device="cuda")
    K = torch.full((n,), 30, dtype=torch.int32, device="cuda")

    def step():
        logits = ctx.rk_matvec4(head, x, out_dtype=torch.float32)[:, 0]
        return (logits,) + ctx.rk_sample(logits, u, temperature=T, top_k=K)

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            logits, tokens, probs = step()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        x.copy_(torch.randn((n, 1, k), generator=g, device="cuda").to(torch.bfloat16))
        u.copy_(torch.rand(n, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        lx, uu = logits.double().cpu().numpy(), u.double().cpu().numpy()
        assert tokens.cpu().tolist() == [X.sample(lx[i], uu[i], float(np.float32(0.8)), 30)[0] for i in range(n)]
    ctx.rk_poll_status()


def test_refusals(rk, ctx):
    x, u = torch.zeros((3, 10), device="cuda"), torch.zeros(3, device="cuda")
    with pytest.raises(rk.RKError) as ei:
        ctx.rk_sample(torch.zeros((1, (1 << 20) + 1), device="cuda"), u[:1])
    assert ei.value.status == 7
    with pytest.raises(rk.RKError):
        ctx.rk_sample(torch.zeros((3, 0), device="cuda"), u)
    with pytest.raises(TypeError):
        ctx.rk_sample(x.half(), u)
    with pytest.raises(TypeError):
        ctx.rk_sample(x, u.double())
    with pytest.raises(TypeError):
        ctx.rk_sample(x, u, top_k=u)
    with pytest.raises(ValueError):
        ctx.rk_sample(x, u[:2])
    with pytest.raises(ValueError):
        ctx.rk_sample(x, u.cpu())
    with pytest.raises(ValueError):
        ctx.rk_sample(x.t(), torch.zeros(10, device="cuda"))
    tokens, probs = ctx.rk_sample(torch.zeros((0, 10), device="cuda"), u[:0])
    assert tokens.shape == (0,) and probs.shape == (0,)


# temperatures at both ends of fp32 (from 2^-100 down the largest logit; infinite: all alike), over logits at both ends
@pytest.mark.parametrize("vocab", [7, 3000])
@pytest.mark.parametrize("temperature", [float("inf"), 3e38, 1e30, 1e-30, 2.0 ** -100, 2.0 ** -101, 1e-44, -1.0, float("nan")])
def test_extreme_temperatures(ctx, vocab, temperature):
    rng = np.random.default_rng(vocab)
    x = rng.standard_normal((4, vocab))
    x[1] = rng.choice([3e38, -3e38, 1.0], size=vocab)
    x[2] *= 1e-37
    x[3, ::2] = -np.inf
    u = rng.random(4)
    for kw in ({}, dict(top_k=3), dict(top_p=0.6), dict(min_p=0.5), dict(top_k=300, top_p=0.6)):
        check(ctx, x, u, temperature=temperature, **kw)


def test_top_k_among_too_many_candidates_is_the_same_every_time(ctx):
    """Rows of which half is one low logit: more tokens reach what the quick search starts from than its list holds, and the
    cluster goes on with bins.  The calls follow one another with other kernels in between, so that the thread blocks of a
    row run apart; all of them have to give the oracle's tokens."""
    rng = np.random.default_rng(28)
    n, vocab = 28, 28479
    x = rng.standard_normal((n, vocab)) * 2.5
    x[:, vocab // 2:] = 0.0
    u = rng.random(n)
    first, probs = check(ctx, x, u, top_k=200, top_p=0.999)
    t, f = dev(x), lambda v, dt=torch.float32: torch.full((n,), v, dtype=dt, device="cuda")  # noqa: E731
    uu = dev(np.array([clear_of_borders(t[i].double().cpu().numpy(), float(u[i]), 1.0, 200, float(np.float32(0.999)), 0.0) for i in range(n)]).astype(np.float32))
    k, p, room = f(200, torch.int32), f(0.999), torch.empty(64 << 20, device="cuda")
    w, tokens = ctx.rk_quant8(torch.randn((1, 2048, 2048), device="cuda").to(torch.bfloat16)), ctx.rk_quant8(torch.randn((300, 2048), device="cuda").to(torch.bfloat16))
    for i in range(200):
        if i % 2:
            room.zero_()
        else:
            ctx.rk_matmul8(w, tokens)
            ctx.rk_moe_route(room[:64 * 1024].view(64, 1024), 8)
        got, got_p = ctx.rk_sample(t, uu, top_k=k, top_p=p)
        assert torch.equal(got, first) and torch.equal(got_p, probs)
    ctx.rk_poll_status()
