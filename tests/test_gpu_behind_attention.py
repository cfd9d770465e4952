"""The operators behind the attention as a program uses them: together in one captured step, on several streams at once, and on
rows of padding.  Sampled tokens of large rows are compared with a 64-bit evaluation in torch."""
import numpy as np
import pytest
import torch

from oracle import experts as X
from tests.test_gpu_matmul8 import bf, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ctx(rk):
    return rk.Context(16, 2, 256, 1024, [0, 8], 0.07)


def test_a_layer_and_the_head_in_one_graph(ctx):
    """Router, fan-out, lists, both expert products, weighted sum, head product, token: captured once, replayed on other
    activations, equal to the same calls made one by one, and the token to the oracle's from the logits."""
    rng = np.random.default_rng(3)
    n, n_e, slots, d, inner, vocab = 24, 32, 6, 256, 128, 5003
    w1, w2, head = weights(ctx, rng, n_e, 2 * inner, d)[0], weights(ctx, rng, n_e, d, inner)[0], weights(ctx, rng, 1, vocab, d)[0]
    gate = torch.randn((d, n_e), device="cuda") * 0.1
    bias = torch.randn(n_e, device="cuda") * 0.05
    x = torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
    u, T = torch.empty(n, device="cuda"), torch.full((n,), 0.7, device="cuda")
    top_k, top_p = torch.full((n,), 40, dtype=torch.int32, device="cuda"), torch.full((n,), 0.9, device="cuda")

    def step():
        ids, wt = ctx.rk_moe_route((x.float()[:, :, None] * gate).sum(1), slots, bias=bias, score="sigmoid", n_groups=4, top_groups=2, group_top=2, renorm=True, scale=1.5)
        _, keep = ctx.rk_moe_fanout(wt, 0.8)
        off, rows = ctx.rk_moe_group(ids, n_e, keep)
        h = ctx.rk_matmul8_experts(w1, ctx.rk_quant8(x), off, rows, slots, y=torch.zeros((n * slots, 2 * inner), dtype=torch.bfloat16, device="cuda"))
        a = (torch.nn.functional.silu(h[:, :inner].float()) * h[:, inner:].float()).to(torch.bfloat16)
        y = ctx.rk_matmul8_experts(w2, ctx.rk_quant8(a), off, rows, 1, y=torch.zeros((n * slots, d), device="cuda"))
        out = (x.float() + (y.view(n, slots, d) * wt[..., None]).sum(1)).to(torch.bfloat16)
        logits = ctx.rk_matmul8(head, ctx.rk_quant8(out), out_dtype=torch.float32)
        return logits, *ctx.rk_sample(logits, u, temperature=T, top_k=top_k, top_p=top_p)

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x.copy_(torch.randn((n, d), generator=g, device="cuda"))
        u.copy_(torch.rand(n, generator=g, device="cuda"))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            captured = step()
    torch.cuda.current_stream().wait_stream(side)
    for seed in (1, 2, 3):
        fill(seed)
        graph.replay()
        again = step()
        torch.cuda.synchronize()
        for a, b in zip(captured, again):
            assert torch.equal(a, b)
        lx, uu = captured[0].double().cpu().numpy(), u.double().cpu().numpy()
        want = [X.sample(lx[i], uu[i], float(np.float32(0.7)), 40, float(np.float32(0.9))) for i in range(n)]
        assert captured[1].cpu().tolist() == [t for t, _ in want]
    ctx.rk_poll_status()


def test_calls_on_two_streams_at_once(ctx):
    """Nothing is shared between calls: interleaved on two streams, with one set of weights, they give what they give alone."""
    rng = np.random.default_rng(5)
    n, n_e, slots, n_out, k = 400, 16, 4, 512, 1024
    w = weights(ctx, rng, n_e, n_out, k)[0]
    jobs = []
    for i in range(2):
        logits = torch.randn((n, n_e), device="cuda")
        jobs.append(dict(x=bf(rng.standard_normal((n, k))), logits=logits, big=torch.randn((8, 40000), device="cuda") * 2, u=torch.rand(8, device="cuda")))

    def run(j):
        ids, wt = ctx.rk_moe_route(j["logits"], slots)
        off, rows = ctx.rk_moe_group(ids, n_e)
        y = ctx.rk_matmul8_experts(w, ctx.rk_quant8(j["x"]), off, rows, slots)
        return ids, wt, off, rows, y, *ctx.rk_sample(j["big"], j["u"], top_p=torch.full((8,), 0.9, device="cuda"))

    alone = [run(j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[] for _ in jobs]
    for _ in range(5):
        for i, (s, j) in enumerate(zip(streams, jobs)):
            with torch.cuda.stream(s):
                got[i].append(run(j))
    torch.cuda.synchronize()
    for i in range(2):
        for rep in got[i]:
            for a, b in zip(rep, alone[i]):
                assert torch.equal(a, b)
    ctx.rk_poll_status()


def test_a_padded_batch(ctx):
    """Rows of padding (no expert eligible, nothing to sample, no pair kept) leave the others as they are alone."""
    rng = np.random.default_rng(6)
    n, n_e, slots, n_out, k = 40, 8, 3, 96, 160
    pad = np.arange(n) % 3 == 1
    logits = rng.standard_normal((n, n_e))
    logits[pad] = -np.inf
    w = weights(ctx, rng, n_e, n_out, k)[0]
    x = bf(rng.standard_normal((n, k)))
    l = torch.from_numpy(logits.astype(np.float32)).cuda()
    ids, wt = ctx.rk_moe_route(l, slots, renorm=True)
    assert (ids[pad] == -1).all() and (wt[pad] == 0).all()
    off, rows = ctx.rk_moe_group(ids, n_e)
    y = ctx.rk_matmul8_experts(w, ctx.rk_quant8(x), off, rows, slots, y=torch.full((n * slots, n_out), 3.0, device="cuda")).view(n, slots, n_out)
    assert (y[pad] == 3.0).all()
    live = torch.from_numpy(np.nonzero(~pad)[0]).cuda()
    ids2, wt2 = ctx.rk_moe_route(l[live], slots, renorm=True)
    off2, rows2 = ctx.rk_moe_group(ids2, n_e)
    y2 = ctx.rk_matmul8_experts(w, ctx.rk_quant8(x[live]), off2, rows2, slots, out_dtype=torch.float32).view(len(live), slots, n_out)
    assert torch.equal(ids[live], ids2) and torch.equal(wt[live], wt2) and torch.equal(y[live], y2)
    big = torch.randn((n, 3001), device="cuda")
    big[torch.from_numpy(pad).cuda()] = float("-inf")
    u = torch.rand(n, device="cuda")
    tokens, probs = ctx.rk_sample(big, u, top_p=torch.full((n,), 0.8, device="cuda"))
    assert (tokens[pad] == -1).all() and torch.isnan(probs[pad]).all()
    t2, p2 = ctx.rk_sample(big[live], u[live], top_p=torch.full((len(live),), 0.8, device="cuda"))
    assert torch.equal(tokens[live], t2) and torch.equal(probs[live], p2)
    ctx.rk_poll_status()


def reference_tokens(x, u, T, k, p, m):
    """The definition in torch, 64 bits; tokens only."""
    x = x.double()
    v = x.shape[1]
    w = torch.exp((x - x.amax(1, keepdim=True)) / T)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    sw = torch.gather(w, 1, order)
    rank = torch.arange(v, device=x.device)[None]
    sw = torch.where(rank < (k if k > 0 else v), sw, torch.zeros_like(sw))
    run = torch.cumsum(sw, 1)
    front = torch.cat([torch.zeros_like(run[:, :1]), run[:, :-1]], 1)
    stay = ((rank < (k if k > 0 else v)) & ((front < p * run[:, -1:]) | (p >= 1)) & (sw >= m)) | (rank == 0)
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(stay, sw, torch.zeros_like(sw)))
    cdf = torch.cumsum(kept, 1)
    return torch.searchsorted(cdf, u.double()[:, None] * cdf[:, -1:], right=True)[:, 0].int()


# every way a cut is found: among the top 256, in estimated bins, by digits where a list overflows (equal logits), and with
# one, two, four and eight thread blocks per row.  A random number within 1e-12 of a border (one in 10^7 here) could differ.
@pytest.mark.parametrize("n, vocab, spread", [(1, 1 << 20, 2.5), (3, 600000, 0.01), (40, 131072, 2.5), (40, 131072, 0.0), (200, 50257, 4.0), (400, 20000, 1.0),
                                              (300, 4096, 0.3)])
@pytest.mark.parametrize("k, p, m", [(0, 1.0, 0.0), (0, 0.9, 0.0), (0, 0.999, 0.001), (3, 0.5, 0.0), (256, 0.99, 0.0), (257, 0.99, 0.0), (5000, 0.9, 0.01), (0, 1.0, 0.1)])
def test_large_rows_against_a_64_bit_evaluation(ctx, n, vocab, spread, k, p, m):
    g = torch.Generator(device="cuda").manual_seed(n + vocab + k)
    for dtype in (torch.float32, torch.bfloat16):
        x = (torch.randn((n, vocab), generator=g, device="cuda") * spread).to(dtype)
        u = torch.rand(n, generator=g, device="cuda")
        f = lambda c: torch.full((n,), c, device="cuda")  # noqa: E731
        T, P, M = 0.8, float(np.float32(p)), float(np.float32(m))
        tokens, _ = ctx.rk_sample(x, u, temperature=f(T), top_k=torch.full((n,), k, dtype=torch.int32, device="cuda"), top_p=f(p), min_p=f(m))
        want = torch.cat([reference_tokens(x[i:i + 16], u[i:i + 16], float(np.float32(T)), k, P, M) for i in range(0, n, 16)])
        assert torch.equal(tokens, want)
    ctx.rk_poll_status()


def test_rows_that_lie_beyond_32_bits(ctx):
    """Three rows 2^30 elements apart: offsets of 2^31 elements, 2^32 bytes and more, into and out of every call."""
    far = 1 << 30
    n, k, n_out = 3, 1000, 264
    g = torch.Generator(device="cuda").manual_seed(9)

    def spread(t):
        room = torch.empty(2 * far + t.shape[1], dtype=t.dtype, device="cuda")
        view = room.as_strided(t.shape, (far, 1))
        view.copy_(t)
        return view

    x = torch.randn((n, k), generator=g, device="cuda").to(torch.bfloat16)
    w = ctx.rk_quant8(torch.randn((1, n_out, k), generator=g, device="cuda").to(torch.bfloat16))
    q = ctx.rk_quant8(x)
    apart = spread(x)
    q2 = ctx.rk_quant8(apart)
    assert torch.equal(q.codes, q2.codes) and torch.equal(q.scales, q2.scales)
    for a, b in zip(ctx.rk_moe_route(x, 6), ctx.rk_moe_route(apart, 6)):
        assert torch.equal(a, b)
    u = torch.rand(n, generator=g, device="cuda")
    p = torch.full((n,), 0.8, device="cuda")
    for a, b in zip(ctx.rk_sample(x, u, top_p=p), ctx.rk_sample(apart, u, top_p=p)):
        assert torch.equal(a, b)
    del apart
    off, rows = torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        want = ctx.rk_matmul8(w, q, out_dtype=dtype)
        y = spread(torch.zeros((n, n_out), dtype=dtype, device="cuda"))
        assert torch.equal(ctx.rk_matmul8(w, q, y=y), want)
        y.zero_()
        assert torch.equal(ctx.rk_matmul8_experts(w, q, off, rows, 1, y=y), want)
        del y
    ctx.rk_poll_status()


def test_codes_that_lie_beyond_32_bits(ctx):
    """140000 rows of 16384 codes (2.3 GB): the last rows give what they give alone, as tokens, as listed pairs and as weights."""
    n, k, tail = 140000, 16384, 40
    g = torch.Generator(device="cuda").manual_seed(10)
    x = torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    x[-tail:] = torch.randn((tail, k), generator=g, device="cuda").to(torch.bfloat16)
    few = x[-tail:].clone()
    w = ctx.rk_quant8(torch.randn((1, 48, k), generator=g, device="cuda").to(torch.bfloat16))
    q, q_few = ctx.rk_quant8(x), ctx.rk_quant8(few)
    assert torch.equal(q.codes[-tail:], q_few.codes) and torch.equal(q.scales[-tail:], q_few.scales)
    want = ctx.rk_matmul8(w, q_few, out_dtype=torch.float32)
    y = ctx.rk_matmul8(w, q, out_dtype=torch.float32)
    assert torch.equal(y[-tail:], want) and (y[:-tail] == 0).all()
    off = torch.tensor([0, tail], dtype=torch.int32, device="cuda")
    rows = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    rows[:tail] = torch.arange(n - tail, n, device="cuda")
    y = torch.full((n, 48), 7.0, device="cuda")
    ctx.rk_matmul8_experts(w, q, off, rows, 1, y=y)
    assert torch.equal(y[-tail:], want) and (y[:-tail] == 7.0).all()
    y = ctx.rk_matmul8(q, w, out_dtype=torch.float32)[:, -tail:]  # the same rows as weights: the scales' two roundings (2^-24 each, on both sides) swap
    assert ((y - want.T).abs() <= 2.0 ** -22 * want.T.abs()).all()
    ctx.rk_poll_status()
