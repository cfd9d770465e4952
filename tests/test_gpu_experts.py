"""Routing to experts and the lists by expert against the float64 oracle.  Ids and lists are compared as they are (scores are
compared in 64 bits on both sides); weights are one fp32 rounding (2^-24) of a 64-bit value whose own error, a softmax of up
to 1024 terms, is below 2^-40: |dw| <= 2^-23 |w| with room, and below the smallest normal number 2^-126 one unit of 2^-149."""
import numpy as np
import pytest
import torch

from oracle import experts as X
from oracle import policy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ctx(rk):
    return rk.Context(16, 2, 256, 1024, [0, 8], 0.07)


def check_route(ctx, logits, k, bias=None, dtype=torch.float32, strided=False, **kw):
    t = torch.from_numpy(np.asarray(logits, dtype=np.float32)).to(dtype).cuda()
    if strided:
        wide = torch.full((t.shape[0], t.shape[1] + 3), float("nan"), dtype=dtype, device="cuda")
        wide[:, 1:-2] = t
        t = wide[:, 1:-2]
    b = None if bias is None else torch.from_numpy(np.asarray(bias, dtype=np.float32)).cuda()
    ids, w = ctx.rk_moe_route(t, k, bias=b, **kw)
    ctx.rk_poll_status()
    want_ids, want_w = X.route(t.double().cpu().numpy(), k, None if bias is None else b.double().cpu().numpy(), **kw)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    got = w.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want_w))
    ok = ~np.isnan(want_w)
    assert (np.abs(got - want_w)[ok] <= 2.0 ** -23 * np.abs(want_w[ok]) + 2.0 ** -149).all()
    return ids, w


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n, e, groups, top, group_top, k", [
    (1, 1, 1, 1, 1, 1), (3, 5, 1, 1, 1, 5), (65, 256, 8, 4, 2, 6), (33, 160, 8, 3, 1, 6), (17, 1024, 1, 1, 2, 16), (9, 1020, 17, 5, 2, 16),
    (40, 64, 32, 7, 2, 8), (31, 33, 11, 11, 1, 8), (8, 128, 4, 1, 2, 8), (1000, 96, 3, 2, 2, 4), (5, 992, 31, 30, 1, 7), (7, 512, 1, 1, 1, 3),
])
def test_route_matches_oracle(ctx, score, n, e, groups, top, group_top, k):
    rng = np.random.default_rng(n * 1000 + e)
    for i, (dtype, biased) in enumerate([(torch.float32, True), (torch.float32, False), (torch.bfloat16, True), (torch.bfloat16, False)]):
        check_route(ctx, rng.standard_normal((n, e)) * 2, k, rng.standard_normal(e) * 0.2 if biased else None, dtype, strided=i % 2 == 1, score=score,
                    n_groups=groups, top_groups=top, group_top=group_top, renorm=i >= 2, scale=[1.0, 2.5][i % 2])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_ties_masks_and_extremes(ctx, score):
    rng = np.random.default_rng(7)
    n, e = 64, 64
    x = rng.integers(-2, 3, size=(n, e)).astype(np.float64)              # many equal scores
    x[1] = 0.0                                                           # all equal
    x[2] = -np.inf                                                       # nothing left
    x[3, 5:] = -np.inf                                                   # five experts left for six slots
    x[4, 8:] = -np.inf                                                   # one group left
    x[5, 10] = np.nan
    x[6] = -np.inf
    x[6, 63] = 3.0                                                       # the last expert only
    x[7] = np.finfo(np.float32).min                                      # the type's lowest value is a number like any other
    x[8, ::2] = np.finfo(np.float32).min
    x[9] = rng.standard_normal(e) * 1e-30
    x[10] = 80.0 + rng.standard_normal(e)
    x[11] = -100.0 + rng.standard_normal(e)
    x[12, 3] = np.inf                                                    # softmax: NaN; sigmoid: 1
    x[13, ::8] = -np.inf                                                 # every group one short
    bias = rng.integers(-1, 2, size=e) * 0.25
    bias[17] = -np.inf
    for groups, top, gt in ((1, 1, 1), (8, 2, 1), (8, 2, 2), (4, 3, 2)):
        for renorm in (False, True):
            check_route(ctx, x, 6, None, score=score, n_groups=groups, top_groups=top, group_top=gt, renorm=renorm)
            check_route(ctx, x, 6, bias, score=score, n_groups=groups, top_groups=top, group_top=gt, renorm=renorm)


def test_route_decides_neighbours_that_fp32_confuses(ctx):
    """Scores that are equal in fp32 and differ in 64 bits: sigmoid of neighbouring large logits, and a bias that swallows them."""
    x = np.zeros((4, 32))
    x[0] = 12.0 + np.arange(32) * 2.0 ** -19           # sigmoid differs by 1e-11
    x[1] = 12.0 + np.arange(32)[::-1] * 2.0 ** -19
    x[2] = 1.0 + (np.arange(32) % 5) * 2.0 ** -22
    x[3, 7] = 2.0 ** -24
    check_route(ctx, x, 8, score="sigmoid")
    check_route(ctx, x, 8, np.full(32, 100.0), score="sigmoid")
    check_route(ctx, x, 8, np.full(32, 100.0), score="softmax", n_groups=4, top_groups=2, group_top=2)


def test_route_nan_bias_marks_every_token(ctx):
    bias = np.zeros(16)
    bias[3] = np.nan
    ids, w = check_route(ctx, np.zeros((5, 16)), 2, bias)
    assert (ids == -1).all() and torch.isnan(w).all()


def check_group(ctx, ids, n_experts, keep=None):
    t = torch.from_numpy(np.asarray(ids, dtype=np.int32)).cuda()
    kp = None if keep is None else torch.from_numpy(np.asarray(keep, dtype=np.uint8)).cuda()
    off, rows = ctx.rk_moe_group(t, n_experts, kp)
    ctx.rk_poll_status()
    want_off, want_rows = X.group(np.asarray(ids), n_experts, keep)
    assert np.array_equal(off.cpu().numpy(), want_off) and np.array_equal(rows.cpu().numpy(), want_rows)


@pytest.mark.parametrize("n, k, e", [(1, 1, 1), (1, 6, 256), (7, 3, 5), (64, 6, 256), (511, 8, 33), (513, 8, 1024), (683, 6, 160), (4097, 1, 2), (3000, 16, 1024),
                                     (20000, 7, 64)])
def test_group_matches_oracle(ctx, n, k, e):
    rng = np.random.default_rng(n + k + e)
    ids = rng.integers(0, e, size=(n, k))
    check_group(ctx, ids, e)
    ids[rng.random((n, k)) < 0.2] = -1                       # routed nowhere
    ids[rng.random((n, k)) < 0.01] = e                       # out of range
    ids[rng.random((n, k)) < 0.01] = -(1 << 31)
    check_group(ctx, ids, e)
    if k <= 8:
        check_group(ctx, ids, e, rng.integers(0, 256, size=n))
        check_group(ctx, ids, e, np.zeros(n))
    check_group(ctx, np.full((n, k), e - 1), e)              # all for one
    check_group(ctx, np.full((n, k), -1), e)                 # none at all


def test_group_without_tokens(ctx):
    off, rows = ctx.rk_moe_group(torch.empty((0, 6), dtype=torch.int32, device="cuda"), 10)
    assert (off == 0).all() and rows.numel() == 0
    ids, w = ctx.rk_moe_route(torch.empty((0, 8), device="cuda"), 2)
    assert ids.shape == (0, 2) and w.shape == (0, 2)


def test_route_fanout_group_in_a_graph(ctx):
    """The chain as a step captures it: route, fan-out on the weights, lists of what stays; replayed on other logits."""
    n, e, k = 300, 128, 6
    logits = torch.randn((n, e), device="cuda")
    bias = torch.randn(e, device="cuda") * 0.1

    def step():
        ids, w = ctx.rk_moe_route(logits, k, bias=bias, score="sigmoid", n_groups=8, top_groups=4, group_top=2, renorm=True)
        k_t, keep = ctx.rk_moe_fanout(w, 0.75)
        return (ids, w, keep) + ctx.rk_moe_group(ids, e, keep)

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ids, w, keep, off, rows = step()
    torch.cuda.current_stream().wait_stream(side)
    for seed in range(3):
        torch.manual_seed(seed)
        logits.copy_(torch.randn((n, e), device="cuda") * 2)
        graph.replay()
        torch.cuda.synchronize()
        want_ids, _ = X.route(logits.double().cpu().numpy(), k, bias.double().cpu().numpy(), "sigmoid", 8, 4, 2, True)
        assert np.array_equal(ids.cpu().numpy(), want_ids)
        _, want_keep = policy.moe_fanout(w.cpu().numpy(), 0.75)
        assert np.array_equal(keep.cpu().numpy(), want_keep)
        want_off, want_rows = X.group(want_ids, e, want_keep)
        assert np.array_equal(off.cpu().numpy(), want_off) and np.array_equal(rows.cpu().numpy(), want_rows)
    ctx.rk_poll_status()


@pytest.mark.parametrize("change, status", [
    (dict(n_groups=0), 7), (dict(n_groups=33), 7), (dict(n_groups=3), 7), (dict(top_groups=0), 2), (dict(n_groups=4, top_groups=5), 2),
    (dict(k=0), 2), (dict(k=17), 2), (dict(k=5, n_groups=16, top_groups=1), 2), (dict(group_top=3), 7), (dict(scale=float("inf")), 2),
])
def test_route_refusals(rk, ctx, change, status):
    kw = dict(k=4)
    kw.update(change)
    with pytest.raises(rk.RKError) as ei:
        ctx.rk_moe_route(torch.zeros((2, 64), device="cuda"), **kw)
    assert ei.value.status == status


def test_wrong_tensors_are_refused(rk, ctx):
    x = torch.zeros((4, 32), device="cuda")
    with pytest.raises(TypeError):
        ctx.rk_moe_route(x.half(), 2)
    with pytest.raises(ValueError):
        ctx.rk_moe_route(x, 2, score="tanh")
    with pytest.raises(ValueError):
        ctx.rk_moe_route(x.t(), 2)
    with pytest.raises(ValueError):
        ctx.rk_moe_route(x[0].expand(4, 32), 2)
    with pytest.raises(ValueError):
        ctx.rk_moe_route(x, 2, bias=torch.zeros(31, device="cuda"))
    with pytest.raises(RuntimeError):
        ctx.rk_moe_route(torch.zeros((1, 1025), device="cuda"), 2)
    ids = torch.zeros((4, 9), dtype=torch.int32, device="cuda")
    with pytest.raises(rk.RKError) as ei:
        ctx.rk_moe_group(ids, 4, torch.zeros(4, dtype=torch.uint8, device="cuda"))     # nine slots, eight mask bits
    assert ei.value.status == 7
    with pytest.raises(rk.RKError):
        ctx.rk_moe_group(ids, 1025)
    with pytest.raises(TypeError):
        ctx.rk_moe_group(ids.long(), 4)


# Scores a few fp32 steps apart, where the order is settled in 64 bits: among a token's own choices, at the last place, over more
# experts than a warp compares at once, and between groups.  Logits are multiples of 2^-23 around a few levels (scores of different
# logits are at least 2^-36 apart, equal ones equal; groups go by one score, as sums of two could differ by less than their
# rounding), biases from two values.
@pytest.mark.parametrize("n_e, k, groups, top_groups, group_top", [(64, 6, 1, 1, 1), (256, 8, 1, 1, 1), (160, 6, 8, 3, 1), (256, 6, 8, 4, 1), (1024, 16, 1, 1, 1), (24, 3, 3, 2, 1)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("steps", [1, 5, 40, 400])
def test_scores_that_are_nearly_equal(ctx, n_e, k, groups, top_groups, group_top, score, biased, steps):
    rng = np.random.default_rng(n_e + k + steps)
    n = 60
    levels = np.array([0.5, 1.0 - 2.0 ** -12, -1.5, 0.0])
    x = levels[rng.integers(0, 4, size=(n, n_e))] + rng.integers(0, steps + 1, size=(n, n_e)) * 2.0 ** -23
    x[n // 2:] = levels[rng.integers(0, 4, size=(n - n // 2, 1))] + rng.integers(0, steps + 1, size=(n - n // 2, n_e)) * 2.0 ** -23
    x[-3, ::2] = 0.0
    x[-3, 1::2] = -0.0
    x = x.astype(np.float32)
    bias = rng.choice([0.0, 0.25], size=n_e) if biased else None
    ids, w = ctx.rk_moe_route(torch.from_numpy(x).cuda(), k, bias=None if bias is None else torch.from_numpy(bias.astype(np.float32)).cuda(),
                              score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)
    want, ww = X.route(x.astype(np.float64), k, bias=bias, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)
    assert np.array_equal(ids.cpu().numpy(), want)
    assert np.abs(w.double().cpu().numpy() - ww).max() <= 2.0 ** -24 + 1e-12
