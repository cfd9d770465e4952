"""Attention over the 4-bit cache against the float64 oracle with the bound of what the kernel computes: the query's turned rope
part enters in two bf16 parts, so a logit, and with it the log-sum-exp, is as good as fp32 sums are.

The bound, per query row.  big = max over the visible keys of sum |q_rope||k_rope| (turned), size the same over all 576 dims, pairs
that of sum over the pairs of dims of (|q0| + |q1|)(|k0| + |k1|) before turning.
  two parts       the high part is off by at most 2^-8 of a value, the low part by 2^-8 of that:            2^-16 big
  turn            cos and sin of an angle reduced in double (2^-26 turns, positions to 2^30 another 4e-8 turns), two ulps
                  each, two products and a sum in fp32: below 1e-6 of |q0| + |q1| per value:              1e-6 pairs
  products        exact in fp32; a step sums 16 and the accumulator, each aligned or rounded to 2^-23 of the step's
                  sum of magnitudes.  8 steps for rope (high and low part), 32 for the latent, which comes first and
                  is 0 where the latent query is 0:                            17 * 2^-23 (8 or 40) * 1.01 size
All of it times sm_scale is a logit's error e.  The log-sum-exp adds the base-2 score's and the maximum's roundings (3 2^-24 of
the largest logit), ex2 (2^-22), the sum over tiles, lanes and parts ((tiles + 40) 2^-24), and the logarithm, the sum with the
maximum and the change of base, here and in the join (4 2^-23 |lse|).
O as in test_gpu_decode.py: p in bf16 and the output's rounding."""
import numpy as np
import pytest
import torch

from oracle import decode as D
from oracle.harness import f64
from tests.test_gpu_decode import BASE, SCALE, U, Pool, bf, chain, fill_pool, make_ctx, plan_for


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


def bounds(q, pos, rows_of, lse, big, size, latent):
    """(error of a logit, error of the log-sum-exp) per query row; rows_of: [(rows [n, 576], delta)]."""
    pairs, keys = np.zeros(len(q)), 0
    a = np.abs(q[:, 512:]).reshape(len(q), 32, 2).sum(axis=2)
    for rows, delta in rows_of:
        b = np.abs(rows[:, 512:]).reshape(len(rows), 32, 2).sum(axis=2)
        seen = (delta + np.arange(len(rows)))[None, :] <= pos[:, None]
        pairs = np.maximum(pairs, np.where(seen, a @ b.T, 0.0).max(axis=1, initial=0.0))
        keys += len(rows)
    e = SCALE * (2.0 ** -16 * big + 1e-6 * pairs + 17 * 2.0 ** -23 * (40 if latent else 8) * 1.01 * size)
    safe = np.where(np.isneginf(lse), 0.0, np.abs(lse))
    return e, e + 3 * 2.0 ** -24 * SCALE * size + 2.0 ** -22 + (keys / 128 + 40) * 2.0 ** -24 + 4 * 2.0 ** -23 * safe


def compare(pool, items, q_pos, q, O, lse, heads, latent=True):
    qh, oh, lh = f64(q), f64(O), lse.double().cpu().numpy()
    for b, mine in enumerate(items):
        ql = q_pos.shape[1]
        rows, pos = qh[b].reshape(ql * heads, 576), np.repeat(q_pos[b], heads)
        rows_of = [(pool.rows(s), d) for s, d in mine]
        o, want, mass, big, size = D.attention(rows, pos, rows_of, SCALE, BASE)
        e, e_lse = bounds(rows, pos, rows_of, want, big, size, latent)
        got_o, got = oh[b].reshape(ql * heads, 512), lh[b].reshape(ql * heads)
        none = np.isneginf(want)
        assert np.array_equal(np.isneginf(got), none), b
        off = np.abs(got[~none] - want[~none]) / e_lse[~none]
        assert (off <= 1.0).all(), (b, float(off.max()))
        tol = (U + np.exp(2 * e) - 1 + 1e-5)[:, None] * mass + U * np.abs(o) + 2.0 ** -126 * (1 + sum(
            len(r) * np.abs(r[:, :512]).max(initial=0.0) for r, _ in rows_of))
        assert (np.abs(got_o - o) <= tol).all(), b


def rope_only(rng, *shape):
    q = rng.standard_normal(shape + (576,)) * 8.0
    q[..., :512] = 0.0
    return q


def test_the_bound_sees_a_lost_low_part():
    """The mistake that the bound is there for, planted in the oracle: turned queries rounded to one bf16 part."""
    rng = np.random.default_rng(101)
    n, delta, rows_n = 700, 4321, 64
    rows = np.concatenate([rng.standard_normal((n, 512)), D.bf16_values(D.bf16_bits(rng.standard_normal((n, 64))))], axis=1)
    q = D.bf16_values(D.bf16_bits(rope_only(rng, rows_n)))
    pos = np.full(rows_n, delta + n - 1)
    _, want, _, big, size = D.attention(q, pos, [(rows, delta)], SCALE, BASE)
    _, e_lse = bounds(q, pos, [(rows, delta)], want, big, size, False)

    def with_parts(parts):
        left = D.turn(q[:, 512:], np.full(rows_n, -float(delta)), BASE)
        total = np.zeros_like(left)
        for _ in range(parts):
            part = D.bf16_values(D.bf16_bits(left))
            total, left = total + part, left - part
        turned = np.concatenate([q[:, :512], total], axis=1)
        return D.attention(turned, np.full(rows_n, n - 1), [(rows, 0)], SCALE, BASE)[1]   # offset 0: no turn is left to do

    assert (np.abs(with_parts(2) - want) <= e_lse).all()
    assert (np.abs(with_parts(1) - want) > e_lse).mean() > 1 / 3


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [16, 32, 64, 72])
@pytest.mark.parametrize("start", [0, 4321, 2 ** 30 - 20000])
def test_rope_scores_keep_fp32_accuracy(rk, heads, start):
    """Queries whose latent part is 0 and whose rope part is large, over segments at small and at the largest offsets."""
    ctx = make_ctx(rk, heads)
    lens = [700, 130, 1, 3000]
    pool = Pool(rk, lens, seed=102)
    fill_pool(ctx, pool, 102)
    items, end = chain(lens, [1, 0, 2, 3], start=start)
    items, q_pos = [items, items[:3]], np.array([[end - 2, end - 1], [start + 500, start + 2]])
    q = bf(rope_only(np.random.default_rng(103), 2, 2, heads))
    O, lse = ctx.rk_cache4_attn(pool.pages, plan_for(ctx, pool, items, q_pos), q)
    ctx.rk_poll_status()
    compare(pool, items, q_pos, q, O, lse, heads, latent=False)


@pytest.mark.gpu
@pytest.mark.parametrize("heads, q_len", [(8, 1), (24, 1), (40, 1), (72, 1), (16, 3), (64, 1)])
@pytest.mark.parametrize("requests, length", [(1, 40000), (40, 1300)])
def test_long_runs_of_tiles_with_rows_that_do_not_fill_a_row_tile(rk, heads, q_len, requests, length):
    """Several key tiles per thread block whose row tile has columns without a query row (64 heads: none), behind requests whose
    queries stand where those columns' would."""
    ctx = make_ctx(rk, heads)
    pool = Pool(rk, [length], seed=104)
    fill_pool(ctx, pool, 104)
    items = [[(0, 7 * b)] for b in range(requests)]
    q_pos = np.array([[7 * b + length - q_len + t for t in range(q_len)] for b in range(requests)])
    rng = np.random.default_rng(105)
    q = bf(rng.standard_normal((requests, q_len, heads, 576)) * (1.0 + 20.0 * (np.arange(requests) % 2))[:, None, None, None])
    O, lse = ctx.rk_cache4_attn(pool.pages, plan_for(ctx, pool, items, q_pos), q)
    ctx.rk_poll_status()
    some = sorted({0, requests // 2, requests - 1})
    compare(pool, [items[b] for b in some], q_pos[some], q[some], O[some], lse[some], heads)
