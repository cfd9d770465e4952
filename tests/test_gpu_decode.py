"""GPU parity of the decode operators through the C ABI against the float64 oracle: the 4-bit paged cache (append,
read), attention of single tokens over it, 4-bit matrix-vector products, and a run of them together.

Error bounds (derived, per element).  u = 2^-8 is half a bf16 step relative to the value.
  latent codes and scales       exact
  rope dims of a cached row     u |v| + 2e-6 (|x0| + |x1|): one bf16 rounding of an fp32 rotation whose angle is
                                reduced in double (error of cos, sin and of the two products below 2e-6)
  attention                     the turned query rope is rounded to bf16: a logit moves by at most
                                e = sm_scale (u sum|q_rope||k_rope| + 48 2^-23 sum|q||k|) (the second part: 36 fp32
                                additions of 16 products each, and the score in base-2 units) + 1e-5, which changes
                                every p by a factor within exp(+-2e); p is rounded to bf16 (u);
                                O is rounded once more:  |dO| <= (u + exp(2e) - 1 + 1e-5) sum p|c| + u |O|.  lse: e + 1e-5.
                                A key whose score lies so far below the largest that p < 2^-126 (fp32's and bf16's
                                smallest normal number) counts as 0: up to n 2^-126 max|c| more for n keys, and 2^-126
                                for an output below the smallest normal number
  matrix-vector                 fp32 sums of exact products: (k / 64 + 40) 2^-23 sum|x w| (+ u |y| for bf16 outputs)
"""
import numpy as np
import pytest
import torch

from oracle import decode as D
from oracle.harness import f64, rel_l2
from tests.helpers import REL_L2

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
BASE, SCALE = 10000.0, float(1.0 / np.sqrt(192.0))


@pytest.fixture(scope="module")
def rk():
    from paper_2609_07008_b200 import binding
    return binding


def make_ctx(rk, heads=16, **kw):
    g = heads // 8
    return rk.Context(heads, g, 256, 1024, [8 * i for i in range(g)], SCALE, BASE, **kw)


@pytest.fixture(scope="module")
def ctx(rk):
    return make_ctx(rk)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def bf(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


class Pool:
    """Segments of given lengths on shuffled pages, host and device side."""

    def __init__(self, rk, lens, seed, extra=2, fill=0xFF):
        rng = np.random.default_rng(seed)
        self.lens = list(lens)
        counts = [(n + 63) // 64 for n in lens]
        self.off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
        self.n_pages = int(self.off[-1]) + extra
        self.ids = rng.permutation(self.n_pages)[:int(self.off[-1])]
        self.host = D.Cache(self.n_pages, fill)          # 0xFF: NaN scales, NaN rope dims wherever no row was written
        self.pages = torch.full((self.n_pages, D.PAGE_BYTES), fill, dtype=torch.uint8, device="cuda")
        self.table = rk.CacheTable(i32(self.lens), i32(self.off), i32(self.ids))

    def page_list(self, s):
        return self.ids[self.off[s]:self.off[s + 1]]

    def rows(self, s, n=None):
        return self.host.rows(self.page_list(s), self.lens[s] if n is None else n)

    def from_device(self):
        self.host.pages = self.pages.cpu().numpy().reshape(self.n_pages, D.UNITS, D.PAGE_ROWS, 16)


def fill_pool(ctx, pool, seed, c_std=1.0, c=None):
    """Appends every segment from index 0 with random rows; returns the inputs (bf16 values)."""
    n = sum(pool.lens)
    rng = np.random.default_rng(seed + 1000)
    c = bf(rng.standard_normal((n, 512)) * c_std if c is None else c)
    kr = bf(rng.standard_normal((n, 64)))
    off = np.concatenate([[0], np.cumsum(pool.lens)])
    ctx.rk_cache4_append(pool.pages, pool.table, c, kr, i32(off))
    ctx.rk_poll_status()
    pool.from_device()
    return f64(c), f64(kr)


# ------------------------------------------------------------------------------------------------------------
# append, read
# ------------------------------------------------------------------------------------------------------------
def special_rows(rng, n):
    """Latents with the values quantisation can go wrong at: ties, zeros, tiny, huge, non-finite, one large value."""
    c = rng.standard_normal((n, 512))
    for i in range(n):
        k = i % 8
        if k == 1:
            c[i] = 0.0
        elif k == 2:
            c[i] = rng.integers(-14, 15, size=512) * 0.5 * 2.0 ** rng.integers(-6, 6)   # halves of a power-of-two scale
            c[i, ::16] = 7.0 * 2.0 ** rng.integers(-6, 6)
        elif k == 3:
            c[i] *= 10.0 ** rng.integers(-12, 6, size=512)
        elif k == 4:
            c[i] *= 1e6
        elif k == 5:
            c[i] *= 1e-9
        elif k == 6:
            c[i, rng.integers(0, 512, size=3)] = [np.inf, -np.inf, np.nan]
        elif k == 7:
            c[i, ::16] = rng.choice([1.0625, 1.1875, 1.3125, 1.9375, 1.4375], size=32) * 7 * 2.0 ** rng.integers(-14, 8)
    return c


@pytest.mark.parametrize("new, old, pad", [
    ([1], [0], 0), ([1, 1, 1], [63, 64, 127], 0), ([0, 5, 0, 200, 0, 1], [3, 60, 0, 1, 64, 5000], 7),
    ([64, 65, 63, 1, 129], [0, 0, 0, 64, 63], 0), ([33] * 40, list(range(40)), 31), ([3, 0, 0], [0, 0, 1], 1),
])
def test_append_matches_oracle_and_touches_nothing_else(rk, ctx, new, old, pad):
    rng = np.random.default_rng(sum(new) + pad)
    pool = Pool(rk, [a + b for a, b in zip(new, old)], seed=5, fill=0xA5)
    n = sum(new)
    c = bf(special_rows(rng, n + pad))
    wide = bf(rng.standard_normal((n + pad, 576)) * 3)         # rope part as a strided slice of a wider row
    kr = wide[:, 512:]
    off = np.concatenate([[0], np.cumsum(new)])
    ctx.rk_cache4_append(pool.pages, pool.table, c, kr, i32(off))
    ctx.rk_poll_status()
    before = pool.host.pages.copy()
    pool.from_device()
    codes, byte = D.quantise_latent(f64(c)[:n])
    x = f64(kr)[:n]
    written = np.zeros((pool.n_pages, 64), dtype=bool)
    at = 0
    for s, (a, b) in enumerate(zip(new, old)):
        for j in range(b, b + a):
            page, slot = pool.page_list(s)[j // 64], j % 64
            written[page, slot] = True
            gc, gb, gr = D.unpack_row(pool.host.pages[page, :, slot])
            assert np.array_equal(gb, byte[at]), (s, j)
            ok = np.repeat(byte[at] != 255, 16)                # codes of a NaN group are of no consequence
            assert np.array_equal(gc[ok], codes[at][ok]), (s, j)
            want = D.turn(x[at][None], [float(j)], BASE)[0]
            tol = U * np.abs(want) + 2e-6 * np.repeat(np.abs(x[at].reshape(32, 2)).sum(axis=1), 2)
            assert (np.abs(gr - want) <= tol).all(), (s, j)
            at += 1
    assert np.array_equal(pool.host.pages.transpose(0, 2, 1, 3)[~written], before.transpose(0, 2, 1, 3)[~written])


def test_append_positions_beyond_float_precision(rk, ctx):
    """Row 20 000 000 of a segment (its page list names one page over and over): the angle is reduced exactly."""
    j = 20_000_001
    n_list = j // 64 + 1
    table = rk.CacheTable(i32([j + 1]), i32([0, n_list]), torch.zeros(n_list, dtype=torch.int32, device="cuda"))
    pages = torch.zeros((1, D.PAGE_BYTES), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(1)
    c, kr = bf(rng.standard_normal((1, 512))), bf(rng.standard_normal((1, 64)))
    ctx.rk_cache4_append(pages, table, c, kr, i32([0, 1]))
    ctx.rk_poll_status()
    got = D.unpack_row(pages.cpu().numpy().reshape(D.UNITS, 64, 16)[:, j % 64])[2]
    want = D.turn(f64(kr), [float(j)], BASE)[0]
    tol = U * np.abs(want) + 2e-6 * np.repeat(np.abs(f64(kr)[0].reshape(32, 2)).sum(axis=1), 2)
    assert (np.abs(got - want) <= tol).all()


def test_append_and_read_with_many_empty_segments(rk, ctx):
    """A block's rows lie in segments far apart, with runs of empty ones between them."""
    rng = np.random.default_rng(11)
    new = rng.choice([0, 0, 0, 0, 0, 1, 2, 40], size=700)
    new[:100] = 0
    new[300:400] = 0
    new[-50:] = 0
    pool = Pool(rk, list(new), seed=11)
    c, _ = fill_pool(ctx, pool, 11)
    off = np.concatenate([[0], np.cumsum(new)])
    want = np.concatenate([pool.rows(s) for s in range(len(new)) if new[s]])
    codes, byte = D.quantise_latent(c)
    assert np.array_equal(want[:, :512], D.latent_values(codes, byte))
    assert np.array_equal(f64(ctx.rk_cache4_read(pool.pages, pool.table, i32(off), int(off[-1]))), want)
    ctx.rk_poll_status()


def test_read_returns_the_stored_values(rk, ctx):
    pool = Pool(rk, [1, 64, 65, 130, 700, 0, 3], seed=6)
    fill_pool(ctx, pool, 6)
    for take in ([1, 64, 65, 130, 700, 0, 3], [1, 1, 64, 66, 65, 0, 0], [0, 0, 0, 0, 1, 0, 3]):
        off = np.concatenate([[0], np.cumsum(take)])
        n, pad = int(off[-1]), 5
        kv = torch.full((n + pad, 576), 17.0, dtype=torch.bfloat16, device="cuda")
        out = ctx.rk_cache4_read(pool.pages, pool.table, i32(off), n + pad, kv=kv)
        ctx.rk_poll_status()
        want = np.concatenate([pool.rows(s)[pool.lens[s] - k:] for s, k in enumerate(take)])
        assert np.array_equal(f64(out)[:n], want)
        assert (out[n:] == 17.0).all()                           # padding rows are left as they were


def test_cache_calls_with_nothing_to_do(rk, ctx):
    pool = Pool(rk, [0, 0], seed=7)
    empty = torch.empty((0, 512), dtype=torch.bfloat16, device="cuda")
    ctx.rk_cache4_append(pool.pages, pool.table, empty, torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), i32([0, 0, 0]))
    assert ctx.rk_cache4_read(pool.pages, pool.table, i32([0, 0, 0]), 0).shape == (0, 576)
    rows = torch.zeros((3, 512), dtype=torch.bfloat16, device="cuda")
    ctx.rk_cache4_append(pool.pages, pool.table, rows, rows[:, :64], i32([0, 0, 0]))      # all padding
    ctx.rk_poll_status()
    assert (pool.pages == 0xFF).all()


def test_bad_tables_are_reported_and_skipped(rk, ctx):
    """Bad entries of the device tables: RK_ERR_ROWS, the row is skipped, good rows are unaffected."""
    rng = np.random.default_rng(8)
    c, kr = bf(rng.standard_normal((4, 512))), bf(rng.standard_normal((4, 64)))
    good = (i32([2, 2]), i32([0, 1, 2]), i32([1, 0]))
    for bad in [(good[0], good[1], i32([1, 7])), (good[0], good[1], i32([1, -1])), (i32([2, 1]), good[1], good[2]),
                (i32([2, 70]), good[1], good[2]), (good[0], i32([0, 1, 1]), good[2]), (good[0], i32([0, -1, 2]), good[2]),
                (good[0], i32([0, 5, 9]), good[2])]:
        pages = torch.full((2, D.PAGE_BYTES), 0xA5, dtype=torch.uint8, device="cuda")
        table = rk.CacheTable(*bad)
        ctx.rk_cache4_append(pages, table, c, kr, i32([0, 2, 4]))
        with pytest.raises(rk.RKError) as ei:
            ctx.rk_poll_status()
        assert ei.value.status == 4
        kv = torch.full((4, 576), 17.0, dtype=torch.bfloat16, device="cuda")
        ctx.rk_cache4_read(pages, table, i32([0, 2, 4]), 4, kv=kv)
        with pytest.raises(rk.RKError) as ei:
            ctx.rk_poll_status()
        assert ei.value.status == 4
        ctx.rk_poll_status()                                     # cleared: the context stays usable
    # malformed row ranges: never out of bounds, reported where a row has no place
    pages = torch.full((2, D.PAGE_BYTES), 0xA5, dtype=torch.uint8, device="cuda")
    ctx.rk_cache4_append(pages, rk.CacheTable(*good), c, kr, i32([3, 1, 4]))
    with pytest.raises(rk.RKError):
        ctx.rk_poll_status()


def test_argument_errors(rk, ctx):
    pool = Pool(rk, [3], seed=9)
    c = torch.zeros((3, 520), dtype=torch.bfloat16, device="cuda")
    kr = torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")

    def status(fn, want):
        with pytest.raises(rk.RKError) as ei:
            fn()
        assert ei.value.status == want, str(ei.value)

    off = i32([0, 3])
    status(lambda: ctx.rk_cache4_append(pool.pages, pool.table, c[:, 1:513], kr, off), 5)         # misaligned base
    odd = torch.zeros((3, 515), dtype=torch.bfloat16, device="cuda")
    status(lambda: ctx.rk_cache4_append(pool.pages, pool.table, odd[:, :512], kr, off), 5)        # odd stride
    with pytest.raises(TypeError):
        ctx.rk_cache4_append(pool.pages, pool.table, c[:, :512].float(), kr, off)
    with pytest.raises(ValueError):
        ctx.rk_cache4_append(pool.pages, pool.table, c[:, :512], kr[:2], off)
    with pytest.raises(ValueError):
        ctx.rk_cache4_append(pool.pages, pool.table, c[:, :512], kr, i32([0, 1, 3]))
    with pytest.raises(ValueError):
        ctx.rk_cache4_append(pool.pages, pool.table, torch.zeros((3, 512, 1), dtype=torch.bfloat16, device="cuda")[..., 0].t().contiguous().t(), kr, off)
    plan = ctx.rk_decode_plan(pool.table, pool.n_pages, i32([0, 1]), i32([0]), i32([0]), i32([[2]]), max_tiles=1)
    q = torch.zeros((1, 1, 16, 576), dtype=torch.bfloat16, device="cuda")
    status(lambda: ctx.rk_cache4_attn(pool.pages, plan, q, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")), 6)
    with pytest.raises(ValueError):
        ctx.rk_cache4_attn(pool.pages, plan, q.expand(1, 2, 16, 576))
    small = rk.DecodePlan(plan.shape, plan.n_pages, plan.buf[:256])
    status(lambda: ctx.rk_cache4_attn(pool.pages, small, q), 6)
    status(lambda: ctx.rk_decode_plan(pool.table, pool.n_pages, i32([0, 1]), i32([0]), i32([0]), i32([[2]]), max_tiles=-1), 3)
    status(lambda: ctx.rk_decode_plan(pool.table, pool.n_pages, i32([0, 1]), i32([0]), i32([0]), i32([[2] * 65]), max_tiles=1), 3)
    phase = make_ctx(rk, value_phase=True)
    status(lambda: phase.rk_cache4_append(pool.pages, pool.table, c[:, :512], kr, off), 7)
    w = torch.zeros((1, 16, 128), dtype=torch.bfloat16, device="cuda")
    for bad, group in [(w, 16), (w[:, :, :64].contiguous(), 128), (torch.zeros((1, 8, 128), dtype=torch.bfloat16, device="cuda"), 32),
                       (torch.zeros((1, 16, 96), dtype=torch.bfloat16, device="cuda"), 32)]:
        status(lambda: ctx.rk_quant4(bad, group), 7)
    w4 = ctx.rk_quant4(w, 32)
    with pytest.raises(ValueError):
        ctx.rk_matvec4(w4, torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda"))
    status(lambda: ctx.rk_matvec4(w4, torch.zeros((1, 1, 136), dtype=torch.bfloat16, device="cuda")[..., 1:129]), 5)
    ctx.rk_poll_status()


# ------------------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------------------
def check_attention(ctx, pool, items, q_pos, q, O, lse, heads, sharp=False):
    """items: per request a list of (segment, delta)."""
    qh, oh, lh = f64(q), f64(O), lse.double().cpu().numpy()
    worst_num = worst_den = 0.0
    for b, mine in enumerate(items):
        ql = q_pos.shape[1]
        rows = qh[b].reshape(ql * heads, 576)
        pos = np.repeat(q_pos[b], heads)
        o, want_lse, mass, big, size = D.attention(rows, pos, [(pool.rows(s), d) for s, d in mine], SCALE, BASE)
        got_o, got_lse = oh[b].reshape(ql * heads, 512), lh[b].reshape(ql * heads)
        e = SCALE * (U * big + 48 * 2.0 ** -23 * size) + 1e-5
        tol = (U + np.exp(2 * e) - 1 + 1e-5)[:, None] * mass + U * np.abs(o)
        tol = tol + 2.0 ** -126 * (1 + sum(pool.lens[s] * np.abs(pool.rows(s)[:, :512]).max(initial=0.0) for s, _ in mine))
        assert np.isfinite(got_o).all(), b
        assert (np.abs(got_o - o) <= tol).all(), (b, float((np.abs(got_o - o) - tol).max()))
        none = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse), none), b
        assert (got_o[none] == 0).all()
        assert (np.abs(got_lse[~none] - want_lse[~none]) <= e[~none] + 1e-5).all(), b
        worst_num += ((got_o - o) ** 2).sum()
        worst_den += (o ** 2).sum()
    if worst_den > 0:
        assert np.sqrt(worst_num / worst_den) <= REL_L2


def plan_for(ctx, pool, items, q_pos, max_tiles=None, **kw):
    seq_off = np.concatenate([[0], np.cumsum([len(m) for m in items])])
    if max_tiles is None:
        max_tiles = sum((pool.lens[s] + 127) // 128 for m in items for s, _ in m)
    return ctx.rk_decode_plan(pool.table, pool.n_pages, i32(seq_off), i32([s for m in items for s, _ in m] or np.zeros(0)),
                              i32([d for m in items for _, d in m] or np.zeros(0)), i32(q_pos), max_tiles=max_tiles, **kw)


def run_attention(ctx, pool, items, q_pos, heads, seed, q_std=1.2, q=None):
    q_pos = np.asarray(q_pos)
    rng = np.random.default_rng(seed + 77)
    if q is None:
        q = bf(rng.standard_normal((len(items), q_pos.shape[1], heads, 576)) * q_std)
    plan = plan_for(ctx, pool, items, q_pos)
    O, lse = ctx.rk_cache4_attn(pool.pages, plan, q)
    ctx.rk_poll_status()
    check_attention(ctx, pool, items, q_pos, q, O, lse, heads)
    return plan, q, O, lse


def chain(lens, segs, start=0):
    """Segments one behind the other in the request: [(segment, delta)], end position."""
    out, run = [], start
    for s in segs:
        out.append((s, run))
        run += lens[s]
    return out, run


@pytest.mark.parametrize("heads", [8, 16, 24, 64, 72, 128])
@pytest.mark.parametrize("q_len", [1, 2, 3])
def test_attention_heads_and_tokens(rk, heads, q_len):
    ctx = make_ctx(rk, heads)
    lens = [130, 64, 200, 7, 65]
    pool = Pool(rk, lens, seed=heads)
    fill_pool(ctx, pool, heads)
    items, pos = [], []
    for segs in ([0, 3], [2, 1, 4], [4]):
        it, end = chain(lens, segs)
        items.append(it)
        pos.append([end - q_len + t for t in range(q_len)])
    run_attention(ctx, pool, items, pos, heads, heads + q_len)


@pytest.mark.parametrize("heads, q_len", [(24, 17), (8, 64), (128, 64)])
def test_attention_many_drafted_tokens(rk, heads, q_len):
    """Many row tiles per request, the last one short; every token has its own mask, the first ones see only the document."""
    ctx = make_ctx(rk, heads)
    lens = [150, q_len + 3, 2]
    pool = Pool(rk, lens, seed=61)
    fill_pool(ctx, pool, 61)
    items = [[(0, 0), (1, 150)], [(2, 0)]]
    q_pos = np.array([np.arange(q_len) + 150 - 2, np.arange(q_len) - 1])
    run_attention(ctx, pool, items, q_pos, heads, 62)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257, 1000])
def test_attention_lengths(rk, ctx, n):
    """One segment of n rows, seen whole, all but the last, one row only, not at all; the rest of its pages is NaN."""
    pool = Pool(rk, [n], seed=n)
    fill_pool(ctx, pool, n)
    items = [[(0, 0)], [(0, 0)], [(0, 0)], [(0, 0)], [], [(0, 5)]]
    run_attention(ctx, pool, items, [[n - 1], [n - 2], [0], [-1], [10], [5 + n // 2]], 16, n)


def test_attention_many_segments_shared_documents_and_gaps(rk, ctx):
    rng = np.random.default_rng(11)
    lens = [int(x) for x in rng.choice([1, 2, 63, 64, 65, 127, 128, 129, 300, 515], size=30)]
    pool = Pool(rk, lens, seed=12)
    fill_pool(ctx, pool, 12)
    items, pos = [], []
    for b in range(9):
        segs = rng.permutation(30)[:int(rng.integers(1, 20))].tolist()
        run, mine = int(rng.integers(0, 1 << 20)), []
        for s in segs:
            mine.append((s, run))
            run += lens[s] + int(rng.integers(0, 40))
        items.append(mine)
        pos.append([run - int(rng.integers(1, 400)), run + 3])
    run_attention(ctx, pool, items, pos, 16, 13)


@pytest.mark.parametrize("heads, seqs, length", [(64, 1, 40000), (16, 5, 9000), (128, 3, 5000), (64, 40, 700)])
def test_attention_split_over_many_ctas(rk, heads, seqs, length):
    ctx = make_ctx(rk, heads)
    rng = np.random.default_rng(heads + seqs)
    lens = [int(length - rng.integers(0, 100)) for _ in range(seqs)]
    pool = Pool(rk, lens, seed=14)
    fill_pool(ctx, pool, 14)
    run_attention(ctx, pool, [[(b, 3 * b)] for b in range(seqs)], [[3 * b + lens[b] - 1] for b in range(seqs)], heads, 15)


def test_attention_rising_scores_take_the_rescale_path(rk, ctx):
    """Keys whose scores grow from tile to tile by more than 2^8, then fall again: every raise of the maximum, and a
    later tile that must not raise it; one head sees the order reversed."""
    n = 128 * 7 + 50
    rng = np.random.default_rng(16)
    c = rng.standard_normal((n, 512)) * 0.05
    level = np.array([0, 10, 30, 90, 60, 200, 5, 1])[np.arange(n) // 128]
    c[:, 0] = level
    pool = Pool(rk, [n], seed=16)
    fill_pool(ctx, pool, 16, c=c)
    q = rng.standard_normal((1, 2, 16, 576)) * 0.1
    q[0, :, :, 0] = np.linspace(-16, 16, 16)[None]
    run_attention(ctx, pool, [[(0, 0)]], [[n - 2, n - 1]], 16, 17, q=bf(q))
    pool64 = Pool(rk, [n * 40], seed=16)                         # the same inside one CTA's long run of tiles
    big = np.tile(c, (40, 1))
    fill_pool(ctx, pool64, 16, c=big)
    run_attention(ctx, pool64, [[(0, 0)]], [[n * 40 - 2, n * 40 - 1]], 16, 17, q=bf(q))


def test_attention_uniform_scores_and_large_scores(rk, ctx):
    pool = Pool(rk, [300], seed=18)
    fill_pool(ctx, pool, 18)
    zero = torch.zeros((1, 1, 16, 576), dtype=torch.bfloat16, device="cuda")
    _, _, O, lse = run_attention(ctx, pool, [[(0, 0)]], [[299]], 16, 18, q=zero)
    assert np.allclose(lse.cpu().numpy(), np.log(300.0), atol=1e-5)
    run_attention(ctx, pool, [[(0, 0)]], [[299]], 16, 18, q_std=40.0)     # near one-hot softmax
    run_attention(ctx, pool, [[(0, 0)]], [[299]], 16, 18, q_std=1e-20)


@pytest.mark.parametrize("heads, n, bad", [(16, 2, "c"), (16, 130, "c"), (64, 130, "rope"), (24, 129, "inf c"), (64, 9000, "c"),
                                           (128, 9000, "rope")])
def test_attention_bad_key_reaches_only_the_tokens_that_see_it(rk, heads, n, bad):
    """The last cached row has a non-finite value.  The last query token sees it and is NaN in every head; the token before it
    and the other request, which ends a row earlier, are what they are without that row."""
    ctx = make_ctx(rk, heads)
    pool = Pool(rk, [n], seed=31)
    rng = np.random.default_rng(32)
    c, kr = rng.standard_normal((n, 512)), rng.standard_normal((n, 64))
    if bad == "rope":
        kr[n - 1, 2:4] = np.nan
    else:
        c[n - 1, 200] = np.nan if bad == "c" else np.inf
    ctx.rk_cache4_append(pool.pages, pool.table, bf(c), bf(kr), i32([0, n]))
    pool.from_device()
    items, q_pos = [[(0, 0)], [(0, 0)]], np.array([[n - 2, n - 1], [n - 3, n - 2]])
    q = bf(rng.standard_normal((2, 2, heads, 576)) * 1.2)
    O, lse = ctx.rk_cache4_attn(pool.pages, plan_for(ctx, pool, items, q_pos), q)
    ctx.rk_poll_status()
    assert torch.isnan(O[0, 1]).all() and torch.isnan(lse[0, 1]).all()
    pool.lens = [n - 1]                                            # the oracle does not see the row either
    check_attention(ctx, pool, [items[0]], q_pos[:1, :1], q[:1, :1], O[:1, :1], lse[:1, :1], heads)
    check_attention(ctx, pool, [items[1]], q_pos[1:], q[1:], O[1:], lse[1:], heads)


def test_attention_long_offsets_in_a_large_pool(rk, ctx):
    """Pages beyond 4 GiB into the pool, segments at large request offsets."""
    n_pages = (9 << 29) // D.PAGE_BYTES
    pages = torch.empty((n_pages, D.PAGE_BYTES), dtype=torch.uint8, device="cuda")
    lens = [200, 130]
    pool = Pool(rk, lens, seed=19)
    ids = np.array([n_pages - 1, n_pages - 9, 3, n_pages - 2, n_pages // 2, 0, 1])[:len(pool.ids)]
    ids = np.concatenate([ids, np.arange(10, 10 + len(pool.ids) - len(ids))]).astype(np.int64)
    rng = np.random.default_rng(20)
    c, kr = bf(rng.standard_normal((330, 512))), bf(rng.standard_normal((330, 64)))
    table = rk.CacheTable(i32(lens), i32(pool.off), i32(ids))
    ctx.rk_cache4_append(pages, table, c, kr, i32([0, 200, 330]))
    back = ctx.rk_cache4_read(pages, table, i32([0, 200, 330]), 330)
    q = bf(rng.standard_normal((1, 1, 16, 576)))
    d = (1 << 30) - 1000
    plan = ctx.rk_decode_plan(table, n_pages, i32([0, 2]), i32([0, 1]), i32([0, d]), i32([[d + 129]]), max_tiles=4)
    O, lse = ctx.rk_cache4_attn(pages, plan, q)
    ctx.rk_poll_status()
    rows = f64(back)
    want, wl, mass, big, size = D.attention(f64(q)[0, 0], np.full(16, d + 129), [(rows[:200], 0), (rows[200:], d)], SCALE, BASE)
    codes, byte = D.quantise_latent(f64(c))
    assert np.array_equal(rows[:, :512], D.latent_values(codes, byte))
    e = SCALE * (U * big + 48 * 2.0 ** -23 * size) + 1e-5
    assert (np.abs(f64(O)[0, 0] - want) <= (U + np.exp(2 * e) - 1 + 1e-5)[:, None] * mass + U * np.abs(want)).all()
    assert (np.abs(lse.double().cpu().numpy()[0, 0] - wl) <= e + 1e-5).all()


def test_attention_repeats_bit_for_bit_and_leaves_other_rows(rk):
    ctx = make_ctx(rk, 64)
    lens = [3000, 1, 777]
    pool = Pool(rk, lens, seed=21)
    fill_pool(ctx, pool, 21)
    items, pos = [[(0, 0), (2, 3000)], [(1, 0)], [(0, 100)]], np.array([[3776], [0], [3099]])
    plan, q, O, lse = run_attention(ctx, pool, items, pos, 64, 22)
    for _ in range(3):
        O2, lse2 = ctx.rk_cache4_attn(pool.pages, plan, q)
        assert torch.equal(O, O2) and torch.equal(lse, lse2)
    # a request's result does not depend on what stands beside it, up to the split of its keys
    big_o = torch.full((5, 1, 64, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    big_l = torch.full((5, 1, 64), 7.0, dtype=torch.float32, device="cuda")
    ctx.rk_cache4_attn(pool.pages, plan, q, O=big_o[1:4], lse=big_l[1:4])
    assert torch.equal(big_o[1:4], O) and (big_o[0] == 7).all() and (big_o[4] == 7).all()
    assert (big_l[0] == 7).all() and (big_l[4] == 7).all()


def test_captured_step_follows_the_tables(rk, ctx):
    """Append, plan and attention in one CUDA graph on a side stream: replayed after lengths, positions and rows changed."""
    cap = 400
    lens = [150, 260]
    pool = Pool(rk, [cap, cap], seed=23)
    fill_pool(ctx, pool, 23)
    seg_len = pool.table.seg_len
    rng = np.random.default_rng(24)
    c, kr = bf(rng.standard_normal((2, 512))), bf(rng.standard_normal((2, 64)))
    q = bf(rng.standard_normal((2, 1, 16, 576)))
    new_off, seq_off = i32([0, 1, 2]), i32([0, 2, 3])
    item_seg, item_delta, q_pos = i32([0, 1, 1]), i32([0, 0, 7]), i32([[0], [0]])
    O = torch.empty((2, 1, 16, 512), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((2, 1, 16), dtype=torch.float32, device="cuda")

    def set_step(n0, n1, delta1):
        seg_len.copy_(i32([n0, n1]))
        item_delta.copy_(i32([0, delta1, 7]))
        q_pos.copy_(i32([[delta1 + n1 - 1], [7 + n1 - 1]]))

    def step(plan=None):
        ctx.rk_cache4_append(pool.pages, pool.table, c, kr, new_off)
        plan = ctx.rk_decode_plan(pool.table, pool.n_pages, seq_off, item_seg, item_delta, q_pos, max_tiles=12, plan=plan)
        ctx.rk_cache4_attn(pool.pages, plan, q, O=O, lse=lse, workspace=ws)
        return plan

    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    set_step(lens[0], lens[1], lens[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan = step()
    torch.cuda.current_stream().wait_stream(side)
    ctx.rk_poll_status()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(plan)
    for n0, n1 in [(150, 260), (151, 261), (192, 300), (400, 1), (1, 400)]:
        set_step(n0, n1, n0 + 3)
        c.copy_(bf(rng.standard_normal((2, 512))))
        q.copy_(bf(rng.standard_normal((2, 1, 16, 576))))
        graph.replay()
        ctx.rk_poll_status()
        pool.from_device()
        pool.lens = [n0, n1]
        codes, byte = D.quantise_latent(f64(c))
        assert np.array_equal(pool.rows(0)[-1, :512], D.latent_values(codes, byte)[0])
        check_attention(ctx, pool, [[(0, 0), (1, n0 + 3)], [(1, 7)]], np.array([[n0 + 3 + n1 - 1], [7 + n1 - 1]]), q, O, lse, 16)


def test_two_streams_at_once_share_the_plan(rk, ctx):
    lens = [2000, 900]
    pool = Pool(rk, lens, seed=25)
    fill_pool(ctx, pool, 25)
    items, pos = [[(0, 0), (1, 2000)]], np.array([[2899]])
    plan, q, O, lse = run_attention(ctx, pool, items, pos, 16, 26)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            outs.append([ctx.rk_cache4_attn(pool.pages, plan, q) for _ in range(4)])
    torch.cuda.synchronize()
    for mine in outs:
        for o2, l2 in mine:
            assert torch.equal(o2, O) and torch.equal(l2, lse)


def test_plan_errors_are_reported(rk, ctx):
    lens = [300, 64]
    pool = Pool(rk, lens, seed=27)
    fill_pool(ctx, pool, 27)
    q = torch.zeros((1, 1, 16, 576), dtype=torch.bfloat16, device="cuda")

    def poll(want):
        with pytest.raises(rk.RKError) as ei:
            ctx.rk_poll_status()
        assert ei.value.status == want, str(ei.value)
        ctx.rk_poll_status()

    # too many tiles: an empty plan; the rows come back as rows that see nothing
    plan = plan_for(ctx, pool, [[(0, 0)]], [[299]], max_tiles=2)
    poll(6)
    O, lse = ctx.rk_cache4_attn(pool.pages, plan, q)
    ctx.rk_poll_status()
    assert (O == 0).all() and torch.isneginf(lse).all()
    # an item without a segment, with a negative offset, with too few pages: left out, the others stand
    for seg, delta in [(2, 0), (-1, 0), (0, -5)]:
        plan = plan_for(ctx, pool, [[(1, 0)]], [[63]])
        want = ctx.rk_cache4_attn(pool.pages, plan, q)
        plan = ctx.rk_decode_plan(pool.table, pool.n_pages, i32([0, 2]), i32([seg, 1]), i32([delta, 0]), i32([[63]]), max_tiles=4)
        poll(4)
        got = ctx.rk_cache4_attn(pool.pages, plan, q)
        ctx.rk_poll_status()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    short = rk.CacheTable(i32([300, 64]), i32([0, 2, 3]), i32(pool.ids[:3]))
    ctx.rk_decode_plan(short, pool.n_pages, i32([0, 1]), i32([0]), i32([0]), i32([[299]]), max_tiles=4)
    poll(4)
    bad_page = rk.CacheTable(i32([300, 64]), i32(pool.off), i32([99] + pool.ids[1:].tolist()))
    plan = ctx.rk_decode_plan(bad_page, pool.n_pages, i32([0, 1]), i32([0]), i32([0]), i32([[299]]), max_tiles=4)
    poll(4)
    O, lse = ctx.rk_cache4_attn(pool.pages, plan, q)            # the tile with the bad page counts as unseen
    ctx.rk_poll_status()
    assert np.allclose(lse.cpu().numpy(), np.log(300 - 128), atol=1e-5)
    bad_off = ctx.rk_decode_plan(pool.table, pool.n_pages, i32([0, 5]), i32([0]), i32([0]), i32([[299]]), max_tiles=4)
    poll(4)
    O, lse = ctx.rk_cache4_attn(pool.pages, bad_off, q)
    assert torch.isneginf(lse).all()
    # a plan of another shape, of another pool, or no plan at all
    plan = plan_for(ctx, pool, [[(0, 0)]], [[299]])
    O = torch.full((1, 1, 16, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    for wrong in (rk.DecodePlan(plan.shape, plan.n_pages, torch.zeros_like(plan.buf)),
                  rk.DecodePlan(rk.rk_decode_shape(1, 1, 1, 2), plan.n_pages, plan.buf)):
        ctx.rk_cache4_attn(pool.pages, wrong, q, O=O)
        poll(3)
        assert (O == 7).all()
    ctx.rk_cache4_attn(pool.pages[:-1], plan, q, O=O)
    poll(3)
    other = make_ctx(rk, 64)
    other.rk_cache4_attn(pool.pages, plan, torch.zeros((1, 1, 64, 576), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(rk.RKError) as ei:
        other.rk_poll_status()
    assert ei.value.status == 3


@pytest.mark.parametrize("far", [2 ** 30 - 1, 2 ** 30, 2 ** 31 - 1])
def test_positions_far_behind_the_last_key(rk, ctx, far):
    """A token at the largest positions sees every key and nothing else (the pages hold NaN behind the last one)."""
    pool = Pool(rk, [130, 65], seed=51)
    fill_pool(ctx, pool, 51)
    items = [[(0, 0), (1, 130)]]
    run_attention(ctx, pool, items, [[194]], 16, 52)
    _, _, O, lse = run_attention(ctx, pool, items, [[far]], 16, 52)
    _, _, near, near_lse = run_attention(ctx, pool, items, [[194]], 16, 52)
    assert torch.equal(O, near) and torch.equal(lse, near_lse)


def test_pool_without_pages(rk, ctx):
    """Tables that name rows of a pool without pages: reported, no tile is made, the rows see nothing."""
    table = rk.CacheTable(i32([100]), i32([0, 2]), i32([0, 1]))
    pages = torch.empty((0, D.PAGE_BYTES), dtype=torch.uint8, device="cuda")
    plan = ctx.rk_decode_plan(table, 0, i32([0, 1]), i32([0]), i32([0]), i32([[99]]), max_tiles=1)
    with pytest.raises(rk.RKError) as ei:
        ctx.rk_poll_status()
    assert ei.value.status == 4
    q = torch.ones((1, 1, 16, 576), dtype=torch.bfloat16, device="cuda")
    O, lse = ctx.rk_cache4_attn(pages, plan, q)
    ctx.rk_poll_status()
    assert (O == 0).all() and torch.isneginf(lse).all()
    empty = rk.CacheTable(i32([0]), i32([0, 0]), torch.empty(0, dtype=torch.int32, device="cuda"))
    plan = ctx.rk_decode_plan(empty, 0, i32([0, 1]), i32([0]), i32([0]), i32([[0]]), max_tiles=1)
    O, lse = ctx.rk_cache4_attn(pages, plan, q)
    ctx.rk_poll_status()
    assert (O == 0).all() and torch.isneginf(lse).all()


def test_decode_agrees_with_the_online_attention_on_the_same_rows(rk):
    """The last query token of an online request, and the same token over the cache: both attend the same rows."""
    from paper_2609_07008_b200 import synth
    w = synth.make_custom([300, 77, 513], 50, n_heads=16, n_groups=2, o_rank=256, d_model=512, pct_bp=700, seed=21)
    ctx = rk.Context.from_profile(w.profile)
    lens = np.diff(w.layout.seg_off).tolist()
    pool = Pool(rk, lens, seed=28)
    n = sum(lens)
    raw = f64(w.kv)
    ctx.rk_cache4_append(pool.pages, pool.table, w.kv[:, :512].cuda(), w.kv[:, 512:].cuda(), i32(w.layout.seg_off))
    kv = ctx.rk_cache4_read(pool.pages, pool.table, i32(w.layout.seg_off), n)
    req = ctx.rk_request_create(w.layout.seg_off, w.layout.seg_delta, w.layout.seg_has_artifact, w.prot_rows)
    q_l, q_g = w.q_l.cuda(), w.q_g.cuda()
    O_g, lse_g, O_l, lse_l = ctx.rk_mla_online_attn(req, kv, q_g, q_l)
    last = n - 1
    q = torch.empty((1, 1, 16, 576), dtype=torch.bfloat16, device="cuda")
    gh, lh = torch.from_numpy(w.profile.global_heads).long().cuda(), torch.from_numpy(w.profile.local_heads).long().cuda()
    q[0, 0, gh] = q_g[last]
    q[0, 0, lh] = q_l[-1]
    end = int(w.layout.seg_delta[-1]) + lens[-1] - 1
    plan = plan_for(ctx, pool, [[(s, int(d)) for s, d in enumerate(w.layout.seg_delta)]], [[end]])
    O, lse = ctx.rk_cache4_attn(pool.pages, plan, q)
    ctx.rk_poll_status()
    for got, want in ((O[0, 0, gh], O_g[last]), (O[0, 0, lh], O_l[-1])):
        assert rel_l2(f64(got), f64(want)) <= REL_L2
    assert (lse[0, 0, gh] - lse_g[last]).abs().max() < 5e-3 and (lse[0, 0, lh] - lse_l[-1]).abs().max() < 5e-3


# ------------------------------------------------------------------------------------------------------------
# 4-bit weights
# ------------------------------------------------------------------------------------------------------------
def check_matvec(got, x, vals, k, bf16):
    """x [t, m, k], vals [m, n, k] float64."""
    want = np.einsum("tmk,mnk->tmn", x, vals)
    mass = np.einsum("tmk,mnk->tmn", np.abs(x), np.abs(vals))
    tol = (k / 64 + 40) * 2.0 ** -23 * mass + (U * np.abs(want) if bf16 else 0.0)
    assert (np.abs(f64(got) - want) <= tol).all(), float((np.abs(f64(got) - want) - tol).max())


@pytest.mark.parametrize("tok", [1, 2, 7, 8, 9, 15, 16, 17, 40])
@pytest.mark.parametrize("mats, n_out, k, group", [(1, 16, 64, 32), (3, 48, 128, 128), (2, 80, 1024, 64), (1, 272, 640, 32),
                                                   (5, 128, 512, 128)])
def test_matvec_matches_oracle(rk, ctx, mats, n_out, k, group, tok):
    rng = np.random.default_rng(k + tok)
    w = bf(rng.standard_normal((mats, n_out, k)) * 0.02)
    vals = D.quantise_weights(f64(w), group)
    w4 = ctx.rk_quant4(w, group)
    wide = bf(rng.standard_normal((tok, mats * k + 8)))
    x = wide[:, :mats * k].unflatten(1, (mats, k))                # token stride wider than a token
    xs = f64(x)
    check_matvec(ctx.rk_matvec4(w4, x), xs, vals, k, True)
    check_matvec(ctx.rk_matvec4(w4, x.contiguous(), out_dtype=torch.float32), xs, vals, k, False)
    y = torch.full((tok, mats * n_out + 3), 7.0, dtype=torch.float32, device="cuda")
    ctx.rk_matvec4(w4, x, y=y[:, :mats * n_out].unflatten(1, (mats, n_out)))
    check_matvec(y[:, :mats * n_out].unflatten(1, (mats, n_out)), xs, vals, k, False)
    assert (y[:, mats * n_out:] == 7).all()
    ctx.rk_poll_status()


@pytest.mark.parametrize("mats, n_out, k, group, tok", [
    (1, 80, 4096, 32, 3), (2, 48, 4160, 64, 9), (1, 32, 8320, 128, 16), (3, 16, 16384, 64, 1), (1, 48, 17024, 128, 5),
    (1, 16, 33088, 64, 17), (1, 5120, 2112, 64, 12), (1, 9600, 128, 128, 4), (40, 256, 192, 32, 2), (1, 13000 // 16 * 16, 2112, 32, 8)])
def test_matvec_long_rows_and_many_rows(rk, ctx, mats, n_out, k, group, tok):
    """k over two, four and eight thread blocks and over several rounds of them, with ragged and empty last slices; several tiles
    of output rows per thread block, with a short last run."""
    rng = np.random.default_rng(n_out + k)
    w = bf(rng.standard_normal((mats, n_out, k)) * 0.02)
    vals = D.quantise_weights(f64(w), group)
    x = bf(rng.standard_normal((tok, mats, k)))
    w4 = ctx.rk_quant4(w, group)
    y = ctx.rk_matvec4(w4, x, out_dtype=torch.float32)
    check_matvec(y, f64(x), vals, k, False)
    assert torch.equal(ctx.rk_matvec4(w4, x, out_dtype=torch.float32), y)
    ctx.rk_poll_status()


def test_matvec_bad_token_stays_alone(rk, ctx):
    """A token with an infinity and one with a NaN, in the first and in the last block of k: the others are untouched."""
    rng = np.random.default_rng(41)
    w = bf(rng.standard_normal((1, 48, 4160)) * 0.02)
    w4 = ctx.rk_quant4(w, 64)
    x = bf(rng.standard_normal((11, 1, 4160)))
    want = ctx.rk_matvec4(w4, x)
    x[2, 0, 4159], x[9, 0, 0] = float("inf"), float("nan")
    y = ctx.rk_matvec4(w4, x)
    good = [t for t in range(11) if t not in (2, 9)]
    assert torch.equal(y[good], want[good])
    assert not torch.isfinite(y[2]).any() and torch.isnan(y[9]).all()
    ctx.rk_poll_status()


def test_weight_codes_at_ties_zeros_and_non_finite_values(rk, ctx):
    w = np.zeros((1, 32, 128))
    w[0, 0] = np.tile(np.arange(-14, 18)[:32] * 0.5, 4)
    w[0, 0, ::32] = 7.0                                            # scale 1: halves sit on ties
    w[0, 1, :32] = np.random.default_rng(0).standard_normal(32) * 1e-30
    w[0, 2] = np.random.default_rng(1).standard_normal(128) * 1e30
    w[0, 4] = np.random.default_rng(2).standard_normal(128)
    w[0, 4, 40] = np.inf
    w[0, 20, 127] = np.nan
    wt = bf(w)
    vals = D.quantise_weights(np.where(np.isfinite(f64(wt)), f64(wt), 0.0), 32)
    w4 = ctx.rk_quant4(wt, 32)
    eye = torch.zeros((128, 1, 128), dtype=torch.bfloat16, device="cuda")
    eye[torch.arange(128), 0, torch.arange(128)] = 1.0
    got = f64(ctx.rk_matvec4(w4, eye, out_dtype=torch.float32))[:, 0].T   # column by column: the values themselves
    rows = [r for r in range(32) if r not in (4, 20)]
    assert np.array_equal(got[rows], vals[0][rows])
    assert np.isnan(got[4]).all() and np.isnan(got[20]).all()       # a NaN scale makes the row's outputs NaN
    ctx.rk_poll_status()


def test_matvec_without_tokens_and_repeats_bit_for_bit(rk, ctx):
    w = bf(np.random.default_rng(3).standard_normal((1, 512, 2048)))
    w4 = ctx.rk_quant4(w, 128)
    assert ctx.rk_matvec4(w4, torch.empty((0, 1, 2048), dtype=torch.bfloat16, device="cuda")).shape == (0, 1, 512)
    x = bf(np.random.default_rng(4).standard_normal((5, 1, 2048)))
    y = ctx.rk_matvec4(w4, x)
    for _ in range(3):
        assert torch.equal(ctx.rk_matvec4(w4, x), y)
    # a token's result does not depend on its neighbours in the same kernel form
    assert torch.equal(ctx.rk_matvec4(w4, x[2:3]), y[2:3])


# ------------------------------------------------------------------------------------------------------------
# a decode step, as it would be used
# ------------------------------------------------------------------------------------------------------------
def test_decode_steps_over_reused_documents(rk):
    """Two requests over three cached documents generate four tokens: append, plan, attention, W_uv, W_a, W_b in
    4 bits.  Each stage is checked against the oracle on that stage's own input."""
    ctx = make_ctx(rk, 16)
    rng = np.random.default_rng(30)
    docs = [200, 333, 64]
    cap = 70
    pool = Pool(rk, docs + [cap, cap], seed=31)
    lens = pool.table.seg_len
    lens.copy_(i32(docs + [0, 0]))
    n = sum(docs)
    ctx.rk_cache4_append(pool.pages, pool.table, bf(rng.standard_normal((n, 512))), bf(rng.standard_normal((n, 64))),
                         i32(np.concatenate([[0], np.cumsum(docs), [n, n]])))
    w = {"uv": bf(rng.standard_normal((16, 128, 512)) * 0.05), "a": bf(rng.standard_normal((2, 256, 1024)) * 0.05),
         "b": bf(rng.standard_normal((1, 1024, 512)) * 0.05)}
    w4 = {k: ctx.rk_quant4(v, g) for (k, v), g in zip(w.items(), (64, 128, 32))}
    vals = {k: D.quantise_weights(f64(v), g) for (k, v), g in zip(w.items(), (64, 128, 32))}
    items = [[(0, 0), (2, 200), (3, 264)], [(1, 0), (0, 333), (4, 540)]]
    plan = None
    for step in range(1, 5):
        lens.copy_(i32(docs + [step, step]))
        ctx.rk_cache4_append(pool.pages, pool.table, bf(rng.standard_normal((2, 512))), bf(rng.standard_normal((2, 64))),
                             i32([0, 0, 0, 0, 1, 2]))
        pos = np.array([[264 + step - 1], [540 + step - 1]])
        plan = plan_for(ctx, pool, items, pos, max_tiles=16, plan=plan)
        q = bf(rng.standard_normal((2, 1, 16, 576)))
        O, lse = ctx.rk_cache4_attn(pool.pages, plan, q)
        o = ctx.rk_matvec4(w4["uv"], O.view(2, 16, 512))
        z = ctx.rk_matvec4(w4["a"], o.view(2, 2, 1024))
        y = ctx.rk_matvec4(w4["b"], z.view(2, 1, 512))
        ctx.rk_poll_status()
        pool.from_device()
        pool.lens = docs + [step, step]
        check_attention(ctx, pool, items, pos, q, O, lse, 16)
        check_matvec(o, f64(O.view(2, 16, 512)), vals["uv"], 512, True)
        check_matvec(z, f64(o.view(2, 2, 1024)), vals["a"], 1024, True)
        check_matvec(y, f64(z.view(2, 1, 512)), vals["b"], 512, True)
        assert y.shape == (2, 1, 1024)
