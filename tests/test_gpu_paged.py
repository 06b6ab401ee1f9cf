"""GPU parity of the paged cache's operators against oracle/paged.py (64 bits), through the C ABI.

Tolerances, derived, not fitted.  A rounding to bf16 is off by at most 2^-8 relative, one to float by 2^-24.
  rotation   two products and a sum in float, rounded once: 2^-8 |x| (bf16) or 2^-24 |x|, + 3 * 2^-24 (|a c| + |b s|).
  attention  out = sum_j p_j v_j / sum_j p_j.  A score is off by delta <= (dim + 16) * 2^-24 * top, where `top` bounds what its terms
             add up to in magnitude (dim products summed in float; scaling, bias and the change to units of ln 2 in the 16; the
             fast tanh of bf16 calls adds softcap * 2^-21), so every probability by a factor within exp(2 delta) of 1; sums over n
             keys in float by n * 2^-24; bf16 probabilities as one term by 2^-8.  All of these weigh sum_j p_j |v_j| = mass, and
             the final rounding |out|.
"""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2604_17701_amd import binding
from parity import record
from wisv_inputs import configs, gen

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    w = configs.get(0)
    c = binding.Context(w.model, gen.make_weights(w.model, w.seed, DEV), 1, 32, 1)
    yield c
    c.wisv_destroy()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def f64(t):
    return t.detach().cpu().double().numpy()


def normal(seed, shape, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


# ------------------------------------------------------------------------------------------------ the plan

def check_plan(ctx, cached, new, free, table, page, max_tokens):
    want = ref.plan(cached, new, free, table, page, max_tokens)
    dev = ints(table)
    got = ctx.wisv_paged_plan(ints(cached), ints(new), ints(free).reshape(-1), dev, page, max_tokens)
    for name, g, w in zip(binding.PagePlan._fields + ("block_table",), tuple(got) + (dev,), want):
        assert g.cpu().numpy().tolist() == w.tolist(), name
    return want


@pytest.mark.parametrize("batch,page,hi_cached,hi_new", [(1, 16, 40, 1), (1, 32, 1, 300), (7, 16, 90, 9), (64, 64, 900, 70), (255, 16, 200, 3),
                                                         (256, 128, 3000, 200), (257, 256, 2000, 40), (1023, 16, 64, 33), (4096, 32, 100, 5)])
def test_plan_matches_the_oracle(ctx, batch, page, hi_cached, hi_new):
    rng = np.random.default_rng(batch + page)
    cached, new = rng.integers(0, hi_cached + 1, batch), rng.integers(0, hi_new + 1, batch)
    table, n = ref.pages_of(list(cached), page, rng)
    need = int(sum(-(-(c + m) // page) - -(-c // page) for c, m in zip(cached, new)))
    wide = np.full((batch, -(-(hi_cached + hi_new) // page) + 1), -1, np.int32)
    wide[:, :table.shape[1]] = table
    total = int(new.sum())
    for n_free, tokens in ((need, max(total, 1)), (need + 9, total + 77), (need // 2, max(total, 1)), (need + 9, max(1, total * 2 // 3)), (0, total + 1)):
        want = check_plan(ctx, cached, new, n + rng.permutation(n_free), wide, page, tokens)
        if n_free >= need and tokens >= total:
            assert want[4][0] == need and not want[5].any()


def test_plan_edges(ctx):
    # idle requests, negative lengths, rows of the table that are full, an entry that is a hole
    t = [[3, 5, -1], [7, -1, -1], [2, 4, 6], [9, -1, -1], [-1, -1, -1], [-1, -1, -1]]
    for cached, new in (([0] * 6, [0] * 6), ([20, 1, 48, 5, 0, -3], [3, 40, 1, 0, 16, 17]), ([32, 16, 33, 0, 0, 0], [0, 1, 16, -5, 48, 49]),
                        ([20, 1, 40, 16, -1, 0], [1, 1, 1, 1, 1, 1]), ([17, 0, 0, 0, 0, 0], [1, 2 ** 31 - 1, 2 ** 31 - 1, 1, 1, 1])):
        for free in ([11, 12, 13, 14, 15, 16, 17, 18, 19, 20], [11, 12, 13], []):
            for tokens in (1, 30, 200):
                check_plan(ctx, cached, new, free, t, 16, tokens)


def test_plan_into_given_tensors_and_twice(ctx):
    cached, new = [5, 40, 0], [4, 1, 33]
    table, n = ref.pages_of(cached, 16)
    wide = np.full((3, 4), -1, np.int32)
    wide[:, :table.shape[1]] = table
    dev, free = ints(wide), ints(n + np.arange(6))
    first = ctx.wisv_paged_plan(ints(cached), ints(new), free, dev, 16, 50)
    again = ctx.wisv_paged_plan(ints(cached), ints(new), free, dev, 16, 50, out=binding.PagePlan(*[torch.full_like(x, -77) for x in first]))
    for x, y in zip(first, again):
        assert torch.equal(x, y)


# ------------------------------------------------------------------------------------------------ rotate and append

def pools(n_pages, g, page, dim, dtype, seed=5):
    return normal(seed, (n_pages, g, page, dim), dtype), normal(seed + 1, (n_pages, g, page // 8, dim, 8), dtype)


def check_append(ctx, dtype, dim, h, g, page, slots, n_pages, positions, rope=True, packed=True, in_place=False, layer=False):
    t, n_rope = len(slots), 50
    qkv = normal(3, (t, h + 2 * g + 1, dim), dtype)     # one head more than the rows need: rows lie apart
    q, k, v = (qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:h + 2 * g]) if packed else (x.clone() for x in (qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:h + 2 * g]))
    kp, vp = pools(3 * n_pages if layer else n_pages, g, page, dim, dtype)
    if layer:   # the second of three layers whose pages lie beside each other
        kp = kp.view(n_pages, 3, g, page, dim)[:, 1]
        vp = vp.view(n_pages, 3, g, page // 8, dim, 8)[:, 1]
    kp0, vp0, q0, k0, v0 = f64(kp), f64(vp), f64(q), f64(k), f64(v)
    ang = np.random.default_rng(1).uniform(-3, 3, (n_rope, dim // 2))
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    at = np.clip(positions, 0, n_rope - 1)
    got = ctx.wisv_paged_append(q if h else None, k, v, ints(positions) if rope else None, ints(slots), kp, vp, torch.from_numpy(cos).to(DEV) if rope else None,
                                torch.from_numpy(sin).to(DEV) if rope else None, q_out=q if in_place else None)
    eps = 2.0 ** -8 if dtype is BF16 else 2.0 ** -24

    def turned(x):
        return (ref.rotate(x, cos[at].astype(np.float64), sin[at].astype(np.float64)),
                ref.rotate(np.abs(x), np.abs(cos[at]).astype(np.float64), -np.abs(sin[at]).astype(np.float64))) if rope else (x, np.zeros_like(x))

    def near(a, want, terms):
        assert (np.abs(a - want) <= (eps * np.abs(want) + 3 * 2.0 ** -24 * np.abs(terms) if rope else 0.0)).all()

    # |a c| + |b s| for the first half of a head; the second half's terms pair up the same way
    if h:
        wq, _ = turned(q0)
        half = dim // 2
        c, s = (np.abs(cos[at])[:, None, :], np.abs(sin[at])[:, None, :])
        a, b = np.abs(q0[..., :half]), np.abs(q0[..., half:])
        near(f64(got), wq, np.concatenate([a * c + b * s, b * c + a * s], -1))
        assert (got.data_ptr() == q.data_ptr()) == in_place
    wk, _ = turned(k0)
    half = dim // 2
    c, s = (np.abs(cos[at])[:, None, :], np.abs(sin[at])[:, None, :])
    a, b = np.abs(k0[..., :half]), np.abs(k0[..., half:])
    terms = np.concatenate([a * c + b * s, b * c + a * s], -1)
    wkp, wvp, lim = kp0.copy(), vp0.copy(), np.zeros_like(kp0)
    ref.store(wkp, wvp, slots, wk, v0)
    ref.store(lim, np.zeros_like(vp0), slots, eps * np.abs(wk) + 3 * 2.0 ** -24 * terms if rope else np.zeros_like(wk), v0)
    assert (np.abs(f64(kp) - wkp) <= lim).all()           # places without a slot keep their bits
    assert np.array_equal(f64(vp), wvp)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim,h,g", [(32, 3, 1), (64, 4, 4), (128, 7, 1), (128, 32, 8), (256, 6, 2)])
@pytest.mark.parametrize("n,start", [(1, 0), (1, 13), (5, 14), (64, 0), (65, 3), (200, 7)])
def test_append_matches_the_oracle(ctx, dtype, dim, h, g, n, start):
    page = 16
    rng = np.random.default_rng(n + start)
    n_pages = -(-(start + n) // page) + 2
    order = rng.permutation(n_pages)
    pos = start + np.arange(n)
    check_append(ctx, dtype, dim, h, g, page, order[pos // page] * page + pos % page, n_pages, pos % 50)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kw", [dict(rope=False), dict(in_place=True), dict(packed=False), dict(layer=True), dict(layer=True, in_place=True)])
def test_append_forms(ctx, dtype, kw):
    rng = np.random.default_rng(3)
    # slots without order, some outside the pool, positions outside the tables
    slots = rng.permutation(6 * 32)[:90] - 5
    slots[::11] = -1
    slots[5::17] = 6 * 32 + np.arange(len(slots[5::17]))
    check_append(ctx, dtype, 64, 6, 2, 32, slots, 6, rng.integers(-3, 60, 90), **kw)


def test_append_without_queries(ctx):
    check_append(ctx, BF16, 128, 0, 2, 16, np.arange(20) + 9, 3, np.arange(20))


def test_append_of_nothing(ctx):
    kp, vp = pools(2, 1, 16, 64, BF16)
    k = torch.empty((0, 1, 64), dtype=BF16, device=DEV)
    none = ints(np.zeros(0))
    out = ctx.wisv_paged_append(torch.empty((0, 2, 64), dtype=BF16, device=DEV), k, k, none, none, kp, vp)
    assert out.shape == (0, 2, 64)


# ------------------------------------------------------------------------------------------------ attention

def setup(dtype, dim, h, g, page, lens, news, seed=1, q_std=2.0, spare_rows=0):
    rng = np.random.default_rng(seed)
    table, n_pages = ref.pages_of(list(lens), page, rng)
    kp, vp = pools(n_pages, g, page, dim, dtype, seed)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = normal(seed + 7, (int(starts[-1]) + spare_rows, h, dim), dtype, q_std)
    return q, kp, vp, table, starts


def limits(dtype, dim, keys, out, mass, top, softcap):
    bf = dtype is BF16
    delta = (dim + 16) * 2.0 ** -24 * top[..., None] + (softcap * 2.0 ** (-21 if bf else -22))
    rel = np.expm1(2 * delta) + (keys + 64) * 2.0 ** -24 + (2.0 ** -8 if bf else 0.0)
    return (2.0 ** -8 if bf else 2.0 ** -23) * np.abs(out) + rel * mass


def check_attention(ctx, q, kp, vp, table, starts, lens, slopes=None, prefix=None, **kw):
    hints = {"max_new": int(np.max(np.diff(starts))), "max_len": int(max(lens))}
    hints.update({k: kw.pop(k) for k in ("max_new", "max_len", "out", "workspace") if k in kw})
    got = ctx.wisv_paged_attention(q, kp, vp, ints(table), ints(starts), ints(lens), slopes=None if slopes is None else torch.tensor(slopes, dtype=F32, device=DEV),
                                   prefix_len=None if prefix is None else ints(prefix), **hints, **kw)
    out, mass, top = ref.attention(f64(q), f64(kp), f64(vp), table, starts, lens, slopes=None if slopes is None else np.float32(slopes), prefix=prefix, **kw)
    n = min(int(starts[-1]), q.shape[0])
    err = np.abs(f64(got)[:n] - out[:n])
    lim = limits(q.dtype, q.shape[2], max(1, int(max(lens))), out, mass, top, kw.get("softcap", 0.0))[:n]
    worst = np.max(err / np.maximum(lim, 1e-300), initial=0.0)
    assert (err <= lim).all(), worst
    return got, out


SHAPES = [(BF16, 128, 32, 8), (BF16, 128, 4, 4), (BF16, 64, 14, 2), (BF16, 32, 5, 1), (BF16, 256, 8, 2), (BF16, 128, 24, 1),
          (F32, 64, 4, 4), (F32, 128, 6, 2), (F32, 32, 9, 3), (F32, 256, 5, 1)]
BATCHES = [([1], [1]), ([16], [1]), ([17], [4]), ([33], [33]), ([500], [1]), ([1000], [8]), ([130], [70]),
           ([64, 1, 0, 31, 200, 90], [3, 1, 0, 31, 5, 60])]


@pytest.mark.parametrize("dtype,dim,h,g", SHAPES)
@pytest.mark.parametrize("lens,news", BATCHES)
def test_attention_matches_the_oracle(ctx, dtype, dim, h, g, lens, news):
    page = (16, 32, 64, 256)[(len(lens) + lens[0] + dim // 32) % 4]
    q, kp, vp, table, starts = setup(dtype, dim, h, g, page, lens, news)
    check_attention(ctx, q, kp, vp, table, starts, lens)


MODS = [dict(softcap=20.0), dict(window=1), dict(window=50), dict(slopes=True), dict(prefix=True), dict(scale=0.3),
        dict(softcap=5.0, window=33, slopes=True, prefix=True), dict(window=40, prefix=True), dict(scale=-0.1, slopes=True)]


@pytest.mark.parametrize("dtype,dim,h,g", [(BF16, 128, 8, 2), (BF16, 64, 7, 1), (BF16, 256, 4, 2), (BF16, 32, 4, 1), (F32, 64, 4, 2)])
@pytest.mark.parametrize("mods", MODS, ids=lambda m: "-".join(m))
@pytest.mark.parametrize("lens,news", [([200, 40, 1, 77], [1, 1, 1, 1]), ([300, 64, 0, 150, 20], [90, 64, 0, 7, 25])])
def test_attention_scores(ctx, dtype, dim, h, g, mods, lens, news):
    """Capped scores, distance bias, window, prefix and a scale, alone and together; new rows that begin before the cache
    (more of them than positions) see the prefix or nothing."""
    kw = dict(mods)
    if kw.pop("slopes", False):
        kw["slopes"] = 2.0 ** (-8.0 * np.arange(1, h + 1) / h)
    if kw.pop("prefix", False):
        kw["prefix"] = [5, 64, 3, 90, 1000][:len(lens)]
    q, kp, vp, table, starts = setup(dtype, dim, h, g, 32, lens, news)
    check_attention(ctx, q, kp, vp, table, starts, lens, **kw)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_rows_without_keys_is_zero(ctx, dtype):
    lens, news = [3, 0, 40], [9, 4, 40]        # six rows lie before the first position; a request without keys
    q, kp, vp, table, starts = setup(dtype, 64, 4, 2, 16, lens, news)
    got, out = check_attention(ctx, q, kp, vp, table, starts, lens)
    assert (f64(got)[:6] == 0).all() and (f64(got)[9:13] == 0).all() and (out[6:9] != 0).any()
    table[2, :] = -1                           # every page is a hole
    got, _ = check_attention(ctx, q, kp, vp, table, starts, lens)
    assert (f64(got)[13:] == 0).all()


@pytest.mark.parametrize("dtype,h", [(BF16, 4), (BF16, 32), (F32, 4)])
@pytest.mark.parametrize("news", [[1, 2, 1], [70, 30, 129]])
def test_attention_reads_nothing_that_it_should_not(ctx, dtype, h, news):
    """NaN and infinities everywhere but in the positions that requests hold: page ends, spare pages, holes."""
    lens, page = [100, 37, 130], 16
    q, kp, vp, table, starts = setup(dtype, 128, h, 4, page, lens, news)
    table[0, 2], table[2, 4], table[2, 5] = -1, 10 ** 6, -7
    clean, _ = check_attention(ctx, q, kp, vp, table, starts, lens)
    held = np.zeros((kp.shape[0], page), bool)
    for b, n in enumerate(lens):
        for j in range(n):
            if 0 <= table[b, j // page] < kp.shape[0]:
                held[table[b, j // page], j % page] = True
    bad = torch.from_numpy(~held).to(DEV)
    kp2 = torch.where(bad[:, None, :, None], torch.full_like(kp, float("nan")), kp)
    vb = bad.view(kp.shape[0], 1, page // 8, 1, 8)
    vp2 = torch.where(vb, torch.full_like(vp, float("inf")), vp)
    vp2[:, :, :, ::2] = torch.where(vb, torch.full_like(vp, float("nan")), vp)[:, :, :, ::2]
    dirty = ctx.wisv_paged_attention(q, kp2, vp2, ints(table), ints(starts), ints(lens), max_new=max(news), max_len=max(lens))
    assert torch.equal(clean, dirty)


@pytest.mark.parametrize("dtype,h", [(BF16, 4), (BF16, 32), (F32, 4)])
@pytest.mark.parametrize("window,prefix", [(0, None), (9, [3]), (0, [40])])
def test_attention_values_that_are_not_finite_reach_only_the_rows_that_see_them(ctx, dtype, h, window, prefix):
    lens, news, page = [90], [60], 32
    q, kp, vp, table, starts = setup(dtype, 64, h, 2, page, lens, news)
    kw = dict(window=window, prefix=prefix)

    def put(pool, pos, feature, x):
        pool[int(table[0, pos // page]), :, (pos % page) // 8, feature, pos % 8] = x

    bad = {50: (3, float("nan")), 64: (5, float("inf")), 77: (63, float("-inf")), 89: (0, float("nan"))}
    for pos, (feature, x) in bad.items():
        put(vp, pos, feature, x)
    got = f64(ctx.wisv_paged_attention(q, kp, vp, ints(table), ints(starts), ints(lens), max_new=60, max_len=90, window=window,
                                       prefix_len=None if prefix is None else ints(prefix)))
    out, mass, top = ref.attention(f64(q), f64(kp), f64(vp), table, starts, lens, **kw)
    fine = np.isfinite(out)
    assert 0 < (~fine).sum() < out.size // 2                   # some rows see such a value, in its feature alone
    # (a probability is two terms hi + lo, lo of either sign: hi inf + lo inf is no number where the formula says infinite)
    assert np.array_equal(np.isfinite(got), fine)
    assert (np.abs(got[fine] - out[fine]) <= limits(dtype, 64, 90, np.where(fine, out, 0.0), mass, top, 0.0)[fine]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hints", [dict(max_new=0, max_len=0), dict(max_new=1, max_len=1), dict(max_new=7, max_len=16), dict(max_new=10 ** 6, max_len=10 ** 9)])
def test_attention_hints_change_no_result_beyond_rounding(ctx, dtype, hints):
    lens, news = [400, 3, 250], [100, 1, 12]
    q, kp, vp, table, starts = setup(dtype, 128, 8, 2, 16, lens, news)
    check_attention(ctx, q, kp, vp, table, starts, lens, **hints)


@pytest.mark.parametrize("dtype,news", [(BF16, [1, 3]), (BF16, [40, 90]), (F32, [4, 30])])
def test_attention_leaves_the_rows_behind_the_last_request(ctx, dtype, news):
    """Rows behind the last request keep their bits in `out`, and the rows of `out` may lie apart."""
    lens = [700, 120]
    q, kp, vp, table, starts = setup(dtype, 64, 6, 2, 32, lens, news, spare_rows=9)
    wide = torch.full((q.shape[0], 8, 64), 7.0, dtype=dtype, device=DEV)
    out = wide[:, 1:7]
    got, _ = check_attention(ctx, q, kp, vp, table, starts, lens, out=out)
    assert got.data_ptr() == out.data_ptr()
    assert (wide[int(starts[-1]):] == 7).all() and (wide[:, 0] == 7).all() and (wide[:, 7] == 7).all()


def test_attention_strided_queries_and_layered_pools(ctx):
    lens, news, g, page, dim = [150, 90], [20, 1], 2, 16, 128
    q, _, _, table, starts = setup(BF16, dim, 8, g, page, lens, news)
    n = int(table.max()) + 4
    kl, vl = normal(2, (n, 3, g, page, dim), BF16), normal(3, (n, 3, g, page // 8, dim, 8), BF16)
    packed = torch.zeros((q.shape[0], 13, dim), dtype=BF16, device=DEV)
    packed[:, 2:10] = q
    check_attention(ctx, packed[:, 2:10], kl[:, 2], vl[:, 2], table, starts, lens)


def test_attention_offsets_beyond_32_bits(ctx):
    """A pool of more than 2^31 elements whose last pages hold a request."""
    g, page, dim = 8, 64, 128
    n_pages = 2 ** 31 // (g * page * dim) + 40
    kp, vp = (torch.zeros((n_pages,) + s, dtype=BF16, device=DEV) for s in ((g, page, dim), (g, page // 8, dim, 8)))
    lens, news = [500], [6]
    q, ks, vs, small, starts = setup(BF16, dim, 16, g, page, lens, news)
    m = ks.shape[0]
    kp[n_pages - m:], vp[n_pages - m:] = ks, vs
    far = np.where(small >= 0, small + n_pages - m, -1)
    near = ctx.wisv_paged_attention(q, ks, vs, ints(small), ints(starts), ints(lens), max_new=6, max_len=500)
    got = ctx.wisv_paged_attention(q, kp, vp, ints(far), ints(starts), ints(lens), max_new=6, max_len=500)
    assert torch.equal(near, got)
    k, v = normal(8, (2, g, dim), BF16), normal(9, (2, g, dim), BF16)
    slots = [n_pages * page - 1, n_pages * page - 64]
    ctx.wisv_paged_append(None, k, v, None, ints(slots), kp, vp)
    assert torch.equal(kp[-1][:, [63, 0]], k.transpose(0, 1)) and torch.equal(vp[-1][:, 7, :, 7], v[0]) and torch.equal(vp[-1][:, 0, :, 0], v[1])


def test_attention_equal_calls_give_equal_bits(ctx):
    lens, news = [4000, 900, 30], [4, 1, 2]
    q, kp, vp, table, starts = setup(BF16, 128, 32, 8, 16, lens, news)
    args = (q, kp, vp, ints(table), ints(starts), ints(lens), 4, 4000)
    first = ctx.wisv_paged_attention(*args)
    for _ in range(3):
        assert torch.equal(first, ctx.wisv_paged_attention(*args))


def test_attention_on_a_long_cache(ctx):
    """Every split of the keys is used; the sums hold over 20000 keys."""
    for dtype, lens in ((BF16, [20011, 17]), (F32, [9001])):
        q, kp, vp, table, starts = setup(dtype, 64, 2, 1, 256, lens, [1] * len(lens))
        check_attention(ctx, q, kp, vp, table, starts, lens)


# ------------------------------------------------------------------------------------------------ refusals in the binding

def test_refusals_name_what_is_wrong(ctx):
    lens, news = [20], [4]
    q, kp, vp, table, starts = setup(BF16, 64, 4, 2, 16, lens, news)
    t, s, n = ints(table), ints(starts), ints(lens)
    ok = dict(q=q, k_pages=kp, v_pages=vp, block_table=t, q_start=s, kv_len=n)
    for change, what in ((dict(q=q.float()), "q must be"), (dict(q=q.cpu()), "q must be"), (dict(q=q[:, :, :32]), "q must be"),
                         (dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), "close together"), (dict(v_pages=vp.float()), "pools"),
                         (dict(v_pages=vp[:, :, :1]), "pools must be"), (dict(block_table=t.long()), "block_table"), (dict(kv_len=n.cpu()), "kv_len"),
                         (dict(q_start=s[:1]), "q_start"), (dict(slopes=torch.zeros(3, device=DEV)), "slopes"),
                         (dict(prefix_len=ints([1, 2])), "prefix_len"), (dict(out=torch.empty_like(q[:2])), "out must be")):
        with pytest.raises(ValueError, match=what):
            ctx.wisv_paged_attention(**{**ok, **change})
    for change, what in ((dict(q=q[:, :3]), "multiple"), (dict(softcap=-1.0), "softcap"), (dict(window=-1), "window"), (dict(scale=float("nan")), "scale")):
        with pytest.raises(binding.WisvError, match=what):
            ctx.wisv_paged_attention(**{**ok, **change})
    long = [3000]
    q, kp, vp, table, starts = setup(BF16, 64, 4, 2, 16, long, news)
    with pytest.raises(binding.WisvError, match="workspace"):
        ctx.wisv_paged_attention(q, kp, vp, ints(table), ints(starts), ints(long), 4, 3000, workspace=torch.empty(64, device=DEV))


# ------------------------------------------------------------------------------------------------ together

def dense(q, k, v, pos, rep):
    """Causal attention of rows at positions `pos` over k, v [len, g, dim], all in 64 bits."""
    out = np.zeros_like(q)
    for h in range(q.shape[1]):
        x = q[:, h] @ k[:, h // rep].T / np.sqrt(q.shape[2])
        x[np.arange(k.shape[0])[None, :] > pos[:, None]] = -np.inf
        e = np.exp(x - x.max(1, keepdims=True))
        out[:, h] = e @ v[:, h // rep] / e.sum(1, keepdims=True)
    return out


@pytest.mark.parametrize("dtype,captured", [(BF16, False), (BF16, True), (F32, False), (F32, True)])
def test_a_server_step_by_step(ctx, dtype, captured):
    """Four requests over one pool: prompts, drafted blocks of unequal length, an idle request, single tokens.  Each step is plan,
    append and attention with no host copy between them; captured: one graph of the three, replayed for every step with the
    server's own eager work between the replays."""
    h, g, dim, page, batch, tokens = 8, 2, 64, 16, 4, 130
    rng = np.random.default_rng(0)
    kp, vp = pools(64, g, page, dim, dtype)
    free, table = ints(rng.permutation(64)), ints(np.full((batch, 16), -1))
    freq = 10000.0 ** (-np.arange(0, dim, 2) / dim)
    ang = np.arange(256)[:, None] * freq[None, :]
    cos, sin = (torch.from_numpy(f(ang).astype(np.float32)).to(DEV) for f in (np.cos, np.sin))
    cached, new = ints([0] * batch), ints([0] * batch)
    qkv = torch.zeros((tokens, h + 2 * g, dim), dtype=dtype, device=DEV)
    out = torch.full((tokens, h, dim), 3.0, dtype=dtype, device=DEV)
    left = free.clone()
    state = {}

    def step():
        plan = state["plan"] = ctx.wisv_paged_plan(cached, new, left, table, page, tokens)
        q = ctx.wisv_paged_append(qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:], plan.positions, plan.slots, kp, vp, cos, sin)
        ctx.wisv_paged_attention(q, kp, vp, table, plan.q_start, plan.kv_len, max_new=60, max_len=256, out=out)

    graph = None
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    history = [[np.zeros((0, h, dim)), np.zeros((0, g, dim)), np.zeros((0, g, dim))] for _ in range(batch)]
    lens, at = [0] * batch, 0
    steps = [[40, 17, 1, 60], [4, 3, 0, 5], [1, 1, 30, 1], [8, 0, 1, 2], [1, 1, 1, 1], [33, 16, 15, 1], [1, 0, 1, 1]]
    for i, ns in enumerate(steps):
        x = normal(100 + i, (sum(ns), h + 2 * g, dim), dtype)
        qkv[:sum(ns)] = x
        cached.copy_(ints(lens))
        new.copy_(ints(ns))
        left.copy_(torch.cat([free[at:], free[:at]]))
        out.fill_(3.0)
        if graph is None:
            step()
        else:
            graph.replay()
            _ = torch.randn(100, device=DEV).sum()
        torch.cuda.synchronize()
        plan = state["plan"]
        assert plan.status.tolist() == [0] * batch
        at += int(plan.n_used)
        row, xs = 0, f64(x)
        got = f64(out)
        for b, n in enumerate(ns):
            pos = lens[b] + np.arange(n)
            c, s = np.cos(ang)[pos], np.sin(ang)[pos]
            qb, kb, vb = xs[row:row + n, :h], xs[row:row + n, h:h + g], xs[row:row + n, h + g:]
            hist = history[b]
            hist[1] = np.concatenate([hist[1], ref.rotate(kb, c, s)])
            hist[2] = np.concatenate([hist[2], vb])
            lens[b] += n
            if n:
                want = dense(ref.rotate(qb, c, s), hist[1], hist[2], pos, h // g)
                # rounded rotated queries and keys move a score of deviation 1 by about 2^-8; float errors stay below 1e-5
                lim = 0.05 if dtype is BF16 else 2e-5
                assert np.abs(got[row:row + n] - want).max() <= lim, (i, b)
            row += n
        assert (got[row:] == 3.0).all()


def test_steps_on_another_stream_and_two_workspaces(ctx):
    """Calls on two streams at once, each with a workspace of its own, give what they give alone."""
    jobs = []
    for seed, lens, news in ((1, [3000, 200], [4, 1]), (2, [2500], [2])):
        q, kp, vp, table, starts = setup(BF16, 128, 16, 4, 32, lens, news, seed=seed)
        jobs.append((q, kp, vp, ints(table), ints(starts), ints(lens), max(news), max(lens)))
    alone = [ctx.wisv_paged_attention(*j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for _ in range(5):
        for i, (s, j) in enumerate(zip(streams, jobs)):
            with torch.cuda.stream(s):
                got[i].append(ctx.wisv_paged_attention(*j))
    torch.cuda.synchronize()
    for i in range(2):
        for o in got[i]:
            assert torch.equal(o, alone[i])


# ------------------------------------------------------------------------------------------------ more shapes and edges

@pytest.mark.parametrize("dtype,dim,h,g", [(BF16, 128, 4, 1), (BF16, 64, 1, 1), (BF16, 256, 2, 1), (BF16, 32, 8, 2), (F32, 64, 2, 1)])
@pytest.mark.parametrize("new", [16, 17, 31, 32, 33, 64, 127, 128, 129])
def test_attention_around_the_tiles(ctx, dtype, dim, h, g, new):
    """Rows that end before, at and behind tiles of 16, 32 and 128 rows; keys that end around a block of 64."""
    for lens, news in (([new], [new]), ([new + 63], [new]), ([new + 64, 65, new + 1], [new, 2, new])):
        q, kp, vp, table, starts = setup(dtype, dim, h, g, 16, lens, news, seed=new)
        check_attention(ctx, q, kp, vp, table, starts, lens)


@pytest.mark.parametrize("dtype,dim,h,g,news", [(BF16, 64, 40, 1, [1, 3]), (BF16, 128, 128, 1, [1, 2]), (BF16, 32, 96, 2, [2, 0]), (BF16, 256, 33, 1, [1, 2]),
                                                (F32, 32, 130, 1, [1, 2])])
def test_attention_with_more_query_heads_than_a_tile_has_rows(ctx, dtype, dim, h, g, news):
    lens = [150, 40]
    q, kp, vp, table, starts = setup(dtype, dim, h, g, 32, lens, news)
    check_attention(ctx, q, kp, vp, table, starts, lens, softcap=8.0)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 512, 1024, 2048, 4096])
@pytest.mark.parametrize("dtype,new", [(BF16, 1), (BF16, 50), (F32, 20)])
def test_every_page_size(ctx, page, dtype, new):
    h, g, dim, n = 4, 2, 64, 5000 if page > 256 else 700
    lens = [n, new]
    q, kp, vp, table, starts = setup(dtype, dim, h, g, page, lens, [new, new])
    check_attention(ctx, q, kp, vp, table, starts, lens, window=600)
    pos = np.arange(lens[0] - 40, lens[0])
    slots = table[0][pos // page].astype(np.int64) * page + pos % page
    check_append(ctx, dtype, dim, h, g, page, slots, kp.shape[0], pos % 50)


@pytest.mark.parametrize("dtype,hi", [(BF16, 70), (F32, 40)])
def test_attention_of_many_requests(ctx, dtype, hi):
    """More requests than the search for a tile's owner takes at a time, idle ones among them."""
    rng = np.random.default_rng(4)
    batch = 1100
    news = np.where(rng.random(batch) < 0.4, 0, rng.integers(1, 4, batch))
    news[[3, 511, 512, 513, 1023, 1024, 1099]] = hi
    lens = news + rng.integers(0, 60, batch)
    q, kp, vp, table, starts = setup(dtype, 32, 2, 1, 16, lens, news)
    check_attention(ctx, q, kp, vp, table, starts, list(lens))


@pytest.mark.parametrize("dtype,lens,news", [(BF16, [2000, 90], [1, 2]), (BF16, [900, 90], [80, 50]), (F32, [1500, 70], [3, 40])])
def test_attention_leaves_the_rows_before_the_first_request(ctx, dtype, lens, news):
    q, kp, vp, table, starts = setup(dtype, 64, 4, 1, 32, lens, news)
    pad = 7
    padded = torch.cat([torch.full_like(q[:1], float("nan")).expand(pad, -1, -1), q]).contiguous()
    out = torch.full_like(padded, 5.0)
    alone = ctx.wisv_paged_attention(q, kp, vp, ints(table), ints(starts), ints(lens), max(news), max(lens))
    got = ctx.wisv_paged_attention(padded, kp, vp, ints(table), ints(starts + pad), ints(lens), max(news), max(lens), out=out)
    assert (got[:pad] == 5.0).all()
    # (tiles do not move with the rows: the same products in the same order, but perhaps another cut of the keys)
    ref_out, mass, top = ref.attention(f64(q), f64(kp), f64(vp), table, starts, lens)
    lim = limits(dtype, 64, max(lens), ref_out, mass, top, 0.0)
    assert (np.abs(f64(got[pad:]) - ref_out) <= lim).all() and (np.abs(f64(alone) - ref_out) <= lim).all()


@pytest.mark.parametrize("dtype,new", [(BF16, 3), (BF16, 60), (F32, 40)])
def test_attention_keys_that_are_no_numbers_reach_only_the_rows_that_see_them(ctx, dtype, new):
    lens, page = [100], 32
    q, kp, vp, table, starts = setup(dtype, 128, 4, 2, page, lens, [new])
    out, mass, top = ref.attention(f64(q), f64(kp), f64(vp), table, starts, lens)
    at = 100 - new + new // 2
    kp[int(table[0, at // page]), 1, at % page, 5] = float("nan")
    got = f64(ctx.wisv_paged_attention(q, kp, vp, ints(table), ints(starts), ints(lens), new, 100))
    lim = limits(dtype, 128, 100, out, mass, top, 0.0)
    p = 100 - new + np.arange(new)
    assert np.isnan(got[p >= at][:, 2:]).all()                                     # the KV head's own query heads
    assert (np.abs(got - out)[:, :2] <= lim[:, :2]).all() and (np.abs(got - out)[p < at] <= lim[p < at]).all()


@pytest.mark.parametrize("dtype,new", [(BF16, 2), (BF16, 40), (F32, 33)])
@pytest.mark.parametrize("kw", [dict(window=2 ** 31 - 1), dict(softcap=1e-3), dict(softcap=1e4), dict(scale=30.0), dict(scale=1e-6),
                                dict(window=5, prefix=[2 ** 31 - 1, -4]), dict(window=70, prefix=[130, 33], slopes=[0.5, 0.0, -0.25, 3.0])],
                         ids=lambda k: "-".join(map(str, k)))
def test_attention_extreme_settings(ctx, dtype, new, kw):
    lens, news = [400, 90], [new, min(new, 9)]
    q, kp, vp, table, starts = setup(dtype, 64, 4, 2, 16, lens, news)
    check_attention(ctx, q, kp, vp, table, starts, lens, **kw)


@pytest.mark.parametrize("dim,softcap,slopes,new", [(32, 9.0, True, 40), (256, 3.0, True, 50), (64, 0.0, True, 1), (128, 7.0, False, 6)])
def test_attention_captured_before_it_has_run(ctx, dim, softcap, slopes, new):
    """A graph captured as the first call of its kind, replayed with other lengths and queries, eager work between the replays."""
    h, g, page, batch = 4, 2, 16, 2
    q, kp, vp, table, starts = setup(BF16, dim, h, g, page, [300, 300], [new, new])
    t, qs, kl = ints(table), ints(starts), ints([300, 300])
    sl = torch.linspace(0.1, 0.4, h, device=DEV) if slopes else None
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx.wisv_paged_attention(q, kp, vp, t, qs, kl, new, 300, softcap=softcap, slopes=sl, out=out)
    for i, lens in enumerate(([300, 300], [17 + new, 250], [new, 299])):
        kl.copy_(ints(lens))
        q.copy_(normal(50 + i, tuple(q.shape), BF16, 2.0))
        out.zero_()
        graph.replay()
        _ = torch.randn(64, device=DEV).sum().item()
        eager = ctx.wisv_paged_attention(q, kp, vp, t, qs, kl, new, 300, softcap=softcap, slopes=sl)
        assert torch.equal(out, eager)
        check_attention(ctx, q, kp, vp, table, starts, lens, softcap=softcap, slopes=None if sl is None else f64(sl), max_new=new, max_len=300)


def test_two_graphs_replayed_at_once(ctx):
    """Graphs captured apart have workspaces apart: replayed on two streams at once they give what they give alone."""
    jobs, graphs, outs = [], [], []
    for seed, lens, news in ((1, [4000, 300], [3, 1]), (2, [3500, 40], [2, 2])):
        q, kp, vp, table, starts = setup(BF16, 128, 8, 2, 32, lens, news, seed=seed)
        args = (q, kp, vp, ints(table), ints(starts), ints(lens), max(news), max(lens))
        alone = ctx.wisv_paged_attention(*args)
        out, graph = torch.zeros_like(alone), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            ctx.wisv_paged_attention(*args, out=out)
        jobs.append((args, alone))
        graphs.append(graph)
        outs.append(out)
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for s, gr in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
        torch.cuda.synchronize()
        for o, (_, alone) in zip(outs, jobs):
            assert torch.equal(o, alone)


def test_plan_with_entries_that_no_pool_has(ctx):
    """Table entries and free pages so large that their slots would not fit an int are left without a slot."""
    t = [[2 ** 31 - 1, -1], [2 ** 27, -1], [2 ** 27 - 1, -1]]
    dev = ints(t)
    plan = ctx.wisv_paged_plan(ints([3, 3, 3]), ints([2, 2, 2]), ints([]).reshape(-1), dev, 16, 6)
    assert plan.slots.tolist() == [-1, -1, -1, -1, (2 ** 27 - 1) * 16 + 3, (2 ** 27 - 1) * 16 + 4] and plan.status.tolist() == [0, 0, 0]


@pytest.mark.parametrize("dtype,news", [(BF16, [1, 2, 1]), (BF16, [50, 3, 20]), (F32, [9, 1, 40])])
def test_attention_over_pages_that_requests_share(ctx, dtype, news):
    """Requests whose tables begin with the same pages (a common prompt), and a page that stands twice in one row."""
    lens, page = [150, 90, 200], 16
    q, kp, vp, table, starts = setup(dtype, 64, 4, 2, page, lens, news)
    table[1, :4] = table[0, :4]
    table[2, :3] = table[0, :3]
    table[2, 7] = table[2, 5]
    check_attention(ctx, q, kp, vp, table, starts, lens)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_of_two_rows_with_one_slot_leaves_either(ctx, dtype):
    kp, vp = pools(4, 2, 16, 64, dtype)
    k, v = normal(1, (70, 2, 64), dtype), normal(2, (70, 2, 64), dtype)
    before = kp.clone(), vp.clone()
    ctx.wisv_paged_append(None, k, v, None, ints([21] * 70), kp, vp)
    assert (k == kp[1, :, 5]).any(0).all() and (v == vp[1, :, 0, :, 5]).any(0).all()
    kp[1, :, 5], vp[1, :, 0, :, 5] = before[0][1, :, 5], before[1][1, :, 0, :, 5]
    assert torch.equal(kp, before[0]) and torch.equal(vp, before[1])


# ------------------------------------------------------------------------------------------------ float prompts of many rows

# (128 or more tiles of 128 rows, at most a quarter of them empty: float calls that reach the kernel of many rows)
FLOAT_PROMPTS = [(128, 32, 16, [290, 260, 512, 256], [256, 256, 230, 256]), (64, 44, 44, [130, 128, 77, 140], [128, 128, 77, 120]),
                 (256, 16, 8, [600, 640], [600, 550]), (64, 64, 8, [300], [290])]


@pytest.mark.parametrize("dim,h,g,lens,news", FLOAT_PROMPTS)
@pytest.mark.parametrize("mods", [{}] + MODS, ids=lambda m: "-".join(m) or "plain")
def test_attention_of_float_prompts(ctx, dim, h, g, lens, news, mods):
    kw = dict(mods)
    if kw.pop("slopes", False):
        kw["slopes"] = 2.0 ** (-8.0 * np.arange(1, h + 1) / h)
    if kw.pop("prefix", False):
        kw["prefix"] = [5, 64, 3, 90][:len(lens)]
    q, kp, vp, table, starts = setup(F32, dim, h, g, 16, lens, news, seed=5)
    check_attention(ctx, q, kp, vp, table, starts, lens, **kw)


def test_attention_of_float_prompts_cut_along_the_keys(ctx):
    lens, news = [2900], [520]
    q, kp, vp, table, starts = setup(F32, 64, 32, 4, 64, lens, news, seed=6)
    check_attention(ctx, q, kp, vp, table, starts, lens)
    check_attention(ctx, q, kp, vp, table, starts, lens, window=300, prefix=[70])


def test_float_prompts_read_nothing_that_they_should_not(ctx):
    """Holes, page ends and spare pages full of NaN; values that are not finite in the places of some rows."""
    lens, news, page, h, g = [290, 270], [256, 250], 16, 64, 32
    q, kp, vp, table, starts = setup(F32, 64, h, g, page, lens, news, seed=8)
    table[0, 2], table[1, 4], table[1, 9] = -1, 10 ** 6, -7
    clean, _ = check_attention(ctx, q, kp, vp, table, starts, lens)
    held = np.zeros((kp.shape[0], page), bool)
    for b, n in enumerate(lens):
        for j in range(n):
            if 0 <= table[b, j // page] < kp.shape[0]:
                held[table[b, j // page], j % page] = True
    bad = torch.from_numpy(~held).to(DEV)
    kp2 = torch.where(bad[:, None, :, None], torch.full_like(kp, float("nan")), kp)
    vp2 = torch.where(bad.view(kp.shape[0], 1, page // 8, 1, 8), torch.full_like(vp, float("inf")), vp)
    args = (ints(table), ints(starts), ints(lens))
    assert torch.equal(clean, ctx.wisv_paged_attention(q, kp2, vp2, *args, max_new=max(news), max_len=max(lens)))
    at, feature = 200, 37
    vp2[int(table[0, at // page]), :, (at % page) // 8, feature, at % 8] = float("nan")
    got = ctx.wisv_paged_attention(q, kp2, vp2, *args, max_new=max(news), max_len=max(lens))
    sees = torch.zeros_like(got, dtype=torch.bool)
    sees[at - (lens[0] - news[0]):news[0], :, feature] = True
    assert torch.equal(got.isnan(), sees) and torch.equal(got[~sees], clean[~sees])


def test_float_prompts_with_strides_and_padding_rows(ctx):
    lens, news, h, dim = [300], [280], 64, 64
    q, kp, vp, table, starts = setup(F32, dim, h, 8, 32, lens, news, seed=9, spare_rows=40)
    wide = torch.full((q.shape[0], h * dim + 36), float("nan"), dtype=F32, device=DEV)
    wide[:, :h * dim] = q.reshape(q.shape[0], -1)
    out = torch.full((q.shape[0], h * dim + 20), 3.0, dtype=F32, device=DEV)
    view = out[:, :h * dim].view(-1, h, dim)
    check_attention(ctx, wide[:, :h * dim].view(-1, h, dim), kp, vp, table, starts, lens, out=view)
    assert (out[:, h * dim:] == 3.0).all() and (view[280:] == 3.0).all()


@pytest.mark.parametrize("dtype,new", [(BF16, 2), (BF16, 40), (F32, 2), (F32, 40)])
def test_attention_of_queries_that_are_no_numbers_over_cut_keys(ctx, dtype, new):
    """Every part of the keys has nothing but NaN scores for such a row: it stays NaN, and no other row changes."""
    lens, h = [4000], 4
    q, kp, vp, table, starts = setup(dtype, 64, h, 2, 64, lens, [new])
    clean, _ = check_attention(ctx, q, kp, vp, table, starts, lens)
    q[1, 3, 7] = float("nan")
    got = ctx.wisv_paged_attention(q, kp, vp, ints(table), ints(starts), ints(lens), new, 4000)
    assert got[1, 3].isnan().all()
    got[1, 3] = clean[1, 3]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype,dim,h,g,lens,news", [(BF16, 128, 8, 2, [200, 40], [2, 1]), (BF16, 64, 8, 2, [300, 70], [90, 64]), (BF16, 256, 4, 2, [170], [60]),
                                                     (F32, 64, 4, 2, [200, 40], [30, 9]), (F32, 128, 32, 16, [290, 512], [256, 512])])
@pytest.mark.parametrize("kw", [dict(scale=-0.2, softcap=7.0), dict(scale=-0.1), dict(scale=-0.3, softcap=3.0, window=40)], ids=lambda k: "-".join(k))
def test_attention_with_a_negative_scale(ctx, dtype, dim, h, g, lens, news, kw):
    q, kp, vp, table, starts = setup(dtype, dim, h, g, 32, lens, news, seed=11)
    check_attention(ctx, q, kp, vp, table, starts, lens, **kw)


@pytest.mark.parametrize("dtype,dim", [(BF16, 32), (BF16, 64), (BF16, 128), (BF16, 256), (F32, 64), (F32, 128), (F32, 256)])
def test_attention_of_prompts_far_into_a_cache_of_ragged_requests(ctx, dtype, dim):
    """Idle requests, single tokens and prompts in one call, holes in the pages of some, over many blocks of keys."""
    lens, news, h = [1500, 0, 700, 33, 900, 64], [300, 0, 1, 33, 257, 64], 32 if dtype is F32 else 4
    q, kp, vp, table, starts = setup(dtype, dim, h, h // 2, 16, lens, news, seed=12)
    table[0, 11] = table[4, 3] = -1
    check_attention(ctx, q, kp, vp, table, starts, lens)
    check_attention(ctx, q, kp, vp, table, starts, lens, window=333, prefix=[100, 0, 50, 0, 17, 64], softcap=11.0)


# ------------------------------------------------------------------------------------------------ a plan that takes up the last one's

@pytest.mark.parametrize("batch,page,hi_cached,hi_new", [(1, 16, 40, 3), (7, 16, 90, 40), (257, 64, 900, 40), (1030, 16, 70, 9), (4096, 32, 100, 5)])
@pytest.mark.parametrize("name", ["kv_len", "q_start", "status", "positions", "slots"])
@pytest.mark.parametrize("which", ["cached", "new"])
def test_plan_over_its_own_lengths(ctx, batch, page, hi_cached, hi_new, name, which):
    """An output that lies over cached_len or new_len, in step with it or an element apart: what apart gives, whoever is refused."""
    rng = np.random.default_rng(batch)
    cached, new = rng.integers(0, hi_cached + 1, batch), rng.integers(0, hi_new + 1, batch)
    table, n = ref.pages_of(list(cached), page, rng)
    wide = np.full((batch, -(-(hi_cached + hi_new) // page)), -1, np.int32)
    wide[:, :table.shape[1]] = table
    wide = wide[:, :max(table.shape[1], wide.shape[1] - 1)]      # the longest requests find no room in their rows
    total = max(int(new.sum()), 1)
    need = int(sum(-(-(c + m) // page) - -(-c // page) for c, m in zip(cached, new)))
    for n_free, tokens in ((need, total), (need // 2, total + 50), (need, max(1, total * 2 // 3))):
        free = n + rng.permutation(n_free)
        want = ref.plan(cached, new, free, wide, page, tokens)
        for apart in (0, 1):
            sizes = dict(q_start=batch + 1, kv_len=batch, positions=tokens, slots=tokens, n_used=1, status=batch)
            both = torch.zeros(max(sizes[name], batch) + 1, dtype=torch.int32, device=DEV)
            lens = both[apart:apart + batch]
            lens.copy_(ints(cached if which == "cached" else new))
            out = binding.PagePlan(**{k: both[:m] if k == name else torch.full((m,), -77, dtype=torch.int32, device=DEV) for k, m in sizes.items()})
            dev = ints(wide)
            got = ctx.wisv_paged_plan(lens if which == "cached" else ints(cached), lens if which == "new" else ints(new), ints(free).reshape(-1), dev, page,
                                      tokens, out=out)
            for k, g, w in zip(binding.PagePlan._fields + ("block_table",), tuple(got) + (dev,), want):
                assert g.cpu().numpy().tolist() == w.tolist(), (k, apart)


@pytest.mark.parametrize("captured", [False, True])
def test_plans_that_take_up_the_last_ones_lengths(ctx, captured):
    """A server's steps over one set of tensors: the lengths that a plan leaves are the next one's, in place or in two sets in turn."""
    rng = np.random.default_rng(2)
    batch, page, tokens, width = 300, 16, 3000, 12
    for sets in (1, 2):
        free = ints(5 + rng.permutation(2000))
        left, new, table = free.clone(), ints(np.zeros(batch)), ints(np.full((batch, width), -1))
        outs = [binding.PagePlan(*[torch.zeros(n, dtype=torch.int32, device=DEV) for n in (batch + 1, batch, tokens, tokens, 1, batch)]) for _ in range(sets)]
        steps = [lambda i=i: ctx.wisv_paged_plan(outs[i - 1].kv_len, new, left, table, page, tokens, out=outs[i]) for i in range(sets)]
        if captured:
            graphs = []
            for step in steps:
                torch.cuda.synchronize()
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(graphs[-1]):
                    step()
            steps = [g.replay for g in graphs]
        lens, at, host = np.zeros(batch, np.int64), 0, np.full((batch, width), -1)
        for i in range(7):
            ns = rng.integers(0, 9, batch) * (rng.random(batch) < 0.9)
            new.copy_(ints(ns))
            left.copy_(torch.cat([free[at:], free[:at]]))
            want = ref.plan(lens, ns, left.tolist(), host, page, tokens)
            steps[i % sets]()
            _ = torch.randn(100, device=DEV).sum()
            torch.cuda.synchronize()
            for k, g, w in zip(binding.PagePlan._fields + ("block_table",), tuple(outs[i % sets]) + (table,), want):
                assert g.cpu().numpy().tolist() == w.tolist(), (sets, i, k)
            lens, host, at = want[1], want[6], at + int(want[4][0])


def test_plan_for_the_most_rows_that_a_step_can_have(ctx):
    """2^31 - 1 rows: the count of a thread's rows ends beyond 32 bits."""
    tokens = 2 ** 31 - 1
    plan = ctx.wisv_paged_plan(ints([3, 70]), ints([2, 20]), ints([9, 8, 7]), ints([[4, -1], [-1] * 2]), 64, tokens)
    assert plan.q_start.tolist() == [0, 2, 22] and plan.kv_len.tolist() == [5, 90] and plan.status.tolist() == [0, 0] and plan.n_used.tolist() == [0]
    assert plan.positions[:22].tolist() == [3, 4] + list(range(70, 90)) and plan.slots[:3].tolist() == [259, 260, -1]
    for rows, want in ((plan.positions, 0), (plan.slots, -1)):
        for part in rows[22:].split(1 << 28):
            assert int(part.min()) == want and int(part.max()) == want


# ------------------------------------------------------------------------------------------------ the terms of a probability

@pytest.mark.parametrize("dim,h,g,news", [(32, 8, 2, [8, 3, 1]), (64, 8, 2, [4, 4, 1]), (64, 12, 3, [8, 8, 5]), (128, 8, 2, [4, 1, 3]), (128, 8, 2, [8, 5, 8]),
                                          (128, 3, 1, [6, 10, 9]), (256, 4, 1, [4, 4, 1]), (256, 8, 2, [8, 1, 7])])
@pytest.mark.parametrize("window", [0, 90])
def test_few_rows_have_probabilities_of_two_terms(ctx, dim, h, g, news, window):
    """Up to 32 rows per KV head, by the hint: probabilities are good to 2^-17, which one bf16 term is not.

    Queries and keys are small integers, so that products and their sums are exact and a score x (in units of ln 2) is off by the
    rounding of the scale, of its product and of the difference to the maximum, 2^-24 * 2 max|x| each.  An exponential adds 2^-23, each
    of at most four moves of the maximum 2^-23 and a rounding, twice (sum and output): delta = (6 max|x| + 20) * 2^-24.  The rest as above,
    with 2^-17 for a probability.  Outputs near zero show it: what is rounded at the end is small there."""
    lens = [160, 97, 130]
    rng = np.random.default_rng(dim + h)
    table, n_pages = ref.pages_of(lens, 16, rng)
    starts = np.concatenate([[0], np.cumsum(news)])
    whole = lambda *shape: torch.from_numpy(rng.integers(-2, 3, shape).astype(np.float32)).to(BF16).to(DEV)  # noqa: E731
    q, kp, scale = whole(int(starts[-1]), h, dim), whole(n_pages, g, 16, dim), 2.0 ** -5
    vp = normal(dim, (n_pages, g, 2, dim, 8), BF16)
    got = f64(ctx.wisv_paged_attention(q, kp, vp, ints(table), ints(starts), ints(lens), max(news), max(lens), scale=scale, window=window))
    qh, kh, vh = f64(q), f64(kp), f64(vp)
    out, mass, _ = ref.attention(qh, kh, vh, table, starts, lens, scale=scale, window=window)
    one, x_max = np.zeros_like(out), 0.0
    for b, n in enumerate(news):     # what one term would give
        k, v, _ = ref.gather(kh, vh, table[b], lens[b])
        p, j = (lens[b] - n + np.arange(n))[:, None], np.arange(lens[b])[None, :]
        sees = (j <= p) & (j > p - (window or 10 ** 6))
        for head in range(h):
            x = np.where(sees, scale * (qh[starts[b]:starts[b + 1], head] @ k[head // (h // g)].T), -np.inf)
            x_max = max(x_max, np.abs(x[sees]).max() / np.log(2.0))
            e = f64(torch.from_numpy(np.exp(x - x.max(1, keepdims=True))).to(BF16))
            one[starts[b]:starts[b + 1], head] = e @ v[head // (h // g)] / e.sum(1, keepdims=True)
    delta = (6 * x_max + 20) * 2.0 ** -24
    lim = 2.0 ** -8 * np.abs(out) + (2.0 ** -17 + 2 * delta + (max(lens) + 64) * 2.0 ** -24) * mass
    assert (np.abs(one - out) > lim).mean() > 0.01
    err = np.abs(got - out)
    record(f"paged_two_terms_{dim}_{h}_{g}_{max(news)}_w{window}", {"err_of_limit": float((err / lim).max()), "one_term_of_limit": float((np.abs(one - out) / lim).max())})
    assert (err <= lim).all(), (err / lim).max()


@pytest.mark.parametrize("dtype,dim,lens,news", [(BF16, 128, [300, 70], [3, 1]), (BF16, 128, [300, 70], [90, 64]), (BF16, 64, [5000], [2]), (BF16, 64, [9000], [60]),
                                                 (F32, 64, [300, 70], [40, 9]), (F32, 64, [5000], [4])])
def test_attention_in_place(ctx, dtype, dim, lens, news):
    """out over q itself, in packed rows: what another tensor gets, and nothing beside the queries is touched."""
    h, g = 8, 2
    q, kp, vp, table, starts = setup(dtype, dim, h, g, 16, lens, news)
    args = (kp, vp, ints(table), ints(starts), ints(lens), max(news), max(lens))
    want = ctx.wisv_paged_attention(q, *args)
    packed = torch.full((q.shape[0], h + 3, dim), 7.0, dtype=dtype, device=DEV)
    packed[:, 1:1 + h] = q
    got = ctx.wisv_paged_attention(packed[:, 1:1 + h], *args, out=packed[:, 1:1 + h])
    assert torch.equal(got, want) and (packed[:, 0] == 7).all() and (packed[:, 1 + h:] == 7).all()


@pytest.mark.parametrize("dim,g,lens,news", [(128, 8, [500, 300], [5, 7]), (128, 8, [700], [300]), (64, 8, [1500], [200]), (256, 4, [300, 90], [60, 90])])
def test_prompts_offsets_beyond_32_bits(ctx, dim, g, lens, news):
    """Pools of more than 2^31 elements whose last pages hold the requests, on the kernel of many rows (both its forms at head_dim 128)."""
    page, h = 64, 4 * g
    n_pages = 2 ** 31 // (g * page * dim) + 40
    kp, vp = (torch.zeros((n_pages,) + s, dtype=BF16, device=DEV) for s in ((g, page, dim), (g, page // 8, dim, 8)))
    q, ks, vs, small, starts = setup(BF16, dim, h, g, page, lens, news)
    m = ks.shape[0]
    kp[n_pages - m:], vp[n_pages - m:] = ks, vs
    far = np.where(small >= 0, small + n_pages - m, -1)
    args = (ints(starts), ints(lens), max(news), max(lens))
    near = ctx.wisv_paged_attention(q, ks, vs, ints(small), *args)
    assert near.any() and torch.equal(near, ctx.wisv_paged_attention(q, kp, vp, ints(far), *args))


def test_float_prompts_offsets_beyond_32_bits(ctx):
    page, h, g, dim, lens, news = 64, 32, 16, 128, [290, 260, 512, 256], [256, 256, 230, 256]
    n_pages = 2 ** 31 // (g * page * dim) + 40
    kp, vp = (torch.zeros((n_pages,) + s, dtype=F32, device=DEV) for s in ((g, page, dim), (g, page // 8, dim, 8)))
    q, ks, vs, small, starts = setup(F32, dim, h, g, page, lens, news)
    m = ks.shape[0]
    kp[n_pages - m:], vp[n_pages - m:] = ks, vs
    far = np.where(small >= 0, small + n_pages - m, -1)
    args = (ints(starts), ints(lens), max(news), max(lens))
    near = ctx.wisv_paged_attention(q, ks, vs, ints(small), *args)
    assert near.any() and torch.equal(near, ctx.wisv_paged_attention(q, kp, vp, ints(far), *args))


CAPTURED_FIRST = '''
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import torch
import test_gpu_paged as t
ctx = t.binding.Context(t.configs.get(0).model, t.gen.make_weights(t.configs.get(0).model, 0, t.DEV), 1, 32, 1)
calls = []
for dtype, dim, h, g, lens, news in {cases!r}:
    q, kp, vp, table, starts = t.setup(getattr(torch, dtype), dim, h, g, 16, lens, news)
    args = (q, kp, vp, t.ints(table), t.ints(starts), t.ints(lens), max(news), max(lens))
    calls.append((args, torch.zeros_like(q)))
torch.cuda.synchronize()
for args, out in calls:
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.wisv_paged_attention(*args, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert out.any() and torch.equal(out, ctx.wisv_paged_attention(*args))
        torch.cuda.synchronize()
    print("captured", args[0].shape, flush=True)
print("done", flush=True)
'''


def test_the_first_paged_call_of_a_process_may_be_captured():
    """In a process of its own: the first call of each kernel of prompts, which asks for its LDS then, is the captured one."""
    import os
    import subprocess
    import sys
    tests = os.path.dirname(os.path.abspath(__file__))
    cases = [("bfloat16", 128, 8, 2, [300, 200], [90, 60]), ("bfloat16", 128, 8, 2, [300, 200], [8, 5]), ("bfloat16", 256, 4, 2, [170], [60]),
             ("bfloat16", 64, 8, 2, [9000], [60]), ("float32", 128, 32, 16, [290, 260, 512, 256], [256, 256, 230, 256])]
    code = CAPTURED_FIRST.format(root=os.path.dirname(tests), tests=tests, cases=cases)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.strip().endswith("done"), r.stdout + r.stderr
