"""What the attention over the quantized cache keeps of its numbers: softmax
weights to fp32's sums, scores and V scales far apart, rows that are not
finite.  Every expected value is float64 arithmetic on the cache's codes."""
import numpy as np
import pytest
import torch

import paper_2311_14114_amd as sq
from oracle import serve
from test_gpu_kv import TYPES, _i32, _random_cache, _tables

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- weights --
def integer_queries(r, T, heads, D):
    return r.integers(-3, 4, (T, heads, D)).astype(np.float32)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_weights_are_two_fp16_numbers(dtype, bits):
    """Few positions carry most of the weight, integer queries leave the
    scores' sums exact: what is left is the weights' own error.  Each is two
    fp16 numbers cut to 11 bits, the second from what the first left: 2^-20 of
    the weight."""
    r = np.random.default_rng(31)
    lens, new = [100, 61], [4, 3]
    pages, table = _tables(r, lens, 16)
    cache, h = _random_cache(r, pages, 16, 2, 128, bits)
    cu = [0, 4, 7]
    q = torch.from_numpy(integer_queries(r, 7, 8, 128)).to(TYPES[dtype]).cuda()
    scale = 0.15 if bits == 8 else 0.1
    out = sq.soniq_kv_attention(cache, q, torch.from_numpy(table).cuda(), _i32(cu), _i32(lens), scale=scale)
    want, _, bound = serve.attention(q.float().cpu().numpy(), h["k"], h["ks"], h["v"], h["vs"], table, cu, lens, bits,
                                     scale, weight=2.0**-20, exact_sums=True)
    far = np.abs(out.double().cpu().numpy() - want)
    half, tiny = torch.finfo(q.dtype).eps / 2, torch.finfo(q.dtype).tiny
    ok = far <= bound + half * (np.maximum(np.abs(want), tiny) + bound)
    assert ok.all(), ((~ok).sum(), ok.size, (far - half * np.abs(want))[~ok].max(), bound.max())


# ------------------------------------------------- scores and scales apart --
LOG2E = float(np.log2(np.e))
LN2 = float(np.float32(np.log(2.0)))                  # a scale of it makes scores count in powers of two


def _told(r, scores, values, D, bits, page=16):
    """A cache of one sequence whose position j scores scores[j] (float32)
    against a query of 1 in element 0 and holds V codes times values[j]."""
    n, top = len(scores), 127 if bits == 8 else 7
    pages, table = _tables(r, [n], page)
    cache, h = _random_cache(r, pages, page, 1, D, bits)
    at = [(int(table[0, j // page]), 0, j % page) for j in range(n)]
    for j, (x, v) in enumerate(zip(np.asarray(scores, np.float32), np.asarray(values, np.float32))):
        code = np.zeros(D, np.int64)
        code[0] = np.sign(x)
        h["k"][at[j]], h["ks"][at[j]] = serve.pack_codes(code, bits), np.abs(x)
        h["vs"][at[j]] = v / np.float32(top)
    for t, x in ((cache.k, "k"), (cache.k_scale, "ks"), (cache.v_scale, "vs")):
        t.copy_(torch.from_numpy(h[x].view(np.int8) if x == "k" else h[x]))
    V = np.stack([serve.unpack_codes(h["v"][a], bits) * h["vs"][a].astype(np.float64) for a in at])
    return cache, table, V


def _check_told(scores, values, dtype, bits, D=64, seed=0):
    """Query heads of 1, 1/2 and -1 in element 0, against float64.  Off by,
    relatively, in each weight: two fp16 numbers 2^-21; the base-2 exponent x
    of a weight that counts is rounded three times (the row's unit, the
    difference from the reference, a moved reference), 2^-23 |x| each as
    exp2 grows by ln 2 < 1; exp2 and its products 8 * 2^-24.  The sums of n
    terms add n * 2^-24.  An exponential below 2^-126 of the row's largest may be
    0, and a weight is off by 2^-30 of the largest one where it is subnormal."""
    r = np.random.default_rng(seed)
    cache, table, V = _told(r, scores, values, D, bits)
    n = len(scores)
    heads = np.array([1.0, 0.5, -1.0])
    q = torch.zeros((1, 3, D), dtype=TYPES[dtype], device="cuda")
    q[0, :, 0] = torch.from_numpy(heads).to(q.dtype)
    lse = torch.zeros((1, 3), device="cuda")
    out = sq.soniq_kv_attention(cache, q, torch.from_numpy(table).cuda(), _i32([0, 1]), _i32([n]), scale=LN2, lse=lse)
    got, got_lse = out.double().cpu().numpy()[0], lse.double().cpu().numpy()[0]
    half, tiny = torch.finfo(q.dtype).eps / 2, torch.finfo(q.dtype).tiny
    s = np.asarray(scores, np.float32).astype(np.float64)
    for g, a in enumerate(heads):
        z = a * s * (LN2 * LOG2E)
        x = z - z.max()
        p = np.exp2(x)
        share = p[:, None] * np.abs(V) / p.sum()
        off = 2.0**-21 + 3 * 2.0**-23 * np.abs(x) + (8 + n) * 2.0**-24
        total = (off * p).sum() / p.sum()             # of the sum below
        want = p @ V / p.sum()
        bound = (share * (off + total)[:, None]).sum(0) + n * (2.0**-126 * np.abs(V).max(0) + 2.0**-30 * share.max())
        limit = bound + half * (np.maximum(np.abs(want), tiny) + bound)
        far = np.abs(got[g] - want)
        assert np.isfinite(got[g]).all(), (g, got[g][:4], want[:4])
        assert (far <= limit).all(), (g, far.max(), limit.min(), got[g][:4], want[:4])
        l = z.max() / LOG2E + np.log(p.sum())
        assert abs(got_lse[g] - l) <= 1e-5 + 2.0**-21 * abs(l), (g, got_lse[g], l)


def _spread(steps, span):
    """Each step's (score, value) for `span` positions."""
    return [x for x, _ in steps for _ in range(span)], [v for _, v in steps for _ in range(span)]


APART = {  # (score in base 2, V's largest element) in the order of the positions
    "zero V, a jump, then V far below": [(0, 0), (75, 0), (-60, 1)],
    "zero V alone": [(0, 0), (75, 0), (-3, 0)],
    "equal scores past 2^24": [(3e7 + 2, 0.01), (3e7 + 2, 10), (3e7 + 2, 3e4)],
    "equal scores past 2^29": [(1e9, 0.01), (1e9, 10)],
    "a rise that V makes up for": [(0, 1), (100, 2.0**-100)],
    "a fall that V makes up for": [(100, 2.0**-50), (0, 2.0**50)],
    "V all tiny": [(0, 2.0**-100), (1, 2.0**-101), (-4, 2.0**-99)],
    "V all huge": [(0, 2.0**120), (3, 2.0**117), (1, 2.0**119)],
    "steps up": [(30 * i, 2.0**(-30 * i)) for i in range(4)],
    "steps down": [(-30 * i, 2.0**(30 * i)) for i in range(4)],
    "up and down": [(0, 1), (90, 2.0**-90), (10, 2.0**-12), (89, 2.0**-91), (-5, 32)],
}


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("span", [32, 128, 700])      # by waves, by steps of a wave, by parts
@pytest.mark.parametrize("name", list(APART))
def test_scores_and_scales_far_apart(name, span, bits):
    _check_told(*_spread(APART[name], span), "bf16", bits)


@pytest.mark.parametrize("span", [32, 128, 700])
def test_scores_far_apart_fp16(span):
    for steps in ([(1e9, 0.01), (1e9, 10)], [(0, 1), (12, 2.0**-12)], [(0, 0), (75, 0), (74, 3)]):
        _check_told(*_spread(steps, span), "fp16", 8)


def test_a_wave_far_below_the_others():
    """One wave meets zero V and a jump, the others scores so far above that
    nothing of that wave counts."""
    scores, values = [], []
    for step in ((0, 0), (75, 0), (-60, 1)):
        for wave in range(4):
            scores += [step[0] if wave == 0 else 215 + wave] * 32
            values += [step[1] if wave == 0 else 0.5] * 32
    _check_told(scores, values, "bf16", 8)


def test_rows_of_zeros_beside_others():
    """V rows of zeros as soniq_kv_write leaves them (scale 0), keys with
    scores on both sides of the others'."""
    r = np.random.default_rng(33)
    for spread in (1.0, 12.0, 60.0):
        scores = spread * r.standard_normal(900)
        values = np.where(r.random(900) < 0.6, 0.0, np.exp2(r.integers(-8, 9, 900)))
        values[:300] = 0
        _check_told(scores, values, "bf16", 8)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("span", [32, 128, 700])
@pytest.mark.parametrize("rise", [20, 39, 60, 79])
def test_a_rise_onto_large_values(rise, span, bits):
    """Scores that rise by less than any step of a reference, onto V whose
    product with an unnormalised exponential would pass fp32's end."""
    _check_told(*_spread([(0, 1), (rise, 2.0**110), (rise - 3, 2.0**113)], span), "bf16", bits)


# ------------------------------------------------------- rows with no value --
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("side", ["k", "v"])
def test_a_visible_row_that_held_an_infinity(side, dtype, bits):
    """A key or value row with an infinity is stored as scale inf and codes 0,
    so its elements are NaN: every query that sees it gets NaN, whatever its
    own values, and no other query does."""
    r = np.random.default_rng(34)
    held, new, heads, group, D = 90, 40, 2, 4, 128
    pages, table = _tables(r, [held + new], 16)
    cache, h = _random_cache(r, pages, 16, heads, D, bits)
    kv = torch.from_numpy(r.standard_normal((2, new, heads, D)).astype(np.float32)).cuda()
    where = 13                                         # this new token's row, in head 1
    kv["kv".index(side), where, 1, 7] = float("inf") if bits == 8 else -float("inf")
    args = (torch.from_numpy(table).cuda(), _i32([0, new]))
    sq.soniq_kv_write(cache, kv[0], kv[1], *args, _i32([held]))
    q = r.standard_normal((new, heads * group, D)).astype(np.float32)
    q[1::4, :, 5] *= 300                               # an outlier channel
    q[2::4] *= np.exp2(r.integers(-12, 5, D))          # a wide range
    q[3::4] *= 0.01
    q = torch.from_numpy(q).to(TYPES[dtype]).cuda()
    out = sq.soniq_kv_attention(cache, q, *args, _i32([held + new]))
    bad = torch.zeros((new, heads * group), dtype=torch.bool)
    bad[where:, group:] = True                         # causal: that token and those after it
    nan = torch.isnan(out).cpu()
    assert bool(nan[bad].all()), int((~nan[bad].all(-1)).sum())
    assert not bool(nan[~bad].any())


@pytest.mark.parametrize("sign", [1, -1])
def test_an_infinite_scale_over_codes(sign):
    """A caller's own cache may hold an infinite K scale over any codes: NaN
    as well, not a score of minus infinity that drops the position."""
    r = np.random.default_rng(35)
    pages, table = _tables(r, [70], 16)
    cache, h = _random_cache(r, pages, 16, 1, 64, 8)
    cache.k_scale[int(table[0, 1]), 0, 3] = sign * float("inf")
    q = torch.from_numpy(r.standard_normal((2, 8, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    out = sq.soniq_kv_attention(cache, q, torch.from_numpy(table).cuda(), _i32([0, 2]), _i32([70]))
    assert bool(torch.isnan(out).all())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_codes_of_zero_add_nothing(dtype, bits):
    """Keys with one outlier channel have codes 0 elsewhere.  Queries that are
    0 in that channel score exactly 0, whatever the scale: the mean of V."""
    r = np.random.default_rng(36)
    n, D = 200, 128
    pages, table = _tables(r, [n], 16)
    cache, h = _random_cache(r, pages, 16, 1, D, bits)
    h["k"][:] = serve.pack_codes(np.where(np.arange(D) == 4, 127 if bits == 8 else 7, 0), bits)
    h["ks"][:] = np.exp2(r.integers(0, 24, h["ks"].shape))
    cache.k.copy_(torch.from_numpy(h["k"].view(np.int8)))
    cache.k_scale.copy_(torch.from_numpy(h["ks"]))
    q = r.standard_normal((5, 8, D)).astype(np.float32)
    q[2] *= np.exp2(r.integers(-9, 6, D))
    q[:, :, 4] = 0
    q = torch.from_numpy(q).to(TYPES[dtype]).cuda()
    lse = torch.zeros((5, 8), device="cuda")
    out = sq.soniq_kv_attention(cache, q, torch.from_numpy(table).cuda(), _i32([0, 5]), _i32([n]), lse=lse)
    V = np.concatenate([serve.unpack_codes(h["v"][p, 0], bits) * h["vs"][p, 0, :, None].astype(np.float64)
                        for p in table[0]])
    half = torch.finfo(q.dtype).eps / 2
    for i in range(5):
        m = n - 4 + i
        want, size = V[:m].mean(0), np.abs(V[:m]).mean(0)
        # a weight 2^-21 and the sums' m roundings, in the numerator and below
        bound = size * (2.0**-21 + 2 * m * 2.0**-24)
        assert (np.abs(out[i].double().cpu().numpy() - want) <= bound + half * (np.abs(want) + bound)).all()
        assert np.abs(lse[i].cpu().numpy() - np.log(m)).max() <= 1e-5


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("outlier", [1, 30, 1000])
def test_a_score_is_an_fp32_sum(outlier, dtype, bits):
    """One position a sequence, so that lse is the score itself, of keys with
    one channel above the others and queries that are 0 there: off by D + 8
    roundings of 2^-24 of the products' sizes (the sum's, the scalings' and
    lse's), and of those alone."""
    r = np.random.default_rng(37)
    B, D = 300, 128
    K = r.standard_normal((B, 2, D)).astype(np.float32)
    K[:, :, 5] *= outlier
    cache = sq.KVCache.empty(B, 16, 2, D, bits)
    table, cu, one = _i32(np.arange(B)[:, None].tolist()), _i32(list(range(B + 1))), _i32([1] * B)
    k = torch.from_numpy(K).cuda()
    sq.soniq_kv_write(cache, k, k, table, cu, _i32([0] * B))
    q = r.standard_normal((B, 8, D)).astype(np.float32)
    q[1::2, :, 5] = 0
    q = torch.from_numpy(q).to(TYPES[dtype]).cuda()
    lse = torch.zeros((B, 8), device="cuda")
    sq.soniq_kv_attention(cache, q, table, cu, one, lse=lse, max_q=1, max_kv=1)
    codes, scales = serve.quantize_rows(K, 127.0 if bits == 8 else 7.0)
    key = np.repeat(codes * scales[..., None].astype(np.float64), 4, axis=1)
    products = q.double().cpu().numpy() * key * D**-0.5
    far = np.abs(lse.double().cpu().numpy() - products.sum(-1))
    assert (far <= (D + 8) * 2.0**-24 * np.abs(products).sum(-1)).all(), far.max()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("power", [-114, -60, 60, 118])
def test_queries_of_any_size(power, bits):
    """Queries of 2^power against keys of its reciprocal: the scores of
    ordinary ones, to the same roundings as above."""
    r = np.random.default_rng(38)
    B, D = 100, 128
    K = (r.standard_normal((B, 1, D)) * 2.0**-power).astype(np.float32)
    cache = sq.KVCache.empty(B, 16, 1, D, bits)
    table, cu, one = _i32(np.arange(B)[:, None].tolist()), _i32(list(range(B + 1))), _i32([1] * B)
    k = torch.from_numpy(K).cuda()
    sq.soniq_kv_write(cache, k, k, table, cu, _i32([0] * B))
    q = torch.from_numpy((r.standard_normal((B, 4, D)) * 2.0**power).astype(np.float32)).to(torch.bfloat16).cuda()
    lse = torch.zeros((B, 4), device="cuda")
    sq.soniq_kv_attention(cache, q, table, cu, one, lse=lse, max_q=1, max_kv=1)
    codes, scales = serve.quantize_rows(K, 127.0 if bits == 8 else 7.0)
    products = q.double().cpu().numpy() * (codes * scales[..., None].astype(np.float64)) * D**-0.5
    far = np.abs(lse.double().cpu().numpy() - products.sum(-1))
    assert (far <= (D + 8) * 2.0**-24 * np.abs(products).sum(-1)).all(), far.max()
