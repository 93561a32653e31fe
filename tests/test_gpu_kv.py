"""The quantized key/value cache and the attention over it.  Codes, scales
and values equal the oracle's bit for bit; attention is held to float64 by
the bound that the oracle derives (half steps of fp16 weights and fp32 sums)
plus half a step of the output's own type."""
import numpy as np
import pytest
import torch

import paper_2311_14114_amd as sq
from oracle import serve

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _tables(r, lengths, page, spare=2, width=0):
    """(pages, table int32 [B, width]) with the sequences' pages scattered."""
    need = [-(-n // page) for n in lengths]
    total = sum(need) + spare
    order = r.permutation(total)
    table = np.full((len(lengths), max([1, width, *need])), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return total, table


def _random_cache(r, pages, page, heads, D, bits):
    top = 127 if bits == 8 else 7
    mk = lambda: serve.pack_codes(r.integers(-top, top + 1, (pages, heads, page, D)), bits)
    sc = lambda: (np.exp(0.3 * r.standard_normal((pages, heads, page))) / top * 2).astype(np.float32)
    h = dict(k=mk(), ks=sc(), v=mk(), vs=sc())
    d = {n: torch.from_numpy(x.view(np.int8) if x.dtype == np.uint8 else x).cuda() for n, x in h.items()}
    return sq.KVCache(d["k"], d["ks"], d["v"], d["vs"], bits=bits), h


def _same(got, want):
    got, want = got.float().cpu().numpy(), want.float().numpy()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


# ---------------------------------------------------------------- writing --
WRITES = [  # new tokens, positions held before, heads, head_dim, page
    ([1], [0], 1, 64, 16), ([1, 1, 1], [15, 16, 31], 8, 128, 16), ([5, 0, 33], [3, 9, 0], 2, 192, 24),
    ([40], [7], 3, 256, 1), ([0, 0, 7], [0, 0, 0], 4, 64, 8), ([300, 17], [100, 1], 2, 128, 64),
    ([1] * 70, list(range(70)), 1, 128, 16)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("new,before,heads,D,page", WRITES, ids=lambda v: "x")
def test_write_and_read(new, before, heads, D, page, dtype, bits):
    r = np.random.default_rng(sum(new) + D)
    pages, table = _tables(r, [a + n for a, n in zip(before, new)], page)
    cache, h = _random_cache(r, pages, page, heads, D, bits)
    T, behind = sum(new), 2
    # keys and values beside each other and beside something else, per token
    kv = torch.from_numpy(r.standard_normal((T + behind, 3, heads, D)).astype(np.float32)).to(TYPES[dtype]).cuda()
    if T > 2:
        kv[1, 0, 0] = 0                              # a row of zeros
        kv[0, 1, heads - 1, 5] = float("nan")        # and one that holds a NaN
        kv[2, 0, 0, D - 1] = float("-inf")
    K, V = kv[:, 0], kv[:, 1]
    cu = np.concatenate(([0], np.cumsum(new)))
    print(f"[gpu] kv_write {new[:4]} heads={heads} D={D} page={page} {dtype} {bits} bits", flush=True)
    args = (torch.from_numpy(table).cuda(), _i32(cu.tolist()), _i32(before))
    sq.soniq_kv_write(cache, K, V, *args)
    for x, codes, scales, rows in (("k", cache.k, cache.k_scale, K), ("v", cache.v, cache.v_scale, V)):
        serve.kv_write(h[x], h[x + "s"], rows.float().cpu().numpy(), table, cu, before, bits)
        np.testing.assert_array_equal(codes.cpu().numpy().view(np.uint8), h[x])     # and the rest untouched
        np.testing.assert_array_equal(scales.cpu().numpy(), h[x + "s"])
    out = torch.full((2, T + behind, heads, D), 3.0, dtype=TYPES[dtype], device="cuda")
    sq.soniq_kv_read(cache, *args, T + behind, out=(out[0], out[1]))
    for i, x in enumerate("kv"):
        want = torch.from_numpy(serve.kv_read(h[x], h[x + "s"], table, cu, before, bits)).to(TYPES[dtype])
        _same(out[i, :T], want)
        assert bool((out[i, T:] == 3.0).all())       # rows behind the last sequence


def test_bad_pages_are_left_out():
    """Entries that name no page, positions past the table or before it:
    nothing is written, zeros are read, nothing is attended to."""
    r = np.random.default_rng(4)
    pages, page, heads, D = 6, 8, 2, 64
    table = np.array([[0, -1, 2], [6, 3, 2**31 - 1], [-2**31, 4, 5]], np.int32)
    new, start = [40, 24, 16], [-5, 0, 4]
    cu = np.concatenate(([0], np.cumsum(new)))
    cache, h = _random_cache(r, pages, page, heads, D, 8)
    T = sum(new)
    K = torch.from_numpy(r.standard_normal((T, heads, D)).astype(np.float32)).cuda()
    args = (torch.from_numpy(table).cuda(), _i32(cu.tolist()), _i32(start))
    sq.soniq_kv_write(cache, K, -K, *args)
    serve.kv_write(h["k"], h["ks"], K.cpu().numpy(), table, cu, start, 8)
    serve.kv_write(h["v"], h["vs"], -K.cpu().numpy(), table, cu, start, 8)
    np.testing.assert_array_equal(cache.k.cpu().numpy().view(np.uint8), h["k"])
    np.testing.assert_array_equal(cache.v_scale.cpu().numpy(), h["vs"])
    k, v = sq.soniq_kv_read(cache, *args, T, dtype=torch.float32)
    _same(k, torch.from_numpy(serve.kv_read(h["k"], h["ks"], table, cu, start, 8)))
    _same(v, torch.from_numpy(serve.kv_read(h["v"], h["vs"], table, cu, start, 8)))
    q = torch.from_numpy(r.standard_normal((3, 4, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    _check_attention(cache, h, q, table, [0, 1, 2, 3], [24, 8, 2**30], 8)


def test_odd_prefix_sums_stay_inside():
    """Prefix sums that fall, start below 0 or end past the batch: whatever
    they say, rows past the batch and other sequences' pages stay as they were."""
    r = np.random.default_rng(5)
    cache, h = _random_cache(r, 4, 8, 2, 64, 8)
    table = torch.from_numpy(np.array([[0, 1], [2, -1]], np.int32)).cuda()
    K = torch.randn((6, 2, 64), device="cuda")
    for cu in ([5, 2, 100], [-3, 4, 2], [0, 2**31 - 1, -2**31]):
        sq.soniq_kv_write(cache, K, K, table, _i32(cu), _i32([0, 0]))
        q = torch.randn((6, 2, 64), device="cuda").to(torch.bfloat16)
        sq.soniq_kv_attention(cache, q, table, _i32(cu), _i32([9, 4]))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(cache.k.cpu().numpy().view(np.uint8)[3], h["k"][3])


# -------------------------------------------------------------- attention --
def _check_attention(cache, h, q, table, cu, kv_len, bits, mask=None, scale=None, max_kv=None, max_q=None):
    scale = cache.head_dim ** -0.5 if scale is None else scale
    T, Hq = q.shape[:2]
    out = torch.full((T, Hq, 2, cache.head_dim), 5.0, dtype=q.dtype, device="cuda")[:, :, 1]
    lse = torch.full((T, Hq), 5.0, device="cuda")
    sq.soniq_kv_attention(cache, q, torch.from_numpy(table).cuda(), _i32(list(cu)), _i32(list(kv_len)), scale=scale,
                          mask=None if mask is None else torch.from_numpy(mask).cuda(), out=out, lse=lse,
                          max_kv=max_kv, max_q=max_q)
    want, wl, bound = serve.attention(q.float().cpu().numpy(), h["k"], h["ks"], h["v"], h["vs"], table, cu, kv_len,
                                      bits, scale, mask)
    n = int(cu[-1])
    got = out.double().cpu().numpy()
    half = torch.finfo(q.dtype).eps / 2
    tiny = torch.finfo(q.dtype).tiny * half            # half a step of the type's subnormals
    far = np.abs(got[:n] - want[:n])
    ok = far <= bound[:n] + half * (np.abs(want[:n]) + bound[:n]) + tiny
    assert ok.all(), (far[~ok].max(), bound[:n][~ok].max(), np.argwhere(~ok)[:4])
    gl = lse.double().cpu().numpy()[:n]
    empty = np.isneginf(wl[:n])
    np.testing.assert_array_equal(np.isneginf(gl), empty)
    assert np.all(got[:n][empty] == 0)
    assert np.all(np.abs(gl[~empty] - wl[:n][~empty]) <= 1e-4 + 1e-5 * np.abs(wl[:n][~empty]))
    assert bool((out[n:] == 5.0).all()) and bool((lse[n:] == 5.0).all())
    return out


ATTEND = [  # new tokens, cached positions (new ones among them), heads, group, head_dim, page
    ([1], [1], 1, 1, 64, 16), ([1], [31], 2, 1, 128, 16), ([1], [33], 1, 4, 128, 1), ([1, 1], [257, 64], 2, 8, 64, 64),
    ([1], [2049], 2, 4, 128, 16), ([1, 1, 1], [700, 1, 0], 2, 3, 192, 24), ([1], [1500], 1, 2, 256, 8),
    ([2, 5], [2, 300], 2, 2, 128, 16), ([16, 1, 0, 7], [100, 129, 40, 7], 1, 4, 128, 32), ([17], [17], 2, 5, 64, 16),
    ([64], [1000], 1, 2, 64, 48), ([40], [333], 1, 8, 128, 7), ([3, 3], [90, 4500], 1, 16, 128, 128),
    ([30], [95], 2, 1, 256, 16), ([100], [130], 1, 3, 192, 32), ([130, 2], [1100, 3], 1, 1, 128, 16)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("new,lens,heads,group,D,page", ATTEND, ids=lambda v: "x")
def test_attention(new, lens, heads, group, D, page, dtype, bits):
    r = np.random.default_rng(sum(new) + sum(lens) + D)
    pages, table = _tables(r, lens, page)
    cache, h = _random_cache(r, pages, page, heads, D, bits)
    T = sum(new)
    q = torch.from_numpy(2 * r.standard_normal((T + 1, heads * group, D)).astype(np.float32)).to(TYPES[dtype]).cuda()
    cu = np.concatenate(([0], np.cumsum(new))).tolist()
    print(f"[gpu] kv_attention new={new} lens={lens} heads={heads}x{group} D={D} page={page} {bits} bits", flush=True)
    _check_attention(cache, h, q, table, cu, lens, bits)
    if max(new) > 1:                                  # a tree (its first token sees nothing but itself)
        W = -(-max(new) // 64)
        mask = np.zeros((T + 1, 64 * W), bool)
        for b, n in enumerate(new):
            for i in range(n):
                p = int(r.integers(-1, i)) if i else -1
                if p >= 0:
                    mask[cu[b] + i] = mask[cu[b] + p]
                mask[cu[b] + i, i] = True
        words = np.packbits(mask.reshape(T + 1, W, 8, 8), axis=-1, bitorder="little").reshape(T + 1, W, 8)
        _check_attention(cache, h, q, table, cu, lens, bits, mask=np.ascontiguousarray(words).view(np.int64).reshape(T + 1, W))


@pytest.mark.parametrize("max_kv", [0, 1, 100, 100000])
def test_the_hint_changes_nothing_but_rounding(max_kv):
    r = np.random.default_rng(8)
    lens = [3000, 40]
    pages, table = _tables(r, lens, 16)
    cache, h = _random_cache(r, pages, 16, 2, 128, 8)
    q = torch.from_numpy(r.standard_normal((2, 8, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
    _check_attention(cache, h, q, table, [0, 1, 2], lens, 8, max_kv=max_kv)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_head_major_operands_and_shared_pages(dtype, bits):
    """[heads, tokens, head_dim] operands, a table that is a slice of a wider
    one, a prefix that two sequences share, a page that one holds twice."""
    r = np.random.default_rng(21)
    page, heads, group, D, B = 16, 2, 4, 128, 3
    wide = np.full((B, 40), 5, np.int32)
    cache, h = _random_cache(r, 30, page, heads, D, bits)
    wide[0, 3:9] = [4, 7, 9, 11, 4, 13]               # page 4 twice
    wide[1, 3:9] = [4, 7, 9, 15, 16, 17]              # the first three shared with sequence 0
    wide[2, 3:9] = [20, 21, 22, 23, 24, -1]
    table = torch.from_numpy(wide).cuda()[:, 3:9]
    start, new = [90, 70, 61], [3, 5, 2]
    cu = [0, 3, 8, 10]
    kv = torch.randn((2, heads, 11, D), device="cuda").to(TYPES[dtype])
    K, V = kv[0].transpose(0, 1), kv[1].transpose(0, 1)
    sq.soniq_kv_write(cache, K, V, table, _i32(cu), _i32(start))
    narrow = np.ascontiguousarray(wide[:, 3:9])
    serve.kv_write(h["k"], h["ks"], K.float().cpu().numpy(), narrow, cu, start, bits)
    serve.kv_write(h["v"], h["vs"], V.float().cpu().numpy(), narrow, cu, start, bits)
    np.testing.assert_array_equal(cache.k.cpu().numpy().view(np.uint8), h["k"])
    np.testing.assert_array_equal(cache.v_scale.cpu().numpy(), h["vs"])
    back = torch.full((2, heads, 11, D), 3.0, dtype=TYPES[dtype], device="cuda")
    sq.soniq_kv_read(cache, table, _i32(cu), _i32(start), 11, out=(back[0].transpose(0, 1), back[1].transpose(0, 1)))
    k, v = sq.soniq_kv_read(cache, table, _i32(cu), _i32(start), 11, dtype=TYPES[dtype])
    assert torch.equal(back[0].transpose(0, 1)[:10], k[:10]) and torch.equal(back[1].transpose(0, 1)[:10], v[:10])
    assert bool((back[:, :, 10] == 3.0).all())
    lens = [a + n for a, n in zip(start, new)]
    q = torch.randn((heads * group, 11, D), device="cuda").to(TYPES[dtype]).transpose(0, 1)
    want = _check_attention(cache, h, q, narrow, cu, lens, bits)
    out = torch.full((heads * group, 11, D), 3.0, dtype=TYPES[dtype], device="cuda")
    work = torch.empty(sq.soniq_kv_attention_workspace(cache, 11, heads * group, B, 8, 200) + 64, dtype=torch.uint8,
                       device="cuda")
    sq.soniq_kv_attention(cache, q, table, _i32(cu), _i32(lens), out=out.transpose(0, 1), work=work, max_q=8, max_kv=200)
    far = (out.transpose(0, 1)[:10].float() - want[:10].float()).abs()
    # Another split of the same sums.  Each result is off by half a step of its
    # type and, for bf16, by half a step of the fp16 weights, 2^-11 of
    # sum |w v| <= max |v| < 8: 2 (eps / 2 |o| + 2^-8) < 4 eps (1 + |o|).
    assert bool((far <= 4 * torch.finfo(q.dtype).eps * (1 + want[:10].float().abs())).all())
    assert bool((out[:, 10] == 3.0).all())


@pytest.mark.parametrize("max_kv", [None, 60])
def test_many_sequences(max_kv):
    """More sequences than a wave has lanes, many of them without new tokens
    or without positions, lengths on both sides of a part's."""
    r = np.random.default_rng(22)
    B = 200
    new = r.choice([0, 1, 1, 2, 9], B).tolist()
    lens = [int(n * r.integers(0, 2) + r.choice([0, 5, 130, 900, 2600])) for n in new]
    pages, table = _tables(r, lens, 64)
    cache, h = _random_cache(r, pages, 64, 1, 64, 8)
    cu = np.concatenate(([0], np.cumsum(new))).tolist()
    q = torch.from_numpy(r.standard_normal((sum(new) + 3, 2, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    _check_attention(cache, h, q, table, cu, lens, 8, max_q=9, max_kv=max_kv)


@pytest.mark.parametrize("B", [3, 40, 64, 65])
@pytest.mark.parametrize("longest,rows", [(9000, 1), (1500, 40)])
@pytest.mark.parametrize("max_kv", [None, 128, 1 << 20])
def test_parts_of_very_different_lengths(B, longest, rows, max_kv):
    """One long sequence among short and empty ones, which the lengths
    themselves cut, with hints far off on both sides."""
    r = np.random.default_rng(24)
    new = [rows] + r.integers(0, rows + 1, B - 1).tolist()
    lens = [longest] + [int(n * (k % 3 > 0) + r.choice([0, 0, 1, 127, 129, 700])) for k, n in enumerate(new[1:])]
    pages, table = _tables(r, lens, 128)
    cache, h = _random_cache(r, pages, 128, 2, 64, 4)
    cu = np.concatenate(([0], np.cumsum(new))).tolist()
    q = torch.from_numpy(r.standard_normal((sum(new) + 1, 2, 64)).astype(np.float32)).to(torch.float16).cuda()
    _check_attention(cache, h, q, table, cu, lens, 4, max_q=rows, max_kv=max_kv)


def test_the_most_sequences_with_the_longest_hint():
    """65535 sequences of 32 heads, told to hold 2^31 - 1 positions: the cut's
    arithmetic stays in range, and empty ones among them stay empty."""
    r = np.random.default_rng(25)
    B = 65535
    cache, h = _random_cache(r, 3, 16, 32, 64, 8)
    table = np.full((B, 2), -1, np.int32)
    table[0], table[B - 1] = [1, 0], [2, -1]
    lens = np.zeros(B, np.int32)
    lens[0], lens[B - 1] = 20, 9
    cu = np.zeros(B + 1, np.int32)
    cu[1:], cu[40000:], cu[B] = 1, 2, 3               # sequence 39999 has a new token and no position
    q = torch.from_numpy(r.standard_normal((4, 32, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    _check_attention(cache, h, q, table, cu, lens, 8, max_q=1, max_kv=2**31 - 1)


def test_two_graphs_share_a_workspace():
    """Two layers' attention captured on one workspace, replayed in turn, with
    eager work on it between the replays."""
    r = np.random.default_rng(23)
    lens = [3000, 41]
    pages, table = _tables(r, lens, 16)
    caches = [_random_cache(r, pages, 16, 2, 128, b)[0] for b in (8, 4)]
    t, cu, ln = torch.from_numpy(table).cuda(), _i32([0, 2, 3]), _i32(lens)
    qs = [torch.randn((3, 8, 128), device="cuda").to(torch.bfloat16) for _ in range(2)]
    work = torch.empty(sq.soniq_kv_attention_workspace(caches[0], 3, 8, 2, 2, 3000), dtype=torch.uint8, device="cuda")
    assert work.numel() > 0
    call = lambda i: sq.soniq_kv_attention(caches[i], qs[i], t, cu, ln, max_q=2, max_kv=3000, work=work)
    want = [call(0), call(1)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for i in range(2):
        with torch.cuda.stream(side):
            call(i)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(call(i))
        graphs.append(g)
    for k in (0, 1, 1, 0, 0, 1):
        outs[k].zero_()
        graphs[k].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[k], want[k])
        assert torch.equal(call(1 - k), want[1 - k])
        torch.cuda.synchronize()


def test_rows_that_see_nothing():
    """No cached position, masks without a bit, lengths shorter than the new
    tokens: zeros and -inf, whatever the cache holds."""
    r = np.random.default_rng(9)
    lens = [0, 5, 2, 70]
    new = [2, 5, 4, 3]
    pages, table = _tables(r, [64, 64, 64, 128], 16)
    cache, h = _random_cache(r, pages, 16, 2, 64, 8)
    cu = np.concatenate(([0], np.cumsum(new))).tolist()
    q = torch.from_numpy(r.standard_normal((sum(new), 4, 64)).astype(np.float32)).to(torch.float16).cuda()
    _check_attention(cache, h, q, table, cu, lens, 8)
    mask = np.zeros((sum(new), 1), np.int64)
    mask[3, 0] = -1                                   # bits past the new tokens count for nothing
    mask[11, 0] = 1 << 2
    _check_attention(cache, h, q, table, cu, lens, 8, mask=mask)


@pytest.mark.parametrize("bits", [8, 4])
def test_what_is_masked_cannot_be_seen(bits):
    """NaN and infinite scales, and scales of 1e30, at masked positions,
    positions past the length and unused pages."""
    r = np.random.default_rng(10)
    lens, new = [90, 300], [6, 6]
    pages, table = _tables(r, lens, 16, spare=5)
    cache, h = _random_cache(r, pages, 16, 2, 128, bits)
    cu = [0, 6, 12]
    q = torch.from_numpy(r.standard_normal((12, 8, 128)).astype(np.float32)).to(torch.bfloat16).cuda()
    mask = np.zeros((12, 1), np.int64)
    for t in range(12):
        mask[t] = (1 << (t % 6)) | (1 if t % 6 != 4 else 0)
    # nobody but token 4 sees new position 4, and nobody at all a position past the length
    used = np.zeros((pages, 16), bool)
    for b, n in enumerate(lens):
        for pos in range(n):
            used[table[b, pos // 16], pos % 16] = True
    bad = [np.nan, np.inf, 1e30, -np.inf]
    for x in ("ks", "vs"):
        for h_ in range(2):
            plane = h[x][:, h_]
            plane[~used] = r.choice(bad, (~used).sum())
        for b, n in enumerate(lens):
            pos = n - 6 + 4
            h[x][table[b, pos // 16], :, pos % 16] = 1e30 if x == "vs" else np.nan
    cache.k_scale.copy_(torch.from_numpy(h["ks"]))
    cache.v_scale.copy_(torch.from_numpy(h["vs"]))
    out = torch.zeros((12, 8, 128), dtype=torch.bfloat16, device="cuda")
    sq.soniq_kv_attention(cache, q, torch.from_numpy(table).cuda(), _i32(cu), _i32(lens),
                          mask=torch.from_numpy(mask).cuda(), out=out)
    want, _, bound = serve.attention(q.float().cpu().numpy(), h["k"], h["ks"], h["v"], h["vs"], table, cu, lens, bits,
                                     128 ** -0.5, mask)
    got = out.double().cpu().numpy()
    for t in range(12):
        if t % 6 == 4:
            assert np.isnan(got[t]).all()             # it sees a NaN key
        else:
            assert (np.abs(got[t] - want[t]) <= bound[t] + 2.0**-8 * (np.abs(want[t]) + bound[t])).all()


@pytest.mark.parametrize("scale", [0.0, -0.125])
def test_scales_of_zero_and_below(scale):
    """A scale of 0 averages what is visible; a negative one turns the order."""
    r = np.random.default_rng(15)
    lens = [70, 9]
    pages, table = _tables(r, lens, 16)
    cache, h = _random_cache(r, pages, 16, 2, 64, 8)
    q = torch.from_numpy(r.standard_normal((6, 4, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    q[1] = 0
    _check_attention(cache, h, q, table, [0, 3, 6], lens, 8, scale=scale)


def test_extreme_scores_and_scales():
    """Scores that leave one position, V scales that span 2^40 and fall where
    the weights rise, q rows that span fp16's range and beyond."""
    r = np.random.default_rng(11)
    lens = [400, 400, 400]
    pages, table = _tables(r, lens, 16)
    cache, h = _random_cache(r, pages, 16, 1, 128, 8)
    h["vs"] *= np.exp2(r.integers(-20, 21, h["vs"].shape)).astype(np.float32)
    cache.v_scale.copy_(torch.from_numpy(h["vs"]))
    q = r.standard_normal((3, 2, 128)).astype(np.float32)
    q[0] *= 100
    q[1] *= 1e-3
    q[2] *= np.exp2(r.integers(-12, 5, 128))
    q = torch.from_numpy(q).to(torch.bfloat16).cuda()
    _check_attention(cache, h, q, table, [0, 1, 2, 3], lens, 8)
    big = (q.float() * 1e9).to(torch.bfloat16)
    _check_attention(cache, h, big, table, [0, 1, 2, 3], lens, 8, scale=128 ** -0.5 / 1e9)


def test_a_bad_query_spoils_itself_alone():
    r = np.random.default_rng(12)
    lens = [200]
    pages, table = _tables(r, lens, 16)
    cache, h = _random_cache(r, pages, 16, 1, 64, 8)
    q = torch.from_numpy(r.standard_normal((5, 4, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    t = torch.from_numpy(table).cuda()
    ref = sq.soniq_kv_attention(cache, q, t, _i32([0, 5]), _i32(lens))
    q[2, 1, 7] = float("nan")
    got = sq.soniq_kv_attention(cache, q, t, _i32([0, 5]), _i32(lens))
    assert bool(torch.isnan(got[2, 1]).all())
    got[2, 1] = ref[2, 1]
    assert torch.equal(got, ref)


def test_repeats_are_identical_and_max_q_bounds_the_rows():
    r = np.random.default_rng(13)
    lens = [2500, 77]
    pages, table = _tables(r, lens, 32)
    cache, h = _random_cache(r, pages, 32, 4, 128, 4)
    q = torch.from_numpy(r.standard_normal((10, 16, 128)).astype(np.float32)).to(torch.float16).cuda()
    t, cu, ln = torch.from_numpy(table).cuda(), _i32([0, 4, 10]), _i32(lens)
    ref = sq.soniq_kv_attention(cache, q, t, cu, ln)
    for _ in range(3):
        assert torch.equal(sq.soniq_kv_attention(cache, q, t, cu, ln), ref)
    out = torch.full_like(q, 9.0)
    sq.soniq_kv_attention(cache, q, t, cu, ln, max_q=4, out=out)
    tail = slice(8, 10)                                # the second sequence's queries from the fifth on
    assert bool((out[tail] == 9.0).all())
    far = (out[:8].float() - ref[:8].float()).abs()
    assert bool((far <= 2.0**-9 * (1 + ref[:8].float().abs())).all())


def test_long_cache_passes_32_bits():
    """A cache of more than 4 GiB of codes a side, used at its far end."""
    page, heads, D = 256, 8, 256
    pages = (9 << 29) // (page * heads * D)
    print("[gpu] cache past 4 GiB", flush=True)
    cache = sq.KVCache.empty(pages, page, heads, D, 8)
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    n = 700
    K = torch.randn((n, heads, D), device="cuda").to(torch.bfloat16)
    V = torch.randn((n, heads, D), device="cuda").to(torch.bfloat16)
    args = (table, _i32([0, n]), _i32([0]))
    sq.soniq_kv_write(cache, K, V, *args)
    q8, s = serve.quantize_rows(K.float().cpu().numpy())
    np.testing.assert_array_equal(cache.k[pages - 1].cpu().numpy().transpose(1, 0, 2), q8[:256])
    np.testing.assert_array_equal(cache.k[pages - 2, :, :188].cpu().numpy().transpose(1, 0, 2), q8[512:])
    k, v = sq.soniq_kv_read(cache, *args, n, dtype=torch.float32)
    _same(k, torch.from_numpy(q8.astype(np.float32) * s[..., None]))
    small = sq.KVCache.empty(3, page, heads, D, 8)
    args0 = (_i32([[0, 1, 2]]), *args[1:])
    sq.soniq_kv_write(small, K, V, *args0)
    q = torch.randn((2, 16, D), device="cuda").to(torch.bfloat16)
    a = sq.soniq_kv_attention(cache, q, table, _i32([0, 2]), _i32([n]))
    b = sq.soniq_kv_attention(small, q, args0[0], _i32([0, 2]), _i32([n]))
    assert torch.equal(a, b)


def test_binding_refusals():
    cache = sq.KVCache.empty(4, 16, 2, 64)
    t, cu, ln = _i32([[0, 1]]), _i32([0, 3]), _i32([20])
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((3, 2, 64), device="cuda")
    att = lambda **kw: sq.soniq_kv_attention(cache, kw.pop("q", q), kw.pop("t", t), kw.pop("cu", cu), kw.pop("ln", ln), **kw)
    bad = [(TypeError, lambda: att(t=t.long())), (ValueError, lambda: att(cu=cu[:1])), (TypeError, lambda: att(ln=ln.cpu())),
           (sq.SoniqError, lambda: att(q=q.float())), (TypeError, lambda: att(q=q.double())),
           (sq.SoniqError, lambda: att(q=q[:, :3])), (ValueError, lambda: att(q=q[..., :32])),
           (TypeError, lambda: att(q=q.transpose(1, 2).contiguous().transpose(1, 2))),
           (TypeError, lambda: att(mask=torch.zeros((3, 1), dtype=torch.int32, device="cuda"))),
           (ValueError, lambda: att(mask=torch.zeros((2, 1), dtype=torch.int64, device="cuda"))),
           (sq.SoniqError, lambda: att(mask=torch.zeros((3, 5), dtype=torch.int64, device="cuda"))),
           (sq.SoniqError, lambda: att(max_q=257)), (ValueError, lambda: att(out=q.half())),
           (TypeError, lambda: att(out=torch.empty_like(q[:1]).expand(3, 4, 64))),
           (TypeError, lambda: att(out=torch.as_strided(torch.empty_like(q), (3, 4, 64), (64, 64, 1)))),
           (TypeError, lambda: att(out=torch.as_strided(torch.empty_like(q), (3, 4, 64), (64, 128, 1)))),
           (sq.SoniqError, lambda: att(scale=float("nan"))),
           (sq.SoniqError, lambda: att(max_kv=5000, work=torch.empty(64, dtype=torch.uint8, device="cuda"))),
           (sq.SoniqError, lambda: att(max_kv=5000, work=torch.empty(1 << 20, dtype=torch.uint8, device="cuda")[8:])),
           (TypeError, lambda: att(work=torch.empty(1 << 20, dtype=torch.float32, device="cuda"))),
           (ValueError, lambda: att(lse=torch.zeros((3, 3), device="cuda"))),
           (ValueError, lambda: sq.soniq_kv_write(cache, k, k[..., ::2], t, cu, ln)),
           (TypeError, lambda: sq.soniq_kv_write(cache, torch.zeros((3, 2, 128), device="cuda")[..., ::2], k, t, cu, ln)),
           (ValueError, lambda: sq.soniq_kv_write(cache, k.half(), k, t, cu, ln)),
           (ValueError, lambda: sq.soniq_kv_write(cache, k[:, :1], k[:, :1], t, cu, ln)),
           (ValueError, lambda: sq.soniq_kv_read(cache, t, cu, ln, 4, out=(k, k))),
           (ValueError, lambda: sq.KVCache.empty(4, 16, 2, 64, bits=2)), (TypeError, lambda: sq.KVCache(k, k, k, k)),
           (ValueError, lambda: sq.KVCache(cache.k, cache.k_scale, cache.v[:1], cache.v_scale))]
    for i, (error, call) in enumerate(bad):
        print("[gpu] refusal", i, flush=True)
        with pytest.raises(error):
            call()


def test_masks_without_a_word_or_a_token():
    """An empty mask has a null address, which is no mask: without words it is
    refused, since it would hide every new token; without tokens there is
    nothing to hide."""
    cache = sq.KVCache.empty(4, 16, 2, 64)
    t, ln = _i32([[0, 1]]), _i32([20])
    for T in (3, 0):
        q = torch.zeros((T, 4, 64), dtype=torch.bfloat16, device="cuda")
        mask = torch.zeros((T, 1), dtype=torch.int64, device="cuda")
        assert sq.soniq_kv_attention(cache, q, t, _i32([0, T]), ln, mask=mask).shape == (T, 4, 64)
        with pytest.raises(ValueError):
            sq.soniq_kv_attention(cache, q, t, _i32([0, T]), ln, mask=mask[:, :0].contiguous())


def test_more_tokens_than_a_sequence_may_have():
    """300 sequences of one new token each: max_q has to be given, and the
    refusal says so."""
    r = np.random.default_rng(26)
    lens = r.integers(1, 40, 300).tolist()
    pages, table = _tables(r, lens, 16)
    cache, h = _random_cache(r, pages, 16, 1, 64, 8)
    q = torch.from_numpy(r.standard_normal((300, 2, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    cu = list(range(301))
    with pytest.raises(ValueError, match="max_q"):
        sq.soniq_kv_attention(cache, q, torch.from_numpy(table).cuda(), _i32(cu), _i32(lens))
    _check_attention(cache, h, q, table, cu, lens, 8, max_q=1)


def test_no_sequences_and_no_tokens():
    cache = sq.KVCache.empty(4, 16, 2, 64)
    none = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    q = torch.full((3, 4, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    sq.soniq_kv_attention(cache, q, none, _i32([0]), _i32([]), out=out)
    assert bool((out == 7.0).all())
    assert sq.soniq_kv_attention(cache, q[:0], _i32([[0]]), _i32([0, 0]), _i32([5])).shape == (0, 4, 64)
    k = torch.zeros((0, 2, 64), device="cuda")
    sq.soniq_kv_write(cache, k, k, _i32([[0]]), _i32([0, 0]), _i32([0]))
    assert sq.soniq_kv_read(cache, _i32([[0]]), _i32([0, 0]), _i32([0]), 0)[0].shape == (0, 2, 64)


# ------------------------------------------------------------ used together --
def _layer(r, hidden, heads, group, D):
    W = {"qkv": ((group + 2) * heads * D, hidden), "out": (hidden, group * heads * D)}
    made = {}
    for n, (rows, cols) in W.items():
        w = torch.from_numpy((r.standard_normal((rows, cols)) / np.sqrt(cols)).astype(np.float32)).cuda()
        made[n] = sq.soniq_quantize_rows(w)
    return made


def _step(layer, x, cache, heads, group, D, table, cu, start, kv_len, mask):
    """One attention block of a decode step: projection, cache write,
    attention, projection."""
    qkv = sq.soniq_quantize_i8_gemm(x, *layer["qkv"]).view(x.shape[0], (group + 2) * heads, D)
    q, k, v = qkv[:, :group * heads], qkv[:, group * heads:-heads], qkv[:, -heads:]
    sq.soniq_kv_write(cache, k, v, table, cu, start)
    o = sq.soniq_kv_attention(cache, q, table, cu, kv_len, mask=mask, max_q=8)
    return qkv, o, sq.soniq_quantize_i8_gemm(o.view(x.shape[0], -1), *layer["out"])


@pytest.mark.parametrize("bits", [8, 4])
def test_decode_block_with_a_draft_tree_eager_and_captured(bits):
    """The calls as a serving loop makes them: a tree of drafted tokens after
    cached prefixes, eager against the oracle step by step, then captured and
    replayed with other inputs, eager work between the replays."""
    r = np.random.default_rng(14)
    hidden, heads, group, D, page = 512, 2, 4, 64, 16
    layer = _layer(r, hidden, heads, group, D)
    held, n = [37, 0, 130], 6
    lens = [a + n for a in held]
    pages, table = _tables(r, lens, page)
    cache, h = _random_cache(r, pages, page, heads, D, bits)
    other, _ = _random_cache(np.random.default_rng(14), pages, page, heads, D, bits)
    for a, b in ((cache.k, other.k), (cache.k_scale, other.k_scale), (cache.v, other.v), (cache.v_scale, other.v_scale)):
        b.copy_(a)
    cu = [0, n, 2 * n, 3 * n]
    parents = [-1, 0, 0, 1, 1, 2]
    seen = []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    mask = np.array(seen * 3, np.int64)[:, None]
    args = (torch.from_numpy(table).cuda(), _i32(cu), _i32(held), _i32(lens), torch.from_numpy(mask).cuda())
    xs = [torch.from_numpy(r.standard_normal((3 * n, hidden)).astype(np.float32)).to(torch.bfloat16).cuda()
          for _ in range(3)]
    qkv, o, y = _step(layer, xs[0], cache, heads, group, D, *args)
    f = lambda t: t.float().cpu().numpy()
    q8, s = serve.quantize_rows(f(xs[0]))
    _same(qkv.view(3 * n, -1), torch.from_numpy(serve.i8_gemm(q8, s, *(t.cpu().numpy() for t in layer["qkv"]))).to(torch.bfloat16))
    serve.kv_write(h["k"], h["ks"], f(qkv[:, group * heads:-heads]), table, cu, held, bits)
    serve.kv_write(h["v"], h["vs"], f(qkv[:, -heads:]), table, cu, held, bits)
    np.testing.assert_array_equal(cache.k.cpu().numpy().view(np.uint8), h["k"])
    np.testing.assert_array_equal(cache.v.cpu().numpy().view(np.uint8), h["v"])
    want, _, bound = serve.attention(f(qkv[:, :group * heads]), h["k"], h["ks"], h["v"], h["vs"], table, cu, lens, bits,
                                     D ** -0.5, mask)
    assert (np.abs(f(o) - want) <= bound + 2.0**-8 * (np.abs(want) + bound)).all()
    q8, s = serve.quantize_rows(f(o).reshape(3 * n, -1))
    _same(y, torch.from_numpy(serve.i8_gemm(q8, s, *(t.cpu().numpy() for t in layer["out"]))).to(torch.bfloat16))

    x = xs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(layer, x, other, heads, group, D, *args)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = _step(layer, x, other, heads, group, D, *args)
    for k in (1, 2, 0, 1):
        x.copy_(xs[k])
        g.replay()
        torch.cuda.synchronize()
        want = _step(layer, xs[k], cache, heads, group, D, *args)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert torch.equal(cache.k, other.k) and torch.equal(cache.v_scale, other.v_scale)
