"""8-bit linear layers with one scale per token and per output channel:
codes, scales and outputs equal the oracle's bit for bit (the order of the
fp32 scaling is fixed, the sums are exact), at sizes on and off every tile,
for tokens that start anywhere and for rows of zeros, infinities and NaN."""
import numpy as np
import pytest
import torch

import paper_2311_14114_amd as sq
from oracle import serve

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _tokens(M, K, dtype, gap=0, seed=0, offset=0):
    """[M, K] tokens inside a wider buffer, `offset` elements from its start."""
    g = torch.Generator().manual_seed(seed + M * 7 + K)
    x = torch.randn((M, K + gap), generator=g)
    x[:, torch.rand(K + gap, generator=g) < 0.01] *= 20
    flat = torch.zeros(M * (K + gap) + offset, dtype=TYPES[dtype], device="cuda")
    flat[offset:] = x.to(TYPES[dtype]).flatten().cuda()
    return flat[offset:].view(M, K + gap)[:, :K]


def _codes(M, K, seed, ld=None, offset=0):
    r = np.random.default_rng(seed)
    ld = K if ld is None else ld
    x = r.integers(-128, 128, (M, ld)).astype(np.int8)
    flat = torch.zeros(M * ld + offset, dtype=torch.int8, device="cuda")
    flat[offset:] = torch.from_numpy(x).flatten().cuda()
    return flat[offset:].view(M, ld)[:, :K], x[:, :K]


def _same(got, want):
    """Bit for bit, with any NaN equal to any other."""
    got, want = got.cpu(), want.cpu()
    assert got.shape == want.shape and got.dtype == want.dtype
    nan = torch.isnan(want) if want.is_floating_point() else torch.zeros(want.shape, dtype=torch.bool)
    if want.is_floating_point():
        assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], want[~nan])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,K,gap,offset", [
    (1, 1, 0, 0), (1, 64, 0, 0), (3, 100, 5, 1), (5, 4091, 3, 3), (2, 4096, 0, 0), (33, 768, 0, 2),
    (700, 130, 1, 0), (9, 8192, 8, 0), (2, 16389, 0, 0), (1, 65536, 0, 1), (4100, 16, 0, 0),
    (300, 512, 0, 0), (257, 513, 1, 0), (300, 1024, 0, 1), (260, 1025, 0, 0), (1025, 1025, 0, 0), (1030, 2048, 0, 0),
    (300, 2048, 0, 0), (3, 2049, 0, 0), (3, 4097, 1, 0), (3, 6144, 0, 0), (3, 6145, 0, 0), (2, 8193, 0, 1), (3, 12288, 0, 0),
    (2, 12289, 0, 0), (2, 18432, 0, 0), (2, 18437, 0, 0)])
def test_quantize_rows(M, K, gap, offset, dtype):
    A = _tokens(M, K, dtype, gap, offset=offset)
    print(f"[gpu] quantize_rows {M}x{K} {dtype}", flush=True)
    back = torch.full((M, K + 7), 99, dtype=torch.int8, device="cuda")
    Q, s = sq.soniq_quantize_rows(A, out=back[:, :K])
    q, sc = serve.quantize_rows(A.float().cpu().numpy())
    _same(Q, torch.from_numpy(q))
    _same(s, torch.from_numpy(sc))
    assert bool((back[:, K:] == 99).all())          # columns past K are left alone


def test_more_rows_than_workgroups():
    """Past 2^20 workgroups each takes several rows."""
    M, K = (1 << 20) + 300, 2056
    A = torch.randn((4096, K), device="cuda").to(torch.bfloat16).repeat(M // 4096 + 1, 1)[:M]
    A[(1 << 20):] *= 3
    print("[gpu] rows past 2^20", flush=True)
    Q, s = sq.soniq_quantize_rows(A)
    for part in (slice(0, 300), slice(M - 700, M)):
        q, t = sq.soniq_quantize_rows(A[part])
        assert torch.equal(Q[part], q) and torch.equal(s[part], t)


def test_quantize_rows_special():
    """Rows of zeros, ties, the smallest and largest values, infinities and
    NaN; each row by itself."""
    K = 300
    A = np.random.default_rng(0).standard_normal((10, K)).astype(np.float32)
    A[1] = 0
    A[2, 7] = np.inf
    A[3, 299] = np.nan
    A[4, 0] = -np.inf
    A[5] = 2.0**-149 * np.arange(K)
    A[6] *= 1e38 / np.abs(A[6]).max()
    A[7] = np.repeat([127, 0.5, 1.5, -2.5, 63.5, -0.5], 50)
    A[8] = -0.0
    A[9] = np.where(np.arange(K) == 4, np.nan, np.inf)
    Q, s = sq.soniq_quantize_rows(torch.from_numpy(A).cuda())
    q, sc = serve.quantize_rows(A)
    _same(Q, torch.from_numpy(q))
    _same(s, torch.from_numpy(sc))
    assert torch.isnan(s[3]) and torch.isinf(s[2]) and s[1] == 0


SHAPES = [  # M, N, K
    (1, 1, 1), (1, 16, 64), (1, 4096, 4096), (1, 100, 16389), (2, 130, 256), (3, 1030, 4091), (4, 64, 65536),
    (5, 11, 127), (7, 515, 512), (8, 4096, 1024), (9, 300, 640), (16, 128, 128), (17, 17, 17), (24, 1100, 96),
    (33, 4099, 257), (40, 256, 4096), (48, 33, 8192), (63, 65, 63), (64, 64, 64), (65, 129, 191), (100, 768, 768),
    (128, 128, 4096), (129, 257, 385), (200, 2304, 768), (256, 256, 256), (257, 511, 1000), (301, 199, 4091),
    (513, 1025, 129), (1000, 300, 2048), (2049, 140, 320), (1, 70000, 64), (4097, 65, 64), (512, 2560, 1152),
    (130, 1300, 2065), (100, 10000, 2049), (70, 19300, 130), (2050, 1300, 100), (300, 9000, 1000), (3900, 4100, 200),
    (4090, 4085, 300), (4096, 4096, 16), (66, 64, 1025), (64, 9999, 16), (200, 64, 15), (90, 30, 2000), (8200, 260, 16)]


@pytest.mark.parametrize("M,N,K", SHAPES, ids=lambda v: str(v))
@pytest.mark.parametrize("form", ["plain", "odd"])
def test_i8_gemm(M, N, K, form):
    """Codes of the whole int8 range; `odd`: leading dimensions and starts
    that no load width divides, a bias, fp16 into a wider output."""
    odd = form == "odd"
    A, a = _codes(M, K, 1, K + 5 if odd else K, 3 if odd else 0)
    W, w = _codes(N, K, 2, K + 9 if odd else K, 1 if odd else 0)
    r = np.random.default_rng(M + N + K)
    sa = np.exp(r.standard_normal(M)).astype(np.float32)
    sw = (np.exp(r.standard_normal(N)) / 1e3).astype(np.float32)
    bias = r.standard_normal(N).astype(np.float32) if odd else None
    dt = torch.float16 if odd else torch.bfloat16
    if odd:
        sa /= 64 * np.sqrt(K)                        # outputs inside fp16's range
    print(f"[gpu] i8_gemm {M}x{N}x{K} {form}", flush=True)
    wide = torch.full((M, N + 3), 7.0, dtype=dt, device="cuda")
    cuda = lambda x: None if x is None else torch.from_numpy(x).cuda()
    Y = sq.soniq_i8_gemm(A, cuda(sa), W, cuda(sw), bias=cuda(bias), out=wide[:, :N])
    want = torch.from_numpy(serve.i8_gemm(a, sa, w, sw, bias))
    _same(Y, want.to(dt))
    assert bool((wide[:, N:] == 7.0).all())
    Y32 = sq.soniq_i8_gemm(A, cuda(sa), W, cuda(sw), bias=cuda(bias), dtype=torch.float32)
    _same(Y32, want)


@pytest.mark.parametrize("M,N,K,gap", [(1, 4096, 4096, 0), (1, 33, 100, 3), (2, 1100, 768, 0), (3, 100, 8191, 1),
                                       (4, 256, 2048, 0), (5, 64, 512, 0), (8, 130, 11008, 0), (9, 40, 65, 0),
                                       (40, 300, 1024, 5), (300, 512, 640, 0), (1, 24, 65536, 0),
                                       (1, 100, 1, 0), (1, 70, 16384, 0), (1, 70, 16385, 1), (2, 40, 8192, 0), (2, 40, 513, 7),
                                       (3, 129, 63, 0), (4, 16, 4089, 0), (4, 16, 4097, 0), (4, 5000, 127, 2), (55, 8200, 300, 0), (16, 70, 1024, 0),
                                       (16, 70, 1025, 1), (13, 8300, 1257, 3), (2, 8300, 8192, 0), (16, 8200, 129, 0),
                                       (7, 33, 2336, 0), (15, 31, 65, 2), (17, 40, 64, 0), (11, 9000, 7, 1)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_quantize_i8_gemm_equals_the_two_calls(M, N, K, gap, dtype):
    A = _tokens(M, K, dtype, gap)
    A[M // 2] *= 0                                   # a token of zeros among the others
    W, w = _codes(N, K, 5)
    sw = torch.rand(N, device="cuda") / 100
    print(f"[gpu] quantize_i8_gemm {M}x{N}x{K} {dtype}", flush=True)
    Y = sq.soniq_quantize_i8_gemm(A, W, sw, dtype=TYPES[dtype])
    q, s = sq.soniq_quantize_rows(A)
    _same(Y, sq.soniq_i8_gemm(q, s, W, sw, dtype=TYPES[dtype]))
    qo, so = serve.quantize_rows(A.float().cpu().numpy())
    _same(Y, torch.from_numpy(serve.i8_gemm(qo, so, w, sw.cpu().numpy())).to(TYPES[dtype]))


@pytest.mark.parametrize("M", [1, 3, 40, 300])
def test_a_bad_token_spoils_itself_alone(M):
    A = _tokens(M, 512, "bf16", seed=3)
    clean = A.clone()
    A[0, 100], A[M // 2, 3] = float("nan"), float("inf")
    W, _ = _codes(200, 512, 5)
    sw = torch.rand(200, device="cuda") / 100
    Y, ref = sq.soniq_quantize_i8_gemm(A, W, sw), sq.soniq_quantize_i8_gemm(clean, W, sw)
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    bad[0] = bad[M // 2] = True
    assert bool(torch.isnan(Y[bad].float()).all())
    assert torch.equal(Y[~bad], ref[~bad])


@pytest.mark.parametrize("M,N", [(65, 300), (3, 40), (300, 70)])
def test_rows_far_apart(M, N):
    """Row strides past 2^24 bytes, and tokens more than 4 GiB from the first."""
    ld = (1 << 24) + 48
    r = np.random.default_rng(7)
    a = r.integers(-128, 128, (M, 200)).astype(np.int8)
    big = torch.empty((M, ld), dtype=torch.int8, device="cuda")
    A = big[:, 8:208]
    A.copy_(torch.from_numpy(a))
    W, w = _codes(N, 200, 8)
    sa, sw = torch.rand(M, device="cuda"), torch.rand(N, device="cuda") / 1000
    want = torch.from_numpy(serve.i8_gemm(a, sa.cpu().numpy(), w, sw.cpu().numpy()))
    _same(sq.soniq_i8_gemm(A, sa, W, sw, dtype=torch.float32), want)
    if M > 64:                                       # and as the weights
        _same(sq.soniq_i8_gemm(W, sw, A, sa, dtype=torch.float32),
              torch.from_numpy(serve.i8_gemm(w, sw.cpu().numpy(), a, sa.cpu().numpy())))


def test_two_graphs_share_a_workspace():
    """Two captured layers on one workspace, replayed in turn with eager calls
    on it between them."""
    W, _ = _codes(600, 512, 5)
    sw = torch.rand(600, device="cuda") / 100
    work = torch.empty(sq.soniq_quantize_i8_gemm_workspace(300, 512), dtype=torch.uint8, device="cuda")
    xs = [_tokens(300, 512, "bf16", seed=1), _tokens(20, 512, "bf16", seed=2)]
    want = [sq.soniq_quantize_i8_gemm(x, W, sw) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for x in xs:
        with torch.cuda.stream(side):
            sq.soniq_quantize_i8_gemm(x, W, sw, work=work)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(sq.soniq_quantize_i8_gemm(x, W, sw, work=work))
        graphs.append(g)
    for k in (0, 1, 1, 0, 0, 1):
        outs[k].zero_()
        graphs[k].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[k], want[k])
        assert torch.equal(sq.soniq_quantize_i8_gemm(xs[1 - k], W, sw, work=work), want[1 - k])
        torch.cuda.synchronize()


def test_a_given_stream_owns_what_the_call_allocates():
    """The current stream gets none of the memory that a call on another one
    still uses: its workspace, freed as the call returns, stays that stream's."""
    W, _ = _codes(256, 512, 5)
    sw = torch.rand(256, device="cuda") / 100
    x = _tokens(4096, 512, "bf16", seed=3)
    want = sq.soniq_quantize_i8_gemm(x, W, sw)
    need = sq.soniq_quantize_i8_gemm_workspace(4096, 512)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)                # the call waits behind this
    got = sq.soniq_quantize_i8_gemm(x, W, sw, stream=side.cuda_stream)
    mine = torch.full((need,), 77, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert bool((mine == 77).all())
    assert torch.equal(got, want)
    q, s = sq.soniq_quantize_rows(x, stream=torch.cuda.default_stream().cuda_stream)
    assert torch.equal(sq.soniq_i8_gemm(q, s, W, sw, stream=0), want)


def test_binding_refusals():
    """What the binding refuses before the library sees it."""
    x = torch.randn((4, 64), device="cuda")
    W, _ = _codes(20, 64, 5)
    sw = torch.rand(20, device="cuda")
    bad = [(TypeError, lambda: sq.soniq_quantize_rows(x.t())), (TypeError, lambda: sq.soniq_quantize_rows(x.double())),
           (TypeError, lambda: sq.soniq_quantize_rows(x[:1].expand(4, 64))), (TypeError, lambda: sq.soniq_quantize_rows(x[0])),
           (ValueError, lambda: sq.soniq_quantize_rows(x, scales=torch.empty(3, device="cuda"))),
           (TypeError, lambda: sq.soniq_quantize_rows(x, out=torch.empty((4, 64), device="cuda"))),
           (ValueError, lambda: sq.soniq_quantize_i8_gemm(x[:, :32], W, sw)),
           (TypeError, lambda: sq.soniq_quantize_i8_gemm(x, W.float(), sw)),
           (ValueError, lambda: sq.soniq_quantize_i8_gemm(x, W, sw[:3])),
           (TypeError, lambda: sq.soniq_quantize_i8_gemm(x, W, sw.cpu())),
           (TypeError, lambda: sq.soniq_quantize_i8_gemm(x, W, sw, dtype=torch.float64)),
           (ValueError, lambda: sq.soniq_quantize_i8_gemm(x, W, sw, out=torch.empty((4, 21), device="cuda"))),
           (sq.SoniqError, lambda: sq.soniq_quantize_i8_gemm(torch.randn((17, 64), device="cuda"), W, sw,
                                                             work=torch.empty(16, dtype=torch.uint8, device="cuda"))),
           (TypeError, lambda: sq.soniq_i8_gemm(x, sw, W, sw))]
    for error, call in bad:
        with pytest.raises(error):
            call()


def test_no_tokens():
    W, _ = _codes(20, 64, 5)
    sw = torch.rand(20, device="cuda")
    assert sq.soniq_quantize_i8_gemm(torch.empty((0, 64), device="cuda"), W, sw).shape == (0, 20)


def test_streams_and_shared_weights():
    """Two streams at once, each with its own workspace, on one weight matrix."""
    W, w = _codes(1024, 1024, 5)
    sw = torch.rand(1024, device="cuda") / 100
    xs = [_tokens(M, 1024, "bf16", seed=M) for M in (1, 200)]
    want = [sq.soniq_quantize_i8_gemm(x, W, sw) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(4):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[k].append(sq.soniq_quantize_i8_gemm(xs[k], W, sw))
    torch.cuda.synchronize()
    for k in (0, 1):
        for y in got[k]:
            assert torch.equal(y, want[k])
