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
