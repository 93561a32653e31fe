"""The attention oracle's bound tells weights of one fp16 number from weights
of two: a plain implementation with either rounding, on the CPU."""
import numpy as np
import pytest

from oracle import serve


def _case(bits, top):
    r = np.random.default_rng(31)
    page, D, G, n = 16, 128, 4, 96
    mk = lambda: serve.pack_codes(r.integers(-top, top + 1, (n // page, 1, page, D)), bits)
    sc = lambda: (np.exp(0.3 * r.standard_normal((n // page, 1, page))) / top * 2).astype(np.float32)
    cache = mk(), sc(), mk(), sc()
    table = np.arange(n // page, dtype=np.int32)[None]
    return cache, table, r.integers(-3, 4, (8, G, D)).astype(np.float32)


def _weighed(cache, table, q, bits, scale, parts):
    """Attention with every weight p * s_v, in units of a power of two below
    the row's largest, held as the sum of `parts` fp16 numbers, each the
    rounded rest of those before."""
    kc, ks, vc, vs = cache
    n = table.shape[1] * kc.shape[2]
    out = np.zeros(q.shape)
    ck, sk, _ = serve.kv_rows(kc, ks, table, 0, range(n), bits)
    cv, sv, _ = serve.kv_rows(vc, vs, table, 0, range(n), bits)
    K, s = ck[:, 0] * sk[:, :1].astype(np.float64), sv[:, 0].astype(np.float64)
    for t in range(q.shape[0]):
        m = n - q.shape[0] + t + 1                    # as far as this token sees
        z = scale * (q[t].astype(np.float64) @ K[:m].T)
        p = np.exp(z - z.max(-1, keepdims=True))
        unit = 2.0**np.floor(np.log2((p * s[:m]).max(-1, keepdims=True)))
        w = p * s[:m] / unit
        held = np.zeros_like(w)
        for _ in range(parts):
            held += (w - held).astype(np.float16).astype(np.float64)
        out[t] = unit * (held @ cv[:m, 0]) / p.sum(-1, keepdims=True)
    return out


@pytest.mark.parametrize("bits,scale", [(8, 0.15), (4, 0.1)])
def test_a_dropped_second_part_is_seen(bits, scale):
    cache, table, q = _case(bits, 127 if bits == 8 else 7)
    args = (q, *cache, table, [0, 8], [96], bits, scale)
    want, _, wide = serve.attention(*args)
    _, _, close = serve.attention(*args, weight=2.0**-21, exact_sums=True)
    one, two = (_weighed(cache, table, q, bits, scale, k) for k in (1, 2))
    assert (np.abs(one - want) <= wide).all()
    assert (np.abs(two - want) <= close).all()
    for eps in (2.0**-11, 2.0**-8):                   # half a step of fp16 and of bf16 outputs
        held = lambda x: (x.astype(np.float16) if eps < 2.0**-9 else _bf16(x)).astype(np.float64)
        limit = close + eps * (np.abs(want) + close)
        assert (np.abs(held(two) - want) <= limit).all()
        assert (np.abs(held(one) - want) > limit).sum() > 10


def _bf16(x):
    u = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + (u >> 16 & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
