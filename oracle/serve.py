"""Plain implementations of the 8-bit linear layers and the quantized
key/value cache, in numpy: written from the formulas, sharing nothing with
the HIP path.  Codes and scales follow the codec's definition (fp32
divisions, ties to even), so they are compared bit for bit; attention is
computed in float64."""
from __future__ import annotations

import numpy as np

F32 = np.float32


def quantize_rows(x, top=127.0):
    """Codes (int8) and scales (float32) over the last axis of float32 x."""
    x = np.asarray(x, F32)
    with np.errstate(all="ignore"):
        amax = np.abs(x).max(-1, keepdims=True)            # NaN where the row has one
        s = (amax / F32(top)).astype(F32)
        q = np.rint((x / s).astype(F32))
        ok = (s > 0) & np.isfinite(s)
        q = np.where(ok, np.clip(np.where(ok, q, 0), -top, top), 0).astype(np.int8)
    return q, s[..., 0]


def i8_gemm(qa, sa, qw, sw, bias=None):
    """float32 outputs before their rounding to the output type: the fixed
    order (float(acc) * s_a) * s_w + bias."""
    acc = qa.astype(np.float64) @ qw.astype(np.float64).T   # sums of integers below 2^53: exact
    assert np.abs(acc).max(initial=0) < 2**31
    acc = acc.astype(np.int32)
    with np.errstate(all="ignore"):
        y = (acc.astype(F32) * sa[:, None].astype(F32)).astype(F32)
        y = (y * sw[None, :].astype(F32)).astype(F32)
        return y if bias is None else (y + bias[None, :].astype(F32)).astype(F32)


def pack_codes(q, bits):
    """Codes [..., D] as stored bytes (uint8)."""
    if bits == 8:
        return q.astype(np.int8).view(np.uint8)
    u = q.astype(np.int64) & 15
    return (u[..., 0::2] | (u[..., 1::2] << 4)).astype(np.uint8)


def unpack_codes(b, bits):
    b = np.asarray(b).view(np.uint8)
    if bits == 8:
        return b.view(np.int8).astype(np.int64)
    lo, hi = (b & 15).astype(np.int64), (b >> 4).astype(np.int64)
    out = np.stack((lo, hi), -1).reshape(*b.shape[:-1], -1)
    return out - 16 * (out > 7)


def place(table, pages, page_size, b, pos):
    """(page, row in it) of a position, or None."""
    if pos < 0 or pos >= table.shape[1] * page_size:
        return None
    p = int(table[b, pos // page_size])
    return (p, pos % page_size) if 0 <= p < pages else None


def kv_write(codes, scales, rows, table, cu, start, bits):
    """Writes float32 rows [T, H, D] into codes [P, H, S, W] and scales
    [P, H, S] in place."""
    P, _, S, _ = codes.shape
    q, s = quantize_rows(rows, 127.0 if bits == 8 else 7.0)
    packed = pack_codes(q, bits)
    for b in range(table.shape[0]):
        for i in range(int(cu[b + 1]) - int(cu[b])):
            at = place(table, P, S, b, int(start[b]) + i)
            if at is not None:
                codes[at[0], :, at[1]] = packed[cu[b] + i]
                scales[at[0], :, at[1]] = s[cu[b] + i]


def kv_rows(codes, scales, table, b, positions, bits):
    """(codes int64 [n, H, D], scales float32 [n, H], present [n])."""
    P, H, S, W = codes.shape
    n = len(positions)
    c = np.zeros((n, H, W * 8 // bits), np.int64)
    s = np.zeros((n, H), F32)
    there = np.zeros(n, bool)
    for k, pos in enumerate(positions):
        at = place(table, P, S, b, int(pos))
        if at is not None:
            c[k], s[k], there[k] = unpack_codes(codes[at[0], :, at[1]], bits), scales[at[0], :, at[1]], True
    return c, s, there


def kv_read(codes, scales, table, cu, start, bits):
    """float32 values [cu[B], H, D] (code * scale in one fp32 product)."""
    out = [np.zeros((0, codes.shape[1], codes.shape[3] * 8 // bits), F32)]
    for b in range(table.shape[0]):
        n = int(cu[b + 1]) - int(cu[b])
        c, s, _ = kv_rows(codes, scales, table, b, [int(start[b]) + i for i in range(n)], bits)
        with np.errstate(all="ignore"):
            out.append(c.astype(F32) * s[..., None])
    return np.concatenate(out)


def attention(q, kc, ks, vc, vs, table, cu, kv_len, bits, scale, mask=None, weight=2.0**-11, exact_sums=False):
    """float64 attention of q [T, Hq, D] over the cache.  Returns (out, lse,
    bound): bound is what rounding the softmax weights and fp32 sums can move
    an output by, before its own rounding:
      - a weight is off by at most `weight` of itself (2^-11: one fp16
        number), or by 2^-25 of the largest weight where it is subnormal;
      - a score is off by (D + 16) roundings of 2^-24 of sum |q k| (and of
        its own size for the scalings and the exponent), which moves a weight
        by that much, relatively, in the numerator and in the sum;
        exact_sums: q and codes are integers whose sums fp32 holds, in any
        order, so that only the roundings of the scalings are left;
      - sums of n terms in fp32 add n roundings of 2^-24."""
    T, Hq, D = q.shape
    P, H, S, _ = kc.shape
    G = Hq // H
    out, lse, bound = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf), np.zeros((T, Hq, D))
    for b in range(table.shape[0]):
        n, length = int(cu[b + 1]) - int(cu[b]), int(kv_len[b])
        L = max(0, min(length, table.shape[1] * S))
        base = length - n
        ck, sk, there = kv_rows(kc, ks, table, b, range(L), bits)
        cv, sv, _ = kv_rows(vc, vs, table, b, range(L), bits)
        pos = np.arange(L)
        for i in range(n):
            t = int(cu[b]) + i
            j = pos - base
            if mask is None:
                seen = j <= i
            else:
                words = mask[t].view(np.uint64)
                bit = np.zeros(L, bool)
                new = (j >= 0) & (j < 64 * len(words))
                bit[new] = [(int(words[x // 64]) >> (x % 64)) & 1 for x in j[new].tolist()]
                seen = (j < 0) | bit
            seen &= there
            if not seen.any():
                continue
            for h in range(H):
                K = ck[seen, h].astype(np.float64) * sk[seen, h].astype(np.float64)[:, None]
                V = cv[seen, h].astype(np.float64) * sv[seen, h].astype(np.float64)[:, None]
                for g in range(G):
                    x = q[t, h * G + g].astype(np.float64)
                    with np.errstate(all="ignore"):
                        z = scale * (K @ x)
                        m = z.max()
                        e = np.exp(z - m)
                        p = e / e.sum()
                        out[t, h * G + g] = p @ V
                        lse[t, h * G + g] = m + np.log(e.sum())
                        size = abs(scale) * (np.abs(K) @ np.abs(x))
                        ds = 8 * 2.0**-24 * (1 + np.abs(z).max())
                        if not exact_sums:
                            ds += (D + 16) * 2.0**-24 * size.max()
                            # the fp16 grid of q: relative to the row's largest element
                            ds += abs(scale) * 2.0**-24 * np.abs(x).max(initial=0) * np.abs(K).sum(1).max()
                        A = p @ np.abs(V)
                        top = (p * sv[seen, h]).max() * np.abs(cv[seen, h]).sum(0)
                        bound[t, h * G + g] = A * (weight + 2 * ds + len(z) * 2.0**-24) + 2.0**-25 * top
    return out, lse, bound
