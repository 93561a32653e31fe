"""The 8-bit linear layers and the quantized cache without a GPU: every
refusal happens on the host, before any device work; the cache's index
arithmetic, compiled here from the header that the kernels include, stays
inside the cache whatever the tables hold; the oracle is held to
hand-worked and brute-force cases."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2311_14114_amd as sq
from oracle import serve

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000                      # never dereferenced: validation fails first
BAD, UNSUP = sq.SONIQ_ERR_INVALID_ARGUMENT, sq.SONIQ_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(sq.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return sq.lib()


def _with(base, **changes):
    return [changes.get(k, v) for k, v in base.items()]


ROWS = dict(A=FAKE, type=0, M=4, K=32, lda=32, Q=FAKE, ldq=32, s=FAKE, stream=None)
GEMM = dict(A=FAKE, lda=32, s_a=FAKE, W=FAKE, ldw=32, s_w=FAKE, bias=None, M=4, N=8, K=32, Y=FAKE, y_type=1, ldy=8,
            stream=None)
BOTH = dict(A=FAKE, type=0, lda=32, W=FAKE, ldw=32, s_w=FAKE, bias=None, M=20, N=8, K=32, Y=FAKE, y_type=1, ldy=8,
            work=FAKE, bytes=1 << 20, stream=None)


@pytest.mark.parametrize("fn,base,changes,status", [
    ("rows", ROWS, dict(A=None), BAD), ("rows", ROWS, dict(type=3), BAD), ("rows", ROWS, dict(type=-1), BAD),
    ("rows", ROWS, dict(M=-1), BAD), ("rows", ROWS, dict(K=0), BAD), ("rows", ROWS, dict(lda=31), BAD),
    ("rows", ROWS, dict(ldq=31), BAD), ("rows", ROWS, dict(Q=None), BAD), ("rows", ROWS, dict(s=None), BAD),
    ("rows", ROWS, dict(A=FAKE + 2), BAD), ("rows", ROWS, dict(s=FAKE + 2), BAD),
    ("rows", ROWS, dict(K=65537, lda=65537, ldq=65537), UNSUP), ("rows", ROWS, dict(M=1 << 31), UNSUP),
    ("gemm", GEMM, dict(A=None), BAD), ("gemm", GEMM, dict(W=None), BAD), ("gemm", GEMM, dict(s_a=None), BAD),
    ("gemm", GEMM, dict(s_w=None), BAD), ("gemm", GEMM, dict(Y=None), BAD), ("gemm", GEMM, dict(lda=31), BAD),
    ("gemm", GEMM, dict(ldw=31), BAD), ("gemm", GEMM, dict(ldy=7), BAD), ("gemm", GEMM, dict(N=0), BAD),
    ("gemm", GEMM, dict(K=0), BAD), ("gemm", GEMM, dict(M=-1), BAD), ("gemm", GEMM, dict(y_type=5), BAD),
    ("gemm", GEMM, dict(Y=FAKE + 1), BAD), ("gemm", GEMM, dict(bias=FAKE + 1), BAD),
    ("gemm", GEMM, dict(K=70000, lda=70000, ldw=70000), UNSUP), ("gemm", GEMM, dict(N=1 << 31, ldy=1 << 31), UNSUP),
    ("gemm", GEMM, dict(M=(1 << 30) - 64), UNSUP), ("gemm", GEMM, dict(M=1 << 16, N=1 << 20, ldy=1 << 20), UNSUP),
    ("both", BOTH, dict(A=None), BAD), ("both", BOTH, dict(W=None), BAD), ("both", BOTH, dict(work=None), BAD),
    ("both", BOTH, dict(work=FAKE + 8), BAD), ("both", BOTH, dict(bytes=20 * 32 + 79), BAD),
    ("both", BOTH, dict(lda=31), BAD), ("both", BOTH, dict(y_type=9), BAD)],
    ids=lambda v: str(v) if isinstance(v, (str, int)) else "-".join(v) if isinstance(v, dict) and len(v) < 4 else "")
def test_linear_refusals(L, fn, base, changes, status):
    f = {"rows": L.soniq_quantize_rows, "gemm": L.soniq_i8_gemm, "both": L.soniq_quantize_i8_gemm}[fn]
    assert f(*_with(base, **changes)) == status
    assert L.soniq_last_error().startswith(b"soniq_")


def _cache(**changes):
    c = dict(k=FAKE, k_scale=FAKE, v=FAKE, v_scale=FAKE, pages=4, page_size=16, heads=2, head_dim=64, bits=8)
    c.update(changes)
    return sq.KVCacheStruct(*c.values())


COPY = dict(cache=None, K=FAKE, kt=128, kh=64, V=FAKE, vt=128, vh=64, type=1, T=3, table=FAKE, ld=2, width=2, B=2,
            cu=FAKE, start=FAKE, stream=None)
ATTEND = dict(cache=None, q=FAKE, qt=256, qh=64, type=1, T=3, heads=4, table=FAKE, ld=2, width=2, B=2, cu=FAKE,
              kv_len=FAKE, mask=None, words=0, scale=0.125, max_q=2, max_kv=32, out=FAKE, ot=256, oh=64, lse=None,
              work=FAKE, bytes=1 << 40, stream=None)
TABLES = [(dict(table=None), BAD), (dict(cu=None), BAD), (dict(ld=1), BAD), (dict(width=0), BAD), (dict(B=-1), BAD),
          (dict(T=-1), BAD), (dict(table=FAKE + 2), BAD), (dict(B=1 << 16), UNSUP),
          (dict(width=1 << 28, ld=1 << 28), UNSUP)]


@pytest.mark.parametrize("changes,status", TABLES + [
    (dict(start=None), BAD), (dict(K=None), BAD), (dict(V=None), BAD), (dict(type=7), BAD), (dict(V=FAKE + 1), BAD)],
    ids=str)
@pytest.mark.parametrize("fn", ["write", "read"])
def test_copy_refusals(L, fn, changes, status):
    c = _cache()
    f = L.soniq_kv_write if fn == "write" else L.soniq_kv_read
    assert f(*_with(COPY, cache=ctypes.addressof(c), **changes)) == status
    assert L.soniq_last_error().startswith(b"soniq_kv_" + fn.encode())


@pytest.mark.parametrize("changes,status", TABLES + [
    (dict(kv_len=None), BAD), (dict(q=None), BAD), (dict(out=None), BAD), (dict(type=0), BAD), (dict(heads=3), BAD),
    (dict(heads=0), BAD), (dict(max_q=0), BAD), (dict(max_kv=-1), BAD), (dict(max_q=257), UNSUP),
    (dict(mask=FAKE), BAD), (dict(words=1), BAD), (dict(mask=FAKE, words=5), BAD), (dict(mask=FAKE + 4, words=1), BAD),
    (dict(work=FAKE + 8), BAD), (dict(lse=FAKE + 2), BAD), (dict(scale=float("nan")), BAD),
    (dict(scale=float("inf")), BAD)], ids=str)
def test_attention_refusals(L, changes, status):
    c = _cache()
    assert L.soniq_kv_attention(*_with(ATTEND, cache=ctypes.addressof(c), **changes)) == status
    assert L.soniq_last_error().startswith(b"soniq_kv_attention")


@pytest.mark.parametrize("changes,status", [
    (dict(k=None), BAD), (dict(v_scale=None), BAD), (dict(k=FAKE + 8), BAD), (dict(k_scale=FAKE + 1), BAD),
    (dict(pages=0), BAD), (dict(page_size=0), BAD), (dict(heads=0), BAD), (dict(head_dim=96), UNSUP),
    (dict(head_dim=512), UNSUP), (dict(bits=2), UNSUP), (dict(pages=1 << 31), UNSUP),
    (dict(pages=1 << 20, page_size=1 << 10), UNSUP)], ids=str)
def test_cache_refusals(L, changes, status):
    c = _cache(**changes)
    at = ctypes.addressof(c)
    assert L.soniq_kv_write(*_with(COPY, cache=at)) == status
    assert L.soniq_kv_attention(*_with(ATTEND, cache=at)) == status
    n = ctypes.c_int64()
    assert L.soniq_kv_attention_workspace(at, 3, 4, 2, 2, 32, ctypes.byref(n)) == status
    assert L.soniq_kv_read(*_with(COPY, cache=None)) == BAD


def test_nothing_to_do_is_ok(L):
    at = ctypes.addressof(c := _cache())
    assert L.soniq_quantize_rows(*_with(ROWS, M=0, A=None, Q=None, s=None)) == 0
    assert L.soniq_i8_gemm(*_with(GEMM, M=0, A=None, s_a=None, Y=None)) == 0
    assert L.soniq_quantize_i8_gemm(*_with(BOTH, M=0, A=None, Y=None, work=None, bytes=0)) == 0
    for k in ("T", "B"):
        assert L.soniq_kv_write(*_with(COPY, cache=at, **{k: 0})) == 0
        assert L.soniq_kv_read(*_with(COPY, cache=at, **{k: 0}, K=None, V=None)) == 0
        assert L.soniq_kv_attention(*_with(ATTEND, cache=at, **{k: 0}, q=None, out=None)) == 0
    assert c.pages == 4


def test_workspaces(L):
    n = ctypes.c_int64(-1)
    for M, K in ((17, 100), (16, 1025), (1, 16385)):
        assert L.soniq_quantize_i8_gemm_workspace(M, K, ctypes.byref(n)) == 0
        assert n.value >= M * K + M * 4
    for M, K in ((0, 100), (1, 16384), (4, 100), (16, 1024)):  # quantized where they are used
        assert L.soniq_quantize_i8_gemm_workspace(M, K, ctypes.byref(n)) == 0 and n.value == 0
    for bad in ((-1, 4), (4, 0)):
        assert L.soniq_quantize_i8_gemm_workspace(*bad, ctypes.byref(n)) == BAD
    assert L.soniq_quantize_i8_gemm_workspace(4, 4, None) == BAD
    c = _cache()
    assert L.soniq_kv_attention_workspace(ctypes.addressof(c), 3, 4, 2, 2, 32, None) == BAD


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros((2, 4))
    with pytest.raises(TypeError):
        sq.soniq_quantize_rows(x)
    with pytest.raises(TypeError):
        sq.KVCache(x, x, x, x)


SLOT_MAIN = r"""
#include "soniq_kv_slot.h"
using namespace soniq;
extern "C" int row(const int32_t* page, int64_t ld, int width, int B, int pages, int page_size, int heads, int b, int64_t pos) {
  return kv_row(KvTable{page, ld, width, B}, KvDims{pages, page_size, heads, 64, 8}, b, pos);
}
extern "C" void span(int lo, int hi, int total, int* out) {
  const KvSpan s = kv_span(lo, hi, total);
  out[0] = s.first;
  out[1] = s.count;
}
extern "C" int length(int width, int page_size, int len) {
  return kv_length(KvTable{nullptr, width, width, 1}, KvDims{1, page_size, 1, 64, 8}, len);
}
"""


@pytest.fixture(scope="module")
def slot(tmp_path_factory):
    d = tmp_path_factory.mktemp("slot")
    (d / "slot.cpp").write_text(SLOT_MAIN)
    so = str(d / "slot.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2311_14114_amd", "csrc"), str(d / "slot.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    i, q, p = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p
    lib.row.argtypes = [p, q, i, i, i, i, i, i, q]
    lib.span.argtypes = [i, i, i, p]
    lib.length.argtypes = [i, i, i]
    return lib


EDGE = [-2**31, -2**31 + 1, -7, -1, 0, 1, 2, 3, 100, 2**31 - 2, 2**31 - 1]


def test_rows_stay_inside_the_cache(slot):
    """Tables of garbage, positions of any sign and size: a row inside the
    cache, the right one, or none."""
    r = np.random.default_rng(0)
    for pages, size, heads, width in ((5, 7, 3, 4), (1, 1, 1, 1), (1 << 14, 16, 8, 300), (3, 1 << 29, 1, 3)):
        if pages * size * heads >= 2**31 or width * size >= 2**31:
            size //= 4
        table = r.integers(-2, pages + 2, (3, width + 1)).astype(np.int32)
        table[0, 0], table[1, -2], table[2, width // 2] = -2**31, 2**31 - 1, pages - 1
        ends = [-1, 0, size - 1, size, width * size - 1, width * size, -2**40, 2**62, -2**63, 2**32]
        for pos in ends + r.integers(-5, width * size + 5, 300).tolist():
            for b in range(3):
                got = slot.row(table.ctypes.data, width + 1, width, 3, pages, size, heads, b, pos)
                at = serve.place(table[:, :width], pages, size, b, pos)
                want = -1 if at is None else at[0] * heads * size + at[1]
                assert got == want
                assert got + (heads - 1) * size < pages * heads * size


def test_spans_and_lengths_stay_inside_the_batch(slot):
    out = (ctypes.c_int * 2)()
    for lo in EDGE:
        for hi in EDGE:
            for total in (0, 1, 3, 2**31 - 1):
                slot.span(lo, hi, total, out)
                assert 0 <= out[0] <= total and 0 <= out[1] <= total - out[0]
                if 0 <= lo <= hi <= total:
                    assert (out[0], out[1]) == (lo, hi - lo)
    for width, size in ((1, 1), (7, 16), (2**20, 2**10 - 1)):
        for n in EDGE:
            assert slot.length(width, size, n) == max(0, min(n, width * size))


# ----------------------------------------------------------------- oracle --
def test_oracle_codec_by_brute_force():
    """Every code is the nearest of the grid to x / s (ties aside), the
    largest element takes the largest code, and 4-bit bytes unpack to what
    was packed."""
    r = np.random.default_rng(1)
    for top, bits in ((127, 8), (7, 4)):
        x = r.standard_normal((50, 64)).astype(np.float32)
        q, s = serve.quantize_rows(x, float(top))
        grid = np.arange(-top, top + 1) * s[:, None, None].astype(np.float64)
        best = np.abs(x[..., None].astype(np.float64) - grid).min(-1)
        mine = np.abs(x - q * s[:, None].astype(np.float64))
        assert (mine <= best * (1 + 1e-5)).all()
        assert (np.abs(q).max(1) == top).all()
        np.testing.assert_array_equal(serve.unpack_codes(serve.pack_codes(q, bits), bits), q)
    q, s = serve.quantize_rows(np.array([[7, 0.5, 1.5, -2.5, 3.5]], np.float32), 7.0)
    assert s[0] == 1 and q[0].tolist() == [7, 0, 2, -2, 4]
    assert serve.pack_codes(np.array([1, -1]), 4).tolist() == [0xF1]


def test_oracle_attention_by_hand():
    """Two positions with equal scores average their values; a mask leaves
    one of them; a weight of 3 to 1 comes out of ln 3."""
    codes = np.zeros((1, 1, 2, 64), np.uint8)
    v = codes.copy()
    v[0, 0, 0, 0], v[0, 0, 1, 0] = 10, 30
    one = np.ones((1, 1, 2), np.float32)
    table, cu = np.zeros((1, 1), np.int32), [0, 1]
    q = np.ones((1, 1, 64), np.float32)
    out, lse, _ = serve.attention(q, codes, one, v, one, table, cu, [2], 8, 1.0)
    assert out[0, 0, 0] == 20 and abs(lse[0, 0] - np.log(2)) < 1e-12
    out, lse, _ = serve.attention(q, codes, one, v, one, table, cu, [2], 8, 1.0, np.zeros((1, 1), np.int64))
    assert out[0, 0, 0] == 10 and lse[0, 0] == 0
    k = codes.copy()
    k[0, 0, 1, 0] = 1
    out, _, _ = serve.attention(q, k, one, v, one, table, cu, [2], 8, float(np.log(3)))
    assert abs(out[0, 0, 0] - 25) < 1e-12
    out, lse, _ = serve.attention(q, k, one, v, one, table, cu, [0], 8, 1.0)
    assert (out == 0).all() and np.isneginf(lse).all()
