// Host side of the 8-bit linear layers and the quantized key/value cache:
// argument checks, workspaces, dispatch.
#include <cmath>
#include <cstdarg>
#include <cstdint>

#include "soniq.h"
#include "soniq_internal.h"
#include "soniq_serve.h"

using namespace soniq;

namespace {

soniq_status fail(soniq_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  set_error(st, fmt, ap);
  va_end(ap);
  return st;
}

#define HIP_TRY(expr)                                                                       \
  do {                                                                                      \
    hipError_t e_ = (expr);                                                                 \
    if (e_ != hipSuccess)                                                                   \
      return fail(e_ == hipErrorOutOfMemory ? SONIQ_ERR_OUT_OF_MEMORY : SONIQ_ERR_HIP,      \
                  "%s failed: %s", #expr, hipGetErrorString(e_));                           \
  } while (0)

// Refuses a call: bad arguments, or sizes beyond this build's limits.
#define NEED(cond, ...)                                              \
  do {                                                               \
    if (!(cond)) return fail(SONIQ_ERR_INVALID_ARGUMENT, __VA_ARGS__); \
  } while (0)
#define LIMIT(cond, ...)                                           \
  do {                                                             \
    if (!(cond)) return fail(SONIQ_ERR_UNSUPPORTED, __VA_ARGS__);    \
  } while (0)

constexpr int64_t kMax31 = (int64_t)1 << 31;
constexpr int64_t kMaxGroups = (int64_t)1 << 24;  // workgroups of 256 threads in a launch: 2^32 threads are too many

int type_size(int type) { return type == SONIQ_F32 ? 4 : type == SONIQ_BF16 || type == SONIQ_F16 ? 2 : 0; }

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

hipStream_t hip_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

soniq_status check_quantize(const char* who, const void* A, int a_type, int64_t M, int64_t K,
                            int64_t lda) {
  NEED(type_size(a_type), "%s: a_type %d is not SONIQ_F32, SONIQ_BF16 or SONIQ_F16", who, a_type);
  NEED(M >= 0 && K >= 1 && lda >= K, "%s: M = %lld, K = %lld, lda = %lld", who, (long long)M,
       (long long)K, (long long)lda);
  NEED(A || M == 0, "%s: null A", who);
  NEED(aligned(A, type_size(a_type)), "%s: A is not aligned to its elements", who);
  LIMIT(K <= SONIQ_MAX_K && M < kMax31, "%s: M = %lld, K = %lld (M < 2^31, K <= %d)", who,
        (long long)M, (long long)K, SONIQ_MAX_K);
  return SONIQ_OK;
}

soniq_status check_gemm(const char* who, const void* W, int64_t ldw, const float* s_w,
                        const float* bias, int64_t M, int64_t N, int64_t K, const void* Y,
                        int y_type, int64_t ldy) {
  NEED(type_size(y_type), "%s: y_type %d is not SONIQ_F32, SONIQ_BF16 or SONIQ_F16", who, y_type);
  NEED(M >= 0 && N >= 1 && K >= 1, "%s: M = %lld, N = %lld, K = %lld", who, (long long)M,
       (long long)N, (long long)K);
  NEED(ldw >= K && ldy >= N, "%s: ldw = %lld < K or ldy = %lld < N", who, (long long)ldw,
       (long long)ldy);
  NEED(W && s_w && (Y || M == 0), "%s: null pointer", who);
  NEED(aligned(s_w, 4) && aligned(bias, 4) && aligned(Y, type_size(y_type)),
       "%s: s_w, bias or Y is not aligned to its elements", who);
  LIMIT(K <= SONIQ_MAX_K && M < kMax31 && N < kMax31 / 32 && ((M + 63) / 64) * ((N + 63) / 64) < kMaxGroups - 8,
        "%s: M = %lld, N = %lld, K = %lld (M < 2^31, N < 2^26, M * N / 4096 < 2^24 - 8, K <= %d)", who,
        (long long)M, (long long)N, (long long)K, SONIQ_MAX_K);
  return SONIQ_OK;
}

// Workspace of soniq_quantize_i8_gemm where it takes two launches: the codes,
// then the scales.  Rows are padded past a multiple of 128 bytes, so that the
// same chunk of neighbouring rows does not fall on one cache channel (8192^3:
// 497 us on token rows of 8192 bytes, 468 on 8320; weights' rows take either).
int64_t codes_ld(int64_t K) { return round_up(K, 128) + 128; }
int64_t i8_work(int64_t M, int64_t K) {
  return i8_fused(M, K) ? 0 : M * codes_ld(K) + round_up(4 * M, 16);
}

soniq_status check_cache(const char* who, const soniq_kv_cache_t* c) {
  NEED(c, "%s: null cache", who);
  NEED(c->k_dev && c->v_dev && c->k_scale_dev && c->v_scale_dev, "%s: null pointer in the cache", who);
  NEED(aligned(c->k_dev, 16) && aligned(c->v_dev, 16) && aligned(c->k_scale_dev, 4) &&
           aligned(c->v_scale_dev, 4),
       "%s: cache codes are 16-byte, scales 4-byte aligned", who);
  NEED(c->pages >= 1 && c->page_size >= 1 && c->heads >= 1,
       "%s: cache of %lld pages, page_size %d, %d heads", who, (long long)c->pages, c->page_size,
       c->heads);
  LIMIT(c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 192 || c->head_dim == 256,
        "%s: head_dim %d (64, 128, 192 and 256 are supported)", who, c->head_dim);
  LIMIT(c->bits == 4 || c->bits == 8, "%s: %d-bit cache (4 and 8 are supported)", who, c->bits);
  LIMIT(c->heads < (1 << 14) && c->pages < kMax31 &&
            (int64_t)c->heads * c->page_size < kMax31 &&
            c->pages * ((int64_t)c->heads * c->page_size) < kMax31,
        "%s: %lld pages of %d rows for %d heads (2^31 rows or more)", who, (long long)c->pages,
        c->page_size, c->heads);
  return SONIQ_OK;
}

soniq_status check_table(const char* who, const soniq_kv_cache_t* c, const int32_t* table,
                         int64_t ld, int64_t width, int64_t B, const int32_t* cu,
                         const int32_t* other, int64_t T) {
  NEED(B >= 0 && T >= 0 && width >= 1 && ld >= width,
       "%s: B = %lld, T = %lld, table_width = %lld, table_ld = %lld", who, (long long)B, (long long)T,
       (long long)width, (long long)ld);
  NEED((table && cu && other) || B == 0 || T == 0, "%s: null table, cu or lengths", who);
  NEED(aligned(table, 4) && aligned(cu, 4) && aligned(other, 4), "%s: tables are int32, 4-byte aligned", who);
  LIMIT(B <= 65535 && T < kMaxGroups && width < kMax31 && width * (int64_t)c->page_size < kMax31,
        "%s: B = %lld, T = %lld, table_width = %lld (B < 2^16, T < 2^24, table_width * page_size < 2^31)",
        who, (long long)B, (long long)T, (long long)width);
  return SONIQ_OK;
}

KvDims dims_of(const soniq_kv_cache_t* c) {
  return {(int32_t)c->pages, c->page_size, c->heads, c->head_dim, c->bits};
}

soniq_status kv_copy(const char* who, bool write, const soniq_kv_cache_t* cache, void* K,
                     int64_t k_ts, int64_t k_hs, void* V, int64_t v_ts, int64_t v_hs, int type,
                     int64_t T, const int32_t* table, int64_t ld, int64_t width, int64_t B,
                     const int32_t* cu, const int32_t* start, void* stream) {
  if (soniq_status st = check_cache(who, cache)) return st;
  if (soniq_status st = check_table(who, cache, table, ld, width, B, cu, start, T)) return st;
  const int e = type_size(type);
  NEED(e, "%s: type %d is not SONIQ_F32, SONIQ_BF16 or SONIQ_F16", who, type);
  NEED((K && V) || B == 0 || T == 0, "%s: null K or V", who);
  NEED(aligned(K, e) && aligned(V, e), "%s: K or V is not aligned to its elements", who);
  if (T == 0 || B == 0) return SONIQ_OK;
  const KvCopy c{{{static_cast<uint8_t*>(cache->k_dev), cache->k_scale_dev, K, k_ts, k_hs},
                  {static_cast<uint8_t*>(cache->v_dev), cache->v_scale_dev, V, v_ts, v_hs}},
                 dims_of(cache), {table, ld, (int32_t)width, (int32_t)B}, cu, start, (int32_t)T, type};
  HIP_TRY(write ? launch_kv_write(c, hip_stream(stream)) : launch_kv_read(c, hip_stream(stream)));
  return SONIQ_OK;
}

soniq_status check_attend(const char* who, const soniq_kv_cache_t* cache, int64_t T, int32_t q_heads,
                          int64_t B, int64_t max_q, int64_t max_kv) {
  if (soniq_status st = check_cache(who, cache)) return st;
  NEED(q_heads >= 1 && q_heads % cache->heads == 0, "%s: %d query heads over a cache of %d", who,
       q_heads, cache->heads);
  NEED(T >= 0 && B >= 0 && max_q >= 1 && max_kv >= 0, "%s: T = %lld, B = %lld, max_q = %lld, max_kv = %lld",
       who, (long long)T, (long long)B, (long long)max_q, (long long)max_kv);
  LIMIT(max_q <= 256 && q_heads <= 65535 && B <= 65535 && max_kv < kMax31 && T * q_heads < kMaxGroups,
        "%s: max_q = %lld, %d query heads, B = %lld, T = %lld (max_q <= 256, heads and B < 2^16, T * heads < 2^24)",
        who, (long long)max_q, q_heads, (long long)B, (long long)T);
  LIMIT(B * cache->heads * ((max_q * (q_heads / cache->heads) + 15) / 16) < (1 << 22),
        "%s: %lld sequences of %d heads and up to %lld new tokens are too many", who, (long long)B,
        cache->heads, (long long)max_q);
  return SONIQ_OK;
}

}  // namespace

extern "C" {

soniq_status soniq_quantize_rows(const void* A_dev, int a_type, int64_t M, int64_t K, int64_t lda,
                                 int8_t* Q_dev, int64_t ldq, float* s_dev, void* stream) {
  const char* who = "soniq_quantize_rows";
  if (soniq_status st = check_quantize(who, A_dev, a_type, M, K, lda)) return st;
  NEED(ldq >= K, "%s: ldq = %lld < K", who, (long long)ldq);
  NEED((Q_dev && s_dev) || M == 0, "%s: null Q or s", who);
  NEED(aligned(s_dev, 4), "%s: s is not aligned to its elements", who);
  if (M == 0) return SONIQ_OK;
  HIP_TRY(launch_quantize_rows(A_dev, a_type, M, K, lda, Q_dev, ldq, s_dev, hip_stream(stream)));
  return SONIQ_OK;
}

soniq_status soniq_i8_gemm(const int8_t* A_dev, int64_t lda, const float* s_a_dev,
                           const int8_t* W_dev, int64_t ldw, const float* s_w_dev,
                           const float* bias_dev, int64_t M, int64_t N, int64_t K, void* Y_dev,
                           int y_type, int64_t ldy, void* stream) {
  const char* who = "soniq_i8_gemm";
  if (soniq_status st = check_gemm(who, W_dev, ldw, s_w_dev, bias_dev, M, N, K, Y_dev, y_type, ldy))
    return st;
  NEED(lda >= K, "%s: lda = %lld < K", who, (long long)lda);
  NEED((A_dev && s_a_dev) || M == 0, "%s: null A or s_a", who);
  NEED(aligned(s_a_dev, 4), "%s: s_a is not aligned to its elements", who);
  if (M == 0) return SONIQ_OK;
  const I8Gemm g{A_dev, lda, s_a_dev, W_dev, ldw, s_w_dev, bias_dev, M, N, K, Y_dev, y_type, ldy};
  HIP_TRY(launch_i8_gemm(g, hip_stream(stream)));
  return SONIQ_OK;
}

soniq_status soniq_quantize_i8_gemm_workspace(int64_t M, int64_t K, int64_t* bytes) {
  const char* who = "soniq_quantize_i8_gemm_workspace";
  NEED(bytes && M >= 0 && K >= 1, "%s: null bytes, or M = %lld, K = %lld", who, (long long)M, (long long)K);
  LIMIT(K <= SONIQ_MAX_K && M < kMax31, "%s: M = %lld, K = %lld", who, (long long)M, (long long)K);
  *bytes = i8_work(M, K);
  return SONIQ_OK;
}

soniq_status soniq_quantize_i8_gemm(const void* A_dev, int a_type, int64_t lda,
                                    const int8_t* W_dev, int64_t ldw, const float* s_w_dev,
                                    const float* bias_dev, int64_t M, int64_t N, int64_t K,
                                    void* Y_dev, int y_type, int64_t ldy, void* work_dev,
                                    int64_t work_bytes, void* stream) {
  const char* who = "soniq_quantize_i8_gemm";
  if (soniq_status st = check_quantize(who, A_dev, a_type, M, K, lda)) return st;
  if (soniq_status st = check_gemm(who, W_dev, ldw, s_w_dev, bias_dev, M, N, K, Y_dev, y_type, ldy))
    return st;
  const int64_t need = i8_work(M, K);
  NEED(work_bytes >= need && (work_dev || need == 0) && aligned(work_dev, 16),
       "%s: a workspace of %lld bytes, 16-byte aligned, is needed", who, (long long)need);
  if (M == 0) return SONIQ_OK;
  if (i8_fused(M, K)) {
    const I8Gemm g{nullptr, 0, nullptr, W_dev, ldw, s_w_dev, bias_dev, M, N, K, Y_dev, y_type, ldy};
    HIP_TRY(launch_i8_fused(g, A_dev, a_type, lda, hip_stream(stream)));
    return SONIQ_OK;
  }
  int8_t* q = static_cast<int8_t*>(work_dev);
  float* s = reinterpret_cast<float*>(q + M * codes_ld(K));
  const I8Gemm g{q, codes_ld(K), s, W_dev, ldw, s_w_dev, bias_dev, M, N, K, Y_dev, y_type, ldy};
  HIP_TRY(launch_quantize_rows(A_dev, a_type, M, K, lda, q, codes_ld(K), s, hip_stream(stream)));
  HIP_TRY(launch_i8_gemm(g, hip_stream(stream)));
  return SONIQ_OK;
}

soniq_status soniq_kv_write(const soniq_kv_cache_t* cache, const void* K_dev,
                            int64_t k_token_stride, int64_t k_head_stride, const void* V_dev,
                            int64_t v_token_stride, int64_t v_head_stride, int type, int64_t T,
                            const int32_t* table_dev, int64_t table_ld, int64_t table_width,
                            int64_t B, const int32_t* cu_dev, const int32_t* start_dev,
                            void* stream) {
  return kv_copy("soniq_kv_write", true, cache, const_cast<void*>(K_dev), k_token_stride,
                 k_head_stride, const_cast<void*>(V_dev), v_token_stride, v_head_stride, type, T,
                 table_dev, table_ld, table_width, B, cu_dev, start_dev, stream);
}

soniq_status soniq_kv_read(const soniq_kv_cache_t* cache, void* K_dev, int64_t k_token_stride,
                           int64_t k_head_stride, void* V_dev, int64_t v_token_stride,
                           int64_t v_head_stride, int type, int64_t T, const int32_t* table_dev,
                           int64_t table_ld, int64_t table_width, int64_t B,
                           const int32_t* cu_dev, const int32_t* start_dev, void* stream) {
  return kv_copy("soniq_kv_read", false, cache, K_dev, k_token_stride, k_head_stride, V_dev,
                 v_token_stride, v_head_stride, type, T, table_dev, table_ld, table_width, B, cu_dev,
                 start_dev, stream);
}

soniq_status soniq_kv_attention_workspace(const soniq_kv_cache_t* cache, int64_t T,
                                          int32_t q_heads, int64_t B, int64_t max_q,
                                          int64_t max_kv, int64_t* bytes) {
  const char* who = "soniq_kv_attention_workspace";
  if (soniq_status st = check_attend(who, cache, T, q_heads, B, max_q, max_kv)) return st;
  NEED(bytes, "%s: null bytes", who);
  *bytes = T && B ? kv_attention_work_bytes(dims_of(cache), T, q_heads, B, max_q, max_kv) : 0;
  return SONIQ_OK;
}

soniq_status soniq_kv_attention(const soniq_kv_cache_t* cache, const void* q_dev,
                                int64_t q_token_stride, int64_t q_head_stride, int type, int64_t T,
                                int32_t q_heads, const int32_t* table_dev, int64_t table_ld,
                                int64_t table_width, int64_t B, const int32_t* cu_dev,
                                const int32_t* kv_len_dev, const uint64_t* mask_dev,
                                int32_t mask_words, float scale, int64_t max_q, int64_t max_kv,
                                void* out_dev, int64_t out_token_stride, int64_t out_head_stride,
                                float* lse_dev, void* work_dev, int64_t work_bytes, void* stream) {
  const char* who = "soniq_kv_attention";
  if (soniq_status st = check_attend(who, cache, T, q_heads, B, max_q, max_kv)) return st;
  if (soniq_status st =
          check_table(who, cache, table_dev, table_ld, table_width, B, cu_dev, kv_len_dev, T))
    return st;
  NEED(type == SONIQ_BF16 || type == SONIQ_F16, "%s: type %d is not SONIQ_BF16 or SONIQ_F16", who, type);
  NEED(mask_dev ? mask_words >= 1 && mask_words <= 4 : mask_words == 0,
       "%s: %d mask words (1 to 4 with a mask, 0 without)", who, mask_words);
  NEED(std::isfinite(scale), "%s: the scale is not finite", who);
  if (T == 0 || B == 0) return SONIQ_OK;
  NEED(q_dev && out_dev, "%s: null q or out", who);
  NEED(aligned(q_dev, 2) && aligned(out_dev, 2) && aligned(mask_dev, 8) && aligned(lse_dev, 4),
       "%s: q, out, mask or lse is not aligned to its elements", who);
  const int64_t need = kv_attention_work_bytes(dims_of(cache), T, q_heads, B, max_q, max_kv);
  NEED(work_bytes >= need && (work_dev || need == 0) && aligned(work_dev, 16),
       "%s: a workspace of %lld bytes, 16-byte aligned, is needed", who, (long long)need);
  const KvAttend a{static_cast<const uint8_t*>(cache->k_dev), cache->k_scale_dev,
                   static_cast<const uint8_t*>(cache->v_dev), cache->v_scale_dev, dims_of(cache),
                   {table_dev, table_ld, (int32_t)table_width, (int32_t)B}, cu_dev, kv_len_dev, q_dev,
                   q_token_stride, q_head_stride, out_dev, out_token_stride, out_head_stride, lse_dev,
                   mask_dev, mask_words, type, (int32_t)T, q_heads, q_heads / cache->heads,
                   (int32_t)max_q, (int32_t)max_kv, scale, static_cast<float*>(work_dev)};
  HIP_TRY(launch_kv_attention(a, hip_stream(stream)));
  return SONIQ_OK;
}

}  // extern "C"
