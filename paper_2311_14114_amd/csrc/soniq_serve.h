// Internal declarations of the 8-bit linear layers (soniq_i8.hip) and the
// quantized key/value cache (soniq_kv.hip), shared with their host side
// (soniq_serve_api.cpp).  Not part of the public ABI.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "soniq_kv_slot.h"

namespace soniq {

// ---- 8-bit linear layers ---------------------------------------------------
// Element types as in soniq.h (SONIQ_F32, SONIQ_BF16, SONIQ_F16).
hipError_t launch_quantize_rows(const void* A, int a_type, int64_t M, int64_t K, int64_t lda,
                                int8_t* Q, int64_t ldq, float* s, hipStream_t stream);

struct I8Gemm {
  const int8_t* A;
  int64_t lda;
  const float* sa;
  const int8_t* W;
  int64_t ldw;
  const float* sw;
  const float* bias;  // or null
  int64_t M, N, K;
  void* Y;
  int y_type;
  int64_t ldy;
};
hipError_t launch_i8_gemm(const I8Gemm& g, hipStream_t stream);
// Quantization and product in one launch, where they are (g.A and g.sa are
// not read).
bool i8_fused(int64_t M, int64_t K);
hipError_t launch_i8_fused(const I8Gemm& g, const void* A, int a_type, int64_t lda, hipStream_t stream);

// ---- key/value cache -------------------------------------------------------
// One side of the cache and the ragged rows that go with it.
struct KvSide {
  uint8_t* codes;
  float* scale;
  void* rows;               // [T, heads, head_dim]
  int64_t token_stride, head_stride;  // elements
};

struct KvCopy {
  KvSide side[2];  // keys, values
  KvDims dims;
  KvTable table;
  const int32_t* cu;
  const int32_t* start;
  int32_t T;
  int type;
};
hipError_t launch_kv_write(const KvCopy& c, hipStream_t stream);
hipError_t launch_kv_read(const KvCopy& c, hipStream_t stream);

struct KvAttend {
  const uint8_t* k;
  const float* ks;
  const uint8_t* v;
  const float* vs;
  KvDims dims;
  KvTable table;
  const int32_t* cu;
  const int32_t* kv_len;
  const void* q;
  int64_t q_ts, q_hs;
  void* out;
  int64_t o_ts, o_hs;
  float* lse;  // or null
  const uint64_t* mask;
  int32_t mask_words;
  int type;
  int32_t T, q_heads, group;
  int32_t max_q, max_kv;
  float scale;
  // work: per (token row, part): max, sum, then the unnormalised outputs
  float* work;
};
int64_t kv_attention_work_bytes(const KvDims& d, int64_t T, int32_t q_heads, int64_t B,
                                int64_t max_q, int64_t max_kv);
hipError_t launch_kv_attention(const KvAttend& a, hipStream_t stream);

}  // namespace soniq
