// gfx950 kernels of the quantized key/value cache and the attention over it.
#include "soniq_serve.h"
#include "soniq_values.h"

namespace soniq {
namespace {

// The sequence of ragged row t: how many of cu[1 .. B] are at most t (B for
// a row behind the last sequence).
__device__ __forceinline__ int row_sequence(const int32_t* cu, int B, int t) {
  int b = 0;
  for (int i = threadIdx.x % 64; i - (int)(threadIdx.x % 64) < B; i += 64)
    b += __popcll(__ballot(i < B && cu[i + 1] <= t));
  return b;
}

__device__ __forceinline__ int code_at(const uint8_t* row, int d, int bits) {
  if (bits == 8) return (int8_t)row[d];
  const int n = (row[d / 2] >> (4 * (d & 1))) & 15;
  return n - 16 * (n > 7);
}

// One wave per (token, side, head).
template <int TYPE, bool WRITE>
__global__ __launch_bounds__(64) void k_kv_copy(KvCopy c) {
  typedef typename Value<TYPE>::T T;
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, D = c.dims.head_dim;
  const KvSide sd = blockIdx.z ? c.side[1] : c.side[0];
  const int b = row_sequence(c.cu, c.table.B, t);
  if (b >= c.table.B) return;
  const int64_t pos = (int64_t)c.start[b] + ((int64_t)t - c.cu[b]);
  const int32_t row0 = kv_row(c.table, c.dims, b, pos);
  T* x = static_cast<T*>(sd.rows) + (int64_t)t * sd.token_stride + h * sd.head_stride;
  if (row0 < 0) {
    if (!WRITE)
      for (int d = lane; d < D; d += 64) x[d] = Value<TYPE>::store(0.0f);
    return;
  }
  const int64_t row = (int64_t)row0 + (int64_t)h * c.dims.page_size;
  uint8_t* codes = sd.codes + row * (D * c.dims.bits / 8);
  if (WRITE) {
    uint32_t mx = 0;
    for (int d = lane; d < D; d += 64) mx = max(mx, __float_as_uint(Value<TYPE>::load(x[d])) & 0x7FFFFFFFu);
    for (int o = 32; o; o >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, o));
    const RowCodec rc = row_codec(mx, c.dims.bits == 8 ? 127.0f : 7.0f);
    if (lane == 0) sd.scale[row] = rc.s;
    if (c.dims.bits == 8) {
      for (int d = lane; d < D; d += 64) codes[d] = (uint8_t)row_code(rc, Value<TYPE>::load(x[d]));
    } else {
      for (int d = lane; d < D / 2; d += 64)
        codes[d] = (uint8_t)((row_code(rc, Value<TYPE>::load(x[2 * d])) & 15) |
                             (row_code(rc, Value<TYPE>::load(x[2 * d + 1])) << 4));
    }
  } else {
    const float s = sd.scale[row];
    for (int d = lane; d < D; d += 64) x[d] = Value<TYPE>::store((float)code_at(codes, d, c.dims.bits) * s);
  }
}

// Whether new position j is visible to new query i.
__device__ __forceinline__ bool sees(const KvAttend& a, int64_t t, int i, int j) {
  if (!a.mask) return j <= i;
  return j < 64 * a.mask_words && (a.mask[t * a.mask_words + j / 64] >> (j % 64)) & 1;
}

// One workgroup per (sequence, query, head): 256 positions at a time, one
// per thread, then the outputs of the chunk, one element per thread.
template <int TYPE>
__global__ __launch_bounds__(256) void k_kv_attend(KvAttend a) {
  typedef typename Value<TYPE>::T T;
  __shared__ float q[256], p[256];
  __shared__ int32_t rows[256];
  __shared__ float red[8];
  const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int D = a.dims.head_dim, bits = a.dims.bits, rb = D * bits / 8;
  const KvSpan sp = kv_span(a.cu[b], a.cu[b + 1], a.T);
  if (i >= sp.count) return;
  const int64_t t = sp.first + i;
  const int len = kv_length(a.table, a.dims, a.kv_len[b]);
  const int64_t base = (int64_t)a.kv_len[b] - sp.count;
  const int h = hq / a.group;
  if (tid < D) q[tid] = Value<TYPE>::load(static_cast<const T*>(a.q)[t * a.q_ts + hq * a.q_hs + tid]);
  float m = -INFINITY, l = 0.0f, o = 0.0f;
  for (int j0 = 0; j0 < len; j0 += 256) {
    __syncthreads();
    const int j = j0 + tid;
    float s = -INFINITY;
    int32_t row = j < len ? kv_row(a.table, a.dims, b, j) : -1;
    if (row >= 0 && (j < base || sees(a, t, i, (int)(j - base)))) {
      row += h * a.dims.page_size;
      float z = 0.0f;
      for (int d = 0; d < D; ++d) z = fmaf(q[d], (float)code_at(a.k + (int64_t)row * rb, d, bits), z);
      s = z * a.ks[row] * a.scale;
    } else {
      row = -1;
    }
    float mx = s;
    for (int x = 32; x; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
    if (tid % 64 == 0) red[tid / 64] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float mn = fmaxf(m, mx), al = mn == -INFINITY ? 1.0f : expf(m - mn);
    const float e = row >= 0 ? expf(s - mn) : 0.0f;
    float sum = e;
    for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
    if (tid % 64 == 0) red[4 + tid / 64] = sum;
    p[tid] = row >= 0 ? e * a.vs[row] : 0.0f;
    rows[tid] = row;
    __syncthreads();
    l = l * al + (red[4] + red[5] + red[6] + red[7]);
    o *= al;
    m = mn;
    if (tid < D)
      for (int x = 0; x < 256; ++x)
        if (rows[x] >= 0) o = fmaf(p[x], (float)code_at(a.v + (int64_t)rows[x] * rb, tid, bits), o);
  }
  if (tid < D)
    static_cast<T*>(a.out)[t * a.o_ts + hq * a.o_hs + tid] = Value<TYPE>::store(l == 0.0f ? 0.0f : o / l);
  if (tid == 0 && a.lse) a.lse[t * a.q_heads + hq] = l == 0.0f ? -INFINITY : m + logf(l);
}

template <bool WRITE>
hipError_t launch_kv_copy(const KvCopy& c, hipStream_t stream) {
  const dim3 grid((unsigned)c.T, (unsigned)c.dims.heads, 2), block(64);
  if (c.type == SONIQ_F32) k_kv_copy<SONIQ_F32, WRITE><<<grid, block, 0, stream>>>(c);
  else if (c.type == SONIQ_BF16) k_kv_copy<SONIQ_BF16, WRITE><<<grid, block, 0, stream>>>(c);
  else k_kv_copy<SONIQ_F16, WRITE><<<grid, block, 0, stream>>>(c);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const KvCopy& c, hipStream_t stream) { return launch_kv_copy<true>(c, stream); }
hipError_t launch_kv_read(const KvCopy& c, hipStream_t stream) { return launch_kv_copy<false>(c, stream); }

int64_t kv_attention_work_bytes(const KvDims&, int64_t, int32_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_kv_attention(const KvAttend& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.max_q, (unsigned)a.q_heads, (unsigned)a.table.B), block(256);
  if (a.type == SONIQ_BF16) k_kv_attend<SONIQ_BF16><<<grid, block, 0, stream>>>(a);
  else k_kv_attend<SONIQ_F16><<<grid, block, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace soniq
