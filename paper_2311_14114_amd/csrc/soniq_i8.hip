// gfx950 kernels of the 8-bit linear layers with one scale per token and per
// output channel.
#include "soniq_serve.h"
#include "soniq_values.h"

namespace soniq {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// One row per workgroup: its largest |x|, then its codes.
template <int TYPE>
__global__ __launch_bounds__(256) void k_rows(const typename Value<TYPE>::T* A, int K, int64_t lda,
                                              int8_t* Q, int64_t ldq, float* s) {
  __shared__ uint32_t part[4];
  const int64_t m = blockIdx.x;
  const typename Value<TYPE>::T* a = A + m * lda;
  uint32_t mx = 0;
  for (int k = threadIdx.x; k < K; k += 256)
    mx = max(mx, __float_as_uint(Value<TYPE>::load(a[k])) & 0x7FFFFFFFu);
  for (int o = 32; o; o >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, o));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = mx;
  __syncthreads();
  mx = max(max(part[0], part[1]), max(part[2], part[3]));
  const RowCodec rc = row_codec(mx, 127.0f);
  if (threadIdx.x == 0) s[m] = rc.s;
  for (int k = threadIdx.x; k < K; k += 256)
    Q[m * ldq + k] = (int8_t)row_code(rc, Value<TYPE>::load(a[k]));
}

template <int TYPE>
__device__ __forceinline__ void store_y(const I8Gemm& g, int64_t m, int64_t n, int acc, float sa,
                                        float sw) {
  float y = __fmul_rn(__fmul_rn((float)acc, sa), sw);
  if (g.bias) y = __fadd_rn(y, g.bias[n]);
  static_cast<typename Value<TYPE>::T*>(g.Y)[m * g.ldy + n] = Value<TYPE>::store(y);
}

// 64x64 tile, four waves of 32x32, 64 channels a step through LDS.
template <int TYPE>
__global__ __launch_bounds__(256) void k_i8_tile(I8Gemm g) {
  __shared__ int8_t As[64][80], Bs[64][80];
  const int64_t m0 = (int64_t)blockIdx.y * 64, n0 = (int64_t)blockIdx.x * 64;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32, r = lane % 16, kq = lane / 16;
  v4i acc[2][2] = {};
  for (int64_t k0 = 0; k0 < g.K; k0 += 64) {
    const int row = tid / 4, c = (tid % 4) * 16;
    for (int e = 0; e < 16; ++e) {
      const int64_t k = k0 + c + e;
      As[row][c + e] = m0 + row < g.M && k < g.K ? g.A[(m0 + row) * g.lda + k] : 0;
      Bs[row][c + e] = n0 + row < g.N && k < g.K ? g.W[(n0 + row) * g.ldw + k] : 0;
    }
    __syncthreads();
    v4i a[2], b[2];
    for (int i = 0; i < 2; ++i) {
      a[i] = *reinterpret_cast<const v4i*>(&As[wm + 16 * i + r][16 * kq]);
      b[i] = *reinterpret_cast<const v4i*>(&Bs[wn + 16 * i + r][16 * kq]);
    }
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j < 2; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[j], acc[i][j], 0, 0, 0);
    __syncthreads();
  }
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      for (int e = 0; e < 4; ++e) {
        const int64_t m = m0 + wm + 16 * i + 4 * kq + e, n = n0 + wn + 16 * j + r;
        if (m < g.M && n < g.N) store_y<TYPE>(g, m, n, acc[i][j][e], g.sa[m], g.sw[n]);
      }
}

}  // namespace

hipError_t launch_quantize_rows(const void* A, int a_type, int64_t M, int64_t K, int64_t lda,
                                int8_t* Q, int64_t ldq, float* s, hipStream_t stream) {
  const dim3 grid((unsigned)M), block(256);
  if (a_type == SONIQ_F32)
    k_rows<SONIQ_F32><<<grid, block, 0, stream>>>(static_cast<const float*>(A), (int)K, lda, Q, ldq, s);
  else if (a_type == SONIQ_BF16)
    k_rows<SONIQ_BF16><<<grid, block, 0, stream>>>(static_cast<const uint16_t*>(A), (int)K, lda, Q, ldq, s);
  else
    k_rows<SONIQ_F16><<<grid, block, 0, stream>>>(static_cast<const _Float16*>(A), (int)K, lda, Q, ldq, s);
  return hipGetLastError();
}

hipError_t launch_i8_gemm(const I8Gemm& g, hipStream_t stream) {
  const dim3 grid((unsigned)((g.N + 63) / 64), (unsigned)((g.M + 63) / 64)), block(256);
  if (g.y_type == SONIQ_F32) k_i8_tile<SONIQ_F32><<<grid, block, 0, stream>>>(g);
  else if (g.y_type == SONIQ_BF16) k_i8_tile<SONIQ_BF16><<<grid, block, 0, stream>>>(g);
  else k_i8_tile<SONIQ_F16><<<grid, block, 0, stream>>>(g);
  return hipGetLastError();
}

}  // namespace soniq
