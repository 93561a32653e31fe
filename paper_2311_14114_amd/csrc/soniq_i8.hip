// gfx950 kernels of the 8-bit linear layers with one scale per token and per
// output channel:
//   Y[m,n] = (float(sum_k Qa[m,k] Qw[n,k]) * s_a[m]) * s_w[n] + bias[n],
//   s_a[m] = max_k |A[m,k]| / 127,  Qa = rint(A / s_a).
//
//   k_rows       codes and scales of rows, one wave or one workgroup a row
//   k_i8_fused   up to 16 short tokens, quantized where they are used: one launch
//   k_i8_skinny  up to 64 tokens: bound by the weights' bytes; the waves of a
//                workgroup split K, each with its own part of LDS
//   k_i8_tile    more tokens: bound by LDS where tiles are few and small, by
//                the matrix cores else; operands staged through LDS
//   k_i8_short   more tokens of fewer than 16 channels
//
// The integer sums are exact, so no split or order of K changes a bit.
// Measured figures in this file are of one MI355X; times "in a graph" leave
// out the host's part of a call.
#include "soniq_serve.h"
#include "soniq_values.h"

#include <algorithm>
#include <type_traits>

namespace soniq {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

// 16 bytes at any address.
__device__ __forceinline__ v4i load16(const int8_t* p) {
  struct __attribute__((packed, aligned(1))) P { v4i v; };
  return reinterpret_cast<const P*>(p)->v;
}

// 16 bytes moved down by `by` >= 0, zeros above: what a load that would end
// `by` bytes past its row holds, from the row's last 16 bytes instead.
__device__ __forceinline__ void move_down(v4i& x, int by) {
  const uint64_t lo = (uint32_t)x[0] | (uint64_t)(uint32_t)x[1] << 32;
  const uint64_t hi = (uint32_t)x[2] | (uint64_t)(uint32_t)x[3] << 32;
  const int sh = 8 * (by & 7);
  const uint64_t up = sh ? hi << (64 - sh) : 0, l = by & 8 ? hi >> sh : lo >> sh | up;
  const uint64_t h = by & 8 ? 0 : hi >> sh;
  x[0] = by >= 16 ? 0 : (int)l, x[1] = by >= 16 ? 0 : (int)(l >> 32);
  x[2] = by >= 16 ? 0 : (int)h, x[3] = by >= 16 ? 0 : (int)(h >> 32);
}

// Bytes [k, k + 16) of a row of K < 16, zeros from K on; reads nothing outside the row.
__device__ __forceinline__ v4i load_short(const int8_t* row, int64_t k, int64_t K) {
  uint32_t b[4] = {0, 0, 0, 0};
  for (int i = 0; i < 16; ++i)
    if (k + i < K) b[i / 4] |= (uint32_t)(uint8_t)row[k + i] << (8 * (i % 4));
  return v4i{(int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ------------------------------------------------------------ quantizing --
__device__ __forceinline__ void store_codes(int8_t* q, int k, int K, uint2 c) {
  if (k + 8 <= K) {
    struct __attribute__((packed, aligned(1))) P { uint32_t x, y; };
    *reinterpret_cast<P*>(q + k) = {c.x, c.y};
  } else {
    for (int i = 0; i < 8; ++i)
      if (k + i < K) q[k + i] = (int8_t)((i < 4 ? c.x : c.y) >> (8 * (i % 4)));
  }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
#pragma unroll
  for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  return m;
}

// T threads a row: a wave, four of them a workgroup, or a workgroup.  A row of
// up to 8 * T * kHeld elements stays in registers between its maximum and its
// codes; longer ones are read again for the rest.  Bytes bound it where rows
// are many: 8192 x 8192 bf16 take 48 us, 202 MB at 4.2 TB/s (a large copy
// reaches 4.8), 4096 x 4096 13.3, 50 MB at 3.8.  Few rows take two dependent
// trips to memory and a barrier: 40 x 4096 4.3 us.
template <int TYPE, int T, int kHeld>
__global__ __launch_bounds__(T < 256 ? 256 : T) void k_rows(const typename Value<TYPE>::T* A, int64_t M, int K,
                                                            int64_t lda, int8_t* Q, int64_t ldq, float* s) {
  static_assert(T == 64 || T >= 256, "a row is a wave's or a workgroup's");
  constexpr int kRows = T < 256 ? 256 / T : 1;  // a workgroup
  __shared__ uint32_t part[T / 64];
  const int t = threadIdx.x % T;
  const int64_t step = (int64_t)gridDim.x * kRows;
  for (int64_t m = (int64_t)blockIdx.x * kRows + threadIdx.x / T; m < M; m += step) {
    const typename Value<TYPE>::T* a = A + m * lda;
    Eight<TYPE> x[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) x[i].load(a, min(8 * (t + T * i), K), K);
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) mx = max(mx, x[i].amax());
    for (int k = 8 * (t + T * kHeld); k < K; k += 8 * T) {
      Eight<TYPE> y;
      y.load(a, k, K);
      mx = max(mx, y.amax());
    }
    mx = wave_max(mx);
    if constexpr (T > 64) {
      __syncthreads();  // the last row's maxima have been read
      if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = mx;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < T / 64; ++w) mx = max(mx, part[w]);
    }
    const RowCoder rc(mx, 127.0f);
    if (t == 0) s[m] = rc.s;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (8 * (t + T * i) < K) store_codes(Q + m * ldq, 8 * (t + T * i), K, x[i].codes(rc));
    for (int k = 8 * (t + T * kHeld); k < K; k += 8 * T) {
      Eight<TYPE> y;
      y.load(a, k, K);
      store_codes(Q + m * ldq, k, K, y.codes(rc));
    }
  }
}

// --------------------------------------------------------------- outputs --
__device__ __forceinline__ void store_y(const I8Gemm& g, int64_t at, float y) {
  if (g.y_type == SONIQ_BF16) static_cast<uint16_t*>(g.Y)[at] = bf16_bits(y);
  else if (g.y_type == SONIQ_F16) static_cast<_Float16*>(g.Y)[at] = Value<SONIQ_F16>::store(y);
  else static_cast<float*>(g.Y)[at] = y;
}
__device__ __forceinline__ float scaled(int acc, float sa, float sw) {
  return __fmul_rn(__fmul_rn((float)acc, sa), sw);
}

// ------------------------------------------------------------ few tokens --
// A workgroup of eight waves takes 16 * NT output channels and all tokens
// (at most 8 * A8); wave w takes the 128-byte segments w, w + 8, ... of K.  A
// load takes whole 128-byte pieces of 8 rows: a cache serves neighbouring
// lanes of one line at once, but an operand of the product has neighbouring
// lanes in different rows (loading operands as they are took 60 accesses an
// instruction and half the speed).  So each wave turns its segments through
// its own part of LDS, with no barrier; sums meet in LDS at the end.
// 40 x 11008 x 4096 take 11.4 us: 45 MB of weights at 4.0 TB/s.
template <int A8, int NT>
__global__ __launch_bounds__(512) void k_i8_skinny(I8Gemm g) {
  constexpr int MT = (A8 + 1) / 2, NL = A8 + 2 * NT;           // loads a lane and segment
  constexpr int U = NL <= 3 ? 4 : NL <= 6 ? 2 : 1;             // segments in flight
  constexpr int kWave = (16 * MT + 16 * NT) * 128;             // LDS bytes of a wave
  constexpr int kRed = 8 * MT * NT * 256 * 4;
  __shared__ __align__(16) int8_t lds[8 * kWave > kRed ? 8 * kWave : kRed];
  const int tid = threadIdx.x, lane = tid % 64, r = lane % 16, q = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NT);
  const int lr = lane / 8, lc = lane % 8;
  const int8_t* row[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i)
    row[i] = i < A8 ? g.A + min((int64_t)(8 * i + lr), g.M - 1) * g.lda
                    : g.W + min(n0 + 8 * (i - A8) + lr, g.N - 1) * g.ldw;
  // rows 0 .. 16 MT - 1 of the wave's LDS are tokens (those past 8 * A8 hold
  // anything: their sums are not stored), then 16 NT channels; chunk c of row
  // x at c ^ (x / 2 % 8), as in the tiles below
  int8_t* mine = lds + wave * kWave;
  const int wat = lr * 128, wsw = lr / 2;
  auto put = [&](int i, v4i x) {
    const int at = i < A8 ? 8 * i : 16 * MT + 8 * (i - A8);  // first row of the load
    *reinterpret_cast<v4i*>(mine + at * 128 + wat + ((lc ^ (at / 2 % 8 + wsw)) << 4)) = x;
  };
  v4i acc[MT][NT] = {};
  auto mma = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = r * 128 + (((4 * h + q) ^ (r / 2)) << 4);
      v4i a[MT], w[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i) a[i] = *reinterpret_cast<const v4i*>(mine + i * 2048 + at);
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j] = *reinterpret_cast<const v4i*>(mine + (MT + j) * 2048 + at);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], w[j], acc[i][j], 0, 0, 0);
    }
  };
  auto order = [&]() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); };
  // The last segment may be partial: chunks that cross the rows' end are taken
  // from the last 16 bytes and moved down (`over` bytes) before they are put.
  // It is loaded in its turn, like the others (40 x 11008 x 4091: 13.2 us, and
  // 17.9 with a load of its own after the loop).
  const int K = (int)g.K, segs = K >= 16 ? (K + 127) / 128 : 0, partial = K % 128 ? segs - 1 : segs;
  const int over = max(0, partial * 128 + 16 * lc + 16 - K);
  v4i x[U][NL];
  auto fetch = [&](int u, int sg) {
    const int k = min(sg * 128 + 16 * lc, K - 16);
#pragma unroll
    for (int i = 0; i < NL; ++i) x[u][i] = load16(row[i] + k);
  };
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (wave + 8 * u < segs) fetch(u, wave + 8 * u);
  for (int sg = wave; sg < segs; sg += 8 * U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (sg + 8 * u < segs) {
        if (sg + 8 * u == partial) {
          asm volatile("");  // a branch, not selects
#pragma unroll
          for (int i = 0; i < NL; ++i) move_down(x[u][i], over);
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) put(i, x[u][i]);
        if (sg + 8 * (u + U) < segs) fetch(u, sg + 8 * (u + U));
        order();
        mma();
        order();
      }
    }
  }
  if (K < 16 && wave == 0) {
#pragma unroll
    for (int i = 0; i < NL; ++i) put(i, load_short(row[i], 16 * lc, K));
    order();
    mma();
  }
  __syncthreads();
  int* red = reinterpret_cast<int*>(lds);  // [wave][tile][e][lane]
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[((wave * MT * NT + i * NT + j) * 4 + e) * 64 + lane] = acc[i][j][e];
  __syncthreads();
  for (int y = tid; y < MT * NT * 256; y += 512) {
    const int tile = y / 256, e = y / 64 % 4, l = y % 64;
    const int64_t m = 16 * (tile / NT) + 4 * (l / 16) + e, n = n0 + 16 * (tile % NT) + l % 16;
    if (m >= g.M || n >= g.N) continue;
    int sum = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) sum += red[((w * MT * NT + tile) * 4 + e) * 64 + l];
    float v = scaled(sum, g.sa[m], g.sw[n]);
    if (g.bias) v = __fadd_rn(v, g.bias[n]);
    store_y(g, m * g.ldy + n, v);
  }
}

// Up to 16 tokens with their quantization in the same launch: every workgroup
// makes the codes for itself (at most kFusedMost elements, 32 a thread), in
// LDS, while its first weights are on their way.  16 output channels a
// workgroup, K over the waves as above, U segments of each in flight.
// 1 x 4096 x 4096 takes 6.1 us in a trace (8.2 from one to the next in a graph):
// 17 MB at 2.8 TB/s, half of it the way from the launch to the codes.  Past 16384 elements the codes cost every workgroup more
// than a launch of their own (8 x 4096 x 4096: 14.9 us in a graph, 10.5 with
// two launches); from 8192 on they are level (16 x 2304 x 768: 7.4 and 7.0),
// and a launch from Python is 4 more.
constexpr int kFusedRows = 16, kFusedMost = 16384;

template <int TYPE, int U>
__global__ __launch_bounds__(512, U == 2 ? 6 : 4) void k_i8_fused(I8Gemm g, const typename Value<TYPE>::T* A, int64_t lda) {
  constexpr int kPad = 144, kHeld = kFusedMost / (8 * 512);
  // codes of token m at m * (K up to a multiple of 128 + 16), then the waves'
  // weights (later the sums), then the largest |x| and the scale of each token
  __shared__ __align__(16) int8_t codes[kFusedMost + kFusedRows * kPad];
  __shared__ __align__(16) int8_t wlds[8 * 2048];
  __shared__ uint32_t amax[kFusedRows];
  __shared__ float sa[kFusedRows];
  const int tid = threadIdx.x, lane = tid % 64, r = lane % 16, q = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int M = (int)g.M, K = (int)g.K, nv = (K + 7) / 8, pitch = (K + 127) / 128 * 128 + 16;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int lr = lane / 8, lc = lane % 8;

  Eight<TYPE> x[kHeld];
  int xm[kHeld], xk[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int v = tid + 512 * i;
    xm[i] = v / nv, xk[i] = v % nv * 8;
    const bool on = xm[i] < M;
    x[i].load(A + (on ? xm[i] : 0) * lda, on ? xk[i] : K, K);  // zeros past the last token
  }
  const int8_t* row[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) row[i] = g.W + min(n0 + 8 * i + lr, g.N - 1) * g.ldw;
  const int segs = K >= 16 ? (K + 127) / 128 : 0, partial = K % 128 ? segs - 1 : segs;  // as above
  const int over = max(0, partial * 128 + 16 * lc + 16 - K);
  v4i w[U][2];
  auto fetch = [&](int u, int sg) {
    const int k = min(sg * 128 + 16 * lc, K - 16);
#pragma unroll
    for (int i = 0; i < 2; ++i) w[u][i] = load16(row[i] + k);
  };
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (wave + 8 * u < segs) fetch(u, wave + 8 * u);
  if (tid < kFusedRows) amax[tid] = 0;
  lds_barrier();
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    if (512 * i >= nv * M) break;
    const uint32_t mx = x[i].amax();
    if (nv % 64 == 0) {  // a wave's pieces are of one token
      const uint32_t wm = wave_max(mx);
      if (lane == 0 && xm[i] < M) atomicMax(&amax[xm[i]], wm);
    } else if (xm[i] < M) {
      atomicMax(&amax[xm[i]], mx);
    }
  }
  lds_barrier();
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    if (xm[i] < M) {
      const RowCoder rc(amax[xm[i]], 127.0f);
      if (xk[i] == 0) sa[xm[i]] = rc.s;
      *reinterpret_cast<uint2*>(codes + xm[i] * pitch + xk[i]) = x[i].codes(rc);
    }
  }
  // the last segment's channels past K: zeros (products with whatever the weights hold there are 0 too)
  for (int i = tid; i < 128 * M; i += 512) {
    const int k = K / 128 * 128 + i % 128;
    if (k >= nv * 8 && k < pitch) codes[i / 128 * pitch + k] = 0;
  }
  lds_barrier();

  int8_t* mine = wlds + wave * 2048;
  const int8_t* arow = codes + min(r, M - 1) * pitch + 16 * q;
  v4i acc = {0, 0, 0, 0};
  auto put = [&](int i, v4i v) {
    *reinterpret_cast<v4i*>(mine + (8 * i + lr) * 128 + ((lc ^ (4 * i + lr / 2)) << 4)) = v;
  };
  auto mma = [&](int sg) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const v4i b = *reinterpret_cast<const v4i*>(mine + r * 128 + (((4 * h + q) ^ (r / 2)) << 4));
      const v4i a = *reinterpret_cast<const v4i*>(arow + sg * 128 + 64 * h);
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, acc, 0, 0, 0);
    }
  };
  auto order = [&]() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); };
  for (int sg = wave; sg < segs; sg += 8 * U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (sg + 8 * u < segs) {
        if (sg + 8 * u == partial) {
          asm volatile("");  // a branch, not selects
#pragma unroll
          for (int i = 0; i < 2; ++i) move_down(w[u][i], over);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) put(i, w[u][i]);
        if (sg + 8 * (u + U) < segs) fetch(u, sg + 8 * (u + U));
        order();
        mma(sg + 8 * u);
        order();
      }
    }
  }
  if (K < 16 && wave == 0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) put(i, load_short(row[i], 16 * lc, K));
    order();
    mma(0);
  }
  __syncthreads();
  int* red = reinterpret_cast<int*>(wlds);  // [wave][token][column]
#pragma unroll
  for (int e = 0; e < 4; ++e) red[(wave * 16 + 4 * q + e) * 16 + r] = acc[e];
  __syncthreads();
  const int64_t n = n0 + tid % 16;
  if (tid < 16 * M && n < g.N) {
    const int m = tid / 16;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += red[(i * 16 + m) * 16 + tid % 16];
    float v = scaled(sum, sa[m], g.sw[n]);
    if (g.bias) v = __fadd_rn(v, g.bias[n]);
    store_y(g, m * g.ldy + n, v);
  }
}

// ----------------------------------------------------------- many tokens --
// A wave's outputs, scaled and stored.  Lane (c, hi) holds row m = c of each
// 32x32 tile, and of it columns 8 g + 4 hi + e: four neighbours, packed into
// this wave's part of LDS as one piece; 32 rows at a time then leave in whole
// 16-byte pieces of consecutive columns.
template <int TYPE, bool BIAS, int TM, int TN, bool CLAMP>
__device__ __forceinline__ void tile_out(const I8Gemm& g, const v16i (&acc)[TM][TN], int8_t* lds, int64_t mw,
                                         int64_t nw, int lane) {
  typedef typename Value<TYPE>::T T;
  constexpr int E = sizeof(T), kCols = 32 * TN, kPitch = kCols * E + 16;  // bytes of a row in LDS
  constexpr int kLanes = kCols * E / 16;                                  // lanes a row on the way out
  const int c = lane % 32, hi = lane / 32;
  struct __attribute__((packed, aligned(4))) F4 { float v[4]; };
  float sw[TN][4][4];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t n = nw + 32 * j + 8 * q + 4 * hi;
      if constexpr (CLAMP) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sw[j][q][e] = g.sw[min(n + e, g.N - 1)];
      } else {
        const F4 x = *reinterpret_cast<const F4*>(g.sw + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) sw[j][q][e] = x.v[e];
      }
    }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = mw + 32 * i + c;
    const float sa = g.sa[CLAMP ? min(m, g.M - 1) : m];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        T y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = scaled(acc[i][j][4 * q + e], sa, sw[j][q][e]);
          if constexpr (BIAS) {
            const int64_t n = nw + 32 * j + 8 * q + 4 * hi + e;
            v = __fadd_rn(v, g.bias[CLAMP ? min(n, g.N - 1) : n]);
          }
          y[e] = Value<TYPE>::store(v);
        }
        __builtin_memcpy(lds + c * kPitch + (32 * j + 8 * q + 4 * hi) * E, y, sizeof y);
      }
    // the wave's own region: its stores above come before its loads below
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += 64 / kLanes) {
      const int r = r0 + lane / kLanes, col = lane % kLanes * (16 / E);
      struct __attribute__((packed, aligned(E))) P { T v[16 / E]; };
      P x;
      __builtin_memcpy(&x, __builtin_assume_aligned(lds + r * kPitch + col * E, 16), 16);
      const int64_t my = mw + 32 * i + r, ny = nw + col;
      T* out = static_cast<T*>(g.Y) + my * g.ldy + ny;
      if constexpr (CLAMP) {
        if (my < g.M) {
#pragma unroll
          for (int e = 0; e < 16 / E; ++e)
            if (ny + e < g.N) out[e] = x.v[e];
        }
      } else {
        *reinterpret_cast<P*>(out) = x;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  }
}

// BM x BN tile, four waves of (BM/2) x (BN/2), 128 channels a stage through
// two LDS buffers.  Rows go from memory to registers one stage ahead, so that
// any alignment and the last partial stage are a matter of that load alone,
// and into LDS within the stage before their own.  LDS rows are 128 bytes;
// the 16-byte chunk c of row r sits at chunk c ^ (r / 2 % 8), which spreads
// the 16 rows that a fragment read touches at once over all banks.
// A stage has four steps of 32 channels: the fragments of the next step are
// read during the products of this one, across the barrier too, and the
// first three steps each move a third of the next stage into LDS and load
// that third of the one after.
//
// A tile that would pass the last row or channel starts earlier instead (its
// neighbour computes the same outputs, to the same bits).  CLAMP: for
// matrices smaller than a tile, and for row strides of 2^24 bytes and more:
// each row's address by itself.
//
// SETS = 2: two sets of four waves take the even and the odd stages, each
// with its own buffers, and the first adds the second's sums before it stores.
// Few tiles leave a CU with one workgroup, whose one stage in flight does not
// cover the memory's latency.
//
// 8192^3 takes 455 to 485 us, 2270 to 2420 TOPS by the card (the matrix cores
// busy 0.65 of the time; a library's product of int8 matrices reached 2035 to
// 2500), 4096 x 4096 x 11008 147 to 159 us, 2320 to 2510.  256x256 spills 292
// bytes a lane, outside its main loop.  Small tiles are bound by
// LDS: a stage of 64x128 writes 24 KB and reads 48, some 770 of the 900
// cycles that it takes (301 x 4099 x 4091: 13.6 us); two stages in flight a
// set, or four sets, changed nothing.  Weights' rows that do not start at
// multiples of 16 bytes take two lines a load: 19 us there.
template <int BM, int BN, bool CLAMP, int SETS>
__global__ __launch_bounds__(256 * SETS, BM * BN * SETS > 128 * 128 ? 1 : 2) void k_i8_tile(I8Gemm g, int tm, int tn) {
  constexpr int TM = BM / 64, TN = BN / 64;        // 32x32 tiles a wave
  constexpr int LA = BM / 32, LB = BN / 32, NS = LA + LB;  // 16-byte loads a thread and stage
  __shared__ __align__(16) int8_t lds_all[SETS][2][(BM + BN) * 128];

  // Workgroup b runs on XCD b % 8: each XCD takes a contiguous run of the
  // tile order, columns of up to four row blocks (bands of one height: 600 x
  // 4096 x 4096 takes 18.3 us, 19.2 with two fours and a two), so that its L2
  // serves the rows that its tiles share.
  int bm, bn;
  {
    const int total = tm * tn, per = (total + 7) / 8;
    const int t = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
    if ((int)(blockIdx.x / 8) >= per || t >= total) return;
    const int bands = (tm + 3) / 4, high = (tm + bands - 1) / bands;
    const int band = t / (high * tn), rows = min(high, tm - high * band), in = t - band * high * tn;
    bm = high * band + in % rows;
    bn = in / rows;
  }
  const int set = SETS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / 256);
  const int tid = threadIdx.x % 256, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  auto& lds = lds_all[set];
  const int64_t m0 = CLAMP ? (int64_t)bm * BM : min((int64_t)bm * BM, g.M - BM);
  const int64_t n0 = CLAMP ? (int64_t)bn * BN : min((int64_t)bn * BN, g.N - BN);
  const int lr = tid / 8, lc = tid % 8;
  // Stages of this set (the second set's last one may lie past K altogether).
  // In a partial last stage, chunks that cross the end of a row are taken from
  // its last 16 bytes (K >= 16 here) and moved down when they are written;
  // `over`: how many bytes past the end this thread's chunk would reach.
  const int stages = ((int)((g.K + 127) / 128) + SETS - 1) / SETS;
  const int left = (int)g.K - ((stages - 1) * SETS + set) * 128;  // of the last stage
  const bool tail = left < 128;
  const int over = max(0, 16 * lc + 16 - left);
  constexpr uint32_t kStep = SETS * 128;
  const int8_t* row[NS];  // uniform without CLAMP
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const bool isA = i < LA;
    const int r = 32 * (isA ? i : i - LA);
    if constexpr (CLAMP)
      row[i] = isA ? g.A + min(m0 + lr + r, g.M - 1) * g.lda : g.W + min(n0 + lr + r, g.N - 1) * g.ldw;
    else
      row[i] = isA ? g.A + (m0 + r) * g.lda : g.W + (n0 + r) * g.ldw;
  }
  const uint32_t va = (CLAMP ? 0 : (uint32_t)(lr * g.lda)) + 16 * lc + 128 * set;
  const uint32_t vb = (CLAMP ? 0 : (uint32_t)(lr * g.ldw)) + 16 * lc + 128 * set;
  v4i st[NS];
  // k: byte of the rows where the stage starts (this thread's chunk is 16 lc further)
  auto load = [&](int i, uint32_t k) { st[i] = load16(row[i] + ((i < LA ? va : vb) + k)); };
  const int wat = lr * 128 + ((lc ^ (lr / 2 % 8)) << 4);
  auto write = [&](int i, int buf) { *reinterpret_cast<v4i*>(&lds[buf][wat + 4096 * i]) = st[i]; };
  const int wm = (wave & 1) * (BM / 2), wn = (wave >> 1) * (BN / 2);
  int rat[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
    rat[ks] = (lane % 32) * 128 + (((2 * ks + lane / 32) ^ (lane / 2 % 8)) << 4);
  struct Frag {
    v4i a[TM], b[TN];
  } f[2];
  auto read = [&](Frag& x, int buf, int ks) {
#pragma unroll
    for (int i = 0; i < TM; ++i) x.a[i] = *reinterpret_cast<const v4i*>(&lds[buf][rat[ks] + (wm + 32 * i) * 128]);
#pragma unroll
    for (int j = 0; j < TN; ++j)
      x.b[j] = *reinterpret_cast<const v4i*>(&lds[buf][rat[ks] + (BM + wn + 32 * j) * 128]);
  };
  v16i acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
  auto mma = [&](const Frag& x) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x.b[j], x.a[i], acc[i][j], 0, 0, 0);
  };
  // What a step issues beside its products, one piece after each product:
  // fragment reads first (the next step waits for them), then LDS writes
  // with the loads that refill their registers.
  auto interleave = [&](auto moved) {
    constexpr int kMoved = decltype(moved)::value, kReads = TM + TN, kMma = TM * TN;
    constexpr int kPer = (kReads + 2 * kMoved + kMma - 1) / kMma;
#pragma unroll
    for (int i = 0; i < kMma; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i * kPer < kReads) {
        __builtin_amdgcn_sched_group_barrier(0x100, kPer, 0);
      } else {
        __builtin_amdgcn_sched_group_barrier(0x200, (kPer + 1) / 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, (kPer + 1) / 2, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr int kCut[4] = {0, (NS + 2) / 3, (NS + 2) / 3 + (NS + 1) / 3, NS};

#pragma unroll
  for (int i = 0; i < NS; ++i) load(i, stages == 1 ? (uint32_t)-over : 0u);
  if (stages == 1 && tail) {
#pragma unroll
    for (int i = 0; i < NS; ++i) move_down(st[i], over);
  }
#pragma unroll
  for (int i = 0; i < NS; ++i) write(i, 0);
  if (stages > 1) {
#pragma unroll
    for (int i = 0; i < NS; ++i) load(i, kStep - (stages == 2 ? over : 0));
  }
  lds_barrier();
  read(f[0], 0, 0);
  int s = 0;
  for (; s + 3 < stages; ++s) {
    const int buf = s & 1;
    const uint32_t k = (uint32_t)(s + 2) * kStep;
#pragma unroll
    for (int ks = 0; ks < 3; ++ks) {
      read(f[(ks + 1) & 1], buf, ks + 1);
      mma(f[ks & 1]);
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (i >= kCut[ks] && i < kCut[ks + 1]) write(i, buf ^ 1), load(i, k);
      interleave(std::integral_constant<int, (NS + 2) / 3>());
    }
    lds_barrier();
    read(f[0], buf ^ 1, 0);
    mma(f[1]);
    interleave(std::integral_constant<int, 0>());
  }
  // the last three stages: nothing to load any more, and perhaps a partial one
  for (; s < stages; ++s) {
    const int buf = s & 1;
    read(f[1], buf, 1);
    mma(f[0]);
    read(f[0], buf, 2);
    mma(f[1]);
    read(f[1], buf, 3);
    if (tail && s + 1 == stages - 1) {
      asm volatile("");  // a branch, not selects
#pragma unroll
      for (int i = 0; i < NS; ++i) move_down(st[i], over);
    }
    if (s + 1 < stages) {
#pragma unroll
      for (int i = 0; i < NS; ++i) write(i, buf ^ 1);
    }
    if (s + 2 < stages) {
      const uint32_t k = (uint32_t)(s + 2) * kStep - (s + 2 == stages - 1 ? over : 0);
#pragma unroll
      for (int i = 0; i < NS; ++i) load(i, k);
    }
    mma(f[0]);
    lds_barrier();
    if (s + 1 < stages) read(f[0], buf ^ 1, 0);
    mma(f[1]);
  }

  __syncthreads();  // the outputs go through the same LDS
  int8_t* mine = &lds_all[0][0][0] + wave * (int)(sizeof lds_all / 4);
  if constexpr (SETS == 2) {
    int* sums = reinterpret_cast<int*>(mine) + lane;
#pragma unroll
    for (int x = 0; x < TM * TN * 16; ++x)
      if (set == 1) sums[64 * x] = acc[x / 16 / TN][x / 16 % TN][x % 16];
    __syncthreads();
    if (set == 1) return;
#pragma unroll
    for (int x = 0; x < TM * TN * 16; ++x) acc[x / 16 / TN][x / 16 % TN][x % 16] += sums[64 * x];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  }
  const int64_t mw = m0 + wm, nw = n0 + wn;
  auto out = [&](auto type) {
    constexpr int T = decltype(type)::value;
    if (g.bias) tile_out<T, true, TM, TN, CLAMP>(g, acc, mine, mw, nw, lane);
    else tile_out<T, false, TM, TN, CLAMP>(g, acc, mine, mw, nw, lane);
  };
  if (g.y_type == SONIQ_BF16) out(std::integral_constant<int, SONIQ_BF16>());
  else if (g.y_type == SONIQ_F16) out(std::integral_constant<int, SONIQ_F16>());
  else out(std::integral_constant<int, SONIQ_F32>());
}

// Many tokens of fewer than 16 channels: one output a thread.
__global__ __launch_bounds__(256) void k_i8_short(I8Gemm g) {
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= g.N) return;
  for (int64_t m = blockIdx.y; m < g.M; m += gridDim.y) {
    int sum = 0;
    for (int k = 0; k < g.K; ++k) sum += (int)g.A[m * g.lda + k] * (int)g.W[n * g.ldw + k];
    float y = scaled(sum, g.sa[m], g.sw[n]);
    if (g.bias) y = __fadd_rn(y, g.bias[n]);
    store_y(g, m * g.ldy + n, y);
  }
}

// Threads a row and pieces of 8 elements that each holds: as few as hold the
// row, since a piece past its end still costs its checks and registers, and
// registers cost waves; two a thread keep enough loads in flight.  us in a
// graph, 16-bit rows, and what 256 threads of four pieces (a wave of four up to
// 2048 elements) take:
//   8192 x  300  64, 1:  6.6   9.7     4096 x  6000  256, 3: 16.7  20.2
//   8192 x 1024  64, 2:  9.2  10.8     8192 x  8192  512, 2: 47.7  50.9
//    300 x 2048 256, 1:  4.3   5.5     4096 x 11008  768, 2: 39.7  40.7
//   4096 x 2560 256, 2: 11.7  17.7     4096 x 14336  768, 3: 46.7  49.3
//   4096 x 4096 256, 2: 13.3  18.3     2000 x 20000  768, 3: 30.1  37.3
template <int TYPE>
void launch_rows(const void* A, int64_t M, int64_t K, int64_t lda, int8_t* Q, int64_t ldq, float* s,
                 hipStream_t stream) {
  const auto* a = static_cast<const typename Value<TYPE>::T*>(A);
  auto go = [&](auto threads, auto held) {
    constexpr int T = decltype(threads)::value, kRows = T < 256 ? 256 / T : 1;
    const unsigned grid = (unsigned)std::min<int64_t>((M + kRows - 1) / kRows, 1 << 20);
    k_rows<TYPE, T, decltype(held)::value><<<grid, T < 256 ? 256 : T, 0, stream>>>(a, M, (int)K, lda, Q, ldq, s);
  };
#define GO(T, H) go(std::integral_constant<int, T>(), std::integral_constant<int, H>())
  if (K <= 512 && M > 256) GO(64, 1);
  else if (K <= 1024 && M > 256) GO(64, 2);
  else if (K <= 2048 && M > 1024) GO(64, 4);
  else if (K <= 2048) GO(256, 1);
  else if (K <= 4096) GO(256, 2);
  else if (K <= 6144) GO(256, 3);
  else if (K <= 8192) GO(512, 2);
  else if (K <= 12288) GO(768, 2);
  else GO(768, 3);
#undef GO
}

template <int BM, int BN, bool CLAMP = false, int SETS = 1>
void launch_tile(const I8Gemm& g, hipStream_t stream) {
  const int64_t tm = (g.M + BM - 1) / BM, tn = (g.N + BN - 1) / BN;
  k_i8_tile<BM, BN, CLAMP, SETS>
      <<<(unsigned)((tm * tn + 7) / 8 * 8), 256 * SETS, 0, stream>>>(g, (int)tm, (int)tn);
}

// The tile of a matrix that is no smaller than it.  Larger tiles move fewer
// bytes a product, smaller ones leave fewer CUs idle; below one tile a CU,
// two sets of waves hide what one stage in flight does not.  Times in us of a
// call in a graph, rows of 4096 + 128 bytes (512 in the last lines; weights'
// rows of K bytes take the same, of K + 16 up to a fifth more):
//                        64x64  2 sets  64x128  2 sets  128x128  256x256
//    65 x  4096 x 4096    10.0     9.5    12.4    11.7       -        -
//    80 x 11008 x 4096    17.7    16.0    15.5    13.3       -        -
//   256 x  4096 x 4096    11.3    10.4    12.9    12.2     15.9     44.9
//   256 x 11008 x 4096    27.1    25.4    23.4    25.4     19.1     46.9
//   512 x  4096 x 4096    21.0    18.9    16.6    16.2     18.3     46.4
//  1024 x  4096 x 4096    36.6    33.6    26.9    28.0     22.0     47.3
//  2048 x 11008 x 4096   151.4   158.1   124.2   147.0    101.7    113.0
//  4096 x  4096 x 4096   112.9   117.7    92.1   108.2     74.5     67.6
//   512 x  1024 x 1024     4.6     4.8     5.5     5.9      7.0     20.1
//  2048 x  2048 x  512     7.2     9.0     6.8     9.2      6.8     17.2
// So: 256x256 where it fills at least 85% of the rounds of one tile a CU that
// it takes; else 128x128 from 160 tiles on; else 64x128 from 150 on; else
// 64x64.  Two sets where the tiles give a CU no second one and K is long
// enough to be shared out.
void launch_tiles(const I8Gemm& g, hipStream_t stream) {
  constexpr int64_t kCus = 256;
  auto tiles = [&](int64_t bm, int64_t bn) {
    return g.M < bm || g.N < bn ? 0 : ((g.M + bm - 1) / bm) * ((g.N + bn - 1) / bn);
  };
  const int64_t t256 = tiles(256, 256), t64x128 = tiles(64, 128);
  if (t256 && 100 * t256 >= 85 * kCus * ((t256 + kCus - 1) / kCus)) launch_tile<256, 256>(g, stream);
  else if (tiles(128, 128) >= 160) launch_tile<128, 128>(g, stream);
  else if (t64x128 >= 150) {
    if (t64x128 <= kCus && g.K >= 2048) launch_tile<64, 128, false, 2>(g, stream);
    else launch_tile<64, 128>(g, stream);
  } else if (g.K > 1024) launch_tile<64, 64, false, 2>(g, stream);
  else launch_tile<64, 64>(g, stream);
}

// Up to 16 tokens and 8192 channels, a workgroup takes 16 channels: the
// weights are all that counts, and more workgroups load them sooner.  Else 48:
// the tokens' codes are read once a workgroup, from L2, and would outweigh the
// weights (40 x 11008 x 4096: 12.8 us a call with 16 channels, 11.9 with 48;
// 64 tokens: 18.8 and 13.0; 48 x 4096 x 4096: 7.1 and 8.7).
template <int A8>
void launch_skinny(const I8Gemm& g, hipStream_t stream) {
  if (A8 <= 2 || g.N <= 8192)
    k_i8_skinny<A8, 1><<<(unsigned)((g.N + 15) / 16), 512, 0, stream>>>(g);
  else
    k_i8_skinny<A8, 3><<<(unsigned)((g.N + 47) / 48), 512, 0, stream>>>(g);
}

// Four segments in flight leave two workgroups a CU their registers, two
// segments three, which more than two a CU gain from (us in a graph, four and
// two: 1 x 11008 x 4096 14.0 and 12.4, 2 x 11008 x 8192 24.6 and 20.8, but
// 1 x 4096 x 4096 8.2 and 8.6, 4 x 4096 x 4096 10.4 and 11.0).
template <int TYPE>
void launch_fused(const I8Gemm& g, const void* A, int64_t lda, hipStream_t stream) {
  const auto* a = static_cast<const typename Value<TYPE>::T*>(A);
  const unsigned grid = (unsigned)((g.N + 15) / 16);
  if (grid <= 512) k_i8_fused<TYPE, 4><<<grid, 512, 0, stream>>>(g, a, lda);
  else k_i8_fused<TYPE, 2><<<grid, 512, 0, stream>>>(g, a, lda);
}

}  // namespace

hipError_t launch_quantize_rows(const void* A, int a_type, int64_t M, int64_t K, int64_t lda,
                                int8_t* Q, int64_t ldq, float* s, hipStream_t stream) {
  if (a_type == SONIQ_F32) launch_rows<SONIQ_F32>(A, M, K, lda, Q, ldq, s, stream);
  else if (a_type == SONIQ_BF16) launch_rows<SONIQ_BF16>(A, M, K, lda, Q, ldq, s, stream);
  else launch_rows<SONIQ_F16>(A, M, K, lda, Q, ldq, s, stream);
  return hipGetLastError();
}

bool i8_fused(int64_t M, int64_t K) { return M <= kFusedRows && M * ((K + 7) / 8 * 8) <= kFusedMost; }

hipError_t launch_i8_fused(const I8Gemm& g, const void* A, int a_type, int64_t lda, hipStream_t stream) {
  if (a_type == SONIQ_F32) launch_fused<SONIQ_F32>(g, A, lda, stream);
  else if (a_type == SONIQ_BF16) launch_fused<SONIQ_BF16>(g, A, lda, stream);
  else launch_fused<SONIQ_F16>(g, A, lda, stream);
  return hipGetLastError();
}

hipError_t launch_i8_gemm(const I8Gemm& g, hipStream_t stream) {
  if (g.M <= 8) launch_skinny<1>(g, stream);
  else if (g.M <= 16) launch_skinny<2>(g, stream);
  else if (g.M <= 32) launch_skinny<4>(g, stream);
  else if (g.M <= 48) launch_skinny<6>(g, stream);
  else if (g.M <= 64) launch_skinny<8>(g, stream);
  else if (g.K < 16) k_i8_short<<<dim3((unsigned)((g.N + 255) / 256), (unsigned)std::min<int64_t>(g.M, 65535)), 256, 0, stream>>>(g);
  else if (std::max(g.lda, g.ldw) >= 1 << 24 || g.N < 64) launch_tile<64, 64, true>(g, stream);
  else launch_tiles(g, stream);
  return hipGetLastError();
}

}  // namespace soniq
