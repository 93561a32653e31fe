// gfx950 kernels of the quantized key/value cache and the attention over it.
#include "soniq_serve.h"
#include "soniq_values.h"

#include <algorithm>
#include <type_traits>

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

// Barrier for LDS alone: loads from memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Rows of 8 codes a lane: 8, 16 or 32 lanes (24 of them busy for 192
// elements) a row, so that a row's maximum stays within a wave.
template <int D>
constexpr int kRowLanes = D == 64 ? 8 : D == 128 ? 16 : 32;
constexpr int kCopyTokens = 16;  // tokens a workgroup, at most

// A workgroup takes `tw` tokens, all heads of both sides.  Its first wave
// finds where each token lives; then every thread moves pieces of 8 elements,
// kAhead of them in flight (one at a time reached 3.7 TB/s on long reads:
// 8 bytes a lane and 32 waves do not cover the memory's latency).
//   write: s = max |x| / top, code = rint(x / s);   read: code * s.
// Bytes bound it: reading 500 MB of prefixes (8 sequences, 8 heads of 128, 8
// bits) takes 106 us, 4.7 TB/s, what a large copy reaches; 700 to 4096 tokens
// of 5 sequences read back from 4 bits 16 us.  Writing them takes 20, bound by
// instructions: 8500 a SIMD are some 14 of those.  A token or a few take 3.8 to
// 4.7 us: launch, tables, then one trip to memory.
template <int TYPE, int D, int BITS, bool WRITE>
__global__ __launch_bounds__(256) void k_kv_copy(KvCopy c, int tw) {
  typedef typename Value<TYPE>::T T;
  constexpr int L = kRowLanes<D>, kAhead = 4;
  struct __attribute__((packed, aligned(sizeof(T)))) P { T v[8]; };
  __shared__ int32_t where[kCopyTokens];  // row for head 0, -1 without a page, -2 behind the last sequence
  const int tid = threadIdx.x, t0 = (int)blockIdx.x * tw, H2 = 2 * c.dims.heads;
  const int tokens = min(tw, c.T - t0), pieces = tokens * H2 * L;
  const int d = tid % L * 8;  // 256 is a multiple of L: the same elements of every row
  const bool on = d < D;

  Eight<TYPE> v[kAhead];
  int64_t at[kAhead];    // element of the side's rows
  int side[kAhead], head[kAhead], tok[kAhead];
  auto place = [&](int k, int x) {
    const int row = x / L;
    tok[k] = row / H2;
    const int y = row - tok[k] * H2;
    side[k] = y >= c.dims.heads;
    head[k] = side[k] ? y - c.dims.heads : y;
    const int64_t t = t0 + tok[k];
    at[k] = side[k] ? t * c.side[1].token_stride + head[k] * c.side[1].head_stride
                    : t * c.side[0].token_stride + head[k] * c.side[0].head_stride;
  };
  auto rows = [&](int k) { return static_cast<T*>(side[k] ? c.side[1].rows : c.side[0].rows) + at[k] + d; };
  auto load_rows = [&](int x0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (x0 + 256 * k < pieces) {
        place(k, x0 + 256 * k);
        if (WRITE && on) v[k].load(rows(k));
      }
  };
  load_rows(tid);

  if (tid < 64) {
    int b = 0;  // how many of cu[1 .. B] are at most this lane's token
    for (int i = 0; i < c.table.B; i += 64) {
      const int32_t end = i + tid < c.table.B ? c.cu[i + tid + 1] : 0;
      const uint64_t live = __ballot(i + tid < c.table.B);
#pragma unroll
      for (int k = 0; k < kCopyTokens; ++k) {
        const int n = __popcll(__ballot(end <= t0 + k) & live);
        b += tid == k ? n : 0;
      }
    }
    if (tid < tokens) {
      int32_t row = -2;
      if (b < c.table.B) row = kv_row(c.table, c.dims, b, (int64_t)c.start[b] + ((int64_t)(t0 + tid) - c.cu[b]));
      where[tid] = row;
    }
  }
  lds_barrier();

  for (int x0 = tid; x0 < pieces;) {
    int32_t row0[kAhead];
    uint32_t w[kAhead][2];
    float sc[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      row0[k] = x0 + 256 * k < pieces ? where[tok[k]] : -2;
      w[k][0] = w[k][1] = 0;
      sc[k] = 0.0f;
      if (!WRITE && row0[k] >= 0 && on) {
        const int64_t row = (int64_t)row0[k] + (int64_t)head[k] * c.dims.page_size;
        const uint8_t* codes = (side[k] ? c.side[1].codes : c.side[0].codes) + row * (D * BITS / 8) + d * BITS / 8;
        sc[k] = (side[k] ? c.side[1].scale : c.side[0].scale)[row];
        if constexpr (BITS == 8) {
          const uint2 x = *reinterpret_cast<const uint2*>(codes);
          w[k][0] = x.x, w[k][1] = x.y;
        } else {
          w[k][0] = *reinterpret_cast<const uint32_t*>(codes);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (WRITE) {
        uint32_t mx = on && row0[k] >= 0 ? v[k].amax() : 0;
#pragma unroll
        for (int o = 1; o < L; o *= 2) mx = max(mx, (uint32_t)__shfl_xor((int)mx, o));
        if (row0[k] < 0) continue;
        const RowCoder rc(mx, BITS == 8 ? 127.0f : 7.0f);
        const int64_t row = (int64_t)row0[k] + (int64_t)head[k] * c.dims.page_size;
        if (d == 0) (side[k] ? c.side[1].scale : c.side[0].scale)[row] = rc.s;
        if (!on) continue;
        uint8_t* codes = (side[k] ? c.side[1].codes : c.side[0].codes) + row * (D * BITS / 8) + d * BITS / 8;
        if constexpr (BITS == 8) *reinterpret_cast<uint2*>(codes) = v[k].codes(rc);
        else *reinterpret_cast<uint32_t*>(codes) = v[k].nibbles(rc);
      } else if (on && row0[k] > -2) {
        P y;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int code = BITS == 8 ? (int8_t)(w[k][i / 4] >> (8 * (i % 4))) : (int)(w[k][0] << (28 - 4 * i)) >> 28;
          y.v[i] = Value<TYPE>::store((float)code * sc[k]);
        }
        *reinterpret_cast<P*>(rows(k)) = y;
      }
    }
    x0 += 256 * kAhead;
    load_rows(x0);
  }
}

// ---------------------------------------------------------- attention --
// One workgroup takes 16 * R query rows (new tokens times the heads that
// share a key/value head) of one sequence and key/value head over one part
// of its positions; four waves take 32 positions each in turn, keep their
// own running softmax, and meet at the end.  Parts meet in k_kv_join.
// Single tokens are bound by the cache's bytes: 32 sequences of 2000 to 32768
// positions, 8 heads of 128, 8 bits, 4 query heads each: 199 us for 1.06 GB,
// 5.3 TB/s (a plain read reaches 6.4), and 7 for the join.  Many rows by the
// vector instructions of codes and softmax: 8 sequences of 3001 to 8191
// positions, 96 rows, 4 bits, fp16: 60 us with the join, of which those 18600 a
// SIMD take 31 (matrix cores 10, 50 MB from memory 10); then the starts and ends
// of parts.
//
// Everything stays transposed, so that no operand crosses lanes: with
// kb = lane / 16 and c = lane % 16,
//   S^T = K Q^T  (v_mfma_f32_16x16x32_f16, rows = positions): lane holds the
//         scores of query row c and of positions 4 kb + i and 16 + 4 kb + i;
//   O^T = V^T P^T: those same eight positions, in that order, are the lane's
//         eight k elements, so P goes from the scores' registers into the
//         product; the V operand is 8 positions of one element d, and a lane
//         that loads elements [c * D/16, (c + 1) * D/16) of its eight rows
//         holds D/16 such operands, a byte permute away.
// K and V go from memory to registers; LDS holds the queries' fragments and
// each position's cache row and scales.
//
// Codes become fp16 exactly: a code moved to unsigned, u = code + zero, is the
// fp16 subnormal u * 2^-24, and one packed fma a pair makes it (u - zero) * 2^-15
// for K and 2^-9 for V.  (K could do without, with scores that start from
// -zero * sum(q): 3 to 4% less with many rows, but their sums then round at the
// size of u, which moved scores of 4-bit keys by 20 times what an fp32 sum is
// off by, and by 2e-4 where one channel was 30 times the others.)
// Queries are scaled by a power of two per row to use fp16's whole range (they
// are exact in it down to 2^-28 of the row's largest element).
//
// Softmax of a row over the positions so far, all in fp32 and base 2:
//   p = exp2(s - r),  l = sum p,  w = p * s_v,  outputs = sum w * code.
// The reference r has to do with scores alone: one that was met, so that l
// neither overflows nor vanishes.  The weights go into the product as fp16, in
// a unit of their own, a power of two that follows the largest w so far
// (between 2^6 and 2^14 units of it): only exponents change with it, so that
// scores and V scales may rise and fall against each other over all of fp32's
// range.  Both are rarely moved: where a p passes 2^80, or a w its 2^14 units.
// Half a step of fp16 in each weight is as much as an fp16 output's own and an
// eighth of a bf16 output's, so a second product takes what the rounding left
// (without it, fp16 outputs' error against 64 bits was 1.4 to 1.5 times that of
// rounding the exact output).  When it came it cost single tokens nothing to
// speak of (201 us and 201 for 32 sequences of 2000 to 32768 positions, bf16),
// many rows 3 to 9% (8 sequences of 3001 to 8191 positions, 96 rows, 8 bits,
// bf16: 52.4 and 57.1).
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kSub = 1024;     // positions whose rows and scales LDS holds at a time

// Over the four lanes that share c: the same result in each.
__device__ __forceinline__ float quad_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t v = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t v = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// One step of a row's softmax over N positions a lane.  x: scores without the
// row's unit qf (positive), -inf at hidden positions, where v is 0.  Leaves
// the weights in x, and calls scale(f) where the outputs so far have to be
// multiplied.  A row starts at r = kHidden, where a visible score's exponential
// is infinite and a hidden one's 0, and stays there while it sees nothing.
constexpr float kHidden = -3.402823466e38f;
struct RowSoftmax {
  float r, l;
  float limit;  // 2^14 units of the weights; a power of two
  __device__ __forceinline__ static int exponent(float x) { return (int)(__float_as_uint(x) >> 23) - 127; }
  __device__ __forceinline__ static float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
  __device__ __forceinline__ float per_weight() const { return power(14 - exponent(limit)); }  // units in 1
};
constexpr float kFirstLimit = 0x1p-112f;  // units in 1: 2^126
template <int N, class Scale>
__device__ __forceinline__ void softmax_step(float (&x)[N], const float (&v)[N], float qf, RowSoftmax& st, Scale scale) {
  float w[N], lt, top;
  auto weigh = [&]() {
    lt = 0.0f, top = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], qf, -st.r));
      lt += p;
      w[e] = p * v[e];
      top = fmaxf(top, fabsf(w[e]));
    }
  };
  weigh();
  const uint64_t hot = __ballot(lt > 0x1p80f || top > st.limit);
  if (hot) {
    uint32_t rows = (uint32_t)(hot | hot >> 32);  // bit c: row c, by any of its four lanes
    rows |= rows >> 16;
    const bool moves = rows >> (threadIdx.x % 16) & 1;
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) mx = fmaxf(mx, x[e]);
    mx = quad_max(mx * qf);
    // A row's reference moves up to the highest score with its weights' unit:
    // with exponentials up to 1 no weight can pass fp32's end before it is
    // scaled, and the sum has room.
    float f = 1.0f;
    if (moves && mx > st.r) {
      f = __builtin_amdgcn_exp2f(st.r - mx);
      st.r = mx;
    }
    weigh();
    top = quad_max(top);
    const int was = RowSoftmax::exponent(st.limit) - 8;  // of the largest weight when the unit was chosen
    const int e = moves ? min(max(RowSoftmax::exponent(fmaxf(ldexpf(f, was), top)), -120), 119) : was;
    st.limit = RowSoftmax::power(e + 8);
    st.l *= f;
    scale(ldexpf(f, was - e));
  }
  st.l += lt;
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = w[e];
}

// Weights in their unit as fp16, and what the rounding left of them, cut: 2^-21
// of the weight at most, or 2^-24 of a unit.
__device__ __forceinline__ void weigh_fine(const float (&w)[8], float units, h8& coarse, h8& fine) {
  union { h2 p[4]; h8 v; } a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    asm("v_fma_mixlo_f16 %0, %1, %2, 0" : "=v"(a.p[i]) : "v"(w[2 * i]), "v"(units));
    asm("v_fma_mixhi_f16 %0, %1, %2, 0" : "+v"(a.p[i]) : "v"(w[2 * i + 1]), "v"(units));
    float lo, hi;  // w * units - a, exact
    asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel_hi:[0,0,1]" : "=v"(lo) : "v"(w[2 * i]), "v"(units), "v"(a.p[i]));
    asm("v_fma_mix_f32 %0, %1, %2, -%3 op_sel:[0,0,1] op_sel_hi:[0,0,1]"
        : "=v"(hi) : "v"(w[2 * i + 1]), "v"(units), "v"(a.p[i]));
    b.p[i] = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(lo, hi));
  }
  coarse = a.v, fine = b.v;
}

// Two codes moved to unsigned and held as fp16 subnormals (UP: times 16, as they
// lie in the odd nibbles): the codes times 2^UNIT, exactly.
template <int BITS, bool UP, int UNIT>
__device__ __forceinline__ h2 signed_half(uint32_t u16pair) {
  constexpr float up = (float)(1 << (24 + UNIT)) / (UP ? 16 : 1), zero = (BITS == 8 ? 128.0f : 8.0f) / (float)(1 << -UNIT);
  constexpr _Float16 m = (_Float16)up, z = (_Float16)-zero;
  return __builtin_elementwise_fma(__builtin_bit_cast(h2, u16pair), h2{m, m}, h2{z, z});
}
constexpr int kUnitK = -15, kUnitV = -9;

// Eight K codes as an operand: from two words of 8-bit codes in order, or
// from one word of 4-bit codes in the order 0 4 1 5 2 6 3 7.
template <int BITS>
__device__ __forceinline__ h8 k_operand(const uint32_t* w) {
  union { h2 p[4]; h8 v; } r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (BITS == 8) {
      const uint32_t u = w[i] ^ 0x80808080u;
      r.p[2 * i] = signed_half<8, false, kUnitK>(__builtin_amdgcn_perm(u, u, 0x0c010c00u));
      r.p[2 * i + 1] = signed_half<8, false, kUnitK>(__builtin_amdgcn_perm(u, u, 0x0c030c02u));
    } else {
      const uint32_t u = w[0] >> (8 * i);
      r.p[2 * i] = signed_half<4, false, kUnitK>((u ^ 0x00080008u) & 0x000F000Fu);
      r.p[2 * i + 1] = signed_half<4, true, kUnitK>((u ^ 0x00800080u) & 0x00F000F0u);
    }
  }
  return r.v;
}
// Where element i of a group of eight goes in that operand.
template <int BITS>
__device__ __forceinline__ constexpr int k_order(int i) {
  return BITS == 8 ? i : i < 4 ? 2 * i : 2 * (i - 4) + 1;
}

// Bytes of a lane's share of a row, loaded in the widest pieces.
template <int BYTES>
struct Raw {
  uint32_t w[(BYTES + 3) / 4];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (BYTES == 2) {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    } else if constexpr (BYTES == 6) {
      struct __attribute__((packed, aligned(2))) P { uint32_t a; uint16_t b; };
      const P x = *reinterpret_cast<const P*>(p);
      w[0] = x.a;
      w[1] = x.b;
    } else {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(p + 16 * i);
        w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
      }
      constexpr int r = BYTES % 16, o = BYTES / 16 * 4;
      if constexpr (r == 4) w[o] = *reinterpret_cast<const uint32_t*>(p + 4 * o);
      if constexpr (r == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(p + 4 * o);
        w[o] = x.x, w[o + 1] = x.y;
      }
      if constexpr (r == 12) {
        const uint3 x = *reinterpret_cast<const uint3*>(p + 4 * o);
        w[o] = x.x, w[o + 1] = x.y, w[o + 2] = x.z;
      }
    }
  }
};

// From a lane's V codes of eight positions the operand of its element j.
template <int VB, int BITS>
__device__ __forceinline__ void v_unsigned(Raw<VB>& r) {
  if constexpr (BITS == 8) {
#pragma unroll
    for (int i = 0; i < (VB + 3) / 4; ++i) r.w[i] ^= 0x80808080u;
  }
}
template <int VB, int BITS, bool ODD>
__device__ __forceinline__ h8 v_operand(const Raw<VB> (&r)[8], int j) {
  union { h2 p[4]; h8 v; } x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t lo = r[2 * i].w[j * BITS / 32], hi = r[2 * i + 1].w[j * BITS / 32];
    if constexpr (BITS == 4) {
      lo = ODD ? (lo ^ 0x80808080u) & 0xF0F0F0F0u : (lo ^ 0x08080808u) & 0x0F0F0F0Fu;
      hi = ODD ? (hi ^ 0x80808080u) & 0xF0F0F0F0u : (hi ^ 0x08080808u) & 0x0F0F0F0Fu;
    }
    const uint32_t by = j * BITS / 8 % 4;
    x.p[i] = signed_half<BITS, BITS == 4 && ODD, kUnitV>(__builtin_amdgcn_perm(hi, lo, 0x0c000c00u | (4 + by) << 16 | by));
  }
  return x.v;
}

// Which of the 32 positions from new position j0 on (negative: older ones)
// new query i of ragged row t sees.
__device__ __forceinline__ uint32_t seen_bits(const KvAttend& a, int64_t t, int i, int64_t j0) {
  if (j0 <= -32) return ~0u;
  const uint32_t old = j0 < 0 ? (1u << -j0) - 1u : 0u;
  if (!a.mask) {
    const int64_t n = i - j0 + 1;
    return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
  }
  const uint64_t* w = a.mask + t * a.mask_words;
  if (j0 < 0) return old | (uint32_t)(w[0] << -j0);
  const int64_t x = j0 / 64;
  const int sh = (int)(j0 % 64);
  if (x >= a.mask_words) return 0u;
  uint64_t v = w[x] >> sh;
  if (sh > 32 && x + 1 < a.mask_words) v |= w[x + 1] << (64 - sh);
  return (uint32_t)v;
}

// How a launch is cut.  Lengths count in pieces of 128 positions here.
struct KvSplit {
  int R;       // 16-row tiles a workgroup
  int RB;      // workgroups over the rows
  int parts;   // parts of a sequence, at most
  int chunk;   // pieces of a part, at least
  int cap;     // and at most, where `parts` allows (0: `chunk` as it is)
  float per;   // parts of all sequences that make one workgroup a CU
  int waves;   // workgroups a CU that are resident at once
  bool pad;    // more LDS than is used, so that no more than two are
  int least;   // and that the parts are to make, at least
};

// Inclusive sums over the lanes of a wave.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

__device__ __forceinline__ uint32_t pieces_of(int len) { return ((uint32_t)len + 127) / 128; }

// Pieces a part takes, from the lengths themselves (lane b: those of sequence
// b, 0 past the last; up to 64 sequences): the parts of all of them are to
// make `least` workgroups a CU, or as many more up to all that are resident,
// or twice, three times those, as `cap` asks for.  Floats only choose;
// whatever they choose is cut exactly by part_of.
__device__ __forceinline__ uint32_t kv_chunk(const KvSplit& sp, uint32_t pieces) {
  if (sp.cap == 0) return sp.chunk;
  const float total = (float)wave_sum(pieces), fl = (float)pieces, cap = (float)sp.cap, all = (float)sp.waves;
  float w = fmaxf(ceilf(total / (sp.per * cap)), (float)sp.least);
  if (w > all) w = ceilf(w / all) * all;
  const float want = w * sp.per;
  float c = fminf(fmaxf(ceilf(total / want), (float)sp.chunk), cap);
  for (int i = 0; i < 8 && c < cap; ++i) {
    const float n = (float)wave_sum((uint32_t)ceilf(fl * __builtin_amdgcn_rcpf(c) - 0.001f));
    if (n <= want) break;
    c = fminf(c + fmaxf(1.0f, floorf(c * 0.0625f)), cap);
  }
  return __builtin_amdgcn_readfirstlane((uint32_t)c);
}
// The same for one sequence: no more than `parts` of them.
__device__ __forceinline__ uint32_t kv_chunk_of(uint32_t pieces, uint32_t chunk, int parts) {
  return max(chunk, (pieces + parts - 1) / (uint32_t)parts);
}

// The positions of one part: [first, first + count).
struct KvPart {
  int first, count, used;  // used: parts of this sequence that hold positions
};
__device__ __forceinline__ KvPart part_of(int len, int part, int parts, uint32_t chunk) {
  // len < 2^31, chunk <= 2^24, part < 2^22
  const uint32_t pieces = pieces_of(len), c = kv_chunk_of(pieces, chunk, parts);
  const uint64_t first = (uint64_t)part * c * 128;
  const int count = first >= (uint64_t)len ? 0 : (int)min((uint64_t)c * 128, len - first);
  return {(int)first, count, (int)((pieces + c - 1) / c)};
}
// Pieces of sequence `lane`, for the two calls above.
__device__ __forceinline__ uint32_t kv_lane_pieces(const KvAttend& a, int lane) {
  return lane < a.table.B ? pieces_of(kv_length(a.table, a.dims, a.kv_len[lane])) : 0;
}

// What a workgroup works on.
struct KvUnit {
  KvSpan span;    // the sequence's rows of the ragged batch
  int nq, len;    // its queries that are computed, its positions
  int64_t base;   // its positions before the new ones (may be negative)
  int b, h, part, row0, rows;  // row0, rows: query rows (query * group + head) of this workgroup
  KvPart pt;
};
// Workgroups of the same positions go to one XCD, one after the other.
// False: there is nothing to do.
__device__ __forceinline__ bool kv_unit(const KvAttend& a, const KvSplit& sp, int lane, KvUnit& u) {
  const uint32_t id = blockIdx.x, x = id / 8;
  const int rb = (int)(x % sp.RB), unit = (int)(x / sp.RB) * 8 + (int)(id % 8);
  const int bp = unit / a.dims.heads;
  u.h = unit % a.dims.heads;
  uint32_t chunk = sp.chunk;
  if (sp.cap == 0) {
    u.part = bp % sp.parts, u.b = bp / sp.parts;
    if (u.b >= a.table.B) return false;
  } else {
    // the parts that hold positions, and one of each sequence without any, come first
    const uint32_t pieces = kv_lane_pieces(a, lane);
    chunk = kv_chunk(sp, pieces);
    const uint32_t c = kv_chunk_of(pieces, chunk, sp.parts);
    const uint32_t n = lane < a.table.B ? max((pieces + c - 1) / c, 1u) : 0, end = wave_scan(n);
    u.b = __popcll(__ballot(end <= (uint32_t)bp));
    if (u.b >= a.table.B) return false;
    u.part = bp - (int)__builtin_amdgcn_readlane(end - n, u.b);
  }
  u.span = kv_span(a.cu[u.b], a.cu[u.b + 1], a.T);
  u.nq = min(u.span.count, a.max_q);
  u.len = kv_length(a.table, a.dims, a.kv_len[u.b]);
  u.base = (int64_t)a.kv_len[u.b] - u.span.count;
  u.row0 = rb * 16 * sp.R;
  u.rows = min(u.nq * a.group - u.row0, 16 * sp.R);
  u.pt = part_of(u.len, u.part, sp.parts, chunk);
  return u.rows > 0 && (u.part == 0 || u.pt.count > 0);
}

// Per query row: the unit of its scores, its query (-1: none).
template <int ROWS>
struct KvRowInfo {
  float qf[ROWS];
  int32_t qi[ROWS];
};

// The queries of 16 * R rows on their way to LDS as operands: loaded before
// anything waits, turned once the K and V loads are out.
template <int D, int BITS, int R>
struct KvQuery {
  // threads a row: a power of two that leaves each a multiple of 8 elements
  static constexpr int kMost = D % 128 == 0 ? 16 : 8, TPR = 16 / R < kMost ? 16 / R : kMost, PER = D / TPR;
  struct __attribute__((packed, aligned(2))) P { uint16_t v[8]; };
  P raw[PER / 8];
  __device__ __forceinline__ void load(const KvAttend& a, const KvUnit& u, int tid) {
    const int r = tid / TPR, d = tid % TPR * PER;
    if (r < u.rows) {  // rows <= 16 R: the threads past them have none
      const int64_t t = u.span.first + (u.row0 + r) / a.group;
      const int64_t at = t * a.q_ts + ((int64_t)u.h * a.group + (u.row0 + r) % a.group) * a.q_hs + d;
      const uint16_t* p = static_cast<const uint16_t*>(a.q) + at;
#pragma unroll
      for (int g = 0; g < PER / 8; ++g) raw[g] = *reinterpret_cast<const P*>(p + 8 * g);
    } else {
#pragma unroll
      for (int g = 0; g < PER / 8; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) raw[g].v[i] = 0;
    }
  }
  __device__ __forceinline__ void stage(const KvAttend& a, const KvUnit& u, int tid, h8 (*q)[D / 32][64],
                                        KvRowInfo<16 * R>& info) const {
    if (tid >= 16 * R * TPR) return;
    const int r = tid / TPR, d0 = tid % TPR * PER;
    auto value = [&](int i) {
      const uint16_t x = raw[i / 8].v[i % 8];
      return a.type == SONIQ_BF16 ? bf16_value(x) : (float)__builtin_bit_cast(_Float16, x);
    };
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) mx = max(mx, __float_as_uint(value(i)) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = 1; o < TPR; o *= 2) mx = max(mx, (uint32_t)__shfl_xor((int)mx, o));
    // largest element to [2^14, 2^15); rows of zeros, infinities or NaN as they are
    int e = (int)(mx >> 23) - 127 - 14;
    e = mx >= 0x7F800000u || mx == 0 ? 0 : max(e, -126);
    const float down = copysignf(__uint_as_float((uint32_t)(127 - e) << 23), a.scale);
#pragma unroll
    for (int g = 0; g < PER / 8; ++g) {
      h8 v;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k_order<BITS>(i)] = (_Float16)(value(8 * g + i) * down);
      const int d = d0 + 8 * g;
      q[r / 16][d % (D / 4) / 8][d / (D / 4) * 16 + r % 16] = v;
    }
    if (tid % TPR == 0) {
      // (never 0: hidden positions stay at -inf)
      info.qf[r] = fmaxf(fabsf(a.scale) * 1.44269504f * (float)(1 << -kUnitK) * __uint_as_float((uint32_t)(127 + e) << 23), 0x1p-126f);
      info.qi[r] = r < u.rows ? (u.row0 + r) / a.group : -1;
    }
  }
};

// Positions [p0, p0 + n) of a sequence, n <= kSub, in LDS: cache row, scales,
// validity (a position without a page has row 0 and a clear bit).
struct KvPositions {
  uint32_t row[kSub];
  float ks[kSub], vs[kSub];
  uint32_t valid[kSub / 32];
};
struct KvFind {
  int32_t at[kSub / 256];
  float ks[kSub / 256], vs[kSub / 256];
  __device__ __forceinline__ void find(const KvAttend& a, const KvUnit& u, int p0, int n, int tid) {
#pragma unroll
    for (int k = 0; k < kSub / 256; ++k) {
      const int x = tid + 256 * k;
      at[k] = x < n ? kv_row(a.table, a.dims, u.b, (int64_t)p0 + x) : -1;
    }
  }
  __device__ __forceinline__ void rows(const KvAttend& a, const KvUnit& u, int n, int tid, KvPositions& L) {
#pragma unroll
    for (int k = 0; k < kSub / 256; ++k) {
      const int x = tid + 256 * k;
      ks[k] = vs[k] = 0.0f;
      if (256 * k < n) {
        const uint64_t there = __ballot(at[k] >= 0);
        if (tid % 64 == 0) L.valid[x / 32] = (uint32_t)there;
        if (tid % 64 == 32) L.valid[x / 32] = (uint32_t)(there >> 32);
        const int32_t row = at[k] < 0 ? 0 : at[k] + u.h * a.dims.page_size;
        L.row[x] = row;
        ks[k] = a.ks[row], vs[k] = a.vs[row];
      }
    }
  }
  // A key whose scale is infinite holds no numbers (soniq_kv_write stores a row
  // with an infinity as codes 0): its score is NaN, never an infinity of the
  // sign of whatever the codes sum up to, since -inf would hide the position.
  __device__ __forceinline__ void scales(int n, int tid, KvPositions& L) const {
#pragma unroll
    for (int k = 0; k < kSub / 256; ++k)
      if (256 * k < n) {
        L.ks[tid + 256 * k] = __builtin_isinf(ks[k]) ? __builtin_nanf("") : ks[k];
        L.vs[tid + 256 * k] = vs[k];
      }
  }
};

template <int D, int R>
struct KvLds {
  KvPositions p;
  h8 q[R][D / 32][64];
  KvRowInfo<16 * R> info;
};

template <int D>
constexpr int kOutPitch = D + 4;  // of the outputs in LDS
template <int D, int R>
constexpr size_t kv_lds() {
  constexpr size_t loop = sizeof(KvLds<D, R>), out = (size_t)4 * 16 * kOutPitch<D> * 4 + 4 * 16 * 12;
  return loop > out ? loop : out;
}

// Waves a SIMD, by the registers that a row tile's outputs take.
constexpr int kv_waves(int D, int R) {
  return D * R <= 64 ? 5 : D * R <= 128 ? 4 : D * R <= 192 || D == 128 ? 3 : 2;
}

template <int D, int BITS, int R>
__global__ __launch_bounds__(256, kv_waves(D, R)) void k_kv_attend(KvAttend a, KvSplit sp) {
  constexpr int RB = D * BITS / 8;   // bytes of a cache row
  constexpr int KB = RB / 4, VB = RB / 16;
  constexpr int NK = D / 32;         // products over d
  constexpr int DB = D / 16;         // elements of d a lane holds, and V operands
  constexpr int OP = kOutPitch<D>;
  __shared__ __align__(16) uint8_t lds_bytes[kv_lds<D, R>()];
  KvLds<D, R>& L = *reinterpret_cast<KvLds<D, R>*>(lds_bytes);

  KvUnit un;
  if (!kv_unit(a, sp, threadIdx.x % 64, un)) return;
  const int h = un.h, G = a.group, nq = un.nq, row0 = un.row0;
  const KvSpan span = un.span;
  const KvPart pt = un.pt;
  const int64_t base = un.base;
  int tid = threadIdx.x, lane = tid % 64, c = lane % 16, kb = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);  // uniform, and known to be

  f4 O[R][DB];
  RowSoftmax sm[R];
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
#pragma unroll
    for (int j = 0; j < DB; ++j) O[rt][j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    sm[rt] = {kHidden, 0.0f, kFirstLimit};
  }

  const uint8_t* kp = a.k + kb * KB;
  const uint8_t* vp = a.v + c * VB;
  Raw<KB> kr[2];
  Raw<VB> vr[8];
  auto load_k = [&](int st) {
#pragma unroll
    for (int t = 0; t < 2; ++t) kr[t].load(kp + (uint64_t)L.p.row[st * 32 + 16 * t + c] * RB);
  };
  auto load_v = [&](int st) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint4 x = *reinterpret_cast<const uint4*>(&L.p.row[st * 32 + 16 * t + 4 * kb]);
      vr[4 * t].load(vp + (uint64_t)x.x * RB);
      vr[4 * t + 1].load(vp + (uint64_t)x.y * RB);
      vr[4 * t + 2].load(vp + (uint64_t)x.z * RB);
      vr[4 * t + 3].load(vp + (uint64_t)x.w * RB);
    }
  };

  // Positions [s0, s0 + kSub) of the part into LDS, with this wave's first K
  // and V on their way.
  auto prepare = [&](int s0, auto first) {
    const int n = min(pt.count - s0, kSub);
    int x = tid;
    asm volatile("" : "+v"(x));  // nothing of this is kept over the loop
    KvFind f;
    KvQuery<D, BITS, R> q;
    f.find(a, un, pt.first + s0, n, x);
    if constexpr (decltype(first)::value) q.load(a, un, x);
    f.rows(a, un, n, x, L.p);
    lds_barrier();
    if (wave < (n + 31) / 32) {
      load_k(wave);
      load_v(wave);
    }
    if constexpr (decltype(first)::value) q.stage(a, un, x, L.q, L.info);
    f.scales(n, x, L.p);
    lds_barrier();
  };

  prepare(0, std::true_type());
  for (int s0 = 0;;) {
    const int n = min(pt.count - s0, kSub), nst = (n + 31) / 32, p0 = pt.first + s0;
    for (int st = wave; st < nst; st += 4) {
      const bool more = st + 4 < nst;
      f4 S[R][2];
#pragma unroll
      for (int rt = 0; rt < R; ++rt) S[rt][0] = S[rt][1] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        if constexpr (D * R > 256) __builtin_amdgcn_sched_barrier(0);
        const h8 k0 = k_operand<BITS>(&kr[0].w[s * (BITS == 8 ? 2 : 1)]);
        const h8 k1 = k_operand<BITS>(&kr[1].w[s * (BITS == 8 ? 2 : 1)]);
#pragma unroll
        for (int rt = 0; rt < R; ++rt) {
          const h8 q = L.q[rt][s][lane];
          S[rt][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q, S[rt][0], 0, 0, 0);
          S[rt][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q, S[rt][1], 0, 0, 0);
        }
      }
      if (more) load_k(st + 4);

      const uint32_t valid = __builtin_amdgcn_readfirstlane(L.p.valid[st]);
      const int64_t j0 = (int64_t)p0 + st * 32 - base;
      const bool whole = valid == ~0u && j0 <= -32;
      h8 P[R], fine[R];
#pragma unroll
      for (int rt = 0; rt < R; ++rt) {
        if constexpr (R > 1) __builtin_amdgcn_sched_barrier(0);
        int x = 16 * rt + c, y = st * 32 + 4 * kb;
        asm volatile("" : "+v"(x), "+v"(y));  // read here: nothing of this is kept over the row tiles
        const float qf = L.info.qf[x];
        const f4 ks0 = *reinterpret_cast<const f4*>(&L.p.ks[y]), ks1 = *reinterpret_cast<const f4*>(&L.p.ks[y + 16]);
        const f4 vs0 = *reinterpret_cast<const f4*>(&L.p.vs[y]), vs1 = *reinterpret_cast<const f4*>(&L.p.vs[y + 16]);
        float s[8], v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[i] = S[rt][0][i] * ks0[i], s[4 + i] = S[rt][1][i] * ks1[i];
          v[i] = vs0[i], v[4 + i] = vs1[i];
        }
        if (!whole) {
          const int i = L.info.qi[x];
          const uint32_t bits = (i >= 0 ? valid & seen_bits(a, span.first + i, i, j0) : 0u) >> (4 * kb);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool on = (bits >> (16 * (e / 4) + e % 4)) & 1;
            s[e] = on ? s[e] : -INFINITY;
            v[e] = on ? v[e] : 0.0f;
          }
        }
        softmax_step<8>(s, v, qf, sm[rt], [&](float f) {
#pragma unroll
          for (int j = 0; j < DB; ++j) O[rt][j] *= f;
        });
        weigh_fine(s, sm[rt].per_weight(), P[rt], fine[rt]);
      }

      // O^T += V^T P^T, one element of d per lane column at a time
      if constexpr (R > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int e = 0; e < 8; ++e) v_unsigned<VB, BITS>(vr[e]);
#pragma unroll
      for (int j = 0; j < DB; ++j) {
        const h8 x = j % 2 ? v_operand<VB, BITS, true>(vr, j) : v_operand<VB, BITS, false>(vr, j);
#pragma unroll
        for (int rt = 0; rt < R; ++rt) {
          O[rt][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, P[rt], O[rt][j], 0, 0, 0);
          O[rt][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, fine[rt], O[rt][j], 0, 0, 0);
        }
      }
      if (more) load_v(st + 4);
    }
    s0 += kSub;
    if (s0 >= pt.count) break;
    lds_barrier();  // this sub-part's rows and scales have been read
    prepare(s0, std::false_type());
  }

  // ---- the four waves meet, one row tile at a time
  asm volatile("" : "+v"(tid), "+v"(c), "+v"(kb));  // nor of this
  float* out = reinterpret_cast<float*>(lds_bytes);       // [wave][16][OP]
  float* ml = out + 4 * 16 * OP;                          // [wave][16]: r, l, limit
  const bool direct = pt.used <= 1;
  float* ml_out = a.work + (int64_t)a.T * a.q_heads * sp.parts * D;
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    __syncthreads();
    const float ls = quad_sum(sm[rt].l);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* o = out + (wave * 16 + c) * OP + (4 * kb + i) * DB;
#pragma unroll
      for (int j = 0; j < DB; ++j) o[j] = O[rt][j][i];
    }
    if (kb == 0) {
      float* x = ml + (wave * 16 + c) * 3;
      x[0] = sm[rt].r, x[1] = ls, x[2] = sm[rt].limit;
    }
    __syncthreads();
    for (int x = tid; x < 16 * (D / 4); x += 256) {
      const int r = x / (D / 4), d = x % (D / 4) * 4, rr = row0 + 16 * rt + r;
      if (rr >= nq * G) continue;
      // Normalised here, also where parts are to meet: V's own range then bounds
      // what is stored.  Codes were taken times 2^kUnitV, weights in units
      // of 2^-14 limit; 2^80 more keeps the factors in range until they meet.
      const float* x4 = ml + 3 * r;
      float M = x4[0], sum = 0.0f, f[4];
#pragma unroll
      for (int w = 1; w < 4; ++w) M = fmaxf(M, x4[48 * w]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        f[w] = __builtin_amdgcn_exp2f(x4[48 * w] - M);
        sum += x4[48 * w + 1] * f[w];
      }
      const float by = sum == 0.0f ? 0.0f : 0x1p80f / sum;
      f4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < 4; ++w)
        o += *reinterpret_cast<const f4*>(out + (w * 16 + r) * OP + d) *
             ldexpf(f[w] * by, RowSoftmax::exponent(x4[48 * w + 2]) - 14 - kUnitV - 80);
      const int64_t t = span.first + rr / G, hq = (int64_t)h * G + rr % G;
      if (direct) {
        const int64_t at = t * a.o_ts + hq * a.o_hs + d;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (a.type == SONIQ_BF16) static_cast<uint16_t*>(a.out)[at + i] = bf16_bits(o[i]);
          else static_cast<_Float16*>(a.out)[at + i] = (_Float16)o[i];
        }
        if (d == 0 && a.lse)
          a.lse[t * a.q_heads + hq] = sum == 0.0f ? -INFINITY : (M + __log2f(sum)) * 0.693147181f;
      } else {
        const int64_t x = (t * a.q_heads + hq) * sp.parts + un.part;
        *reinterpret_cast<f4*>(a.work + x * D + d) = o;
        if (d == 0) ml_out[2 * x] = M, ml_out[2 * x + 1] = sum;
      }
    }
  }
}

// Weighted means o of sums l relative to exp2(m), joined with K more.  A part
// that met a NaN alone has no maximum, but its sum.
template <int K, int E>
__device__ __forceinline__ void join_parts(float& m, float& l, float (&o)[E], const float (&pm)[K], const float (&pl)[K],
                                           const float (&po)[K][E]) {
  float M = m, b[K];
#pragma unroll
  for (int k = 0; k < K; ++k) M = fmaxf(M, pm[k]);
  const float a = l * __builtin_amdgcn_exp2f(m - M);
  l = a;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    b[k] = pl[k] * __builtin_amdgcn_exp2f(pm[k] - M);
    l += b[k];
  }
  m = M;
  const float by = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    o[i] *= a * by;
#pragma unroll
    for (int k = 0; k < K; ++k) o[i] += po[k][i] * (b[k] * by);
  }
}

// Joins the parts of one (token, query head): W waves take every W-th part
// each and meet in LDS (W = 1: a wave by itself, four rows a workgroup).  4
// to 7 us: one look at the lengths, then a trip to memory every four parts.
template <int D, int W>
__global__ __launch_bounds__(256) void k_kv_join(KvAttend a, KvSplit sp) {
  constexpr int E = D / 64, kAhead = 4;
  __shared__ float out[W == 1 ? 1 : W][D], ml[W == 1 ? 1 : W][2];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t x = (int64_t)blockIdx.x * (4 / W) + (W == 1 ? wave : 0);
  const int64_t t = x / a.q_heads;
  const int hq = (int)(x % a.q_heads), first = W == 1 ? 0 : wave;
  if (t >= a.T) return;
  const int b = row_sequence(a.cu, a.table.B, (int)t);
  if (b >= a.table.B) return;
  const KvSpan span = kv_span(a.cu[b], a.cu[b + 1], a.T);
  if (t < span.first || t - span.first >= min(span.count, a.max_q)) return;
  const uint32_t chunk = sp.cap == 0 ? sp.chunk : kv_chunk(sp, kv_lane_pieces(a, lane));
  const KvPart pt = part_of(kv_length(a.table, a.dims, a.kv_len[b]), 0, sp.parts, chunk);
  if (pt.used <= 1) return;  // written where it was computed
  const float* w = a.work + x * sp.parts * D;
  const float* wml = a.work + (int64_t)a.T * a.q_heads * sp.parts * D + x * sp.parts * 2;
  float m = kHidden, l = 0.0f, o[E] = {};
  // kAhead parts' loads at a time (past the last one: the first again, weightless)
  for (int p0 = first; p0 < pt.used; p0 += W * kAhead) {
    float pm[kAhead], pl[kAhead], po[kAhead][E];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const bool on = p0 + W * k < pt.used;
      const int p = on ? p0 + W * k : p0;
      pm[k] = on ? wml[2 * p] : kHidden, pl[k] = on ? wml[2 * p + 1] : 0.0f;
#pragma unroll
      for (int i = 0; i < E; ++i) po[k][i] = on ? w[(int64_t)p * D + E * lane + i] : 0.0f;
    }
    join_parts(m, l, o, pm, pl, po);
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int i = 0; i < E; ++i) out[wave][E * lane + i] = o[i];
    if (lane == 0) ml[wave][0] = m, ml[wave][1] = l;
    __syncthreads();
    if (wave) return;
    float pm[W - 1], pl[W - 1], po[W - 1][E];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
      pm[k] = ml[k + 1][0], pl[k] = ml[k + 1][1];
#pragma unroll
      for (int i = 0; i < E; ++i) po[k][i] = out[k + 1][E * lane + i];
    }
    join_parts(m, l, o, pm, pl, po);
  }
  const int64_t at = t * a.o_ts + hq * a.o_hs + E * lane;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    if (a.type == SONIQ_BF16) static_cast<uint16_t*>(a.out)[at + i] = bf16_bits(o[i]);
    else static_cast<_Float16*>(a.out)[at + i] = (_Float16)o[i];
  }
  if (lane == 0 && a.lse) a.lse[x] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * 0.693147181f;
}

// Rows a workgroup takes, and how the positions are cut.  A part costs its
// workgroup a start of several dependent loads, and 4 bytes an output written
// and read again; and parts that are not all resident end unevenly.  So up to
// 64 sequences are cut on the device, by their lengths (see kv_chunk).  Times
// below are us a call in a graph, 8 heads of 128, 8 bits, bf16.
//  - Parts have at most 1024 positions a row tile, or more where that would
//    make more than eight thousand workgroups (32 sequences of 2000 to 32768
//    positions: 203, 217 with two thousand, 203 with 32 thousand; 64 of 20000
//    to 32768: 648, 659, 658).
//  - Two row tiles and short parts: two workgroups a CU, held there by LDS that
//    nobody uses, finish sooner than three with shorter parts yet; three where
//    two would have parts past nine pieces.  Cut by the longest sequence, and by
//    lengths with two and with three:
//      sequences  positions     rows   longest   two   three
//          4     1001 to 4191     96     30.6    29.0   31.7
//          4     3001 to 8191     32     31.4    26.9   29.2
//          8     3001 to 8191     20     31.1    31.1   31.6
//          8     3001 to 8191     64     45.5    50.4   46.1
//          8     3001 to 8191     96     66.8    73.0   62.9
//         16     3001 to 8191     40     93.4    98.2   88.8
//  - `least`: as many parts as are resident with two row tiles (the 96 rows of
//    8 sequences take 69.7 with two a CU), two a CU with one.
// More sequences, or few positions: by the longest one's length, about a
// thousand workgroups.  Up to 512 positions (384 with two row tiles) stay in
// one part, which needs no second launch, and that is 3 more from Python (one
// sequence, 4 query heads a head: 200 positions 7.7 and 8.9 in two launches, 384
// 8.9 and 9.2, 512 10.1 and 9.0, 768 12.2 and 9.6; 48 rows: 200 positions 11.3
// and 12.0, 384 13.2 and 12.3, 512 15.0 and 12.1).
// Four row tiles a wave spill, and so do two with 8-bit heads of 256 elements
// (32 bytes a lane).
KvSplit kv_split(const KvDims& d, int32_t q_heads, int64_t B, int64_t max_q, int64_t max_kv) {
  const int64_t rows = max_q * (q_heads / d.heads);
  KvSplit s;
  s.R = rows <= 16 ? 1 : 2;
  s.RB = (int)((rows + 16 * s.R - 1) / (16 * s.R));
  const int64_t units = B * d.heads * s.RB, pieces = max_kv < 1 ? 1 : (max_kv + 127) / 128;
  auto over = [&](int64_t n) { return std::min((pieces * units + n - 1) / n, (int64_t)1 << 24); };
  const bool by_lengths = B <= 64 && pieces * units > 512;
  const int64_t cap = std::max<int64_t>(8 * s.R, over(8192));
  const int64_t chunk = pieces <= (s.R == 1 ? 4 : 3) ? pieces : std::min(over(1024), cap);
  const int64_t parts = std::min((pieces + chunk - 1) / chunk, std::max<int64_t>(((int64_t)1 << 22) / units, 1));
  s.chunk = (int)chunk;
  s.parts = (int)parts;
  s.cap = by_lengths && parts > 1 ? (int)cap : 0;
  s.per = 256.0f / ((float)d.heads * (float)s.RB);
  s.waves = kv_waves(d.head_dim, s.R);
  s.pad = s.R == 2 && s.waves > 2 && s.cap && over(3 * 256) <= 9;
  if (s.pad) s.waves = 2;
  s.least = s.R == 2 ? s.waves : 2;
  return s;
}

template <int D, int BITS>
void launch_attend(const KvAttend& a, const KvSplit& s, hipStream_t stream) {
  const int64_t u = (int64_t)a.table.B * a.dims.heads * s.parts;
  const dim3 grid((unsigned)((u + 7) / 8 * 8 * s.RB)), block(256);
  constexpr size_t kTwo = 56 << 10;  // of 160 KB
  const size_t pad = s.pad ? kTwo - std::min(kTwo, kv_lds<D, 2>()) : 0;
  if (s.R == 1) k_kv_attend<D, BITS, 1><<<grid, block, 0, stream>>>(a, s);
  else k_kv_attend<D, BITS, 2><<<grid, block, pad, stream>>>(a, s);
  if (s.parts <= 1) return;
  const int64_t x = (int64_t)a.T * a.q_heads;
  // a wave a row, or four where rows are few and parts many (us a call, a wave
  // and four: 16 sequences of 501 to 2191 positions, 4096 rows, 26.8 and 31.2;
  // one token over 200000 positions 122 and 98)
  if (s.parts <= 8 || (s.parts <= 32 && x >= 2048)) k_kv_join<D, 1><<<(unsigned)((x + 3) / 4), 256, 0, stream>>>(a, s);
  else k_kv_join<D, 4><<<(unsigned)x, 256, 0, stream>>>(a, s);
}

template <bool WRITE, int D, int BITS>
void launch_kv_copy(const KvCopy& c, hipStream_t stream) {
  // one token a workgroup until there are two thousand workgroups, then whole
  // rounds of its pieces; writes take one round, whose codes cost arithmetic
  // that other workgroups' loads hide
  const int round = std::max(4 * 256 / (2 * c.dims.heads * kRowLanes<D>), 1);
  int tw = std::min(std::max(c.T / 2048, 1), WRITE ? std::min(round, kCopyTokens) : kCopyTokens);
  if (tw > round) tw = tw / round * round;
  const unsigned grid = (unsigned)((c.T + tw - 1) / tw);
  if (c.type == SONIQ_F32) k_kv_copy<SONIQ_F32, D, BITS, WRITE><<<grid, 256, 0, stream>>>(c, tw);
  else if (c.type == SONIQ_BF16) k_kv_copy<SONIQ_BF16, D, BITS, WRITE><<<grid, 256, 0, stream>>>(c, tw);
  else k_kv_copy<SONIQ_F16, D, BITS, WRITE><<<grid, 256, 0, stream>>>(c, tw);
}
template <bool WRITE>
hipError_t launch_kv_copy(const KvCopy& c, hipStream_t stream) {
  const bool b8 = c.dims.bits == 8;
  switch (c.dims.head_dim) {
    case 64: b8 ? launch_kv_copy<WRITE, 64, 8>(c, stream) : launch_kv_copy<WRITE, 64, 4>(c, stream); break;
    case 128: b8 ? launch_kv_copy<WRITE, 128, 8>(c, stream) : launch_kv_copy<WRITE, 128, 4>(c, stream); break;
    case 192: b8 ? launch_kv_copy<WRITE, 192, 8>(c, stream) : launch_kv_copy<WRITE, 192, 4>(c, stream); break;
    default: b8 ? launch_kv_copy<WRITE, 256, 8>(c, stream) : launch_kv_copy<WRITE, 256, 4>(c, stream); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const KvCopy& c, hipStream_t stream) { return launch_kv_copy<true>(c, stream); }
hipError_t launch_kv_read(const KvCopy& c, hipStream_t stream) { return launch_kv_copy<false>(c, stream); }

int64_t kv_attention_work_bytes(const KvDims& d, int64_t T, int32_t q_heads, int64_t B,
                                int64_t max_q, int64_t max_kv) {
  const KvSplit s = kv_split(d, q_heads, B, max_q, max_kv);
  return s.parts > 1 ? T * q_heads * s.parts * (d.head_dim + 2) * 4 : 0;
}

hipError_t launch_kv_attention(const KvAttend& a, hipStream_t stream) {
  const KvSplit s = kv_split(a.dims, a.q_heads, a.table.B, a.max_q, a.max_kv);
  const bool b8 = a.dims.bits == 8;
  switch (a.dims.head_dim) {
    case 64: b8 ? launch_attend<64, 8>(a, s, stream) : launch_attend<64, 4>(a, s, stream); break;
    case 128: b8 ? launch_attend<128, 8>(a, s, stream) : launch_attend<128, 4>(a, s, stream); break;
    case 192: b8 ? launch_attend<192, 8>(a, s, stream) : launch_attend<192, 4>(a, s, stream); break;
    default: b8 ? launch_attend<256, 8>(a, s, stream) : launch_attend<256, 4>(a, s, stream); break;
  }
  return hipGetLastError();
}

}  // namespace soniq
