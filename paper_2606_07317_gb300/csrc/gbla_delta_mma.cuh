// Pieces shared by the chunked kernels of the gated delta rule: warp-level matrix products
// whose left operand is the result of another (in registers), tiles in shared memory, and
// the layout of what a chunk prepares.
#pragma once

#include <type_traits>

#include "gbla_decay.cuh"
#include "gbla_internal.cuh"
#include "gbla_sm100.cuh"

namespace gbla {
namespace delta {

using namespace sm100;

// ------------------------------------------------------------- matrix products
// c (16 x 8, fp32) += a b with the row index of c in lane / 4 (and + 8) and its column
// pair in lane % 4.  A tile c of one product is, register by register, half the left
// operand of the next one in bf16 (k = 16), and the whole one in tf32 (k = 8, with the
// columns 2t and 2t + 1 in the places of t and t + 4): chains of products stay in registers.
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// (Tiles that these read are written by asynchronous copies alone; volatile keeps the loads
// behind the barrier after those.)
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// x = hi + lo to 23 bits: hi rounded by integer operations (B2 H8 N32768 D64 418 us, 449 with
// conversion instructions), lo, which has at most 12 bits, cut off.  (A NaN may leave hi a number;
// lo keeps it.)
__device__ __forceinline__ void tf32_split(float x, uint32_t &hi, uint32_t &lo) {
  hi = (__float_as_uint(x) + 0x1000u) & 0xFFFFE000u;
  lo = __float_as_uint(x - __uint_as_float(hi)) & 0xFFFFE000u;
}

// The left operand of tf32 products made of a result tile, in three terms: hi + lo on both sides (the
// product of the two small parts is left out: 2^-22).  The tensor cores cut off what their
// accumulator cannot hold, so that long sums shrink: where results are fp32 (kSums), the products
// of 8 are summed from zero and added in one rounding (the gradient of the keys 1.9e-6 of its norm
// off, 0.4e-6 with it).
template <bool kSums = false>
struct LeftTf32 {
  uint32_t hi[4], lo[4];
  __device__ __forceinline__ explicit LeftTf32(const float (&c)[4]) {
    const float x[4] = {c[0], c[2], c[1], c[3]};
#pragma unroll
    for (int i = 0; i < 4; ++i) tf32_split(x[i], hi[i], lo[i]);
  }
  // The right operand's values at rows 2t and 2t + 1 of this lane's column: as they are,
  __device__ __forceinline__ void times(float (&c)[4], float b0, float b1) const {
    uint32_t h0, l0, h1, l1;
    tf32_split(b0, h0, l0);
    tf32_split(b1, h1, l1);
    times(c, make_uint4(h0, h1, l0, l1));
  }
  // or split before.
  __device__ __forceinline__ void times(float (&c)[4], const uint4 &b) const {
    if (kSums) {
      float z[4] = {};
      mma_tf32(z, lo, b.x, b.y);
      mma_tf32(z, hi, b.z, b.w);
      mma_tf32(z, hi, b.x, b.y);
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] += z[i];
      return;
    }
    mma_tf32(c, lo, b.x, b.y);
    mma_tf32(c, hi, b.z, b.w);
    mma_tf32(c, hi, b.x, b.y);
  }
};
// The left operand of bf16 products made of two result tiles, as kTerms bf16 numbers each
// (8 kTerms bits); the right operand is exact in bf16, or two bf16 numbers too.
template <int kTerms>
struct LeftBf16 {
  uint32_t part[kTerms][4];
  __device__ __forceinline__ LeftBf16() {}
  __device__ __forceinline__ LeftBf16(const float (&c)[4], const float (&d)[4]) {
    float x[8] = {c[0], c[1], c[2], c[3], d[0], d[1], d[2], d[3]};
#pragma unroll
    for (int p = 0; p < kTerms; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        part[p][i] = f2_to_bf2(x[2 * i], x[2 * i + 1]);
        const float2 f = bf2_to_f2(part[p][i]);
        x[2 * i] -= f.x, x[2 * i + 1] -= f.y;
      }
  }
  __device__ __forceinline__ void times(float (&c)[4], uint32_t b0, uint32_t b1) const {
#pragma unroll
    for (int p = kTerms - 1; p >= 0; --p) mma_bf16(c, part[p], b0, b1);
  }
  // (the product of the two small parts is left out: 2^-16)
  __device__ __forceinline__ void times(float (&c)[4], const uint4 &b) const {
    if constexpr (kTerms > 1) mma_bf16(c, part[1], b.x, b.y);
    mma_bf16(c, part[0], b.z, b.w);
    mma_bf16(c, part[0], b.x, b.y);
  }
};

// ------------------------------------------------------------- tiles
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void cp_async_or_zero(uint32_t dst, const void *src, bool valid) {
  const int n = valid ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n)
               : "memory");
}

// The sequence that the place-th blocks of a scan take: the place-th longest, so that a long one
// does not begin when the others end (lengths of at most 256 sequences; equal ones, and more
// than those, in their order).  Ends with a barrier.
__device__ __forceinline__ int longest_first(const int32_t *seq_lens, int B, int place) {
  if (!seq_lens || B > 256 || B == 1) return place;
  __shared__ int found;
  for (int i = threadIdx.x; i < B; i += blockDim.x) {
    const int mine = __ldg(seq_lens + i);
    int rank = 0;
    for (int j = 0; j < B; ++j) {
      const int o = __ldg(seq_lens + j);
      rank += o > mine || (o == mine && j < i);
    }
    if (rank == place) found = i;
  }
  __syncthreads();
  return found;
}

// Tokens of a chunk: bf16 64; fp32 32, whose tiles are twice the bytes a token.
template <typename T>
constexpr int kChunkOf = sizeof(T) == 2 ? 64 : 32;

// Elements of a padded row of kCols values: rows 4 banks (bf16: ldmatrix) or 8 (fp32: pairs of
// two) apart.
template <typename T>
constexpr int pad_row(int cols) { return cols + 8; }
// kRows tokens of kCols values into padded rows; rows from n on become zeros.  A thread keeps its
// columns and goes down the rows: a copy costs two or three instructions.
template <typename T, int kRows, int kCols, int kThreads>
__device__ __forceinline__ void load_rows(T *to, const T *from, long long stride, int n, int tid) {
  constexpr int kVec = 16 / sizeof(T), kPer = kCols / kVec, kStep = kThreads / kPer;
  constexpr int kTimes = kRows / kStep;
  static_assert(kThreads % kPer == 0 && kRows % kStep == 0, "whole rows at a time");
  const int r = tid / kPer, c = tid % kPer * kVec;
  const uint32_t dst = smem_u32(to + r * pad_row<T>(kCols) + c);
  const T *src = from + r * stride + c;
#pragma unroll
  for (int i = 0; i < kTimes; ++i) {
    const bool valid = r + i * kStep < n;
    cp_async_or_zero(dst + i * (kStep * pad_row<T>(kCols) * (int)sizeof(T)), valid ? src : from, valid);
    src += kStep * stride;
  }
}
template <int kFloats, int kThreads>
__device__ __forceinline__ void load_flat(float *to, const float *from, int tid) {
  constexpr int kTimes = (kFloats / 4 + kThreads - 1) / kThreads;
  const uint32_t dst = smem_u32(to + tid * 4);
  from += tid * 4;
#pragma unroll
  for (int i = 0; i < kTimes; ++i)
    if ((i + 1) * kThreads * 4 <= kFloats || tid * 4 + i * kThreads * 4 < kFloats)
      cp_async_16(dst + i * kThreads * 16, from + i * kThreads * 4);
}

// Right operands from a raw tile of tokens x channels, for products with the left operands
// above.  bf16: k = 16; fp32: k = 8.
// by_token: column n of the product is a token, k its channels; by_channel: the other way round.
struct PairBf16 {
  uint32_t b[2][2];  // two adjacent column tiles
};
template <int kRow>
__device__ __forceinline__ PairBf16 by_token(const __nv_bfloat16 *tile, int token0, int ch0) {
  const int l = threadIdx.x & 31;
  uint32_t r[4];
  ldmatrix4(r, smem_u32(tile + (token0 + (l & 7) + ((l >> 4) & 1) * 8) * kRow + ch0 +
                        ((l >> 3) & 1) * 8));
  return {{{r[0], r[1]}, {r[2], r[3]}}};
}
template <int kRow>
__device__ __forceinline__ PairBf16 by_channel(const __nv_bfloat16 *tile, int token0, int ch0) {
  const int l = threadIdx.x & 31;
  uint32_t r[4];
  ldmatrix4_t(r, smem_u32(tile + (token0 + (l & 7) + ((l >> 3) & 1) * 8) * kRow + ch0 +
                          ((l >> 4) & 1) * 8));
  return {{{r[0], r[1]}, {r[2], r[3]}}};
}

// ------------------------------------------------------------- what a chunk prepares
// Lower triangular C x C matrices as right operands, tile by tile on and below the diagonal, with a
// vector a lane, so that a warp's loads lie side by side.
//
// In fp32, tiles of 8 x 8 for tf32 products of three terms: the triangular inverses.  Where keys are
// alike and beta is near 2 their entries are near 2 and of either sign, and what they make of a
// chunk's misses nearly cancels: in one tf32 number (2^-11) results were off by a tenth and more, in
// two bf16 ones by up to 6e-3.  kSplit: stored as the products' two parts (B2 H8 N32768 D64 403 us,
// 418 where each warp splits them), else split where they are used, in half the bytes: with bf16 at
// D = 128 shared memory has no room for parts.
template <int C, bool kSplit>
struct Whole {
  static constexpr int kWide = 1;  // result tiles that a left operand takes
  static constexpr int kFloats = (C / 8) * (C / 8 + 1) / 2 * 32 * (kSplit ? 4 : 2);
  static __device__ __forceinline__ int at(int m, int j) {
    return (m * (m + 1) / 2 + j) * 32 + (threadIdx.x & 31);
  }
  static __device__ __forceinline__ uint4 load(const float *base, int m, int j) {
    if (kSplit) return ((const uint4 *)base)[at(m, j)];
    const float2 x = ((const float2 *)base)[at(m, j)];
    return parts(x.x, x.y);
  }
  static __device__ __forceinline__ uint4 parts(float x, float y) {
    uint4 v;  // hi, hi, lo, lo
    tf32_split(x, v.x, v.z);
    tf32_split(y, v.y, v.w);
    return v;
  }
  static __device__ __forceinline__ void store(float *base, int m, int j, float b0, float b1) {
    if (kSplit) ((uint4 *)base)[at(m, j)] = parts(b0, b1);
    else ((float2 *)base)[at(m, j)] = make_float2(b0, b1);
  }
  template <bool kSums, int kN>
  static __device__ __forceinline__ LeftTf32<kSums> left(const float (&r)[kN][4], int j) {
    return LeftTf32<kSums>(r[j]);
  }
};
// As two bf16 numbers a value, for products of 16.  Summed over columns: 8 rows m by 16 columns j;
// over rows (kRows): 16 rows m by 8 columns j.
template <int C, bool kRows>
struct Halves {
  static constexpr int kWide = 2;
  static constexpr int kFloats = (C / 16) * (C / 16 + 1) * 32 * 4;
  static __device__ __forceinline__ int at(int m, int j) {
    const int tile = kRows ? m * (m + 1) + j : (m / 2 + (m & 1)) * (m / 2 + 1) + j;
    return tile * 32 + (threadIdx.x & 31);
  }
  static __device__ __forceinline__ uint4 load(const float *base, int m, int j) {
    return ((const uint4 *)base)[at(m, j)];
  }
  // values at 2t, 2t + 1, 2t + 8 and 2t + 9 along the sum
  static __device__ __forceinline__ void store(float *base, int m, int j, const float (&x)[4]) {
    uint4 v = {f2_to_bf2(x[0], x[1]), f2_to_bf2(x[2], x[3]), 0, 0};
    const float2 a = bf2_to_f2(v.x), b = bf2_to_f2(v.y);
    v.z = f2_to_bf2(x[0] - a.x, x[1] - a.y), v.w = f2_to_bf2(x[2] - b.x, x[3] - b.y);
    ((uint4 *)base)[at(m, j)] = v;
  }
  template <bool kSums, int kN>
  static __device__ __forceinline__ LeftBf16<2> left(const float (&r)[kN][4], int j) {
    return LeftBf16<2>(r[2 * j], r[2 * j + 1]);
  }
};
// Powers of a chunk's gates.
template <int C>
struct Gates {
  // e^G_i, e^(G_C - G_i), beta_i; G_i log2 e as two floats; e^G_C as two
  static constexpr int kUp = 0, kDown = C, kBeta = 2 * C, kHi = 3 * C, kLo = 4 * C, kWhole = 5 * C;
  static constexpr int kFloats = 5 * C + 4;
};

// A chunk's record.  For the forward pass beta M, P and the powers of its gates.  For the backward
// pass (kBack) M - 1, and, for products that sum over the row index, T - 1 with T = (1 + beta X)^-1,
// and P the other way round.  The inverses in fp32; P, whose products nothing multiplies up, as two
// bf16 numbers where what it makes is bf16 (kExact: the gradient of a state, in fp32, is not:
// 1.0e-6 of its norm off, 0.3e-6 in fp32).
template <typename T, int D, bool kBack, bool kExact = false>
struct Record {
  static constexpr int C = kChunkOf<T>;
  using M = Whole<C, sizeof(T) == 4 || D < 128>;
  using P = std::conditional_t<sizeof(T) == 2 && !kExact, Halves<C, kBack>, M>;
  static constexpr int kM = 0, kGates = M::kFloats, kP = kGates + Gates<C>::kFloats;
  static constexpr int kT = kP + P::kFloats, kFloats = kT + (kBack ? M::kFloats : 0);
};

// ------------------------------------------------------------- a warp's part of a state
// A state's 16 columns as left operands, handed to another warp through shared memory: a uint4 a
// lane for each 8 (fp32) or twice for each 16 (bf16, two numbers a value) of its rows.
template <int D>
constexpr int kHandWords = D / 8;

// Products of the state's 16 columns (transposed: D / 8 tiles) with the rows of a tile of keys.
// kHand: leaves the left operands in `hand`.
template <int kTerms, int D, int C, bool kHand>
__device__ __forceinline__ void key_products(const float (&S)[D / 8][4], const __nv_bfloat16 *ks,
                                             float (&kv)[C / 8][4], uint4 *hand) {
  constexpr int kRow = pad_row<__nv_bfloat16>(D);
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 0; d < D / 16; ++d) {
    const LeftBf16<kTerms> a(S[2 * d], S[2 * d + 1]);
    if (kHand) {
#pragma unroll
      for (int p = 0; p < 2; ++p)
        hand[(2 * d + p) * 32 + lane] = make_uint4(a.part[p][0], a.part[p][1], a.part[p][2], a.part[p][3]);
    }
#pragma unroll
    for (int n = 0; n < C / 16; ++n) {
      const PairBf16 k = by_token<kRow>(ks, 16 * n, 16 * d);
      a.times(kv[2 * n], k.b[0][0], k.b[0][1]);
      a.times(kv[2 * n + 1], k.b[1][0], k.b[1][1]);
    }
  }
}
template <int kTerms, int D, int C, bool kHand>
__device__ __forceinline__ void key_products(const float (&S)[D / 8][4], const float *ks,
                                             float (&kv)[C / 8][4], uint4 *hand) {
  constexpr int kRow = pad_row<float>(D);
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int d = 0; d < D / 8; ++d) {
    const LeftTf32<true> a(S[d]);
    if (kHand) ((float4 *)hand)[d * 32 + lane] = make_float4(S[d][0], S[d][1], S[d][2], S[d][3]);
#pragma unroll
    for (int n = 0; n < C / 8; ++n) {
      const float2 k = *(const float2 *)(ks + (8 * n + g) * kRow + 8 * d + 2 * t);
      a.times(kv[n], k.x, k.y);
    }
  }
}
// The same with a state handed over, in 16 bits where results are bf16.
template <int D, int C>
__device__ __forceinline__ void query_products(const uint4 *hand, const __nv_bfloat16 *qs,
                                               float (&qv)[C / 8][4]) {
  constexpr int kRow = pad_row<__nv_bfloat16>(D);
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 0; d < D / 16; ++d) {
    const uint4 x = hand[2 * d * 32 + lane], y = hand[(2 * d + 1) * 32 + lane];
    const uint32_t hi[4] = {x.x, x.y, x.z, x.w}, lo[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int n = 0; n < C / 16; ++n) {
      const PairBf16 q = by_token<kRow>(qs, 16 * n, 16 * d);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mma_bf16(qv[2 * n + i], lo, q.b[i][0], q.b[i][1]);
        mma_bf16(qv[2 * n + i], hi, q.b[i][0], q.b[i][1]);
      }
    }
  }
}
template <int D, int C>
__device__ __forceinline__ void query_products(const uint4 *hand, const float *qs,
                                               float (&qv)[C / 8][4]) {
  constexpr int kRow = pad_row<float>(D);
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int d = 0; d < D / 8; ++d) {
    const float4 s = ((const float4 *)hand)[d * 32 + lane];
    const float c[4] = {s.x, s.y, s.z, s.w};
    const LeftTf32<true> a(c);
#pragma unroll
    for (int n = 0; n < C / 8; ++n) {
      const float2 q = *(const float2 *)(qs + (8 * n + g) * kRow + 8 * d + 2 * t);
      a.times(qv[n], q.x, q.y);
    }
  }
}
// The warp's columns e0 .. e0 + 15 of a D x D matrix in global memory (NULL: zeros).
template <int D>
__device__ __forceinline__ void load_state(float (&S)[D / 8][4], const float *from, int e0) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
  for (int d = 0; d < D / 8; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      S[d][i] = from ? from[(8 * d + 2 * t + (i & 1)) * D + e0 + g + (i >> 1) * 8] : 0.f;
}
template <int D>
__device__ __forceinline__ void store_state(float *to, const float (&S)[D / 8][4], int e0) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
  for (int d = 0; d < D / 8; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      to[(8 * d + 2 * t + (i & 1)) * D + e0 + g + (i >> 1) * 8] = S[d][i];
}
// The same between the launches of the backward pass, as the warps hold it: a float4 a lane for
// each 8 of a matrix's rows (kTiles; or of a chunk's tokens), one 16 columns after the other.
template <int kTiles>
__device__ __forceinline__ void store_packed(float *to, const float (&x)[kTiles][4], int e0) {
  float4 *at = (float4 *)to + e0 / 16 * kTiles * 32 + (threadIdx.x & 31);
#pragma unroll
  for (int i = 0; i < kTiles; ++i) at[i * 32] = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
}
// S = (hi + lo) S + w^T k over the chunk's tokens.  The chunk's own sum starts from zero and is
// added in one rounding: the tensor cores cut off what their accumulator cannot hold, which
// over the chunks of a long sequence would shrink the state.
template <int kTerms, int D, int C>
__device__ __forceinline__ void state_update(float (&S)[D / 8][4], float hi, float lo,
                                             const float (&w)[C / 8][4], const __nv_bfloat16 *ks) {
  constexpr int kRow = pad_row<__nv_bfloat16>(D);
  static_assert(C == 64, "four left operands");
  const LeftBf16<kTerms> a[4] = {{w[0], w[1]}, {w[2], w[3]}, {w[4], w[5]}, {w[6], w[7]}};
#pragma unroll
  for (int d = 0; d < D / 16; d += 2) {  // four sums at a time
    float x[4][4] = {};
#pragma unroll
    for (int j = 0; j < C / 16; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const PairBf16 k = by_channel<kRow>(ks, 16 * j, 16 * (d + e));
        a[j].times(x[2 * e], k.b[0][0], k.b[0][1]);
        a[j].times(x[2 * e + 1], k.b[1][0], k.b[1][1]);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float &s = S[2 * d + i][e];
        s = fmaf(hi, s, fmaf(lo, s, x[i][e]));
      }
  }
}
template <int kTerms, int D, int C>
__device__ __forceinline__ void state_update(float (&S)[D / 8][4], float hi, float lo,
                                             const float (&w)[C / 8][4], const float *ks) {
  constexpr int kRow = pad_row<float>(D);
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
  for (int d = 0; d < D / 8; ++d) {
    float x[4] = {};
#pragma unroll
    for (int j = 0; j < C / 8; ++j) {
      const LeftTf32<true> a(w[j]);
      a.times(x, ks[(8 * j + 2 * t) * kRow + 8 * d + g], ks[(8 * j + 2 * t + 1) * kRow + 8 * d + g]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) S[d][e] = fmaf(hi, S[d][e], fmaf(lo, S[d][e], x[e]));
  }
}
// The values of the warp's columns e0 .. e0 + 15 at the tokens of tiles 2n and 2n + 1, as
// product tiles hold them.
template <int kRow>
__device__ __forceinline__ void values_of(float (&a)[4], float (&b)[4], const __nv_bfloat16 *vs,
                                          int n, int e0) {
  const int l = threadIdx.x & 31;
  uint32_t r[4];
  ldmatrix4_t(r, smem_u32(vs + (16 * n + (l >> 4) * 8 + (l & 7)) * kRow + e0 + ((l >> 3) & 1) * 8));
  const float2 f[4] = {bf2_to_f2(r[0]), bf2_to_f2(r[1]), bf2_to_f2(r[2]), bf2_to_f2(r[3])};
  a[0] = f[0].x, a[1] = f[0].y, a[2] = f[1].x, a[3] = f[1].y;
  b[0] = f[2].x, b[1] = f[2].y, b[2] = f[3].x, b[3] = f[3].y;
}
template <int kRow>
__device__ __forceinline__ void values_of(float (&a)[4], float (&b)[4], const float *vs, int n,
                                          int e0) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const float *v = vs + (16 * n + 2 * t) * kRow + e0 + g;
  a[0] = v[0], a[1] = v[kRow], a[2] = v[8], a[3] = v[kRow + 8];
  v += 8 * kRow;
  b[0] = v[0], b[1] = v[kRow], b[2] = v[8], b[3] = v[kRow + 8];
}
// A result tile (16 columns of the values, 8 tokens from `token` on) to global memory.
__device__ __forceinline__ void store_tile(__nv_bfloat16 *o, size_t stride, const float (&c)[4],
                                           int token, int n) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const uint32_t lo = transpose8(f2_to_bf2(c[0], c[1])), hi = transpose8(f2_to_bf2(c[2], c[3]));
  if (token + g < n) {
    uint32_t *at = (uint32_t *)(o + (size_t)(token + g) * stride + 2 * t);
    at[0] = lo, at[4] = hi;
  }
}
__device__ __forceinline__ void store_tile(float *o, size_t stride, const float (&c)[4], int token,
                                           int n) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (token + 2 * t + e < n) {
      float *at = o + (size_t)(token + 2 * t + e) * stride + g;
      at[0] = c[e], at[8] = c[2 + e];
    }
}

// ------------------------------------------------------------- between the files
template <typename T>
int chunks_of(const DeltaArgs &a) { return (a.N + kChunkOf<T> - 1) / kChunkOf<T>; }
// A sequence is cut into `count` segments of `chunks` chunks (the last one shorter).  Scratch: a
// state and a matrix for each, [B H][count][D][D].
struct Segments {
  int count, chunks;
  size_t floats(const DeltaArgs &a) const {
    return count > 1 ? (size_t)a.B * a.H * count * a.D * a.D : 0;
  }
};
Segments segments_of(const DeltaArgs &a, bool back);
// First part of the backward pass: records (of the backward's form), the states before all
// chunks and the misses, packed; `moves`: the matrices that segments move a state by.  exact:
// states meet keys and writes in three terms.
cudaError_t save_forward(const DeltaArgs &a, const Segments &g, bool exact, float *records,
                         float *states, float *misses, float *before, float *moves,
                         cudaStream_t st);
// Turns what each segment adds to the gradient of the state into that before it, in place:
// A' = move^T A + own, from the last segment on.
cudaError_t join_back(const DeltaArgs &a, const Segments &g, const float *init, float *own,
                      const float *moves, cudaStream_t st);

}  // namespace delta
}  // namespace gbla
