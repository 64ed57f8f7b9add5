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
// fp32 rounded to the 11 significant bits that tf32 products read.
__device__ __forceinline__ uint32_t tf32_of(float x) {
  uint32_t r;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
  return r;
}
// x = hi + lo to 22 bits.
__device__ __forceinline__ void tf32_split(float x, uint32_t &hi, uint32_t &lo) {
  hi = tf32_of(x);
  lo = tf32_of(x - __uint_as_float(hi));
}

// The left operand of tf32 products made of a result tile; kTerms 1: rounded to 11 bits,
// 3: hi + lo (the product of the two small parts is left out: 2^-22).
template <int kTerms>
struct LeftTf32 {
  uint32_t hi[4], lo[4];
  __device__ __forceinline__ explicit LeftTf32(const float (&c)[4]) {
    const float x[4] = {c[0], c[2], c[1], c[3]};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (kTerms == 1) hi[i] = tf32_of(x[i]);
      else tf32_split(x[i], hi[i], lo[i]);
    }
  }
  // The right operand's values at rows 2t and 2t + 1 of this lane's column: as they are,
  __device__ __forceinline__ void times(float (&c)[4], float b0, float b1) const {
    if (kTerms == 1) {
      mma_tf32(c, hi, tf32_of(b0), tf32_of(b1));
      return;
    }
    uint32_t h0, l0, h1, l1;
    tf32_split(b0, h0, l0);
    tf32_split(b1, h1, l1);
    times(c, make_uint4(h0, h1, l0, l1));
  }
  // or rounded or split before.
  __device__ __forceinline__ void times(float (&c)[4], const uint2 &b) const {
    mma_tf32(c, hi, b.x, b.y);
  }
  __device__ __forceinline__ void times(float (&c)[4], const uint4 &b) const {
    mma_tf32(c, lo, b.x, b.y);
    mma_tf32(c, hi, b.z, b.w);
    mma_tf32(c, hi, b.x, b.y);
  }
};
// The left operand of bf16 products made of two result tiles, as kTerms bf16 numbers each
// (8 kTerms bits); the right operand is exact in bf16.
template <int kTerms>
struct LeftBf16 {
  uint32_t part[kTerms][4];
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
};

// ------------------------------------------------------------- tiles
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void cp_async_or_zero(uint32_t dst, const void *src, bool valid) {
  const int n = valid ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n)
               : "memory");
}

// Tokens of a chunk: bf16 64; fp32 32, whose tiles are twice the bytes a token.
template <typename T>
constexpr int kChunkOf = sizeof(T) == 2 ? 64 : 32;

// Elements of a padded row of kCols values: rows 4 banks (bf16: ldmatrix) or 8 (fp32: pairs of
// two) apart.
template <typename T>
constexpr int pad_row(int cols) { return cols + 8; }
// kRows tokens of kCols values into padded rows; rows from n on become zeros.
template <typename T, int kRows, int kCols, int kThreads>
__device__ __forceinline__ void load_rows(T *to, const T *from, long long stride, int n) {
  constexpr int kVec = 16 / sizeof(T), kPer = kCols / kVec;
  for (int i = threadIdx.x; i < kRows * kPer; i += kThreads) {
    const int r = i / kPer, c = i % kPer * kVec;
    cp_async_or_zero(smem_u32(to + r * pad_row<T>(kCols) + c), from + (r < n ? r * stride + c : 0),
                     r < n);
  }
}
template <int kFloats, int kThreads>
__device__ __forceinline__ void load_flat(float *to, const float *from) {
  for (int i = threadIdx.x * 4; i < kFloats; i += kThreads * 4)
    cp_async_16(smem_u32(to + i), from + i);
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
// Lower triangular C x C matrices, as the right operands of tf32 products: tiles of 8 x 8 on
// and below the diagonal, row by row of tiles, each with a uint2 (one term: rounded) or uint4
// (three: two hi, two lo) a lane, so that a warp's loads lie side by side.
template <int C, int kTerms>
struct Tiles {
  static constexpr int kLane = kTerms == 1 ? 2 : 4;  // floats
  static constexpr int kTiles = (C / 8) * (C / 8 + 1) / 2, kFloats = kTiles * 32 * kLane;
  using Word = std::conditional_t<kTerms == 1, uint2, uint4>;
  static __device__ __forceinline__ int at(int m, int j) {
    return (m * (m + 1) / 2 + j) * 32 + (threadIdx.x & 31);
  }
  static __device__ __forceinline__ Word load(const float *base, int m, int j) {
    return ((const Word *)base)[at(m, j)];
  }
  static __device__ __forceinline__ void store(float *base, int m, int j, float b0, float b1) {
    if constexpr (kTerms == 1) {
      ((uint2 *)base)[at(m, j)] = make_uint2(tf32_of(b0), tf32_of(b1));
    } else {
      uint4 v;
      tf32_split(b0, v.x, v.z);
      tf32_split(b1, v.y, v.w);
      ((uint4 *)base)[at(m, j)] = v;
    }
  }
};
// Powers of a chunk's gates.
template <int C>
struct Gates {
  static constexpr int kUp = 0, kDown = C, kBeta = 2 * C, kWhole = 3 * C, kFloats = 4 * C;
};

}  // namespace delta
}  // namespace gbla
