// Attention by the gated delta rule in chunks of C tokens.
//
// With G_i the sum of the log decays of a chunk's tokens up to i, S the state before it and
//   X_ij = (k_i . k_j) e^(G_i - G_j)  (j < i),   P_ij = scale (q_i . k_j) e^(G_i - G_j)  (j <= i),
// the misses of the chunk's tokens solve a triangular system,
//   miss_i + sum_j X_ij beta_j miss_j = v_i - e^(G_i) S^T k_i = r_i,
// so miss = M r with M = (1 + X beta)^-1, u = beta miss, and
//   o_i = scale e^(G_i) S^T q_i + sum_j P_ij u_j,
//   S'  = e^(G_C) S + sum_j e^(G_C - G_j) k_j u_j^T.
// M and P need no state: a first launch forms them for all chunks at once.  A second one
// goes through the chunks, and in it the columns of S are independent of one another: each
// warp carries 16 of them, transposed, through the whole sequence, in registers.
#include <math.h>

#include "gbla_delta_mma.cuh"

namespace gbla {
namespace delta {
namespace {

// A chunk's record: M, P and the powers of its gates.  M in kSolve terms; P in one where results
// are bf16.
template <typename T, int kSolve>
struct Record {
  static constexpr int C = kChunkOf<T>;
  using M = Tiles<C, kSolve>;
  using P = Tiles<C, sizeof(T) == 2 ? 1 : 3>;
  static constexpr int kM = 0, kP = M::kFloats, kGates = kP + P::kFloats;
  static constexpr int kFloats = kGates + Gates<C>::kFloats;
};

// --------------------------------------------------------------- first launch
// One block a (chunk, head, batch), a warp for each 16 of its tokens.
template <typename T, int D>
struct PrepShape {
  static constexpr int C = kChunkOf<T>, kWarps = C / 16, kThreads = kWarps * 32;
  static constexpr int kRow = pad_row<T>(D), kMat = C + 4;
  static constexpr int kBytes = 2 * C * kRow * (int)sizeof(T) + 2 * C * kMat * 4 + 4 * C * 4 + 16;
};

// Products of 16 rows of `left` with every row of `right` up to the block's last row, fp32 tiles
// of 16 x 8 in acc.
template <int D, int C>
__device__ __forceinline__ void rows_times_rows(float (&acc)[C / 8][4], const __nv_bfloat16 *left,
                                                const __nv_bfloat16 *right, int w) {
  constexpr int kRow = pad_row<__nv_bfloat16>(D);
  const int l = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    uint32_t a[4];
    ldmatrix4(a, smem_u32(left + (16 * w + (l & 15)) * kRow + 16 * k + (l >> 4) * 8));
#pragma unroll
    for (int n = 0; n < C / 16; ++n)
      if (n <= w) {
        const PairBf16 p = by_token<kRow>(right, 16 * n, 16 * k);
        mma_bf16(acc[2 * n], a, p.b[0][0], p.b[0][1]);
        mma_bf16(acc[2 * n + 1], a, p.b[1][0], p.b[1][1]);
      }
  }
}
template <int D, int C>
__device__ __forceinline__ void rows_times_rows(float (&acc)[C / 8][4], const float *left,
                                                const float *right, int w) {
  constexpr int kRow = pad_row<float>(D);
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll 2
  for (int k = 0; k < D / 8; ++k) {
    const float2 x = *(const float2 *)(left + (16 * w + g) * kRow + 8 * k + 2 * t);
    const float2 y = *(const float2 *)(left + (16 * w + g + 8) * kRow + 8 * k + 2 * t);
    const float c[4] = {x.x, x.y, y.x, y.y};
    const LeftTf32<3> a(c);
#pragma unroll
    for (int n = 0; n < C / 8; ++n)
      if (n <= 2 * w + 1) {
        const float2 b = *(const float2 *)(right + (8 * n + g) * kRow + 8 * k + 2 * t);
        a.times(acc[n], b.x, b.y);
      }
  }
}

// Parts of C x C matrices in shared memory (rows of C + 4 floats) as operands: 16 rows from i on
// at columns j .. j + 7 on the left, columns j .. j + 7 of rows i .. i + 7 on the right.
template <int C>
__device__ __forceinline__ LeftTf32<3> left_of(const float *m, int i, int j) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const float2 x = *(const float2 *)(m + (i + g) * (C + 4) + j + 2 * t);
  const float2 y = *(const float2 *)(m + (i + g + 8) * (C + 4) + j + 2 * t);
  const float c[4] = {x.x, x.y, y.x, y.y};
  return LeftTf32<3>(c);
}
template <int C>
__device__ __forceinline__ void times_right(float (&c)[4], const LeftTf32<3> &a, const float *m,
                                            int i, int j) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const float *at = m + (i + 2 * t) * (C + 4) + j + g;
  a.times(c, at[0], at[C + 4]);
}

// to = (1 + A)^-1 for strictly lower triangular A, on and below its diagonal blocks of 16.
// Those by forward substitution, the rest from
//   (1 + A)^-1 = [ M0 0; -M1 A10 M0 M1 ]
// for pairs of blocks of 16 and then of 32, in products of three tf32 terms.  (No powers of A,
// which grow where the inverse does not: keys that repeat.)  Begins and ends with all of A, and
// of `to`, visible to the block.
template <int C>
__device__ __forceinline__ void invert(float *to, const float *A, int w) {
  constexpr int kMat = C + 4;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  auto put = [&](const float (&c)[4], int i, int j) {  // minus the product
    *(float2 *)(to + (i + g) * kMat + j + 2 * t) = make_float2(-c[0], -c[1]);
    *(float2 *)(to + (i + g + 8) * kMat + j + 2 * t) = make_float2(-c[2], -c[3]);
  };
  {
    const float *a = A + 16 * w * kMat + 16 * w;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = i == (lane & 15) ? 1.f : 0.f, s1 = 0.f;
#pragma unroll
      for (int m = 0; m < i; m += 4) {
        const float4 v = *(const float4 *)(a + i * kMat + m);
        s = fmaf(-v.x, x[m], s);
        if (m + 1 < i) s1 = fmaf(-v.y, x[m + 1], s1);
        if (m + 2 < i) s = fmaf(-v.z, x[m + 2], s);
        if (m + 3 < i) s1 = fmaf(-v.w, x[m + 3], s1);
      }
      x[i] = s + s1;
      if (lane < 16) to[(16 * w + i) * kMat + 16 * w + lane] = x[i];
    }
  }
  __syncthreads();
  if (w & 1) {
    const int i = 16 * w, j = i - 16;
    float z[2][4] = {}, y[2][4] = {};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const LeftTf32<3> a = left_of<C>(to, i, i + 8 * k);
#pragma unroll
      for (int n = 0; n < 2; ++n) times_right<C>(z[n], a, A, i + 8 * k, j + 8 * n);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const LeftTf32<3> a(z[k]);
#pragma unroll
      for (int n = 0; n < 2; ++n) times_right<C>(y[n], a, to, j + 8 * k, j + 8 * n);
    }
    put(y[0], i, j), put(y[1], i, j + 8);
  }
  __syncthreads();
  if (C == 64) {
    // rows 32 .. 63, columns 0 .. 31: a warp takes 16 of each
    const int i = 32 + 16 * (w & 1), j = 16 * (w >> 1);
    float z[4][4] = {}, y[2][4] = {};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < 2 || (w & 1)) {
        const LeftTf32<3> a = left_of<C>(to, i, 32 + 8 * k);
#pragma unroll
        for (int n = 0; n < 4; ++n) times_right<C>(z[n], a, A, 32 + 8 * k, 8 * n);
      }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k >= 2 || j == 0) {
        const LeftTf32<3> a(z[k]);
#pragma unroll
        for (int n = 0; n < 2; ++n) times_right<C>(y[n], a, to, 8 * k, j + 8 * n);
      }
    put(y[0], i, j), put(y[1], i, j + 8);
    __syncthreads();
  }
}

template <typename T, int D, int kSolve>
__global__ void __launch_bounds__(PrepShape<T, D>::kThreads)
    prepare_kernel(const DeltaArgs p, float *records, int nc) {
  using Sh = PrepShape<T, D>;
  using Rec = Record<T, kSolve>;
  constexpr int C = Sh::C, kThreads = Sh::kThreads, kRow = Sh::kRow, kMat = Sh::kMat;
  extern __shared__ __align__(16) char raw[];
  T *ks = (T *)raw, *qs = ks + C * kRow;
  float *A = (float *)(qs + C * kRow), *inv = A + C * kMat;
  float *hi = inv + C * kMat, *lo = hi + C, *beta = lo + C;
  double *first = (double *)(beta + 2 * C);
  grid_dep_wait();
  const int h = blockIdx.y, b = blockIdx.z, hk = h / (p.H / p.Hk), tid = threadIdx.x;
  const int L = p.seq_lens ? min(max(__ldg(p.seq_lens + b), 0), p.N) : p.N;
  const int t0 = blockIdx.x * C, n = min(C, L - t0);
  if (n <= 0) return;
  load_rows<T, C, D, kThreads>(ks, (const T *)p.k + b * p.sk[0] + t0 * p.sk[1] + (long long)hk * D,
                               p.sk[1], n);
  load_rows<T, C, D, kThreads>(qs, (const T *)p.q + b * p.sq[0] + t0 * p.sq[1] + (long long)hk * D,
                               p.sq[1], n);
  cp_async_commit();
  // Sums of the log decays in 64 bits: differences of two of them are what counts, also
  // behind a token that ends the memory (-inf: a number whose power is 0 next to any other).
  double G = 0.;
  if (tid < C) {
    float lg = 0.f, be = 0.f;
    if (tid < n) {
      lg = to_f(((const T *)p.log_decay)[b * p.sg[0] + (t0 + tid) * p.sg[1] + h]);
      be = to_f(((const T *)p.beta)[b * p.sb[0] + (t0 + tid) * p.sb[1] + h]);
    }
    beta[tid] = be;
    G = fmax((double)lg, -1e3);
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const double o = __shfl_up_sync(0xFFFFFFFFu, G, m);
      if ((tid & 31) >= m) G += o;
    }
    if (tid == 31) *first = G;
  }
  cp_async_wait_all();
  __syncthreads();
  float *rec = records + (((size_t)b * p.H + h) * nc + blockIdx.x) * Rec::kFloats;
  float *gt = rec + Rec::kGates;
  if (tid < C) {
    if (tid >= 32) G += *first;
    const double G2 = G * 1.4426950408889634;  // powers of two from here on
    hi[tid] = (float)G2, lo[tid] = (float)(G2 - (double)hi[tid]);
    gt[Gates<C>::kUp + tid] = expf((float)G);
    gt[Gates<C>::kBeta + tid] = beta[tid];
    if (tid == C - 1) {
      const DecayFactor f = G < -300. ? DecayFactor{0.f, 0.f} : decay_factor((float)G);
      gt[Gates<C>::kWhole] = f.hi, gt[Gates<C>::kWhole + 1] = f.lo;
    }
  }
  __syncthreads();
  if (tid < C)
    gt[Gates<C>::kDown + tid] = exp2f((hi[C - 1] - hi[tid]) + (lo[C - 1] - lo[tid]));
  // the warp's 16 rows of both products, weighted
  const int w = tid / 32, g = (tid & 31) >> 2, t = tid & 3;
  float kk[C / 8][4] = {}, qk[C / 8][4] = {};
  rows_times_rows<D, C>(kk, ks, ks, w);
  rows_times_rows<D, C>(qk, qs, ks, w);
#pragma unroll
  for (int m = 0; m < C / 8; ++m) {
    if (m > 2 * w + 1) continue;
    const int j = 8 * m + 2 * t;
    const float2 hj = *(const float2 *)(hi + j), lj = *(const float2 *)(lo + j);
    const float2 bj = *(const float2 *)(beta + j);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int i = 16 * w + g + 8 * half;
      const float f0 = i >= j ? ex2_approx((hi[i] - hj.x) + (lo[i] - lj.x)) : 0.f;
      const float f1 = i >= j + 1 ? ex2_approx((hi[i] - hj.y) + (lo[i] - lj.y)) : 0.f;
      *(float2 *)(A + i * kMat + j) =
          make_float2(i > j ? kk[m][2 * half] * f0 * bj.x : 0.f,
                      i > j + 1 ? kk[m][2 * half + 1] * f1 * bj.y : 0.f);
      if (2 * w + half >= m)
        Rec::P::store(rec + Rec::kP, 2 * w + half, m, p.scale * qk[m][2 * half] * f0,
                      p.scale * qk[m][2 * half + 1] * f1);
    }
  }
  __syncthreads();
  invert<C>(inv, A, w);
  // M - 1, whose diagonal is 0: the identity's part of a product needs no rounding
  for (int m = w; m < C / 8; m += Sh::kWarps)
    for (int j = 0; j <= m; ++j) {
      const float2 v = *(const float2 *)(inv + (8 * m + g) * kMat + 8 * j + 2 * t);
      Rec::M::store(rec + Rec::kM, m, j, j == m && g == 2 * t ? 0.f : v.x,
                    j == m && g == 2 * t + 1 ? 0.f : v.y);
    }
}

// --------------------------------------------------------------- second launch
template <typename T, int D, int kSolve>
struct ScanShape {
  static constexpr int C = kChunkOf<T>, kWarps = D / 16, kThreads = kWarps * 32;
  static constexpr int kRow = pad_row<T>(D);
  static constexpr int kTile = C * kRow * (int)sizeof(T);        // bytes of k, q or v
  static constexpr int kStage = 3 * kTile + Record<T, kSolve>::kFloats * 4;
  static constexpr int kBytes = 2 * kStage;
};

// Products of the state's 16 columns (transposed: D / 8 tiles) with keys and queries.
template <int kTerms, int D, int C>
__device__ __forceinline__ void state_products(const float (&S)[D / 8][4], const __nv_bfloat16 *ks,
                                               const __nv_bfloat16 *qs, float (&kv)[C / 8][4],
                                               float (&qv)[C / 8][4]) {
  constexpr int kRow = pad_row<__nv_bfloat16>(D);
#pragma unroll
  for (int d = 0; d < D / 16; ++d) {
    const LeftBf16<kTerms> a(S[2 * d], S[2 * d + 1]);
#pragma unroll
    for (int n = 0; n < C / 16; ++n) {
      const PairBf16 k = by_token<kRow>(ks, 16 * n, 16 * d), q = by_token<kRow>(qs, 16 * n, 16 * d);
      a.times(kv[2 * n], k.b[0][0], k.b[0][1]);
      a.times(kv[2 * n + 1], k.b[1][0], k.b[1][1]);
#pragma unroll
      for (int i = 0; i < 2; ++i)  // results are bf16: 16 bits of the state do
#pragma unroll
        for (int p = 1; p >= 0; --p) mma_bf16(qv[2 * n + i], a.part[p], q.b[i][0], q.b[i][1]);
    }
  }
}
template <int kTerms, int D, int C>
__device__ __forceinline__ void state_products(const float (&S)[D / 8][4], const float *ks,
                                               const float *qs, float (&kv)[C / 8][4],
                                               float (&qv)[C / 8][4]) {
  constexpr int kRow = pad_row<float>(D);
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
  for (int d = 0; d < D / 8; ++d) {
    const LeftTf32<3> a(S[d]);
#pragma unroll
    for (int n = 0; n < C / 8; ++n) {
      const float2 k = *(const float2 *)(ks + (8 * n + g) * kRow + 8 * d + 2 * t);
      const float2 q = *(const float2 *)(qs + (8 * n + g) * kRow + 8 * d + 2 * t);
      a.times(kv[n], k.x, k.y);
      a.times(qv[n], q.x, q.y);
    }
  }
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
  for (int d = 0; d < D / 16; ++d) {
    float x[2][4] = {};
#pragma unroll
    for (int j = 0; j < C / 16; ++j) {
      const PairBf16 k = by_channel<kRow>(ks, 16 * j, 16 * d);
      a[j].times(x[0], k.b[0][0], k.b[0][1]);
      a[j].times(x[1], k.b[1][0], k.b[1][1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
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
      const LeftTf32<3> a(w[j]);
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

// kTerms: bf16 numbers that stand for a value of the state where it meets a key or takes a
// write (fp32: 3 tf32 products); kSolve: terms of the product with M.
template <typename T, int D, int kTerms, int kSolve>
__global__ void __launch_bounds__(ScanShape<T, D, kSolve>::kThreads)
    scan_kernel(const DeltaArgs p, const float *records, int nc) {
  using Sh = ScanShape<T, D, kSolve>;
  using Rec = Record<T, kSolve>;
  constexpr int C = Sh::C, kThreads = Sh::kThreads, kRow = Sh::kRow;
  constexpr int kOut = sizeof(T) == 2 ? 1 : 3;  // terms of the product with P
  extern __shared__ __align__(16) char raw[];
  grid_dep_wait();
  const int h = blockIdx.x, b = blockIdx.y, hk = h / (p.H / p.Hk), tid = threadIdx.x;
  const int w = tid / 32, g = (tid & 31) >> 2, t = tid & 3, e0 = 16 * w;
  const int L = p.seq_lens ? min(max(__ldg(p.seq_lens + b), 0), p.N) : p.N;
  const size_t bh = (size_t)b * p.H + h;
  const T *kg = (const T *)p.k + b * p.sk[0] + (long long)hk * D;
  const T *qg = (const T *)p.q + b * p.sq[0] + (long long)hk * D;
  const T *vg = (const T *)p.v + b * p.sv[0] + (long long)h * D;
  T *og = (T *)p.o + ((size_t)b * p.N * p.H + h) * D + e0;
  const size_t orow = (size_t)p.H * D;
  const int chunks = (L + C - 1) / C;
  auto load = [&](int c) {
    char *s = raw + (c & 1) * Sh::kStage;
    const long long t0 = (long long)c * C;
    const int n = min(C, L - c * C);
    load_rows<T, C, D, kThreads>((T *)s, kg + t0 * p.sk[1], p.sk[1], n);
    load_rows<T, C, D, kThreads>((T *)(s + Sh::kTile), qg + t0 * p.sq[1], p.sq[1], n);
    load_rows<T, C, D, kThreads>((T *)(s + 2 * Sh::kTile), vg + t0 * p.sv[1], p.sv[1], n);
    load_flat<Rec::kFloats, kThreads>((float *)(s + 3 * Sh::kTile),
                                      records + (bh * nc + c) * Rec::kFloats);
  };
  float S[D / 8][4];  // rows: columns e0 + g, + 8 of the state; columns: its rows
#pragma unroll
  for (int d = 0; d < D / 8; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      S[d][i] = p.init ? p.init[bh * D * D + (size_t)(8 * d + 2 * t + (i & 1)) * D + e0 + g + (i >> 1) * 8]
                       : 0.f;
  if (chunks > 0) load(0);
  cp_async_commit();
  for (int c = 0; c < chunks; ++c) {
    cp_async_wait_all();
    __syncthreads();  // this chunk's tiles are in, the other buffer is read
    if (c + 1 < chunks) load(c + 1);
    cp_async_commit();
    const char *s = raw + (c & 1) * Sh::kStage;
    const T *ks = (const T *)s, *qs = (const T *)(s + Sh::kTile), *vs = (const T *)(s + 2 * Sh::kTile);
    const float *rec = (const float *)(s + 3 * Sh::kTile), *gt = rec + Rec::kGates;
    const int n = min(C, L - c * C);
    float r[C / 8][4] = {}, o[C / 8][4] = {};
    state_products<kTerms, D, C>(S, ks, qs, r, o);
#pragma unroll
    for (int m = 0; m < C / 16; ++m) {
      float v[2][4];
      values_of<kRow>(v[0], v[1], vs, m, e0);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 up = *(const float2 *)(gt + Gates<C>::kUp + 16 * m + 8 * i + 2 * t);
        float(&x)[4] = r[2 * m + i], (&y)[4] = o[2 * m + i];
        x[0] = fmaf(-up.x, x[0], v[i][0]), x[1] = fmaf(-up.y, x[1], v[i][1]);
        x[2] = fmaf(-up.x, x[2], v[i][2]), x[3] = fmaf(-up.y, x[3], v[i][3]);
        const float ux = up.x * p.scale, uy = up.y * p.scale;
        y[0] *= ux, y[1] *= uy, y[2] *= ux, y[3] *= uy;
      }
    }
    // r += (M - 1) r: the later half of the tokens first, which needs the earlier ones as
    // they are; then those
#pragma unroll
    for (int half = 1; half >= 0; --half) {
      constexpr int kHalf = C / 16;
      float x[kHalf][4] = {};
#pragma unroll
      for (int j = 0; j < (half + 1) * kHalf; ++j) {
        const LeftTf32<kSolve> a(r[j]);
#pragma unroll
        for (int m = 0; m < kHalf; ++m)
          if (half * kHalf + m >= j) a.times(x[m], Rec::M::load(rec + Rec::kM, half * kHalf + m, j));
      }
#pragma unroll
      for (int m = 0; m < kHalf; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) r[half * kHalf + m][i] += x[m][i];
    }
    // u, and the results
#pragma unroll
    for (int j = 0; j < C / 8; ++j) {
      const float2 be = *(const float2 *)(gt + Gates<C>::kBeta + 8 * j + 2 * t);
      r[j][0] *= be.x, r[j][1] *= be.y, r[j][2] *= be.x, r[j][3] *= be.y;
      const LeftTf32<kOut> a(r[j]);
#pragma unroll
      for (int m = j; m < C / 8; ++m) a.times(o[m], Rec::P::load(rec + Rec::kP, m, j));
      store_tile(og + (size_t)c * C * orow, orow, o[j], 8 * j, n);  // no later u meets it
      const float2 dn = *(const float2 *)(gt + Gates<C>::kDown + 8 * j + 2 * t);
      r[j][0] *= dn.x, r[j][1] *= dn.y, r[j][2] *= dn.x, r[j][3] *= dn.y;
    }
    state_update<kTerms, D, C>(S, gt[Gates<C>::kWhole], gt[Gates<C>::kWhole + 1], r, ks);
  }
  if (p.fin) {
#pragma unroll
    for (int d = 0; d < D / 8; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        p.fin[bh * D * D + (size_t)(8 * d + 2 * t + (i & 1)) * D + e0 + g + (i >> 1) * 8] = S[d][i];
  }
}

template <typename T>
int chunks_of(const DeltaArgs &a) { return (a.N + kChunkOf<T> - 1) / kChunkOf<T>; }

// Terms of the product with M: bf16 results alone need one (2^-11 of what M adds to a miss).
bool exact_state(const DeltaArgs &a) { return a.dtype == GBLA_FP32 || a.fin; }

template <typename T, int D, int kTerms, int kSolve>
cudaError_t launch(const DeltaArgs &a, float *scratch, cudaStream_t st) {
  using Pr = PrepShape<T, D>;
  using Sc = ScanShape<T, D, kSolve>;
  const int nc = chunks_of<T>(a);
  const auto prep = prepare_kernel<T, D, kSolve>;
  const auto scan = scan_kernel<T, D, kTerms, kSolve>;
  cudaError_t e;
  if ((e = cudaFuncSetAttribute(prep, cudaFuncAttributeMaxDynamicSharedMemorySize, Pr::kBytes)) !=
      cudaSuccess)
    return e;
  if ((e = cudaFuncSetAttribute(scan, cudaFuncAttributeMaxDynamicSharedMemorySize, Sc::kBytes)) !=
      cudaSuccess)
    return e;
  count_launch();
  if ((e = launch_pdl(prep, dim3(nc, a.H, a.B), dim3(Pr::kThreads), Pr::kBytes, st, a, scratch,
                      nc)) != cudaSuccess)
    return e;
  count_launch();
  return launch_pdl(scan, dim3(a.H, a.B), dim3(Sc::kThreads), Sc::kBytes, st, a,
                    (const float *)scratch, nc);
}

template <int D>
cudaError_t launch_d(const DeltaArgs &a, float *scratch, cudaStream_t st) {
  if (a.dtype == GBLA_FP32) return launch<float, D, 3, 3>(a, scratch, st);
  if (exact_state(a)) return launch<__nv_bfloat16, D, 3, 3>(a, scratch, st);
  return launch<__nv_bfloat16, D, 2, 1>(a, scratch, st);
}

}  // namespace
}  // namespace delta

size_t delta_forward_floats(const DeltaArgs &a) {
  using namespace delta;
  const size_t bh = (size_t)a.B * a.H;
  if (a.dtype == GBLA_FP32) return bh * chunks_of<float>(a) * Record<float, 3>::kFloats;
  return bh * chunks_of<__nv_bfloat16>(a) *
         (exact_state(a) ? Record<__nv_bfloat16, 3>::kFloats : Record<__nv_bfloat16, 1>::kFloats);
}

cudaError_t delta_forward(const DeltaArgs &a, float *scratch, cudaStream_t st) {
  if (a.D == 32) return delta::launch_d<32>(a, scratch, st);
  if (a.D == 64) return delta::launch_d<64>(a, scratch, st);
  return delta::launch_d<128>(a, scratch, st);
}

}  // namespace gbla
