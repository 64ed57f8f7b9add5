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

// --------------------------------------------------------------- first launch
// One block a (chunk, head, batch).
template <typename T, int D>
struct PrepShape {
  static constexpr int C = kChunkOf<T>, kWarps = C / 16, kThreads = kWarps * 32;
  static constexpr int kRow = pad_row<T>(D), kMat = C + 4;
  static constexpr int kBytes = (2 * C * kRow) * sizeof(T) + C * kMat * 4 + 4 * C * 4 + 16;
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

template <typename T, int D>
__global__ void __launch_bounds__(PrepShape<T, D>::kThreads)
    prepare_kernel(const DeltaArgs p, float *mats, float *scores, float *gates, int nc) {
  using Sh = PrepShape<T, D>;
  constexpr int C = Sh::C, kThreads = Sh::kThreads, kRow = Sh::kRow, kMat = Sh::kMat;
  extern __shared__ __align__(16) char raw[];
  T *ks = (T *)raw, *qs = ks + C * kRow;
  float *A = (float *)(qs + C * kRow);
  float *hi = A + C * kMat, *lo = hi + C, *beta = lo + C;
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
  const size_t at = ((size_t)b * p.H + h) * nc + blockIdx.x;
  float *gt = gates + at * Prepared<C>::kGates;
  if (tid < C) {
    if (tid >= 32) G += *first;
    const double G2 = G * 1.4426950408889634;  // powers of two from here on
    hi[tid] = (float)G2, lo[tid] = (float)(G2 - (double)hi[tid]);
    gt[Prepared<C>::kUp + tid] = expf((float)G);
    gt[Prepared<C>::kBeta + tid] = beta[tid];
    if (tid == C - 1) {
      const DecayFactor f = G < -300. ? DecayFactor{0.f, 0.f} : decay_factor((float)G);
      gt[Prepared<C>::kWhole] = f.hi, gt[Prepared<C>::kWhole + 1] = f.lo;
    }
  }
  __syncthreads();
  if (tid < C)
    gt[Prepared<C>::kDown + tid] = exp2f((hi[C - 1] - hi[tid]) + (lo[C - 1] - lo[tid]));
  // the warp's 16 rows of both products, weighted
  const int w = tid / 32, g = (tid & 31) >> 2, t = tid & 3;
  float kk[C / 8][4] = {}, qk[C / 8][4] = {};
  rows_times_rows<D, C>(kk, ks, ks, w);
  rows_times_rows<D, C>(qk, qs, ks, w);
  float *P = scores + at * C * C;
#pragma unroll
  for (int m = 0; m < C / 8; ++m) {
    if (m > 2 * w + 1) continue;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int i = 16 * w + g + 8 * half, j = 8 * m + 2 * t;
      float x[2], y[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float f = i >= j + e ? ex2_approx((hi[i] - hi[j + e]) + (lo[i] - lo[j + e])) : 0.f;
        x[e] = i > j + e ? kk[m][2 * half + e] * f * beta[j + e] : 0.f;
        y[e] = p.scale * qk[m][2 * half + e] * f;
        if (sizeof(T) == 2) y[e] = __uint_as_float(tf32_of(y[e]));  // as the products read it
      }
      *(float2 *)(A + i * kMat + j) = make_float2(x[0], x[1]);
      *(float2 *)(P + i * C + j) = make_float2(y[0], y[1]);
    }
  }
  __syncthreads();
  // M - 1 by forward substitution, a column a thread: x_i = [i = j] - sum_m A_im x_m.
  float x[C];
  float *M = mats + at * C * C;
  if (tid < C) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      float s = i == tid ? 1.f : 0.f, s1 = 0.f;
#pragma unroll
      for (int m = 0; m < i; m += 4) {
        const float4 a = *(const float4 *)(A + i * kMat + m);
        s = fmaf(-a.x, x[m], s);
        if (m + 1 < i) s1 = fmaf(-a.y, x[m + 1], s1);
        if (m + 2 < i) s = fmaf(-a.z, x[m + 2], s);
        if (m + 3 < i) s1 = fmaf(-a.w, x[m + 3], s1);
      }
      x[i] = s + s1;
      M[i * C + tid] = x[i] - (i == tid ? 1.f : 0.f);
    }
  }
}

// --------------------------------------------------------------- second launch
template <typename T, int D>
struct ScanShape {
  static constexpr int C = kChunkOf<T>, kWarps = D / 16, kThreads = kWarps * 32;
  static constexpr int kRow = pad_row<T>(D);
  static constexpr int kTile = C * kRow * sizeof(T);             // bytes of k, q or v
  static constexpr int kMatBytes = C * mat_row(C) * 4;
  static constexpr int kStage = 3 * kTile + 2 * kMatBytes + Prepared<C>::kGates * 4;
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
#pragma unroll
  for (int d = 0; d < D / 16; ++d) {
    float x[2][4] = {};
#pragma unroll
    for (int j = 0; j < C / 16; ++j) {
      const LeftBf16<kTerms> a(w[2 * j], w[2 * j + 1]);
      const PairBf16 k = by_channel<kRow>(ks, 16 * j, 16 * d);
      a.times(x[0], k.b[0][0], k.b[0][1]);
      a.times(x[1], k.b[1][0], k.b[1][1]);
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
__global__ void __launch_bounds__(ScanShape<T, D>::kThreads)
    scan_kernel(const DeltaArgs p, const float *mats, const float *scores, const float *gates,
                int nc) {
  using Sh = ScanShape<T, D>;
  constexpr int C = Sh::C, kThreads = Sh::kThreads, kRow = Sh::kRow, kMat = mat_row(C);
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
    const size_t at = bh * nc + c;
    load_rows<T, C, D, kThreads>((T *)s, kg + t0 * p.sk[1], p.sk[1], n);
    load_rows<T, C, D, kThreads>((T *)(s + Sh::kTile), qg + t0 * p.sq[1], p.sq[1], n);
    load_rows<T, C, D, kThreads>((T *)(s + 2 * Sh::kTile), vg + t0 * p.sv[1], p.sv[1], n);
    load_lower<C, kThreads>((float *)(s + 3 * Sh::kTile), mats + at * C * C);
    load_lower<C, kThreads>((float *)(s + 3 * Sh::kTile + Sh::kMatBytes), scores + at * C * C);
    load_flat<Prepared<C>::kGates, kThreads>((float *)(s + 3 * Sh::kTile + 2 * Sh::kMatBytes),
                                             gates + at * Prepared<C>::kGates);
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
    const float *M = (const float *)(s + 3 * Sh::kTile), *P = M + C * kMat, *gt = P + C * kMat;
    const int n = min(C, L - c * C);
    float r[C / 8][4] = {}, o[C / 8][4] = {};
    state_products<kTerms, D, C>(S, ks, qs, r, o);
#pragma unroll
    for (int m = 0; m < C / 16; ++m) {
      float v[2][4];
      values_of<kRow>(v[0], v[1], vs, m, e0);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 up = *(const float2 *)(gt + Prepared<C>::kUp + 16 * m + 8 * i + 2 * t);
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
          if (half * kHalf + m >= j) {
            const float2 f = *(const float2 *)(M + (8 * (half * kHalf + m) + g) * kMat + 8 * j + 2 * t);
            a.times(x[m], f.x, f.y);
          }
      }
#pragma unroll
      for (int m = 0; m < kHalf; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) r[half * kHalf + m][i] += x[m][i];
    }
    // u, and the results
#pragma unroll
    for (int j = 0; j < C / 8; ++j) {
      const float2 be = *(const float2 *)(gt + Prepared<C>::kBeta + 8 * j + 2 * t);
      r[j][0] *= be.x, r[j][1] *= be.y, r[j][2] *= be.x, r[j][3] *= be.y;
      const LeftTf32<kOut> a(r[j]);
#pragma unroll
      for (int m = j; m < C / 8; ++m) {
        const float2 f = *(const float2 *)(P + (8 * m + g) * kMat + 8 * j + 2 * t);
        a.times(o[m], f.x, f.y);
      }
      store_tile(og + (size_t)c * C * orow, orow, o[j], 8 * j, n);  // no later u meets it
      const float2 dn = *(const float2 *)(gt + Prepared<C>::kDown + 8 * j + 2 * t);
      r[j][0] *= dn.x, r[j][1] *= dn.y, r[j][2] *= dn.x, r[j][3] *= dn.y;
    }
    state_update<kTerms, D, C>(S, gt[Prepared<C>::kWhole], gt[Prepared<C>::kWhole + 1], r, ks);
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

template <typename T, int D, int kTerms, int kSolve>
cudaError_t launch(const DeltaArgs &a, float *scratch, cudaStream_t st) {
  using Pr = PrepShape<T, D>;
  using Sc = ScanShape<T, D>;
  constexpr int C = Pr::C;
  const int nc = chunks_of<T>(a);
  const size_t all = (size_t)a.B * a.H * nc;
  float *mats = scratch, *scores = mats + all * C * C, *gates = scores + all * C * C;
  const auto prep = prepare_kernel<T, D>;
  const auto scan = scan_kernel<T, D, kTerms, kSolve>;
  cudaError_t e;
  if ((e = cudaFuncSetAttribute(prep, cudaFuncAttributeMaxDynamicSharedMemorySize, Pr::kBytes)) !=
      cudaSuccess)
    return e;
  if ((e = cudaFuncSetAttribute(scan, cudaFuncAttributeMaxDynamicSharedMemorySize, Sc::kBytes)) !=
      cudaSuccess)
    return e;
  count_launch();
  if ((e = launch_pdl(prep, dim3(nc, a.H, a.B), dim3(Pr::kThreads), Pr::kBytes, st, a, mats, scores,
                      gates, nc)) != cudaSuccess)
    return e;
  count_launch();
  return launch_pdl(scan, dim3(a.H, a.B), dim3(Sc::kThreads), Sc::kBytes, st, a,
                    (const float *)mats, (const float *)scores, (const float *)gates, nc);
}

template <typename T, int D>
cudaError_t launch_terms(const DeltaArgs &a, float *scratch, cudaStream_t st) {
  if (sizeof(T) == 4 || a.fin) return launch<T, D, 3, 3>(a, scratch, st);
  return launch<T, D, 2, 3>(a, scratch, st);
}

}  // namespace
}  // namespace delta

size_t delta_forward_floats(const DeltaArgs &a) {
  const int C = a.dtype == GBLA_FP32 ? delta::kChunkOf<float> : delta::kChunkOf<__nv_bfloat16>;
  return (size_t)a.B * a.H * ((a.N + C - 1) / C) * (2 * C * C + 4 * C);
}

cudaError_t delta_forward(const DeltaArgs &a, float *scratch, cudaStream_t st) {
  if (a.dtype == GBLA_FP32) {
    if (a.D == 32) return delta::launch_terms<float, 32>(a, scratch, st);
    if (a.D == 64) return delta::launch_terms<float, 64>(a, scratch, st);
    return delta::launch_terms<float, 128>(a, scratch, st);
  }
  if (a.D == 32) return delta::launch_terms<__nv_bfloat16, 32>(a, scratch, st);
  if (a.D == 64) return delta::launch_terms<__nv_bfloat16, 64>(a, scratch, st);
  return delta::launch_terms<__nv_bfloat16, 128>(a, scratch, st);
}

}  // namespace gbla
