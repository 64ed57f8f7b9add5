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
// A block takes `each` chunks of a (head, batch) one after the other, a warp for each 16 tokens.
// One, but for large ragged batches four: the blocks that find no chunk are then a quarter as
// many (ragged D = 128 404 us, 452 with one, 415 with two and 406 with eight; full lengths, B2 H8
// N32768 D64, 90 us with one).  Blocks that stay and number the chunks that there are took a third
// longer.
template <typename T, int D>
struct PrepShape {
  static constexpr int C = kChunkOf<T>, kWarps = C / 16, kThreads = kWarps * 32;
  static constexpr int kRow = pad_row<T>(D), kMat = C + 4;
  // keys and queries, then the inverse in their place; A; the gates
  static constexpr int kTiles = 2 * C * kRow * (int)sizeof(T), kInverse = C * kMat * 4;
  static constexpr int kFirst = kTiles > kInverse ? kTiles : kInverse;
  static constexpr int kBytes = kFirst + kInverse + 4 * C * 4 + 16;
  static constexpr int kBlocks = sizeof(T) == 2 ? 5 : 8;  // an SM
};


// Products of the warp's 16 rows of keys and of queries with every row of keys up to them, fp32
// tiles of 16 x 8.
template <int D, int C>
__device__ __forceinline__ void rows_times_keys(float (&kk)[C / 8][4], float (&qk)[C / 8][4],
                                                const __nv_bfloat16 *ks, const __nv_bfloat16 *qs,
                                                int w) {
  constexpr int kRow = pad_row<__nv_bfloat16>(D);
  const int l = threadIdx.x & 31, at = (16 * w + (l & 15)) * kRow + (l >> 4) * 8;
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    uint32_t a[4], b[4];
    ldmatrix4(a, smem_u32(ks + at + 16 * k));
    ldmatrix4(b, smem_u32(qs + at + 16 * k));
#pragma unroll
    for (int n = 0; n < C / 16; ++n)
      if (n <= w) {
        const PairBf16 p = by_token<kRow>(ks, 16 * n, 16 * k);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mma_bf16(kk[2 * n + i], a, p.b[i][0], p.b[i][1]);
          mma_bf16(qk[2 * n + i], b, p.b[i][0], p.b[i][1]);
        }
      }
  }
}
template <int D, int C>
__device__ __forceinline__ void rows_times_keys(float (&kk)[C / 8][4], float (&qk)[C / 8][4],
                                                const float *ks, const float *qs, int w) {
  constexpr int kRow = pad_row<float>(D);
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll 2
  for (int k = 0; k < D / 8; ++k) {
    const int at = (16 * w + g) * kRow + 8 * k + 2 * t;
    const float2 x = *(const float2 *)(ks + at), y = *(const float2 *)(ks + at + 8 * kRow);
    const float2 u = *(const float2 *)(qs + at), v = *(const float2 *)(qs + at + 8 * kRow);
    const float c[4] = {x.x, x.y, y.x, y.y}, d[4] = {u.x, u.y, v.x, v.y};
    const LeftTf32<> a(c), q(d);
#pragma unroll
    for (int n = 0; n < C / 8; ++n)
      if (n <= 2 * w + 1) {
        const float2 b = *(const float2 *)(ks + (8 * n + g) * kRow + 8 * k + 2 * t);
        a.times(kk[n], b.x, b.y);
        q.times(qk[n], b.x, b.y);
      }
  }
}

struct TwoFloat {
  float hi, lo;
};
// a + b to 2^-45 or so of the larger (the rounding of a sum, found and carried along).
__device__ __forceinline__ TwoFloat sum_of(const TwoFloat &a, const TwoFloat &b) {
  const float s = a.hi + b.hi, r = s - a.hi;
  const float e = (a.hi - (s - r)) + (b.hi - r) + (a.lo + b.lo);
  const float hi = s + e;
  return {hi, e - (hi - s)};
}

// Parts of C x C matrices in shared memory (rows of C + 4 floats) as operands: 16 rows from i on
// at columns j .. j + 7 on the left, columns j .. j + 7 of rows i .. i + 7 on the right.
template <int C>
__device__ __forceinline__ LeftTf32<> left_of(const float *m, int i, int j) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const float2 x = *(const float2 *)(m + (i + g) * (C + 4) + j + 2 * t);
  const float2 y = *(const float2 *)(m + (i + g + 8) * (C + 4) + j + 2 * t);
  const float c[4] = {x.x, x.y, y.x, y.y};
  return LeftTf32<>(c);
}
template <int C>
__device__ __forceinline__ void times_right(float (&c)[4], const LeftTf32<> &a,
                                            const float *m, int i, int j) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const float *at = m + (i + 2 * t) * (C + 4) + j + g;
  a.times(c, at[0], at[C + 4]);
}

// to = (1 + A)^-1 for strictly lower triangular A, on and below its diagonal blocks of 16.
// Those by forward substitution, the rest from
//   (1 + A)^-1 = [ M0 0; -M1 A10 M0 M1 ]
// for pairs of blocks of 16 and then of 32, in tf32 products of three terms.  (No powers of A,
// which grow where the inverse does not: keys that repeat.)  Begins and ends with all of A, and of
// `to`, visible to the block.
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
      const auto a = left_of<C>(to, i, i + 8 * k);
#pragma unroll
      for (int n = 0; n < 2; ++n) times_right<C>(z[n], a, A, i + 8 * k, j + 8 * n);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const LeftTf32<> a(z[k]);
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
        const auto a = left_of<C>(to, i, 32 + 8 * k);
#pragma unroll
        for (int n = 0; n < 4; ++n) times_right<C>(z[n], a, A, 32 + 8 * k, 8 * n);
      }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k >= 2 || j == 0) {
        const LeftTf32<> a(z[k]);
#pragma unroll
        for (int n = 0; n < 2; ++n) times_right<C>(y[n], a, to, 8 * k, j + 8 * n);
      }
    put(y[0], i, j), put(y[1], i, j + 8);
    __syncthreads();
  }
}

// One chunk of head h of sequence b, n of its tokens there; ends without a barrier.
template <typename T, int D, bool kBack, bool kExact>
__device__ __forceinline__ void prepare_chunk(const DeltaArgs &p, char *raw, float *rec, int h,
                                              int b, int t0, int n) {
  using Sh = PrepShape<T, D>;
  using Rec = Record<T, D, kBack, kExact>;
  constexpr int C = Sh::C, kThreads = Sh::kThreads, kRow = Sh::kRow, kMat = Sh::kMat;
  T *ks = (T *)raw, *qs = ks + C * kRow;
  float *A = (float *)(raw + Sh::kFirst), *inv = (float *)raw;
  float *hi = A + C * kMat, *lo = hi + C, *beta = lo + C;
  TwoFloat *first = (TwoFloat *)(beta + 2 * C);
  const int hk = h / (p.H / p.Hk), tid = threadIdx.x;
  load_rows<T, C, D, kThreads>(ks, (const T *)p.k + b * p.sk[0] + t0 * p.sk[1] + (long long)hk * D,
                               p.sk[1], n, tid);
  load_rows<T, C, D, kThreads>(qs, (const T *)p.q + b * p.sq[0] + t0 * p.sq[1] + (long long)hk * D,
                               p.sq[1], n, tid);
  cp_async_commit();
  // Sums of the log decays (times log2 e) as two floats: differences of two of them are what
  // counts, also behind a token that ends the memory (-inf: a number whose power is 0 next to
  // any other).
  TwoFloat G = {0.f, 0.f};
  if (tid < C) {
    float lg = 0.f, be = 0.f;
    if (tid < n) {
      lg = to_f(((const T *)p.log_decay)[b * p.sg[0] + (t0 + tid) * p.sg[1] + h]);
      be = to_f(((const T *)p.beta)[b * p.sb[0] + (t0 + tid) * p.sb[1] + h]);
    }
    beta[tid] = be;
    lg = lg < -1e3f ? -1e3f : lg;  // (a NaN stays)
    constexpr float kLog2e = 1.4426950408889634f, kRest = (float)(1.4426950408889634 - (double)kLog2e);
    G.hi = lg * kLog2e;
    G.lo = fmaf(lg, kLog2e, -G.hi) + lg * kRest;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const TwoFloat o = {__shfl_up_sync(0xFFFFFFFFu, G.hi, m), __shfl_up_sync(0xFFFFFFFFu, G.lo, m)};
      if ((tid & 31) >= m) G = sum_of(o, G);
    }
    if (tid == 31) *first = G;
  }
  cp_async_wait_all();
  __syncthreads();
  float *gt = rec + Rec::kGates;
  if (tid < C) {
    if (tid >= 32) G = sum_of(*first, G);
    hi[tid] = G.hi, lo[tid] = G.lo;
    if (kBack) gt[Gates<C>::kHi + tid] = G.hi, gt[Gates<C>::kLo + tid] = G.lo;
    const float x = (G.hi + G.lo) * 0.6931471805599453f;
    gt[Gates<C>::kUp + tid] = expf(x);
    gt[Gates<C>::kBeta + tid] = beta[tid];
    if (tid == C - 1) {
      const DecayFactor f = x < -300.f ? DecayFactor{0.f, 0.f} : decay_factor(x);
      gt[Gates<C>::kWhole] = f.hi, gt[Gates<C>::kWhole + 1] = f.lo;
    }
  }
  __syncthreads();
  if (tid < C)
    gt[Gates<C>::kDown + tid] = exp2f((hi[C - 1] - hi[tid]) + (lo[C - 1] - lo[tid]));
  // the warp's 16 rows of both products, weighted.  Columns before the warp's first row meet
  // the power in two factors, both at most 1 (rows to that one, that one to the columns).
  const int w = tid / 32, g = (tid & 31) >> 2, t = tid & 3, i0 = 16 * w;
  float kk[C / 8][4] = {}, qk[C / 8][4] = {};
  rows_times_keys<D, C>(kk, qk, ks, qs, w);
  if (kBack) __syncthreads();  // P takes their place
  const float hr = hi[i0], lr = lo[i0];
  float row[2], pair[2][4];  // (pair: a row's two values of P in two adjacent tiles)
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int i = i0 + g + 8 * half;
    row[half] = ex2_approx((hi[i] - hr) + (lo[i] - lr));
  }
#pragma unroll
  for (int m = 0; m < C / 8; ++m) {
    if (m > 2 * w + 1) continue;
    const int j = 8 * m + 2 * t;
    const float2 hj = *(const float2 *)(hi + j), lj = *(const float2 *)(lo + j);
    const float2 bj = *(const float2 *)(beta + j);
    float f[2][2];
    if (m < 2 * w) {
      const float c0 = ex2_approx((hr - hj.x) + (lr - lj.x)), c1 = ex2_approx((hr - hj.y) + (lr - lj.y));
#pragma unroll
      for (int half = 0; half < 2; ++half) f[half][0] = row[half] * c0, f[half][1] = row[half] * c1;
    } else {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int i = i0 + g + 8 * half;
        f[half][0] = i >= j ? ex2_approx((hi[i] - hj.x) + (lo[i] - lj.x)) : 0.f;
        f[half][1] = i >= j + 1 ? ex2_approx((hi[i] - hj.y) + (lo[i] - lj.y)) : 0.f;
      }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int i = i0 + g + 8 * half;
      float &x0 = kk[m][2 * half], &x1 = kk[m][2 * half + 1];
      x0 *= f[half][0], x1 *= f[half][1];
      if (m >= 2 * w) x0 = i > j ? x0 : 0.f, x1 = i > j + 1 ? x1 : 0.f;
      *(float2 *)(A + i * kMat + j) = make_float2(x0 * bj.x, x1 * bj.y);
      const float p0 = p.scale * qk[m][2 * half] * f[half][0];
      const float p1 = p.scale * qk[m][2 * half + 1] * f[half][1];
      if constexpr (kBack) {
        *(float2 *)(inv + i * kMat + j) = make_float2(p0, p1);
      } else if constexpr (sizeof(T) == 2) {
        pair[half][m % 2 * 2] = p0, pair[half][m % 2 * 2 + 1] = p1;
        if (m % 2 == 1) Rec::P::store(rec + Rec::kP, 2 * w + half, m / 2, pair[half]);
      } else if (2 * w + half >= m) {
        Rec::P::store(rec + Rec::kP, 2 * w + half, m, p0, p1);
      }
    }
  }
  __syncthreads();
  // a matrix in shared memory, tile by tile: as it is, or (flip) for sums over its rows; the
  // backward's inverses without their diagonal of 1 (that part of a product needs no rounding),
  // the forward's multiplied by beta
  auto put = [&](float *to, bool flip, bool inverse) {
    for (int m = w; m < C / 8; m += Sh::kWarps)
      for (int j = 0; j <= m; ++j) {
        const float *at = inv + (8 * m + (flip ? 2 * t : g)) * kMat + 8 * j + (flip ? g : 2 * t);
        const bool one = inverse && kBack && j == m;
        const float by = inverse && !kBack ? beta[8 * m + g] : 1.f;
        Rec::M::store(to, m, j, one && g == 2 * t ? 0.f : by * at[0],
                      one && g == 2 * t + 1 ? 0.f : by * at[flip ? kMat : 1]);
      }
  };
  if (kBack) {
    if constexpr (Rec::P::kWide == 2) {  // 16 rows a warp
      for (int j = 0; j < 2 * w + 2; ++j) {
        const float *at = inv + (16 * w + 2 * t) * kMat + 8 * j + g;
        const float x[4] = {at[0], at[kMat], at[8 * kMat], at[9 * kMat]};
        Rec::P::store(rec + Rec::kP, w, j, x);
      }
    } else {
      put(rec + Rec::kP, true, false);
    }
    __syncthreads();
  }
  invert<C>(inv, A, w);
  put(rec + Rec::kM, false, true);
  if (kBack) {  // (1 + beta X)^-1: the rows weighted in place of the columns
    __syncthreads();
#pragma unroll
    for (int m = 0; m < C / 8; ++m) {
      if (m > 2 * w + 1) continue;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int i = 16 * w + g + 8 * half;
        *(float2 *)(A + i * kMat + 8 * m + 2 * t) =
            make_float2(kk[m][2 * half] * beta[i], kk[m][2 * half + 1] * beta[i]);
      }
    }
    __syncthreads();
    invert<C>(inv, A, w);
    put(rec + Rec::kT, true, true);
  }
}

template <typename T, int D, bool kBack, bool kExact>
__global__ void __launch_bounds__(PrepShape<T, D>::kThreads, PrepShape<T, D>::kBlocks)
    prepare_kernel(const DeltaArgs p, float *records, int nc, int each) {
  constexpr int C = PrepShape<T, D>::C;
  extern __shared__ __align__(16) char raw[];
  grid_dep_wait();
  const int h = blockIdx.y, b = blockIdx.z;
  const int L = p.seq_lens ? min(max(__ldg(p.seq_lens + b), 0), p.N) : p.N;
  const int first = blockIdx.x * each, end = min(first + each, (L + C - 1) / C);
  for (int c = first; c < end; ++c) {
    if (c > first) __syncthreads();  // the chunk before is done with
    prepare_chunk<T, D, kBack, kExact>(
        p, raw, records + (((size_t)b * p.H + h) * nc + c) * Record<T, D, kBack, kExact>::kFloats, h,
        b, c * C, min(C, L - c * C));
  }
}

// --------------------------------------------------------------- the scan
// A block carries E = min(D, 64) of the state's columns through the chunks of a segment of a
// sequence, 16 a warp in kCarry warps.  What the columns need for the next chunk is a chain:
//   S^T k -> r -> miss = M r -> u -> S',
// and everything else is taken off it: other warps fetch tiles, and form the results of the chunk
// before, from the state and u that the first ones leave in shared memory.  One barrier a chunk.
//
// What it is for: results (kResults), the states and misses that the backward pass needs
// (kSave), or what a segment does to the state before it (kSegment): E columns of its own
// state, from zero, or of the matrix that takes the state before the segment to the one after
// it, from the identity and with no values.
enum Purpose { kResults, kSave, kSegment };

template <typename T, int D, int kTerms, Purpose kFor>
struct ScanShape {
  using Rec = Record<T, D, kFor == kSave>;
  static constexpr int C = kChunkOf<T>, E = D < 64 ? D : 64, kSplit = D / E;
  // (without results the other warps only fetch, half as many do, and two blocks fit an SM)
  static constexpr int kCarry = E / 16, kHelp = kFor != kResults && kCarry > 2 ? 2 : kCarry;
  static constexpr int kThreads = (kCarry + kHelp) * 32;
  static constexpr int kBlocks = kFor != kResults && (D < 128 || kTerms == 2) ? 2 : 1;
  static constexpr int kRow = pad_row<T>(D), kValRow = pad_row<T>(E);
  // bytes: keys, values, M and gates of a chunk; queries, P and gates of the one before
  static constexpr int kKeys = C * kRow * (int)sizeof(T), kVals = C * kValRow * (int)sizeof(T);
  static constexpr int kRecord = Rec::kP * 4, kFirst = kKeys + kVals + kRecord;
  static constexpr int kSecond = kFor == kResults ? kKeys + (Rec::P::kFloats + C) * 4 : 0;
  // what a warp hands on: its state before the chunk and u
  static constexpr int kHand = kFor != kResults ? 0 : (kHandWords<D> + C / 8) * 32 * 16;
  static constexpr int kBytes = 2 * (kFirst + kSecond + kCarry * kHand);
  static_assert(kBytes <= 227 * 1024, "shared memory of a block");
};

// kTerms: bf16 numbers that stand for a value of the state where it meets a key or takes a
// write (fp32: 3 tf32 products).
// Segments have `seg` chunks; `before` holds the states after all but the last, or takes what
// kSegment forms, the matrices in `moves`, [B H][count][D][D] both.  Records are `stride` floats
// apart (their M and gates lie at the same place in both forms).
// kFold: M comes multiplied by beta (the forward pass's records) and gives u at once; else
// without its diagonal of 1, and gives the misses.
template <typename T, int D, int kTerms, Purpose kFor, bool kFold>
__global__ void __launch_bounds__(ScanShape<T, D, kTerms, kFor>::kThreads,
                                  ScanShape<T, D, kTerms, kFor>::kBlocks)
    scan_kernel(const DeltaArgs p, const float *records, float *states, float *misses,
                float *before, float *moves, int nc, int seg, int count, int stride) {
  using Sh = ScanShape<T, D, kTerms, kFor>;
  using Rec = typename Sh::Rec;
  constexpr int C = Sh::C, E = Sh::E, kCarry = Sh::kCarry, kFetch = Sh::kHelp * 32;
  constexpr bool kSums = sizeof(T) == 4;
  constexpr int kColumns = kFor == kSegment ? 2 * Sh::kSplit : Sh::kSplit;  // blocks a head
  extern __shared__ __align__(16) char raw[];
  grid_dep_wait();
  const int h = blockIdx.x / kColumns, part = blockIdx.x % kColumns, s = blockIdx.z;
  const int b = longest_first(p.seq_lens, p.B, blockIdx.y);
  const int hk = h / (p.H / p.Hk), tid = threadIdx.x, warp = tid / 32, lane = tid & 31, t = tid & 3;
  const bool carry = warp < kCarry;
  const bool move = part >= Sh::kSplit;  // kSegment: columns of the matrix
  const int x0 = part % Sh::kSplit * E, e0 = x0 + warp % kCarry * 16;
  const int L = p.seq_lens ? min(max(__ldg(p.seq_lens + b), 0), p.N) : p.N;
  const size_t bh = (size_t)b * p.H + h;
  const int chunks = (L + C - 1) / C, first = s * seg, end = min(chunks, first + seg);
  // (gridDim.z: all segments, or, for kSegment in the forward pass, those that another follows)
  if (s > 0 && first >= chunks) return;
  if (kFor == kSegment && (chunks == 0 || ((int)gridDim.z < count && end == chunks))) return;
  const T *kg = (const T *)p.k + b * p.sk[0] + (long long)hk * D;
  const T *qg = (const T *)p.q + b * p.sq[0] + (long long)hk * D;
  const T *vg = (const T *)p.v + b * p.sv[0] + (long long)h * D + x0;
  const size_t orow = (size_t)p.H * D;
  char *hands = raw + 2 * (Sh::kFirst + Sh::kSecond) + warp % kCarry * Sh::kHand;
  auto first_of = [&](int c) { return raw + (c & 1) * Sh::kFirst; };
  auto second_of = [&](int c) { return raw + 2 * Sh::kFirst + (c & 1) * Sh::kSecond; };
  auto hand_of = [&](int c) { return (uint4 *)(hands + (c & 1) * (kCarry * Sh::kHand)); };
  const int ftid = tid - kCarry * 32;
  auto fetch_first = [&](int c) {
    char *to = first_of(c);
    const long long t0 = (long long)c * C;
    const int n = min(C, L - c * C);
    load_rows<T, C, D, kFetch>((T *)to, kg + t0 * p.sk[1], p.sk[1], n, ftid);
    load_rows<T, C, E, kFetch>((T *)(to + Sh::kKeys), vg + t0 * p.sv[1], p.sv[1], move ? 0 : n, ftid);
    load_flat<Rec::kP, kFetch>((float *)(to + Sh::kKeys + Sh::kVals),
                               records + (bh * nc + c) * stride, ftid);
  };
  auto fetch_second = [&](int c) {
    char *to = second_of(c);
    const long long t0 = (long long)c * C;
    const float *rec = records + (bh * nc + c) * stride;
    load_rows<T, C, D, kFetch>((T *)to, qg + t0 * p.sq[1], p.sq[1], min(C, L - c * C), ftid);
    load_flat<Rec::P::kFloats, kFetch>((float *)(to + Sh::kKeys), rec + Rec::kP, ftid);
    load_flat<C, kFetch>((float *)(to + Sh::kKeys) + Rec::P::kFloats,
                         rec + Rec::kGates + Gates<C>::kUp, ftid);
  };
  float S[D / 8][4];  // rows: columns e0 + g, + 8 of the state; columns: its rows
  if (carry) {
    if (move) {
      const int g = lane >> 2;
#pragma unroll
      for (int d = 0; d < D / 8; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          S[d][i] = 8 * d + 2 * t + (i & 1) == e0 + g + (i >> 1) * 8 ? 1.f : 0.f;
    } else {
      const float *from = kFor == kSegment ? nullptr
                          : s > 0          ? before + (bh * count + s - 1) * D * D
                          : p.init         ? p.init + bh * D * D
                                           : nullptr;
      load_state<D>(S, from, e0);
    }
  } else {
    if (first < end) fetch_first(first);
    cp_async_commit();
    cp_async_wait_all();
  }
  const int turns = kFor == kResults ? end + 1 : end;
  for (int c = first; c < turns; ++c) {
    __syncthreads();  // this turn's tiles and what was handed on are there, the others are read
    if (carry) {
      if (c >= end) break;
      const char *in = first_of(c);
      const T *ks = (const T *)in, *vs = (const T *)(in + Sh::kKeys);
      const float *M = (const float *)(in + Sh::kKeys + Sh::kVals), *gt = M + Rec::kGates;
      uint4 *hand = hand_of(c);
      float r[C / 8][4] = {};
      if (kFor == kSave) store_packed(states + (bh * nc + c) * D * D, S, e0);
      key_products<kTerms, D, C, kFor == kResults>(S, ks, r, hand);
#pragma unroll
      for (int m = 0; m < C / 16; ++m) {
        float v[2][4];
        values_of<Sh::kValRow>(v[0], v[1], vs, m, e0 - x0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 up = *(const float2 *)(gt + Gates<C>::kUp + 16 * m + 8 * i + 2 * t);
          float(&x)[4] = r[2 * m + i];
          x[0] = fmaf(-up.x, x[0], v[i][0]), x[1] = fmaf(-up.y, x[1], v[i][1]);
          x[2] = fmaf(-up.x, x[2], v[i][2]), x[3] = fmaf(-up.y, x[3], v[i][3]);
        }
      }
      // r = beta M r, or r += (M - 1) r: the later half of the tokens first, which needs the
      // earlier ones as they are; then those
#pragma unroll
      for (int half = 1; half >= 0; --half) {
        constexpr int kHalf = C / 16;
        float x[kHalf][4] = {};
#pragma unroll
        for (int j = 0; j < (half + 1) * kHalf; ++j) {
          const auto a = Rec::M::template left<kSums>(r, j);
#pragma unroll
          for (int m = 0; m < kHalf; ++m)
            if (half * kHalf + m >= j) a.times(x[m], Rec::M::load(M, half * kHalf + m, j));
        }
#pragma unroll
        for (int m = 0; m < kHalf; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            r[half * kHalf + m][i] = kFold ? x[m][i] : r[half * kHalf + m][i] + x[m][i];
      }
      if (kFor == kSave) store_packed(misses + (bh * nc + c) * C * D, r, e0);
#pragma unroll
      for (int j = 0; j < C / 8; ++j) {
        float4 *to = (float4 *)hand + (kHandWords<D> + j) * 32 + lane;
        if (!kFold) {
          const float2 be = *(const float2 *)(gt + Gates<C>::kBeta + 8 * j + 2 * t);
          r[j][0] *= be.x, r[j][1] *= be.y, r[j][2] *= be.x, r[j][3] *= be.y;
        }
        if (kFor == kResults) *to = make_float4(r[j][0], r[j][1], r[j][2], r[j][3]);
        const float2 dn = *(const float2 *)(gt + Gates<C>::kDown + 8 * j + 2 * t);
        r[j][0] *= dn.x, r[j][1] *= dn.y, r[j][2] *= dn.x, r[j][3] *= dn.y;
      }
      state_update<kTerms, D, C>(S, gt[Gates<C>::kWhole], gt[Gates<C>::kWhole + 1], r, ks);
    } else {
      if (c + 1 < end) fetch_first(c + 1);
      if (kFor == kResults && c < end) fetch_second(c);
      cp_async_commit();
      if constexpr (kFor == kResults)
        if (c > first) {  // the chunk before
          const int d0 = c - 1;
          const uint4 *hand = hand_of(d0);
          const float4 *us = (const float4 *)hand + kHandWords<D> * 32 + lane;
          const char *in = second_of(d0);
          const float *P = (const float *)(in + Sh::kKeys), *ups = P + Rec::P::kFloats;
          T *og = (T *)p.o + (((size_t)b * p.N + (size_t)d0 * C) * p.H + h) * D + e0;
          const int n = min(C, L - d0 * C);
          float o[C / 8][4] = {};
          query_products<D, C>(hand, (const T *)in, o);
#pragma unroll
          for (int j = 0; j < C / 8; ++j) {
            const float2 up = *(const float2 *)(ups + 8 * j + 2 * t);
            const float ux = up.x * p.scale, uy = up.y * p.scale;
            o[j][0] *= ux, o[j][1] *= uy, o[j][2] *= ux, o[j][3] *= uy;
          }
          constexpr int kWide = Rec::P::kWide;
#pragma unroll
          for (int j = 0; j < C / 8 / kWide; ++j) {
            float u[kWide][4];
#pragma unroll
            for (int i = 0; i < kWide; ++i) {
              const float4 v = us[(j * kWide + i) * 32];
              u[i][0] = v.x, u[i][1] = v.y, u[i][2] = v.z, u[i][3] = v.w;
            }
            const auto a = Rec::P::template left<kSums>(u, 0);
#pragma unroll
            for (int m = j * kWide; m < C / 8; ++m) a.times(o[m], Rec::P::load(P, m, j));
#pragma unroll
            for (int i = j * kWide; i < (j + 1) * kWide; ++i)
              store_tile(og, orow, o[i], 8 * i, n);  // no later u meets it
          }
        }
      cp_async_wait_all();
    }
  }
  if (!carry) return;
  if (kFor == kSegment) {
    const size_t at = (bh * count + s) * D * D;
    store_state<D>((move ? moves : before) + at, S, e0);
  } else if (kFor == kResults && p.fin && (end == chunks)) {
    store_state<D>(p.fin + bh * D * D, S, e0);
  }
}

// --------------------------------------------------------------- between segments
// A block takes E of the state's columns of one (batch, head).
template <int D>
struct JoinShape {
  static constexpr int E = D < 64 ? D : 64, kThreads = E * 2, kRow = D + 8;
  static constexpr int kBytes = 2 * D * kRow * 4;
};
template <int D, bool kBack>
__global__ void __launch_bounds__(JoinShape<D>::kThreads)
    join_kernel(const float *init, const int32_t *seq_lens, float *own, const float *moves, int N,
                int H, int tokens, int count) {
  using Sh = JoinShape<D>;
  constexpr int kThreads = Sh::kThreads, kRow = Sh::kRow;
  extern __shared__ __align__(16) char raw[];
  float *tile = (float *)raw;
  grid_dep_wait();
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, g = (tid & 31) >> 2, t = tid & 3;
  const int e0 = blockIdx.x * Sh::E + tid / 32 * 16;
  const int L = seq_lens ? min(max(__ldg(seq_lens + b), 0), N) : N;
  const int ns = (L + tokens - 1) / tokens, steps = ns - 1;
  if (steps <= 0) return;
  const size_t bh = (size_t)b * H + h;
  own += bh * count * D * D, moves += bh * count * D * D;
  // the i-th segment in order, 0 .. ns - 2 or ns - 1 .. 1
  auto at = [&](int i) { return (size_t)(kBack ? ns - 1 - i : i) * D * D; };
  auto fetch = [&](int i) {
    load_rows<float, D, D, kThreads>(tile + (i & 1) * D * kRow, moves + at(i), D, D, tid);
  };
  float S[D / 8][4];
  load_state<D>(S, init ? init + bh * D * D : nullptr, e0);
  fetch(0);
  cp_async_commit();
  for (int i = 0; i < steps; ++i) {
    float add[D / 8][4], x[D / 8][4] = {};
    load_state<D>(add, own + at(i), e0);
    cp_async_wait_all();
    __syncthreads();
    if (i + 1 < steps) fetch(i + 1);
    cp_async_commit();
    const float *m = tile + (i & 1) * D * kRow;
#pragma unroll
    for (int k = 0; k < D / 8; ++k) {
      const LeftTf32<> a(S[k]);
#pragma unroll
      for (int n = 0; n < D / 8; ++n) {
        if (kBack) {
          const float *v = m + (8 * k + 2 * t) * kRow + 8 * n + g;
          a.times(x[n], v[0], v[kRow]);
        } else {
          const float2 v = *(const float2 *)(m + (8 * n + g) * kRow + 8 * k + 2 * t);
          a.times(x[n], v.x, v.y);
        }
      }
    }
#pragma unroll
    for (int d = 0; d < D / 8; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[d][e] = x[d][e] + add[d][e];
    store_state<D>(own + at(i), S, e0);
  }
}

// Where a state is a result it meets keys and writes in three terms; bf16 results alone need two
// (2^-16, beside 2^-8 of their own rounding).
bool exact_state(const DeltaArgs &a) { return a.dtype == GBLA_FP32 || a.fin; }

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
    return 152;
  return n;
}

template <typename K>
cudaError_t allow_smem(K kernel, int bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <int D, bool kBack>
cudaError_t join_launch(const DeltaArgs &a, const Segments &g, const float *init, float *own,
                        const float *moves, cudaStream_t st) {
  using Jo = JoinShape<D>;
  const auto join = join_kernel<D, kBack>;
  cudaError_t e;
  if ((e = allow_smem(join, Jo::kBytes)) != cudaSuccess) return e;
  const int C = a.dtype == GBLA_FP32 ? kChunkOf<float> : kChunkOf<__nv_bfloat16>;
  count_launch();
  return launch_pdl(join, dim3(D / Jo::E, a.H, a.B), dim3(Jo::kThreads), Jo::kBytes, st, init,
                    a.seq_lens, own, moves, a.N, a.H, g.chunks * C, g.count);
}

template <typename T, int D, int kTerms, Purpose kFor>
cudaError_t launch(const DeltaArgs &a, const Segments &g, float *records, float *states,
                   float *misses, float *before, float *moves, cudaStream_t st) {
  using Pr = PrepShape<T, D>;
  using Sc = ScanShape<T, D, kTerms, kFor>;
  using Se = ScanShape<T, D, kTerms, kSegment>;
  static_assert(kFor != kSegment, "");
  constexpr bool kExact = kFor == kSave && kTerms == 3;
  const int nc = chunks_of<T>(a), stride = Record<T, D, kFor == kSave, kExact>::kFloats;
  cudaError_t e;
  const auto prep = prepare_kernel<T, D, kFor == kSave, kExact>;
  if ((e = allow_smem(prep, Pr::kBytes)) != cudaSuccess) return e;
  const int each = a.seq_lens && (long long)nc * a.H * a.B >= 64ll * sm_count() ? 4 : 1;
  count_launch();
  if ((e = launch_pdl(prep, dim3((nc + each - 1) / each, a.H, a.B), dim3(Pr::kThreads), Pr::kBytes,
                      st, a, records, nc, each)) != cudaSuccess)
    return e;
  if (g.count > 1) {
    const auto own = scan_kernel<T, D, kTerms, kSegment, kFor == kResults>;
    if ((e = allow_smem(own, Se::kBytes)) != cudaSuccess) return e;
    count_launch();
    // (the backward pass moves its gradients by the last segment's matrix too)
    if ((e = launch_pdl(own, dim3(2 * Se::kSplit * a.H, a.B, kFor == kSave ? g.count : g.count - 1),
                        dim3(Se::kThreads), Se::kBytes, st, a, (const float *)records,
                        (float *)nullptr, (float *)nullptr, before, moves, nc, g.chunks, g.count,
                        stride)) != cudaSuccess)
      return e;
    if ((e = join_launch<D, false>(a, g, a.init, before, moves, st)) != cudaSuccess) return e;
  }
  const auto scan = scan_kernel<T, D, kTerms, kFor, kFor == kResults>;
  if ((e = allow_smem(scan, Sc::kBytes)) != cudaSuccess) return e;
  count_launch();
  return launch_pdl(scan, dim3(Sc::kSplit * a.H, a.B, g.count), dim3(Sc::kThreads), Sc::kBytes, st,
                    a, (const float *)records, states, misses, before, moves, nc, g.chunks, g.count,
                    stride);
}

template <int D>
cudaError_t forward_d(const DeltaArgs &a, const Segments &g, float *rec, float *before, float *moves,
                      cudaStream_t st) {
  if (a.dtype == GBLA_FP32)
    return launch<float, D, 3, kResults>(a, g, rec, nullptr, nullptr, before, moves, st);
  if (exact_state(a))
    return launch<__nv_bfloat16, D, 3, kResults>(a, g, rec, nullptr, nullptr, before, moves, st);
  return launch<__nv_bfloat16, D, 2, kResults>(a, g, rec, nullptr, nullptr, before, moves, st);
}
template <int D>
cudaError_t save_d(const DeltaArgs &a, const Segments &g, bool exact, float *rec, float *states,
                   float *misses, float *before, float *moves, cudaStream_t st) {
  if (a.dtype == GBLA_FP32)
    return launch<float, D, 3, kSave>(a, g, rec, states, misses, before, moves, st);
  if (exact)
    return launch<__nv_bfloat16, D, 3, kSave>(a, g, rec, states, misses, before, moves, st);
  return launch<__nv_bfloat16, D, 2, kSave>(a, g, rec, states, misses, before, moves, st);
}

}  // namespace

// How many segments.  In units of a chunk in a scan of whole sequences (measured, bf16 D = 64:
// 2.4 us, 2.8 with states of full precision): a round of blocks takes a segment's chunks; the scan
// that forms the segments' own states and matrices has twice the blocks, two an SM, and as much
// for a round of these; 0.6 where there is one an SM, which pays neither with states of full
// precision at D = 128 nor in fp32 nor for the backward's three further passes; a segment that is
// joined 1.2.
// Any count and the rule's: B2 H8 N32768: 1 segment 1338 us, 4 599, 8 437, 9 404 (taken), 10 469,
// 19 411; the same at D = 128, N8192: 1 464, 3 313 (taken), 4 307, 6 377; at D = 32: 1 185, 9 83
// (taken), 12 96; B8 H8 N2048, states out: 1 117, 2 107 (taken), 3 133; without: 106, 97, 119;
// backward B4 H8 N8192: 1 939, 4 661 (taken), 9 654; fp32 B3 H6 N517: 1 139, 4 117, 6 104 (taken).
Segments segments_of(const DeltaArgs &a, bool back) {
  const int nc = a.dtype == GBLA_FP32 ? chunks_of<float>(a) : chunks_of<__nv_bfloat16>(a);
  const long long blocks = (long long)a.B * a.H * (a.D > 64 ? 2 : 1), sms = sm_count();
  const double lone = back || (exact_state(a) && (a.D > 64 || a.dtype == GBLA_FP32)) ? 1. : 0.6;
  Segments best = {1, nc};
  double least = 0.;
  for (int want = 1; want <= 64 && want <= nc; ++want) {
    const int chunks = (nc + want - 1) / want, count = (nc + chunks - 1) / chunks;
    double cost = (double)((blocks * count + sms - 1) / sms) * chunks;
    const long long half = (2 * blocks * (count - 1) + sms - 1) / sms;
    if (count > 1) cost += (half / 2 + lone * (half % 2)) * chunks + 1.2 * (count - 1) + 4.;
    if (want == 1 || cost < least) least = cost, best = {count, chunks};
  }
  return best;
}

cudaError_t save_forward(const DeltaArgs &a, const Segments &g, bool exact, float *rec,
                         float *states, float *misses, float *before, float *moves,
                         cudaStream_t st) {
  if (a.D == 32) return save_d<32>(a, g, exact, rec, states, misses, before, moves, st);
  if (a.D == 64) return save_d<64>(a, g, exact, rec, states, misses, before, moves, st);
  return save_d<128>(a, g, exact, rec, states, misses, before, moves, st);
}

cudaError_t join_back(const DeltaArgs &a, const Segments &g, const float *init, float *own,
                      const float *moves, cudaStream_t st) {
  if (a.D == 32) return join_launch<32, true>(a, g, init, own, moves, st);
  if (a.D == 64) return join_launch<64, true>(a, g, init, own, moves, st);
  return join_launch<128, true>(a, g, init, own, moves, st);
}

}  // namespace delta

static size_t record_floats(const DeltaArgs &a) {
  using namespace delta;
  const size_t bh = (size_t)a.B * a.H;
  if (a.dtype == GBLA_FP32) return bh * chunks_of<float>(a) * Record<float, 128, false>::kFloats;
  return bh * chunks_of<__nv_bfloat16>(a) *
         (a.D < 128 ? Record<__nv_bfloat16, 64, false>::kFloats : Record<__nv_bfloat16, 128, false>::kFloats);
}

size_t delta_forward_floats(const DeltaArgs &a) {
  return record_floats(a) + 2 * delta::segments_of(a, false).floats(a);
}

cudaError_t delta_forward(const DeltaArgs &a, float *scratch, cudaStream_t st) {
  const delta::Segments g = delta::segments_of(a, false);
  float *before = scratch + record_floats(a), *moves = before + g.floats(a);
  if (a.D == 32) return delta::forward_d<32>(a, g, scratch, before, moves, st);
  if (a.D == 64) return delta::forward_d<64>(a, g, scratch, before, moves, st);
  return delta::forward_d<128>(a, g, scratch, before, moves, st);
}

}  // namespace gbla
