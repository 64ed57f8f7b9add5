// Backward pass of attention by the gated delta rule, in chunks of C tokens.
//
// With the notation of the forward pass (S before the chunk, A the gradient of the state
// after it, m the misses, u = beta m, T = (1 + beta X)^-1), d the gradients of the results:
//   du_j  = sum_i P_ij d_i + e^(G_C - G_j) A^T k_j,   w = T^T du,   dv = beta w,
//   dbeta_j = w_j . m_j,
//   A'    = e^(G_C) A + sum_i e^(G_i) (scale q_i d_i^T - k_i dv_i^T)   (before the chunk),
// and with dP_ij = scale e^(G_i - G_j) d_i . u_j (j <= i), E_ij = -e^(G_i - G_j) dv_i . u_j (j < i)
//   dq_i = scale e^(G_i) S d_i + sum_j dP_ij k_j,
//   dk_i = e^(G_C - G_i) A u_i - e^(G_i) S dv_i + sum_j E_ij k_j + sum_j (dP_ji q_j + E_ji k_j).
// Every product with a power e^(+-G_i) gives G_i its share, +- itself; the gradient of a token's
// log decay is the sum of those of G_i from it to the chunk's end.
//
// Four launches: what every chunk can prepare by itself, the misses and states from the first
// chunk on, w, dv and A from the last one back, and the rest of each chunk's gradients.  Sequences
// that are cut into segments take four more (each segment's own state and matrix, what it adds to
// A, a join after each), heads that share keys a sum.
#include <math.h>

#include "gbla_delta_mma.cuh"

namespace gbla {
namespace delta {
namespace {

// ------------------------------------------------------------- from the last chunk back
// The forward scan's counterpart: a block carries E = min(D, 64) of the columns of A, 16 a warp,
// from a segment's last chunk to its first.  On the chain are A^T k -> du -> w -> A'; what does
// not need A (sum_i P_ij d_i, and what the results and queries add to A') other warps form one
// chunk ahead and leave in shared memory.  kOwn: what a segment adds to A, from zero and with
// nothing written.
template <typename T, int D, int kTerms>
struct ReverseShape {
  using Rec = Record<T, D, true, kTerms == 3>;
  static constexpr int C = kChunkOf<T>, E = D < 64 ? D : 64, kSplit = D / E;
  static constexpr int kCarry = E / 16, kThreads = 2 * kCarry * 32;
  static constexpr int kRow = pad_row<T>(D), kValRow = pad_row<T>(E);
  // bytes: keys, gates and T of a chunk; queries, d, gates and P of the one ahead
  static constexpr int kKeys = C * kRow * (int)sizeof(T), kVals = C * kValRow * (int)sizeof(T);
  static constexpr int kGate = Gates<C>::kFloats * 4;
  static constexpr int kFirst = kKeys + kGate + Rec::M::kFloats * 4;
  static constexpr int kSecond = kKeys + kVals + kGate + Rec::P::kFloats * 4;
  static constexpr int kHand = (C / 8 + D / 8) * 32 * 16;
  static constexpr int kBytes = 2 * (kFirst + kSecond + kCarry * kHand);
  static_assert(kBytes <= 227 * 1024, "shared memory of a block");
};

template <typename T, int D, int kTerms, bool kOwn>
__global__ void __launch_bounds__(ReverseShape<T, D, kTerms>::kThreads)
    reverse_kernel(const DeltaBackArgs p, const float *records, float *after, float *weights,
                   float *own, int nc, int seg, int count) {
  using Sh = ReverseShape<T, D, kTerms>;
  using Rec = typename Sh::Rec;
  constexpr int C = Sh::C, E = Sh::E, kCarry = Sh::kCarry, kFetch = kCarry * 32;
  constexpr bool kSums = sizeof(T) == 4;
  extern __shared__ __align__(16) char raw[];
  grid_dep_wait();
  const DeltaArgs &f = p.f;
  const int h = blockIdx.x / Sh::kSplit, s = blockIdx.z;
  const int b = longest_first(f.seq_lens, f.B, blockIdx.y);
  const int hk = h / (f.H / f.Hk), tid = threadIdx.x, warp = tid / 32, lane = tid & 31, t = tid & 3;
  const bool carry = warp < kCarry;
  const int x0 = blockIdx.x % Sh::kSplit * E, e0 = x0 + warp % kCarry * 16;
  const int L = f.seq_lens ? min(max(__ldg(f.seq_lens + b), 0), f.N) : f.N;
  const size_t bh = (size_t)b * f.H + h;
  const int chunks = (L + C - 1) / C, first = s * seg, end = min(chunks, first + seg);
  if (s > 0 && first >= chunks) return;
  if (kOwn && s == 0) return;  // nobody reads it
  const T *kg = (const T *)f.k + b * f.sk[0] + (long long)hk * D;
  const T *qg = (const T *)f.q + b * f.sq[0] + (long long)hk * D;
  const size_t orow = (size_t)f.H * D;
  const T *dg = (const T *)p.d_o + ((size_t)b * f.N * f.H + h) * D + x0;
  T *vg = (T *)p.dv + ((size_t)b * f.N * f.H + h) * D + e0;
  char *hands = raw + 2 * (Sh::kFirst + Sh::kSecond) + warp % kCarry * Sh::kHand;
  auto first_of = [&](int c) { return raw + (c & 1) * Sh::kFirst; };
  auto second_of = [&](int c) { return raw + 2 * Sh::kFirst + (c & 1) * Sh::kSecond; };
  auto hand_of = [&](int c) { return (float4 *)(hands + (c & 1) * (kCarry * Sh::kHand)) + lane; };
  const int ftid = tid - kCarry * 32;
  auto fetch_first = [&](int c) {
    char *to = first_of(c);
    const long long t0 = (long long)c * C;
    const float *rec = records + (bh * nc + c) * Rec::kFloats;
    load_rows<T, C, D, kFetch>((T *)to, kg + t0 * f.sk[1], f.sk[1], min(C, L - c * C), ftid);
    load_flat<Gates<C>::kFloats, kFetch>((float *)(to + Sh::kKeys), rec + Rec::kGates, ftid);
    load_flat<Rec::M::kFloats, kFetch>((float *)(to + Sh::kKeys + Sh::kGate), rec + Rec::kT, ftid);
  };
  auto fetch_second = [&](int c) {
    char *to = second_of(c);
    const long long t0 = (long long)c * C;
    const int n = min(C, L - c * C);
    load_rows<T, C, D, kFetch>((T *)to, qg + t0 * f.sq[1], f.sq[1], n, ftid);
    load_rows<T, C, E, kFetch>((T *)(to + Sh::kKeys), dg + t0 * orow, (long long)orow, n, ftid);
    load_flat<Gates<C>::kFloats + Rec::P::kFloats, kFetch>(  // (side by side)
        (float *)(to + Sh::kKeys + Sh::kVals),
        records + (bh * nc + c) * Rec::kFloats + Rec::kGates, ftid);
  };
  float A[D / 8][4];
  if (carry) {
    const float *from = kOwn           ? nullptr
                        : end < chunks ? own + (bh * count + s + 1) * D * D
                        : p.dstate     ? p.dstate + bh * D * D
                                       : nullptr;
    load_state<D>(A, from, e0);
  } else {
    if (first < end) fetch_second(end - 1);
    cp_async_commit();
    cp_async_wait_all();
  }
  // turn c: the chain's chunk c, the others' chunk c - 1
  for (int c = end; c >= first; --c) {
    __syncthreads();  // this turn's tiles and what was left are there, the others are read
    if (carry) {
      if (c == end) continue;
      const char *in = first_of(c);
      const T *ks = (const T *)in;
      const float *gt = (const float *)(in + Sh::kKeys), *Tm = gt + Gates<C>::kFloats;
      const float4 *hand = hand_of(c);
      const int n = min(C, L - c * C);
      if (!kOwn) store_packed(after + (bh * nc + c) * D * D, A, e0);
      float r[C / 8][4] = {};
      key_products<kTerms, D, C, false>(A, ks, r, nullptr);
#pragma unroll
      for (int j = 0; j < C / 8; ++j) {
        const float2 dn = *(const float2 *)(gt + Gates<C>::kDown + 8 * j + 2 * t);
        const float4 x = hand[j * 32];
        r[j][0] = fmaf(dn.x, r[j][0], x.x), r[j][1] = fmaf(dn.y, r[j][1], x.y);
        r[j][2] = fmaf(dn.x, r[j][2], x.z), r[j][3] = fmaf(dn.y, r[j][3], x.w);
      }
      // r += (T - 1)^T r: the earlier half of the tokens first, which needs the later ones as
      // they are
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        constexpr int kHalf = C / 16;
        float x[kHalf][4] = {};
#pragma unroll
        for (int i = half * kHalf; i < C / 8; ++i) {
          const auto a = Rec::M::template left<kSums>(r, i);
#pragma unroll
          for (int j = 0; j < kHalf; ++j)
            if (half * kHalf + j <= i) a.times(x[j], Rec::M::load(Tm, i, half * kHalf + j));
        }
#pragma unroll
        for (int j = 0; j < kHalf; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) r[half * kHalf + j][i] += x[j][i];
      }
      if (!kOwn) store_packed(weights + (bh * nc + c) * C * D, r, e0);
#pragma unroll
      for (int j = 0; j < C / 8; ++j) {
        const float2 be = *(const float2 *)(gt + Gates<C>::kBeta + 8 * j + 2 * t);
        r[j][0] *= be.x, r[j][1] *= be.y, r[j][2] *= be.x, r[j][3] *= be.y;
        if (!kOwn) store_tile(vg + (size_t)c * C * orow, orow, r[j], 8 * j, n);
        const float2 up = *(const float2 *)(gt + Gates<C>::kUp + 8 * j + 2 * t);
        r[j][0] *= -up.x, r[j][1] *= -up.y, r[j][2] *= -up.x, r[j][3] *= -up.y;
      }
      state_update<kTerms, D, C>(A, gt[Gates<C>::kWhole], gt[Gates<C>::kWhole + 1], r, ks);
#pragma unroll
      for (int d = 0; d < D / 8; ++d) {
        const float4 y = hand[(C / 8 + d) * 32];
        A[d][0] += y.x, A[d][1] += y.y, A[d][2] += y.z, A[d][3] += y.w;
      }
    } else {
      if (c > first) {
        fetch_first(c - 1);
        if (c - 1 > first) fetch_second(c - 2);
      }
      cp_async_commit();
      if (c > first) {
        const char *in = second_of(c - 1);
        const T *qs = (const T *)in, *ds = (const T *)(in + Sh::kKeys);
        const float *gt = (const float *)(in + Sh::kKeys + Sh::kVals), *P = gt + Gates<C>::kFloats;
        float4 *hand = hand_of(c - 1);
        float x[C / 8][4] = {}, r[C / 8][4];
#pragma unroll
        for (int m = 0; m < C / 16; ++m) {
          values_of<Sh::kValRow>(r[2 * m], r[2 * m + 1], ds, m, e0 - x0);
          if constexpr (Rec::P::kWide == 2) {
            const LeftBf16<1> a(r[2 * m], r[2 * m + 1]);  // exact
#pragma unroll
            for (int j = 0; j <= 2 * m + 1; ++j) a.times(x[j], Rec::P::load(P, m, j));
          } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const auto a = Rec::P::template left<kSums>(r, 2 * m + i);
#pragma unroll
              for (int j = 0; j <= 2 * m + i; ++j) a.times(x[j], Rec::P::load(P, 2 * m + i, j));
            }
          }
        }
#pragma unroll
        for (int j = 0; j < C / 8; ++j) {
          hand[j * 32] = make_float4(x[j][0], x[j][1], x[j][2], x[j][3]);
          const float2 up = *(const float2 *)(gt + Gates<C>::kUp + 8 * j + 2 * t);
          const float ux = up.x * f.scale, uy = up.y * f.scale;
          r[j][0] *= ux, r[j][1] *= uy, r[j][2] *= ux, r[j][3] *= uy;
        }
        float y[D / 8][4] = {};
        state_update<kTerms, D, C>(y, 0.f, 0.f, r, qs);
#pragma unroll
        for (int d = 0; d < D / 8; ++d)
          hand[(C / 8 + d) * 32] = make_float4(y[d][0], y[d][1], y[d][2], y[d][3]);
      }
      cp_async_wait_all();
    }
  }
  if (!carry) return;
  if (kOwn) store_state<D>(own + (bh * count + s) * D * D, A, e0);
  else if (p.dstate_in && s == 0) store_state<D>(p.dstate_in + bh * D * D, A, e0);
}

// ------------------------------------------------------------- the chunks' own gradients
// One block a (chunk, head, batch), a warp for each 16 of its tokens; results in registers,
// 16 x D of dq and of dk a warp.  Products with states, u and w in three tf32 terms, or, where results
// are bf16, in two bf16 numbers a value (2^-16; in one tf32 number dq was up to 3e-3 of its norm off
// where keys are alike): B4 H8 N8192 D64 212 us, bound by shared memory (56 % of its wavefronts)
// at two blocks an SM.
template <typename T, int D>
struct GradShape {
  static constexpr int C = kChunkOf<T>, kWarps = C / 16, kThreads = kWarps * 32;
  static constexpr int kRow = pad_row<T>(D), kWide = D + 8, kMat = C + 4;
  static constexpr int kTile = C * kRow * (int)sizeof(T);
  static constexpr int kStateFloats = D * kWide > 2 * C * kMat ? D * kWide : 2 * C * kMat;
  static constexpr int kSmall = Gates<C>::kFloats + 2 * C + 2 * kWarps * C + 4 + kWarps;
  // words of packed matrices a thread fetches: of C x D and D x D, the latter at most 16 at a time
  static constexpr int kRowWords = C * D / 4 / kThreads, kStateWords = D * D / 4 / kThreads;
  static constexpr int kBatch = kStateWords < 16 ? kStateWords : 16;
  static constexpr int kBytes = 3 * kTile + (2 * C * kWide + kStateFloats + kSmall) * 4;
};

__device__ __forceinline__ float2 pair_at(const float *p) { return *(const float2 *)p; }
__device__ __forceinline__ float2 pair_at(const __nv_bfloat16 *p) { return bf2_to_f2(*(const uint32_t *)p); }

// Two bf16 numbers that stand for a value, in its place: the larger part above.
__device__ __forceinline__ void halves_of(uint32_t &a, uint32_t &b, float x, float y) {
  const uint32_t hi = f2_to_bf2(x, y);
  const float2 r = bf2_to_f2(hi);
  const uint32_t lo = f2_to_bf2(x - r.x, y - r.y);
  a = __byte_perm(lo, hi, 0x5410), b = __byte_perm(lo, hi, 0x7632);
}
// Those of a row's values at 2t, 2t + 1 and 8 further on, as operands of bf16 products: both large
// parts, both small ones.
__device__ __forceinline__ uint4 halves_at(const float *p) {
  const uint2 x = *(const uint2 *)p, y = *(const uint2 *)(p + 8);
  return make_uint4(__byte_perm(x.x, x.y, 0x7632), __byte_perm(y.x, y.y, 0x7632),
                    __byte_perm(x.x, x.y, 0x5410), __byte_perm(y.x, y.y, 0x5410));
}

// What store_packed left of a kTiles * 8 x D matrix (rows: tiles; columns: 16 by 16): words
// first, first + kThreads, ... of a thread, all in flight before the first is used, and into rows
// of D + 8 floats, or of as many pairs of bf16 numbers.
template <int kThreads, int kN>
__device__ __forceinline__ void fetch_packed(float4 (&v)[kN], const float *from, int first) {
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = __ldg((const float4 *)from + first + i * kThreads);
}
template <int D, int kTiles, bool kHalves, int kThreads, int kN>
__device__ __forceinline__ void spread(float *to, const float4 (&v)[kN], int first) {
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    const int i = first + n * kThreads, tile = i / 32, g = (i & 31) >> 2, t = i & 3;
    uint32_t x[4] = {__float_as_uint(v[n].x), __float_as_uint(v[n].y), __float_as_uint(v[n].z),
                     __float_as_uint(v[n].w)};
    if (kHalves) halves_of(x[0], x[1], v[n].x, v[n].y), halves_of(x[2], x[3], v[n].z, v[n].w);
    uint32_t *at = (uint32_t *)to + (tile % kTiles * 8 + 2 * t) * (D + 8) + tile / kTiles * 16 + g;
    at[0] = x[0], at[D + 8] = x[1], at[8] = x[2], at[D + 16] = x[3];
  }
}

// 16 rows from i on at columns k .. k + 7 of a tile, as the left operand of tf32 products; times
// the rows' factors.
template <int kRow>
__device__ __forceinline__ LeftTf32<true> left_rows(const float *tile, int i, int k, float fx = 1.f,
                                                    float fy = 1.f) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const float2 x = pair_at(tile + (i + g) * kRow + k + 2 * t);
  const float2 y = pair_at(tile + (i + g + 8) * kRow + k + 2 * t);
  const float c[4] = {fx * x.x, fx * x.y, fy * y.x, fy * y.y};
  return LeftTf32<true>(c);
}
// The same at columns k .. k + 15 for bf16 products, of fp32 rows (in two bf16 numbers), of rows
// that are pairs of them, and of bf16 rows.
template <int kRow>
__device__ __forceinline__ LeftBf16<2> left_wide(const float *tile, int i, int k, float fx = 1.f,
                                                 float fy = 1.f) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const float *p = tile + (i + g) * kRow + k + 2 * t, *q = p + 8 * kRow;
  const float2 x = pair_at(p), y = pair_at(q), u = pair_at(p + 8), v = pair_at(q + 8);
  const float c[4] = {fx * x.x, fx * x.y, fy * y.x, fy * y.y};
  const float d[4] = {fx * u.x, fx * u.y, fy * v.x, fy * v.y};
  return LeftBf16<2>(c, d);
}
template <int kRow>
__device__ __forceinline__ LeftBf16<2> left_halves(const float *tile, int i, int k) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const uint4 a = halves_at(tile + (i + g) * kRow + k + 2 * t);
  const uint4 b = halves_at(tile + (i + g + 8) * kRow + k + 2 * t);
  LeftBf16<2> l;
  l.part[0][0] = a.x, l.part[0][1] = b.x, l.part[0][2] = a.y, l.part[0][3] = b.y;
  l.part[1][0] = a.z, l.part[1][1] = b.z, l.part[1][2] = a.w, l.part[1][3] = b.w;
  return l;
}
template <int kRow>
__device__ __forceinline__ LeftBf16<1> left_exact(const __nv_bfloat16 *tile, int i, int k) {
  const int l = threadIdx.x & 31;
  LeftBf16<1> r;
  ldmatrix4(r.part[0], smem_u32(tile + (i + (l & 15)) * kRow + k + (l >> 4) * 8));
  return r;
}
// x += (16 x 16 coefficients a, b) times rows i .. i + 15 of a raw tile.
template <int D>
__device__ __forceinline__ void add_rows(float (&x)[D / 8][4], const float (&a)[4],
                                         const float (&b)[4], const __nv_bfloat16 *tile, int i) {
  const LeftBf16<2> l(a, b);
#pragma unroll
  for (int d = 0; d < D / 16; ++d) {
    const PairBf16 k = by_channel<pad_row<__nv_bfloat16>(D)>(tile, i, 16 * d);
    l.times(x[2 * d], k.b[0][0], k.b[0][1]);
    l.times(x[2 * d + 1], k.b[1][0], k.b[1][1]);
  }
}
template <int D>
__device__ __forceinline__ void add_rows(float (&x)[D / 8][4], const float (&a)[4],
                                         const float (&b)[4], const float *tile, int i) {
  constexpr int kRow = pad_row<float>(D);
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const LeftTf32<true> l0(a), l1(b);
#pragma unroll
  for (int d = 0; d < D / 8; ++d) {
    const float *at = tile + (i + 2 * t) * kRow + 8 * d + g;
    l0.times(x[d], at[0], at[kRow]);
    l1.times(x[d], at[8 * kRow], at[9 * kRow]);
  }
}
// Products of 16 rows of q and of k with rows j .. j + 15 of k.
template <int D>
__device__ __forceinline__ void score_tiles(float (&qk)[2][4], float (&kk)[2][4],
                                            const __nv_bfloat16 *qs, const __nv_bfloat16 *ks, int i,
                                            int j) {
  constexpr int kRow = pad_row<__nv_bfloat16>(D);
  const int l = threadIdx.x & 31;
#pragma unroll
  for (int d = 0; d < D / 16; ++d) {
    const auto a = left_exact<kRow>(qs, i, 16 * d), c = left_exact<kRow>(ks, i, 16 * d);
    const PairBf16 k = by_token<kRow>(ks, j, 16 * d);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      a.times(qk[n], k.b[n][0], k.b[n][1]);
      c.times(kk[n], k.b[n][0], k.b[n][1]);
    }
  }
}
template <int D>
__device__ __forceinline__ void score_tiles(float (&qk)[2][4], float (&kk)[2][4], const float *qs,
                                            const float *ks, int i, int j) {
  constexpr int kRow = pad_row<float>(D);
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll 2
  for (int d = 0; d < D / 8; ++d) {
    const auto a = left_rows<kRow>(qs, i, 8 * d), c = left_rows<kRow>(ks, i, 8 * d);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const float2 k = *(const float2 *)(ks + (j + 8 * n + g) * kRow + 8 * d + 2 * t);
      a.times(qk[n], k.x, k.y);
      c.times(kk[n], k.x, k.y);
    }
  }
}
// Sums over each of the warp's 16 rows of x times a raw tile's rows, in every lane of a row.
template <int D, typename T>
__device__ __forceinline__ void row_dots(float &top, float &bottom, const float (&x)[D / 8][4],
                                         const T *tile, int i) {
  constexpr int kRow = pad_row<T>(D);
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  top = bottom = 0.f;
#pragma unroll
  for (int d = 0; d < D / 8; ++d) {
    const float2 a = pair_at(tile + (i + g) * kRow + 8 * d + 2 * t);
    const float2 b = pair_at(tile + (i + g + 8) * kRow + 8 * d + 2 * t);
    top = fmaf(x[d][0], a.x, fmaf(x[d][1], a.y, top));
    bottom = fmaf(x[d][2], b.x, fmaf(x[d][3], b.y, bottom));
  }
#pragma unroll
  for (int m = 1; m < 4; m <<= 1) {
    top += __shfl_xor_sync(0xFFFFFFFFu, top, m);
    bottom += __shfl_xor_sync(0xFFFFFFFFu, bottom, m);
  }
}
__device__ __forceinline__ void store2(float *p, float x, float y) { *(float2 *)p = make_float2(x, y); }
__device__ __forceinline__ void store2(__nv_bfloat16 *p, float x, float y) {
  *(uint32_t *)p = f2_to_bf2(x, y);
}
__device__ __forceinline__ void store1(float *p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

// O: the type dq and dk leave in (fp32 planes where heads are shared).
template <typename T, typename O, int D>
__global__ void __launch_bounds__(GradShape<T, D>::kThreads)
    grads_kernel(const DeltaBackArgs p, const float *records, const float *states,
                 const float *misses, const float *after, const float *weights, O *dq, O *dk, int nc,
                 int stride) {
  using Sh = GradShape<T, D>;
  constexpr int C = Sh::C, kThreads = Sh::kThreads, kRow = Sh::kRow, kWide = Sh::kWide;
  constexpr int kMat = Sh::kMat, kWarps = Sh::kWarps;
  constexpr bool kHalves = sizeof(T) == 2;  // u and the states as two bf16 numbers
  extern __shared__ __align__(16) char raw[];
  T *ks = (T *)raw, *qs = (T *)(raw + Sh::kTile), *ds = (T *)(raw + 2 * Sh::kTile);
  float *us = (float *)(raw + 3 * Sh::kTile), *vs = us + C * kWide, *st = vs + C * kWide;
  float *gt = st + Sh::kStateFloats, *share = gt + Gates<C>::kFloats, *end = share + C;
  float *cols = end + C, *below = cols + kWarps * C, *dots = below + kWarps * C;
  float *dP = st, *E = st + C * kMat;  // once the states are done with
  grid_dep_wait();
  const DeltaArgs &f = p.f;
  const int h = blockIdx.y, b = blockIdx.z, hk = h / (f.H / f.Hk), tid = threadIdx.x;
  const int w = tid / 32, lane = tid & 31, g = lane >> 2, t = lane & 3, i0 = 16 * w;
  const int L = f.seq_lens ? min(max(__ldg(f.seq_lens + b), 0), f.N) : f.N;
  const int t0 = blockIdx.x * C, n = min(max(L - t0, 0), C), rows = min(f.N - t0, C);
  const size_t bt = (size_t)b * f.N + t0, row0 = bt * f.H + h;  // first token's row of a head
  const size_t orow = (size_t)f.H * D;
  dq += row0 * D, dk += row0 * D;
  T *dlog = (T *)p.dlog_decay + row0, *dbeta = (T *)p.dbeta + row0;
  // rows past the end
  for (int i = tid; i < (rows - n) * (D / 2); i += kThreads) {
    const size_t at = (size_t)(n + i / (D / 2)) * orow + i % (D / 2) * 2;
    store2(dq + at, 0.f, 0.f);
    store2(dk + at, 0.f, 0.f);
    store2((T *)p.dv + row0 * D + at, 0.f, 0.f);
  }
  for (int i = n + tid; i < rows; i += kThreads) {
    store1(dlog + (size_t)i * f.H, 0.f);
    store1(dbeta + (size_t)i * f.H, 0.f);
  }
  if (n == 0) return;
  const size_t at = ((size_t)b * f.H + h) * nc + blockIdx.x;
  const float *S0 = states + at * D * D, *A1 = after + at * D * D;
  load_rows<T, C, D, kThreads>(ks, (const T *)f.k + b * f.sk[0] + t0 * f.sk[1] + (long long)hk * D,
                               f.sk[1], n, tid);
  load_rows<T, C, D, kThreads>(qs, (const T *)f.q + b * f.sq[0] + t0 * f.sq[1] + (long long)hk * D,
                               f.sq[1], n, tid);
  load_rows<T, C, D, kThreads>(ds, (const T *)p.d_o + row0 * D, (long long)orow, n, tid);
  load_flat<Gates<C>::kFloats, kThreads>(gt, records + at * stride + Record<T, D, true>::kGates, tid);
  cp_async_commit();
  // the misses and w (as they are: dbeta is a product of both), A, and where it is small S, with
  // their inner product
  constexpr int kRW = Sh::kRowWords, kSW = Sh::kStateWords, kBatch = Sh::kBatch;
  constexpr bool kKeep = kSW <= 8;
  float4 kept[kKeep ? kSW : 1];
  float dot = 0.f;
  {
    float4 m[kRW], x[kRW], a[kBatch];
    fetch_packed<kThreads>(m, misses + at * C * D, tid);
    fetch_packed<kThreads>(x, weights + at * C * D, tid);
    if constexpr (kKeep) {
      fetch_packed<kThreads>(a, A1, tid);
      fetch_packed<kThreads>(kept, S0, tid);
    }
    spread<D, C / 8, false, kThreads>(us, m, tid);
    spread<D, C / 8, false, kThreads>(vs, x, tid);
    if constexpr (!kKeep) {
#pragma unroll 1
      for (int i = tid; i < D * D / 4; i += kBatch * kThreads) {
        fetch_packed<kThreads>(a, A1, i);
        spread<D, D / 8, kHalves, kThreads>(st, a, i);
      }
    } else {
      spread<D, D / 8, kHalves, kThreads>(st, a, tid);
#pragma unroll
      for (int i = 0; i < kSW; ++i)
        dot = fmaf(a[i].x, kept[i].x, fmaf(a[i].y, kept[i].y, fmaf(a[i].z, kept[i].z, fmaf(a[i].w, kept[i].w, dot))));
    }
  }
  cp_async_wait_all();
  __syncthreads();
  // dbeta, then u and dv in the places of the misses and w; four lanes a row
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int i = i0 + g + 8 * half;
    const float be = gt[Gates<C>::kBeta + i];
    float sum = 0.f;
#pragma unroll
    for (int d = 4 * t; d < D; d += 16) {
      float4 &m = *(float4 *)(us + i * kWide + d), &x = *(float4 *)(vs + i * kWide + d);
      const float4 a = m, c = x;
      sum = fmaf(a.x, c.x, fmaf(a.y, c.y, fmaf(a.z, c.z, fmaf(a.w, c.w, sum))));
      x = make_float4(be * c.x, be * c.y, be * c.z, be * c.w);
      if constexpr (kHalves) {
        uint4 u;
        halves_of(u.x, u.y, be * a.x, be * a.y), halves_of(u.z, u.w, be * a.z, be * a.w);
        *(uint4 *)&m = u;
      } else {
        m = make_float4(be * a.x, be * a.y, be * a.z, be * a.w);
      }
    }
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
    if (t == 0 && i < n) store1(dbeta + (size_t)i * f.H, sum);
  }
  __syncwarp();
  // products with the states.  G's shares: sums of rows of each term with the token's own vector
  const float up0 = gt[Gates<C>::kUp + i0 + g], up1 = gt[Gates<C>::kUp + i0 + g + 8];
  const float dn0 = gt[Gates<C>::kDown + i0 + g], dn1 = gt[Gates<C>::kDown + i0 + g + 8];
  float x[D / 8][4] = {}, y[D / 8][4] = {};  // dq, dk
  if constexpr (kHalves) {
#pragma unroll 2
    for (int e = 0; e < D; e += 16) {
      const auto a = left_halves<kWide>(us, i0, e);
#pragma unroll
      for (int d = 0; d < D / 8; ++d) a.times(y[d], halves_at(st + (8 * d + g) * kWide + e + 2 * t));
    }
#pragma unroll
    for (int d = 0; d < D / 8; ++d) y[d][0] *= dn0, y[d][1] *= dn0, y[d][2] *= dn1, y[d][3] *= dn1;
  } else {
#pragma unroll 2
    for (int e = 0; e < D; e += 8) {
      const auto a = left_rows<kWide>(us, i0, e, dn0, dn1);
#pragma unroll
      for (int d = 0; d < D / 8; ++d) {
        const float2 s = *(const float2 *)(st + (8 * d + g) * kWide + e + 2 * t);
        a.times(y[d], s.x, s.y);
      }
    }
  }
  float to0, to1, all0, all1, q0, q1;
  row_dots<D>(to0, to1, y, ks, i0);
  __syncthreads();
  {
    if constexpr (kKeep) {
      spread<D, D / 8, kHalves, kThreads>(st, kept, tid);
    } else {
#pragma unroll 1
      for (int i = tid; i < D * D / 4; i += kBatch * kThreads) {
        float4 a[kBatch], v[kBatch];
        fetch_packed<kThreads>(a, A1, i);
        fetch_packed<kThreads>(v, S0, i);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          dot = fmaf(a[j].x, v[j].x, fmaf(a[j].y, v[j].y, fmaf(a[j].z, v[j].z, fmaf(a[j].w, v[j].w, dot))));
        spread<D, D / 8, kHalves, kThreads>(st, v, i);
      }
    }
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, m);
    if (lane == 0) dots[w] = dot;
  }
  __syncthreads();
  const float uq0 = up0 * f.scale, uq1 = up1 * f.scale;
  if constexpr (kHalves) {
#pragma unroll 2
    for (int e = 0; e < D; e += 16) {
      const auto a = left_exact<kRow>(ds, i0, e);
      const auto c = left_wide<kWide>(vs, i0, e, -up0, -up1);
#pragma unroll
      for (int d = 0; d < D / 8; ++d) {
        const uint4 s = halves_at(st + (8 * d + g) * kWide + e + 2 * t);
        a.times(x[d], s);
        c.times(y[d], s);
      }
    }
#pragma unroll
    for (int d = 0; d < D / 8; ++d) x[d][0] *= uq0, x[d][1] *= uq0, x[d][2] *= uq1, x[d][3] *= uq1;
  } else {
#pragma unroll 2
    for (int e = 0; e < D; e += 8) {
      const auto a = left_rows<kRow>(ds, i0, e, uq0, uq1);
      const auto c = left_rows<kWide>(vs, i0, e, -up0, -up1);
#pragma unroll
      for (int d = 0; d < D / 8; ++d) {
        const float2 s = *(const float2 *)(st + (8 * d + g) * kWide + e + 2 * t);
        a.times(x[d], s.x, s.y);
        c.times(y[d], s.x, s.y);
      }
    }
  }
  row_dots<D>(q0, q1, x, qs, i0);
  row_dots<D>(all0, all1, y, ks, i0);
  if (t == 0) {
    share[i0 + g] = q0 + (all0 - to0) - to0, share[i0 + g + 8] = q1 + (all1 - to1) - to1;
    end[i0 + g] = to0, end[i0 + g + 8] = to1;
  }
  __syncthreads();  // the states are done with
  // dP and E, blocks of 16 x 16 on and below the diagonal, warp by warp
  for (int blk = w; blk < kWarps * (kWarps + 1) / 2; blk += kWarps) {
    int ib = 0;
    while ((ib + 1) * (ib + 2) / 2 <= blk) ++ib;
    const int jb = blk - ib * (ib + 1) / 2, i1 = 16 * ib, j1 = 16 * jb;
    float qk[2][4] = {}, kk[2][4] = {}, a[2][4] = {}, c[2][4] = {};
    score_tiles<D>(qk, kk, qs, ks, i1, j1);
    if constexpr (kHalves) {
#pragma unroll 2
      for (int e = 0; e < D; e += 16) {
        const auto l = left_exact<kRow>(ds, i1, e);
        const auto m = left_wide<kWide>(vs, i1, e);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint4 u = halves_at(us + (j1 + 8 * q + g) * kWide + e + 2 * t);
          l.times(a[q], u);
          m.times(c[q], u);
        }
      }
    } else {
#pragma unroll 4
      for (int e = 0; e < D; e += 8) {
        const auto l = left_rows<kRow>(ds, i1, e);
        const auto m = left_rows<kWide>(vs, i1, e);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float2 u = *(const float2 *)(us + (j1 + 8 * q + g) * kWide + e + 2 * t);
          l.times(a[q], u.x, u.y);
          m.times(c[q], u.x, u.y);
        }
      }
    }
    // powers e^(G_i - G_j); off the diagonal in two factors, by way of the block's first row
    const float hr = gt[Gates<C>::kHi + i1], lr = gt[Gates<C>::kLo + i1];
    float hi[2], lo[2], pr[2], row[2] = {};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      hi[half] = gt[Gates<C>::kHi + i1 + g + 8 * half], lo[half] = gt[Gates<C>::kLo + i1 + g + 8 * half];
      pr[half] = ex2_approx((hi[half] - hr) + (lo[half] - lr));
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int j = j1 + 8 * q + 2 * t;
      const float2 hj = *(const float2 *)(gt + Gates<C>::kHi + j), lj = *(const float2 *)(gt + Gates<C>::kLo + j);
      float pw[4], col[2] = {};
      if (ib != jb) {
        const float c0 = ex2_approx((hr - hj.x) + (lr - lj.x)), c1 = ex2_approx((hr - hj.y) + (lr - lj.y));
        pw[0] = pr[0] * c0, pw[1] = pr[0] * c1, pw[2] = pr[1] * c0, pw[3] = pr[1] * c1;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool on = i1 + g + (e >> 1) * 8 >= j + (e & 1), same = i1 + g + (e >> 1) * 8 == j + (e & 1);
          const float gap = (hi[e >> 1] - (e & 1 ? hj.y : hj.x)) + (lo[e >> 1] - (e & 1 ? lj.y : lj.x));
          pw[e] = on ? ex2_approx(gap) : 0.f;
          if (same) c[q][e] = 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[q][e] *= f.scale * pw[e];
        c[q][e] *= -pw[e];
        const float m = fmaf(a[q][e], qk[q][e], c[q][e] * kk[q][e]);
        row[e >> 1] += m;
        col[e & 1] += m;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int at2 = (i1 + g + 8 * half) * kMat + j;
        *(float2 *)(dP + at2) = make_float2(a[q][2 * half], a[q][2 * half + 1]);
        *(float2 *)(E + at2) = make_float2(c[q][2 * half], c[q][2 * half + 1]);
      }
#pragma unroll
      for (int m = 4; m < 32; m <<= 1) {
        col[0] += __shfl_xor_sync(0xFFFFFFFFu, col[0], m);
        col[1] += __shfl_xor_sync(0xFFFFFFFFu, col[1], m);
      }
      if (g == 0) *(float2 *)(cols + ib * C + j) = make_float2(col[0], col[1]);
    }
#pragma unroll
    for (int m = 1; m < 4; m <<= 1) {
      row[0] += __shfl_xor_sync(0xFFFFFFFFu, row[0], m);
      row[1] += __shfl_xor_sync(0xFFFFFFFFu, row[1], m);
    }
    if (t == 0) below[jb * C + i1 + g] = row[0], below[jb * C + i1 + g + 8] = row[1];
  }
  __syncthreads();
  // their products: the warp's rows with the tokens before, its columns with those after
#pragma unroll 1
  for (int j0 = 0; j0 <= i0; j0 += 16) {
    float a[2][4], c[2][4];
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int at2 = (i0 + g + 8 * half) * kMat + j0 + 8 * q + 2 * t;
        const float2 u = *(const float2 *)(dP + at2), v = *(const float2 *)(E + at2);
        a[q][2 * half] = u.x, a[q][2 * half + 1] = u.y, c[q][2 * half] = v.x, c[q][2 * half + 1] = v.y;
      }
    add_rows<D>(x, a[0], a[1], ks, j0);
    add_rows<D>(y, c[0], c[1], ks, j0);
  }
#pragma unroll 1
  for (int j0 = i0; j0 < C; j0 += 16) {
    float a[2][4], c[2][4];
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at2 = (j0 + 8 * q + 2 * t + (e & 1)) * kMat + i0 + g + (e >> 1) * 8;
        a[q][e] = dP[at2], c[q][e] = E[at2];
      }
    add_rows<D>(y, a[0], a[1], qs, j0);
    add_rows<D>(y, c[0], c[1], ks, j0);
  }
#pragma unroll
  for (int half = 0; half < 2; ++half)
    if (i0 + g + 8 * half < n) {
      const size_t to = (size_t)(i0 + g + 8 * half) * orow + 2 * t;
#pragma unroll
      for (int d = 0; d < D / 8; ++d) {
        store2(dq + to + 8 * d, x[d][2 * half], x[d][2 * half + 1]);
        store2(dk + to + 8 * d, y[d][2 * half], y[d][2 * half + 1]);
      }
    }
  // the log decays: sums from each token to the chunk's end
  if (tid < C) {
    float mine = share[tid];
    for (int v = 0; v <= tid / 16; ++v) mine += below[v * C + tid];
    for (int v = tid / 16; v < kWarps; ++v) mine -= cols[v * C + tid];
    double G = mine;
    // the last one has what all keys sent to the chunk's end, and the state's own share
    double sent = end[tid];
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) sent += __shfl_xor_sync(0xFFFFFFFFu, sent, m);
    double *other = (double *)cols;
    if (C > 32) {
      named_barrier(1, C);  // cols are read
      if (lane == 0) other[w] = sent;
      named_barrier(1, C);
      sent = other[0] + other[1];
    }
    if (tid == C - 1) {
      float own = dots[0];
      for (int v = 1; v < kWarps; ++v) own += dots[v];
      G += sent + (double)gt[Gates<C>::kWhole] * own;
    }
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const double o = __shfl_down_sync(0xFFFFFFFFu, G, m);
      if (lane + m < 32) G += o;
    }
    if (C > 32) {
      if (tid == 32) other[2] = G;
      named_barrier(1, C);
      if (tid < 32) G += other[2];
    }
    if (tid < n) {
      const float lg = to_f(((const T *)f.log_decay)[b * f.sg[0] + (t0 + tid) * f.sg[1] + h]);
      store1(dlog + (size_t)tid * f.H, lg == -INFINITY ? 0.f : (float)G);
    }
  }
}

// Scratch of the backward pass, in floats from one base.
struct Layout {
  size_t records, states, misses, after, weights, before, own, moves, dq, dk, total;
  Segments segments;
};
// Floats of a chunk's record.  exact: see exact_back.
template <typename T>
int record_floats(int D, bool exact) {
  if (exact) return D < 128 ? Record<T, 64, true, true>::kFloats : Record<T, 128, true, true>::kFloats;
  return D < 128 ? Record<T, 64, true>::kFloats : Record<T, 128, true>::kFloats;
}
template <typename T>
Layout layout_of(const DeltaBackArgs &p, bool exact) {
  const DeltaArgs &a = p.f;
  constexpr int C = kChunkOf<T>;
  const size_t all = (size_t)a.B * a.H * chunks_of<T>(a);
  Layout l = {};
  size_t at = 0;
  auto take = [&](size_t &to, size_t floats) { to = at, at += (floats + 63) / 64 * 64; };
  take(l.records, all * record_floats<T>(a.D, exact));
  take(l.states, all * a.D * a.D);
  take(l.after, all * a.D * a.D);
  take(l.misses, all * C * a.D);
  take(l.weights, all * C * a.D);
  l.segments = segments_of(a, true);
  for (size_t *to : {&l.before, &l.own, &l.moves}) take(*to, l.segments.floats(a));
  const size_t plane = a.H == a.Hk ? 0 : (size_t)a.B * a.N * a.H * a.D;
  take(l.dq, plane);
  take(l.dk, plane);
  l.total = at;
  return l;
}
// States and their gradients meet keys and writes in three terms where a state's gradient is a
// result.
bool exact_back(const DeltaBackArgs &p) { return p.f.dtype == GBLA_FP32 || p.dstate_in; }

template <typename T, typename O, int D>
cudaError_t grads_launch(const DeltaBackArgs &p, const Layout &l, bool exact, float *s, O *dq, O *dk,
                         cudaStream_t st) {
  using Sh = GradShape<T, D>;
  const int nc = chunks_of<T>(p.f);
  const auto kernel = grads_kernel<T, O, D>;
  cudaError_t e;
  if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes)) !=
      cudaSuccess)
    return e;
  count_launch();
  return launch_pdl(kernel, dim3(nc, p.f.H, p.f.B), dim3(Sh::kThreads), Sh::kBytes, st, p,
                    (const float *)(s + l.records), (const float *)(s + l.states),
                    (const float *)(s + l.misses), (const float *)(s + l.after),
                    (const float *)(s + l.weights), dq, dk, nc, record_floats<T>(D, exact));
}

template <typename T, int D, int kTerms>
cudaError_t back_launch(const DeltaBackArgs &p, float *s, cudaStream_t st) {
  using Sh = ReverseShape<T, D, kTerms>;
  constexpr bool kExact = kTerms == 3;
  const DeltaArgs &a = p.f;
  const Layout l = layout_of<T>(p, kExact);
  const int nc = chunks_of<T>(a);
  cudaError_t e;
  if ((e = save_forward(a, l.segments, kExact, s + l.records, s + l.states, s + l.misses,
                        s + l.before, s + l.moves, st)) != cudaSuccess)
    return e;
  const Segments &g = l.segments;
  const float *records = s + l.records;
  const dim3 grid(a.H * Sh::kSplit, a.B, g.count), block(Sh::kThreads);
  if (g.count > 1) {
    const auto own = reverse_kernel<T, D, kTerms, true>;
    if ((e = cudaFuncSetAttribute(own, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes)) !=
        cudaSuccess)
      return e;
    count_launch();
    if ((e = launch_pdl(own, grid, block, Sh::kBytes, st, p, records, (float *)nullptr,
                        (float *)nullptr, s + l.own, nc, g.chunks, g.count)) != cudaSuccess)
      return e;
    if ((e = join_back(a, g, p.dstate, s + l.own, s + l.moves, st)) != cudaSuccess) return e;
  }
  const auto reverse = reverse_kernel<T, D, kTerms, false>;
  if ((e = cudaFuncSetAttribute(reverse, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes)) !=
      cudaSuccess)
    return e;
  count_launch();
  if ((e = launch_pdl(reverse, grid, block, Sh::kBytes, st, p, records, s + l.after, s + l.weights,
                      s + l.own, nc, g.chunks, g.count)) != cudaSuccess)
    return e;
  if (a.H == a.Hk) return grads_launch<T, T, D>(p, l, kExact, s, (T *)p.dq, (T *)p.dk, st);
  float *dq = s + l.dq, *dk = s + l.dk;
  if ((e = grads_launch<T, float, D>(p, l, kExact, s, dq, dk, st)) != cudaSuccess) return e;
  return sum_shared_heads(dq, dk, p.dq, p.dk, (long long)a.B * a.N, a.Hk, a.H / a.Hk, D, a.dtype, st);
}

template <int D>
cudaError_t back_d(const DeltaBackArgs &p, float *s, cudaStream_t st) {
  if (p.f.dtype == GBLA_FP32) return back_launch<float, D, 3>(p, s, st);
  if (exact_back(p)) return back_launch<__nv_bfloat16, D, 3>(p, s, st);
  return back_launch<__nv_bfloat16, D, 2>(p, s, st);
}

}  // namespace
}  // namespace delta

size_t delta_backward_floats(const DeltaBackArgs &p) {
  using namespace delta;
  return (p.f.dtype == GBLA_FP32 ? layout_of<float>(p, true)
                                 : layout_of<__nv_bfloat16>(p, exact_back(p))).total;
}

cudaError_t delta_backward(const DeltaBackArgs &p, float *scratch, cudaStream_t st) {
  if (p.f.D == 32) return delta::back_d<32>(p, scratch, st);
  if (p.f.D == 64) return delta::back_d<64>(p, scratch, st);
  return delta::back_d<128>(p, scratch, st);
}

}  // namespace gbla
