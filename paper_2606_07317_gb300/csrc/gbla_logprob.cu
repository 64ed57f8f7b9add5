// Log probabilities of given tokens, entropy and top alternatives of rows of logits,
// and their gradients.
//
// With y = scale x, one pass over a row keeps the running maximum m of x and, in powers
// of two of t = (x - m) scale log2 e,
//   z = sum 2^t,  w = sum 2^t t;
// when t moves by delta, z becomes 2^delta z and w becomes 2^delta (w + delta z).  Then
//   lse = scale m + ln z,  entropy = ln z - ln 2 w / z,
//   log p(token) = scale (x_token - m) - ln z.
// Ruled-out logits (-inf) weigh 0; a row of nothing else has lse = -inf and entropy 0.
#include <cooperative_groups.h>
#include <math.h>

#include "gbla_internal.cuh"
#include "gbla_sm100.cuh"

namespace gbla {
namespace {

using namespace sm100;
namespace cg = cooperative_groups;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void unpack(const uint4 &v, float (&f)[4]) {
  f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y);
  f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack(const uint4 &v, float (&f)[8]) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = bf2_to_f2(u[i]);
    f[2 * i] = p.x, f[2 * i + 1] = p.y;
  }
}
__device__ __forceinline__ uint4 pack(const float (&f)[4]) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                    __float_as_uint(f[3]));
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
  return make_uint4(f2_to_bf2(f[0], f[1]), f2_to_bf2(f[2], f[3]), f2_to_bf2(f[4], f[5]),
                    f2_to_bf2(f[6], f[7]));
}
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
// Maximum that keeps a NaN (fmaxf drops it).
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A row as scalars up to the first 16-byte boundary, vectors of 16 bytes, scalars behind
// the last whole one: nothing outside the row is read, whatever its length and place.
template <typename T>
struct Row {
  static constexpr int kVec = 16 / sizeof(T);
  const T *p;
  int head, vecs, V;
  __device__ __forceinline__ Row(const T *at, int n) : p(at), V(n) {
    head = (int)((0u - (uint32_t)(uintptr_t)at) % 16u / sizeof(T));
    if (head > V) head = V;
    vecs = (V - head) / kVec;
  }
  __device__ __forceinline__ const uint4 *vec(int i) const { return (const uint4 *)(p + head) + i; }
  __device__ __forceinline__ int loose() const { return V - vecs * kVec; }  // scalars
  // place of scalar j: those of the head, then those behind the vectors
  __device__ __forceinline__ int place(int j) const { return j < head ? j : j + vecs * kVec; }
};

struct Sums {
  float m, z, w;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// c: scale log2 e.
__device__ __forceinline__ Sums joined(const Sums &a, const Sums &b, float c) {
  Sums r;
  r.m = max_nan(a.m, b.m);
  const float base = base_of(r.m);
  // an empty side has z = w = 0: any finite distance does
  const float da = fmaxf((a.m - base) * c, -1e4f), db = fmaxf((b.m - base) * c, -1e4f);
  const float ea = exp2f(da), eb = exp2f(db);
  r.z = __fadd_rn(__fmul_rn(a.z, ea), __fmul_rn(b.z, eb));
  r.w = __fadd_rn(__fmul_rn(fmaf(da, a.z, a.w), ea), __fmul_rn(fmaf(db, b.z, b.w), eb));
  return r;
}

// The sums of all 32 lanes of a warp, or of the first kLanes where each kLanes hold the same ones:
// moved to their common maximum first, added then.
__device__ __forceinline__ float lanes_max(float m) {
  float r;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(m));
  return r;
}
template <int kLanes>
__device__ __forceinline__ Sums joined_lanes(Sums s, float c) {
  const float m = lanes_max(s.m), d = fmaxf((s.m - base_of(m)) * c, -1e4f), e = exp2f(d);
  // products rounded by themselves: a sum is the same from both its sides
  s.w = __fmul_rn(fmaf(d, s.z, s.w), e), s.z = __fmul_rn(s.z, e), s.m = m;
#pragma unroll
  for (int i = kLanes / 2; i > 0; i >>= 1) {
    s.z += __shfl_xor_sync(0xFFFFFFFFu, s.z, i);
    s.w += __shfl_xor_sync(0xFFFFFFFFu, s.w, i);
  }
  return s;
}

// Order of candidates: larger logits first, equal ones by their tokens (lowest first).
// NaN counts as below -inf.  0 stands for none.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 1u;
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  if (o == 1u) return NAN;
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
__device__ __forceinline__ uint64_t key_of(uint32_t order, uint32_t index) {
  return ((uint64_t)order << 32) | (uint32_t)~index;
}

// done(key, rank) for each of n different keys in shared memory (0 is none of them): how many are
// larger.  A thread ranks kEach at a time.
template <int kThreads, int kEach, typename F>
__device__ __forceinline__ void ranked(const uint64_t *keys, int n, F done) {
  for (int i0 = threadIdx.x; i0 < n; i0 += kThreads * kEach) {
    uint64_t mine[kEach];
    int rank[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      mine[u] = i0 + u * kThreads < n ? keys[i0 + u * kThreads] : 0;
      rank[u] = 0;
    }
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
      const uint64_t k = keys[j];
#pragma unroll
      for (int u = 0; u < kEach; ++u) rank[u] += k > mine[u];
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u)
      if (mine[u]) done(mine[u], rank[u]);
  }
}

// What the blocks of a cluster that share a row tell one another.
template <int kThreads>
struct Shared {
  static constexpr int kCandidates = kThreads == 32 ? 640 : 1280;
  Sums part[kThreads / 32];
  Sums whole;                    // of this block
  int count, strips;             // candidates, threads whose logits may hold some
  uint64_t bound;
  uint64_t key[128];
  int strip[kThreads];
  uint64_t most[kThreads];
  uint64_t cand[kCandidates];
  uint64_t best[GBLA_MAX_TOP];   // this block's, in order
};

// Maximum of a vector that keeps a NaN.
__device__ __forceinline__ float max_of(const uint4 &v, float) {
  float f[4];
  unpack(v, f);
  return max_nan(max_nan(f[0], f[1]), max_nan(f[2], f[3]));
}
__device__ __forceinline__ float max_of(const uint4 &v, __nv_bfloat16) {
  uint32_t a, b, c;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
  const float2 f = bf2_to_f2(c);
  return max_nan(f.x, f.y);
}

// Two floats side by side.
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 halves(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// z += 2^t, w += 2^t t with t = (x - base) c, of the values of a vector.  kLifted: bf16 values
// below -2^100 are taken as that first, two in an instruction, for t to be finite (-inf would
// make 0 times infinity of its share of w); else t itself is kept above -1e4.  With a base within
// 2^99 of 0 and c between 2^-60 and 2^20, |t| is below 2^121, and both weigh such values 0.
template <bool kLifted, typename T>
__device__ __forceinline__ void weigh(uint64_t &z, uint64_t &w, uint4 v, uint64_t base, uint64_t c,
                                      T) {
  constexpr int kVec = Row<T>::kVec;
  if (kLifted && sizeof(T) == 2) {
    constexpr uint32_t kLow = 0xF180F180u;  // -2^100 twice
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.x) : "r"(kLow));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.y) : "r"(kLow));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.z) : "r"(kLow));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.w) : "r"(kLow));
  }
  float x[kVec];
  unpack(v, x);
#pragma unroll
  for (int i = 0; i < kVec; i += 2) {
    uint64_t t = mul2(add2(pair_of(x[i], x[i + 1]), base), c);
    float2 f = halves(t);
    if (!(kLifted && sizeof(T) == 2)) {
      f.x = max_nan(f.x, -1e4f), f.y = max_nan(f.y, -1e4f);
      t = pair_of(f.x, f.y);
    }
    const uint64_t e = pair_of(ex2_approx(f.x), ex2_approx(f.y));
    z = add2(z, e), w = fma2(e, t, w);
  }
}

// One row by kThreads threads of each of `split` blocks.  A thread takes kBatch vectors at a
// time: their loads are in flight together, their maximum moves the sums once.  Bound by the
// logits' bytes, beside issue slots (packed arithmetic: 6 or 7 a bf16 logit, 12 without) and one
// exponential a logit.
//
// Top alternatives: the K-th largest of at least 2 K maxima of groups of vectors bounds the
// K-th logit from below, and only the logits of threads that reach it are looked at again, by all
// threads: a little over K candidates, whose ranks are counted (2048 rows of 8191 fp32, K = 32:
// 27 us; 35 where each such thread looks at its own and lanes' sums are joined in pairs).  The rule
// for a row's threads does not ask for K: the other results are the same to the bit without.
template <typename T, int kThreads, bool kTop>
__global__ void __launch_bounds__(kThreads) logprob_kernel(const LogprobArgs p, int split) {
  constexpr int kVec = Row<T>::kVec, kBatch = 4, kWarps = kThreads / 32;
  constexpr int kMaxima = kThreads == 32 ? kBatch : 1;  // of a thread
  using Sh = Shared<kThreads>;
  __shared__ Sh sm;
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid % 32, part = split > 1 ? (int)cluster.block_rank() : 0;
  const float c = p.scale * kLog2e;
  const bool lift = c > 0x1p-60f && c < 0x1p20f;
  const int rows = p.B * p.N, step = gridDim.x / split;
  grid_dep_wait();
  grid_dep_launch();
  for (int r = blockIdx.x / split; r < rows; r += step) {
    const int b = r / p.N, t = r % p.N;
    if (p.seq_lens && t >= __ldg(p.seq_lens + b)) continue;  // the whole cluster skips it
    const Row<T> row((const T *)p.logits + b * p.s[0] + t * p.s[1], p.V);
    const int per = (row.vecs + split - 1) / split, v0 = min(part * per, row.vecs),
              v1 = min(v0 + per, row.vecs);
    const bool last = part == split - 1;
    Sums s = {-INFINITY, 0.f, 0.f};
    float tmax[kMaxima];  // of the vectors, the first of them that has it
    int most[kMaxima];
#pragma unroll
    for (int j = 0; j < kMaxima; ++j) tmax[j] = NAN, most[j] = -1;
    auto move = [&](float m) {  // the sums' base to a larger maximum
      if (!(m <= s.m)) {
        const float base = base_of(max_nan(m, s.m)), d = fmaxf((s.m - base) * c, -1e4f), e = exp2f(d);
        s.w = __fmul_rn(fmaf(d, s.z, s.w), e), s.z = __fmul_rn(s.z, e), s.m = max_nan(m, s.m);
      }
    };
    uint4 v[kBatch], ahead[kBatch];
    auto fetch = [&](uint4 (&to)[kBatch], int i0) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (i0 + u * kThreads < v1) to[u] = __ldg(row.vec(i0 + u * kThreads));
    };
    const uint64_t c2 = pair_of(c, c);
    auto take = [&](int i0, int n) {  // v's first n vectors
      float m[kBatch], all = -INFINITY;
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (u < n) {
          m[u] = max_of(v[u], T());
          all = max_nan(all, m[u]);
          if (kTop && !(m[u] <= tmax[u % kMaxima]))
            tmax[u % kMaxima] = m[u], most[u % kMaxima] = i0 + u * kThreads;
        }
      move(all);
      const float base = base_of(s.m);
      uint64_t z = 0, w = 0;
      const uint64_t base2 = pair_of(-base, -base);
      if (lift && fabsf(base) < 0x1p99f) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (u < n) weigh<true>(z, w, v[u], base2, c2, T());
      } else {
#pragma unroll 1
        for (int u = 0; u < n; ++u) {
          weigh<false>(z, w, v[0], base2, c2, T());
#pragma unroll
          for (int q = 0; q + 1 < kBatch; ++q) v[q] = v[q + 1];
        }
      }
      const float2 zs = halves(z), ws = halves(w);
      s.z += zs.x + zs.y, s.w += ws.x + ws.y;
    };
    int i0 = v0 + tid;
    fetch(v, i0);
    for (; i0 + (kBatch - 1) * kThreads < v1; i0 += kBatch * kThreads) {
      fetch(ahead, i0 + kBatch * kThreads);
      take(i0, kBatch);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) v[u] = ahead[u];
    }
    if (i0 < v1) take(i0, (v1 - i0 + kThreads - 1) / kThreads);
    uint64_t own[kMaxima], key = 0;
#pragma unroll
    for (int j = 0; j < kMaxima; ++j)
      own[j] = kTop && most[j] >= 0
                   ? key_of(order_of(tmax[j]), most[j] * kVec + row.head + kVec - 1)
                   : 0;
    if (last)
      for (int j = tid; j < row.loose(); j += kThreads) {
        const int at = row.place(j);
        const float x = to_f(row.p[at]);
        move(x);
        const float d = max_nan((x - base_of(s.m)) * c, -1e4f), e = ex2_approx(d);
        s.z += e, s.w = fmaf(e, d, s.w);
        if (kTop) {
          const uint64_t k = key_of(order_of(x), at);
          if (k > own[0]) own[0] = k;
        }
      }
    const int token = p.tokens ? __ldg(p.tokens + r) : -1;
    float given = 0.f;  // its logit, on the way early
    if (tid == 0 && part == 0 && token >= 0 && token < p.V) given = to_f(row.p[token]);
    // a NaN hides what else its vector and, before it, its thread hold: they are looked over
    const bool hidden = kTop && s.m != s.m;
    s = joined_lanes<32>(s, c);
#pragma unroll
    for (int j = 0; j < kMaxima; ++j) key = own[j] > key ? own[j] : key;
    // groups of threads, or a warp's threads' maxima: 32, 64 or 128, at least twice K
    const int lg = p.K <= 16 ? 5 : p.K <= 32 ? 6 : 7;
    const int width = kThreads >> lg;  // threads of a group
    uint64_t top = key;
    if (kTop)
      for (int m = 1; m < width; m <<= 1) {
        const uint64_t o = __shfl_xor_sync(0xFFFFFFFFu, top, m);
        if (o > top) top = o;
      }
    __syncthreads();  // the row before is done with
    if (lane == 0) sm.part[tid / 32] = s;
    if (kTop && kMaxima > 1 && lg > 5) {
#pragma unroll
      for (int j = 0; j < kMaxima; j += 2) {
        const uint64_t a = own[j], b = own[(j + 1) % kMaxima];
        if (lg == 6)
          sm.key[tid * 2 + j / 2] = a > b ? a : b;
        else
          sm.key[tid * 4 + j] = a, sm.key[tid * 4 + j + 1] = b;
      }
    } else if (kTop && tid % width == 0) {
      sm.key[tid / width] = top;
    }
    if (tid == 0) sm.count = 0, sm.strips = 0, sm.bound = 0;
    __syncthreads();
    if (kWarps > 1) s = joined_lanes<kWarps>(sm.part[lane % kWarps], c);
    if (kTop) {
      ranked<kThreads, kMaxima>(sm.key, 1 << lg, [&](uint64_t k, int rank) {
        if (rank == p.K - 1) sm.bound = k;
      });
      __syncthreads();
      const uint64_t bound = sm.bound;
      if ((key >= bound && key) || hidden) {
        sm.strip[atomicAdd(&sm.strips, 1)] = tid;
        if (last)
          for (int j = tid; j < row.loose(); j += kThreads) {
            const uint64_t k = key_of(order_of(to_f(row.p[row.place(j)])), row.place(j));
            if (k < bound) continue;
            const int at = atomicAdd(&sm.count, 1);
            if (at < Sh::kCandidates) sm.cand[at] = k;
          }
      }
      __syncthreads();
      const int strips = sm.strips, each = (v1 - v0 + kThreads - 1) / kThreads;
      const int shift = each > 16 ? 5 : each > 8 ? 4 : each > 4 ? 3 : 2, across = kThreads >> shift;
      const bool every = (uint32_t)(bound >> 32) <= 1u;  // no bound, or that of a NaN
      const float least = every ? -INFINITY : value_of((uint32_t)(bound >> 32));
      const int until = (int)~(uint32_t)bound;
      for (int k = tid & ((1 << shift) - 1); k < each; k += 1 << shift)
        for (int e0 = tid >> shift; e0 < strips; e0 += kBatch * across) {
          int at[kBatch];
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            at[u] = e0 + u * across < strips ? v0 + sm.strip[e0 + u * across] + k * kThreads : v1;
            if (at[u] < v1) v[u] = __ldg(row.vec(at[u]));
          }
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            if (at[u] >= v1 || (!every && max_of(v[u], T()) < least)) continue;
            float x[kVec];
            unpack(v[u], x);
            uint32_t hits = 0;  // above the bound, or like it and not behind it
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              if (every || x[e] > least || (x[e] == least && at[u] * kVec + row.head + e <= until))
                hits |= 1u << e;
            int to = hits ? atomicAdd(&sm.count, __popc(hits)) : 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              if (hits >> e & 1) {
                if (to < Sh::kCandidates)
                  sm.cand[to] = key_of(order_of(x[e]), at[u] * kVec + row.head + e);
                ++to;
              }
          }
        }
      __syncthreads();
      const int n = sm.count;
      if (n <= Sh::kCandidates) {
        ranked<kThreads, kMaxima>(sm.cand, n, [&](uint64_t k, int rank) {
          if (rank < p.K) sm.best[rank] = k;
        });
        for (int i = n + tid; i < p.K; i += kThreads) sm.best[i] = 0;
      } else {  // too many (one thread's logits the largest): the best below the one before, K times
        uint64_t before = ~0ull;
        for (int round = 0; round < p.K; ++round) {
          uint64_t mine = 0;
          auto look = [&](uint64_t k) {
            if (k < before && k > mine) mine = k;
          };
          for (int i = v0 + tid; i < v1; i += kThreads) {
            float x[kVec];
            unpack(__ldg(row.vec(i)), x);
#pragma unroll
            for (int e = 0; e < kVec; ++e) look(key_of(order_of(x[e]), i * kVec + row.head + e));
          }
          if (last)
            for (int j = tid; j < row.loose(); j += kThreads)
              look(key_of(order_of(to_f(row.p[row.place(j)])), row.place(j)));
          __syncthreads();
          sm.most[tid] = mine;
          __syncthreads();
          for (int i = 0; i < kThreads; ++i) mine = sm.most[i] > mine ? sm.most[i] : mine;
          if (tid == 0) sm.best[round] = mine;
          before = mine;
        }
      }
      __syncthreads();
    }
    if (split > 1) {
      if (tid == 0) sm.whole = s;
      cluster.sync();
      if (part == 0) {
        for (int i = 1; i < split; ++i) s = joined(s, cluster.map_shared_rank(&sm, i)->whole, c);
        if (kTop) {
          const int n = split * p.K;
          for (int i = tid; i < n; i += kThreads)
            sm.cand[i] = cluster.map_shared_rank(&sm, i / p.K)->best[i % p.K];
          __syncthreads();
          ranked<kThreads, 1>(sm.cand, n, [&](uint64_t k, int rank) {
            if (rank < p.K) sm.best[rank] = k;
          });
          __syncthreads();
        }
      }
    }
    if (part == 0 && tid < (kTop ? p.K : 1)) {
      const bool bad = s.m != s.m || s.m == INFINITY;
      const float lnz = logf(s.z);
      const float lse = bad ? NAN : s.z > 0.f ? fmaf(s.m, p.scale, lnz) : -INFINITY;
      auto logp = [&](float x) {  // (half the distance: the whole one may pass fp32's range)
        return bad              ? NAN
               : x == -INFINITY ? -INFINITY
                                : fmaf(0.5f * x - 0.5f * s.m, 2.f * p.scale, -lnz);
      };
      if (tid == 0) {
        p.lse[r] = lse;
        p.entropy[r] = bad ? NAN : s.z > 0.f ? fmaf(-kLn2, s.w / s.z, lnz) : 0.f;
        if (p.logprob) p.logprob[r] = token >= 0 && token < p.V ? logp(given) : 0.f;
      }
      if (kTop)
        for (int i = tid; i < p.K; i += kThreads) {
          const uint64_t k = sm.best[i];
          p.top_token[(size_t)r * p.K + i] = (int)~(uint32_t)k;
          p.top_logprob[(size_t)r * p.K + i] = logp(value_of((uint32_t)(k >> 32)));
        }
    }
    if (split > 1) cluster.sync();  // the other parts' results are read
  }
}

// d x = scale [ p (dlse - dlogprob - dentropy (ln p + entropy)) + (dlogprob at the token) ],
// a tile of a row at a time: bound by the bytes of logits and gradient.  A thread holds kVecs
// vectors, all on their way before the first is used: 8192 rows of 32768 in bf16 165 us (96 % of
// the measured copy rate), 178 with 4 and 226 with 2.  Short rows take a warp each.
template <typename T, int kBackThreads, int kBackVecs>
__global__ void __launch_bounds__(kBackThreads) logprob_backward_kernel(const LogprobArgs p,
                                                                         int tiles) {
  constexpr int kVec = Row<T>::kVec;
  grid_dep_wait();
  grid_dep_launch();
  const int tid = threadIdx.x;
  const long long all = (long long)p.B * p.N * tiles;
  for (long long w = blockIdx.x; w < all; w += gridDim.x) {
    const int r = (int)(w / tiles), tile = (int)(w % tiles), b = r / p.N, t = r % p.N;
    T *out = (T *)p.dlogits + (size_t)r * p.V;
    const Row<T> row(out, p.V);  // cut by the gradient's place
    const T *in = (const T *)p.logits + b * p.s[0] + t * p.s[1];
    const bool whole = ((uintptr_t)(in + row.head) & 15) == 0;
    float lse = 0.f, ent = 0.f, A = 0.f, dh = 0.f, dlp = 0.f;
    int token = -1;
    const bool valid = !p.seq_lens || t < __ldg(p.seq_lens + b);
    if (valid) {
      lse = p.lse[r], ent = p.entropy[r];
      token = p.tokens ? __ldg(p.tokens + r) : -1;
      if (token < 0 || token >= p.V) token = -1;
      if (p.dlogprob && token >= 0) dlp = p.dlogprob[r];
      if (p.dentropy) dh = p.dentropy[r];
      if (dh == 0.f) ent = 0.f;  // not asked for: whatever it is has no share
      A = (p.dlse ? p.dlse[r] : 0.f) - dlp;
    }
    // padding, or a row of nothing but masks (also such of a type's lowest value, whose
    // lse cannot tell one token from many)
    const bool none = !valid || lse < -1e30f;
    auto grad = [&](float lp, int at) {
      float d = ex2_approx(lp * kLog2e) * fmaf(-dh, lp + ent, A);
      if (at == token) d += dlp;
      return none ? 0.f : d * p.scale;
    };
    auto log_of = [&](float x) { return max_nan(fmaf(x, p.scale, -lse), -1e4f); };
    // A far lse has been rounded by more than 2^-11, and an exact product next to it would be off
    // by as much (an infinity where logits are 1e36): the product rounded in the same way is not.
    // Where both are infinite, the row's largest logits share its probability, exp(-entropy) each.
    // A loop of its own, so that near rows keep their registers (165 us, 181 with a choice an
    // element; rows that are all far 225).
    const int v0 = tile * kBackThreads * kBackVecs + tid;
    auto fetch = [&](int i) {
      if (whole) return *((const uint4 *)(in + row.head) + i);
      float f[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) f[e] = to_f(in[row.head + i * kVec + e]);
      return pack(f);
    };
    if (!none && fabsf(lse) >= 0x1p14f) {
      const float most = -p.entropy[r];
      auto far = [&](float x, int at) {
        const float y = __fmul_rn(x, p.scale);
        return grad(y == INFINITY ? most : max_nan(__fsub_rn(y, lse), -1e4f), at);
      };
#pragma unroll 1
      for (int j = 0; j < kBackVecs; ++j) {
        const int i = v0 + j * kBackThreads;
        if (i >= row.vecs) break;
        float f[kVec];
        unpack(fetch(i), f);
#pragma unroll
        for (int e = 0; e < kVec; ++e) f[e] = far(f[e], row.head + i * kVec + e);
        *((uint4 *)(out + row.head) + i) = pack(f);
      }
      if (tile == 0 && tid < row.loose()) {
        const int at = row.place(tid);
        store1(out + at, far(to_f(in[at]), at));
      }
      continue;
    }
    uint4 v[kBackVecs];
#pragma unroll
    for (int j = 0; j < kBackVecs; ++j) {
      const int i = v0 + j * kBackThreads;
      if (i < row.vecs && !none) v[j] = fetch(i);
    }
#pragma unroll
    for (int j = 0; j < kBackVecs; ++j) {
      const int i = v0 + j * kBackThreads;
      if (i >= row.vecs) continue;
      float f[kVec];
      if (none) v[j] = make_uint4(0, 0, 0, 0);
      unpack(v[j], f);
#pragma unroll
      for (int e = 0; e < kVec; ++e) f[e] = grad(log_of(f[e]), row.head + i * kVec + e);
      *((uint4 *)(out + row.head) + i) = pack(f);
    }
    if (tile == 0 && tid < row.loose()) {
      const int at = row.place(tid);
      store1(out + at, none ? 0.f : grad(log_of(to_f(in[at])), at));
    }
  }
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
    return 152;
  return n;
}

template <typename T, int kThreads, bool kTop>
cudaError_t forward_launch(const LogprobArgs &a, int split, int blocks, cudaStream_t st) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = split, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks * split);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  count_launch();
  return cudaLaunchKernelEx(&cfg, logprob_kernel<T, kThreads, kTop>, a, split);
}

template <typename T>
cudaError_t forward_t(const LogprobArgs &a, cudaStream_t st) {
  const long long rows = (long long)a.B * a.N;
  const int sms = sm_count();
  const int vecs = a.V / Row<T>::kVec;
  // few rows: several blocks share one, while each still has some vectors a thread
  int split = 1;
  while (split < 8 && rows * split * 2 <= sms * 4 && vecs / (split * 2) >= 256) split *= 2;
  long long blocks = 8ll * sms / split;
  if (blocks > rows) blocks = rows;
  // a warp a row where that leaves each lane a few vectors
  if (split == 1 && a.V <= 1024) {
    blocks = 24ll * sms;
    if (blocks > rows) blocks = rows;
    if (a.K > 0) return forward_launch<T, 32, true>(a, 1, (int)blocks, st);
    return forward_launch<T, 32, false>(a, 1, (int)blocks, st);
  }
  // and half the threads for all but the longest rows: what a row costs beside its logits it costs
  // each warp (V = 50021 bf16: 136 us, 148 with 256 threads; V = 8191 fp32, 32 of them: 27 and 31)
  if (split == 1 && vecs <= 16384) {
    blocks = 8ll * sms;
    if (blocks > rows) blocks = rows;
    if (a.K > 0) return forward_launch<T, 128, true>(a, 1, (int)blocks, st);
    return forward_launch<T, 128, false>(a, 1, (int)blocks, st);
  }
  if (a.K > 0) return forward_launch<T, 256, true>(a, split, (int)blocks, st);
  return forward_launch<T, 256, false>(a, split, (int)blocks, st);
}

template <typename T, int kThreads, int kVecs>
cudaError_t backward_launch(const LogprobArgs &a, cudaStream_t st) {
  const int vecs = a.V / Row<T>::kVec, each = kThreads * kVecs;
  const int tiles = vecs < each ? 1 : (vecs + each - 1) / each;
  const long long all = (long long)a.B * a.N * tiles;
  long long blocks = (kThreads == 32 ? 32ll : 16ll) * sm_count();
  if (blocks > all) blocks = all;
  count_launch();
  return launch_pdl(logprob_backward_kernel<T, kThreads, kVecs>, dim3((unsigned)blocks),
                    dim3(kThreads), 0, st, a, tiles);
}

template <typename T>
cudaError_t backward_t(const LogprobArgs &a, cudaStream_t st) {
  const int vecs = a.V / Row<T>::kVec;
  if (vecs <= 128) return backward_launch<T, 32, 4>(a, st);
  if (vecs <= 1024) return backward_launch<T, 256, 4>(a, st);
  return backward_launch<T, 256, 8>(a, st);
}

}  // namespace

cudaError_t logprob_forward(const LogprobArgs &a, cudaStream_t st) {
  return a.dtype == GBLA_FP32 ? forward_t<float>(a, st) : forward_t<__nv_bfloat16>(a, st);
}

cudaError_t logprob_backward(const LogprobArgs &a, cudaStream_t st) {
  return a.dtype == GBLA_FP32 ? backward_t<float>(a, st) : backward_t<__nv_bfloat16>(a, st);
}

}  // namespace gbla
