// Norm of each query and key head with the position rotation in the same pass,
// forward and backward.  Per token and head x[D] with the head's weight w:
//   r = 1 / sqrt(mean(x^2) + eps),  y = x r w,
// then every pair (a, b) of the first R values turns by its position's angle,
//   (a, b) -> (a cos - b sin, a sin + b cos);
// backward, with g = the incoming gradient turned by the opposite angles and
// n = x r:  dw = sum g n,  u = g w,  dx = r (u - n mean(u n)).
//
// About 5 flops a byte: bound by memory.  A head vector is spread over D / 8
// lanes of 8 values (one 16-byte copy in bf16), so a warp holds 256 / D heads
// at once, the mean is a butterfly over those lanes, and the half-split pairs
// (i, i + R / 2) meet by one shuffle per value.  A warp keeps its kU groups of
// heads while it walks over the tokens: their weights stay in registers, and a
// token's row of cosines and sines is read once for all of them.  The tokens to
// come are on their way into shared memory meanwhile (loads into registers left
// memory idle while a token was computed: 69 us where it is 45 now).  Measured at
// B2 H8 N32768 D64 bf16: forward 45 us, 6.2 TB/s (91 % of the measured copy rate);
// backward at B4 N8192: 39 us, 5.2 TB/s (77 %, two kernels).
#include "gbla_internal.cuh"
#include "gbla_sm100.cuh"

namespace gbla {
namespace {

using namespace sm100;

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kBlocks = 2;  // resident blocks an SM
constexpr int kBwdU = 2;    // groups of heads a warp of the backward keeps

// 8 consecutive values of a head: as loaded, and as four pairs in fp32 (the
// packed fp32 instructions halve what this kernel has to issue).
template <typename T>
struct Pack8;
template <>
struct Pack8<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void load(uint32_t at) { u = lds_v4(at); }
  __device__ __forceinline__ void get(float2 (&f)[4]) const {
    f[0] = bf2_to_f2(u.x), f[1] = bf2_to_f2(u.y), f[2] = bf2_to_f2(u.z), f[3] = bf2_to_f2(u.w);
  }
  __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float2 (&f)[4]) {
    *(uint4 *)p = make_uint4(f2_to_bf2(f[0].x, f[0].y), f2_to_bf2(f[1].x, f[1].y),
                             f2_to_bf2(f[2].x, f[2].y), f2_to_bf2(f[3].x, f[3].y));
  }
};
template <>
struct Pack8<float> {
  uint4 a, b;
  __device__ __forceinline__ void load(uint32_t at) {
    a = lds_v4(at);
    b = lds_v4(at + 512);
  }
  __device__ __forceinline__ void get(float2 (&f)[4]) const {
    f[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
    f[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
    f[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
    f[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
  }
  __device__ __forceinline__ static void store(float *p, const float2 (&f)[4]) {
    *(float4 *)p = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    *(float4 *)(p + 4) = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
  }
};

__device__ __forceinline__ void load_f8(const float *p, float2 (&f)[4]) {
  const float4 a = __ldg((const float4 *)p), b = __ldg((const float4 *)p + 1);
  f[0] = make_float2(a.x, a.y), f[1] = make_float2(a.z, a.w);
  f[2] = make_float2(b.x, b.y), f[3] = make_float2(b.z, b.w);
}
__device__ __forceinline__ void load_s8(uint32_t at, float2 (&f)[4]) {
  const uint4 a = lds_v4(at), b = lds_v4(at + 16);
  f[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
  f[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
  f[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
  f[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
// 1 / sqrt(v) within 2^-22 (v a mean of squares plus eps, which may be subnormal: a zero
// head times an infinity would be NaN)
__device__ __forceinline__ float rsqrt_approx(float v) {
  float r;
  asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// The lane's cosines and sines of one token.  Half-split pairs: value e of the
// first half turns with partner e + R/2, so out = y cos + y_partner sin with
// the sine negated in the first half.  Neighbouring pairs (2i, 2i + 1): four
// cosines and four sines.  Lanes past R get cos = 1, sin = 0.  kDir = -1 turns
// by the opposite angles.
template <bool kNext, int kDir>
struct Turn {
  float2 c[kNext ? 2 : 4], s[kNext ? 2 : 4];
  __device__ __forceinline__ void load(uint32_t row, int e0, int R) {
    constexpr int n = kNext ? 2 : 4;
    if (e0 >= R) {
#pragma unroll
      for (int i = 0; i < n; ++i) c[i] = both(1.f), s[i] = both(0.f);
      return;
    }
    if constexpr (kNext) {
      const uint4 a = lds_v4(row + 2 * e0), b = lds_v4(row + 2 * R + 2 * e0);
      c[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
      c[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
      const float2 d = both((float)kDir);
      s[0] = __fmul2_rn(d, make_float2(__uint_as_float(b.x), __uint_as_float(b.y)));
      s[1] = __fmul2_rn(d, make_float2(__uint_as_float(b.z), __uint_as_float(b.w)));
    } else {
      const int half = R / 2, i0 = e0 < half ? e0 : e0 - half;
      load_s8(row + 4 * i0, c);
      load_s8(row + 4 * (half + i0), s);
      const float sign = e0 < half ? -(float)kDir : (float)kDir;
#pragma unroll
      for (int i = 0; i < n; ++i) s[i] = __fmul2_rn(s[i], both(sign));
    }
  }
  __device__ __forceinline__ void apply(float2 (&y)[4], int partner) const {
    if constexpr (kNext) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float cc = i & 1 ? c[i / 2].y : c[i / 2].x, ss = i & 1 ? s[i / 2].y : s[i / 2].x;
        const float2 t = __fmul2_rn(make_float2(-y[i].y, y[i].x), both(ss));
        y[i] = __ffma2_rn(y[i], both(cc), t);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 o = make_float2(__shfl_sync(0xffffffffu, y[i].x, partner),
                                     __shfl_sync(0xffffffffu, y[i].y, partner));
        y[i] = __ffma2_rn(y[i], c[i], __fmul2_rn(o, s[i]));
      }
    }
  }
};

template <int kLanes>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int m = kLanes / 2; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}

struct RotParams {
  const void *q, *k, *dqo, *dko;
  const float *wq, *wk, *rot;
  const int32_t *positions, *seq_lens;
  void *qo, *ko;  // forward: the results; backward: dq, dk
  float *part;    // backward: [slabs][(H + Hk) * D] partial sums of dw
  long long sqb, sqt, skb, skt;  // element strides of q and k (batch, token)
  long long tokens;              // B * N
  int N, H, Hk, R, P;
  float eps;
};

// Walks over tokens first, first + step, ... as (b, t) without a division each.
struct Walk {
  long long tok, step, b, db;
  int t, dt, N;
  __device__ __forceinline__ Walk(long long first, long long stride, int n)
      : tok(first), step(stride), N(n) {
    b = first / n, t = (int)(first % n);
    db = step / n, dt = (int)(step % n);
  }
  __device__ __forceinline__ void next() {
    tok += step;
    b += db, t += dt;
    if (t >= N) t -= N, ++b;
  }
  __device__ __forceinline__ bool live(const RotParams &p) const {
    return tok < p.tokens && !(p.seq_lens && t >= __ldg(p.seq_lens + b));
  }
  // not yet clamped: nothing waits for the load until the position is used
  __device__ __forceinline__ int position(const RotParams &p) const {
    if (tok >= p.tokens) return 0;
    return p.positions ? __ldg(p.positions + b * p.N + t) : t;
  }
};

// A lane's share of a token: its piece of each of kU groups of heads, at a
// distance of off[u] values from the token's first q or k value.
template <int D, int kU>
struct Lane {
  int off[kU], e0, partner;
  bool is_q[kU], on[kU];
  float2 w[kU][4];
  __device__ __forceinline__ Lane(const RotParams &p) {
    constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
    const int lane = threadIdx.x & 31, hop = p.R / 16;
    e0 = (lane % kLanes) * 8;
    partner = e0 >= p.R ? lane : (e0 < p.R / 2 ? lane + hop : lane - hop);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int head = (blockIdx.y * kU + u) * kHeads + lane / kLanes;
      is_q[u] = head < p.H, on[u] = head < p.H + p.Hk;
      off[u] = (is_q[u] ? head : head - p.H) * D + e0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[u][i] = both(0.f);
      if (on[u]) load_f8((is_q[u] ? p.wq : p.wk) + off[u], w[u]);
    }
  }
};

// A warp's ring of tokens on their way in, in shared memory (cp.async): kIn
// tensors' pieces and the row of the table.  Two tokens (fp32: one) are out while
// one is computed, which the registers could not hold.
template <typename T, int D, int kU, int kIn>
struct Ring {
  static constexpr int kStages = sizeof(T) == 2 ? 3 : 2;
  static constexpr int kPiece = 8 * (int)sizeof(T);  // bytes a lane
  static constexpr int kRow = kIn * kU * 32 * kPiece, kBytes = kRow + 512;
  static constexpr int kSmem = kWarps * kStages * kBytes;
  uint32_t base;
  Walk ahead;
  int pos;  // of the next token to send for
  __device__ __forceinline__ Ring(const RotParams &p, uint32_t smem, long long first, long long step)
      : base(smem + (threadIdx.x >> 5) * kStages * kBytes), ahead(first, step, p.N) {
    pos = ahead.position(p);
  }
  __device__ __forceinline__ uint32_t piece(int stage, int in, int u) const {
    return base + stage * kBytes + (in * kU + u) * 32 * kPiece + (threadIdx.x & 31) * 16;
  }
  __device__ __forceinline__ uint32_t row(int stage) const { return base + stage * kBytes + kRow; }
  __device__ __forceinline__ void copy(uint32_t to, const T *from) {
    cp_async_16(to, from);
    if (sizeof(T) == 4) cp_async_16(to + 512, from + 4);
  }
  // Sends for the next token; one copy group whether it is valid or not.
  __device__ __forceinline__ void send(const RotParams &p, const Lane<D, kU> &ln, int stage) {
    const bool live = ahead.live(p);
    const int at = min(max(pos, 0), p.P - 1);
    const long long tok = ahead.tok, b = ahead.b;
    const int t = ahead.t;
    ahead.next();
    pos = ahead.position(p);
    if (live) {
      const T *q = (const T *)p.q + b * p.sqb + t * p.sqt, *k = (const T *)p.k + b * p.skb + t * p.skt;
      const T *gq = (const T *)p.dqo + tok * p.H * D, *gk = (const T *)p.dko + tok * p.Hk * D;
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (ln.on[u]) {
          copy(piece(stage, 0, u), (ln.is_q[u] ? q : k) + ln.off[u]);
          if (kIn == 2) copy(piece(stage, 1, u), (ln.is_q[u] ? gq : gk) + ln.off[u]);
        }
      const int lane = threadIdx.x & 31;
      if (4 * lane < p.R) cp_async_16(row(stage) + 16 * lane, p.rot + (long long)at * p.R + 4 * lane);
    }
    cp_async_commit();
  }
  // Waits for the oldest token in flight, for every lane's copies of it.
  __device__ __forceinline__ void arrive() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncwarp();
  }
};

// Grid (slabs, head blocks); block y serves the heads of its kU groups.
template <typename T, int D, int kU, bool kNext>
__global__ void __launch_bounds__(kThreads, kBlocks) rotate_kernel(const RotParams p) {
  using R = Ring<T, D, kU, 1>;
  extern __shared__ __align__(16) uint8_t smem[];
  grid_dep_wait();
  grid_dep_launch();
  const Lane<D, kU> ln(p);
  const long long first = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const long long step = (long long)gridDim.x * kWarps;
  R ring(p, smem_u32(smem), first, step);
#pragma unroll
  for (int i = 0; i < R::kStages - 1; ++i) ring.send(p, ln, i);
  int stage = 0;
  for (Walk at(first, step, p.N); at.tok < p.tokens; at.next()) {
    ring.arrive();
    ring.send(p, ln, stage == 0 ? R::kStages - 1 : stage - 1);
    if (at.live(p)) {  // the same for the whole warp
      Turn<kNext, 1> turn;
      turn.load(ring.row(stage), ln.e0, p.R);
      T *qo = (T *)p.qo + at.tok * p.H * D, *ko = (T *)p.ko + at.tok * p.Hk * D;
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        Pack8<T> in;
        in.load(ring.piece(stage, 0, u));
        float2 x[4];
        in.get(x);
        float2 sq = __fmul2_rn(x[0], x[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) sq = __ffma2_rn(x[i], x[i], sq);
        const float r = rsqrt_approx(fmaf(head_sum<D / 8>(sq.x + sq.y), 1.f / D, p.eps));
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __fmul2_rn(__fmul2_rn(x[i], ln.w[u][i]), both(r));
        turn.apply(x, ln.partner);
        if (ln.on[u]) Pack8<T>::store((ln.is_q[u] ? qo : ko) + ln.off[u], x);
      }
    }
    stage = stage == R::kStages - 1 ? 0 : stage + 1;
  }
}

template <typename T, int D, int kU, bool kNext>
__global__ void __launch_bounds__(kThreads, kBlocks) rotate_bwd_kernel(const RotParams p) {
  using R = Ring<T, D, kU, 2>;
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
  extern __shared__ __align__(16) uint8_t smem[];
  grid_dep_wait();
  grid_dep_launch();
  const Lane<D, kU> ln(p);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, HT = p.H + p.Hk;
  float2 dw[kU][4];
#pragma unroll
  for (int u = 0; u < kU; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[u][i] = both(0.f);
  const long long first = (long long)blockIdx.x * kWarps + warp;
  const long long step = (long long)gridDim.x * kWarps;
  R ring(p, smem_u32(smem), first, step);
#pragma unroll
  for (int i = 0; i < R::kStages - 1; ++i) ring.send(p, ln, i);
  int stage = 0;
  for (Walk at(first, step, p.N); at.tok < p.tokens; at.next()) {
    ring.arrive();
    ring.send(p, ln, stage == 0 ? R::kStages - 1 : stage - 1);
    T *dq = (T *)p.qo + at.tok * p.H * D, *dk = (T *)p.ko + at.tok * p.Hk * D;
    if (at.live(p)) {  // the same for the whole warp
      Turn<kNext, -1> turn;
      turn.load(ring.row(stage), ln.e0, p.R);
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        Pack8<T> in, gin;
        in.load(ring.piece(stage, 0, u));
        gin.load(ring.piece(stage, 1, u));
        float2 x[4], g[4];
        in.get(x);
        gin.get(g);
        turn.apply(g, ln.partner);
        float2 sq = __fmul2_rn(x[0], x[0]);
        float2 gx[4], dot = both(0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i) sq = __ffma2_rn(x[i], x[i], sq);
          gx[i] = __fmul2_rn(g[i], x[i]);
          dot = __ffma2_rn(gx[i], ln.w[u][i], dot);
        }
        const float r = rsqrt_approx(fmaf(head_sum<kLanes>(sq.x + sq.y), 1.f / D, p.eps));
        // dx = r (u - x r^2 mean(u x)); r^3 would overflow first
        const float m = head_sum<kLanes>(dot.x + dot.y) * (-1.f / D) * r * r;
        float2 dx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (ln.on[u]) dw[u][i] = __ffma2_rn(gx[i], both(r), dw[u][i]);
          dx[i] = __fmul2_rn(__ffma2_rn(x[i], both(m), __fmul2_rn(g[i], ln.w[u][i])), both(r));
        }
        if (ln.on[u]) Pack8<T>::store((ln.is_q[u] ? dq : dk) + ln.off[u], dx);
      }
    } else {  // past the end: zeros
      const float2 zero[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (ln.on[u]) Pack8<T>::store((ln.is_q[u] ? dq : dk) + ln.off[u], zero);
    }
    stage = stage == R::kStages - 1 ? 0 : stage + 1;
  }
  // the block's sums of dw, through the ring's memory
  float(*red)[kU][32][9] = (float(*)[kU][32][9])smem;
  static_assert(sizeof(float) * kWarps * kU * 32 * 9 <= R::kSmem, "sums fit the ring");
  cp_async_wait_all();
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kU; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      red[warp][u][lane][2 * i] = dw[u][i].x, red[warp][u][lane][2 * i + 1] = dw[u][i].y;
  __syncthreads();
  for (int e = threadIdx.x; e < kU * 256; e += kThreads) {
    const int u = e >> 8, l = (e >> 3) & 31, i = e & 7;
    const int hd = (blockIdx.y * kU + u) * kHeads + l / kLanes;
    if (hd >= HT) continue;
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < kWarps; ++v) s += red[v][u][l][i];
    p.part[((size_t)blockIdx.x * HT + hd) * D + (l % kLanes) * 8 + i] = s;
  }
}

// dnorm_q, dnorm_k: the slabs' sums in slab order (8 interleaved runs, then
// those in order), 32 columns a block.
__global__ void __launch_bounds__(256) rotate_dw_kernel(const float *__restrict__ part, int slabs,
                                                        int cols, int qcols,
                                                        float *__restrict__ dwq,
                                                        float *__restrict__ dwk) {
  __shared__ float red[8][33];
  grid_dep_wait();
  grid_dep_launch();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
  float s = 0.f;  // cols is a multiple of 32
  for (int i = g; i < slabs; i += 8) s += part[(size_t)i * cols + c];
  red[g][threadIdx.x & 31] = s;
  __syncthreads();
  if (g == 0) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += red[i][threadIdx.x];
    if (c < qcols)
      dwq[c] = t;
    else
      dwk[c - qcols] = t;
  }
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
    return 152;
  return n;
}

// Blocks along the tokens: enough to fill the device's SMs `per_sm` deep over
// all head blocks, never more than there are tokens for its warps.
int slab_count(long long tokens, int head_blocks, int per_sm) {
  const long long want = (tokens + kWarps - 1) / kWarps;
  long long most = ((long long)sm_count() * per_sm + head_blocks - 1) / head_blocks;
  if (most < 1) most = 1;
  return (int)(want < most ? want : most);
}

template <typename T, int D, int kU>
cudaError_t launch_fwd(const RotParams &p, bool next, cudaStream_t st) {
  const int groups = (p.H + p.Hk + 256 / D - 1) / (256 / D), blocks = (groups + kU - 1) / kU;
  const dim3 grid(slab_count(p.tokens, blocks, kBlocks), blocks);
  const auto kernel = next ? rotate_kernel<T, D, kU, true> : rotate_kernel<T, D, kU, false>;
  constexpr int smem = Ring<T, D, kU, 1>::kSmem;
  const cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  count_launch();
  return launch_pdl(kernel, grid, dim3(kThreads), smem, st, p);
}

template <typename T, int D>
cudaError_t fwd_d(const RotParams &p, bool next, cudaStream_t st) {
  const int groups = (p.H + p.Hk + 256 / D - 1) / (256 / D);
  // Groups of heads a warp: one where there are too few tokens for the warps, so
  // that all loads go out at once; four in bf16 (one row of the table for 4
  // groups; B4 H8 N8192 D64: 23.1 us, with two 26.5), two in fp32 (46.8 and 44.5)
  // or where there are no more.
  if (p.tokens * groups < (long long)sm_count() * kBlocks * kWarps)
    return launch_fwd<T, D, 1>(p, next, st);
  if (sizeof(T) == 4 || groups <= 2) return launch_fwd<T, D, 2>(p, next, st);
  return launch_fwd<T, D, 4>(p, next, st);
}

template <int D>
int bwd_blocks(const RotParams &p) {
  return ((p.H + p.Hk + 256 / D - 1) / (256 / D) + kBwdU - 1) / kBwdU;
}

template <typename T, int D>
cudaError_t bwd_d(const RotParams &p, bool next, float *dwq, float *dwk, cudaStream_t st) {
  const int blocks = bwd_blocks<D>(p), slabs = slab_count(p.tokens, blocks, kBlocks);
  const dim3 grid(slabs, blocks);
  const auto kernel = next ? rotate_bwd_kernel<T, D, kBwdU, true> : rotate_bwd_kernel<T, D, kBwdU, false>;
  constexpr int smem = Ring<T, D, kBwdU, 2>::kSmem;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  count_launch(2);
  if ((e = launch_pdl(kernel, grid, dim3(kThreads), smem, st, p)) != cudaSuccess) return e;
  const int cols = (p.H + p.Hk) * D;
  return launch_pdl(rotate_dw_kernel, dim3(cols / 32), dim3(256), 0, st, (const float *)p.part,
                    slabs, cols, p.H * D, dwq, dwk);
}

RotParams rot_params(const RotateArgs &a) {
  RotParams p = {};
  p.q = a.q, p.k = a.k, p.dqo = a.dqo, p.dko = a.dko;
  p.wq = a.norm_q, p.wk = a.norm_k, p.rot = a.rot;
  p.positions = a.positions, p.seq_lens = a.seq_lens;
  p.qo = a.qo, p.ko = a.ko;
  p.sqb = a.sq[0], p.sqt = a.sq[1], p.skb = a.sk[0], p.skt = a.sk[1];
  p.tokens = (long long)a.B * a.N;
  p.N = a.N, p.H = a.H, p.Hk = a.Hk, p.R = a.R, p.P = a.P;
  p.eps = a.eps;
  return p;
}

}  // namespace

cudaError_t rotate_forward(const RotateArgs &a, cudaStream_t st) {
  const RotParams p = rot_params(a);
  if (a.dtype == GBLA_FP32) {
    if (a.D == 32) return fwd_d<float, 32>(p, a.interleaved, st);
    if (a.D == 64) return fwd_d<float, 64>(p, a.interleaved, st);
    return fwd_d<float, 128>(p, a.interleaved, st);
  }
  if (a.D == 32) return fwd_d<__nv_bfloat16, 32>(p, a.interleaved, st);
  if (a.D == 64) return fwd_d<__nv_bfloat16, 64>(p, a.interleaved, st);
  return fwd_d<__nv_bfloat16, 128>(p, a.interleaved, st);
}

size_t rotate_backward_floats(const RotateArgs &a) {
  const RotParams p = rot_params(a);
  const int blocks = a.D == 32 ? bwd_blocks<32>(p) : a.D == 64 ? bwd_blocks<64>(p) : bwd_blocks<128>(p);
  return (size_t)slab_count(p.tokens, blocks, kBlocks) * (a.H + a.Hk) * a.D;
}

cudaError_t rotate_backward(const RotateArgs &a, float *part, float *dnorm_q, float *dnorm_k,
                            cudaStream_t st) {
  RotParams p = rot_params(a);
  p.part = part;
  const bool n = a.interleaved;
  if (a.dtype == GBLA_FP32) {
    if (a.D == 32) return bwd_d<float, 32>(p, n, dnorm_q, dnorm_k, st);
    if (a.D == 64) return bwd_d<float, 64>(p, n, dnorm_q, dnorm_k, st);
    return bwd_d<float, 128>(p, n, dnorm_q, dnorm_k, st);
  }
  if (a.D == 32) return bwd_d<__nv_bfloat16, 32>(p, n, dnorm_q, dnorm_k, st);
  if (a.D == 64) return bwd_d<__nv_bfloat16, 64>(p, n, dnorm_q, dnorm_k, st);
  return bwd_d<__nv_bfloat16, 128>(p, n, dnorm_q, dnorm_k, st);
}

}  // namespace gbla
