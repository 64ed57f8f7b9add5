// Norm of each query and key head with the position rotation in the same pass,
// forward and backward.  Per token and head x[D] with the head's weight w:
//   r = 1 / sqrt(mean(x^2) + eps),  y = x r w,
// then every pair (a, b) of the first R values turns by its position's angle,
//   (a, b) -> (a cos - b sin, a sin + b cos);
// backward, with g = the incoming gradient turned by the opposite angles and
// n = x r:  dw = sum g n,  u = g w,  dx = r (u - n mean(u n)).
//
// About 5 flops a byte: bound by memory.  A head vector is spread over D / 8
// lanes of 8 values (one 16-byte load in bf16), so a warp holds 256 / D heads
// at once, the mean is a butterfly over those lanes, and the half-split pairs
// (i, i + R / 2) meet by one shuffle per value.  A warp keeps its kU groups of
// heads while it walks over the tokens: their weights stay in registers, and a
// token's row of cosines and sines is read once for all of them.
#include "gbla_internal.cuh"
#include "gbla_sm100.cuh"

namespace gbla {
namespace {

using namespace sm100;

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;

template <typename T>
struct Pack8;  // 8 consecutive values of a head as loaded
template <>
struct Pack8<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void load(const __nv_bfloat16 *p) { u = ldg_nc_v4(p); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = bf2_to_f2(w[i]);
      f[2 * i] = v.x;
      f[2 * i + 1] = v.y;
    }
  }
  __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float (&f)[8]) {
    *(uint4 *)p = make_uint4(f2_to_bf2(f[0], f[1]), f2_to_bf2(f[2], f[3]), f2_to_bf2(f[4], f[5]),
                             f2_to_bf2(f[6], f[7]));
  }
};
template <>
struct Pack8<float> {
  uint4 a, b;
  __device__ __forceinline__ void load(const float *p) {
    a = ldg_nc_v4(p);
    b = ldg_nc_v4(p + 4);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
  }
  __device__ __forceinline__ static void store(float *p, const float (&f)[8]) {
    *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
    *(float4 *)(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
  }
};

__device__ __forceinline__ void load_f8(const float *p, float (&f)[8]) {
  const float4 a = __ldg((const float4 *)p), b = __ldg((const float4 *)p + 1);
  f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
  f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}

// The lane's cosines and sines of one token.  Half-split pairs: value e of the
// first half turns with partner e + R/2, so out = y cos + y_partner sin with
// the sine negated in the first half.  Neighbouring pairs (2i, 2i + 1): four
// cosines and four sines.  Lanes past R get cos = 1, sin = 0.
template <bool kNext>
struct Turn {
  float c[kNext ? 4 : 8], s[kNext ? 4 : 8];
  __device__ __forceinline__ void load(const float *row, int e0, int R) {
    if (e0 >= R) {
#pragma unroll
      for (int i = 0; i < (kNext ? 4 : 8); ++i) c[i] = 1.f, s[i] = 0.f;
      return;
    }
    if (kNext) {
      const float4 a = __ldg((const float4 *)(row + e0 / 2));
      const float4 b = __ldg((const float4 *)(row + R / 2 + e0 / 2));
      c[0] = a.x, c[1] = a.y, c[2] = a.z, c[3] = a.w;
      s[0] = b.x, s[1] = b.y, s[2] = b.z, s[3] = b.w;
    } else {
      const int half = R / 2, i0 = e0 < half ? e0 : e0 - half;
      float a[8], b[8];
      load_f8(row + i0, a);
      load_f8(row + half + i0, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = a[i], s[i] = e0 < half ? -b[i] : b[i];
    }
  }
  // dir = 1 turns by the angles, -1 by the opposite ones
  __device__ __forceinline__ void apply(float (&y)[8], int partner, float dir) const {
    if (kNext) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = y[2 * i], b = y[2 * i + 1], sd = s[i] * dir;
        y[2 * i] = a * c[i] - b * sd;
        y[2 * i + 1] = a * sd + b * c[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float o = __shfl_sync(0xffffffffu, y[i], partner);
        y[i] = fmaf(y[i], c[i], o * (s[i] * dir));
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
  long long b, db;
  int t, dt, N;
  __device__ __forceinline__ Walk(long long first, long long step, int n) : N(n) {
    b = first / n, t = (int)(first % n);
    db = step / n, dt = (int)(step % n);
  }
  __device__ __forceinline__ void next() {
    b += db, t += dt;
    if (t >= N) t -= N, ++b;
  }
};

__device__ __forceinline__ const float *rot_row(const RotParams &p, long long b, int t) {
  int pos = p.positions ? __ldg(p.positions + b * p.N + t) : t;
  pos = min(max(pos, 0), p.P - 1);
  return p.rot + (long long)pos * p.R;
}

// Grid (slabs, head blocks); block y serves the heads of its kU groups.
template <typename T, int D, int kU, bool kNext>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotParams p) {
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
  grid_dep_wait();
  grid_dep_launch();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = lane / kLanes, e0 = (lane % kLanes) * 8, HT = p.H + p.Hk;
  int head[kU];
  float w[kU][8] = {};
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    head[u] = (blockIdx.y * kU + u) * kHeads + sub;
    if (head[u] < HT)
      load_f8((head[u] < p.H ? p.wq + (size_t)head[u] * D : p.wk + (size_t)(head[u] - p.H) * D) +
                  e0,
              w[u]);
  }
  const int hop = p.R / 16;
  const int partner = e0 >= p.R ? lane : (e0 < p.R / 2 ? lane + hop : lane - hop);
  const long long step = (long long)gridDim.x * kWarps;
  Walk at((long long)blockIdx.x * kWarps + warp, step, p.N);
  for (long long tok = (long long)blockIdx.x * kWarps + warp; tok < p.tokens;
       tok += step, at.next()) {
    if (p.seq_lens && at.t >= __ldg(p.seq_lens + at.b)) continue;
    Pack8<T> in[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (head[u] < HT)
        in[u].load(head[u] < p.H
                       ? (const T *)p.q + at.b * p.sqb + at.t * p.sqt + (long long)head[u] * D + e0
                       : (const T *)p.k + at.b * p.skb + at.t * p.skt +
                             (long long)(head[u] - p.H) * D + e0);
    Turn<kNext> turn;
    turn.load(p.R ? rot_row(p, at.b, at.t) : nullptr, e0, p.R);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float x[8] = {};
      if (head[u] < HT) in[u].get(x);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
      const float r = rsqrtf(head_sum<kLanes>(ss) * (1.f / D) + p.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[u][i];
      turn.apply(x, partner, 1.f);
      if (head[u] < HT) {
        T *o = head[u] < p.H ? (T *)p.qo + (tok * p.H + head[u]) * D + e0
                             : (T *)p.ko + (tok * p.Hk + (head[u] - p.H)) * D + e0;
        Pack8<T>::store(o, x);
      }
    }
  }
}

template <typename T, int D, int kU, bool kNext>
__global__ void __launch_bounds__(kThreads) rotate_bwd_kernel(const RotParams p) {
  constexpr int kLanes = D / 8, kHeads = 32 / kLanes;
  __shared__ float red[kWarps][kU][32][9];
  grid_dep_wait();
  grid_dep_launch();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = lane / kLanes, e0 = (lane % kLanes) * 8, HT = p.H + p.Hk;
  int head[kU];
  float w[kU][8] = {}, dw[kU][8] = {};
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    head[u] = (blockIdx.y * kU + u) * kHeads + sub;
    if (head[u] < HT)
      load_f8((head[u] < p.H ? p.wq + (size_t)head[u] * D : p.wk + (size_t)(head[u] - p.H) * D) +
                  e0,
              w[u]);
  }
  const int hop = p.R / 16;
  const int partner = e0 >= p.R ? lane : (e0 < p.R / 2 ? lane + hop : lane - hop);
  const long long step = (long long)gridDim.x * kWarps;
  Walk at((long long)blockIdx.x * kWarps + warp, step, p.N);
  for (long long tok = (long long)blockIdx.x * kWarps + warp; tok < p.tokens;
       tok += step, at.next()) {
    const bool live = !(p.seq_lens && at.t >= __ldg(p.seq_lens + at.b));
    Pack8<T> in[kU], gin[kU];
    if (live) {
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (head[u] < HT) {
          const bool isq = head[u] < p.H;
          const int hk = head[u] - p.H;
          in[u].load(isq ? (const T *)p.q + at.b * p.sqb + at.t * p.sqt + (long long)head[u] * D + e0
                         : (const T *)p.k + at.b * p.skb + at.t * p.skt + (long long)hk * D + e0);
          gin[u].load(isq ? (const T *)p.dqo + (tok * p.H + head[u]) * D + e0
                          : (const T *)p.dko + (tok * p.Hk + hk) * D + e0);
        }
    }
    Turn<kNext> turn;
    if (live) turn.load(p.R ? rot_row(p, at.b, at.t) : nullptr, e0, p.R);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float dx[8] = {};
      if (live) {  // the same for the whole warp
        float x[8] = {}, g[8] = {};
        if (head[u] < HT) in[u].get(x), gin[u].get(g);
        turn.apply(g, partner, -1.f);
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          ss = fmaf(x[i], x[i], ss);
          dot = fmaf(g[i] * w[u][i], x[i], dot);
        }
        const float r = rsqrtf(head_sum<kLanes>(ss) * (1.f / D) + p.eps);
        const float m = head_sum<kLanes>(dot) * (1.f / D) * r * r;  // mean(u n) r
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dw[u][i] = fmaf(g[i], x[i] * r, dw[u][i]);
          dx[i] = r * (g[i] * w[u][i] - x[i] * m);
        }
      }
      if (head[u] < HT) {  // rows past the end get zeros
        T *o = head[u] < p.H ? (T *)p.qo + (tok * p.H + head[u]) * D + e0
                             : (T *)p.ko + (tok * p.Hk + (head[u] - p.H)) * D + e0;
        Pack8<T>::store(o, dx);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kU; ++u)
#pragma unroll
    for (int i = 0; i < 8; ++i) red[warp][u][lane][i] = dw[u][i];
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

constexpr int kPerSm = 4;

template <typename T, int D, int kU>
cudaError_t launch_fwd(const RotParams &p, bool next, cudaStream_t st) {
  const int groups = (p.H + p.Hk + 256 / D - 1) / (256 / D), blocks = (groups + kU - 1) / kU;
  const dim3 grid(slab_count(p.tokens, blocks, kPerSm), blocks);
  count_launch();
  return next ? launch_pdl(rotate_kernel<T, D, kU, true>, grid, dim3(kThreads), 0, st, p)
              : launch_pdl(rotate_kernel<T, D, kU, false>, grid, dim3(kThreads), 0, st, p);
}

template <typename T, int D>
cudaError_t fwd_d(const RotParams &p, bool next, cudaStream_t st) {
  const int groups = (p.H + p.Hk + 256 / D - 1) / (256 / D);
  // Few tokens: one group of heads a warp, so that all loads go out at once.
  if (p.tokens * ((groups + 3) / 4) < (long long)sm_count() * kWarps)
    return launch_fwd<T, D, 1>(p, next, st);
  return launch_fwd<T, D, 4>(p, next, st);
}

constexpr int kBwdU = 2, kBwdPerSm = 2;

template <int D>
int bwd_blocks(const RotParams &p) {
  return ((p.H + p.Hk + 256 / D - 1) / (256 / D) + kBwdU - 1) / kBwdU;
}

template <typename T, int D>
cudaError_t bwd_d(const RotParams &p, bool next, float *dwq, float *dwk, cudaStream_t st) {
  const int blocks = bwd_blocks<D>(p), slabs = slab_count(p.tokens, blocks, kBwdPerSm);
  const dim3 grid(slabs, blocks);
  count_launch(2);
  cudaError_t e =
      next ? launch_pdl(rotate_bwd_kernel<T, D, kBwdU, true>, grid, dim3(kThreads), 0, st, p)
           : launch_pdl(rotate_bwd_kernel<T, D, kBwdU, false>, grid, dim3(kThreads), 0, st, p);
  if (e != cudaSuccess) return e;
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
  return (size_t)slab_count(p.tokens, blocks, kBwdPerSm) * (a.H + a.Hk) * a.D;
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
