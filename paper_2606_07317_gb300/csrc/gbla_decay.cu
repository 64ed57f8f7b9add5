// Decayed linear attention on CUDA cores: the chunked scan for every type and
// head size (fp32 arithmetic), the sum over heads that share a key / value
// head, and the single-token form.
//
// With gamma = exp(log_decay[h]), tokens in chunks of C, r the place in a chunk
// and S the state before it,
//   out_r = scale [ sum_{j <= r} gamma^{r-j} (x_r . y_j) z_j + gamma^{r+1} x_r^T S ],
//   S'    = gamma^C S + sum_j gamma^{C-1-j} y_j z_j^T.
// The scan in reverse (the gradients of keys and values) is the same with the
// powers counted from the chunk's other end.
#include <math.h>

#include "gbla_internal.cuh"
#include "gbla_sm100.cuh"

namespace gbla {
namespace {

using namespace sm100;

// gamma^n for n >= 0 with l2 = log2 gamma; gamma^0 is 1 also for gamma = 0.
__device__ __forceinline__ float decay_pow(float l2, float n) {
  return n == 0.f ? 1.f : exp2f(n * l2);
}
__device__ __forceinline__ float log2_decay(const float *log_decay, int h) {
  return __ldg(log_decay + h) * 1.4426950408889634f;
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void load4(const float *p, float (&f)[4]) {
  const float4 v = __ldg((const float4 *)p);
  f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16 *p, float (&f)[4]) {
  const uint2 v = __ldg((const uint2 *)p);
  const float2 a = bf2_to_f2(v.x), b = bf2_to_f2(v.y);
  f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y;
}
__device__ __forceinline__ void store4(float *p, const float (&f)[4]) {
  *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16 *p, const float (&f)[4]) {
  *(uint2 *)p = make_uint2(f2_to_bf2(f[0], f[1]), f2_to_bf2(f[2], f[3]));
}

// ------------------------------------------------------------------ the scan
constexpr int kC = 32;        // tokens per chunk
constexpr int kThreads = 256;

struct ScanDev {
  const void *x, *y, *z;
  long long sx[2], sy[2], sz[2];
  int gx, gy, gz;
  void *out;
  bool zero_pad, init_t, reverse;
  const float *log_decay;
  const int32_t *seq_lens;
  const float *init;
  float init_scale, fin_scale, scale;
  float *fin, *part;
  int N, H, seg, nseg;  // tokens per segment (a multiple of kC), most segments
};

template <int D>
struct ScanShape {
  static constexpr int kRow = D + 4;                  // padded row of a tile, in floats
  static constexpr int kTile = kC * kRow;
  static constexpr int kSmemFloats = 3 * kTile + kC * (kC + 4) + D * kRow + kC + 1;
  // the state in registers: a kS x kS tile a thread (4 x 4 at D = 64)
  static constexpr int kSt = D / 16;
  // outputs: 4 columns and kOr rows a thread
  static constexpr int kOc = D / 4, kOrows = kThreads / kOc, kOr = kC / kOrows;
};

// One segment of one (batch, head).  kState: only its own state (zero before
// it) goes to `part`; else the results, from the state that the segments before
// it in scan order leave.  The state lives in registers, D / 16 rows by D / 16
// columns a thread (rows ty + 16 i, columns tx * (D / 16) + j), and is laid
// out in shared memory for the product with x.
template <typename T, typename O, int D, bool kState>
__global__ void __launch_bounds__(kThreads) scan_kernel(const ScanDev p) {
  using Sh = ScanShape<D>;
  constexpr int kRow = Sh::kRow, kSt = Sh::kSt, kOr = Sh::kOr;
  extern __shared__ __align__(16) float sm[];
  float *xs = sm, *ys = xs + Sh::kTile, *zs = ys + Sh::kTile;
  float *ps = zs + Sh::kTile;          // [kC][kC + 4] weighted scores
  float *ss = ps + kC * (kC + 4);      // [D][kRow] the state
  float *gp = ss + D * kRow;           // gamma^0 .. gamma^kC
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int seg = blockIdx.x, h = blockIdx.y;
  const int b = blockIdx.z;
  const int L = p.seq_lens ? min(max(p.seq_lens[b], 0), p.N) : p.N;
  const int ns = (L + p.seg - 1) / p.seg;
  const size_t bh = (size_t)b * p.H + h;
  O *out = (O *)p.out + ((size_t)b * p.N * p.H + h) * D;  // row t at t * H * D
  const size_t orow = (size_t)p.H * D;
  if (!kState && p.zero_pad) {  // this segment's share of the rows past the end
    const int t1 = min(p.N, (seg + 1) * p.seg);
    const float z4[4] = {};
    for (int i = tid; i < (t1 - max(L, seg * p.seg)) * (D / 4); i += kThreads)
      store4(out + (max(L, seg * p.seg) + i / (D / 4)) * orow + i % (D / 4) * 4, z4);
  }
  // the last segment in scan order also writes the final state; an empty
  // sequence has none, so segment 0 passes the first state on
  const int last = p.reverse ? 0 : (ns > 0 ? ns - 1 : 0);
  if (seg >= ns && !(seg == 0 && !kState && p.fin)) return;
  if (kState && seg == (p.reverse ? 0 : ns - 1)) return;  // nobody reads it
  const float l2 = log2_decay(p.log_decay, h);
  if (tid <= kC) gp[tid] = decay_pow(l2, (float)tid);

  float S[kSt][kSt];
#pragma unroll
  for (int i = 0; i < kSt; ++i)
#pragma unroll
    for (int j = 0; j < kSt; ++j) S[i][j] = 0.f;
  const bool first = p.reverse ? seg == ns - 1 : seg == 0;
  const int s_end = min(L, (seg + 1) * p.seg);
  if (!kState) {
    if (p.init) {
      // tokens between the first state and this segment
      const float n = p.reverse ? (first || ns == 0 ? 0.f : (float)(L - 1 - s_end)) : (float)seg * p.seg;
      const float w = decay_pow(l2, n) * p.init_scale;
      const float *s0 = p.init + bh * D * D;
#pragma unroll
      for (int i = 0; i < kSt; ++i)
#pragma unroll
        for (int j = 0; j < kSt; ++j) {
          const int d = ty + 16 * i, e = tx * kSt + j;
          S[i][j] = w * (p.init_t ? s0[(size_t)e * D + d] : s0[(size_t)d * D + e]);
        }
    }
    const int lo = p.reverse ? seg + 1 : 0, hi = p.reverse ? ns : seg;
    for (int s = lo; s < hi; ++s) {
      const int gap = p.reverse ? s - seg - 1 : seg - 1 - s;
      const float w = decay_pow(l2, (float)gap * p.seg);
      const float *u = p.part + (bh * p.nseg + s) * (size_t)D * D;
#pragma unroll
      for (int i = 0; i < kSt; ++i)
#pragma unroll
        for (int j = 0; j < kSt; ++j) S[i][j] = fmaf(w, u[(ty + 16 * i) * D + tx * kSt + j], S[i][j]);
    }
  }

  const T *xg = (const T *)p.x + b * p.sx[0] + (long long)(h / p.gx) * D;
  const T *yg = (const T *)p.y + b * p.sy[0] + (long long)(h / p.gy) * D;
  const T *zg = (const T *)p.z + b * p.sz[0] + (long long)(h / p.gz) * D;
  constexpr int kLoads = kC * D / 4 / kThreads;  // float4s of a tile a thread
  const int nc = seg < ns ? (s_end - seg * p.seg + kC - 1) / kC : 0;
  for (int ci = 0; ci < nc; ++ci) {
    const int c0 = seg * p.seg + (p.reverse ? nc - 1 - ci : ci) * kC;
    const int n = min(kC, L - c0);
    __syncthreads();  // the tiles and the state of the chunk before are read
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = tid + i * kThreads, r = at / (D / 4), c = at % (D / 4) * 4;
      float fx[4] = {}, fy[4] = {}, fz[4] = {};
      if (r < n) {
        const long long t = c0 + r;
        if (!kState) load4(xg + t * p.sx[1] + c, fx);
        load4(yg + t * p.sy[1] + c, fy);
        load4(zg + t * p.sz[1] + c, fz);
      }
      if (!kState) store4(xs + r * kRow + c, fx);
      store4(ys + r * kRow + c, fy);
      store4(zs + r * kRow + c, fz);
    }
    if (!kState) {
#pragma unroll
      for (int i = 0; i < kSt; ++i)
#pragma unroll
        for (int j = 0; j < kSt; ++j) ss[(ty + 16 * i) * kRow + tx * kSt + j] = S[i][j];
    }
    __syncthreads();
    // powers: inter weight gamma^{a0 + a1 r}, carry gamma^{span}
    const int span = p.reverse ? (first && ci == 0 ? L - 1 - c0 : kC) : n;
    if (!kState) {
      // scores, 2 rows by 2 columns a thread: rows ty, ty + 16, columns tx, tx + 16
      float s[2][2] = {};
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        float4 xv[2], yv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          xv[i] = *(const float4 *)(xs + (ty + 16 * i) * kRow + d);
          yv[i] = *(const float4 *)(ys + (tx + 16 * i) * kRow + d);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            s[i][j] = fmaf(xv[i].x, yv[j].x, s[i][j]);
            s[i][j] = fmaf(xv[i].y, yv[j].y, s[i][j]);
            s[i][j] = fmaf(xv[i].z, yv[j].z, s[i][j]);
            s[i][j] = fmaf(xv[i].w, yv[j].w, s[i][j]);
          }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = ty + 16 * i, c = tx + 16 * j, gap = p.reverse ? c - r : r - c;
          ps[r * (kC + 4) + c] = gap >= 0 ? s[i][j] * gp[gap] : 0.f;
        }
      __syncthreads();
      // results: kOr rows by 4 columns a thread
      const int oc = tid % Sh::kOc * 4, o0 = tid / Sh::kOc;
      float a[kOr][4] = {};
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        float4 sv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) sv[k] = *(const float4 *)(ss + (d + k) * kRow + oc);
#pragma unroll
        for (int i = 0; i < kOr; ++i) {
          const float4 xv = *(const float4 *)(xs + (o0 + i * Sh::kOrows) * kRow + d);
          const float xk[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            a[i][0] = fmaf(xk[k], sv[k].x, a[i][0]);
            a[i][1] = fmaf(xk[k], sv[k].y, a[i][1]);
            a[i][2] = fmaf(xk[k], sv[k].z, a[i][2]);
            a[i][3] = fmaf(xk[k], sv[k].w, a[i][3]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kOr; ++i) {
        const int r = o0 + i * Sh::kOrows;
        // rows past the end are not written: any power in range does
        const int m = p.reverse ? max(span - r, 0) : r + 1;
        const float w = gp[m];
#pragma unroll
        for (int k = 0; k < 4; ++k) a[i][k] *= w;
      }
#pragma unroll 2
      for (int j = 0; j < kC; j += 4) {
        float4 zv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) zv[k] = *(const float4 *)(zs + (j + k) * kRow + oc);
#pragma unroll
        for (int i = 0; i < kOr; ++i) {
          const float4 pv = *(const float4 *)(ps + (o0 + i * Sh::kOrows) * (kC + 4) + j);
          const float pk[4] = {pv.x, pv.y, pv.z, pv.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            a[i][0] = fmaf(pk[k], zv[k].x, a[i][0]);
            a[i][1] = fmaf(pk[k], zv[k].y, a[i][1]);
            a[i][2] = fmaf(pk[k], zv[k].z, a[i][2]);
            a[i][3] = fmaf(pk[k], zv[k].w, a[i][3]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kOr; ++i) {
        const int r = o0 + i * Sh::kOrows;
        if (r >= n) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) a[i][k] *= p.scale;
        store4(out + (size_t)(c0 + r) * orow + oc, a[i]);
      }
    }
    // the state after the chunk
    const float carry = gp[span];
#pragma unroll
    for (int i = 0; i < kSt; ++i)
#pragma unroll
      for (int j = 0; j < kSt; ++j) S[i][j] *= carry;
    for (int j = 0; j < n; ++j) {
      const float w = gp[p.reverse ? j : n - 1 - j];
      float yv[kSt], zv[kSt];
#pragma unroll
      for (int i = 0; i < kSt; ++i) {
        yv[i] = w * ys[j * kRow + ty + 16 * i];
        zv[i] = zs[j * kRow + tx * kSt + i];
      }
#pragma unroll
      for (int i = 0; i < kSt; ++i)
#pragma unroll
        for (int k = 0; k < kSt; ++k) S[i][k] = fmaf(yv[i], zv[k], S[i][k]);
    }
  }
  if (kState || (p.fin && seg == last)) {
    // reverse: what the gradient of the first state still decays by
    const float w = kState ? 1.f : p.fin_scale * (p.reverse && L > 0 ? decay_pow(l2, 1.f) : 1.f);
    float *dst = kState ? p.part + (bh * p.nseg + seg) * (size_t)D * D : p.fin + bh * D * D;
#pragma unroll
    for (int i = 0; i < kSt; ++i)
#pragma unroll
      for (int j = 0; j < kSt; ++j) dst[(ty + 16 * i) * D + tx * kSt + j] = S[i][j] * w;
  }
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
    return 152;
  return n;
}

// Segments along the sequence: none while the (batch, head) pairs fill the SMs
// twice; else as many as do, of at least 8 chunks (a segment costs its keys and
// values a second time, and the states of those before it).
int scan_segment(const ScanArgs &a) {
  const long long pairs = (long long)a.B * a.H, chunks = (a.N + kC - 1) / kC;
  long long n = pairs > 0 ? (2ll * sm_count() + pairs - 1) / pairs : 1;
  if (n > 64) n = 64;
  if (n > chunks / 8) n = chunks / 8;
  if (n < 1) n = 1;
  return (int)((chunks + n - 1) / n) * kC;
}

ScanDev scan_dev(const ScanArgs &a, float *part) {
  ScanDev p = {};
  p.x = a.x, p.y = a.y, p.z = a.z;
  for (int i = 0; i < 2; ++i) p.sx[i] = a.sx[i], p.sy[i] = a.sy[i], p.sz[i] = a.sz[i];
  p.gx = a.gx, p.gy = a.gy, p.gz = a.gz;
  p.out = a.out, p.zero_pad = a.zero_pad, p.init_t = a.init_t, p.reverse = a.reverse;
  p.log_decay = a.log_decay, p.seq_lens = a.seq_lens, p.init = a.init;
  p.init_scale = a.init_scale, p.fin_scale = a.fin_scale, p.scale = a.scale;
  p.fin = a.fin, p.part = part;
  p.N = a.N, p.H = a.H, p.seg = scan_segment(a);
  p.nseg = (a.N + p.seg - 1) / p.seg;
  return p;
}

template <typename T, typename O, int D>
cudaError_t scan_launch(const ScanArgs &a, float *part, cudaStream_t st) {
  const ScanDev p = scan_dev(a, part);
  constexpr int smem = ScanShape<D>::kSmemFloats * 4;
  const dim3 grid(p.nseg, a.H, a.B);
  cudaError_t e;
  if (p.nseg > 1) {
    if ((e = cudaFuncSetAttribute(scan_kernel<T, O, D, true>,
                                  cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess)
      return e;
    scan_kernel<T, O, D, true><<<grid, kThreads, smem, st>>>(p);
    count_launch();
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  if ((e = cudaFuncSetAttribute(scan_kernel<T, O, D, false>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess)
    return e;
  scan_kernel<T, O, D, false><<<grid, kThreads, smem, st>>>(p);
  count_launch();
  return cudaGetLastError();
}

template <typename T, typename O>
cudaError_t scan_d(const ScanArgs &a, float *part, cudaStream_t st) {
  if (a.D == 32) return scan_launch<T, O, 32>(a, part, st);
  if (a.D == 64) return scan_launch<T, O, 64>(a, part, st);
  return scan_launch<T, O, 128>(a, part, st);
}

// ------------------------------------------------ sum over shared heads
template <typename T>
__global__ void __launch_bounds__(256) shared_sum_kernel(const float *__restrict__ src,
                                                         T *__restrict__ dst, long long quads,
                                                         int G, int D4) {
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < quads; i += gridDim.x * 256ll) {
    const long long head = i / D4;  // (token, key head)
    const int c = (int)(i % D4);
    float a[4] = {};
    for (int g = 0; g < G; ++g) {
      const float4 v = __ldg((const float4 *)src + (head * G + g) * D4 + c);
      a[0] += v.x, a[1] += v.y, a[2] += v.z, a[3] += v.w;
    }
    store4(dst + i * 4, a);
  }
}

// ---------------------------------------------------------- the single token
// S = gamma S + k v^T in place and o = scale q^T S, one block a (sequence,
// head): bound by the state's bytes, 8 D^2 a head.  A thread holds 4 columns of
// kRows rows, all loads in flight before the first product.
template <int D>
struct StepShape {
  static constexpr int kCols = D / 4;                       // column quads
  static constexpr int kThreads = D == 32 ? 64 : 256;
  static constexpr int kGroups = kThreads / kCols;          // rows at a time
  static constexpr int kRows = D / kGroups;
};

template <typename T, int D>
__global__ void __launch_bounds__(StepShape<D>::kThreads) step_kernel(
    const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v, long long sq,
    long long sk, long long sv, const float *__restrict__ log_decay,
    const int32_t *__restrict__ slots, float *__restrict__ state, T *__restrict__ o, int H, int G,
    int n_slots, float scale) {
  using Sh = StepShape<D>;
  __shared__ __align__(16) float qk[2][D];
  __shared__ __align__(16) float red[Sh::kGroups][D];
  grid_dep_wait();
  grid_dep_launch();
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int slot = slots ? __ldg(slots + b) : b;
  if (slot < 0 || slot >= n_slots) return;
  const int c = tid % Sh::kCols, g = tid / Sh::kCols;
  float4 *s = (float4 *)(state + ((size_t)slot * H + h) * D * D) + c;
  float4 r[Sh::kRows];
#pragma unroll
  for (int i = 0; i < Sh::kRows; ++i) r[i] = s[(g + i * Sh::kGroups) * Sh::kCols];
  float vv[4];
  load4(v + b * sv + (long long)(h / G) * D + 4 * c, vv);
  for (int i = tid; i < 2 * D; i += Sh::kThreads)
    qk[i / D][i % D] = i < D ? to_f(q[b * sq + (long long)h * D + i])
                             : to_f(k[b * sk + (long long)(h / G) * D + i - D]);
  const float gamma = decay_pow(log2_decay(log_decay, h), 1.f);
  __syncthreads();
  float a[4] = {};
#pragma unroll
  for (int i = 0; i < Sh::kRows; ++i) {
    const int d = g + i * Sh::kGroups;
    const float kd = qk[1][d], qd = qk[0][d];
    r[i].x = fmaf(kd, vv[0], gamma * r[i].x);
    r[i].y = fmaf(kd, vv[1], gamma * r[i].y);
    r[i].z = fmaf(kd, vv[2], gamma * r[i].z);
    r[i].w = fmaf(kd, vv[3], gamma * r[i].w);
    s[d * Sh::kCols] = r[i];
    a[0] = fmaf(qd, r[i].x, a[0]);
    a[1] = fmaf(qd, r[i].y, a[1]);
    a[2] = fmaf(qd, r[i].z, a[2]);
    a[3] = fmaf(qd, r[i].w, a[3]);
  }
  store4(&red[g][4 * c], a);
  __syncthreads();
  if (g == 0) {
#pragma unroll
    for (int i = 1; i < Sh::kGroups; ++i) {
      const float4 t = *(const float4 *)&red[i][4 * c];
      a[0] += t.x, a[1] += t.y, a[2] += t.z, a[3] += t.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] *= scale;
    store4(o + ((size_t)b * H + h) * D + 4 * c, a);
  }
}

template <typename T, int D>
cudaError_t step_launch(const StepArgs &a, cudaStream_t st) {
  count_launch();
  return launch_pdl(step_kernel<T, D>, dim3(a.H, a.B), dim3(StepShape<D>::kThreads), 0, st,
                    (const T *)a.q, (const T *)a.k, (const T *)a.v, a.sq, a.sk, a.sv, a.log_decay,
                    a.slots, a.state, (T *)a.o, a.H, a.H / a.Hk, a.n_slots, a.scale);
}

}  // namespace

size_t simt_scan_floats(const ScanArgs &a) {
  const int seg = scan_segment(a), nseg = (a.N + seg - 1) / seg;
  return nseg > 1 ? (size_t)a.B * a.H * nseg * a.D * a.D : 0;
}

cudaError_t simt_scan(const ScanArgs &a, float *scratch, cudaStream_t st) {
  if (a.dtype == GBLA_FP32) return scan_d<float, float>(a, scratch, st);
  if (a.out_f32) return scan_d<__nv_bfloat16, float>(a, scratch, st);
  return scan_d<__nv_bfloat16, __nv_bfloat16>(a, scratch, st);
}

cudaError_t sum_shared_heads(const float *src, void *dst, long long tokens, int Hk, int G, int D,
                             gbla_dtype dtype, cudaStream_t st) {
  const long long quads = tokens * Hk * (D / 4);
  long long blocks = (quads + 255) / 256;
  if (blocks > 8ll * sm_count()) blocks = 8ll * sm_count();
  if (dtype == GBLA_FP32)
    shared_sum_kernel<float><<<(int)blocks, 256, 0, st>>>(src, (float *)dst, quads, G, D / 4);
  else
    shared_sum_kernel<__nv_bfloat16>
        <<<(int)blocks, 256, 0, st>>>(src, (__nv_bfloat16 *)dst, quads, G, D / 4);
  count_launch();
  return cudaGetLastError();
}

cudaError_t decay_step(const StepArgs &a, cudaStream_t st) {
  if (a.dtype == GBLA_FP32) {
    if (a.D == 32) return step_launch<float, 32>(a, st);
    if (a.D == 64) return step_launch<float, 64>(a, st);
    return step_launch<float, 128>(a, st);
  }
  if (a.D == 32) return step_launch<__nv_bfloat16, 32>(a, st);
  if (a.D == 64) return step_launch<__nv_bfloat16, 64>(a, st);
  return step_launch<__nv_bfloat16, 128>(a, st);
}

}  // namespace gbla
