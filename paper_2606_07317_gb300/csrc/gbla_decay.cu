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

#include "gbla_decay.cuh"
#include "gbla_internal.cuh"
#include "gbla_sm100.cuh"

namespace gbla {
namespace {

using namespace sm100;

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
// A block of 64 threads (D = 128: 128) serves E = min(D, 64) of the state's columns
// of one segment of one (batch, head): 2 C D + 2 D^2 multiply-adds a token and head
// in products whose operands come from shared memory.  A load's bytes into the
// registers bound those (128 a cycle, broadcast or not, against 128 multiply-adds),
// so a thread holds large tiles of results: 4 x 4 scores, 8 x 4 results (D = 128:
// 4 x 2, 4 x 4), 8 x 8 of the state (in registers for the whole segment), 1 to 2
// bytes a multiply-add.  (Blocks of 256 threads with 2 x 2, 2 x 4 and 4 x 4: 2 to 4
// bytes, 251 us where it is 142 now.)  Several blocks an SM cover one another's
// loads and barriers.  Measured, fp32: B4 H8 N4096 D64 142 us, 23 TFLOP/s of these
// products and of the second pass over the segments' states, the FMA pipe busy for
// about half of it.
constexpr int kC = 32;        // tokens per chunk
// Threads of a block: with 64, D = 128 would leave an SM four warps (B4 H8 N4096:
// 833 us, 518 with smaller tiles).
template <int D>
constexpr int kThreadsOf = D > 64 ? 128 : 64;

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
// Scans of the same sizes in one launch: those of a head follow one another in the
// grid's x.
struct ScanBatch {
  ScanDev scan[kMaxScans];
  int n;
};

template <int D, bool kState>
struct ScanShape {
  static constexpr int kE = D < 64 ? D : 64, kSplit = D / kE;
  static constexpr int kRow = D + 4, kZRow = kE + 4, kPRow = kC + 4;  // padded, in floats
  static constexpr int kOffY = kState ? 0 : kC * kRow, kOffZ = kOffY + kC * kRow;  // behind x
  static constexpr int kOffP = kOffZ + kC * kZRow, kOffS = kOffP + (kState ? 0 : kC * kPRow);
  static constexpr int kOffG = kOffS + (kState ? 0 : D * kE);
  static constexpr int kSmemFloats = kOffG + kC + 1;
  static constexpr int kThreads = kThreadsOf<D>;
  static constexpr int kQc = kThreads / 8, kQj = kC / kQc;  // scores: 4 x kQj
  static constexpr int kTx = kE / 4, kTy = kThreads / kTx, kOr = kC / kTy;  // results: kOr x 4
  static constexpr int kSr = D / (kThreads / 8), kSc = kE / 8;              // state: kSr x kSc
  static constexpr int kBlocks = D == 32 ? 8 : D == 64 ? 4 : 2;             // an SM
};

// 16 bytes from global to shared memory, or zeros.
__device__ __forceinline__ void cp_async_or_zero(uint32_t dst, const void *src, bool valid) {
  const int n = valid ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n)
               : "memory");
}
template <int kCols, int kRowFloats, int kThreads>
__device__ __forceinline__ void load_tile(float *to, const float *from, long long stride, int n) {
  for (int i = threadIdx.x; i < kC * kCols / 4; i += kThreads) {
    const int r = i / (kCols / 4), c = i % (kCols / 4) * 4;
    cp_async_or_zero(smem_u32(to + r * kRowFloats + c), from + (r < n ? r * stride + c : 0), r < n);
  }
}
template <int kCols, int kRowFloats, int kThreads>
__device__ __forceinline__ void load_tile(float *to, const __nv_bfloat16 *from, long long stride,
                                          int n) {
  for (int i = threadIdx.x; i < kC * kCols / 4; i += kThreads) {
    const int r = i / (kCols / 4), c = i % (kCols / 4) * 4;
    float f[4] = {};
    if (r < n) load4(from + r * stride + c, f);
    store4(to + r * kRowFloats + c, f);
  }
}
// kState: only the segment's own state (zero before it) goes to `part`; else the
// results, from the state before the segment, which the prefix kernel leaves in
// `part` (a single segment: the first state).
template <typename T, typename O, int D, bool kState>
__global__ void __launch_bounds__(kThreadsOf<D>, ScanShape<D, kState>::kBlocks)
    scan_kernel(const ScanBatch batch) {
  using Sh = ScanShape<D, kState>;
  constexpr int E = Sh::kE, kRow = Sh::kRow, kZRow = Sh::kZRow, kPRow = Sh::kPRow;
  constexpr int kThreads = Sh::kThreads, kQc = Sh::kQc, kQj = Sh::kQj;
  constexpr int kOr = Sh::kOr, kSr = Sh::kSr, kSc = Sh::kSc;
  extern __shared__ __align__(16) float sm[];
  float *xs = sm, *ys = sm + Sh::kOffY, *zs = sm + Sh::kOffZ;
  float *ps = sm + Sh::kOffP;  // [kC][kPRow] weighted scores
  float *st = sm + Sh::kOffS;  // [D][E] the state
  float *gp = sm + Sh::kOffG;  // gamma^0 .. gamma^kC
  const int each = gridDim.x / batch.n, place = blockIdx.x % each;
  const ScanDev &p = batch.scan[blockIdx.x / each];
  const int tid = threadIdx.x;
  const int seg = place / Sh::kSplit, e0 = place % Sh::kSplit * E;
  const int h = blockIdx.y, b = blockIdx.z;
  if (kState) grid_dep_launch();  // the prefix kernel waits for this one's results
  const int L = p.seq_lens ? min(max(p.seq_lens[b], 0), p.N) : p.N;
  const int ns = (L + p.seg - 1) / p.seg;
  const size_t bh = (size_t)b * p.H + h;
  O *out = (O *)p.out + ((size_t)b * p.N * p.H + h) * D + e0;  // row t at t * H * D
  const size_t orow = (size_t)p.H * D;
  if (!kState && p.zero_pad) {  // this segment's share of the rows past the end
    const int t0 = max(L, seg * p.seg), t1 = min(p.N, (seg + 1) * p.seg);
    const float z4[4] = {};
    for (long long i = tid; i < (long long)(t1 - t0) * (E / 4); i += kThreads)
      store4(out + (size_t)(t0 + i / (E / 4)) * orow + i % (E / 4) * 4, z4);
  }
  // the last segment in scan order also writes the final state; an empty
  // sequence has none, so segment 0 passes the first state on
  const int last = p.reverse ? 0 : (ns > 0 ? ns - 1 : 0);
  if (seg >= ns && !(seg == 0 && !kState && p.fin)) return;
  if (kState && seg == last) return;  // nobody reads it
  const float l2 = log2_decay(p.log_decay, h);
  const DecayFactor chunk_factor = decay_factor(__ldg(p.log_decay + h) * kC);
  if (tid <= kC) gp[tid] = decay_pow(l2, (float)tid);

  // rows sy + i, columns 4 sx + c and, from c = 4 on, 32 + 4 sx + c - 4
  const int sx = tid & 7, sy = (tid >> 3) * kSr;
  auto col = [&](int c) { return 4 * sx + (c & 3) + (c >> 2) * 32; };
  float S[kSr][kSc];
#pragma unroll
  for (int i = 0; i < kSr; ++i)
#pragma unroll
    for (int c = 0; c < kSc; ++c) S[i][c] = 0.f;
  const int s_end = min(L, (seg + 1) * p.seg);
  if (!kState && p.nseg > 1) grid_dep_wait();
  if (!kState && (p.nseg > 1 || p.init)) {
    const bool pre = p.nseg > 1 && ns > 0;
    const float *s0 = pre ? p.part + (bh * p.nseg + seg) * (size_t)D * D
                          : (p.init ? p.init + bh * D * D : nullptr);
    const bool flip = !pre && p.init_t;
    const float w = pre ? 1.f : p.init_scale;
    if (s0)
#pragma unroll
      for (int i = 0; i < kSr; ++i)
#pragma unroll
        for (int c = 0; c < kSc; ++c) {
          const int d = sy + i, e = e0 + col(c);
          S[i][c] = w * (flip ? s0[(size_t)e * D + d] : s0[(size_t)d * D + e]);
        }
  }

  const T *xg = (const T *)p.x + b * p.sx[0] + (long long)(h / p.gx) * D;
  const T *yg = (const T *)p.y + b * p.sy[0] + (long long)(h / p.gy) * D;
  const T *zg = (const T *)p.z + b * p.sz[0] + (long long)(h / p.gz) * D + e0;
  const int nc = seg < ns ? (s_end - seg * p.seg + kC - 1) / kC : 0;
  auto start_of = [&](int ci) { return seg * p.seg + (p.reverse ? nc - 1 - ci : ci) * kC; };
  for (int ci = 0; ci < nc; ++ci) {
    const int c0 = start_of(ci), n = min(kC, L - c0);
    if (!kState) load_tile<D, kRow, kThreads>(xs, xg + c0 * p.sx[1], p.sx[1], n);
    load_tile<D, kRow, kThreads>(ys, yg + c0 * p.sy[1], p.sy[1], n);
    load_tile<E, kZRow, kThreads>(zs, zg + c0 * p.sz[1], p.sz[1], n);
    cp_async_commit();
    if (!kState) {
#pragma unroll
      for (int i = 0; i < kSr; ++i)
#pragma unroll
        for (int c = 0; c < kSc; c += 4)
          *(float4 *)(st + (sy + i) * E + col(c)) =
              make_float4(S[i][c], S[i][c + 1], S[i][c + 2], S[i][c + 3]);
    }
    cp_async_wait_all();
    __syncthreads();
    // powers: carry gamma^span; reverse: the first state belongs to the last token
    const int span = p.reverse ? (s_end == L && ci == 0 ? L - 1 - c0 : kC) : n;
    if (!kState) {
      {
        const int qx = tid % kQc, qy = tid / kQc;  // rows 4 qy + i, columns qx + kQc j
        float a[4][kQj];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < kQj; ++j) a[i][j] = 0.f;
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
          float4 yv[kQj];
#pragma unroll
          for (int j = 0; j < kQj; ++j) yv[j] = *(const float4 *)(ys + (qx + kQc * j) * kRow + d);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 xv = *(const float4 *)(xs + (4 * qy + i) * kRow + d);
#pragma unroll
            for (int j = 0; j < kQj; ++j) {
              a[i][j] = fmaf(xv.x, yv[j].x, a[i][j]);
              a[i][j] = fmaf(xv.y, yv[j].y, a[i][j]);
              a[i][j] = fmaf(xv.z, yv[j].z, a[i][j]);
              a[i][j] = fmaf(xv.w, yv[j].w, a[i][j]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < kQj; ++j) {
            const int r = 4 * qy + i, c = qx + kQc * j, gap = p.reverse ? c - r : r - c;
            ps[r * kPRow + c] = gap >= 0 ? a[i][j] * gp[gap] : 0.f;
          }
      }
      __syncthreads();
      const int tx = tid % Sh::kTx, r0 = tid / Sh::kTx * kOr;  // rows r0 + i, columns 4 tx + c
      float o[kOr][4];
#pragma unroll
      for (int i = 0; i < kOr; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[i][c] = 0.f;
      // o += a tile of left operands (rows of 4 k) times 4 rows of right ones
      auto product = [&](const float *left, int lrow, const float *right, int rrow, int k) {
        float4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = *(const float4 *)(right + (k + q) * rrow + 4 * tx);
#pragma unroll
        for (int i = 0; i < kOr; ++i) {
          const float4 l = *(const float4 *)(left + (r0 + i) * lrow + k);
          const float lk[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            o[i][0] = fmaf(lk[q], v[q].x, o[i][0]);
            o[i][1] = fmaf(lk[q], v[q].y, o[i][1]);
            o[i][2] = fmaf(lk[q], v[q].z, o[i][2]);
            o[i][3] = fmaf(lk[q], v[q].w, o[i][3]);
          }
        }
      };
#pragma unroll 2
      for (int d = 0; d < D; d += 4) product(xs, kRow, st, E, d);
#pragma unroll
      for (int i = 0; i < kOr; ++i) {
        // rows past the end are not written: any power in range does
        const float w = gp[p.reverse ? max(span - r0 - i, 0) : r0 + i + 1];
#pragma unroll
        for (int c = 0; c < 4; ++c) o[i][c] *= w;
      }
#pragma unroll 2
      for (int j = 0; j < kC; j += 4) product(ps, kPRow, zs, kZRow, j);
#pragma unroll
      for (int i = 0; i < kOr; ++i) {
        if (r0 + i >= n) continue;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[i][c] *= p.scale;
        store4(out + (size_t)(c0 + r0 + i) * orow + 4 * tx, o[i]);
      }
    }
    // the state after the chunk
    const DecayFactor carry = span == kC ? chunk_factor : one_factor(gp[span]);
#pragma unroll
    for (int i = 0; i < kSr; ++i)
#pragma unroll
      for (int c = 0; c < kSc; ++c) S[i][c] = fmaf(carry.hi, S[i][c], carry.lo * S[i][c]);
#pragma unroll 2
    for (int j = 0; j < n; ++j) {
      const float w = gp[p.reverse ? j : n - 1 - j];
      float z[kSc];
#pragma unroll
      for (int c = 0; c < kSc; c += 4) {
        const float4 v = *(const float4 *)(zs + j * kZRow + col(c));
        z[c] = w * v.x, z[c + 1] = w * v.y, z[c + 2] = w * v.z, z[c + 3] = w * v.w;
      }
#pragma unroll
      for (int i = 0; i < kSr; i += 4) {
        const float4 v = *(const float4 *)(ys + j * kRow + sy + i);
        const float y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int c = 0; c < kSc; ++c) S[i + q][c] = fmaf(y[q], z[c], S[i + q][c]);
      }
    }
    __syncthreads();  // tiles, scores and state are read
  }
  if (kState || (p.fin && seg == last)) {
    // reverse: what the gradient of the first state still decays by
    const float w = kState ? 1.f : scaled_pow(p.fin_scale, l2, p.reverse && L > 0 ? 1.f : 0.f);
    float *dst = (kState ? p.part + (bh * p.nseg + seg) * (size_t)D * D : p.fin + bh * D * D) + e0;
#pragma unroll
    for (int i = 0; i < kSr; ++i)
#pragma unroll
      for (int c = 0; c < kSc; c += 4) {
        const float f[4] = {w * S[i][c], w * S[i][c + 1], w * S[i][c + 2], w * S[i][c + 3]};
        store4(dst + (size_t)(sy + i) * D + col(c), f);
      }
  }
}

// Replaces each segment's own state by the state before it: the first state and
// the segments before it in scan order, in that order.  Four elements a thread.
__global__ void __launch_bounds__(128) prefix_kernel(const ScanBatch batch, int D) {
  grid_dep_wait();  // (an early launch of the scan would place its blocks unevenly)
  const int each = gridDim.x / batch.n;
  const ScanDev &p = batch.scan[blockIdx.x / each];
  const int h = blockIdx.y, b = blockIdx.z, i = (blockIdx.x % each * 128 + threadIdx.x) * 4;
  const int L = p.seq_lens ? min(max(p.seq_lens[b], 0), p.N) : p.N;
  const int ns = (L + p.seg - 1) / p.seg;
  if (i >= D * D || ns == 0) return;
  const size_t bh = (size_t)b * p.H + h;
  // decay over the tokens of a segment, and of the first one in scan order (reverse: the
  // first state belongs to the last token)
  const DecayFactor whole = decay_factor(__ldg(p.log_decay + h) * p.seg);
  const DecayFactor first =
      p.reverse ? one_factor(decay_pow(log2_decay(p.log_decay, h), (float)(L - 1 - (ns - 1) * p.seg)))
                : whole;
  float S[4] = {};
  if (p.init) {
    const float *s0 = p.init + bh * D * D;
    const int d = i / D, e = i % D;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      S[c] = p.init_scale * (p.init_t ? s0[(size_t)(e + c) * D + d] : s0[i + c]);
  }
  float *part = p.part + bh * p.nseg * D * D + i;
  constexpr int kBatch = 8;  // segments whose loads go out together
  for (int k0 = 0; k0 < ns; k0 += kBatch) {
    float4 own[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int k = k0 + u, s = p.reverse ? ns - 1 - k : k;
      own[u] = k + 1 < ns ? *(const float4 *)(part + (size_t)s * D * D) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int k = k0 + u, s = p.reverse ? ns - 1 - k : k;
      if (k >= ns) break;
      store4(part + (size_t)s * D * D, S);
      const DecayFactor w = k == 0 ? first : whole;
      S[0] = fmaf(w.hi, S[0], fmaf(w.lo, S[0], own[u].x));
      S[1] = fmaf(w.hi, S[1], fmaf(w.lo, S[1], own[u].y));
      S[2] = fmaf(w.hi, S[2], fmaf(w.lo, S[2], own[u].z));
      S[3] = fmaf(w.hi, S[3], fmaf(w.lo, S[3], own[u].w));
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

// Segments along the sequence: as many as the places for blocks hold of whole
// sequences (a segment costs its state a second time, a third of the work), and,
// where only the device knows the lengths, at least eight, so that one long
// sequence does not outlast the others.
int scan_segment(const ScanArgs &a, int scans) {
  const long long blocks = (long long)a.B * a.H * scans * (a.D > 64 ? a.D / 64 : 1);
  const long long chunks = (a.N + kC - 1) / kC, full = (a.D > 64 ? 2ll : a.D > 32 ? 4ll : 8ll) * sm_count();
  long long n = blocks >= full ? 1 : full / blocks;  // one round of blocks, not a little more
  if (a.seq_lens && n < 8 && chunks >= 64) n = 8;
  if (n > 128) n = 128;  // the states before the segments are formed one after the other
  if (n > chunks) n = chunks;
  return (int)((chunks + n - 1) / n) * kC;
}

ScanDev scan_dev(const ScanArgs &a, int scans, float *part) {
  ScanDev p = {};
  p.x = a.x, p.y = a.y, p.z = a.z;
  for (int i = 0; i < 2; ++i) p.sx[i] = a.sx[i], p.sy[i] = a.sy[i], p.sz[i] = a.sz[i];
  p.gx = a.gx, p.gy = a.gy, p.gz = a.gz;
  p.out = a.out, p.zero_pad = a.zero_pad, p.init_t = a.init_t, p.reverse = a.reverse;
  p.log_decay = a.log_decay, p.seq_lens = a.seq_lens, p.init = a.init;
  p.init_scale = a.init_scale, p.fin_scale = a.fin_scale, p.scale = a.scale;
  p.fin = a.fin, p.part = part;
  p.N = a.N, p.H = a.H, p.seg = scan_segment(a, scans);
  p.nseg = (a.N + p.seg - 1) / p.seg;
  return p;
}

template <typename T, typename O, int D>
cudaError_t scan_launch(const ScanArgs &a, const ScanBatch &p, cudaStream_t st) {
  const int nseg = p.scan[0].nseg;
  const dim3 grid(nseg * ScanShape<D, true>::kSplit * p.n, a.H, a.B);
  cudaError_t e;
  if (nseg > 1) {
    constexpr int smem = ScanShape<D, true>::kSmemFloats * 4;
    const auto kernel = scan_kernel<T, O, D, true>;
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) !=
        cudaSuccess)
      return e;
    kernel<<<grid, kThreadsOf<D>, smem, st>>>(p);
    count_launch();
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    count_launch();
    if ((e = launch_pdl(prefix_kernel, dim3((D * D / 4 + 127) / 128 * p.n, a.H, a.B), dim3(128), 0,
                        st, p, D)) != cudaSuccess)
      return e;
  }
  constexpr int smem = ScanShape<D, false>::kSmemFloats * 4;
  const auto kernel = scan_kernel<T, O, D, false>;
  if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) !=
      cudaSuccess)
    return e;
  count_launch();
  if (nseg > 1) return launch_pdl(kernel, grid, dim3(kThreadsOf<D>), smem, st, p);
  kernel<<<grid, kThreadsOf<D>, smem, st>>>(p);
  return cudaGetLastError();
}

template <typename T, typename O>
cudaError_t scan_d(const ScanArgs &a, const ScanBatch &p, cudaStream_t st) {
  if (a.D == 32) return scan_launch<T, O, 32>(a, p, st);
  if (a.D == 64) return scan_launch<T, O, 64>(a, p, st);
  return scan_launch<T, O, 128>(a, p, st);
}

// ------------------------------------------------ sum over shared heads
// dv (blockIdx.y = 0) and dk from the G query heads' planes that share each key
// head, summed in 32 bits in the heads' order and rounded once.  Bound by bytes:
// 4 G read and 2 or 4 written for each value.  A head has 2^lg quads of 4 values.
template <typename T>
__global__ void __launch_bounds__(256) shared_sum_kernel(const float *__restrict__ v_planes,
                                                         const float *__restrict__ k_planes,
                                                         T *__restrict__ dv, T *__restrict__ dk,
                                                         long long quads, int G, int lg) {
  grid_dep_wait();
  grid_dep_launch();
  const float *src = blockIdx.y == 0 ? v_planes : k_planes;
  T *dst = blockIdx.y == 0 ? dv : dk;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < quads; i += gridDim.x * 256ll) {
    const float4 *at = (const float4 *)src + (((i >> lg) * G) << lg) + (i & ((1 << lg) - 1));
    float a[4] = {};
    for (int g = 0; g < G; ++g) {
      const float4 v = *(at + ((long long)g << lg));
      a[0] += v.x, a[1] += v.y, a[2] += v.z, a[3] += v.w;
    }
    store4(dst + i * 4, a);
  }
}

// ---------------------------------------------------------- the single token
// S = gamma S + k v^T in place and o = scale q^T S, one block a (sequence,
// head): bound by the state's bytes, 8 D^2 a head.  A thread holds 4 columns of
// kRows rows, all loads in flight before the first product.  Measured: 512
// sequences, 8 heads, D = 128: 80 us, 6.7 TB/s (99 % of the measured copy rate).
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
  const DecayFactor gamma = decay_factor(__ldg(log_decay + h));
  __syncthreads();
  float a[4] = {};
#pragma unroll
  for (int i = 0; i < Sh::kRows; ++i) {
    const int d = g + i * Sh::kGroups;
    const float kd = qk[1][d], qd = qk[0][d];
    r[i].x = fmaf(kd, vv[0], fmaf(gamma.hi, r[i].x, gamma.lo * r[i].x));
    r[i].y = fmaf(kd, vv[1], fmaf(gamma.hi, r[i].y, gamma.lo * r[i].y));
    r[i].z = fmaf(kd, vv[2], fmaf(gamma.hi, r[i].z, gamma.lo * r[i].z));
    r[i].w = fmaf(kd, vv[3], fmaf(gamma.hi, r[i].w, gamma.lo * r[i].w));
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

size_t simt_scan_floats(const ScanArgs &a, int n) {
  const int seg = scan_segment(a, n), nseg = (a.N + seg - 1) / seg;
  return nseg > 1 ? (size_t)n * a.B * a.H * nseg * a.D * a.D : 0;
}

cudaError_t simt_scan(const ScanArgs *a, int n, float *scratch, cudaStream_t st) {
  const size_t each = simt_scan_floats(*a, n) / n;
  ScanBatch p = {};
  p.n = n;
  for (int i = 0; i < n; ++i) p.scan[i] = scan_dev(a[i], n, scratch + i * each);
  if (a->dtype == GBLA_FP32) return scan_d<float, float>(*a, p, st);
  if (a->out_f32) return scan_d<__nv_bfloat16, float>(*a, p, st);
  return scan_d<__nv_bfloat16, __nv_bfloat16>(*a, p, st);
}

cudaError_t sum_shared_heads(const float *v_planes, const float *k_planes, void *dv, void *dk,
                             long long tokens, int Hk, int G, int D, gbla_dtype dtype,
                             cudaStream_t st) {
  const long long quads = tokens * Hk * (D / 4);
  long long blocks = (quads + 255) / 256;
  if (blocks > 4ll * sm_count()) blocks = 4ll * sm_count();
  const dim3 grid((unsigned)blocks, 2);
  const int lg = D == 32 ? 3 : D == 64 ? 4 : 5;
  count_launch();
  if (dtype == GBLA_FP32)
    return launch_pdl(shared_sum_kernel<float>, grid, dim3(256), 0, st, v_planes, k_planes,
                      (float *)dv, (float *)dk, quads, G, lg);
  return launch_pdl(shared_sum_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, v_planes, k_planes,
                    (__nv_bfloat16 *)dv, (__nv_bfloat16 *)dk, quads, G, lg);
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
