// Decayed linear attention on tensor cores (tcgen05 + TMA): bf16, every D.
//
// The scan of ScanArgs in chunks of C = 64 tokens, in scan order.  With r, j the
// places in a chunk, S the state before it and gamma the head's decay,
//   scores  A_rj  = x_r . y_j                        (M64 N64 KD)
//   results out_r = scale [ sum_j (w_rj A_rj) z_j + u_r x_r^T S ]
//                                                    (M64 ND K64, M64 ND KD)
//   state   S'    = c S + sum_j (v_j y_j) z_j^T      (MD ND K64, a time for each term)
// forward: w = gamma^{r-j} (j <= r), u = gamma^{r+1}, v = gamma^{n-1-j}, c = gamma^n
// for n tokens in the chunk; reverse: w = gamma^{j-r} (j >= r), u = gamma^{64-r},
// v = gamma^j, c = gamma^64, and u = gamma^{n-1-r}, c = gamma^{n-1} in the first
// chunk, whose state before it (the gradient of the final state) belongs to the
// last token itself.
//
// Rounding: the weighted scores and the state as it meets a query are rounded
// once to bf16, in the gradients too: the product that reads them takes bf16, and
// the results are rounded to bf16 themselves.  Against 64 bits the results are
// 2.35e-3 of their norm off, 1.66e-3 by their own rounding alone, which is what the
// CUDA-core family leaves (its scores and state stay in fp32).  The state is held in
// fp32 registers and is never rebuilt from rounded values: v_j y_j goes into the
// product as a sum of bf16 numbers, two (2^-17 of a term) where the state only
// serves the results, three (the term rounded to fp32 once, 2^-24) where it is a
// result itself.  The decay powers are fp32.
//
// One CTA scans a run of chunks (a segment) of one (batch, head).  A sequence is
// cut into several where whole ones would leave SMs idle or one long sequence
// would outlast the rest; a first kernel then sums the state of every segment but
// the last in scan order (y and z alone, the chunk that the scan starts with read
// last, so that it is still in L2), a second one turns them into the states before
// the segments, and the scan starts from those.  Each launch begins while the one
// before it ends.
//
// What bounds a chunk (D = 64): memory takes 32 KB of it, 1430 cycles of an SM's
// share of the measured bandwidth; shared memory some 144 KB (operands of the
// MMAs 64, weighted keys 24, loads 24, scores, state and staged results 32), 1150;
// the tensor pipe 650 at M = 64 (33 cycles an MMA of N = 64, 65 of N = 128).  Hence
// C = 64 and not 128: twice the tokens would read the keys' and values' tiles half
// as often, but the scores would be written and read for twice the pairs.  And so
// y's tile and the state (transposed) lie one behind the other, and scores and
// x_r^T S are one product of N = 128 that reads x once; the terms of the state's
// product are side by side in one of N = 128 in the same way.  Measured: B19 H8
// N4096 (one whole sequence an SM) 55 us, 5.8 TB/s, 85 % of the measured copy rate;
// B2 H8 N32768, where segments cost y and z twice, 82 us, 3.3 TB/s of what the
// operation needs.  D = 128 has operands twice as wide for a state four times as
// large: 336 KB and 2600 cycles of shared memory against 2870 of memory, 127 us at
// B19 H8 N4096 (74 %).
//
// Warps of the scan: 0-3 weight the scores, 4-7 form v_j y_j, the next 4 (D = 128:
// 8) hold the state, the next 4 write results, then one warp issues the TMA loads (a
// lane for each 64-channel block of each tensor: one thread issues a box in half
// a microsecond) and one the MMAs (one elected lane: issued from a plain branch on
// the lane number, each MMA took 160 cycles).  M = 64 accumulators lie in lanes 0-15
// of each TMEM quarter and are read with the 16-lane shapes.
//
// Every mbarrier wait is bounded (2 s); one that runs out sets a bit in
// g_decay_error and raises the CTA's abort flag.
#include <mutex>

#include "gbla_decay.cuh"
#include "gbla_internal.cuh"
#include "gbla_sm100.cuh"

namespace gbla {

__device__ unsigned int g_decay_error;

namespace {

using namespace sm100;

constexpr int kC = 64;                 // tokens per chunk
constexpr int kBlk = kC * 128;         // 8 KB: 64 tokens x 64 channels, 128B swizzle

template <int D, int kTerms>
struct Shape {
  static constexpr bool kMerged = D == 64;                 // scores and inter results in one MMA
  static constexpr int kB = D / 64;                        // 64-channel blocks
  static constexpr int kTile = kB * kBlk;                  // one tensor's chunk
  static constexpr int kSBytes = D * D * 2;                // the state rounded to bf16
  // rings of x, y and z tiles; merged: the state's tile follows y's in its slot
  static constexpr int kNX = D == 64 ? 4 : 2, kNY = D == 64 ? (kTerms == 2 ? 5 : 4) : 3,
                       kNZ = D == 64 ? (kTerms == 2 ? 6 : 5) : (kTerms == 2 ? 4 : 3);
  static constexpr int kYSlot = kTile + (kMerged ? kSBytes : 0);
  static constexpr int kConv = D == 64 ? 2 : 1;            // buffers of v_j y_j
  static constexpr int kP = D == 64 ? 2 : 1;               // of weighted scores
  static constexpr int kOffX = 0, kOffY = kOffX + kNX * kTile, kOffZ = kOffY + kNY * kYSlot;
  static constexpr int kOffConv = kOffZ + kNZ * kTile;
  static constexpr int kOffP = kOffConv + kConv * kTerms * kTile;
  static constexpr int kOffS = kOffP + kP * kBlk;
  static constexpr int kOffOut = kOffS + (kMerged ? 0 : kSBytes);  // 2 KB a result warp
  static constexpr int kOffBar = kOffOut + kBlk;
  static constexpr int kBars = 2 * (kNX + kNY + kNZ + kConv + kP) + 2 * 5 + 3;
  static constexpr int kOffMisc = kOffBar + kBars * 8;
  static constexpr int kSmem = kOffMisc + 16 + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr int kSWarps = D == 64 ? 4 : 8;
  static constexpr int kOutWarp = 8 + kSWarps, kTmaWarp = kOutWarp + 4, kMmaWarp = kTmaWarp + 1;
  static constexpr int kThreads = (kMmaWarp + 1) * 32;
  static constexpr int kLoads = 3 * kB;                    // issuing lanes
  // TMEM columns.  Merged: two buffers of scores | inter results, two of intra
  // results, the chunk's state (its large and its small terms side by side).
  // Else two of scores, two of results (inter, weighted in place, then intra
  // added), the chunk's state.
  static constexpr uint32_t kColSc = 0, kScStep = kMerged ? 128 : 64;
  static constexpr uint32_t kColInter = kMerged ? 64 : 128, kInterStep = 128;
  static constexpr uint32_t kColIntra = kMerged ? 256 : 128, kIntraStep = kMerged ? 64 : 128;
  static constexpr uint32_t kColDs = 384;
};

struct TcParams {
  void *out;
  const float *log_decay;
  const int32_t *seq_lens;
  const float *init;
  float *fin, *part;
  float init_scale, fin_scale, scale;
  int N, H, gx, gy, gz;
  int seg, ranks;  // chunks of a segment, most segments of a sequence
  bool zero_pad, init_t, reverse;
  bool before;     // `part` holds the states before the segments, not their own
};

__device__ __forceinline__ void decay_error(unsigned code, const AbortFlag &ab) {
  if (!ab.raised()) atomicOr(&g_decay_error, code);
  ab.raise();
}

// 16 lanes x 64 columns: thread t gets rows t / 4 (v[4 i], v[4 i + 1]) and
// t / 4 + 8 (v[4 i + 2], v[4 i + 3]), columns 8 i + 2 (t % 4) and the next.
__device__ __forceinline__ void tmem_ld_16x64(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st_16x64(uint32_t taddr, const float (&v)[32]) {
  uint32_t r[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(v[i]);
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// The warp's 16 x 64 values in the layout above, as bf16 into 16 rows of 128
// bytes (128-byte swizzle; the first row a multiple of 8 of the tile).
__device__ __forceinline__ void store_16x64(uint32_t rows, int lane, const float (&v)[32]) {
  const uint32_t row = rows + (lane & 15) * 128;  // lane l: row l % 16, piece k + l / 16
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    const uint32_t at = row + (((k + (lane >> 4)) ^ (lane & 7)) << 4);
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at),
                 "r"(f2_to_bf2(v[4 * k], v[4 * k + 1])), "r"(f2_to_bf2(v[4 * k + 2], v[4 * k + 3])),
                 "r"(f2_to_bf2(v[4 * k + 4], v[4 * k + 5])),
                 "r"(f2_to_bf2(v[4 * k + 6], v[4 * k + 7]))
                 : "memory");
  }
}
// The same transposed: the values' rows become 16 columns of a tile of 64 rows of
// 128 bytes, from its 16-byte piece `piece` on.
__device__ __forceinline__ void store_16x64_t(uint32_t tile, int piece, int lane,
                                              const float (&v)[32]) {
  // lane l: the row 8 (k + l / 16) + l % 8 of the tile, piece + (l / 8) % 2 of it
  const uint32_t row = tile + (8 * (lane >> 4) + (lane & 7)) * 128 +
                       (((piece + ((lane >> 3) & 1)) ^ (lane & 7)) << 4);
#pragma unroll
  for (int k = 0; k < 8; k += 2)
    asm volatile(
        "stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(row + k * 1024),
        "r"(f2_to_bf2(v[4 * k], v[4 * k + 1])), "r"(f2_to_bf2(v[4 * k + 2], v[4 * k + 3])),
        "r"(f2_to_bf2(v[4 * k + 4], v[4 * k + 5])), "r"(f2_to_bf2(v[4 * k + 6], v[4 * k + 7]))
        : "memory");
}
// A result warp's 16 x 64 values (rows 16 ow on of the chunk, the first n of its
// rows valid) to rows of `orow` values; bf16 as whole 128-byte rows through the
// warp's 2 KB of staging.
template <int V, typename O>
__device__ __forceinline__ void write_rows(O *dst, size_t orow, uint32_t stage, int ow, int lane,
                                           int n, const float (&a)[32]) {
  if constexpr (sizeof(O) == 4) {
    const int r0 = 16 * ow + (lane >> 2);
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (r0 + 8 * q < n && 8 * k < V)
          *(float2 *)(dst + (size_t)(r0 + 8 * q) * orow + 8 * k + 2 * (lane & 3)) =
              make_float2(a[4 * k + 2 * q], a[4 * k + 2 * q + 1]);
  } else {
    __syncwarp();
    store_16x64(stage, lane, a);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = (lane >> 3) + 4 * k;
      const uint4 v = lds_v4(stage + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
      if (16 * ow + r < n && 8 * (lane & 7) < V)
        *(uint4 *)(dst + (size_t)(16 * ow + r) * orow + 8 * (lane & 7)) = v;
    }
  }
}
__device__ __forceinline__ uint32_t bf2_mul(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t bf2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// Shared-memory matrix descriptor (128-byte swizzle) of a tile, and the same
// moved by a constant number of bytes: the address field's carry never leaves
// the low word, so a step costs one addition.
__device__ __forceinline__ uint64_t desc_at(uint64_t d, uint32_t bytes) {
  return (d & 0xFFFFFFFF00000000ull) | (uint32_t)((uint32_t)d + (bytes >> 4));
}
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(r));
  return r != 0;
}

// A row's weight: for two terms as a sum of two bf16 numbers, doubled up.
struct RowWeight {
  float f;
  uint32_t hi, lo;
  __device__ __forceinline__ void set(float w) {
    f = w;
    hi = f2_to_bf2(w, w);
    const float rest = w - bf2_to_f2(hi).x;
    lo = f2_to_bf2(rest, rest);
  }
};
// 8 values of y times a row's weight as sums of kTerms bf16 numbers, one in each
// tile from `to` on.  Two terms stay in packed bf16: h = rn(y hi), y hi - h is
// exact, l = rn(y lo + that).
template <int kTerms, int kTile>
__device__ __forceinline__ void weigh_piece(const uint4 &u, const RowWeight &w, uint32_t to) {
  const uint32_t in[4] = {u.x, u.y, u.z, u.w};
  uint32_t o[kTerms][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (kTerms == 2) {
      o[0][e] = bf2_mul(in[e], w.hi);
      o[1][e] = bf2_fma(in[e], w.lo, bf2_fma(in[e], w.hi, o[0][e] ^ 0x80008000u));
    } else {
      float2 f = bf2_to_f2(in[e]);
      f.x *= w.f, f.y *= w.f;
#pragma unroll
      for (int t = 0; t < kTerms; ++t) {
        o[t][e] = f2_to_bf2(f.x, f.y);
        if (t + 1 < kTerms) {
          const float2 q = bf2_to_f2(o[t][e]);
          f.x -= q.x, f.y -= q.y;  // exact
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < kTerms; ++t)
    sts_v4(to + t * kTile, make_uint4(o[t][0], o[t][1], o[t][2], o[t][3]));
}
// The chunk that holds the sequence's end, from its n valid tokens: keys, values
// and weighted keys past the end become 0 (padding may hold NaN).  ys, zs, cs:
// the thread's piece of row rr; rows rr + 16 k.
template <int kTerms, int kTile>
__device__ __forceinline__ void weigh_end(uint32_t ys, uint32_t zs, uint32_t cs, int rr, int n,
                                          float l2, float gain, bool reverse) {
  const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll 1
  for (int k = 0; k < 4 * kTile / kBlk; ++k) {
    const int r = rr + 16 * (k & 3), off = (k >> 2) * kBlk + (k & 3) * 2048;
    if (r < n) {
      RowWeight w;
      w.set(gain * decay_pow(l2, (float)(reverse ? r : n - 1 - r)));
      weigh_piece<kTerms, kTile>(lds_v4(ys + off), w, cs + off);
      continue;
    }
    sts_v4(ys + off, zero);
    sts_v4(zs + off, zero);
#pragma unroll
    for (int t = 0; t < kTerms; ++t) sts_v4(cs + t * kTile + off, zero);
  }
}

// The chunk's own state, sum of (v_j y_j) z_j^T, into (keep: added to) the
// columns at d.  D = 64: transposed (M = e), the first two terms side by side in
// N, the third onto the second; D = 128: all onto one another, the small first.
template <int D, int kTerms, int kTile>
__device__ __forceinline__ void state_product(uint32_t d, uint32_t zs, uint32_t cs, bool keep) {
  const uint64_t zd = sw128_desc(zs, kBlk, 1024), cd = sw128_desc(cs, kBlk, 1024);
  if constexpr (D == 64) {
    constexpr uint32_t id2 = idesc_bf16_f32(64, 128, 1, 1), id1 = idesc_bf16_f32(64, 64, 1, 1);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      mma_bf16(d, desc_at(zd, k * 2048), desc_at(cd, k * 2048), id2, keep || k != 0);
    if constexpr (kTerms == 3)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        mma_bf16(d + 64, desc_at(zd, k * 2048), desc_at(cd, 2 * kTile + k * 2048), id1, 1);
  } else {
    constexpr uint32_t id_s = idesc_bf16_f32(D, D, 1, 1);
#pragma unroll
    for (int t = kTerms - 1; t >= 0; --t)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        mma_bf16(d, desc_at(cd, t * kTile + k * 2048), desc_at(zd, k * 2048), id_s,
                 keep || t != kTerms - 1 || k != 0);
  }
}

// Place of a state thread's value i: D = 64, held transposed, as tmem_ld_16x64
// gives it (rows e); D = 128, one row d and 64 columns.
template <int D>
__device__ __forceinline__ int state_at(int sw, int lane, int i, int *e) {
  if (D == 64) {
    *e = 16 * sw + (lane >> 2) + 8 * ((i >> 1) & 1);
    return 8 * (i >> 2) + 2 * (lane & 3) + (i & 1);
  }
  *e = 64 * (sw >> 2) + i;
  return 32 * (sw & 3) + lane;
}

// A state thread's value i of the scan's first state (V: its size in memory).
template <int D, int V>
__device__ __forceinline__ float first_state(const TcParams &p, size_t bh, int sw, int lane,
                                             int i) {
  int e;
  const int d = state_at<D>(sw, lane, i, &e);
  if (V < D && (d >= V || e >= V)) return 0.f;
  return p.init_scale * __ldg(p.init + bh * V * V + (p.init_t ? e * V + d : d * V + e));
}

// S = S + f v (own) or S = f S + v over a state thread's values, from the columns
// at src (D = 64: the small terms' columns first).
template <int D, bool kOwn, int kNV>
__device__ __forceinline__ void take_state(float (&S)[kNV], uint32_t src, DecayFactor f) {
  const float2 f2 = make_float2(f.hi, f.hi), g2 = make_float2(f.lo, f.lo);
  auto add = [&](int i, float2 v) {
    const float2 q = make_float2(S[i], S[i + 1]);
    const float2 r = kOwn ? __ffma2_rn(f2, v, q) : __ffma2_rn(f2, q, __ffma2_rn(g2, q, v));
    S[i] = r.x, S[i + 1] = r.y;
  };
  if constexpr (D == 64) {
    float small[32], large[32];
    tmem_ld_16x64(src + 64, small);
    tmem_ld_16x64(src, large);
    tmem_ld_wait_regs(small);
    tmem_pin(large);
#pragma unroll
    for (int i = 0; i < 32; i += 2) add(i, make_float2(small[i], small[i + 1]));
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      if (kOwn) {
        add(i, make_float2(large[i], large[i + 1]));
      } else {
        const float2 r = __fadd2_rn(make_float2(S[i], S[i + 1]), make_float2(large[i], large[i + 1]));
        S[i] = r.x, S[i + 1] = r.y;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {  // (16 at a time spilled)
      float v[8];
      tmem_ld8(src + 8 * k, v);
      tmem_ld_wait_regs(v);
#pragma unroll
      for (int e = 0; e < 8; e += 2) add(8 * k + e, make_float2(v[e], v[e + 1]));
    }
  }
}

// The CTA's segment in scan order: places [q0, q0 + cnt) of the nc chunks.
struct Segment {
  int L, nc, q0, cnt;
  bool last, reverse;
  __device__ __forceinline__ Segment(const TcParams &p, int b, int rank) : reverse(p.reverse) {
    L = p.seq_lens == nullptr ? p.N : min(max(p.seq_lens[b], 0), p.N);
    nc = (L + kC - 1) / kC;
    q0 = rank * p.seg;
    cnt = max(0, min(p.seg, nc - q0));
    last = cnt > 0 && q0 + cnt == nc;
  }
  __device__ __forceinline__ int token_of(int place) const {
    return (reverse ? nc - 1 - place : place) * kC;
  }
  // Tokens that the first state decays by before the segment (in reverse it belongs to
  // the last token).
  __device__ __forceinline__ int tokens_before() const {
    return !reverse ? q0 * kC : q0 == 0 ? 0 : L - 1 - (nc - q0) * kC;
  }
};

// D = 64: the state before segment `rank`, from part or from the segments' own
// states and the first one, into S = 0.
template <int V>
__device__ __forceinline__ void start_state(float (&S)[32], const TcParams &p, const Segment &sg,
                                            size_t bh, int rank, int sw, int lane, float l2) {
  if (p.ranks > 1) {
    grid_dep_wait();
    const float *part = p.part + bh * p.ranks * 64 * 64 + 32 * sw + lane;
    const int end = p.before ? rank + 1 : rank;
    for (int s = p.before ? rank : 0; s < end; ++s) {
      const float f = decay_pow(l2, (float)(end - 1 - s) * p.seg * kC);
#pragma unroll
      for (int i = 0; i < 32; ++i) S[i] = fmaf(f, __ldcg(part + ((size_t)s * 32 + i) * 128), S[i]);
    }
  }
  if (p.init && !p.before) {
    const float f = decay_pow(l2, (float)sg.tokens_before());
#pragma unroll
    for (int i = 0; i < 32; ++i) S[i] = fmaf(f, first_state<64, V>(p, bh, sw, lane, i), S[i]);
  }
}

// ---------------------------------------------------------------------------
// The state of each segment but the last, without what comes before it.  Chunks
// go by from the segment's end in scan order to its start; kGroup of them add up
// in TMEM (their distance from the first is in the weights), then the state warps
// take the sum.  (The tensor cores' sums are cut, not rounded: where the state is a
// result, 96 additions in a row showed at 1e-6 of it, so there are fewer.)  Warps:
// 0-7 form v_j y_j (two groups, alternate chunks), the next 4 (D = 128: 8) hold the
// state, then loads and MMAs.

template <int D, int kTerms>
struct OwnShape {
  static constexpr int kGroup = kTerms == 3 ? 2 : 8;
  static constexpr int kB = D / 64, kTile = kB * kBlk;
  // Even, so that a slot always meets the same one of the two groups: a parity
  // wait tells a phase from the one before it only, and a group that missed a
  // phase of a slot would take an old one for the one it waits for.
  static constexpr int kNY = 4, kNZ = 4;
  static constexpr int kOffY = 0, kOffZ = kNY * kTile, kOffConv = kOffZ + kNZ * kTile;
  static constexpr int kOffBar = kOffConv + 2 * kTerms * kTile;
  static constexpr int kBars = 2 * (kNY + kNZ) + 2 * 4 + 1;
  static constexpr int kOffMisc = kOffBar + kBars * 8;
  static constexpr int kSmem = kOffMisc + 16 + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr int kSWarps = D == 64 ? 4 : 8;
  static constexpr int kTmaWarp = 8 + kSWarps, kMmaWarp = kTmaWarp + 1;
  static constexpr int kThreads = (kMmaWarp + 1) * 32;
  static constexpr int kLoads = 2 * kB;
  static constexpr uint32_t kTmemCols = 256;  // two buffers of 128
  static constexpr int kPerSm = D == 64 && kTerms == 2 ? 2 : 1;  // as the shared memory allows
};

template <int D, int kTerms>
__global__ void __launch_bounds__(OwnShape<D, kTerms>::kThreads, OwnShape<D, kTerms>::kPerSm)
    own_state_kernel(const TcParams p, const __grid_constant__ CUtensorMap tm_y,
                     const __grid_constant__ CUtensorMap tm_z) {
  using Sh = OwnShape<D, kTerms>;
  constexpr int kNV = D == 64 ? 32 : 64;
  grid_dep_launch();
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t *fy = (uint64_t *)(smem + Sh::kOffBar), *ey = fy + Sh::kNY, *fz = ey + Sh::kNY,
           *ez = fz + Sh::kNZ, *conv_full = ez + Sh::kNZ, *conv_empty = conv_full + 2,
           *ds_full = conv_empty + 2, *ds_empty = ds_full + 2, *drained = ds_empty + 2;
  uint32_t *tmem_slot = (uint32_t *)(smem + Sh::kOffMisc);
  const AbortFlag ab{smem_u32(smem + Sh::kOffMisc + 4)};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const Segment sg(p, b, rank);
  if (sg.cnt == 0 || sg.last) return;
  const float l2 = __ldg(p.log_decay + h) * 1.4426950408889634f;

  // The loading warp sets the barriers up and starts at once; the others also wait
  // for the TMEM allocation.
  if (warp == Sh::kTmaWarp && lane == 0) {
    *(volatile int *)(smem + Sh::kOffMisc + 4) = 0;
    for (int i = 0; i < Sh::kNY; ++i) mbar_init(&fy[i], Sh::kB), mbar_init(&ey[i], 1);
    for (int i = 0; i < Sh::kNZ; ++i) mbar_init(&fz[i], Sh::kB), mbar_init(&ez[i], 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&conv_full[i], 4);
      mbar_init(&conv_empty[i], 1);
      mbar_init(&ds_full[i], 1);
      mbar_init(&ds_empty[i], Sh::kSWarps);
    }
    mbar_init(drained, 1);
    fence_mbar_init();
  }
  if (warp == Sh::kTmaWarp && lane == 0) {
    tma_prefetch_desc(&tm_y);
    tma_prefetch_desc(&tm_z);
  }
  if (warp == Sh::kMmaWarp) tmem_alloc(tmem_slot, Sh::kTmemCols);
  if (warp == Sh::kTmaWarp) {
    __syncwarp();
    named_barrier_arrive(1, Sh::kThreads);
  } else {
    tc_fence_before();
    named_barrier(1, Sh::kThreads);
    tc_fence_after();
  }
  const uint32_t tmem = *tmem_slot;
  auto token_at = [&](int g) { return sg.token_of(sg.q0 + sg.cnt - 1 - g); };

  if (warp == Sh::kTmaWarp) {
    if (lane < Sh::kLoads) {
      const int t = lane / Sh::kB, blk = lane % Sh::kB;
      const CUtensorMap *tm = t == 0 ? &tm_y : &tm_z;
      const int hd = h / (t == 0 ? p.gy : p.gz), slots = t == 0 ? Sh::kNY : Sh::kNZ;
      uint64_t *f = t == 0 ? fy : fz, *e = t == 0 ? ey : ez;
      uint8_t *to = smem + (t == 0 ? Sh::kOffY : Sh::kOffZ) + blk * kBlk;
      int i = 0;
      for (; i < sg.cnt; ++i) {
        const int s = i % slots;
        if (!mbar_wait(&e[s], ((i / slots) & 1) ^ 1, &ab)) {
          decay_error(1, ab);
          break;
        }
        mbar_arrive_expect_tx(&f[s], kBlk);
        tma_load_4d(to + s * Sh::kTile, tm, &f[s], blk * 64, hd, token_at(i), b);
      }
      if (i < sg.cnt)  // gave up: no copy may land after the CTA is gone
        for (int k = max(0, i - slots); k < i; ++k)
          mbar_wait(&f[k % slots], (k / slots) & 1, nullptr);
    }
    __syncwarp();
  } else if (warp == Sh::kMmaWarp) {
    if (elect_one()) {
      const uint32_t base = smem_u32(smem);
      bool ok = true;
      auto wait = [&](uint64_t *m, uint32_t parity) {
        if (ok && !mbar_wait(m, parity, &ab)) decay_error(2, ab), ok = false;
        return ok;
      };
      for (int g = 0; g < sg.cnt && ok; ++g) {
        const int cb = g & 1, q = g / Sh::kGroup, db = q & 1;
        if (g % Sh::kGroup == 0 && q >= 2 && !wait(&ds_empty[db], ((q >> 1) & 1) ^ 1)) break;
        if (!wait(&conv_full[cb], (g >> 1) & 1)) break;
        tc_fence_after();
        state_product<D, kTerms, Sh::kTile>(
            tmem + 128 * db, base + Sh::kOffZ + (g % Sh::kNZ) * Sh::kTile,
            base + Sh::kOffConv + cb * kTerms * Sh::kTile, g % Sh::kGroup != 0);
        mma_commit(&conv_empty[cb]);
        mma_commit(&ey[g % Sh::kNY]);
        mma_commit(&ez[g % Sh::kNZ]);
        if (g % Sh::kGroup == Sh::kGroup - 1 || g == sg.cnt - 1) mma_commit(&ds_full[db]);
      }
      mma_commit(drained);  // nothing is in flight when TMEM is freed
      if (!mbar_wait(drained, 0, nullptr)) decay_error(512, ab);
    }
    __syncwarp();
  } else if (warp < 8) {
    const int ct = tid & 127, ch = ct & 7, rr = ct >> 3;
    float wr[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      wr[k] = decay_pow(l2, (float)(p.reverse ? rr + 16 * k : kC - 1 - rr - 16 * k));
    const uint32_t piece = rr * 128 + ((ch ^ (rr & 7)) << 4);
    for (int g = warp >> 2; g < sg.cnt; g += 2) {
      const int sy = g % Sh::kNY, sz = g % Sh::kNZ, cb = g & 1;
      const int n = min(kC, sg.L - token_at(g));
      const float gain = decay_pow(l2, (float)(g % Sh::kGroup) * kC);
      if (!mbar_wait(&fy[sy], (g / Sh::kNY) & 1, &ab)) decay_error(16, ab);
      if (!mbar_wait(&fz[sz], (g / Sh::kNZ) & 1, &ab)) decay_error(16, ab);  // for the MMAs
      if (g >= 2 && !mbar_wait(&conv_empty[cb], ((g >> 1) & 1) ^ 1, &ab)) decay_error(32, ab);
      const uint32_t ys = smem_u32(smem + Sh::kOffY + sy * Sh::kTile) + piece;
      const uint32_t cs = smem_u32(smem + Sh::kOffConv + cb * kTerms * Sh::kTile) + piece;
      if (n == kC) {
        RowWeight w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k].set(gain * wr[k]);
#pragma unroll
        for (int blk = 0; blk < Sh::kB; ++blk) {
          uint4 u[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) u[k] = lds_v4(ys + blk * kBlk + k * 2048);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            weigh_piece<kTerms, Sh::kTile>(u[k], w[k], cs + blk * kBlk + k * 2048);
        }
      } else {
        weigh_end<kTerms, Sh::kTile>(ys, smem_u32(smem + Sh::kOffZ + sz * Sh::kTile) + piece, cs, rr,
                                     n, l2, gain, p.reverse);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&conv_full[cb]);
    }
  } else {
    const int sw = warp - 8, st = tid - 8 * 32;
    const uint32_t src = tmem + ((uint32_t)(32 * (sw & 3)) << 16) + (D == 64 ? 0 : 64 * (sw >> 2));
    float S[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) S[i] = 0.f;
    for (int q = 0; q * Sh::kGroup < sg.cnt; ++q) {
      if (!mbar_wait(&ds_full[q & 1], (q >> 1) & 1, &ab)) decay_error(64, ab);
      tc_fence_after();
      take_state<D, true>(S, src + 128 * (q & 1), {decay_pow(l2, (float)q * (Sh::kGroup * kC)), 0.f});
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ds_empty[q & 1]);
    }
    float *part = p.part + (((size_t)b * p.H + h) * p.ranks + rank) * D * D + st;
#pragma unroll
    for (int i = 0; i < kNV; ++i) part[i * Sh::kSWarps * 32] = S[i];
  }
  tc_fence_before();
  __syncthreads();
  if (warp == Sh::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, Sh::kTmemCols);
  }
}

// ---------------------------------------------------------------------------
// The state before each segment in place of its own state, from the scan's first
// state on: for each value the segments go by in scan order, 8 loads at a time.
// D = 64 up to 12 segments: without this launch, the scan's state warps sum the
// segments before theirs while others still run (9: B2 H8 N32768 81 us, with it 84; 32:
// B1 H4 N32768 42 us, with it 33).  At D = 128 they have no registers for enough loads
// in flight (4.5 us a segment; 32 of them: B1 H3 N8192 101 us, with this launch 25; 9:
// B2 H8 N16384 108 and 93; 2: B8 H8 N2048 54 and 56).
template <int D, int V>
__global__ void __launch_bounds__(256) before_kernel(const TcParams p) {
  constexpr int kT = D == 64 ? 128 : 256, kBatch = 8;  // the state's threads in a scan
  grid_dep_launch();
  const int h = blockIdx.y, b = blockIdx.z, at = (blockIdx.x * 256 + threadIdx.x) * 4;
  const size_t bh = (size_t)b * p.H + h;
  const Segment sg(p, b, 0);
  const int ns = max(1, (sg.nc + p.seg - 1) / p.seg);
  float S[4] = {};
  if (p.init)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      S[c] = first_state<D, V>(p, bh, (at + c) % kT >> 5, (at + c) & 31, at / kT);
  // tokens of the first segment that the first state decays by (reverse: it belongs
  // to the last token), and of the others
  const float ld = __ldg(p.log_decay + h);
  const int first = p.reverse ? sg.L - 1 - (sg.nc - p.seg) * kC : p.seg * kC;  // as tokens_before
  const DecayFactor w0 = decay_factor(ld * first), w1 = decay_factor(ld * (p.seg * kC));
  float *part = p.part + bh * p.ranks * D * D + at;
  grid_dep_wait();  // also with one segment: a grid never ends before the kernels ahead of it
  for (int r0 = 0; r0 < ns; r0 += kBatch) {
    float4 own[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      own[u] = r0 + u + 1 < ns ? __ldcg((const float4 *)(part + (size_t)(r0 + u) * D * D))
                               : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int r = r0 + u;
      if (r >= ns) break;
      *(float4 *)(part + (size_t)r * D * D) = make_float4(S[0], S[1], S[2], S[3]);
      const DecayFactor w = r == 0 ? w0 : w1;
      S[0] = fmaf(w.hi, S[0], fmaf(w.lo, S[0], own[u].x));
      S[1] = fmaf(w.hi, S[1], fmaf(w.lo, S[1], own[u].y));
      S[2] = fmaf(w.hi, S[2], fmaf(w.lo, S[2], own[u].z));
      S[3] = fmaf(w.hi, S[3], fmaf(w.lo, S[3], own[u].w));
    }
  }
}

// ---------------------------------------------------------------------------
// The scan of each segment.  V: the heads' size in memory (32 runs as D = 64 with
// the missing channels loaded as zeros).
template <int D, int V, int kTerms, typename O>
__global__ void __launch_bounds__(Shape<D, kTerms>::kThreads, 1)
    decay_kernel(const TcParams p, const __grid_constant__ CUtensorMap tm_x,
                 const __grid_constant__ CUtensorMap tm_y,
                 const __grid_constant__ CUtensorMap tm_z) {
  using Sh = Shape<D, kTerms>;
  constexpr int kNV = D == 64 ? 32 : 64;  // state values a thread
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t *bar = (uint64_t *)(smem + Sh::kOffBar);
  // *_ready: everything that its MMAs wait for, on one barrier (a wait costs the
  // issuing thread more than an MMA)
  uint64_t *fx = bar, *ex = fx + Sh::kNX, *fy = ex + Sh::kNX, *ey = fy + Sh::kNY, *fz = ey + Sh::kNY, *ez = fz + Sh::kNZ,
           *state_ready = ez + Sh::kNZ, *conv_empty = state_ready + Sh::kConv,
           *intra_ready = conv_empty + Sh::kConv, *p_empty = intra_ready + Sh::kP,
           *score_ready = p_empty + Sh::kP, *sc_full = score_ready + 2,
           *inter_ready = sc_full + 2, *inter_full = inter_ready + 2, *o_full = inter_full + 2,
           *s_empty = o_full + 2, *ds_full = s_empty + 1, *drained = ds_full + 1;
  uint32_t *tmem_slot = (uint32_t *)(smem + Sh::kOffMisc);
  const AbortFlag ab{smem_u32(smem + Sh::kOffMisc + 4)};

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.y, b = blockIdx.z;
  const int rank = blockIdx.x;
  const Segment sg(p, b, rank);
  const int L = sg.L, q0 = sg.q0, cnt = sg.cnt;
  const size_t bh = (size_t)b * p.H + h, orow = (size_t)p.H * V;
  O *out = (O *)p.out + ((size_t)b * p.N * p.H + h) * V;  // token t at t * orow

  if (p.zero_pad) {  // the rows past the end, shared among the sequence's CTAs
    constexpr int kPer = V * (int)sizeof(O) / 16;
    for (long long i = (long long)rank * Sh::kThreads + tid; i < (long long)(p.N - L) * kPer;
         i += (long long)p.ranks * Sh::kThreads)
      ((uint4 *)(out + (L + i / kPer) * orow))[i % kPer] = make_uint4(0, 0, 0, 0);
  }
  if (cnt == 0) {
    if (p.ranks > 1) grid_dep_wait();  // a grid never ends before the kernels ahead of it
    if (rank == 0 && p.fin)  // an empty sequence passes its state on
      for (int i = tid; i < V * V; i += Sh::kThreads)
        p.fin[bh * V * V + i] = p.init ? p.init[bh * V * V + i] * p.init_scale * p.fin_scale : 0.f;
    return;
  }
  const float l2 = __ldg(p.log_decay + h) * 1.4426950408889634f;

  // The loading warp sets the barriers up and starts at once; the others also wait
  // for the TMEM allocation.
  if (warp == Sh::kTmaWarp && lane == 0) {
    *(volatile int *)(smem + Sh::kOffMisc + 4) = 0;
    for (int i = 0; i < Sh::kNX; ++i) mbar_init(&fx[i], Sh::kB), mbar_init(&ex[i], 1);
    for (int i = 0; i < Sh::kNY; ++i) mbar_init(&fy[i], Sh::kB), mbar_init(&ey[i], 1);
    for (int i = 0; i < Sh::kNZ; ++i) mbar_init(&fz[i], Sh::kB), mbar_init(&ez[i], 1);
    for (int i = 0; i < Sh::kConv; ++i)  // weighted keys there, last step's state taken
      mbar_init(&state_ready[i], 4 + Sh::kSWarps), mbar_init(&conv_empty[i], 1);
    for (int i = 0; i < Sh::kP; ++i)  // scores weighted, results' columns free (D = 128: weighted)
      mbar_init(&intra_ready[i], 8), mbar_init(&p_empty[i], 1);
    for (int i = 0; i < 2; ++i) {
      // scores' columns free (D = 64: and inter results', state there)
      mbar_init(&score_ready[i], Sh::kMerged ? 12 : 4);
      mbar_init(&inter_ready[i], 4 + Sh::kSWarps);  // D = 128: results' columns free, state there
      mbar_init(&sc_full[i], 1);
      mbar_init(&inter_full[i], 1);
      mbar_init(&o_full[i], 1);
    }
    mbar_init(s_empty, 1);
    mbar_init(ds_full, 1);
    mbar_init(drained, 1);
    fence_mbar_init();
  }
  if (warp == Sh::kTmaWarp && lane == 0) {
    tma_prefetch_desc(&tm_x);
    tma_prefetch_desc(&tm_y);
    tma_prefetch_desc(&tm_z);
  }
  if (warp == Sh::kMmaWarp) tmem_alloc(tmem_slot, 512);
  if (warp == Sh::kTmaWarp) {
    __syncwarp();
    named_barrier_arrive(1, Sh::kThreads);
  } else {
    tc_fence_before();
    named_barrier(1, Sh::kThreads);
    tc_fence_after();
  }
  const uint32_t tmem = *tmem_slot;
  if (warp == Sh::kTmaWarp) {
    // ---------------------------------------------------------------- loads
    if (lane < Sh::kLoads) {
      const int t = lane / Sh::kB, blk = lane % Sh::kB;  // tensor, 64-channel block
      const CUtensorMap *tm = t == 0 ? &tm_x : t == 1 ? &tm_y : &tm_z;
      const int hd = h / (t == 0 ? p.gx : t == 1 ? p.gy : p.gz);
      uint64_t *f = t == 0 ? fx : t == 1 ? fy : fz, *e = t == 0 ? ex : t == 1 ? ey : ez;
      const int slots = t == 0 ? Sh::kNX : t == 1 ? Sh::kNY : Sh::kNZ;
      uint8_t *to = smem + (t == 0 ? Sh::kOffX : t == 1 ? Sh::kOffY : Sh::kOffZ) + blk * kBlk;
      const int size = t == 1 ? Sh::kYSlot : Sh::kTile;
      int i = 0;
      for (; i < cnt; ++i) {
        const int s = i % slots;
        if (!mbar_wait(&e[s], ((i / slots) & 1) ^ 1, &ab)) {
          decay_error(1, ab);
          break;
        }
        mbar_arrive_expect_tx(&f[s], kBlk);
        tma_load_4d(to + s * size, tm, &f[s], blk * 64, hd, sg.token_of(q0 + i), b);
      }
      if (i < cnt)  // gave up: no copy may land after the CTA is gone
        for (int k = max(0, i - slots); k < i; ++k)
          mbar_wait(&f[k % slots], (k / slots) & 1, nullptr);
    }
    __syncwarp();
  } else if (warp == Sh::kMmaWarp) {
    // ----------------------------------------------------------------- MMAs
    if (elect_one()) {
      const uint32_t base = smem_u32(smem);
      bool ok = true;
      auto wait = [&](uint64_t *m, uint32_t parity) {
        if (ok && !mbar_wait(m, parity, &ab)) decay_error(2, ab), ok = false;
        return ok;
      };
      auto state_mma = [&](int i) {
        const int cb = i % Sh::kConv;
        if (!wait(&fz[i % Sh::kNZ], (i / Sh::kNZ) & 1)) return;
        if (!wait(&state_ready[cb], (i / Sh::kConv) & 1)) return;
        tc_fence_after();
        state_product<D, kTerms, Sh::kTile>(
            tmem + Sh::kColDs, base + Sh::kOffZ + (i % Sh::kNZ) * Sh::kTile,
            base + Sh::kOffConv + cb * kTerms * Sh::kTile, false);
        mma_commit(ds_full);
        mma_commit(&conv_empty[cb]);
      };
      // scores of chunk i; merged: and x_r^T S.  The chunk's state
      // went before, so its keys are there and those past the end are zero.
      auto score_mma = [&](int i) {
        const int sx = i % Sh::kNX, sy = i % Sh::kNY;
        if (!wait(&fx[sx], (i / Sh::kNX) & 1)) return;
        if (!wait(&score_ready[i & 1], (i >> 1) & 1)) return;
        tc_fence_after();
        constexpr uint32_t id = idesc_bf16_f32(64, Sh::kMerged ? 128 : 64, 0, 0);
        const uint64_t xd = sw128_desc(base + Sh::kOffX + sx * Sh::kTile, 16, 1024);
        const uint64_t yd = sw128_desc(base + Sh::kOffY + sy * Sh::kYSlot, 16, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = (k >> 2) * kBlk + (k & 3) * 32;
          mma_bf16(tmem + Sh::kColSc + Sh::kScStep * (i & 1), desc_at(xd, off), desc_at(yd, off), id,
                   k != 0);
        }
        mma_commit(&sc_full[i & 1]);
        mma_commit(&ey[sy]);
        if constexpr (Sh::kMerged) mma_commit(&ex[sx]);
      };
      auto inter_mma = [&](int i) {  // x_r^T S on its own
        const int sx = i % Sh::kNX;
        if (!wait(&inter_ready[i & 1], (i >> 1) & 1)) return;
        tc_fence_after();
        constexpr uint32_t id = idesc_bf16_f32(64, D, 0, 1);
        const uint64_t xd = sw128_desc(base + Sh::kOffX + sx * Sh::kTile, 16, 1024);
        const uint64_t sd = sw128_desc(base + Sh::kOffS, D * 128, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_bf16(tmem + Sh::kColInter + Sh::kInterStep * (i & 1), desc_at(xd, (k >> 2) * kBlk + (k & 3) * 32),
                   desc_at(sd, k * 2048), id, k != 0);
        mma_commit(&inter_full[i & 1]);
        mma_commit(s_empty);
        mma_commit(&ex[sx]);
      };
      auto intra_mma = [&](int j) {  // sum_j (w_rj A_rj) z_j
        const int sz = j % Sh::kNZ, pb = j % Sh::kP, ob = j & 1;
        if (!wait(&intra_ready[pb], (j / Sh::kP) & 1)) return;
        tc_fence_after();
        constexpr uint32_t id = idesc_bf16_f32(64, D, 0, 1);
        const uint64_t pd = sw128_desc(base + Sh::kOffP + pb * kBlk, 16, 1024);
        const uint64_t zd = sw128_desc(base + Sh::kOffZ + sz * Sh::kTile, kBlk, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16(tmem + Sh::kColIntra + Sh::kIntraStep * ob, desc_at(pd, k * 32),
                   desc_at(zd, k * 2048), id, !Sh::kMerged || k != 0);
        mma_commit(&p_empty[pb]);
        mma_commit(&o_full[ob]);
        mma_commit(&ez[sz]);
      };
      state_mma(0);
      // Scores of chunk i, results of chunk i - 1 (whose scores have been
      // weighted meanwhile), state of chunk i + 1 (which leaves a whole round for
      // the state to reach the scores of i + 1).
      for (int i = 0; i <= cnt && ok; ++i) {
        if (i < cnt) score_mma(i);
        if constexpr (!Sh::kMerged)
          if (i < cnt && ok) inter_mma(i);
        if (i >= 1 && ok) intra_mma(i - 1);
        if (i + 1 < cnt && ok) state_mma(i + 1);
      }
      mma_commit(drained);  // nothing is in flight when TMEM is freed
      if (!mbar_wait(drained, 0, nullptr)) decay_error(512, ab);
    }
    __syncwarp();
  } else if (warp < 4) {
    // ------------------------------------------- weighted scores (warps 0-3)
    const int r0 = 16 * warp + (lane >> 2), c = 2 * (lane & 3);
    float2 w[9];  // exponent e0 -+ 8 k, one less (more) for the second column
#pragma unroll
    for (int k = 0; k < 9; ++k) {
      float e[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int n = (p.reverse ? -1 : 1) * (r0 - c - q - 8 * (k - 1));
        e[q] = n >= 0 ? p.scale * decay_pow(l2, (float)n) : 0.f;
      }
      w[k] = make_float2(e[0], e[1]);
    }
    if (lane == 0) mbar_arrive(&score_ready[0]), mbar_arrive(&score_ready[1]);
    for (int i = 0; i < cnt; ++i) {
      const int pb = i % Sh::kP;
      if (!mbar_wait(&sc_full[i & 1], (i >> 1) & 1, &ab)) decay_error(4, ab);
      tc_fence_after();
      float a[32];
      tmem_ld_16x64(tmem + ((uint32_t)(32 * warp) << 16) + Sh::kColSc + Sh::kScStep * (i & 1), a);
      tmem_ld_wait_regs(a);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&score_ready[i & 1]);
      if (i >= Sh::kP && !mbar_wait(&p_empty[pb], ((i / Sh::kP) & 1) ^ 1, &ab)) decay_error(8, ab);
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float2 m = __fmul2_rn(make_float2(a[4 * k + 2 * q], a[4 * k + 2 * q + 1]), w[k + 1 - q]);
          a[4 * k + 2 * q] = m.x, a[4 * k + 2 * q + 1] = m.y;
        }
      store_16x64(smem_u32(smem + Sh::kOffP + pb * kBlk) + 16 * warp * 128, lane, a);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&intra_ready[pb]);
    }
  } else if (warp < 8) {
    // --------------------------------------------- weighted keys (warps 4-7)
    const int ct = tid - 128, ch = ct & 7, rr = ct >> 3;  // 16-byte chunk, first row
    const uint32_t piece = rr * 128 + ((ch ^ (rr & 7)) << 4);
    RowWeight w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[k].set(decay_pow(l2, (float)(p.reverse ? rr + 16 * k : kC - 1 - rr - 16 * k)));
    for (int i = 0; i < cnt; ++i) {
      const int sy = i % Sh::kNY, sz = i % Sh::kNZ, cb = i % Sh::kConv;
      const int n = min(kC, L - sg.token_of(q0 + i));
      if (!mbar_wait(&fy[sy], (i / Sh::kNY) & 1, &ab)) decay_error(16, ab);
      if (i >= Sh::kConv && !mbar_wait(&conv_empty[cb], ((i / Sh::kConv) & 1) ^ 1, &ab))
        decay_error(32, ab);
      const uint32_t ys = smem_u32(smem + Sh::kOffY + sy * Sh::kYSlot) + piece;
      const uint32_t cs = smem_u32(smem + Sh::kOffConv + cb * kTerms * Sh::kTile) + piece;
      if (n == kC) {
#pragma unroll
        for (int blk = 0; blk < Sh::kB; ++blk) {
          uint4 u[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) u[k] = lds_v4(ys + blk * kBlk + k * 2048);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            weigh_piece<kTerms, Sh::kTile>(u[k], w[k], cs + blk * kBlk + k * 2048);
        }
      } else {
        if (!mbar_wait(&fz[sz], (i / Sh::kNZ) & 1, &ab)) decay_error(16, ab);
        weigh_end<kTerms, Sh::kTile>(ys, smem_u32(smem + Sh::kOffZ + sz * Sh::kTile) + piece, cs, rr,
                                     n, l2, 1.f, p.reverse);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&state_ready[cb]);
    }
  } else if (warp < 8 + Sh::kSWarps) {
    // ------------------------------------------------- the state, in registers
    const int sw = warp - 8;
    const DecayFactor chunk_factor = decay_factor(__ldg(p.log_decay + h) * kC);
    float S[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) S[i] = 0.f;
    const uint32_t src = tmem + ((uint32_t)(32 * (sw & 3)) << 16) + Sh::kColDs +
                         (D == 64 ? 0 : 64 * (sw >> 2));
    if (lane == 0) mbar_arrive(&state_ready[0]);
    if constexpr (D == 64) {
      start_state<V>(S, p, sg, bh, rank, sw, lane, l2);
    } else {
      // The state before the segment, or the first one, in one loop: in two they cost the
      // kernel more spilled registers (B19 H8 N4096 132 us, so 127).
      const float *from = nullptr;
      int step = 0;
      float f = 0.f;
      if (p.ranks > 1) {
        grid_dep_wait();
        from = p.part + (bh * p.ranks + rank) * D * D + (tid - 8 * 32), step = Sh::kSWarps * 32;
        f = 1.f;
      } else if (p.init) {
        int e;
        const int d = state_at<D>(sw, lane, 0, &e);
        from = p.init + bh * D * D + (p.init_t ? e * D + d : d * D + e), step = p.init_t ? D : 1;
        f = p.init_scale;
      }
      if (from)
#pragma unroll
        for (int i = 0; i < kNV; ++i, from += step) S[i] = f * __ldcg(from);
    }
    for (int j = 0; j < cnt; ++j) {
      if constexpr (D == 64) {  // behind the chunk's keys, once their slot is free
        const int sy = j % Sh::kNY;
        if (!mbar_wait(&ey[sy], ((j / Sh::kNY) & 1) ^ 1, &ab)) decay_error(128, ab);
        store_16x64(smem_u32(smem + Sh::kOffY + sy * Sh::kYSlot + Sh::kTile) + 16 * sw * 128, lane, S);
      } else {
        if (j >= 1 && !mbar_wait(s_empty, (j & 1) ^ 1, &ab)) decay_error(128, ab);
        const int d = 32 * (sw & 3) + lane;
        const uint32_t row = smem_u32(smem + Sh::kOffS) + (sw >> 2) * (D * 128) + d * 128;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          sts_v4(row + ((k ^ (d & 7)) << 4),
                 make_uint4(f2_to_bf2(S[8 * k], S[8 * k + 1]), f2_to_bf2(S[8 * k + 2], S[8 * k + 3]),
                            f2_to_bf2(S[8 * k + 4], S[8 * k + 5]),
                            f2_to_bf2(S[8 * k + 6], S[8 * k + 7])));
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(Sh::kMerged ? &score_ready[j & 1] : &inter_ready[j & 1]);
      const int t0 = sg.token_of(q0 + j), n = min(kC, L - t0);
      const int span = !p.reverse ? n : (q0 + j == 0 ? n - 1 : kC);
      if (!mbar_wait(ds_full, j & 1, &ab)) decay_error(64, ab);
      tc_fence_after();
      take_state<D, false>(S, src, span == kC ? chunk_factor : one_factor(decay_pow(l2, (float)span)));
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&state_ready[(j + 1) % Sh::kConv]);
    }
    if (p.fin && sg.last) {
      const float f = scaled_pow(p.fin_scale, l2, p.reverse ? 1.f : 0.f);
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        int e;
        const int d = state_at<D>(sw, lane, i, &e);
        if (V == D || (d < V && e < V)) p.fin[bh * V * V + d * V + e] = S[i] * f;
      }
    }
  } else {
    // ---------------------------------------------------------------- results
    const int ow = warp - Sh::kOutWarp, r0 = 16 * ow + (lane >> 2);
    const uint32_t quarter = tmem + ((uint32_t)(32 * ow) << 16);
    const uint32_t stage = smem_u32(smem + Sh::kOffOut + ow * 2048);
    float u[2];  // weights of x_r^T S in the rows r0 and r0 + 8
#pragma unroll
    for (int k = 0; k < 2; ++k)
      u[k] = scaled_pow(p.scale, l2, (float)(p.reverse ? kC - (r0 + 8 * k) : r0 + 8 * k + 1));
    float s[32];  // D = 64: the inter results of the chunk at hand
    // They are read as soon as the scores are there, before the intra results, so
    // that the next but one product may take their columns.
    auto load_inter = [&](int j) {
      if (!mbar_wait(&sc_full[j & 1], (j >> 1) & 1, &ab)) decay_error(256, ab);
      tc_fence_after();
      tmem_ld_16x64(quarter + Sh::kColInter + Sh::kInterStep * (j & 1), s);
      tmem_ld_wait_regs(s);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&score_ready[j & 1]);
    };
    if (lane == 0) {
      uint64_t *inter = Sh::kMerged ? score_ready : inter_ready;
      mbar_arrive(&inter[0]), mbar_arrive(&inter[1]);
      if (Sh::kMerged) mbar_arrive(&intra_ready[0]), mbar_arrive(&intra_ready[1 % Sh::kP]);
    }
    if constexpr (Sh::kMerged) load_inter(0);
    for (int j = 0; j < cnt; ++j) {
      const int ob = j & 1, t0 = sg.token_of(q0 + j), n = min(kC, L - t0);
      float ur[2] = {u[0], u[1]};
      if (p.reverse && q0 + j == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          ur[k] = scaled_pow(p.scale, l2, (float)max(n - 1 - (r0 + 8 * k), 0));
      }
      if constexpr (!Sh::kMerged) {  // weight the inter results in place; intra is added to them
        if (!mbar_wait(&inter_full[ob], (j >> 1) & 1, &ab)) decay_error(256, ab);
        tc_fence_after();
#pragma unroll
        for (int blk = 0; blk < Sh::kB; ++blk) {
          const uint32_t at = quarter + Sh::kColInter + Sh::kInterStep * ob + blk * 64;
          tmem_ld_16x64(at, s);
          tmem_ld_wait_regs(s);
#pragma unroll
          for (int i = 0; i < 32; ++i) s[i] *= ur[(i >> 1) & 1];
          tmem_st_16x64(at, s);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&intra_ready[j % Sh::kP]);
      }
      if (!mbar_wait(&o_full[ob], (j >> 1) & 1, &ab)) decay_error(256, ab);
      tc_fence_after();
#pragma unroll
      for (int blk = 0; blk < Sh::kB; ++blk) {
        float a[32];
        tmem_ld_16x64(quarter + Sh::kColIntra + Sh::kIntraStep * ob + blk * 64, a);
        tmem_ld_wait_regs(a);
        if (blk == Sh::kB - 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(Sh::kMerged ? &intra_ready[ob % Sh::kP] : &inter_ready[ob]);
        }
        if constexpr (Sh::kMerged) {
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float w = ur[(i >> 1) & 1];
            const float2 r = __ffma2_rn(make_float2(w, w), make_float2(s[i], s[i + 1]),
                                        make_float2(a[i], a[i + 1]));
            a[i] = r.x, a[i + 1] = r.y;
          }
          if (j + 1 < cnt) load_inter(j + 1);
        }
        write_rows<(V < 64 ? V : 64), O>(out + (size_t)t0 * orow + blk * 64, orow, stage, ow, lane, n,
                                         a);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == Sh::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ---------------------------------------------------------------------------
// The gradients of keys and values together (D <= 64), in reverse.  Both meet the
// same state A = sum gamma^.. q d_o^T, whose keys and values are q and d_o:
//   dv_r = scale [ sum_{j >= r} gamma^{j-r} (k_r . q_j) d_o_j + u_r A^T k_r ],
//   dk_r = scale [ sum_{j >= r} gamma^{j-r} (v_r . d_o_j) q_j + u_r A v_r ].
// So a chunk is two jobs of the scan above, dv then dk, over tiles that are loaded
// once, and one state, which the state warps write behind both: transposed behind
// q (dv's columns are those of d_o) and as it is behind d_o.  Against two scans
// this saves half the loads, a state product and its weighted keys, and the second
// own-state kernel.  Scores, weighting and results see jobs as they see chunks.
template <int kTerms>
struct KvShape {
  static constexpr int kNX = kTerms == 2 ? 2 : 1;  // slots of k and of v each
  static constexpr int kN = 4;                     // slots of q and of d_o, a state behind each
  static constexpr int kSlot = 2 * kBlk;
  static constexpr int kOffX = 0, kOffQ = 2 * kNX * kBlk, kOffG = kOffQ + kN * kSlot;
  static constexpr int kOffConv = kOffG + kN * kSlot, kOffP = kOffConv + 2 * kTerms * kBlk;
  static constexpr int kOffOut = kOffP + 2 * kBlk, kOffBar = kOffOut + kBlk;
  static constexpr int kBars = 2 * (2 * kNX) + 4 * kN + 8 * 2 + 1 + 1 + 2;
  static constexpr int kOffMisc = kOffBar + kBars * 8;
  static constexpr int kSmem = kOffMisc + 16 + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr int kTmaWarp = 16, kMmaWarp = 17, kThreads = 18 * 32;
  // scores | inter results of two jobs, intra results of two, the chunk's state
  static constexpr uint32_t kColSc = 0, kColIntra = 256, kColDs = 384;
};

struct KvParams {
  TcParams c;  // y = q, z = d_o; out = dv
  void *dk;
};

template <int V, int kTerms, typename O>
__global__ void __launch_bounds__(KvShape<kTerms>::kThreads, 1)
    kv_kernel(const KvParams kp, const __grid_constant__ CUtensorMap tm_k,
              const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_q,
              const __grid_constant__ CUtensorMap tm_g) {
  using Sh = KvShape<kTerms>;
  constexpr int D = 64, kNX = Sh::kNX, kN = Sh::kN;
  const TcParams &p = kp.c;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t *fx = (uint64_t *)(smem + Sh::kOffBar), *ex = fx + 2 * kNX, *fq = ex + 2 * kNX,
           *eq = fq + kN, *fg = eq + kN, *eg = fg + kN, *state_ready = eg + kN,
           *conv_empty = state_ready + 2, *score_ready = conv_empty + 2, *sc_full = score_ready + 2,
           *intra_ready = sc_full + 2, *p_empty = intra_ready + 2, *o_full = p_empty + 2,
           *s_full = o_full + 2, *ds_full = s_full + 2, *drained = ds_full + 1;
  uint32_t *tmem_slot = (uint32_t *)(smem + Sh::kOffMisc);
  const AbortFlag ab{smem_u32(smem + Sh::kOffMisc + 4)};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const Segment sg(p, b, rank);
  const int L = sg.L, q0 = sg.q0, cnt = sg.cnt, jobs = 2 * cnt;
  const size_t bh = (size_t)b * p.H + h, orow = (size_t)p.H * V;
  const size_t first = ((size_t)b * p.N * p.H + h) * V;  // token t at first + t * orow
  {  // the rows past the end, shared among the sequence's CTAs
    constexpr int kPer = V * (int)sizeof(O) / 16;
    for (long long i = (long long)rank * Sh::kThreads + tid; i < (long long)(p.N - L) * kPer * 2;
         i += (long long)p.ranks * Sh::kThreads) {
      O *out = (O *)(i & 1 ? kp.dk : p.out) + first;
      ((uint4 *)(out + (L + (i >> 1) / kPer) * orow))[(i >> 1) % kPer] = make_uint4(0, 0, 0, 0);
    }
  }
  if (cnt == 0) {
    if (p.ranks > 1) grid_dep_wait();  // a grid never ends before the kernels ahead of it
    if (rank == 0 && p.fin)  // an empty sequence passes its state on
      for (int i = tid; i < V * V; i += Sh::kThreads)
        p.fin[bh * V * V + i] = p.init ? p.init[bh * V * V + i] * p.init_scale * p.fin_scale : 0.f;
    return;
  }
  const float l2 = __ldg(p.log_decay + h) * 1.4426950408889634f;
  // The loading warp sets the barriers up and starts at once; the others also wait
  // for the TMEM allocation.
  if (warp == Sh::kTmaWarp && lane == 0) {
    *(volatile int *)(smem + Sh::kOffMisc + 4) = 0;
    for (int i = 0; i < 2 * kNX; ++i) mbar_init(&fx[i], 1), mbar_init(&ex[i], 1);
    for (int i = 0; i < kN; ++i) {
      mbar_init(&fq[i], 1), mbar_init(&eq[i], 1);
      mbar_init(&fg[i], 1), mbar_init(&eg[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&state_ready[i], 8);  // weighted q there, the last chunk's state taken
      mbar_init(&conv_empty[i], 1);
      mbar_init(&score_ready[i], 8);  // scores' and inter results' columns free
      mbar_init(&sc_full[i], 1);
      mbar_init(&intra_ready[i], 8);  // scores weighted, intra results' columns free
      mbar_init(&p_empty[i], 1);
      mbar_init(&o_full[i], 1);
      mbar_init(&s_full[i], 4);
    }
    mbar_init(ds_full, 1);
    mbar_init(drained, 1);
    fence_mbar_init();
  }
  if (warp == Sh::kTmaWarp && lane == 0) {
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_g);
  }
  if (warp == Sh::kMmaWarp) tmem_alloc(tmem_slot, 512);
  if (warp == Sh::kTmaWarp) {
    __syncwarp();
    named_barrier_arrive(1, Sh::kThreads);
  } else {
    tc_fence_before();
    named_barrier(1, Sh::kThreads);
    tc_fence_after();
  }
  const uint32_t tmem = *tmem_slot;
  if (warp == Sh::kTmaWarp) {
    // ---------------------------------------------------------------- loads
    if (lane < 4) {  // k, v, q, d_o
      const CUtensorMap *tm = lane == 0 ? &tm_k : lane == 1 ? &tm_v : lane == 2 ? &tm_q : &tm_g;
      const int hd = lane < 2 ? h / p.gx : h, slots = lane < 2 ? kNX : kN;
      uint64_t *f = lane < 2 ? fx + lane * kNX : lane == 2 ? fq : fg;
      uint64_t *e = lane < 2 ? ex + lane * kNX : lane == 2 ? eq : eg;
      uint8_t *to = smem + (lane < 2 ? Sh::kOffX + lane * kNX * kBlk : lane == 2 ? Sh::kOffQ : Sh::kOffG);
      const int size = lane < 2 ? kBlk : Sh::kSlot;
      int i = 0;
      for (; i < cnt; ++i) {
        const int s = i % slots;
        if (!mbar_wait(&e[s], ((i / slots) & 1) ^ 1, &ab)) {
          decay_error(1, ab);
          break;
        }
        mbar_arrive_expect_tx(&f[s], kBlk);
        tma_load_4d(to + s * size, tm, &f[s], 0, hd, sg.token_of(q0 + i), b);
      }
      if (i < cnt)  // gave up: no copy may land after the CTA is gone
        for (int k = max(0, i - slots); k < i; ++k)
          mbar_wait(&f[k % slots], (k / slots) & 1, nullptr);
    }
    __syncwarp();
  } else if (warp == Sh::kMmaWarp) {
    // ----------------------------------------------------------------- MMAs
    if (elect_one()) {
      const uint32_t base = smem_u32(smem);
      bool ok = true;
      auto wait = [&](uint64_t *m, uint32_t parity) {
        if (ok && !mbar_wait(m, parity, &ab)) decay_error(2, ab), ok = false;
        return ok;
      };
      auto slot = [&](bool g, int i) { return base + (g ? Sh::kOffG : Sh::kOffQ) + (i % kN) * Sh::kSlot; };
      auto state_mma = [&](int i) {
        if (!wait(&fg[i % kN], (i / kN) & 1)) return;
        if (!wait(&state_ready[i & 1], (i >> 1) & 1)) return;
        tc_fence_after();
        state_product<D, kTerms, kBlk>(tmem + Sh::kColDs, slot(true, i),
                                       base + Sh::kOffConv + (i & 1) * kTerms * kBlk, false);
        mma_commit(ds_full);
        mma_commit(&conv_empty[i & 1]);
      };
      // job 2 i (dv): k against q and the state behind it; 2 i + 1 (dk): v against d_o
      auto score_mma = [&](int job) {
        const int i = job >> 1, w = job & 1, sx = w * kNX + i % kNX;
        if (!wait(&fx[sx], (i / kNX) & 1)) return;
        if (w == 0 && !wait(&s_full[i & 1], (i >> 1) & 1)) return;
        if (!wait(&score_ready[w], i & 1)) return;
        tc_fence_after();
        constexpr uint32_t id = idesc_bf16_f32(64, 128, 0, 0);
        const uint64_t xd = sw128_desc(base + Sh::kOffX + sx * kBlk, 16, 1024);
        const uint64_t yd = sw128_desc(slot(w != 0, i), 16, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16(tmem + Sh::kColSc + 128 * w, desc_at(xd, k * 32), desc_at(yd, k * 32), id, k != 0);
        mma_commit(&sc_full[w]);
        mma_commit(&ex[sx]);
      };
      auto intra_mma = [&](int job) {
        const int i = job >> 1, w = job & 1;
        if (!wait(&intra_ready[w], i & 1)) return;
        tc_fence_after();
        constexpr uint32_t id = idesc_bf16_f32(64, D, 0, 1);
        const uint64_t pd = sw128_desc(base + Sh::kOffP + w * kBlk, 16, 1024);
        const uint64_t zd = sw128_desc(slot(w == 0, i), kBlk, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16(tmem + Sh::kColIntra + 64 * w, desc_at(pd, k * 32), desc_at(zd, k * 2048), id, k != 0);
        mma_commit(&p_empty[w]);
        mma_commit(&o_full[w]);
        if (w == 1) mma_commit(&eq[i % kN]), mma_commit(&eg[i % kN]);
      };
      state_mma(0);
      for (int job = 0; job <= jobs && ok; ++job) {
        if (job < jobs) score_mma(job);
        if (job >= 1 && ok) intra_mma(job - 1);
        if ((job & 1) && job < jobs && (job >> 1) + 1 < cnt && ok) state_mma((job >> 1) + 1);
      }
      mma_commit(drained);  // nothing is in flight when TMEM is freed
      if (!mbar_wait(drained, 0, nullptr)) decay_error(512, ab);
    }
    __syncwarp();
  } else if (warp < 4) {
    // ------------------------------------------- weighted scores (warps 0-3)
    const int r0 = 16 * warp + (lane >> 2), c = 2 * (lane & 3);
    float2 w[9];  // gamma^{column - row} in steps of 8 columns, as in the scan
#pragma unroll
    for (int k = 0; k < 9; ++k) {
      float e[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int n = c + q + 8 * (k - 1) - r0;
        e[q] = n >= 0 ? p.scale * decay_pow(l2, (float)n) : 0.f;
      }
      w[k] = make_float2(e[0], e[1]);
    }
    if (lane == 0) mbar_arrive(&score_ready[0]), mbar_arrive(&score_ready[1]);
    for (int job = 0; job < jobs; ++job) {
      const int i = job >> 1, s = job & 1;
      if (!mbar_wait(&sc_full[s], i & 1, &ab)) decay_error(4, ab);
      tc_fence_after();
      float a[32];
      tmem_ld_16x64(tmem + ((uint32_t)(32 * warp) << 16) + Sh::kColSc + 128 * s, a);
      tmem_ld_wait_regs(a);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&score_ready[s]);
      if (i >= 1 && !mbar_wait(&p_empty[s], (i & 1) ^ 1, &ab)) decay_error(8, ab);
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float2 m = __fmul2_rn(make_float2(a[4 * k + 2 * q], a[4 * k + 2 * q + 1]), w[k + 1 - q]);
          a[4 * k + 2 * q] = m.x, a[4 * k + 2 * q + 1] = m.y;
        }
      store_16x64(smem_u32(smem + Sh::kOffP + s * kBlk) + 16 * warp * 128, lane, a);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&intra_ready[s]);
    }
  } else if (warp < 8) {
    // ------------------------------------------------ weighted q (warps 4-7)
    const int ct = tid - 128, ch = ct & 7, rr = ct >> 3;
    const uint32_t piece = rr * 128 + ((ch ^ (rr & 7)) << 4);
    RowWeight w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k].set(decay_pow(l2, (float)(rr + 16 * k)));
    for (int i = 0; i < cnt; ++i) {
      const int s = i % kN, cb = i & 1, n = min(kC, L - sg.token_of(q0 + i));
      if (!mbar_wait(&fq[s], (i / kN) & 1, &ab)) decay_error(16, ab);
      if (i >= 2 && !mbar_wait(&conv_empty[cb], ((i >> 1) & 1) ^ 1, &ab)) decay_error(32, ab);
      const uint32_t ys = smem_u32(smem + Sh::kOffQ + s * Sh::kSlot) + piece;
      const uint32_t cs = smem_u32(smem + Sh::kOffConv + cb * kTerms * kBlk) + piece;
      if (n == kC) {
        uint4 u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = lds_v4(ys + k * 2048);
#pragma unroll
        for (int k = 0; k < 4; ++k) weigh_piece<kTerms, kBlk>(u[k], w[k], cs + k * 2048);
      } else {
        if (!mbar_wait(&fg[s], (i / kN) & 1, &ab)) decay_error(16, ab);
        weigh_end<kTerms, kBlk>(ys, smem_u32(smem + Sh::kOffG + s * Sh::kSlot) + piece, cs, rr, n, l2,
                                1.f, true);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&state_ready[cb]);
    }
  } else if (warp < 12) {
    // --------------------- the state, transposed (rows of d_o), in registers
    const int sw = warp - 8;
    const uint32_t src = tmem + ((uint32_t)(32 * sw) << 16) + Sh::kColDs;
    const DecayFactor chunk_factor = decay_factor(__ldg(p.log_decay + h) * kC);
    float S[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) S[i] = 0.f;
    if (lane == 0) mbar_arrive(&state_ready[0]);
    start_state<V>(S, p, sg, bh, rank, sw, lane, l2);
    for (int i = 0; i < cnt; ++i) {
      const int s = i % kN;
      if (!mbar_wait(&eq[s], ((i / kN) & 1) ^ 1, &ab)) decay_error(128, ab);
      if (!mbar_wait(&eg[s], ((i / kN) & 1) ^ 1, &ab)) decay_error(128, ab);
      store_16x64(smem_u32(smem + Sh::kOffQ + s * Sh::kSlot + kBlk) + 16 * sw * 128, lane, S);
      store_16x64_t(smem_u32(smem + Sh::kOffG + s * Sh::kSlot + kBlk), 2 * sw, lane, S);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_full[i & 1]);
      const int n = min(kC, L - sg.token_of(q0 + i));
      if (!mbar_wait(ds_full, i & 1, &ab)) decay_error(64, ab);
      tc_fence_after();
      take_state<64, false>(S, src, q0 + i > 0 ? chunk_factor : one_factor(decay_pow(l2, (float)(n - 1))));
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&state_ready[(i + 1) & 1]);
    }
    if (p.fin && sg.last) {
      const float f = scaled_pow(p.fin_scale, l2, 1.f);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        int e;
        const int d = state_at<64>(sw, lane, i, &e);
        if (V == D || (d < V && e < V)) p.fin[bh * V * V + d * V + e] = S[i] * f;
      }
    }
  } else {
    // ---------------------------------------------------------------- results
    const int ow = warp - 12, r0 = 16 * ow + (lane >> 2);
    const uint32_t quarter = tmem + ((uint32_t)(32 * ow) << 16);
    const uint32_t stage = smem_u32(smem + Sh::kOffOut + ow * 2048);
    float u[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) u[k] = scaled_pow(p.scale, l2, (float)(kC - (r0 + 8 * k)));
    float s[32];
    auto load_inter = [&](int job) {
      const int w = job & 1;
      if (!mbar_wait(&sc_full[w], (job >> 1) & 1, &ab)) decay_error(256, ab);
      tc_fence_after();
      tmem_ld_16x64(quarter + Sh::kColSc + 128 * w + 64, s);
      tmem_ld_wait_regs(s);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&score_ready[w]);
    };
    if (lane == 0) {
      mbar_arrive(&score_ready[0]), mbar_arrive(&score_ready[1]);
      mbar_arrive(&intra_ready[0]), mbar_arrive(&intra_ready[1]);
    }
    load_inter(0);
    for (int job = 0; job < jobs; ++job) {
      const int i = job >> 1, w = job & 1, t0 = sg.token_of(q0 + i), n = min(kC, L - t0);
      float ur[2] = {u[0], u[1]};
      if (q0 + i == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          ur[k] = scaled_pow(p.scale, l2, (float)max(n - 1 - (r0 + 8 * k), 0));
      }
      if (!mbar_wait(&o_full[w], i & 1, &ab)) decay_error(256, ab);
      tc_fence_after();
      float a[32];
      tmem_ld_16x64(quarter + Sh::kColIntra + 64 * w, a);
      tmem_ld_wait_regs(a);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&intra_ready[w]);
#pragma unroll
      for (int k = 0; k < 32; k += 2) {
        const float f = ur[(k >> 1) & 1];
        const float2 r = __ffma2_rn(make_float2(f, f), make_float2(s[k], s[k + 1]),
                                    make_float2(a[k], a[k + 1]));
        a[k] = r.x, a[k + 1] = r.y;
      }
      if (job + 1 < jobs) load_inter(job + 1);
      O *dst = (O *)(w ? kp.dk : p.out) + first + (size_t)t0 * orow;
      write_rows<V, O>(dst, orow, stage, ow, lane, n, a);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == Sh::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                   const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                   const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = (EncodeTiledFn)f;
  });
  return fn;
}

// Boxes of 64 channels x 1 head x 64 tokens, 128-byte swizzle.
cudaError_t make_map(CUtensorMap *m, const void *base, int B, int N, int heads, int D,
                     const long long (&s)[2]) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return cudaErrorNotSupported;
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)N, (cuuint64_t)B};
  const cuuint64_t strides[3] = {(cuuint64_t)D * 2, (cuuint64_t)s[1] * 2, (cuuint64_t)s[0] * 2};
  const cuuint32_t box[4] = {64, 1, kC, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  const CUresult r =
      fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, box, estr,
         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
         CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
    return 152;
  return n;
}

// Chunks of a segment.  In units of a scanned chunk (0.75 us at D = 64, 1.5 at
// D = 128), as measured: a CTA costs what its pipeline takes to fill and drain and
// its chunks, one of the own-state kernel 0.6 of a unit a chunk.  Equal lengths:
// whole rounds of CTAs over the SMs.  Lengths that only the device knows are taken
// to be uneven, a quarter of the longest on average; the kernels then last as long as
// all the work over the SMs and half a segment of tail, or as their longest CTA (B32
// H8 D128, log-normal about 4096 to 32768: 524 us; cut as if all were the longest,
// 1030).  A batch of about equal lengths pays for that: all 4096 of B19 H8 D64 96 us
// for 56 without lengths, all 8192 of B16 H8 D128 360 for 238.
// The pass over keys and values takes `chunk` = 1.6 scanned chunks a chunk.  Starting a
// CTA: 9 units, at D = 128 4.2 (B8 H8 N8192: 169 us, with 3.5 186; 7 sequences ragged to
// 21623: 147 us, with 5 176).
int segment_for(const ScanArgs &a, double chunk) {
  const double fill = (a.D > 64 ? 4.2 : 9) / chunk, own_chunk = 0.6 / chunk;
  const int nc = (a.N + kC - 1) / kC, sms = sm_count();
  const double pairs = (double)a.B * a.H;
  auto rounds = [&](double ctas) { return (double)(long long)(ctas / sms + 0.999999); };
  auto more = [](double x, double y) { return x > y ? x : y; };
  int best = nc;
  double least = 0;
  for (int r = 1; r <= 32 && nc >= 4 * r; ++r) {
    const int seg = (nc + r - 1) / r;
    double t;
    if (a.seq_lens) {
      const double all = pairs * nc / 4 / sms, fills = fill * pairs * (r / 4.0 + 0.5) / sms;
      t = more(all + fills + seg / 2, seg + fill);
      if (r > 1)
        t += more(own_chunk * (all * (r - 1) / r + seg / 2) + fills, own_chunk * seg + fill);
    } else {
      t = rounds(pairs * r) * (seg + fill);
      if (r > 1) t += rounds(pairs * (r - 1)) * own_chunk * seg + fill;
    }
    if (r == 1 || t < 0.97 * least) best = seg, least = t;
  }
  return best;
}

constexpr double kKvChunk = 1.6;

int ranks_for(const ScanArgs &a, double chunk) {
  const int seg = segment_for(a, chunk);
  return ((a.N + kC - 1) / kC + seg - 1) / seg;
}
size_t part_floats(const ScanArgs &a, double chunk) {
  const size_t d = a.D < 64 ? 64 : a.D;
  const int ranks = ranks_for(a, chunk);
  return ranks > 1 ? (size_t)a.B * a.H * ranks * d * d : 0;
}

// A scan ready to launch.
struct Scan {
  ScanArgs a;
  TcParams p;
  CUtensorMap x, y, z;
  cudaError_t set(const ScanArgs &args, float *scratch, double chunk = 1) {
    a = args;
    p = TcParams{};
    p.out = a.out, p.log_decay = a.log_decay, p.seq_lens = a.seq_lens;
    p.init = a.init, p.fin = a.fin, p.part = scratch;
    p.init_scale = a.init_scale, p.fin_scale = a.fin_scale, p.scale = a.scale;
    p.N = a.N, p.H = a.H, p.gx = a.gx, p.gy = a.gy, p.gz = a.gz;
    p.zero_pad = a.zero_pad, p.init_t = a.init_t, p.reverse = a.reverse;
    p.seg = segment_for(a, chunk), p.ranks = ranks_for(a, chunk);
    p.before = p.ranks > (a.D > 64 ? 1 : 12);
    cudaError_t e;
    if ((e = make_map(&x, a.x, a.B, a.N, a.H / a.gx, a.D, a.sx)) != cudaSuccess) return e;
    if ((e = make_map(&y, a.y, a.B, a.N, a.H / a.gy, a.D, a.sy)) != cudaSuccess) return e;
    return make_map(&z, a.z, a.B, a.N, a.H / a.gz, a.D, a.sz);
  }
};

template <int D, int kTerms>
cudaError_t launch_own(const Scan &s, cudaStream_t st) {
  using Sh = OwnShape<D, kTerms>;
  const auto kernel = own_state_kernel<D, kTerms>;
  const cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kSmem);
  if (e != cudaSuccess) return e;
  kernel<<<dim3(s.p.ranks - 1, s.a.H, s.a.B), Sh::kThreads, Sh::kSmem, st>>>(s.p, s.y, s.z);
  count_launch();
  return cudaGetLastError();
}

// The states of the segments, where a sequence is cut into any.  (The backward's in
// one launch ahead of its scans were slower: 120 us where it is 117 at B4 H8 N8192
// D64, 363 for 320 at B2 N16384 D128; each scan finds less of its own in L2.)
cudaError_t states_before(const Scan &s, cudaStream_t st) {
  if (s.p.ranks <= 1) return cudaSuccess;
  const bool wide = s.a.D > 64;
  const cudaError_t e =
      wide ? s.a.fin ? launch_own<128, 3>(s, st) : launch_own<128, 2>(s, st)
           : s.a.fin ? launch_own<64, 3>(s, st) : launch_own<64, 2>(s, st);
  if (e != cudaSuccess) return e;
  if (!s.p.before) return cudaSuccess;
  count_launch();
  return launch_pdl(wide          ? before_kernel<128, 128>
                    : s.a.D == 64 ? before_kernel<64, 64>
                                  : before_kernel<64, 32>,
                    dim3(wide ? 16 : 4, s.a.H, s.a.B), dim3(256), 0, st, s.p);
}

// Launches a scan right behind the kernels that form the states before its segments:
// it may start while they end, as only its state warps read what they write, and
// those wait for it.
template <typename... KArgs, typename... Args>
cudaError_t launch_behind(void (*kernel)(KArgs...), const Scan &s, int threads, int smem,
                          cudaStream_t st, Args... args) {
  const cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const dim3 grid(s.p.ranks, s.a.H, s.a.B);
  count_launch();
  if (s.p.ranks > 1) return launch_pdl(kernel, grid, dim3(threads), smem, st, args...);
  kernel<<<grid, threads, smem, st>>>(args...);
  return cudaGetLastError();
}

template <int D, int V>
cudaError_t launch_scan_as(const Scan &s, cudaStream_t st) {
  auto go = [&](auto *kernel, auto shape) {
    using Sh = decltype(shape);
    return launch_behind(kernel, s, Sh::kThreads, Sh::kSmem, st, s.p, s.x, s.y, s.z);
  };
  if (s.a.fin)
    return s.a.out_f32 ? go(decay_kernel<D, V, 3, float>, Shape<D, 3>{})
                       : go(decay_kernel<D, V, 3, __nv_bfloat16>, Shape<D, 3>{});
  return s.a.out_f32 ? go(decay_kernel<D, V, 2, float>, Shape<D, 2>{})
                     : go(decay_kernel<D, V, 2, __nv_bfloat16>, Shape<D, 2>{});
}
cudaError_t launch_scan(const Scan &s, cudaStream_t st) {
  const cudaError_t e = states_before(s, st);
  if (e != cudaSuccess) return e;
  if (s.a.D == 32) return launch_scan_as<64, 32>(s, st);
  return s.a.D == 64 ? launch_scan_as<64, 64>(s, st) : launch_scan_as<128, 128>(s, st);
}

template <int V>
cudaError_t launch_kv_as(const Scan &dv, const Scan &dk, cudaStream_t st) {
  auto go = [&](auto *kernel, auto shape) {
    using Sh = decltype(shape);
    return launch_behind(kernel, dv, Sh::kThreads, Sh::kSmem, st, KvParams{dv.p, dk.a.out}, dv.x,
                         dk.x, dv.y, dv.z);
  };
  if (dv.a.fin)
    return dv.a.out_f32 ? go(kv_kernel<V, 3, float>, KvShape<3>{})
                        : go(kv_kernel<V, 3, __nv_bfloat16>, KvShape<3>{});
  return dv.a.out_f32 ? go(kv_kernel<V, 2, float>, KvShape<2>{})
                      : go(kv_kernel<V, 2, __nv_bfloat16>, KvShape<2>{});
}
cudaError_t launch_kv(const Scan &dv, const Scan &dk, cudaStream_t st) {
  const cudaError_t e = states_before(dv, st);
  if (e != cudaSuccess) return e;
  return dv.a.D == 32 ? launch_kv_as<32>(dv, dk, st) : launch_kv_as<64>(dv, dk, st);
}

// Keys and values together where the state fits beside both (D <= 64).
bool together(const ScanArgs &a) { return a.D <= 64; }

}  // namespace

bool tc_scan_supports(const ScanArgs &a) {
  if (a.dtype != GBLA_BF16) return false;
  for (const auto &s : {a.sx, a.sy, a.sz})  // the stride limit of a tensor map
    if (s[0] >= (1ll << 39) || s[1] >= (1ll << 39)) return false;
  int dev = 0, major = 0, minor = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
  cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
  return major == 10 && minor == 3 && encode_fn() != nullptr;
}

size_t tc_scan_floats(const ScanArgs &a) { return part_floats(a, 1); }

cudaError_t tc_scan(const ScanArgs &a, float *scratch, cudaStream_t st) {
  Scan s;
  const cudaError_t e = s.set(a, scratch);
  return e == cudaSuccess ? launch_scan(s, st) : e;
}

// The scans follow one another, so one scratch serves them.
size_t tc_backward_floats(const ScanArgs *scan) {
  const size_t one = part_floats(scan[0], 1);
  const size_t two = part_floats(scan[1], together(scan[0]) ? kKvChunk : 1);
  return one > two ? one : two;
}

cudaError_t tc_backward(const ScanArgs *scan, float *scratch, cudaStream_t st) {
  Scan s[3];
  const bool kv = together(scan[0]);
  cudaError_t e;
  for (int i = 0; i < 3; ++i)
    if ((e = s[i].set(scan[i], scratch, kv && i > 0 ? kKvChunk : 1)) != cudaSuccess) return e;
  if ((e = launch_scan(s[0], st)) != cudaSuccess) return e;
  if (kv) return launch_kv(s[1], s[2], st);
  if ((e = launch_scan(s[1], st)) != cudaSuccess) return e;
  return launch_scan(s[2], st);
}

unsigned decay_device_error(bool reset) {
  unsigned v = 0;
  if (cudaMemcpyFromSymbol(&v, g_decay_error, sizeof(v)) != cudaSuccess) return 0xFFFFFFFFu;
  if (reset) {
    const unsigned z = 0;
    if (cudaMemcpyToSymbol(g_decay_error, &z, sizeof(z)) != cudaSuccess) return 0xFFFFFFFFu;
  }
  return v;
}

}  // namespace gbla
