// Decayed linear attention on tensor cores (tcgen05 + TMA): bf16, D in {64, 128}.
//
// The scan of ScanArgs in chunks of C = 64 tokens, in scan order.  With r, j the
// places in a chunk, S the state before it and gamma the head's decay,
//   scores  A_rj  = x_r . y_j                        (M64 N64 KD)
//   results out_r = scale [ sum_j (w_rj A_rj) z_j + u_r x_r^T S ]
//                                                    (M64 ND K64, M64 ND KD)
//   state   S'    = c S + sum_j (v_j y_j) z_j^T      (MD ND K64, a time for each term)
// D = 64: y's tile and the state (transposed) lie one behind the other, so that
// scores and x_r^T S are one product of N = 128, and the terms of the state's
// product share one of N = 128: an MMA of M = 64 takes about as long at N = 64.
// forward: w = gamma^{r-j} (j <= r), u = gamma^{r+1}, v = gamma^{n-1-j}, c = gamma^n
// for n tokens in the chunk; reverse: w = gamma^{j-r} (j >= r), u = gamma^{64-r},
// v = gamma^j, c = gamma^64, and u = gamma^{n-1-r}, c = gamma^{n-1} in the first
// chunk, whose state before it (the gradient of the final state) belongs to the
// last token itself.
//
// Rounding: the weighted scores and the state as it meets a query are rounded
// once to bf16 (the results are bf16 too).  The state is held in fp32 registers
// and is never rebuilt from rounded values: v_j y_j goes into the product as a
// sum of bf16 numbers, two (2^-17 of a term) where the state only serves the
// results, three (2^-25) where it is a result itself.  The decay powers are fp32.
//
// One CTA serves a run of chunks (a segment) of one (batch, head); a cluster of
// 1, 2, 4 or 8 CTAs serves the whole sequence.  Every CTA but the last in scan
// order first sums its own segment's state (y and z alone, the chunk it will need
// last read first, so that what it reads again soonest is still in L2), the
// cluster meets once, and each CTA starts its scan from the weighted sum of the
// segments before it.  That costs y and z a second read and saves any launch
// besides this one.
//
// Warps: 0-3 weight the scores, 4-7 form v_j y_j, the next 4 (D = 128: 8) hold
// the state, the next 4 write results, then one warp issues the TMA loads (a
// lane for each 64-channel block of each tensor: one thread issues a box in half
// a microsecond) and one the MMAs.  M = 64 accumulators lie in lanes 0-15 of each
// TMEM quarter and are read with the 16-lane shapes.
//
// Every mbarrier wait is bounded (2 s); one that runs out sets a bit in
// g_decay_error and raises the CTA's abort flag.
#include <mutex>

#include "gbla_internal.cuh"
#include "gbla_sm100.cuh"

namespace gbla {

__device__ unsigned int g_decay_error;

namespace {

using namespace sm100;

constexpr int kC = 64;                 // tokens per chunk
constexpr int kBlk = kC * 128;         // 8 KB: 64 tokens x 64 channels, 128B swizzle
constexpr int kMaxCluster = 8;

template <int D, int kTerms>
struct Shape {
  static constexpr bool kMerged = D == 64;                 // scores and inter results in one MMA
  static constexpr int kB = D / 64;                        // 64-channel blocks
  static constexpr int kTile = kB * kBlk;                  // one tensor's chunk
  static constexpr int kSBytes = D * D * 2;                // the state rounded to bf16
  // rings of x, y and z tiles; merged: the state's tile follows y's in its slot
  static constexpr int kNX = D == 64 ? 4 : (kTerms == 2 ? 3 : 2), kNY = D == 64 ? 4 : 3,
                       kNZ = D == 64 ? 5 : 3;
  static constexpr int kYSlot = kTile + (kMerged ? kSBytes : 0);
  static constexpr int kConv = D == 64 ? 2 : 1;            // buffers of v_j y_j
  static constexpr int kP = D == 64 ? 2 : 1;               // of weighted scores
  static constexpr int kO = D == 64 ? 2 : 1;               // of the results' accumulators
  static constexpr int kOffX = 0, kOffY = kOffX + kNX * kTile, kOffZ = kOffY + kNY * kYSlot;
  static constexpr int kOffConv = kOffZ + kNZ * kTile;
  static constexpr int kOffP = kOffConv + kConv * kTerms * kTile;
  static constexpr int kOffS = kOffP + kP * kBlk;
  static constexpr int kOffBar = kOffS + (kMerged ? 0 : kSBytes);
  static constexpr int kBars = 2 * (kNX + kNY + kNZ + kConv + kP + kO) + 2 + 1 + 2 + 4 + 1;
  static constexpr int kOffMisc = kOffBar + kBars * 8;
  static constexpr int kSmem = kOffMisc + 16 + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr int kSWarps = D == 64 ? 4 : 8;
  static constexpr int kOutWarp = 8 + kSWarps, kTmaWarp = kOutWarp + 4, kMmaWarp = kTmaWarp + 1;
  static constexpr int kThreads = (kMmaWarp + 1) * 32;
  static constexpr int kLoads = 3 * kB;                    // issuing lanes
  // TMEM columns.  Merged: two buffers of scores | inter results, two of intra
  // results, the chunk's state (its large and its small terms side by side);
  // else two of scores, inter, intra, state.
  static constexpr uint32_t kColSc = 0, kScStep = kMerged ? 128 : 64;
  static constexpr uint32_t kColInter = kMerged ? 64 : 128, kInterStep = kMerged ? 128 : 0;
  static constexpr uint32_t kColIntra = 256, kIntraStep = kMerged ? 64 : 0;
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
  bool zero_pad, init_t, reverse;
};

__device__ __forceinline__ void decay_error(unsigned code, const AbortFlag &ab) {
  if (!ab.raised()) atomicOr(&g_decay_error, code);
  ab.raise();
}
__device__ __forceinline__ float decay_pow(float l2, float n) {
  return n == 0.f ? 1.f : exp2f(n * l2);
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
__device__ __forceinline__ void sts_u32(uint32_t a, uint32_t v) {
  asm volatile("st.shared.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
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
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
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

template <int D, int kTerms, typename O>
__global__ void __launch_bounds__(Shape<D, kTerms>::kThreads, 1)
    decay_kernel(const TcParams p, const __grid_constant__ CUtensorMap tm_x,
                 const __grid_constant__ CUtensorMap tm_y,
                 const __grid_constant__ CUtensorMap tm_z) {
  using Sh = Shape<D, kTerms>;
  constexpr int kNV = D == 64 ? 32 : 64;  // state values a thread
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t *bar = (uint64_t *)(smem + Sh::kOffBar);
  uint64_t *fx = bar, *ex = fx + Sh::kNX, *fy = ex + Sh::kNX, *ey = fy + Sh::kNY,
           *fz = ey + Sh::kNY, *ez = fz + Sh::kNZ, *conv_full = ez + Sh::kNZ,
           *conv_empty = conv_full + Sh::kConv, *p_full = conv_empty + Sh::kConv,
           *p_empty = p_full + Sh::kP, *o_full = p_empty + Sh::kP, *o_empty = o_full + Sh::kO,
           *s_full = o_empty + Sh::kO, *s_empty = s_full + 2, *ds_full = s_empty + 1,
           *ds_empty = ds_full + 1, *sc_full = ds_empty + 1, *sc_empty = sc_full + 2,
           *drained = sc_empty + 2;
  uint32_t *tmem_slot = (uint32_t *)(smem + Sh::kOffMisc);
  const AbortFlag ab{smem_u32(smem + Sh::kOffMisc + 4)};

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.y, b = blockIdx.z;
  const int rank = (int)cluster_rank(), ranks = (int)cluster_size();
  const int L = p.seq_lens == nullptr ? p.N : min(max(p.seq_lens[b], 0), p.N);
  const size_t bh = (size_t)b * p.H + h, orow = (size_t)p.H * D;
  O *out = (O *)p.out + ((size_t)b * p.N * p.H + h) * D;  // token t at t * orow

  if (p.zero_pad) {  // the rows past the end, shared among the cluster's CTAs
    constexpr int kPer = D * (int)sizeof(O) / 16;
    for (long long i = (long long)rank * Sh::kThreads + tid; i < (long long)(p.N - L) * kPer;
         i += (long long)ranks * Sh::kThreads)
      ((uint4 *)(out + (L + i / kPer) * orow))[i % kPer] = make_uint4(0, 0, 0, 0);
  }
  // The CTA's chunks by their place in scan order: [q0, q0 + cnt) of nc.
  const int nc = (L + kC - 1) / kC;
  const int seg = max(1, (nc + ranks - 1) / ranks);
  const int last_rank = nc > 0 ? min(ranks - 1, (nc - 1) / seg) : 0;
  const int q0 = rank * seg;
  const int cnt = rank > last_rank ? 0 : (rank == last_rank ? nc - q0 : seg);
  const bool is_last = rank == last_rank;
  if (cnt == 0) {
    if (rank == 0 && p.fin)  // an empty sequence passes its state on
      for (int i = tid; i < D * D; i += Sh::kThreads)
        p.fin[bh * D * D + i] = p.init ? p.init[bh * D * D + i] * p.init_scale * p.fin_scale : 0.f;
    return;
  }
  const int pre = is_last ? 0 : cnt;  // chunks of the pass over the segment's own state
  const float l2 = __ldg(p.log_decay + h) * 1.4426950408889634f;

  if (tid == 0) {
    *(volatile int *)(smem + Sh::kOffMisc + 4) = 0;
    for (int i = 0; i < Sh::kNX; ++i) mbar_init(&fx[i], Sh::kB), mbar_init(&ex[i], 1);
    for (int i = 0; i < Sh::kNY; ++i) mbar_init(&fy[i], Sh::kB), mbar_init(&ey[i], 1);
    for (int i = 0; i < Sh::kNZ; ++i) mbar_init(&fz[i], Sh::kB), mbar_init(&ez[i], 1);
    for (int i = 0; i < Sh::kConv; ++i) mbar_init(&conv_full[i], 4), mbar_init(&conv_empty[i], 1);
    for (int i = 0; i < Sh::kP; ++i) mbar_init(&p_full[i], 4), mbar_init(&p_empty[i], 1);
    for (int i = 0; i < Sh::kO; ++i) mbar_init(&o_full[i], 1), mbar_init(&o_empty[i], 4);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], Sh::kSWarps);
      mbar_init(&sc_full[i], 1);
      mbar_init(&sc_empty[i], 4);
    }
    mbar_init(s_empty, 1);
    mbar_init(ds_full, 1);
    mbar_init(ds_empty, Sh::kSWarps);
    mbar_init(drained, 1);
    fence_mbar_init();
  }
  if (warp == Sh::kTmaWarp && lane == 0) {
    tma_prefetch_desc(&tm_x);
    tma_prefetch_desc(&tm_y);
    tma_prefetch_desc(&tm_z);
  }
  if (warp == Sh::kMmaWarp) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const bool state_warp = warp >= 8 && warp < 8 + Sh::kSWarps;
  if (ranks > 1 && !state_warp) cluster_arrive();

  // Step g of the CTA (its own-state pass, then the scan): the chunk's place in
  // scan order, and its first token.
  auto place_of = [&](int g) { return g < pre ? q0 + cnt - 1 - g : q0 + g - pre; };
  auto token_of = [&](int place) { return (p.reverse ? nc - 1 - place : place) * kC; };

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
      const int first = t == 0 ? pre : 0, steps = pre + cnt - first;  // x: the scan alone
      int i = 0;
      for (; i < steps; ++i) {
        const int s = i % slots;
        if (!mbar_wait(&e[s], ((i / slots) & 1) ^ 1, &ab)) {
          decay_error(1, ab);
          break;
        }
        mbar_arrive_expect_tx(&f[s], kBlk);
        tma_load_4d(to + s * size, tm, &f[s], blk * 64, hd, token_of(place_of(first + i)), b);
      }
      if (i < steps)  // gave up: no copy may land after the CTA is gone
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
      // the chunk's own state, sum of (v_j y_j) z_j^T; own: in the pass over the
      // segment's own state, after which the tiles are free
      auto state_mma = [&](int g, bool own) {
        const int cb = g % Sh::kConv, sz = g % Sh::kNZ;
        if (!wait(&fz[sz], (g / Sh::kNZ) & 1)) return;
        if (!wait(&conv_full[cb], (g / Sh::kConv) & 1)) return;
        if (g >= 1 && !wait(ds_empty, (g & 1) ^ 1)) return;
        tc_fence_after();
        const uint64_t zd = sw128_desc(base + Sh::kOffZ + sz * Sh::kTile, kBlk, 1024);
        const uint64_t cd =
            sw128_desc(base + Sh::kOffConv + cb * kTerms * Sh::kTile, kBlk, 1024);
        const uint32_t d = tmem + Sh::kColDs;
        if constexpr (Sh::kMerged) {
          // transposed (M = e): the first two terms side by side in N, the third
          // onto the second
          constexpr uint32_t id2 = idesc_bf16_f32(64, 128, 1, 1), id1 = idesc_bf16_f32(64, 64, 1, 1);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_bf16(d, desc_at(zd, k * 2048), desc_at(cd, k * 2048), id2, k != 0);
          if constexpr (kTerms == 3)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_bf16(d + 64, desc_at(zd, k * 2048), desc_at(cd, 2 * Sh::kTile + k * 2048), id1, 1);
        } else {
          constexpr uint32_t id_s = idesc_bf16_f32(D, D, 1, 1);
#pragma unroll
          for (int t = kTerms - 1; t >= 0; --t)  // the small terms first
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_bf16(d, desc_at(cd, t * Sh::kTile + k * 2048), desc_at(zd, k * 2048), id_s,
                       t != kTerms - 1 || k != 0);
        }
        mma_commit(ds_full);
        mma_commit(&conv_empty[cb]);
        if (own) {
          mma_commit(&ey[g % Sh::kNY]);
          mma_commit(&ez[sz]);
        }
      };
      // scores of the scan's chunk i; merged: and x_r^T S.  The chunk's state
      // went before, so its keys are there and those past the end are zero.
      auto score_mma = [&](int i) {
        const int sx = i % Sh::kNX, sy = (pre + i) % Sh::kNY;
        if (!wait(&fx[sx], (i / Sh::kNX) & 1)) return;
        if (i >= 2 && !wait(&sc_empty[i & 1], ((i >> 1) & 1) ^ 1)) return;
        if constexpr (Sh::kMerged) {
          if (i >= 2 && !wait(&o_empty[i & 1], ((i >> 1) & 1) ^ 1)) return;
          if (!wait(&s_full[i & 1], (i >> 1) & 1)) return;
        }
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
        if (i >= 1 && !wait(&o_empty[0], (i & 1) ^ 1)) return;
        if (!wait(&s_full[i & 1], (i >> 1) & 1)) return;
        tc_fence_after();
        constexpr uint32_t id = idesc_bf16_f32(64, D, 0, 1);
        const uint64_t xd = sw128_desc(base + Sh::kOffX + sx * Sh::kTile, 16, 1024);
        const uint64_t sd = sw128_desc(base + Sh::kOffS, D * 128, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_bf16(tmem + Sh::kColInter, desc_at(xd, (k >> 2) * kBlk + (k & 3) * 32),
                   desc_at(sd, k * 2048), id, k != 0);
        mma_commit(s_empty);
        mma_commit(&ex[sx]);
      };
      auto intra_mma = [&](int j) {  // sum_j (w_rj A_rj) z_j
        const int g = pre + j, sz = g % Sh::kNZ, pb = j % Sh::kP, ob = j % Sh::kO;
        if (!wait(&p_full[pb], (j / Sh::kP) & 1)) return;
        tc_fence_after();
        constexpr uint32_t id = idesc_bf16_f32(64, D, 0, 1);
        const uint64_t pd = sw128_desc(base + Sh::kOffP + pb * kBlk, 16, 1024);
        const uint64_t zd = sw128_desc(base + Sh::kOffZ + sz * Sh::kTile, kBlk, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16(tmem + Sh::kColIntra + Sh::kIntraStep * ob, desc_at(pd, k * 32),
                   desc_at(zd, k * 2048), id, k != 0);
        mma_commit(&p_empty[pb]);
        mma_commit(&o_full[ob]);
        mma_commit(&ez[sz]);
      };
      for (int g = 0; g < pre && ok; ++g) state_mma(g, true);
      if (ok) state_mma(pre, false);
      // Scores of chunk i, results of chunk i - 1 (whose scores have been
      // weighted meanwhile), state of chunk i + 1 (which leaves a whole round for
      // the state to reach the scores of i + 1).
      for (int i = 0; i <= cnt && ok; ++i) {
        if (i < cnt) score_mma(i);
        if (i >= 1 && ok) intra_mma(i - 1);
        if (i + 1 < cnt && ok) state_mma(pre + i + 1, false);
        if constexpr (!Sh::kMerged)
          if (i < cnt && ok) inter_mma(i);
      }
      mma_commit(drained);  // nothing is in flight when TMEM is freed
      if (!mbar_wait(drained, 0, nullptr)) decay_error(512, ab);
    }
    __syncwarp();
  } else if (warp < 4) {
    // ------------------------------------------- weighted scores (warps 0-3)
    const int r0 = 16 * warp + (lane >> 2), c = 2 * (lane & 3);
    float w[9][2];  // exponent e0 -+ 8 k, one less (more) for the second column
#pragma unroll
    for (int k = 0; k < 9; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int n = (p.reverse ? -1 : 1) * (r0 - c - e - 8 * (k - 1));
        w[k][e] = n >= 0 ? decay_pow(l2, (float)n) : 0.f;
      }
    for (int i = 0; i < cnt; ++i) {
      const int pb = i % Sh::kP;
      if (!mbar_wait(&sc_full[i & 1], (i >> 1) & 1, &ab)) decay_error(4, ab);
      tc_fence_after();
      float a[32];
      tmem_ld_16x64(tmem + ((uint32_t)(32 * warp) << 16) + Sh::kColSc + Sh::kScStep * (i & 1), a);
      tmem_ld_wait_regs(a);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sc_empty[i & 1]);
      if (i >= Sh::kP && !mbar_wait(&p_empty[pb], ((i / Sh::kP) & 1) ^ 1, &ab)) decay_error(8, ab);
      const uint32_t ps = smem_u32(smem + Sh::kOffP + pb * kBlk) + r0 * 128 + c * 2;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t at = ps + ((k ^ (r0 & 7)) << 4);  // row r0 + 8 has the same swizzle
        sts_u32(at, f2_to_bf2(a[4 * k] * w[k + 1][0], a[4 * k + 1] * w[k + 1][1]));
        sts_u32(at + 8 * 128, f2_to_bf2(a[4 * k + 2] * w[k][0], a[4 * k + 3] * w[k][1]));
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[pb]);
    }
  } else if (warp < 8) {
    // --------------------------------------------- weighted keys (warps 4-7)
    const int ct = tid - 128, ch = ct & 7, rr = ct >> 3;  // 16-byte chunk, first row
    float wr[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = rr + 16 * k;
      wr[k] = decay_pow(l2, (float)(p.reverse ? r : kC - 1 - r));
    }
    // one 16-byte piece: kTerms bf16 numbers for each of its 8 products
    auto split = [&](const uint4 &u, float w, uint32_t to) {
      const uint32_t in[4] = {u.x, u.y, u.z, u.w};
      uint32_t o[kTerms][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float2 f = bf2_to_f2(in[e]);
        f.x *= w, f.y *= w;
#pragma unroll
        for (int t = 0; t < kTerms; ++t) {
          o[t][e] = f2_to_bf2(f.x, f.y);
          if (t + 1 < kTerms) {
            const float2 q = bf2_to_f2(o[t][e]);
            f.x -= q.x, f.y -= q.y;  // exact
          }
        }
      }
#pragma unroll
      for (int t = 0; t < kTerms; ++t)
        sts_v4(to + t * Sh::kTile, make_uint4(o[t][0], o[t][1], o[t][2], o[t][3]));
    };
    for (int g = 0; g < pre + cnt; ++g) {
      const int sy = g % Sh::kNY, cb = g % Sh::kConv;
      const int n = min(kC, L - token_of(place_of(g)));
      if (!mbar_wait(&fy[sy], (g / Sh::kNY) & 1, &ab)) decay_error(16, ab);
      if (g >= Sh::kConv && !mbar_wait(&conv_empty[cb], ((g / Sh::kConv) & 1) ^ 1, &ab))
        decay_error(32, ab);
      const uint32_t ys = smem_u32(smem + Sh::kOffY + sy * Sh::kYSlot) + rr * 128 + ((ch ^ (rr & 7)) << 4);
      const uint32_t cs = smem_u32(smem + Sh::kOffConv + cb * kTerms * Sh::kTile) + rr * 128 +
                          ((ch ^ (rr & 7)) << 4);
      if (n == kC) {
#pragma unroll
        for (int blk = 0; blk < Sh::kB; ++blk) {
          uint4 u[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) u[k] = lds_v4(ys + blk * kBlk + k * 2048);
#pragma unroll
          for (int k = 0; k < 4; ++k) split(u[k], wr[k], cs + blk * kBlk + k * 2048);
        }
      } else {
        // the chunk with the sequence's end: padding may hold NaN, so keys, values
        // and weighted keys past the end become 0
        const int sz = g % Sh::kNZ;
        if (!mbar_wait(&fz[sz], (g / Sh::kNZ) & 1, &ab)) decay_error(16, ab);
        const uint32_t zs = smem_u32(smem + Sh::kOffZ + sz * Sh::kTile) + rr * 128 + ((ch ^ (rr & 7)) << 4);
        const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll 1
        for (int k = 0; k < 4 * Sh::kB; ++k) {
          const int r = rr + 16 * (k & 3), off = (k >> 2) * kBlk + (k & 3) * 2048;
          if (r < n) {
            split(lds_v4(ys + off), decay_pow(l2, (float)(p.reverse ? r : n - 1 - r)), cs + off);
            continue;
          }
          sts_v4(ys + off, zero);
          sts_v4(zs + off, zero);
#pragma unroll
          for (int t = 0; t < kTerms; ++t) sts_v4(cs + t * Sh::kTile + off, zero);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&conv_full[cb]);
    }
  } else if (state_warp) {
    // ------------------------------------------------- the state, in registers
    const int sw = warp - 8;
    float S[kNV];
#pragma unroll
    for (int i = 0; i < kNV; ++i) S[i] = 0.f;
    const uint32_t src = tmem + ((uint32_t)(32 * (sw & 3)) << 16) + Sh::kColDs +
                         (D == 64 ? 0 : 64 * (sw >> 2));
    // S = a S + f (the state of step g's chunk)
    auto take = [&](int g, float a, float f) {
      if (!mbar_wait(ds_full, g & 1, &ab)) decay_error(64, ab);
      tc_fence_after();
      if constexpr (D == 64) {
#pragma unroll
        for (int i = 0; i < 32; ++i) S[i] *= a;
#pragma unroll
        for (int t = 0; t < 2; ++t) {  // the small terms first
          float v[32];
          tmem_ld_16x64(src + 64 * (1 - t), v);
          tmem_ld_wait_regs(v);
#pragma unroll
          for (int i = 0; i < 32; ++i) S[i] = fmaf(f, v[i], S[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v[16];
          tmem_ld16(src + 16 * i, v);
          tmem_ld_wait_regs(v);
#pragma unroll
          for (int e = 0; e < 16; ++e) S[16 * i + e] = fmaf(f, v[e], a * S[16 * i + e]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(ds_empty);
    };
    if (ranks > 1) {
      // the segment's own state: chunks from its end in scan order to its start
      for (int g = 0; g < pre; ++g) take(g, 1.f, decay_pow(l2, (float)g * kC));
      constexpr int kThr = Sh::kSWarps * 32;
      const int st = tid - 8 * 32;
      float *part = p.part + bh * ranks * D * D;
      if (pre) {
#pragma unroll
        for (int i = 0; i < kNV; ++i) {
          __stcg(part + ((size_t)rank * kNV + i) * kThr + st, S[i]);
          S[i] = 0.f;
        }
      }
      cluster_arrive();
      cluster_wait();
      for (int s = 0; s < rank; ++s) {
        const float f = decay_pow(l2, (float)(rank - 1 - s) * seg * kC);
#pragma unroll
        for (int i = 0; i < kNV; ++i)
          S[i] = fmaf(f, __ldcg(part + ((size_t)s * kNV + i) * kThr + st), S[i]);
      }
    }
    if (p.init) {
      // tokens between the first state and this segment (reverse: and the last
      // token, which that state belongs to)
      const float n = !p.reverse ? (float)q0 * kC : q0 == 0 ? 0.f : (float)(L - 1 - (nc - q0) * kC);
      const float f = decay_pow(l2, n) * p.init_scale;
      const float *s0 = p.init + bh * D * D;
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        int e;
        const int d = state_at<D>(sw, lane, i, &e);
        S[i] = fmaf(f, __ldg(s0 + (p.init_t ? e * D + d : d * D + e)), S[i]);
      }
    }
    for (int j = 0; j < cnt; ++j) {
      if constexpr (D == 64) {  // behind the chunk's keys, once their slot is free
        const int g = pre + j, sy = g % Sh::kNY;
        if (!mbar_wait(&ey[sy], ((g / Sh::kNY) & 1) ^ 1, &ab)) decay_error(128, ab);
        const int e = 16 * sw + (lane >> 2);
        const uint32_t row = smem_u32(smem + Sh::kOffY + sy * Sh::kYSlot + Sh::kTile) + e * 128 +
                             (lane & 3) * 4;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t at = row + ((k ^ (e & 7)) << 4);
          sts_u32(at, f2_to_bf2(S[4 * k], S[4 * k + 1]));
          sts_u32(at + 8 * 128, f2_to_bf2(S[4 * k + 2], S[4 * k + 3]));
        }
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
      if (lane == 0) mbar_arrive(&s_full[j & 1]);
      const int t0 = token_of(q0 + j), n = min(kC, L - t0);
      const int span = !p.reverse ? n : (q0 + j == 0 ? n - 1 : kC);
      take(pre + j, decay_pow(l2, (float)span), 1.f);
    }
    if (p.fin && is_last) {
      const float f = p.fin_scale * (p.reverse ? decay_pow(l2, 1.f) : 1.f);
#pragma unroll
      for (int i = 0; i < kNV; ++i) {
        int e;
        const int d = state_at<D>(sw, lane, i, &e);
        p.fin[bh * D * D + d * D + e] = S[i] * f;
      }
    }
  } else {
    // ---------------------------------------------------------------- results
    const int ow = warp - Sh::kOutWarp, r0 = 16 * ow + (lane >> 2);
    const uint32_t quarter = tmem + ((uint32_t)(32 * ow) << 16);
    float u[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
      u[k] = p.scale * decay_pow(l2, (float)(p.reverse ? kC - (r0 + 8 * k) : r0 + 8 * k + 1));
    for (int j = 0; j < cnt; ++j) {
      const int ob = j % Sh::kO, t0 = token_of(q0 + j), n = min(kC, L - t0);
      float ur[2] = {u[0], u[1]};
      if (p.reverse && q0 + j == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
          ur[k] = p.scale * decay_pow(l2, (float)max(n - 1 - (r0 + 8 * k), 0));
      }
      if (!mbar_wait(&o_full[ob], (j / Sh::kO) & 1, &ab)) decay_error(256, ab);
      tc_fence_after();
#pragma unroll
      for (int blk = 0; blk < Sh::kB; ++blk) {
        float a[32], s[32];
        tmem_ld_16x64(quarter + Sh::kColIntra + Sh::kIntraStep * ob + blk * 64, a);
        tmem_ld_16x64(quarter + Sh::kColInter + Sh::kInterStep * ob + blk * 64, s);
        tmem_ld_wait_regs(a);
        tmem_pin(s);
        if (blk == Sh::kB - 1) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&o_empty[ob]);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) a[i] = fmaf(ur[(i >> 1) & 1], s[i], a[i] * p.scale);
        if constexpr (sizeof(O) == 4) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int q = 0; q < 2; ++q)
              if (r0 + 8 * q < n)
                *(float2 *)(out + (size_t)(t0 + r0 + 8 * q) * orow + blk * 64 + 8 * k +
                            2 * (lane & 3)) = make_float2(a[4 * k + 2 * q], a[4 * k + 2 * q + 1]);
        } else {
          // four lanes hold the four words of a 16-byte piece: each lane gathers
          // the whole pieces lane % 4 and lane % 4 + 4 of both rows
          const int l4 = lane & 3;
#pragma unroll
          for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              uint32_t m[4], t[4];
#pragma unroll
              for (int k = 0; k < 4; ++k)
                m[k] = f2_to_bf2(a[16 * hf + 4 * k + 2 * q], a[16 * hf + 4 * k + 2 * q + 1]);
              // 4 x 4 transpose over the lanes: exchange with lane ^ 1, then lane ^ 2
              const bool b0 = l4 & 1, b1 = l4 & 2;
              const uint32_t x0 = __shfl_xor_sync(0xffffffffu, b0 ? m[0] : m[1], 1);
              const uint32_t x1 = __shfl_xor_sync(0xffffffffu, b0 ? m[2] : m[3], 1);
              t[0] = b0 ? x0 : m[0], t[1] = b0 ? m[1] : x0;
              t[2] = b0 ? x1 : m[2], t[3] = b0 ? m[3] : x1;
              const uint32_t y0 = __shfl_xor_sync(0xffffffffu, b1 ? t[0] : t[2], 2);
              const uint32_t y1 = __shfl_xor_sync(0xffffffffu, b1 ? t[1] : t[3], 2);
              const uint4 v = b1 ? make_uint4(y0, y1, t[2], t[3]) : make_uint4(t[0], t[1], y0, y1);
              if (r0 + 8 * q < n)
                *(uint4 *)(out + (size_t)(t0 + r0 + 8 * q) * orow + blk * 64 + 8 * (4 * hf + l4)) = v;
            }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == Sh::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (ranks > 1 && !state_warp) cluster_wait();
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

// CTAs per sequence.  A CTA's time is its chunks, half of them again for the
// pass over its own state; a launch takes the longest sequence's CTA or, where
// that is more, all of them over the SMs (in whole rounds when the lengths are
// known to be equal).  Lengths that only the device knows are taken to be a
// quarter of the longest on average.
int cluster_for(const ScanArgs &a) {
  const int nc = (a.N + kC - 1) / kC, sms = sm_count();
  const double pairs = (double)a.B * a.H;
  int best = 1;
  double least = 0;
  for (int cs = 1; cs <= kMaxCluster; cs *= 2) {
    if (cs > 1 && nc < 4 * cs) break;
    const double one = cs == 1 ? nc : 1.5 * ((nc + cs - 1) / cs);
    const double rounds = pairs * cs / sms;
    double t;
    if (a.seq_lens)
      t = one > one * rounds / 4 ? one : one * rounds / 4;
    else
      t = one * (double)(long long)(rounds + 0.999999);
    if (cs == 1 || t < 0.95 * least) best = cs, least = t;
  }
  return best;
}

template <int D, int kTerms, typename O>
cudaError_t launch(const ScanArgs &a, const TcParams &p, int cs, const CUtensorMap &tx,
                   const CUtensorMap &ty, const CUtensorMap &tz, cudaStream_t st) {
  using Sh = Shape<D, kTerms>;
  const auto kernel = decay_kernel<D, kTerms, O>;
  cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cs;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cs, a.H, a.B);
  cfg.blockDim = dim3(Sh::kThreads);
  cfg.dynamicSmemBytes = Sh::kSmem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, p, tx, ty, tz);
}

template <int D>
cudaError_t launch_d(const ScanArgs &a, const TcParams &p, int cs, const CUtensorMap &tx,
                     const CUtensorMap &ty, const CUtensorMap &tz, cudaStream_t st) {
  if (a.fin)
    return a.out_f32 ? launch<D, 3, float>(a, p, cs, tx, ty, tz, st)
                     : launch<D, 3, __nv_bfloat16>(a, p, cs, tx, ty, tz, st);
  return a.out_f32 ? launch<D, 2, float>(a, p, cs, tx, ty, tz, st)
                   : launch<D, 2, __nv_bfloat16>(a, p, cs, tx, ty, tz, st);
}

}  // namespace

bool tc_scan_supports(const ScanArgs &a) {
  if (a.dtype != GBLA_BF16 || (a.D != 64 && a.D != 128)) return false;
  for (const auto &s : {a.sx, a.sy, a.sz})  // the stride limit of a tensor map
    if (s[0] >= (1ll << 39) || s[1] >= (1ll << 39)) return false;
  int dev = 0, major = 0, minor = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
  cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
  return major == 10 && minor == 3 && encode_fn() != nullptr;
}

size_t tc_scan_floats(const ScanArgs &a) {
  const int cs = cluster_for(a);
  return cs > 1 ? (size_t)a.B * a.H * cs * a.D * a.D : 0;
}

cudaError_t tc_scan(const ScanArgs &a, float *scratch, cudaStream_t st) {
  CUtensorMap tx, ty, tz;
  cudaError_t e;
  if ((e = make_map(&tx, a.x, a.B, a.N, a.H / a.gx, a.D, a.sx)) != cudaSuccess) return e;
  if ((e = make_map(&ty, a.y, a.B, a.N, a.H / a.gy, a.D, a.sy)) != cudaSuccess) return e;
  if ((e = make_map(&tz, a.z, a.B, a.N, a.H / a.gz, a.D, a.sz)) != cudaSuccess) return e;
  TcParams p = {};
  p.out = a.out, p.log_decay = a.log_decay, p.seq_lens = a.seq_lens;
  p.init = a.init, p.fin = a.fin, p.part = scratch;
  p.init_scale = a.init_scale, p.fin_scale = a.fin_scale, p.scale = a.scale;
  p.N = a.N, p.H = a.H, p.gx = a.gx, p.gy = a.gy, p.gz = a.gz;
  p.zero_pad = a.zero_pad, p.init_t = a.init_t, p.reverse = a.reverse;
  const int cs = cluster_for(a);
  return a.D == 64 ? launch_d<64>(a, p, cs, tx, ty, tz, st)
                   : launch_d<128>(a, p, cs, tx, ty, tz, st);
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
