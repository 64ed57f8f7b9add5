// Decayed linear attention on tensor cores (tcgen05 + TMA): bf16, D in {64, 128}.
//
// The scan of ScanArgs in chunks of C = 64 tokens, in scan order.  With r, j the
// places in a chunk, S the state before it and gamma the head's decay,
//   scores  A_rj  = x_r . y_j                        (M64 N64 KD)
//   results out_r = scale [ sum_j (w_rj A_rj) z_j + u_r x_r^T S ]
//                                                    (M64 ND K64, M64 ND KD)
//   state   S'    = c S + sum_j (v_j y_j) z_j^T      (MD ND K64)
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
  static constexpr int kB = D / 64;                        // 64-channel blocks
  static constexpr int kTile = kB * kBlk;                  // one tensor's chunk
  static constexpr int kStages = D == 64 ? 5 : (kTerms == 2 ? 3 : 2);
  static constexpr int kConv = D == 64 ? 2 : 1;            // buffers of v_j y_j
  static constexpr int kP = D == 64 ? 2 : 1;               // of weighted scores
  static constexpr int kS = D == 64 ? 2 : 1;               // of the rounded state
  static constexpr int kO = D == 64 ? 2 : 1;               // of the results' accumulators
  static constexpr int kDs = D == 64 ? 2 : 1;              // of the chunk's state
  static constexpr int kSBytes = D * D * 2;
  static constexpr int kOffConv = kStages * 3 * kTile;
  static constexpr int kOffP = kOffConv + kConv * kTerms * kTile;
  static constexpr int kOffS = kOffP + kP * kBlk;
  static constexpr int kOffBar = kOffS + kS * kSBytes;
  static constexpr int kBars = 2 * (kStages + kConv + kP + kS + kO + kDs) + 5;
  static constexpr int kOffMisc = kOffBar + kBars * 8;
  static constexpr int kSmem = kOffMisc + 16 + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
  static constexpr int kSWarps = D == 64 ? 4 : 8;
  static constexpr int kOutWarp = 8 + kSWarps, kTmaWarp = kOutWarp + 4, kMmaWarp = kTmaWarp + 1;
  static constexpr int kThreads = (kMmaWarp + 1) * 32;
  static constexpr int kLoads = 3 * kB;                    // issuing lanes
  // TMEM columns: scores [0, 128), per result buffer intra and inter, then the state
  static constexpr uint32_t kColO = 128, kColDs = 384;
  static_assert(kColO + kO * 2 * D <= kColDs && kColDs + kDs * D <= 512, "TMEM");
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

// The state rows of a thread: D = 64, rows and columns as tmem_ld_16x64 gives
// them; D = 128, one row and 64 columns.
template <int D>
__device__ __forceinline__ int state_at(int sw, int lane, int i, int *e) {
  if (D == 64) {
    *e = 8 * (i >> 2) + 2 * (lane & 3) + (i & 1);
    return 16 * sw + (lane >> 2) + 8 * ((i >> 1) & 1);
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
  uint64_t *full = bar, *empty = full + Sh::kStages, *conv_full = empty + Sh::kStages,
           *conv_empty = conv_full + Sh::kConv, *p_full = conv_empty + Sh::kConv,
           *p_empty = p_full + Sh::kP, *s_full = p_empty + Sh::kP, *s_empty = s_full + Sh::kS,
           *o_full = s_empty + Sh::kS, *o_empty = o_full + Sh::kO, *ds_full = o_empty + Sh::kO,
           *ds_empty = ds_full + Sh::kDs, *sc_full = ds_empty + Sh::kDs, *sc_empty = sc_full + 2,
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
    for (int i = 0; i < Sh::kStages; ++i) mbar_init(&full[i], Sh::kLoads), mbar_init(&empty[i], 1);
    for (int i = 0; i < Sh::kConv; ++i) mbar_init(&conv_full[i], 4), mbar_init(&conv_empty[i], 1);
    for (int i = 0; i < Sh::kP; ++i) mbar_init(&p_full[i], 4), mbar_init(&p_empty[i], 1);
    for (int i = 0; i < Sh::kS; ++i) mbar_init(&s_full[i], Sh::kSWarps), mbar_init(&s_empty[i], 1);
    for (int i = 0; i < Sh::kO; ++i) mbar_init(&o_full[i], 1), mbar_init(&o_empty[i], 4);
    for (int i = 0; i < Sh::kDs; ++i)
      mbar_init(&ds_full[i], 1), mbar_init(&ds_empty[i], Sh::kSWarps);
    for (int i = 0; i < 2; ++i) mbar_init(&sc_full[i], 1), mbar_init(&sc_empty[i], 4);
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
      int g = 0;
      for (; g < pre + cnt; ++g) {
        const int s = g % Sh::kStages;
        if (!mbar_wait(&empty[s], ((g / Sh::kStages) & 1) ^ 1, &ab)) {
          decay_error(1, ab);
          break;
        }
        if (t == 0 && g < pre) {
          mbar_arrive(&full[s]);
          continue;
        }
        mbar_arrive_expect_tx(&full[s], kBlk);
        tma_load_4d(smem + (s * 3 + t) * Sh::kTile + blk * kBlk, tm, &full[s], blk * 64, hd,
                    token_of(place_of(g)), b);
      }
      if (g < pre + cnt)  // gave up: no copy may land after the CTA is gone
        for (int f = max(0, g - Sh::kStages); f < g; ++f)
          mbar_wait(&full[f % Sh::kStages], (f / Sh::kStages) & 1, nullptr);
    }
    __syncwarp();
  } else if (warp == Sh::kMmaWarp) {
    // ----------------------------------------------------------------- MMAs
    if (elect_one()) {
      constexpr uint32_t id_sc = idesc_bf16_f32(64, 64, 0, 0);
      constexpr uint32_t id_o = idesc_bf16_f32(64, D, 0, 1);
      constexpr uint32_t id_s = idesc_bf16_f32(D, D, 1, 1);
      const uint32_t base = smem_u32(smem);
      bool ok = true;
      auto wait = [&](uint64_t *m, uint32_t parity) {
        if (ok && !mbar_wait(m, parity, &ab)) decay_error(2, ab), ok = false;
        return ok;
      };
      // the chunk's own state: sum of (v_j y_j) z_j^T, the small terms first
      auto state_mma = [&](int g) {
        const int s = g % Sh::kStages, cb = g % Sh::kConv, db = g % Sh::kDs;
        if (!wait(&conv_full[cb], (g / Sh::kConv) & 1)) return;
        if (g >= Sh::kDs && !wait(&ds_empty[db], ((g / Sh::kDs) & 1) ^ 1)) return;
        tc_fence_after();
        const uint32_t zs = base + (s * 3 + 2) * Sh::kTile;
        const uint32_t d = tmem + Sh::kColDs + db * D;
#pragma unroll
        for (int t = kTerms - 1; t >= 0; --t) {
          const uint32_t cs = base + Sh::kOffConv + (cb * kTerms + t) * Sh::kTile;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_bf16(d, sw128_desc(cs + k * 2048, kBlk, 1024), sw128_desc(zs + k * 2048, kBlk, 1024),
                     id_s, t != kTerms - 1 || k != 0);
        }
        mma_commit(&ds_full[db]);
        mma_commit(&conv_empty[cb]);
      };
      for (int g = 0; g < pre && ok; ++g) {
        const int s = g % Sh::kStages;
        if (!wait(&full[s], (g / Sh::kStages) & 1)) break;
        state_mma(g);
        mma_commit(&empty[s]);
      }
      auto score_mma = [&](int i) {
        const int g = pre + i, s = g % Sh::kStages;
        if (!wait(&full[s], (g / Sh::kStages) & 1)) return;
        // rows past the end are zeroed with the weighted keys of the same chunk
        if (token_of(q0 + i) + kC > L && !wait(&conv_full[g % Sh::kConv], (g / Sh::kConv) & 1))
          return;
        if (i >= 2 && !wait(&sc_empty[i & 1], ((i >> 1) & 1) ^ 1)) return;
        tc_fence_after();
        const uint32_t xs = base + s * 3 * Sh::kTile, ys = xs + Sh::kTile;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = (k >> 2) * kBlk + (k & 3) * 32;
          mma_bf16(tmem + 64 * (i & 1), sw128_desc(xs + off, 16, 1024),
                   sw128_desc(ys + off, 16, 1024), id_sc, k != 0);
        }
        mma_commit(&sc_full[i & 1]);
      };
      auto rest_mma = [&](int j) {
        const int g = pre + j, s = g % Sh::kStages, ob = j % Sh::kO, sb = j % Sh::kS,
                  pb = j % Sh::kP;
        state_mma(g);
        if (!ok) return;
        if (j >= Sh::kO && !wait(&o_empty[ob], ((j / Sh::kO) & 1) ^ 1)) return;
        if (!wait(&s_full[sb], (j / Sh::kS) & 1)) return;
        tc_fence_after();
        const uint32_t xs = base + s * 3 * Sh::kTile, zs = xs + 2 * Sh::kTile;
        const uint32_t ss = base + Sh::kOffS + sb * Sh::kSBytes;
        const uint32_t intra = tmem + Sh::kColO + ob * 2 * D, inter = intra + D;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_bf16(inter, sw128_desc(xs + (k >> 2) * kBlk + (k & 3) * 32, 16, 1024),
                   sw128_desc(ss + k * 2048, D * 128, 1024), id_o, k != 0);
        mma_commit(&s_empty[sb]);
        if (!wait(&p_full[pb], (j / Sh::kP) & 1)) return;
        tc_fence_after();
        const uint32_t ps = base + Sh::kOffP + pb * kBlk;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16(intra, sw128_desc(ps + k * 32, 16, 1024), sw128_desc(zs + k * 2048, kBlk, 1024),
                   id_o, k != 0);
        mma_commit(&p_empty[pb]);
        mma_commit(&o_full[ob]);
        mma_commit(&empty[s]);
      };
      for (int i = 0; i <= cnt && ok; ++i) {
        // the scores of the next chunk go out before the rest of this one; not
        // those of a chunk cut short, which wait for its weighted keys
        const bool cut = i < cnt && token_of(q0 + i) + kC > L;
        if (i < cnt && !cut) score_mma(i);
        if (i >= 1 && ok) rest_mma(i - 1);
        if (cut && ok) score_mma(i);
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
      tmem_ld_16x64(tmem + ((uint32_t)(32 * warp) << 16) + 64 * (i & 1), a);
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
    for (int g = 0; g < pre + cnt; ++g) {
      const int s = g % Sh::kStages, cb = g % Sh::kConv;
      const int n = min(kC, L - token_of(place_of(g)));
      if (!mbar_wait(&full[s], (g / Sh::kStages) & 1, &ab)) decay_error(16, ab);
      if (g >= Sh::kConv && !mbar_wait(&conv_empty[cb], ((g / Sh::kConv) & 1) ^ 1, &ab))
        decay_error(32, ab);
      const uint32_t ys = smem_u32(smem + (s * 3 + 1) * Sh::kTile);
      const uint32_t cs = smem_u32(smem + Sh::kOffConv + cb * kTerms * Sh::kTile);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = rr + 16 * k;
        float w = wr[k];
        if (n < kC && !p.reverse) w = r < n ? decay_pow(l2, (float)(n - 1 - r)) : 0.f;
#pragma unroll
        for (int blk = 0; blk < Sh::kB; ++blk) {
          const uint32_t at = blk * kBlk + r * 128 + ((ch ^ (r & 7)) << 4);
          if (r >= n) {  // padding may hold NaN: keys, values and weighted keys become 0
            const uint4 z = make_uint4(0, 0, 0, 0);
            sts_v4(ys + at, z);
            sts_v4(ys + Sh::kTile + at, z);
#pragma unroll
            for (int t = 0; t < kTerms; ++t) sts_v4(cs + t * Sh::kTile + at, z);
            continue;
          }
          const uint4 u = lds_v4(ys + at);
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
            sts_v4(cs + t * Sh::kTile + at, make_uint4(o[t][0], o[t][1], o[t][2], o[t][3]));
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
    const uint32_t dst = tmem + ((uint32_t)(32 * (sw & 3)) << 16) + Sh::kColDs +
                         (D == 64 ? 0 : 64 * (sw >> 2));
    // S = a S + f (the state of step g's chunk)
    auto take = [&](int g, float a, float f) {
      const int db = g % Sh::kDs;
      if (!mbar_wait(&ds_full[db], (g / Sh::kDs) & 1, &ab)) decay_error(64, ab);
      tc_fence_after();
      if constexpr (D == 64) {
        float v[32];
        tmem_ld_16x64(dst + db * D, v);
        tmem_ld_wait_regs(v);
#pragma unroll
        for (int i = 0; i < 32; ++i) S[i] = fmaf(f, v[i], a * S[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v[16];
          tmem_ld16(dst + db * D + 16 * i, v);
          tmem_ld_wait_regs(v);
#pragma unroll
          for (int e = 0; e < 16; ++e) S[16 * i + e] = fmaf(f, v[e], a * S[16 * i + e]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ds_empty[db]);
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
      const int sb = j % Sh::kS;
      if (j >= Sh::kS && !mbar_wait(&s_empty[sb], ((j / Sh::kS) & 1) ^ 1, &ab))
        decay_error(128, ab);
      const uint32_t ss = smem_u32(smem + Sh::kOffS + sb * Sh::kSBytes);
      if constexpr (D == 64) {
        const int d = 16 * sw + (lane >> 2);
        const uint32_t row = ss + d * 128 + (lane & 3) * 4;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t at = row + ((k ^ (d & 7)) << 4);
          sts_u32(at, f2_to_bf2(S[4 * k], S[4 * k + 1]));
          sts_u32(at + 8 * 128, f2_to_bf2(S[4 * k + 2], S[4 * k + 3]));
        }
      } else {
        const int d = 32 * (sw & 3) + lane;
        const uint32_t row = ss + (sw >> 2) * (D * 128) + d * 128;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          sts_v4(row + ((k ^ (d & 7)) << 4),
                 make_uint4(f2_to_bf2(S[8 * k], S[8 * k + 1]), f2_to_bf2(S[8 * k + 2], S[8 * k + 3]),
                            f2_to_bf2(S[8 * k + 4], S[8 * k + 5]),
                            f2_to_bf2(S[8 * k + 6], S[8 * k + 7])));
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_full[sb]);
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
    const uint32_t quarter = tmem + ((uint32_t)(32 * ow) << 16) + Sh::kColO;
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
        tmem_ld_16x64(quarter + ob * 2 * D + blk * 64, a);
        tmem_ld_16x64(quarter + ob * 2 * D + D + blk * 64, s);
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
