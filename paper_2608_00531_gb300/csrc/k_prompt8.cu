// Attention of packed rows over a cache held in 8 bits (e4m3 codes, a scale for each block
// of 16 slots and head), on tcgen05 tensor cores: causal (cure_prompt_attn8), or a repair
// tree's rows in place (cure_tree_attn8).
//
//   out_i = sum_j softmax_j(c q_i k_j) v_j,   k_j = ks_j K_j,  v_j = vs_j V_j
//
// with codes K, V and their blocks' scales ks, vs.
//
// Scores.  K goes from memory to the tensor cores as it is.  q (8 significant bits) is two
// e4m3 values (4 bits each): with its row scaled by a power of two to at most 448,
//   q = q1 + q2,  q1 = e4m3(q),  q2 = e4m3(q - q1)
// is exact but for q2's smallest step, 2^-9: at most 2^-10 where the row's largest value is above 224, 2^-17 of that.
// S = q1 K + q2 K are 8 products of 32 dims where bf16 has 8 of 16, at twice the rate.
//
// Weights.  V's codes are widened to fp16 (exact), and P is fp16 with the block's scale in it:
//   P'_j = 2^(s_j + log2 vs_j - M + 7),  M the running maximum of s_j + log2 vs_j
// so that a rounding is relative to what a term adds to the output, whatever the scales, and
// the smallest steps (2^-24 of fp16) are 2^-31 of the largest term.  The sum of weights is
// kept in float32 as sum_blocks (sum P') / vs.
//
// Units, pieces and the scheduler are those of the bf16 kernel (prompt_units.cuh).  Roles (16
// warps):
//   warps 0-3 / 4-7   Q of M tile 0 / 1 into its parts, and its softmax, a thread a row
//   warp 8            TMA producer: Q, K and V tiles (16 KiB each), and the blocks' scales
//   warp 9            issues S = Q K^T (M128 N128, K 2 x 128) of M tiles 0 and 1 in turn
//   warp 10           issues O += P' V (A = P' from TMEM)
//   warp 11           lays out the CTA's pieces of work
//   warps 12-15       V tiles to fp16, and the epilogue: a piece's rows go out behind the next one's
//                     first V tile
// TMEM as there: S (128) | P[2] (64 each) | O[2] (128 each).  A piece whose rows fit one M
// tile (single tokens, small trees) takes its tiles in turn with both softmax groups, each
// with an O and sums of its own, which the epilogue adds up: a group's exponentials would
// otherwise take longer than a tile's bytes.
//
// Bound: the softmax warps' chain.  A tile of 128 keys and two M tiles takes 1.5 us of their exponentials,
// sums and conversions (the products' own time is 1.1), and a unit about 5 us on top until its first scores
// are there and its last rows out.  One document of 16384 tokens, 64 heads and 8 of K and V: 2.83 ms, 1.55
// PFLOP/s of the attention's operations; 32 prompts of 33 to 4096 tokens, 28 heads and 4: 247 us.  The blocks'
// largest scores come with the scores from TMEM (tcgen05.ld.red): found in registers, 260 us and 3.06 ms.  Q taken
// apart by warps 12-15 in front of the piece's V tiles cost 25 us of the prompts, Q asked for behind the first
// V tile instead of in front of the first K tile 6.  Registers of a thread for softmax, warps 12-15 and the
// rest: 168 / 88 / 88 (184 / 80 / 64 took 274 us where they took 263, 160 / 104 / 88 282; a few words spill in each).
#include "prompt8.cuh"

namespace cure {
namespace {

using namespace prompt;

constexpr int kBlk = CURE_KV8_BLOCK;
constexpr int kBlocks = BN / kBlk;      // of a tile
constexpr int kTile = BN * D;           // 16 KiB of codes
constexpr int kTileW = kTile * 2;
constexpr int kQuad = 4;                // tiles whose pages and scales are looked up together
constexpr int kScaleSlots = 8;          // quads whose scales lie in shared memory
constexpr int kScaleFloats = 7 * kBlocks;  // of a tile: ks and log2 vs of each block twice, and ks, log2 vs, 1 / vs once

// Shared memory and barriers of the kernel for units of MT M tiles.  With one, Q takes half
// the place, and two more tiles are on their way (which gains nothing where units are cut).
template <int MT>
struct Layout {
  static constexpr int m_tiles = MT, threads = kThreads;
  static constexpr int NK = MT == 1 ? 4 : 3, NV = MT == 1 ? 3 : 2, NW = 2;  // stages: K tiles, V tiles, V tiles in fp16
  enum : int {
    B_QFULL = 0, B_QRAW = 2, B_QEMPTY = 4, B_SFREE = 6,
    B_KFULL, B_KEMPTY = B_KFULL + NK, B_VFULL = B_KEMPTY + NK, B_VEMPTY = B_VFULL + NV,
    B_WFULL = B_VEMPTY + NV, B_WEMPTY = B_WFULL + NW, B_SFULL = B_WEMPTY + NW, B_PFULL = B_SFULL + 2,
    B_PVDONE = B_PFULL + 2, B_STAT = B_PVDONE + 2, B_OFREE = B_STAT + 2, B_DRAIN = B_OFREE + 2, B_JOIN = B_DRAIN + 2,
    B_SCALES = B_JOIN + 1, piece_bar = B_SCALES + kScaleSlots, taken_bar = piece_bar + kPieces,
    B_NEVER = taken_bar + kPieces, num_bars
  };
  static constexpr int q = 0;                        // Q[m][part]
  static constexpr int k = q + MT * 2 * kQHalf;      // K[stage]
  static constexpr int v = k + NK * kTile;           // V[stage]
  static constexpr int w = v + NV * kTile;           // V in fp16[stage]: chunks of 16 keys, [d half][16 keys][64 d]
  static constexpr int bars = w + NW * kTileW;
  static constexpr int tmem_slot = bars + 8 * num_bars;
  static constexpr int abort = tmem_slot + 4;
  static constexpr int joins = abort + 4;                      // units that this CTA joins at its end
  static constexpr int pieces = (joins + 4 + 15) / 16 * 16;    // int [kPieces][kPieceInts], then [2] to join
  static constexpr int prefix = pieces + (kPieces + 2) * kPieceInts * 4;  // int64 first position of each sequence [B+1]
  static constexpr int scales = (prefix + 8 * (kAttnMaxBatch + 1) + 15) / 16 * 16;  // float [slot][tile][kScaleFloats]
  static constexpr int q_scale = scales + kScaleSlots * kQuad * kScaleFloats * 4;   // float [piece % 2][m][row]
  static constexpr int inv = q_scale + 4 * BM * 4;             // float [group][row]: reciprocal row sums
  static constexpr int lse = inv + 2 * BM * 4;                 // float [group][row]: base-2 log-sum-exps
  static constexpr int kept = lse + 2 * BM * 4;                // the epilogue's piece, a copy for each of its warps
  static constexpr int bytes = kept + 4 * kPieceInts * 4;
  static_assert(bytes <= 232448, "fits the 227 KiB opt-in");
};

struct Args8 : PromptArgs {
  const float *k_scale, *v_scale;
  // a tree's rows (Tree8)
  const int32_t* n_nodes;
  const uint64_t* anc;
  int n_max;
  int cluster;  // CTAs of a unit's cluster (CLUSTER)
};
struct Tree8 : Args8 {
  static constexpr bool kTree = true;
};

// Two float as fp16 (lo in the low half), and e4m3 pairs to and from fp16 pairs.
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}\n"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ uint32_t narrow(uint32_t lo, uint32_t hi) {
  uint32_t w;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 a, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, %2;\n\t"
      "mov.b32 %0, {a, b};\n\t}\n"
      : "=r"(w)
      : "r"(lo), "r"(hi));
  return w;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// Lane i of the warp reads TMEM lane (taddr.lane + i), 16 columns.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}

// S = Q_m K^T: 4 steps of 32 dims with q1, then with q2 (kQHalf further on).
__device__ __forceinline__ void issue_s(uint32_t d, uint32_t q, uint32_t q_hi, uint32_t k, uint32_t k_hi, uint32_t idesc,
                                        uint32_t full) {
  static_assert(kQHalf >> 4 == 1024, "as the steps are written");
  asm volatile(
      "{\n\t.reg .pred pf, pt, el;\n\t.reg .b64 a, b0, b1, b2, b3;\n\t.reg .b32 x;\n\t"
      "elect.sync _|el, 0xffffffff;\n\t"
      "setp.ne.b32 pf, 0, 0;\n\t"
      "setp.eq.b32 pt, 0, 0;\n\t"
      "mov.b64 a, {%1, %2};\n\tmov.b64 b0, {%3, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b0, %5, pf;\n\t"
      "add.u32 x, %1, 2;\n\tmov.b64 a, {x, %2};\n\tadd.u32 x, %3, 2;\n\tmov.b64 b1, {x, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b1, %5, pt;\n\t"
      "add.u32 x, %1, 4;\n\tmov.b64 a, {x, %2};\n\tadd.u32 x, %3, 4;\n\tmov.b64 b2, {x, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b2, %5, pt;\n\t"
      "add.u32 x, %1, 6;\n\tmov.b64 a, {x, %2};\n\tadd.u32 x, %3, 6;\n\tmov.b64 b3, {x, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b3, %5, pt;\n\t"
      "add.u32 x, %1, 1024;\n\tmov.b64 a, {x, %2};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b0, %5, pt;\n\t"
      "add.u32 x, %1, 1026;\n\tmov.b64 a, {x, %2};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b1, %5, pt;\n\t"
      "add.u32 x, %1, 1028;\n\tmov.b64 a, {x, %2};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b2, %5, pt;\n\t"
      "add.u32 x, %1, 1030;\n\tmov.b64 a, {x, %2};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b3, %5, pt;\n\t"
      "@el tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%6];\n\t}\n" ::"r"(d),
      "r"(q), "r"(q_hi), "r"(k), "r"(k_hi), "r"(idesc), "r"(full)
      : "memory");
}

// Instruction descriptor with float32 D and A, B of format 0: fp16 in kind::f16, e4m3 in kind::f8f6f4.
__host__ __device__ constexpr uint32_t idesc_0(int M, int N, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

constexpr uint32_t kGaveUp = 0x7fc0dead;  // a NaN that no arithmetic gives: the log-sum-exps of a CTA that gave up
constexpr float kLift = 7.f;  // P' is 2^kLift times what it stands for: at most 2^15 with the lag of 2^8

// ---- clusters: barrier, a peer's address of a shared-memory variable, loads from it
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();  // (what stands before may have left the warp's lanes apart, which an aligned barrier must not meet)
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float ld_cluster(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_cluster_v4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}

// 16 columns of TMEM of the lane's row, and the largest of them.
__device__ __forceinline__ void tmem_ld16_max(uint32_t taddr, uint32_t* r, float& top) {
  asm volatile(
      "tcgen05.ld.red.sync.aligned.32x32b.x16.max.f32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, %16, [%17];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=f"(top)
      : "r"(taddr));
}

// Units of two M tiles; or with CLUSTER (a tree's rows) of one, each with a cluster of A.cluster CTAs to
// itself, which take an equal part of its tiles each and join them through distributed shared memory.  EXPIRE
// (self-test): one wait of one warp runs out.
template <class Args, bool CLUSTER, bool EXPIRE>
__global__ void __launch_bounds__(kThreads, 1)
attn8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
             const __grid_constant__ CUtensorMap tm_q, const Args A) {
  constexpr bool kTree = Args::kTree;
  using Lay = Layout<CLUSTER ? 1 : 2>;
  constexpr int MT = Lay::m_tiles;
  constexpr int NK = Lay::NK, NV = Lay::NV, NW = Lay::NW;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sb = smem_u32(smem);
  if (sb & 1023u) {  // the swizzled tiles need a 1 KiB-aligned base
    if (tid == 0) flag(A.err, CURE_DEVERR_ALIGN);
    return;
  }
  const int G = A.G, npb = BM / G;
  const Bar bar{sb + Lay::bars};
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + Lay::abort);
  const uint32_t aborted = sb + Lay::abort;
  volatile int* n_joins = reinterpret_cast<volatile int*>(smem + Lay::joins);
  float* q_scale = reinterpret_cast<float*>(smem + Lay::q_scale);
  float* row_inv = reinterpret_cast<float*>(smem + Lay::inv);
  float* lse_of = reinterpret_cast<float*>(smem + Lay::lse);

  // ---------------------------------------------------------------- set-up
  if (tid == 0) {
    mbar_init(bar(Lay::B_QFULL), BM);
    mbar_init(bar(Lay::B_QFULL + 1), BM);
    mbar_init(bar(Lay::B_QEMPTY), 1);
    mbar_init(bar(Lay::B_QEMPTY + 1), 1);
    mbar_init(bar(Lay::B_QRAW), 1);
    mbar_init(bar(Lay::B_QRAW + 1), 1);
    mbar_init(bar(Lay::B_SFREE), BM);
    for (int i = 0; i < NK; ++i) {
      mbar_init(bar(Lay::B_KFULL + i), 1);
      mbar_init(bar(Lay::B_KEMPTY + i), 1);
    }
    for (int i = 0; i < NV; ++i) {
      mbar_init(bar(Lay::B_VFULL + i), 1);
      mbar_init(bar(Lay::B_VEMPTY + i), 4);
    }
    for (int i = 0; i < NW; ++i) {
      mbar_init(bar(Lay::B_WFULL + i), 4);
      mbar_init(bar(Lay::B_WEMPTY + i), 1);
    }
    for (int m = 0; m < 2; ++m) {
      mbar_init(bar(Lay::B_SFULL + m), 1);
      mbar_init(bar(Lay::B_PFULL + m), BM);
      mbar_init(bar(Lay::B_PVDONE + m), 1);
      mbar_init(bar(Lay::B_STAT + m), BM);
      mbar_init(bar(Lay::B_OFREE + m), BM);
      mbar_init(bar(Lay::B_DRAIN + m), 1);
    }
    mbar_init(bar(Lay::B_JOIN), BM);
    for (int i = 0; i < kScaleSlots; ++i) mbar_init(bar(Lay::B_SCALES + i), 1);
    for (int i = 0; i < kPieces; ++i) {
      mbar_init(bar(Lay::piece_bar + i), 1);
      mbar_init(bar(Lay::taken_bar + i), kTakers);
    }
    if constexpr (EXPIRE) mbar_init(bar(Lay::B_NEVER), 1);
    *abort_flag = 0;
    *n_joins = 0;
    fence_mbar_init();
  }
  if (warp == 0) tmem_alloc(sb + Lay::tmem_slot, kTmemCols);
  if (warp == 8 && lane == 0) {
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
    tma_prefetch_desc(&tm_q);
  }
  pdl_begin();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + Lay::tmem_slot);
  Await<EXPIRE> await;
  if constexpr (EXPIRE) {
    await.never = bar(Lay::B_NEVER);
    await.left = blockIdx.x == 0 && warp == A.expire_warp ? (uint32_t)A.expire_wait : 0u;
  }
  Pieces pieces{0};
  Piece x;
  // Whether a piece has rows in both M tiles; else both softmax groups take M tile 0's, a tile each in turn.
  auto two_tiles = [&](const Piece& x) { return MT == 2 && (2 * x.rg + 1) * npb < x.n; };

  // (128 * (2 * 168 + 88 + 88) = 512 * 128 registers, what the block was launched with)
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    // ================================================================ softmax
    const int m = warp >> 2;
    const int row = tid & 127;  // row within the M tile = TMEM lane
    const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t tS = tl + kColS, tP = tl + kColP + m * 64, tO = tl + kColO + m * D;
    uint32_t sc = 0, quads = 0, pc = 0;  // tiles of this group, quads and pieces of the CTA
    bool ok = true;
    uint32_t done = 0;  // pieces of this group
    // Q of the group's M tile: bf16 rows (dims 0-63 where q1 goes, the others in q2's place), which each thread
    // takes out and puts back as its row's parts
    uint32_t got = 0;
    const uint32_t q_row = sb + Lay::q + m * 2 * kQHalf + row * 128;
    while (ok && pieces.next<Lay>(await, bar, smem, aborted, x)) {
      const uint32_t at = quads * kQuad;  // the piece's first place among the scales
      quads += (uint32_t)(x.t1 - x.t0 + kQuad - 1) / kQuad;
      const bool two = two_tiles(x);
      const int mq = two ? m : 0, step = two ? 1 : 2;  // the M tile whose rows these are
      const int first = x.t0 + m - mq;
      if (two || m == 0) {
        if (!await(bar(Lay::B_QRAW + m), got++ & 1u, aborted)) break;
        uint4 w[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) w[k] = ld_shared_v4(q_row + (k >> 3) * kQHalf + (((k & 7) ^ (row & 7)) << 4));
        if (row >= npb * G || (MT * x.rg + m) * npb + row / G >= x.n) {
#pragma unroll
          for (int k = 0; k < 16; ++k) w[k] = make_uint4(0u, 0u, 0u, 0u);
        }
        // the row's largest value: bf16 magnitudes in order as integers, two at a time
        __nv_bfloat162 big = __float2bfloat162_rn(0.f);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) big = __hmax2(big, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&u[e])));
        }
        const float amax = fmaxf(__low2float(big), __high2float(big));
        // 2^e, the least with amax <= 448 * 2^e (448 = 1.75 * 2^8), not below 2^-60
        const uint32_t bits = __float_as_uint(amax);
        const int e = min(max((int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u), -60), 120);
        q_scale[((pc & 1u) * 2 + m) * BM + row] = __uint_as_float((uint32_t)(127 + e) << 23);
        const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
        for (int u = 0; u < 8; ++u) {  // 16 dims
          const uint32_t in[8] = {w[2 * u].x,     w[2 * u].y,     w[2 * u].z,     w[2 * u].w,
                                  w[2 * u + 1].x, w[2 * u + 1].y, w[2 * u + 1].z, w[2 * u + 1].w};
          uint32_t q1[4], q2[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t f[2], r[2];
#pragma unroll
            for (int z = 0; z < 2; ++z)
              f[z] = pack_f16(__uint_as_float(in[2 * k + z] << 16) * inv,
                              __uint_as_float(in[2 * k + z] & 0xffff0000u) * inv);
            q1[k] = narrow(f[0], f[1]);
            widen(q1[k], r[0], r[1]);
            q2[k] = narrow(sub_f16x2(f[0], r[0]), sub_f16x2(f[1], r[1]));
          }
          const uint32_t to = q_row + ((u ^ (row & 7)) << 4);
          st_shared_v4(to, q1[0], q1[1], q1[2], q1[3]);
          st_shared_v4(to + kQHalf, q2[0], q2[1], q2[2], q2[3]);
        }
        fence_proxy_async_smem();
        mbar_arrive(bar(Lay::B_QFULL + m));
      }
      const float* qs = q_scale + ((pc++ & 1u) * 2 + mq) * BM + row;
      if (first >= x.t1) continue;
      const int i0 = (MT * x.rg + mq) * npb;
      const int i = i0 + row / G;  // the row's place in its sequence
      const bool idle = (warp & 3) * 32 >= min(npb, x.n - i0) * G;  // no row of the warp is one of the sequence's
      // keys that the row sees (a tree's: at most), the fewest and the most that a row of this warp sees
      const int sees = kTree ? x.L + x.n : x.L + i + 1;
      const int least = kTree ? x.L : __shfl_sync(0xffffffffu, sees, 0), most = __shfl_sync(0xffffffffu, sees, 31);
      float m_run = -INFINITY, l_run = 0.f, c = 0.f;
      for (int t = first; t < x.t1; t += step) {
        if (!await(bar(Lay::B_SFULL + m), sc & 1u, aborted)) { ok = false; break; }
        ++sc;
        tc_fence_after();
        if (idle) {  // its rows of P' and O may hold anything
          mbar_arrive(bar(Lay::B_SFREE));
          if (sc > 1 && !await(bar(Lay::B_PVDONE + m), (sc - 2) & 1u, aborted)) { ok = false; break; }
          mbar_arrive(bar(Lay::B_PFULL + m));
          continue;
        }
        uint32_t v[BN];
        float top[kBlocks];  // each block's largest score
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) tmem_ld16_max(tS + kBlk * b, v + kBlk * b, top[b]);
        tmem_wait_ld();
        tc_fence_before();
        // The row's factor, read before S is given back: that of the piece after the next takes its place.
        // (Within bounds where a block's factor is never 0, which would meet -infinity.)
        if (t == first) c = fminf(fmaxf(A.scale_log2 * *qs, 0x1p-80f), 0x1p80f);
        mbar_arrive(bar(Lay::B_SFREE));  // the next product may take S
        // The tile's scales (the S product has waited for them).  They stay for as long as it takes: their
        // slot is written again for the eighth quad from here, once S of all but its last three tiles is done.
        const float4* scales =
            reinterpret_cast<const float4*>(smem + Lay::scales + (at + (uint32_t)(t - x.t0)) % (kScaleSlots * kQuad) * (kScaleFloats * 4));
        float x_[BN];
#pragma unroll
        for (int k = 0; k < BN; ++k) x_[k] = __uint_as_float(v[k]);
        if ((t + 1) * BN > least) {
          auto largest = [&](int b) -> float {
            const float* y = x_ + b * kBlk;
            float a0 = fmax3(y[0], y[1], y[2]), a1 = fmax3(y[3], y[4], y[5]);
            a0 = fmax3(a0, y[6], y[7]);
            a1 = fmax3(a1, y[8], y[9]);
            a0 = fmax3(a0, y[10], y[11]);
            a1 = fmax3(a1, y[12], y[13]);
            return fmax3(fmaxf(a0, a1), y[14], y[15]);
          };
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int key = t * BN + 32 * q;  // the block's first
            if (key + 32 > least) {
              const int left = min(max(sees - key, 0), 32);  // keys of the block that the row sees
              uint32_t seen = left == 32 ? 0xffffffffu : (1u << left) - 1u;
              if constexpr (kTree) {
                const int words = 2 * ((A.n_max + 63) / 64), base = key - x.L;  // the node of the block's first key
                const uint32_t* anc = reinterpret_cast<const uint32_t*>(A.anc) + (int64_t)(x.r0 + i) * words;
                auto word = [&](int k) -> uint32_t { return i < x.n && k < words ? __ldg(anc + k) : 0u; };
                seen &= base >= 0 ? __funnelshift_r(word(base >> 5), word((base >> 5) + 1), base & 31)
                                  : (word(0) << -base) | ((1u << -base) - 1u);
              }
#pragma unroll
              for (int k = 0; k < 32; ++k) x_[32 * q + k] = (seen >> k) & 1u ? x_[32 * q + k] : -INFINITY;
              top[2 * q] = largest(2 * q);
              top[2 * q + 1] = largest(2 * q + 1);
            }
          }
        }
        // the maximum of s + log2 vs
        float mt = -INFINITY;
#pragma unroll
        for (int b = 0; b < kBlocks; b += 2) {
          const float4 ks = scales[b / 2], lv = scales[kBlocks / 2 + b / 2];
          mt = fmax3(mt, fmaf(top[b], c * ks.x, lv.x), fmaf(top[b + 1], c * ks.z, lv.z));
        }
        const float m_new = fmaxf(m_run, mt);
        const bool need = m_new > m_run + 8.0f;
        const float alpha = need ? ex2(m_run - m_new) : 1.f;
        if (need) m_run = m_new;
        // P's place and O are free once this group's PV product before is done
        if (sc > 1) {
          if (!await(bar(Lay::B_PVDONE + m), (sc - 2) & 1u, aborted)) { ok = false; break; }
          tc_fence_after();
        }
        const float nbase = m_run == -INFINITY ? 0.f : kLift - m_run;
        uint64_t sum = f2_pack(0.f, 0.f);
        auto exponentials = [&](int q) {  // of 32 keys
          // (a block's once each here, twice in the maximum's loads: twice here too takes a document 1.5 % longer, once
          // there too 32 trees 3 %)
          const float2 ks = reinterpret_cast<const float2*>(scales)[2 * kBlocks + q];
          const float2 lv = reinterpret_cast<const float2*>(scales)[2 * kBlocks + kBlocks / 2 + q];
          const float2 iv = reinterpret_cast<const float2*>(scales)[3 * kBlocks + q];
          const float e0 = c * ks.x, e1 = c * ks.y, n0 = nbase + lv.x, n1 = nbase + lv.y;
          const uint64_t c2[2] = {f2_pack(e0, e0), f2_pack(e1, e1)}, nb2[2] = {f2_pack(n0, n0), f2_pack(n1, n1)};
          uint32_t pk[16];
          uint64_t part[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const int u = k >> 3;
            float a0, a1;
            f2_unpack(f2_fma(f2_pack(x_[32 * q + 2 * k], x_[32 * q + 2 * k + 1]), c2[u], nb2[u]), a0, a1);
            const float p0 = ex2(a0), p1 = ex2(a1);
            part[u] = f2_add(part[u], f2_pack(p0, p1));
            pk[k] = pack_f16(p0, p1);
          }
          sum = f2_fma(part[0], f2_pack(iv.x, iv.x), f2_fma(part[1], f2_pack(iv.y, iv.y), sum));
          tmem_st16(tP + 16 * q, pk);
        };
        exponentials(0);
        exponentials(1);
        if (t * BN + BN / 2 < most) {
          exponentials(2);
          exponentials(3);
        } else {  // keys that no row of the warp sees
          const uint32_t zero[16] = {};
          tmem_st16(tP + 32, zero);
          tmem_st16(tP + 48, zero);
        }
        float s0, s1;
        f2_unpack(sum, s0, s1);
        l_run = l_run * alpha + (s0 + s1);
        if (t > first && __any_sync(0xffffffffu, need)) {
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            uint32_t o[32];
            tmem_ld32(tO + q * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
            tmem_st32(tO + q * 32, o);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(bar(Lay::B_PFULL + m));
      }
      if (!ok) break;
      // What the epilogue needs to know of the row, once it is done with the piece before.
      if (done > 0 && !await(bar(Lay::B_OFREE + m), (done - 1) & 1u, aborted)) break;
      row_inv[m * BM + row] = l_run > 0.f ? 1.f / l_run : 0.f;
      lse_of[m * BM + row] = row_lse(m_run - kLift, l_run);
      mbar_arrive(bar(Lay::B_STAT + m));
      ++done;
    }
  } else if (warp >= 12) {
    // ================================================================ V tiles, epilogue
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    const int row = tid & 127;  // row within an M tile = TMEM lane
    const uint32_t tO = tmem + ((uint32_t)((warp & 3) * 32) << 16) + kColO;
    const bool wide = (reinterpret_cast<uintptr_t>(A.out) & 31) == 0;
    uint32_t done0 = 0, done1 = 0, tiles0 = 0, tiles1 = 0, joins = 0, vt = 0;
    bool ok = true, have = false;
    Piece* kept = reinterpret_cast<Piece*>(smem + Lay::kept) + (warp & 3);  // (registers are short)
    // The epilogue's threads meet (an mbarrier, for a wait that ends when the CTA gives up).
    auto meet = [&]() -> bool {
      mbar_arrive(bar(Lay::B_JOIN));
      return ok = await(bar(Lay::B_JOIN), joins++ & 1u, aborted);
    };
    while (ok) {
      const bool more = pieces.next<Lay>(await, bar, smem, aborted, x);
      if (!more && !have) break;
      for (int t = more ? x.t0 : 0, t_end = more ? x.t1 : 1; ok && t < t_end; ++t) {
        if (more) {
          // ---- a V tile to fp16: 16 codes a load; keys behind the unit's last one count as zeros,
          // so that what lies there cannot reach O through 0 * NaN
          const uint32_t vs = vt % NV, ws = vt % NW;
          if (!await(bar(Lay::B_VFULL + vs), (vt / NV) & 1u, aborted) ||
              !await(bar(Lay::B_WEMPTY + ws), ((vt / NW) & 1u) ^ 1u, aborted)) {
            ok = false;
            break;
          }
          ++vt;
          // A lane's 16 dims of keys 16 j + key.  Eight lanes take 64 dims of each of two keys whose
          // numbers differ by 5: in the swizzled tiles their loads then lie on all banks (bit 2), and
          // so do their stores, every second unit of a key (bit 0).
          const int hf = (row >> 3) & 1, s4 = row & 3, key = ((row >> 4) * 2) ^ ((row >> 2) & 1 ? 5 : 0);
          const uint32_t src = sb + Lay::v + vs * kTile + key * D + (((hf * 4 + s4) ^ (key & 7)) << 4);
          uint4 w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = ld_shared_v4(src + j * (16 * D));
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(Lay::B_VEMPTY + vs));
          const int valid = x.keys - t * BN;
          if (valid < BN) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (16 * j + key >= valid) w[j] = make_uint4(0u, 0u, 0u, 0u);
          }
          const uint32_t dst = sb + Lay::w + ws * kTileW + hf * kVHalf + key * 128, u0 = (uint32_t)((2 * s4) ^ (key & 7)) << 4;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            uint32_t a[8];
            widen(w[j].x, a[0], a[1]);
            widen(w[j].y, a[2], a[3]);
            widen(w[j].z, a[4], a[5]);
            widen(w[j].w, a[6], a[7]);
            const uint32_t to = dst + j * kVChunk;
            st_shared_v4(to + u0, a[0], a[1], a[2], a[3]);
            st_shared_v4(to + (u0 ^ 16), a[4], a[5], a[6], a[7]);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(Lay::B_WFULL + ws));
        }
        if (!have) continue;
        // ---- the piece before: its rows
        have = false;
        const Piece prev = *kept;
        const int nt = prev.t1 - prev.t0;
        const bool whole = nt == prev.T, two = two_tiles(prev), both = !two && nt > 1;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (prev.t0 == 0);
        tiles0 += (uint32_t)(two ? nt : (nt + 1) / 2);
        tiles1 += (uint32_t)(two ? nt : nt / 2);
#pragma unroll 1
        for (int m = 0; m < (two ? 2 : 1); ++m) {
          // STAT first: the softmax has then seen all PV products but the last
          if (!await(bar(Lay::B_STAT + m), (m ? done1++ : done0++) & 1u, aborted) ||
              !await(bar(Lay::B_PVDONE + m), ((m ? tiles1 : tiles0) - 1) & 1u, aborted)) {
            ok = false;
            break;
          }
          float f0 = row_inv[m * BM + row], f1 = 0.f, lse = lse_of[m * BM + row];
          if (both) {
            if (!await(bar(Lay::B_STAT + 1), done1++ & 1u, aborted) ||
                !await(bar(Lay::B_PVDONE + 1), (tiles1 - 1) & 1u, aborted)) {
              ok = false;
              break;
            }
            const float l1 = lse_of[BM + row], top = fmaxf(lse, l1), w0 = ex2(lse - top), w1 = ex2(l1 - top);
            const float r = 1.f / (w0 + w1);
            f0 *= w0 * r;
            f1 = row_inv[BM + row] * w1 * r;
            lse = top + log2f(w0 + w1);
          }
          tc_fence_after();
          const int i = (MT * prev.rg + m) * npb + row / G;
          const bool vrow = row < npb * G && i < prev.n;
          uint16_t* orow = A.out + ((int64_t)(prev.r0 + i) * A.heads_q + prev.h * G + row % G) * D;
          float4* po = reinterpret_cast<float4*>(A.ws_o) + slot * (32 * 2 * BM) + m * BM + row;
          constexpr int kPlaces = CLUSTER ? BM : 2 * BM;  // rows of a float4 column
          if (CLUSTER) {  // (no product reads V any more)
            po = reinterpret_cast<float4*>(smem + Lay::w) + row;
            lse_of[row] = lse;
          } else if (!whole) {
            __stcg(A.ws_lse + slot * (2 * BM) + m * BM + row, lse);
          }
#pragma unroll 1
          for (int q = 0; q < 8; ++q) {  // 16 columns
            uint32_t o[16];
            tmem_ld16(tO + m * D + q * 16, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f0);
            if (both) {
              uint32_t o1[16];
              tmem_ld16(tO + D + q * 16, o1);
              tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 16; ++k)
                o[k] = __float_as_uint(fmaf(__uint_as_float(o1[k]), f1, __uint_as_float(o[k])));
            }
            if (!vrow) {
            } else if (whole && !CLUSTER) {
              uint32_t v[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) v[k] = pack_bf16(__uint_as_float(o[2 * k]), __uint_as_float(o[2 * k + 1]));
              st_global_32(orow + q * 16, v, wide);
            } else {
              // a part of a unit: normalised O to the workspace, float4 columns [32][256 rows]
#pragma unroll
              for (int k = 0; k < 4; ++k)
                po[(q * 4 + k) * kPlaces] = make_float4(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1]),
                                                         __uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3]));
            }
          }
          tc_fence_before();
          mbar_arrive(bar(Lay::B_OFREE + m));
          if (both) mbar_arrive(bar(Lay::B_OFREE + 1));
        }
        if (!ok || whole || CLUSTER) continue;
        // The CTA whose part arrives last joins the unit when its own pieces are done.
        __threadfence();
        if (!meet()) break;
        if (tid == 12 * 32 && !*abort_flag && arrive_at(A.cnt + prev.o0, A.tag) == prev.parts) {
          A.cnt[prev.o0] = 0;  // a completed unit leaves a zero word behind
          *reinterpret_cast<Piece*>(smem + Lay::pieces + (kPieces + *n_joins) * (kPieceInts * 4)) = prev;
          *n_joins = *n_joins + 1;
        }
      }
      if (!more) break;
      __syncwarp();
      if (lane == 0) *kept = x;
      __syncwarp();
      have = true;
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 8) {
      // ================================================================ producer
      const int ps = A.kv.page_size;
      const bool paged = A.kv.layout == 1;
      const int ppt = paged ? BN / ps : 0;  // pages (boxes) of a tile: 2 .. 8
      uint32_t kt = 0, vt = 0, quads = 0;   // tiles issued, quads whose scales are out
      uint32_t q0 = 0, q1 = 0;              // pieces whose M tile of Q is issued
      while (pieces.next<Lay>(await, bar, smem, aborted, x)) {
        // Pages and scales are looked up a quad of tiles at a time, two quads and one ahead of their
        // use (one tile ahead, a tile took as long as a load).  Lane 8 i + p: page p of the quad's tile
        // i (a missing one reads zeros), and the scales of its block p.
        auto pages_of = [&](int q) -> int {
          const int t = x.t0 + q * kQuad + (lane >> 3), p = lane & 7, tok = t * BN + p * ps;
          if (p >= ppt || t >= x.t1 || tok >= x.keys) return -1;
          const int page = A.kv.block_table[(int64_t)x.b * A.kv.max_len + tok / ps];
          if (page < 0 || page >= A.kv.num_pages) {
            flag(A.err, CURE_DEVERR_PAGE);
            return -1;
          }
          return page;
        };
        auto scales_of = [&](int q, int pages) -> float2 {
          const int t = x.t0 + q * kQuad + (lane >> 3), blk = lane & 7;
          int64_t place;
          if (paged) {
            const int page = __shfl_sync(0xffffffffu, pages, (lane & 24) | (blk * kBlk / ps));
            place = page < 0 ? -1 : (int64_t)page * (ps / kBlk) + blk * kBlk % ps / kBlk;
          } else {
            place = (int64_t)x.b * ((A.kv.max_len + kBlk - 1) / kBlk) + t * kBlocks + blk;
          }
          if (t >= x.t1 || t * BN + blk * kBlk >= x.keys || place < 0) return make_float2(1.f, 1.f);
          return make_float2(__ldg(A.k_scale + place * A.kv.heads_kv + x.h), __ldg(A.v_scale + place * A.kv.heads_kv + x.h));
        };
        const int nt = x.t1 - x.t0;
        // of this quad and the next one
        int pages0 = pages_of(0), pages1 = pages_of(1);
        float2 scales0 = scales_of(0, pages0), scales1;
        bool is_v = false, unsaid = false;  // what comes next; whether the quad's scales are still to be put into shared memory
        auto say = [&]() {
          float2* to = reinterpret_cast<float2*>(smem + Lay::scales) +
                       (quads % kScaleSlots * kQuad + (lane >> 3)) * (kScaleFloats / 2) + (lane & 7);
          const float ks = fminf(fmaxf(scales0.x, 0x1p-40f), 0x1p40f), vs = fminf(fmaxf(scales0.y, 0x1p-40f), 0x1p40f);
          const float lv = log2f(vs), rv = 1.f / vs;
          to[0] = make_float2(ks, ks);
          to[kBlocks] = make_float2(lv, lv);
          float* once = reinterpret_cast<float*>(to - (lane & 7) + 2 * kBlocks) + (lane & 7);
          once[0] = ks;
          once[kBlocks] = lv;
          once[2 * kBlocks] = rv;
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(Lay::B_SCALES + quads % kScaleSlots));
          ++quads;
          unsaid = false;
        };
        // Q of the piece, an M tile once the S products of the one before in its place are done
        auto ask = [&]() -> bool {
          for (int m = 0; m < (two_tiles(x) ? 2 : 1); ++m) {
            if (!await(bar(Lay::B_QEMPTY + m), ((m ? q1 : q0) & 1u) ^ 1u, aborted)) return false;
            if (m) ++q1;
            else ++q0;
            if (lane == 0) mbar_arrive_expect_tx(bar(Lay::B_QRAW + m), (uint32_t)(2 * npb * G * 128));
            __syncwarp();
            if (lane < 2)
              tma_load_4d(sb + Lay::q + (2 * m + lane) * kQHalf, &tm_q, bar(Lay::B_QRAW + m), lane * 64, 0, x.h,
                          x.r0 + (MT * x.rg + m) * npb);
            __syncwarp();
          }
          return true;
        };
        if (!ask()) goto produced;
        // K and V tiles in turn (with a second K tile in front of the first V tile 25 nodes behind 4096 tokens
        // take 15.7, not 15.1 us)
        for (int t = 0; t < nt;) {
          if (is_v && unsaid && t > 0) say();
          if (!await(is_v ? bar(Lay::B_VEMPTY + vt % NV) : bar(Lay::B_KEMPTY + kt % NK),
                     ((is_v ? vt / NV : kt / NK) & 1u) ^ 1u, aborted))
            goto produced;
          if (!is_v && t % kQuad == 0) {
            if (t > 0) {
              pages0 = pages1;
              scales0 = scales1;
              pages1 = pages_of(t / kQuad + 1);
            }
            scales1 = scales_of(t / kQuad + 1, pages1);
            unsaid = true;
          }
          const int page = __shfl_sync(0xffffffffu, pages0, t % kQuad * 8 | (lane & 7));
          const uint32_t st = is_v ? vt++ % NV : kt++ % NK;
          const uint32_t full = bar((is_v ? Lay::B_VFULL : Lay::B_KFULL) + st);
          const uint32_t dst = sb + (is_v ? Lay::v : Lay::k) + st * kTile;
          if (lane == 0) mbar_arrive_expect_tx(full, kTile);
          __syncwarp();
          const CUtensorMap* map = is_v ? &tm_v : &tm_k;
          if (paged) {
            if (lane < ppt) tma_load_4d(dst + lane * ps * D, map, full, 0, x.h, 0, page);
          } else if (lane == 0) {
            tma_load_4d(dst, map, full, 0, x.h, (x.t0 + t) * BN, x.b);
          }
          __syncwarp();
          t += is_v;
          is_v = !is_v;
        }
        if (unsaid) say();
      }
    produced:
      if (*abort_flag) {  // let copies in flight land before the CTA's smem goes away
        for (uint32_t i = (kt > NK ? kt - NK : 0); i < kt; ++i)
          wait_bounded(bar(Lay::B_KFULL + i % NK), (i / NK) & 1u, abort_flag, A.err, false);
        for (uint32_t i = (vt > NV ? vt - NV : 0); i < vt; ++i)
          wait_bounded(bar(Lay::B_VFULL + i % NV), (i / NV) & 1u, abort_flag, A.err, false);
        if (q0 > 0) wait_bounded(bar(Lay::B_QRAW), (q0 - 1) & 1u, abort_flag, A.err, false);
        if (q1 > 0) wait_bounded(bar(Lay::B_QRAW + 1), (q1 - 1) & 1u, abort_flag, A.err, false);
      }
    } else if (warp == 9) {
      // ================================================================ S products
      constexpr uint32_t idS = idesc_0(BM, BN, false);
      uint32_t q0 = 0, q1 = 0, c = 0, kt = 0, quads = 0;  // pieces of each M tile, products, K tiles, quads of scales
      const uint64_t qd = sdesc_sw128(sb + Lay::q, 16, 1024), kd = sdesc_sw128(sb + Lay::k, 16, 1024);
      while (pieces.next<Lay>(await, bar, smem, aborted, x)) {
        const bool two = two_tiles(x);
        for (int t = x.t0; t < x.t1; ++t, ++kt) {
          const uint32_t st = kt % NK;
          if (!await(bar(Lay::B_KFULL + st), (kt / NK) & 1u, aborted)) goto scored;
          if ((t - x.t0) % kQuad == 0) {  // the softmax reads them once it has S
            if (!await(bar(Lay::B_SCALES + quads % kScaleSlots), (quads / kScaleSlots) & 1u, aborted)) goto scored;
            ++quads;
          }
#pragma unroll 1
          for (int m = 0; m < (two ? 2 : 1); ++m) {
            // (the first product waits for the phase before the first, which counts as done)
            if (!await(bar(Lay::B_SFREE), (c++ & 1u) ^ 1u, aborted)) goto scored;
            if (t == x.t0 && !await(bar(Lay::B_QFULL + m), (m ? q1++ : q0++) & 1u, aborted)) goto scored;
            tc_fence_after();
            issue_s(tmem + kColS, (uint32_t)qd + m * (2 * kQHalf >> 4), (uint32_t)(qd >> 32),
                    (uint32_t)kd + st * (kTile >> 4), (uint32_t)(kd >> 32), idS,
                    bar(Lay::B_SFULL + (two ? m : (t - x.t0) & 1)));
            if (t == x.t1 - 1) commit_elect(bar(Lay::B_QEMPTY + m));  // the piece's last use of the M tile of Q
          }
          commit_elect(bar(Lay::B_KEMPTY + st));
        }
      }
    scored:
      __syncwarp();
      commit_elect(bar(Lay::B_DRAIN));
      wait_bounded(bar(Lay::B_DRAIN), 0, abort_flag, A.err, false);
    } else if (warp == 10) {
      // ================================================================ PV products
      constexpr uint32_t idO = idesc_0(BM, D, true);
      uint32_t c0 = 0, c1 = 0, done0 = 0, done1 = 0, vt = 0;  // products and pieces of each group, V tiles
      // V as an MN-major operand: the d halves LBO apart, 8-key groups SBO apart
      const uint64_t vd = sdesc_sw128(sb + Lay::w, kVHalf, 1024);
      while (pieces.next<Lay>(await, bar, smem, aborted, x)) {
        const bool two = two_tiles(x);
        for (int t = x.t0; t < x.t1; ++t, ++vt) {
          const uint32_t st = vt % NW;
          if (!await(bar(Lay::B_WFULL + st), (vt / NW) & 1u, aborted)) goto multiplied;
          const int turn = two ? 0 : (t - x.t0) & 1;
#pragma unroll 1
          for (int m = turn; m < (two ? 2 : turn + 1); ++m) {
            // a group's first product of a piece takes O over from the epilogue of the one before
            // (from none at first: the phase before the first counts as done)
            const bool fresh = t - x.t0 == turn;
            if (fresh && !await(bar(Lay::B_OFREE + m), ((m ? done1++ : done0++) & 1u) ^ 1u, aborted)) goto multiplied;
            if (!await(bar(Lay::B_PFULL + m), (m ? c1++ : c0++) & 1u, aborted)) goto multiplied;
            tc_fence_after();
            issue_pv(tmem + kColO + m * D, tmem + kColP + m * 64, (uint32_t)vd + st * (kTileW >> 4),
                     (uint32_t)(vd >> 32), idO, !fresh, bar(Lay::B_PVDONE + m));
          }
          commit_elect(bar(Lay::B_WEMPTY + st));
        }
      }
    multiplied:
      __syncwarp();
      commit_elect(bar(Lay::B_DRAIN + 1));
      wait_bounded(bar(Lay::B_DRAIN + 1), 0, abort_flag, A.err, false);
    } else {
      // ================================================================ scheduler
      if constexpr (CLUSTER) {
        // the one piece of this CTA, if the unit has so many tiles
        const int rank = (int)blockIdx.x % A.cluster, u = (int)blockIdx.x / A.cluster, Hkv = A.kv.heads_kv;
        const int groups = (A.n_max + npb - 1) / npb;
        int bad;
        x = Piece{};
        x.b = u / (Hkv * groups);
        x.h = u % Hkv;
        x.rg = u / Hkv % groups;
        const Seq q = sequence(A, x.b, &bad);
        if (bad && rank == 0 && x.h == 0 && x.rg == 0) flag(A.err, bad);
        x.r0 = q.r0;
        x.n = q.n;
        x.L = q.L;
        x.keys = q.L + q.n;
        x.T = (x.keys + BN - 1) / BN;
        x.t0 = x.T * rank / A.cluster;
        x.t1 = x.T * (rank + 1) / A.cluster;
        if (x.rg * npb >= q.n) x.t1 = x.t0 = 0;  // no rows
        if (lane == 0) {
          Piece* to = reinterpret_cast<Piece*>(smem + Lay::pieces);
          to[0] = x;
          mbar_arrive(bar(Lay::piece_bar));
          if (x.t0 < x.t1) {
            to[1] = Piece{};
            mbar_arrive(bar(Lay::piece_bar + 1));
          }
        }
        __syncwarp();
      } else {
        schedule<Lay>(A, npb, await, bar, smem, aborted, lane);
      }
    }
  }

  // ---- the units that this CTA joins, by all warps and with equal registers again
  // (behind the barrier: a warp that had nothing to do must not take back the registers
  // that a softmax warp still waits for)
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp < 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 128;");
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 128;");
  if (*abort_flag && tid == 0) flag(A.err, CURE_DEVERR_TIMEOUT);
  if constexpr (CLUSTER) {
    // Each CTA of the cluster joins some of the unit's rows, a float4 a thread:
    //   O = sum_p 2^(lse_p) O_p / sum_p 2^(lse_p) over the parts that saw a key
    const Piece& p = *reinterpret_cast<const Piece*>(smem + Lay::pieces);
    // this CTA has given up (the unit's rows are then left unwritten), or its part has no keys
    const float none = *abort_flag ? __uint_as_float(kGaveUp) : -FLT_MAX;
    if (p.t0 >= p.t1 || *abort_flag)
      for (int i = tid; i < BM; i += kThreads) lse_of[i] = none;
    cluster_sync();
    const int rank = (int)blockIdx.x % A.cluster;
    const int rows = min(npb, p.n - p.rg * npb) * G, each = (max(rows, 0) + A.cluster - 1) / A.cluster;
    const int first = rank * each, mine = min(each, rows - first);
    for (int i = tid; i < mine * 32; i += kThreads) {
      const int r = first + i % mine, c = i / mine;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float top = -FLT_MAX, total = 0.f;
      bool gave_up = false;
      const uint32_t l_at = sb + Lay::lse + r * 4, o_at = sb + Lay::w + (c * BM + r) * 16;
      for (int q0 = 0; q0 < A.cluster; q0 += 4) {
        float w[4], best = top;
        float4 o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int from = min(q0 + q, A.cluster - 1);
          w[q] = ld_cluster(map_rank(l_at, from));
          o[q] = ld_cluster_v4(map_rank(o_at, from));
          if (q0 + q >= A.cluster) w[q] = -FLT_MAX;
          gave_up |= __float_as_uint(w[q]) == kGaveUp;
          best = fmaxf(best, w[q]);
        }
        const float a = ex2(top - best);
        top = best;
        total *= a;
        acc = make_float4(acc.x * a, acc.y * a, acc.z * a, acc.w * a);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (w[q] == -FLT_MAX) continue;  // (what stands there may be anything)
          const float wq = ex2(w[q] - top);
          total += wq;
          acc = make_float4(fmaf(wq, o[q].x, acc.x), fmaf(wq, o[q].y, acc.y), fmaf(wq, o[q].z, acc.z),
                            fmaf(wq, o[q].w, acc.w));
        }
      }
      if (gave_up) continue;
      const float inv = total > 0.f ? 1.f / total : 0.f;
      uint16_t* orow = A.out + ((int64_t)(p.r0 + p.rg * npb + r / G) * A.heads_q + p.h * G + r % G) * D;
      *reinterpret_cast<uint2*>(orow + 4 * c) =
          make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    }
    cluster_sync();  // the peers have read this CTA's shared memory
  } else if (!*abort_flag) {
    join_units<Lay>(A, npb, smem, *n_joins, warp, lane);
  }
  __syncwarp();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Dynamic shared memory (and clusters above the portable size), once per device.
template <class Args, bool CLUSTER, bool EXPIRE = false>
cudaError_t set_up() {
  static std::atomic<uint64_t> ready;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (ready.load() & bit) return cudaSuccess;
  const auto kernel = attn8_kernel<Args, CLUSTER, EXPIRE>;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<CLUSTER ? 1 : 2>::bytes);
  if (e == cudaSuccess && CLUSTER) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) ready.fetch_or(bit);
  return e;
}

// Clusters of `size` CTAs that the device holds at once (a cluster lies within one GPC, so fewer than
// SMs / size).
int max_clusters(int size) {
  static std::atomic<int> known[64][kAttnMaxCluster + 1];  // 1 + the count; 0: not asked yet
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64 || set_up<Tree8, true>() != cudaSuccess) return 0;
  int n = known[dev][size].load();
  if (n == 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(size);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Layout<1>::bytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, attn8_kernel<Tree8, true, false>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    known[dev][size].store(++n);
  }
  return n - 1;
}

// CTAs of each unit's cluster for `units` units of one M tile; 0: units cut among all CTAs instead (the
// faster form where a cluster would have two).  us cut and in clusters, trees of 17 to 33 nodes behind 1024 to 8192
// tokens, 28/4 heads: 8 of them 45.6 and, in clusters of 2, 47.6; 6 41.6 and 51.6; 5 42.3 and, of 3, 39.3; 4 45.2 and,
// of 4, 31.2; 2 43.7 and 24.1.  One of 25 nodes behind 4096, 32/8 heads: 26.5 and 14.7.
int cluster_size(int64_t units) {
  for (int c = kAttnMaxCluster; c >= 3; --c)
    if (units <= max_clusters(c)) return c;
  return 0;
}

template <bool CLUSTER, bool EXPIRE, class Args>
cudaError_t launch(const Attn8Call& c, Args& A, int grid, cudaStream_t s) {
  const cudaError_t e = set_up<Args, CLUSTER, EXPIRE>();
  if (e != cudaSuccess) return e;
  CUtensorMap mk, mv, mq;
  const int box = c.kv.layout == 1 ? c.kv.page_size : BN;
  if (!make_codes_map(&mk, c.k_cache, c.kv, c.batch, box) || !make_codes_map(&mv, c.v_cache, c.kv, c.batch, box) ||
      !make_q_map(&mq, c.q, (uint64_t)c.rows, c.kv.heads_kv, c.heads_q / c.kv.heads_kv, BM * c.kv.heads_kv / c.heads_q))
    return cudaErrorInvalidValue;
  fill_args8(c, &A);
  A.k_scale = c.k_scale;
  A.v_scale = c.v_scale;
  A.n_nodes = c.n_nodes;
  A.anc = c.anc;
  A.n_max = c.n_max;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(Layout<CLUSTER ? 1 : 2>::threads);
  cfg.dynamicSmemBytes = Layout<CLUSTER ? 1 : 2>::bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  if (CLUSTER) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = A.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.numAttrs = 1;
  }
  // many units: after the whole of the call before (as in k_prompt.cu)
  if ((int64_t)c.rows * c.heads_q <= (int64_t)4 * 2 * BM * num_sms()) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  return cudaLaunchKernelEx(&cfg, attn8_kernel<Args, CLUSTER, EXPIRE>, mk, mv, mq, A);
}
template <bool CLUSTER, class Args>
cudaError_t launch(const Attn8Call& c, Args& A, int grid, cudaStream_t s) {
  return c.expire_wait > 0 ? launch<CLUSTER, true>(c, A, grid, s) : launch<CLUSTER, false>(c, A, grid, s);
}

}  // namespace

size_t attn8_workspace() {
  const int ctas = num_sms();
  return counter_bytes8(ctas) + (size_t)ctas * 2 * 2 * BM * (D + 1) * sizeof(float);
}

cudaError_t launch_attn8(const Attn8Call& c, cudaStream_t s) {
  if (tokens8_fits(c)) return launch_tokens8(c, s);
  const int sms = num_sms();
  if (c.n_nodes) {
    Tree8 A = {};
    // few units: a cluster of CTAs each
    const int npb = BM / (c.heads_q / c.kv.heads_kv);
    const int64_t units = (int64_t)c.batch * c.kv.heads_kv * ((c.n_max + npb - 1) / npb);
    A.cluster = units * 2 <= sms ? cluster_size(units) : 0;
    return A.cluster > 0 ? launch<true>(c, A, (int)units * A.cluster, s) : launch<false>(c, A, sms, s);
  }
  Args8 A = {};
  return launch<false>(c, A, sms, s);
}

}  // namespace cure
