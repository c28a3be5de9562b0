// Causal grouped-head attention of packed prompt rows over the cache (the input
// of Alg. 1: the target reads the prompt before the first step), on tcgen05
// tensor cores.
//
//   out_i = sum_{j <= L + i} softmax_j(scale q_i k_j) v_j     (row i of a sequence
//                                                             with L tokens before)
//
// Work.  A unit is (sequence, row group, kv head): 2 * npb rows' heads of one kv
// head, packed (row, group head) into two M tiles of 128 (npb = 128 / G rows
// each), against its keys 0 .. L + last row in 128-key tiles.  Two M tiles share
// each K and V tile from shared memory, and one runs its softmax while the
// other's products run.
//
// Roles (16 warps):
//   warps 0-3 / 4-7   softmax of M tile 0 / 1, a thread a row: reads S from TMEM,
//                     writes P (bf16) to TMEM, keeps the row's running maximum
//                     and sum, rescales O (only where the maximum has grown by
//                     more than 2^8)
//   warp 8            TMA producer: Q, and K and V tiles in turn through a ring
//                     of 5 stages of 32 KiB
//   warp 9            issues S = Q K^T (M128 N128 K128) of M tiles 0 and 1 in turn
//   warp 10           issues O += P V (A = P from TMEM) once P is published
//   warp 11           lays out the CTA's pieces of work, a few ahead
//   warps 12-15       epilogue: write O while the softmax warps are in the next piece
// TMEM (512 columns): S (128) | P[2] (64 each) | O[2] (128 each).  There is one S
// for both M tiles: a softmax frees it as soon as it has loaded its row (128
// registers), long before its exponentials are done, and the other M tile's
// product takes it.  That keeps the two M tiles half a tile apart, one in its
// softmax while the tensor cores work for the other, and no product waits for
// the PV product of its own M tile.  (With an S for each M tile and P over it, S
// had to wait for PV to finish; both M tiles then ran in step, 1870 cycles of
// softmax and 1940 of products a tile, one after the other.)
//
// Bound and measured (us back to back; part of the measured 1929 TFLOP/s or 6.78 TB/s).
// Many keys: the products, M128 N128 at one S at a time, with the softmax of the other
// M tile under them.  One prompt of 16384, 64/8 heads: 2530, 1738 TFLOP/s, 0.90 (2700 in
// runs of a second under the power cap: 0.94 of what a library product keeps up then).
// Shorter units add what starting and ending one costs, 1 to 2 tiles of time: chunks of
// 8 prompts behind 1024 to 16000 tokens, 28/4 heads, 260, 0.74 (279 in long runs); 32
// prompts of 33 to 4096 305, 0.71 (329).  Single tokens: the cache's bytes, 64 sequences of 500 to 16000 tokens 183,
// 6.0 TB/s, 0.88.  One prompt of 200: 11.4, latency.
//
// Code.  All roles run at once, and what they run between them is about what the
// instruction cache holds: 169 KB of code, most of it the scheduler's copies of its
// parts and the waits, made short units a seventh slower (200 prompts of 20 to 150: 73,
// and 64 with 100 KB, 61 with 95).  Hence one copy of everything, waits of ten instructions, and
// nothing unrolled that need not be.  (Q of each M tile on barriers of its own, and O
// packed into registers before it is stored: no faster, and a third slower on short
// units, for that reason.)
#include "prompt_units.cuh"

namespace cure {
namespace {

using namespace prompt;

constexpr int NS = 5;                   // ring stages, a K or a V tile each
constexpr int kKHalf = BN * 64 * 2;     // 16 KiB: [128 keys][64 d]
constexpr int kTile = 2 * kKHalf;       // 32 KiB
// from a paged cache: [8-key group][d half][8 keys][64 d], as in the tree attention
constexpr int kPgGroup = 8 * D * 2;
constexpr int kPgHalf = kPgGroup / 2;
constexpr int kOffQ = 0;                       // Q[m][half]
constexpr int kOffRing = kOffQ + 4 * kQHalf;   // K/V[stage]
constexpr int kOffMisc = kOffRing + NS * kTile;
enum {
  B_QFULL = 0, B_QEMPTY = 1, B_SFREE = 2, B_FULL = 3, B_EMPTY = B_FULL + NS, B_SFULL = B_EMPTY + NS,
  B_PFULL = B_SFULL + 2, B_PVDONE = B_PFULL + 2, B_STAT = B_PVDONE + 2, B_OFREE = B_STAT + 2, B_DRAIN = B_OFREE + 2,
  B_JOIN = B_DRAIN + 2, B_PIECE = B_JOIN + 1, B_TAKEN = B_PIECE + kPieces, B_NEVER = B_TAKEN + kPieces,
  kNumBars = B_NEVER + 1
};
constexpr int kOffTmemSlot = kOffMisc + 8 * kNumBars;
constexpr int kOffAbort = kOffTmemSlot + 4;
constexpr int kOffJoins = kOffAbort + 4;                              // units that this CTA joins at its end
constexpr int kOffPieces = (kOffJoins + 4 + 15) / 16 * 16;            // int [kPieces][kPieceInts], then [2] to join
constexpr int kOffPrefix = kOffPieces + (kPieces + 2) * kPieceInts * 4;  // int64 first position of each sequence [B+1]
constexpr int kSmemBytes = kOffPrefix + 8 * (kAttnMaxBatch + 1);
static_assert(kSmemBytes <= 232448, "fits the 227 KiB opt-in");
struct Lay {  // where the pieces lie, for what prompt_units.cuh shares
  static constexpr int m_tiles = 2, threads = kThreads, pieces = kOffPieces, prefix = kOffPrefix, piece_bar = B_PIECE, taken_bar = B_TAKEN;
};

// The products of a tile and one M tile, issued by a lane that is elected once for them
// and the commit behind them, on descriptors in halves, so that a step is one addition.
// (Groups of steps on 64-bit descriptors and a commit with its own election: 2 % more
// time, 6 % on a prompt of 16384.  The ring stage's and Q's commits in here as well,
// under conditions: 2 % more.)
//
// S = Q_m K^T: 8 steps of 16 dims, the second 64 dims kQHalf and (K: k2) further on.
__device__ __forceinline__ void issue_s(uint32_t d, uint32_t q, uint32_t q_hi, uint32_t k, uint32_t k_hi, uint32_t k2,
                                        uint32_t idesc, uint32_t full) {
  static_assert(kQHalf >> 4 == 1024, "as the steps are written");
  asm volatile(
      "{\n\t.reg .pred pf, pt, el;\n\t.reg .b64 a, b;\n\t.reg .b32 x, y;\n\t"
      "elect.sync _|el, 0xffffffff;\n\t"
      "setp.ne.b32 pf, 0, 0;\n\t"
      "setp.eq.b32 pt, 0, 0;\n\t"
      "mov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %6, pf;\n\t"
      "add.u32 x, %1, 2;\n\tadd.u32 y, %3, 2;\n\tmov.b64 a, {x, %2};\n\tmov.b64 b, {y, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %6, pt;\n\t"
      "add.u32 x, %1, 4;\n\tadd.u32 y, %3, 4;\n\tmov.b64 a, {x, %2};\n\tmov.b64 b, {y, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %6, pt;\n\t"
      "add.u32 x, %1, 6;\n\tadd.u32 y, %3, 6;\n\tmov.b64 a, {x, %2};\n\tmov.b64 b, {y, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %6, pt;\n\t"
      "add.u32 x, %1, 1024;\n\tmov.b64 a, {x, %2};\n\tmov.b64 b, {%5, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %6, pt;\n\t"
      "add.u32 x, %1, 1026;\n\tadd.u32 y, %5, 2;\n\tmov.b64 a, {x, %2};\n\tmov.b64 b, {y, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %6, pt;\n\t"
      "add.u32 x, %1, 1028;\n\tadd.u32 y, %5, 4;\n\tmov.b64 a, {x, %2};\n\tmov.b64 b, {y, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %6, pt;\n\t"
      "add.u32 x, %1, 1030;\n\tadd.u32 y, %5, 6;\n\tmov.b64 a, {x, %2};\n\tmov.b64 b, {y, %4};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %6, pt;\n\t"
      "@el tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%7];\n\t}\n" ::"r"(d),
      "r"(q), "r"(q_hi), "r"(k), "r"(k_hi), "r"(k2),
      "r"(idesc), "r"(full)
      : "memory");
}


template <bool EXPIRE>
__global__ void __launch_bounds__(kThreads, 1)
prompt_attn_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const __grid_constant__ CUtensorMap tm_q, const PromptArgs A) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sb = smem_u32(smem);
  if (sb & 1023u) {  // the swizzled tiles need a 1 KiB-aligned base
    if (tid == 0) flag(A.err, CURE_DEVERR_ALIGN);
    return;
  }
  const int G = A.G, npb = BM / G;
  const Bar bar{sb + kOffMisc};
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffAbort);
  const uint32_t aborted = sb + kOffAbort;
  volatile int* n_joins = reinterpret_cast<volatile int*>(smem + kOffJoins);

  // ---------------------------------------------------------------- set-up
  if (tid == 0) {
    mbar_init(bar(B_QFULL), 1);
    mbar_init(bar(B_QEMPTY), 1);
    mbar_init(bar(B_SFREE), BM);
    for (int i = 0; i < NS; ++i) {
      mbar_init(bar(B_FULL + i), 1);
      mbar_init(bar(B_EMPTY + i), 1);
    }
    for (int m = 0; m < 2; ++m) {
      mbar_init(bar(B_SFULL + m), 1);
      mbar_init(bar(B_PFULL + m), BM);
      mbar_init(bar(B_PVDONE + m), 1);
      mbar_init(bar(B_STAT + m), BM);
      mbar_init(bar(B_OFREE + m), BM);
      mbar_init(bar(B_DRAIN + m), 1);
    }
    mbar_init(bar(B_JOIN), BM);
    for (int i = 0; i < kPieces; ++i) {
      mbar_init(bar(B_PIECE + i), 1);
      mbar_init(bar(B_TAKEN + i), kTakers);
    }
    if constexpr (EXPIRE) mbar_init(bar(B_NEVER), 1);
    *abort_flag = 0;
    *n_joins = 0;
    fence_mbar_init();
  }
  if (warp == 0) tmem_alloc(sb + kOffTmemSlot, kTmemCols);
  if (warp == 8 && lane == 0) {
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  // Q rows at or past npb * G are never written by the Q copies: zero them once
  const int pad_rows = BM - npb * G;
  for (int c = tid; c < 4 * pad_rows * 8; c += kThreads) {
    const int q16 = c & 7, rr = npb * G + ((c >> 3) % pad_rows), mh = (c >> 3) / pad_rows;
    st_shared_v4(sb + kOffQ + mh * kQHalf + rr * 128 + q16 * 16, 0u, 0u, 0u, 0u);
  }
  pdl_begin();
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + kOffTmemSlot);
  Await<EXPIRE> await;
  if constexpr (EXPIRE) {
    await.never = bar(B_NEVER);
    await.left = blockIdx.x == 0 && warp == A.expire_warp ? (uint32_t)A.expire_wait : 0u;
  }
  Pieces pieces{0};
  Piece x;
  // M tile 1 of a piece is active when its first row is one of the sequence's
  auto active1 = [&](const Piece& x) { return (2 * x.rg + 1) * npb < x.n; };

  // The softmax warps hold a row of S each: they get registers from the other
  // warpgroups (128 * (2 * 160 + 96 + 96) = 512 * 128, what the block was launched with).
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    // ================================================================ softmax
    const int m = warp >> 2;
    const int row = tid & 127;  // row within the M tile = TMEM lane
    const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t tS = tl + kColS, tP = tl + kColP + m * 64, tO = tl + kColO + m * D;
    const float c = A.scale_log2;
    uint32_t sc = 0, r = 0;  // tiles of this M tile, ring tiles
    bool ok = true;
    uint32_t done = 0;  // pieces of this M tile
    while (ok && pieces.next<Lay>(await, bar, smem, aborted, x)) {
      const uint32_t r_piece = r;
      r += 2 * (uint32_t)(x.t1 - x.t0);
      if (m == 1 && !active1(x)) continue;
      const int i = (2 * x.rg + m) * npb + row / G;  // the row's place in its sequence
      const int sees = x.L + i + 1;                  // keys that it sees
      // the fewest and the most that a row of this warp sees
      const int least = __shfl_sync(0xffffffffu, sees, 0), most = __shfl_sync(0xffffffffu, sees, 31);
      float m_run = -INFINITY, l_run = 0.f;
      for (int t = x.t0; t < x.t1; ++t) {
        if (!await(bar(B_SFULL + m), sc & 1u, aborted)) { ok = false; break; }
        ++sc;
        tc_fence_after();
        uint32_t v[4][32];
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(tS + 32 * q, v[q]);
        tmem_wait_ld();
        tc_fence_before();
        mbar_arrive(bar(B_SFREE));  // the next product may take S
        float x_[BN];
#pragma unroll
        for (int k = 0; k < BN; ++k) x_[k] = __uint_as_float(v[k >> 5][k & 31]);
        if ((t + 1) * BN > least) {
          const int lim = sees - t * BN;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (t * BN + 32 * (q + 1) > least) {
              const int left = min(max(lim - 32 * q, 0), 32);  // keys of the block that the row sees
              const uint32_t seen = left == 32 ? 0xffffffffu : (1u << left) - 1u;
#pragma unroll
              for (int k = 0; k < 32; ++k) x_[32 * q + k] = (seen >> k) & 1u ? x_[32 * q + k] : -INFINITY;
            }
          }
        }
        float mx[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) mx[k] = fmaxf(x_[k], x_[8 + k]);
#pragma unroll
        for (int j = 16; j < BN; j += 16)
#pragma unroll
          for (int k = 0; k < 8; ++k) mx[k] = fmax3(mx[k], x_[j + k], x_[j + 8 + k]);
        const float mt = fmax3(fmax3(mx[0], mx[1], mx[2]), fmax3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * c;
        const float m_new = fmaxf(m_run, mt);
        const bool need = m_new > m_run + 8.0f;
        const float alpha = need ? ex2(m_run - m_new) : 1.f;
        if (need) m_run = m_new;
        // P's place and O are free once this M tile's PV product before is done
        if (sc > 1) {
          if (!await(bar(B_PVDONE + m), (sc - 2) & 1u, aborted)) { ok = false; break; }
          tc_fence_after();
        }
        const float nbase = m_run == -INFINITY ? 0.f : -m_run;
        const uint64_t c2 = f2_pack(c, c), nb2 = f2_pack(nbase, nbase);
        uint64_t sm2[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
        auto exponentials = [&](int q) {  // of 32 keys
          uint32_t pk[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float a0, a1;
            f2_unpack(f2_fma(f2_pack(x_[32 * q + 2 * k], x_[32 * q + 2 * k + 1]), c2, nb2), a0, a1);
            const float p0 = ex2(a0), p1 = ex2(a1);
            sm2[k & 1] = f2_add(sm2[k & 1], f2_pack(p0, p1));
            pk[k] = pack_bf16(p0, p1);
          }
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
        float s4[4];
        f2_unpack(sm2[0], s4[0], s4[1]);
        f2_unpack(sm2[1], s4[2], s4[3]);
        l_run = l_run * alpha + ((s4[0] + s4[1]) + (s4[2] + s4[3]));
        if (t > x.t0 && __any_sync(0xffffffffu, need)) {
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
        // V rows past the unit's last key are zeroed so that what lies there cannot reach
        // O through 0 * NaN: by M tile 0, whose PV product of a tile is issued first; up to
        // the end of the last page or 16-row copy, behind which zeros were read
        const int valid = x.keys - t * BN;
        if (m == 0 && valid < BN) {
          const uint32_t rv = r_piece + 2 * (uint32_t)(t - x.t0) + 1;
          if (!await(bar(B_FULL + rv % NS), (rv / NS) & 1u, aborted)) { ok = false; break; }
          const uint32_t vb = sb + kOffRing + (rv % NS) * kTile;
          const bool paged = A.kv.layout == 1;
          const int unit = paged ? A.kv.page_size : 16;
          for (int q = row; q < (unit - 1 - (valid - 1) % unit) * 16; q += BM) {
            const int rr = valid + (q >> 4), hf = (q >> 3) & 1, cc = q & 7;
            const uint32_t off = paged ? (rr >> 3) * kPgGroup + hf * kPgHalf + (rr & 7) * 128
                                       : (rr >> 4) * kVChunk + hf * kVHalf + (rr & 15) * 128;
            st_shared_v4(vb + off + cc * 16, 0u, 0u, 0u, 0u);
          }
          fence_proxy_async_smem();
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(bar(B_PFULL + m));
      }
      if (!ok) break;
      // What the epilogue needs to know of the row, once it is done with the piece before
      // (so that it also sees every phase of STAT).
      if (done > 0 && !await(bar(B_OFREE + m), (done - 1) & 1u, aborted)) break;
      __stcg(A.ws_inv + ((int64_t)blockIdx.x * 2 + m) * BM + row, l_run > 0.f ? 1.f / l_run : 0.f);
      if (x.t1 - x.t0 < x.T)
        __stcg(A.ws_lse + (2 * (int64_t)blockIdx.x + (x.t0 == 0)) * (2 * BM) + m * BM + row, row_lse(m_run, l_run));
      mbar_arrive(bar(B_STAT + m));
      ++done;
    }
  } else if (warp >= 12) {
    // ================================================================ epilogue
    // Writes a piece's rows while the softmax warps are in the next one.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    const int row = tid & 127;  // row within an M tile = TMEM lane
    const uint32_t tO = tmem + ((uint32_t)((warp & 3) * 32) << 16) + kColO;
    const bool wide = (reinterpret_cast<uintptr_t>(A.out) & 31) == 0;
    uint32_t done0 = 0, done1 = 0, tiles0 = 0, tiles1 = 0, joins = 0;
    bool ok = true;
    // The epilogue's threads meet (an mbarrier, for a wait that ends when the CTA gives up).
    auto meet = [&]() -> bool {
      mbar_arrive(bar(B_JOIN));
      return ok = await(bar(B_JOIN), joins++ & 1u, aborted);
    };
    while (ok && pieces.next<Lay>(await, bar, smem, aborted, x)) {
      const bool whole = x.t1 - x.t0 == x.T;
      const int64_t slot = 2 * (int64_t)blockIdx.x + (x.t0 == 0);
#pragma unroll 1
      for (int m = 0; m < 2; ++m) {
        if (m == 1 && !active1(x)) break;
        // STAT first: the softmax has then seen all PV products but the last
        const uint32_t done = m ? done1++ : done0++;  // pieces before, and tiles with this one
        const uint32_t tiles = m ? tiles1 += (uint32_t)(x.t1 - x.t0) : tiles0 += (uint32_t)(x.t1 - x.t0);
        if (!await(bar(B_STAT + m), done & 1u, aborted)) { ok = false; break; }
        const float inv = __ldcg(A.ws_inv + ((int64_t)blockIdx.x * 2 + m) * BM + row);
        if (!await(bar(B_PVDONE + m), (tiles - 1) & 1u, aborted)) { ok = false; break; }
        tc_fence_after();
        const int i = (2 * x.rg + m) * npb + row / G;
        const bool vrow = row < npb * G && i < x.n;
        uint16_t* orow = A.out + ((int64_t)(x.r0 + i) * A.heads_q + x.h * G + row % G) * D;
        float4* po = reinterpret_cast<float4*>(A.ws_o) + slot * (32 * 2 * BM) + m * BM + row;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {  // 32 columns
          uint32_t o[32];
          tmem_ld32(tO + m * D + q * 32, o);
          tmem_wait_ld();
          if (whole) {
            uint32_t v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k)
              v[k] = pack_bf16(__uint_as_float(o[2 * k]) * inv, __uint_as_float(o[2 * k + 1]) * inv);
            if (vrow) {
              st_global_32(orow + q * 32, v, wide);
              st_global_32(orow + q * 32 + 16, v + 8, wide);
            }
          } else if (vrow) {
            // a part of a unit: normalised O to the workspace, float4 columns [32][256 rows]
#pragma unroll
            for (int k = 0; k < 8; ++k)
              po[(q * 8 + k) * (2 * BM)] =
                  make_float4(__uint_as_float(o[4 * k]) * inv, __uint_as_float(o[4 * k + 1]) * inv,
                              __uint_as_float(o[4 * k + 2]) * inv, __uint_as_float(o[4 * k + 3]) * inv);
          }
        }
        tc_fence_before();
        mbar_arrive(bar(B_OFREE + m));
      }
      if (!ok || whole) continue;
      // The CTA whose part arrives last joins the unit when its own pieces are done.
      __threadfence();
      if (!meet()) break;
      if (tid == 12 * 32 && !*abort_flag && arrive(A.cnt + x.o0, A.tag) == x.parts) {
        A.cnt[x.o0] = 0;  // a completed unit leaves a zero word behind
        *reinterpret_cast<Piece*>(smem + kOffPieces + (kPieces + *n_joins) * (kPieceInts * 4)) = x;
        *n_joins = *n_joins + 1;
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    if (warp == 8) {
      // ================================================================ producer
      const int ps = A.kv.page_size;
      const int ppt = A.kv.layout == 1 ? BN / ps : 0;  // pages (boxes) of a tile: 2 .. 16
      const uint32_t qbytes = (uint32_t)(npb * G * 128);
      uint32_t qc = 0, issued = 0;   // pieces, ring tiles
      uint32_t st = 0, parity = 1u;  // the next ring tile's stage, and its wait's parity
      while (pieces.next<Lay>(await, bar, smem, aborted, x)) {
        auto page_of = [&](int t) -> int {  // lane p: page p of tile t; a missing one reads zeros
          const int tok = t * BN + lane * ps;
          if (lane >= ppt || tok >= x.keys) return -1;
          const int page = A.kv.block_table[(int64_t)x.b * A.kv.max_len + tok / ps];
          if (page < 0 || page >= A.kv.num_pages) {
            flag(A.err, CURE_DEVERR_PAGE);
            return -1;
          }
          return page;
        };
        int page = -1, next = page_of(x.t0);
        for (int i = 2 * x.t0; i < 2 * x.t1; ++i) {  // K and V tiles in turn
          const int t = i >> 1, kv = i & 1;
          if (!kv) {
            page = next;
            next = t + 1 < x.t1 ? page_of(t + 1) : -1;
          }
          if (!await(bar(B_EMPTY + st), parity, aborted)) goto produced;
          const uint32_t full = bar(B_FULL + st), dst = sb + kOffRing + st * kTile;
          if (lane == 0) mbar_arrive_expect_tx(full, kTile);
          __syncwarp();
          if (A.kv.layout == 1) {
            if (lane < ppt) tma_load_5d(dst + lane * ps * 256, kv ? &tm_v : &tm_k, full, 0, 0, 2 * x.h, 0, page);
          } else if (kv == 0) {
            if (lane < 2) tma_load_3d(dst + lane * kKHalf, &tm_k, full, lane * 64, x.h, x.b * A.kv.max_len + t * BN);
          } else if (lane < BN / 16) {
            // 16 rows each; those past the unit's keys from behind the tensor, which reads zeros
            const int row = t * BN + 16 * lane;
            tma_load_4d(dst + lane * kVChunk, &tm_v, full, 0,
                        row < x.keys ? x.b * A.kv.max_len + row : A.batch * A.kv.max_len, 0, x.h);
          }
          __syncwarp();
          ++issued;
          if (++st == NS) {
            st = 0;
            parity ^= 1u;
          }
          if (i == 2 * x.t0) {  // Q of both M tiles once the previous piece's S products are done
            if (!await(bar(B_QEMPTY), (qc & 1u) ^ 1u, aborted)) goto produced;
            ++qc;
            if (lane == 0) mbar_arrive_expect_tx(bar(B_QFULL), 4 * qbytes);
            __syncwarp();
            if (lane < 4)  // M tile lane / 2, d half lane % 2
              tma_load_4d(sb + kOffQ + lane * kQHalf, &tm_q, bar(B_QFULL), (lane & 1) * 64, 0, x.h,
                          x.r0 + (2 * x.rg + (lane >> 1)) * npb);
            __syncwarp();
          }
        }
      }
    produced:
      if (*abort_flag) {  // let copies in flight land before the CTA's smem goes away
        for (uint32_t i = (issued > NS ? issued - NS : 0); i < issued; ++i)
          wait_bounded(bar(B_FULL + i % NS), (i / NS) & 1u, abort_flag, A.err, false);
        if (qc > 0) wait_bounded(bar(B_QFULL), (qc - 1) & 1u, abort_flag, A.err, false);
      }
    } else if (warp == 9) {
      // ================================================================ S products
      constexpr uint32_t idS = idesc_bf16_f32(BM, BN, false);
      const bool paged = A.kv.layout == 1;
      uint32_t qc = 0, c = 0;        // pieces, products
      uint32_t st = 0, parity = 0u;  // the next K tile's stage, and its wait's parity
      const uint64_t qd = sdesc_sw128(sb + kOffQ, 16, 1024);
      const uint64_t kd = sdesc_sw128(sb + kOffRing, 16, paged ? kPgGroup : 1024u);
      const uint32_t k2 = (paged ? kPgHalf : kKHalf) >> 4;
      while (pieces.next<Lay>(await, bar, smem, aborted, x)) {
        if (!await(bar(B_QFULL), qc++ & 1u, aborted)) break;
        const int mts = active1(x) ? 2 : 1;
        for (int t = x.t0; t < x.t1; ++t) {
          const uint32_t k = (uint32_t)kd + st * (kTile >> 4);
#pragma unroll 1
          for (int m = 0; m < mts; ++m) {
            // (the first product waits for the phase before the first, which counts as done)
            if (!await(bar(B_SFREE), (c++ & 1u) ^ 1u, aborted)) goto scored;
            // The K tile, after SFREE: a parity wait is sound from the phase before on and
            // not later, and the stage's tile before this one, V of three tiles before, has
            // landed when the softmax of M tile 0 has loaded S of the tile before (it then
            // has seen the PV product of that V tile done).
            if (m == 0 && !await(bar(B_FULL + st), parity, aborted)) goto scored;
            tc_fence_after();
            issue_s(tmem + kColS, (uint32_t)qd + m * (2 * kQHalf >> 4), (uint32_t)(qd >> 32), k, (uint32_t)(kd >> 32),
                    k + k2, idS, bar(B_SFULL + m));
          }
          commit_elect(bar(B_EMPTY + st));
          if (t == x.t1 - 1) commit_elect(bar(B_QEMPTY));  // the piece's last use of Q
          st += 2;
          if (st >= NS) {
            st -= NS;
            parity ^= 1u;
          }
        }
      }
    scored:
      __syncwarp();
      commit_elect(bar(B_DRAIN));
      wait_bounded(bar(B_DRAIN), 0, abort_flag, A.err, false);
    } else if (warp == 10) {
      // ================================================================ PV products
      constexpr uint32_t idO = idesc_bf16_f32(BM, D, true);
      const bool paged = A.kv.layout == 1;
      uint32_t c0 = 0, c1 = 0, done0 = 0, done1 = 0;  // products and pieces of each M tile
      uint32_t st = 1, parity = 0u;                   // the next V tile's stage, and its wait's parity
      // V as an MN-major operand: the d halves LBO apart, 8-key groups SBO apart
      const uint64_t vd = sdesc_sw128(sb + kOffRing, paged ? kPgHalf : kVHalf, paged ? kPgGroup : 1024u);
      while (pieces.next<Lay>(await, bar, smem, aborted, x)) {
        const int mts = active1(x) ? 2 : 1;
        for (int t = x.t0; t < x.t1; ++t) {
          // (the stage's K tile of two tiles before has landed: its S became the P that this
          // warp has waited for)
          if (!await(bar(B_FULL + st), parity, aborted)) goto multiplied;
#pragma unroll 1
          for (int m = 0; m < mts; ++m) {
            // the first product of a piece takes O over from the epilogue of the one before
            // (from none at first: the phase before the first counts as done)
            if (t == x.t0 && !await(bar(B_OFREE + m), ((m ? done1++ : done0++) & 1u) ^ 1u, aborted)) goto multiplied;
            if (!await(bar(B_PFULL + m), (m ? c1++ : c0++) & 1u, aborted)) goto multiplied;
            tc_fence_after();
            issue_pv(tmem + kColO + m * D, tmem + kColP + m * 64, (uint32_t)vd + st * (kTile >> 4),
                     (uint32_t)(vd >> 32), idO, t > x.t0, bar(B_PVDONE + m));
          }
          commit_elect(bar(B_EMPTY + st));
          st += 2;
          if (st >= NS) {
            st -= NS;
            parity ^= 1u;
          }
        }
      }
    multiplied:
      __syncwarp();
      commit_elect(bar(B_DRAIN + 1));
      wait_bounded(bar(B_DRAIN + 1), 0, abort_flag, A.err, false);
    } else {
      // ================================================================ scheduler
      schedule<Lay>(A, npb, await, bar, smem, aborted, lane);
    }
  }

  // ---- the units that this CTA joins, by all warps and with equal registers again
  // (behind the barrier: a warp that had nothing to do must not take back the registers
  // that a softmax warp still waits for, or with all of them gone that wait has no end)
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp < 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 128;");
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 128;");
  if (*abort_flag) {
    if (tid == 0) flag(A.err, CURE_DEVERR_TIMEOUT);
  } else {
    join_units<Lay>(A, npb, smem, *n_joins, warp, lane);
  }
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace

// Workspace: piece counters [CTAs] (256-byte rounded), partial outputs and their
// log-sum-exps [2 * CTAs]: of a CTA's pieces at most its first and its last are
// parts of a unit; and the row sums that softmax warps leave for the epilogue.
namespace {
size_t counter_bytes(int ctas) { return ((size_t)ctas * sizeof(PieceCount) + 255) / 256 * 256; }
}  // namespace

size_t prompt_attn_workspace() {
  const int ctas = num_sms();
  return counter_bytes(ctas) + (size_t)ctas * 2 * BM * (2 * (D + 1) + 1) * sizeof(float);
}

cudaError_t launch_prompt_attn(const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                               const cure_kv_desc& kv, const int32_t* row_start, const int32_t* cache_len, int rows,
                               int batch, int heads_q, float scale, uint16_t* out, void* workspace, int* err,
                               cudaStream_t s, int expire_warp, int expire_wait) {
  const bool expire = expire_warp >= 0;
  const auto kernel = expire ? prompt_attn_kernel<true> : prompt_attn_kernel<false>;
  static std::atomic<uint64_t> ready[2];  // devices on which each has its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready[expire].load() & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    ready[expire].fetch_or(bit);
  }
  const int Hkv = kv.heads_kv, G = heads_q / Hkv;
  CUtensorMap mk, mv, mq;
  bool ok;
  if (kv.layout == 0) {
    const uint64_t n = (uint64_t)batch * kv.max_len;
    ok = make_kv_map(&mk, k_cache, n, Hkv, BN) && make_v_rows_map(&mv, v_cache, n, Hkv);
  } else {
    ok = make_page_map(&mk, k_cache, (uint64_t)kv.num_pages, kv.page_size, Hkv) &&
         make_page_map(&mv, v_cache, (uint64_t)kv.num_pages, kv.page_size, Hkv);
  }
  ok = ok && make_q_map(&mq, q, (uint64_t)rows, Hkv, G, BM / G);
  if (!ok) return cudaErrorInvalidValue;
  PromptArgs A;
  A.kv = kv;
  A.row_start = row_start;
  A.cache_len = cache_len;
  A.rows = rows;
  A.batch = batch;
  A.heads_q = heads_q;
  A.G = G;
  A.cap = std::min(kv.layout == 0 ? kv.max_len : kv.max_len * kv.page_size, INT32_MAX - 2 * BN);
  A.scale_log2 = scale * 1.4426950408889634f;
  A.out = out;
  A.err = err;
  A.expire_warp = expire_warp;
  A.expire_wait = expire_wait;
  A.tag = next_launch_tag();  // whatever the workspace's counters hold counts as zero
  const int ctas = num_sms();
  char* ws = static_cast<char*>(workspace);
  A.cnt = reinterpret_cast<PieceCount*>(ws);
  A.ws_o = reinterpret_cast<float*>(ws + counter_bytes(ctas));
  A.ws_lse = A.ws_o + (size_t)2 * ctas * 2 * BM * D;
  A.ws_inv = A.ws_lse + (size_t)2 * ctas * 2 * BM;
  // Many units: after the whole of the call before.  CTAs that start under it take the SMs
  // as they fall free, and then CTAs of neighbouring numbers, which take units side by
  // side, are not close to each other.  us back to back, so and as a programmatic
  // dependent: 17 units a CTA (32 ragged prompts) 332 and 359, 7 (8 of them) 96 and 102;
  // 3.5 (chunks of 8 prompts) 276 and 275; one prompt of 200 13.1 and 12.1.
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemBytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = (int64_t)rows * heads_q > (int64_t)4 * 2 * BM * ctas ? 0 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, mk, mv, mq, A);
}

}  // namespace cure
