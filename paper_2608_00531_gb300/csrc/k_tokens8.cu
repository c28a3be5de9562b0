// Attention of few rows a sequence over a cache held in 8 bits (cure_prompt_attn8 of single
// tokens): units of at most 16 (row, group head) pairs.
//
// The cache's bytes are the work, and tiles of 128 rows on tcgen05 would be nearly empty: an
// S and a PV product of a tile take 1024 cycles there, with the waits between them more than
// the tile's 1390 cycles of memory time.  Here a warp holds the unit's 16 rows in the
// fragments of mma.sync (m16n8k16, fp16) and goes through its keys alone:
//   - 32 keys a step, K and V by TMA into a ring of its own, no other warp to wait for;
//   - codes go from shared memory to the fragments in registers: K's four codes in a row are a lane's two
//     B registers of a step (the dims are numbered so), V's are paired by key;
//   - q is exact in fp16 under a power of two a row, P' = 2^(s + log2 vs - M + 7) as in k_prompt8.cu.
// The warps of a CTA take a piece's steps in turn, and add up their sums behind its last one, with the next
// piece's first steps on their way.  That costs a unit some 5 us; where there are many short units, each warp
// takes units of its own instead, and nothing is added up.
//
// Bound: HBM for long sequences but for the units' starts and ends, the warps' instructions for 8 heads of K and
// V (4 rows of 16 used).  64 tokens behind 500 to 16000 keys (28 heads, 4 of K and V) 96 us, 5.2 TB/s; 256 behind
// 1500 (32 and 8) 167 us (208 by whole CTAs), 200 behind 20 to 300 29 us (83).
// Units, pieces, the scheduler and joins: prompt_units.cuh.
#include <type_traits>

#include "prompt8.cuh"

namespace cure {
namespace {

using namespace prompt;

constexpr int kRows = 16;               // (row, group head) pairs of a unit
constexpr int kStep = 32;               // keys of a step
constexpr int kSteps = BN / kStep;      // of a tile
constexpr int kWorkers = 11;            // warps that attend; the last one lays out the pieces
constexpr int kThreads12 = 32 * (kWorkers + 1);
constexpr int NS = 2;                   // steps of a warp in shared memory
constexpr int kBlk = CURE_KV8_BLOCK;
constexpr int kHalf = kStep * D;        // 4 KiB: K or V of a step
constexpr int kQBytes = 8 * 32 * 16;    // a unit's Q
constexpr int kBatch = 8;               // steps whose pages and scales are looked up together
constexpr float kLift = 7.f;            // P' is 2^kLift times what it stands for

struct Lay {
  static constexpr int m_tiles = 1, threads = kThreads12, alone = kWorkers;
  enum : int { B_FULL = 0, B_DONE = B_FULL + kWorkers * NS, B_FREE, B_JOIN, piece_bar, taken_bar = piece_bar + kPieces, B_NEVER = taken_bar + kPieces, num_bars };
  static constexpr int ring = 0;                                   // [warp][stage][K, V][32 keys][128]
  static_assert(kRows * D * 4 == 2 * kHalf, "a warp's sums take a stage's place");
  static constexpr int lse = ring + kWorkers * NS * 2 * kHalf;     // float [warp][16 rows]
  static constexpr int q = lse + kWorkers * kRows * 4;             // uint [product][lane][4]: Q's fragments
  static constexpr int q_scale = q + kQBytes;                      // float [16 rows]
  static constexpr int place = q_scale + kRows * 4;                // int [warp]: where its sums are
  static constexpr int bars = (place + kWorkers * 4 + 7) / 8 * 8;
  static constexpr int abort = bars + 8 * num_bars;
  static constexpr int joins = abort + 4;
  static constexpr int pieces = (joins + 4 + 15) / 16 * 16;
  static constexpr int prefix = pieces + (kPieces + 2) * kPieceInts * 4;
  static constexpr int kept = (prefix + 8 * (kAttnMaxBatch + 1) + 15) / 16 * 16;  // the piece that is added up, a copy for each warp
  static constexpr int mode = kept + kWorkers * kPieceInts * 4;    // int: whether the warps attend alone
  static constexpr int bytes = mode + 16;
  // .. and where they may: [slot][warp] their pieces, [warp] Q's fragments (of the first at q) and factors.  (What shared memory takes
  // is lost to the L1 cache: where it is not used, this costs 3 %.)
  static constexpr int own = bytes;
  static constexpr int own_q = own + kPieces * kWorkers * kPieceInts * 4;
  static constexpr int own_scale = own_q + (kWorkers - 1) * kQBytes;
  static constexpr int bytes_alone = own_scale + kWorkers * kRows * 4;
  static_assert(bytes_alone <= 232448, "fits the 227 KiB opt-in");
};

// ALONE: warps may attend to units of their own.
template <bool ALONE>
struct TokenArgs : PromptArgs {
  // Its start and end cost a unit 5 us; a tile, 0.55 (64 sequences of 500 to 16000 keys: 111 us with 2, 106 with 4,
  // 99 with 6, 96 with 8 to 10, 99 with 16).
  static constexpr int kUnitCost = 9 * BN;
  // 256 sequences of 100 to 3000 keys, 8 heads of K and V: 212 us cut, 234 in turn; what cuts those leaves whole the
  // 208 us of 1500 keys each.
  static constexpr float kSpread = 0.8f;
  // A warp alone takes as long for a key as the CTA does for 6.5.
  static constexpr float kAloneTail = ALONE ? 6.5f : 0.f;
  const uint16_t* q;
  const float *k_scale, *v_scale;
};

__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}\n"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// c (16 x 8) += a (16 x 16) b (16 x 8)
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// EXPIRE (self-test): one wait of one warp runs out.
template <bool MAY_ALONE, bool EXPIRE>
__global__ void __launch_bounds__(kThreads12, 1)
tokens8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
               const TokenArgs<MAY_ALONE> A) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sb = smem_u32(smem);
  if (sb & 1023u) {  // the swizzled tiles need a 1 KiB-aligned base
    if (tid == 0) flag(A.err, CURE_DEVERR_ALIGN);
    return;
  }
  const int G = A.G, npb = kRows / G;
  const Bar bar{sb + Lay::bars};
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + Lay::abort);
  const uint32_t aborted = sb + Lay::abort;
  volatile int* n_joins = reinterpret_cast<volatile int*>(smem + Lay::joins);
  if (tid == 0) {
    for (int i = 0; i < kWorkers * NS; ++i) mbar_init(bar(Lay::B_FULL + i), 1);
    mbar_init(bar(Lay::B_DONE), 32 * kWorkers);
    mbar_init(bar(Lay::B_FREE), 32 * kWorkers);
    mbar_init(bar(Lay::B_JOIN), 32 * kWorkers);
    for (int i = 0; i < kPieces; ++i) {
      mbar_init(bar(Lay::piece_bar + i), 1);
      mbar_init(bar(Lay::taken_bar + i), kWorkers);
    }
    if constexpr (EXPIRE) mbar_init(bar(Lay::B_NEVER), 1);
    *abort_flag = 0;
    *n_joins = 0;
    *reinterpret_cast<volatile int*>(smem + Lay::mode) = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  pdl_begin();
  __syncthreads();
  Await<EXPIRE> await;
  if constexpr (EXPIRE) {
    await.never = bar(Lay::B_NEVER);
    await.left = blockIdx.x == 0 && warp == A.expire_warp ? (uint32_t)A.expire_wait : 0u;
  }

  if (warp == kWorkers) {
    schedule<Lay>(A, npb, await, bar, smem, aborted, lane);
  } else {
    // The scheduler's first piece says whether each warp attends to units of its own.
    auto attend = [&](auto tag) {
      constexpr bool ALONE = decltype(tag)::value;
    const int g = lane >> 2, t4 = lane & 3;  // fragment row (and key, and dims), fragment columns
    const int ps = A.kv.page_size;
    const bool paged = A.kv.layout == 1;
    const int per = paged ? ps / kBlk : 1;  // blocks of a page
    const int box = paged ? min(ps, kStep) : kStep, boxes = kStep / box;  // tokens of a copy, copies of K or V of a step
    const uint32_t ring = sb + Lay::ring + warp * (NS * 2 * kHalf);
    float* lses = reinterpret_cast<float*>(smem + Lay::lse);
    volatile int* place_of_sums = reinterpret_cast<volatile int*>(smem + Lay::place);
    Piece* kept = reinterpret_cast<Piece*>(smem + Lay::kept) + warp;
    Pieces pieces{0};
    Piece x;
    uint32_t issued = 0, used = 0, done = 0, joins = 0;
    // The piece's steps of this warp, of those with keys of the unit: warp, warp + 11, .., or all.
    constexpr int S = ALONE ? 1 : kWorkers;
    constexpr int kRaw = ALONE ? 4 : 2;  // rows of Q on their way
    const uint32_t qs = ALONE && warp > 0 ? Lay::own_q + (warp - 1) * kQBytes : Lay::q;
    float* q_scale = reinterpret_cast<float*>(smem + (ALONE ? Lay::own_scale + warp * kRows * 4 : Lay::q_scale));
    int s0, n;
    // Pages and scales are looked up kBatch steps at a time, two batches and one ahead.  Lane 4 k + 2 v + p:
    // where block p of the batch's step k lies in a paged cache (page * blocks + block; -1: nowhere, zeros), and
    // its scale of K (v = 0) or V.
    int place0, place1, place2;
    float scale0, scale1;
    auto look_up = [&](int batch) -> int {
      const int k = batch * kBatch + (lane >> 2), tok = (s0 + k * S) * kStep + (lane & 1) * kBlk;
      if (k >= n || tok >= x.keys) return -1;
      if (!paged) return 0;
      const int page = A.kv.block_table[(int64_t)x.b * A.kv.max_len + tok / ps];
      if (page < 0 || page >= A.kv.num_pages) {
        flag(A.err, CURE_DEVERR_PAGE);
        return -1;
      }
      return page * per + tok % ps / kBlk;
    };
    auto scale_of = [&](int batch, int place) -> float {
      if (place < 0) return 1.f;
      int64_t at = place;
      if (!paged)
        at = (int64_t)x.b * ((A.kv.max_len + kBlk - 1) / kBlk) + (s0 + (batch * kBatch + (lane >> 2)) * S) * (kStep / kBlk) +
             (lane & 1);
      return __ldg((lane & 2 ? A.v_scale : A.k_scale) + at * A.kv.heads_kv + x.h);
    };
    // The copies of step k; `ahead`: it is one of the batch behind the one that place0 is of.
    auto issue = [&](int k, bool ahead) {
      const uint32_t st = issued % NS, full = bar(Lay::B_FULL + warp * NS + st);
      const int place = __shfl_sync(0xffffffffu, ahead ? place1 : place0, (k % kBatch) * 4 + (lane & 1));
      if (lane == 0) mbar_arrive_expect_tx(full, 2 * kHalf);
      __syncwarp();
      if (lane < 4 && (lane & 1) < boxes) {  // K's boxes, V's boxes
        const uint32_t dst = ring + st * (2 * kHalf) + (lane >> 1) * kHalf + (lane & 1) * (box * D);
        const CUtensorMap* map = lane < 2 ? &tm_k : &tm_v;
        if (paged) tma_load_4d(dst, map, full, 0, x.h, place < 0 ? 0 : place % per * kBlk, place < 0 ? -1 : place / per);
        else tma_load_4d(dst, map, full, 0, x.h, (s0 + k * S) * kStep, x.b);
      }
      __syncwarp();
      ++issued;
    };
    // The next piece, its look-ups, and its first step on the way.
    auto begin = [&]() -> bool {
      if constexpr (ALONE) {
        const uint32_t slot = pieces.k % kPieces;
        if (!await(bar(Lay::piece_bar + slot), (pieces.k / kPieces) & 1u, aborted)) return false;
        x = reinterpret_cast<const Piece*>(smem + Lay::own)[slot * kWorkers + warp];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(Lay::taken_bar + slot));
        ++pieces.k;
        if (x.t0 >= x.t1) return false;
      } else {
        if (!pieces.next<Lay>(await, bar, smem, aborted, x)) return false;
      }
      s0 = x.t0 * kSteps + (ALONE ? 0 : warp);
      const int s_end = min(x.t1 * kSteps, (x.keys + kStep - 1) / kStep);
      n = s0 < s_end ? (s_end - s0 + S - 1) / S : 0;
      place0 = look_up(0);
      place1 = look_up(1);
      place2 = look_up(2);
      if (n > 0) issue(0, false);
      scale0 = scale_of(0, place0);
      scale1 = scale_of(1, place1);
      return true;
    };
    // Q: rows first, first + each of the unit (the warp's: warp, warp + 11), 4 dims a lane, on their way
    uint2 raw[kRaw];
    auto load_q = [&](int first, int each) {
#pragma unroll
      for (int r = 0; r < kRaw; ++r) {
        const int row = first + each * r, i = x.rg * npb + row / G;
        raw[r] = make_uint2(0u, 0u);
        if (row < npb * G && i < x.n)
          raw[r] = __ldg(reinterpret_cast<const uint2*>(
              A.q + ((int64_t)(x.r0 + i) * A.heads_q + x.h * G + row % G) * D + 4 * lane));
      }
    };
    // .. in fp16 under a power of two that brings a row below 448, as the products' fragments: dims 4 L ..
    // 4 L + 3 of row r are registers r / 8 and 2 + r / 8 of product L % 8 in lane 4 (r % 8) + L / 8
    auto put_q = [&](int first, int each) {
#pragma unroll
      for (int r = 0; r < kRaw; ++r) {
        const int row = first + each * r;
        if (row >= kRows) break;
        const float v[4] = {__uint_as_float(raw[r].x << 16), __uint_as_float(raw[r].x & 0xffff0000u),
                            __uint_as_float(raw[r].y << 16), __uint_as_float(raw[r].y & 0xffff0000u)};
        const float mine = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
        const uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(mine));
        const int e = min(max((int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u), -60), 120);
        const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
        uint32_t* to = reinterpret_cast<uint32_t*>(smem + qs) + ((lane & 7) * 32 + 4 * (row & 7) + (lane >> 3)) * 4 + (row >> 3);
        to[0] = pack_f16(v[0] * inv, v[1] * inv);
        to[2] = pack_f16(v[2] * inv, v[3] * inv);
        if (lane == 0)
          q_scale[row] =
              fminf(fmaxf(A.scale_log2 * __uint_as_float((uint32_t)(127 + e) << 23), 0x1p-80f), 0x1p80f);
      }
    };
    bool more = begin();
    if (more && !ALONE) {
      load_q(warp, kWorkers);
      put_q(warp, kWorkers);
      mbar_arrive(bar(Lay::B_FREE));
    }
    while (more) {
      if constexpr (ALONE) {
#pragma unroll 1
        for (int row = 0; row < kRows; row += kRaw) {
          load_q(row, 1);
          put_q(row, 1);
        }
        __syncwarp();
      } else {  // all have read this warp's sums, and Q is there
        if (!await(bar(Lay::B_FREE), done & 1u, aborted)) break;
      }
      if (n > 1) issue(1, false);
      float c[2];
      int sees[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        c[r] = q_scale[g + 8 * r];
        sees[r] = x.L + x.rg * npb + (g + 8 * r) / G + 1;
      }
      const int least = x.L + x.rg * npb + 1;  // keys that all rows see

      float o[16][4], m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
#pragma unroll 1
      for (int k = 0; k < n; ++k) {
        if (k > 0 && k % kBatch == 0) {
          place0 = place1;
          scale0 = scale1;
          place1 = place2;
          scale1 = scale_of(k / kBatch + 1, place1);
          place2 = look_up(k / kBatch + 2);
        }
        const uint32_t st = used % NS;
        if (!await(bar(Lay::B_FULL + warp * NS + st), (used / NS) & 1u, aborted)) goto out;
        ++used;
        const uint32_t kb = ring + st * (2 * kHalf), vb = kb + kHalf;
        const int key0 = (s0 + k * S) * kStep;
        // ---- S: key 8 nt + g of the step; codes 4 w .. + 3 of 16 are a lane's B registers of one product
        float s[4][4];
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint4 w[4];
#pragma unroll
          for (int nt = 0; nt < 4; ++nt) w[nt] = ld_shared_v4(kb + (8 * nt + g) * D + (((2 * t4 + j) ^ g) << 4));
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const uint4 q = ld_shared_v4(sb + qs + ((4 * j + z) * 32 + lane) * 16);
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) {
              uint32_t b0, b1;
              widen(z == 0 ? w[nt].x : z == 1 ? w[nt].y : z == 2 ? w[nt].z : w[nt].w, b0, b1);
              mma(s[nt], q.x, q.y, q.z, q.w, b0, b1);
            }
          }
        }
        // ---- the step's scales, masks, the maximum of s + log2 vs
        float ks[2], lv[2], iv[2];
        {
          const float sc = fminf(fmaxf(scale0, 0x1p-40f), 0x1p40f), lg = log2f(sc), rc = 1.f / sc;
          const int at = k % kBatch * 4;
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            ks[b] = __shfl_sync(0xffffffffu, sc, at + b);
            lv[b] = __shfl_sync(0xffffffffu, lg, at + 2 + b);
            iv[b] = __shfl_sync(0xffffffffu, rc, at + 2 + b);
          }
        }
        if (key0 + kStep > least) {
#pragma unroll
          for (int nt = 0; nt < 4; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (key0 + 8 * nt + 2 * t4 + (e & 1) >= sees[e >> 1]) s[nt][e] = -INFINITY;
        }
        float alpha[2];
        bool need = false;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float mt = -INFINITY;
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const float top = fmaxf(fmaxf(s[2 * b][2 * r], s[2 * b][2 * r + 1]), fmaxf(s[2 * b + 1][2 * r], s[2 * b + 1][2 * r + 1]));
            mt = fmaxf(mt, fmaf(top, c[r] * ks[b], lv[b]));
          }
          mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, 1));
          mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, 2));
          const bool grows = mt > m_run[r] + 8.f;
          alpha[r] = grows ? ex2(m_run[r] - mt) : 1.f;
          if (grows) m_run[r] = mt;
          need |= grows;
        }
        if (__any_sync(0xffffffffu, need)) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] *= alpha[e >> 1];
          l_run[0] *= alpha[0];
          l_run[1] *= alpha[1];
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          uint32_t a[4];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float nb = (m_run[r] == -INFINITY ? 0.f : kLift - m_run[r]) + lv[b], cb = c[r] * ks[b];
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = ex2(fmaf(s[2 * b + (e >> 1)][2 * r + (e & 1)], cb, nb));
            l_run[r] = fmaf((p[0] + p[1]) + (p[2] + p[3]), iv[b], l_run[r]);
            a[r] = pack_f16(p[0], p[1]);
            a[2 + r] = pack_f16(p[2], p[3]);
          }
          // ---- O: dims 16 g + i of product i, keys 16 b + 2 t4, + 1, + 8, + 9; codes of two keys in a register
          uint4 v[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const int key = 16 * b + 2 * t4 + (z & 1) + 8 * (z >> 1);
            v[z] = ld_shared_v4(vb + key * D + ((g ^ (key & 7)) << 4));
            // what lies behind the unit's last key must not reach O through 0 * NaN
            if (key0 + kStep > x.keys && key0 + key >= x.keys) v[z] = make_uint4(0u, 0u, 0u, 0u);
          }
          if (b == 1) {  // the stage is read
            __syncwarp();
            if (k + NS < n) issue(k + NS, (k + NS) / kBatch != k / kBatch);
          }
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t u0 = w == 0 ? v[0].x : w == 1 ? v[0].y : w == 2 ? v[0].z : v[0].w;
            const uint32_t u1 = w == 0 ? v[1].x : w == 1 ? v[1].y : w == 2 ? v[1].z : v[1].w;
            const uint32_t u2 = w == 0 ? v[2].x : w == 1 ? v[2].y : w == 2 ? v[2].z : v[2].w;
            const uint32_t u3 = w == 0 ? v[3].x : w == 1 ? v[3].y : w == 2 ? v[3].z : v[3].w;
            uint32_t x0[4], x1[4];
            widen(__byte_perm(u0, u1, 0x5140), x0[0], x0[1]);
            widen(__byte_perm(u0, u1, 0x7362), x0[2], x0[3]);
            widen(__byte_perm(u2, u3, 0x5140), x1[0], x1[1]);
            widen(__byte_perm(u2, u3, 0x7362), x1[2], x1[3]);
#pragma unroll
            for (int z = 0; z < 4; ++z) mma(o[4 * w + z], a[0], a[1], a[2], a[3], x0[z], x1[z]);
          }
        }
      }
      // ---- the next piece is on its way before this one is added up; the sums lie in the stage behind its
      // first step's
      if (lane == 0) *kept = x;
      __syncwarp();
      more = begin();
      if constexpr (ALONE) {
        // a lane's 32 dims of rows g and g + 8
        const Piece prev = *kept;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float l = l_run[r];
          l += __shfl_xor_sync(0xffffffffu, l, 1);
          l += __shfl_xor_sync(0xffffffffu, l, 2);
          const float inv = l > 0.f ? 1.f / l : 0.f;
          const int row = g + 8 * r, i = prev.rg * npb + row / G;
          if (row >= npb * G || i >= prev.n) continue;
          uint16_t* orow = A.out + ((int64_t)(prev.r0 + i) * A.heads_q + prev.h * G + row % G) * D + 32 * t4;
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int d = 0; d < 16; d += 8) {
              uint32_t w[4];
#pragma unroll
              for (int z = 0; z < 4; ++z)
                w[z] = pack_bf16(o[d + 2 * z][2 * r + e] * inv, o[d + 2 * z + 1][2 * r + e] * inv);
              *reinterpret_cast<uint4*>(orow + 16 * e + d) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        __syncwarp();  // (all lanes have read the piece)
        continue;
      }
      const uint32_t st = issued % NS;
      float* mine = reinterpret_cast<float*>(smem + Lay::ring + warp * (NS * 2 * kHalf) + st * (2 * kHalf));
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float l = l_run[r];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        const float inv = l > 0.f ? 1.f / l : 0.f;
        if (t4 == 0) lses[warp * kRows + g + 8 * r] = row_lse(m_run[r] - kLift, l);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<float4*>(mine + (g + 8 * r) * D + 32 * t4 + 16 * e + i) =
                make_float4(o[i][2 * r + e] * inv, o[i + 1][2 * r + e] * inv, o[i + 2][2 * r + e] * inv,
                            o[i + 3][2 * r + e] * inv);
      }
      if (lane == 0) place_of_sums[warp] = (int)(warp * (NS * 2 * kHalf) + st * (2 * kHalf));
      if (more) load_q(warp, kWorkers);
      mbar_arrive(bar(Lay::B_DONE));
      if (!await(bar(Lay::B_DONE), done & 1u, aborted)) break;
      ++done;
      // ---- a row's 8 dims a thread: O = sum_w 2^(lse_w) O_w / sum_w 2^(lse_w)
      const Piece prev = *kept;
      const bool whole = prev.t1 - prev.t0 == prev.T;
      if (tid < kRows * D / 8) {
        const int row = tid >> 4, d0 = (tid & 15) * 8, i = prev.rg * npb + row / G;
        const bool vrow = row < npb * G && i < prev.n;
        float top = -FLT_MAX, total = 0.f;
#pragma unroll
        for (int k = 0; k < kWorkers; ++k) top = fmaxf(top, lses[k * kRows + row]);
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
#pragma unroll
        for (int k = 0; k < kWorkers; ++k) {
          const float wk = ex2(lses[k * kRows + row] - top);
          total += wk;
          const float4* src = reinterpret_cast<const float4*>(smem + Lay::ring + place_of_sums[k]) + (row * D + d0) / 4;
          const float4 y = src[0], z = src[1];
          a = make_float4(fmaf(wk, y.x, a.x), fmaf(wk, y.y, a.y), fmaf(wk, y.z, a.z), fmaf(wk, y.w, a.w));
          b = make_float4(fmaf(wk, z.x, b.x), fmaf(wk, z.y, b.y), fmaf(wk, z.z, b.z), fmaf(wk, z.w, b.w));
        }
        const float r = 1.f / total;
        a = make_float4(a.x * r, a.y * r, a.z * r, a.w * r);
        b = make_float4(b.x * r, b.y * r, b.z * r, b.w * r);
        if (whole && vrow) {
          uint16_t* orow = A.out + ((int64_t)(prev.r0 + i) * A.heads_q + prev.h * G + row % G) * D + d0;
          *reinterpret_cast<uint4*>(orow) =
              make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
        } else if (vrow) {
          // a part of a unit: to the workspace, float4 columns [32][256 rows]
          const int64_t slot = 2 * (int64_t)blockIdx.x + (prev.t0 == 0);
          float4* po = reinterpret_cast<float4*>(A.ws_o) + (slot * 32 + d0 / 4) * (2 * BM) + row;
          po[0] = a;
          po[2 * BM] = b;
          if ((tid & 15) == 0) __stcg(A.ws_lse + slot * (2 * BM) + row, top + log2f(total));
        }
      }
      if (more) put_q(warp, kWorkers);
      fence_proxy_async_smem();  // (the sums' places get copies next)
      mbar_arrive(bar(Lay::B_FREE));
      if (whole) continue;
      // The CTA whose part arrives last joins the unit when its own pieces are done.
      __threadfence();
      mbar_arrive(bar(Lay::B_JOIN));
      if (!await(bar(Lay::B_JOIN), joins++ & 1u, aborted)) break;
      if (tid == 0 && !*abort_flag && arrive_at(A.cnt + prev.o0, A.tag) == prev.parts) {
        A.cnt[prev.o0] = 0;  // a completed unit leaves a zero word behind
        *reinterpret_cast<Piece*>(smem + Lay::pieces + (kPieces + *n_joins) * (kPieceInts * 4)) = prev;
        *n_joins = *n_joins + 1;
      }
    }
  out:
    if (*abort_flag)  // let copies in flight land before the CTA's smem goes away
      for (; used < issued; ++used)
        wait_bounded(bar(Lay::B_FULL + warp * NS + used % NS), (used / NS) & 1u, abort_flag, A.err, false);
    };
    if constexpr (MAY_ALONE) {
      if (await(bar(Lay::piece_bar), 0, aborted)) {
        if (*reinterpret_cast<volatile int*>(smem + Lay::mode)) attend(std::true_type{});
        else attend(std::false_type{});
      }
    } else {
      attend(std::false_type{});
    }
  }
  __syncthreads();
  if (*abort_flag) {
    if (tid == 0) flag(A.err, CURE_DEVERR_TIMEOUT);
  } else {
    join_units<Lay>(A, npb, smem, *n_joins, warp, lane);
  }
}

}  // namespace

// Sequences whose rows fit one unit on average.  Against k_prompt8.cu: 64 sequences of 1 / 2 rows behind
// 500 to 8000 keys (28 and 4 heads) 65 / 71 and 97 / 104 us, of 2 / 4 rows (32 and 8 heads) 108 / 122 and 170 / 192.
// A long chunk among them is read again for each of its units: one of 64 rows beside 63 single tokens 70 and 79,
// one of 300 rows beside 128 169 and 262, one of 100 rows behind 8000 keys beside 40 114 and 92, one of 600 behind
// 4000 beside 255 417 and 311.  (A launch of each for the sequences that it suits was slower in most of these.)
bool tokens8_fits(const Attn8Call& c) {
  const int G = c.heads_q / c.kv.heads_kv;
  return !c.n_nodes && G <= kRows && c.rows <= (int64_t)c.batch * (kRows / G);
}

template <bool ALONE, bool EXPIRE>
static cudaError_t launch(const Attn8Call& c, cudaStream_t s) {
  constexpr int bytes = ALONE ? Lay::bytes_alone : Lay::bytes;
  static std::atomic<uint64_t> ready;  // devices on which it has its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready.load() & bit)) {
    e = cudaFuncSetAttribute(tokens8_kernel<ALONE, EXPIRE>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit);
  }
  CUtensorMap mk, mv;
  const int box = c.kv.layout == 1 ? std::min(c.kv.page_size, kStep) : kStep;
  if (!make_codes_map(&mk, c.k_cache, c.kv, c.batch, box) || !make_codes_map(&mv, c.v_cache, c.kv, c.batch, box))
    return cudaErrorInvalidValue;
  TokenArgs<ALONE> A = {};
  fill_args8(c, &A);
  A.q = c.q;
  A.k_scale = c.k_scale;
  A.v_scale = c.v_scale;
  return launch_pdl(tokens8_kernel<ALONE, EXPIRE>, dim3((unsigned)num_sms()), dim3(kThreads12), (size_t)bytes, s, mk, mv, A);
}

// Fewer units than two to an SM are never a warp's each; the kernel that asks is 2 to 3 % slower where the answer is
// no (64 sequences of 500 to 16000 keys, 4 heads of K and V: 98 us, not 96).
cudaError_t launch_tokens8(const Attn8Call& c, cudaStream_t s) {
  const bool alone = c.batch > 32 && (int64_t)c.rows * c.kv.heads_kv >= (int64_t)2 * num_sms();
  if (c.expire_wait > 0) return alone ? launch<true, true>(c, s) : launch<false, true>(c, s);
  return alone ? launch<true, false>(c, s) : launch<false, false>(c, s);
}

}  // namespace cure
