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
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "attn_tc.cuh"

namespace cure {
namespace {

using namespace tc;

constexpr int BM = kAttnRowsCta;  // 128 rows per M tile
constexpr int BN = 128;           // keys per tile
constexpr int D = kAttnD;
constexpr int NS = 5;             // ring stages, a K or a V tile each
constexpr int kThreads = 512;
constexpr uint32_t kTmemCols = 512;
constexpr int kPieces = 4;        // pieces that the scheduler may be ahead
constexpr int kTakers = 15;       // warps that take pieces: all but the scheduler

constexpr int kQHalf = kAttnQHalf;      // 16 KiB: [128 rows][64 d]
constexpr int kKHalf = BN * 64 * 2;     // 16 KiB: [128 keys][64 d]
constexpr int kTile = 2 * kKHalf;       // 32 KiB
constexpr int kVChunk = kAttnVChunk;    // 4 KiB: V keys 16c..16c+15, both d halves
constexpr int kVHalf = kVChunk / 2;
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
constexpr int kPieceInts = 12;
constexpr int kOffPieces = (kOffJoins + 4 + 15) / 16 * 16;            // int [kPieces][kPieceInts], then [2] to join
constexpr int kOffPrefix = kOffPieces + (kPieces + 2) * kPieceInts * 4;  // int64 first position of each sequence [B+1]
constexpr int kSmemBytes = kOffPrefix + 8 * (kAttnMaxBatch + 1);
static_assert(kSmemBytes <= 232448, "fits the 227 KiB opt-in");

constexpr uint32_t kColS = 0;    // S:    columns 0 .. 127
constexpr uint32_t kColP = 128;  // P[m]: columns 128 + m*64
constexpr uint32_t kColO = 256;  // O[m]: columns 256 + m*128

struct PromptArgs {
  cure_kv_desc kv;
  const int32_t* row_start;
  const int32_t* cache_len;
  int rows, batch, heads_q, G, cap;
  float scale_log2;
  PieceCount* cnt;  // [CTAs] (launch tag << 9) | pieces arrived of the unit whose first piece the CTA has
  uint64_t tag;     // this launch's tag
  float* ws_o;    // [2 * CTAs][32][256] float4 partial outputs
  float* ws_lse;  // [2 * CTAs][256] their base-2 log-sum-exps
  float* ws_inv;  // [CTAs][2 M tiles][128 rows] reciprocal row sums, softmax to epilogue
  uint16_t* out;
  int* err;
  int expire_warp, expire_wait;  // self-test: the wait of CTA 0 that runs out, by its warp and number from 1
};

// Positions.  Every unit takes kUnitCost positions (what starting and ending a
// piece costs, in key times) and then one for each key of the last row that its
// row group could have; tile t of it stands at the position of its first key.
constexpr int kUnitCost = 2 * BN;
// What joining the parts of units costs a call (7 to 8 us: a prompt of 200 or 1024 cut
// needlessly), and the fewest positions worth a CTA.
constexpr int kJoinCost = 8 * BN;
constexpr int kMinShare = 3 * BN;
// Units of fewer positions on average, and those of a batch of more than 32, are
// dealt out in turn: the reckoning that evens them out would take longer than they do.
constexpr int kShortUnit = kUnitCost + 5 * BN;
// A share's border that lies nearer to a unit's border than this moves there.
constexpr int kSnap = 4 * BN;

// A sequence's rows and the tokens before them; n = 0 where they do not make sense.
struct Seq {
  int r0, n, L;
};
__device__ __forceinline__ Seq sequence(const PromptArgs& A, int b, int* bad) {
  Seq s;
  s.r0 = A.row_start[b];
  s.L = A.cache_len[b];
  const int64_t n = (int64_t)A.row_start[b + 1] - s.r0;
  s.n = (int)n;
  *bad = 0;
  if (s.r0 < 0 || n < 0 || s.r0 + n > A.rows) *bad = CURE_DEVERR_NODES;
  else if (n > 0 && (s.L < 0 || s.L + n > A.cap)) *bad = CURE_DEVERR_SLOT;
  if (*bad) s.n = 0;
  return s;
}

// Tiles [t0, t1) of one unit.
struct alignas(16) Piece {
  int b, h, rg;    // sequence, kv head, row group
  int r0, n, L;    // the sequence's rows and the tokens before them
  int keys, T;     // keys that any of the unit's rows sees, and their tiles
  int t0, t1;      // t0 == t1: no more pieces
  int o0, parts;   // the unit's pieces: of CTAs o0 .. o0 + parts - 1
};
static_assert(sizeof(Piece) == 4 * kPieceInts, "as it lies in shared memory");

__device__ __forceinline__ float sqrt_approx(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// a / b of nonnegative numbers for a quotient of at most `most` (below 2^22 or so).
__device__ __forceinline__ int small_quotient(int64_t a, int64_t b, int most) {
  int q = min(most, (int)__fdividef((float)a, (float)b));  // off by one or two at most
  while (q * b > a) --q;
  while (q < most && (q + 1) * b <= a) ++q;
  return q;
}

// The units of a call, laid end to end, as the scheduler warp walks them.  Either
// they are cut (positions as above, an even share of them for every CTA) or they
// are dealt out whole, one position each; `falling`: the long ones first, the
// sequences in the order of their lengths, their row groups from the last one down.
//
// A batch of up to 32 sequences stays in the warp's registers, a sequence a lane;
// of a larger one the first positions lie in shared memory and the rest is read
// again.  (A call's first piece was 5,000 cycles away, most of it dependent loads.)
struct Walk {
  const int64_t* start;   // large batches: first position of each sequence
  bool few, falling;
  Seq mine;               // few: the lane's sequence, its number and its first position
  int number_of_mine;
  int64_t first_of_mine;
  int B, Hkv, R;          // R: rows of a row group
  bool split;
  int P;                  // CTAs that take part
  int64_t share;          // positions of one CTA (the last one takes the rest)
  int64_t near;           // how far a share's border moves to a unit's border at most
  // the unit at position ustart: sequence i (number b), the k-th row group, head h
  Seq s;
  int i, b, k, h, groups;
  int64_t ustart, cost;

  __device__ __forceinline__ int groups_of(int n) const {  // row groups of n rows
    const int a = n + R - 1;  // below 2^24
    int q = (int)__fdividef((float)a, (float)R);
    while (q * R > a) --q;
    while ((q + 1) * R <= a) ++q;
    return q;
  }
  // the k-th row group's positions for a head: of the first, and what each adds
  __device__ __forceinline__ int base() const { return split ? kUnitCost + s.L : 1; }
  __device__ __forceinline__ int step() const { return split ? R : 0; }
  __device__ __forceinline__ int64_t before(int k) const {  // a head's positions in front of the k-th row group
    return k * (int64_t)base() + (int64_t)step() * k * (k + 1) / 2;
  }
  __device__ __forceinline__ int owner(int64_t p) const { return small_quotient(p, share, P - 1); }
  __device__ __forceinline__ void load(const PromptArgs& A) {
    if (few) {
      s.r0 = __shfl_sync(0xffffffffu, mine.r0, i);
      s.n = __shfl_sync(0xffffffffu, mine.n, i);
      s.L = __shfl_sync(0xffffffffu, mine.L, i);
      b = __shfl_sync(0xffffffffu, number_of_mine, i);
    } else {
      int bad;
      b = i;
      s = sequence(A, b, &bad);
    }
    groups = groups_of(s.n);
  }
  __device__ __forceinline__ void price() { cost = base() + (int64_t)(k + 1) * step(); }
  __device__ __forceinline__ void seek(const PromptArgs& A, int64_t g) {  // the unit that holds position g
    int64_t first;  // of the last sequence that starts at or before it
    if (few) {
      i = __popc(__ballot_sync(0xffffffffu, (int)(threadIdx.x & 31) < B && first_of_mine <= g)) - 1;
      first = __shfl_sync(0xffffffffu, first_of_mine, i);
    } else {
      int lo = 0, hi = B;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= g) lo = mid;
        else hi = mid;
      }
      i = lo;
      first = start[i];
    }
    load(A);
    const int64_t local = g - first;
    // the last row group that starts at or before it: local = Hkv before(k), off by one or two at most
    const float d = (float)step(), each = (float)base() + 0.5f * d, l = __fdividef((float)local, (float)Hkv);
    k = min(groups - 1, (int)__fdividef(2.f * l, each + sqrt_approx(each * each + 2.f * d * l)));
    int64_t at = Hkv * before(k);
    while (k > 0 && at > local) at = Hkv * before(--k);
    while (k < groups - 1) {
      const int64_t next = Hkv * before(k + 1);
      if (next > local) break;
      at = next;
      ++k;
    }
    price();
    h = small_quotient(local - at, cost, Hkv - 1);
    ustart = first + at + h * cost;
  }
  __device__ __forceinline__ void advance(const PromptArgs& A) {  // to the next unit (there is one)
    ustart += cost;
    if (++h < Hkv) return;
    h = 0;
    if (++k == groups) {
      k = 0;
      do {
        ++i;
        load(A);
      } while (groups == 0 && i + 1 < B);
    }
    price();
  }
  __device__ __forceinline__ int row_group() const { return falling ? groups - 1 - k : k; }
  __device__ __forceinline__ int keys() const { return s.L + min((row_group() + 1) * R, s.n); }
  __device__ __forceinline__ int tiles() const { return (keys() + BN - 1) / BN; }
  // Where the border p of a share, which lies in this unit, is drawn: at one of the
  // unit's borders if that is near (or if one side would be left without a tile).
  __device__ __forceinline__ int64_t border(int64_t p) const {
    const int64_t first = ustart + kUnitCost;
    if (p < first + near) return ustart;
    if (p > first + (int64_t)(tiles() - 1) * BN || ustart + cost - p < near) return ustart + cost;
    return p;
  }
  // The unit's tiles in the range [g, g_end) between drawn borders.
  __device__ __forceinline__ Piece within(int64_t g, int64_t g_end) const {
    Piece x;
    x.b = b;
    x.h = h;
    x.rg = row_group();
    x.r0 = s.r0;
    x.n = s.n;
    x.L = s.L;
    x.keys = keys();
    x.T = tiles();
    x.t0 = 0;
    x.t1 = x.T;
    x.o0 = (int)blockIdx.x;
    x.parts = 1;
    if (split) {
      const int64_t first = ustart + kUnitCost;  // tile 0's position
      if (g > first) x.t0 = (int)min((int64_t)x.T, (g - first + BN - 1) / BN);
      x.t1 = g_end <= first ? 0 : (int)min((int64_t)x.T, (g_end - first + BN - 1) / BN);
      if (x.t0 < x.t1 && x.t1 - x.t0 < x.T) {
        // the shares that the first and the last tile lie in, and theirs after the borders moved
        int o1 = owner(first + (int64_t)(x.T - 1) * BN);
        x.o0 = owner(first);
        if (x.o0 < P - 1 && (x.o0 + 1) * share < first + near) ++x.o0;
        if (o1 * share >= first + near && ustart + cost - o1 * share < near) --o1;
        x.parts = o1 - x.o0 + 1;
      }
    }
    return x;
  }
};

// The roles' waits.  What the roles run between them fits the instruction cache or does
// not: with tc::wait_warp in the 17 places 8 prompts of 2048 took 213 us, so 206.
template <bool EXPIRE>
struct Await {
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity, uint32_t abort_flag) {
    return wait_compact<(uint32_t)kWaitTimeoutCycles>(bar, parity, abort_flag);
  }
};
// In the self-test's kernel one wait of one warp is for what never comes.
template <>
struct Await<true> {
  uint32_t never;  // a barrier that nothing completes
  uint32_t left;   // waits up to and with that one (0: none)
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity, uint32_t abort_flag) {
    if (left > 0 && --left == 0) return wait_compact<1u << 20>(never, 0, abort_flag);
    return wait_compact<(uint32_t)kWaitTimeoutCycles>(bar, parity, abort_flag);
  }
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
// O_m (+)= P_m V: 8 steps of 16 keys, P 8 columns of bf16 pairs and V a chunk further on each.
__device__ __forceinline__ void issue_pv(uint32_t d, uint32_t p, uint32_t v, uint32_t v_hi, uint32_t idesc,
                                         uint32_t accumulate, uint32_t done) {
  static_assert(kVChunk >> 4 == 256, "as the steps are written");
  asm volatile(
      "{\n\t.reg .pred p0, pt, el;\n\t.reg .b64 b;\n\t.reg .b32 x, y;\n\t"
      "elect.sync _|el, 0xffffffff;\n\t"
      "setp.ne.b32 p0, %5, 0;\n\t"
      "setp.eq.b32 pt, 0, 0;\n\t"
      "mov.b64 b, {%2, %3};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p0;\n\t"
      "add.u32 x, %1, 8;\n\tadd.u32 y, %2, 256;\n\tmov.b64 b, {y, %3};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, pt;\n\t"
      "add.u32 x, %1, 16;\n\tadd.u32 y, %2, 512;\n\tmov.b64 b, {y, %3};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, pt;\n\t"
      "add.u32 x, %1, 24;\n\tadd.u32 y, %2, 768;\n\tmov.b64 b, {y, %3};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, pt;\n\t"
      "add.u32 x, %1, 32;\n\tadd.u32 y, %2, 1024;\n\tmov.b64 b, {y, %3};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, pt;\n\t"
      "add.u32 x, %1, 40;\n\tadd.u32 y, %2, 1280;\n\tmov.b64 b, {y, %3};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, pt;\n\t"
      "add.u32 x, %1, 48;\n\tadd.u32 y, %2, 1536;\n\tmov.b64 b, {y, %3};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, pt;\n\t"
      "add.u32 x, %1, 56;\n\tadd.u32 y, %2, 1792;\n\tmov.b64 b, {y, %3};\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %4, pt;\n\t"
      "@el tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%6];\n\t}\n" ::"r"(d),
      "r"(p), "r"(v), "r"(v_hi), "r"(idesc), "r"(accumulate), "r"(done)
      : "memory");
}

// A role's place in the pieces that the scheduler has laid out.
struct Pieces {
  uint32_t k;
  // The next one; false when there is none or the CTA has given up.  (All lanes of a warp.)
  template <class Wait>
  __device__ __forceinline__ bool next(Wait& await, const Bar& bar, const uint8_t* smem, uint32_t aborted, Piece& x) {
    const uint32_t slot = k % kPieces;
    if (!await(bar(B_PIECE + slot), (k / kPieces) & 1u, aborted)) return false;
    const int4* p = reinterpret_cast<const int4*>(smem + kOffPieces + slot * (kPieceInts * 4));
    int4* d = reinterpret_cast<int4*>(&x);
#pragma unroll
    for (int i = 0; i < kPieceInts / 4; ++i) d[i] = p[i];
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar(B_TAKEN + slot));
    ++k;
    return x.t0 < x.t1;
  }
};

// 32 bytes of a row: one store where the output is aligned to it (whole sectors at
// a time), else two.
__device__ __forceinline__ void st_global_32(uint16_t* p, const uint32_t* v, bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                 "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
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
    while (ok && pieces.next(await, bar, smem, aborted, x)) {
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
    while (ok && pieces.next(await, bar, smem, aborted, x)) {
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
      while (pieces.next(await, bar, smem, aborted, x)) {
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
      while (pieces.next(await, bar, smem, aborted, x)) {
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
      while (pieces.next(await, bar, smem, aborted, x)) {
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
      int64_t* start = reinterpret_cast<int64_t*>(smem + kOffPrefix);
      Walk walk;
      walk.start = start;
      walk.B = A.batch;
      walk.Hkv = A.kv.heads_kv;
      walk.R = 2 * npb;
      // Totals first: whether to cut units is chosen by them.
      struct Size {
        int64_t units, cost;
      };
      auto size_of = [&](const Seq& s) -> Size {  // a sequence's positions of both kinds
        const int64_t k = walk.groups_of(s.n);
        return {walk.Hkv * k, walk.Hkv * (k * (kUnitCost + s.L) + walk.R * k * (k + 1) / 2)};
      };
      auto scan = [&](int64_t v) -> int64_t {  // sum over the lanes up to this one
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int64_t y = __shfl_up_sync(0xffffffffu, v, off);
          if (lane >= off) v += y;
        }
        return v;
      };
      // A sequence a lane (of a large batch the last 32), and the totals.
      int64_t units = 0, cost = 0;
      int longest = 0;
      Seq own{0, 0, 0};
      walk.few = A.batch <= 32;
      for (int base = 0; base < A.batch; base += 32) {
        const int b = base + lane;
        own = Seq{0, 0, 0};
        if (b < A.batch) {
          int bad;
          own = sequence(A, b, &bad);
          if (bad && blockIdx.x == 0) flag(A.err, bad);
        }
        if (own.n > 0) longest = max(longest, own.L + own.n);
        units += size_of(own).units;
        cost += size_of(own).cost;
      }
      units = __shfl_sync(0xffffffffu, scan(units), 31);
      cost = __shfl_sync(0xffffffffu, scan(cost), 31);
      longest = __reduce_max_sync(0xffffffffu, longest);
      walk.P = (int)gridDim.x;
      // Which is faster, in positions.  Whole units end with the longest one if every CTA has
      // one at most.  In turn they end with an even share and, in the CTAs that end last,
      // half of the longest one.  Longest first they end with an even share, or with the
      // (k + 1)-th round of units as long as those that it starts with; some 3 % more.  Cut
      // units end with an even share, which the pieces' fixed costs upset by some 8 %, and
      // the joins.  Both ways, forced, us whole / cut, with whole : cut as estimated here:
      //   one prompt of 200, 32/8 heads  10.9 / 18.5 (0.41)   8 chunks of up to 1024  477 / 551 (0.93)
      //   one of 1024                    20.2 / 27.3 (0.73)   32 prompts up to 4096   801 / 884 (0.94)
      //   8 of 700, 28/4 heads           43.9 / 41.8 (0.81)   64 chunks of up to 300  636 / 702 (0.99)
      //   8 of 2048, 32/8 heads           208 / 223 (0.91)    single tokens of 256     202 / 189 (0.99)
      //   100 of up to 1500, 28/4 heads   523 / 578 (0.92)    of 64, 4000 keys each   86.9 / 92.6 (1.06)
      //   one of 16384, 64/8 heads       2687 / 2757 (0.95)   of 64, 500 to 16000      219 / 174 (1.34)
      // The wrong side is taken by up to 7 %, within some 20 % of the border.
      const float share = __fdividef((float)cost, (float)walk.P);
      const float cut = 1.08f * share + kJoinCost;
      float whole = (float)(longest + kUnitCost);
      walk.falling = walk.few && units > walk.P && cost >= units * kShortUnit && whole <= cut;
      walk.mine = own;
      walk.number_of_mine = lane;
      if (walk.falling) {
        // to each lane the sequence that comes lane-th
        const int length = own.n > 0 ? own.L + own.n : 0;
        int rank = 0, from = lane;
#pragma unroll 1
        for (int l = 0; l < 32; ++l) {
          const int o = __shfl_sync(0xffffffffu, length, l);
          rank += o > length || (o == length && l < lane);
        }
#pragma unroll 1
        for (int l = 0; l < 32; ++l)
          if (__shfl_sync(0xffffffffu, rank, l) == lane) from = l;
        walk.mine.r0 = __shfl_sync(0xffffffffu, own.r0, from);
        walk.mine.n = __shfl_sync(0xffffffffu, own.n, from);
        walk.mine.L = __shfl_sync(0xffffffffu, own.L, from);
        walk.number_of_mine = from;
        // the keys of the units that the rounds begin with, where the lane's sequence has them
        const int n = (int)size_of(walk.mine).units, first = (int)scan(n) - n;
        float most = fmaxf(whole, share);
#pragma unroll 1
        for (int r = 1; r < 4; ++r) {
          const int local = r * walk.P - first;
          if (local >= 0 && local < n) {
            const int rg = (n - 1 - local) / walk.Hkv;
            const int keys = walk.mine.L + min((rg + 1) * walk.R, walk.mine.n);
            most = fmaxf(most, (float)(r + 1) * (float)(keys + kUnitCost));
          }
        }
        whole = 1.03f * __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
      } else if (units > walk.P) {
        whole = share + 0.5f * whole;
      }
      walk.split = whole > cut;
      if (walk.split) {
        walk.falling = false;
        walk.mine = own;
        walk.number_of_mine = lane;
      }
      const int64_t run = walk.split ? cost : units;  // positions
      if (walk.few) {
        const Size z = size_of(walk.mine);
        const int64_t v = walk.split ? z.cost : z.units;
        walk.first_of_mine = scan(v) - v;
      } else {
        int64_t upto = 0;
        for (int base = 0; base < A.batch; base += 32) {
          const int b = base + lane;
          int64_t v = 0;
          if (b < A.batch) {
            int bad;
            const Size z = size_of(sequence(A, b, &bad));
            v = walk.split ? z.cost : z.units;
          }
          const int64_t to = scan(v);
          if (b < A.batch) start[b] = upto + to - v;
          upto += __shfl_sync(0xffffffffu, to, 31);
        }
        __syncwarp();
      }
      uint32_t k = 0;
      auto put = [&](const Piece& p) -> bool {
        const uint32_t slot = k % kPieces;
        if (!await(bar(B_TAKEN + slot), ((k / kPieces) & 1u) ^ 1u, aborted)) return false;
        ++k;
        if (lane == 0) {
          int4* d = reinterpret_cast<int4*>(smem + kOffPieces + slot * (kPieceInts * 4));
          const int4* v = reinterpret_cast<const int4*>(&p);
#pragma unroll
          for (int i = 0; i < kPieceInts / 4; ++i) d[i] = v[i];
          mbar_arrive(bar(B_PIECE + slot));
        }
        __syncwarp();
        return true;
      };
      // Whole units, every P-th; or longest first, the first ones by number and then in
      // chunks of `team` units for a team of neighbouring CTAs, each chunk to the team that
      // has the least to do by then: every CTA follows the same reckoning.  Neighbours take
      // units side by side (the same rows' other heads, the same head's other rows): SMs
      // close to each other get the same K and V tiles faster, 8 to 12 % of a tile's time.
      // 32 ragged prompts of 28/4 heads: 334 us so, 355 every P-th (the busiest CTA 15 %
      // above the mean); 64 prompts of 300: 105 so, 98 every P-th.
      const int c = (int)blockIdx.x, team = min(8, walk.P), teams = min(32, walk.P / team);
      uint32_t load = 0;  // of the lane's team, in tiles
      // the next chunk's first unit: head ch of the ck-th row group of the cs-th sequence
      int at = 0, cs = 0, ck = 0, ch = 0;
      int cL = __shfl_sync(0xffffffffu, walk.mine.L, 0), cn = __shfl_sync(0xffffffffu, walk.mine.n, 0);
      auto next_of_team = [&]() -> int64_t {  // the CTA's next unit after its first; `run`: none
        while (at < (int)run) {
          // tiles of the chunk's longest unit: its first, or the first of a sequence that
          // begins in it
          int groups = walk.groups_of(cn);
          int T = (cL + min((groups - ck) * walk.R, cn) + BN - 1) / BN;
          ck += team / walk.Hkv;
          ch += team % walk.Hkv;
          if (ch >= walk.Hkv) {
            ch -= walk.Hkv;
            ++ck;
          }
          while (ck >= groups && cs + 1 < A.batch) {
            ck -= groups;
            ++cs;
            cL = __shfl_sync(0xffffffffu, walk.mine.L, cs);
            cn = __shfl_sync(0xffffffffu, walk.mine.n, cs);
            groups = walk.groups_of(cn);
            if (groups > 0 && ck + ch > 0) T = max(T, (cL + cn + BN - 1) / BN);
          }
          const uint32_t least = __reduce_min_sync(0xffffffffu, lane < teams ? load * 32 + lane : 0xffffffffu);
          const int to = (int)(least & 31u), u = at + c % team;
          const bool first = at == to * team;
          if (lane == to) load += (uint32_t)T + 1;
          at += team;
          if (to == c / team && !first && u < (int)run) return u;
        }
        return run;
      };
      // every CTA that takes part in cut units has a tile of each unit that its range lies in
      if (walk.split) {
        if (share < (float)kMinShare) walk.P = max(1, (int)((float)run * (1.f / kMinShare)));
        walk.share = (int64_t)(__fdividef((float)run, (float)walk.P) * 0.999999f);
        walk.near = min((int64_t)kSnap, max((int64_t)1, (walk.share - kUnitCost) / 2));
      }
      // A CTA of cut units finds its range's end first, then takes the units inside the range
      // and the range's first and last piece, which may be parts of units.
      bool ending = walk.split && c < walk.P - 1, ok = true;
      int64_t g = walk.split ? (ending ? c + 1 : c) * walk.share : c;
      int64_t g_end = run, last = run;  // the range's end, and the unit that it ends in
      if (walk.split ? c >= walk.P : walk.falling && c >= teams * team) g = run;
      while (ok && g < run) {
        walk.seek(A, g);
        if (walk.split && g > 0) g = walk.border(g);
        if (ending) {
          g_end = g;
          last = walk.ustart;
          ending = false;
          g = c * walk.share;
          continue;
        }
        while (true) {
          x = walk.within(g, g_end);
          if (x.t0 < x.t1) ok = put(x);
          if (!walk.split || !ok || walk.ustart >= last || walk.ustart + walk.cost >= run) break;
          walk.advance(A);
        }
        g = walk.split ? run : walk.falling ? next_of_team() : g + walk.P;
      }
      x = Piece{};
      if (ok) put(x);  // the end
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
    for (int d = 0; d < *n_joins; ++d) {
      x = *reinterpret_cast<const Piece*>(smem + kOffPieces + (kPieces + d) * (kPieceInts * 4));
      __threadfence();
      // rows 0 .. v0 - 1 of M tile 0 and 0 .. v1 - 1 of M tile 1
      const int v0 = min(npb, x.n - 2 * x.rg * npb) * G, v1 = max(0, min(npb, x.n - (2 * x.rg + 1) * npb)) * G;
      const int rows8 = (v0 + v1 + 7) / 8;
      // A warp takes 8 rows and 4 * C of the 32 float4 columns, N parts' loads in flight:
      //   O = sum_p 2^(lse_p) O_p / sum_p 2^(lse_p), relative to the maximum so far
      auto join = [&](auto ctag, auto ntag) {
        constexpr int C = decltype(ctag)::value, N = decltype(ntag)::value;
        for (int task = warp; task < rows8 * (8 / C); task += kThreads / 32) {
          const int k = task / (8 / C) * 8 + (lane >> 2), c0 = task % (8 / C) * 4 * C + (lane & 3);
          if (k >= v0 + v1) continue;
          const int mt = k >= v0, rr = mt ? k - v0 : k;
          const int64_t at = mt * BM + rr;
          float4 acc[C];
#pragma unroll
          for (int j = 0; j < C; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
          float M = -INFINITY, wsum = 0.f;
          for (int p0 = 0; p0 < x.parts; p0 += N) {
            float w[N];
            float4 o[N][C];
#pragma unroll
            for (int p = 0; p < N; ++p) {
              if (p0 + p < x.parts) {
                const int64_t sl = 2 * (int64_t)(x.o0 + p0 + p) + (p0 + p == 0);
                w[p] = __ldcg(A.ws_lse + sl * (2 * BM) + at);
#pragma unroll
                for (int j = 0; j < C; ++j)
                  o[p][j] = __ldcg(reinterpret_cast<const float4*>(A.ws_o) + (sl * 32 + c0 + 4 * j) * (2 * BM) + at);
              } else {
                w[p] = -INFINITY;
#pragma unroll
                for (int j = 0; j < C; ++j) o[p][j] = make_float4(0.f, 0.f, 0.f, 0.f);
              }
            }
            float Mn = M;
#pragma unroll
            for (int p = 0; p < N; ++p) Mn = fmaxf(Mn, w[p]);
            const float a = ex2(M - Mn);
            M = Mn;
            wsum *= a;
#pragma unroll
            for (int j = 0; j < C; ++j) acc[j] = make_float4(acc[j].x * a, acc[j].y * a, acc[j].z * a, acc[j].w * a);
#pragma unroll
            for (int p = 0; p < N; ++p) {
              const float wp = ex2(w[p] - Mn);
              wsum += wp;
#pragma unroll
              for (int j = 0; j < C; ++j) {
                acc[j].x += wp * o[p][j].x;
                acc[j].y += wp * o[p][j].y;
                acc[j].z += wp * o[p][j].z;
                acc[j].w += wp * o[p][j].w;
              }
            }
          }
          const float winv = 1.f / wsum;
          uint16_t* orow =
              A.out + ((int64_t)(x.r0 + (2 * x.rg + mt) * npb + rr / G) * A.heads_q + x.h * G + rr % G) * D;
#pragma unroll
          for (int j = 0; j < C; ++j)
            *reinterpret_cast<uint2*>(orow + (c0 + 4 * j) * 4) =
                make_uint2(pack_bf16(acc[j].x * winv, acc[j].y * winv), pack_bf16(acc[j].z * winv, acc[j].w * winv));
        }
      };
      if (rows8 >= 8) join(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
      else join(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
    }
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
