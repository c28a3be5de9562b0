// What the causal attention kernels over the cache share (k_prompt.cu: a bf16 cache;
// k_prompt8.cu: one in 8 bits): how a call's work is cut into pieces and dealt out, the
// roles' waits, the PV products, and the joining of units that were cut.
//
// A unit is (sequence, row group, kv head): 2 * npb rows' heads of one kv head, packed
// (row, group head) into two M tiles of 128 (npb = 128 / G rows each), against its keys
// in 128-key tiles.  A piece is the tiles of a unit that one CTA takes.
#pragma once

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "attn_tc.cuh"

namespace cure {
namespace prompt {

using namespace tc;

constexpr int BM = kAttnRowsCta;  // 128 rows per M tile
constexpr int BN = 128;           // keys per tile
constexpr int D = kAttnD;
constexpr int kThreads = 512;
constexpr uint32_t kTmemCols = 512;
constexpr int kPieces = 4;        // pieces that the scheduler may be ahead
constexpr int kTakers = 15;       // warps that take pieces: all but the scheduler
constexpr int kPieceInts = 12;

constexpr int kQHalf = kAttnQHalf;      // 16 KiB: [128 rows][128 bytes]
constexpr int kVChunk = kAttnVChunk;    // 4 KiB: V keys 16c..16c+15, both d halves
constexpr int kVHalf = kVChunk / 2;

constexpr uint32_t kColS = 0;    // S:    columns 0 .. 127
constexpr uint32_t kColP = 128;  // P[m]: columns 128 + m*64
constexpr uint32_t kColO = 256;  // O[m]: columns 256 + m*128

struct PromptArgs {
  static constexpr bool kTree = false;  // rows see the keys up to their own
  static constexpr int kUnitCost = 2 * BN;  // what a unit's start and end cost (below)
  static constexpr float kAloneTail = 0.f;  // > 0: warps may take units of their own, and how much slower (schedule)
  static constexpr float kSpread = 0.f;     // what unlike lengths add to units dealt out in turn (schedule)
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

// Positions.  Every unit takes Args::kUnitCost positions (what starting and ending a
// piece costs, in a kernel's key times) and then one for each key of the last row that its
// row group could have; tile t of it stands at the position of its first key.
// What joining the parts of units costs a call (7 to 8 us: a prompt of 200 or 1024 cut
// needlessly), and the fewest positions worth a CTA.
constexpr int kJoinCost = 8 * BN;
constexpr int kMinShare = 3 * BN;
// Units of fewer positions on average, and those of a batch of more than 32, are
// dealt out in turn: the reckoning that evens them out would take longer than they do.
constexpr int kShortUnit = 7 * BN;
// A share's border that lies nearer to a unit's border than this moves there.
constexpr int kSnap = 4 * BN;

// A sequence's rows and the tokens before them; n = 0 where they do not make sense.
struct Seq {
  int r0, n, L;
};
template <class Args>
__device__ __forceinline__ Seq sequence(const Args& A, int b, int* bad) {
  Seq s;
  s.L = A.cache_len[b];
  int64_t n;
  *bad = 0;
  if constexpr (Args::kTree) {
    s.r0 = b * A.n_max;
    n = A.n_nodes[b];
    if (n < 1 || n > A.n_max) *bad = CURE_DEVERR_NODES;
  } else {
    s.r0 = A.row_start[b];
    n = (int64_t)A.row_start[b + 1] - s.r0;
    if (s.r0 < 0 || n < 0 || s.r0 + n > A.rows) *bad = CURE_DEVERR_NODES;
  }
  s.n = (int)n;
  if (!*bad && n > 0 && (s.L < 0 || s.L + n > A.cap)) *bad = CURE_DEVERR_SLOT;
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
template <class Args>
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
  // (a tree's row groups all see its last node)
  __device__ __forceinline__ int base() const { return split ? Args::kUnitCost + s.L + (Args::kTree ? groups * R : 0) : 1; }
  __device__ __forceinline__ int step() const { return split && !Args::kTree ? R : 0; }
  __device__ __forceinline__ int64_t before(int k) const {  // a head's positions in front of the k-th row group
    return k * (int64_t)base() + (int64_t)step() * k * (k + 1) / 2;
  }
  __device__ __forceinline__ int owner(int64_t p) const { return small_quotient(p, share, P - 1); }
  __device__ __forceinline__ void load(const Args& A) {
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
  __device__ __forceinline__ void seek(const Args& A, int64_t g) {  // the unit that holds position g
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
  __device__ __forceinline__ void advance(const Args& A) {  // to the next unit (there is one)
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
  __device__ __forceinline__ int keys() const { return s.L + (Args::kTree ? s.n : min((row_group() + 1) * R, s.n)); }
  __device__ __forceinline__ int tiles() const { return (keys() + BN - 1) / BN; }
  // Where the border p of a share, which lies in this unit, is drawn: at one of the
  // unit's borders if that is near (or if one side would be left without a tile).
  __device__ __forceinline__ int64_t border(int64_t p) const {
    const int64_t first = ustart + Args::kUnitCost;
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
      const int64_t first = ustart + Args::kUnitCost;  // tile 0's position
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
  template <class LAY, class Wait>
  __device__ __forceinline__ bool next(Wait& await, const Bar& bar, const uint8_t* smem, uint32_t aborted, Piece& x) {
    const uint32_t slot = k % kPieces;
    if (!await(bar(LAY::piece_bar + slot), (k / kPieces) & 1u, aborted)) return false;
    const int4* p = reinterpret_cast<const int4*>(smem + LAY::pieces + slot * (kPieceInts * 4));
    int4* d = reinterpret_cast<int4*>(&x);
#pragma unroll
    for (int i = 0; i < kPieceInts / 4; ++i) d[i] = p[i];
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar(LAY::taken_bar + slot));
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

// The scheduler warp: lays out the CTA's pieces of work, up to kPieces ahead.  LAY: where
// the kernel's shared memory and barriers hold them.
template <class LAY, class Args, class Wait>
__device__ __forceinline__ void schedule(const Args& A, int npb, Wait& await, const Bar& bar, uint8_t* smem,
                                         uint32_t aborted, int lane) {
  Piece x;
  int64_t* start = reinterpret_cast<int64_t*>(smem + LAY::prefix);
  Walk<Args> walk;
  walk.start = start;
  walk.B = A.batch;
  walk.Hkv = A.kv.heads_kv;
  walk.R = LAY::m_tiles * npb;
  // Totals first: whether to cut units is chosen by them.
  struct Size {
    int64_t units, cost;
  };
  auto size_of = [&](const Seq& s) -> Size {  // a sequence's positions of both kinds
    const int64_t k = walk.groups_of(s.n);
    return {walk.Hkv * k, walk.Hkv * (k * (Args::kUnitCost + s.L) + walk.R * (Args::kTree ? k * k : k * (k + 1) / 2))};
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
  float whole = (float)(longest + Args::kUnitCost);
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
        most = fmaxf(most, (float)(r + 1) * (float)(keys + Args::kUnitCost));
      }
    }
    whole = 1.03f * __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
  } else if (units > walk.P) {
    // (unlike lengths add up to unlike sums of units / P of them)
    const float over = whole - __fdividef((float)cost, (float)units);
    whole = share + 0.5f * whole;
    if constexpr (Args::kSpread > 0)
      whole += Args::kSpread * fmaxf(0.f, over) * sqrt_approx(__fdividef((float)units, (float)walk.P));
  }
  walk.split = whole > cut;
  // Units of a warp each, where that is faster: they start and end under each other's copies, and at the call's
  // end the last ones go on at a warp's pace.
  bool alone = false;
  if constexpr (Args::kAloneTail > 0)
    if (!walk.few && longest <= 1 << 22) {  // (a warp's unit of so many keys stays well within the waits' limit)
      const float keys = (float)(cost - units * (Args::kUnitCost - BN));
      alone = __fdividef(keys, (float)walk.P) + Args::kAloneTail * (float)longest < fminf(whole, cut);
      if (alone) walk.split = false;
    }
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
    if (!await(bar(LAY::taken_bar + slot), ((k / kPieces) & 1u) ^ 1u, aborted)) return false;
    ++k;
    if (lane == 0) {
      int4* d = reinterpret_cast<int4*>(smem + LAY::pieces + slot * (kPieceInts * 4));
      const int4* v = reinterpret_cast<const int4*>(&p);
#pragma unroll
      for (int i = 0; i < kPieceInts / 4; ++i) d[i] = v[i];
      mbar_arrive(bar(LAY::piece_bar + slot));
    }
    __syncwarp();
    return true;
  };
  if constexpr (Args::kAloneTail > 0)
    if (alone) {
      if (lane == 0) *reinterpret_cast<volatile int*>(smem + LAY::mode) = 1;
      // the units of LAY::alone warps, a unit a lane
      bool some = true;
      for (int64_t base = 0; some; base += (int64_t)LAY::alone * walk.P) {
        const int64_t u = base + (int64_t)lane * walk.P + blockIdx.x;
        some = base + blockIdx.x < units;  // (behind the last: the end)
        Piece own_piece = Piece{};
        if (lane < LAY::alone && u < units) {
          walk.seek(A, u);
          own_piece = walk.within(0, units);
        }
        const uint32_t slot = k % kPieces;
        if (!await(bar(LAY::taken_bar + slot), ((k / kPieces) & 1u) ^ 1u, aborted)) return;
        ++k;
        if (lane < LAY::alone) *(reinterpret_cast<Piece*>(smem + LAY::own) + slot * LAY::alone + lane) = own_piece;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(LAY::piece_bar + slot));
      }
      return;
    }
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
    walk.near = min((int64_t)kSnap, max((int64_t)1, (walk.share - Args::kUnitCost) / 2));
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

// Joins the units whose last part came from this CTA: all warps, with equal registers.
template <class LAY, class Args>
__device__ __forceinline__ void join_units(const Args& A, int npb, const uint8_t* smem, int n_joins, int warp, int lane) {
  const int G = A.G;
  Piece x;
  for (int d = 0; d < n_joins; ++d) {
    x = *reinterpret_cast<const Piece*>(smem + LAY::pieces + (kPieces + d) * (kPieceInts * 4));
    __threadfence();
    // rows 0 .. v0 - 1 of M tile 0 and 0 .. v1 - 1 of M tile 1
    const int v0 = min(npb, x.n - LAY::m_tiles * x.rg * npb) * G,
              v1 = LAY::m_tiles == 1 ? 0 : max(0, min(npb, x.n - (2 * x.rg + 1) * npb)) * G;
    const int rows8 = (v0 + v1 + 7) / 8;
    // A warp takes 8 rows and 4 * C of the 32 float4 columns, N parts' loads in flight:
    //   O = sum_p 2^(lse_p) O_p / sum_p 2^(lse_p), relative to the maximum so far
    auto join = [&](auto ctag, auto ntag) {
      constexpr int C = decltype(ctag)::value, N = decltype(ntag)::value;
      for (int task = warp; task < rows8 * (8 / C); task += LAY::threads / 32) {
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
            A.out + ((int64_t)(x.r0 + (LAY::m_tiles * x.rg + mt) * npb + rr / G) * A.heads_q + x.h * G + rr % G) * D;
#pragma unroll
        for (int j = 0; j < C; ++j)
          *reinterpret_cast<uint2*>(orow + (c0 + 4 * j) * 4) =
              make_uint2(pack_bf16(acc[j].x * winv, acc[j].y * winv), pack_bf16(acc[j].z * winv, acc[j].w * winv));
      }
    };
    if (rows8 >= 8) join(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
    else join(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());
  }
  __syncwarp();  // (what comes next is aligned: TMEM is given back)
}

}  // namespace prompt
}  // namespace cure
