// K and V rows into a cache held in 8 bits (e4m3 codes, a scale for each block of 16 slots
// and head): cure_append_kv8, from the rows of a layer's projection, and the accepted
// path's rows of every layer (cure_resync_kv8).
//
//   s = 2^e, the least with max |x| <= 448 s over what the block then holds
//   code = e4m3(x / s)
//
// With a power of two x / s is exact, and a held value that is expressed anew under another
// scale keeps its digits, as e4m3 is a floating type: only what falls below its normal
// range (2^-6 s) is rounded again.
//
// Layout.  A CTA takes the blocks that begin in its range of packed rows (a block's rows in
// one call are neighbours).  Each of its 16 half warps has one slot of a block for all heads, 8 values a
// lane: a row of the call, with the row's cosines and sines in registers, or one that the block
// holds already.  Two or four heads of K and V at a time are loaded, normed and turned, and their rows'
// largest values meet in shared memory; behind the barrier each half warp writes its codes, while the next
// heads' values are on their way.  Heads of Q go the same way without meeting; where a block gains few
// rows, all half warps share those rows' heads.
//
// Bound: latency.  A block is a chain of look-ups (sequence, length, page: 2.5 us), its rows' angles, and
// a meeting of 1 to 1.5 us for each group of heads.  Single tokens of 200 sequences (32 and 8 heads): 12.5 us;
// 19241 rows in 32 chunks behind cached ones (28 and 4 heads, norms, three axes): 91 us, 3.7 TB/s, of which
// finding the places takes 20 us, K and V 40 and Q 45 when left out in turn.  A head a warp with its 16 rows
// in registers took 143 us there (100 KB of code), rows staged in shared memory 117, Q in a launch of its own
// 116.  The accepted paths' rows (a block's four heads of one layer at a time, no rotation): 32 paths in 28
// layers 19 us with the lengths' launch.
#include <algorithm>

#include "rope_math.cuh"

namespace cure {
namespace {

using rope::hi_f;
using rope::lo_f;
using rope::Raw;

constexpr int kThreads = 256;
constexpr int kD = 128;
constexpr int kBlk = CURE_KV8_BLOCK;
static_assert(kBlk == 16, "a half warp a slot, 16 lanes a row");

// Four values as codes (ties to even; beyond 448: 448; NaN stays one), and back.
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}\n"
      : "=r"(r)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ void from_codes(uint32_t w, float* y) {
  uint32_t a, b;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "mov.b32 {lo, hi}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, lo;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, hi;\n\t}\n"
      : "=r"(a), "=r"(b)
      : "r"(w));
  const float2 p = __half22float2(*reinterpret_cast<__half2*>(&a)), q = __half22float2(*reinterpret_cast<__half2*>(&b));
  y[0] = p.x;
  y[1] = p.y;
  y[2] = q.x;
  y[3] = q.y;
}

// The exponent of a block's scale: the least e from -40 to 40 with amax <= 448 * 2^e
// (448 = 1.75 * 2^8).
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return min(max(e, -40), 40);
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Where a lane's 8 values lie in a head, as two runs of 4: in the half layout the first
// and second values of its four pairs, else 8 values on end (interleaved, or not rotated).
struct Lane {
  int off_a, off_b;
  bool rot;
};
template <bool INTER>
__device__ __forceinline__ Lane lane_of(int l16, int rot_dim) {
  const int r8 = rot_dim >> 3;
  Lane p;
  p.rot = l16 < r8;
  p.off_a = INTER ? 8 * l16 : p.rot ? 4 * l16 : 8 * l16;
  p.off_b = INTER ? 8 * l16 + 4 : p.rot ? 4 * l16 + 4 * r8 : 8 * l16 + 4;
  return p;
}

__device__ __forceinline__ Raw load_raw(const uint16_t* row, const Lane& p) {
  Raw x;
  x.a = *reinterpret_cast<const uint2*>(row + p.off_a);
  x.b = *reinterpret_cast<const uint2*>(row + p.off_b);
  return x;
}
// y[0..3] the values at off_a, y[4..7] those at off_b.
__device__ __forceinline__ void widen(const Raw& x, float* y) {
  y[0] = lo_f(x.a.x);
  y[1] = hi_f(x.a.x);
  y[2] = lo_f(x.a.y);
  y[3] = hi_f(x.a.y);
  y[4] = lo_f(x.b.x);
  y[5] = hi_f(x.b.x);
  y[6] = lo_f(x.b.y);
  y[7] = hi_f(x.b.y);
}

// The rotation (and, before it, the head norm: weights w times the row's factor rs) of a lane's
// values by its four pairs' cosines and sines.
template <bool INTER>
__device__ __forceinline__ void norm_rotate(float* y, const float* w, bool norm, float rs, const float* c, const float* sn,
                                            bool rot) {
  if (norm) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = y[e] * rs * w[e];
  }
  if (rot) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = INTER ? 2 * e : e, j = INTER ? 2 * e + 1 : e + 4;
      const float a = y[i], b = y[j];
      y[i] = fmaf(-b, sn[e], a * c[e]);
      y[j] = fmaf(a, sn[e], b * c[e]);
    }
  }
}
// The norm's factor of a row that half a warp holds.
__device__ __forceinline__ float norm_factor(const float* y, float eps) {
  float ss = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  return rsqrtf(ss * (1.f / kD) + eps);
}

constexpr int kHeadsP = 4;  // of K and V between two barriers: in the commit

// What a half warp has in the slot of its block.
enum Slot { kNone, kHeld, kFresh };

// N heads of a block's K or V, all threads of the CTA: y the rows' values (kNone: any), `codes` each
// head's codes of the half warp's slot (NULL: no head), `scale` its place.
template <int N>
__device__ __forceinline__ void quantise(float (&y)[N][8], Slot what, uint8_t* const (&codes)[N],
                                         float* const (&scale)[N], const float (&old)[N], const Lane& p,
                                         uint32_t (*part)[kThreads / 32]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(y[u][e]));  // (a NaN counts for nothing)
    // of both half warps' slots; as integers, which are ordered as the values are
    const uint32_t top = __reduce_max_sync(0xffffffffu, what == kNone ? 0u : __float_as_uint(amax));
    if (lane == 0) part[u][warp] = top;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < N; ++u) {
    if (!codes[u]) break;
    const uint4 p0 = reinterpret_cast<const uint4*>(part[u])[0], p1 = reinterpret_cast<const uint4*>(part[u])[1];
    const uint32_t top = max(max(max(p0.x, p0.y), max(p0.z, p0.w)), max(max(p1.x, p1.y), max(p1.z, p1.w)));
    const int e = scale_exponent(__uint_as_float(top));
    const float s = power(e), inv = power(-e);
    if (what == kFresh || (what == kHeld && s != old[u])) {  // (what is held stays as it is under the same scale)
      *reinterpret_cast<uint32_t*>(codes[u] + p.off_a) =
          to_codes(y[u][0] * inv, y[u][1] * inv, y[u][2] * inv, y[u][3] * inv);
      *reinterpret_cast<uint32_t*>(codes[u] + p.off_b) =
          to_codes(y[u][4] * inv, y[u][5] * inv, y[u][6] * inv, y[u][7] * inv);
    }
    if (threadIdx.x == 0) *scale[u] = s;
  }
}

// A half warp's values of a head as they lie: a row's, or the block's codes.
__device__ __forceinline__ Raw load_slot(Slot what, const uint16_t* row, const uint8_t* codes, const Lane& p) {
  Raw x;
  x.a = x.b = make_uint2(0u, 0u);
  if (what == kFresh) x = load_raw(row, p);
  if (what == kHeld) {
    x.a.x = *reinterpret_cast<const uint32_t*>(codes + p.off_a);
    x.a.y = *reinterpret_cast<const uint32_t*>(codes + p.off_b);
  }
  return x;
}
__device__ __forceinline__ void value_of(const Raw& x, Slot what, float old, float* y) {
  if (what == kHeld) {
    from_codes(x.a.x, y);
    from_codes(x.a.y, y + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= old;
  } else {
    widen(x, y);
  }
}

// The page of a block of 16 slots, or the sequence's own range: the row of its slot 0 in the
// cache and its place among the scales; false where there is none.
__device__ __forceinline__ bool place_of(const cure_kv_desc& kv, int seq, int blk, int64_t* row, int64_t* place) {
  if (kv.layout == 0) {
    *row = (int64_t)seq * kv.max_len + (int64_t)blk * kBlk;
    *place = (int64_t)seq * ((kv.max_len + kBlk - 1) / kBlk) + blk;
    return true;
  }
  const int per = kv.page_size / kBlk;
  const int page = kv.block_table[(int64_t)seq * kv.max_len + blk / per];
  if (page < 0 || page >= kv.num_pages) return false;
  *place = (int64_t)page * per + blk % per;
  *row = *place * kBlk;
  return true;
}

struct Append8Args {
  RopeArgs r;
  float *k_scale, *v_scale;
  int range;  // packed rows whose blocks a CTA takes
};

// CTAs to an SM, with kHeads heads of K or V between two barriers.
constexpr int resident(int kHeads) { return kHeads == 2 ? 3 : 2; }

template <bool INTER, int kHeads>
__global__ void __launch_bounds__(kThreads, resident(kHeads))
append8_kernel(const __grid_constant__ Append8Args G) {
  const RopeArgs& A = G.r;
  __shared__ uint64_t turns[64];
  __shared__ __align__(16) uint32_t part[2][kHeads][kThreads / 32];
  if (threadIdx.x < 64) turns[threadIdx.x] = A.rope.turns[threadIdx.x];
  __syncthreads();
  pdl_begin();
  const int tid = threadIdx.x, lane = tid & 31, l16 = lane & 15, hw = tid >> 4;
  const int Hq = A.heads_q, Hkv = A.heads_kv;
  const int first = blockIdx.x * G.range;
  const int end = min(first + G.range, A.rows);
  const Lane turned = lane_of<INTER>(l16, A.rope.rot_dim), plain = lane_of<true>(l16, 0);
  const int n_axes = A.axes.axes;
  const int64_t cap = A.kv.layout == 0 ? A.kv.max_len : (int64_t)A.kv.max_len * A.kv.page_size;
  const bool tell = tid == 0 && blockIdx.y == 0;
  int buf = 0;

  for (int row = first; row < end;) {
    // The row's sequence: as many of the ends row_start[1..B] are at or before it.  Its first row, the
    // row behind its last and its length come along with the search.
    int seq = 0, start = A.row_start[0], stop = A.rows, L = 0;
    for (int base = 0; base < A.batch; base += 256) {
      int e[8], len[8], n = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int b = base + 32 * i + lane;
        e[i] = b < A.batch ? A.row_start[b + 1] : INT32_MAX;
        len[i] = b < A.batch ? A.cache_len[b] : 0;
      }
      const int last = base + 256 < A.batch ? __shfl_sync(0xffffffffu, e[7], 31) : INT32_MAX;
      if (last <= row) {  // (ascending: all of these are)
        seq += 256;
        start = last;
        continue;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) n += __popc(__ballot_sync(0xffffffffu, e[i] <= row));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (n > 0 && (n - 1) / 32 == i) start = __shfl_sync(0xffffffffu, e[i], (n - 1) & 31);
        if (n / 32 == i) {
          stop = min(stop, __shfl_sync(0xffffffffu, e[i], n & 31));
          L = __shfl_sync(0xffffffffu, len[i], n & 31);
        }
      }
      seq += n;
      break;
    }
    if (seq >= A.batch) return;  // behind the last sequence
    const int i = row - start;
    if (i < 0 || start < 0 || row >= stop) {  // before the first sequence, or row_start does not ascend
      if ((seq > 0 || i >= 0) && tell) flag(A.err, CURE_DEVERR_NODES);
      ++row;
      continue;
    }
    const int64_t slot = (int64_t)L + i;
    if (slot < 0 || slot >= cap) {
      bool none = false;  // a row that holds no token needs no slot
      for (int a = 0; A.pos && a < max(1, n_axes); ++a) none |= A.pos[(int64_t)a * A.rows + row] < 0;
      if (tell && !none) flag(A.err, CURE_DEVERR_SLOT);
      ++row;
      continue;
    }
    const int blk = (int)(slot / kBlk), t0 = (int)(slot % kBlk);
    const int m = (int)min((int64_t)min(kBlk - t0, stop - row), cap - slot);  // the block's rows from here on
    if (i > 0 && t0 > 0) {  // it begins before this row: its CTA takes it (but not what lies past the capacity)
      row += m;
      continue;
    }
    const int row0 = row;
    row += m;
    int64_t crow = 0, place = 0;
    const bool there = place_of(A.kv, seq, blk, &crow, &place);

    // Half warps 0 .. m - 1 have the rows, the last t0 what the block holds; for Q row r = hw % m.
    const int r = hw % m, t = (t0 + hw) & (kBlk - 1);
    int p = (int)(slot + r);
    bool none = false;  // row r holds no token
    if (n_axes > 0) {
      // lane a: the position on axis a
      p = l16 < n_axes ? A.pos[(int64_t)l16 * A.rows + row0 + r] : 0;
      none = __ballot_sync(0xffffffffu, p < 0) >> (lane & 16) & 0xffffu;
    } else if (A.pos) {
      p = A.pos[row0 + r];
      none = p < 0;
    }
    const Slot what = hw < m ? (none ? kNone : kFresh) : t < t0 && i == 0 ? kHeld : kNone;
    if (!__syncthreads_or(what == kFresh)) continue;  // (also: the block before is done with `part`)
    if (!there) {
      if (tell) flag(A.err, CURE_DEVERR_PAGE);
      continue;
    }

    // cosines and sines of the lane's pairs
    float c[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
    int at[4] = {p, p, p, p};
    if (n_axes > 0) {
      const uint32_t axis = reinterpret_cast<const uint32_t*>(A.axes.axis)[l16];
#pragma unroll
      for (int e = 0; e < 4; ++e) at[e] = __shfl_sync(0xffffffffu, p, (lane & 16) | ((axis >> (8 * e)) & 7u));
    }
    if (turned.rot) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // the fraction of a turn in 2^-32, as a signed number of half turns
        const int32_t f = (int32_t)(uint32_t)(((uint64_t)(uint32_t)at[e] * turns[4 * l16 + e]) >> 32);
        sincospif((float)f * 0x1p-31f, &sn[e], &c[e]);
        c[e] *= A.rope.amplitude;
        sn[e] *= A.rope.amplitude;
      }
    }

    // ---- heads of K, then of V
    const int64_t ld = (int64_t)Hkv * kD, at_slot = (crow + t) * ld;
    float w[8];
    if (A.k_norm) widen(load_raw(A.k_norm, turned), w);
    const int groups = (Hkv + kHeads - 1) / kHeads;  // of K, and of V; the next one's values are on their way
    Raw x[kHeads];
    float old[kHeads];
    auto load = [&](int g) {
      const bool kv = g >= groups;
      const int h = (kv ? g - groups : g) * kHeads;
      const uint16_t* in = kv ? A.v + (row0 + hw) * A.ld_v : A.k + (row0 + hw) * A.ld_k;
      const uint8_t* codes = reinterpret_cast<const uint8_t*>(kv ? A.v_out : A.k_out) + at_slot;
      const float* scales = (kv ? G.v_scale : G.k_scale) + place * Hkv;
      const Lane lp = kv ? plain : turned;
#pragma unroll
      for (int u = 0; u < kHeads; ++u) {
        const bool is = g < 2 * groups && h + u < Hkv;
        x[u] = load_slot(is ? what : kNone, in + (h + u) * kD, codes + (h + u) * kD, lp);
        old[u] = is && t0 > 0 ? scales[h + u] : 1.f;
      }
    };
    load(blockIdx.y);
#pragma unroll 1
    for (int g = blockIdx.y; g < 2 * groups; g += gridDim.y) {
      const bool kv = g >= groups;
      const int h = (kv ? g - groups : g) * kHeads;
      const Lane lp = kv ? plain : turned;
      uint8_t* base = reinterpret_cast<uint8_t*>(kv ? A.v_out : A.k_out) + at_slot;
      float* scales = (kv ? G.v_scale : G.k_scale) + place * Hkv;
      float y[kHeads][8], was[kHeads];
      uint8_t* codes[kHeads];
      float* scale[kHeads];
#pragma unroll
      for (int u = 0; u < kHeads; ++u) {
        codes[u] = h + u < Hkv ? base + (h + u) * kD : nullptr;
        scale[u] = scales + h + u;
        was[u] = old[u];
        value_of(x[u], what, was[u], y[u]);
      }
      load(g + gridDim.y);
      if (!kv) {
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
          const float rs = A.k_norm ? norm_factor(y[u], A.eps) : 1.f;  // (all lanes, whatever they have)
          if (what == kFresh) norm_rotate<INTER>(y[u], w, A.k_norm != nullptr, rs, c, sn, lp.rot);
        }
      }
      quantise(y, what, codes, scale, was, lp, part[buf]);
      buf ^= 1;
    }

    // ---- heads of Q: half warp hw those of row hw % m from the (hw / m)-th on
    if (A.q) {
      const int shares = kBlk / m, parts = gridDim.y * shares;
      if (A.q_norm) widen(load_raw(A.q_norm, turned), w);
      const uint16_t* in = A.q + (int64_t)(row0 + r) * A.ld_q;
      uint16_t* out = A.q_out + (int64_t)(row0 + r) * A.ld_q_out;
      const bool mine = hw < m * shares && !none;
      constexpr int U = 4;
      Raw x[U];
      auto load = [&](int h0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = h0 + u * parts + blockIdx.y * shares + hw / m;
          x[u] = load_slot(mine && h < Hq ? kFresh : kNone, in + h * kD, nullptr, turned);
        }
      };
      load(0);
      for (int h0 = 0; h0 < Hq; h0 += U * parts) {
        Raw now[U];
#pragma unroll
        for (int u = 0; u < U; ++u) now[u] = x[u];
        load(h0 + U * parts);  // (none behind the last)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = h0 + u * parts + blockIdx.y * shares + hw / m;
          float y[8];
          widen(now[u], y);
          const float rs = A.q_norm ? norm_factor(y, A.eps) : 1.f;
          norm_rotate<INTER>(y, w, A.q_norm != nullptr, rs, c, sn, turned.rot);
          if (mine && h < Hq) {
            *reinterpret_cast<uint2*>(out + h * kD + turned.off_a) =
                make_uint2(tc::pack_bf16(y[0], y[1]), tc::pack_bf16(y[2], y[3]));
            *reinterpret_cast<uint2*>(out + h * kD + turned.off_b) =
                make_uint2(tc::pack_bf16(y[4], y[5]), tc::pack_bf16(y[6], y[7]));
          }
        }
      }
    }
  }
}

struct Paths8Args {
  LayerPtrs caches;
  LayerScales scales;
  cure_kv_desc kv;
  const uint16_t *tree_k, *tree_v;
  int layers, batch, n_max, block;
  const int32_t *path_nodes, *accept_len, *cache_len;
  int* err;
};

// The k-th block that sequence b's accepted path reaches (blockIdx.x = b * blocks + k).
__global__ void __launch_bounds__(kThreads, 3)
paths8_kernel(const __grid_constant__ Paths8Args A) {
  __shared__ __align__(16) uint32_t part[2][kHeadsP][kThreads / 32];
  pdl_begin();
  const int tid = threadIdx.x, l16 = tid & 15, hw = tid >> 4;
  const int blocks = (A.block + 1 + kBlk - 2) / kBlk + 1;
  const int b = blockIdx.x / blocks, k = blockIdx.x % blocks;
  const int Hkv = A.kv.heads_kv, P = A.block + 2;
  const int n = min(A.accept_len[b], A.block) + 1;  // rows of the path
  const int L = A.cache_len[b];
  const bool tell = tid == 0 && blockIdx.y == 0;
  const int64_t cap = A.kv.layout == 0 ? A.kv.max_len : (int64_t)A.kv.max_len * A.kv.page_size;
  if (n < 1) return;
  if (L < 0 || (int64_t)L + n > cap) {
    if (tell && k == 0) flag(A.err, CURE_DEVERR_SLOT);
    if (L < 0) return;
  }
  const int blk = L / kBlk + k;
  const int64_t slot0 = (int64_t)blk * kBlk;
  const int from = (int)max((int64_t)0, L - slot0);  // slots of the block that are held, or come before its rows
  const int to = (int)min((int64_t)kBlk, min((int64_t)L + n, cap) - slot0);
  if (from >= to) return;
  int64_t crow, place;
  if (!place_of(A.kv, b, blk, &crow, &place)) {
    if (tell) flag(A.err, CURE_DEVERR_PAGE);
    return;
  }
  Slot what = hw < from ? kHeld : kNone;
  int node = 0;
  if (hw >= from && hw < to) {
    node = A.path_nodes[(int64_t)b * P + (int)(slot0 + hw - L)];
    if (node >= 0 && node < A.n_max) what = kFresh;
    else if (l16 == 0 && blockIdx.y == 0) flag(A.err, CURE_DEVERR_NODES);
  }
  if (!__syncthreads_or(what == kFresh)) return;
  const Lane plain = lane_of<true>(l16, 0);
  const int64_t ld = (int64_t)Hkv * kD, at_slot = (crow + hw) * ld;
  const int groups = (Hkv + kHeadsP - 1) / kHeadsP;
  int buf = 0;
  for (int item = blockIdx.y; item < A.layers * 2 * groups; item += gridDim.y) {
    const int l = item / (2 * groups), kv = item / groups & 1, h = item % groups * kHeadsP;
    const uint16_t* in = (kv ? A.tree_v : A.tree_k) + (((int64_t)l * A.batch + b) * A.n_max + node) * ld;
    uint8_t* base = static_cast<uint8_t*>(kv ? A.caches.v[l] : A.caches.k[l]) + at_slot;
    float* scales = (kv ? A.scales.v[l] : A.scales.k[l]) + place * Hkv;
    Raw x[kHeadsP];
    float old[kHeadsP], y[kHeadsP][8];
    uint8_t* codes[kHeadsP];
    float* scale[kHeadsP];
#pragma unroll
    for (int u = 0; u < kHeadsP; ++u) {
      const bool is = h + u < Hkv;
      codes[u] = is ? base + (h + u) * kD : nullptr;
      scale[u] = scales + h + u;
      x[u] = load_slot(is ? what : kNone, in + (h + u) * kD, codes[u], plain);
      old[u] = is && from > 0 ? *scale[u] : 1.f;
    }
#pragma unroll
    for (int u = 0; u < kHeadsP; ++u) value_of(x[u], what, old[u], y[u]);
    quantise(y, what, codes, scale, old, plain, part[buf]);
    buf ^= 1;
  }
}

struct HeldArgs {
  LayerPtrs caches;
  LayerScales scales;
  cure_kv_desc kv;
  const int32_t* cache_len;
  uint8_t* saved;  // codes [layer][K, V][sequence][16 slots][heads][128], then scales [layer][K, V][sequence][heads]
  int layers, batch;
};

// What sequence blockIdx.x holds of the block that the next row behind it would share (none where its length is a
// multiple of 16), with the block's scales: of every layer's K and V out of the caches, or back.  A block's slots lie
// end to end in either layout.  28 layers of 32 sequences, 4 heads: 7 MB each way, 5 us.
template <bool SAVE>
__global__ void __launch_bounds__(kThreads)
held8_kernel(const __grid_constant__ HeldArgs A) {
  pdl_begin();
  const int b = blockIdx.x, L = A.cache_len[b], Hkv = A.kv.heads_kv;
  const int64_t cap = A.kv.layout == 0 ? A.kv.max_len : (int64_t)A.kv.max_len * A.kv.page_size;
  if (L <= 0 || L % kBlk == 0 || L > cap) return;
  int64_t row, place;
  if (!place_of(A.kv, b, L / kBlk, &row, &place)) return;  // (nothing can be appended there either)
  const int n = L % kBlk * Hkv * (kD / 16);  // 16 codes each
  const int64_t all = (int64_t)2 * A.layers * A.batch;
  for (int item = blockIdx.y; item < 2 * A.layers; item += gridDim.y) {
    const int l = item >> 1, v = item & 1;
    const int64_t at = (int64_t)item * A.batch + b;
    uint4* codes = reinterpret_cast<uint4*>(static_cast<uint8_t*>(v ? A.caches.v[l] : A.caches.k[l]) + row * Hkv * kD);
    uint4* kept = reinterpret_cast<uint4*>(A.saved + at * kBlk * Hkv * kD);
    float* scales = (v ? A.scales.v[l] : A.scales.k[l]) + place * Hkv;
    float* kept_scales = reinterpret_cast<float*>(A.saved + all * kBlk * Hkv * kD) + at * Hkv;
    for (int i = threadIdx.x; i < n; i += kThreads) (SAVE ? kept : codes)[i] = (SAVE ? codes : kept)[i];
    for (int i = threadIdx.x; i < Hkv; i += kThreads) (SAVE ? kept_scales : scales)[i] = (SAVE ? scales : kept_scales)[i];
  }
}

}  // namespace

size_t held8_bytes(int layers, int batch, const cure_kv_desc& kv) {
  return (size_t)2 * layers * batch * kv.heads_kv * (kBlk * kD + sizeof(float));
}

cudaError_t launch_held8(bool save, int layers, const LayerPtrs& caches, const LayerScales& scales, const cure_kv_desc& kv,
                         int batch, const int32_t* cache_len, void* saved, cudaStream_t s) {
  HeldArgs a;
  a.caches = caches;
  a.scales = scales;
  a.kv = kv;
  a.cache_len = cache_len;
  a.saved = static_cast<uint8_t*>(saved);
  a.layers = layers;
  a.batch = batch;
  return launch_pdl(save ? held8_kernel<true> : held8_kernel<false>, dim3((unsigned)batch, (unsigned)(2 * layers)),
                    dim3(kThreads), 0, s, a);
}

cudaError_t launch_append8(const RopeArgs& args, float* k_scale, float* v_scale, cudaStream_t s) {
  Append8Args a;
  a.r = args;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  // A CTA for each block where sequences have many rows; for each row where they have one.
  a.range = 1;
  while (a.range < kBlk && (int64_t)2 * a.range * args.batch <= args.rows) a.range *= 2;
  const int64_t ctas = ((int64_t)args.rows + a.range - 1) / a.range;
  // Few blocks: their heads in parts, a pair of heads each where that leaves every SM at most one CTA.
  const int64_t sms = num_sms();
  const int groups = (args.heads_kv + 1) / 2;  // pairs of heads of K, and of V
  const int most = ctas * 2 * groups <= sms ? 2 * groups : std::max(groups, (args.heads_q + 7) / 8);
  auto parts_of = [&](int heads) -> int {
    return (int)std::max<int64_t>(1, std::min<int64_t>(sms * resident(heads) / ctas, most));
  };
  // Calls of few rows wait for meetings: four heads meet at a time, in fewer CTAs to an SM.  Single tokens of
  // 64 / 300 / 500 sequences 8.8 -> 7.0, 18.0 -> 12.8, 26.7 -> 22.9 us (8 heads of K and V), 32 trees of 33
  // rows 22.2 -> 18.0, 100 of 9 rows 19.9 -> 20.3.  Longer calls want the CTAs: 32 chunks of 100 rows 33.8 with
  // two heads, 39.3 with four; 19241 rows 91 and 94.
  const bool four = args.rows < 8 * sms && parts_of(2) < 2 * groups;
  const int parts = parts_of(four ? 4 : 2);
  auto kernel = args.rope.style == 1 ? four ? append8_kernel<true, 4> : append8_kernel<true, 2>
                                     : four ? append8_kernel<false, 4> : append8_kernel<false, 2>;
  return launch_pdl(kernel, dim3((unsigned)ctas, (unsigned)parts), dim3(kThreads), 0, s, a);
}

cudaError_t launch_paths8(int layers, const LayerPtrs& caches, const LayerScales& scales, const cure_kv_desc& kv,
                          const uint16_t* tree_k, const uint16_t* tree_v, int batch, int n_max, int block,
                          const int32_t* path_nodes, const int32_t* accept_len, const int32_t* cache_len, int* err,
                          cudaStream_t s) {
  Paths8Args a;
  a.caches = caches;
  a.scales = scales;
  a.kv = kv;
  a.tree_k = tree_k;
  a.tree_v = tree_v;
  a.layers = layers;
  a.batch = batch;
  a.n_max = n_max;
  a.block = block;
  a.path_nodes = path_nodes;
  a.accept_len = accept_len;
  a.cache_len = cache_len;
  a.err = err;
  const int blocks = (block + 1 + kBlk - 2) / kBlk + 1;
  const int parts = layers * 2 * ((kv.heads_kv + kHeadsP - 1) / kHeadsP);
  return launch_pdl(paths8_kernel, dim3((unsigned)(batch * blocks), (unsigned)(parts < 65535 ? parts : 65535)),
                    dim3(kThreads), 0, s, a);
}

}  // namespace cure
