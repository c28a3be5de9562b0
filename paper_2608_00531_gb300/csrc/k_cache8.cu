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
// Layout.  A CTA takes the blocks that begin in its range of packed rows (a block's
// rows in one call are neighbours), a warp one head of K or V of a block at a time: half a
// warp a row, 8 values a lane, all 16 rows in registers (rows that the block holds already
// are decoded into the same places), so that every value is read once, the largest is
// found by one reduction, and the codes go out behind it.  The rows' cosines and sines
// are made once a block in shared memory, for all heads of K and Q.
#include <cuda_bf16.h>

#include "attn_tc.cuh"
#include "common.cuh"

namespace cure {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kD = 128;
constexpr int kBlk = CURE_KV8_BLOCK;
static_assert(kBlk == 16, "16 rows in 8 steps of two");

__device__ __forceinline__ float lo_f(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

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

struct Raw {  // a lane's values of one row as they lie in memory
  uint2 a, b;
};
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

// Head norm and rotation of a lane's values (all 16 lanes of the half warp).  cs: the row's
// cosines and sines.
template <bool INTER>
__device__ __forceinline__ void norm_rotate(float* y, const float* w, bool norm, float eps, const float2* cs, bool rot,
                                            int l16) {
  if (norm) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float rs = rsqrtf(ss * (1.f / kD) + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = y[e] * rs * w[e];
  }
  if (rot) {
    const float4* t = reinterpret_cast<const float4*>(cs + 4 * l16);
    const float4 t0 = t[0], t1 = t[1];
    const float c[4] = {t0.x, t0.z, t1.x, t1.z}, s[4] = {t0.y, t0.w, t1.y, t1.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = INTER ? 2 * e : e, j = INTER ? 2 * e + 1 : e + 4;
      const float a = y[i], b = y[j];
      y[i] = fmaf(-b, s[e], a * c[e]);
      y[j] = fmaf(a, s[e], b * c[e]);
    }
  }
}

// One head of a block (a warp): rows `fresh` (bits of the block's slots) from row(t), those of
// `held` as they stand; the new codes and scale.  `codes`: the head's codes of the block's
// slot 0, `ld` bytes from slot to slot.
template <bool INTER, bool TURN, class Row>
__device__ __forceinline__ void quantise_head(const Row& row, uint32_t fresh, uint32_t held, uint8_t* codes, int64_t ld,
                                              float* scale, const Lane& p, const float* w, bool norm, float eps,
                                              const float2 (*cs)[64], int lane) {
  const int l16 = lane & 15, half = lane >> 4;
  float y[8][8];
  Raw x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = 2 * j + half;
    x[j].a = x[j].b = make_uint2(0u, 0u);
    if (fresh >> t & 1u) {
      x[j] = load_raw(row(t), p);
    } else if (held >> t & 1u) {
      x[j].a.x = *reinterpret_cast<const uint32_t*>(codes + t * ld + p.off_a);
      x[j].a.y = *reinterpret_cast<const uint32_t*>(codes + t * ld + p.off_b);
    }
  }
  const float old = held ? *scale : 1.f;
  float amax = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = 2 * j + half;
    if ((fresh | held) >> (2 * j) & 3u) {  // (both halves of the warp: the norm's sums take all lanes)
      if (held >> t & 1u) {
        from_codes(x[j].a.x, y[j]);
        from_codes(x[j].a.y, y[j] + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[j][e] *= old;
      } else {
        widen(x[j], y[j]);
      }
      if (TURN) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = y[j][e];
        norm_rotate<INTER>(z, w, norm, eps, cs[t], p.rot, l16);
        if (fresh >> t & 1u) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[j][e] = z[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(y[j][e]));  // (a NaN counts for nothing)
    }
  }
  // as integers, which are ordered as the values are
  const int e = scale_exponent(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax))));
  const float s = power(e), inv = power(-e);
  const uint32_t out = s == old ? fresh : fresh | held;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int t = 2 * j + half;
    if (out >> t & 1u) {
      *reinterpret_cast<uint32_t*>(codes + t * ld + p.off_a) =
          to_codes(y[j][0] * inv, y[j][1] * inv, y[j][2] * inv, y[j][3] * inv);
      *reinterpret_cast<uint32_t*>(codes + t * ld + p.off_b) =
          to_codes(y[j][4] * inv, y[j][5] * inv, y[j][6] * inv, y[j][7] * inv);
    }
  }
  if (lane == 0) *scale = s;
}

// The page of a block of 16 slots, or the sequence's own range: the row of its slot 0 in the
// cache and its place among the scales; false (error word set) where there is none.
__device__ __forceinline__ bool place_of(const cure_kv_desc& kv, int seq, int blk, int64_t* row, int64_t* place, int* err,
                                         bool tell) {
  if (kv.layout == 0) {
    *row = (int64_t)seq * kv.max_len + (int64_t)blk * kBlk;
    *place = (int64_t)seq * ((kv.max_len + kBlk - 1) / kBlk) + blk;
    return true;
  }
  const int per = kv.page_size / kBlk;
  const int page = kv.block_table[(int64_t)seq * kv.max_len + blk / per];
  if (page < 0 || page >= kv.num_pages) {
    if (tell) flag(err, CURE_DEVERR_PAGE);
    return false;
  }
  *place = (int64_t)page * per + blk % per;
  *row = *place * kBlk;
  return true;
}

struct Append8Args {
  RopeArgs r;
  float *k_scale, *v_scale;
  int range;  // packed rows whose blocks a CTA takes
};

template <bool INTER>
__global__ void __launch_bounds__(kThreads, 2)
append8_kernel(const __grid_constant__ Append8Args G) {
  const RopeArgs& A = G.r;
  __shared__ uint64_t turns[64];
  __shared__ float2 cs[kBlk][64];
  __shared__ uint32_t skip;  // rows of the block with a negative position
  if (threadIdx.x < 64) turns[threadIdx.x] = A.rope.turns[threadIdx.x];
  pdl_begin();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, l16 = lane & 15, half = lane >> 4;
  const int Hq = A.heads_q, Hkv = A.heads_kv;
  const int first = blockIdx.x * G.range;
  const int end = min(first + G.range, A.rows);
  const Lane turned = lane_of<INTER>(l16, A.rope.rot_dim), plain = lane_of<true>(l16, 0);
  const int n_axes = A.axes.axes;
  const int64_t cap = A.kv.layout == 0 ? A.kv.max_len : (int64_t)A.kv.max_len * A.kv.page_size;

  for (int row = first; row < end;) {
    // the row's sequence: as many of the ends row_start[1..B] are at or before it
    int seq = 0;
    for (int base = 0; base < A.batch; base += 256) {
      int e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int b = base + 32 * i + lane;
        e[i] = b < A.batch ? A.row_start[b + 1] : INT32_MAX;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) seq += __popc(__ballot_sync(0xffffffffu, e[i] <= row));
    }
    if (seq >= A.batch) return;  // behind the last sequence
    const int start = A.row_start[seq], stop = min(A.row_start[seq + 1], A.rows);
    const int i = row - start;
    if (i < 0 || start < 0 || row >= stop) {  // before the first sequence, or row_start does not ascend
      if ((seq > 0 || i >= 0) && tid == 0 && blockIdx.y == 0) flag(A.err, CURE_DEVERR_NODES);
      ++row;
      continue;
    }
    const int L = A.cache_len[seq];
    const int64_t slot = (int64_t)L + i;
    if (slot < 0 || slot >= cap) {
      if (tid == 0 && blockIdx.y == 0) flag(A.err, CURE_DEVERR_SLOT);
      ++row;
      continue;
    }
    const int blk = (int)(slot / kBlk), t0 = (int)(slot % kBlk);
    if (i > 0 && t0 > 0) {  // the block begins before this row: its CTA takes it
      row += min(kBlk - t0, stop - row);
      continue;
    }
    const int m = (int)min((int64_t)min(kBlk - t0, stop - row), cap - slot);  // the block's rows
    const int row0 = row;
    row += m;
    int64_t crow, place;
    if (!place_of(A.kv, seq, blk, &crow, &place, A.err, tid == 0 && blockIdx.y == 0)) continue;

    // ---- the rows' angles, and which of them hold no token
    __syncthreads();  // (the block before is done with them)
    if (tid == 0) skip = 0;
    __syncthreads();
    if (A.pos && tid < m) {
      bool none = false;
      for (int a = 0; a < max(1, n_axes); ++a) none |= A.pos[(int64_t)a * A.rows + row0 + tid] < 0;
      if (none) atomicOr(&skip, 1u << (t0 + tid));
    }
    const int pairs = A.rope.rot_dim / 2;
    for (int k = tid; k < m * 64; k += kThreads) {
      const int r = k >> 6, pair = k & 63;
      if (pair < pairs) {
        const int axis = n_axes > 0 ? A.axes.axis[pair] : 0;
        const int p = A.pos ? A.pos[(int64_t)axis * A.rows + row0 + r] : (int)(slot + r);
        // the fraction of a turn in 2^-32, as a signed number of half turns
        const int32_t f = (int32_t)(uint32_t)(((uint64_t)(uint32_t)p * turns[pair]) >> 32);
        float2 c;
        sincospif((float)f * 0x1p-31f, &c.y, &c.x);
        cs[t0 + r][pair] = make_float2(c.x * A.rope.amplitude, c.y * A.rope.amplitude);
      }
    }
    __syncthreads();
    const uint32_t rows_in = ((1u << m) - 1u) << t0;
    const uint32_t fresh = rows_in & ~skip;
    const uint32_t held = i == 0 ? (1u << t0) - 1u : 0u;
    if (fresh == 0) continue;

    // ---- heads of K and V, then those of Q
    const int64_t ld = (int64_t)Hkv * kD;
    for (int h = blockIdx.y * kWarps + warp; h < 2 * Hkv; h += gridDim.y * kWarps) {
      const bool is_v = h >= Hkv;
      const int hh = is_v ? h - Hkv : h;
      if (is_v) {
        auto src = [&](int t) { return A.v + (int64_t)(row0 + t - t0) * A.ld_v + hh * kD; };
        quantise_head<true, false>(src, fresh, held, reinterpret_cast<uint8_t*>(A.v_out) + crow * ld + hh * kD, ld,
                                   G.v_scale + place * Hkv + hh, plain, nullptr, false, 0.f, nullptr, lane);
      } else {
        float w[8];
        if (A.k_norm) widen(load_raw(A.k_norm, turned), w);
        auto src = [&](int t) { return A.k + (int64_t)(row0 + t - t0) * A.ld_k + hh * kD; };
        quantise_head<INTER, true>(src, fresh, held, reinterpret_cast<uint8_t*>(A.k_out) + crow * ld + hh * kD, ld,
                                   G.k_scale + place * Hkv + hh, turned, w, A.k_norm != nullptr, A.eps, cs, lane);
      }
    }
    if (A.q) {
      // (row, head) pairs, half a warp each, four at a time
      float w[8];
      if (A.q_norm) widen(load_raw(A.q_norm, turned), w);
      const int todo = m * Hq;
      constexpr int U = 4;
      for (int k0 = (blockIdx.y * kWarps + warp) * 2 * U; k0 < todo; k0 += gridDim.y * kWarps * 2 * U) {
        Raw x[U];
        int r[U], hh[U];
        bool there[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = k0 + 2 * u + half;
          r[u] = k / Hq;
          hh[u] = k - r[u] * Hq;
          there[u] = k < todo && (fresh >> (t0 + r[u]) & 1u);
          x[u].a = x[u].b = make_uint2(0u, 0u);
          if (there[u]) x[u] = load_raw(A.q + (int64_t)(row0 + r[u]) * A.ld_q + hh[u] * kD, turned);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float y[8];
          widen(x[u], y);
          norm_rotate<INTER>(y, w, A.q_norm != nullptr, A.eps, cs[(t0 + r[u]) & 15], turned.rot, l16);
          if (there[u]) {
            uint16_t* out = A.q_out + (int64_t)(row0 + r[u]) * A.ld_q_out + hh[u] * kD;
            *reinterpret_cast<uint2*>(out + turned.off_a) =
                make_uint2(tc::pack_bf16(y[0], y[1]), tc::pack_bf16(y[2], y[3]));
            *reinterpret_cast<uint2*>(out + turned.off_b) =
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

// The k-th block that sequence b's accepted path reaches (blockIdx.x = b * blocks + k), a
// head of K or V of a layer a warp.
__global__ void __launch_bounds__(kThreads, 2)
paths8_kernel(const __grid_constant__ Paths8Args A) {
  pdl_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int blocks = (A.block + 1 + kBlk - 2) / kBlk + 1;
  const int b = blockIdx.x / blocks, k = blockIdx.x % blocks;
  const int Hkv = A.kv.heads_kv, P = A.block + 2;
  const int n = min(A.accept_len[b], A.block) + 1;  // rows of the path
  const int L = A.cache_len[b];
  const bool tell = threadIdx.x == 0 && blockIdx.y == 0;
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
  if (!place_of(A.kv, b, blk, &crow, &place, A.err, tell)) return;
  // lane t: the node of slot t
  int node = -1;
  if (lane >= from && lane < to) {
    node = A.path_nodes[(int64_t)b * P + (int)(slot0 + lane - L)];
    if (node < 0 || node >= A.n_max) {
      if (warp == 0 && blockIdx.y == 0) flag(A.err, CURE_DEVERR_NODES);
      node = -1;
    }
  }
  const uint32_t fresh = __ballot_sync(0xffffffffu, node >= 0), held = (1u << from) - 1u;
  if (fresh == 0) return;
  int nodes[8];  // of the half warp's rows
#pragma unroll
  for (int j = 0; j < 8; ++j) nodes[j] = __shfl_sync(0xffffffffu, node, 2 * j + (lane >> 4));
  const Lane plain = lane_of<true>(lane & 15, 0);
  const int64_t ld = (int64_t)Hkv * kD;
  const int total = A.layers * 2 * Hkv;
  for (int item = blockIdx.y * kWarps + warp; item < total; item += gridDim.y * kWarps) {
    const int l = item / (2 * Hkv), h = item % (2 * Hkv);
    const bool is_v = h >= Hkv;
    const int hh = is_v ? h - Hkv : h;
    const uint16_t* tree = (is_v ? A.tree_v : A.tree_k) + ((int64_t)l * A.batch + b) * A.n_max * ld + hh * kD;
    uint8_t* codes = static_cast<uint8_t*>(is_v ? A.caches.v[l] : A.caches.k[l]) + crow * ld + hh * kD;
    float* scale = (is_v ? A.scales.v[l] : A.scales.k[l]) + place * Hkv + hh;
    auto src = [&](int t) { return tree + nodes[t >> 1] * ld; };
    quantise_head<true, false>(src, fresh, held, codes, ld, scale, plain, nullptr, false, 0.f, nullptr, lane);
  }
}

}  // namespace

cudaError_t launch_append8(const RopeArgs& args, float* k_scale, float* v_scale, cudaStream_t s) {
  Append8Args a;
  a.r = args;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  // A CTA for each block where sequences have many rows; for each row where they have one.
  a.range = 1;
  while (a.range < kBlk && (int64_t)2 * a.range * args.batch <= args.rows) a.range *= 2;
  const int64_t ctas = ((int64_t)args.rows + a.range - 1) / a.range;
  // few blocks: their heads in parts
  const int64_t want = (int64_t)num_sms() * 2;
  const int most = (2 * args.heads_kv + kWarps - 1) / kWarps;
  int parts = (int)((want + ctas - 1) / ctas);
  if (parts > most) parts = most;
  auto kernel = args.rope.style == 1 ? append8_kernel<true> : append8_kernel<false>;
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
  const int items = layers * 2 * kv.heads_kv;
  const int parts = (items + kWarps - 1) / kWarps;
  return launch_pdl(paths8_kernel, dim3((unsigned)(batch * blocks), (unsigned)(parts < 65535 ? parts : 65535)),
                    dim3(kThreads), 0, s, a);
}

}  // namespace cure
