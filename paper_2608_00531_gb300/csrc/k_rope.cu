// Between a layer's Q/K/V projection and its attention (Sec. 3.2, 3.4: the
// target runs its own attention over the tree's nodes at their positions): the
// per-head RMS norm of Q and K and the rotary rotation in one pass, the results
// as rows (cure_rope_qkv) or, for K and V, as rows of the cache
// (cure_append_kv).
//
//   y = x * w / sqrt(mean(x^2) + eps)                      (with norm weights)
//   a' = A (a cos(p f_i) - b sin(p f_i)), b' = A (b cos(p f_i) + a sin(p f_i))
//
// for the pair (a, b) of frequency i of a head at position p.  The angle is
// kept in turns: f_i / 2 pi is a 64-bit binary fraction, so that p times it
// modulo 2^64 is the exact fraction of a turn of that product at any position
// (an error of p 2^-65 turns, below 2^-34 at every int32 position); its upper
// 32 bits go to a float and through sincospif.
//
// Layout.  Half a warp holds a head, 8 values (16 bytes) a lane; a warp takes a
// range of one row's heads, with the row's cosines and sines (times the norm
// weights) in registers: they are the same for all heads.  In the half layout
// the partner of a value lies rot_dim / 16 lanes away, in the interleaved
// layout in the same lane.
#include <cuda_bf16.h>

#include "common.cuh"

namespace cure {
namespace {

constexpr int kWarps = 8;
constexpr int kD = 128;
constexpr int kUnroll = 4;  // loads in flight a lane: heads of one pass of a warp = 2 * kUnroll

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float lo_f(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

struct Rows {  // bf16 rows of heads
  const uint16_t* in;
  uint16_t* out;
  int64_t ld_in, ld_out;  // values from row to row
  int heads;
};

// A lane's 8 dims of a row's rotation: own = cos, other = -sin / +sin, with the
// norm's weights of the value itself and of its partner.
struct Turn {
  float own[8], other[8];
};

template <bool APPEND>
__global__ void __launch_bounds__(32 * kWarps)
rope_kernel(const __grid_constant__ RopeArgs A) {
  __shared__ uint64_t turns[64];
  if (threadIdx.x < 64) turns[threadIdx.x] = A.rope.turns[threadIdx.x];
  __syncthreads();
  pdl_begin();
  const int lane = threadIdx.x & 31, l16 = lane & 15, half = lane >> 4;
  const int64_t item = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int64_t row = item / A.chunks;
  const int chunk = (int)(item % A.chunks);
  if (row >= A.rows) return;
  int h = chunk * A.chunk_heads;  // this warp's heads of Q, K, V end to end: [h, h_end)
  const int h_end = min(h + A.chunk_heads, A.heads_q + 2 * A.heads_kv);

  int p = A.pos ? A.pos[row] : 0;
  if (p < 0) return;  // a row that holds no token
  int64_t crow = -1;  // APPEND: the row's place in the cache
  if (APPEND) {
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
    const int64_t i = row - A.row_start[seq];
    if (i < 0) {  // before the first sequence, or row_start does not ascend
      if (seq > 0 && lane == 0) flag(A.err, CURE_DEVERR_NODES);
      return;
    }
    const int64_t slot = A.cache_len[seq] + i;
    if (!A.pos) p = (int)slot;
    const int64_t cap = A.kv.layout == 0 ? A.kv.max_len : (int64_t)A.kv.max_len * A.kv.page_size;
    if (slot < 0 || slot >= cap) {
      if (lane == 0) flag(A.err, CURE_DEVERR_SLOT);
      return;
    }
    if (A.kv.layout == 0) {
      crow = (int64_t)seq * A.kv.max_len + slot;
    } else {
      const int page = A.kv.block_table[(int64_t)seq * A.kv.max_len + slot / A.kv.page_size];
      if (page < 0 || page >= A.kv.num_pages) {
        if (lane == 0) flag(A.err, CURE_DEVERR_PAGE);
        return;
      }
      crow = (int64_t)page * A.kv.page_size + slot % A.kv.page_size;
    }
  }

  // cosines and sines of the lane's dims
  const int r16 = A.rope.rot_dim >> 4;  // lanes of one half of the rotated dims
  const bool inter = A.rope.style == 1;
  const bool rot = l16 < 2 * r16;
  const bool first = l16 < r16;             // half layout: the lane holds the pairs' first values
  const int partner = inter || !rot ? lane : first ? lane + r16 : lane - r16;
  Turn t;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    t.own[e] = 1.f;
    t.other[e] = 0.f;
  }
  if (rot && h < A.heads_q + A.heads_kv) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (inter && (e & 1)) {
        t.own[e] = t.own[e - 1];
        t.other[e] = -t.other[e - 1];
        continue;
      }
      const int i = inter ? 4 * l16 + e / 2 : 8 * (first ? l16 : l16 - r16) + e;
      // the fraction of a turn in 2^-32, as a signed number of half turns
      const int32_t f = (int32_t)(uint32_t)(((uint64_t)(uint32_t)p * turns[i]) >> 32);
      float s, c;
      sincospif((float)f * 0x1p-31f, &s, &c);
      t.own[e] = c * A.rope.amplitude;
      t.other[e] = (inter || first ? -s : s) * A.rope.amplitude;
    }
  }

  // heads [a, b) of one tensor
  auto pass = [&](const Rows& R, int a, int b, const uint16_t* norm, bool turn) {
    if (a >= b) return;
    const uint16_t* src = R.in + row * R.ld_in + 8 * l16;
    uint16_t* dst = R.out + row * R.ld_out + 8 * l16;
    Turn w = t;
    if (turn && norm) {
      const uint4 v = *reinterpret_cast<const uint4*>(norm + 8 * l16);
      const uint4 u = *reinterpret_cast<const uint4*>(norm + 8 * (partner & 15));
      const uint32_t vv[4] = {v.x, v.y, v.z, v.w}, uu[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        w.own[2 * q] *= lo_f(vv[q]);
        w.own[2 * q + 1] *= hi_f(vv[q]);
        w.other[2 * q] *= inter ? hi_f(uu[q]) : lo_f(uu[q]);
        w.other[2 * q + 1] *= inter ? lo_f(uu[q]) : hi_f(uu[q]);
      }
    }
    for (int h0 = a; h0 < b; h0 += 2 * kUnroll) {
      uint4 x[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int hh = h0 + 2 * u + half;
        x[u] = hh < b ? *reinterpret_cast<const uint4*>(src + (int64_t)hh * kD) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int hh = h0 + 2 * u + half;
        uint32_t v[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
        if (turn) {
          float rs = 1.f;
          if (norm) {
            float ss = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) ss += lo_f(v[q]) * lo_f(v[q]) + hi_f(v[q]) * hi_f(v[q]);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            rs = rsqrtf(ss * (1.f / kD) + A.eps);
          }
          uint32_t g[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            g[q] = __shfl_sync(0xffffffffu, v[q], partner);
            if (inter) g[q] = __byte_perm(g[q], 0, 0x1032);
            if (!rot) g[q] = 0u;  // a value without a partner must not meet 0 * infinity
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float lo = rs * (lo_f(v[q]) * w.own[2 * q] + lo_f(g[q]) * w.other[2 * q]);
            const float hi = rs * (hi_f(v[q]) * w.own[2 * q + 1] + hi_f(g[q]) * w.other[2 * q + 1]);
            v[q] = pack2(lo, hi);
          }
        }
        if (hh < b) *reinterpret_cast<uint4*>(dst + (int64_t)hh * kD) = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
  };
  Rows Q{A.q, A.q_out, A.ld_q, A.ld_q_out, A.heads_q};
  Rows K{A.k, A.k_out, A.ld_k, A.ld_k_out, A.heads_kv};
  Rows V{A.v, A.v_out, A.ld_v, A.ld_v_out, A.heads_kv};
  if (APPEND) {  // K and V rows go to the row's place in the cache
    K.out += (crow - row) * K.ld_out;
    V.out += (crow - row) * V.ld_out;
  }
  const int k0 = A.heads_q, v0 = k0 + A.heads_kv;
  if (A.q) pass(Q, h, min(h_end, k0), A.q_norm, true);
  if (A.k) pass(K, max(h, k0) - k0, min(h_end, v0) - k0, A.k_norm, true);
  if (A.v) pass(V, max(h, v0) - v0, h_end - v0, nullptr, false);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& args, bool append, cudaStream_t s) {
  RopeArgs a = args;
  const int heads = a.heads_q + 2 * a.heads_kv;
  a.chunk_heads = heads;
  a.chunks = 1;
  const int64_t blocks = ((int64_t)a.rows * a.chunks + kWarps - 1) / kWarps;
  return launch_pdl(append ? rope_kernel<true> : rope_kernel<false>, dim3((unsigned)blocks), dim3(32 * kWarps), 0, s, a);
}

}  // namespace cure
