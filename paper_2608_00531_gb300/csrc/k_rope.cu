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
// modulo 2^64 is the exact fraction of a turn of that product at any position;
// what the table's entry is off by (it comes from 64-bit floats: below 2^-53 turns
// for the plain frequencies) counts p times.  The fraction's upper 32 bits go to a
// float, which rounds them by up to 2^-26 of a turn, and through sincospif.
//
// Layout.  Half a warp holds a head, 8 values a lane, and a warp takes a range of
// one row's heads with the row's cosines and sines (times the norm weights) in
// registers: they are the same for all heads.  A lane's 8 values are four whole
// pairs, so that no lane needs another's: in the half layout two runs of 4 values
// rot_dim / 2 apart, two 8-byte loads; in the interleaved layout 8 values on end.
// The arithmetic is on pairs of floats (f32x2).
//
// Bound and measured.  Every value is read once and written once: HBM bounds many
// rows.  32768 rows of 64 + 2 x 8 heads 204 us, 6.59 TB/s (0.97 of a plain copy's
// 6.78); 10940 rows of 28 + 2 x 4 heads with norms into 16-token pages 42 us, 4.76
// TB/s: three waves of warps, each with its look-ups and six rounds of loads, and the
// norm's sums (39 us without them).  Few rows are bound by latency: 17 rows of 32 + 2 x
// 8 heads 2.6 us, 758 rows of 28 + 2 x 4 heads with norms 7.4 us (1.9 TB/s).  (Loads of
// the next step into each place as it falls free: 63 us for the 10940 rows, as the
// four places' sums then run one after the other.)
#include <cuda_bf16.h>

#include "attn_tc.cuh"
#include "common.cuh"

namespace cure {
namespace {

constexpr int kWarps = 8;
constexpr int kD = 128;
constexpr int kUnroll = 4;  // heads of one step of a warp: 2 * kUnroll, their loads in flight together

__device__ __forceinline__ float lo_f(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_f(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

struct Raw {  // a lane's values of one head as they lie in memory
  uint2 a, b;
};
// Its four pairs: first and second values, two pairs to a register pair.
template <bool INTER>
__device__ __forceinline__ void unpack(const Raw& x, uint64_t (&a)[2], uint64_t (&b)[2]) {
  if (INTER) {
    a[0] = tc::f2_pack(lo_f(x.a.x), lo_f(x.a.y));
    b[0] = tc::f2_pack(hi_f(x.a.x), hi_f(x.a.y));
    a[1] = tc::f2_pack(lo_f(x.b.x), lo_f(x.b.y));
    b[1] = tc::f2_pack(hi_f(x.b.x), hi_f(x.b.y));
  } else {
    a[0] = tc::f2_pack(lo_f(x.a.x), hi_f(x.a.x));
    a[1] = tc::f2_pack(lo_f(x.a.y), hi_f(x.a.y));
    b[0] = tc::f2_pack(lo_f(x.b.x), hi_f(x.b.x));
    b[1] = tc::f2_pack(lo_f(x.b.y), hi_f(x.b.y));
  }
}
template <bool INTER>
__device__ __forceinline__ Raw pack(const uint64_t (&a)[2], const uint64_t (&b)[2]) {
  float a0, a1, a2, a3, b0, b1, b2, b3;
  tc::f2_unpack(a[0], a0, a1);
  tc::f2_unpack(a[1], a2, a3);
  tc::f2_unpack(b[0], b0, b1);
  tc::f2_unpack(b[1], b2, b3);
  Raw y;
  if (INTER) {
    y.a = make_uint2(tc::pack_bf16(a0, b0), tc::pack_bf16(a1, b1));
    y.b = make_uint2(tc::pack_bf16(a2, b2), tc::pack_bf16(a3, b3));
  } else {
    y.a = make_uint2(tc::pack_bf16(a0, a1), tc::pack_bf16(a2, a3));
    y.b = make_uint2(tc::pack_bf16(b0, b1), tc::pack_bf16(b2, b3));
  }
  return y;
}

template <bool APPEND, bool INTER>
__global__ void __launch_bounds__(32 * kWarps, 3)
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
  // this warp's heads of Q, K and V end to end: [h, h_end)
  const int h = chunk * A.chunk_heads, k0 = A.heads_q, v0 = k0 + A.heads_kv;
  const int h_end = min(h + A.chunk_heads, v0 + A.heads_kv);

  // where the lane's values lie in a head: with rotated dims left, the pairs 4 l16
  // .. 4 l16 + 3; the lanes behind them take the dims that are not rotated
  const int r8 = A.rope.rot_dim >> 3;  // lanes that rotate
  const bool rot = l16 < r8;
  const int off_a = INTER ? 8 * l16 : rot ? 4 * l16 : 8 * l16;
  const int off_b = INTER ? 8 * l16 + 4 : rot ? 4 * l16 + 4 * r8 : 8 * l16 + 4;

  auto load = [&](const uint16_t* in, int a, int b, Raw (&x)[kUnroll]) {  // heads a .. b - 1, at most 2 * kUnroll
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int hh = a + 2 * u + half;
      x[u].a = x[u].b = make_uint2(0u, 0u);
      if (hh < b) {
        x[u].a = *reinterpret_cast<const uint2*>(in + hh * kD + off_a);
        x[u].b = *reinterpret_cast<const uint2*>(in + hh * kD + off_b);
      }
    }
  };
  const uint16_t* in_q = A.q ? A.q + row * A.ld_q : nullptr;
  const uint16_t* in_k = A.k ? A.k + row * A.ld_k : nullptr;
  const uint16_t* in_v = A.v ? A.v + row * A.ld_v : nullptr;
  // the first step's loads go out before anything is looked up
  Raw x[kUnroll];
  if (h < k0) {
    if (in_q) load(in_q, h, min(h_end, k0), x);
  } else if (h < v0) {
    if (in_k) load(in_k, h - k0, min(h_end, v0) - k0, x);
  } else if (in_v) {
    load(in_v, h - v0, h_end - v0, x);
  }

  int p = A.pos ? A.pos[row] : 0;
  if (p < 0) return;  // a row that holds no token
  int64_t crow = row;  // the row of K's and V's outputs
  if (APPEND) {
    // the row's sequence: as many of the ends row_start[1..B] are at or before it
    int seq = 0;
    if (A.batch <= 32) {
      const int e = lane < A.batch ? A.row_start[lane + 1] : INT32_MAX;
      seq = __popc(__ballot_sync(0xffffffffu, e <= row));
    } else {
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
    }
    if (seq >= A.batch) return;  // behind the last sequence
    const int start = A.row_start[seq];
    const int64_t i = row - start;
    if (i < 0 || start < 0 || row >= A.row_start[seq + 1]) {  // before the first sequence, or row_start does not ascend
      if ((seq > 0 || i >= 0) && lane == 0) flag(A.err, CURE_DEVERR_NODES);
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
      const int ps = A.kv.page_size;
      const int page = A.kv.block_table[(int64_t)seq * A.kv.max_len + (int)slot / ps];
      if (page < 0 || page >= A.kv.num_pages) {
        if (lane == 0) flag(A.err, CURE_DEVERR_PAGE);
        return;
      }
      crow = (int64_t)page * ps + (int)slot % ps;
    }
  }

  // cosines and sines of the lane's pairs: a' = a c + b ms, b' = b c + a s
  float c[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (rot && h < v0) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // the fraction of a turn in 2^-32, as a signed number of half turns
      const int32_t f = (int32_t)(uint32_t)(((uint64_t)(uint32_t)p * turns[4 * l16 + e]) >> 32);
      sincospif((float)f * 0x1p-31f, &sn[e], &c[e]);
      c[e] *= A.rope.amplitude;
      sn[e] *= A.rope.amplitude;
    }
  }

  // heads [a, b) of one tensor; `have`: x holds the first step's values
  auto pass = [&](const uint16_t* in, uint16_t* out, int a, int b, const uint16_t* norm, bool have) {
    uint64_t ca[2], cb[2], sa[2], sb[2];  // factors of a and b: a' = ca a + sb b, b' = cb b + sa a
    {
      float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f};
      if (norm) {
        Raw w;
        w.a = *reinterpret_cast<const uint2*>(norm + off_a);
        w.b = *reinterpret_cast<const uint2*>(norm + off_b);
        uint64_t pa[2], pb[2];
        unpack<INTER>(w, pa, pb);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          tc::f2_unpack(pa[e], wa[2 * e], wa[2 * e + 1]);
          tc::f2_unpack(pb[e], wb[2 * e], wb[2 * e + 1]);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        ca[e] = tc::f2_pack(c[2 * e] * wa[2 * e], c[2 * e + 1] * wa[2 * e + 1]);
        cb[e] = tc::f2_pack(c[2 * e] * wb[2 * e], c[2 * e + 1] * wb[2 * e + 1]);
        sa[e] = tc::f2_pack(sn[2 * e] * wa[2 * e], sn[2 * e + 1] * wa[2 * e + 1]);
        sb[e] = tc::f2_pack(-sn[2 * e] * wb[2 * e], -sn[2 * e + 1] * wb[2 * e + 1]);
      }
    }
    for (int h0 = a; h0 < b; h0 += 2 * kUnroll) {
      if (!have) load(in, h0, b, x);
      have = false;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int hh = h0 + 2 * u + half;
        if (h0 + 2 * u >= b) break;
        uint64_t va[2], vb[2], ya[2], yb[2];
        unpack<INTER>(x[u], va, vb);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          ya[e] = f2_mul(va[e], ca[e]);
          yb[e] = f2_mul(vb[e], cb[e]);
          if (rot) {  // a value that is not rotated must not meet 0 * infinity
            ya[e] = tc::f2_fma(vb[e], sb[e], ya[e]);
            yb[e] = tc::f2_fma(va[e], sa[e], yb[e]);
          }
        }
        if (norm) {
          uint64_t ss = f2_mul(va[0], va[0]);
          ss = tc::f2_fma(va[1], va[1], ss);
          ss = tc::f2_fma(vb[0], vb[0], ss);
          ss = tc::f2_fma(vb[1], vb[1], ss);
          float s0, s1;
          tc::f2_unpack(ss, s0, s1);
          s0 += s1;
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, o);
          const float rs = rsqrtf(s0 * (1.f / kD) + A.eps);
          const uint64_t rs2 = tc::f2_pack(rs, rs);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            ya[e] = f2_mul(ya[e], rs2);
            yb[e] = f2_mul(yb[e], rs2);
          }
        }
        if (hh < b) {
          const Raw y = pack<INTER>(ya, yb);
          *reinterpret_cast<uint2*>(out + hh * kD + off_a) = y.a;
          *reinterpret_cast<uint2*>(out + hh * kD + off_b) = y.b;
        }
      }
    }
  };
  if (in_q && h < k0) pass(in_q, A.q_out + row * A.ld_q_out, h, min(h_end, k0), A.q_norm, true);
  const int ka = max(h, k0) - k0, kb = min(h_end, v0) - k0;
  if (in_k && ka < kb) pass(in_k, A.k_out + crow * A.ld_k_out, ka, kb, A.k_norm, h >= k0);
  const int va = max(h, v0) - v0, vb = h_end - v0;
  if (in_v && va < vb) {
    uint16_t* out = A.v_out + crow * A.ld_v_out;
    for (int h0 = va; h0 < vb; h0 += 2 * kUnroll) {
      if (h0 > va || h < v0) load(in_v, h0, vb, x);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int hh = h0 + 2 * u + half;
        if (hh < vb) {
          *reinterpret_cast<uint2*>(out + hh * kD + off_a) = x[u].a;
          *reinterpret_cast<uint2*>(out + hh * kD + off_b) = x[u].b;
        }
      }
    }
  }
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& args, bool append, cudaStream_t s) {
  RopeArgs a = args;
  const int heads = a.heads_q + 2 * a.heads_kv;
  // Few rows: a row's heads in parts, of one step's heads where all parts are resident
  // at once, so that a row is over after one round of loads (us replayed, parts of 8 / 16
  // / 32 heads / whole rows: 300 rows of 36 normed heads 3.8 / 4.5 / 6.5 / 6.8; 758 6.2 /
  // 6.2 / 6.8 / 7.2; 1000 6.8 / 6.5 / 7.9 / 7.2; 758 rows of 80 heads 8.6 / 7.9 / 8.7 /
  // 12.0).  Many: a warp a row, so that its angles serve all heads (2566 rows of 36 normed
  // heads 16.1 / 16.7 / 17.7 / 13.6, 9000 of them 47.8 / 44.1 / 43.8 / 35.2).  In a second
  // wave of whole rows that is mostly idle, parts of two steps are faster: up to some 11/8
  // of a wave, and with 40 heads or more (with 36 the third part is a quarter full).  Parts
  // of 16 / whole rows, normed: 80 heads, 4096 rows 34.9 / 39.2, 5000 41.6 / 42.0, 5472
  // 45.2 / 43.6, 7200 58.0 / 50.2; 40 heads, 4096 21.7 / 23.1, 5000 25.8 / 24.6; 36 heads,
  // 4096 22.9 / 21.6, 7200 35.8 / 27.2.
  const int64_t resident = (int64_t)num_sms() * 3 * kWarps;
  a.chunk_heads = heads;
  for (int n = 2 * kUnroll; n < heads; n *= 2)
    if (a.rows * (int64_t)((heads + n - 1) / n) <= resident) {
      a.chunk_heads = n;
      break;
    }
  if (a.chunk_heads == heads && heads >= 40 && a.rows > resident && 8 * (int64_t)a.rows < 11 * resident)
    a.chunk_heads = 4 * kUnroll;
  a.chunks = (heads + a.chunk_heads - 1) / a.chunk_heads;
  const int64_t blocks = ((int64_t)a.rows * a.chunks + kWarps - 1) / kWarps;
  auto kernel = a.rope.style == 1 ? (append ? rope_kernel<true, true> : rope_kernel<false, true>)
                                  : (append ? rope_kernel<true, false> : rope_kernel<false, false>);
  return launch_pdl(kernel, dim3((unsigned)blocks), dim3(32 * kWarps), 0, s, a);
}

}  // namespace cure
