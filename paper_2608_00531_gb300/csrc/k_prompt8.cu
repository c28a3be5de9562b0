// Attention of packed rows over a cache held in 8 bits (e4m3 codes, a scale for each block
// of 16 slots and head): causal (cure_prompt_attn8), or a repair tree's rows in place
// (cure_tree_attn8).
//
//   out_i = sum_j softmax_j(scale q_i k_j) v_j,   k_j = ks_j K_j,  v_j = vs_j V_j
//
// A CTA takes a row's query head, its four warps every fourth key, a lane four dims;
// one pass with the running maximum and sum.
#include "attn_tc.cuh"
#include "common.cuh"

namespace cure {
namespace {

using namespace tc;

constexpr int kD = 128;
constexpr int kBlk = CURE_KV8_BLOCK;

__device__ __forceinline__ float4 widen(uint32_t w) {
  uint32_t a, b;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}\n"
      : "=r"(a), "=r"(b)
      : "r"(w));
  const float2 p = __half22float2(*reinterpret_cast<__half2*>(&a)), q = __half22float2(*reinterpret_cast<__half2*>(&b));
  return make_float4(p.x, p.y, q.x, q.y);
}

__global__ void __launch_bounds__(128) attn8_kernel(const Attn8Call A) {
  pdl_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.x, h = blockIdx.y, Hkv = A.kv.heads_kv, hk = h / (A.heads_q / Hkv);
  int b, i, n;
  if (A.n_nodes) {
    b = row / A.n_max;
    i = row % A.n_max;
    n = A.n_nodes[b];
    if (n < 1 || n > A.n_max) {
      if (threadIdx.x == 0) flag(A.err, CURE_DEVERR_NODES);
      return;
    }
    if (i >= n) return;
  } else {
    for (b = 0; b < A.batch && A.row_start[b + 1] <= row; ++b) {}
    if (b == A.batch || row < A.row_start[b]) return;
    i = row - A.row_start[b];
    n = A.row_start[b + 1] - A.row_start[b];
    if (A.row_start[b] < 0 || A.row_start[b + 1] > A.rows) {
      if (threadIdx.x == 0) flag(A.err, CURE_DEVERR_NODES);
      return;
    }
  }
  const int L = A.cache_len[b];
  const int64_t cap = A.kv.layout == 0 ? A.kv.max_len : (int64_t)A.kv.max_len * A.kv.page_size;
  if (L < 0 || (int64_t)L + n > cap) {
    if (threadIdx.x == 0) flag(A.err, CURE_DEVERR_SLOT);
    return;
  }
  const uint64_t* anc = A.n_nodes ? A.anc + (int64_t)row * ((A.n_max + 63) / 64) : nullptr;
  const int keys = A.n_nodes ? L + n : L + i + 1;
  const uint2 qw = *reinterpret_cast<const uint2*>(A.q + ((int64_t)row * A.heads_q + h) * kD + 4 * lane);
  const float c = A.scale * 1.4426950408889634f;
  const float q0 = __uint_as_float(qw.x << 16) * c, q1 = __uint_as_float(qw.x & 0xffff0000u) * c,
              q2 = __uint_as_float(qw.y << 16) * c, q3 = __uint_as_float(qw.y & 0xffff0000u) * c;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = warp; j < keys; j += 4) {
    if (anc && j >= L && !(anc[(j - L) >> 6] >> ((j - L) & 63) & 1u)) continue;
    int64_t crow, place;
    float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
    bool there = true;
    if (A.kv.layout == 0) {
      crow = (int64_t)b * A.kv.max_len + j;
      place = (int64_t)b * ((A.kv.max_len + kBlk - 1) / kBlk) + j / kBlk;
    } else {
      const int ps = A.kv.page_size, page = A.kv.block_table[(int64_t)b * A.kv.max_len + j / ps];
      there = page >= 0 && page < A.kv.num_pages;
      crow = (int64_t)page * ps + j % ps;
      place = crow / kBlk;
      if (!there && threadIdx.x == 0) flag(A.err, CURE_DEVERR_PAGE);
    }
    float ks = 0.f, vs = 0.f;
    if (there) {
      k = widen(*reinterpret_cast<const uint32_t*>(A.k_cache + (crow * Hkv + hk) * kD + 4 * lane));
      v = widen(*reinterpret_cast<const uint32_t*>(A.v_cache + (crow * Hkv + hk) * kD + 4 * lane));
      ks = fminf(fmaxf(A.k_scale[place * Hkv + hk], 0x1p-40f), 0x1p40f);
      vs = fminf(fmaxf(A.v_scale[place * Hkv + hk], 0x1p-40f), 0x1p40f);
    }
    float x = (q0 * k.x + q1 * k.y) + (q2 * k.z + q3 * k.w);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    x *= ks;
    const float mn = fmaxf(m, x), a = ex2(m - mn), p = ex2(x - mn);
    m = mn;
    l = l * a + p;
    o = make_float4(o.x * a + p * vs * v.x, o.y * a + p * vs * v.y, o.z * a + p * vs * v.z, o.w * a + p * vs * v.w);
  }
  __shared__ float sm[4], sl[4];
  __shared__ float4 so[4][32];
  if (lane == 0) {
    sm[warp] = m;
    sl[warp] = l;
  }
  so[warp][lane] = o;
  __syncthreads();
  if (warp > 0) return;
  const float M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  float L4 = 0.f;
  o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int w = 0; w < 4; ++w) {
    if (sm[w] == -INFINITY) continue;
    const float a = ex2(sm[w] - M);
    L4 += a * sl[w];
    const float4 t = so[w][lane];
    o = make_float4(o.x + a * t.x, o.y + a * t.y, o.z + a * t.z, o.w + a * t.w);
  }
  const float inv = L4 > 0.f ? 1.f / L4 : 0.f;
  *reinterpret_cast<uint2*>(A.out + ((int64_t)row * A.heads_q + h) * kD + 4 * lane) =
      make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
}

}  // namespace

size_t attn8_workspace() { return prompt_attn_workspace(); }

cudaError_t launch_attn8(const Attn8Call& c, cudaStream_t s) {
  return launch_pdl(attn8_kernel, dim3((unsigned)c.rows, (unsigned)c.heads_q), dim3(128), 0, s, c);
}

}  // namespace cure
