// A lane's values of a head, half a warp a head, 8 values a lane: how they lie in memory, as pairs of
// floats, and their rotation (k_rope.cu; k_cache8.cu: into a cache in 8 bits).
#pragma once

#include <cuda_bf16.h>

#include "attn_tc.cuh"
#include "common.cuh"

namespace cure {
namespace rope {

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

// The norm and the rotation of a lane's four pairs as factors: a' = ca a + sb b, b' = cb b + sa a.
struct Factors {
  uint64_t ca[2], cb[2], sa[2], sb[2];
};
// From the pairs' cosines and sines and the norm's weights (NULL: none) where the lane's values lie.
template <bool INTER>
__device__ __forceinline__ Factors factors(const float (&c)[4], const float (&sn)[4], const uint16_t* norm, int off_a,
                                           int off_b) {
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
  Factors f;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    f.ca[e] = tc::f2_pack(c[2 * e] * wa[2 * e], c[2 * e + 1] * wa[2 * e + 1]);
    f.cb[e] = tc::f2_pack(c[2 * e] * wb[2 * e], c[2 * e + 1] * wb[2 * e + 1]);
    f.sa[e] = tc::f2_pack(sn[2 * e] * wa[2 * e], sn[2 * e + 1] * wa[2 * e + 1]);
    f.sb[e] = tc::f2_pack(-sn[2 * e] * wb[2 * e], -sn[2 * e + 1] * wb[2 * e + 1]);
  }
  return f;
}
// A head's pairs normed (all 16 lanes of the half warp, whatever they hold) and rotated (`rot`: a value that is
// not must not meet 0 * infinity).
__device__ __forceinline__ void norm_rotate(uint64_t (&a)[2], uint64_t (&b)[2], const Factors& f, bool norm, float eps,
                                            bool rot) {
  uint64_t rs2 = 0;
  if (norm) {
    uint64_t ss = f2_mul(a[0], a[0]);
    ss = tc::f2_fma(a[1], a[1], ss);
    ss = tc::f2_fma(b[0], b[0], ss);
    ss = tc::f2_fma(b[1], b[1], ss);
    float s0, s1;
    tc::f2_unpack(ss, s0, s1);
    s0 += s1;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, o);
    const float rs = rsqrtf(s0 * (1.f / 128) + eps);
    rs2 = tc::f2_pack(rs, rs);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    uint64_t ya = f2_mul(a[e], f.ca[e]), yb = f2_mul(b[e], f.cb[e]);
    if (rot) {
      ya = tc::f2_fma(b[e], f.sb[e], ya);
      yb = tc::f2_fma(a[e], f.sa[e], yb);
    }
    a[e] = norm ? f2_mul(ya, rs2) : ya;
    b[e] = norm ? f2_mul(yb, rs2) : yb;
  }
}

}  // namespace rope
}  // namespace cure
