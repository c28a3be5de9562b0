// What the attention kernels on tcgen05 share: TMA loads and maps, commits, piece
// counters and packed arithmetic; and the tree attention's MMA groups and waits by
// whole warps (the prompt attention issues a tile of 128 keys at a time, with its
// commit, and waits in less code: k_prompt.cu).
#pragma once

#include <cuda_bf16.h>
#include <cudaTypedefs.h>
#include <float.h>

#include <atomic>

#include "attn_common.cuh"
#include "tc_ptx.cuh"

namespace cure {
namespace tc {

constexpr int kAttnQHalf = kAttnRowsCta * 64 * 2;  // 16 KiB: [128 rows][64 d]
constexpr int kAttnVChunk = 16 * kAttnD * 2;       // 4 KiB: V keys 16c..16c+15, both d halves

// One S product group, S_m = Q_m K^T over K = 128 (8 MMAs), in one asm
// block: the descriptors step by constant adds (16-byte units: 32 bytes
// within a 64-element half); kd and kd2 describe the two d halves of K.
__device__ __forceinline__ void mma_s_group(uint32_t d, uint64_t qd, uint64_t kd, uint64_t kd2, uint32_t idesc) {
  asm volatile(
      "{\n\t.reg .pred pf, pt, el;\n\t.reg .b64 a, b;\n\t"
      "elect.sync _|el, 0xffffffff;\n\t"
      "setp.ne.b32 pf, %4, %4;\n\t"
      "setp.eq.b32 pt, %4, %4;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, pf;\n\t"
      "add.s64 a, %1, 2;\n\tadd.s64 b, %2, 2;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, pt;\n\t"
      "add.s64 a, %1, 4;\n\tadd.s64 b, %2, 4;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, pt;\n\t"
      "add.s64 a, %1, 6;\n\tadd.s64 b, %2, 6;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, pt;\n\t"
      "add.s64 a, %1, %5;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, %6, %3, pt;\n\t"
      "add.s64 a, %1, %5 + 2;\n\tadd.s64 b, %6, 2;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, pt;\n\t"
      "add.s64 a, %1, %5 + 4;\n\tadd.s64 b, %6, 4;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, pt;\n\t"
      "add.s64 a, %1, %5 + 6;\n\tadd.s64 b, %6, 6;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, pt;\n\t}\n" ::"r"(d),
      "l"(qd), "l"(kd), "r"(idesc), "r"(0), "n"(kAttnQHalf >> 4), "l"(kd2)
      : "memory");
}
// One PV product group, O_m (+)= P_m V over 64 keys (4 MMAs): A from TMEM
// (8 columns of bf16 pairs per step), B stepping by one V chunk.
__device__ __forceinline__ void mma_pv_group(uint32_t d, uint32_t pa, uint64_t vd, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p0, pt, el;\n\t.reg .b64 b;\n\t.reg .b32 t;\n\t"
      "elect.sync _|el, 0xffffffff;\n\t"
      "setp.ne.b32 p0, %4, 0;\n\t"
      "setp.eq.b32 pt, %4, %4;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p0;\n\t"
      "add.u32 t, %1, 8;\n\tadd.s64 b, %2, %5;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, pt;\n\t"
      "add.u32 t, %1, 16;\n\tadd.s64 b, %2, 2 * %5;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, pt;\n\t"
      "add.u32 t, %1, 24;\n\tadd.s64 b, %2, 3 * %5;\n\t"
      "@el tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, pt;\n\t}\n" ::"r"(d),
      "r"(pa), "l"(vd), "r"(idesc), "r"(accumulate), "n"(kAttnVChunk >> 4)
      : "memory");
}

// Arrive on `bar` once the products this warp's elected lane issued are done.
// The issuing warps run converged and elect the lane inside the asm instead of
// branching to lane 0 (in the LM head's issuer, which steps the same way, four
// products then take 124 cycles to issue instead of 265).  28 q / 4 kv heads, 16
// sequences of 5001-8191 keys, trees of up to 65 nodes 112 -> 107 us; 32 of
// 1024-8192 keys and 64 x 8 kv heads x 32768 keys within 1-2 %, about what runs
// differ by; one M tile on 8- and 16-token pages lost up to 2 % on stream-K (see
// attn_ping_pong).
__device__ __forceinline__ void commit_elect(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred el;\n\telect.sync _|el, 0xffffffff;\n\t"
      "@el tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}\n" ::"r"(bar)
      : "memory");
}

struct Bar {
  uint32_t base;
  __device__ __forceinline__ uint32_t operator()(int i) const { return base + 8u * (uint32_t)i; }
};

// All lanes of the warp wait; the warp proceeds only if every lane succeeded.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                          int* err) {
  const bool ok = wait_bounded(bar, parity, abort_flag, err, true);
  return __all_sync(0xffffffffu, ok);
}

// Pairs of floats in one 64-bit register pair, for the packed f32x2
// arithmetic of sm_100 and later (two lanes of work per instruction).
__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t r, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// max of three (sm_100 and later have a three-input float max)
__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// The base-2 log-sum-exp of a row of a piece.  A row that saw no key gets the lowest
// finite value: its O is 0, so a merge over pieces that all saw none gives 0
// (-inf would give NaN there).  A NaN stays one.
__device__ __forceinline__ float row_lse(float m, float l) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(m + log2f(l)), "f"(-FLT_MAX));
  return d;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c,
                                             uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c),
               "r"(d)
               : "memory");
}

// A unit's piece counter holds (launch tag << 9) | pieces arrived.  A word
// whose tag is not this launch's (left by an aborted launch or by another user
// of the memory, or never written) counts as zero, so the workspace needs no
// reset.  Tags have 55 bits, far from each other and from small integers
// (next_launch_tag): with 23 bits counted up from 1, words such as token ids
// were taken for counts.  A completed unit leaves zero behind, which counts as
// zero for the same call replayed from a graph, with the same tag.
constexpr int kCountBits = 9;
constexpr int kCountMask = (1 << kCountBits) - 1;
__device__ __forceinline__ int count_of(PieceCount v, uint64_t tag) {
  return (v >> kCountBits) == tag ? (int)(v & kCountMask) : 0;
}
// This piece's arrival (after its release fence): the pieces arrived so far,
// this one included.
__device__ __forceinline__ int arrive(PieceCount* cnt, uint64_t tag) {
  PieceCount old = *reinterpret_cast<volatile PieceCount*>(cnt);
  while (true) {
    const PieceCount nw = (PieceCount)(tag << kCountBits) | (PieceCount)(count_of(old, tag) + 1);
    const PieceCount prev = atomicCAS(cnt, old, nw);
    if (prev == old) return (int)(nw & kCountMask);
    old = prev;
  }
}

__device__ __forceinline__ PieceCount ld_acquire(const PieceCount* p) {
  PieceCount v;
  asm volatile("ld.acquire.gpu.global.b64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
  return v;
}

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, uint32_t bar,
                                            int c0, int c1, int c2, int c3, int c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
// An L2 prefetch of one 4-D box (no shared memory, no barrier).
__device__ __forceinline__ void tma_prefetch_4d(const CUtensorMap* map, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(c0), "r"(c1), "r"(c2), "r"(c3)
               : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar,
                                            int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

// ---- tensor maps (host)
inline PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) ==
                        cudaSuccess &&
                    q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p) : nullptr;
  }();
  return fn;
}

// [rows][Hkv][128] bf16 viewed as (d, head, row); boxes of 64 d x 1 head x box_rows.
inline bool make_kv_map(CUtensorMap* m, const void* base, uint64_t rows, int Hkv, int box_rows) {
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)kAttnD, (cuuint64_t)Hkv, (cuuint64_t)rows};
  cuuint64_t strides[2] = {(cuuint64_t)kAttnD * 2, (cuuint64_t)Hkv * kAttnD * 2};
  cuuint32_t box[3] = {64, 1, (cuuint32_t)box_rows};
  cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// V rows [rows][Hkv][128] bf16 viewed as (d in half, row, d half, head);
// boxes of 64 d x 16 rows x 2 halves: [half][16 rows][64 d], one 4 KiB chunk.
inline bool make_v_rows_map(CUtensorMap* m, const void* base, uint64_t rows, int Hkv) {
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[4] = {64, (cuuint64_t)rows, 2, (cuuint64_t)Hkv};
  cuuint64_t strides[3] = {(cuuint64_t)Hkv * kAttnD * 2, 128, (cuuint64_t)kAttnD * 2};
  cuuint32_t box[4] = {64, 16, 2, 1};
  cuuint32_t es[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Paged K or V [pages][ps][Hkv][128] bf16 viewed as (d in half, row in an
// 8-row group, d half + 2 * head, group in page, page); one box is a whole
// page of one head: [group][d half][8 rows][64 d], ps * 256 bytes.
inline bool make_page_map(CUtensorMap* m, const void* base, uint64_t pages, int ps, int Hkv) {
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[5] = {64, 8, 2 * (cuuint64_t)Hkv, (cuuint64_t)(ps / 8), (cuuint64_t)pages};
  cuuint64_t strides[4] = {(cuuint64_t)Hkv * kAttnD * 2, 128, (cuuint64_t)8 * Hkv * kAttnD * 2,
                           (cuuint64_t)ps * Hkv * kAttnD * 2};
  cuuint32_t box[5] = {64, 8, 2, (cuuint32_t)(ps / 8), 1};
  cuuint32_t es[5] = {1, 1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// q [tokens][Hkv][G][128] bf16 viewed as (d, group head, kv head, token); boxes
// of 64 d x G x 1 x npb tokens: the rows of one M tile, (node, g) packed.
inline bool make_q_map(CUtensorMap* m, const void* base, uint64_t tokens, int Hkv, int G, int npb) {
  auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[4] = {(cuuint64_t)kAttnD, (cuuint64_t)G, (cuuint64_t)Hkv, (cuuint64_t)tokens};
  cuuint64_t strides[3] = {(cuuint64_t)kAttnD * 2, (cuuint64_t)G * kAttnD * 2, (cuuint64_t)Hkv * G * kAttnD * 2};
  cuuint32_t box[4] = {64, (cuuint32_t)G, 1, (cuuint32_t)npb};
  cuuint32_t es[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace tc
}  // namespace cure
