// What the attention kernels over a cache in 8 bits share: the codes' tensor maps, the workspace's
// layout and the arguments (k_prompt8.cu: tiles of 128 rows; k_tokens8.cu: few rows a sequence).
#pragma once

#include "prompt_units.cuh"

namespace cure {

// Calls whose sequences have so few rows on average that k_tokens8.cu takes them.
bool tokens8_fits(const Attn8Call& c);
cudaError_t launch_tokens8(const Attn8Call& c, cudaStream_t s);

namespace prompt {

// One layer's codes as (d, head, token in its page or sequence, page or sequence); boxes of 128 d x
// 1 head x box_tokens tokens, swizzled by 128 bytes, what lies outside reads as zeros.
inline bool make_codes_map(CUtensorMap* m, const uint8_t* base, const cure_kv_desc& kv, int batch, int box_tokens) {
  auto fn = encode_fn();
  if (!fn) return false;
  const bool paged = kv.layout == 1;
  const cuuint64_t tokens = paged ? kv.page_size : kv.max_len > 0 ? kv.max_len : 1;
  const cuuint64_t row = (cuuint64_t)kv.heads_kv * D;
  cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)kv.heads_kv, tokens, (cuuint64_t)(paged ? kv.num_pages : batch)};
  cuuint64_t strides[3] = {(cuuint64_t)D, row, row * tokens};
  cuuint32_t box[4] = {(cuuint32_t)D, 1, (cuuint32_t)box_tokens, 1};
  cuuint32_t es[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<uint8_t*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Workspace: piece counters [CTAs] (256-byte rounded), partial outputs and their log-sum-exps
// [2 * CTAs]: of a CTA's pieces at most its first and its last are parts of a unit.
inline size_t counter_bytes8(int ctas) { return ((size_t)ctas * sizeof(PieceCount) + 255) / 256 * 256; }

// This part's arrival at its unit's counter, as tc::arrive: the parts so far, this one included.  By
// additions, of which many at once are as fast as one (by exchanges, 38 parts of a unit that end together took
// 15 us).  An addition to a word without this launch's tag is not counted, whatever it leaves there: who
// made it sets the word, or finds it set and adds again.
__device__ __forceinline__ int arrive_at(PieceCount* cnt, uint64_t tag) {
  PieceCount old = atomicAdd(cnt, (PieceCount)1);
  while ((old >> kCountBits) != tag) {
    const PieceCount now = old = *reinterpret_cast<volatile PieceCount*>(cnt);
    if ((now >> kCountBits) == tag) {
      old = atomicAdd(cnt, (PieceCount)1);
    } else if (atomicCAS(cnt, now, (PieceCount)(tag << kCountBits) | 1u) == now) {
      return 1;
    }
  }
  return (int)(old & kCountMask) + 1;
}

inline void fill_args8(const Attn8Call& c, PromptArgs* A) {
  A->kv = c.kv;
  A->row_start = c.row_start;
  A->cache_len = c.cache_len;
  A->rows = c.rows;
  A->batch = c.batch;
  A->heads_q = c.heads_q;
  A->G = c.heads_q / c.kv.heads_kv;
  A->cap = std::min(c.kv.layout == 0 ? c.kv.max_len : c.kv.max_len * c.kv.page_size, INT32_MAX - 2 * BN);
  A->scale_log2 = c.scale * 1.4426950408889634f;
  A->out = c.out;
  A->err = c.err;
  A->expire_warp = c.expire_warp;
  A->expire_wait = c.expire_wait;
  A->tag = next_launch_tag();  // whatever the workspace's counters hold counts as zero
  const int ctas = num_sms();
  char* ws = static_cast<char*>(c.workspace);
  A->cnt = reinterpret_cast<PieceCount*>(ws);
  A->ws_o = reinterpret_cast<float*>(ws + counter_bytes8(ctas));
  A->ws_lse = A->ws_o + (size_t)2 * ctas * 2 * BM * D;
}

}  // namespace prompt
}  // namespace cure
