// What the kernels of the paged cache share (paged.hip, paged_attention.hip). Not installed.
#pragma once
#include "../../include/amxfp4_paged.h"
#include "../../include/amxfp4_scoring.h"
#include "device_formats.h"

namespace amx {

constexpr int64_t kPagedMaxSeqs = 4096;

// The pool as the kernels see it. Byte offsets are 64-bit: a cache has more than 2^32 of them.
struct PagedPool {
  uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  uint32_t pages, page_log2, kv_heads;
};

hipError_t launch_paged_attention(int scale_kind, bool asym, int head_dim, const PagedPool& pool, const uint16_t* q, int64_t rows,
                                  int64_t q_heads, const int32_t* table, int64_t seqs, int64_t max_pages, const int32_t* lens,
                                  const int32_t* starts, const int32_t* positions, float scale, const amx_scores_t* scores,
                                  int64_t max_keys, uint16_t* out, void* workspace, hipStream_t s);
size_t paged_attention_workspace(int head_dim, int64_t rows, int64_t q_heads, int64_t kv_heads, int64_t seqs, int64_t max_keys);

}  // namespace amx
