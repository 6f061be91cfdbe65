// The masked attention for heads of 128, the checks of a call and how it is divided (attention_masked.h has the kernel).
#include "attention_masked.h"

namespace amx {
namespace {

// Up to so many workgroups all run at once. They are dealt to the compute units in turns, of which every other one goes backwards, so that a
// unit that got a long block in one gets a short one in the next: nine documents in 2048 rows 47 -> 42 us, five prefixes in 1504 rows (64 heads)
// 48 -> 40. Of more workgroups the longest start first.
constexpr int64_t kAtOnce = 768;
// Keys from which tiles too far for a slope are looked for, where no `first` cuts the rows shorter (the norms are a launch more). With and without, us: 32 / 8 heads
// x 8192 with slopes from 2^-0.25 to 2^-8 367 and 590, of heads of 64 309 and 443, 40 / 8 heads x 4096 156 and 211, 32 / 8 x 2048 69 and 67.
constexpr int64_t kFarKeys = 4096;
constexpr int64_t kMostBlocks = 64;  // (a lane to each)

// Few workgroups with long rows are split over the keys, kLeastOfChunk key tiles or more to a chunk, into as many as run at once: two to a
// compute unit, or three with heads of 64, where the chunks stay long. us for up to 512, 768 and 1024 workgroups: 10 rows behind 30000 keys, 32 / 8 heads of
// 128, 114, 131 and 117 (786 without a split), 200 rows of 40 heads behind 8000 90, 111 and 100, heads of 64, 100 rows behind 8000 42, 45 and 50 (185), 10 rows
// behind 30000 81, 66 and 81. 10 rows behind 3000 keys in chunks of eight tiles 33, of four 37.
constexpr int64_t kSplitBelow = 256, kLeastOfChunk = 8, kLongChunk = 32, kMostChunks = 64;

// Chunks that the key tiles of a block of queries are cut into.
int chunks_of(int64_t Hq, int64_t Sq, int64_t tiles, int64_t D) {
  const int64_t workgroups = Hq * ((Sq + kQueries - 1) / kQueries);
  if (workgroups > kSplitBelow) return 1;
  int64_t c = 768 / workgroups;
  if (D == 128 || tiles / c < kLongChunk) c = 512 / workgroups;
  if (c > tiles / kLeastOfChunk) c = tiles / kLeastOfChunk;
  return (int)(c > kMostChunks ? kMostChunks : c < 2 ? 1 : c);
}
// (the most for fewer tiles too)
int most_chunks_of(int64_t Hq, int64_t Sq, int64_t tiles, int64_t D) {
  const int a = chunks_of(Hq, Sq, tiles, D), b = chunks_of(Hq, Sq, tiles, 128);
  return a > b ? a : b;
}

size_t panels_bytes(int64_t Hq, int64_t Hkv, int64_t Sq, int64_t Sk, int64_t D) { return (attention_workspace_bytes(Hq, Hkv, Sq, Sk, D) + 255) & ~(size_t)255; }
size_t rows_bytes(int64_t Hq, int64_t Sq, int chunks, int64_t floats) { return ((size_t)(Hq * Sq * chunks * floats) * sizeof(float) + 255) & ~(size_t)255; }
size_t workspace_bytes_of(int64_t Hq, int64_t Hkv, int64_t Sq, int64_t Sk, int64_t D) {
  const int c = most_chunks_of(Hq, Sq, Sk / 32, D);
  return panels_bytes(Hq, Hkv, Sq, Sk, D) + (size_t)(Hkv * (Sk / 32)) * sizeof(float) + (c == 1 ? 0 : rows_bytes(Hq, Sq, c, 1) + rows_bytes(Hq, Sq, c, 2) + rows_bytes(Hq, Sq, c, D));
}
// Workgroups of a launch whose waves take two key tiles to a step: where two of them to a compute unit, which is what the registers leave room for, are
// all there are. us with one tile and with two: 32 / 8 heads x 2048, capped, 79.0 and 74.7, of heads of 64 60.9 and 56.1, 256 workgroups with a window of 4096
// (not split) 121 and 114; 768 workgroups (64 / 8 x 1504) 39.9 and 45.8.
constexpr int64_t kMostOfPairs = 512;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace
}  // namespace amx

using namespace amx;

extern "C" {

size_t amxfp4_attention_masked_workspace_bytes(const amx_format_t* fmt, int64_t q_heads, int64_t kv_heads, int64_t Sq, int64_t Sk,
                                               int64_t head_dim) {
  if (!fmt || q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads || q_heads > 65535 || Sq <= 0 || Sk <= 0 || Sk % 32 || Sq > (1 << 20) ||
      Sk > (1 << 20) || (head_dim != 128 && head_dim != 64))
    return 0;
  return workspace_bytes_of(q_heads, kv_heads, Sq, Sk, head_dim);
}

int amxfp4_attention_masked(const amx_format_t* fmt, int64_t q_heads, int64_t kv_heads, int64_t Sq, int64_t Sk,
                                       int64_t head_dim, const uint8_t* Q_codes, const uint8_t* Q_scales, const uint8_t* K_codes,
                                       const uint8_t* K_scales, const uint8_t* V_codes, const uint8_t* V_scales, float scale,
                                       const amx_scores_t* scores, int32_t causal, int64_t pos0, const int32_t* first,
                                       const int32_t* last, void* out_bf16, void* workspace, size_t workspace_bytes, void* stream) {
  if (!fmt) return report_error(AMX_ERR_INVALID_ARG, "attention_masked: fmt is NULL");
  if (fmt->elem != AMX_ELEM_FP4_E2M1 || fmt->scale < AMX_SCALE_E8M0_FLOOR || fmt->scale > AMX_SCALE_FP8_E4M3 ||
      (fmt->asymmetric != 0 && fmt->asymmetric != 1) || fmt->group_size == 0 || fmt->group_size < -1)
    return report_error(AMX_ERR_INVALID_ARG, "attention_masked: bad format");
  if (fmt->group_size != 32) return report_error(AMX_ERR_UNSUPPORTED, "attention_masked: groups of 32 only (one group per key tile)");
  if (head_dim != 128 && head_dim != 64) return report_error(AMX_ERR_UNSUPPORTED, "attention_masked: head_dim must be 128 or 64");
  if (q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads != 0 || q_heads > 65535)
    return report_error(AMX_ERR_INVALID_ARG, "attention_masked: q_heads must be a positive multiple of kv_heads (at most 65535)");
  if (Sq <= 0 || Sk <= 0 || Sk % 32 != 0 || Sk > (1 << 20) || Sq > (1 << 20))
    return report_error(AMX_ERR_INVALID_ARG, "attention_masked: Sq and Sk must be positive, at most 2^20, and Sk a multiple of 32");
  if ((causal != 0 && causal != 1) || pos0 < 0 || pos0 > (1 << 30))
    return report_error(AMX_ERR_INVALID_ARG, "attention_masked: causal must be 0 or 1, pos0 0 to 2^30");
  if (!(scale > 0.0f) || !(scale < 1.0e30f)) return report_error(AMX_ERR_INVALID_ARG, "attention_masked: scale must be a positive finite number");
  if (!scores_valid(scores))
    return report_error(AMX_ERR_INVALID_ARG, "attention_masked: cap must be 0 or 2^-20 to 2^20, slopes 4-byte aligned, reserved 0");
  if (!Q_codes || !Q_scales || !K_codes || !K_scales || !V_codes || !V_scales || !out_bf16)
    return report_error(AMX_ERR_INVALID_ARG, "attention_masked: NULL data pointer");
  if (!aligned(Q_codes, 16) || !aligned(K_codes, 16) || !aligned(V_codes, 16) || !aligned(Q_scales, 2) || !aligned(K_scales, 2) ||
      !aligned(V_scales, 2) || !aligned(out_bf16, 16) || !aligned(first, 4) || !aligned(last, 4))
    return report_error(AMX_ERR_INVALID_ARG, "attention_masked: codes and out need 16-byte, scales 2-byte, first and last 4-byte alignment");
  if (!workspace || workspace_bytes < workspace_bytes_of(q_heads, kv_heads, Sq, Sk, head_dim) || !aligned(workspace, 256))
    return report_error(AMX_ERR_WORKSPACE, "attention_masked: workspace missing, too small or not 256-byte aligned");

  MaskedWork w = {};
  w.first = first, w.last = last, w.Sq = (int)Sq, w.Sk = (int)Sk, w.kv_group = (int)(q_heads / kv_heads), w.causal = causal, w.pos0 = (int)pos0;
  w.scores = scores_of(scores, scale);
  // (keys behind the last row's position are not seen: no more chunks than there is room for)
  const int64_t keys = causal && pos0 + Sq < Sk ? pos0 + Sq : Sk;
  const int chunks = chunks_of(q_heads, Sq, (keys + 31) / 32, head_dim);
  const int64_t blocks = (Sq + kQueries - 1) / kQueries, workgroups = q_heads * blocks;
  const bool small = chunks == 1 && workgroups <= kMostOfPairs && Sk * head_dim <= kHeldElements, pairs = workgroups <= kMostOfPairs;
  if (workgroups > 256 && blocks > 1 && blocks <= kMostBlocks)
    w.turn = workgroups > kAtOnce ? (first || last ? (int)blocks : 0) : q_heads < 256 ? (int)(256 / q_heads) : 1;
  if (chunks > 1) {
    uint8_t* at = static_cast<uint8_t*>(workspace) + panels_bytes(q_heads, kv_heads, Sq, Sk, head_dim);
    w.maxima = reinterpret_cast<float*>(at);
    w.ends = reinterpret_cast<float2*>(at += rows_bytes(q_heads, Sq, chunks, 1));
    w.parts = reinterpret_cast<float*>(at += rows_bytes(q_heads, Sq, chunks, 2));
  }
  if (w.scores.slopes && !first && chunks == 1 && Sk >= kFarKeys)
    w.norms = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + panels_bytes(q_heads, kv_heads, Sq, Sk, head_dim));
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool asym = fmt->asymmetric != 0;
  uint16_t* Kp = static_cast<uint16_t*>(workspace);
  uint16_t* Vp = Kp + kv_heads * Sk * head_dim;
  hipError_t e = hipSuccess;
  if (!small) e = launch_expand_kv(fmt->scale, asym, K_codes, K_scales, Kp, V_codes, V_scales, Vp, Sk, head_dim, kv_heads, s);
  if (e != hipSuccess) return report_hip_error(e, "attention_masked: expansion launch");
  const MaskedOperands m = {Q_codes, Q_scales, K_codes, K_scales, V_codes, V_scales, asym ? 1 : 0, Kp, Vp, static_cast<uint16_t*>(out_bf16)};
  e = head_dim == 128 ? launch_masked<128>(fmt->scale, m, w, q_heads, chunks, small, pairs, s)
                      : launch_attention_masked_64(fmt->scale, m, w, q_heads, chunks, small, pairs, s);
  return e == hipSuccess ? AMX_OK : report_hip_error(e, "attention_masked launch");
}

}  // extern "C"
