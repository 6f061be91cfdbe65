// Fused quantized attention whose rows see a range of keys each, with capped scores and biases that fall with distance
// (include/amxfp4_scoring.h): the recurrence of attention.hip, on the same panels.
//
//   S^T[key, query] = K_tile[32 keys x D] . Q^T[D x 32 queries]        (MFMA 32x32x16 BF16, A = K rows, B = Q rows)
//   O^T[d, query]  += V^T[d x 32 keys]    . P^T[32 keys x 32 queries]  (A = V^T rows, B = the probabilities)
// In a 32x32 accumulator lane l holds column l % 32 (one query) and rows 8c + 4(l/32) + r (c, r = 0..3) in register 4c + r.
// Workgroup = 4 waves x 32 queries; a key tile's K and V fragments are brought into LDS once per workgroup by direct-to-LDS
// loads, double buffered.
//
// Ranges. A lane keeps its query's first key and the number of keys behind it; the mask of a score is one subtraction and one
// unsigned comparison. The wave's smallest first and largest last key bound the tiles it computes, the workgroup's those it loads; tiles that
// all of a wave's queries see wholly skip the mask. A query that has seen no key yet keeps its sums as they are.
#include "attention_tile.h"
#include "cast_math.h"
#include "dequant_regs.h"
#include "gemm_common.h"
#include "kernels.h"
#include "scoring.h"

namespace amx {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // (what is not a number stays so)
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}
constexpr int kWaves = 4, kQueries = 32 * kWaves;  // waves and queries of a workgroup

// What one launch reads beside the operands.
struct MaskedWork {
  const int32_t *first, *last;
  int Sq, Sk, kv_group, causal, pos0;
  Scores scores;
};

__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max(int v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
  return __builtin_amdgcn_readfirstlane(v);
}

template <int SCALE_KIND, int D, bool CAP, bool SLOPE>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 4 : 3) void attention_masked_kernel(const uint8_t* __restrict__ Q_codes, const uint8_t* __restrict__ Q_scales,
                                                                     int asym, const uint16_t* __restrict__ Kp,
                                                                     const uint16_t* __restrict__ Vp, uint16_t* __restrict__ out, MaskedWork w) {
  // FP8-E5M2 scales: probabilities as FP16 times 2^8, V^T biased by 2^-3, the 2^5 taken out with the row sum at the end
  constexpr bool kPF16 = SCALE_KIND == kScaleE5M2;
  constexpr int kFrags = D / 16;  // of K, and of V, in a key tile
  // two stages of (K tile, V tile), separate arrays so that loads into one stage are known not to alias reads of the other
  __shared__ __attribute__((aligned(1024))) uint8_t ldsK0[kFrags * kFragBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t ldsV0[kFrags * kFragBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t ldsK1[kFrags * kFragBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t ldsV1[kFrags * kFragBytes];
  __shared__ int edges[2][kWaves];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // x walks the query heads, a contiguous range of them per XCD where their number is a multiple of 8; y the query blocks,
  // the last ones, which have the most key tiles under a causal mask, first
  const int nheads = (int)gridDim.x;
  const int h = (nheads & 7) == 0 ? (int)(blockIdx.x & 7) * (nheads >> 3) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
  const int g = h / w.kv_group;
  const int qw = (int)(gridDim.y - 1 - blockIdx.y) * kQueries + wave * 32;
  const int Skv = (w.Sk + 63) & ~63;  // the V panel's keys

  // ---- the keys that this lane's query sees: from lo on, span more; rows past Sq repeat the last one
  const int query = min(qw + (lane & 31), w.Sq - 1), position = w.pos0 + query;
  int lo = 0, hi = w.Sk - 1;
  if (w.first) lo = max(w.first[query], 0);
  if (w.last) hi = min(w.last[query], hi);
  if (w.causal) hi = min(hi, position);
  const bool none = lo > hi || qw >= w.Sq;
  // (of the wave: the least and the greatest key that any query sees, and the range that all of them see)
  const int from = wave_min(none ? 0x7FFFFFFF : lo), to = wave_max(none ? -1 : hi);
  const int all_from = wave_max(none ? 0x7FFFFFFF : lo), all_to = wave_min(none ? -1 : hi);
  const uint32_t span = none ? 0u : (uint32_t)(hi - lo);
  if (none) lo = -0x7FFFFFFF;  // (no key is 0 keys behind it)
  if (lane == 0) edges[0][wave] = from, edges[1][wave] = to;
  __syncthreads();
  const int least = min(min(edges[0][0], edges[0][1]), min(edges[0][2], edges[0][3]));
  const int most = max(max(edges[1][0], edges[1][1]), max(edges[1][2], edges[1][3]));
  // key tiles that the workgroup loads, and that this wave computes (uniform)
  const int t_begin = most < 0 ? 0 : __builtin_amdgcn_readfirstlane(least >> 5);
  const int t_end = most < 0 ? 0 : __builtin_amdgcn_readfirstlane((most >> 5) + 1);
  const int own_begin = to < 0 ? 0 : from >> 5, own_end = to < 0 ? 0 : (to >> 5) + 1;

  const int64_t frags_k = (int64_t)(w.Sk / 32) * kFrags, frags_v = (int64_t)(D / 32) * (Skv / 16);
  const __amdgpu_buffer_rsrc_t Kr = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(Kp) + g * frags_k * kFragBytes), 0, (int)(frags_k * kFragBytes), 0x00020000);
  const __amdgpu_buffer_rsrc_t Vr = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(Vp) + g * frags_v * kFragBytes), 0, (int)(frags_v * kFragBytes), 0x00020000);
  const int lane_off = lane * 16;

  // this wave's share of tile T into stage (DK, DV): every fourth fragment of K, and of V (fragment f: row block f / 2, k-step f % 2)
#define AMX_MASKED_LOAD(T, DK, DV)                                                                                 \
  _Pragma("unroll") for (int i = 0; i < kFrags / kWaves; ++i) {                                                    \
    const int f = wave + kWaves * i;                                                                               \
    __builtin_amdgcn_raw_ptr_buffer_load_lds(Kr, (lds_ptr_t)((DK) + f * kFragBytes), 16, lane_off,                 \
                                             ((T) * kFrags + f) * kFragBytes, 0, 0);                               \
    __builtin_amdgcn_raw_ptr_buffer_load_lds(Vr, (lds_ptr_t)((DV) + f * kFragBytes), 16, lane_off,                 \
                                             ((f >> 1) * (Skv / 16) + (f & 1) + 2 * (T)) * kFragBytes, 0, 0);      \
  }

  // ---- this wave's 32 queries as the B operand of the first product, dequantized here from their codes
  bf16x8 qf[kFrags];
  {
    const int64_t row = (int64_t)h * w.Sq + query;
    const u32x4* codes = reinterpret_cast<const u32x4*>(Q_codes + row * (D / 2));
    const uint8_t* sb = Q_scales + row * (D / 32) * (asym ? 2 : 1);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {  // a group of 32: k-steps 2 i and 2 i + 1; lane half l takes words l, 2 + l
      const u32x4 c = codes[i];
      const uint32_t bp = sb[asym ? 2 * i : i], bn = asym ? sb[2 * i + 1] : bp;
      const uint32_t s_pos = f2u(scale_value<SCALE_KIND>(bp)), s_neg = f2u(scale_value<SCALE_KIND>(bn));
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t word = (lane >> 5) ? c[2 * k + 1] : c[2 * k];
        qf[2 * i + k] = __builtin_bit_cast(
            bf16x8, u32x4{dequant2_f32<true, 0>(word, s_pos, s_neg), dequant2_f32<true, 1>(word, s_pos, s_neg),
                          dequant2_f32<true, 2>(word, s_pos, s_neg), dequant2_f32<true, 3>(word, s_pos, s_neg)});
      }
    }
  }

  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  // Running maximum (in units of log2) and sum of this lane's query; the sum of the keys that this lane has, until the end. The maximum
  // starts finite: a query that has seen no key yet then has weights of 0 and a factor of 1 without any test.
  float m = -0x1.fffffep127f, l = 0.f;
  const int row_in_tile = 4 * (lane >> 5);    // key of register v: 8 (v / 4) + row_in_tile + v % 4
  // Distances are taken from the nearest key that the query sees: all its scores shift alike, and stay small where it sees far keys
  // only. In a tile in front of all the wave's nearest keys a score is f(q.k) + slope (key in the tile) - slope (distance of the tile's first
  // key): the second term is the last addition of f, the third is left to the maximum.
  const float slope = SLOPE ? w.scores.slopes[h] * kLog2e : 0.f;
  const int nearest = none ? 0 : max(lo, min(position, lo + (int)span));
  const int all_nearest = SLOPE ? wave_min(none ? 0x7FFFFFFF : nearest) : 0;
  float step[16];
  if constexpr (SLOPE) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      // (in scalar registers: an instruction takes one of those, and the scale is the one to move)
      float of = slope * (float)(8 * (v >> 2) + (v & 3));
      asm volatile("" : "+v"(of));
      step[v] = u2f((uint32_t)__builtin_amdgcn_readfirstlane((int)f2u(of)));
    }
  }
  float scale = w.scores.scale;
  if constexpr (SLOPE && !CAP) asm volatile("" : "+v"(scale));

  // scores X of the raw products S, plus PLUS (an expression in v)
#define AMX_MASKED_SCORES(X, S, SMALL, PLUS)                                                                       \
  if constexpr (!CAP) {                                                                                            \
    _Pragma("unroll") for (int v = 0; v < 16; ++v) (X)[v] = __builtin_fmaf((S)[v], scale, PLUS);                   \
  } else if (SMALL) {                                                                                              \
    asm volatile("");                                                                                              \
    _Pragma("unroll") for (int v = 0; v < 16; ++v) (X)[v] = capped_small((S)[v], w.scores, PLUS);                  \
  } else {                                                                                                         \
    asm volatile("");                                                                                              \
    _Pragma("unroll") for (int v = 0; v < 16; ++v) (X)[v] = capped((S)[v], w.scores.in, w.scores.cap) + (PLUS);    \
  }
  // one key tile from stage (CK, CV)
#define AMX_MASKED_TILE(T, CK, CV)                                                                                 \
  if ((T) >= own_begin && (T) < own_end) {                                                                         \
    f32x16 s;                                                                                                      \
    _Pragma("unroll") for (int v = 0; v < 16; ++v) s[v] = 0.f;                                                     \
    _Pragma("unroll") for (int kb = 0; kb < kFrags; ++kb) {                                                        \
      const bf16x8 a = *reinterpret_cast<const bf16x8*>((CK) + kb * kFragBytes + lane_off);                        \
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[kb], s, 0, 0, 0);                                          \
    }                                                                                                              \
    float x[16], shift = 0.f;                                                                                      \
    const int key0 = (T) * 32 + row_in_tile;                                                                       \
    bool small = false;                                                                                            \
    if constexpr (CAP) {                                                                                           \
      float size = __builtin_fabsf(s[0]);                                                                          \
      _Pragma("unroll") for (int v = 1; v < 16; ++v) size = fmaxf(size, __builtin_fabsf(s[v]));                    \
      small = __builtin_amdgcn_ballot_w64(size > w.scores.small) == 0; /* uniform */                               \
    }                                                                                                              \
    if (SLOPE && (T) * 32 + 31 <= all_nearest) { /* uniform: in front of the nearest keys */                       \
      asm volatile("");                                                                                            \
      AMX_MASKED_SCORES(x, s, small, step[v])                                                                      \
      shift = slope * (float)(nearest - key0);                                                                     \
    } else {                                                                                                       \
      asm volatile("");                                                                                            \
      AMX_MASKED_SCORES(x, s, small, 0.f)                                                                          \
      if constexpr (SLOPE) {                                                                                       \
        const float away = (float)(nearest - key0);                                                                \
        _Pragma("unroll") for (int v = 0; v < 16; ++v)                                                             \
          x[v] = __builtin_fmaf(-slope, __builtin_fabsf(away - (float)(8 * (v >> 2) + (v & 3))), x[v]);            \
      }                                                                                                            \
    }                                                                                                              \
    if ((T) * 32 < all_from || (T) * 32 + 31 > all_to) { /* some key of the tile is not seen by some query */      \
      asm volatile(""); /* (keeps the branch: most tiles skip the masking altogether) */                           \
      _Pragma("unroll") for (int v = 0; v < 16; ++v)                                                               \
        if ((uint32_t)(key0 + 8 * (v >> 2) + (v & 3)) - (uint32_t)lo > span) x[v] = -__builtin_inff();             \
    }                                                                                                              \
    float mx = x[0];                                                                                               \
    _Pragma("unroll") for (int v = 1; v < 16; ++v) mx = fmaxf(mx, x[v]);                                           \
    const float own = mx - shift; /* the lane's largest score; the query's other keys are in lane ^ 32 */          \
    const auto both = __builtin_amdgcn_permlane32_swap(f2u(own), f2u(own), false, false);                          \
    const float top = fmaxf(u2f(both[0]), u2f(both[1])), m_new = fmaxf(m, top);                                    \
    const float alpha = __builtin_amdgcn_exp2f(m - m_new), pmax = __builtin_amdgcn_exp2f(top - m_new);             \
    /* what is subtracted from x. The score that holds the maximum gives exactly 0, whatever the shift rounds */   \
    float base = m_new;                                                                                            \
    if constexpr (SLOPE) base = own == m_new ? mx : m_new + shift;                                                 \
    m = m_new;                                                                                                     \
    /* The cast of the 32 weights of each query as one group, of which pmax is the largest. FP8 scales: the exponentials are of the    \
       quotients, 2^(x - base - log2 S) (the rounding of base + log2 S is that of a score), and their sum takes S back.                \
       A scale of 0 (all weights below 2^-17) casts them to 0. */                                                  \
    uint32_t pb[8];                                                                                                \
    float sum = 0.f;                                                                                               \
    if constexpr (SCALE_KIND == kScaleE5M2 || SCALE_KIND == kScaleE4M3) {                                          \
      float S, R;                                                                                                  \
      fp8_scale_inexact<SCALE_KIND>(pmax, S, R);                                                                   \
      const float divide = S > 0.f ? S : 1.0f;                                                                     \
      base += __builtin_amdgcn_logf(divide);                                                                       \
      _Pragma("unroll") for (int v = 0; v < 16; ++v) x[v] = __builtin_amdgcn_exp2f(x[v] - base), sum += x[v];      \
      sum *= divide;                                                                                               \
      const _Float16 s_half = (_Float16)S; /* E5M2: exact, subnormals included */                                  \
      _Pragma("unroll") for (int i = 0; i < 8; ++i) {                                                              \
        const uint32_t code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(f2u(x[2 * i]), x[2 * i], x[2 * i + 1], 1.0f, 0); \
        if constexpr (kPF16) {                                                                                     \
          const f16x2 e = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, 256.0f, 0);                               \
          pb[i] = __builtin_bit_cast(uint32_t, e * (f16x2){s_half, s_half});                                       \
        } else {                                                                                                   \
          const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0);                                 \
          pb[i] = __builtin_amdgcn_perm(f2u(e[1] * S), f2u(e[0] * S), 0x07060302u); /* exact: 6 significant bits */ \
        }                                                                                                          \
      }                                                                                                            \
    } else {                                                                                                       \
      _Pragma("unroll") for (int v = 0; v < 16; ++v) x[v] = __builtin_amdgcn_exp2f(x[v] - base), sum += x[v];      \
      AMX_ATTENTION_TILE_CAST(x, pmax, pb, false)                                                                  \
    }                                                                                                              \
    l = __builtin_fmaf(l, alpha, sum);                                                                             \
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) { /* the maximum moved for some query: rescale */        \
      _Pragma("unroll") for (int db = 0; db < D / 32; ++db)                                                        \
        _Pragma("unroll") for (int v = 0; v < 16; ++v) o[db][v] *= alpha;                                          \
    }                                                                                                              \
    _Pragma("unroll") for (int j = 0; j < 2; ++j) {                                                                \
      const u32x4 b = {pb[4 * j], pb[4 * j + 1], pb[4 * j + 2], pb[4 * j + 3]};                                    \
      _Pragma("unroll") for (int db = 0; db < D / 32; ++db) {                                                      \
        const u32x4 a = *reinterpret_cast<const u32x4*>((CV) + (db * 2 + j) * kFragBytes + lane_off);              \
        if constexpr (kPF16)                                                                                       \
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), \
                                                         o[db], 0, 0, 0);                                          \
        else                                                                                                       \
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),                           \
                                                          __builtin_bit_cast(bf16x8, b), o[db], 0, 0, 0);          \
      }                                                                                                            \
    }                                                                                                              \
  }

  if (t_begin < t_end) AMX_MASKED_LOAD(t_begin, ldsK0, ldsV0);
  AMX_WAIT_VMCNT(0);
  AMX_BARRIER();
  for (int t = t_begin; t < t_end; t += 2) {
    // stage 1 was last read during tile t - 1; the barrier that ended it lets every wave refill it now
    if (t + 1 < t_end) AMX_MASKED_LOAD(t + 1, ldsK1, ldsV1);
    AMX_MASKED_TILE(t, ldsK0, ldsV0);
    AMX_WAIT_VMCNT(0);
    AMX_BARRIER();
    if (t + 1 < t_end) {  // uniform over the workgroup
      if (t + 2 < t_end) AMX_MASKED_LOAD(t + 2, ldsK0, ldsV0);
      AMX_MASKED_TILE(t + 1, ldsK1, ldsV1);
      AMX_WAIT_VMCNT(0);
      AMX_BARRIER();
    }
  }
#undef AMX_MASKED_TILE
#undef AMX_MASKED_SCORES
#undef AMX_MASKED_LOAD

  // out[query][h * D + d] = O^T[d][query] / l; register 4c + r of row block db is d = 32 db + 8 c + 4 (lane / 32) + r
  const auto halves = __builtin_amdgcn_permlane32_swap(f2u(l), f2u(l), false, false);
  l = u2f(halves[0]) + u2f(halves[1]);
  if (qw + (lane & 31) < w.Sq) {
    const float inv = l == 0.f ? 0.f : (kPF16 ? 0.03125f : 1.0f) / l;
    uint16_t* dst = out + ((int64_t)query * nheads + h) * D + row_in_tile;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<uint2*>(dst + db * 32 + c * 8) = make_uint2(
            pack_bf16(o[db][4 * c] * inv, o[db][4 * c + 1] * inv), pack_bf16(o[db][4 * c + 2] * inv, o[db][4 * c + 3] * inv));
  }
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace
}  // namespace amx

using namespace amx;

extern "C" int amxfp4_attention_masked(const amx_format_t* fmt, int64_t q_heads, int64_t kv_heads, int64_t Sq, int64_t Sk,
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
  if (!workspace || workspace_bytes < attention_workspace_bytes(q_heads, kv_heads, Sq, Sk, head_dim) || !aligned(workspace, 256))
    return report_error(AMX_ERR_WORKSPACE, "attention_masked: workspace missing, too small or not 256-byte aligned");

  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool asym = fmt->asymmetric != 0;
  uint16_t* Kp = static_cast<uint16_t*>(workspace);
  uint16_t* Vp = Kp + kv_heads * Sk * head_dim;
  hipError_t e = launch_expand_kv(fmt->scale, asym, K_codes, K_scales, Kp, V_codes, V_scales, Vp, Sk, head_dim, kv_heads, s);
  if (e != hipSuccess) return report_hip_error(e, "attention_masked: expansion launch");
  const MaskedWork w = {first, last, (int)Sq, (int)Sk, (int)(q_heads / kv_heads), causal, (int)pos0, scores_of(scores, scale)};
  const dim3 grid((unsigned)q_heads, (unsigned)((Sq + kQueries - 1) / kQueries));
  auto go = [&]<int SK, int D, bool CAP, bool SLOPE>() {
    hipLaunchKernelGGL((attention_masked_kernel<SK, D, CAP, SLOPE>), grid, dim3(64 * kWaves), 0, s, Q_codes, Q_scales, asym ? 1 : 0,
                       Kp, Vp, static_cast<uint16_t*>(out_bf16), w);
  };
  auto with_scores = [&]<int SK, int D>() {
    if (w.scores.cap > 0.f)
      w.scores.slopes ? go.template operator()<SK, D, true, true>() : go.template operator()<SK, D, true, false>();
    else
      w.scores.slopes ? go.template operator()<SK, D, false, true>() : go.template operator()<SK, D, false, false>();
  };
  auto with_scale = [&]<int SK>() { head_dim == 128 ? with_scores.template operator()<SK, 128>() : with_scores.template operator()<SK, 64>(); };
  switch (fmt->scale) {
    case AMX_SCALE_FP8_E5M2: with_scale.template operator()<kScaleE5M2>(); break;
    case AMX_SCALE_FP8_E4M3: with_scale.template operator()<kScaleE4M3>(); break;
    case AMX_SCALE_E8M0_FLOOR: with_scale.template operator()<kScaleE8M0Floor>(); break;
    default: with_scale.template operator()<kScaleE8M0Round>();
  }
  e = hipGetLastError();
  return e == hipSuccess ? AMX_OK : report_hip_error(e, "attention_masked launch");
}
