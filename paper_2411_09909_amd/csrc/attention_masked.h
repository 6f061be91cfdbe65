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
// all of a wave's queries see wholly skip the mask. The running maximum begins at the lowest finite number, so that a query that has seen no
// key yet has weights of 0 and a factor of 1 without a test.
// Scores. In units of log2. Where they rise with the products (no slopes) the maximum is taken of those, and a score less the maximum and the
// scale's logarithm is one multiply-add (capped: the last step of a polynomial). A slope is a constant of the key's place in the tile, added by
// that step too, and one number for the tile, which only the maximum sees.
// Split rows (kMaxima, kPart). The cast of a tile depends on the running maximum of all keys before it, so chunks of the keys are not
// independent; but the maximum is a fifth of the work (half of the products and no exponentials). One launch takes every chunk's
// maxima, the next starts each chunk with those of the chunks before it, and the join adds the sums up: the same numbers as without the split.
//
// Bound and measured (us a call with the expansion of K and V in front; cards differ by 4 %): 32 / 8 heads of 128 x 8192 with nothing but the causal mask 536 = 1026
// TFLOP/s of the visible half (amxfp4_attention: 567), the rate of a library's product of 8192^3 being 1380 to 1420. A tile of a wave is 16 products of
// 32 cycles and some 600 to 860 cycles of vector instructions (with slopes the maximum moves in every tile, and 64 registers of the output with it); counters: the
// vector unit 83 % busy, the products 44 %, one beside the other. With slopes 590, and 364 to 392 without the tiles that are too far to count. 2048 rows of nine
// documents with capped scores 39 to 42, of which the expansion is 8: blocks of very different length, all running at once (the longest alone takes 37). The first form took 834 and 55: the
// accumulator in the second half of the register file, copied back and forth (waves_per_eu given no lower bound), the mask computed for every
// tile, exp2 and a reciprocal for each capped score, two exchanges through LDS to a tile.
#pragma once
#include "attention_tile.h"
#include "cast_math.h"
#include "dequant_regs.h"
#include "gemm_common.h"
#include "kernels.h"
#include "scoring.h"

namespace amx {

// What one launch reads beside the operands.
struct MaskedWork {
  const int32_t *first, *last;
  int Sq, Sk, kv_group, causal, pos0;
  float *maxima, *parts;  // of split rows: [head][row][chunk]; [head][chunk][row][D]
  float2* ends;           // [head][chunk][row]: maximum and sum
  const float* norms;     // [key head][key tile]: the largest norm of a key of the tile; nullptr: no tiles are left out
  int turn;  // query blocks to a turn of the workgroups over the compute units (0: the last block first)
  Scores scores;
};

// The operands, the panels of K and V and the output of a launch.
struct MaskedOperands {
  const uint8_t *Q_codes, *Q_scales, *K_codes, *K_scales, *V_codes, *V_scales;
  int asym;
  const uint16_t *K_panel, *V_panel;
  uint16_t* out;
};

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // (what is not a number stays so)
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}
// Elements of a head's keys up to which K and V, 64 KB of LDS, are held whole: every workgroup reads them as codes then, with no expansion in front.
// 12 heads of 64 x 77 10.0 -> 8.3 us, 32 / 8 heads of 128 x 20 and x 128 9.6 -> 8.0; 64 heads of 64 x 250 13.6 either way.
constexpr int kHeldElements = 16384;
constexpr float kLowest = -0x1.fffffep127f;
// Added to a sum of up to 128 squares that is to bound a norm from above: squares below 2^-126, those of numbers below 2^-63, are too small or lost
// (a scale of 2^80 makes large scores of such numbers).
constexpr float kLostSquares = 0x1p-118f;
constexpr int kWaves = 4, kQueries = 32 * kWaves;  // waves and queries of a workgroup

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

// NT: key tiles to a step, 1 or 2. PASS: kWhole; kMaxima and kPart, a chunk of a workgroup's key tiles; kHeld, all of K and V out of
// their codes (the last four pointers, which only it reads) into LDS at once.
enum { kWhole, kMaxima, kPart, kHeld };
template <int SCALE_KIND, int D, bool CAP, bool SLOPE, int NT, int PASS>
__global__ __launch_bounds__(64 * kWaves, NT == 2 ? 2 : D == 64 ? 4 : 3) void attention_masked_kernel(
    const uint8_t* __restrict__ Q_codes, const uint8_t* __restrict__ Q_scales, int asym, const uint16_t* __restrict__ Kp,
    const uint16_t* __restrict__ Vp, uint16_t* __restrict__ out, MaskedWork w, const uint8_t* __restrict__ K_codes,
    const uint8_t* __restrict__ K_scales, const uint8_t* __restrict__ V_codes, const uint8_t* __restrict__ V_scales) {
  // FP8-E5M2 scales: probabilities as FP16 times 2^8, V^T biased by 2^-3, the 2^5 taken out with the row sum at the end
  constexpr bool kPF16 = SCALE_KIND == kScaleE5M2;
  // Whether a wave goes before the others of its SIMD while it multiplies: 32 / 8 heads of 128 x 4096, causal, 160 -> 154 us, 64 / 8 x 1504 39.7 -> 38.7,
  // a window of 4096 over 1000 rows of heads of 64, split, 110 -> 106; pairs of tiles, 2048 rows, 74.6 -> 76.2, heads of 64 tile by tile 435 -> 444.
  constexpr bool kProductsFirst = PASS == kPart || (PASS == kWhole && NT == 1 && D == 128);
  constexpr int kFrags = D / 16, kTileBytes = kFrags * kFragBytes;  // of K, and of V, in a key tile
  // two stages of (K tiles, V tiles), separate arrays so that loads into one stage are known not to alias reads of the other
  __shared__ __attribute__((aligned(1024))) uint8_t ldsK0[PASS == kHeld ? 1 : NT * kTileBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t ldsV0[PASS == kMaxima || PASS == kHeld ? 1 : NT * kTileBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t ldsK1[PASS == kHeld ? 1 : NT * kTileBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t ldsV1[PASS == kMaxima || PASS == kHeld ? 1 : NT * kTileBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t all_tiles[PASS == kHeld ? 2 * kHeldElements * 2 : 1];  // K's tiles, then V's, an even number
  __shared__ int edges[2][kWaves];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // x walks the query heads, a contiguous range of them per XCD where their number is a multiple of 8; y the query blocks: without ranges the
  // last ones, which have the most key tiles under a causal mask, first
  const int nheads = (int)gridDim.x;
  int h = (nheads & 7) == 0 ? (int)(blockIdx.x & 7) * (nheads >> 3) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
  // (With far tiles left out heads of steep slopes have little to do: neighbours go to different XCDs, back and forth, and a compute unit's next
  // workgroup, some 32 further on its XCD, is of another head than its last.)
  if (SLOPE && w.norms && (nheads & 7) == 0) {
    const int n = nheads >> 3, slot = (int)((blockIdx.x >> 3) + blockIdx.y * (uint32_t)n / 32) % n, xcd = (int)(blockIdx.x & 7);
    h = 8 * slot + (slot & 1 ? 7 - xcd : xcd);
  }
  const int g = h / w.kv_group;
  const int blocks = (int)gridDim.y;
  int block = blocks - 1 - (int)blockIdx.y;
  if (w.turn > 0) {  // uniform: the blocks by the keys between their first row's first and their last row's last, longest first
    const int b = min(lane, blocks - 1), row0 = b * kQueries, row1 = min(row0 + kQueries, w.Sq) - 1;
    int a = 0, z = w.Sk - 1;
    if (w.first) a = max(w.first[row0], 0);
    if (w.last) z = min(w.last[row1], z);
    if (w.causal) z = min(z, w.pos0 + row1);
    const int length = lane < blocks ? max(z - a + 1, 0) : -1;
    int rank = 0;
    for (int o = 0; o < blocks; ++o) {
      const int other = __builtin_amdgcn_readlane(length, o);
      rank += other > length || (other == length && o > lane) ? 1 : 0;
    }
    const int turn = (int)blockIdx.y / w.turn, in_turn = (int)blockIdx.y - turn * w.turn, size = min(w.turn, blocks - turn * w.turn);
    const int wanted = turn & 1 ? turn * w.turn + size - 1 - in_turn : (int)blockIdx.y;
    block = (int)__builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < blocks && rank == wanted));
  }
  const int qw = block * kQueries + wave * 32;
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
  int t_begin = most < 0 ? 0 : __builtin_amdgcn_readfirstlane(least >> 5);
  int t_end = most < 0 ? 0 : __builtin_amdgcn_readfirstlane((most >> 5) + 1);
  int own_begin = to < 0 ? 0 : from >> 5, own_end = to < 0 ? 0 : (to >> 5) + 1;
  const int chunk = (int)blockIdx.z, chunks = (int)gridDim.z;
  if constexpr (PASS == kMaxima || PASS == kPart) {
    // (whole steps: what a step has beyond the block's last tile is masked, what it had beyond a chunk's would not be)
    static_assert(NT == 2, "chunks of pairs");
    const int steps = (t_end - t_begin + 1) / 2;
    t_end = min(t_end, t_begin + 2 * (steps * (chunk + 1) / chunks)), t_begin += 2 * (steps * chunk / chunks);
    own_begin = max(own_begin, t_begin), own_end = min(own_end, t_end);
  }

  const int64_t frags_k = (int64_t)(w.Sk / 32) * kFrags, frags_v = (int64_t)(D / 32) * (Skv / 16);
  const __amdgpu_buffer_rsrc_t Kr = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(Kp) + g * frags_k * kFragBytes), 0, (int)(frags_k * kFragBytes), 0x00020000);
  const __amdgpu_buffer_rsrc_t Vr = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(Vp) + g * frags_v * kFragBytes), 0, (int)(frags_v * kFragBytes), 0x00020000);
  const int lane_off = lane * 16;

  // this wave's share of the tiles from `t` on into stage (K, V): every fourth fragment of either (fragment f of V: row block f / 2, k-step
  // f % 2). Behind the last tile that one comes again.
  auto load = [&](int t, uint8_t* K, uint8_t* V) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int tile = NT == 1 ? t : min(t + n, t_end - 1);
#pragma unroll
      for (int i = 0; i < kFrags / kWaves; ++i) {
        const int f = wave + kWaves * i;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(Kr, (lds_ptr_t)(K + n * kTileBytes + f * kFragBytes), 16, lane_off,
                                                 (tile * kFrags + f) * kFragBytes, 0, 0);
        if constexpr (PASS != kMaxima)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(Vr, (lds_ptr_t)(V + n * kTileBytes + f * kFragBytes), 16, lane_off,
                                                   ((f >> 1) * (Skv / 16) + (f & 1) + 2 * tile) * kFragBytes, 0, 0);
      }
    }
  };

  const int small_tiles = (t_end - t_begin + 1) & ~1;
  if constexpr (PASS == kHeld) {
    // fragments of both, dealt over the waves; lane l holds row l % 32 (a key; a dimension of V), elements 8 (l / 32) .. of 16, V's keys in
    // the accumulator's order
    const int r = lane & 31, half = lane >> 5;
    auto scales = [&](const uint8_t* from, int64_t group) {
      return asym ? (uint32_t) * reinterpret_cast<const uint16_t*>(from + 2 * group) : from[group] * 0x101u;
    };
    for (int i = wave; i < small_tiles * kFrags; i += kWaves) {
      const int n = i / kFrags, f = i % kFrags, tile = min(t_begin + n, t_end - 1);
      const int64_t key = (int64_t)g * w.Sk + tile * 32 + r;
      const uint32_t kw = *reinterpret_cast<const uint32_t*>(K_codes + key * (D / 2) + 8 * f + 4 * half);
      const uint32_t kb = scales(K_scales, key * (D / 32) + f / 2);
      const int64_t dim = (int64_t)g * D + 32 * (f >> 1) + r;
      const uint16_t* v = reinterpret_cast<const uint16_t*>(V_codes + dim * (w.Sk / 2) + tile * 16 + 8 * (f & 1) + 2 * half);
      const uint32_t vw = v[0] | (uint32_t)v[2] << 16;
      const uint32_t vb = scales(V_scales, dim * (w.Sk / 32) + tile);
      auto exact = [&](uint32_t word, uint32_t bytes) {
        const uint32_t p = f2u(scale_value<SCALE_KIND>(bytes & 0xFF)), q = f2u(scale_value<SCALE_KIND>(bytes >> 8));
        return u32x4{dequant2_f32<true, 0>(word, p, q), dequant2_f32<true, 1>(word, p, q), dequant2_f32<true, 2>(word, p, q),
                     dequant2_f32<true, 3>(word, p, q)};
      };
      *reinterpret_cast<u32x4*>(all_tiles + i * kFragBytes + lane_off) = exact(kw, kb);
      u32x4 values;
      if constexpr (kPF16) {
        const uint32_t p = (vb & 0x7F) << 8, q = vb & 0x7F00;  // the byte is the upper byte of an FP16, and the scale is wanted twice
        values = dequant_word<kScaleE5M2, true>(vw, p | p << 16, q | q << 16);
      } else {
        values = exact(vw, vb);
      }
      *reinterpret_cast<u32x4*>(all_tiles + (small_tiles * kFrags + i) * kFragBytes + lane_off) = values;
    }
  } else if (!(SLOPE && PASS == kWhole)) {
    if (t_begin < t_end) load(t_begin, ldsK0, ldsV0);
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

  // ---- far tiles. A key whose score is 60 below a row's maximum in units of log2 has less than 2^-60 of the row's sum, and is left out where a bound
  // on its score says so: the result is off by that much of the key's value. (Values as large as to show it, 2^50 times the near ones, are the caller's
  // to keep out.) Tiles in front of the first that may have others need not be looked at: their maximum is as far below, so that what is
  // cast against it would be as small. |q . k| <= |q| |k| bounds the scores: a tile's by its largest key, the maximum's by the nearest
  // key, from which the distances count.
  const float slope = SLOPE ? slope_of(w.scores, (uint32_t)h) : 0.f;
  const int nearest = none ? 0 : max(lo, min(position, lo + (int)span));
  const int all_nearest = SLOPE ? wave_min(none ? 0x7FFFFFFF : nearest) : 0;
  if constexpr (SLOPE && PASS == kWhole) {
    if (w.norms && slope > 0.f) {  // uniform
      float size = 0.f;
#pragma unroll
      for (int kb = 0; kb < kFrags; ++kb)
#pragma unroll
        for (int i = 0; i < 8; ++i) size = __builtin_fmaf((float)qf[kb][i], (float)qf[kb][i], size);
      size += __shfl_xor(size, 32, 64);
      const float* norms = w.norms + (int64_t)g * (w.Sk / 32);
      size = __builtin_sqrtf(size + kLostSquares) * w.scores.scale * 1.001f;  // (the cap makes scores smaller only)
      float near = none ? 0.f : norms[nearest >> 5];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) size = fmaxf(size, __shfl_xor(size, d, 64)), near = fmaxf(near, __shfl_xor(near, d, 64));
      int skipped = own_begin;
      for (; skipped < own_end; skipped += 64) {
        const int t = skipped + lane;
        const bool far = t < own_end && size * (norms[min(t, w.Sk / 32 - 1)] + near) + 60.f < slope * (float)(all_nearest - 32 * t - 31);
        const uint64_t needed = ~__builtin_amdgcn_ballot_w64(far);
        if (needed) {
          skipped += (int)__builtin_ctzll(needed);
          break;
        }
      }
      own_begin = min(skipped, own_end);
      __syncthreads();  // (the edges have been read)
      if (lane == 0) edges[0][wave] = own_begin < own_end ? own_begin : 0x7FFFFFFF;
      __syncthreads();
      const int first = min(min(edges[0][0], edges[0][1]), min(edges[0][2], edges[0][3]));
      t_begin = __builtin_amdgcn_readfirstlane(min(max(first, t_begin), t_end));
    }
    if (t_begin < t_end) load(t_begin, ldsK0, ldsV0);
  }

  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
  // Running maximum (in units of log2) and sum of this lane's query; the sum of the keys that this lane has, until the end. The maximum
  // starts finite: a query that has seen no key yet then has weights of 0 and a factor of 1 without any test.
  float m = kLowest, l = 0.f;
  if constexpr (PASS == kPart)
    for (int c = 0; c < chunk; ++c) m = fmaxf(m, w.maxima[((int64_t)h * w.Sq + query) * chunks + c]);
  const int row_in_tile = 4 * (lane >> 5);    // key of register v: 8 (v / 4) + row_in_tile + v % 4
  // Distances are taken from the nearest key that the query sees: all its scores shift alike, and stay small where it sees far keys
  // only. In a tile in front of all the wave's nearest keys a score is f(q.k) + slope (key in the tile) - slope (distance of the tile's first
  // key): the second term is the last addition of f, the third is left to the maximum.
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

  // Scores of a tile's raw products, each plus plus(v). (The empty statements keep the branches, here and below: without them both sides are
  // computed and selected from.)
  auto scores = [&](const f32x16& s, bool small, float (&x)[16], auto plus) __attribute__((always_inline)) {
    if constexpr (!CAP) {
#pragma unroll
      for (int v = 0; v < 16; ++v) x[v] = __builtin_fmaf(s[v], scale, plus(v));
    } else if (small) {
      asm volatile("");
#pragma unroll
      for (int v = 0; v < 16; ++v) x[v] = capped_small(s[v], w.scores, plus(v));
    } else {
      asm volatile("");
#pragma unroll
      for (int v = 0; v < 16; ++v) x[v] = capped(s[v], w.scores.in, w.scores.cap) + plus(v);
    }
  };

  // NT key tiles from `t` on, out of stage (K, V)
  auto step_of = [&](int t, const uint8_t* K, const uint8_t* V) __attribute__((always_inline)) {
    if (t + NT <= own_begin || t >= own_end) return;
    f32x16 s[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[n][v] = 0.f;
    if constexpr (kProductsFirst) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kb = 0; kb < kFrags; ++kb)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const bf16x8 a = *reinterpret_cast<const bf16x8*>(K + n * kTileBytes + kb * kFragBytes + lane_off);
        s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[kb], s[n], 0, 0, 0);
      }
    if constexpr (kProductsFirst) __builtin_amdgcn_s_setprio(0);
    const bool all_seen = t * 32 >= all_from && (t + NT) * 32 - 1 <= all_to;  // every key of the tiles, by every query (uniform)
    bool small = false;
    if constexpr (CAP) {
      float size = __builtin_fabsf(s[0][0]);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) size = fmaxf(size, __builtin_fabsf(s[n][v]));
      small = __builtin_amdgcn_ballot_w64(size > w.scores.small) == 0;
    }
    // ---- the lane's largest score of each tile, the query's (its other keys are in lane ^ 32), and the running maxima. own: what is
    // subtracted from a score for it (the one that holds the maximum gives exactly 0, whatever the shift rounds)
    float x[NT][16], base[NT], alpha[NT], pmax[NT];
    auto maxima = [&](int n, float own, float shift) __attribute__((always_inline)) {
      if constexpr (PASS == kMaxima) {
        m = fmaxf(m, own - shift);
        return;
      }
      const auto both = __builtin_amdgcn_permlane32_swap(f2u(own - shift), f2u(own - shift), false, false);
      const float top = fmaxf(u2f(both[0]), u2f(both[1])), m_new = fmaxf(m, top);
      alpha[n] = __builtin_amdgcn_exp2f(m - m_new), pmax[n] = __builtin_amdgcn_exp2f(top - m_new);
      // A power-of-two scale halves where the largest weight falls just below 1. Scores that tie with the running maximum (with dyadic slopes and
      // scales they often do) are up to some roundings away from it here: they count as it.
      if constexpr (SCALE_KIND != kScaleE5M2 && SCALE_KIND != kScaleE4M3)
        pmax[n] = m_new - top <= __builtin_fmaf(__builtin_fabsf(m_new), 0x1p-22f, 0x1p-16f) ? 1.0f : pmax[n];
      base[n] = !SLOPE ? m_new : own - shift == m_new ? own : m_new + shift;
      m = m_new;
    };
    // The scale of the cast, as a divisor: FP8 scales take the exponentials of the quotients, 2^(x - base - log2 S) (the rounding of base +
    // log2 S is that of a score), and their sum takes S back. A scale of 0 (all weights below 2^-17) casts them to 0.
    float S[NT], divide[NT];
    auto scale_of_cast = [&](int n) __attribute__((always_inline)) {
      if constexpr (SCALE_KIND == kScaleE5M2 || SCALE_KIND == kScaleE4M3) {
        float inverse;
        fp8_scale_inexact<SCALE_KIND>(pmax[n], S[n], inverse);
        divide[n] = S[n] > 0.f ? S[n] : 1.0f;
        base[n] += __builtin_amdgcn_logf(divide[n]);
      } else {
        float inverse;
        (void)encode_scale_sr<SCALE_KIND>(pmax[n], S[n], inverse);
        divide[n] = 1.0f;
      }
    };
    if (!SLOPE && all_seen) {  // scores rise with the products: the largest of those first, then each less its base in one go
      asm volatile("");
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float most = s[n][0];
#pragma unroll
        for (int v = 1; v < 16; ++v) most = fmaxf(most, s[n][v]);
        float top = most * scale;
        if constexpr (CAP) top = small ? capped_small(most, w.scores, 0.f) : capped(most, w.scores.in, w.scores.cap);
        maxima(n, top, 0.f);
        if constexpr (PASS == kMaxima) continue;
        scale_of_cast(n);
        const float less = -base[n];
        scores(s[n], small, x[n], [&](int) { return less; });
      }
    } else {
      asm volatile("");
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int key0 = (t + n) * 32 + row_in_tile;
        float shift = 0.f;
        if (SLOPE && (t + n) * 32 + 31 <= all_nearest) {  // uniform: in front of the nearest keys
          asm volatile("");
          scores(s[n], small, x[n], [&](int v) { return step[v]; });
          shift = slope * (float)(nearest - key0);
        } else {
          asm volatile("");
          scores(s[n], small, x[n], [](int) { return 0.f; });
          if constexpr (SLOPE) {
            const float away = (float)(nearest - key0);
#pragma unroll
            for (int v = 0; v < 16; ++v) x[n][v] = __builtin_fmaf(-slope, __builtin_fabsf(away - (float)(8 * (v >> 2) + (v & 3))), x[n][v]);
          }
        }
        if (!all_seen) {
          asm volatile("");
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if ((uint32_t)(key0 + 8 * (v >> 2) + (v & 3)) - (uint32_t)lo > span) x[n][v] = -__builtin_inff();
        }
        float own = x[n][0];
#pragma unroll
        for (int v = 1; v < 16; ++v) own = fmaxf(own, x[n][v]);
        maxima(n, own, shift);
        if constexpr (PASS == kMaxima) continue;
        scale_of_cast(n);
#pragma unroll
        for (int v = 0; v < 16; ++v) x[n][v] -= base[n];
      }
    }
    if constexpr (PASS == kMaxima) return;
    // ---- the weights, their sum and their cast, 32 of a query as one group
    uint32_t pb[NT][8];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float sum = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) x[n][v] = __builtin_amdgcn_exp2f(x[n][v]), sum += x[n][v];
      l = __builtin_fmaf(l, alpha[n], sum * divide[n]);
      const _Float16 s_half = (_Float16)S[n];  // (E5M2: exact, subnormals included)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = x[n][2 * i], b = x[n][2 * i + 1];
        if constexpr (SCALE_KIND == kScaleE5M2) {
          const uint32_t code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(f2u(a), a, b, 1.0f, 0);
          pb[n][i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, 256.0f, 0) * (f16x2){s_half, s_half});
        } else if constexpr (SCALE_KIND == kScaleE4M3) {
          const uint32_t code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(f2u(a), a, b, 1.0f, 0);
          const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0);
          pb[n][i] = __builtin_amdgcn_perm(f2u(e[1] * S[n]), f2u(e[0] * S[n]), 0x07060302u);  // exact: 6 significant bits
        } else {  // the conversions apply a power of two themselves (its exponent field: the first divides, the second multiplies)
          const uint32_t code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(f2u(a), a, b, S[n], 0);
          pb[n][i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, S[n], 0));
        }
      }
    }
    // ---- O^T
    if constexpr (kProductsFirst) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (__builtin_amdgcn_ballot_w64(alpha[n] != 1.0f) != 0) {  // the maximum moved for some query: rescale
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[db][v] *= alpha[n];
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x4 b = {pb[n][4 * j], pb[n][4 * j + 1], pb[n][4 * j + 2], pb[n][4 * j + 3]};
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const u32x4 a = *reinterpret_cast<const u32x4*>(V + n * kTileBytes + (db * 2 + j) * kFragBytes + lane_off);
          if constexpr (kPF16)
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), o[db], 0, 0, 0);
          else
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), o[db], 0, 0, 0);
        }
      }
    }
    if constexpr (kProductsFirst) __builtin_amdgcn_s_setprio(0);
  };

  if constexpr (PASS == kHeld) {
    __syncthreads();
    for (int t = t_begin; t < t_end; t += NT)
      step_of(t, all_tiles + (t - t_begin) * kTileBytes, all_tiles + (small_tiles + t - t_begin) * kTileBytes);
  } else {
    AMX_WAIT_VMCNT(0);
    AMX_BARRIER();
    for (int t = t_begin; t < t_end; t += 2 * NT) {
      // stage 1 was last read in the step before; the barrier that ended it lets every wave refill it now
      if (t + NT < t_end) load(t + NT, ldsK1, ldsV1);
      step_of(t, ldsK0, ldsV0);
      AMX_WAIT_VMCNT(0);
      AMX_BARRIER();
      if (t + NT < t_end) {  // uniform over the workgroup
        if (t + 2 * NT < t_end) load(t + 2 * NT, ldsK0, ldsV0);
        step_of(t + NT, ldsK1, ldsV1);
        AMX_WAIT_VMCNT(0);
        AMX_BARRIER();
      }
    }
  }

  const bool stored = qw + (lane & 31) < w.Sq;
  if constexpr (PASS == kMaxima) {
    const auto both = __builtin_amdgcn_permlane32_swap(f2u(m), f2u(m), false, false);
    if (stored && lane < 32) w.maxima[((int64_t)h * w.Sq + query) * chunks + chunk] = fmaxf(u2f(both[0]), u2f(both[1]));
    return;
  }
  // out[query][h * D + d] = O^T[d][query] / l; register 4c + r of row block db is d = 32 db + 8 c + 4 (lane / 32) + r
  const auto halves = __builtin_amdgcn_permlane32_swap(f2u(l), f2u(l), false, false);
  l = u2f(halves[0]) + u2f(halves[1]);
  if (!stored) return;
  if constexpr (PASS == kPart) {
    const int64_t row = ((int64_t)h * chunks + chunk) * w.Sq + query;
    if (lane < 32) w.ends[row] = make_float2(m, l);
    float* dst = w.parts + row * D + row_in_tile;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4*>(dst + db * 32 + c * 8) = make_float4(o[db][4 * c], o[db][4 * c + 1], o[db][4 * c + 2], o[db][4 * c + 3]);
  } else {
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

// The chunks' sums against their own maxima, of which the last one's is the row's: a thread to four dimensions of a row and head.
template <int D>
__global__ __launch_bounds__(256) void attention_masked_join_kernel(const float* __restrict__ parts, const float2* __restrict__ ends,
                                                                    uint16_t* __restrict__ out, int Sq, int heads, int chunks, float bias) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, at = i / (D / 4);
  if (at >= (int64_t)Sq * heads) return;
  const int h = (int)(at / Sq), row = (int)(at - (int64_t)h * Sq), d = (int)(i % (D / 4)) * 4;
  const int64_t first = (int64_t)h * chunks * Sq + row;
  const float top = ends[first + (int64_t)(chunks - 1) * Sq].x;
  float4 sum = make_float4(0, 0, 0, 0);
  float l = 0.f;
#pragma unroll 4
  for (int c = 0; c < chunks; ++c) {
    const int64_t r = first + (int64_t)c * Sq;
    const float2 end = ends[r];
    const float f = __builtin_amdgcn_exp2f(end.x - top);
    const float4 v = *reinterpret_cast<const float4*>(parts + r * D + d);
    sum.x += v.x * f, sum.y += v.y * f, sum.z += v.z * f, sum.w += v.w * f, l += end.y * f;
  }
  const float inv = l == 0.f ? 0.f : bias / l;
  *reinterpret_cast<uint2*>(out + ((int64_t)row * heads + h) * D + d) = make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
}

}  // namespace

// The largest norm of the keys of a tile, to a wave.
template <int SCALE_KIND>
__global__ __launch_bounds__(256) void key_norms_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int asym, int64_t tiles, int D,
                                                        float* __restrict__ norms) {
  const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= tiles) return;
  const int lane = threadIdx.x & 63;
  const int64_t key = tile * 32 + (lane & 31);  // (tiles of a head after another)
  float sum = 0.f;
  for (int i = lane >> 5; i < D / 32; i += 2) {
    const u32x4 c = *reinterpret_cast<const u32x4*>(codes + key * (D / 2) + 16 * i);
    const uint8_t* sb = scales + (key * (D / 32) + i) * (asym ? 2 : 1);
    const float p = scale_value<SCALE_KIND>(sb[0]), n = asym ? scale_value<SCALE_KIND>(sb[1]) : p;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t word = c[j];
      const f32x2 e[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 3)};
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float v = e[k >> 1][k & 1], x = v * (v < 0.f ? n : p);
        sum = __builtin_fmaf(x, x, sum);
      }
    }
  }
  sum += __shfl_xor(sum, 32, 64);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum = fmaxf(sum, __shfl_xor(sum, d, 64));
  if (lane == 0) norms[tile] = __builtin_sqrtf(sum + kLostSquares) * 1.001f;
}

// The launches of a checked call with heads of D. chunks > 1: split rows; small: kHeld; else pairs of key tiles to a step or not.
template <int D>
hipError_t launch_masked(int scale_kind, const MaskedOperands& m, const MaskedWork& w, int64_t q_heads, int chunks, bool small, bool pairs,
                         hipStream_t s) {
  dim3 grid((unsigned)q_heads, (unsigned)((w.Sq + kQueries - 1) / kQueries), (unsigned)chunks);
  auto go = [&]<int SK, bool CAP, bool SLOPE>() {
    auto pass = [&]<int NT, int PASS>() {
      hipLaunchKernelGGL((attention_masked_kernel<SK, D, CAP, SLOPE, NT, PASS>), grid, dim3(64 * kWaves), 0, s, m.Q_codes, m.Q_scales, m.asym,
                         m.K_panel, m.V_panel, m.out, w, m.K_codes, m.K_scales, m.V_codes, m.V_scales);
    };
    if (SLOPE && w.norms) {
      const int64_t tiles = q_heads / w.kv_group * (w.Sk / 32);
      hipLaunchKernelGGL((key_norms_kernel<SK>), dim3((unsigned)((tiles + 3) / 4)), dim3(256), 0, s, m.K_codes, m.K_scales, m.asym, tiles, D,
                         const_cast<float*>(w.norms));
    }
    if (chunks > 1) {
      pass.template operator()<2, kMaxima>();
      pass.template operator()<2, kPart>();
      hipLaunchKernelGGL((attention_masked_join_kernel<D>), dim3((unsigned)((w.Sq * q_heads * (D / 4) + 255) / 256)), dim3(256), 0, s, w.parts, w.ends,
                         m.out, w.Sq, (int)q_heads, chunks, SK == kScaleE5M2 ? 0.03125f : 1.0f);
    } else if (small) {
      pass.template operator()<2, kHeld>();
    } else if (pairs) {
      pass.template operator()<2, kWhole>();
    } else {
      pass.template operator()<1, kWhole>();
    }
  };
  auto with_scale = [&]<int SK>() {
    if (w.scores.cap > 0.f)
      w.scores.slopes ? go.template operator()<SK, true, true>() : go.template operator()<SK, true, false>();
    else
      w.scores.slopes ? go.template operator()<SK, false, true>() : go.template operator()<SK, false, false>();
  };
  switch (scale_kind) {
    case kScaleE5M2: with_scale.template operator()<kScaleE5M2>(); break;
    case kScaleE4M3: with_scale.template operator()<kScaleE4M3>(); break;
    case kScaleE8M0Floor: with_scale.template operator()<kScaleE8M0Floor>(); break;
    default: with_scale.template operator()<kScaleE8M0Round>();
  }
  return hipGetLastError();
}

// attention_masked.hip: heads of 128; attention_masked_64.hip: of 64 (two files because there are many kernels)
hipError_t launch_attention_masked_64(int scale_kind, const MaskedOperands& m, const MaskedWork& w, int64_t q_heads, int chunks, bool small, bool pairs,
                                      hipStream_t s);

}  // namespace amx
