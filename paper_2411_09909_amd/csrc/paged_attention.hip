// Attention over the paged cache (include/amxfp4_paged.h): split over the keys, joined by a second kernel.
//
// Columns. A matrix instruction has 16 columns and a decoding step few rows of queries (4 query heads share a key head in the
// models this is for), so the columns of a tile are (combination, group): a combination is a row and a query head that read
// the same key head, a group one of the head dimension's D / 32 groups of the cast. Column (c, g) multiplies combination c with
// group g of the keys alone (the query's other groups are zeros there), so that the group's scales, which are those of a token,
// can be applied to the product: s[c][j] = sum_g S[j][g] (q . elements)[c][j][g]. The keys' elements are converted to BF16, which
// holds them, and not scaled.
//   sign pair   S_p q.e+ + S_n q.e-: a product to each sign class. (S_n q.e + (S_p - S_n) q.e+ would save separating e-, but where S_n is much the
//               larger the positive class is the difference of two terms of its size: with S_n / S_p = 2^16 and a query of zeros on the negative
//               elements' dimensions a score was off by 2^-10 of sum |q k|, with 2^28 it was lost.)
//   (The codes as they are on the block-scaled instruction, the query as two E4M3 parts, saves the conversion and costs
//   exactness: that instruction adds its products in a window of 2^-13 of the largest, and a score was off by 2^-12 of it.)
// Values. The codes of 64 tokens are transposed by ds_read_b64_tr_b4 (16 lanes read 16 rows of 16 codes and get one column
// each), converted to BF16 elements and multiplied with p[c][j] S[j][g], rounded to BF16: O[d][c] = sum_j (p S)[j][c] e[j][d].
// The two sign classes stay apart here too (e+ with p S_p, e- with p S_n). The columns of the other groups compute products nobody reads.
// Layout of a tile of 64 tokens in a wave: lane (column or row r = l % 16, quarter u = l / 16). S^T comes out of the matrix
// instruction t (of 4) with tile rows 4 u + i in lane (r, u): those rows are keys 16 u + 4 t + i, so that a lane holds the 16 keys
// 16 u .. of its column, in the order in which the second product wants them, and needs the scales of 16 neighbouring tokens, 32 bytes.
//
// Division of the work, by the host's rules at the end of this file:
//   split    units of 64 tokens (more where there could be 2^31 of them) of one sequence, key head and tile of combinations, in
//            that order, are dealt out evenly over the workgroups, whatever the sequences' lengths are. Every workgroup finds its own
//            range from the lengths (a prefix sum over the sequences, in LDS). A range may begin and end within a sequence: those
//            partial results (O, m, l) go to the workspace, at most two to a workgroup, and paged_attention_join_kernel adds them up.
//   whole    short sequences: a sequence and key head to a workgroup or, where there are many, to a wave, with all its tokens.
//
// Bound and measured (a pass of both kernels, back to back; medians; cards differ by some 4 %). 64 sequences of up to 16384 tokens, 32 / 8 heads of
// 128, pairs of E5M2 scales, 612 MB: 145 us = 4.2 TB/s (140 before the scores kept the sign classes apart); pieces of 4 KB from all over the memory
// are read at 5.9 TB/s by loads alone (104 us), and the vector instructions (conversion, scales, softmax: 787 to a tile and wave) hide in that but
// for their unevenness. One of 131000 tokens, 151 MB: 49 us, of which 7 to 10 are the join. 16 of up to 4000 with up to 4 rows of 8 query heads to a
// key head, 42 MB: 39 us, bound by the vector instructions. One of 700: 10 us, the chain from the lengths to the codes and the waves' join.
// Not dealt out evenly are sequences taken whole (tables, or max_keys, of up to 1024 tokens) of which a few have many rows: see is_whole().
#include "paged.h"

#include "kernels.h"
#include "layer_math.h"

namespace amx {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = 64;        // tokens of a unit
// Workgroups of a launch that splits sequences, which are all to run at once: the registers leave room for three to a compute unit with four
// columns to a combination and for two with two or one and asymmetric scales. 16 sequences of 4 rows and 8 query heads to a key head 41 us on
// 512 and 52 on 768, 40 of up to 3000 tokens with 8 query heads to a key head 41 and 48. Where three or four have room with fewer columns, 512 are as
// good: symmetric scales and two columns, the same 40 sequences 31.2 us and 31.7, 16 of up to 8000 28.1 and 26.8, 4 of up to 30000 27.0 and 27.6;
// heads of 64, 8 sequences of up to 16000 tokens 21 and 22.
constexpr int most_workers(int gc) { return gc == 4 ? 768 : 512; }
// A sequence, key head and tile of combinations takes as long as this many tiles before its first one is in: the chain from the lengths
// over the table to the keys, and the joining of the waves.
constexpr uint32_t kStart = 12;

// What one launch reads, beside the arrays of the sequences.
struct PagedWork {
  const uint16_t* q;
  uint16_t* out;
  uint8_t* workspace;
  int64_t rows, max_pages;
  int seqs, q_heads, per;  // per: query heads to a key head
  float scale_log2;
  int whole, unit_log2;    // tiles of 64 tokens to a unit
};

// What a workgroup leaves behind for the joining kernel, at the front of the workspace.
struct PagedTail {
  uint32_t units, end;    // all units; one past the last of the sequence, key head and tile that it began and did not end
  uint32_t groups, owner;  // workgroups among which the units are divided; 1: it began such a one
  uint32_t first, rows, head, tile;  // the sequence's rows; key head; tile of combinations
};

// units of a worker: [first_unit(g), first_unit(g + 1))
__device__ __forceinline__ uint32_t first_unit(uint32_t units, uint32_t groups, uint32_t g) {
  return units / groups * g + (units % groups) * g / groups;  // (groups <= 768)
}

template <int NC, int D>
constexpr int kPartFloats = NC * (D + 2);

// A sequence as the units see it. NT: tiles of tokens (one at least, so that a row without keys is written), CT: tiles of combinations.
struct PagedSequence {
  int64_t first;  // its first row
  uint32_t rows, keys, NT, CT;
};
template <int NC>
__device__ __forceinline__ void paged_tiles(const PagedWork& w, PagedSequence& s) {
  s.NT = max((s.keys + kTile - 1) / kTile, 1u);
  s.CT = (s.rows * (uint32_t)w.per + NC - 1) / NC;  // (rows * q_heads <= 2^31)
}
template <int NC>
__device__ __forceinline__ PagedSequence paged_sequence(const PagedWork& w, uint32_t page_log2, const int32_t* __restrict__ lens,
                                                        const int32_t* __restrict__ starts, int b) {
  PagedSequence s;
  const int64_t a = max((int64_t)starts[b], (int64_t)0), e = min((int64_t)starts[b + 1], w.rows);
  const int n = lens[b];
  s.first = a;
  s.rows = e > a ? (uint32_t)(e - a) : 0u;
  s.keys = (uint32_t)max(0, min(n, (int)(w.max_pages << page_log2)));  // (at most 2^30)
  paged_tiles<NC>(w, s);
  return s;
}

// LDS that a launch which splits sequences takes for them
constexpr int kKept = 512;
__host__ __device__ constexpr size_t sequences_bytes(int64_t seqs) { return ((size_t)seqs * (seqs <= kKept ? 16 : 4) + 63) & ~(size_t)63; }

// max over the four quarters of a wave (lanes of the same column)
__device__ __forceinline__ float quarters_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(f2u(v), f2u(v), false, false);
  v = fmaxf(u2f(a[0]), u2f(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false);
  return fmaxf(u2f(b[0]), u2f(b[1]));
}
__device__ __forceinline__ float quarters_sum(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(f2u(v), f2u(v), false, false);
  v = u2f(a[0]) + u2f(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false);
  return u2f(b[0]) + u2f(b[1]);
}

// A lane's neighbours among the GC columns of a combination (GC 2 or 4): lane ^ 1, lane ^ 2.
template <int X>
__device__ __forceinline__ float neighbour(float v) {
  return u2f((uint32_t)__builtin_amdgcn_mov_dpp((int)f2u(v), X == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true));
}
// the value of column G of the combination, in all its columns
template <int GC, int G>
__device__ __forceinline__ float of_column(float v) {
  if constexpr (GC == 1) return v;
  constexpr int kPerm = GC == 4 ? G * 0x55 : G + (G << 2) + ((2 + G) << 4) + ((2 + G) << 6);
  return u2f((uint32_t)__builtin_amdgcn_mov_dpp((int)f2u(v), kPerm, 0xF, 0xF, true));
}

// Two scales (bytes 2 HALF and 2 HALF + 1 of a word) as floats.
template <int SCALE_KIND, bool HALF>
__device__ __forceinline__ f32x2 two_scales(uint32_t word) {
  if constexpr (SCALE_KIND == kScaleE5M2) {
    return __builtin_amdgcn_cvt_pk_f32_bf8((int)word, HALF);
  } else if constexpr (SCALE_KIND == kScaleE4M3) {
    return __builtin_amdgcn_cvt_pk_f32_fp8((int)word, HALF);
  } else {  // the exponent's field (byte 0: 2^-127, as good as the 0 it becomes)
    const uint32_t a = HALF ? word << 7 : word << 23, b = HALF ? word >> 1 : word << 15;
    return f32x2{u2f(a & 0x7F800000u), u2f(b & 0x7F800000u)};
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// eight codes -> eight elements, BF16
__device__ __forceinline__ u32x4 elements(uint32_t word) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.0f, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.0f, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.0f, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, 1.0f, 3))};
}

// The elements of one sign class, zeros for the others: as 16-bit integers negative numbers lie below 0. (The words one by one, through
// a variable: a bit cast of a vector's element itself takes element 0.)
__device__ __forceinline__ u32x4 positive(u32x4 e) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = e[i];
    v[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, two), (i16x2{0, 0})));
  }
  return v;
}
__device__ __forceinline__ u32x4 negative(u32x4 e) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t two = e[i];
    v[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2, two), (i16x2{0, 0})));
  }
  return v;
}

template <int SCALE_KIND, bool ASYM, int D, int GC>
struct PagedTile {
  static constexpr int kGroups = D / 32, GS = kGroups / GC;
  static constexpr bool kAsLoaded = D == 128 && GC == 4;  // a lane has the four words of the group of its quarter, and the products take one each
  static constexpr int NK = D / 32, NV = D / 32;          // loads of 16 bytes: codes of K, of V
  static constexpr int kScaleWords = (ASYM ? 8 : 4);      // scales of 16 tokens
  u32x4 k[NK], v[NV];
  u32x4 ks[GS][kScaleWords / 4], vs[GS][kScaleWords / 4];
};

// SHARE: waves to a sequence and key head, 4 or 1.
template <int SCALE_KIND, bool ASYM, int D, int GC, int SHARE>
__global__ __launch_bounds__(256, D == 64 || GC == 4 || (!ASYM && GC == 2) ? 3 : 2) void paged_attention_kernel(
    PagedPool pool, PagedWork w, const int32_t* __restrict__ table, const int32_t* __restrict__ lens, const int32_t* __restrict__ starts,
    const int32_t* __restrict__ positions) {
  using Tile = PagedTile<SCALE_KIND, ASYM, D, GC>;
  constexpr int GS = Tile::GS, NC = 16 / GC, DT = D / 16;
  constexpr int kValueBytes = kTile * D / 2;  // of a wave's tile of V
  constexpr int kShareFloats = NC * D;
  extern __shared__ __align__(64) uint8_t lds[];
  __shared__ float top_of[4][NC], sum_of[4][NC];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool whole = SHARE == 1 || w.whole;
  // split: units up to and with a sequence; of up to kKept sequences also what paged_sequence() reads
  uint32_t* const ends = reinterpret_cast<uint32_t*>(lds);
  uint32_t* const kept = ends + w.seqs;
  const bool keep = w.seqs <= kKept;
  uint8_t* const region = lds + (whole ? 0 : sequences_bytes(w.seqs));
  uint8_t* const mine = region + wave * kValueBytes;

  int b, head;
  uint32_t ct = 0, unit = 0, hi = 0;
  const uint32_t worker = SHARE == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  // units of a sequence, key head and tile of combinations
  auto units_of = [&](uint32_t NT) { return kStart + ((NT + (1u << w.unit_log2) - 1) >> w.unit_log2); };
  if (whole) {
    if (worker >= (uint32_t)w.seqs * pool.kv_heads) return;  // (SHARE == 1: the wave; nobody waits for it)
    b = __builtin_amdgcn_readfirstlane((int)(worker / pool.kv_heads)), head = (int)worker - b * (int)pool.kv_heads;
    ct = blockIdx.y;
  } else {
    const int lane = threadIdx.x & 63;
    // ---- the worker's range of units. The sums stay at kMostUnits once they reach it, which only rows that sequences share
    // can bring about: then units are missing, but each is one of its sequence's.
    constexpr uint32_t kMostUnits = 0x7FFFFFFF;
    __shared__ uint32_t edge[4];
    const int each = (w.seqs + 255) >> 8, b0 = threadIdx.x * each, b1 = min(w.seqs, b0 + each);
    uint32_t sum = 0;
    for (int i = b0; i < b1; ++i) {
      const PagedSequence s = paged_sequence<NC>(w, pool.page_log2, lens, starts, i);
      if (keep) kept[i] = (uint32_t)s.first, kept[w.seqs + i] = s.rows, kept[2 * w.seqs + i] = s.keys;
      const uint64_t own = min((uint64_t)s.CT * units_of(s.NT), (uint64_t)kMostUnits) * pool.kv_heads;
      ends[i] = sum = (uint32_t)min(sum + own, (uint64_t)kMostUnits);
    }
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t v = __shfl_up(upto, o, 64);
      if (lane >= o) upto = min(upto + v, kMostUnits);
    }
    if (lane == 63) edge[wave] = upto;
    __syncthreads();
    uint32_t before = __shfl_up(upto, 1, 64);
    if (lane == 0) before = 0;
    for (int i = 0; i < wave; ++i) before = min(before + edge[i], kMostUnits);
    for (int i = b0; i < b1; ++i) ends[i] = min(ends[i] + before, kMostUnits);
    __syncthreads();
    const uint32_t units = __builtin_amdgcn_readfirstlane(ends[w.seqs - 1]);
    // four units at least
    const uint32_t groups = max(1u, min((uint32_t)gridDim.x, w.unit_log2 ? units : (units + 3) / 4));
    if (threadIdx.x == 0) reinterpret_cast<PagedTail*>(w.workspace)[worker] = PagedTail{units, 0, groups, 0, 0, 0, 0, 0};
    if (worker >= groups || units == 0) return;
    unit = first_unit(units, groups, worker), hi = first_unit(units, groups, worker + 1);
    // the first sequence whose units end behind the range's first: its 64th of the sequences, then in there
    const int part = (w.seqs + 63) >> 6;
    const int chunk = (int)__popcll(__builtin_amdgcn_ballot_w64(ends[min((lane + 1) * part, w.seqs) - 1] <= unit));
    const int at = chunk * part + lane;
    b = chunk * part + (int)__popcll(__builtin_amdgcn_ballot_w64(lane < part && at < w.seqs && ends[min(at, w.seqs - 1)] <= unit));
    head = 0;
  }

  for (;;) {
    // (the lane anew here and below the tiles: what depends on it would otherwise be worked out before and take 50 registers)
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const int lane = thread & 63, r = lane & 15, u = lane >> 4, c = r / GC, gc = r % GC;
    uint32_t t0 = 0, t1, after = 0;  // tiles of tokens; the unit behind the segment's last
    bool complete = true;
    if (!whole) {
      if (unit >= hi) return;
      while (__builtin_amdgcn_readfirstlane(ends[b]) <= unit) ++b;
    }
    PagedSequence s;
    if (!whole && keep) {
      s.first = __builtin_amdgcn_readfirstlane(kept[b]), s.rows = __builtin_amdgcn_readfirstlane(kept[w.seqs + b]);
      s.keys = __builtin_amdgcn_readfirstlane(kept[2 * w.seqs + b]);
      paged_tiles<NC>(w, s);
    } else {
      s = paged_sequence<NC>(w, pool.page_log2, lens, starts, b);
    }
    if (whole) {
      if (ct >= s.CT) return;
      t1 = s.NT;
    } else {
      const uint32_t base = b ? __builtin_amdgcn_readfirstlane(ends[b - 1]) : 0u;
      const uint32_t per_segment = units_of(s.NT);
      const uint32_t seg = (unit - base) / per_segment, first = (unit - base) - seg * per_segment;
      head = (int)(seg / s.CT), ct = seg - (uint32_t)head * s.CT;
      after = base + (seg + 1) * per_segment;
      const uint32_t end = min(per_segment, first + (hi - unit));
      unit += end - first;
      if (end <= kStart) continue;  // its start alone: what comes after is the next worker's
      t0 = first > kStart ? (first - kStart) << w.unit_log2 : 0u, t1 = min(s.NT, (end - kStart) << w.unit_log2);
      complete = t0 == 0 && end == per_segment;
    }
    t0 = __builtin_amdgcn_readfirstlane(t0), t1 = __builtin_amdgcn_readfirstlane(t1);
    ct = __builtin_amdgcn_readfirstlane(ct), head = __builtin_amdgcn_readfirstlane(head);
    const int32_t* row_table = table + (int64_t)b * w.max_pages;
    const uint32_t last_entry = (uint32_t)(w.max_pages - 1);

    // ---- this lane's combination
    const uint32_t combination = ct * NC + c;
    const bool asked = combination < s.rows * (uint32_t)w.per;
    const uint32_t row_of = asked ? combination / (uint32_t)w.per : 0u, head_of = asked ? combination - row_of * (uint32_t)w.per : 0u;
    const int64_t row = s.first + row_of;
    const int position = positions[row < w.rows ? row : 0];

    // ---- the query: dimensions 32 j + 8 u .. of group j, zeros where the column is not the group's; where the keys' words stay as
    // they are loaded (all groups in the columns), dimensions 32 u + 8 j .. of group u
    u32x4 q[Tile::kGroups];
#pragma unroll
    for (int j = 0; j < Tile::kGroups; ++j) {
      q[j] = u32x4{0, 0, 0, 0};
      if (asked && (Tile::kAsLoaded ? u : j % GC) == gc)
        q[j] = *reinterpret_cast<const u32x4*>(w.q + (row * w.q_heads + (int64_t)head * w.per + head_of) * D +
                                               (Tile::kAsLoaded ? 32 * u + 8 * j : 32 * j + 8 * u));
    }

    // ---- requests. A tile's registers take the next tile's data once they have been used: K, its scales and V (which is in LDS by
    // then) after the scores, V's scales after the weights.
    const int64_t page_stride = (int64_t)pool.kv_heads << pool.page_log2;
    const uint32_t mask = (1u << pool.page_log2) - 1;
    // Pages of the four sub-blocks of 16 tokens of the tile that is requested next (four variables: an array would be indexed). Asked for a
    // tile ahead, one to a lane, through the vector memory: a scalar load in flight would make every wait for LDS wait for it.
    uint32_t id0, id1, id2, id3, ahead;
    auto look_up = [&](uint32_t tile) { ahead = (uint32_t)row_table[min((tile * kTile + 16 * (lane & 3)) >> pool.page_log2, last_entry)]; };
    auto found = [&]() {
      id0 = (uint32_t)__builtin_amdgcn_readlane((int)ahead, 0), id1 = (uint32_t)__builtin_amdgcn_readlane((int)ahead, 1);
      id2 = (uint32_t)__builtin_amdgcn_readlane((int)ahead, 2), id3 = (uint32_t)__builtin_amdgcn_readlane((int)ahead, 3);
    };
    auto in_pool = [&](uint32_t id) { return id < pool.pages ? id : 0u; };
    auto pick = [&](int k) {  // of a sub-block that depends on the lane
      const uint32_t a = k & 1 ? id1 : id0, z = k & 1 ? id3 : id2;
      return in_pool(k & 2 ? z : a);
    };
    auto first_token = [&](uint32_t page, uint32_t token) {  // of the pool, for this head: place of a token
      return (int64_t)page * page_stride + ((int64_t)head << pool.page_log2) + (token & mask);
    };
    // scales of tokens 16 u .. of group st * GC + gc
    auto request_scales = [&](uint32_t tile, const uint8_t* from, u32x4 (&to)[GS][Tile::kScaleWords / 4]) {
      const uint32_t place = (tile * kTile + 16 * u) & mask;
      const int64_t at = (((int64_t)pick(u) * pool.kv_heads + head) * Tile::kGroups + gc) << pool.page_log2;
      const uint8_t* p = from + (at + place) * (ASYM ? 2 : 1);
#pragma unroll
      for (int st = 0; st < GS; ++st)
#pragma unroll
        for (int i = 0; i < Tile::kScaleWords / 4; ++i)
          to[st][i] = *reinterpret_cast<const u32x4*>(p + (((int64_t)st * GC) << pool.page_log2) * (ASYM ? 2 : 1) + 16 * i);
    };
    // K: tile row r of product t is key 16 (r / 4) + 4 t + r % 4
    auto request_keys = [&](uint32_t tile, Tile& d) {
      const int k = r >> 2;
      const uint32_t token = tile * kTile + 16 * k + (r & 3) + (D == 64 ? 4 * (u >> 1) : 0);
      const uint8_t* p = pool.k_codes + first_token(pick(k), token) * (D / 2) + 16 * (D == 64 ? (u & 1) : u);
#pragma unroll
      for (int t = 0; t < Tile::NK; ++t) d.k[t] = *reinterpret_cast<const u32x4*>(p + t * (D == 64 ? 8 : 4) * (D / 2));
      request_scales(tile, pool.k_scales, d.ks);
    };
    auto request_values = [&](uint32_t tile, Tile& d) {
#pragma unroll
      for (int n = 0; n < Tile::NV; ++n) {
        constexpr int kParts = D / 32;  // pieces of 16 bytes in a row
        const uint32_t token = tile * kTile + n * (64 / kParts) + lane / kParts;
        const uint32_t page = in_pool(D == 128 ? (n == 0 ? id0 : n == 1 ? id1 : n == 2 ? id2 : id3) : n == 0 ? (lane < 32 ? id0 : id1) : (lane < 32 ? id2 : id3));
        d.v[n] = *reinterpret_cast<const u32x4*>(pool.v_codes + first_token(page, token) * (D / 2) + 16 * (lane % kParts));
      }
    };
    auto bad_pages = [&]() {
      return (id0 >= pool.pages ? 1u : 0u) | (id1 >= pool.pages ? 2u : 0u) | (id2 >= pool.pages ? 4u : 0u) | (id3 >= pool.pages ? 8u : 0u);
    };
    Tile d;
    uint32_t tile = t0 + (SHARE == 1 ? 0 : wave), bad = 0;
    look_up(tile);
    if (tile < t1) {
      found();
      bad = bad_pages();
      request_values(tile, d);
      request_keys(tile, d);
      request_scales(tile, pool.v_scales, d.vs);
    }
    look_up(tile + SHARE);

    // tokens it sees; columns that nobody asked for see all and are not looked at
    // (positions may be the type's ends: one is added only below the keys' number)
    const int limit = asked ? min(max(position, -1), (int)s.keys - 1) + 1 : 0x7FFFFFFF;
    int least = limit, most = asked ? limit : 0;  // (the same in all quarters and in the columns of a combination)
#pragma unroll
    for (int o = GC; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o, 64)), most = max(most, __shfl_xor(most, o, 64));
    least = __builtin_amdgcn_readfirstlane(least), most = __builtin_amdgcn_readfirstlane(most);
    const uint32_t stop = min(t1, (uint32_t)(most + kTile - 1) / kTile);

    // ---- the tiles
    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.f;
    const float sc = w.scale_log2;

    for (; tile < stop; tile += SHARE) {
      const bool more = tile + SHARE < stop;
      // V into LDS, piece p of row j at p ^ (some bits of j): rows that 16 lanes read at once lie in different banks
      // (the LDS of a launch and `mine` begin at multiples of 64 bytes)
#pragma unroll
      for (int n = 0; n < Tile::NV; ++n) {
        constexpr int kParts = D / 32;
        const int j = n * (64 / kParts) + lane / kParts, part = (lane % kParts) ^ (D == 128 ? (j >> 2) & 3 : (j >> 3) & 1);
        *reinterpret_cast<u32x4*>(mine + j * (D / 2) + 16 * part) = d.v[n];
      }

      // ---- scores
      float x[16];
      const int first = (int)tile * kTile;
      const int count = (bad >> u) & 1 ? 0 : max(0, min(limit - first - 16 * u, 16));
      const bool all = first + kTile <= least && bad == 0;
      uint32_t kw[4 * Tile::NK];
#pragma unroll
      for (int n = 0; n < Tile::NK; ++n) {
        if constexpr (Tile::kAsLoaded) {
          for (int j = 0; j < 4; ++j) kw[4 * n + j] = d.k[n][j];
          continue;
        }
        // a lane has the four words of one group; it is to have word u of each of the four: the quarters' 4 x 4 words transposed
        const auto a = __builtin_amdgcn_permlane32_swap(d.k[n][0], d.k[n][2], false, false);
        const auto z = __builtin_amdgcn_permlane32_swap(d.k[n][1], d.k[n][3], false, false);
        const auto y0 = __builtin_amdgcn_permlane16_swap(a[0], z[0], false, false), y1 = __builtin_amdgcn_permlane16_swap(a[1], z[1], false, false);
        kw[4 * n] = y0[0], kw[4 * n + 1] = y0[1], kw[4 * n + 2] = y1[0], kw[4 * n + 3] = y1[1];
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * t + i] = 0.f;
#pragma unroll
        for (int st = 0; st < GS; ++st) {
          f32x4 dot = {0, 0, 0, 0}, negatives = {0, 0, 0, 0};  // (both signs, where they have one scale; the positive class else)
#pragma unroll
          for (int j = st * GC; j < (st + 1) * GC; ++j) {
            const u32x4 e = elements(kw[Tile::kGroups * t + j]);  // (heads of 64: two tiles' words in turn)
            const bf16x8 qj = __builtin_bit_cast(bf16x8, q[j]);
            dot = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ASYM ? positive(e) : e), qj, dot, 0, 0, 0);
            if constexpr (ASYM) negatives = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, negative(e)), qj, negatives, 0, 0, 0);
          }
          if constexpr (ASYM) {
            const uint32_t s0 = d.ks[st][t >> 1][2 * t & 3], s1 = d.ks[st][t >> 1][(2 * t + 1) & 3];
            const f32x2 a[4] = {two_scales<SCALE_KIND, false>(s0), two_scales<SCALE_KIND, true>(s0), two_scales<SCALE_KIND, false>(s1),
                                two_scales<SCALE_KIND, true>(s1)};
#pragma unroll
            for (int i = 0; i < 4; ++i)
              x[4 * t + i] = __builtin_fmaf(a[i][1], negatives[i], __builtin_fmaf(a[i][0], dot[i], x[4 * t + i]));
          } else {
            const uint32_t s0 = d.ks[st][0][t];
            const f32x2 a = two_scales<SCALE_KIND, false>(s0), z = two_scales<SCALE_KIND, true>(s0);
            x[4 * t] = __builtin_fmaf(a[0], dot[0], x[4 * t]), x[4 * t + 1] = __builtin_fmaf(a[1], dot[1], x[4 * t + 1]);
            x[4 * t + 2] = __builtin_fmaf(z[0], dot[2], x[4 * t + 2]), x[4 * t + 3] = __builtin_fmaf(z[1], dot[3], x[4 * t + 3]);
          }
        }
      }
      // (the scores are there before K's registers are asked for again: otherwise the scaling is moved behind the branch, and both the
      // products and the old scales are kept across it; the same with V's scales below)
#pragma unroll
      for (int i = 0; i < 16; ++i) asm volatile("" : "+v"(x[i]));
      if (more) {
        found();
        request_keys(tile + SHARE, d);
        request_values(tile + SHARE, d);
      }
      // The columns' sums, each column keeping those of its share of the lane's 16 keys: key GC k + gc as y[k]. The rest of the softmax
      // is done for those alone.
      constexpr int kMine = 16 / GC;
      float y[kMine];
      if constexpr (GC == 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const bool odd = gc & 1, high = gc & 2;
          const float a = (odd ? x[4 * k + 1] : x[4 * k]) + neighbour<1>(odd ? x[4 * k] : x[4 * k + 1]);
          const float z = (odd ? x[4 * k + 3] : x[4 * k + 2]) + neighbour<1>(odd ? x[4 * k + 2] : x[4 * k + 3]);
          y[k] = (high ? z : a) + neighbour<2>(high ? a : z);
        }
      } else if constexpr (GC == 2) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = (gc ? x[2 * k + 1] : x[2 * k]) + neighbour<1>(gc ? x[2 * k] : x[2 * k + 1]);
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) y[k] = x[k];
      }
      if (!all) {
#pragma unroll
        for (int k = 0; k < kMine; ++k) y[k] = GC * k + gc < count ? y[k] : -INFINITY;
        // scales of V that belong to no token seen become zeros: they may be infinite, and weights of 0 would be NaN
#pragma unroll
        for (int st = 0; st < GS; ++st)
#pragma unroll
          for (int i = 0; i < Tile::kScaleWords; ++i) {
            constexpr int kTokens = ASYM ? 2 : 4;  // of a word
            const int seen = max(0, min(count - kTokens * i, kTokens));
            d.vs[st][i >> 2][i & 3] &= seen == kTokens ? ~0u : (1u << (32 / kTokens * seen)) - 1;
          }
      }

      // ---- running maximum and sum
      float top = y[0];
#pragma unroll
      for (int k = 1; k < kMine; ++k) top = fmaxf(top, y[k]);
      if constexpr (GC >= 2) top = fmaxf(top, neighbour<1>(top));
      if constexpr (GC >= 4) top = fmaxf(top, neighbour<2>(top));
      top = fmaxf(m, quarters_max(top));
      const float to = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f((m - to) * sc), shift = to * sc;
      m = top;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < kMine; ++k) y[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[k], sc, -shift)), sum += y[k];
      l = __builtin_fmaf(l, alpha, sum);
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] *= alpha;
      }

      // ---- values. Token 16 u + r's row, its piece 0; piece p is 16 p bytes away in the bits of its place (again for every tile: one
      // register instead of one to a piece)
      uint32_t row_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)mine + (16 * u + r) * (D / 2) + 16 * (D == 128 ? (r >> 2) & 3 : (r >> 3) & 1);
      asm volatile("" : "+v"(row_at));
#pragma unroll
      for (int st = 0; st < GS; ++st) {
        uint32_t wp[8], wn[8];  // weights of this lane's 16 keys, pairs
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f32x2 s0, s1;  // (S_p, S_n) of keys 2 i and 2 i + 1
          if constexpr (ASYM) {
            const uint32_t word = d.vs[st][i >> 2][i & 3];
            s0 = two_scales<SCALE_KIND, false>(word), s1 = two_scales<SCALE_KIND, true>(word);
          } else {
            const uint32_t word = d.vs[st][0][i >> 1];
            const f32x2 pair = i & 1 ? two_scales<SCALE_KIND, true>(word) : two_scales<SCALE_KIND, false>(word);
            s0 = f32x2{pair[0], pair[0]}, s1 = f32x2{pair[1], pair[1]};
          }
          // keys 2 i and 2 i + 1: each from the column that has it
          const float v = y[2 * i / GC], z = y[(2 * i + 1) / GC];
          const float a = GC == 4 && (i & 1) ? of_column<GC, GC == 4 ? 2 : 0>(v) : of_column<GC, 0>(v);
          const float e = GC == 4 && (i & 1) ? of_column<GC, GC == 4 ? 3 : 0>(z) : of_column<GC, GC >= 2 ? 1 : 0>(z);
          wp[i] = pack_bf16(a * s0[0], e * s1[0]);
          if constexpr (ASYM) wn[i] = pack_bf16(a * s0[1], e * s1[1]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          asm volatile("" : "+v"(wp[i]));
          if constexpr (ASYM) asm volatile("" : "+v"(wn[i]));
        }
        if (st == GS - 1 && more) {
          request_scales(tile + SHARE, pool.v_scales, d.vs);
          bad = bad_pages();
          look_up(tile + 2 * SHARE);
        }
        const bf16x8 p0 = __builtin_bit_cast(bf16x8, (u32x4{wp[0], wp[1], wp[2], wp[3]})), p1 = __builtin_bit_cast(bf16x8, (u32x4{wp[4], wp[5], wp[6], wp[7]}));
        bf16x8 n0, n1;
        if constexpr (ASYM)
          n0 = __builtin_bit_cast(bf16x8, (u32x4{wn[0], wn[1], wn[2], wn[3]})), n1 = __builtin_bit_cast(bf16x8, (u32x4{wn[4], wn[5], wn[6], wn[7]}));
#pragma unroll
        for (int dt = 2 * GC * st; dt < 2 * GC * (st + 1); ++dt) {
          typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
          const i32x2 codes = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2*)(uintptr_t)((row_at ^ (16 * (dt >> 1))) + 8 * (dt & 1)));
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4 e = elements((uint32_t)codes[h]);
            if constexpr (ASYM) {
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, positive(e)), h ? p1 : p0, o[dt], 0, 0, 0);
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, negative(e)), h ? n1 : n0, o[dt], 0, 0, 0);
            } else {
              o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, e), h ? p1 : p0, o[dt], 0, 0, 0);
            }
          }
        }
      }
    }

    l = quarters_sum(l);
    if constexpr (GC >= 2) l += neighbour<1>(l);
    if constexpr (GC >= 4) l += neighbour<2>(l);
    thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const int to_u = (int)(thread & 63) >> 4, to_c = (int)(thread & 15) / GC, to_gc = (int)(thread & 15) % GC;
    // where a combination's result goes
    auto destination = [&](uint32_t which) {
      const uint32_t i = which / (uint32_t)w.per, h = which - i * (uint32_t)w.per;
      return w.out + ((s.first + i) * w.q_heads + (int64_t)head * w.per + h) * D;
    };
    if constexpr (SHARE == 1) {
      const float inv = l > 0.f ? 1.0f / l : 0.f;
      const uint32_t which = ct * NC + to_c;
      if (which < s.rows * (uint32_t)w.per) {
        uint16_t* to = destination(which) + 4 * to_u;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          if ((dt >> 1) % GC == to_gc) {
            const f32x4 v = o[dt] * inv;
            *reinterpret_cast<uint2*>(to + dt * 16) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
          }
      }
      ct += gridDim.y;
      continue;
    }

    // ---- the four waves' shares, each against its own maximum, become one
    if (to_u == 0 && to_gc == 0) top_of[wave][to_c] = m, sum_of[wave][to_c] = l;
    __syncthreads();  // (and all waves have read their V)
    const float top = fmaxf(fmaxf(top_of[0][to_c], top_of[1][to_c]), fmaxf(top_of[2][to_c], top_of[3][to_c]));
    const float factor = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * sc);
    float* share = reinterpret_cast<float*>(region);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      if ((dt >> 1) % GC == to_gc) *reinterpret_cast<f32x4*>(share + wave * kShareFloats + to_c * D + dt * 16 + 4 * to_u) = o[dt] * factor;
    __syncthreads();
    float* part = nullptr;
    if (!complete)  // slot 0: begun by another worker, 1: begun here
      part = reinterpret_cast<float*>(w.workspace + (((size_t)gridDim.x * sizeof(PagedTail) + 255) & ~(size_t)255)) +
             (2 * (size_t)worker + (t0 == 0 ? 1 : 0)) * kPartFloats<NC, D>;
    for (int i = (int)thread; i < kShareFloats / 2; i += 256) {
      const int combo = 2 * i / D, dim = 2 * i % D;
      float2 v = *reinterpret_cast<const float2*>(share + 2 * i);
#pragma unroll
      for (int k = 1; k < 4; ++k) {
        const float2 z = *reinterpret_cast<const float2*>(share + k * kShareFloats + 2 * i);
        v.x += z.x, v.y += z.y;
      }
      float best = top_of[0][combo], total = 0.f;
#pragma unroll
      for (int k = 1; k < 4; ++k) best = fmaxf(best, top_of[k][combo]);
#pragma unroll
      for (int k = 0; k < 4; ++k) total += top_of[k][combo] == -INFINITY ? 0.f : sum_of[k][combo] * __builtin_amdgcn_exp2f((top_of[k][combo] - best) * sc);
      if (complete) {
        const uint32_t which = ct * NC + combo;
        if (which < s.rows * (uint32_t)w.per) {
          const float inv = total > 0.f ? 1.0f / total : 0.f;
          *reinterpret_cast<uint32_t*>(destination(which) + dim) = pack_bf16(v.x * inv, v.y * inv);
        }
      } else {
        *reinterpret_cast<float2*>(part + 2 * i) = v;
        if (dim == 0) part[NC * D + combo] = best * sc, part[NC * D + NC + combo] = total;
      }
    }
    if (whole) {
      ct += gridDim.y;
    } else if (!complete && t0 == 0 && threadIdx.x == 0) {
      PagedTail* tail = reinterpret_cast<PagedTail*>(w.workspace) + worker;
      tail->end = after, tail->owner = 1, tail->first = (uint32_t)s.first, tail->rows = s.rows, tail->head = (uint32_t)head, tail->tile = ct;
    }
    __syncthreads();  // the share has been read
  }
}

// Adds up the partial results of one sequence, key head and tile of combinations: the second slot of the worker that began it, then
// the first slots of those after it, in their order. SLICES workgroups to a worker of the other kernel; most have nothing to do. A part's
// floats are shared out over the slices and `kLanes` threads, the parts over the rest, eight requests of each under way at once.
template <int D, int NC, int SLICES>
__global__ __launch_bounds__(512) void paged_attention_join_kernel(PagedWork w, uint32_t workers) {
  constexpr int kLanes = NC * D / 4 / SLICES, kSets = 512 / kLanes;
  static_assert(kLanes <= 512, "one pass");
  const uint32_t g = blockIdx.x;
  const PagedTail t = reinterpret_cast<const PagedTail*>(w.workspace)[g];
  if (!t.owner) return;
  // the worker that has the segment's last unit: about (end - 1) groups / units
  uint32_t last = (uint32_t)((uint64_t)(t.end - 1) * t.groups / t.units);
  last = min(last, t.groups - 1);
  while (last + 1 < t.groups && first_unit(t.units, t.groups, last + 1) < t.end) ++last;
  while (first_unit(t.units, t.groups, last) >= t.end) --last;
  const uint32_t count = last - g + 1;
  const float* parts = reinterpret_cast<const float*>(w.workspace + (((size_t)workers * sizeof(PagedTail) + 255) & ~(size_t)255));
  auto part = [&](uint32_t i) { return parts + (2 * (size_t)(g + i) + (i == 0 ? 1 : 0)) * kPartFloats<NC, D>; };
  __shared__ float4 sums[kSets][kLanes];
  __shared__ float2 rest[kSets][kLanes];
  const int set = threadIdx.x / kLanes, lane = threadIdx.x % kLanes, at = (int)blockIdx.y * kLanes + lane;
  const int combo = at / (D / 4), dim = 4 * (at % (D / 4));
  float4 sum = make_float4(0, 0, 0, 0);
  float total = 0.f, top = -INFINITY;
  // a set's parts, against their own running maximum
  for (uint32_t i0 = set; i0 < count; i0 += 8 * kSets) {
    float4 v[8];
    float m[8], l[8], best = top;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float* p = part(min(i0 + k * kSets, count - 1));
      v[k] = *reinterpret_cast<const float4*>(p + 4 * at), m[k] = p[NC * D + combo], l[k] = p[NC * D + NC + combo];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (i0 + k * kSets >= count) m[k] = -INFINITY;
      best = fmaxf(best, m[k]);
    }
    const float to = best == -INFINITY ? 0.f : best, old = __builtin_amdgcn_exp2f(top - to);
    top = best;
    sum.x *= old, sum.y *= old, sum.z *= old, sum.w *= old, total *= old;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (m[k] == -INFINITY) continue;  // (one that saw no key, or none)
      const float f = __builtin_amdgcn_exp2f(m[k] - to);
      sum.x += v[k].x * f, sum.y += v[k].y * f, sum.z += v[k].z * f, sum.w += v[k].w * f, total += l[k] * f;
    }
  }
  sums[set][lane] = sum, rest[set][lane] = make_float2(top, total);
  __syncthreads();
  const uint32_t which = t.tile * NC + combo;
  if (set != 0 || which >= t.rows * (uint32_t)w.per) return;
  float best = top;
#pragma unroll
  for (int k = 1; k < kSets; ++k) best = fmaxf(best, rest[k][lane].x);
  float4 all = make_float4(0, 0, 0, 0);
  total = 0.f;
#pragma unroll
  for (int k = 0; k < kSets; ++k) {
    const float4 v = sums[k][lane];
    const float2 ml = rest[k][lane];
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - best);
    all.x += v.x * f, all.y += v.y * f, all.z += v.z * f, all.w += v.w * f, total += ml.y * f;
  }
  const float inv = total > 0.f ? 1.0f / total : 0.f;
  const uint32_t i = which / (uint32_t)w.per, h = which - i * (uint32_t)w.per;
  uint16_t* to = w.out + (((int64_t)t.first + i) * w.q_heads + (int64_t)t.head * w.per + h) * D + dim;
  *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16(all.x * inv, all.y * inv), pack_bf16(all.z * inv, all.w * inv));
}

// Columns to a combination: as many of the groups as leave room for the combinations that a sequence has on average. (Fewer columns are less
// work to a combination, but all combinations of a tile pay for it: 40 sequences of up to 3000 tokens with 8 query heads to a key head take
// 40 us with two columns and 52 with four and two tiles; with 16 query heads 8 of up to 16000 41 us with one column and 51 with two.)
int columns_of(int head_dim, int64_t rows, int64_t seqs, int64_t per) {
  const int64_t combinations = per * ((rows + seqs - 1) / seqs);
  if (head_dim == 128 && combinations <= 4) return 4;
  return combinations <= 8 ? 2 : 1;
}

// Tokens up to which a sequence is not split over workgroups: with 8 key heads, 64 sequences of up to 1000 tokens take 21 us whole and
// 27 split, one of 700 10.4 and 11.9; one of 2000 20 whole and 12 split, 200 of them 105 and 86 (64 of them 39 and 43).
// All measured with as many rows to each sequence. A sequence with many rows among others with few has its tiles of combinations one after
// another, in as many workgroups to a key head as the sequences need on average (the launch's y), where splitting would deal them out.
bool is_whole(int64_t most_keys) { return most_keys <= 1024; }

// Short sequences, and many for their length: a wave that has a sequence alone has nothing to share through LDS and to wait for, but the
// longest takes four times as long as with four waves. 128 sequences with 8 key heads and up to 120, 300, 600 and 1000 tokens take 10, 16,
// 25 and 37 us by the wave and 15, 19, 26 and 34 by four waves; 200 of up to 300, 500 and 600 23, 32 and 39 against 25, 29 and 34; 400 and
// 1000 of up to 500 50 and 104 against 55 and 119; 64 of up to 120 8.3 and 8.5, of up to 600 24 and 17.
bool is_by_wave(int64_t segments, int64_t most_keys) { return is_whole(most_keys) && 3 * segments >= 10 * most_keys; }

// Workgroups that join the parts of a segment. With parts of 2048 floats one is left with a single set of threads, which takes them eight
// at a time, one after another: up to 32 segments, of 24 parts and more, four of them do it sooner (16 rows and query heads to a key head, 4 key
// heads: one sequence of 20000 tokens 31 -> 23 us, 4 of up to 30000 34 -> 28, 8 of up to 16000 42 -> 41); with more segments the workgroups
// without work cost more (128 segments 52 -> 56), with smaller parts they do throughout (8 segments of 512 floats and 96 parts 52 -> 54).
constexpr int join_slices(int floats) { return floats == 2048 ? 4 : 1; }
constexpr int64_t kSlicedTiles = 64;  // (a bound that counts up to one tile too many to a sequence and key head)

}  // namespace

size_t paged_attention_workspace(int head_dim, int64_t rows, int64_t q_heads, int64_t kv_heads, int64_t seqs, int64_t) {
  // (whatever max_keys says: a sequence may be longer)
  const int64_t nc = 16 / columns_of(head_dim, rows, seqs, q_heads / kv_heads), workers = most_workers(16 / (int)nc);
  return ((workers * sizeof(PagedTail) + 255) & ~(size_t)255) + 2 * workers * nc * (head_dim + 2) * sizeof(float);
}

hipError_t launch_paged_attention(int scale_kind, bool asym, int head_dim, const PagedPool& pool, const uint16_t* q, int64_t rows,
                                  int64_t q_heads, const int32_t* table, int64_t seqs, int64_t max_pages, const int32_t* lens,
                                  const int32_t* starts, const int32_t* positions, float scale, int64_t max_keys, uint16_t* out,
                                  void* workspace, hipStream_t s) {
  const int64_t per = q_heads / pool.kv_heads, width = max_pages << pool.page_log2;
  const int64_t most_keys = max_keys > 0 && max_keys < width ? max_keys : width;
  const int gc = columns_of(head_dim, rows, seqs, per), nc = 16 / gc;
  const bool whole = is_whole(most_keys);
  // at most so many tiles of combinations have all sequences together, and so many units
  const int64_t tiles = (rows * per / nc + (seqs < rows ? seqs : rows)) * pool.kv_heads, tokens = (width + kTile - 1) / kTile;
  int unit_log2 = 0;
  while (tiles >= (int64_t(1) << 31) / ((tokens >> unit_log2) + 1 + kStart)) ++unit_log2;
  const PagedWork w = {q, out, static_cast<uint8_t*>(workspace), rows, max_pages, (int)seqs, (int)q_heads, (int)per,
                       scale * 1.4426950408889634f, whole ? 1 : 0, unit_log2};
  const size_t values = 4 * kTile * (size_t)head_dim / 2, shares = 4 * (size_t)nc * head_dim * sizeof(float);
  const int64_t segments = seqs * pool.kv_heads;
  const bool by_wave = is_by_wave(segments, most_keys);
  dim3 grid;
  int64_t workers = 0;
  size_t lds = by_wave || shares < values ? values : shares;
  if (whole) {
    // tiles of combinations of one sequence: as many as there are on average, at least
    const int64_t ct = (rows * per + seqs * nc - 1) / (seqs * nc);
    grid = dim3((unsigned)(by_wave ? (segments + 3) / 4 : segments), (unsigned)(ct < 1024 ? ct : 1024));
  } else {
    const int64_t units = tiles * ((((most_keys + kTile - 1) / kTile) >> unit_log2) + 1 + kStart) / 4 + 1;
    workers = units < most_workers(gc) ? units : most_workers(gc);
    grid = dim3((unsigned)workers);
    lds += sequences_bytes(seqs);
  }
  auto go = [&]<int SK, bool ASYM, int D, int GC>() {
    if (!by_wave)
      hipLaunchKernelGGL((paged_attention_kernel<SK, ASYM, D, GC, 4>), grid, dim3(256), lds, s, pool, w, table, lens, starts, positions);
    else
      hipLaunchKernelGGL((paged_attention_kernel<SK, ASYM, D, GC, 1>), grid, dim3(256), lds, s, pool, w, table, lens, starts, positions);
    if (whole) return hipGetLastError();
    constexpr int kSlices = join_slices(16 / GC * D);
    if (kSlices > 1 && tiles <= kSlicedTiles)
      hipLaunchKernelGGL((paged_attention_join_kernel<D, 16 / GC, kSlices>), dim3((unsigned)workers, kSlices), dim3(512), 0, s, w, (uint32_t)workers);
    else
      hipLaunchKernelGGL((paged_attention_join_kernel<D, 16 / GC, 1>), dim3((unsigned)workers), dim3(512), 0, s, w, (uint32_t)workers);
    return hipGetLastError();
  };
  auto with_format = [&]<int SK, bool ASYM>() {
    if (head_dim == 128)
      return gc == 4 ? go.template operator()<SK, ASYM, 128, 4>()
             : gc == 2 ? go.template operator()<SK, ASYM, 128, 2>()
                       : go.template operator()<SK, ASYM, 128, 1>();
    return gc == 2 ? go.template operator()<SK, ASYM, 64, 2>() : go.template operator()<SK, ASYM, 64, 1>();
  };
  switch (scale_kind) {
    case kScaleE5M2: return asym ? with_format.template operator()<kScaleE5M2, true>() : with_format.template operator()<kScaleE5M2, false>();
    case kScaleE4M3: return asym ? with_format.template operator()<kScaleE4M3, true>() : with_format.template operator()<kScaleE4M3, false>();
    default: return asym ? with_format.template operator()<kScaleE8M0Floor, true>() : with_format.template operator()<kScaleE8M0Floor, false>();
  }
}

}  // namespace amx
