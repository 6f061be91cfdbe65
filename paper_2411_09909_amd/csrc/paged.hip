// The paged key / value cache (include/amxfp4_paged.h): a step's bookkeeping, the rows that are written and read back.
#include "../../include/amxfp4_paged.h"

#include <math.h>

#include "cast_core.h"
#include "device_formats.h"
#include "kernels.h"
#include "layer_math.h"
#include "paged.h"

namespace amx {
namespace {

// ---- bookkeeping ----------------------------------------------------------------------------------------------------

// Three inclusive prefix sums over 256 threads that stay at their caps once they reach them (cap + cap fits; min(a + b, cap) is
// associative); before: the sums up to the thread before.
struct Sums {
  uint32_t rows, given, want;
};
__device__ __forceinline__ Sums add_capped(Sums a, Sums b, Sums cap) {
  return {min(a.rows + b.rows, cap.rows), min(a.given + b.given, cap.given), min(a.want + b.want, cap.want)};
}
__device__ __forceinline__ Sums scan_before(Sums v, Sums cap, Sums* waves) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const Sums u = {__shfl_up(v.rows, o, 64), __shfl_up(v.given, o, 64), __shfl_up(v.want, o, 64)};
    if (lane >= o) v = add_capped(v, u, cap);
  }
  if (lane == 63) waves[wave] = v;
  Sums before = {__shfl_up(v.rows, 1, 64), __shfl_up(v.given, 1, 64), __shfl_up(v.want, 1, 64)};
  if (lane == 0) before = {0, 0, 0};
  __syncthreads();
  for (int w = 0; w < wave; ++w) before = add_capped(before, waves[w], cap);
  return before;
}

// the first of n ascending numbers that is greater than x, n if none is
__device__ __forceinline__ int first_above(const uint32_t* v, int n, uint32_t x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (v[mid] > x)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

// Every workgroup works out the sums over the sequences for itself (a few words a thread, out of the caches), then takes its
// share of the rows and of the pages given back: one launch, and no workgroup waits for another. What is read (lens, state, the
// queue's entries in use, table entries of pages held) is nowhere written.
// One scan does for all: a sequence that ends behind the batch's last row is refused, and so are all after it, so what they would have
// taken changes nothing.
// Bound by the chain of one load, the scan and one more load, not by bytes: 4.7 us for 64 sequences of a token each, 8.8 us for 1000
// sequences with 28000 rows. The rows of a sequence with few of them (decoding) are written by the thread that has the sequence; those
// of longer ones are shared out, a row to a thread, each finding its sequence in the sums. With the search for all rows, a scan to each
// sum and four rows to a thread the same took 6.4 and 13.3 us.
constexpr int kDirectRows = 8;
__global__ __launch_bounds__(256) void paged_plan_kernel(const int32_t* __restrict__ lens, const int32_t* __restrict__ new_rows,
                                                         int seqs, uint32_t rows, int page_log2, uint32_t pages,
                                                         uint32_t max_pages, const int32_t* __restrict__ state,
                                                         int32_t* queue, int32_t* table, int32_t* __restrict__ lens_out,
                                                         int32_t* __restrict__ starts, int32_t* __restrict__ slots,
                                                         int32_t* __restrict__ positions, int32_t* __restrict__ state_out) {
  extern __shared__ uint32_t sums[];
  __shared__ Sums waves[4];
  __shared__ uint32_t taken_of[4], refused_of[4], shared_out;
  uint32_t* ends = sums;                  // rows up to and with the sequence
  uint32_t* first = sums + seqs;          // its new rows; then: pages taken before it, kRefused if it is refused or has no rows
  uint32_t* back = sums + 2 * seqs;       // pages given back up to and with it
  uint32_t* held_in = sums + 3 * seqs;    // the tokens it has
  constexpr uint32_t kRefused = ~0u;
  const uint32_t most = max_pages << page_log2, page_mask = (1u << page_log2) - 1;
  const int each = (seqs + 255) >> 8, b0 = threadIdx.x * each, b1 = min(seqs, b0 + each);
  auto held_of = [&](int len) { return len < 0 ? 0u : min((uint32_t)len, most); };
  auto pages_of = [&](uint32_t tokens) { return (tokens + page_mask) >> page_log2; };
  const Sums cap = {rows + 1, pages, pages + 1};
  auto sums_of = [&](uint32_t held, int n) {
    const bool room = n > 0 && (uint32_t)n <= most - held;
    const uint32_t more = n > 0 ? (uint32_t)n : 0u, given = n < 0 ? pages_of(held) : 0u;
    const uint32_t want = room ? pages_of(held + more) - pages_of(held) : 0u;
    return add_capped(Sums{more < cap.rows ? more : cap.rows, given, want < cap.want ? want : cap.want}, Sums{0, 0, 0}, cap);
  };
  for (int b = threadIdx.x; b < seqs; b += 256) held_in[b] = held_of(lens[b]), first[b] = (uint32_t)new_rows[b];
  const int32_t state0 = state[0], state1 = state[1];
  if (threadIdx.x == 0) shared_out = 0;
  __syncthreads();
  Sums mine = {0, 0, 0};
  for (int b = b0; b < b1; ++b) mine = add_capped(mine, sums_of(held_in[b], (int)first[b]), cap);
  Sums upto = scan_before(mine, cap, waves);
  const uint32_t head = (uint32_t)state0 % pages, count = state1 < 0 ? 0u : min((uint32_t)state1, pages);

  auto place = [&](uint32_t t, int b, uint32_t held, uint32_t before, uint32_t i) {  // row t: the sequence's i-th new one
    const uint32_t p = held + i, number = p >> page_log2, old = pages_of(held);
    int32_t* entry = table + (int64_t)b * max_pages + number;
    int32_t page;
    if (number >= old) {
      page = queue[(head + (before + number - old)) % pages];
      if ((p & page_mask) == 0) *entry = page;
    } else {
      page = *entry;
    }
    positions[t] = (int32_t)p;
    // (an id outside the pool has no slot)
    slots[t] = (uint32_t)page < pages ? (int32_t)(((uint32_t)page << page_log2) + (p & page_mask)) : -1;
  };
  uint32_t taken = 0, refused = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = (int)first[b];
    const uint32_t held = held_in[b];
    const Sums own = sums_of(held, n), now = add_capped(upto, own, cap);
    const bool fits = n > 0 && (uint32_t)n <= most - held && now.rows <= rows, ok = fits && (own.want == 0 || now.want <= count);
    if (ok && now.want <= count) taken = now.want;  // (behind one refused for its pages the sum stays above count)
    refused += n > 0 && !ok;
    ends[b] = now.rows, first[b] = ok ? upto.want : kRefused, back[b] = now.given;
    // rows of the last sequence that is cut off end with the batch
    const uint32_t begin = min(upto.rows, rows), end = min(now.rows, rows);
    if (end - begin > kDirectRows) {
      shared_out = 1;
    } else if ((uint32_t)(b - b0) % gridDim.x == blockIdx.x) {
      for (uint32_t t = begin; t < end; ++t) {
        if (ok)
          place(t, b, held, upto.want, t - begin);
        else
          slots[t] = -1, positions[t] = -1;
      }
    }
    if (blockIdx.x == 0) {
      lens_out[b] = n < 0 ? 0 : (int32_t)(held + (ok ? (uint32_t)n : 0u));
      starts[b + 1] = (int32_t)end;
    }
    upto = now;
  }
  __syncthreads();

  const uint32_t total = min(ends[seqs - 1], rows);
  const uint32_t stride = gridDim.x * 256u, me = blockIdx.x * 256u + threadIdx.x;
  for (uint64_t t = (shared_out ? 0 : total) + (uint64_t)me; t < rows; t += stride) {
    if (t >= total) {
      slots[t] = -1, positions[t] = -1;
      continue;
    }
    const int b = first_above(ends, seqs, (uint32_t)t);
    const uint32_t begin = b ? ends[b - 1] : 0u, end = min(ends[b], rows);
    if (end - begin <= kDirectRows) continue;  // its sequence's thread has written it
    if (first[b] != kRefused)
      place((uint32_t)t, b, held_in[b], first[b], (uint32_t)t - begin);
    else
      slots[t] = -1, positions[t] = -1;
  }
  const uint32_t given_all = min(back[seqs - 1], pages - count);
  for (uint32_t i = me; i < given_all; i += stride) {
    const int b = first_above(back, seqs, i);
    const uint32_t p = i - (b ? back[b - 1] : 0);
    queue[(head + count + i) % pages] = table[(int64_t)b * max_pages + p];
  }
  if (blockIdx.x != 0) return;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    taken = max(taken, (uint32_t)__shfl_xor(taken, o, 64));
    refused += __shfl_xor(refused, o, 64);
  }
  if ((threadIdx.x & 63) == 0) taken_of[threadIdx.x >> 6] = taken, refused_of[threadIdx.x >> 6] = refused;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4; ++w) taken = max(taken, taken_of[w]), refused += refused_of[w];
    starts[0] = 0;
    state_out[0] = (int32_t)((head + taken) % pages), state_out[1] = (int32_t)(count - taken + given_all);
    state_out[2] = (int32_t)refused, state_out[3] = (int32_t)total;
  }
}

// ---- rows into the cache --------------------------------------------------------------------------------------------

// The work is cut as in rope_quantize_kernel (layer_ops.hip): items of (row, head, run of 8 dimensions below head_dim / 2 and
// the 8 head_dim / 2 further on), four neighbouring threads to a group of 32; the workgroup's threads first work out the FP64
// sines and cosines of its rows, while the loads of their first items are under way. Heads 0 .. q_heads - 1 are queries, the next
// kv_heads keys, the rest values. Same arithmetic as split_heads_rope_kernel and the cast: same bits.
// A thread keeps its row and run and goes from head to head, so that a sine and cosine leaves the LDS once.
// `per_group` heads to a workgroup: with few rows the eight of one go (sixteen of 64 dimensions), so that there are workgroups enough
// (1 row of 48 heads 3.7 us against 5.2 with all heads, 256 rows of 80 heads 6.0 against 9.6); with many all of them, so that the
// angles are worked out once: 9500 rows of 48 heads 66 us against 68, 330 MB read and written at 5.0 TB/s.
constexpr int kWriteRows = 4, kWriteManyGroups = 512;
__device__ __forceinline__ uint32_t pack_rne(float a, float b) {
  typedef __bf16 bf16_2 __attribute__((ext_vector_type(2)));
  typedef float float_2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float_2{a, b}), bf16_2));
}
template <int SCALE_KIND, bool ASYM, int D>
__global__ __launch_bounds__(256) void paged_write_kernel(const float* __restrict__ in, int64_t rows, int64_t ld, int q_heads,
                                                          const int32_t* __restrict__ slots, const int32_t* __restrict__ positions,
                                                          double log_theta, int per_group, uint16_t* __restrict__ q_out, PagedPool pool) {
  constexpr int kHalf = D / 2, kRuns = D / 16;
  __shared__ double2 turn[kWriteRows * kHalf];  // dimension 8 j + e of row t at [e][t][j]
  const int heads = q_heads + 2 * (int)pool.kv_heads;
  const int h0 = blockIdx.y * per_group, nh = min(heads - h0, per_group);
  const int64_t t0 = (int64_t)blockIdx.x * kWriteRows;
  const int nt = (int)min(rows - t0, (int64_t)kWriteRows);
  const int turned = q_heads + (int)pool.kv_heads;
  const int j = threadIdx.x % kRuns, t = threadIdx.x / kRuns % kWriteRows;
  constexpr int kHeads = 256 / (kRuns * kWriteRows);  // of one go
  const int first = threadIdx.x / (kRuns * kWriteRows), last = t < nt ? h0 + nh : 0;
  float4 next[4];
  const float* row_in = in + (t0 + min(t, nt - 1)) * ld + 8 * j;
  auto request = [&](int h) {  // (past the last head: the last one again, not used)
    const float* p = row_in + (int64_t)min(h, heads - 1) * D;
    next[0] = *reinterpret_cast<const float4*>(p), next[1] = *reinterpret_cast<const float4*>(p + 4);
    next[2] = *reinterpret_cast<const float4*>(p + kHalf), next[3] = *reinterpret_cast<const float4*>(p + kHalf + 4);
  };
  request(h0 + first);
  if (h0 < turned)
    for (int a = threadIdx.x; a < nt * kHalf; a += 256) {
      const int ta = a / kHalf, i = a % kHalf;
      const int32_t pos = positions[t0 + ta];
      const double inv = exp(-log_theta * (double)i / (double)kHalf);
      double sn, cs;
      sincos((double)pos * inv, &sn, &cs);
      turn[(i & 7) * (kWriteRows * kRuns) + ta * kRuns + (i >> 3)] = make_double2(sn, cs);
    }
  __syncthreads();
  const uint64_t size = (uint64_t)pool.pages << pool.page_log2;
  double2 r[8];
  int32_t position = 0, slot = -1;
  if (t < nt) {
    position = positions[t0 + t], slot = slots[t0 + t];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = turn[e * (kWriteRows * kRuns) + t * kRuns + j];
  }
  for (int h = h0 + first; h < last; h += kHeads) {  // (the same h for the four threads of a group)
    float x1[8] = {next[0].x, next[0].y, next[0].z, next[0].w, next[1].x, next[1].y, next[1].z, next[1].w};
    float x2[8] = {next[2].x, next[2].y, next[2].z, next[2].w, next[3].x, next[3].y, next[3].z, next[3].w};
    if (h + kHeads < last) request(h + kHeads);
    if (h < turned) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = x1[e], b = x2[e];
        x1[e] = (float)((double)a * r[e].y - (double)b * r[e].x);
        x2[e] = (float)((double)b * r[e].y + (double)a * r[e].x);
      }
    }
    const uint32_t d1[4] = {pack_rne(x1[0], x1[1]), pack_rne(x1[2], x1[3]), pack_rne(x1[4], x1[5]), pack_rne(x1[6], x1[7])};
    const uint32_t d2[4] = {pack_rne(x2[0], x2[1]), pack_rne(x2[2], x2[3]), pack_rne(x2[4], x2[5]), pack_rne(x2[6], x2[7])};
    if (h < q_heads) {
      if (position < 0) continue;
      uint16_t* q = q_out + ((t0 + t) * q_heads + h) * D + 8 * j;
      *reinterpret_cast<uint4*>(q) = make_uint4(d1[0], d1[1], d1[2], d1[3]);
      *reinterpret_cast<uint4*>(q + kHalf) = make_uint4(d2[0], d2[1], d2[2], d2[3]);
      continue;
    }
    if (slot < 0 || (uint64_t)slot >= size) continue;
    uint32_t c1[1], c2[1], p1, n1, p2, n2;
    cast_words_bf16<SCALE_KIND, ASYM, 8>(d1, 2, c1, p1, n1);
    cast_words_bf16<SCALE_KIND, ASYM, 8>(d2, 2, c2, p2, n2);
    const bool value = h >= turned;
    const int g = h - (value ? turned : q_heads);
    const int64_t page_head = (int64_t)((uint32_t)slot >> pool.page_log2) * pool.kv_heads + g;
    const uint32_t place = (uint32_t)slot & ((1u << pool.page_log2) - 1);
    uint8_t* codes = (value ? pool.v_codes : pool.k_codes) + ((page_head << pool.page_log2) + place) * kHalf;
    *reinterpret_cast<uint32_t*>(codes + 4 * j) = c1[0];
    *reinterpret_cast<uint32_t*>(codes + kHalf / 2 + 4 * j) = c2[0];
    if ((j & 3) == 0) {
      constexpr int kGroups = D / 32;
      uint8_t* scales = value ? pool.v_scales : pool.k_scales;
      const int64_t s1 = ((page_head * kGroups + (j >> 2)) << pool.page_log2) + place;
      const int64_t s2 = s1 + ((int64_t)(kGroups / 2) << pool.page_log2);
      if constexpr (ASYM) {
        *reinterpret_cast<uint16_t*>(scales + 2 * s1) = (uint16_t)(p1 | (n1 << 8));
        *reinterpret_cast<uint16_t*>(scales + 2 * s2) = (uint16_t)(p2 | (n2 << 8));
      } else {
        scales[s1] = (uint8_t)p1, scales[s2] = (uint8_t)p2;
      }
    }
  }
}

// ---- rows out of the cache ------------------------------------------------------------------------------------------

// One thread to 8 elements of K or V (blockIdx.y).
template <int SCALE_KIND, bool ASYM, int D, bool OUT_BF16>
__global__ __launch_bounds__(256) void paged_read_kernel(const int32_t* __restrict__ slots, int64_t rows, PagedPool pool,
                                                         void* __restrict__ k_out, void* __restrict__ v_out) {
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int j = (int)(item % (D / 8));
  const int64_t th = item / (D / 8), row = th / pool.kv_heads;
  if (row >= rows) return;
  const int g = (int)(th - row * pool.kv_heads);
  const uint8_t* codes = blockIdx.y ? pool.v_codes : pool.k_codes;
  const uint8_t* scales = blockIdx.y ? pool.v_scales : pool.k_scales;
  const int32_t slot = slots[row];
  uint32_t w = 0;
  float s_pos = 0.f, s_neg = 0.f;
  if (slot >= 0 && (uint64_t)slot < (uint64_t)pool.pages << pool.page_log2) {
    const int64_t page_head = (int64_t)((uint32_t)slot >> pool.page_log2) * pool.kv_heads + g;
    const uint32_t place = (uint32_t)slot & ((1u << pool.page_log2) - 1);
    w = *reinterpret_cast<const uint32_t*>(codes + ((page_head << pool.page_log2) + place) * (D / 2) + 4 * j);
    const int64_t s = ((page_head * (D / 32) + (j >> 2)) << pool.page_log2) + place;
    if constexpr (ASYM) {
      const uint32_t sb = *reinterpret_cast<const uint16_t*>(scales + 2 * s);
      s_pos = scale_value<SCALE_KIND>(sb & 255u), s_neg = scale_value<SCALE_KIND>(sb >> 8);
    } else {
      s_pos = s_neg = scale_value<SCALE_KIND>(scales[s]);
    }
  }
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t n = (w >> (4 * e)) & 15u;
    v[e] = (float)e2m1_twice(n & 7u) * ((n & 8u) ? -0.5f * s_neg : 0.5f * s_pos);  // at most 6 significant bits: exact
  }
  void* out = blockIdx.y ? v_out : k_out;
  if constexpr (OUT_BF16) {
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (f2u(v[2 * e]) >> 16) | (f2u(v[2 * e + 1]) & 0xFFFF0000u);
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + item * 8) = make_uint4(o[0], o[1], o[2], o[3]);
  } else {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(out) + item * 8);
    o[0] = make_float4(v[0], v[1], v[2], v[3]), o[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
int done(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AMX_OK : report_hip_error(e, what);
}
constexpr int64_t kMaxTokens = int64_t(1) << 30, kMaxRows = int64_t(1) << 24, kMaxHeads = 1024, kMaxQueries = int64_t(1) << 31;

// log2 of a page size that is taken, else -1
int page_log2(int64_t page_size) {
  for (int l = 4; l <= 10; ++l)
    if (page_size == int64_t(1) << l) return l;
  return -1;
}

int check(const amx_format_t* fmt, const amx_paged_pool_t* pool) {
  if (!fmt || !pool) return report_error(AMX_ERR_INVALID_ARG, "paged cache: fmt or pool is NULL");
  if (fmt->elem != AMX_ELEM_FP4_E2M1 || fmt->scale < AMX_SCALE_E8M0_FLOOR || fmt->scale > AMX_SCALE_FP8_E4M3 ||
      (fmt->asymmetric != 0 && fmt->asymmetric != 1) || fmt->group_size == 0 || fmt->group_size < -1)
    return report_error(AMX_ERR_INVALID_ARG, "paged cache: bad format");
  if (fmt->group_size != 32) return report_error(AMX_ERR_UNSUPPORTED, "paged cache: groups of 32 only");
  if (pool->pages <= 0 || pool->page_size <= 0 || pool->kv_heads <= 0 || pool->head_dim <= 0 || pool->reserved != 0)
    return report_error(AMX_ERR_INVALID_ARG, "paged cache: pages, page_size, kv_heads and head_dim must be positive, reserved 0");
  if (page_log2(pool->page_size) < 0)
    return report_error(AMX_ERR_UNSUPPORTED, "paged cache: page_size must be a power of two from 16 to 1024");
  if (pool->head_dim != 64 && pool->head_dim != 128) return report_error(AMX_ERR_UNSUPPORTED, "paged cache: head_dim must be 64 or 128");
  if (pool->pages > kMaxTokens / pool->page_size || pool->kv_heads > kMaxHeads)
    return report_error(AMX_ERR_INVALID_ARG, "paged cache: pages * page_size at most 2^30, kv_heads at most 1024");
  return AMX_OK;
}

int check_memory(const amx_paged_pool_t* pool) {
  if (!pool->k_codes || !pool->k_scales || !pool->v_codes || !pool->v_scales)
    return report_error(AMX_ERR_INVALID_ARG, "paged cache: NULL pointer in the pool");
  if (!aligned16(pool->k_codes) || !aligned16(pool->k_scales) || !aligned16(pool->v_codes) || !aligned16(pool->v_scales))
    return report_error(AMX_ERR_INVALID_ARG, "paged cache: the pool's memory must be 16-byte aligned");
  return AMX_OK;
}

PagedPool view(const amx_paged_pool_t* p) {
  return {p->k_codes, p->k_scales, p->v_codes, p->v_scales, (uint32_t)p->pages, (uint32_t)page_log2(p->page_size), (uint32_t)p->kv_heads};
}

// go<scale format, asymmetric, head_dim>() for the checked arguments
template <class Go>
void for_pool(const amx_format_t* fmt, const amx_paged_pool_t* pool, Go go) {
  auto with_dim = [&]<int SK, bool ASYM>() {
    pool->head_dim == 128 ? go.template operator()<SK, ASYM, 128>() : go.template operator()<SK, ASYM, 64>();
  };
  const bool asym = fmt->asymmetric != 0;
  switch (fmt->scale) {
    case AMX_SCALE_FP8_E5M2:
      asym ? with_dim.template operator()<kScaleE5M2, true>() : with_dim.template operator()<kScaleE5M2, false>();
      break;
    case AMX_SCALE_FP8_E4M3:
      asym ? with_dim.template operator()<kScaleE4M3, true>() : with_dim.template operator()<kScaleE4M3, false>();
      break;
    case AMX_SCALE_E8M0_FLOOR:
      asym ? with_dim.template operator()<kScaleE8M0Floor, true>() : with_dim.template operator()<kScaleE8M0Floor, false>();
      break;
    default: asym ? with_dim.template operator()<kScaleE8M0Round, true>() : with_dim.template operator()<kScaleE8M0Round, false>();
  }
}

}  // namespace
}  // namespace amx

using namespace amx;

extern "C" {

size_t amxfp4_paged_codes_bytes(const amx_format_t* fmt, const amx_paged_pool_t* pool) {
  if (check(fmt, pool) != AMX_OK) return 0;
  return (size_t)pool->pages * pool->page_size * pool->kv_heads * (pool->head_dim / 2);
}

size_t amxfp4_paged_scales_bytes(const amx_format_t* fmt, const amx_paged_pool_t* pool) {
  if (check(fmt, pool) != AMX_OK) return 0;
  return (size_t)pool->pages * pool->page_size * pool->kv_heads * (pool->head_dim / 32) * (fmt->asymmetric ? 2 : 1);
}

int amxfp4_paged_plan(const int32_t* lens, const int32_t* new_rows, int64_t seqs, int64_t rows, int64_t page_size, int64_t pages,
                      int64_t max_pages, const int32_t* state, int32_t* queue, int32_t* table, int32_t* lens_out, int32_t* starts,
                      int32_t* slots, int32_t* positions, int32_t* state_out, void* stream) {
  if (!lens || !new_rows || !state || !queue || !table || !lens_out || !starts || !slots || !positions || !state_out)
    return report_error(AMX_ERR_INVALID_ARG, "paged_plan: NULL pointer");
  for (const void* p : {(const void*)lens, (const void*)new_rows, (const void*)state, (const void*)queue, (const void*)table,
                        (const void*)lens_out, (const void*)starts, (const void*)slots, (const void*)positions, (const void*)state_out})
    if (!aligned4(p)) return report_error(AMX_ERR_INVALID_ARG, "paged_plan: pointers must be 4-byte aligned");
  if (seqs <= 0 || seqs > kPagedMaxSeqs || rows <= 0 || rows > kMaxTokens || page_size <= 0 || pages <= 0 || max_pages <= 0)
    return report_error(AMX_ERR_INVALID_ARG, "paged_plan: bad shape (1 to 4096 sequences, rows, pages and max_pages positive)");
  const int l = page_log2(page_size);
  if (l < 0) return report_error(AMX_ERR_UNSUPPORTED, "paged_plan: page_size must be a power of two from 16 to 1024");
  if (pages > kMaxTokens >> l || max_pages > kMaxTokens >> l)
    return report_error(AMX_ERR_INVALID_ARG, "paged_plan: pages and max_pages times page_size at most 2^30");
  if (lens_out == lens || state_out == state)
    return report_error(AMX_ERR_INVALID_ARG, "paged_plan: lens_out and state_out must be buffers of their own");
  const int64_t blocks = (rows + 255) / 256;
  hipLaunchKernelGGL(paged_plan_kernel, dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(256), 4 * sizeof(uint32_t) * (size_t)seqs,
                     reinterpret_cast<hipStream_t>(stream), lens, new_rows, (int)seqs, (uint32_t)rows, l, (uint32_t)pages,
                     (uint32_t)max_pages, state, queue, table, lens_out, starts, slots, positions, state_out);
  return done("paged_plan launch");
}

int amxfp4_paged_write(const amx_format_t* fmt, const amx_paged_pool_t* pool, const float* in, int64_t rows, int64_t ld,
                       int64_t q_heads, const int32_t* slots, const int32_t* positions, double theta, void* q_out_bf16,
                       void* stream) {
  if (int rc = check(fmt, pool); rc != AMX_OK) return rc;
  if (int rc = check_memory(pool); rc != AMX_OK) return rc;
  if (!in || !slots || !positions || !q_out_bf16) return report_error(AMX_ERR_INVALID_ARG, "paged_write: NULL pointer");
  if (rows <= 0 || rows > kMaxRows || q_heads <= 0 || q_heads > kMaxHeads || ld < (q_heads + 2 * pool->kv_heads) * pool->head_dim)
    return report_error(AMX_ERR_INVALID_ARG, "paged_write: bad shape (ld at least the width of queries, keys and values)");
  if (!(theta > 1.0) || isinf(theta)) return report_error(AMX_ERR_INVALID_ARG, "paged_write: theta must exceed 1 and be finite");
  if (!aligned16(in) || ld % 4 || !aligned16(q_out_bf16) || !aligned4(slots) || !aligned4(positions))
    return report_error(AMX_ERR_INVALID_ARG, "paged_write: in and q_out must be 16-byte aligned, ld a multiple of 4");
  const int64_t heads = q_heads + 2 * pool->kv_heads, groups = (rows + kWriteRows - 1) / kWriteRows;
  const int per_group = groups >= kWriteManyGroups ? (int)heads : (int)(256 / (pool->head_dim / 16 * kWriteRows));
  const dim3 grid((unsigned)groups, (unsigned)((heads + per_group - 1) / per_group));
  for_pool(fmt, pool, [&]<int SK, bool ASYM, int D>() {
    hipLaunchKernelGGL((paged_write_kernel<SK, ASYM, D>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), in, rows, ld,
                       (int)q_heads, slots, positions, log(theta), per_group, static_cast<uint16_t*>(q_out_bf16), view(pool));
  });
  return done("paged_write launch");
}

int amxfp4_paged_read(const amx_format_t* fmt, const amx_paged_pool_t* pool, const int32_t* slots, int64_t rows, int32_t out_dtype,
                      void* k_out, void* v_out, void* stream) {
  if (int rc = check(fmt, pool); rc != AMX_OK) return rc;
  if (int rc = check_memory(pool); rc != AMX_OK) return rc;
  if (!slots || !k_out || !v_out) return report_error(AMX_ERR_INVALID_ARG, "paged_read: NULL pointer");
  if (rows <= 0 || rows > kMaxRows) return report_error(AMX_ERR_INVALID_ARG, "paged_read: rows must be positive, at most 2^24");
  if (out_dtype != 0 && out_dtype != 1) return report_error(AMX_ERR_INVALID_ARG, "paged_read: out_dtype must be 0 or 1");
  if (!aligned16(k_out) || !aligned16(v_out) || !aligned4(slots))
    return report_error(AMX_ERR_INVALID_ARG, "paged_read: outputs must be 16-byte aligned");
  for_pool(fmt, pool, [&]<int SK, bool ASYM, int D>() {
    constexpr int kFormat = SK == kScaleE8M0Round ? kScaleE8M0Floor : SK;  // one encoding of the bytes
    // (a launch has fewer than 2^32 threads: rows at a time, which are all of them up to 2^34 elements of K)
    const int64_t row_items = (int64_t)pool->kv_heads * (D / 8), most = (int64_t(1) << 31) / row_items;
    for (int64_t r = 0; r < rows; r += most) {
      const int64_t n = rows - r < most ? rows - r : most, at = r * row_items * 8 * (out_dtype == 1 ? 2 : 4);
      const dim3 grid((unsigned)((n * row_items + 255) / 256), 2);
      void *k = static_cast<uint8_t*>(k_out) + at, *v = static_cast<uint8_t*>(v_out) + at;
      if (out_dtype == 1)
        hipLaunchKernelGGL((paged_read_kernel<kFormat, ASYM, D, true>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream),
                           slots + r, n, view(pool), k, v);
      else
        hipLaunchKernelGGL((paged_read_kernel<kFormat, ASYM, D, false>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream),
                           slots + r, n, view(pool), k, v);
    }
  });
  return done("paged_read launch");
}

size_t amxfp4_paged_attention_workspace_bytes(const amx_format_t* fmt, const amx_paged_pool_t* pool, int64_t rows, int64_t q_heads,
                                              int64_t seqs, int64_t max_keys) {
  if (check(fmt, pool) != AMX_OK || rows <= 0 || rows > kMaxRows || q_heads <= 0 || q_heads > kMaxHeads || q_heads % pool->kv_heads ||
      seqs <= 0 || seqs > kPagedMaxSeqs || max_keys < 0 || max_keys > kMaxTokens || rows * q_heads > kMaxQueries)
    return 0;
  return paged_attention_workspace(pool->head_dim, rows, q_heads, pool->kv_heads, seqs, max_keys);
}

int amxfp4_paged_attention(const amx_format_t* fmt, const amx_paged_pool_t* pool, const void* q_bf16, int64_t rows, int64_t q_heads,
                           const int32_t* table, int64_t seqs, int64_t max_pages, const int32_t* lens, const int32_t* starts,
                           const int32_t* positions, float scale, int64_t max_keys, void* out_bf16, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (int rc = check(fmt, pool); rc != AMX_OK) return rc;
  if (int rc = check_memory(pool); rc != AMX_OK) return rc;
  if (!q_bf16 || !table || !lens || !starts || !positions || !out_bf16)
    return report_error(AMX_ERR_INVALID_ARG, "paged_attention: NULL pointer");
  if (rows <= 0 || rows > kMaxRows || q_heads <= 0 || q_heads > kMaxHeads || q_heads % pool->kv_heads || seqs <= 0 ||
      seqs > kPagedMaxSeqs || max_pages <= 0 || max_pages > kMaxTokens / pool->page_size || max_keys < 0 || max_keys > kMaxTokens ||
      rows * q_heads > kMaxQueries)
    return report_error(AMX_ERR_INVALID_ARG, "paged_attention: bad shape (q_heads a multiple of kv_heads, 1 to 4096 sequences)");
  // (the kernel's scale is this times log2 e, which has to be finite too)
  if (!(scale > 0.f) || scale > 0x1p127f) return report_error(AMX_ERR_INVALID_ARG, "paged_attention: scale must be positive, at most 2^127");
  if (!aligned16(q_bf16) || !aligned16(out_bf16) || !aligned4(table) || !aligned4(lens) || !aligned4(starts) || !aligned4(positions))
    return report_error(AMX_ERR_INVALID_ARG, "paged_attention: q and out must be 16-byte aligned");
  const size_t need = paged_attention_workspace(pool->head_dim, rows, q_heads, pool->kv_heads, seqs, max_keys);
  if (need && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255)))
    return report_error(AMX_ERR_WORKSPACE, "paged_attention: workspace missing, too small or not 256-byte aligned");
  const hipError_t e =
      launch_paged_attention(fmt->scale, fmt->asymmetric != 0, pool->head_dim, view(pool), static_cast<const uint16_t*>(q_bf16), rows,
                             q_heads, table, seqs, max_pages, lens, starts, positions, scale, max_keys,
                             static_cast<uint16_t*>(out_bf16), workspace, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? AMX_OK : report_hip_error(e, "paged_attention launch");
}

}  // extern "C"
