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

// Inclusive prefix sums over 256 threads that stay at `cap` once they reach it (cap + cap fits; min(a + b, cap) is associative).
__device__ __forceinline__ uint32_t scan_capped(uint32_t v, uint32_t cap, uint32_t* waves) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(v, o, 64);
    if (lane >= o) v = v + u < cap ? v + u : cap;
  }
  __syncthreads();  // `waves` may still be read from the scan before
  if (lane == 63) waves[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v = v + waves[w] < cap ? v + waves[w] : cap;
  return v;
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
__global__ __launch_bounds__(256) void paged_plan_kernel(const int32_t* __restrict__ lens, const int32_t* __restrict__ new_rows,
                                                         int seqs, uint32_t rows, int page_log2, uint32_t pages,
                                                         uint32_t max_pages, const int32_t* __restrict__ state,
                                                         int32_t* queue, int32_t* table, int32_t* __restrict__ lens_out,
                                                         int32_t* __restrict__ starts, int32_t* __restrict__ slots,
                                                         int32_t* __restrict__ positions, int32_t* __restrict__ state_out) {
  extern __shared__ uint32_t sums[];
  __shared__ uint32_t waves[4], taken_of[4], refused_of[4];
  uint32_t* ends = sums;                  // rows up to and with the sequence
  uint32_t* first = sums + seqs;          // pages taken before it, kRefused if it is refused or has no rows
  uint32_t* back = sums + 2 * seqs;       // pages given back up to and with it
  constexpr uint32_t kRefused = ~0u;
  const uint32_t most = max_pages << page_log2, page_mask = (1u << page_log2) - 1;
  const uint32_t head = (uint32_t)state[0] % pages;
  const uint32_t count = state[1] < 0 ? 0u : min((uint32_t)state[1], pages);
  const int each = (seqs + 255) >> 8, b0 = threadIdx.x * each, b1 = min(seqs, b0 + each);
  auto held = [&](int b) { return lens[b] < 0 ? 0u : min((uint32_t)lens[b], most); };
  auto pages_of = [&](uint32_t tokens) { return (tokens + page_mask) >> page_log2; };

  uint32_t sum = 0, given = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = new_rows[b];
    sum = min(sum + min((uint32_t)max(n, 0), rows + 1), rows + 1);
    given = min(given + (n < 0 ? pages_of(held(b)) : 0u), pages);
    ends[b] = sum, back[b] = given;
  }
  const uint32_t sum_here = scan_capped(sum, rows + 1, waves), given_here = scan_capped(given, pages, waves);
  // what lies before this thread's sequences: the sums up to the thread before
  __shared__ uint32_t edge[256], edge2[256];
  edge[threadIdx.x] = sum_here, edge2[threadIdx.x] = given_here;
  __syncthreads();
  const uint32_t sum_before = threadIdx.x ? edge[threadIdx.x - 1] : 0, given_before = threadIdx.x ? edge2[threadIdx.x - 1] : 0;
  uint32_t want = 0;
  for (int b = b0; b < b1; ++b) {
    ends[b] = min(ends[b] + sum_before, rows + 1);
    back[b] = min(back[b] + given_before, pages);
    const int n = new_rows[b];
    const uint32_t h = held(b);
    const bool fits = n > 0 && (uint32_t)n <= most - h && ends[b] <= rows;
    const uint32_t w = fits ? pages_of(h + n) - pages_of(h) : 0u;
    first[b] = fits ? w : kRefused;
    want = min(want + w, pages + 1);
  }
  const uint32_t want_here = scan_capped(want, pages + 1, waves);
  __syncthreads();
  edge[threadIdx.x] = want_here;
  __syncthreads();
  uint32_t upto = threadIdx.x ? edge[threadIdx.x - 1] : 0, taken = 0, refused = 0;
  for (int b = b0; b < b1; ++b) {
    const uint32_t w = first[b];
    const bool fits = w != kRefused;
    const uint32_t before = upto;
    if (fits) upto = min(upto + w, pages + 1);
    const bool ok = fits && (w == 0 || upto <= count);
    if (upto <= count) taken = upto;
    first[b] = ok ? before : kRefused;
    refused += !ok && new_rows[b] > 0;
  }
  __syncthreads();

  const uint32_t total = min(ends[seqs - 1], rows);
  const uint32_t stride = gridDim.x * 256u, me = blockIdx.x * 256u + threadIdx.x;
  for (uint64_t t64 = me; t64 < rows; t64 += stride) {
    const uint32_t t = (uint32_t)t64;
    int32_t pos = -1, slot = -1;
    if (t < total) {
      const int b = first_above(ends, seqs, t);
      const uint32_t begin = first[b];
      if (begin != kRefused) {
        const uint32_t h = held(b), p = h + (t - (b ? ends[b - 1] : 0)), number = p >> page_log2, old = pages_of(h);
        int32_t* entry = table + (int64_t)b * max_pages + number;
        int32_t page;
        if (number >= old) {
          page = queue[(head + (begin + number - old)) % pages];
          if ((p & page_mask) == 0) *entry = page;
        } else {
          page = *entry;
        }
        pos = (int32_t)p;
        // (an id outside the pool has no slot)
        slot = (uint32_t)page < pages ? (int32_t)(((uint32_t)page << page_log2) + (p & page_mask)) : -1;
      }
    }
    slots[t] = slot, positions[t] = pos;
  }
  const uint32_t given_all = min(back[seqs - 1], pages - count);
  for (uint32_t i = me; i < given_all; i += stride) {
    const int b = first_above(back, seqs, i);
    const uint32_t p = i - (b ? back[b - 1] : 0);
    queue[(head + count + i) % pages] = table[(int64_t)b * max_pages + p];
  }
  if (blockIdx.x != 0) return;
  for (int b = threadIdx.x; b < seqs; b += 256) {
    const int n = new_rows[b];
    lens_out[b] = n < 0 ? 0 : (int32_t)(held(b) + (first[b] != kRefused ? (uint32_t)n : 0u));
    starts[b + 1] = (int32_t)min(ends[b], rows);
  }
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
// sines and cosines of its rows. Heads 0 .. q_heads - 1 are queries, the next kv_heads keys, the rest values. Same
// arithmetic as split_heads_rope_kernel and the cast: same bits.
constexpr int kWriteRows = 4, kWriteHeads = 16;
template <int SCALE_KIND, bool ASYM, int D>
__global__ __launch_bounds__(256) void paged_write_kernel(const float* __restrict__ in, int64_t rows, int64_t ld, int q_heads,
                                                          const int32_t* __restrict__ slots, const int32_t* __restrict__ positions,
                                                          double log_theta, uint16_t* __restrict__ q_out, PagedPool pool) {
  constexpr int kHalf = D / 2, kRuns = D / 16;
  __shared__ double2 turn[kWriteRows * kHalf];  // dimension 8 j + e of row t at [e][t][j]
  const int heads = q_heads + 2 * (int)pool.kv_heads;
  const int h0 = blockIdx.y * kWriteHeads, nh = min(heads - h0, kWriteHeads);
  const int64_t t0 = (int64_t)blockIdx.x * kWriteRows;
  const int nt = (int)min(rows - t0, (int64_t)kWriteRows);
  const int turned = q_heads + (int)pool.kv_heads;
  if (h0 < turned)
    for (int a = threadIdx.x; a < nt * kHalf; a += 256) {
      const int t = a / kHalf, i = a % kHalf;
      const double ang = (double)positions[t0 + t] * exp(-log_theta * (double)i / (double)kHalf);
      double sn, cs;
      sincos(ang, &sn, &cs);
      turn[(i & 7) * (kWriteRows * kRuns) + t * kRuns + (i >> 3)] = make_double2(sn, cs);
    }
  __syncthreads();
  const uint64_t size = (uint64_t)pool.pages << pool.page_log2;
  for (int it = threadIdx.x; it < nt * nh * kRuns; it += 256) {
    const int j = it % kRuns, th = it / kRuns, t = th / nh, h = h0 + th % nh;  // (the same t and h for the four threads of a group)
    const float* p = in + (t0 + t) * ld + (int64_t)h * D + 8 * j;
    float x1[8], x2[8];
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 a = *reinterpret_cast<const float4*>(p + e), b = *reinterpret_cast<const float4*>(p + kHalf + e);
      x1[e] = a.x, x1[e + 1] = a.y, x1[e + 2] = a.z, x1[e + 3] = a.w;
      x2[e] = b.x, x2[e + 1] = b.y, x2[e + 2] = b.z, x2[e + 3] = b.w;
    }
    if (h < turned) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double2 r = turn[e * (kWriteRows * kRuns) + t * kRuns + j];
        const float a = x1[e], b = x2[e];
        x1[e] = (float)((double)a * r.y - (double)b * r.x);
        x2[e] = (float)((double)b * r.y + (double)a * r.x);
      }
    }
    const uint32_t d1[4] = {pack2(x1[0], x1[1]), pack2(x1[2], x1[3]), pack2(x1[4], x1[5]), pack2(x1[6], x1[7])};
    const uint32_t d2[4] = {pack2(x2[0], x2[1]), pack2(x2[2], x2[3]), pack2(x2[4], x2[5]), pack2(x2[6], x2[7])};
    if (h < q_heads) {
      if (positions[t0 + t] < 0) continue;
      uint16_t* q = q_out + ((t0 + t) * q_heads + h) * D + 8 * j;
      *reinterpret_cast<uint4*>(q) = make_uint4(d1[0], d1[1], d1[2], d1[3]);
      *reinterpret_cast<uint4*>(q + kHalf) = make_uint4(d2[0], d2[1], d2[2], d2[3]);
      continue;
    }
    const int32_t slot = slots[t0 + t];
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
  const int64_t blocks = (rows + 1023) / 1024;
  hipLaunchKernelGGL(paged_plan_kernel, dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(256), 3 * sizeof(uint32_t) * (size_t)seqs,
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
  const int64_t heads = q_heads + 2 * pool->kv_heads;
  const dim3 grid((unsigned)((rows + kWriteRows - 1) / kWriteRows), (unsigned)((heads + kWriteHeads - 1) / kWriteHeads));
  for_pool(fmt, pool, [&]<int SK, bool ASYM, int D>() {
    hipLaunchKernelGGL((paged_write_kernel<SK, ASYM, D>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), in, rows, ld,
                       (int)q_heads, slots, positions, log(theta), static_cast<uint16_t*>(q_out_bf16), view(pool));
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
    const dim3 grid((unsigned)((rows * pool->kv_heads * (D / 8) + 255) / 256), 2);
    if (out_dtype == 1)
      hipLaunchKernelGGL((paged_read_kernel<kFormat, ASYM, D, true>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), slots,
                         rows, view(pool), k_out, v_out);
    else
      hipLaunchKernelGGL((paged_read_kernel<kFormat, ASYM, D, false>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), slots,
                         rows, view(pool), k_out, v_out);
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
  if (!(scale > 0.f) || isinf(scale)) return report_error(AMX_ERR_INVALID_ARG, "paged_attention: scale must be positive and finite");
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
