// Attention over the paged cache (include/amxfp4_paged.h).
#include "paged.h"

#include "kernels.h"
#include "layer_math.h"

namespace amx {
namespace {

// One workgroup to a row and query head, its four waves take turns with the keys, the lanes share out the head dimension; running
// maximum and sum per wave, joined at the end.
template <int SCALE_KIND, bool ASYM, int D>
__global__ __launch_bounds__(256) void paged_attention_kernel(PagedPool pool, const uint16_t* __restrict__ q, int64_t rows, int q_heads,
                                                              const int32_t* __restrict__ table, int seqs, int64_t max_pages,
                                                              const int32_t* __restrict__ lens, const int32_t* __restrict__ starts,
                                                              const int32_t* __restrict__ positions, float scale_log2,
                                                              uint16_t* __restrict__ out) {
  __shared__ float share[4][D + 2];
  const int64_t t = blockIdx.x;
  const int h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int lo = 0, hi = seqs;  // the first sequence that ends behind the row
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid + 1] > t)
      hi = mid;
    else
      lo = mid + 1;
  }
  if (lo >= seqs || starts[lo] > t) return;
  const int64_t most = max_pages << pool.page_log2;
  const int64_t keys = min(min((int64_t)positions[t] + 1, (int64_t)lens[lo]), most);
  const int g = h / (q_heads / (int)pool.kv_heads);
  constexpr int E = D / 64;  // elements of a lane
  float qv[E], o[E] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) qv[e] = u2f((uint32_t)q[(t * q_heads + h) * D + lane * E + e] << 16);
  for (int64_t j = wave; j < keys; j += 4) {
    const uint32_t page = (uint32_t)table[lo * max_pages + (j >> pool.page_log2)];
    if (page >= pool.pages) continue;
    const int64_t page_head = (int64_t)page * pool.kv_heads + g, place = j & ((1 << pool.page_log2) - 1);
    auto value = [&](const uint8_t* codes, const uint8_t* scales, int d) {
      const uint32_t n = (codes[((page_head << pool.page_log2) + place) * (D / 2) + d / 2] >> (4 * (d & 1))) & 15u;
      const int64_t s = ((page_head * (D / 32) + d / 32) << pool.page_log2) + place;
      const float S = scale_value<SCALE_KIND>(ASYM ? scales[2 * s + (n >> 3)] : scales[s]);
      return (float)e2m1_twice(n & 7u) * (n & 8u ? -0.5f * S : 0.5f * S);
    };
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += qv[e] * value(pool.k_codes, pool.k_scales, lane * E + e);
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) s += __shfl_xor(s, w, 64);
    s *= scale_log2;
    const float m_new = fmaxf(m, s), alpha = __builtin_amdgcn_exp2f(m - m_new), p = __builtin_amdgcn_exp2f(s - m_new);
    m = m_new, l = l * alpha + p;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * alpha + p * value(pool.v_codes, pool.v_scales, lane * E + e);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) share[wave][lane * E + e] = o[e];
  share[wave][D] = m, share[wave][D + 1] = l;
  __syncthreads();
  if (threadIdx.x < D) {
    const float top = fmaxf(fmaxf(share[0][D], share[1][D]), fmaxf(share[2][D], share[3][D]));
    float sum = 0.f, total = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float f = share[w][D] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(share[w][D] - top);
      sum += share[w][threadIdx.x] * f, total += share[w][D + 1] * f;
    }
    out[(t * q_heads + h) * D + threadIdx.x] = (uint16_t)bf16_rne(total > 0.f ? sum / total : 0.f);
  }
}

}  // namespace

size_t paged_attention_workspace(int, int64_t, int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_paged_attention(int scale_kind, bool asym, int head_dim, const PagedPool& pool, const uint16_t* q, int64_t rows,
                                  int64_t q_heads, const int32_t* table, int64_t seqs, int64_t max_pages, const int32_t* lens,
                                  const int32_t* starts, const int32_t* positions, float scale, int64_t max_keys, uint16_t* out,
                                  void* workspace, hipStream_t s) {
  auto go = [&]<int SK, bool ASYM>() {
    auto kernel = head_dim == 128 ? paged_attention_kernel<SK, ASYM, 128> : paged_attention_kernel<SK, ASYM, 64>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows, (unsigned)q_heads), dim3(256), 0, s, pool, q, rows, (int)q_heads, table, (int)seqs,
                       max_pages, lens, starts, positions, scale * 1.4426950408889634f, out);
    return hipGetLastError();
  };
  switch (scale_kind) {
    case kScaleE5M2: return asym ? go.template operator()<kScaleE5M2, true>() : go.template operator()<kScaleE5M2, false>();
    case kScaleE4M3: return asym ? go.template operator()<kScaleE4M3, true>() : go.template operator()<kScaleE4M3, false>();
    default: return asym ? go.template operator()<kScaleE8M0Floor, true>() : go.template operator()<kScaleE8M0Floor, false>();
  }
}

}  // namespace amx
