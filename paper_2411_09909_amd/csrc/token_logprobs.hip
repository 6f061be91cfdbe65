// Log probabilities of given tokens, entropy and the likeliest alternatives out of logits (include/amxfp4_scoring.h), in one
// pass over them.
//
// With y the logit (or the capped one), a thread keeps of what it has read the maximum m and, against it,
//     S = sum e^(y - m)   and   T = sum e^(y - m) (y - m);
// two such triples join at M = max(m, m'):  S + S' with factors f = e^(m - M), and T as f (T + S (m - M)) + .... At the end
//     logprob = (y_t - m) - log S,   entropy = log S - T / S.
// (Differences first and log2 e after them: the largest logit's is exactly 0, whatever its size.)
//
// A capped logit is x (1 + u P(u)), u = (x / cap)^2, up to 0.6 of the cap, which is most segments; in the others each value takes what
// is its due. Logits of -inf, or so far below the largest that FP32 does not hold the difference, have a path of their own too: there the
// differences are kept from 0 times infinity.
//
// Alternatives. A row is read in segments (chunks of 16 bytes to a lane, side by side over the wave); each leaves its largest logit
// in LDS, each thread keeps its own. The top-th largest of a wave's 64 and of the segments' bound the result from below, so only
// segments that reach the bound are read again, from the cache, and the few elements at or above it are put in order by counting for
// each how many are better. Rows in which more than kList elements reach the bound (equal logits by the hundred) take them one after the other.
//
// Bound and measured: 4096 rows of 128000 float32 logits, 10 alternatives, 381 us = 5.5 TB/s (reads alone reach 6.2), 700 of 256000, capped, 139 us = 5.1 TB/s, where the
// vector unit is 67 % busy; one row of 128000 11.5 us, two launches of a chain each: read, bound, list, order. The first form took 391, 156 and 22 us: it ranked the
// threads' maxima through LDS, read every segment again, took one place in the list at a time and both functions of a cap for every logit.
#include "kernels.h"
#include "scoring.h"

namespace amx {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kSegment = 1024;  // elements, 16 to a lane
constexpr int kSegments = 512;  // of a part, at most
constexpr int kList = 512;      // candidates that are put in order at once
constexpr int kMostTop = 64;
constexpr int kMostParts = 64;
constexpr float kLn2 = 0.6931471805599453f;
// P: fitted here for the least absolute error of tanh z = z (1 + u P(u)) for |z| <= 0.6, 2.8e-8 (one term more than in scoring.h: logits are
// answers themselves)
constexpr float kWide = 0.6f, kP[4] = {-0.33332247f, 0.13308099f, -0.051994339f, 0.015319208f};

struct Sums {
  float m, s, t;
};

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return u2f((uint32_t)__builtin_amdgcn_mov_dpp((int)f2u(v), CTRL, 0xF, 0xF, true));
}
// over the wave, in all lanes: quads, rows of 16, and the swaps of 16 and 32 lanes
template <class Op>
__device__ __forceinline__ float wave_reduce(float v, Op op) {
  v = op(v, moved<0xB1>(v));
  v = op(v, moved<0x4E>(v));
  v = op(v, moved<0x124>(v));
  v = op(v, moved<0x128>(v));
  const auto a = __builtin_amdgcn_permlane16_swap(f2u(v), f2u(v), false, false);
  v = op(u2f(a[0]), u2f(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(f2u(v), f2u(v), false, false);
  return op(u2f(b[0]), u2f(b[1]));
}
__device__ __forceinline__ float wave_max(float v) { return wave_reduce(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_min(float v) { return wave_reduce(v, [](float a, float b) { return fminf(a, b); }); }
// (lanes add in orders of their own: the first one's sum, so that all go on with the same)
__device__ __forceinline__ float wave_sum(float v) {
  return u2f((uint32_t)__builtin_amdgcn_readfirstlane((int)f2u(wave_reduce(v, [](float a, float b) { return a + b; }))));
}

// sums against their own maximum, against the maximum `to`
__device__ __forceinline__ Sums shifted(Sums a, float to) {
  // (nothing in it: sums of 0, or NaN; far below: 0 times a number)
  const float d = a.m == -INFINITY ? 0.f : fmaxf(a.m - to, -1000.f), f = __builtin_amdgcn_exp2f(d * kLog2e);
  return {to, a.s * f, (a.t + a.s * d) * f};
}
__device__ __forceinline__ Sums wave_joined(Sums a) {
  const float m = wave_max(a.m);
  a = shifted(a, m);
  return {m, wave_sum(a.s), wave_sum(a.t)};
}

struct LogprobWork {
  const void* logits;
  const int32_t* targets;
  float *logprob, *entropy, *top_logprobs;
  int32_t* top_ids;
  int64_t ld;
  int vocab, top, parts, per_part;  // per_part: segments
  float in, cap, inverse, small;    // in as in Scores; the cap, its inverse, and how far the polynomial goes
  float4* sums;                     // workspace: (m, S, T) of each row and part
  uint2* tops;                      // workspace: (logit, id) [row][part][top], best first
};

__device__ __forceinline__ float capped_small(const LogprobWork& w, float x) {
  const float z = x * w.inverse, u = z * z;
  const float p = __builtin_fmaf(u, __builtin_fmaf(u, __builtin_fmaf(u, kP[3], kP[2]), kP[1]), kP[0]);
  return x * __builtin_fmaf(u, p, 1.0f);
}
// A logit, capped; -inf stays.
template <bool CAP>
__device__ __forceinline__ float value_of(const LogprobWork& w, float x) {
  if constexpr (!CAP) return x;
  return x == -INFINITY ? x : __builtin_fabsf(x) <= w.small ? capped_small(w, x) : capped(x, w.in, w.cap);
}

// A logit and its id as one number, larger for what is better (no NaN; zeros of both signs are equal).
__device__ __forceinline__ uint64_t key_of(float v, int id) {
  const uint32_t u = f2u(v + 0.f), up = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return (uint64_t)up << 32 | (uint32_t)~id;
}
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t up = (uint32_t)(key >> 32);
  return u2f(up ^ ((uint32_t)((int32_t)~up >> 31) | 0x80000000u));
}
__device__ __forceinline__ int id_of(uint64_t key) { return (int)~(uint32_t)key; }

struct Selection {
  uint64_t list[kList];
  uint64_t wave_best[kWaves];
  int count;
};

// The k best of the elements that each(f) hands to this thread as f(logit, id, there), k in all threads together, in order: emit(rank, logit,
// id). f comes for N elements at a time, `there` false for those that are none. No element below `bound` is among them. What is not there (of
// rows with NaN) comes out as id -1. l.count is 0. Where the bound is -inf and the list too short, it is made again of what is not ruled out and of
// those others that `early` says yes to, the lowest ids: no more of them can be wanted.
template <int N, class Each, class Emit>
__device__ __forceinline__ void select_best(Selection& l, int k, float bound, Each each, Emit emit) {
  const int t = threadIdx.x;
  each([&](const float (&v)[N], auto id, auto there, auto) {
    int mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) mine += v[i] >= bound && there(i) ? 1 : 0;
    if (mine == 0) return;
    int at = atomicAdd(&l.count, mine);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (v[i] >= bound && there(i)) {
        if (at < kList) l.list[at] = key_of(v[i], id(i));
        ++at;
      }
  });
  __syncthreads();
  int n = l.count;
  if (n > kList && bound == -INFINITY) {  // (uniform) parts of a row that are ruled out: 20 rows of 60000, half of them so, 42 us without, 16 with it
    __syncthreads();
    if (t == 0) l.count = 0;
    __syncthreads();
    each([&](const float (&v)[N], auto id, auto there, auto early) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (there(i) && (v[i] > -INFINITY || (v[i] == -INFINITY && early(i)))) {
          const int at = atomicAdd(&l.count, 1);
          if (at < kList) l.list[at] = key_of(v[i], id(i));
        }
    });
    __syncthreads();
    n = l.count;
  }
  if (n <= kList) {
    for (int c = t; c < n; c += kThreads) {
      const uint64_t key = l.list[c];
      int rank = 0;
#pragma unroll 8
      for (int o = 0; o < n; ++o) rank += l.list[o] > key ? 1 : 0;
      if (rank < k) emit(rank, logit_of(key), id_of(key));
    }
    for (int r = n + t; r < k; r += kThreads) emit(r, NAN, -1);
    return;
  }
  uint64_t last = ~uint64_t(0);
  for (int r = 0; r < k; ++r) {
    uint64_t best = 0;  // (less than any element's)
    each([&](const float (&v)[N], auto id, auto there, auto) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (v[i] >= bound && there(i)) {
          const uint64_t key = key_of(v[i], id(i));
          if (key < last && key > best) best = key;
        }
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t other = __shfl_xor(best, o, 64);
      best = other > best ? other : best;
    }
    __syncthreads();  // (the last round's have been read)
    if ((t & 63) == 0) l.wave_best[t >> 6] = best;
    __syncthreads();
#pragma unroll
    for (int o = 0; o < kWaves; ++o) best = l.wave_best[o] > best ? l.wave_best[o] : best;
    if (t == 0) emit(r, best ? logit_of(best) : NAN, best ? id_of(best) : -1);
    last = best;
  }
}

// the k-th largest of a wave's values (k <= 64; none is NaN): the least of those that fewer than k exceed
__device__ __forceinline__ float kth_of_wave(float mine, int k) {
  int above = 0;
#pragma unroll
  for (int o = 0; o < 64; ++o) above += u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(mine), o)) > mine ? 1 : 0;
  return wave_min(above < k ? mine : INFINITY);
}

// What is left to do for a row of which everything is known: one thread.
template <bool CAP>
__device__ __forceinline__ void finish(const LogprobWork& w, int64_t row, Sums all, float log_s, float target) {
  const bool nothing = all.m == -INFINITY && all.s == 0.f;
  if (w.targets) {
    const int at = w.targets[row];
    w.logprob[row] = at < 0 || at >= w.vocab ? 0.f : nothing ? -INFINITY : (value_of<CAP>(w, target) - all.m) - log_s;
  }
  if (w.entropy) w.entropy[row] = nothing ? 0.f : log_s - all.t / all.s;
}
template <bool CAP>
__device__ __forceinline__ float logprob_of(const LogprobWork& w, Sums all, float log_s, float x) {
  return all.m == -INFINITY && all.s == 0.f ? -INFINITY : (value_of<CAP>(w, x) - all.m) - log_s;
}

template <bool BF16, bool CAP, bool TOP>
__global__ __launch_bounds__(kThreads) void token_logprobs_kernel(LogprobWork w) {
  using Element = std::conditional_t<BF16, uint16_t, float>;
  constexpr int kE = 16 / (int)sizeof(Element), kN = kSegment / 64, kChunks = kN / kE;  // elements of a chunk of 16 bytes; of a lane; its chunks
  __shared__ Selection l;
  __shared__ Sums wave_sums[kWaves];
  __shared__ float segment_best[TOP ? kSegments : 1];
  __shared__ int chosen[TOP ? kSegments : 1], chosen_count;
  __shared__ float bounds[2][kWaves];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t row = blockIdx.x / (uint32_t)w.parts;
  const int part = (int)(blockIdx.x - (uint32_t)row * (uint32_t)w.parts);
  const Element* x = static_cast<const Element*>(w.logits) + row * w.ld;
  // elements that lie between the 16-byte boundary before the row and its first
  const int off = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(Element));
  const int s0 = part * w.per_part, s1 = min(s0 + w.per_part, (w.vocab + off + kSegment - 1) / kSegment);
  auto value = [&](Element e) { if constexpr (BF16) return u2f((uint32_t)e << 16); else return e; };
  float target = 0.f;  // (asked for now: it is here when it is wanted)
  if (t == 0 && w.parts == 1 && w.targets) {
    const int at = w.targets[row];
    if (at >= 0 && at < w.vocab) target = value(x[at]);
  }

  // a lane's elements of segment `s`: v[c kE + e] is element first + 64 kE c + e; outside the row -inf
  auto load = [&](int s, float (&v)[kN]) {
    const int first = s * kSegment - off + lane * kE;
    if (s * kSegment - off >= 0 && (s + 1) * kSegment - off <= w.vocab) {  // uniform
      u32x4 r[kChunks];
#pragma unroll
      for (int c = 0; c < kChunks; ++c) r[c] = *reinterpret_cast<const u32x4*>(x + first + c * 64 * kE);
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t word = r[c][i];
          if constexpr (BF16)
            v[c * kE + 2 * i] = u2f(word << 16), v[c * kE + 2 * i + 1] = u2f(word & 0xFFFF0000u);
          else
            v[c * kE + i] = u2f(word);
        }
    } else {  // chunks that lie within the row still come whole
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int i = first + c * 64 * kE;
        if (i >= 0 && i + kE <= w.vocab) {
          const u32x4 r = *reinterpret_cast<const u32x4*>(x + i);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t word = r[e];
            if constexpr (BF16)
              v[c * kE + 2 * e] = u2f(word << 16), v[c * kE + 2 * e + 1] = u2f(word & 0xFFFF0000u);
            else
              v[c * kE + e] = u2f(word);
          }
        } else {
#pragma unroll
          for (int e = 0; e < kE; ++e) {  // (all asked for before the first is looked at)
            const float at = value(x[min(max(i + e, 0), w.vocab - 1)]);
            v[c * kE + e] = i + e >= 0 && i + e < w.vocab ? at : -INFINITY;
          }
        }
      }
    }
  };

  // ---- the pass
  if (t == 0) l.count = 0, chosen_count = 0;
  Sums mine = {-INFINITY, 0.f, 0.f};
  float best = -INFINITY;  // of the thread, as logits
  float v[kN];
  for (int s = s0 + wave; s < s1; s += kWaves) {
    load(s, v);
    float most = v[0], edge = CAP ? __builtin_fabsf(v[0]) : v[0];  // edge: the largest size, or the smallest value
#pragma unroll
    for (int i = 1; i < kN; ++i) {
      most = fmaxf(most, v[i]);
      edge = CAP ? fmaxf(edge, __builtin_fabsf(v[i])) : fminf(edge, v[i]);
    }
    most = fmaxf(most, -INFINITY);  // (a NaN alone)
    if constexpr (TOP) {
      best = fmaxf(best, most);
      const float all = wave_max(most);
      if (lane == 0) segment_best[s - s0] = all;
    }
    const float m = fmaxf(mine.m, value_of<CAP>(w, most)), to = m == -INFINITY ? 0.f : m;
    mine = shifted(mine, to);
    mine.m = m;
    if (__builtin_amdgcn_ballot_w64(CAP ? edge > w.small : edge - to == -INFINITY) == 0) {  // uniform
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const float z = (CAP ? capped_small(w, v[i]) : v[i]) - to, e = __builtin_amdgcn_exp2f(z * kLog2e);
        mine.s += e, mine.t = __builtin_fmaf(e, z, mine.t);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const float z = value_of<CAP>(w, v[i]) - to, e = __builtin_amdgcn_exp2f(z * kLog2e);
        mine.s += e, mine.t = __builtin_fmaf(e, fmaxf(z, -1000.f), mine.t);  // (0 times -inf, which a difference of large ones may be too)
      }
    }
  }
  mine = wave_joined(mine);
  const float bound_here = TOP ? kth_of_wave(best, w.top) : 0.f;
  if (lane == 0) wave_sums[wave] = mine, bounds[0][wave] = bound_here;
  __syncthreads();
  const float m = fmaxf(fmaxf(wave_sums[0].m, wave_sums[1].m), fmaxf(wave_sums[2].m, wave_sums[3].m));
  Sums all = {m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const Sums a = shifted(wave_sums[i], m);
    all.s += a.s, all.t += a.t;
  }
  const float log_s = kLn2 * __builtin_amdgcn_logf(all.s);
  if (t == 0) {
    if (w.parts == 1)
      finish<CAP>(w, row, all, log_s, target);
    else
      w.sums[blockIdx.x] = make_float4(all.m, all.s, all.t, 0.f);
  }
  if constexpr (TOP) {
    const int segments = max(s1 - s0, 0), k = w.top;
    float bound = fmaxf(fmaxf(bounds[0][0], bounds[0][1]), fmaxf(bounds[0][2], bounds[0][3]));
    if (segments >= k) {  // (uniform) the k-th largest of the segments' as well
      float least = INFINITY;
      for (int s = t; s < segments; s += kThreads) {
        const float v = segment_best[s];
        int above = 0;
#pragma unroll 8
        for (int o = 0; o < segments; ++o) above += segment_best[o] > v ? 1 : 0;
        if (above < k) least = fminf(least, v);
      }
      least = wave_min(least);
      if (lane == 0) bounds[1][wave] = least;
      __syncthreads();
      bound = fmaxf(bound, fminf(fminf(bounds[1][0], bounds[1][1]), fminf(bounds[1][2], bounds[1][3])));
    }
    int count = 0;
    if (segments > kWaves) {  // (uniform)
      for (int s = t; s < segments; s += kThreads)
        if (segment_best[s] >= bound) chosen[atomicAdd(&chosen_count, 1)] = s;
      __syncthreads();
      count = chosen_count;
    }
    auto each = [&](auto f) {
      auto segment = [&](int s) {
        const int first = s * kSegment - off + lane * kE;
        auto id = [&](int i) { return first + i / kE * 64 * kE + i % kE; };
        // (fewer than k of a part's first 2 k ids are not ruled out where any that is may be wanted)
        f(v, id, [&](int i) { return id(i) >= 0 && id(i) < w.vocab; }, [&](int i) { return id(i) < max(s0 * kSegment - off, 0) + 2 * k; });
      };
      if (segments <= kWaves) {  // a wave has read one at most, and has it still
        if (wave < segments) segment(s0 + wave);
        return;
      }
      for (int c = wave; c < count; c += kWaves) {
        const int s = s0 + chosen[c];
        load(s, v);
        segment(s);
      }
    };
    auto emit = [&](int rank, float v, int id) {
      if (w.parts == 1)
        w.top_logprobs[row * k + rank] = logprob_of<CAP>(w, all, log_s, v), w.top_ids[row * k + rank] = id;
      else
        w.tops[(int64_t)blockIdx.x * k + rank] = make_uint2(f2u(v), (uint32_t)id);
    };
    select_best<kN>(l, k, bound, each, emit);
  }
}

// Adds up the parts of a row. (A part with fewer elements than `top` has ids of -1 at its end.)
template <bool BF16, bool CAP, bool TOP>
__global__ __launch_bounds__(kThreads) void token_logprobs_join_kernel(LogprobWork w) {
  __shared__ Selection l;
  const int t = threadIdx.x, lane = t & 63, k = w.top, parts = w.parts;
  const int64_t row = blockIdx.x;
  if (t == 0) l.count = 0;
  float target = 0.f;
  if (t == 0 && w.targets) {
    const int at = w.targets[row];
    if (at >= 0 && at < w.vocab) {
      if constexpr (BF16)
        target = u2f((uint32_t)static_cast<const uint16_t*>(w.logits)[row * w.ld + at] << 16);
      else
        target = static_cast<const float*>(w.logits)[row * w.ld + at];
    }
  }
  // every wave for itself
  Sums all = {-INFINITY, 0.f, 0.f};
  if (lane < parts) {
    const float4 v = w.sums[row * parts + lane];
    all = {v.x, v.y, v.z};
  }
  const uint2* tops = w.tops + row * parts * k;
  float bound = -INFINITY;
  if constexpr (TOP) {
    // A part's k-th bounds the result, and so does the k-th largest of the parts' first where there are so many (a NaN: none there)
    float head = -INFINITY, tail = -INFINITY;
    if (lane < parts) head = fmaxf(u2f(tops[lane * k].x), -INFINITY), tail = fmaxf(u2f(tops[lane * k + k - 1].x), -INFINITY);
    bound = wave_max(tail);
    if (parts >= k) bound = fmaxf(bound, kth_of_wave(head, k));
  }
  all = wave_joined(all);
  const float log_s = kLn2 * __builtin_amdgcn_logf(all.s);
  if (t == 0) finish<CAP>(w, row, all, log_s, target);
  if constexpr (TOP) {
    __syncthreads();
    auto each = [&](auto f) {
      for (int i = t; i < parts * k; i += kThreads) {
        const uint2 entry = tops[i];
        const float v[1] = {u2f(entry.x)};
        // (the first part, of more than k ids, names as many as can be wanted)
        f(v, [&](int) { return (int)entry.y; }, [&](int) { return (int)entry.y >= 0; }, [&](int) { return i < k; });
      }
    };
    auto emit = [&](int rank, float v, int id) {
      w.top_logprobs[row * k + rank] = logprob_of<CAP>(w, all, log_s, v), w.top_ids[row * k + rank] = id;
    };
    select_best<1>(l, k, bound, each, emit);
  }
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Parts that a row is read in, and segments of each: as many as give 1024 workgroups, and more for long rows, up to 3000 workgroups, as long as a part has
// 128 KB (so up to 1500 rows of 256 KB and more are read in two parts at least, from 1501 on whole); whatever the number of rows, as many as keep a part's
// segments within kSegments. us with up to 1024, 2048 and 4096 workgroups: 300 rows of 32000 BF16 logits 16.5, 21.5 and
// 19.1, 2000 of 128000 BF16 120, 132 and 146, 700 of 256000 float32 154, 140 and 135, 4000 of 32001 float32 108, 108 and 122.
int parts_of(int dtype, int64_t rows, int64_t vocab, int& per_part) {
  const int64_t segments = (vocab + 7 + kSegment - 1) / kSegment;  // (a row may begin up to 7 elements behind a boundary)
  const int64_t large = vocab * (dtype == 1 ? 2 : 4) >> 17, many = 3000 / rows;
  int64_t parts = (1024 + rows - 1) / rows;
  const int64_t more = many < large ? many : large;
  parts = parts > more ? parts : more;
  const int64_t most = (segments + kWaves - 1) / kWaves, least = (segments + kSegments - 1) / kSegments;
  parts = parts < most ? parts : most;
  parts = parts < kMostParts ? parts : kMostParts;
  parts = parts > least ? parts : least;
  per_part = (int)((segments + parts - 1) / parts);
  // (a segment to each wave, or as many: with one more the others wait, and up to one each they need not be read again. 96 rows of 50001 BF16
  // logits in parts of four 13.7 us, of five 15.3; 14.3 since ruled-out parts are listed once more)
  const int even = per_part / kWaves * kWaves;
  if (parts > 1 && even > 0 && per_part < 4 * kWaves && (segments + even - 1) / even <= kMostParts) per_part = even;
  return (int)((segments + per_part - 1) / per_part);
}

constexpr int64_t kMostVocab = int64_t(1) << 24, kMostRows = int64_t(1) << 23;
static_assert(kMostVocab / kSegment / kSegments < kMostParts, "a part's segments fit");

bool bad_shape(int32_t dtype, int64_t rows, int64_t vocab, int64_t top) {
  return (dtype != 0 && dtype != 1) || rows <= 0 || rows > kMostRows || vocab <= 0 || vocab > kMostVocab || top < 0 || top > kMostTop || top > vocab;
}

size_t sums_bytes(int64_t rows, int parts) { return ((size_t)rows * parts * sizeof(float4) + 255) & ~(size_t)255; }

}  // namespace
}  // namespace amx

using namespace amx;

extern "C" {

size_t amxfp4_token_logprobs_workspace_bytes(int32_t dtype, int64_t rows, int64_t vocab, int64_t top) {
  if (bad_shape(dtype, rows, vocab, top)) return 0;
  int per_part;
  const int parts = parts_of(dtype, rows, vocab, per_part);
  return parts == 1 ? 0 : sums_bytes(rows, parts) + (size_t)rows * parts * top * sizeof(uint2);
}

int amxfp4_token_logprobs(const void* logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t ld, const int32_t* targets, float cap,
                          int64_t top, float* logprob, float* entropy, float* top_logprobs, int32_t* top_ids, void* workspace,
                          size_t workspace_bytes, void* stream) {
  if (!logits) return report_error(AMX_ERR_INVALID_ARG, "token_logprobs: logits is NULL");
  if (bad_shape(dtype, rows, vocab, top))
    return report_error(AMX_ERR_INVALID_ARG, "token_logprobs: dtype 0 or 1, 1 to 2^23 rows and 2^24 columns, top 0 to 64 and at most vocab");
  if (ld < vocab || ld > (int64_t(1) << 31) || rows > (int64_t(1) << 40) / ld)
    return report_error(AMX_ERR_INVALID_ARG, "token_logprobs: ld at least vocab, at most 2^31, rows * ld at most 2^40");
  if (!(targets == nullptr) != !(logprob == nullptr))
    return report_error(AMX_ERR_INVALID_ARG, "token_logprobs: targets and logprob go together");
  if ((top > 0) != (top_logprobs != nullptr) || (top > 0) != (top_ids != nullptr))
    return report_error(AMX_ERR_INVALID_ARG, "token_logprobs: top_logprobs and top_ids are wanted exactly when top is positive");
  if (!targets && !entropy && !top) return report_error(AMX_ERR_INVALID_ARG, "token_logprobs: nothing is asked for");
  if (!(cap == 0.f || (cap >= 0x1p-20f && cap <= 0x1p20f)))
    return report_error(AMX_ERR_INVALID_ARG, "token_logprobs: cap must be 0 or 2^-20 to 2^20");
  if (!aligned(logits, dtype == 1 ? 2 : 4) || !aligned(targets, 4) || !aligned(logprob, 4) || !aligned(entropy, 4) ||
      !aligned(top_logprobs, 4) || !aligned(top_ids, 4))
    return report_error(AMX_ERR_INVALID_ARG, "token_logprobs: pointers must be aligned to their elements");
  LogprobWork w = {logits, targets, logprob, entropy, top_logprobs, top_ids, ld, (int)vocab, (int)top, 0, 0, 0.f, 0.f, 0.f, 0.f, nullptr, nullptr};
  w.parts = parts_of(dtype, rows, vocab, w.per_part);
  if (cap > 0.f) w.in = 2 * kLog2e / cap, w.cap = cap, w.inverse = 1.0f / cap, w.small = kWide * cap;
  if (w.parts > 1) {
    if (!workspace || workspace_bytes < amxfp4_token_logprobs_workspace_bytes(dtype, rows, vocab, top) || !aligned(workspace, 256))
      return report_error(AMX_ERR_WORKSPACE, "token_logprobs: workspace missing, too small or not 256-byte aligned");
    w.sums = static_cast<float4*>(workspace);
    w.tops = reinterpret_cast<uint2*>(static_cast<uint8_t*>(workspace) + sums_bytes(rows, w.parts));
  }
  auto go = [&]<bool BF16, bool CAP, bool TOP>() {
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipLaunchKernelGGL((token_logprobs_kernel<BF16, CAP, TOP>), dim3((unsigned)(rows * w.parts)), dim3(kThreads), 0, s, w);
    if (w.parts > 1) hipLaunchKernelGGL((token_logprobs_join_kernel<BF16, CAP, TOP>), dim3((unsigned)rows), dim3(kThreads), 0, s, w);
  };
  auto with_type = [&]<bool BF16>() {
    if (cap > 0.f)
      top ? go.template operator()<BF16, true, true>() : go.template operator()<BF16, true, false>();
    else
      top ? go.template operator()<BF16, false, true>() : go.template operator()<BF16, false, false>();
  };
  dtype == 1 ? with_type.template operator()<true>() : with_type.template operator()<false>();
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AMX_OK : report_hip_error(e, "token_logprobs launch");
}

}  // extern "C"
