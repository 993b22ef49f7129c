// A token and its confidence from a row of logits and one uniform number (reflex_sample_tokens).
//
// Weights and their sums are fp64 where a draw or a filter compares them: with u given, the
// token is a matter of which side of a border u lies on, and sums in fp32 (relative error 1e-7
// times some) would take another token in one row of a hundred where 1e5 tokens share the mass.
// w = 2^((l - max) log2(e) / temperature) by a table of 64 powers and a cubic (relative error
// 4e-11, some 15 vector instructions); the confidence's denominator sums fp32 powers.
//
// Launches:
//  1. The logits are read once from HBM, a wave a part of a row (rows are cut so that few rows fill the
//     GPU too): each part's maximum with its first index, its sum of weights and its sum for the
//     confidence.  Every lane sums relative to a logit of its own, which it moves when one lies 2^24
//     above it.  Groups of eight lanes leave their maxima, from which a bound for top-k follows.
//  2. With filters: each part's elements above a bound that no kept logit lies below are listed, in
//     index order, if they are few enough, as they mostly are.
//  3. A wave a row.  Without filters it finds the part that u falls into and scans that one.  With
//     filters it holds the list in registers, finds the last kept logit of top-k and of top-p bit by
//     bit of the 32-bit order keys (counts by ballots, weights in fixed point), and draws.
//  4. With filters: a workgroup of 16 waves for each row whose list did not fit (flat rows, mostly of
//     top-p).  For top-p alone the numbers and mean logits of 2048 linear bins say nearly where the
//     border lies; one more pass sums the weights above that place and lists the bins around it, where the
//     border is then sought.  Otherwise, or where that fails, the last kept logit is found by counts
//     or weights in the bins, first linear ones between the bound and the maximum, then over the order
//     keys of one bin, in passes over the row (in the memory-side cache by then) until what is left
//     fits a list in LDS.  (Fixed-point weights: the sums do not depend on the order of the atomics.)  The
//     draw goes over the row's sixteenths and a scan of one.
// Everything is inlined and in registers: no stack.  (Keep it so, ScratchSize 0 in the build's resource report: a
// form that used one gave a wrong token and a GPU fault whose cause was never shown.)
//
// Measured, us (bf16 logits, temperature 1): 1024 rows of 100003 without filters 95 (launch 1: 86, bound by its
// 29 vector instructions an element, where reading the logits takes 34; 114 at another temperature, whose
// confidences want sums of their own; greedy 47), top-k 50 166, min-p 0.02 202, top-p 0.9 394 (launch 4:
// 262 for the flat rows, 75 a row, bound by 50 vector instructions an element on the row's own CU); 32 rows of
// 131072 16, 28, 65 and 106, with all filters (temperature 0.7, top-k 50, top-p 0.9, min-p 0.02) 34, of which launch 3
// takes 17: one wave's chain of loads and the bit by bit search for two borders; one row of 32000 10, two launches.
#include <algorithm>
#include <cmath>
#include <limits>
#include <type_traits>

#include "fp8.h"

namespace rfx {
namespace {

constexpr int SS_THREADS = 256, SS_WAVES = SS_THREADS / kWave;      // launches 1 to 3
constexpr int SP_THREADS = 1024, SP_WAVES = SP_THREADS / kWave;     // launch 4
constexpr int SP_PARTS = 256;                                       // most parts of a row
constexpr int SP_BIN_BITS = 11, SP_BINS = 1 << SP_BIN_BITS;
constexpr int SP_LANE = 4, SP_SEG = SP_LANE * kWave;      // list entries of a lane and of a wave
constexpr int SL_LANE = 16, SL_MOST = SL_LANE * kWave;    // a row's list: entries of a lane, of all
constexpr int SL_LIST = 4 * SL_MOST;                      // the parts' shares of it are larger
constexpr int SP_AROUND = 4;                              // bins listed on either side of a border's likely one
constexpr int SP_ROWS = 1 << 16;                          // rows of a launch
constexpr int SP_SCAN = 8;                                // consecutive elements of a thread in a scan
static_assert(SP_BINS == 2 * SP_THREADS && SP_PARTS <= SP_THREADS, "two bins a thread");
constexpr double SP_LOG2E = 1.4426950408889634074;
constexpr float SP_NONE = -__builtin_huge_valf(), SP_LOWEST = -3.402823466e38f;
// What stands in for a logit without weight where weights are summed.  Less any logit and times the least scale
// (4.2e-39, the highest temperature's) it is below -4000, and finite times the largest (1e45).
constexpr double SP_WEIGHTLESS = -1e42;

#define SP_INLINE __attribute__((always_inline))

// What the first launch leaves of a part: sums relative to `top`.
struct Part {
  double sum, flat;
  float top;           // the maximum
  int first;           // its first index
  float group[8];      // maxima of the groups of eight lanes
};

// An element that the second launch lists.
struct Listed {
  uint32_t key;
  int index;
};

struct SampleArgs {
  const int32_t *rows, *n_rows;      // rows: from row0 on
  int M, V, T, parts, row0;          // M: rows of this launch; row0: the rows before them
  const float* u;
  double scale;          // log2(e) / temperature; 0: temperature 0
  double floor2;         // log2(min_p), -inf for none
  int top_k;             // 1 .. V
  double top_p;
  int32_t* tokens;
  float* conf;
  Part* part;            // [M, parts]
  float* pair;           // [M, parts, 32]: maxima of the pairs of lanes
  int32_t* listed;       // [M, parts]: the parts' numbers of listed elements, -1 for too many
  Listed* list;          // [M, SP_LIST]: parts' shares one after the other
};

// Rows of this launch that are in use, and row j's position.
RFX_DEVICE int rows_used(const SampleArgs& a) {
  return a.n_rows == nullptr ? a.M : min(max(a.n_rows[0], 0) - a.row0, a.M);
}
RFX_DEVICE int position_of(const SampleArgs& a, int j) { return a.rows == nullptr ? a.row0 + j : a.rows[j]; }

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
constexpr double kMagic = 0x1.8p46;      // its last place is 1 / 64

// a b + c as one instruction with a destination of its own.  (The compiler prefers the form that adds
// into its destination, and copies the polynomial's constants there for every use.)
RFX_DEVICE double fma64(double a, double b, double c) {
#ifdef __HIP_DEVICE_COMPILE__
  double d;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
#else
  return fma(a, b, c);
#endif
}

// Entry j of the table: 2^(j / 64), its high word less j << 14, so that n << 14 added to it multiplies
// by 2^((n - j) / 64) for n % 64 = j.
RFX_DEVICE double pow2_entry(int j) {
  return __longlong_as_double(__double_as_longlong(exp2(j / 64.0)) - (static_cast<long long>(j) << 46));
}

// 2^x as a product p t, given y = x + kMagic (rounded) and r = x - (y - kMagic), |r| <= 1 / 128.
RFX_DEVICE void pow2_parts(double y, double r, const double* table, double& p, double& t) {
  const uint32_t n = static_cast<uint32_t>(__double_as_longlong(y));      // 64 x, rounded
  p = fma64(r, fma64(r, fma64(r, 0.05550410866482158, 0.24022650695910071), 0.69314718055994531), 1.0);
  u32x2_t e = __builtin_bit_cast(
      u32x2_t, *reinterpret_cast<const double*>(reinterpret_cast<const char*>(table) + ((n << 3) & 0x1f8u)));
  e[1] += n << 14;
  t = __builtin_bit_cast(double, e);
}
RFX_DEVICE double pow2_of(double y, double r, const double* table) {
  double p, t;
  pow2_parts(y, r, table, p, t);
  return p * t;
}

// 2^x for x <= 1000, zero below 2^-1020.
RFX_DEVICE double pow2_or_0(double x, const double* table) {
  const double y = x + kMagic;
  return x >= -1020.0 ? pow2_of(y, x - (y - kMagic), table) : 0.0;
}

// Of one number a wave in LDS: the sum of those of the waves before wave w, and of all (for every lane).
template <class T>
RFX_DEVICE T waves_before(const T* of_wave, int w, T& all) {
  const int lane = threadIdx.x & 63;
  const T mine = lane < SP_WAVES ? of_wave[lane] : T(0);
  all = wave_sum64(mine);
  return wave_sum64(lane < w ? mine : T(0));
}
RFX_DEVICE int waves_before(const int* of_wave, int w, int& all) {
  const int lane = threadIdx.x & 63;
  const int mine = lane < SP_WAVES ? of_wave[lane] : 0;
  all = wave_sum_i32(mine);
  return wave_sum_i32(lane < w ? mine : 0);
}

// A row of logits in parts of whole 16-byte vectors; the elements before the first 16-byte boundary
// belong to the first part, those behind the last vector to the last.
template <class E>
struct Row {
  static constexpr int VEC = 16 / sizeof(E);
  typedef float Values __attribute__((ext_vector_type(VEC)));
  const E* p;
  int V, head, vecs, parts, per;

  RFX_DEVICE Row(const E* p_, int V_, int parts_) : p(p_), V(V_), parts(parts_) {
    head = min(V, static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(E)));
    vecs = (V - head) / VEC;
    per = (vecs + parts - 1) / parts;
  }
  // First index of a part (parts: V).
  RFX_DEVICE int begin(int part) const { return part == 0 ? 0 : (part >= parts ? V : head + min(part * per, vecs) * VEC); }
  RFX_DEVICE float at(int i) const {
    if constexpr (sizeof(E) == 2)
      return bf16_to_f32(p[i]);
    else
      return p[i];
  }
  // A wave's walk over a part, in index order, all 64 lanes in every call: f(values, n, index of the
  // first, whole), n = VEC, or fewer (0 or 1 too) where `whole` is false_type.  WHOLE: whole waves of
  // vectors get a call site of their own.
  template <bool WHOLE, class F>
  RFX_DEVICE void each(int part, F&& f) const {
    const int lane = threadIdx.x & 63;
    const uint4* const vec = reinterpret_cast<const uint4*>(p + head);
    const int begin = min(part * per, vecs), end = min(begin + per, vecs);
    auto load = [&](int at) SP_INLINE { return at < end ? vec[at] : make_uint4(0, 0, 0, 0); };
    auto unpack = [](const uint4& q) SP_INLINE {
      const uint32_t b[4] = {q.x, q.y, q.z, q.w};
      Values v;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(E) == 2) {
          v[2 * j] = __uint_as_float(b[j] << 16);
          v[2 * j + 1] = __uint_as_float(b[j] & 0xffff0000u);
        } else {
          v[j] = __uint_as_float(b[j]);
        }
      }
      return v;
    };
    int i = begin + lane;
    uint4 q0 = load(i);      // three vectors ahead
    uint4 q1 = load(i + kWave);
    uint4 q2 = load(i + 2 * kWave);
    uint4 q3 = load(i + 3 * kWave);
    auto next = [&]() SP_INLINE {
      q0 = q1;
      q1 = q2;
      q2 = q3;
      q3 = load(i + 4 * kWave);
      i += kWave;
    };
    auto aside = [&](int first, int stop, int& n) SP_INLINE {      // an element a lane
      Values v;
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[j] = SP_NONE;
      n = first < stop ? 1 : 0;
      if (n) v[0] = at(first);
      return v;
    };
    const int steps = (end - begin + kWave - 1) / kWave;
    for (int st = part == 0 ? -1 : 0; st < steps + (part == parts - 1 ? 1 : 0); ++st) {
      if (WHOLE) {
        auto whole = [&](uint4& q) SP_INLINE {      // (the four loads take turns: no copies between them)
          const Values v = unpack(q);
          q = load(i + 4 * kWave);
          f(v, VEC, head + i * VEC, std::true_type{});
          i += kWave;
        };
        for (; st >= 0 && begin + (st + 4) * kWave <= end; st += 4) {
          whole(q0);
          whole(q1);
          whole(q2);
          whole(q3);
        }
        if (st >= steps + (part == parts - 1 ? 1 : 0)) break;
      }
      Values v;
      int n, first;
      if (st < 0) {
        first = lane;
        v = aside(first, head, n);
      } else if (st == steps) {
        first = head + vecs * VEC + lane;
        v = aside(first, V, n);
      } else {
        first = head + i * VEC;
        n = i < end ? VEC : 0;
        v = unpack(q0);
        next();
      }
      f(v, n, first, std::false_type{});
    }
  }
};

// FLAT: the confidence's sum is another one than the weights'.  PAIRS: top-k, whose bound may want the pairs' maxima.
template <class E, bool DRAWS, bool FLAT, bool PAIRS>
__global__ __launch_bounds__(SS_THREADS) void sample_sums_kernel(const E* __restrict__ logits, SampleArgs a) {
  constexpr int VEC = Row<E>::VEC;
  using Values = typename Row<E>::Values;
  __shared__ double table[64];
  const int tid = threadIdx.x, lane = tid & 63;
  if (DRAWS && tid < 64) table[tid] = pow2_entry(tid);
  __syncthreads();
  const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * SS_WAVES + (tid >> 6));
  const int j = item / a.parts, part = item - j * a.parts;
  if (j >= rows_used(a)) return;
  const Row<E> row(logits + static_cast<size_t>(j) * a.V, a.V, a.parts);
  const double scale = a.scale, step = fmax(scale, SP_LOG2E);
  float best = SP_NONE, ref = SP_LOWEST;
  int at = 0x7fffffff;
  double sum = 0.0, flat = 0.0;
  row.template each<true>(part, [&](Values v, int n, int i, auto whole) SP_INLINE {
    constexpr bool WHOLE = decltype(whole)::value;
    // (fmaxf passes NaN by)
    float m = fmaxf(v[0], SP_NONE);
#pragma unroll
    for (int k = 1; k < VEC; ++k) m = fmaxf(m, v[k]);
    if ((WHOLE || n > 0) && (m > best || at == 0x7fffffff)) {
      best = m;
      at = i;
#pragma unroll
      for (int k = VEC - 1; k >= 0; --k)
        if (v[k] == m) at = i + k;
      const double up = static_cast<double>(m) - static_cast<double>(ref);
      if (up * step > 24.0 && m < -SP_NONE) {      // move the reference here
        if (DRAWS) sum *= pow2_or_0(-up * scale, table);
        if (FLAT) flat *= exp2(-up * SP_LOG2E);
        ref = m;
      }
    }
    float z = 0.0f;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      if (DRAWS) {
        // (NaN and -inf: far below every number that they may be relative to, at the highest temperature too)
        const double d = fmax(static_cast<double>(v[k]), SP_WEIGHTLESS) - static_cast<double>(ref);
        const double y = fmax(fma(d, scale, kMagic), kMagic - 1020.0);      // (below 2^-1020: next to nothing)
        double p, t;
        pow2_parts(y, fma(d, scale, kMagic - y), table, p, t);
        if (WHOLE)
          sum = fma(p, t, sum);
        else
          sum += k < n ? p * t : 0.0;
      }
      if (FLAT) {
        const float w = __builtin_amdgcn_exp2f((v[k] - ref) * static_cast<float>(SP_LOG2E));
        z += WHOLE || k < n ? w : 0.0f;
      }
    }
    if (FLAT && z != z) {      // NaN among them, as -inf (told by the sum: no instruction an element)
      z = 0.0f;
#pragma unroll
      for (int k = 0; k < VEC; ++k)
        z += (WHOLE || k < n) && v[k] == v[k] ? __builtin_amdgcn_exp2f((v[k] - ref) * static_cast<float>(SP_LOG2E)) : 0.0f;
    }
    if (FLAT) flat += static_cast<double>(z);
  });
  const uint64_t key =
      wave_max_u64((static_cast<uint64_t>(f32_order_key(best)) << 32) | (0x7fffffffu - static_cast<uint32_t>(at)));
  const float top = f32_from_order_key(static_cast<uint32_t>(key >> 32));
  const double down = fmin(static_cast<double>(ref) - static_cast<double>(top), 0.0);      // (top -inf: +inf)
  if (DRAWS) sum = wave_sum64(sum * pow2_or_0(down * scale, table));
  if (FLAT) flat = wave_sum64(flat * exp2(down * SP_LOG2E));
  if (top == SP_NONE) sum = flat = 0.0;
  Part* const out = a.part + item;
  if (lane == 0) {
    out->sum = sum;
    out->flat = flat;
    out->top = top;
    out->first = static_cast<int>(0x7fffffffu - static_cast<uint32_t>(key));
  }
  // maxima of the pairs and of the groups of eight lanes (no elements: -inf)
  uint32_t group = f32_order_key(best);
  group = max(group, dpp_u32<kDppXor1>(group));
  if (PAIRS && lane % 2 == 0) a.pair[static_cast<size_t>(item) * (kWave / 2) + lane / 2] = f32_from_order_key(group);
  group = max(group, dpp_u32<kDppXor2>(group));
  group = max(group, dpp_u32<kDppHalfMirror>(group));
  if (lane % 8 == 0) out->group[lane / 8] = f32_from_order_key(group);
}

// The bound of a row's filters, by one wave: no kept logit lies below it.
//  - Top-k: as many groups of lanes as have elements have a maximum each; top_k of them are at least
//    the bound (its key's low 16 bits zero), so top_k elements are.  Of G groups of random elements some
//    G ln(G / (G - top_k)) elements lie above; pairs serve where the groups of eight lanes are too few.
//  - Top-p: the tokens of less than the share (1 - top_p) / V together weigh less than what may be left
//    out.
//  - Min-p itself; not where top-p needs the weight of what top-k leaves, min-p's part among it.
// In fp32, with a margin.  m: the row's maximum, total: its sum of weights.
RFX_DEVICE float filter_bound(const SampleArgs& a, const Part* part, double m, double total) {
  const int lane = threadIdx.x & 63, groups = 8 * a.parts;
  const float top = static_cast<float>(m);
  const bool by_count = a.top_k < a.V, by_mass = a.top_p < 1.0;
  float cut = SP_LOWEST;
  if (by_count && 2 * a.top_k <= a.parts) {      // (enough parts: their maxima do)
    uint32_t bound = 0;
    uint32_t key[SP_PARTS / kWave];
#pragma unroll
    for (int q = 0; q < SP_PARTS / kWave; ++q) {
      const int p = q * kWave + lane;
      key[q] = p < a.parts ? f32_order_key(part[p].top) : 0u;
    }
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t t = bound | (1u << bit);
      int n = 0;
#pragma unroll
      for (int q = 0; q < SP_PARTS / kWave; ++q) n += __popcll(__ballot(key[q] >= t));
      if (n >= a.top_k) bound = t;
    }
    if (bound > f32_order_key(SP_LOWEST)) cut = f32_from_order_key(bound);
  } else if (by_count) {
    // the top_k-th of n entries, if they are enough
    auto bound_of = [&](int n_entries, auto&& entry) SP_INLINE {
      if (a.top_k > n_entries) return;
      uint32_t bound = 0;
      uint32_t key[8 * SP_PARTS / kWave];
#pragma unroll
      for (int q = 0; q < 8 * SP_PARTS / kWave; ++q) {
        const int g = q * kWave + lane;
        key[q] = g < n_entries ? f32_order_key(entry(g)) : 0u;
      }
      for (int bit = 31; bit >= 16; --bit) {
        const uint32_t t = bound | (1u << bit);
        int n = 0;
#pragma unroll
        for (int q = 0; q < 8 * SP_PARTS / kWave; ++q)
          if (q * kWave < n_entries) n += __popcll(__ballot(key[q] >= t));
        if (n >= a.top_k) bound = t;
      }
      if (bound > f32_order_key(SP_LOWEST)) cut = f32_from_order_key(bound);
    };
    if (8 * a.top_k <= 7 * groups || a.parts > SP_PARTS / 4) {
      bound_of(groups, [&](int g) SP_INLINE { return part[g / 8].group[g % 8]; });
    } else {
      const float* const pair = a.pair + (part - a.part) * (kWave / 2);
      bound_of(kWave / 2 * a.parts, [&](int g) SP_INLINE { return pair[g]; });
    }
  } else if (!by_count && by_mass) {
    cut = static_cast<float>(m + (log2((1.0 - a.top_p) * total / a.V) - 0.001) / a.scale);
  }
  if (a.floor2 > -1.0e300 && !(by_count && by_mass)) cut = fmaxf(cut, static_cast<float>(m + (a.floor2 - 0.001) / a.scale));
  return fminf(fmaxf(cut - 1e-6f * fmaxf(fabsf(cut), fabsf(top)), SP_LOWEST), top);
}

// Weights in fixed point: times the power of two that brings the sum of all between 2^50 and 2^51, and
// rounded.  (A power of two: equal logits at the maximum have weight 1 and borders that are exact.)
RFX_DEVICE double fixed_scale(double total) {
  return __longlong_as_double((2096ll - (__double_as_longlong(total) >> 52)) << 52);
}
RFX_DEVICE uint64_t fixed_point(double w, double scale) {
  return static_cast<uint64_t>(__double_as_longlong(fma(w, scale, 0x1p52))) - 0x4330000000000000ull;
}

// A row's maximum and sum of weights from its parts, by one wave.
RFX_DEVICE void row_sums(const SampleArgs& a, const Part* part, const double* table, float& top, double& total) {
  const int lane = threadIdx.x & 63;
  float best = SP_NONE;
  for (int p = lane; p < a.parts; p += kWave) best = fmaxf(best, part[p].top);
  top = f32_from_order_key(wave_max_u32(f32_order_key(best)));
  total = 0.0;
  for (int p = lane; p < a.parts; p += kWave)
    total += part[p].sum * pow2_or_0((static_cast<double>(part[p].top) - static_cast<double>(top)) * a.scale, table);
  total = wave_sum64(total);
}

template <class E>
__global__ __launch_bounds__(SS_THREADS) void sample_list_kernel(const E* __restrict__ logits, SampleArgs a) {
  constexpr int VEC = Row<E>::VEC;
  using Values = typename Row<E>::Values;
  __shared__ double table[64];
  __shared__ float s_cut;
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid < 64) table[tid] = pow2_entry(tid);
  __syncthreads();
  const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * SS_WAVES + (tid >> 6));
  const int j = item / a.parts, p = item - j * a.parts;      // (one row a workgroup: parts % SS_WAVES = 0)
  if (j >= rows_used(a)) return;
  const Part* const part = a.part + static_cast<size_t>(j) * a.parts;
  if (tid < kWave) {
    float top;
    double total;
    row_sums(a, part, table, top, total);
    const float cut = top > SP_NONE && top < -SP_NONE ? filter_bound(a, part, top, total) : -SP_NONE;
    if (lane == 0) s_cut = cut;
  }
  __syncthreads();
  const float cut = s_cut;      // (+inf: a row without weight, or with +inf: no list)
  const int room = SL_LIST / a.parts;
  int n_list = 0;      // (uniform in the wave)
  if (cut < -SP_NONE) {
    Listed* const list = a.list + static_cast<size_t>(j) * SL_LIST + static_cast<size_t>(p) * room;
    const Row<E> row(logits + static_cast<size_t>(j) * a.V, a.V, a.parts);
    row.template each<false>(p, [&](Values v, int n, int i, auto) SP_INLINE {
      uint32_t on = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e) on |= e < n && v[e] >= cut ? 1u << e : 0u;
      if (__ballot(on != 0) == 0 || n_list > room) return;
      const int count = __popc(on), incl = wave_inclusive_scan_i32(count, lane);
      int to = n_list + incl - count;
      n_list += __builtin_amdgcn_readlane(incl, 63);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if ((on >> e) & 1u) {
          if (to < room) list[to] = Listed{f32_order_key(v[e]), i + e};
          ++to;
        }
      }
    });
  }
  if (lane == 0) a.listed[static_cast<size_t>(j) * a.parts + p] = n_list > room ? -1 : n_list;
}

// A row's parts, lane l with parts l, l + 64, .. (none: nothing of them), loaded together: a row's launch is a
// chain of loads from other launches' results, 1 us each.
constexpr int SP_PARTS_LANE = (SP_PARTS + kWave - 1) / kWave;
struct RowParts {
  double sum[SP_PARTS_LANE], flat[SP_PARTS_LANE];
  float top[SP_PARTS_LANE];
  int first[SP_PARTS_LANE];
};
RFX_DEVICE RowParts load_parts(const SampleArgs& a, const Part* part) {
  RowParts r;
#pragma unroll
  for (int q = 0; q < SP_PARTS_LANE; ++q) {
    const int p = kWave * q + static_cast<int>(threadIdx.x & 63);
    r.sum[q] = r.flat[q] = 0.0;
    r.top[q] = SP_NONE;
    r.first[q] = 0x7fffffff;
    if (p < a.parts) {
      r.sum[q] = part[p].sum;
      r.flat[q] = part[p].flat;
      r.top[q] = part[p].top;
      r.first[q] = part[p].first;
    }
  }
  return r;
}

// A row's sums from its parts', by one wave; first: the maximum's first index.
RFX_DEVICE void row_flat(const SampleArgs& a, const RowParts& part, const double* table, float& top, int& first,
                         double& total, double& flat) {
  uint64_t most = 0;
#pragma unroll
  for (int q = 0; q < SP_PARTS_LANE; ++q)
    if (kWave * q < a.parts)
      most = max(most, (static_cast<uint64_t>(f32_order_key(part.top[q])) << 32) |
                           (0x7fffffffu - static_cast<uint32_t>(part.first[q])));
  most = wave_max_u64(most);
  top = f32_from_order_key(static_cast<uint32_t>(most >> 32));
  first = static_cast<int>(0x7fffffffu - static_cast<uint32_t>(most));
  total = flat = 0.0;
#pragma unroll
  for (int q = 0; q < SP_PARTS_LANE; ++q) {
    if (kWave * q < a.parts) {
      const double down = static_cast<double>(part.top[q]) - static_cast<double>(top);
      total += part.sum[q] * pow2_or_0(down * a.scale, table);
      flat += part.flat[q] * pow2_or_0(down * SP_LOG2E, table);
    }
  }
  total = wave_sum64(total);
  flat = a.scale == SP_LOG2E ? total : wave_sum64(flat);
}

// Of the lanes' weights in lane order, the lane that `target` falls into, and what is left of it there;
// else (the order of the additions) the last lane with weight, +inf; -1: none has weight.
RFX_DEVICE int pick_lane(double w, double target, double before, double& rest, bool& hit) {
  const double incl = wave_inclusive_scan64(w);
  const uint64_t hits = __ballot(w > 0.0 && before + incl > target), any = __ballot(w > 0.0);
  hit = hits != 0;
  rest = hit ? target - (before + incl - w) : __builtin_huge_val();
  return hit ? __builtin_ctzll(hits) : (any != 0 ? 63 - __builtin_clzll(any) : -1);
}

template <class E, bool FILTERS>
__global__ __launch_bounds__(SS_THREADS) void sample_row_kernel(const E* __restrict__ logits, SampleArgs a) {
  __shared__ double table[64];
  __shared__ int s_at[SS_WAVES][SP_PARTS + 1];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = __builtin_amdgcn_readfirstlane(blockIdx.x * SS_WAVES + wv), V = a.V, parts = a.parts;
  // (loads of a row of the workspace, ahead of what decides whether there is such a row)
  const size_t row_of = static_cast<size_t>(min(j, a.M - 1)) * parts;
  const Part* const part = a.part + row_of;
  const RowParts of_row = load_parts(a, part);
  int listed[SP_PARTS_LANE];
#pragma unroll
  for (int q = 0; q < SP_PARTS_LANE; ++q)
    listed[q] = FILTERS && kWave * q + lane < parts ? a.listed[row_of + kWave * q + lane] : 0;
  if (tid < 64) table[tid] = pow2_entry(tid);
  __syncthreads();
  if (j >= rows_used(a)) return;
  const int pos = position_of(a, j);
  if (pos < 0 || pos >= a.T) return;
  const Row<E> row(logits + static_cast<size_t>(j) * V, V, parts);
  float top;
  int token;
  double total, flat;
  row_flat(a, of_row, table, top, token, total, flat);
  float u = a.u[pos];
  u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
  const double m = top, scale = a.scale;
  auto weight = [&](uint32_t k) SP_INLINE {
    return pow2_or_0((static_cast<double>(f32_from_order_key(k)) - m) * scale, table);
  };
  if (top == SP_NONE) {            // nothing has weight
    token = -1;
    flat = 1.0;
  } else if (top == -SP_NONE) {    // the +inf ones have the same weight each, the others none
    int n = 0;
    for (int i = lane; i < V; i += kWave) n += row.at(i) == top ? 1 : 0;
    n = wave_sum_i32(n);
    flat = n;
    if (scale > 0.0) {
      if (a.top_k < n) n = a.top_k;
      if (a.top_p < 1.0) n = max(1, static_cast<int>(ceil(a.top_p * n)));
      int want = min(static_cast<int>(u * static_cast<double>(n)), n - 1);      // the want-th of them
      for (int i0 = 0; i0 < V; i0 += kWave) {
        uint64_t on = __ballot(i0 + lane < V && row.at(min(i0 + lane, V - 1)) == top);
        const int here = __popcll(on);
        if (want < here) {
          for (; want > 0; --want) on &= on - 1;
          token = i0 + __builtin_ctzll(on);
          break;
        }
        want -= here;
      }
    }
  } else if (FILTERS) {
    // the list, lane l's entries R l .. R l + R - 1 of it
    int all = 0;
    bool fits = true;
#pragma unroll
    for (int q = 0; q < SP_PARTS_LANE; ++q) {
      if (kWave * q < parts) {
        const int n = listed[q], p = kWave * q + lane;
        fits = fits && __ballot(n < 0) == 0;
        const int incl = wave_inclusive_scan_i32(n, lane);
        if (p < parts) s_at[wv][p] = all + incl - n;
        all += __builtin_amdgcn_readlane(incl, 63);
      }
    }
    if (!fits || all > SL_MOST) return;      // the fourth launch's
    if (lane == 0) s_at[wv][parts] = all;
    __builtin_amdgcn_wave_barrier();
    const int R = (all + kWave - 1) / kWave, room = SL_LIST / parts;
    const Listed* const list = a.list + static_cast<size_t>(j) * SL_LIST;
    uint32_t key[SL_LANE];
    int index[SL_LANE];
    {
      int at = R * lane, p = 0;
      for (int step = 128; step > 0; step >>= 1)      // the part that holds entry `at`
        if (p + step < parts && s_at[wv][p + step] <= at) p += step;
#pragma unroll
      for (int r = 0; r < SL_LANE; ++r) {
        key[r] = 0;
        index[r] = 0;
        if (r < R && at < all) {
          while (s_at[wv][p + 1] <= at) ++p;
          const Listed l = list[static_cast<size_t>(p) * room + (at - s_at[wv][p])];
          key[r] = l.key;
          index[r] = l.index;
          ++at;
        }
      }
    }
    // The border: keys above it are kept, and the first `ties` equal to it.  Keys are tried bit by bit
    // from the first in which the listed ones differ.
    const bool by_count = a.top_k < V, by_mass = a.top_p < 1.0;
    const uint32_t key_top = f32_order_key(top);
    uint32_t least = key[0] != 0 ? key[0] : key_top;
#pragma unroll
    for (int r = 1; r < SL_LANE; ++r) least = min(least, key[r] != 0 ? key[r] : key_top);
    least = ~wave_max_u32(~least);
    const int bits = least == key_top ? 0 : 32 - __builtin_clz(least ^ key_top);      // that differ
    const uint32_t common = bits == 32 ? 0u : key_top >> bits << bits;
    // A lane's entries, four at a time (those past the list have key 0, below every key that is tried).
    auto each_listed = [&](auto&& f) SP_INLINE {
#pragma unroll
      for (int r0 = 0; r0 < SL_LANE; r0 += 4)
        if (r0 < R) {
#pragma unroll
          for (int r = r0; r < r0 + 4; ++r) f(r);
        }
    };
    uint32_t border = 0;
    int ties = 0x7fffffff;
    if (by_count && a.top_k < all) {
      border = common;
      for (int bit = bits - 1; bit >= 0; --bit) {
        const uint32_t t = border | (1u << bit);
        if (t > key_top) continue;
        int n = 0;
        each_listed([&](int r) SP_INLINE { n += key[r] >= t ? 1 : 0; });
        if (wave_sum_i32(n) >= a.top_k) border = t;
      }
      int above = 0;
      each_listed([&](int r) SP_INLINE { above += key[r] > border ? 1 : 0; });
      ties = a.top_k - wave_sum_i32(above);
    }
    // Of what is equal to `border`, this lane's first's rank.
    auto tie_rank = [&]() SP_INLINE {
      int n = 0;
#pragma unroll
      for (int r = 0; r < SL_LANE; ++r) n += key[r] == border ? 1 : 0;
      return wave_inclusive_scan_i32(n, lane) - n;
    };
    double w[SL_LANE];
    {
      int rank = tie_rank();
#pragma unroll
      for (int r = 0; r < SL_LANE; ++r) {
        const bool tie = key[r] == border;
        w[r] = r < R && key[r] != 0 && (key[r] > border || (tie && rank < ties)) ? weight(key[r]) : 0.0;
        rank += tie ? 1 : 0;
      }
    }
    if (by_mass) {
      const double fixed = fixed_scale(total);
      uint64_t q[SL_LANE], sum = 0;
#pragma unroll
      for (int r = 0; r < SL_LANE; ++r) {
        q[r] = r < R ? fixed_point(w[r], fixed) : 0;
        sum += q[r];
      }
      const double want = a.top_p * (by_count ? static_cast<double>(wave_sum64(sum)) : total * fixed);
      const uint64_t least_sum = static_cast<uint64_t>(ceil(want));      // (below 2^52)
      uint32_t last = common;      // the largest key from which on the weights sum to `want`
      for (int bit = bits - 1; bit >= 0; --bit) {
        const uint32_t t = last | (1u << bit);
        if (t > key_top) continue;
        sum = 0;
        each_listed([&](int r) SP_INLINE { sum += key[r] >= t ? q[r] : 0; });
        if (wave_sum64(sum) >= least_sum) last = t;
      }
      uint64_t above = 0;
#pragma unroll
      for (int r = 0; r < SL_LANE; ++r) above += key[r] > last ? q[r] : 0;
      above = wave_sum64(above);
      const double each = static_cast<double>(fixed_point(weight(last), fixed));
      border = last;      // (below all keys: all are needed)
      ties = each > 0.0 ? max(1, static_cast<int>(fmin(ceil((want - static_cast<double>(above)) / each), 2e9))) : 0;
      int rank = tie_rank();
#pragma unroll
      for (int r = 0; r < SL_LANE; ++r) {
        const bool tie = key[r] == border;
        if (!(key[r] > border || (tie && rank < ties))) w[r] = 0.0;
        rank += tie ? 1 : 0;
      }
    }
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < SL_LANE; ++r) {
      if (r < R) {
        if ((static_cast<double>(f32_from_order_key(key[r])) - m) * scale < a.floor2) w[r] = 0.0;
        sum += w[r];
      }
    }
    double rest;
    bool hit;
    const int lane_of = pick_lane(sum, u * wave_sum64(sum), 0.0, rest, hit);
    double cum = 0.0;
    int mine = -1;
    bool past = false;
    rest = lane == lane_of ? rest : 0.0;
#pragma unroll
    for (int r = 0; r < SL_LANE; ++r) {
      if (r < R && w[r] > 0.0 && !past) {
        cum += w[r];
        mine = index[r];
        past = cum > rest;
      }
    }
    if (lane_of >= 0) token = __builtin_amdgcn_readlane(mine, lane_of);
  } else if (scale > 0.0) {
    // the part that u falls into, 64 parts at a time, then its elements, eight consecutive ones a lane
    double target = u * total, before = 0.0, rest = 0.0;
    int last_part = 0;
    for (int p0 = 0; p0 < parts; p0 += kWave) {
      const double w = p0 + lane < parts ? part[p0 + lane].sum * pow2_or_0((static_cast<double>(part[p0 + lane].top) - m) * scale, table) : 0.0;
      bool hit;
      double left;
      const int lane_of = pick_lane(w, target, before, left, hit);
      before += wave_sum64(w);
      if (lane_of >= 0) {
        last_part = p0 + lane_of;
        const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(left));
        rest = __longlong_as_double(static_cast<long long>(
            (static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(bits >> 32), lane_of))) << 32) |
            static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(bits), lane_of))));
      }
      if (hit) break;
    }
    const int begin = row.begin(last_part), end = row.begin(last_part + 1);
    uint32_t next[SP_SCAN];
    auto load = [&](int i0) SP_INLINE {
#pragma unroll
      for (int e = 0; e < SP_SCAN; ++e) {
        const int i = i0 + SP_SCAN * lane + e;
        next[e] = i < end ? f32_order_key(fmaxf(row.at(i), SP_NONE)) : 0u;
      }
    };
    before = 0.0;
    load(begin);
    for (int i0 = begin; i0 < end; i0 += SP_SCAN * kWave) {
      double w[SP_SCAN], sum = 0.0;
#pragma unroll
      for (int e = 0; e < SP_SCAN; ++e) {
        w[e] = next[e] > f32_order_key(SP_NONE) ? weight(next[e]) : 0.0;
        sum += w[e];
      }
      load(i0 + SP_SCAN * kWave);
      bool hit;
      double left;
      const int lane_of = pick_lane(sum, rest, before, left, hit);
      before += wave_sum64(sum);
      double cum = 0.0;
      int mine = -1;
      bool past = false;
#pragma unroll
      for (int e = 0; e < SP_SCAN; ++e) {
        if (w[e] > 0.0 && !past) {
          cum += w[e];
          mine = i0 + SP_SCAN * lane + e;
          past = cum > left;
        }
      }
      if (lane_of >= 0) token = __builtin_amdgcn_readlane(mine, lane_of);
      if (hit) break;
    }
  }
  if (lane == 0) {
    a.tokens[pos] = token;
    if (a.conf != nullptr) {
      double w = 0.0;
      if (token >= 0) {
        const float l = row.at(token);
        w = l == top ? 1.0 : pow2_or_0((static_cast<double>(l) - m) * SP_LOG2E, table);
      }
      a.conf[pos] = static_cast<float>(w / flat);
    }
  }
}

struct SampleShared {
  double table[64];
  double sum[SP_WAVES];
  uint64_t wave_mass[SP_WAVES];
  int wave_count[SP_WAVES], ties[SP_WAVES], seg_n[SP_WAVES];
  uint32_t first[SP_WAVES], last[SP_WAVES];
  double target;
  uint64_t above;
  uint32_t bin;
  int token;
  uint64_t hist[SP_BINS];
  uint32_t key[SP_WAVES][SP_SEG];      // the list: order keys and indices, wave w's part in row w
  int index[SP_WAVES][SP_SEG];
};

template <class E>
__global__ __launch_bounds__(SP_THREADS) void sample_flat_kernel(const E* __restrict__ logits, SampleArgs a) {
  constexpr int VEC = Row<E>::VEC;
  using Values = typename Row<E>::Values;
  __shared__ SampleShared s;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = blockIdx.x, V = a.V, parts = a.parts;
  const double scale = a.scale, least = a.floor2;
  if (j >= rows_used(a)) return;
  const int pos = position_of(a, j);
  if (pos < 0 || pos >= a.T) return;
  bool fits = true;
  int all = 0;
  for (int p0 = 0; p0 < parts; p0 += kWave) {
    const int n = p0 + lane < parts ? a.listed[static_cast<size_t>(j) * parts + p0 + lane] : 0;
    fits = fits && __ballot(n < 0) == 0;
    all += wave_sum_i32(n);
  }
  if (fits && all <= SL_MOST) return;      // the third launch's
  if (tid < 64) s.table[tid] = pow2_entry(tid);
  __syncthreads();
  const Part* const part_of = a.part + static_cast<size_t>(j) * parts;
  const Row<E> row(logits + static_cast<size_t>(j) * V, V, SP_WAVES);      // (a wave a sixteenth)
  float top;
  int token;
  double total, flat;
  row_flat(a, load_parts(a, part_of), s.table, top, token, total, flat);
  const double m = top;
  const uint32_t key_top = f32_order_key(top);
  auto power = [&](uint32_t k) SP_INLINE { return (static_cast<double>(f32_from_order_key(k)) - m) * scale; };
  auto key_of = [&](float l) SP_INLINE { return f32_order_key(fmaxf(l, SP_NONE)); };      // (NaN as -inf)
  auto weight = [&](uint32_t k) SP_INLINE { return pow2_or_0(power(k), s.table); };

  // Of the threads' weights in thread order, the thread that `target` (of_all: times the sum) falls
  // into: s.target is then what is left of it; else the last thread with weight, s.target inf; -1: none
  // has weight.  `sum`: all weights.  hit: whether it falls into one.
  auto pick = [&](double w, double target, bool of_all, double& sum, bool& hit) SP_INLINE {
    const double incl = wave_inclusive_scan64(w);
    if (lane == 63) s.sum[wv] = incl;
    __syncthreads();
    const double before = waves_before(s.sum, wv, sum);
    if (of_all) target *= sum;
    const uint64_t hits = __ballot(w > 0.0 && before + incl > target), any = __ballot(w > 0.0);
    if (lane == 0) {      // (the first thread counted from the end, so that the largest is meant; 0: none)
      s.first[wv] = hits != 0 ? SP_THREADS - (kWave * wv + __builtin_ctzll(hits)) : 0;
      s.last[wv] = any != 0 ? kWave * wv + kWave - __builtin_clzll(any) : 0;
    }
    __syncthreads();
    const int first = static_cast<int>(wave_max_u32(lane < SP_WAVES ? s.first[lane] : 0));
    const int last = static_cast<int>(wave_max_u32(lane < SP_WAVES ? s.last[lane] : 0));
    hit = first != 0;
    const int winner = hit ? SP_THREADS - first : last - 1;
    if (tid == winner) s.target = hit ? target - (before + incl - w) : __builtin_huge_val();
    __syncthreads();
    return winner;
  };
  {
    float u = a.u[pos];
    u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
    // ---- filters: keys above `border` are kept, and the first `border_ties` of those equal to it; of
    // both only those with power() >= least
    const bool by_count = a.top_k < V, by_mass = a.top_p < 1.0;
    uint32_t border = f32_order_key(SP_NONE);
    int border_ties = 0;
    bool listed = false;      // the list holds all elements that may be kept
    double sum_above = 0.0;   // kept weights of this wave's sixteenth above the elements on the list,
    bool summed = false;      // which are all that may be the border
    {
      const float cut = filter_bound(a, part_of, m, total);
      const uint32_t key_low = f32_order_key(cut);
      // Bins of the first pass: linear in the logit, bin 0 at the cut (so that more is higher), or at
      // weights of 2^-64, where the lower ones are in it too.
      const float range = fminf(top - cut, static_cast<float>(64.0 / scale));
      const float inv = range > 1e-30f ? (SP_BINS - 0.5f) / range : 0.0f;
      auto linear_bin = [&](float l) SP_INLINE {
        return SP_BINS - 1 - static_cast<int>(fminf((top - l) * inv, SP_BINS - 1.0f));
      };
      const double fixed = fixed_scale(total);
      auto fixed_weight = [&](uint32_t k) SP_INLINE { return fixed_point(weight(k), fixed); };
      enum { LINEAR, KEYS, LIST };
      int stage = by_count || by_mass ? LINEAR : LIST;
      int within = -1, shift = 0;
      uint32_t lo = key_low, hi = key_top;
      bool weigh = !by_count, have = false;      // have: the list holds them all
      auto add = [&](uint32_t k, float l) SP_INLINE {
        const uint32_t bin = stage == LINEAR ? linear_bin(l) : (k - lo) >> shift;
        atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[bin]),
                  static_cast<unsigned long long>(weigh ? fixed_weight(k) : 1u));
      };
      // One pass over the elements with keys in [lo, hi] (within: only those of this linear bin; -1:
      // all): adds them to the bins, linear ones or those of (key - lo) >> shift, by number or by
      // weight; over the row it also lists them, in index order, as long as they fit, and over the keys
      // of the last criterion's bin sums the kept weights above.
      auto pass = [&]() SP_INLINE {
        for (int b = tid; b < SP_BINS; b += SP_THREADS) s.hist[b] = 0;
        __syncthreads();
        const float lo_f = f32_from_order_key(lo), hi_f = f32_from_order_key(hi);
        if (have) {
          const int n = s.seg_n[wv];
          for (int e = lane; e < n; e += kWave) {
            const uint32_t k = s.key[wv][e];
            const float l = f32_from_order_key(k);
            if (k >= lo && k <= hi && (within < 0 || linear_bin(l) == within)) add(k, l);
          }
          __syncthreads();
          return;
        }
        const bool sum_up = stage == KEYS && !summed && (weigh || !by_mass);
        int n_list = 0;      // (uniform in the wave)
        row.template each<false>(wv, [&](Values v, int n, int i, auto) SP_INLINE {
          uint32_t on = 0, up = 0;
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            if (e < n && v[e] >= lo_f) {
              const int bin = within < 0 ? 0 : linear_bin(v[e]) - within;
              on |= bin == 0 && v[e] <= hi_f ? 1u << e : 0u;
              up |= bin > 0 || v[e] > hi_f ? 1u << e : 0u;
            }
          }
          if (sum_up && __ballot(up != 0) != 0) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              const double x = (static_cast<double>(v[e]) - m) * scale;
              if (((up >> e) & 1u) && x >= least) sum_above += pow2_or_0(x, s.table);
            }
          }
          if (__ballot(on != 0) == 0) return;
          if (n_list <= SP_SEG) {
            const int count = __popc(on), incl = wave_inclusive_scan_i32(count, lane);
            int to = n_list + incl - count;
            n_list += __builtin_amdgcn_readlane(incl, 63);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              if ((on >> e) & 1u) {
                if (to < SP_SEG) {
                  s.key[wv][to] = f32_order_key(v[e]);
                  s.index[wv][to] = i + e;
                }
                ++to;
              }
            }
          }
          if (stage != LIST) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
              if ((on >> e) & 1u) add(f32_order_key(v[e]), v[e]);
          }
        });
        if (lane == 0) s.seg_n[wv] = n_list;
        __syncthreads();
        have = __ballot(lane < SP_WAVES && s.seg_n[lane] > SP_SEG) == 0;
        if (sum_up) {
          summed = have;
          if (!have) sum_above = 0.0;
        }
      };
      // From the top, the first bin with anything in it that brings the sum of the bins (and `above`)
      // to the aim, or the last with anything; s.above: the sum before it.  The aim is `want`, or
      // with `share` that share of all but `less`.
      auto choose = [&](uint64_t above, double want, double share, uint64_t less) SP_INLINE {
        const int top_bin = SP_BINS - 1 - 2 * tid;
        const uint64_t h[2] = {s.hist[top_bin], s.hist[top_bin - 1]};
        const uint64_t incl = wave_inclusive_scan64(h[0] + h[1]);
        if (lane == 63) s.wave_mass[wv] = incl;
        if (tid == 0) s.bin = 0;
        __syncthreads();
        uint64_t all;
        uint64_t q = above + waves_before(s.wave_mass, wv, all) + incl - h[0] - h[1];
        all += above;
        if (share > 0.0) want = share * static_cast<double>(all - less);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (h[e] > 0 && (q == 0 || static_cast<double>(q) < want) &&
              (static_cast<double>(q + h[e]) >= want || q + h[e] == all)) {
            s.bin = top_bin - e;
            s.above = q;
          }
          q += h[e];
        }
        __syncthreads();
        return want;
      };
      // Top-k, then top-p of what it leaves: a linear pass, then passes over the keys of its bin, each
      // over the row until what is left fits the list.  What top-k leaves is listed if it fits.  Min-p
      // alone needs no pass.
      uint32_t from = key_low;      // elements below are cut off, of those equal to it all but `room`
      int room = 0x7fffffff;
      uint64_t above = 0, less = 0;
      double want = by_count ? static_cast<double>(a.top_k) : a.top_p * (total * fixed);
      double share = 0.0;
      if (stage == LIST) border = key_low - 1;
      // Top-p alone: the bins' numbers of elements and mean logits (a fifth of the instructions of a
      // weight) say nearly where its border lies.  One pass over the row then sums the weights above a few
      // bins around it and lists those bins' elements, and the border is sought in the list; if it is not
      // there after all, or the list is too long, the passes below find it.
      // (Rows that fit the list whole need no such search.)
      if (by_mass && !by_count && V > SP_WAVES * SP_SEG && top < __builtin_huge_valf()) {
        for (int b = tid; b < SP_BINS; b += SP_THREADS) s.hist[b] = 0;      // (number, sum of places in the bin)
        if (tid == 0) s.bin = 0;
        __syncthreads();
        row.template each<true>(wv, [&](Values v, int n, int, auto whole) SP_INLINE {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            if ((decltype(whole)::value || e < n) && v[e] >= cut) {
              const float down = (top - v[e]) * inv;      // (as in linear_bin)
              const int bin = static_cast<int>(fminf(down, SP_BINS - 1.0f));
              const float place = fminf(down - static_cast<float>(bin), 1.0f);      // (V 2^11 < 2^32)
              atomicAdd(reinterpret_cast<unsigned long long*>(&s.hist[SP_BINS - 1 - bin]),
                        (1ull << 32) | static_cast<uint32_t>(place * 2047.0f));
            }
          }
        });
        __syncthreads();
        {
          const int top_bin = SP_BINS - 1 - 2 * tid;
          double h[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const double n = static_cast<double>(s.hist[top_bin - e] >> 32);
            const double places = static_cast<double>(static_cast<uint32_t>(s.hist[top_bin - e])) / 2047.0;
            h[e] = n > 0.0 && inv > 0.0f ? n * pow2_or_0(-(2 * tid + e + places / n) / inv * scale, s.table) : n;
          }
          const double incl = wave_inclusive_scan64(h[0] + h[1]);
          if (lane == 63) s.sum[wv] = incl;
          __syncthreads();
          double all;
          const double q = waves_before(s.sum, wv, all) + incl - h[0] - h[1], aim = a.top_p * total;
          if (q < aim && q + h[0] + h[1] >= aim) s.bin = top_bin - (q + h[0] >= aim ? 0 : 1);
          __syncthreads();
        }
        // as many bins on either side as half of the list has room for (wide bins: one is enough)
        const int middle = static_cast<int>(s.bin), side = abs(lane - SP_AROUND), at_bin = middle + lane - SP_AROUND;
        const int near = side <= SP_AROUND && at_bin >= 0 && at_bin < SP_BINS ? static_cast<int>(s.hist[at_bin] >> 32) : 0;
        int around = SP_AROUND;
        while (around > 1 && wave_sum_i32(side <= around ? near : 0) > SP_WAVES * SP_SEG / 2) --around;
        const int first = middle - around, last = middle + around;
        // bins above the last: (top - l) inv < up_to; the listed ones and above: < list_to
        const float up_to = static_cast<float>(SP_BINS - 1 - last);
        const float list_to = first <= 0 ? __builtin_huge_valf() : static_cast<float>(SP_BINS - first);
        const uint32_t by_fixed = static_cast<uint32_t>(__double_as_longlong(fixed) >> 32) - (1023u << 20);
        const bool floored = least > -__builtin_huge_val();
        uint64_t mass = 0;      // (a weight in fixed point as the bits of 2^52 and it)
        uint32_t key_min = 0xffffffffu, key_max = 0;
        int n_list = 0, added = 0;      // (uniform in the wave)
        row.template each<false>(wv, [&](Values v, int n, int i, auto) SP_INLINE {
          uint32_t on = 0;
          added += VEC;
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float l = e < n ? v[e] : SP_NONE;
            const float at = fmaxf(l, cut), down = (top - at) * inv;
            const bool up = down < up_to;
            on |= !up && down < list_to && l >= cut ? 1u << e : 0u;
            const double d = static_cast<double>(at) - m, y = fma(d, scale, kMagic);
            double p, t;
            pow2_parts(y, fma(d, scale, kMagic - y), s.table, p, t);
            u32x2_t word = __builtin_bit_cast(u32x2_t, t);      // (times the fixed point's scale; nothing below)
            word[1] = up ? word[1] + by_fixed : 0u;
            const double f = fma(p, __builtin_bit_cast(double, word), 0x1p52);
            mass += static_cast<uint64_t>(__double_as_longlong(f));
            if (floored) sum_above += up && d * scale >= least ? f - 0x1p52 : 0.0;
          }
          if (n_list > SP_SEG || __ballot(on != 0) == 0) return;
          const int ones = __popc(on), incl = wave_inclusive_scan_i32(ones, lane);
          int to = n_list + incl - ones;
          n_list += __builtin_amdgcn_readlane(incl, 63);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            if ((on >> e) & 1u) {
              const uint32_t k = f32_order_key(v[e]);
              key_min = min(key_min, k);
              key_max = max(key_max, k);
              if (to < SP_SEG) {
                s.key[wv][to] = k;
                s.index[wv][to] = i + e;
              }
              ++to;
            }
          }
        });
        mass -= static_cast<uint64_t>(added) * 0x4330000000000000ull;
        sum_above = (floored ? sum_above : static_cast<double>(mass)) / fixed;
        uint64_t mass_listed = 0;      // (of the list as far as there is room for it)
        for (int e = lane; e < min(n_list, SP_SEG); e += kWave) mass_listed += fixed_weight(s.key[wv][e]);
        mass = wave_sum64(mass);
        mass_listed = wave_sum64(mass_listed);
        key_min = ~wave_max_u32(~key_min);
        key_max = wave_max_u32(key_max);
        uint64_t sum_listed;
        if (lane == 0) {
          s.seg_n[wv] = n_list;
          s.wave_mass[wv] = mass;
          s.first[wv] = key_min;
          s.last[wv] = key_max;
        }
        __syncthreads();
        waves_before(s.wave_mass, wv, above);
        key_min = ~wave_max_u32(lane < SP_WAVES ? ~s.first[lane] : 0u);
        key_max = wave_max_u32(lane < SP_WAVES ? s.last[lane] : 0u);
        have = __ballot(lane < SP_WAVES && s.seg_n[lane] > SP_SEG) == 0;
        __syncthreads();
        if (lane == 0) s.wave_mass[wv] = mass_listed;
        __syncthreads();
        waves_before(s.wave_mass, wv, sum_listed);
        __syncthreads();
        have = have && sum_listed > 0 && (above == 0 || static_cast<double>(above) < want) &&
               (first <= 0 || static_cast<double>(above + sum_listed) >= want);
        summed = have;
        if (have) {
          stage = KEYS;
          lo = key_min;
          hi = key_max;
        } else {
          above = 0;
          sum_above = 0.0;
        }
      }
      while (by_count || by_mass) {
        if (stage == KEYS) {
          const uint32_t span = hi - lo;
          const int bits = span == 0 ? 0 : 32 - __builtin_clz(span);
          shift = bits > SP_BIN_BITS ? bits - SP_BIN_BITS : 0;
        }
        pass();
        if (stage == LIST) {
          listed = have;
          if (!by_count || !by_mass) break;
        } else {
          if (stage == KEYS && shift == 0 && lo == from && room < 0x7fffffff) {
            const uint64_t most_here = (weigh ? fixed_weight(lo) : 1u) * static_cast<uint64_t>(room);
            if (tid == 0) s.hist[0] = min(s.hist[0], most_here);
            __syncthreads();
          }
          want = choose(above, want, share, less);
          share = 0.0;
          const uint32_t at = s.bin;
          above = s.above;
          const uint64_t here = s.hist[at];
          __syncthreads();
          if (stage == LINEAR) {
            listed = listed || have;      // (all from key_low, or from top-k's border, on)
            within = static_cast<int>(at);
            stage = KEYS;
            continue;
          }
          lo += at << shift;
          hi = min(hi, lo + ((1u << shift) - 1u));
          if (shift > 0) continue;
          border = lo;
          if (weigh) {
            // as many of the border's elements as bring the sum to the aim
            const double each = static_cast<double>(fixed_weight(lo));
            border_ties = each > 0.0 ? static_cast<int>(fmax(1.0, fmin(ceil((want - static_cast<double>(above)) / each),
                                                                       rint(static_cast<double>(here) / each))))
                                     : 1;
            break;
          }
          border_ties = static_cast<int>(fmin(want - static_cast<double>(above), static_cast<double>(here)));
          less = here - static_cast<uint64_t>(border_ties);      // (their number yet)
          if (summed) break;
          if (!listed) {
            stage = LIST;
            within = -1;
            lo = border;
            hi = key_top;
            have = false;
            continue;
          }
          if (!by_mass) break;
        }
        weigh = true;
        stage = LINEAR;
        within = -1;
        from = lo = border;
        hi = key_top;
        room = border_ties;
        have = listed;
        above = 0;
        less *= fixed_weight(border);
        share = a.top_p;
      }
    }
    // ---- the draw
    auto kept = [&](uint32_t k, bool tie_kept) SP_INLINE {
      return (k > border || (k == border && tie_kept)) && k > f32_order_key(SP_NONE) && power(k) >= least;
    };
    // Ranks of a thread's `n` ties among all threads' in thread order; `all`: how many there are.
    auto tie_rank = [&](int n, int& all) SP_INLINE {
      const int incl = wave_inclusive_scan_i32(n, lane);
      if (lane == 63) s.wave_count[wv] = incl;
      __syncthreads();
      const int rank = waves_before(s.wave_count, wv, all) + incl - n;
      __syncthreads();
      return rank;
    };
    // The weights of the list's entries, kept ones: wave w has segment w, lane l its entries 4 l ..;
    // and how many ties among them are kept.
    double w[SP_LANE];
    double sum = 0.0;
    int ties_kept = 0;
    if (listed || summed) {
      const int n = s.seg_n[wv];
      uint32_t k[SP_LANE];
      int ties = 0, all;
#pragma unroll
      for (int e = 0; e < SP_LANE; ++e) {
        const int at = SP_LANE * lane + e;
        k[e] = at < n ? s.key[wv][at] : 0u;
        ties += k[e] == border ? 1 : 0;
      }
      int rank = tie_rank(ties, all);
#pragma unroll
      for (int e = 0; e < SP_LANE; ++e) {
        const bool tie = k[e] == border;
        w[e] = kept(k[e], tie && rank < border_ties) ? weight(k[e]) : 0.0;
        ties_kept += tie && rank < border_ties ? 1 : 0;
        rank += tie ? 1 : 0;
        sum += w[e];
      }
    }
    if (listed) {
      double sum_all;
      bool hit;
      const int winner = pick(sum, u, true, sum_all, hit);
      if (tid == winner) {
        double cum = 0.0;
        int to = -1;
        bool past = false;
#pragma unroll
        for (int e = 0; e < SP_LANE; ++e) {
          cum += w[e];
          if (w[e] > 0.0 && !past) {
            to = s.index[wv][SP_LANE * lane + e];
            past = cum > s.target;
          }
        }
        s.token = to;
      }
      __syncthreads();
      if (winner >= 0) token = s.token;
    } else {
      int part, begin, end, tie_room = 0;
      double unused;
      bool hit;
      if (summed) {
        sum = wave_sum64(sum + sum_above);
        ties_kept = wave_sum_i32(ties_kept);
        if (lane == 0) s.ties[wv] = ties_kept;
      } else {
        int ties = 0;
        row.template each<false>(wv, [&](Values v, int n, int, auto) SP_INLINE {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const uint32_t k = key_of(v[e]);
            if (e < n && kept(k, false)) sum += weight(k);
            ties += e < n && k == border ? 1 : 0;
          }
        });
        sum = wave_sum64(sum);
        ties = wave_sum_i32(ties);
        if (lane == 0) s.ties[wv] = ties;
        __syncthreads();
        int all;
        const int mine_kept = min(ties, max(border_ties - waves_before(s.ties, wv, all), 0));
        if (kept(border, true)) sum += mine_kept * weight(border);
        __syncthreads();
        if (lane == 0) s.ties[wv] = mine_kept;
      }
      part = pick(lane == 0 ? sum : 0.0, u, true, unused, hit) / kWave;      // (-1 / 64 is 0: weights are there)
      tie_room = s.ties[part];
      begin = row.begin(part);
      end = row.begin(part + 1);
      // that part, eight consecutive elements a thread; the last kept token stands in where the order
      // of the additions leaves the target at the part's end
      double target = s.target;
      int tie_base = 0;
      __syncthreads();
      for (int i0 = begin; i0 < end; i0 += SP_SCAN * SP_THREADS) {
        const int i1 = i0 + SP_SCAN * tid;
        uint32_t k[SP_SCAN];
        int ties = 0, all = 0;
#pragma unroll
        for (int e = 0; e < SP_SCAN; ++e) {
          k[e] = i1 + e < end ? key_of(row.at(i1 + e)) : 0u;
          ties += k[e] == border ? 1 : 0;
        }
        int rank = 0;
        rank = tie_base + tie_rank(ties, all);
        double w[SP_SCAN], sum = 0.0;
#pragma unroll
        for (int e = 0; e < SP_SCAN; ++e) {
          const bool tie = k[e] == border;
          w[e] = kept(k[e], tie && rank < tie_room) ? weight(k[e]) : 0.0;
          rank += tie ? 1 : 0;
          sum += w[e];
        }
        double sum_all;
        const int winner = pick(sum, target, false, sum_all, hit);
        if (tid == winner) {
          double cum = 0.0;
          int to = -1;
          bool past = false;
#pragma unroll
          for (int e = 0; e < SP_SCAN; ++e) {
            cum += w[e];
            if (w[e] > 0.0 && !past) {
              to = i1 + e;
              past = cum > s.target;
            }
          }
          s.token = to;
        }
        __syncthreads();
        if (winner >= 0) token = s.token;
        __syncthreads();
        if (hit) break;
        target -= sum_all;
        tie_base += all;
      }
    }
  }
  if (tid == 0) {
    a.tokens[pos] = token;
    if (a.conf != nullptr) {
      const double x = (static_cast<double>(row.at(token)) - m) * SP_LOG2E;
      a.conf[pos] = static_cast<float>(pow2_or_0(x, s.table) / flat);
    }
  }
}

// Parts of a row, a wave each: 4096 elements at most (the third launch scans one), more parts for few
// rows (4096 waves fill the GPU, but not for fewer than 512 elements); a multiple of a workgroup's waves.
int parts_of(int M, int V) {
  const int least = (V + 4095) / 4096;
  const int fill = std::min((4096 + M - 1) / std::max(M, 1), V / 512);
  return std::min((std::max({least, fill, 1}) + SS_WAVES - 1) / SS_WAVES * SS_WAVES, SP_PARTS);
}

}  // namespace

static bool filters(const SampleArgs& a) { return a.top_k < a.V || a.top_p < 1.0 || a.floor2 > -1.0e300; }

// Rows are taken SP_ROWS at a time, each with all launches (a launch has less than 2^32 threads, and the
// workspace, 33 to 81 KB a row, serves the next rows again).  Of those of a launch: the parts' records, the
// numbers of elements listed, the maxima of pairs, the lists.
static size_t part_bytes(int M, int V) { return align_up(sizeof(Part) * static_cast<size_t>(M) * parts_of(M, V)); }
static size_t listed_bytes(int M, int V) { return align_up(sizeof(int32_t) * static_cast<size_t>(M) * parts_of(M, V)); }
static size_t pair_bytes(int M, int V) {
  return align_up(sizeof(float) * (kWave / 2) * static_cast<size_t>(M) * parts_of(M, V));
}
size_t sample_ws_bytes(int M, int V) {
  M = std::min(M, SP_ROWS);
  return part_bytes(M, V) + listed_bytes(M, V) + pair_bytes(M, V) + align_up(sizeof(Listed) * static_cast<size_t>(M) * SL_LIST);
}

template <class E>
static int launch_sample_as(const E* logits, const SampleArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((static_cast<size_t>(a.M) * a.parts + SS_WAVES - 1) / SS_WAVES));
  auto sums = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(SS_THREADS), 0, s, logits, a); };
  if (a.scale == 0.0)
    sums(sample_sums_kernel<E, false, true, false>);
  else if (a.scale == SP_LOG2E)
    a.top_k < a.V ? sums(sample_sums_kernel<E, true, false, true>) : sums(sample_sums_kernel<E, true, false, false>);
  else
    a.top_k < a.V ? sums(sample_sums_kernel<E, true, true, true>) : sums(sample_sums_kernel<E, true, true, false>);
  const dim3 rows(static_cast<unsigned>((a.M + SS_WAVES - 1) / SS_WAVES));
  if (a.scale > 0.0 && filters(a)) {
    hipLaunchKernelGGL((sample_list_kernel<E>), grid, dim3(SS_THREADS), 0, s, logits, a);
    hipLaunchKernelGGL((sample_row_kernel<E, true>), rows, dim3(SS_THREADS), 0, s, logits, a);
    hipLaunchKernelGGL((sample_flat_kernel<E>), dim3(static_cast<unsigned>(a.M)), dim3(SP_THREADS), 0, s, logits, a);
  } else {
    hipLaunchKernelGGL((sample_row_kernel<E, false>), rows, dim3(SS_THREADS), 0, s, logits, a);
  }
  return launch_status();
}

int launch_sample(const void* logits, int logits_type, const int32_t* rows, const int32_t* n_rows, int M, int V,
                  const float* u, const reflex_sample_params& p, int T, int32_t* tokens, float* conf, void* ws,
                  hipStream_t s) {
  const int most = std::min(M, SP_ROWS);
  char* at[4] = {static_cast<char*>(ws)};
  at[1] = at[0] + part_bytes(most, V);
  at[2] = at[1] + listed_bytes(most, V);
  at[3] = at[2] + pair_bytes(most, V);
  SampleArgs a{rows, n_rows, most, V, T, parts_of(most, V), 0, u,
               p.temperature > 0.0f ? SP_LOG2E / static_cast<double>(p.temperature) : 0.0,
               p.min_p > 0.0f ? std::log2(static_cast<double>(p.min_p)) : -std::numeric_limits<double>::infinity(),
               p.top_k > 0 && p.top_k < V ? p.top_k : V, static_cast<double>(p.top_p), tokens, conf,
               reinterpret_cast<Part*>(at[0]), reinterpret_cast<float*>(at[2]), reinterpret_cast<int32_t*>(at[1]),
               reinterpret_cast<Listed*>(at[3])};
  for (; a.row0 < M; a.row0 += most) {
    a.M = std::min(most, M - a.row0);
    a.rows = rows == nullptr ? nullptr : rows + a.row0;
    const size_t first = static_cast<size_t>(a.row0) * V;
    const int rc = logits_type == REFLEX_TYPE_F32 ? launch_sample_as(static_cast<const float*>(logits) + first, a, s)
                                                  : launch_sample_as(static_cast<const uint16_t*>(logits) + first, a, s);
    if (rc != REFLEX_OK) return rc;
  }
  return REFLEX_OK;
}

}  // namespace rfx
