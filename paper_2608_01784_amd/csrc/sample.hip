// A token and its confidence from a row of logits and one uniform number (reflex_sample_tokens).
//
// Weights and their sums are fp64 where a draw or a filter compares them: with u given, the
// token is a matter of which side of a border u lies on, and sums in fp32 (relative error 1e-7
// times some) would take another token in one row of a hundred where 1e5 tokens share the mass.
// w = 2^((l - max) log2(e) / temperature) by a table of 64 powers and a cubic (relative error
// 4e-11, a dozen vector instructions); the confidence's denominator sums fp32 powers.
//
// One workgroup of 16 waves holds a row, wave w the w-th sixteenth of it, in 16-byte loads.
//  1. One pass: maximum with its first index, sum of weights, sum for the confidence.  Every
//     thread sums relative to a logit of its own, which it moves when one lies 2^60 above it;
//     the sums are scaled to the row's maximum at the end.
//  2. Filters, if any.  The last kept logit is found by narrowing a range of 32-bit order keys, 11
//     bits a pass, by counts (top-k) or weights (top-p; fixed point, 2^-43, so that the sums do
//     not depend on the order of the atomics).  The range starts at a bound that no kept logit
//     lies below (at_least()); a pass over the row also lists the range's elements in LDS, in index
//     order, and when they fit (4096), as they mostly do, everything that follows works on the list.
//  3. The draw: the kept weights' sums by sixteenth (of the list, or of the row in one more pass),
//     the one that u falls into, and a scan of that one alone.
// Everything is inlined and in registers: no stack.
#include <cmath>
#include <limits>

#include "fp8.h"

namespace rfx {
namespace {

constexpr int SP_THREADS = 1024, SP_WAVES = SP_THREADS / kWave;
constexpr int SP_BIN_BITS = 11, SP_BINS = 1 << SP_BIN_BITS;
constexpr int SP_LANE = 4, SP_SEG = SP_LANE * kWave;      // list entries of a lane and of a wave
constexpr double SP_FIXED = 8796093022208.0;              // 2^43: 2^20 weights of 1 fit 64 bits
static_assert(REFLEX_MAX_VOCAB <= (1 << 20), "fixed-point sums");
static_assert(SP_BINS == 2 * SP_THREADS, "two bins a thread");
constexpr double SP_LOG2E = 1.4426950408889634074;
constexpr float SP_NONE = -__builtin_huge_valf();

#define SP_INLINE __attribute__((always_inline))

struct SampleArgs {
  const int32_t *rows, *n_rows;
  int M, V, T;
  const float* u;
  double scale;          // log2(e) / temperature; 0: temperature 0
  double floor2;         // log2(min_p), -inf for none
  int top_k;             // 1 .. V
  double top_p;
  int32_t* tokens;
  float* conf;
};

// 2^x for -1020 <= x <= 1000.
RFX_DEVICE double pow2(double x, const double* table) {
  constexpr double kMagic = 0x1.8p46;            // its last place is 1 / 64
  const double y = x + kMagic;
  const double r = x - (y - kMagic);             // |r| <= 1 / 128
  const int n = static_cast<int>(__double_as_longlong(y));
  double p = fma(r, 0.05550410866482158, 0.24022650695910071);
  p = fma(r, p, 0.69314718055994531);
  p = fma(r, p, 1.0) * table[n & 63];
  return __longlong_as_double(__double_as_longlong(p) + static_cast<long long>(static_cast<unsigned long long>(n >> 6) << 52));
}

// 2^x for x <= 1000, zero below 2^-1020.
RFX_DEVICE double pow2_or_0(double x, const double* table) { return x >= -1020.0 ? pow2(x, table) : 0.0; }

RFX_DEVICE double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

template <class T>
RFX_DEVICE T wave_inclusive_shfl(T v, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const T up = __shfl_up(v, o, kWave);
    v += lane >= o ? up : T(0);
  }
  return v;
}

struct SampleShared {
  double table[64];
  double sum[SP_WAVES], flat[SP_WAVES];
  uint64_t best[SP_WAVES], wave_mass[SP_WAVES];
  int wave_count[SP_WAVES], ties[SP_WAVES], seg_n[SP_WAVES];
  float low[SP_WAVES];
  double target;
  uint64_t above_mass;
  uint32_t bin, above, key_count;
  int part, token;
  uint32_t count[SP_BINS];
  uint64_t mass[SP_BINS];
  uint32_t key[SP_WAVES][SP_SEG];      // the list: order keys and indices, wave w's part in row w
  int index[SP_WAVES][SP_SEG];
};

// A row of logits: elements before the first 16-byte boundary, vectors, a wave's share of those.
template <class E>
struct Row {
  static constexpr int VEC = 16 / sizeof(E);
  const E* p;
  int V, head, vecs, per_wave;

  RFX_DEVICE Row(const E* p_, int V_) : p(p_), V(V_) {
    head = min(V, static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(E)));
    vecs = (V - head) / VEC;
    per_wave = (vecs + SP_WAVES - 1) / SP_WAVES;
  }
  // First index of wave w's part (w = 16: V).
  RFX_DEVICE int begin(int w) const { return w == 0 ? 0 : (w == SP_WAVES ? V : head + min(w * per_wave, vecs) * VEC); }
  // NaN as -inf; inf_row: where some are +inf, those are 0 and the others -inf.
  RFX_DEVICE static float value(float l, bool inf_row) {
    l = fmaxf(l, SP_NONE);
    return inf_row ? (l == -SP_NONE ? 0.0f : SP_NONE) : l;
  }
  RFX_DEVICE float at(int i, bool inf_row) const {
    if constexpr (sizeof(E) == 2)
      return value(bf16_to_f32(p[i]), inf_row);
    else
      return value(p[i], inf_row);
  }
  // f(values, n, index of the first) in index order for this wave's part, 64 lanes at a time: n is VEC,
  // or less (0 and 1 too) before the first and behind the last vector; every lane is active in every call.
  template <class F>
  RFX_DEVICE void each(bool inf_row, F&& f) const {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float v[VEC];
    auto single = [&](int i, bool on) SP_INLINE {
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[j] = SP_NONE;
      if (on) v[0] = at(i, inf_row);
      f(v, on ? 1 : 0, i);
    };
    if (w == 0) single(lane, lane < head);
    const uint4* const vec = reinterpret_cast<const uint4*>(p + head);
    const int begin = min(w * per_wave, vecs), end = min((w + 1) * per_wave, vecs);
    const uint4 none = make_uint4(0, 0, 0, 0);
    auto load = [&](int i) SP_INLINE { return i < end ? vec[i] : none; };
    uint4 q[4];      // three vectors ahead
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = load(begin + j * kWave + lane);
    for (int i0 = begin; i0 < end; i0 += kWave) {
      const int i = i0 + lane;
      const uint32_t b[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
      q[0] = q[1];
      q[1] = q[2];
      q[2] = q[3];
      q[3] = load(i + 4 * kWave);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(E) == 2) {
          v[2 * j] = value(__uint_as_float(b[j] << 16), inf_row);
          v[2 * j + 1] = value(__uint_as_float(b[j] & 0xffff0000u), inf_row);
        } else {
          v[j] = value(__uint_as_float(b[j]), inf_row);
        }
      }
      f(v, i < end ? VEC : 0, head + i * VEC);
    }
    if (w == SP_WAVES - 1) single(head + vecs * VEC + lane, head + vecs * VEC + lane < V);
  }
};

template <class E>
__global__ __launch_bounds__(SP_THREADS) void sample_kernel(const E* __restrict__ logits, SampleArgs a) {
  constexpr int VEC = Row<E>::VEC;
  __shared__ SampleShared s;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = blockIdx.x, V = a.V;
  const double scale = a.scale, least = a.floor2;
  const int used = a.n_rows == nullptr ? a.M : min(a.n_rows[0], a.M);
  if (j >= used) return;
  const int pos = a.rows == nullptr ? j : a.rows[j];
  if (pos < 0 || pos >= a.T) return;
  if (tid < 64) s.table[tid] = exp2(tid / 64.0);
  __syncthreads();
  const Row<E> row(logits + static_cast<size_t>(j) * V, V);
  const bool draws = scale > 0.0, same = scale == SP_LOG2E;
  const double step = fmax(scale, SP_LOG2E);

  // ---- 1. maximum and sums
  bool inf_row = false;
  float top, low;      // the maximum; the least of the threads' own maxima
  int first;
  double flat;
  for (;;) {
    float best = SP_NONE, ref = -3.402823466e38f;
    int at = 0x7fffffff;
    double sum = 0.0, z = 0.0;
    row.each(inf_row, [&](const float (&v)[VEC], int n, int i) SP_INLINE {
      float m = v[0];
#pragma unroll
      for (int k = 1; k < VEC; ++k) m = fmaxf(m, v[k]);
      if (n > 0 && (m > best || at == 0x7fffffff)) {
        best = m;
        at = i;
#pragma unroll
        for (int k = VEC - 1; k >= 0; --k)
          if (v[k] == m) at = i + k;
      }
      const double up = static_cast<double>(m) - static_cast<double>(ref);
      if (n > 0 && up * step > 60.0 && m < -SP_NONE) {      // move the reference here
        sum *= pow2_or_0(-up * scale, s.table);
        z *= pow2_or_0(-up * SP_LOG2E, s.table);
        ref = m;
      }
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        if (k < n) {
          const double x = static_cast<double>(v[k]) - static_cast<double>(ref);
          if (draws) sum += pow2_or_0(fmin(x * scale, 60.0), s.table);
          if (!same) z += __builtin_amdgcn_exp2f(static_cast<float>(x * SP_LOG2E));
        }
      }
    });
    float mine = best;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine = fminf(mine, __shfl_xor(mine, o, kWave));
    const uint64_t key = wave_max_u64((static_cast<uint64_t>(f32_order_key(best)) << 32) |
                                      (0x7fffffffu - static_cast<uint32_t>(at)));
    if (lane == 0) {
      s.best[wv] = key;
      s.low[wv] = mine;
    }
    __syncthreads();
    uint64_t most = 0;
    low = -SP_NONE;
#pragma unroll
    for (int x = 0; x < SP_WAVES; ++x) {
      most = max(most, s.best[x]);
      low = fminf(low, s.low[x]);
    }
    top = f32_from_order_key(static_cast<uint32_t>(most >> 32));
    first = static_cast<int>(0x7fffffffu - static_cast<uint32_t>(most));
    __syncthreads();
    if (top == -SP_NONE) {       // some +inf: once more, among them
      inf_row = true;
      continue;
    }
    if (top == SP_NONE) {        // nothing has weight
      if (tid == 0) {
        a.tokens[pos] = -1;
        if (a.conf != nullptr) a.conf[pos] = 0.0f;
      }
      return;
    }
    const double down = static_cast<double>(ref) - static_cast<double>(top);
    sum = wave_sum_f64(sum * pow2_or_0(down * scale, s.table));
    z = wave_sum_f64(z * pow2_or_0(down * SP_LOG2E, s.table));
    if (lane == 0) {
      s.sum[wv] = sum;
      s.flat[wv] = same ? sum : z;
    }
    __syncthreads();
    flat = 0.0;
#pragma unroll
    for (int x = 0; x < SP_WAVES; ++x) flat += s.flat[x];
    __syncthreads();
    break;
  }
  const double m = top;
  auto power = [&](float l) SP_INLINE { return (static_cast<double>(l) - m) * scale; };
  auto key_power = [&](uint32_t k) SP_INLINE { return power(f32_from_order_key(k)); };
  int token = first;
  if (draws) {
    // ---- 2. filters: keys above `border` are kept, and the first `border_ties` of those equal to
    // it; of both only those with power() >= least
    const bool some = a.top_k < V || a.top_p < 1.0 || least > -1.0e300;
    uint32_t border = f32_order_key(SP_NONE);
    int border_ties = 0;
    bool listed = false;      // the list holds all elements that may be kept
    if (some) {
      // A logit that no kept one lies below: by top-k, as many threads as have elements (1024, or V)
      // have a maximum of at least `low`; by top-p, tokens of less than the share (1 - top_p) / V
      // together hold less than what may be left out; and min-p itself.  (fp32 after a margin.)
      float cut = a.top_k <= min(V / VEC, SP_THREADS) ? low : SP_NONE;
      if (cut == SP_NONE || a.top_k >= V) {
        cut = SP_NONE;
        double total = 0.0;
        if (a.top_p < 1.0 && a.top_k >= V) {
          for (int x = 0; x < SP_WAVES; ++x) total += s.sum[x];
          cut = static_cast<float>(m + (log2((1.0 - a.top_p) * total / V) - 0.001) / scale);
        }
      }
      // (not where top-p needs the weight of what top-k leaves, min-p's part among it)
      if (least > -1.0e300 && (a.top_k >= V || a.top_p >= 1.0))
        cut = fmaxf(cut, static_cast<float>(m + (least - 0.001) / scale));
      cut = cut < top ? cut - 1e-6f * fmaxf(fabsf(cut), fabsf(top)) : top;
      cut = fminf(cut, top);
      const uint32_t key_low = f32_order_key(fmaxf(cut, -3.402823466e38f)), key_top = f32_order_key(top);
      // Lists the elements with keys in [lo, hi], in index order, as long as they fit; and counts and
      // weighs them by bins of (key - lo) >> shift.
      auto row_pass = [&](uint32_t lo, uint32_t hi, int shift, bool weigh) SP_INLINE {
        for (int b = tid; b < SP_BINS; b += SP_THREADS) {
          s.count[b] = 0;
          s.mass[b] = 0;
        }
        __syncthreads();
        int n_list = 0;      // (uniform in the wave)
        row.each(inf_row, [&](const float (&v)[VEC], int n, int i) SP_INLINE {
          uint32_t in = 0;
          uint32_t k[VEC];
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            k[e] = f32_order_key(v[e]);
            in |= e < n && k[e] >= lo && k[e] <= hi ? 1u << e : 0u;
          }
          if (__ballot(in != 0) == 0) return;
          const int mine = __popc(in), incl = wave_inclusive_scan_i32(mine, lane);
          int to = n_list + incl - mine;
          n_list += __builtin_amdgcn_readlane(incl, 63);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            if ((in >> e) & 1u) {
              if (to < SP_SEG) {
                s.key[wv][to] = k[e];
                s.index[wv][to] = i + e;
              }
              ++to;
              const uint32_t b = (k[e] - lo) >> shift;
              atomicAdd(&s.count[b], 1u);
              if (weigh)
                atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[b]),
                          static_cast<unsigned long long>(pow2_or_0(power(v[e]), s.table) * SP_FIXED + 0.5));
            }
          }
        });
        if (lane == 0) s.seg_n[wv] = n_list;
        __syncthreads();
      };
      auto list_pass = [&](uint32_t lo, uint32_t hi, int shift, bool weigh) SP_INLINE {
        for (int b = tid; b < SP_BINS; b += SP_THREADS) {
          s.count[b] = 0;
          s.mass[b] = 0;
        }
        __syncthreads();
        const int n = s.seg_n[wv];
        for (int e = lane; e < n; e += kWave) {
          const uint32_t k = s.key[wv][e];
          if (k >= lo && k <= hi) {
            const uint32_t b = (k - lo) >> shift;
            atomicAdd(&s.count[b], 1u);
            if (weigh)
              atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[b]),
                        static_cast<unsigned long long>(pow2_or_0(key_power(k), s.table) * SP_FIXED + 0.5));
          }
        }
        __syncthreads();
      };
      auto list_fits = [&]() SP_INLINE {
        bool fits = true;
#pragma unroll
        for (int x = 0; x < SP_WAVES; ++x) fits = fits && s.seg_n[x] <= SP_SEG;
        return fits;
      };
      // Sums over all bins above bin SP_BINS - 1 - 2 tid (exclusive), then the first bin from the top
      // that has elements and reaches the aim, or the last with elements: s.bin, and what is above.
      auto choose = [&](bool weigh, uint32_t above, uint64_t above_mass, double want) SP_INLINE {
        const int hi = SP_BINS - 1 - 2 * tid;
        const int n2 = static_cast<int>(s.count[hi] + s.count[hi - 1]);
        const uint64_t q2 = weigh ? s.mass[hi] + s.mass[hi - 1] : 0;
        const int incl = wave_inclusive_scan_i32(n2, lane);
        const uint64_t incl_q = weigh ? wave_inclusive_shfl(q2, lane) : 0;
        if (lane == 63) {
          s.wave_count[wv] = incl;
          s.wave_mass[wv] = incl_q;
        }
        if (tid == 0) s.bin = 0;
        __syncthreads();
        uint32_t c = above + incl - n2, all = above;
        uint64_t q = above_mass + incl_q - q2;
#pragma unroll
        for (int x = 0; x < SP_WAVES; ++x) {
          c += x < wv ? s.wave_count[x] : 0;
          q += x < wv ? s.wave_mass[x] : 0;
          all += s.wave_count[x];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t n = s.count[hi - e];
          const uint64_t w = weigh ? s.mass[hi - e] : 0;
          const bool before = weigh ? (c == 0 || static_cast<double>(q) < want) : static_cast<double>(c) < want;
          const bool after = weigh ? static_cast<double>(q + w) >= want : static_cast<double>(c + n) >= want;
          if (n > 0 && before && (after || c + n == all)) {
            s.bin = hi - e;
            s.above = c;
            s.above_mass = q;
            s.key_count = n;
          }
          c += n;
          q += w;
        }
        __syncthreads();
      };
      // Narrows [lo, hi] to the border by count (want elements) or weight (a prefix of `want`); room:
      // elements equal to the first lo that count (the others were cut off before).
      auto narrow = [&](uint32_t lo, uint32_t hi, bool weigh, double want, int room, uint32_t& key, int& ties,
                        bool on_list) SP_INLINE {
        const uint32_t lo0 = lo;
        uint32_t above = 0;
        uint64_t above_mass = 0;
        bool have = on_list;       // the list holds all of [lo, hi]
        for (;;) {
          const uint32_t span = hi - lo;
          const int bits = span == 0 ? 0 : 32 - __builtin_clz(span), shift = bits > SP_BIN_BITS ? bits - SP_BIN_BITS : 0;
          if (have) {
            list_pass(lo, hi, shift, weigh);
          } else {
            row_pass(lo, hi, shift, weigh);
            have = list_fits();
            if (lo == key_low && hi == key_top) listed = have;
          }
          if (shift == 0 && lo == lo0) {
            if (tid == 0 && static_cast<uint32_t>(room) < s.count[0]) {
              s.mass[0] = s.mass[0] / s.count[0] * static_cast<uint32_t>(room);
              s.count[0] = room;
            }
            __syncthreads();
          }
          choose(weigh, above, above_mass, want);
          const uint32_t bin = s.bin;
          above = s.above;
          above_mass = s.above_mass;
          const uint32_t n = s.key_count;
          const double each = weigh ? static_cast<double>(s.mass[bin]) / n : 0.0;
          __syncthreads();
          lo += bin << shift;
          hi = min(hi, lo + ((1u << shift) - 1u));
          if (shift == 0) {
            key = lo;
            if (weigh) {
              const double need = (want - static_cast<double>(above_mass)) / each;
              ties = each > 0.0 && need < n ? max(1, static_cast<int>(ceil(need))) : static_cast<int>(n);
            } else {
              ties = min(static_cast<int>(want) - static_cast<int>(above), static_cast<int>(n));
            }
            return;
          }
        }
      };
      int room = 0x7fffffff;
      uint32_t from = key_low;
      if (a.top_k < V) {
        narrow(key_low, key_top, false, static_cast<double>(a.top_k), room, border, border_ties, false);
        from = border;
        room = border_ties;
      }
      if (a.top_p < 1.0) {
        // the weight of what top-k leaves (without top-k: of all), in fixed point
        uint64_t q = 0;
        auto add = [&](uint32_t k) SP_INLINE {
          if (k > from || (a.top_k >= V && k == from))
            q += static_cast<uint64_t>(pow2_or_0(key_power(k), s.table) * SP_FIXED + 0.5);
        };
        if (a.top_k >= V) from = f32_order_key(-3.402823466e38f);
        if (listed && a.top_k < V) {
          for (int e = lane; e < s.seg_n[wv]; e += kWave) add(s.key[wv][e]);
        } else {
          row.each(inf_row, [&](const float (&v)[VEC], int n, int) SP_INLINE {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
              if (e < n) add(f32_order_key(v[e]));
          });
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) q += __shfl_xor(q, o, kWave);
        if (lane == 0) s.wave_mass[wv] = q;
        __syncthreads();
        q = 0;
#pragma unroll
        for (int x = 0; x < SP_WAVES; ++x) q += s.wave_mass[x];
        __syncthreads();
        double mass = static_cast<double>(q);
        if (a.top_k < V) mass += static_cast<double>(static_cast<uint64_t>(pow2_or_0(key_power(border), s.table) * SP_FIXED + 0.5)) * border_ties;
        narrow(a.top_k < V ? border : key_low, key_top, true, a.top_p * mass, room, border, border_ties, listed);
      }
      if (a.top_k >= V && !(a.top_p < 1.0)) {       // min-p alone
        row_pass(key_low, key_top, 31, false);
        listed = list_fits();
        border = key_low - 1;
      }
    }
    // ---- 3. the draw
    auto kept = [&](uint32_t k, bool tie_kept) SP_INLINE {
      return (k > border || (k == border && tie_kept)) && k > f32_order_key(SP_NONE) && key_power(k) >= least;
    };
    float u = a.u[pos];
    u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
    // The part that u falls into, from the parts' weights in s.sum: s.part (-1: none has weight), and
    // what is left of u in s.target.
    auto choose_part = [&]() SP_INLINE {
      __syncthreads();
      if (tid == 0) {
        double all = 0.0, cum = 0.0, before = 0.0;
        for (int x = 0; x < SP_WAVES; ++x) all += s.sum[x];
        const double target = u * all;
        int part = -1;
        for (int x = 0; x < SP_WAVES; ++x) {
          if (s.sum[x] <= 0.0) continue;
          part = x;
          before = cum;
          cum += s.sum[x];
          if (target < cum) break;
        }
        s.part = part;
        s.target = target < cum ? target - before : __builtin_huge_val();
      }
      __syncthreads();
    };
    if (some && listed) {
      // wave w has segment w, lane l its entries 4 l ..
      const int n = s.seg_n[wv];
      uint32_t k[SP_LANE];
      int ties = 0;
#pragma unroll
      for (int e = 0; e < SP_LANE; ++e) {
        const int at = SP_LANE * lane + e;
        k[e] = at < n ? s.key[wv][at] : 0u;
        ties += k[e] == border ? 1 : 0;
      }
      int rank = wave_inclusive_scan_i32(ties, lane);
      if (lane == 63) s.ties[wv] = rank;
      __syncthreads();
      rank -= ties;
      for (int x = 0; x < wv; ++x) rank += s.ties[x];
      double w[SP_LANE], mine = 0.0;
#pragma unroll
      for (int e = 0; e < SP_LANE; ++e) {
        const bool tie = k[e] == border;
        w[e] = kept(k[e], tie && rank < border_ties) ? pow2_or_0(key_power(k[e]), s.table) : 0.0;
        rank += tie ? 1 : 0;
        mine += w[e];
      }
      const double incl = wave_inclusive_shfl(mine, lane);
      if (lane == 63) s.sum[wv] = incl;
      if (tid == 0) s.token = -1;
      choose_part();
      if (s.part == wv) {
        // the first entry past the target, else the last kept one
        const double target = s.target;
        double cum = incl - mine;
        int hit = -1, last = -1;
#pragma unroll
        for (int e = 0; e < SP_LANE; ++e) {
          cum += w[e];
          if (w[e] > 0.0) {
            last = SP_LANE * lane + e;
            if (hit < 0 && cum > target) hit = last;
          }
        }
        const uint64_t hits = __ballot(hit >= 0), any = __ballot(last >= 0);
        const int to = hits != 0 ? __shfl(hit, __builtin_ctzll(hits), kWave)
                                 : (any != 0 ? __shfl(last, 63 - __builtin_clzll(any), kWave) : -1);
        if (lane == 0 && to >= 0) s.token = s.index[wv][to];
      }
      __syncthreads();
      token = s.token >= 0 ? s.token : token;
    } else {
      if (some) {
        double sum = 0.0;
        int ties = 0;
        row.each(inf_row, [&](const float (&v)[VEC], int n, int) SP_INLINE {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const uint32_t k = f32_order_key(v[e]);
            if (e < n && kept(k, false)) sum += pow2_or_0(power(v[e]), s.table);
            ties += e < n && k == border ? 1 : 0;
          }
        });
        sum = wave_sum_f64(sum);
        ties = wave_sum_i32(ties);
        if (lane == 0) {
          s.sum[wv] = sum;
          s.ties[wv] = ties;
        }
        __syncthreads();
        if (tid == 0) {
          const double tie = kept(border, true) ? pow2_or_0(key_power(border), s.table) : 0.0;
          int left = border_ties;
          for (int x = 0; x < SP_WAVES; ++x) {
            const int n = min(s.ties[x], left);
            s.sum[x] += n * tie;
            s.ties[x] = n;        // the part's kept ties
            left -= n;
          }
        }
      }
      choose_part();
      const int part = s.part;
      if (part >= 0) {
        const double target = s.target;
        const int end = row.begin(part + 1), tie_room = some ? s.ties[part] : 0;
        double base = 0.0;
        int tie_base = 0;
        // 1024 elements at a time; the last kept token stands in where the order of the additions
        // leaves the target at the part's end
        for (int i0 = row.begin(part); i0 < end; i0 += SP_THREADS) {
          const int i = i0 + tid;
          const uint32_t k = i < end ? f32_order_key(row.at(i, inf_row)) : 0u;
          const bool tie = some && k == border;
          const int tie_incl = wave_inclusive_scan_i32(tie ? 1 : 0, lane);
          if (lane == 63) s.wave_count[wv] = tie_incl;
          __syncthreads();
          int rank = tie_base + tie_incl - 1, tie_all = 0;
#pragma unroll
          for (int x = 0; x < SP_WAVES; ++x) {
            rank += x < wv ? s.wave_count[x] : 0;
            tie_all += s.wave_count[x];
          }
          const bool keep = some ? kept(k, tie && rank < tie_room) : k > f32_order_key(SP_NONE);
          const double w = keep ? pow2_or_0(key_power(k), s.table) : 0.0;
          const double incl = wave_inclusive_shfl(w, lane);
          if (lane == 63) s.flat[wv] = incl;
          __syncthreads();
          double before = base, all = base;
#pragma unroll
          for (int x = 0; x < SP_WAVES; ++x) {
            before += x < wv ? s.flat[x] : 0.0;
            all += s.flat[x];
          }
          const uint64_t hits = __ballot(w > 0.0 && before + incl > target), any = __ballot(w > 0.0);
          if (lane == 0) {
            const int hit = hits != 0 ? i0 + kWave * wv + __builtin_ctzll(hits) : 0x7fffffff;
            const int last = any != 0 ? i0 + kWave * wv + 63 - __builtin_clzll(any) : -1;
            s.best[wv] = (static_cast<uint64_t>(static_cast<uint32_t>(hit)) << 32) | static_cast<uint32_t>(last);
          }
          __syncthreads();
          int hit = 0x7fffffff, last = -1;
#pragma unroll
          for (int x = 0; x < SP_WAVES; ++x) {
            hit = min(hit, static_cast<int>(s.best[x] >> 32));
            last = max(last, static_cast<int>(static_cast<uint32_t>(s.best[x])));
          }
          __syncthreads();
          if (last >= 0) token = last;
          if (hit != 0x7fffffff) {
            token = hit;
            break;
          }
          base = all;
          tie_base += tie_all;
        }
      }
    }
  }
  if (tid == 0) {
    a.tokens[pos] = token;
    if (a.conf != nullptr)
      a.conf[pos] = static_cast<float>(pow2_or_0((static_cast<double>(row.at(token, inf_row)) - m) * SP_LOG2E, s.table) / flat);
  }
}

}  // namespace

size_t sample_ws_bytes(int, int) { return 0; }

int launch_sample(const void* logits, int logits_type, const int32_t* rows, const int32_t* n_rows, int M, int V,
                  const float* u, const reflex_sample_params& p, int T, int32_t* tokens, float* conf, void*,
                  hipStream_t s) {
  SampleArgs a{rows, n_rows, M, V, T, u, p.temperature > 0.0f ? SP_LOG2E / static_cast<double>(p.temperature) : 0.0,
               p.min_p > 0.0f ? std::log2(static_cast<double>(p.min_p)) : -std::numeric_limits<double>::infinity(),
               p.top_k > 0 && p.top_k < V ? p.top_k : V, static_cast<double>(p.top_p), tokens, conf};
  if (logits_type == REFLEX_TYPE_F32)
    hipLaunchKernelGGL(sample_kernel<float>, dim3(M), dim3(SP_THREADS), 0, s, static_cast<const float*>(logits), a);
  else
    hipLaunchKernelGGL(sample_kernel<uint16_t>, dim3(M), dim3(SP_THREADS), 0, s, static_cast<const uint16_t*>(logits), a);
  return launch_status();
}

}  // namespace rfx
