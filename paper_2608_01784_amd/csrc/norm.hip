// What stands between a block's output and the next block's input (reflex_block_norm): the norm after the block,
// its gate, the scaled residual stream, the norm before the next block and that one's 8-bit rows.
//
//   y = the block's row, or sum_j alpha_j y_sorted[j] (+ the shared expert's row), in fp32
//   u = residual_scale x + gate (y r(y) w_post), rounded to the stream's type;  r(v) = 1 / sqrt(mean v^2 + eps)
//   n = bf16(u r(u) w_pre);  codes and scale of n (int8.h)
// One pass: W waves hold a row in registers, 16 numbers a lane, from the loads to the codes, and the weights over all
// the rows that a workgroup takes.  Sums of squares are taken in fp64 (a square of fp32 is exact there), so r is the
// rounded quotient in whatever order they are added (but for a row in some 10^8, next to a border), and each product and
// sum is rounded to fp32 by itself: results are those of the formulas, operation by operation, except for the experts'
// rows, which are added with fused multiply-adds in rank order as the combine does.  n is the norm of the stream as it is
// stored, so that a later call on x_out gives the same, and the codes are those of the bf16 n, so that the router and the
// experts read one input: that rounding moves a number by up to a quarter to a half of a code's step where it is within a
// factor of two of the row's largest (half a bf16 step is 2^(k-8) from 2^k on, a code's step a / 127), by half as much for
// each factor of two below, beside the half step that every code is off by.
//
// Bound by HBM.  16384 rows of 2048, bf16 stream, a gate for each sequence and both norms, 302 MB: 56 to 62 us (cards
// differ) or 4.9 to 5.4 TB/s, what a large copy moves; 8192 tokens of 1 to 12 experts' rows with a shared one, 352 MB: 67 us.
// What that took: 16 numbers a lane, not 32 (80 -> 75 us, joined rows 95 -> 82: more rows in flight), loads and stores that
// pass the caches by (80 -> 70), all of a row's loads ahead of its first sum, and weights loaded once a workgroup (together
// 59).  The fp64 sums cost 5 % of the given rows, 62 us to 59 with fp32 ones on one card, and nothing of the joined ones (67).
// Other widths, one gate, both norms, as many numbers, bf16 / fp32 stream, TB/s: given rows of 512 4.5 / 4.8, of 1024 5.4 /
// 5.0, of 4096 5.2 / 5.0, of 8192 5.0 / 5.0, of 16384 4.6 / 4.5; 1 to 8 joined rows of 512 4.3 / 4.8, of 4096 5.2 / 5.1, of
// 16384 4.6 / 4.6 (the instance for fp32 ones spills 8 registers).  Rows of 128 leave three quarters of a wave's lanes idle:
// 1.5 / 2.2.
#include "int8.h"

namespace rfx {
namespace {

constexpr int BN_VECS = 2;                          // groups of 8 numbers of a lane
constexpr int BN_COLS = kWave * 8 * BN_VECS;        // numbers of a wave: 1024
constexpr int BN_STEP = kWave * 8;                  // columns between a lane's groups
constexpr int BN_WAVES = 32;                        // waves a CU of the persistent grid

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

// 16 bytes that are read or written once (STREAM), or not.
template <bool STREAM>
__device__ __forceinline__ uint4 load16(const void* p) {
  if constexpr (STREAM) {
    const u32x4_t v = __builtin_nontemporal_load(static_cast<const u32x4_t*>(p));
    return make_uint4(v.x, v.y, v.z, v.w);
  } else {
    return *static_cast<const uint4*>(p);
  }
}
template <bool STREAM>
__device__ __forceinline__ void store16(void* p, uint4 v) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, static_cast<u32x4_t*>(p));
  else
    *static_cast<uint4*>(p) = v;
}

__device__ __forceinline__ void widen8(const uint4& b, float (&v)[8]) {
  const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(w[j] << 16);
    v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  }
}
__device__ __forceinline__ void floats8(const uint4& a, const uint4& b, float (&v)[8]) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

// The sequence of row i: how many of seq_offsets[1 .. B-1] are at most i, 64 probes at a time.
__device__ __forceinline__ int sequence_of(const int32_t* seq_offsets, int B, int i, int lane) {
  int lo = 1, n = B - 1;      // entries lo .. lo + n - 1 are undecided, those before are at most i
  while (n > 0) {
    const int step = (n + 63) / 64, at = lo + (lane + 1) * step - 1;
    const bool below = at < lo + n && seq_offsets[at] <= i;
    const int c = __popcll(__ballot(below));      // whole steps at most i
    lo += c * step;
    n = min(n - c * step, step - 1);
  }
  return min(lo, B) - 1;
}

template <int W, bool WIDE, bool PAIRS, bool STREAM>
__device__ __forceinline__ void block_norm_rows(const reflex_norm_args& a, uint64_t* shared) {
  constexpr int WAVES = W < 4 ? 4 : W, ROWS = WAVES / W;
  // Expert rows in flight: more take registers that hold a second workgroup (8192 tokens of 1 to 12 rows of 2048, 67.8 us
  // with 4, 72.4 with 8); rows of 16 waves have 128 registers.
  constexpr int BN_PAIRS = W < 16 ? 4 : 1;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int used = a.n_rows == nullptr ? a.T : min(a.n_rows[0], a.T), d = a.d;
  const int col = (wave % W) * BN_COLS + 8 * lane;
  bool in[BN_VECS];
#pragma unroll
  for (int i = 0; i < BN_VECS; ++i) in[i] = col + BN_STEP * i < d;
  // What the waves of a row add up or compare meets in one of two arrays in turn, so that one barrier is enough: a
  // wave that writes an array again has passed the other's barrier, which all waves reach after reading this one.
  int turn = 0;
  auto meet = [&](uint64_t mine, auto join) {
    if constexpr (W > 1) {
      uint64_t* const at = shared + WAVES * turn;
      turn ^= 1;
      if (lane == 0) at[wave] = mine;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < W; ++i) join(at[wave / W * W + i]);
    } else {
      join(mine);
    }
  };
  auto inverse_rms = [&](const float (&v)[BN_VECS][8]) {      // (columns past d hold zeros)
    double s[2] = {}, sum = 0.0;
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j % 2] = __builtin_fma(static_cast<double>(v[i][j]), static_cast<double>(v[i][j]), s[j % 2]);
    meet(__builtin_bit_cast(uint64_t, wave_sum64(s[0] + s[1])), [&](uint64_t x) { sum += __builtin_bit_cast(double, x); });
    return static_cast<float>(1.0 / __builtin_sqrt(sum / d + static_cast<double>(a.eps)));
  };
  // the weights of the lane's columns, for all rows
  float w_post[BN_VECS][8], w_pre[BN_VECS][8];
#pragma unroll
  for (int i = 0; i < BN_VECS; ++i) {
    const uint4* const post = reinterpret_cast<const uint4*>(a.w_post + col + BN_STEP * i);
    const uint4* const pre = reinterpret_cast<const uint4*>(a.w_pre + col + BN_STEP * i);
    if (a.w_post != nullptr && in[i]) floats8(post[0], post[1], w_post[i]);
    if (a.w_pre != nullptr && in[i]) floats8(pre[0], pre[1], w_pre[i]);
  }
  for (int first = static_cast<int>(blockIdx.x) * ROWS; first < used; first += static_cast<int>(gridDim.x) * ROWS) {
    const int row = first + wave / W;
    const bool on = row < used;
    const int r = on ? row : first;
    const size_t at = static_cast<size_t>(r) * d;
    // everything the row reads, ahead of what is computed from it
    uint4 xv[BN_VECS][WIDE ? 2 : 1], yv[BN_VECS], gv[BN_VECS];
    if (a.x != nullptr) {
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (in[i]) {
          const char* const p = static_cast<const char*>(a.x) + (at + col + BN_STEP * i) * (WIDE ? 4 : 2);
          xv[i][0] = load16<STREAM>(p);
          if constexpr (WIDE) xv[i][1] = load16<STREAM>(p + 16);
        }
    }
    const uint16_t* const y = PAIRS ? a.shared_y : a.y;
    if (y != nullptr) {
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (in[i]) yv[i] = load16<STREAM>(y + at + col + BN_STEP * i);
    }
    if (a.gate != nullptr) {
      int g = 0;
      if (a.seq_offsets != nullptr)
        g = sequence_of(a.seq_offsets, a.gate_rows, r, lane);
      else if (a.gate_rows > 1)
        g = r;
      const size_t from = static_cast<size_t>(g) * d;
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (in[i]) gv[i] = load16<false>(a.gate + from + col + BN_STEP * i);
    }
    float u[BN_VECS][8];
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) u[i][j] = 0.0f;
    if constexpr (PAIRS) {
      const int cap = a.pair_capacity;
      const int p0 = min(max(a.pair_offsets[r], 0), cap), p1 = min(max(a.pair_offsets[r + 1], p0), cap);
      for (int p = p0; p < p1; p += kWave) {      // lane j has pair p + j
        const int np = min(p1 - p, kWave);
        int prow = 0;
        float pw = 0.0f;
        if (lane < np) {
          prow = min(max(a.pair_to_sorted[p + lane], 0), cap - 1);
          pw = a.pair_weight[p + lane];
        }
        for (int q = 0; q < np; q += BN_PAIRS) {
          uint4 v[BN_PAIRS][BN_VECS];
#pragma unroll
          for (int k = 0; k < BN_PAIRS; ++k)
            if (q + k < np) {
              const size_t from = static_cast<size_t>(__builtin_amdgcn_readlane(prow, q + k)) * d;
#pragma unroll
              for (int i = 0; i < BN_VECS; ++i)
                if (in[i]) v[k][i] = load16<STREAM>(a.y_sorted + from + col + BN_STEP * i);
            }
#pragma unroll
          for (int k = 0; k < BN_PAIRS; ++k)
            if (q + k < np) {
              const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(pw), q + k));
#pragma unroll
              for (int i = 0; i < BN_VECS; ++i)
                if (in[i]) {
                  float e[8];
                  widen8(v[k][i], e);
#pragma unroll
                  for (int j = 0; j < 8; ++j) u[i][j] = __builtin_fmaf(w, e[j], u[i][j]);
                }
            }
        }
      }
    }
    if (y != nullptr) {
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (in[i]) {
          float e[8];
          widen8(yv[i], e);
#pragma unroll
          for (int j = 0; j < 8; ++j) u[i][j] = PAIRS ? add_rn(u[i][j], e[j]) : e[j];
        }
    }
    if (a.w_post != nullptr) {
      const float f = inverse_rms(u);
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (in[i]) {
#pragma unroll
          for (int j = 0; j < 8; ++j) u[i][j] = mul_rn(mul_rn(u[i][j], f), w_post[i][j]);
        }
    }
    if (a.gate != nullptr) {
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (in[i]) {
          float g[8];
          widen8(gv[i], g);
#pragma unroll
          for (int j = 0; j < 8; ++j) u[i][j] = mul_rn(g[j], u[i][j]);
        }
    }
    if (a.x != nullptr) {
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (in[i]) {
          float x[8];
          if constexpr (WIDE)
            floats8(xv[i][0], xv[i][1], x);
          else
            widen8(xv[i][0], x);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float s = mul_rn(a.residual_scale, x[j]);
            u[i][j] = PAIRS || a.y != nullptr ? add_rn(s, u[i][j]) : s;
          }
        }
    }
    // the stream's new row, and from here on its rounded numbers
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i) {
      if constexpr (WIDE) {
        if (on && a.x_out != nullptr && in[i]) {
          uint4* const to = reinterpret_cast<uint4*>(static_cast<float*>(a.x_out) + at + col + BN_STEP * i);
          uint32_t b[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) b[j] = __float_as_uint(u[i][j]);
          store16<STREAM>(to, make_uint4(b[0], b[1], b[2], b[3]));
          store16<STREAM>(to + 1, make_uint4(b[4], b[5], b[6], b[7]));
        }
      } else {
        const uint4 b = pack8(u[i]);
        if (on && a.x_out != nullptr && in[i])
          store16<STREAM>(static_cast<uint16_t*>(a.x_out) + at + col + BN_STEP * i, b);
        widen8(b, u[i]);
      }
    }
    if (a.w_pre == nullptr) continue;      // (for all rows alike)
    const float f = inverse_rms(u);
    uint4 n[BN_VECS];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i) {
      n[i] = make_uint4(0, 0, 0, 0);
      if (in[i]) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = mul_rn(mul_rn(u[i][j], f), w_pre[i][j]);
        n[i] = pack8(v);
        most = max(most, i8_amax8(n[i]));
        if (on && a.n_out != nullptr) store16<STREAM>(a.n_out + at + col + BN_STEP * i, n[i]);
      }
    }
    if (a.q_out == nullptr) continue;
    const uint32_t mine = wave_max_u32(most);
    meet(mine, [&](uint64_t x) { most = max(most, static_cast<uint32_t>(x)); });
    const float factor = i8_factor(most);
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i)
      if (on && in[i]) {
        const u32x2_t c = {i8_pack4(n[i].x, n[i].y, factor), i8_pack4(n[i].z, n[i].w, factor)};
        u32x2_t* const to = reinterpret_cast<u32x2_t*>(a.q_out + at + col + BN_STEP * i);
        if constexpr (STREAM)
          __builtin_nontemporal_store(c, to);
        else
          *to = c;
      }
    if (on && lane == 0 && wave % W == 0) a.q_scale[row] = i8_scale(most);
  }
}

// Rows that are read and written once pass the caches by where there are more of them than the Infinity Cache holds.
template <int W, bool WIDE, bool PAIRS>
__global__ __launch_bounds__(kWave* (W < 4 ? 4 : W)) void block_norm_kernel(reflex_norm_args a) {
  __shared__ uint64_t shared[2 * (W < 4 ? 4 : W)];
  size_t row = 2 * (a.n_out != nullptr) + (a.q_out != nullptr) + (WIDE ? 4 : 2) * ((a.x != nullptr) + (a.x_out != nullptr)) +
               2 * (a.y != nullptr || a.shared_y != nullptr);
  row *= static_cast<size_t>(a.T);
  if (PAIRS) row += 2 * static_cast<size_t>(min(max(a.pair_offsets[a.T], 0), a.pair_capacity));
  if (row * a.d > kStreamBytes)
    block_norm_rows<W, WIDE, PAIRS, true>(a, shared);
  else
    block_norm_rows<W, WIDE, PAIRS, false>(a, shared);
}

template <int W, bool WIDE, bool PAIRS>
int launch_as(const reflex_norm_args& a, hipStream_t s) {
  constexpr int WAVES = W < 4 ? 4 : W, ROWS = WAVES / W;
  const int blocks = (a.T + ROWS - 1) / ROWS, most = device_cus() * BN_WAVES / WAVES;
  hipLaunchKernelGGL((block_norm_kernel<W, WIDE, PAIRS>), dim3(blocks < most ? blocks : most), dim3(kWave * WAVES), 0, s, a);
  return launch_status();
}

template <int W>
int launch_of(const reflex_norm_args& a, hipStream_t s) {
  const bool wide = a.stream_type == REFLEX_TYPE_F32, pairs = a.y_sorted != nullptr;
  if (wide) return pairs ? launch_as<W, true, true>(a, s) : launch_as<W, true, false>(a, s);
  return pairs ? launch_as<W, false, true>(a, s) : launch_as<W, false, false>(a, s);
}

}  // namespace

int launch_block_norm(const reflex_norm_args& a, hipStream_t s) {
  if (a.d <= BN_COLS) return launch_of<1>(a, s);
  if (a.d <= 2 * BN_COLS) return launch_of<2>(a, s);
  if (a.d <= 4 * BN_COLS) return launch_of<4>(a, s);
  if (a.d <= 8 * BN_COLS) return launch_of<8>(a, s);
  return launch_of<16>(a, s);
}

}  // namespace rfx
