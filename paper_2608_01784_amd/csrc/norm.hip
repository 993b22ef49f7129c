// What stands between a block's output and the next block's input (reflex_block_norm): the norm after the block,
// its gate, the scaled residual stream, the norm before the next block and that one's 8-bit rows.
//
//   y = the block's row, or sum_j alpha_j y_sorted[j] (+ the shared expert's row), in fp32
//   u = residual_scale x + gate (y r(y) w_post), rounded to the stream's type;  r(v) = 1 / sqrt(mean v^2 + eps)
//   n = bf16(u r(u) w_pre);  codes and scale of n (int8.h)
// One pass: W waves hold a row in registers, 32 numbers a lane, from the loads to the codes.  Sums of squares are
// taken in fp64 (a square of fp32 is exact there), so r is the rounded quotient whatever the order, and each product
// and sum is rounded to fp32 by itself: results do not depend on W, and are those of the formulas, operation by
// operation, except for the experts' rows, which are added with fused multiply-adds in rank order as the combine does.
#include "int8.h"

namespace rfx {
namespace {

constexpr int BN_VECS = 4;                          // groups of 8 numbers of a lane
constexpr int BN_COLS = kWave * 8 * BN_VECS;        // numbers of a wave: 2048
constexpr int BN_PAIRS = 4;                         // expert rows in flight

// 8 numbers of a row of fp32 or bf16.
template <bool WIDE>
__device__ __forceinline__ void load8(const void* base, size_t at, float* v) {
  if constexpr (WIDE) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
    const float4 a = p[0], b = p[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
}

__device__ __forceinline__ uint4 pack8(const float* v) {
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

template <int W, bool WIDE, bool PAIRS>
__global__ __launch_bounds__(kWave* (W < 4 ? 4 : W)) void block_norm_kernel(reflex_norm_args a) {
  constexpr int WAVES = W < 4 ? 4 : W, ROWS = WAVES / W;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int used = a.n_rows == nullptr ? a.T : min(a.n_rows[0], a.T), d = a.d;
  const int col = (wave % W) * BN_COLS + 8 * lane;
  // a row's sum and maximum over its waves
  auto row_sum = [&](double v) {
    v = wave_sum64(v);
    if constexpr (W > 1) {
      __shared__ double s_sum[WAVES];
      __syncthreads();      // the last row's are read
      if (lane == 0) s_sum[wave] = v;
      __syncthreads();
      v = 0.0;
#pragma unroll
      for (int i = 0; i < W; ++i) v += s_sum[wave / W * W + i];
    }
    return v;
  };
  auto row_max = [&](uint32_t v) {
    v = wave_max_u32(v);
    if constexpr (W > 1) {
      __shared__ uint32_t s_max[WAVES];
      __syncthreads();
      if (lane == 0) s_max[wave] = v;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < W; ++i) v = max(v, s_max[wave / W * W + i]);
    }
    return v;
  };
  auto inverse_rms = [&](const float (&v)[BN_VECS][8]) {      // (columns past d hold zeros)
    double s[2] = {};
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j % 2] = __builtin_fma(static_cast<double>(v[i][j]), static_cast<double>(v[i][j]), s[j % 2]);
    return static_cast<float>(1.0 / __builtin_sqrt(row_sum(s[0] + s[1]) / d + static_cast<double>(a.eps)));
  };
  for (int first = static_cast<int>(blockIdx.x) * ROWS; first < used; first += static_cast<int>(gridDim.x) * ROWS) {
    const int row = first + wave / W;
    const bool on = row < used;
    const size_t at = static_cast<size_t>(on ? row : first) * d;
    float u[BN_VECS][8], x[BN_VECS][8];
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) u[i][j] = x[i][j] = 0.0f;
    if (a.x != nullptr) {
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (col + 512 * i < d) load8<WIDE>(a.x, at + col + 512 * i, x[i]);
    }
    if constexpr (PAIRS) {
      const int r = on ? row : first, cap = a.pair_capacity;
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
                if (col + 512 * i < d) v[k][i] = *reinterpret_cast<const uint4*>(a.y_sorted + from + col + 512 * i);
            }
#pragma unroll
          for (int k = 0; k < BN_PAIRS; ++k)
            if (q + k < np) {
              const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(pw), q + k));
#pragma unroll
              for (int i = 0; i < BN_VECS; ++i)
                if (col + 512 * i < d) {
                  const uint32_t b[4] = {v[k][i].x, v[k][i].y, v[k][i].z, v[k][i].w};
#pragma unroll
                  for (int j = 0; j < 4; ++j) {
                    u[i][2 * j] = __builtin_fmaf(w, __uint_as_float(b[j] << 16), u[i][2 * j]);
                    u[i][2 * j + 1] = __builtin_fmaf(w, __uint_as_float(b[j] & 0xffff0000u), u[i][2 * j + 1]);
                  }
                }
            }
        }
      }
      if (a.shared_y != nullptr) {
#pragma unroll
        for (int i = 0; i < BN_VECS; ++i)
          if (col + 512 * i < d) {
            float v[8];
            load8<false>(a.shared_y, at + col + 512 * i, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[i][j] = add_rn(u[i][j], v[j]);
          }
      }
    } else if (a.y != nullptr) {
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (col + 512 * i < d) load8<false>(a.y, at + col + 512 * i, u[i]);
    }
    if (a.w_post != nullptr) {
      const float r = inverse_rms(u);
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (col + 512 * i < d) {
          float w[8];
          load8<true>(a.w_post, col + 512 * i, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) u[i][j] = mul_rn(mul_rn(u[i][j], r), w[j]);
        }
    }
    if (a.gate != nullptr) {
      int g = 0;
      if (a.seq_offsets != nullptr)
        g = sequence_of(a.seq_offsets, a.gate_rows, on ? row : first, lane);
      else if (a.gate_rows > 1)
        g = on ? row : first;
      const size_t from = static_cast<size_t>(g) * d;
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
        if (col + 512 * i < d) {
          float w[8];
          load8<false>(a.gate, from + col + 512 * i, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) u[i][j] = mul_rn(w[j], u[i][j]);
        }
    }
    if (a.x != nullptr) {
#pragma unroll
      for (int i = 0; i < BN_VECS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float s = mul_rn(a.residual_scale, x[i][j]);
          u[i][j] = PAIRS || a.y != nullptr ? add_rn(s, u[i][j]) : s;
        }
    }
    // the stream's new row, and from here on its rounded numbers
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i) {
      if constexpr (WIDE) {
        if (on && a.x_out != nullptr && col + 512 * i < d) {
          float4* const to = reinterpret_cast<float4*>(static_cast<float*>(a.x_out) + at + col + 512 * i);
          to[0] = make_float4(u[i][0], u[i][1], u[i][2], u[i][3]);
          to[1] = make_float4(u[i][4], u[i][5], u[i][6], u[i][7]);
        }
      } else {
        const uint4 b = pack8(u[i]);
        if (on && a.x_out != nullptr && col + 512 * i < d)
          *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.x_out) + at + col + 512 * i) = b;
        const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u[i][2 * j] = __uint_as_float(w[j] << 16);
          u[i][2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
      }
    }
    if (a.w_pre == nullptr) continue;      // (for all rows alike)
    const float r = inverse_rms(u);
    uint4 n[BN_VECS];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i) {
      n[i] = make_uint4(0, 0, 0, 0);
      if (col + 512 * i < d) {
        float w[8];
        load8<true>(a.w_pre, col + 512 * i, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = mul_rn(mul_rn(u[i][j], r), w[j]);
        n[i] = pack8(w);
        most = max(most, i8_amax8(n[i]));
        if (on && a.n_out != nullptr) *reinterpret_cast<uint4*>(a.n_out + at + col + 512 * i) = n[i];
      }
    }
    if (a.q_out == nullptr) continue;
    most = row_max(most);
    const float factor = i8_factor(most);
#pragma unroll
    for (int i = 0; i < BN_VECS; ++i)
      if (on && col + 512 * i < d)
        *reinterpret_cast<uint2*>(a.q_out + at + col + 512 * i) =
            make_uint2(i8_pack4(n[i].x, n[i].y, factor), i8_pack4(n[i].z, n[i].w, factor));
    if (on && lane == 0 && wave % W == 0) a.q_scale[row] = i8_scale(most);
  }
}

template <int W, bool WIDE, bool PAIRS>
int launch_as(const reflex_norm_args& a, hipStream_t s) {
  constexpr int WAVES = W < 4 ? 4 : W, ROWS = WAVES / W;
  const int blocks = (a.T + ROWS - 1) / ROWS, most = device_cus() * 16 / WAVES * 4;
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
  return launch_of<8>(a, s);
}

}  // namespace rfx
