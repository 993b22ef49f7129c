// bf16 rows and weights to 8-bit integers with a scale for each row (int8.h).
//
// One pass over the data, a row in registers between the maximum and the rounding: W waves hold a row, 32 numbers
// (four 16-byte loads) a lane, and where W > 1 their maxima meet in LDS.  Bound by HBM (3 bytes a number).
#include "int8.h"

namespace rfx {
namespace {

constexpr int QI_VECS = 4;                           // 16-byte loads of a lane
constexpr int QI_COLS = kWave * 8 * QI_VECS;         // numbers of a wave: 2048

template <int W>
__global__ __launch_bounds__(kWave* (W < 4 ? 4 : W)) void quantize_i8_kernel(
    const uint16_t* __restrict__ x, const int32_t* __restrict__ rows, const int32_t* __restrict__ n_rows, size_t x_rows,
    size_t M, size_t extra, int K, int8_t* __restrict__ q, float* __restrict__ scale) {
  constexpr int WAVES = W < 4 ? 4 : W;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t block = static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x;
  const size_t row = block * (WAVES / W) + wave / W;
  const size_t used = n_rows == nullptr ? M : static_cast<size_t>(max(n_rows[0], 0));
  const bool on = row < M && (row < used || row >= extra);
  size_t src = row;
  bool inside = on;
  if (on && rows != nullptr) {
    const int r = rows[row];
    inside = r >= 0 && static_cast<size_t>(r) < x_rows;
    src = static_cast<size_t>(r);
  }
  uint4 v[QI_VECS];
  uint32_t m = 0;
  const int col = (wave % W) * QI_COLS + 8 * lane;
#pragma unroll
  for (int i = 0; i < QI_VECS; ++i) {
    v[i] = make_uint4(0, 0, 0, 0);
    const int c = col + i * kWave * 8;
    if (inside && c < K) v[i] = *reinterpret_cast<const uint4*>(x + src * K + c);
  }
#pragma unroll
  for (int i = 0; i < QI_VECS; ++i) m = max(m, i8_amax8(v[i]));
  m = wave_max_u32(m);
  if constexpr (W > 1) {
    __shared__ uint32_t s_max[WAVES];
    if (lane == 0) s_max[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) m = max(m, s_max[wave / W * W + i]);
  }
  if (!on) return;
  const float factor = i8_factor(m);
#pragma unroll
  for (int i = 0; i < QI_VECS; ++i) {
    const int c = col + i * kWave * 8;
    if (c < K)
      *reinterpret_cast<uint2*>(q + row * K + c) =
          make_uint2(i8_pack4(v[i].x, v[i].y, factor), i8_pack4(v[i].z, v[i].w, factor));
  }
  if (lane == 0 && wave % W == 0) scale[row] = i8_scale(m);
}

template <int W>
int launch_as(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, size_t x_rows, size_t M, size_t extra, int K,
              int8_t* q, float* scale, hipStream_t s) {
  constexpr int WAVES = W < 4 ? 4 : W;
  // (a dimension of a grid has less than 2^32 threads)
  const size_t blocks = (M + WAVES / W - 1) / (WAVES / W), x_blocks = size_t(1) << 20;
  const dim3 grid(static_cast<unsigned>(blocks < x_blocks ? blocks : x_blocks),
                  static_cast<unsigned>((blocks + x_blocks - 1) / x_blocks));
  hipLaunchKernelGGL(quantize_i8_kernel<W>, grid, dim3(kWave * WAVES), 0, s, x, rows, n_rows, x_rows, M, extra, K, q, scale);
  return launch_status();
}

}  // namespace

int launch_quantize_i8(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, size_t x_rows, size_t M,
                       size_t extra, int K, int8_t* q, float* scale, hipStream_t s) {
  if (K <= QI_COLS) return launch_as<1>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
  if (K <= 2 * QI_COLS) return launch_as<2>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
  if (K <= 4 * QI_COLS) return launch_as<4>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
  return launch_as<8>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
}

}  // namespace rfx
