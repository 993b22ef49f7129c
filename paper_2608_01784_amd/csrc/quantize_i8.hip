// bf16 rows and weights to 8-bit integers with a scale for each row (int8.h).
//
// One pass over the data, a row in registers between the maximum and the rounding.  A lane has four 16-byte loads in
// flight: W waves hold a row of more than 2048 numbers and their maxima meet in LDS, a wave holds R rows of up to
// 2048 / R.  Bound by HBM (3 bytes a number): 16384 rows of 2048, 101 MB, 16 to 18 us or 5.6 to 6.3 TB/s (a large copy
// moves 5.1); 65536 rows of 512 with four rows a wave 20.6 us, with one 23.6.
#include "int8.h"

namespace rfx {
namespace {

constexpr int QI_VECS = 4;                           // 16-byte loads of a lane
constexpr int QI_COLS = kWave * 8 * QI_VECS;         // numbers of a wave: 2048

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

// STREAM: more rows than the Infinity Cache holds, which pass the caches by.
template <int W, int R, bool STREAM>
__global__ __launch_bounds__(kWave* (W < 4 ? 4 : W)) void quantize_i8_kernel(
    const uint16_t* __restrict__ x, const int32_t* __restrict__ rows, const int32_t* __restrict__ n_rows, size_t x_rows,
    size_t M, size_t extra, int K, int8_t* __restrict__ q, float* __restrict__ scale) {
  static_assert(W == 1 || R == 1, "rows of several waves, or waves of several rows");
  constexpr int WAVES = W < 4 ? 4 : W, VECS = QI_VECS / R;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t block = static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x;
  const size_t row0 = (block * (WAVES / W) + wave / W) * R;
  const size_t used = n_rows == nullptr ? M : static_cast<size_t>(max(n_rows[0], 0));
  const int col = (wave % W) * QI_COLS + 8 * lane;
  bool on[R];
  uint4 v[R][VECS];
  uint32_t m[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const size_t row = row0 + r;
    on[r] = row < M && (row < used || row >= extra);
    size_t src = row;
    bool inside = on[r];
    if (on[r] && rows != nullptr) {
      const int i = rows[row];
      inside = i >= 0 && static_cast<size_t>(i) < x_rows;
      src = static_cast<size_t>(i);
    }
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      v[r][i] = make_uint4(0, 0, 0, 0);
      const int c = col + i * kWave * 8;
      if (inside && c < K) {
        const u32x4_t* const p = reinterpret_cast<const u32x4_t*>(x + src * K + c);
        const u32x4_t b = STREAM ? __builtin_nontemporal_load(p) : *p;
        v[r][i] = make_uint4(b.x, b.y, b.z, b.w);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = 0;
#pragma unroll
    for (int i = 0; i < VECS; ++i) m[r] = max(m[r], i8_amax8(v[r][i]));
    m[r] = wave_max_u32(m[r]);
  }
  if constexpr (W > 1) {
    __shared__ uint32_t s_max[WAVES];
    if (lane == 0) s_max[wave] = m[0];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) m[0] = max(m[0], s_max[wave / W * W + i]);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (!on[r]) continue;
    const size_t row = row0 + r;
    const float factor = i8_factor(m[r]);
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int c = col + i * kWave * 8;
      if (c < K) {
        const u32x2_t b = {i8_pack4(v[r][i].x, v[r][i].y, factor), i8_pack4(v[r][i].z, v[r][i].w, factor)};
        u32x2_t* const to = reinterpret_cast<u32x2_t*>(q + row * K + c);
        if constexpr (STREAM)
          __builtin_nontemporal_store(b, to);
        else
          *to = b;
      }
    }
    if (lane == 0 && wave % W == 0) scale[row] = i8_scale(m[r]);
  }
}

template <int W, int R>
int launch_as(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, size_t x_rows, size_t M, size_t extra, int K,
              int8_t* q, float* scale, hipStream_t s) {
  constexpr int WAVES = W < 4 ? 4 : W, ROWS = WAVES / W * R;
  // (a dimension of a grid has less than 2^32 threads)
  const size_t blocks = (M + ROWS - 1) / ROWS, x_blocks = size_t(1) << 20;
  const dim3 grid(static_cast<unsigned>(blocks < x_blocks ? blocks : x_blocks),
                  static_cast<unsigned>((blocks + x_blocks - 1) / x_blocks));
  auto* kernel = 3 * M * K > kStreamBytes ? &quantize_i8_kernel<W, R, true> : &quantize_i8_kernel<W, R, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kWave * WAVES), 0, s, x, rows, n_rows, x_rows, M, extra, K, q, scale);
  return launch_status();
}

}  // namespace

int launch_quantize_i8(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, size_t x_rows, size_t M,
                       size_t extra, int K, int8_t* q, float* scale, hipStream_t s) {
  if (K <= QI_COLS / 4) return launch_as<1, 4>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
  if (K <= QI_COLS / 2) return launch_as<1, 2>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
  if (K <= QI_COLS) return launch_as<1, 1>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
  if (K <= 2 * QI_COLS) return launch_as<2, 1>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
  if (K <= 4 * QI_COLS) return launch_as<4, 1>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
  return launch_as<8, 1>(x, rows, n_rows, x_rows, M, extra, K, q, scale, s);
}

}  // namespace rfx
