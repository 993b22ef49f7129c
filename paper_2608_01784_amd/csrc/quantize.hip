// bf16 rows and weights to 8 bits with a power-of-two scale for each block of 128 (fp8.h).
//
// Both kernels make one pass over the data, a block in registers between the maximum and the
// rounding, and are bound by HBM (3 bytes a number): 8192 rows of 2048, 50 MB, 11.6 us or 4.3 TB/s,
// where a large copy moves 5.1.
//  - rows: a wave holds four blocks of a row (512 columns, 16 lanes and 16 bytes a lane per
//    block), so their four scale bytes leave as one dword;
//  - weights: a workgroup holds a 128 x 128 block, eight rows of 8 numbers in each thread (8 experts
//    of 4096 x 2048, 201 MB, 33 us).
#include "fp8.h"

namespace rfx {
namespace {

constexpr int QR_THREADS = 256, QR_WAVES = QR_THREADS / kWave;

// Largest finite magnitude of eight bf16 numbers, as fp32 bits.
__device__ __forceinline__ uint32_t amax8(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = (w[i] << 16) & 0x7fffffffu, hi = w[i] & 0x7fff0000u;
    m = max(m, lo < 0x7f800000u ? lo : 0u);
    m = max(m, hi < 0x7f800000u ? hi : 0u);
  }
  return m;
}

// The codes of eight bf16 numbers; inv: one over their scale.
__device__ __forceinline__ uint2 codes8(const uint4& v, float inv) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t q[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t b[4] = {w[2 * i] << 16, w[2 * i] & 0xffff0000u, w[2 * i + 1] << 16, w[2 * i + 1] & 0xffff0000u};
    q[i] = f8_pack4(__uint_as_float(b[0]) * inv, __uint_as_float(b[1]) * inv, __uint_as_float(b[2]) * inv,
                    __uint_as_float(b[3]) * inv);
#pragma unroll
    for (int j = 0; j < 4; ++j)       // infinities and NaN: the one NaN code
      if ((b[j] & 0x7fffffffu) >= 0x7f800000u) q[i] = (q[i] & ~(0xffu << (8 * j))) | (0x7fu << (8 * j));
  }
  return make_uint2(q[0], q[1]);
}

// Maximum over the 16 lanes of a DPP row.
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
  v = max(v, dpp_u32<kDppXor1>(v));
  v = max(v, dpp_u32<kDppXor2>(v));
  v = max(v, dpp_u32<kDppHalfMirror>(v));
  return max(v, dpp_u32<kDppMirror>(v));
}

__global__ __launch_bounds__(QR_THREADS) void quantize_rows_kernel(
    const uint16_t* __restrict__ x, const int32_t* __restrict__ rows, const int32_t* __restrict__ n_rows,
    int x_rows, int M, int K, int groups, uint8_t* __restrict__ q, uint32_t* __restrict__ scale) {
  const int lane = threadIdx.x & 63;
  const size_t item = (static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x) * QR_WAVES + (threadIdx.x >> 6);
  const int row = static_cast<int>(item / groups), group = static_cast<int>(item % groups);
  const int used = n_rows == nullptr ? M : min(n_rows[0], M);
  if (row >= used) return;
  const int src = rows == nullptr ? row : rows[row];
  const int col = 512 * group + 8 * lane;
  uint4 v = make_uint4(0, 0, 0, 0);
  if (col < K && src >= 0 && src < x_rows)
    v = *reinterpret_cast<const uint4*>(x + static_cast<size_t>(src) * K + col);
  const uint32_t byte = f8_scale_byte(row_max_u32(amax8(v)));
  if (col < K) *reinterpret_cast<uint2*>(q + static_cast<size_t>(row) * K + col) = codes8(v, f8_inverse(byte));
  // the group's four bytes; K is a multiple of 128, so a block is inside K or past it
  const uint32_t mine = col < K ? byte : 0u;
  const uint32_t b0 = __builtin_amdgcn_readlane(mine, 0), b1 = __builtin_amdgcn_readlane(mine, 16);
  const uint32_t b2 = __builtin_amdgcn_readlane(mine, 32), b3 = __builtin_amdgcn_readlane(mine, 48);
  if (lane == 0) scale[static_cast<size_t>(group) * M + row] = b0 | (b1 << 8) | (b2 << 16) | (b3 << 24);
}

__global__ __launch_bounds__(QR_THREADS) void quantize_weight_kernel(const uint16_t* __restrict__ w, int N, int K,
                                                                     int n_blocks, int groups, uint8_t* __restrict__ q,
                                                                     uint8_t* __restrict__ scale) {
  __shared__ uint32_t s_max[QR_WAVES];
  const int tid = threadIdx.x, k_blocks = K / F8_BLOCK;
  const int kb = blockIdx.x % k_blocks, nb = blockIdx.x / k_blocks % n_blocks, e = blockIdx.x / k_blocks / n_blocks;
  const int r0 = F8_BLOCK * nb + tid / 16, col = F8_BLOCK * kb + 8 * (tid % 16);
  const size_t base = (static_cast<size_t>(e) * N + r0) * K + col;
  uint4 v[8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = make_uint4(0, 0, 0, 0);
    if (r0 + 16 * i < N) v[i] = *reinterpret_cast<const uint4*>(w + base + static_cast<size_t>(16 * i) * K);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, amax8(v[i]));
  m = wave_max_u32(m);
  if ((tid & 63) == 0) s_max[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < QR_WAVES; ++x) m = max(m, s_max[x]);
  const uint32_t byte = f8_scale_byte(m);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (r0 + 16 * i < N)
      *reinterpret_cast<uint2*>(q + base + static_cast<size_t>(16 * i) * K) = codes8(v[i], f8_inverse(byte));
  // the block's byte, and the padding after the last block of a row of blocks
  uint8_t* out = scale + (static_cast<size_t>(e) * n_blocks + nb) * 4 * groups;
  if (tid == 0) out[kb] = static_cast<uint8_t>(byte);
  if (kb == k_blocks - 1 && tid > kb && tid < 4 * groups) out[tid] = 0;
}

}  // namespace

int launch_quantize_rows(const uint16_t* x, const int32_t* rows, const int32_t* n_rows, int x_rows, int M, int K,
                         uint8_t* q, uint8_t* scale, hipStream_t s) {
  const int groups = f8_groups(K);
  // (a dimension of a grid has less than 2^32 threads: 2^20 workgroups in x, the others in y)
  const size_t blocks = (static_cast<size_t>(M) * groups + QR_WAVES - 1) / QR_WAVES, x_blocks = size_t(1) << 20;
  const dim3 grid(static_cast<unsigned>(blocks < x_blocks ? blocks : x_blocks),
                  static_cast<unsigned>((blocks + x_blocks - 1) / x_blocks));
  hipLaunchKernelGGL(quantize_rows_kernel, grid,
                     dim3(QR_THREADS), 0, s, x, rows, n_rows, x_rows, M, K, groups, q,
                     reinterpret_cast<uint32_t*>(scale));
  return launch_status();
}

int launch_quantize_weight(const uint16_t* w, int E, int N, int K, uint8_t* q, uint8_t* scale, hipStream_t s) {
  const int n_blocks = (N + F8_BLOCK - 1) / F8_BLOCK;
  hipLaunchKernelGGL(quantize_weight_kernel, dim3(static_cast<unsigned>(E) * n_blocks * (K / F8_BLOCK)),
                     dim3(QR_THREADS), 0, s, w, N, K, n_blocks, f8_groups(K), q, scale);
  return launch_status();
}

}  // namespace rfx
