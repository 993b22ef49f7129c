// SwiGLU experts and plain products on 8-bit integer rows and weights (int8.h): the launches of gemm8_impl.h.
//
// A row of the activation has one scale, so its codes wait for all of its columns: the up product leaves bf16 rows,
// which quantize_i8_kernel rounds to 8 bits ahead of the down product (53000 rows of 1024: 32 of 454 us; 26 rows an expert
// on 256 experts of width 512: 5 of 170).  bf16 ahead of the rounding: it moves a number by up to a quarter to a half of an
// 8-bit step where it is within a factor of two of the row's largest, by half as much for each factor of two below, beside
// the half step that every code is off by; fp32 rows would be twice the bytes.  (The kernels for few rows save the launch:
// there a workgroup reads a tile's whole rows anyway.)
#include "gemm8_impl.h"

namespace rfx {
namespace {

const uint8_t* codes(const int8_t* p) { return reinterpret_cast<const uint8_t*>(p); }
const uint32_t* bits(const float* p) { return reinterpret_cast<const uint32_t*>(p); }

// ---- experts of few rows ----------------------------------------------------------------------------------
// With a few rows an expert the time of a product is a chain of latencies and its weights' stream, which the tiles of
// gemm8(), 512 KB of weights each, share out unevenly (18 experts with a row: 144 tiles for 256 CUs).  Here a workgroup
// has 32 rows x 32 columns of gate and of up (UP) or x 64 columns (DOWN), 128 KB of weights at K = 2048, and its waves take
// every FEW_W-th slice of 128 of K each, straight from global memory into the MFMAs' registers, a slice ahead of the
// products (two took the registers that hold a second workgroup, 31 -> 37 us for the 4 tokens below); their sums meet in
// LDS.  The first weights are asked for ahead of what the rows wait for (31 -> 29 us).  DOWN reads the activation's bf16
// rows and rounds them to 8 bits itself, a row's maximum over the waves first,
// which saves a launch.  Sums of integers are exact, so the results are those of the tiles.

// 16 codes of 32 bytes of bf16.
__device__ __forceinline__ i32x4_t codes16(const uint4& a, const uint4& b, float factor) {
  return i32x4_t{static_cast<int>(i8_pack4(a.x, a.y, factor)), static_cast<int>(i8_pack4(a.z, a.w, factor)),
                 static_cast<int>(i8_pack4(b.x, b.y, factor)), static_cast<int>(i8_pack4(b.z, b.w, factor))};
}

template <Mode MODE, int FEW_W>
__global__ __launch_bounds__(64 * FEW_W) void int8_few_kernel(Args8 a, const uint16_t* __restrict__ act) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem8[];
  int* const sums = reinterpret_cast<int*>(smem8);      // [W][2][16][SLIM_PITCH]
  __shared__ uint32_t s_max[FEW_W][32];
  __shared__ float s_scale[32];
  constexpr int BN = MODE == UP ? 32 : 64;
  const int K = a.K, N = a.N, E = a.E, nk = K / G8_BK, n_tiles = (N + BN - 1) / BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int m = static_cast<int>(blockIdx.x) / n_tiles;
  const int n0 = (static_cast<int>(blockIdx.x) - m * n_tiles) * BN;
  // the tile's rows: the always-on expert's first, then 32 at a time of the experts that have some
  int e = E, row0 = a.sh_row0 + 32 * m, row_end = a.sh_row0 + a.sh_rows;
  const int sh_m = (a.sh_rows + 31) / 32;
  if (m >= sh_m) {
    m -= sh_m;
    int before = 0;
    e = -1;
#pragma unroll
    for (int q = 0; q < REFLEX_MAX_EXPERTS / 64; ++q) {
      if (64 * q < E && e < 0) {
        const int i = 64 * q + lane, lo = a.expert_offsets[min(i, E)], hi = min(a.expert_offsets[min(i + 1, E)], a.out_rows);
        const int tiles = (max(hi - lo, 0) + 31) / 32, incl = before + wave_inclusive_scan_i32(tiles, lane);
        const uint64_t here = __ballot(i < E && m >= incl - tiles && m < incl);
        if (here != 0) {
          const int at = __ffsll(static_cast<unsigned long long>(here)) - 1;
          e = 64 * q + at;
          row0 = __builtin_amdgcn_readlane(lo, at) + 32 * (m - __builtin_amdgcn_readlane(incl - tiles, at));
          row_end = __builtin_amdgcn_readlane(hi, at);
        }
        before = __builtin_amdgcn_readlane(incl, 63);
      }
    }
  }
  if (e < 0 || row0 < 0 || row0 >= row_end) return;
  const bool on = e == E;
  // (rows past the last are the last one's again, and not stored)
  const int row = min(row0 + lane % 32, row_end - 1);
  int src = row;
  if (MODE == UP && !on) src = a.gather[row];
  const size_t e0 = on ? size_t(0) : static_cast<size_t>(e) * N;
  const uint8_t* w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int n = min(n0 + (MODE == UP ? 0 : 32 * j) + lane % 32, N - 1);
    const uint8_t* const base = MODE == UP && j == 1 ? (on ? a.sw1 : a.w1) : (on ? a.sw0 : a.w0);
    w[j] = base + (e0 + n) * K + 32 * (lane / 32);
  }
  // A slice: lane l has bytes 32 (l / 32) .. of each half of its rows' 128 (of both operands alike)
  struct Slice {
    i32x4_t w[2][4], x[4];
    uint4 r[4][2];
  } slice;
  auto load_weights = [&](Slice& f, int k) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        f.w[j][q] =
            *reinterpret_cast<const i32x4_t*>(w[j] + static_cast<size_t>(k) * G8_BK + 64 * (q / 2) + 16 * (q % 2));
  };
  // (an access waits for those before it: UP's weights are asked for behind the rows' numbers and ahead of the rows, DOWN's
  // behind its first rows)
  if constexpr (MODE == UP) {
    if (wave < nk) load_weights(slice, wave);
    __builtin_amdgcn_sched_barrier(0);
    if (on) src -= a.sh_row0;
  }
  src = min(max(src, 0), a.x_rows - 1);
  const uint8_t* const x = a.x + static_cast<size_t>(src) * K + 32 * (lane / 32);
  const uint16_t* const xr = act + static_cast<size_t>(src) * K + 32 * (lane / 32);
  auto load_rows = [&](Slice& f, int k) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const size_t at = static_cast<size_t>(k) * G8_BK + 64 * (q / 2) + 16 * (q % 2);
      if constexpr (MODE == UP) {
        f.x[q] = *reinterpret_cast<const i32x4_t*>(x + at);
      } else {
        f.r[q][0] = *reinterpret_cast<const uint4*>(xr + at);
        f.r[q][1] = *reinterpret_cast<const uint4*>(xr + at + 8);
      }
    }
  };
  if (wave < nk) load_rows(slice, wave);
  uint32_t most = 0;
  if constexpr (MODE == DOWN) {
    __builtin_amdgcn_sched_barrier(0);
    auto maximum = [&](const Slice& f) {
#pragma unroll
      for (int q = 0; q < 4; ++q) most = max(most, max(i8_amax8(f.r[q][0]), i8_amax8(f.r[q][1])));
    };
    if (wave < nk) {
      load_weights(slice, wave);
      __builtin_amdgcn_sched_barrier(0);
      maximum(slice);
    }
    for (int k = wave + FEW_W; k < nk; k += FEW_W) {
      Slice f;
      load_rows(f, k);
      maximum(f);
    }
  }
  float factor = 0.0f;
  if constexpr (MODE == DOWN) {
    uint32_t lower, upper;      // the two halves of a row's slices
    rows_swap32(most, lower, upper);
    most = max(lower, upper);
    if (lane < 32) s_max[wave][lane] = most;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < FEW_W; ++v) most = max(most, s_max[v][lane % 32]);
    factor = i8_factor(most);
    if (threadIdx.x < 32) s_scale[threadIdx.x] = i8_scale(most);
  } else if (threadIdx.x < 32) {
    s_scale[threadIdx.x] = __uint_as_float(a.x_scale[src]);
  }
  i32x16_t acc[2] = {};
  for (int k = wave; k < nk; k += FEW_W) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const i32x4_t xv = MODE == UP ? slice.x[q] : codes16(slice.r[q][0], slice.r[q][1], factor);
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(slice.w[j][q], xv, acc[j], 0, 0, 0);
    }
    if (k + FEW_W < nk) {
      load_weights(slice, k + FEW_W);
      load_rows(slice, k + FEW_W);
    }
  }
  // lane l, register r: row l % 32, column 8 (r / 4) + 4 (l / 32) + r % 4
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) sums[((wave * 2 + j) * 16 + r) * SLIM_PITCH + lane] = acc[j][r];
  __syncthreads();
  uint16_t* const out = static_cast<uint16_t*>(a.out);
  auto value = [&](int j, int i, int c) {      // row i, column c of block j
    const int* const at = sums + (j * 16 + (c / 8) * 4 + c % 4) * SLIM_PITCH + i + 32 * ((c / 4) % 2);
    int sum = at[0];
#pragma unroll
    for (int v = 1; v < FEW_W; ++v) sum += at[v * 2 * 16 * SLIM_PITCH];
    const uint32_t* const scale = MODE == UP && j == 1 ? (on ? a.ss1 : a.s1) : (on ? a.ss0 : a.s0);
    return static_cast<float>(sum) * (s_scale[i] * __uint_as_float(scale[e0 + n0 + (MODE == UP ? 0 : 32 * j) + c]));
  };
  for (int t = threadIdx.x; t < 32 * BN; t += 64 * FEW_W) {
    const int i = t / BN, c = t % BN;
    if (row0 + i >= row_end || n0 + c >= N) continue;
    const float v = MODE == UP ? silu_mul(value(0, i, c), value(1, i, c)) : value(c / 32, i, c % 32);
    out[static_cast<size_t>(row0 + i) * N + n0 + c] = f32_to_bf16(v);
  }
}

template <Mode MODE, int FEW_W>
int launch_few_as(const Args8& a, const uint16_t* act, hipStream_t s) {
  constexpr size_t lds = sizeof(int) * FEW_W * 2 * 16 * SLIM_PITCH;
  auto* kernel = &int8_few_kernel<MODE, FEW_W>;
  static std::atomic<uint64_t> set_on{0};
  const int rc = allow_lds(reinterpret_cast<const void*>(kernel), lds, set_on);
  if (rc != REFLEX_OK) return rc;
  // tiles at most: of the always-on rows, and of the routed ones one an expert and pair more than whole ones
  const int m_tiles = (a.sh_rows + 31) / 32 + std::min(a.E, a.out_rows) + a.out_rows / 32, bn = MODE == UP ? 32 : 64;
  hipLaunchKernelGGL(kernel, dim3(m_tiles * ((a.N + bn - 1) / bn)), dim3(64 * FEW_W), lds, s, a, act);
  return launch_status();
}

template <Mode MODE>
int launch_few(const Args8& a, const uint16_t* act, hipStream_t s) {
  return a.K < 8 * G8_BK ? launch_few_as<MODE, 4>(a, act, s) : launch_few_as<MODE, 8>(a, act, s);
}

// Whether experts of so many rows (when all are loaded alike) take these kernels: while their weights are a short stream.
// Both products and the rounding between, up to 8 experts a token, us, tiles / here: 64 experts of 3 x 2048 x 1024, 1
// token 27 / 16, 4 36 / 29, 16 73 / 64, 32 80 / 75, 64 85 / 84; 256 of 512, 8 tokens 42 / 38, 16 67 / 56, 32 82 / 89,
// 128 149 / 159; 256 of 1024 with up to 4, 16 tokens 69 / 66, 32 102 / 108; 8 of 4096 with up to 2, 8 tokens 55 / 46, 96
// 54 / 53; 33 of 640 with up to 4, 16 tokens 32 / 23, 200 42 / 42.
bool few_rows(int likely, int E, int cap, int d, int f, int sh_rows) {
  const double bytes = 3.0 * d * f * std::max(std::min(E, cap), 1);
  // (room for many rows of few tokens: a workgroup for every tile that there may be would be too many)
  return likely <= 32 && cap <= 64 * E && sh_rows <= 128 && bytes <= 4.5e8 && likely * bytes <= 3e9;
}

size_t act_bytes(int rows, int f) { return align_up(2 * static_cast<size_t>(rows) * f + 1); }
size_t code_bytes(int rows, int f) { return align_up(static_cast<size_t>(rows) * f + 1); }

}  // namespace

size_t swiglu_i8_ws_bytes(int rows, int f) {
  return act_bytes(rows, f) + code_bytes(rows, f) + align_up(sizeof(float) * (static_cast<size_t>(rows) + 1));
}

int launch_swiglu_i8(const int8_t* h, const float* hs, const int32_t* sorted_token, const int32_t* expert_offsets,
                     const Int8Weights& w, int T, int E, int d, int f, int cap, const AlwaysOnI8& sh, void* act,
                     uint16_t* y_sorted, hipStream_t s) {
  if (cap <= 0 && sh.rows <= 0) return REFLEX_OK;
  const int rows = cap + sh.rows;
  uint16_t* const a = static_cast<uint16_t*>(act);
  int8_t* const q = reinterpret_cast<int8_t*>(static_cast<char*>(act) + act_bytes(rows, f));
  float* const qs = reinterpret_cast<float*>(reinterpret_cast<char*>(q) + code_bytes(rows, f));
  const int likely = expected_rows(T, E, cap, sh.rows);
  const Args8 up{codes(h), bits(hs), sorted_token, expert_offsets, codes(w.w_gate), codes(w.w_up), bits(w.s_gate),
                 bits(w.s_up), codes(sh.w.w_gate), codes(sh.w.w_up), bits(sh.w.s_gate), bits(sh.w.s_up), E, d, f, T, cap,
                 sh.row0, sh.rows, nullptr, a, nullptr, 0};
  const Args8 down{codes(q), bits(qs), nullptr, expert_offsets, codes(w.w_down), nullptr, bits(w.s_down), nullptr,
                   codes(sh.w.w_down), nullptr, bits(sh.w.s_down), nullptr, E, f, d, rows, cap, sh.row0, sh.rows, nullptr,
                   y_sorted, nullptr, 0};
  if (few_rows(likely, E, cap, d, f, sh.rows)) {
    const int rc = launch_few<UP>(up, nullptr, s);
    return rc != REFLEX_OK ? rc : launch_few<DOWN>(down, a, s);
  }
  int rc = launch_gemm8<I8, UP, uint16_t>(up, likely, s);
  if (rc != REFLEX_OK) return rc;
  // (without routed experts the rows are the always-on expert's)
  rc = launch_quantize_i8(a, nullptr, E > 0 ? expert_offsets + E : nullptr, rows, rows, sh.rows > 0 ? sh.row0 : rows, f, q,
                          qs, s);
  if (rc != REFLEX_OK) return rc;
  return launch_gemm8<I8, DOWN, uint16_t>(down, likely, s);
}

int launch_matmul_i8(const int8_t* x, const float* xs, const int8_t* w, const float* ws, const int32_t* n_rows, int M,
                     int N, int K, int out_type, void* out, hipStream_t s) {
  const Args8 a{codes(x), bits(xs), nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, codes(w), nullptr, bits(ws), nullptr,
                0, K, N, M, M, 0, M, n_rows, out, nullptr, 0};
  return out_type == REFLEX_TYPE_F32 ? launch_gemm8<I8, PLAIN, float>(a, M, s) : launch_gemm8<I8, PLAIN, uint16_t>(a, M, s);
}

}  // namespace rfx
