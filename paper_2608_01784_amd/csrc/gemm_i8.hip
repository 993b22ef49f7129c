// SwiGLU experts and plain products on 8-bit integer rows and weights (int8.h).
//
// A wave has 32 rows x 32 columns (of gate and of up in UP) and reads both operands from global memory, 16 bytes of a
// row a lane, into v_mfma_i32_32x32x32_i8.  Weights are the MFMA's first operand: lane l, register r hold row l % 32
// and column 8 (r / 4) + 4 (l / 32) + r % 4.
#include "int8.h"

namespace rfx {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));
enum Mode { UP, DOWN, PLAIN };
constexpr int GI_WAVES = 4;

struct ArgsI8 {
  const int8_t* x;                          // [x_rows, K]
  const float* x_scale;                     // [x_rows]
  const int32_t *gather, *expert_offsets;
  const int8_t *w0, *w1;                    // routed weights [E, N, K]: gate and up (UP), or w0 alone
  const float *s0, *s1;                     // their scales [E, N]
  const int8_t *sw0, *sw1;                  // the always-on expert's (PLAIN: the weights)
  const float *ss0, *ss1;
  int E, K, N, x_rows, out_rows;
  int sh_row0, sh_rows;
  const int32_t* n_rows;
  void* out;
};

__device__ __forceinline__ float silu_mul(float g, float u) {
  return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f)) * u;
}

template <Mode MODE, class OUT>
__global__ __launch_bounds__(64 * GI_WAVES) void gemm_i8_kernel(ArgsI8 a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n_tiles = (a.N + 32 * GI_WAVES - 1) / (32 * GI_WAVES);
  const int n0 = (static_cast<int>(blockIdx.x % n_tiles) * GI_WAVES + wave) * 32;
  int m = blockIdx.x / n_tiles, e = a.E, row0 = 0, row_end = 0, sh_rows = a.sh_rows;
  if (MODE == PLAIN && a.n_rows != nullptr) sh_rows = min(max(a.n_rows[0], 0), sh_rows);
  const int sh_m = (sh_rows + 31) / 32;
  if (m < sh_m) {
    row0 = a.sh_row0 + 32 * m;
    row_end = a.sh_row0 + sh_rows;
  } else {
    m -= sh_m;
    for (e = 0; e < a.E; ++e) {
      const int lo = a.expert_offsets[e], hi = min(a.expert_offsets[e + 1], a.out_rows), tiles = (max(hi - lo, 0) + 31) / 32;
      if (m < tiles) {
        row0 = lo + 32 * m;
        row_end = hi;
        break;
      }
      m -= tiles;
    }
  }
  if (row0 < 0 || row0 >= row_end || n0 >= a.N) return;
  const bool on = e == a.E;      // the always-on expert's, or a plain product
  const int row = min(row0 + lane % 32, row_end - 1);
  int src = row;
  if (MODE == UP) src = on ? row - a.sh_row0 : a.gather[row];
  src = min(max(src, 0), a.x_rows - 1);
  const int n = min(n0 + lane % 32, a.N - 1);
  const int8_t* const x = a.x + static_cast<size_t>(src) * a.K + 16 * (lane / 32);
  const size_t at = (on ? size_t(0) : static_cast<size_t>(e) * a.N) + n;
  const int8_t* const w0 = (on ? a.sw0 : a.w0) + at * a.K + 16 * (lane / 32);
  const int8_t* const w1 = MODE == UP ? (on ? a.sw1 : a.w1) + at * a.K + 16 * (lane / 32) : nullptr;
  i32x16_t c0 = {}, c1 = {};
  for (int k = 0; k < a.K; k += 32) {
    const i32x4_t xv = *reinterpret_cast<const i32x4_t*>(x + k);
    c0 = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4_t*>(w0 + k), xv, c0, 0, 0, 0);
    if (MODE == UP) c1 = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4_t*>(w1 + k), xv, c1, 0, 0, 0);
  }
  if (row0 + lane % 32 >= row_end) return;
  const float sx = a.x_scale[src];
  const size_t base = on ? size_t(0) : static_cast<size_t>(e) * a.N;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int col = n0 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
    if (col >= a.N) continue;
    float v = static_cast<float>(c0[r]) * (sx * (on ? a.ss0 : a.s0)[base + col]);
    if (MODE == UP) v = silu_mul(v, static_cast<float>(c1[r]) * (sx * (on ? a.ss1 : a.s1)[base + col]));
    OUT* const out = static_cast<OUT*>(a.out) + static_cast<size_t>(row) * a.N + col;
    if constexpr (sizeof(OUT) == 4)
      *out = v;
    else
      *out = f32_to_bf16(v);
  }
}

template <Mode MODE, class OUT>
int launch(const ArgsI8& a, hipStream_t s) {
  const size_t m_tiles = (a.sh_rows + 31) / 32 + (a.E > 0 ? a.out_rows / 32 + a.E : 0);
  const size_t tiles = m_tiles * ((a.N + 32 * GI_WAVES - 1) / (32 * GI_WAVES));
  hipLaunchKernelGGL((gemm_i8_kernel<MODE, OUT>), dim3(static_cast<unsigned>(tiles)), dim3(64 * GI_WAVES), 0, s, a);
  return launch_status();
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
  const ArgsI8 up{h, hs, sorted_token, expert_offsets, w.w_gate, w.w_up, w.s_gate, w.s_up, sh.w.w_gate, sh.w.w_up,
                  sh.w.s_gate, sh.w.s_up, E, d, f, T, cap, sh.row0, sh.rows, nullptr, a};
  int rc = launch<UP, uint16_t>(up, s);
  if (rc != REFLEX_OK) return rc;
  // (without routed experts the rows are the always-on expert's)
  rc = launch_quantize_i8(a, nullptr, E > 0 ? expert_offsets + E : nullptr, rows, rows, sh.rows > 0 ? sh.row0 : rows, f, q,
                          qs, s);
  if (rc != REFLEX_OK) return rc;
  const ArgsI8 down{q, qs, nullptr, expert_offsets, w.w_down, nullptr, w.s_down, nullptr, sh.w.w_down, nullptr,
                    sh.w.s_down, nullptr, E, f, d, rows, cap, sh.row0, sh.rows, nullptr, y_sorted};
  return launch<DOWN, uint16_t>(down, s);
}

int launch_matmul_i8(const int8_t* x, const float* xs, const int8_t* w, const float* ws, const int32_t* n_rows, int M,
                     int N, int K, int out_type, void* out, hipStream_t s) {
  const ArgsI8 a{x, xs, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, w, nullptr, ws, nullptr,
                 0, K, N, M, 0, 0, M, n_rows, out};
  return out_type == REFLEX_TYPE_F32 ? launch<PLAIN, float>(a, s) : launch<PLAIN, uint16_t>(a, s);
}

}  // namespace rfx
