// SwiGLU experts and plain products on e4m3 rows and weights (fp8.h): the launches of gemm8_impl.h.
#include "gemm8_impl.h"

namespace rfx {
namespace {

const uint32_t* dwords(const uint8_t* p) { return reinterpret_cast<const uint32_t*>(p); }

}  // namespace

// codes [rows, f], then their scales
size_t swiglu8_act_bytes(int rows, int f) { return align_up(std::max<size_t>(static_cast<size_t>(rows) * f, 1)); }
size_t swiglu8_ws_bytes(int rows, int f) {
  return swiglu8_act_bytes(rows, f) + align_up(std::max<size_t>(4 * static_cast<size_t>(f8_groups(f)) * rows, 1));
}

int launch_swiglu8_up(const uint8_t* h, const uint8_t* hs, const int32_t* sorted_token, const int32_t* expert_offsets,
                      const Fp8Weights& w, int T, int E, int d, int f, int cap, const AlwaysOn8& sh, uint8_t* act,
                      hipStream_t s) {
  if (cap <= 0 && sh.rows <= 0) return REFLEX_OK;
  const int rows = cap + sh.rows;
  const Args8 a{h, dwords(hs), sorted_token, expert_offsets, w.w_gate, w.w_up, dwords(w.s_gate), dwords(w.s_up),
                sh.w.w_gate, sh.w.w_up, dwords(sh.w.s_gate), dwords(sh.w.s_up), E, d, f, T, cap, sh.row0, sh.rows,
                nullptr, act, act + swiglu8_act_bytes(rows, f), rows};
  return launch_gemm8<F8, UP, uint8_t>(a, expected_rows(T, E, cap, sh.rows), s);
}

int launch_swiglu8_down(const int32_t* expert_offsets, const Fp8Weights& w, int T, int E, int d, int f, int cap,
                        const AlwaysOn8& sh, const uint8_t* act, uint16_t* y_sorted, hipStream_t s) {
  if (cap <= 0 && sh.rows <= 0) return REFLEX_OK;
  const int rows = cap + sh.rows;
  const Args8 a{act, dwords(act + swiglu8_act_bytes(rows, f)), nullptr, expert_offsets, w.w_down, nullptr,
                dwords(w.s_down), nullptr, sh.w.w_down, nullptr, dwords(sh.w.s_down), nullptr, E, f, d, rows, cap,
                sh.row0, sh.rows, nullptr, y_sorted, nullptr, 0};
  return launch_gemm8<F8, DOWN, uint16_t>(a, expected_rows(T, E, cap, sh.rows), s);
}

int launch_swiglu8_dense(const uint8_t* x, const uint8_t* xs, const Fp8Weights& w, int M, int d, int f, uint16_t* y,
                         uint8_t* act, hipStream_t s) {
  if (M <= 0) return REFLEX_OK;
  const AlwaysOn8 sh{w, 0, M};
  const Fp8Weights none{};
  int rc = launch_swiglu8_up(x, xs, nullptr, nullptr, none, M, 0, d, f, 0, sh, act, s);
  if (rc == REFLEX_OK) rc = launch_swiglu8_down(nullptr, none, M, 0, d, f, 0, sh, act, y, s);
  return rc;
}

int launch_matmul8(const uint8_t* x, const uint8_t* xs, const uint8_t* w, const uint8_t* ws, const int32_t* n_rows,
                   int M, int N, int K, int out_type, void* out, hipStream_t s) {
  const Args8 a{x, dwords(xs), nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, w, nullptr, dwords(ws), nullptr,
                0, K, N, M, M, 0, M, n_rows, out, nullptr, 0};
  return out_type == REFLEX_TYPE_F32 ? launch_gemm8<F8, PLAIN, float>(a, M, s) : launch_gemm8<F8, PLAIN, uint16_t>(a, M, s);
}

}  // namespace rfx
