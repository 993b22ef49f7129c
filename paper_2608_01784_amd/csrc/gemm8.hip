// SwiGLU experts and plain products on 8-bit rows and weights (fp8.h), on the f8f6f4 MFMA.
//
//  UP:    act[j, :] = quantize(SiLU(x_j W_gate[e]^T) * (x_j W_up[e]^T)),  x_j = h[sorted_token[j]]
//  DOWN:  y[j, :]   = act[j, :] W_down[e]^T
//  PLAIN: out[i, :] = x[i, :] W^T, any N, the first n_rows rows (fp8_slim_kernel where there are few tiles)
// Both operands are K-contiguous codes.  Rows of one expert are contiguous; each workgroup counts
// the experts' M tiles itself from expert_offsets, so no launch shape depends on device-resident
// counts.  One more expert may follow the routed ones, the always-on one: every token is one of
// its rows, in token order.  In UP the first half of a tile's weight rows are gate rows and the
// second half the matching up rows, so gate and up of a column meet in one lane and register.
//
// Scales: a K slice of the loop is one block of 128 codes, so it has one scale byte per input
// row and one per 128 weight rows, and v_mfma_scale_f32_32x32x64_f8f6f4 takes both bytes as they
// are, at the rate of the unscaled instruction and with no vector instruction between the
// products.  A lane multiplies the same input rows in every slice: it loads their bytes four
// slices at once, a group ahead.  The weights' bytes of a whole tile lie in one register, a dword
// a lane.
//
// Precision: the f8f6f4 MFMA adds its 64 products with about 17 bits below the largest of them
// (measured: 1.4e-5 relative in the 2-norm, whatever K is), far inside the rounding to bf16 or e4m3
// that follows (but a code of the activation next to a border may be the other one: experts are 1.8e-3 to
// 2.1e-3 from 64 bits where fp32 sums leave 1.7e-3), and not what an fp32 result promises.  PLAIN with fp32
// results therefore widens the codes to bf16 (one instruction for two, scale included; e4m3 numbers times
// powers of two are bf16 numbers, at the ends of the range with move_scales) and multiplies on
// v_mfma_f32_32x32x16_bf16, whose products are exact and whose sums are fp32: a quarter of the rate,
// unnoticed where the weights' stream bounds the product.
//
// Data movement: operands go from global memory straight into LDS (16 bytes a lane) through rings
// of slices.  LDS rows are 128 bytes (8 chunks of 16) with chunk c of row r in slot
// c ^ ((r / 2) % 8): of the 16 rows that a 16-byte read serves at a time, all (row parity, slot)
// pairs are distinct, so fragment reads are free of bank conflicts, while a wave's copy writes
// 1 KB (8 whole rows) contiguously.  Each lane reads chunks fsel and 2 + fsel of its row for the
// first MFMA of a slice and 4 + fsel and 6 + fsel for the second, of both operands alike (which
// products of a block meet in one instruction is free).
//
// Scheduling: a persistent grid walks a flattened sequence of (tile, slice) steps, so copying
// ahead continues across tile boundaries.  Tiles are dealt to the 8 XCDs in contiguous runs
// (workgroup b runs on XCD b % 8).  Of an expert the N tiles of one M tile are adjacent (its
// gathered rows stay in L2); of a plain product the M tiles of one N tile (the weights are the
// large operand).
//
// What bounds it, measured: many rows by the MFMAs (8192 x 8192 x 8192 2.3 PFLOP/s, where a large
// library product of this type reaches 2.7) and, with a short K, by the tiles' stores, which come from all
// workgroups at once and are not hidden (8192 x 8192 x 2048 2.0; 64 experts of 3 x 2048 x 1024 with 53000
// rows 1.65); few rows by the weights' stream (48 rows of 131072 x 2048 6.2 TB/s for bf16 results, 4.8 for
// fp32 ones; experts 3.5 to 4.5 TB/s, whose launches are short and start with two dependent
// loads).  Letting every second workgroup start half a tile later, so that stores meet products of others, cost
// its delay (490 -> 512 us).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "fp8.h"

namespace rfx {

namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int G8_XCDS = 8;
constexpr int G8_BK = F8_BLOCK;                  // bytes of a slice's row
constexpr int G8_CHUNKS = G8_BK / 16;
constexpr int G8_OP_ROWS = 64 / G8_CHUNKS;       // rows of one wave's copy (1 KB)
constexpr int G8_NJ = 4;                         // 32-row weight blocks per wave
enum Mode { UP, DOWN, PLAIN };

// s_waitcnt vmcnt(N) with expcnt and lgkmcnt left at their maxima (vmcnt in bits [3:0] and
// [15:14], expcnt [6:4], lgkmcnt [11:8]).
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0f70);
}

// Workgroup barrier without the fences of __syncthreads(), which would drain the copies in
// flight.  lgkmcnt(0): this wave's LDS reads are done before any wave refills what they read.
__device__ __forceinline__ void lds_barrier8() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Cache policy of the copies: work-group scope; a line is read once per workgroup.
constexpr int kCopyPolicy = 1;

// One wave's 1 KB copy with 64-bit addresses.  (Out of line of the kernel's lambdas, so that the
// host-side pass of the kernel stays valid.)
__device__ __forceinline__ void copy_far(const uint8_t* src, uint8_t* dst) {
  __builtin_amdgcn_global_load_lds(src, dst, 16, 0, kCopyPolicy);
}

// Eight codes times a power of two as bf16 numbers.
__device__ __forceinline__ bf16x8_t widen8(int lo, int hi, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Widened codes are bf16 numbers under scale bytes 3 .. 246.  Codes next to 448 under 247 are past bf16 (the
// largest bf16 numbers round to 256 2^120), subnormal ones under 1 and 2 below its last place.  There a power of two
// moves between the bytes of the wave's rows, x[i] a lane, and the byte w of the weights, which all of them share;
// four slices' bytes at once.  (A row at the other end of the range then keeps its numbers to within 2^-133.)
template <int MI>
__device__ __forceinline__ void move_scales(uint32_t (&x)[MI], uint32_t& w) {
  // below 16 or from 240 on: the upper four bits of a byte alike
  auto maybe = [](uint32_t v) {
    const uint32_t differ = (v ^ (v << 1)) & 0xe0e0e0e0u;
    return ((differ - 0x01010101u) & ~differ & 0x80808080u) != 0;
  };
  bool some = maybe(w);
#pragma unroll
  for (int i = 0; i < MI; ++i) some = some || maybe(x[i]);
  if (!__any(some)) return;
#pragma unroll 1
  for (int at = 0; at < 32; at += 8) {
    uint32_t least = 255, most = 0;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      least = min(least, (x[i] >> at) & 0xffu);
      most = max(most, (x[i] >> at) & 0xffu);
    }
    const bool high = __any(most > 246), near_high = __any(most > 244), low = __any(least < 3);
    const uint32_t wb = (w >> at) & 0xffu;
    int move = 0;
    if (high)
      move = -1;
    else if (low)
      move = near_high || wb < 5 ? 0 : 2;
    else if (wb > 246)
      move = near_high ? 0 : 1;
    else if (wb < 3)
      move = -2;
#pragma unroll
    for (int i = 0; i < MI; ++i) x[i] += static_cast<uint32_t>(move) << at;
    w -= static_cast<uint32_t>(move) << at;
  }
}

__device__ __forceinline__ float silu_mul(float g, float u) {
  return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f)) * u;
}

// The lane number, as a value that is computed where it is used: what depends on it is not moved out of the
// loops around, where it would hold registers over a whole tile.
__device__ __forceinline__ int lane_here() {
  int l = threadIdx.x & 63;
  asm volatile("" : "+v"(l));
  return l;
}

// ---- epilogue stores of a tile of DOWN or PLAIN ---------------------------------------------------------
// A wave has 32 rows x 128 columns of a pair block as four accumulators of 32 columns: lane l, register r
// holds row l % 32 and column 8 (r/4) + 4 (l/32) + r%4.  Rows go through the wave's 4 KB of scratch in
// LDS, 128 bytes of each at a time (64 bf16 or 32 fp32 columns), and come back with neighbouring lanes
// on neighbouring columns, so that a store writes whole 128-byte pieces of rows.  Chunk c (16 bytes) of row r
// lies at c ^ (r % 8), free of bank conflicts both ways.  (Inline assembly: the compiler cannot tell
// the scratch from the ring that copies in flight write, and would wait for those.)
constexpr int G8_STAGE = 32 * 128;

__device__ __forceinline__ void lds_write64(uint32_t at, uint32_t a, uint32_t b) {
  asm volatile("ds_write_b64 %0, %1" ::"v"(at), "v"(u32x2_t{a, b}) : "memory");
}
__device__ __forceinline__ void lds_write128(uint32_t at, float a, float b, float c, float d) {
  asm volatile("ds_write_b128 %0, %1" ::"v"(at), "v"(f32x4_t{a, b, c, d}) : "memory");
}
__device__ __forceinline__ uint32_t stage_at(uint32_t stage, int row, int chunk) {
  return stage + row * 128 + ((chunk ^ (row & 7)) * 16);
}

// The staged 32 rows x (128 / sizeof(OUT)) columns to `out`: rows row_base .. below row_end, columns
// col_base .. below N.  8 lanes a row, 16 bytes each, at any address that the elements allow (rows of
// an odd N start anywhere; global stores need no alignment beyond that).
template <class OUT, bool ANY_N>
__device__ __forceinline__ void store_staged(int row_base, int col_base, int row_end, int N, OUT* __restrict__ out,
                                             uint32_t stage) {
  constexpr int VEC = 16 / sizeof(OUT), COLS = 128 / sizeof(OUT);
  const int lane = lane_here();
  if (ANY_N && col_base + COLS > N && N % VEC != 0) {      // the rows' end inside a vector: an element a lane
#pragma unroll 1
    for (int q = 0; q < 32 * COLS / 64; ++q) {
      const int r = (64 / COLS) * q + lane / COLS, c = lane % COLS;
      const uint32_t at = stage_at(stage, r, c / VEC) + sizeof(OUT) * (c % VEC);
      uint32_t v;
      if constexpr (sizeof(OUT) == 4)
        asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v) : "v"(at) : "memory");
      else
        asm volatile("ds_read_u16 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v) : "v"(at) : "memory");
      if (row_base + r < row_end && col_base + c < N) {
        OUT* const to = out + static_cast<size_t>(row_base + r) * N + col_base + c;
        if constexpr (sizeof(OUT) == 4)
          *to = __uint_as_float(v);
        else
          *to = static_cast<OUT>(v);
      }
    }
    return;
  }
  u32x4_t v[4];
  uint32_t at[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) at[q] = stage_at(stage, (lane >> 3) + 8 * q, lane & 7);
  asm volatile(
      "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3])
      : "memory");
  const int col = col_base + VEC * (lane & 7);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = row_base + (lane >> 3) + 8 * q;
    if (row < row_end && col < N) __builtin_memcpy(out + static_cast<size_t>(row) * N + col, &v[q], 16);
  }
}

// A tile shape: 2 x 2 waves, one a SIMD, MI 32-row pair blocks by 128 weight rows each (wave (wm, wn) has
// the pair blocks wm, wm + 2, ..: an expert's last tile then shortens all waves alike); rings of
// A_SLOTS input-row and B_SLOTS weight slices, copied A_SLOTS - 1 and B_SLOTS - 1 steps ahead.  (Blocks of
// 128 x 128 a wave read half as much LDS per product as eight waves' of 128 x 64, whose reads and copies
// alone would take all of the LDS's rate.)
template <int MI_, int A_SLOTS_, int B_SLOTS_>
struct Shape8 {
  static constexpr int MI = MI_, WM = 2, WN = 2, WAVES = 4, A_SLOTS = A_SLOTS_, B_SLOTS = B_SLOTS_;
  static constexpr int THREADS = 64 * WAVES;
  static constexpr int BM = 32 * MI * WM, BROWS = 32 * G8_NJ * WN;      // pair and weight rows of a tile
  static constexpr int A_BYTES = BM * G8_BK, B_BYTES = BROWS * G8_BK;   // one slice
  static constexpr int A_OPS = BM / G8_OP_ROWS / WAVES, B_OPS = BROWS / G8_OP_ROWS / WAVES;   // a wave's copies
  static constexpr int B_WROWS = BROWS / WAVES;                         // weight rows a wave copies
  static constexpr size_t LDS = size_t(A_SLOTS) * A_BYTES + size_t(B_SLOTS) * B_BYTES;
  // Copies that may be in flight when a step starts: those issued after its own input rows
  // (A_SLOTS - 1 steps ago) and weights (no later than the rows).
  static constexpr int IN_FLIGHT = (B_SLOTS > A_SLOTS ? B_OPS : 0) + (A_SLOTS - 2) * (A_OPS + B_OPS);
  static_assert(A_SLOTS >= 2 && B_SLOTS >= A_SLOTS, "shape");
  static_assert(A_OPS * G8_OP_ROWS * WAVES == BM && B_OPS * G8_OP_ROWS * WAVES == BROWS, "whole copies");
  static_assert(WAVES * G8_STAGE <= B_BYTES && 8 * BM <= B_BYTES, "the epilogue's scratch fits a weight slot");
  static_assert(BROWS == 2 * F8_BLOCK && B_WROWS == F8_BLOCK / 2, "UP: half of the waves copy gate rows, half up rows");
  static_assert(4 * (REFLEX_MAX_EXPERTS + 1) <= LDS, "start-up scratch in the rings");
  static_assert(LDS <= 160 * 1024 && IN_FLIGHT < 64, "LDS and vmcnt range");
};

struct Args8 {
  const uint8_t* x;                    // [x_rows, K] codes
  const uint32_t* x_scale;             // [ceil(K / 512)][x_rows], four blocks' bytes each
  const int32_t *gather, *expert_offsets;
  const uint8_t *w0, *w1;              // routed weights [E, N, K]: gate and up (UP), or w0 alone
  const uint32_t *s0, *s1;             // their scales, a dword per four blocks of a row of blocks
  const uint8_t *sw0, *sw1;            // the always-on expert's (PLAIN: the weights)
  const uint32_t *ss0, *ss1;
  int E, K, N, x_rows, out_rows;       // out_rows: rows the routed experts may write
  int sh_row0, sh_rows;                // the always-on expert's rows of x (UP: of `out` alone)
  const int32_t* n_rows;               // PLAIN: on the device, NULL: sh_rows
  void* out;
  uint8_t* out_scale;                  // UP: the activation's, [ceil(N / 512)][act_rows][4]
  int act_rows;
};

// BIG: x of 2^31 bytes or more, addressed with 64-bit pointers (a buffer resource's byte offset
// has 32 bits, of which the upper half is kept for skipped copies).
template <Mode MODE, class S, bool BIG, class OUT>
__global__ __launch_bounds__(S::THREADS, 1) void fp8_gemm_kernel(Args8 a) {
  constexpr int MI = S::MI, A_OPS = S::A_OPS, B_OPS = S::B_OPS;
  constexpr bool WIDE = MODE == PLAIN && sizeof(OUT) == 4;       // fp32 results
  constexpr int BN = MODE == UP ? S::BROWS / 2 : S::BROWS;       // output columns of a tile
  extern __shared__ __attribute__((aligned(16))) uint8_t smem8[];
  uint8_t* const a_ring = smem8;
  uint8_t* const b_ring = smem8 + S::A_SLOTS * S::A_BYTES;
  const int K = a.K, N = a.N, E = a.E;
  int sh_rows = a.sh_rows;
  if (MODE == PLAIN && a.n_rows != nullptr) sh_rows = min(max(a.n_rows[0], 0), sh_rows);
  const int n_tiles = (N + BN - 1) / BN, nk = K / G8_BK, groups = (nk + 3) / 4;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN;
  // ---- expert row offsets and the prefix of M tiles, in registers: lane l holds experts l,
  // l + 64, l + 128, l + 192
  int toff_r[4] = {}, eo_r[4] = {}, eo_E = 0, m_total = 0;
  if (MODE != PLAIN) {
    int* s_eo = reinterpret_cast<int*>(smem8);       // (the rings are empty yet)
    for (int e = tid; e <= E; e += S::THREADS) s_eo[e] = E > 0 ? a.expert_offsets[e] : 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int e = lane + 64 * q;
      eo_r[q] = s_eo[e < E ? e : E];
      const int n = s_eo[e < E ? e + 1 : E] - eo_r[q];
      const int tiles = n < 0 ? 0 : (n + S::BM - 1) / S::BM;
      const int incl = wave_inclusive_scan_i32(tiles, lane);
      toff_r[q] = e < E ? (m_total + incl - tiles) * n_tiles : INT32_MAX;
      m_total += __builtin_amdgcn_readlane(incl, 63);
    }
    eo_E = __builtin_amdgcn_readfirstlane(s_eo[E]);
    __syncthreads();     // all scratch reads done before the first copies land
  }
  auto table_at = [&](const int (&r)[4], int e) {      // entry e (< 256) of a per-lane table
    const int q = e >> 6;
    const int v = q == 0 ? r[0] : (q == 1 ? r[1] : (q == 2 ? r[2] : r[3]));
    return __builtin_amdgcn_readlane(v, e & 63);
  };
  struct Tile {
    int expert, row0, row_end, n0, rot;      // rot: the K group that the tile starts with
  };
  // Tiles of one height, in whole 64-row steps: no tile of few rows at an expert's end.
  auto height_of = [](int rows, int tiles) {
    return tiles > 1 ? min(((rows + tiles - 1) / tiles + 63) & ~63, S::BM) : S::BM;
  };
  const int sh_m = (sh_rows + S::BM - 1) / S::BM;
  auto decode = [&](bool always_on, int L) {
    Tile t;
    if (MODE == PLAIN || always_on) {
      // (PLAIN: M inner; an always-on expert: N inner, as the routed ones)
      const int n = MODE == PLAIN ? L / sh_m : L % n_tiles, m = MODE == PLAIN ? L - n * sh_m : L / n_tiles;
      const int height = height_of(sh_rows, sh_m);
      t.expert = E;
      t.n0 = n * BN;
      t.row0 = a.sh_row0 + min(m * height, sh_rows);
      t.row_end = min(a.sh_row0 + sh_rows, t.row0 + height);
      t.rot = n % groups;
      return t;
    }
    int e = -1;      // four ballots count the experts whose first tile lies at or before L
#pragma unroll
    for (int q = 0; q < 4; ++q) e += __popcll(__ballot(toff_r[q] <= L));
    e = e < 0 ? 0 : e;
    const int local = L - table_at(toff_r, e), m = local / n_tiles, n = local - m * n_tiles;
    const int er0 = table_at(eo_r, e), er1 = e + 1 < E ? table_at(eo_r, e + 1) : eo_E;
    const int height = height_of(er1 - er0, (er1 - er0 + S::BM - 1) / S::BM);
    t.expert = e;
    t.n0 = n * BN;
    t.row0 = er0 + m * height;
    t.row_end = min(min(er1, a.out_rows), t.row0 + height);
    if (t.row0 < 0 || t.row0 >= t.row_end) t.row_end = t.row0;   // inconsistent offsets: no rows
    // Tiles that stream weights at the same time start at different groups of their rows
    t.rot = (MODE == UP ? n % 2 + 5 * e : n) % groups;
    return t;
  };
  // ---- this workgroup's tiles: a contiguous run of the routed (PLAIN: of all) tiles per XCD,
  // strided over the XCD's workgroups; ahead of it the XCD's share of the always-on expert's
  const int xcd = blockIdx.x % G8_XCDS, per_xcd = gridDim.x / G8_XCDS, j0 = blockIdx.x / G8_XCDS;
  const int sh_tiles = MODE == PLAIN ? 0 : sh_m * n_tiles;
  const int sh_mine = (max(sh_tiles - xcd, 0) + G8_XCDS - 1) / G8_XCDS;
  const int run_tiles = (MODE == PLAIN ? sh_m : m_total) * n_tiles;
  const int chunk = (run_tiles + G8_XCDS - 1) / G8_XCDS;
  const int r_begin = xcd * chunk, r_mine = max(min(run_tiles - r_begin, chunk), 0);
  if (j0 >= sh_mine + r_mine) return;
  const int n_my = (sh_mine + r_mine - j0 + per_xcd - 1) / per_xcd;
  auto tile_at = [&](int i) {
    const int j = j0 + i * per_xcd;
    return j < sh_mine ? decode(true, xcd + G8_XCDS * j) : decode(false, r_begin + j - sh_mine);
  };
  // ---- copies: op q of a slice fills rows OP_ROWS q ..; lane L writes row r = OP_ROWS q + L / 8 at
  // slot L % 8, holding chunk (L % 8) ^ ((r / 2) % 8).  Each loader (input rows, weights) has a
  // current tile and slice and holds the next tile's setup ready: a tile's K loop takes it
  // across one tile boundary at most (unless short_k, when setups are made at the boundary).
  const bool short_k = nk < S::B_SLOTS;
  auto lane_row = [](int l, int q) { return q * G8_OP_ROWS + l / G8_CHUNKS; };
  auto lane_chunk = [&](int l, int q) { return ((l % G8_CHUNKS) ^ ((lane_row(l, q) / 2) % G8_CHUNKS)) * 16; };
  // Gathered rows (UP) have an offset a copy; contiguous ones a first row, copies j and j + 2 being 16 rows
  // apart with the same swizzle.  (Contiguous rows past the tile's last are other rows of x, or past
  // its end, where the range check, BIG: a clamp, keeps the copy inside.)
  constexpr int A_REGS = MODE == UP ? A_OPS : 2;
  using Off = typename std::conditional<BIG && MODE == UP, size_t, uint32_t>::type;
  int a_tile = -1, a_k = nk, a_rot = 0, a_ops = 0, a_row0 = 0, na_rot = 0, na_ops = 0, na_row0 = 0;
  bool na_ready = false, na_gather = false;
  Off a_off[A_REGS];
  int na_row = 0;      // UP: lane l has the source row of the wave's row l of the next tile
  auto set_a = [&](const Tile& t) {
    const int valid = t.row_end - t.row0;
    // copies wholly past the expert's last row are not issued; rows past it inside a 32-row block
    // hold whatever the slot held before, enter only their own row of the product, and are not stored
    const int n = (valid + G8_OP_ROWS - 1) / G8_OP_ROWS - A_OPS * wave;
    na_ops = __builtin_amdgcn_readfirstlane(min(max(n, 0), A_OPS));
    na_rot = t.rot;
    na_gather = MODE == UP && t.expert != E;
    na_row0 = valid > 0 ? t.row0 : 0;
    if constexpr (MODE == UP) {
      const int r = G8_OP_ROWS * A_OPS * wave + lane_here() % (G8_OP_ROWS * A_OPS);
      na_row = valid > 0 ? t.row0 + (r < valid ? r : 0) : 0;
      if (!na_gather) na_row -= a.sh_row0;
    }
  };
  auto gather_a = [&]() {
    if constexpr (MODE == UP) {
      if (na_ready && na_gather) na_row = a.gather[na_row];
    }
  };
  int b_tile = -1, b_k = nk, b_rot = 0, nb_rot = 0, b_len = 0, nb_len = 0;
  bool nb_ready = false;
  uint32_t b_lo = 0, b_hi = 0, nb_lo = 0, nb_hi = 0;
  uint32_t b_off[2];       // copies j and j + 2 are 16 rows apart and share the swizzle
#pragma unroll
  for (int j = 0; j < 2; ++j) b_off[j] = static_cast<uint32_t>(lane_row(lane, j) * K + lane_chunk(lane, B_OPS * wave + j));
  auto set_b = [&](const Tile& t) {
    nb_rot = t.rot;
    constexpr int W = S::B_WROWS, HALF = S::WAVES / 2;
    const bool second = MODE == UP && wave >= HALF;
    // rows past N are not copied, and their columns not stored
    const int row = min(t.n0 + W * (second ? wave - HALF : wave), N);
    nb_len = min(W, N - row) * K;
    const uint8_t* base = t.expert == E ? (second ? a.sw1 : a.sw0)
                                        : (second ? a.w1 : a.w0) + static_cast<size_t>(t.expert) * N * K;
    const uint64_t at = reinterpret_cast<uint64_t>(base + static_cast<size_t>(row) * K);
    nb_lo = static_cast<uint32_t>(at);
    nb_hi = static_cast<uint32_t>(at >> 32);
  };
  auto ready_a = [&]() {
    na_ready = a_tile + 1 < n_my;
    if (!na_ready) return;
    set_a(tile_at(a_tile + 1));
    gather_a();
  };
  auto ready_b = [&]() {
    nb_ready = b_tile + 1 < n_my;
    if (nb_ready) set_b(tile_at(b_tile + 1));
  };
  // The byte offset of a loader's next slice; then it advances (past the workgroup's last tile it
  // stays on its last slice, so the issue never branches and every address stays in bounds).
  auto a_next = [&]() {
    if (a_k == nk) {
      if (na_ready) {
        na_ready = false;
        ++a_tile;
        a_k = 0;
        a_rot = 4 * na_rot;
        a_ops = na_ops;
        a_row0 = na_row0;
        const int l = lane_here();
#pragma unroll
        for (int j = 0; j < A_REGS; ++j) {
          const int at = A_OPS * wave + j;
          const int src = MODE == UP ? min(max(__shfl(na_row, lane_row(l, j)), 0), a.x_rows - 1) : na_row0 + lane_row(l, at);
          a_off[j] = static_cast<Off>(src) * static_cast<Off>(K) + static_cast<Off>(lane_chunk(l, at));
        }
      } else {
        a_k = nk - 1;
      }
    }
    const int k = a_k + a_rot;
    ++a_k;
    return (k >= nk ? k - nk : k) * G8_BK;
  };
  auto b_next = [&]() {
    if (b_k == nk) {
      if (nb_ready) {
        nb_ready = false;
        ++b_tile;
        b_k = 0;
        b_rot = 4 * nb_rot;
        b_lo = nb_lo;
        b_hi = nb_hi;
        b_len = nb_len;
      } else {
        b_k = nk - 1;
      }
    }
    const int k = b_k + b_rot;
    ++b_k;
    return (k >= nk ? k - nk : k) * G8_BK;
  };
  // Input rows go through a resource of the operand's size; a skipped copy gets an offset past it,
  // which the range check turns into no memory access (no branch in the step).
  const __amdgpu_buffer_rsrc_t x_rsrc = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(a.x), static_cast<short>(0),
      BIG ? 0 : static_cast<int>(static_cast<uint32_t>(a.x_rows) * static_cast<uint32_t>(K)), 0x00020000);
  auto copy_a = [&](int j, uint8_t* slot, int k0) {
    uint8_t* to = slot + (A_OPS * wave + j) * 1024;
    if constexpr (BIG && MODE == UP) {
      copy_far(a.x + a_off[j] + k0, to);
    } else if constexpr (BIG) {
      const int l = lane_here(), row = min(a_row0 + lane_row(l, A_OPS * wave + j), a.x_rows - 1);
      copy_far(a.x + static_cast<size_t>(row) * K + lane_chunk(l, A_OPS * wave + j) + k0, to);
    } else {
      const uint32_t at = MODE == UP ? a_off[j] : a_off[j % 2] + static_cast<uint32_t>(16 * (j / 2) * K);
      const uint32_t off = j < a_ops ? at + static_cast<uint32_t>(k0) : 0x80000000u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rsrc, (__attribute__((address_space(3))) void*)to, 16, off, 0, 0,
                                               kCopyPolicy);
    }
  };
  auto copy_b = [&](int j, uint8_t* slot, int k0) {
    // the resource is rebuilt from wave-uniform values at each use, so that it lives in scalar registers
    const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b_lo)));
    const uint64_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b_hi)));
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(lo | (hi << 32)), static_cast<short>(0), __builtin_amdgcn_readfirstlane(b_len), 0x00020000);
    const uint32_t off = b_off[j % 2] + static_cast<uint32_t>(k0 + 16 * (j / 2) * K);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rsrc, (__attribute__((address_space(3))) void*)(slot + (B_OPS * wave + j) * 1024), 16, off, 0, 0, kCopyPolicy);
  };
  // ---- multiply: pair blocks WM i + wm, weight blocks b_row[j] of the tile
  // (UP: two blocks of gate rows, then the matching two of up rows)
  int b_row[G8_NJ];
#pragma unroll
  for (int j = 0; j < G8_NJ; ++j)
    b_row[j] = MODE == UP ? (j / 2) * (S::BROWS / 2) + 64 * wn + 32 * (j % 2) : 128 * wn + 32 * j;
  // ---- scales: source rows of this lane's row of each pair block, of this tile and of the next;
  // their bytes of the current group; the weights' bytes of all K (UP: gate and up rows)
  constexpr int SR = (MI + 1) / 2;      // lane l has row l % 32 of pair block 2 q + l / 32
  int s_row[SR], ns_row[SR];
  uint32_t s_cur[SR], w_cur[2] = {0, 0}, w_next[2] = {0, 0};
  auto set_scales = [&](const Tile& t) {
    const int valid = t.row_end - t.row0, l = lane_here();
#pragma unroll
    for (int q = 0; q < SR; ++q) {
      const int r = 32 * (S::WM * (2 * q + l / 32) + wm) + l % 32;
      int src = valid > 0 ? t.row0 + (r < valid ? r : 0) : 0;
      if (MODE == UP) src = t.expert == E ? src - a.sh_row0 : a.gather[src];
      ns_row[q] = min(max(src, 0), a.x_rows - 1);
    }
    const int block = min(t.n0 + (MODE == UP ? 0 : 128 * wn), N - 1) / F8_BLOCK;
    const size_t stride = static_cast<size_t>((N + F8_BLOCK - 1) / F8_BLOCK) * groups;
#pragma unroll
    for (int j = 0; j < (MODE == UP ? 2 : 1); ++j) {
      const uint32_t* base = t.expert == E ? (j ? a.ss1 : a.ss0) : (j ? a.s1 : a.s0) + t.expert * stride;
      w_next[j] = l < groups ? base[static_cast<size_t>(block) * groups + l] : 0u;
    }
  };
  auto load_scale = [&](int q, int row, int group) { s_cur[q] = a.x_scale[static_cast<size_t>(group) * a.x_rows + row]; };
  auto take_scales = [&]() {      // the next tile's become the current tile's
#pragma unroll
    for (int q = 0; q < SR; ++q) s_row[q] = ns_row[q];
    w_cur[0] = w_next[0];
    w_cur[1] = w_next[1];
  };
  // ---- prologue: the first tile's scales (ahead of the copies: an access waits for all that were issued before
  // it), then the copies that the steps before the first would have issued, in their order
  ready_a();
  Tile t = tile_at(0), next_t = t;
  set_scales(t);
  take_scales();
#pragma unroll
  for (int q = 0; q < SR; ++q) load_scale(q, s_row[q], t.rot);
#pragma unroll
  for (int v = 1 - S::B_SLOTS; v < 0; ++v) {
    const int qa = v + S::A_SLOTS - 1, qb = v + S::B_SLOTS - 1;
    if (qa >= 0) {
      if (qa > 0 && a_k == nk) ready_a();
      const int k = a_next();
#pragma unroll
      for (int j = 0; j < A_OPS; ++j) copy_a(j, a_ring + qa * S::A_BYTES, k);
    }
    if (b_k == nk) ready_b();
    const int k = b_next();
#pragma unroll
    for (int j = 0; j < B_OPS; ++j) copy_b(j, b_ring + qb * S::B_BYTES, k);
  }
  // The K loop of one tile with NB active pair blocks (0: this wave only copies), group by group; at its
  // end s_cur holds the next tile's first group.
  //
  // A SIMD has one wave, so the wave itself keeps its matrix core fed: a unit is one pair block times the
  // four weight blocks of half a slice (four MFMAs, 256 cycles), a slice 2 NB units.  A unit's fragments
  // are read while an earlier one multiplies, and a slice's last LATE units run after the next step's
  // barrier, while that slice's first fragments are read.  Units alternate between two fragment
  // registers; the late ones have their own.
  int s = 0;              // steps so far (the rings' slot counter)
  // One tile: K loop and epilogue, an instance per count of active blocks (with the accumulators inside,
  // which would be copied together from five places otherwise).
  auto tile = [&](auto nb_c) {
    constexpr int NB = decltype(nb_c)::value;
    const int l = lane_here(), frow = l & 31, fsel = l >> 5, fx = (frow / 2) % G8_CHUNKS;
    f32x16_t acc[NB > 0 ? NB : 1][G8_NJ];
    constexpr int UNITS = 2 * NB, LATE = NB > 1 ? 2 : 1;
    i32x8_t af[2 + LATE], bf[2][G8_NJ];
    uint32_t late_sx[LATE], late_sw[2];      // the late units' scales
    auto slot_of = [](int u) { return u >= UNITS - LATE ? 2 + u - (UNITS - LATE) : u % 2; };
    // (fresh: the first products of a tile add to nothing)
    auto multiply = [&](auto fresh_c, int u, uint32_t sx, const uint32_t (&sw)[2]) {
      constexpr bool FRESH = decltype(fresh_c)::value;
      const f32x16_t zero = {};
      const int kk = u / (NB > 0 ? NB : 1), i = u - kk * NB;
      // weights as the MFMA's A operand: a lane ends up with 4 consecutive columns of one row
      if constexpr (WIDE) {
        const float sws = __uint_as_float((sw[0] & 0xffu) << 23);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bf16x8_t xb =
              widen8(af[slot_of(u)][2 * q], af[slot_of(u)][2 * q + 1], __uint_as_float((sx & 0xffu) << 23));
#pragma unroll
          for (int j = 0; j < G8_NJ; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(bf[kk][j][2 * q], bf[kk][j][2 * q + 1], sws), xb,
                                                                FRESH && q == 0 ? zero : acc[i][j], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int j = 0; j < G8_NJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
              bf[kk][j], af[slot_of(u)], FRESH ? zero : acc[i][j], 0, 0, 0, static_cast<int>(sw[MODE == UP ? j / 2 : 0]), 0,
              static_cast<int>(sx));
      }
    };
    auto late_units = [&]() {
#pragma unroll
      for (int l = 0; l < LATE; ++l) multiply(std::false_type{}, UNITS - LATE + l, late_sx[l], late_sw);
    };
    auto step = [&](auto first_c, const uint32_t (&sx)[MI], const uint32_t (&sw)[2]) {
      constexpr bool FIRST = decltype(first_c)::value;
      const int ka = a_next(), kb = b_next();
      // slice s has landed (copies land in order; other outstanding accesses only lengthen the
      // wait) and is visible to all waves; the slots that the previous step read are free
      wait_copies<S::IN_FLIGHT>();
      lds_barrier8();
      uint8_t* const An = a_ring + ((s + S::A_SLOTS - 1) % S::A_SLOTS) * S::A_BYTES;
      uint8_t* const Bn = b_ring + ((s + S::B_SLOTS - 1) % S::B_SLOTS) * S::B_BYTES;
      if constexpr (NB == 0) {
#pragma unroll
        for (int j = 0; j < A_OPS; ++j) copy_a(j, An, ka);
#pragma unroll
        for (int j = 0; j < B_OPS; ++j) copy_b(j, Bn, kb);
      } else {
        constexpr int kMfmas = WIDE ? 4 * G8_NJ : G8_NJ;      // of a unit
        const uint8_t* const As = a_ring + (s % S::A_SLOTS) * S::A_BYTES;
        const uint8_t* const Bs = b_ring + (s % S::B_SLOTS) * S::B_BYTES;
        auto read = [&](const uint8_t* row, int kk) {
          const i32x4_t lo = *reinterpret_cast<const i32x4_t*>(row + ((4 * kk + fsel) ^ fx) * 16);
          const i32x4_t hi = *reinterpret_cast<const i32x4_t*>(row + ((4 * kk + 2 + fsel) ^ fx) * 16);
          return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        auto read_b = [&](int kk, int j) { bf[kk][j] = read(Bs + (b_row[j] + frow) * G8_BK, kk); };
        auto read_a = [&](int u) {
          const int kk = u / NB, i = u - kk * NB;
          af[slot_of(u)] = read(As + (32 * (S::WM * i + wm) + frow) * G8_BK, kk);
        };
        // The copies, a few after each unit.
        constexpr int SPOTS = FIRST ? UNITS - LATE : UNITS, OPS = A_OPS + B_OPS;
        int done = 0, spot = 0;
        auto copies = [&](int spots) {
          spot += spots;
          const int until = spot >= SPOTS ? OPS : OPS * spot / SPOTS;
#pragma unroll
          for (int c = 0; c < OPS; ++c)
            if (c >= done && c < until) {
              if (c < A_OPS)
                copy_a(c, An, ka);
              else
                copy_b(c - A_OPS, Bn, kb);
              __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            }
          done = until;
        };
#pragma unroll
        for (int j = 0; j < G8_NJ; ++j) read_b(0, j);
        // (not the late units' yet: their registers hold the previous slice's)
        constexpr int AHEAD = UNITS - LATE < 2 ? UNITS - LATE : 2;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) read_a(u);
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * G8_NJ + 2 * AHEAD, 0);
        if constexpr (!FIRST) {
#pragma unroll
          for (int l = 0; l < LATE; ++l) {
            multiply(std::false_type{}, UNITS - LATE + l, late_sx[l], late_sw);
            __builtin_amdgcn_sched_group_barrier(0x008, kMfmas, 0);
            copies(1);
          }
        }
#pragma unroll
        for (int u = 0; u < UNITS - LATE; ++u) {
          // what is read during this unit: its share of the second half's weights, a later unit's rows
          int reads = 0;
          if (u < NB) {
#pragma unroll
            for (int j = 0; j < G8_NJ; ++j)
              if (j >= G8_NJ * u / NB && j < G8_NJ * (u + 1) / NB) {
                read_b(1, j);
                reads += 2;
              }
          }
          if (FIRST && u < NB)
            multiply(std::true_type{}, u, sx[u % (NB > 0 ? NB : 1)], sw);
          else
            multiply(std::false_type{}, u, sx[u % (NB > 0 ? NB : 1)], sw);
          if (u + AHEAD < UNITS) {
            read_a(u + AHEAD);
            reads += 2;
          }
          if (reads == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          if (reads == 4) __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
          if (reads == 6) __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
          if (reads == 10) __builtin_amdgcn_sched_group_barrier(0x100, 10, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, kMfmas, 0);
          copies(1);
        }
#pragma unroll
        for (int l = 0; l < LATE; ++l) late_sx[l] = sx[(UNITS - LATE + l) % NB];
        late_sw[0] = sw[0];
        late_sw[1] = sw[1];
      }
    };
    int g = t.rot;
    for (int done = 0; done < nk;) {
      const int len = min(4, nk - 4 * g);
      const bool last = done + len >= nk;
      uint32_t sx[MI], sw[2];
#pragma unroll
      for (int q = 0; q < SR; ++q) {
        uint32_t lower, upper;      // both halves' rows, in all lanes
        rows_swap32(s_cur[q], lower, upper);
        sx[2 * q] = lower;
        if (2 * q + 1 < MI) sx[2 * q + 1] = upper;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) sw[j] = __builtin_amdgcn_readlane(static_cast<int>(w_cur[j]), g);
      if constexpr (WIDE) {
        move_scales(sx, sw[0]);
        sw[0] = __builtin_amdgcn_readfirstlane(static_cast<int>(sw[0]));
      }
      if (done == 0 && !short_k) gather_a();
      g = last ? next_t.rot : (g + 1 < groups ? g + 1 : 0);
#pragma unroll
      for (int q = 0; q < SR; ++q) load_scale(q, last ? ns_row[q] : s_row[q], g);
      int q = 0;
      auto shift = [&]() {
#pragma unroll
        for (int i = 0; i < MI; ++i) sx[i] >>= 8;
#pragma unroll
        for (int j = 0; j < 2; ++j) sw[j] >>= 8;
        ++q;
        ++s;
      };
      if (done == 0) {
        step(std::true_type{}, sx, sw);
        shift();
      }
      while (q < len) {
        step(std::false_type{}, sx, sw);
        shift();
      }
      done += len;
    }
    if constexpr (NB > 0) late_units();
    take_scales();
    // every wave has read the tile's last slices: the weight slot takes the epilogue's scratch (the
    // next tile's first step refills it only after its own barrier)
    lds_barrier8();
    const uint32_t scratch = static_cast<uint32_t>(
        reinterpret_cast<uintptr_t>(b_ring + ((s + S::B_SLOTS - 1) % S::B_SLOTS) * S::B_BYTES));
    const int el = lane_here(), erow = el & 31, esel = el >> 5;
    if constexpr (MODE == UP) {
      // A pair block at a time: the activation and its rows' maxima over this wave's 64 columns, then the
      // codes, with the maximum of the two waves that share the rows.  All waves pass MI barriers, whatever
      // their blocks.
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        __builtin_amdgcn_sched_barrier(0);      // (one block's registers at a time)
        if constexpr (NB > 0) {
          float v[2][16];
          uint32_t lo = 0, hi = 0;
          const int in_tile = 32 * (S::WM * i + wm) + erow, row = t.row0 + in_tile;
          bool odd = false;      // infinities or NaN in the block
          if (i < NB) {
            float m = 0.0f, bad = 0.0f;
#pragma unroll
            for (int jj = 0; jj < 2; ++jj)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                v[jj][r] = silu_mul(acc[i < NB ? i : 0][jj][r], acc[i < NB ? i : 0][jj + 2][r]);
                m = fmaxf(m, fabsf(v[jj][r]));
                bad = fmaf(v[jj][r], 0.0f, bad);
              }
            odd = __any(bad != 0.0f);      // (NaN compares unequal)
            uint32_t mb = __float_as_uint(m);
            if (odd) {                     // the maximum of the finite values
              mb = 0;
#pragma unroll
              for (int jj = 0; jj < 2; ++jj)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                  const uint32_t b = __float_as_uint(v[jj][r]) & 0x7fffffffu;
                  mb = max(mb, b < 0x7f800000u ? b : 0u);
                }
            }
            rows_swap32(mb, lo, hi);
            asm volatile("ds_write_b32 %0, %1" ::"v"(scratch + 8u * in_tile + 4u * wn), "v"(max(lo, hi)) : "memory");
          }
          lds_barrier8();
          if (i < NB) {
            u32x2_t both;
            asm volatile("ds_read_b64 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(both) : "v"(scratch + 8u * in_tile) : "memory");
            const uint32_t byte = f8_scale_byte(max(both[0], both[1]));
            const float inv = f8_inverse(byte);
            const int kb = t.n0 / F8_BLOCK;
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
              uint32_t c[4];
#pragma unroll
              for (int g = 0; g < 4; ++g)
                c[g] = f8_pack4(v[jj][4 * g] * inv, v[jj][4 * g + 1] * inv, v[jj][4 * g + 2] * inv, v[jj][4 * g + 3] * inv);
              if (odd) {      // infinities and NaN: the one NaN code
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                  for (int h = 0; h < 4; ++h)
                    if ((__float_as_uint(v[jj][4 * g + h]) & 0x7fffffffu) >= 0x7f800000u)
                      c[g] = (c[g] & ~(0xffu << (8 * h))) | (0x7fu << (8 * h));
              }
              // a lane holds columns 8 g + 4 esel ..; with the wave's halves swapped the lower one holds
              // columns 0-15 of each row, the upper one 16-31
              const auto p = __builtin_amdgcn_permlane32_swap(c[0], c[2], false, false);
              const auto q = __builtin_amdgcn_permlane32_swap(c[1], c[3], false, false);
              if (row < t.row_end)
                *reinterpret_cast<u32x4_t*>(static_cast<uint8_t*>(a.out) + static_cast<size_t>(row) * N + t.n0 + 64 * wn +
                                            32 * jj + 16 * esel) = u32x4_t{p[0], p[1], q[0], q[1]};
            }
            if (row < t.row_end && wn == 0 && esel == 0)
              a.out_scale[(static_cast<size_t>(kb >> 2) * a.act_rows + row) * 4 + (kb & 3)] = static_cast<uint8_t>(byte);
          }
        } else {
          lds_barrier8();
        }
      }
    } else {
      OUT* const out = static_cast<OUT*>(a.out);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        __builtin_amdgcn_sched_barrier(0);      // (one block's registers at a time)
        {
          const int rb = t.row0 + 32 * (S::WM * i + wm);
          const uint32_t stage = scratch + wave * G8_STAGE;
#pragma unroll
          for (int j = 0; j < G8_NJ; j += sizeof(OUT) == 4 ? 1 : 2) {
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (sizeof(OUT) == 4) {
              const f32x16_t& c = acc[i][j];
#pragma unroll
              for (int g = 0; g < 4; ++g)
                lds_write128(stage_at(stage, erow, 2 * g + esel), c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]);
            } else {
#pragma unroll
              for (int jj = 0; jj < 2; ++jj) {
                const f32x16_t& c = acc[i][j + jj];
#pragma unroll
                for (int g = 0; g < 4; ++g)
                  lds_write64(stage_at(stage, erow, 4 * jj + g) + 8 * esel, pack_bf16x2(c[4 * g], c[4 * g + 1]),
                              pack_bf16x2(c[4 * g + 2], c[4 * g + 3]));
              }
            }
            store_staged<OUT, MODE == PLAIN>(rb, t.n0 + 128 * wn + 32 * j, t.row_end, N, out, stage);
          }
        }
      }
    }
  };
  for (int tile_i = 0; tile_i < n_my; ++tile_i) {
    const bool more = tile_i + 1 < n_my;
    if (more) next_t = tile_at(tile_i + 1);
    if (short_k) {
      ready_a();
      ready_b();
    } else {
      na_ready = nb_ready = more;
      if (more) {
        set_a(next_t);
        set_b(next_t);
      }
    }
    set_scales(next_t);
    // pair blocks of this wave that hold pairs: blocks wm, wm + WM, .. of the tile
    const int blocks = (t.row_end - t.row0 + 31) >> 5;
    const int nb = __builtin_amdgcn_readfirstlane(min(max(blocks - wm + S::WM - 1, 0) / S::WM, MI));
    switch (nb) {
      case 4:
        if constexpr (MI >= 4) tile(std::integral_constant<int, 4>{});
        break;
      case 3:
        if constexpr (MI >= 3) tile(std::integral_constant<int, 3>{});
        break;
      case 2:
        if constexpr (MI >= 2) tile(std::integral_constant<int, 2>{});
        break;
      case 1: tile(std::integral_constant<int, 1>{}); break;
      default: tile(std::integral_constant<int, 0>{}); break;
    }
    t = next_t;
  }
  wait_copies<0>();     // the last (unused) copies land before the workgroup's LDS is released
}

// ---- plain products of few tiles -------------------------------------------------------------------
// A product with fewer 256-column tiles than the GPU has CUs leaves most of them idle, and its time is
// its K loop's, slice after slice.  Here a workgroup has a small tile, 32 MI rows x 32 NJ columns, and its W
// waves take every W-th slice of K each, straight from global memory into the MFMAs' registers (whole
// 128-byte lines of rows, SLIM_AHEAD slices ahead: nothing to share, no barrier in the loop); their sums meet in
// LDS, added in wave order.  Bound by a load's latency: K = 4096 is four slices a wave.
constexpr int SLIM_AHEAD = 2;
constexpr int SLIM_PITCH = 65;      // floats between an accumulator's registers in LDS: no bank conflicts either way

template <int MI, int NJ, int W, class OUT>
__global__ __launch_bounds__(64 * W) void fp8_slim_kernel(Args8 a) {
  constexpr bool WIDE = sizeof(OUT) == 4;
  extern __shared__ __attribute__((aligned(16))) float slim_sums[];      // [W][MI][NJ][16][SLIM_PITCH]
  const int K = a.K, N = a.N, nk = K / G8_BK, groups = (nk + 3) / 4;
  int rows = a.sh_rows;
  if (a.n_rows != nullptr) rows = min(max(a.n_rows[0], 0), rows);
  const int m_tiles = (a.sh_rows + 32 * MI - 1) / (32 * MI);
  const int row0 = static_cast<int>(blockIdx.x) % m_tiles * 32 * MI, n0 = static_cast<int>(blockIdx.x) / m_tiles * 32 * NJ;
  if (row0 >= rows) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (rows and columns past the last are the last one's again, and not stored)
  const uint8_t *x[MI], *w[NJ];
  const uint32_t* xs[MI];
  static_assert(F8_BLOCK % (32 * NJ) == 0, "a tile's columns in one block of weights");
  const uint32_t* const ws = a.ss0 + static_cast<size_t>(n0 / F8_BLOCK) * groups;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int r = min(row0 + 32 * i + lane % 32, rows - 1);
    x[i] = a.x + static_cast<size_t>(r) * K + 32 * (lane / 32);
    xs[i] = a.x_scale + r;
  }
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int n = min(n0 + 32 * j + lane % 32, N - 1);
    w[j] = a.sw0 + static_cast<size_t>(n) * K + 32 * (lane / 32);
  }
  // A slice: lane l has bytes 32 (l / 32) .. of each half of its rows' 128 (of both operands alike)
  struct Slice {
    i32x4_t x[MI][4], w[NJ][4];
    uint32_t sx[MI], sw;
  } slice[SLIM_AHEAD];
  auto load = [&](Slice& f, int k) {
    k = min(k, nk - 1);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        f.x[i][q] = *reinterpret_cast<const i32x4_t*>(x[i] + static_cast<size_t>(k) * G8_BK + 64 * (q / 2) + 16 * (q % 2));
      f.sx[i] = xs[i][static_cast<size_t>(k >> 2) * a.x_rows];
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        f.w[j][q] = *reinterpret_cast<const i32x4_t*>(w[j] + static_cast<size_t>(k) * G8_BK + 64 * (q / 2) + 16 * (q % 2));
    }
    f.sw = ws[k >> 2];
  };
  f32x16_t acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x16_t{};
  auto multiply = [&](const Slice& f, int k) {
    const int shift = 8 * (k & 3);
    uint32_t rows_scale[MI], weights_scale = f.sw;      // (the tile's columns lie in one block of 128)
#pragma unroll
    for (int i = 0; i < MI; ++i) rows_scale[i] = f.sx[i];
    if constexpr (WIDE) move_scales(rows_scale, weights_scale);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const uint32_t sx = (rows_scale[i] >> shift) & 0xffu, sw = (weights_scale >> shift) & 0xffu;
          if constexpr (WIDE) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const i32x4_t &xv = f.x[i][2 * kk + q / 2], &wv = f.w[j][2 * kk + q / 2];
              const int at = 2 * (q % 2);
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(wv[at], wv[at + 1], __uint_as_float(sw << 23)),
                                                                  widen8(xv[at], xv[at + 1], __uint_as_float(sx << 23)),
                                                                  acc[i][j], 0, 0, 0);
            }
          } else {
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                __builtin_shufflevector(f.w[j][2 * kk], f.w[j][2 * kk + 1], 0, 1, 2, 3, 4, 5, 6, 7),
                __builtin_shufflevector(f.x[i][2 * kk], f.x[i][2 * kk + 1], 0, 1, 2, 3, 4, 5, 6, 7), acc[i][j], 0, 0, 0,
                static_cast<int>(sw), 0, static_cast<int>(sx));
          }
        }
  };
  if (wave < nk) {
#pragma unroll
    for (int d = 0; d < SLIM_AHEAD; ++d) load(slice[d], wave + d * W);
    for (int k = wave; k < nk; k += SLIM_AHEAD * W) {
#pragma unroll
      for (int d = 0; d < SLIM_AHEAD; ++d) {
        if (k + d * W < nk) multiply(slice[d], k + d * W);
        if (k + (d + SLIM_AHEAD) * W < nk) load(slice[d], k + (d + SLIM_AHEAD) * W);
      }
    }
  }
  // lane l, register r: row l % 32, column 8 (r / 4) + 4 (l / 32) + r % 4
  auto sums = [&](int v, int i, int j) { return slim_sums + ((v * MI + i) * NJ + j) * 16 * SLIM_PITCH; };
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) sums(wave, i, j)[r * SLIM_PITCH + lane] = acc[i][j][r];
  __syncthreads();
  OUT* const out = static_cast<OUT*>(a.out);
  for (int t = threadIdx.x; t < 1024 * MI * NJ; t += 64 * W) {      // neighbouring threads: neighbouring columns
    const int col = t % (32 * NJ), row = t / (32 * NJ), c = col % 32;
    if (row0 + row >= rows || n0 + col >= N) continue;
    const float* const at = sums(0, row / 32, col / 32) + ((c / 8) * 4 + c % 4) * SLIM_PITCH + row % 32 + 32 * ((c / 4) % 2);
    float sum = at[0];
#pragma unroll
    for (int v = 1; v < W; ++v) sum += at[v * MI * NJ * 16 * SLIM_PITCH];
    if constexpr (WIDE)
      out[static_cast<size_t>(row0 + row) * N + n0 + col] = sum;
    else
      out[static_cast<size_t>(row0 + row) * N + n0 + col] = f32_to_bf16(sum);
  }
}

// The tile shapes (pair rows x weight rows).  The activation's blocks of 128 columns need 256
// weight rows a tile (128 of gate, 128 of up).
using Tall = Shape8<4, 2, 3>;       // 256 x 256, 160 KB of LDS, one workgroup per CU
using Half = Shape8<2, 3, 3>;       // 128 x 256, 144 KB
using Quarter = Shape8<1, 3, 4>;    // 64 x 256, 152 KB

// Lets a kernel have `lds` bytes of LDS; set_on: a bit a device (the attribute is the device's own).
int allow_lds(const void* kernel, size_t lds, std::atomic<uint64_t>& set_on) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return REFLEX_ERR_LAUNCH;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if ((set_on.load(std::memory_order_relaxed) & bit) == 0) {
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds)) != hipSuccess)
      return REFLEX_ERR_LAUNCH;
    set_on.fetch_or(bit, std::memory_order_relaxed);
  }
  return REFLEX_OK;
}

template <int MI, int NJ, int W, class OUT>
int launch_slim(const Args8& a, hipStream_t s) {
  constexpr size_t lds = sizeof(float) * W * MI * NJ * 16 * SLIM_PITCH;
  static_assert(lds <= 160 * 1024, "LDS");
  auto* kernel = &fp8_slim_kernel<MI, NJ, W, OUT>;
  static std::atomic<uint64_t> set_on{0};
  const int rc = allow_lds(reinterpret_cast<const void*>(kernel), lds, set_on);
  if (rc != REFLEX_OK) return rc;
  const int tiles = (a.sh_rows + 32 * MI - 1) / (32 * MI) * ((a.N + 32 * NJ - 1) / (32 * NJ));
  hipLaunchKernelGGL(kernel, dim3(tiles), dim3(64 * W), lds, s, a);
  return launch_status();
}

template <Mode MODE, class S, bool BIG, class OUT>
int launch_as(const Args8& a, hipStream_t s) {
  auto* kernel = &fp8_gemm_kernel<MODE, S, BIG, OUT>;
  static std::atomic<uint64_t> set_on{0};
  const int rc = allow_lds(reinterpret_cast<const void*>(kernel), S::LDS, set_on);
  if (rc != REFLEX_OK) return rc;
  const int grid = (device_cus() + G8_XCDS - 1) / G8_XCDS * G8_XCDS;      // one workgroup per CU
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(S::THREADS), S::LDS, s, a);
  return launch_status();
}

// rows: the rows of an expert when all are loaded alike and every token takes its most.  What bounds a
// product of few rows is the weights' stream, which a deeper ring of weights keeps a little fuller; more rows
// need tall tiles, which read the weights once.  131072 x 2048 weights, bf16 results, us with 64 / 128 / 256 rows a
// tile: 64 rows 47.7 / 47.6 / 49.5, 128 rows 73 / 56 / 57, 256 rows 128 / 92 / 80, 512 rows 255 / 172 / 143.  64 experts
// of 3 x 2048 x 1024: 8 rows each at most 94 / 98 / 99, 64 rows 105 / 106 / 105, 128 rows 134 / 115 / 120, 256 rows
// 182 / 169 / 134, 512 rows 285 / 230 / 220.
template <Mode MODE, class OUT>
int launch_gemm8(const Args8& a, int rows, hipStream_t s) {
  if constexpr (MODE == PLAIN) {
    // Small tiles while they find a CU each (32 x 32: two to a CU).  2048 columns of K, bf16 / fp32 results, us:
    // 16 x 4096 9.8 / 9.9 in 32 x 32 tiles, 12.7 / 18.1 in 64 x 256; 256 x 2048 11.6 / 10.9, in 64 x 64 12.6 / 13.3,
    // in 256 x 256 26.8 / 46.6; 1024 x 1024 20.6 / 18.4, 12.8 / 14.1, 27.0 / 46.7; 64 x 16384 21.7 / 18.3, 13.2 / 14.4,
    // 15.4 / 21.9; 64 x 24576 31.5 / 25.4, 24.2 / 25.8, 15.7 / 22.8.
    const auto tiles = [&](int side) { return static_cast<long long>((rows + side - 1) / side) * ((a.N + side - 1) / side); };
    if (tiles(32) <= 2 * device_cus()) return launch_slim<1, 1, 8, OUT>(a, s);
    if (tiles(64) <= device_cus()) return launch_slim<2, 2, 4, OUT>(a, s);
  }
  if (static_cast<size_t>(a.x_rows) * static_cast<size_t>(a.K) >= (size_t(1) << 31))
    return launch_as<MODE, Tall, true, OUT>(a, s);
  // Half tiles too where whole ones would leave half of the CUs idle (1024 x 4096 x 2048 28.8 -> 20.0 us, 413 x 13071 x
  // 768 33.9 -> 21.3; a little beyond, 264 x 17745 x 1152, 140 tiles, 28.9)
  constexpr int BN = MODE == UP ? Tall::BROWS / 2 : Tall::BROWS;
  const bool half = static_cast<long long>(std::max(a.E, 1)) * ((rows + Tall::BM - 1) / Tall::BM) * ((a.N + BN - 1) / BN) <=
                    device_cus() / 2;
  if (rows <= Quarter::BM) return launch_as<MODE, Quarter, false, OUT>(a, s);
  if (rows <= Half::BM || half) return launch_as<MODE, Half, false, OUT>(a, s);
  return launch_as<MODE, Tall, false, OUT>(a, s);
}

const uint32_t* dwords(const uint8_t* p) { return reinterpret_cast<const uint32_t*>(p); }

int expected_rows(int T, int E, int cap, int sh_rows) {
  const int experts = std::min(E, cap);
  const int routed = experts > 0 ? std::min(T, (cap + experts - 1) / experts) : 0;
  return std::max(routed, E == 0 ? sh_rows : 0);
}

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
  return launch_gemm8<UP, uint8_t>(a, expected_rows(T, E, cap, sh.rows), s);
}

int launch_swiglu8_down(const int32_t* expert_offsets, const Fp8Weights& w, int T, int E, int d, int f, int cap,
                        const AlwaysOn8& sh, const uint8_t* act, uint16_t* y_sorted, hipStream_t s) {
  if (cap <= 0 && sh.rows <= 0) return REFLEX_OK;
  const int rows = cap + sh.rows;
  const Args8 a{act, dwords(act + swiglu8_act_bytes(rows, f)), nullptr, expert_offsets, w.w_down, nullptr,
                dwords(w.s_down), nullptr, sh.w.w_down, nullptr, dwords(sh.w.s_down), nullptr, E, f, d, rows, cap,
                sh.row0, sh.rows, nullptr, y_sorted, nullptr, 0};
  return launch_gemm8<DOWN, uint16_t>(a, expected_rows(T, E, cap, sh.rows), s);
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
  return out_type == REFLEX_TYPE_F32 ? launch_gemm8<PLAIN, float>(a, M, s) : launch_gemm8<PLAIN, uint16_t>(a, M, s);
}

}  // namespace rfx
