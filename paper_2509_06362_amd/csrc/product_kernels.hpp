// Products of rows with weights whose rows are channels, for one matrix (8-bit integers with scales) or for many, each with
// its own ragged group of rows (experts), with the gate in the epilogue.
//
// Both operands hold what is summed over along a row, so that a lane's 16 bytes of a row are an operand of the matrix units as
// they are, 8 elements of 16 bits or 16 of 8: every type goes through the same addresses, in bytes.  Which bytes of a row
// meet in which instruction does not matter as long as both operands agree.  The weights are the instructions' first operand:
// a lane then ends with four neighbouring channels of one row.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "gate.hpp"

namespace maaso {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

struct Int8 { int8_t bits; };  // the 8-bit integers, as a template's argument

template <typename T> struct Operand;
template <> struct Operand<__bf16> {
  using Sum = f32x4;
  static __device__ inline f32x4 mfma(u32x4 w, u32x4 a, f32x4 c) {
    return mfma_16x16x32(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, a), c);
  }
};
template <> struct Operand<_Float16> {
  using Sum = f32x4;
  static __device__ inline f32x4 mfma(u32x4 w, u32x4 a, f32x4 c) {
    return mfma_16x16x32(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, a), c);
  }
};
template <> struct Operand<Int8> {
  using Sum = i32x4;
  static __device__ inline i32x4 mfma(u32x4 w, u32x4 a, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, a), c, 0, 0, 0);
  }
};

struct ProductArgs {
  const char* a;
  const char* w;
  void* out;
  const float* a_scale;
  const float* w_scale;
  const float* bias;
  const int32_t* start;    // NULL: one group of all rows
  const int32_t* token;
  uint64_t a_stride, w_stride, expert_stride;  // bytes
  uint64_t out_stride;                         // elements
  uint32_t n_a, n_rows, n_experts, in_bytes, n_out, channels;  // channels: rows of an expert's weights
  uint32_t out_type;
  uint32_t col_tiles;
  bool wide;    // rows of out begin at multiples of 16 bytes
  bool turned;  // tiles begin at unlike steps
  uint32_t* status;
};

// The rows of one tile: `rows` rows of out from `begin` on (0: there is no such tile), of this expert.
struct RowTile {
  uint32_t expert, begin, rows;
};

__device__ inline uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// Inclusive sum / maximum over the lanes below.
__device__ inline uint32_t lanes_sum(uint32_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = (uint32_t)__shfl_up((int)v, d);
    v += (int)(threadIdx.x & 63u) >= d ? o : 0u;
  }
  return v;
}
__device__ inline uint32_t lanes_max(uint32_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = (uint32_t)__shfl_up((int)v, d);
    v = max(v, (int)(threadIdx.x & 63u) >= d ? o : 0u);
  }
  return v;
}

// 64 experts at a time, one to a lane: their rows [lo, hi) and the tiles of `Rows` rows up to and with each of them.
// A start out of order is taken as the nearest that is not.
template <uint32_t Rows> struct Groups {
  uint32_t base = 0, seen = 0, last = 0, lo = 0, hi = 0, upto = 0;
  bool bad = false;
  __device__ inline void look(const ProductArgs& a) {
    const uint32_t e = base + (threadIdx.x & 63u);
    const bool in = e < a.n_experts;
    const int32_t s0 = in ? a.start[e] : 0, s1 = in ? a.start[e + 1u] : 0;
    lo = (uint32_t)min(max(s0, 0), (int32_t)a.n_rows);
    hi = (uint32_t)min(max(s1, 0), (int32_t)a.n_rows);
    const bool off = in && (hi < lo || lo != (uint32_t)s0 || hi != (uint32_t)s1 || lo < last);
    if (__ballot(off)) {
      bad = true;
      lo = lanes_max(max(lo, last));
      hi = lanes_max(max(lo, hi));
    }
    last = (uint32_t)__builtin_amdgcn_readlane((int)hi, (int)min(63u, a.n_experts - 1u - base));
    if (!in) lo = hi = 0u;
    upto = seen + lanes_sum((hi - lo + Rows - 1u) / Rows);
    seen = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  }
  // The tile among the experts looked at; it is there: `tile` is below `seen`, and was not below what was seen before.
  __device__ inline RowTile take(uint32_t tile) const {
    const int l = (int)__builtin_ctzll(__ballot(tile < upto));
    const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)lo, l), end = (uint32_t)__builtin_amdgcn_readlane((int)hi, l);
    const uint32_t tiles = (end - first + Rows - 1u) / Rows, to = (uint32_t)__builtin_amdgcn_readlane((int)upto, l);
    const uint32_t begin = first + (tile - (to - tiles)) * Rows;
    return {base + (uint32_t)l, begin, min(Rows, end - begin)};
  }
};

template <uint32_t Rows> __device__ inline RowTile row_tile(const ProductArgs& a, uint32_t tile) {
  if (!a.start) return {0u, tile * Rows, tile * Rows < a.n_rows ? min(Rows, a.n_rows - tile * Rows) : 0u};
  Groups<Rows> g;
  for (; g.base < a.n_experts; g.base += 64u) {
    g.look(a);
    if (tile < g.seen) return g.take(tile);
  }
  return {0u, 0u, 0u};
}

// Whoever is first: starts out of order are told once, and by a block that would look at them all the same.
__device__ inline void check_starts(const ProductArgs& a) {
  if (!a.start) return;
  Groups<16u> g;
  for (; g.base < a.n_experts; g.base += 64u) g.look(a);
  if (g.bad && (threadIdx.x & 63u) == 0u) atomicOr(a.status, MAASO_INST_BAD_BOUND);
}

// The row of a that row `r` of out is made of; `ok`: there is one.
__device__ inline uint32_t source_row(const ProductArgs& a, uint32_t r, bool& ok) {
  const uint32_t t = a.token ? (uint32_t)a.token[r] : r;
  ok = t < a.n_a;
  return ok ? t : 0u;
}

// The first `left` of 16 bytes, the others zeros.
__device__ inline u32x4 first_bytes(u32x4 v, int left) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int keep = left - 4 * d;
    v[d] = keep >= 4 ? v[d] : keep <= 0 ? 0u : v[d] & ((1u << (8 * keep)) - 1u);
  }
  return v;
}

// 16 bytes from byte `at` of a row on, zeros from the row's end on.  (Rows begin at multiples of 16 bytes: what is read beside
// a row's last byte lies in the same 16.)
__device__ inline u32x4 row_bytes(const char* row, uint32_t at, uint32_t in_bytes) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(row + (at < in_bytes ? at : 0u));
  return first_bytes(v, (int)in_bytes - (int)at);
}

// N neighbouring numbers that begin anywhere.
template <int N> struct __attribute__((packed, aligned(4))) Floats { float v[N]; };

// What N neighbouring channels of an expert, from `col` on, are scaled by and raised by, gate and gated.
template <typename T, int N, bool Gated> struct Channels {
  static constexpr int kBoth = Gated ? 2 : 1;
  static constexpr bool kScaled = sizeof(T) == 1;
  float scale[kBoth][N], bias[kBoth][N];
  __device__ inline void take(const float* from, uint64_t at, uint32_t left, float none, float (&to)[N]) {
    if (!from) {
#pragma unroll
      for (int k = 0; k < N; ++k) to[k] = none;
    } else if (left >= (uint32_t)N) {
      const Floats<N> f = *reinterpret_cast<const Floats<N>*>(from + at);
#pragma unroll
      for (int k = 0; k < N; ++k) to[k] = f.v[k];
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) to[k] = (uint32_t)k < left ? from[at + k] : none;
    }
  }
  __device__ inline void load(const ProductArgs& a, uint32_t expert, uint32_t col) {
    const uint64_t at = (uint64_t)expert * a.channels + col;
#pragma unroll
    for (int h = 0; h < kBoth; ++h) {
      if constexpr (kScaled) take(a.w_scale, at + (uint64_t)h * a.n_out, a.n_out - col, 1.0f, scale[h]);
      take(a.bias, at + (uint64_t)h * a.n_out, a.n_out - col, 0.0f, bias[h]);
    }
  }
};

// N neighbouring channels of one row: scales, bias, gate, the one rounding.  (Adding the bias that is not there changes no number but -0.)
template <typename T, int N, bool Gated>
__device__ inline void finish(const ProductArgs& a, const Channels<T, N, Gated>& c, uint32_t row, float row_scale, uint32_t col, float (&y)[N], float (&up)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if constexpr (sizeof(T) == 1) y[k] = y[k] * row_scale * c.scale[0][k];
    y[k] += c.bias[0][k];
    if constexpr (Gated) {
      if constexpr (sizeof(T) == 1) up[k] = up[k] * row_scale * c.scale[Gated][k];
      y[k] = silu(y[k]) * (up[k] + c.bias[Gated][k]);
    }
  }
  const uint64_t to = (uint64_t)row * a.out_stride + col;
  const bool whole = a.wide && col + (uint32_t)N <= a.n_out;
  if (a.out_type == MAASO_FP32) {
    float* p = static_cast<float*>(a.out) + to;
    if (whole) {
#pragma unroll
      for (int k = 0; k < N; k += 4) *reinterpret_cast<f32x4*>(p + k) = (f32x4){y[k], y[k + 1], y[k + 2], y[k + 3]};
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (col + (uint32_t)k < a.n_out) p[k] = y[k];
    }
    return;
  }
  uint32_t pair[N / 2];
  if (a.out_type == MAASO_BF16) {
#pragma unroll
    for (int k = 0; k < N / 2; ++k) pair[k] = __builtin_bit_cast(uint32_t, narrow2<__bf16>(y[2 * k], y[2 * k + 1]));
  } else {
#pragma unroll
    for (int k = 0; k < N / 2; ++k) pair[k] = __builtin_bit_cast(uint32_t, narrow2<_Float16>(y[2 * k], y[2 * k + 1]));
  }
  uint16_t* p = static_cast<uint16_t*>(a.out) + to;
  if (whole) {
    if constexpr (N == 8) *reinterpret_cast<u32x4*>(p) = (u32x4){pair[0], pair[1], pair[2], pair[3]};
    else *reinterpret_cast<u32x2*>(p) = (u32x2){pair[0], pair[1]};
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (col + (uint32_t)k < a.n_out) p[k] = (uint16_t)(pair[k / 2] >> (16 * (k & 1)));
  }
}

// Few rows: the weights are read once, straight into registers, and what bounds it is that reading, or the latency of a launch and two loads
// (one row, 8 bits, 2048 to 4096: 4.0 us; 16 rows 4.6; in tiles 7.3).  A block is 16 rows by
// 16 channels, those that gate them beside them; its waves share what is summed over, 128 bytes of a row in turn, and their sums meet in
// shared memory, in the order of the waves.
template <typename T, bool Gated, int Waves>
__global__ void __launch_bounds__(64 * Waves) product_stream_kernel(ProductArgs a) {
  using Sum = typename Operand<T>::Sum;
  constexpr int kAhead = 4, kTiles = Gated ? 2 : 1;  // 128-byte steps whose loads are under way at once
  __shared__ Sum sums[Waves][kTiles][64];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64u, i = lane & 15u, g = lane / 16u;
  if (blockIdx.x == 0u && blockIdx.y == 0u && wave == 0u) check_starts(a);
  const RowTile t = row_tile<16>(a, blockIdx.y);
  if (t.rows == 0u) return;
  const uint32_t n0 = blockIdx.x * 16u;
  bool ok;
  const uint32_t source = source_row(a, t.begin + (i < t.rows ? i : 0u), ok);
  const char* ap = a.a + source * a.a_stride;
  const char* wp[kTiles];
#pragma unroll
  for (int n = 0; n < kTiles; ++n) wp[n] = a.w + t.expert * a.expert_stride + (min(n0 + i, a.n_out - 1u) + n * a.n_out) * a.w_stride;
  Sum sum[kTiles] = {};
  const uint32_t whole = a.in_bytes / 128u, steps = (a.in_bytes + 127u) / 128u;
  uint32_t at = wave;
  u32x4 wv[kAhead][kTiles][2], av[kAhead][2];
  auto multiply = [&]() {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int n = 0; n < kTiles; ++n) sum[n] = Operand<T>::mfma(wv[u][n][h], av[u][h], sum[n]);
  };
  for (; at + (kAhead - 1) * Waves < whole; at += kAhead * Waves) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t byte = (at + u * Waves) * 128u + g * 32u + h * 16u;
#pragma unroll
        for (int n = 0; n < kTiles; ++n) wv[u][n][h] = *reinterpret_cast<const u32x4*>(wp[n] + byte);
        av[u][h] = *reinterpret_cast<const u32x4*>(ap + byte);
      }
    multiply();
  }
  if (at < steps) {  // what is left, all of it under way at once; bytes from the rows' end on are zeros in both
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t byte = (at + u * Waves) * 128u + g * 32u + h * 16u;
#pragma unroll
        for (int n = 0; n < kTiles; ++n) wv[u][n][h] = row_bytes(wp[n], byte, a.in_bytes);
        av[u][h] = row_bytes(ap, byte, a.in_bytes);
      }
    multiply();
  }
#pragma unroll
  for (int n = 0; n < kTiles; ++n) sums[wave][n][lane] = sum[n];
  __syncthreads();
  if (wave != 0u) return;
  Sum y[kTiles];
#pragma unroll
  for (int n = 0; n < kTiles; ++n) {
    y[n] = sums[0][n][lane];
#pragma unroll
    for (int w = 1; w < Waves; ++w) y[n] += sums[w][n][lane];
  }
  const uint32_t col = n0 + g * 4u;
  if (i >= t.rows || col >= a.n_out) return;
  if (!ok) {
    atomicOr(a.status, MAASO_INST_BAD_ROW);
    return;
  }
  float yf[4], uf[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    yf[k] = (float)y[0][k];
    uf[k] = Gated ? (float)y[kTiles - 1][k] : 0.0f;
  }
  Channels<T, 4, Gated> c;
  c.load(a, t.expert, col);
  finish<T, 4, Gated>(a, c, t.begin + i, a.a_scale ? a.a_scale[source] : 1.0f, col, yf, uf);
}

// Waits until no more than N of this wave's loads to shared memory are under way, its other accesses to shared memory are done, and all
// waves have come here.
template <uint32_t N> __device__ inline void meet() {
  static_assert(N < 64u, "the counter has six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// ... of the steps of Loads loads that are under way, no more than `steps`, at most Most.
template <uint32_t Loads, uint32_t Most> __device__ inline void meet_behind(uint32_t steps) {
  if constexpr (Most == 0u) {
    meet<0>();
  } else {
    if (steps >= Most) meet<Most * Loads>();
    else meet_behind<Loads, Most - 1u>(steps);
  }
}

// More rows.  In the largest tiles matrix units are busy 53 % of a launch (8 bits, 8192 x 4096 x 8192, gated: 247 us, 2220 T/s, where the library's plain
// product of 8192 cubed reaches 2060) or 64 % (16 bits, 8192 cubed: 829 us, 1330 T/s, the library 671 and 84 %); 16 bits, 8192 x 2048 x 8192
// 243 us, 1130 T/s.  The 829 us are 705 without the loads, 798 without the reads of shared memory, 626 without both, 646 on another card without the barrier as well:
// loads are what a step waits for.  Begin and end of a tile are 13 us of 61 at 4096 bytes.  The largest tiles have 14 registers too few: the rows' ends, which whole
// steps do without, find their addresses in scratch and are brought one by one (8192 x 4104 x 8192 264 us, 4096 236).  Slower were four waves of 128 by 128 (3 %), steps of
// 64 bytes in three to five stages (7 to 30 %, half lines), blocks that go from tile to tile (12 %, registers), lines brought to the cache ahead (8 %).
// A block is kRows rows by kCols channels, a wave MI by NI times 16 of each.  Steps of 128 bytes of both come to shared
// memory asynchronously, Stages of them under way or in use.  A step is two halves: while one is multiplied the operands of the next
// are read, and the waves meet between the halves, where their operands lie in registers already; there a step's place becomes free for the step
// Stages later.  A row's eight pieces of 16 bytes lie crossed with the row's lowest three bits, so that reads of one piece of neighbouring
// rows meet different banks.
template <typename T, int WM, int WN, int MI, int NI, int Stages, bool Gated>
__global__ void __launch_bounds__(64 * WM * WN, Stages * (WM * MI + WN * NI) * 2 <= 80 ? 2 : 1) product_tile_kernel(ProductArgs a) {
  using Sum = typename Operand<T>::Sum;
  constexpr uint32_t kWaves = WM * WN, kRows = WM * MI * 16, kCols = WN * NI * 16, kStage = (kRows + kCols) * 128;
  constexpr uint32_t kALoads = kRows / 8 / kWaves, kBLoads = kCols / 8 / kWaves, kLoads = kALoads + kBLoads;
  constexpr int H = Gated ? NI / 2 : NI;  // channel tiles of a wave's outputs
  constexpr uint32_t kOut = WN * H * 16, kAcross = 8, kTwo = H % 2 ? 1 : 2;
  static_assert(kRows % (8 * kWaves) == 0 && kCols % (8 * kWaves) == 0 && (!Gated || NI % 2 == 0), "whole loads, whole gates");
  static_assert(Stages >= 2 && (Stages - 1) * kLoads < 64, "loads under way that can be counted");
  __shared__ __attribute__((aligned(1024))) char lds[Stages * kStage];
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x / 64u), i = lane & 15u, g = lane / 16u;
  const uint32_t wm = wave / WN, wn = wave % WN;
  if (blockIdx.x == 0u && wave == 0u) check_starts(a);

  // Which tile: those of one eighth of the list run on one die, neighbours of up to kAcross row tiles at once, so that the die's
  // cache holds what they share.
  uint32_t tiles_down = (a.n_rows + kRows - 1u) / kRows;
  Groups<kRows> groups;
  if (a.start) {
    for (;; groups.base += 64u) {
      groups.look(a);
      if (groups.base + 64u >= a.n_experts) break;
    }
    tiles_down = groups.seen;
  }
  const uint32_t tiles = tiles_down * a.col_tiles, share = (tiles + 7u) / 8u;
  const uint32_t at = (blockIdx.x & 7u) * share + blockIdx.x / 8u;
  if (blockIdx.x / 8u >= share || at >= tiles) return;
  const uint32_t band = at / (kAcross * a.col_tiles), in_band = at - band * kAcross * a.col_tiles, high = min(kAcross, tiles_down - band * kAcross);
  const uint32_t col_tile = in_band / high, down = band * kAcross + in_band % high;
  const RowTile t = a.start && a.n_experts <= 64u ? groups.take(down) : row_tile<kRows>(a, down);
  if (t.rows == 0u) return;
  const uint32_t n0 = col_tile * kOut;

  const char* from[kLoads];  // a's, then w's
  const uint32_t piece = ((lane & 7u) ^ (lane / 8u)) * 16u;
#pragma unroll
  for (uint32_t q = 0; q < kALoads; ++q) {
    const uint32_t r = (wave * kALoads + q) * 8u + lane / 8u;
    bool ok;
    from[q] = a.a + source_row(a, t.begin + (r < t.rows ? r : 0u), ok) * a.a_stride + piece;
  }
  const char* weights = a.w + t.expert * a.expert_stride;
#pragma unroll
  for (uint32_t q = 0; q < kBLoads; ++q) {
    // Row p of a wave's channels lies where its sums come out beside their neighbours': a lane of the matrix unit's result has four
    // rows of each tile, and those of two tiles are to be eight channels in a row, those of four lanes then 64 bytes of 16-bit outputs.
    const uint32_t b = (wave * kBLoads + q) * 8u + lane / 8u, p = b % (NI * 16u), n = p / 16u, r = p % 16u;
    const uint32_t c = n0 + b / (NI * 16u) * (H * 16u) + n % H / kTwo * (kTwo * 16u) + r / 4u * (kTwo * 4u) + n % H % kTwo * 4u + r % 4u;
    from[kALoads + q] = weights + (min(c, a.n_out - 1u) + (Gated && n >= (uint32_t)H ? a.n_out : 0u)) * a.w_stride + piece;
  }

  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const uint32_t whole = a.in_bytes / 128u, steps = (a.in_bytes + 127u) / 128u;
  // Written out, because the compiler would have every later read of shared memory wait for it.  (m0 is named as changed, so that none of the
  // compiler's own uses of it, from its setting on, has this between; that it warns of, as of any reserved register.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  auto async16 = [&](const char* p, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_base + to), "v"(p) : "memory", "m0");
  };
#pragma clang diagnostic pop
  auto place_of = [&](uint32_t q) { return q < kALoads ? (wave * kALoads + q) * 1024u : kRows * 128u + (wave * kBLoads + (q - kALoads)) * 1024u; };
  // Many weights and few rows wait for memory, and rows a power of two apart have every block read the same channels at a time: a tile
  // begins where it lies in the list and goes round.  8 experts of 8192 channels of 2048 elements in 16 bits, 64 rows 59 to 50.5 us, 5.3 TB/s; 512
  // rows 73 to 61; the largest tiles, which wait for the matrix unit, are 2 % slower so.
  constexpr bool kTurns = MI * NI <= 16;
  const uint32_t turned = kTurns && a.turned && whole ? (col_tile * 5u + t.expert * 3u) % whole : 0u;
  auto step_at = [&](uint32_t step) {
    if constexpr (!kTurns) return step;
    const uint32_t to = step + turned;
    return to >= whole ? to - whole : to;
  };
  // (Rows that are not there are not brought, where every wait is for all that is under way: what lies in their place meets no sum that is kept.)
  constexpr bool kSkips = Stages == 2;
  auto bring = [&](uint32_t step, uint32_t q) {
    if (kSkips && q < kALoads && (wave * kALoads + q) * 8u >= t.rows) return;
    async16(from[q] + step_at(step) * 128u, step % Stages * kStage + place_of(q));
  };
  auto bring_end = [&](uint32_t step) {  // the rows' end lies in this step: zeros behind it in both
    for (uint32_t q = 0; q < kLoads; ++q)
      *reinterpret_cast<u32x4*>(lds + step % Stages * kStage + place_of(q) + lane * 16u) = row_bytes(from[q] - piece, step * 128u + piece, a.in_bytes);
  };

  const uint32_t row_at = (wm * MI * 16u + i) * 128u, col_at = kRows * 128u + (wn * NI * 16u + i) * 128u;
  const uint32_t half_at[2] = {(g ^ (i & 7u)) * 16u, ((4u + g) ^ (i & 7u)) * 16u};
  u32x4 av[2][MI], bv[2][NI];
  auto read = [&](uint32_t step, int half, int k) {  // operand k of both
    const char* at = lds + step % Stages * kStage + half_at[half];
    if (k < NI) bv[half][k] = *reinterpret_cast<const u32x4*>(at + col_at + k * 2048);
    if (k < MI) av[half][k] = *reinterpret_cast<const u32x4*>(at + row_at + k * 2048);
  };
  Sum sum[MI][NI] = {};
  auto multiply = [&](int half, int m) {
#pragma unroll
    for (int n = 0; n < NI; ++n) sum[m][n] = Operand<T>::mfma(bv[half][n], av[half][m], sum[m][n]);
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr int kReads = MI > NI ? MI : NI;

#pragma unroll
  for (uint32_t s = 0; s < (uint32_t)Stages; ++s) {
    if (s < whole) {
#pragma unroll
      for (uint32_t q = 0; q < kLoads; ++q) bring(s, q);
    } else if (s < steps) {
      bring_end(s);
    }
  }
  if (kSkips && (wave * kALoads + kALoads - 1u) * 8u >= t.rows) meet<0>();  // (fewer loads a step than are counted)
  else meet_behind<kLoads, Stages - 1>(steps - 1u);
  if (wm * MI * 16u >= t.rows) {  // none of this wave's rows are there: it brings its share and leaves the matrix unit to the others
    for (uint32_t step = 0; step + 1u < steps; ++step) {
      meet_behind<kLoads, Stages - 2>(steps - 2u - step);
      const uint32_t next = step + Stages;
      if (next < whole) {
#pragma unroll
        for (uint32_t q = 0; q < kLoads; ++q) bring(next, q);
      } else if (next < steps) {
        bring_end(next);
      }
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < kReads; ++k) read(0u, 0, k);
  for (uint32_t step = 0; step < steps; ++step) {
#pragma unroll
    for (int m = 0; m < MI; ++m) {
#pragma unroll
      for (int k = m * kReads / MI; k < (m + 1) * kReads / MI; ++k) read(step, 1, k);
      multiply(0, m);
    }
    if (step + 1u < steps) meet_behind<kLoads, Stages - 2>(steps - 2u - step);
    const uint32_t next = step + Stages;
    if (next >= whole && next < steps) bring_end(next);
#pragma unroll
    for (int m = 0; m < MI; ++m) {
#pragma unroll
      for (int k = m * kReads / MI; k < (m + 1) * kReads / MI; ++k) read(step + 1u, 0, k);  // (behind the last step what is read is not used)
      if (next < whole) {
#pragma unroll
        for (uint32_t q = m * kLoads / MI; q < (m + 1) * kLoads / MI; ++q) bring(next, q);
      }
      multiply(1, m);
    }
  }
  bool ok[MI];
  float row_scale[MI];
#pragma unroll
  for (int m = 0; m < MI; ++m) {
    const uint32_t r = wm * MI * 16u + m * 16u + i;
    ok[m] = r < t.rows;
    bool there = true;
    const uint32_t source = source_row(a, t.begin + (ok[m] ? r : 0u), there);
    row_scale[m] = sizeof(T) == 1 && a.a_scale ? a.a_scale[source] : 1.0f;
    if (ok[m] && !there) {
      ok[m] = false;
      atomicOr(a.status, MAASO_INST_BAD_ROW);
    }
  }
#pragma unroll
  for (int n = 0; n < H; n += (int)kTwo) {
    const uint32_t col = n0 + wn * (H * 16u) + (uint32_t)n * 16u + g * (kTwo * 4u);
    if (col >= a.n_out) continue;
    Channels<T, 4 * (int)kTwo, Gated> c;
    c.load(a, t.expert, col);
#pragma unroll
    for (int m = 0; m < MI; ++m) {
      if (!ok[m]) continue;
      float y[4 * kTwo], up[4 * kTwo];
#pragma unroll
      for (int k = 0; k < 4 * (int)kTwo; ++k) {
        y[k] = (float)sum[m][n + k / 4][k % 4];
        up[k] = Gated ? (float)sum[m][n + k / 4 + (Gated ? H : 0)][k % 4] : 0.0f;
      }
      finish<T, 4 * (int)kTwo, Gated>(a, c, t.begin + wm * MI * 16u + m * 16u + i, row_scale[m], col, y, up);
    }
  }
}

}  // namespace maaso
