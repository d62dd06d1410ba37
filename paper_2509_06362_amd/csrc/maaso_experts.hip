// Host side of the products, the experts and the rows in 8 bits (include/maaso_instance.h): argument validation, launch shapes.
#include "../../include/maaso_instance.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "instance_host.hpp"
#include "product_forms.hpp"
#include "product_kernels.hpp"
#include "route_kernels.hpp"
#include "rows_kernels.hpp"

using namespace maaso;

namespace {

// A launch holds fewer than 2^32 threads.  Rows beyond kPieceRows of one launch, and threads beyond kPieceThreads, go to another, and so do tokens that are
// chosen for alone; tokens that are put in order cannot (16 threads to a token), and channels have a launch's x to themselves (16 threads to a channel).
constexpr uint32_t kPieceRows = 1u << 22, kMostTokens = (1u << 26) - 1u, kMostOut = (1u << 27) - 1u;
constexpr uint64_t kPieceThreads = 1u << 30;

bool whole16(uint64_t elements, uint64_t size) { return elements % (16u / size) == 0; }

template <typename T, int Form, int Threads, int Held>
void launch_quantize_held(const QuantizeArgs& a, hipStream_t s) {
  constexpr uint32_t kRows = Threads == 64 ? 4u : 1u;
  hipLaunchKernelGGL((quantize_kernel<T, Form, Threads, Held>), dim3((a.n + kRows - 1u) / kRows), dim3(Threads == 64 ? 256 : Threads), 0, s, a);
}

template <typename T, int Form, int Threads>
void launch_quantize_threads(const QuantizeArgs& a, hipStream_t s) {
  const uint32_t turns = (a.width + 8u * Threads - 1u) / (8u * Threads);
  if (turns == 1u) launch_quantize_held<T, Form, Threads, 1>(a, s);
  else if (turns == 2u) launch_quantize_held<T, Form, Threads, 2>(a, s);
  else launch_quantize_held<T, Form, Threads, 4>(a, s);
}

// Threads to a row: a wave where there are many short rows (8192 rows of 1024, 16 bits, 6.2 us for 9.2 by 256 threads), 1024 where there are
// few (one row of 8192 3.4 for 4.2), 512 where the norm's weight takes registers as well (2000 rows of 8192 13.6 for 16.4); else 256 (8000 rows of 4096
// with a norm 25.0, 3.9 TB/s, by 128 threads 29.3; without 4.9 TB/s).
template <typename T, int Form>
void launch_quantize_form(const QuantizeArgs& a, uint32_t n_cu, hipStream_t s) {
  if (a.width <= 1024u && a.n >= 1024u) launch_quantize_threads<T, Form, 64>(a, s);
  else if (a.width > 2048u && a.n <= n_cu) launch_quantize_threads<T, Form, 1024>(a, s);
  else if (Form == MAASO_ROWS_NORM && a.width > 4096u) launch_quantize_threads<T, Form, 512>(a, s);
  else launch_quantize_threads<T, Form, 256>(a, s);
}

template <typename T>
void launch_quantize(uint32_t form, const QuantizeArgs& a, uint32_t n_cu, hipStream_t s) {
  if (form == MAASO_ROWS_PLAIN) launch_quantize_form<T, MAASO_ROWS_PLAIN>(a, n_cu, s);
  else if (form == MAASO_ROWS_NORM) launch_quantize_form<T, MAASO_ROWS_NORM>(a, n_cu, s);
  else launch_quantize_form<T, MAASO_ROWS_GATED>(a, n_cu, s);
}

// What a product's arguments have to be, of one matrix and of experts alike.
int check_product(const maaso_product* p) {
  if (p->type != MAASO_INT8 && p->type != MAASO_BF16 && p->type != MAASO_FP16) return MAASO_E_INVALID_ARG;
  if (p->out_type > MAASO_FP32 || (p->type != MAASO_INT8 && p->out_type != MAASO_FP32 && p->out_type != p->type)) return MAASO_E_INVALID_ARG;
  if (p->type != MAASO_INT8 && (p->a_scale || p->w_scale)) return MAASO_E_INVALID_ARG;
  if (p->n_in == 0 || p->n_in > MAASO_PRODUCT_MAX_IN || p->n_out == 0 || p->n_out > kMostOut) return MAASO_E_SHAPE;
  const uint64_t size = element_size(p->type), channels = (uint64_t)p->n_out * (p->gated ? 2u : 1u);
  if (p->n_a > 1u && (!whole16(p->a_stride, size) || p->a_stride < p->n_in)) return MAASO_E_SHAPE;
  if (channels > 1u && (!whole16(p->w_stride, size) || p->w_stride < p->n_in)) return MAASO_E_SHAPE;
  if (!aligned(p->a, 16) || !aligned(p->w, 16) || !aligned(p->out, element_size(p->out_type))) return MAASO_E_SHAPE;
  return MAASO_OK;
}

ProductArgs product_args(const maaso_instance* inst, const maaso_product* p, uint32_t n_rows) {
  const uint64_t size = element_size(p->type), out_size = element_size(p->out_type);
  ProductArgs a{};
  a.a = static_cast<const char*>(p->a); a.w = static_cast<const char*>(p->w); a.out = p->out;
  a.a_scale = p->a_scale; a.w_scale = p->w_scale; a.bias = p->bias;
  a.a_stride = p->a_stride * size; a.w_stride = p->w_stride * size; a.out_stride = p->out_stride;
  a.n_a = p->n_a; a.n_rows = n_rows; a.n_experts = 1u;
  a.in_bytes = p->n_in * (uint32_t)size; a.n_out = p->n_out; a.channels = p->n_out * (p->gated ? 2u : 1u);
  a.out_type = p->out_type;
  a.wide = aligned(p->out, 16) && (n_rows <= 1u || p->out_stride * out_size % 16u == 0u);
  a.status = inst->status;
  return a;
}

// Row tiles of `rows` rows that there can be.
uint64_t most_tiles(const ProductArgs& a, uint32_t rows) {
  return a.start ? a.n_rows / rows + std::min(a.n_experts, a.n_rows) : (a.n_rows + rows - 1u) / rows;
}

template <typename T, bool Gated>
int launch_stream(ProductArgs& a, hipStream_t s) {
  const uint64_t down = most_tiles(a, 16u);
  if (down > 65535u) return MAASO_E_SHAPE;
  hipLaunchKernelGGL((product_stream_kernel<T, Gated, 4>), dim3((a.n_out + 15u) / 16u, (uint32_t)down), dim3(256), 0, s, a);
  return launched();
}

template <typename T, int WM, int WN, int MI, int NI, int Stages, bool Gated>
int launch_tiles(ProductArgs& a, hipStream_t s) {
  const uint32_t cols = WN * NI * 16u / (Gated ? 2u : 1u);
  a.col_tiles = (a.n_out + cols - 1u) / cols;
  const uint64_t most = (most_tiles(a, WM * MI * 16u) * a.col_tiles + 7u) / 8u * 8u;
  if (most * (64u * WM * WN) > 0xffffffffull) return MAASO_E_SHAPE;
  hipLaunchKernelGGL((product_tile_kernel<T, WM, WN, MI, NI, Stages, Gated>), dim3((uint32_t)most), dim3(64 * WM * WN), 0, s, a);
  return launched();
}

template <typename T, bool Gated>
int launch_product(ProductArgs& a, uint32_t n_cu, hipStream_t s) {
  const ProductShape shape{a.n_rows, a.n_experts, a.channels, a.in_bytes, a.start != nullptr};
  a.turned = begins_unlike(shape);
  switch (product_form(shape, n_cu)) {
    case kStream: return launch_stream<T, Gated>(a, s);
    case kTiles64: return launch_tiles<T, 2, 2, 2, 2, 4, Gated>(a, s);
    case kTiles128Four: return launch_tiles<T, 2, 2, 4, 4, 4, Gated>(a, s);
    case kTiles128Two: return launch_tiles<T, 2, 2, 4, 4, 2, Gated>(a, s);
    default: return launch_tiles<T, 2, 4, 8, 4, 2, Gated>(a, s);
  }
}

template <typename T>
int launch_product(ProductArgs& a, bool gated, uint32_t n_cu, hipStream_t s) {
  return gated ? launch_product<T, true>(a, n_cu, s) : launch_product<T, false>(a, n_cu, s);
}

int launch_product(uint32_t type, ProductArgs& a, bool gated, uint32_t n_cu, hipStream_t s) {
  if (type == MAASO_INT8) return launch_product<Int8>(a, gated, n_cu, s);
  if (type == MAASO_BF16) return launch_product<__bf16>(a, gated, n_cu, s);
  return launch_product<_Float16>(a, gated, n_cu, s);
}

// The launches.  One, by one block, for a handful of tokens; choosing by small blocks all over the card and one block for the order while that has
// some two thousand choices; beyond that counts by chunks, their sums, and places by chunks.  256 experts, 8 chosen, with a bias, us by one block, by two
// launches, by three: 16 tokens 8.8, 10.3, 17; 64 tokens 13.2, 10.6, 17; 256 tokens 41, 12.6, 17; 512 tokens -, 20.3, 17.3; 64 experts, 6 chosen,
// 64 tokens 5.4, 6.4, 9; 512 tokens -, 12.3, 9.5; 8 experts, 2 chosen, 512 tokens -, 6.7, 9.0; 1024 tokens -, 10.6, 8.8.
bool one_block(const RouteArgs& a, uint32_t held) { return a.start && a.n <= kOneBlock / held; }
uint32_t order_room(const RouteArgs& a) { return a.n_experts * ((a.n + 31u) / 32u + 1u) * 4u; }
bool one_order(const RouteArgs& a) { return a.n <= kOrderTokens && a.n * a.k <= kOrderChoices && order_room(a) <= kOrderRoom; }

template <typename T, int Lanes, int Quads, bool Biased>
void launch_route(const RouteArgs& a, hipStream_t s) {
  if (one_block(a, Quads * Lanes / 16)) {
    hipLaunchKernelGGL((route_kernel<T, Lanes, Quads, Biased>), dim3(1), dim3(1024), order_room(a), s, a);
    return;
  }
  if (a.before) {
    hipLaunchKernelGGL((route_choose_kernel<T, Lanes, Quads, Biased>), dim3(a.chunks), dim3(1024), 0, s, a);
  } else {
    for (uint32_t first = 0; first < a.n; first += kPieceRows) {
      RouteArgs piece = a;
      piece.logits = static_cast<const T*>(a.logits) + first * a.stride;
      piece.expert = a.expert + (uint64_t)first * a.k;
      piece.weight = a.weight + (uint64_t)first * a.k;
      piece.n = std::min(a.n - first, kPieceRows);
      hipLaunchKernelGGL((route_choose_kernel<T, Lanes, Quads, Biased>), dim3((piece.n + 256u / Lanes - 1u) / (256u / Lanes)), dim3(256), 0, s, piece);
    }
  }
  if (!a.start) return;
  if (!a.before) {
    hipLaunchKernelGGL(route_order_kernel, dim3(1), dim3(1024), order_room(a), s, a);
    return;
  }
  hipLaunchKernelGGL(route_before_kernel, dim3((a.n_experts + 15u) / 16u), dim3(1024), 0, s, a);
  hipLaunchKernelGGL(route_place_kernel, dim3(a.chunks), dim3(1024), 0, s, a);
}

template <typename T, bool Biased>
void launch_route(const RouteArgs& a, hipStream_t s) {
  if (a.n_experts <= 64u) launch_route<T, 16, 1, Biased>(a, s);
  else if (a.n_experts <= 128u) launch_route<T, 16, 2, Biased>(a, s);
  else if (a.n_experts <= 256u) launch_route<T, 16, 4, Biased>(a, s);
  else if (a.n_experts <= 512u) launch_route<T, 32, 4, Biased>(a, s);
  else launch_route<T, 64, 4, Biased>(a, s);
}

template <typename T>
void launch_route(const RouteArgs& a, hipStream_t s) {
  if (a.bias) launch_route<T, true>(a, s);
  else launch_route<T, false>(a, s);
}

}  // namespace

extern "C" {

int maaso_rows_quantize(maaso_instance* inst, const maaso_rows_quantize_args* p, void* hip_stream) {
  if (!inst || !p) return MAASO_E_INVALID_ARG;
  if (p->type > MAASO_FP32 || p->form > MAASO_ROWS_GATED || (p->weight && p->form != MAASO_ROWS_NORM)) return MAASO_E_INVALID_ARG;
  if (p->width == 0 || p->width > 0x3fffffffu) return MAASO_E_SHAPE;
  if (p->n == 0) return MAASO_OK;
  if (p->n > 0x7fffffffu) return MAASO_E_SHAPE;
  if (!p->x || !p->q || !p->scale) return MAASO_E_INVALID_ARG;
  if (p->form == MAASO_ROWS_NORM && (!(p->eps >= 0.0f) || !std::isfinite(p->eps))) return MAASO_E_INVALID_ARG;
  const uint64_t size = element_size(p->type), elements = (uint64_t)p->width * (p->form == MAASO_ROWS_GATED ? 2u : 1u);
  if (!aligned(p->x, size) || !aligned(p->q, 16) || !aligned(p->weight, size)) return MAASO_E_SHAPE;
  if (p->n > 1u && (p->q_stride % 16u || p->x_stride < elements || p->q_stride < p->width)) return MAASO_E_SHAPE;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  for (uint64_t first = 0; first < p->n; first += kPieceRows) {
    const QuantizeArgs a{static_cast<const char*>(p->x) + first * p->x_stride * size, p->weight, p->q + first * p->q_stride, p->scale + first,
                         p->x_stride, p->q_stride, (uint32_t)std::min<uint64_t>(p->n - first, kPieceRows), p->width, p->eps};
    if (p->type == MAASO_BF16) launch_quantize<__bf16>(p->form, a, (uint32_t)inst->n_cu, s);
    else if (p->type == MAASO_FP16) launch_quantize<_Float16>(p->form, a, (uint32_t)inst->n_cu, s);
    else launch_quantize<float>(p->form, a, (uint32_t)inst->n_cu, s);
  }
  return launched();
}

int maaso_scaled_product(maaso_instance* inst, const maaso_product* p, void* hip_stream) {
  if (!inst || !p) return MAASO_E_INVALID_ARG;
  if (p->type != MAASO_INT8) return MAASO_E_INVALID_ARG;
  if (const int rc = check_product(p)) return rc;
  if (p->n_a == 0) return MAASO_OK;
  if (!p->a || !p->w || !p->out) return MAASO_E_INVALID_ARG;
  if (p->n_a > 0x7fffffffu || (p->n_a > 1u && p->out_stride < p->n_out)) return MAASO_E_SHAPE;
  ProductArgs a = product_args(inst, p, p->n_a);
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  return launch_product(p->type, a, p->gated != 0u, (uint32_t)inst->n_cu, s);
}

int maaso_expert_product(maaso_instance* inst, const maaso_expert_product_args* p, void* hip_stream) {
  if (!inst || !p) return MAASO_E_INVALID_ARG;
  if (const int rc = check_product(&p->product)) return rc;
  if (p->n_experts == 0 || p->n_experts > MAASO_EXPERT_MAX) return MAASO_E_SHAPE;
  if (p->n_rows == 0) return MAASO_OK;
  if (!p->product.a || !p->product.w || !p->product.out || !p->start || p->product.n_a == 0) return MAASO_E_INVALID_ARG;
  if (p->n_rows > 0x7fffffffu || p->product.n_a > 0x7fffffffu || (p->n_rows > 1u && p->product.out_stride < p->product.n_out)) return MAASO_E_SHAPE;
  const uint64_t size = element_size(p->product.type), channels = (uint64_t)p->product.n_out * (p->product.gated ? 2u : 1u);
  if (p->n_experts > 1u && (!whole16(p->expert_stride, size) || p->expert_stride < (channels - 1u) * p->product.w_stride + p->product.n_in)) return MAASO_E_SHAPE;
  ProductArgs a = product_args(inst, &p->product, p->n_rows);
  a.start = p->start; a.token = p->token; a.n_experts = p->n_experts; a.expert_stride = p->expert_stride * size;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  return launch_product(p->product.type, a, p->product.gated != 0u, (uint32_t)inst->n_cu, s);
}

int maaso_expert_route(maaso_instance* inst, const maaso_expert_route_args* p, void* hip_stream) {
  if (!inst || !p) return MAASO_E_INVALID_ARG;
  if (p->type > MAASO_FP32 || (p->bias && !p->sigmoid) || !std::isfinite(p->scale)) return MAASO_E_INVALID_ARG;
  if (p->n_experts == 0 || p->n_experts > MAASO_EXPERT_MAX || p->k == 0 || p->k > p->n_experts || p->k > MAASO_EXPERT_MAX_CHOSEN) return MAASO_E_SHAPE;
  const bool order = p->start || p->token || p->place;
  if (order && !(p->start && p->token && p->place) && p->n) return MAASO_E_INVALID_ARG;
  if (p->n && (!p->logits || !p->expert || !p->weight)) return MAASO_E_INVALID_ARG;
  if (p->n > kMostTokens || (uint64_t)p->n * p->k > 0x7fffffffull || (p->n > 1u && p->stride < p->n_experts)) return MAASO_E_SHAPE;
  if (p->n == 0 && !p->start) return MAASO_OK;
  RouteArgs a{p->logits, p->bias, p->expert, p->weight, p->start, p->token, p->place, p->stride, p->n, p->n_experts, p->k,
              p->sigmoid != 0u, p->renorm != 0u, p->scale, (p->n + kChunk - 1u) / kChunk, nullptr, nullptr};
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  if (order && !one_order(a)) {
    Carve ws{inst->ws, inst->ws_bytes};
    a.before = ws.take<uint32_t>((size_t)a.chunks * a.n_experts);
    a.total = ws.take<uint32_t>(a.n_experts);
    if (!ws.fits) return MAASO_E_WORKSPACE;
  }
  if (p->type == MAASO_BF16) launch_route<__bf16>(a, s);
  else if (p->type == MAASO_FP16) launch_route<_Float16>(a, s);
  else launch_route<float>(a, s);
  return launched();
}

int maaso_expert_combine(maaso_instance* inst, const maaso_expert_combine_args* p, void* hip_stream) {
  if (!inst || !p) return MAASO_E_INVALID_ARG;
  if (p->type > MAASO_FP32) return MAASO_E_INVALID_ARG;
  if (p->width == 0 || p->width > 0x3fffffffu || p->k == 0 || p->k > MAASO_EXPERT_MAX_CHOSEN) return MAASO_E_SHAPE;
  if (p->n == 0) return MAASO_OK;
  if (!p->out || !p->place || (!p->y && p->n_rows)) return MAASO_E_INVALID_ARG;
  const uint64_t size = element_size(p->type), per = (p->width + 7u) / 8u, piece = kPieceThreads / per;
  if (p->n > 0x7fffffffu || p->n_rows > 0x7fffffffu) return MAASO_E_SHAPE;
  if (!aligned(p->y, size) || !aligned(p->residual, size) || !aligned(p->out, size)) return MAASO_E_SHAPE;
  auto rows_ok = [&](uint32_t rows, uint64_t stride) { return rows <= 1u || stride >= p->width; };
  if (!rows_ok(p->n_rows, p->y_stride) || !rows_ok(p->n, p->out_stride) || (p->residual && !rows_ok(p->n, p->residual_stride))) return MAASO_E_SHAPE;
  if (p->residual == p->out && p->n > 1u && p->residual_stride != p->out_stride) return MAASO_E_INVALID_ARG;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  for (uint64_t first = 0; first < p->n; first += piece) {
    const uint32_t n = (uint32_t)std::min<uint64_t>(p->n - first, piece), blocks = (uint32_t)((n * per + 255u) / 256u);
    const CombineArgs a{p->y, p->residual ? static_cast<const char*>(p->residual) + first * p->residual_stride * size : nullptr,
                        static_cast<char*>(p->out) + first * p->out_stride * size, p->place + first * p->k, p->weight ? p->weight + first * p->k : nullptr,
                        p->y_stride, p->residual_stride, p->out_stride, n, p->k, p->width, p->n_rows, inst->status};
    if (p->type == MAASO_BF16) hipLaunchKernelGGL(combine_kernel<__bf16>, dim3(blocks), dim3(256), 0, s, a);
    else if (p->type == MAASO_FP16) hipLaunchKernelGGL(combine_kernel<_Float16>, dim3(blocks), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(combine_kernel<float>, dim3(blocks), dim3(256), 0, s, a);
  }
  return launched();
}

}  // extern "C"
