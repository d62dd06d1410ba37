// Host side of the C ABI declared in include/maaso_instance.h: argument validation, the instance, launch shapes.
#include "../../include/maaso_instance.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <new>

#include "host_common.hpp"
#include "kv_append_kernels.hpp"
#include "kv_attention_kernels.hpp"
#include "kv_pages_kernels.hpp"
#include "logits_kernels.hpp"

using namespace maaso;

struct maaso_instance {
  int device;
  int n_cu;
  uint32_t* status;  // device status word, and behind it the one that maaso_instance_status reads
  LogitsRow* rows;   // [kFewRows] behind it, zeros between calls (made so again by maaso_instance_status)
  char* ws;          // device workspace
  size_t ws_bytes;
  // one call at a time, as for maaso_ctx
  std::atomic<int> in_call;
  hipEvent_t order_ev;
  hipStream_t last_stream;
  bool has_last;
};

namespace {

// Exclusive use by one call, and order behind the previous call's stream (calls that are captured are left to the caller, and
// so is the order behind a stream that is being captured by now: an event recorded there would be a node of its graph, and the
// wait for it would draw this call's stream into the capture).
struct InstanceCall {
  maaso_instance* inst;
  DeviceGuard device;
  int rc;
  InstanceCall(maaso_instance* in, hipStream_t s) : inst(in), device(in->device), rc(MAASO_OK) {
    int idle = 0;
    if (!inst->in_call.compare_exchange_strong(idle, 1, std::memory_order_acquire)) {
      inst = nullptr;
      rc = MAASO_E_BUSY;
      return;
    }
    if (!device.ok) { rc = MAASO_E_HIP; return; }
    if (inst->has_last && inst->last_stream == s) return;
    if (is_captured(s)) return;
    if (inst->has_last && !is_captured(inst->last_stream)) {
      const bool ordered = hipEventRecord(inst->order_ev, inst->last_stream) == hipSuccess &&
                           hipStreamWaitEvent(s, inst->order_ev, 0) == hipSuccess;
      if (!ordered) {
        (void)hipGetLastError();
        if (!hip_ok(hipDeviceSynchronize())) rc = MAASO_E_HIP;
      }
    }
    inst->last_stream = s;
    inst->has_last = true;
  }
  ~InstanceCall() {
    if (inst) inst->in_call.store(0, std::memory_order_release);
  }
  InstanceCall(const InstanceCall&) = delete;
  InstanceCall& operator=(const InstanceCall&) = delete;
};

// Takes the status bits and leaves none, in one step: a copy and a clear of their own would lose what is raised between them.
// The rows are made zeros, as calls leave them: two few-row calls that have run at once, which the caller has to order, may
// have left counts behind that every later call would go wrong by.
__global__ void __launch_bounds__(256) take_status_kernel(uint32_t* status, LogitsRow* rows) {
  const uint32_t i = blockIdx.x * 256u + threadIdx.x;
  rows[i].key = 0ull;
  rows[i].done = 0u;
  if (i == 0u) status[1] = atomicExch(status, 0u);
}
static_assert(kFewRows % 256u == 0u, "a thread to a row");

constexpr size_t kOwnBytes = 256u + kFewRows * sizeof(LogitsRow);  // the status word, then the rows

int launched() { return hip_ok(hipGetLastError()) ? MAASO_OK : MAASO_E_HIP; }

// Parts of the workspace, 256 bytes apart.
struct Carve {
  char* at;
  size_t left;
  bool fits = true;
  template <typename T> T* take(size_t n) {
    const size_t bytes = (n * sizeof(T) + 255) & ~size_t(255);
    if (bytes > left) { fits = false; return nullptr; }
    T* p = reinterpret_cast<T*>(at);
    at += bytes;
    left -= bytes;
    return p;
  }
};

// The copy is behind the kernel on the null stream and has come when it returns: nothing is under way then that later calls,
// on streams that do not wait for the null stream, could run beside.
int take_status(maaso_instance* in, uint32_t* bits) {
  DeviceGuard guard(in->device);
  if (!guard.ok) return MAASO_E_HIP;
  uint32_t v = 0;
  if (!hip_ok(hipDeviceSynchronize())) return MAASO_E_HIP;
  hipLaunchKernelGGL(take_status_kernel, dim3(kFewRows / 256u), dim3(256), 0, nullptr, in->status, in->rows);
  if (!hip_ok(hipGetLastError())) return MAASO_E_HIP;
  if (!hip_ok(hipMemcpy(&v, in->status + 1, 4, hipMemcpyDeviceToHost))) return MAASO_E_HIP;
  if (bits) *bits = v;
  return v ? MAASO_E_INVALID_ARG : MAASO_OK;
}

bool page_size_ok(uint32_t s) { return s == 16u || s == 32u || s == 64u || s == 128u; }
uint32_t log2_of(uint32_t x) { return 31u - (uint32_t)__builtin_clz(x); }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

int check_pages(const maaso_kv_pages* p) {
  if (!p || !p->refs || !p->table || !p->length) return MAASO_E_INVALID_ARG;
  if (p->n_pages == 0 || p->n_rows == 0 || p->width == 0) return MAASO_E_INVALID_ARG;
  if (!page_size_ok(p->page_size) || p->n_pages > MAASO_KV_MAX_PAGES) return MAASO_E_SHAPE;
  if ((uint64_t)p->width * p->page_size > 0x7fffffffull) return MAASO_E_SHAPE;
  return MAASO_OK;
}

PageArgs page_args(const maaso_instance* inst, const maaso_kv_pages* p) {
  return {p->n_pages, log2_of(p->page_size), p->n_rows, p->width, p->refs, p->table, p->length, inst->status};
}

uint64_t element_size(uint32_t type) { return type == MAASO_E4M3 ? 1u : type == MAASO_FP32 ? 4u : 2u; }

int check_cache(const maaso_kv_cache* c) {
  if (!c || !c->k || !c->v) return MAASO_E_INVALID_ARG;
  if (c->type != MAASO_BF16 && c->type != MAASO_FP16 && c->type != MAASO_E4M3) return MAASO_E_INVALID_ARG;
  if (c->type != MAASO_E4M3 && (c->k_scale || c->v_scale)) return MAASO_E_INVALID_ARG;
  if (c->n_layers == 0 || c->n_pages == 0 || c->n_kv_heads == 0) return MAASO_E_INVALID_ARG;
  if (!page_size_ok(c->page_size) || c->n_pages > MAASO_KV_MAX_PAGES || c->n_kv_heads > 1024u || c->n_layers > 65535u) return MAASO_E_SHAPE;
  if (c->head_dim != 64u && c->head_dim != 128u && c->head_dim != 256u) return MAASO_E_SHAPE;
  const uint64_t page = (uint64_t)c->n_kv_heads * c->page_size * c->head_dim, size = element_size(c->type);
  if (c->n_pages > 1u && c->page_stride < page) return MAASO_E_SHAPE;
  // (layers of pages or pages of layers: their elements only must not be the same)
  if (c->n_layers > 1u && c->layer_stride < page) return MAASO_E_SHAPE;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || c->page_stride * size % 16u || c->layer_stride * size % 16u) return MAASO_E_SHAPE;
  return MAASO_OK;
}

}  // namespace

extern "C" {

int maaso_instance_create(int device, uint64_t workspace_bytes, maaso_instance** out) {
  if (!out) return MAASO_E_INVALID_ARG;
  *out = nullptr;
  if (workspace_bytes == 0) workspace_bytes = MAASO_INSTANCE_WORKSPACE_BYTES;
  if (workspace_bytes > (1ull << 40)) return MAASO_E_SHAPE;
  int count = 0;
  if (!hip_ok(hipGetDeviceCount(&count)) || device < 0 || device >= count) return MAASO_E_HIP;
  DeviceGuard guard(device);
  if (!guard.ok) return MAASO_E_HIP;
  maaso_instance* in = new (std::nothrow) maaso_instance();
  if (!in) return MAASO_E_NOMEM;
  in->device = device;
  in->ws_bytes = ((size_t)workspace_bytes + 255) & ~size_t(255);
  int rc = MAASO_OK;
  if (!hip_ok(hipDeviceGetAttribute(&in->n_cu, hipDeviceAttributeMultiprocessorCount, device))) rc = MAASO_E_HIP;
  if (rc == MAASO_OK && !hip_ok(hipMalloc(reinterpret_cast<void**>(&in->status), kOwnBytes))) rc = MAASO_E_NOMEM;
  if (rc == MAASO_OK && !hip_ok(hipMalloc(reinterpret_cast<void**>(&in->ws), in->ws_bytes))) rc = MAASO_E_NOMEM;
  if (rc == MAASO_OK && !hip_ok(hipEventCreateWithFlags(&in->order_ev, hipEventDisableTiming))) rc = MAASO_E_HIP;
  if (rc == MAASO_OK && (!hip_ok(hipMemset(in->status, 0, kOwnBytes)) || !hip_ok(hipDeviceSynchronize()))) rc = MAASO_E_HIP;
  if (rc != MAASO_OK) {
    if (in->order_ev) (void)hipEventDestroy(in->order_ev);
    if (in->ws) (void)hipFree(in->ws);
    if (in->status) (void)hipFree(in->status);
    (void)hipGetLastError();
    delete in;
    return rc;
  }
  in->rows = reinterpret_cast<LogitsRow*>(in->status + 64);
  *out = in;
  return MAASO_OK;
}

void maaso_instance_destroy(maaso_instance* in) {
  if (!in) return;
  DeviceGuard guard(in->device);
  (void)hipDeviceSynchronize();
  (void)hipEventDestroy(in->order_ev);
  (void)hipFree(in->ws);
  (void)hipFree(in->status);
  (void)hipGetLastError();
  delete in;
}

int maaso_instance_status(maaso_instance* in, uint32_t* bits) {
  if (bits) *bits = 0;
  if (!in) return MAASO_E_INVALID_ARG;
  int idle = 0;
  if (!in->in_call.compare_exchange_strong(idle, 1, std::memory_order_acquire)) return MAASO_E_BUSY;
  const int rc = take_status(in, bits);
  in->in_call.store(0, std::memory_order_release);
  return rc;
}

int maaso_kv_extend(maaso_instance* inst, const maaso_kv_pages* pages, const int32_t* rows, uint32_t n, const int32_t* q_start,
                    uint32_t n_tok, int64_t* slot, int32_t* pos, int32_t* copies, void* hip_stream) {
  if (!inst) return MAASO_E_INVALID_ARG;
  if (const int rc = check_pages(pages)) return rc;
  if (n == 0 && n_tok == 0) return MAASO_OK;
  if (n == 0 || !rows || !q_start || !copies || (n_tok != 0 && !slot)) return MAASO_E_INVALID_ARG;
  if (n > MAASO_KV_MAX_ROWS || n_tok > 0x7fffffffu || (uint64_t)n * pages->width > 0x7fffffffull) return MAASO_E_SHAPE;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  Carve ws{inst->ws, inst->ws_bytes};
  ExtendArgs a{page_args(inst, pages), rows, q_start, n, n_tok, slot, pos, copies, ws.take<uint32_t>(1), ws.take<int32_t>(n),
               ws.take<uint32_t>(n + 1u), ws.take<int32_t>(n), ws.take<int32_t>(pages->n_pages)};
  if (!ws.fits) return MAASO_E_WORKSPACE;
  if (n_tok <= 4u * kPageThreads) {
    hipLaunchKernelGGL(extend_kernel, dim3(1), dim3(kPageThreads), 0, s, a);
  } else {
    hipLaunchKernelGGL(extend_plan_kernel, dim3(1), dim3(kPageThreads), 0, s, a);
    hipLaunchKernelGGL(extend_apply_kernel, dim3(std::min(1024u, (n_tok + 255u) / 256u)), dim3(256), 0, s, a);
  }
  return launched();
}

int maaso_kv_fork(maaso_instance* inst, const maaso_kv_pages* pages, const int32_t* parents, const int32_t* children, uint32_t n,
                  void* hip_stream) {
  if (!inst) return MAASO_E_INVALID_ARG;
  if (const int rc = check_pages(pages)) return rc;
  if (n == 0) return MAASO_OK;
  if (!parents || !children) return MAASO_E_INVALID_ARG;
  if (n > MAASO_KV_MAX_ROWS) return MAASO_E_SHAPE;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  hipLaunchKernelGGL(fork_kernel, dim3(n), dim3(256), 0, s, page_args(inst, pages), parents, children);
  return launched();
}

int maaso_kv_trim(maaso_instance* inst, const maaso_kv_pages* pages, const int32_t* rows, const int32_t* keep, uint32_t n,
                  void* hip_stream) {
  if (!inst) return MAASO_E_INVALID_ARG;
  if (const int rc = check_pages(pages)) return rc;
  if (n == 0) return MAASO_OK;
  if (!rows || !keep) return MAASO_E_INVALID_ARG;
  if (n > MAASO_KV_MAX_ROWS) return MAASO_E_SHAPE;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  hipLaunchKernelGGL(trim_kernel, dim3(n), dim3(256), 0, s, page_args(inst, pages), rows, keep);
  return launched();
}

int maaso_kv_compact(maaso_instance* inst, const maaso_kv_pages* pages, int32_t* refs_out, int32_t* table_out, int32_t* moves,
                     int32_t* n_live, void* hip_stream) {
  if (!inst) return MAASO_E_INVALID_ARG;
  if (const int rc = check_pages(pages)) return rc;
  if (!refs_out || !table_out || !n_live || (!moves && pages->n_pages > 1u)) return MAASO_E_INVALID_ARG;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  Carve ws{inst->ws, inst->ws_bytes};
  const uint32_t chunks = (pages->n_pages + kCompactChunk - 1u) / kCompactChunk;
  CompactArgs a{page_args(inst, pages), refs_out, table_out, moves, n_live, chunks, ws.take<uint32_t>(chunks),
                ws.take<uint32_t>(pages->n_pages + 1u), ws.take<int32_t>(pages->n_pages)};
  if (!ws.fits) return MAASO_E_WORKSPACE;
  const uint64_t entries = std::max<uint64_t>((uint64_t)pages->n_rows * pages->width, pages->n_pages);
  if (chunks == 1u && entries <= kCompactEntries) {
    hipLaunchKernelGGL(compact_kernel, dim3(1), dim3(kPageThreads), 0, s, a);
    return launched();
  }
  if (chunks > 1u) hipLaunchKernelGGL(compact_count_kernel, dim3(chunks), dim3(kPageThreads), 0, s, a);
  hipLaunchKernelGGL(compact_rank_kernel, dim3(chunks), dim3(kPageThreads), 0, s, a);
  hipLaunchKernelGGL(compact_apply_kernel, dim3((uint32_t)std::min<uint64_t>(2048u, (entries + 255u) / 256u)), dim3(256), 0, s, a);
  return launched();
}

int maaso_kv_copy(maaso_instance* inst, const maaso_kv_cache* cache, const int32_t* pairs, uint32_t n, void* hip_stream) {
  if (!inst) return MAASO_E_INVALID_ARG;
  if (const int rc = check_cache(cache)) return rc;
  if (n == 0) return MAASO_OK;
  if (!pairs) return MAASO_E_INVALID_ARG;
  const uint64_t size = element_size(cache->type), bytes = (uint64_t)cache->n_kv_heads * cache->page_size * cache->head_dim * size;
  const uint64_t chunks = (bytes + kCopyChunk - 1u) / kCopyChunk;
  if (n > MAASO_KV_MAX_PAGES || chunks * n > 0x7fffffffull) return MAASO_E_SHAPE;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  CopyArgs a{pairs, n, cache->n_pages, (uint32_t)chunks, cache->n_layers, bytes, cache->page_stride * size, cache->layer_stride * size,
             static_cast<char*>(cache->k), static_cast<char*>(cache->v), bytes * n * cache->n_layers * 2u > kCopyPast, inst->status};
  hipLaunchKernelGGL(copy_kernel, dim3((uint32_t)(chunks * n), cache->n_layers, 2), dim3(256), 0, s, a);
  return launched();
}

}  // extern "C"

namespace {

template <typename T, typename C, int D>
void launch_append(const AppendArgs& a, uint32_t blocks, bool interleaved, hipStream_t s) {
  if (interleaved) hipLaunchKernelGGL((append_kernel<T, C, D, true>), dim3(blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((append_kernel<T, C, D, false>), dim3(blocks), dim3(256), 0, s, a);
}

template <typename T, typename C>
void launch_append_d(uint32_t d, const AppendArgs& a, uint32_t blocks, bool interleaved, hipStream_t s) {
  if (d == 64u) launch_append<T, C, 64>(a, blocks, interleaved, s);
  else if (d == 128u) launch_append<T, C, 128>(a, blocks, interleaved, s);
  else launch_append<T, C, 256>(a, blocks, interleaved, s);
}

// Few rows of a sequence or group go through the stream kernel, more through the tile kernel; which, the kernels see
// from the device's arrays.  The bounds tell the host whether there can be tiles, but not that there is nothing of few rows:
// n * max_q == n_tok does not say that every sequence has max_q queries, for they need not fill n_tok.
template <typename T, typename C, int D>
void launch_attention(AttentionArgs a, hipStream_t s) {
  const uint32_t heads = a.n_kv_heads;
  const bool tiles = a.max_q * a.group > kStreamRows, shared_tiles = a.shared_parts && (uint64_t)a.n_tok * a.group > kStreamRows;
  a.stream_shared = a.n_groups * heads * a.shared_parts;
  const uint32_t items = a.stream_shared + a.n * heads * a.own_parts;
  a.stream_blocks = a.alone ? (items + 3u) / 4u : items;
  if (tiles || shared_tiles) {
    a.tile_shared = shared_tiles ? a.shared_tiles * heads * a.shared_parts : 0u;
    a.tile_blocks = a.tile_shared + (tiles ? a.own_tiles * heads * a.own_parts : 0u);
    hipLaunchKernelGGL((attention_tile_kernel<T, C, D, D == 256 ? 32 : 64>), dim3(a.tile_blocks + a.stream_blocks), dim3(256), 0, s, a);
  } else if (a.alone) {
    hipLaunchKernelGGL((attention_stream_kernel<T, C, D, 1>), dim3(a.stream_blocks), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL((attention_stream_kernel<T, C, D, 4>), dim3(a.stream_blocks), dim3(256), 0, s, a);
  }
  if (a.part_o) {
    constexpr uint32_t kHeads = 256 / D;  // of a wave
    const uint32_t groups = (a.n_heads + kHeads - 1u) / kHeads;
    if ((uint64_t)a.n_tok * groups < 1024u)
      hipLaunchKernelGGL((attention_join_kernel<T, C, D, 4, 1>), dim3(a.n_tok, groups), dim3(256), 0, s, a);
    else if ((uint64_t)a.n_tok * groups < 32768u)
      hipLaunchKernelGGL((attention_join_kernel<T, C, D, 1, 1>), dim3(a.n_tok, (groups + 3u) / 4u), dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((attention_join_kernel<T, C, D, 1, 8>), dim3((a.n_tok + 7u) / 8u, (groups + 3u) / 4u), dim3(256), 0, s, a);
  }
}

template <typename T, typename C>
void launch_attention_d(uint32_t d, const AttentionArgs& a, hipStream_t s) {
  if (d == 64u) launch_attention<T, C, 64>(a, s);
  else if (d == 128u) launch_attention<T, C, 128>(a, s);
  else launch_attention<T, C, 256>(a, s);
}

uint32_t round_up(uint64_t x, uint32_t to) { return (uint32_t)((x + to - 1u) / to * to); }

template <typename T, typename O>
void launch_logits(const LogitsArgs& a, hipStream_t s) {
  const dim3 g(a.n * a.slices);
  if (a.meet) hipLaunchKernelGGL((logits_kernel<T, O, kFewThreads, kFewPieces>), g, dim3(kFewThreads), 0, s, a);
  else hipLaunchKernelGGL((logits_kernel<T, O, kManyThreads, kManyPieces>), g, dim3(kManyThreads), 0, s, a);
}

}  // namespace

extern "C" {

int maaso_kv_append(maaso_instance* inst, const maaso_kv_cache* cache, uint32_t layer, const maaso_kv_append_args* p,
                    void* hip_stream) {
  if (!inst || !p) return MAASO_E_INVALID_ARG;
  if (const int rc = check_cache(cache)) return rc;
  if (layer >= cache->n_layers) return MAASO_E_INVALID_ARG;
  if (p->type != MAASO_BF16 && p->type != MAASO_FP16) return MAASO_E_INVALID_ARG;
  if (cache->type != p->type && cache->type != MAASO_E4M3) return MAASO_E_INVALID_ARG;
  const uint32_t d = cache->head_dim;
  if (p->n_heads == 0 || p->n_heads > 1024u || p->rotary > d || p->rotary % 16u) return MAASO_E_SHAPE;
  if (p->n_tok == 0) return MAASO_OK;
  if (p->n_tok > 0x7fffffffu) return MAASO_E_SHAPE;
  if (!p->q || !p->k || !p->v || !p->q_out || !p->slot) return MAASO_E_INVALID_ARG;
  if (p->rotary && (!p->cos_sin || !p->pos || p->n_pos == 0 || p->n_pos > 0x7fffffffu || !aligned(p->cos_sin, 16))) return MAASO_E_INVALID_ARG;
  if (!(p->eps >= 0.0f) || !std::isfinite(p->eps)) return MAASO_E_INVALID_ARG;
  if (p->n_tok > 1u && (p->q_stride < (uint64_t)p->n_heads * d || p->q_out_stride < (uint64_t)p->n_heads * d ||
                        p->k_stride < (uint64_t)cache->n_kv_heads * d || p->v_stride < (uint64_t)cache->n_kv_heads * d))
    return MAASO_E_SHAPE;
  if (p->q == p->q_out && p->n_tok > 1u && p->q_stride != p->q_out_stride) return MAASO_E_INVALID_ARG;
  const uint64_t size = element_size(cache->type);
  AppendArgs a{};
  a.q = p->q; a.k = p->k; a.v = p->v; a.q_out = p->q_out; a.q_weight = p->q_weight; a.k_weight = p->k_weight;
  a.cos_sin = p->cos_sin; a.pos = p->pos; a.slot = p->slot; a.k_scale = cache->k_scale; a.v_scale = cache->v_scale;
  a.k_pages = static_cast<char*>(cache->k) + layer * cache->layer_stride * size;
  a.v_pages = static_cast<char*>(cache->v) + layer * cache->layer_stride * size;
  a.q_stride = p->q_stride; a.k_stride = p->k_stride; a.v_stride = p->v_stride; a.q_out_stride = p->q_out_stride;
  a.page_stride = cache->page_stride;
  a.page_log2 = log2_of(cache->page_size);
  a.n_slots = (uint64_t)cache->n_pages << a.page_log2;
  a.n_tok = p->n_tok; a.n_heads = p->n_heads; a.n_kv_heads = cache->n_kv_heads; a.rotary = p->rotary; a.n_pos = p->n_pos;
  a.eps = p->eps;
  a.past = (uint64_t)p->n_tok * p->n_heads * d * 2u > kCopyPast;
  a.status = inst->status;
  const bool turned = p->n_tok >= 512u;  // values through shared memory
  const uint64_t heads = p->n_heads + cache->n_kv_heads * (turned ? 1u : 2u), per = 256u / (d / 8u) * kAppendHeads;
  const uint64_t head_blocks = (heads * p->n_tok + per - 1u) / per;
  const uint64_t value_blocks = turned ? (uint64_t)(p->n_tok + kTurnTokens - 1u) / kTurnTokens * cache->n_kv_heads * (d / 64u) : 0u;
  if (head_blocks + value_blocks > 0x7fffffffull) return MAASO_E_SHAPE;
  a.value_blocks = (uint32_t)value_blocks;
  const uint32_t blocks = (uint32_t)(head_blocks + value_blocks);
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  const bool inter = p->interleaved != 0u;
  if (p->type == MAASO_BF16 && cache->type == MAASO_BF16) launch_append_d<__bf16, __bf16>(d, a, blocks, inter, s);
  else if (p->type == MAASO_BF16) launch_append_d<__bf16, E4m3>(d, a, blocks, inter, s);
  else if (cache->type == MAASO_FP16) launch_append_d<_Float16, _Float16>(d, a, blocks, inter, s);
  else launch_append_d<_Float16, E4m3>(d, a, blocks, inter, s);
  return launched();
}

int maaso_kv_attention(maaso_instance* inst, const maaso_kv_cache* cache, uint32_t layer, const maaso_kv_pages* pages,
                       const maaso_kv_attention_args* p, void* hip_stream) {
  if (!inst || !p) return MAASO_E_INVALID_ARG;
  if (const int rc = check_cache(cache)) return rc;
  if (const int rc = check_pages(pages)) return rc;
  if (layer >= cache->n_layers || pages->page_size != cache->page_size || pages->n_pages != cache->n_pages) return MAASO_E_INVALID_ARG;
  if (p->type != MAASO_BF16 && p->type != MAASO_FP16) return MAASO_E_INVALID_ARG;
  if (cache->type != p->type && cache->type != MAASO_E4M3) return MAASO_E_INVALID_ARG;
  if (p->n_heads == 0 || p->n_heads > 1024u || p->n_heads % cache->n_kv_heads) return MAASO_E_SHAPE;
  if (!std::isfinite(p->scale)) return MAASO_E_INVALID_ARG;
  if (p->n == 0 || p->n_tok == 0) return p->n_tok == 0 ? MAASO_OK : MAASO_E_INVALID_ARG;
  if (p->n > MAASO_KV_MAX_ROWS || p->n_groups > p->n || p->n_tok > 0x7fffffu || p->max_q == 0 || p->max_q > p->n_tok) return MAASO_E_SHAPE;
  if (!p->q || !p->out || !p->q_start || (p->n_groups && (!p->group_start || !p->shared))) return MAASO_E_INVALID_ARG;
  const uint32_t d = cache->head_dim;
  if (!aligned(p->q, 16) || !aligned(p->out, 16) || p->q_stride % 8u || p->out_stride % 8u) return MAASO_E_SHAPE;
  if (p->n_tok > 1u && (p->q_stride < (uint64_t)p->n_heads * d || p->out_stride < (uint64_t)p->n_heads * d)) return MAASO_E_SHAPE;
  if (p->max_len > 0x7fffffffu) return MAASO_E_SHAPE;
  const uint64_t size = element_size(cache->type), rows = (uint64_t)p->n_tok * p->n_heads;
  AttentionArgs a{};
  a.q = p->q; a.out = p->out; a.lse = p->lse; a.q_stride = p->q_stride; a.out_stride = p->out_stride;
  a.k_pages = static_cast<const char*>(cache->k) + layer * cache->layer_stride * size;
  a.v_pages = static_cast<const char*>(cache->v) + layer * cache->layer_stride * size;
  a.page_stride = cache->page_stride;
  a.k_scale = cache->k_scale; a.v_scale = cache->v_scale;
  a.table = pages->table; a.length = pages->length;
  a.q_start = p->q_start; a.rows = p->rows; a.group_start = p->group_start; a.shared = p->shared;
  a.n = p->n; a.n_tok = p->n_tok; a.n_heads = p->n_heads; a.n_kv_heads = cache->n_kv_heads; a.group = p->n_heads / cache->n_kv_heads;
  a.n_groups = p->max_shared ? p->n_groups : 0u;
  a.n_pages = pages->n_pages; a.page_log2 = log2_of(pages->page_size); a.n_rows = pages->n_rows; a.width = pages->width;
  a.max_q = p->max_q; a.max_len = p->max_len; a.most_shared = a.n_groups ? (uint32_t)std::min<uint64_t>(std::min(p->max_shared, p->max_len), (uint64_t)pages->width * pages->page_size) : 0u;
  a.scale_log2 = (float)((double)p->scale * 1.4426950408889634);
  a.status = inst->status;
  const uint64_t group_rows = (uint64_t)p->n_tok * a.group;
  a.own_tiles = (uint32_t)(group_rows / kTileRows + p->n);
  a.shared_tiles = a.n_groups ? (uint32_t)(group_rows / kTileRows + a.n_groups) : 0u;
  const bool tiles = (uint64_t)p->max_q * a.group > kStreamRows, shared_tiles = group_rows > kStreamRows;
  // How keys are split.  Many rows: until there are two blocks to a compute unit, and where there are less than eight, into
  // parts of no more than 2048 keys, so that long rows end when the others do.  Few: so that the keys, as far as the lengths'
  // sum tells, come to even parts for every place that a unit has, but into none below 256 or 128 keys; a row may be longer
  // than the others and still be cut as finely.
  const uint64_t cus = (uint64_t)inst->n_cu, heads = a.n_kv_heads, most_len = std::max(1u, p->max_len);
  auto split = [&](uint64_t keys, uint64_t items) {
    const uint64_t want = 2u * cus, parts = items >= want ? 1u : (want + items - 1u) / items;
    const uint32_t chunk = std::max(256u, round_up((keys + parts - 1u) / parts, 256u));
    return items < 8u * cus ? std::min(chunk, 2048u) : chunk;
  };
  const uint64_t total = p->total_len && p->total_len < p->n * most_len ? p->total_len : p->n * most_len;
  const uint64_t in_common = (uint64_t)p->n * a.most_shared, own = total > in_common ? total - in_common : p->n;
  // Items to a wave each, where there are many of few keys: four waves that share one have little to do and wait for each other
  // twice.  512 to 1024 sequences of 8 key heads (heads of 256: 1024 of 4), a block to an item against a wave, us: heads of 64
  // in 16 bits, 64 keys 25 : 16, 300 keys 68 : 66, 500 keys 97 : 105; in 8 bits, 300 keys 41 : 34, 1000 keys 96 : 100; heads of 256, 200
  // keys 212 : 164, 1000 keys 726 : 724; heads of 128 in 8 bits, 200 keys 60 : 58, 300 keys 74 : 78; in 16 bits, 40 keys 42 : 30,
  // 100 keys 58 : 61, 300 keys 126 : 143.
  a.alone = p->n * heads >= 4096u && own <= p->n * (d == 128u && size == 2u ? 64u : 256u);
  const uint64_t places = (a.alone ? 8u : 4u) * cus;
  auto even = [&](uint64_t keys) { return std::max(a.alone ? 128u : 256u, round_up(keys * heads / places, 64u)); };
  if (tiles) {
    a.own_least = split(most_len, (uint64_t)a.own_tiles * heads);
    a.own_parts = (uint32_t)((most_len + a.own_least - 1u) / a.own_least);
  } else {
    a.own_least = a.alone ? 128u : 256u;
    const uint64_t chunk = even(own), parts = (most_len + chunk - 1u) / chunk;
    const uint64_t bound = (2u * own / p->n + a.own_least - 1u) / a.own_least + (places + p->n * heads - 1u) / (p->n * heads);
    a.own_parts = (uint32_t)std::min(parts, bound);
  }
  a.shared_chunk = !a.n_groups ? 256u : shared_tiles ? split(a.most_shared, (uint64_t)a.shared_tiles * heads) : even((uint64_t)a.n_groups * a.most_shared);
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  for (;;) {
    a.shared_parts = (a.most_shared + a.shared_chunk - 1u) / a.shared_chunk;
    if (a.own_parts + a.shared_parts == 1u) break;
    Carve ws{inst->ws, inst->ws_bytes};
    a.part_ml = ws.take<float>(rows * (a.own_parts + a.shared_parts) * 2u);
    a.part_o = ws.take<float>(rows * (a.own_parts + a.shared_parts) * d);
    if (ws.fits) break;
    a.part_o = nullptr;
    if (a.own_parts == 1u && a.shared_parts <= 1u) return MAASO_E_WORKSPACE;
    // half as many parts, where there are more of them
    if (a.own_parts >= a.shared_parts) a.own_parts = (a.own_parts + 1u) / 2u;
    else a.shared_chunk *= 2u;
  }
  const uint64_t shared_blocks = (uint64_t)(a.shared_tiles + a.n_groups) * a.n_kv_heads * a.shared_parts;
  const uint64_t own_blocks = (uint64_t)(a.own_tiles + p->n) * a.n_kv_heads * a.own_parts;
  if (shared_blocks + own_blocks > 0x7fffffffull || (rows + 3u) / 4u > 0x7fffffffull) return MAASO_E_SHAPE;
  if (p->type == MAASO_BF16 && cache->type == MAASO_BF16) launch_attention_d<__bf16, __bf16>(d, a, s);
  else if (p->type == MAASO_BF16) launch_attention_d<__bf16, E4m3>(d, a, s);
  else if (cache->type == MAASO_FP16) launch_attention_d<_Float16, _Float16>(d, a, s);
  else launch_attention_d<_Float16, E4m3>(d, a, s);
  return launched();
}

int maaso_logits_adjust(maaso_instance* inst, const maaso_logits_args* p, void* hip_stream) {
  if (!inst || !p) return MAASO_E_INVALID_ARG;
  if (p->type > MAASO_FP32 || (p->out_type != MAASO_FP32 && p->out_type != p->type)) return MAASO_E_INVALID_ARG;
  if (p->vocab == 0 || p->vocab > 0x7fffffffu) return MAASO_E_SHAPE;
  if (p->n == 0) return MAASO_OK;
  if (!p->logits || (!p->out && !p->chosen)) return MAASO_E_INVALID_ARG;
  if ((p->history == nullptr) != (p->history_start == nullptr) && p->n_history) return MAASO_E_INVALID_ARG;
  if (p->n_bias && (!p->bias_token || !p->bias_value || !p->bias_start)) return MAASO_E_INVALID_ARG;
  if (p->mask && p->n_mask == 0) return MAASO_E_INVALID_ARG;
  if (p->n > 1u && (p->stride < p->vocab || (p->out && p->out_stride < p->vocab))) return MAASO_E_SHAPE;
  if (p->out == p->logits && (p->out_type != p->type || (p->n > 1u && p->out_stride != p->stride))) return MAASO_E_INVALID_ARG;
  if (p->n_history > 0x7fffffffu || p->n_bias > 0x7fffffffu) return MAASO_E_SHAPE;
  LogitsArgs a{};
  a.logits = p->logits; a.out = p->out; a.chosen = p->chosen; a.stride = p->stride; a.out_stride = p->out_stride;
  a.n = p->n; a.vocab = p->vocab; a.slices = (p->vocab + kManySlice - 1u) / kManySlice;
  a.n_history = p->n_history; a.n_bias = p->n_bias; a.n_mask = p->n_mask; a.mask_words = (p->vocab + 31u) / 32u;
  a.repetition = p->repetition; a.frequency = p->frequency; a.presence = p->presence; a.temperature = p->temperature;
  if (p->n_history) { a.history = p->history; a.history_start = p->history_start; }
  if (p->n_bias) { a.bias_token = p->bias_token; a.bias_value = p->bias_value; a.bias_start = p->bias_start; }
  a.mask = p->mask; a.mask_row = p->mask_row;
  a.status = inst->status;
  // Fewer large slices than eight to a compute unit, which takes as many at once: small ones, whose blocks meet in the
  // instance's own memory instead of a launch of their own.
  if (a.n <= kFewRows && (uint64_t)a.n * a.slices < 8u * (uint64_t)inst->n_cu) {
    a.slices = (p->vocab + kFewSlice - 1u) / kFewSlice;
    a.meet = inst->rows;
  }
  if ((uint64_t)a.n * a.slices > 0x7fffffffull) return MAASO_E_SHAPE;
  const uint64_t out_size = element_size(p->out_type);
  a.past = p->out && (uint64_t)p->n * p->vocab * out_size > kLogitPast && aligned(p->out, 16) && (p->n == 1u || p->out_stride * out_size % 16u == 0u);
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  InstanceCall call(inst, s);
  if (call.rc != MAASO_OK) return call.rc;
  Carve ws{inst->ws, inst->ws_bytes};
  a.best = ws.take<unsigned long long>(a.chosen && !a.meet ? (size_t)a.n * a.slices : 1u);
  if (!ws.fits) return MAASO_E_WORKSPACE;
  if (p->type == MAASO_FP32) launch_logits<float, float>(a, s);
  else if (p->type == MAASO_BF16 && p->out_type == MAASO_FP32) launch_logits<__bf16, float>(a, s);
  else if (p->type == MAASO_BF16) launch_logits<__bf16, __bf16>(a, s);
  else if (p->out_type == MAASO_FP32) launch_logits<_Float16, float>(a, s);
  else launch_logits<_Float16, _Float16>(a, s);
  if (a.chosen && !a.meet) hipLaunchKernelGGL(choose_kernel, dim3(a.n), dim3(64), 0, s, a.best, a.slices, a.chosen);
  return launched();
}

}  // extern "C"
