// The instance as its host sides hold it: exclusive use by one call, the workspace's parts, checks that entry points share.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

#include "../../include/maaso_instance.h"
#include "host_common.hpp"

namespace maaso {
struct LogitsRow;
}

struct maaso_instance {
  int device;
  int n_cu;
  uint32_t* status;         // device status word, and behind it the one that maaso_instance_status reads
  maaso::LogitsRow* rows;   // [kFewRows] behind it, zeros between calls (made so again by maaso_instance_status)
  char* ws;                 // device workspace
  size_t ws_bytes;
  // one call at a time, as for maaso_ctx
  std::atomic<int> in_call;
  hipEvent_t order_ev;
  hipStream_t last_stream;
  bool has_last;
};

namespace maaso {

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

inline int launched() { return hip_ok(hipGetLastError()) ? MAASO_OK : MAASO_E_HIP; }

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

inline bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline uint64_t element_size(uint32_t type) { return type == MAASO_E4M3 || type == MAASO_INT8 ? 1u : type == MAASO_FP32 ? 4u : 2u; }

}  // namespace maaso
