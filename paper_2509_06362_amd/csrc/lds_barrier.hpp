// A barrier for shared memory that atomics have changed.
#pragma once

#include <hip/hip_runtime.h>

namespace maaso {

// Barrier that publishes LDS atomics.  For atomics whose result is unused the compiler emits no wait
// on the LDS counter before the s_barrier of __syncthreads(), and on gfx950 a wavefront reading behind
// that barrier can then see the location without some of the additions (observed as run-to-run
// differences in the per-window admission counts).  Waiting for this wavefront's outstanding LDS
// operations (s_waitcnt lgkmcnt(0), all other counters left at their maxima) before the barrier
// closes that window.  Atomics whose result is used need nothing: the use already waits.
__device__ __forceinline__ void lds_atomics_barrier() {
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __syncthreads();
}

}  // namespace maaso
