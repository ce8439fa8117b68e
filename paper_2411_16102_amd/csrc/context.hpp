// What the entry points outside api.hip use of a context.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <exception>
#include <new>

#include "../../include/blendstep.h"
#include "staging.hpp"

namespace bs {

struct HipRuntime {  // what Staging asks of the runtime
  typedef hipStream_t Stream;
  typedef hipEvent_t Event;
  int create(Event *e) { return hipEventCreateWithFlags(e, hipEventDisableTiming); }
  int destroy(Event e) { return hipEventDestroy(e); }
  int alloc(int32_t **p, long words) {
    return hipHostMalloc(reinterpret_cast<void **>(p), (size_t)words * sizeof(int32_t), hipHostMallocDefault);
  }
  int release(int32_t *p) { return hipHostFree(p); }
  int record(Event e, Stream s) { return hipEventRecord(e, s); }
  int wait(Event e) { return hipEventSynchronize(e); }
  int wait_all() { return hipDeviceSynchronize(); }
  int capturing(Stream s, bool *yes) {
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    const hipError_t e = hipStreamIsCapturing(s, &status);
    *yes = status == hipStreamCaptureStatusActive;
    return e;
  }
};

struct CtxView {
  const bs_layer_cfg *cfg;  // max_positions filled in
  int device;               // BS_DEVICE_NONE: host only
  const float *rope_cos, *rope_sin;  // [max_positions][head_dim / 2]
  float *ws;                // floats that any call on the context may use while it runs, ws_floats of them
  unsigned *counters;       // zero between launches, n_counters of them
  size_t ws_floats;
  int n_counters, n_cu;
};
CtxView ctx_view(const bs_ctx *c);
// keeps the message for bs_last_error and returns the code
int ctx_fail(bs_ctx *c, int code, const char *fmt, ...);
// pinned words that what `stream` is given next may read (see Staging::place)
int ctx_stage(bs_ctx *c, long words, hipStream_t stream, int32_t **out);

// No exception crosses the C boundary: host allocations (vectors that grow with the batch) can throw.
template <class F>
int ctx_guarded(bs_ctx *c, F &&body) {
  try {
    return body();
  } catch (const std::bad_alloc &) {
    return ctx_fail(c, BS_ENOMEM, "out of host memory");
  } catch (const std::exception &e) {
    return ctx_fail(c, BS_EINVAL, "unexpected exception: %s", e.what());
  } catch (...) {
    return ctx_fail(c, BS_EINVAL, "unexpected exception");
  }
}

}  // namespace bs

#define CTX_HIP_TRY(ctx, expr)                                                                             \
  do {                                                                                                     \
    const hipError_t e_ = (expr);                                                                          \
    if (e_ != hipSuccess) return ::bs::ctx_fail(ctx, BS_EHIP, "%s: %s", #expr, hipGetErrorString(e_));      \
  } while (0)
