// kia_host.hpp -- host helpers shared by the files with entry points.
#pragma once

#include <hip/hip_runtime.h>

namespace kia {

// Compute units of the current device (kia_abi.hip).
int host_cus();

// One kernel launch on stream s, recorded under `name` while the timing hook is
// on (kia_abi.hip).
void timed_launch(const char *name, hipStream_t s, void (*launch)(void *), void *ctx);
template <class F> void timed_call(const char *name, hipStream_t s, F launch) {
  timed_launch(name, s, [](void *f) { (*static_cast<F *>(f))(); }, &launch);
}

}  // namespace kia
