// Host helpers shared by the library's entry points: the error detail, the
// checks of pointers and the device, and the launch steps of a call.
// Definitions in api.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdlib.h>

#include "headguard.h"

namespace hg {

// Records the detail of a status for hg_last_error and returns the status;
// ok() clears the detail.
int fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int ok();

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

int check_device_ptr(const void* p, const char* name);

// Checks that a HIP device is present.
int check_device();

// Buffers the call reads or writes, with their sizes, for NULL, alignment and
// device-memory checks.
struct Buf {
  const void* p;
  uint64_t bytes;
  uintptr_t align;
  const char* name;
};

int check_buffers(const Buf* bufs, int nb);

// Launch steps of one call.  Test hook: with HG_FAIL_LAUNCH=i in the
// environment, step i (0-based) of every call reports hipErrorLaunchFailure
// without enqueuing anything, so the mapping of a launch error to HG_ERR_HIP
// can be exercised on a working device.  Step 0 failing leaves every output
// untouched; a later step failing leaves the earlier steps enqueued.
struct LaunchSteps {
  int fail_at = -1;
  int next = 0;
  LaunchSteps() {
    const char* s = getenv("HG_FAIL_LAUNCH");
    if (s && *s) fail_at = atoi(s);
  }
  template <class F>
  hipError_t operator()(F&& launch) {
    if (next++ == fail_at) return hipErrorLaunchFailure;
    return launch();
  }
};

}  // namespace hg
