// Host-side helpers shared by the C entry points: the calling thread's error
// message and the library-managed workspaces.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <mutex>

namespace dion2 {

constexpr int64_t kMaxDim = int64_t(1) << 20;   // longest side of a weight matrix

// Sets the calling thread's dion2_last_error message and returns status.
int fail(int status, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char* what);

// A layer call's hold on the library workspace that (current device, stream)
// has for these calls, apart from the steps': at least the bytes asked for, kept
// from other host threads while it lives.
struct WorkspaceLease {
    std::unique_lock<std::mutex> lock;
    char* dev = nullptr;
};
int lease_layer_workspace(hipStream_t s, size_t bytes, WorkspaceLease* out);

}  // namespace dion2
