// What entry points outside api.hip use of it: the thread's stream and error state, the
// device, the per-stream workspace and the checks of strided operands.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <exception>
#include <mutex>

#include "attn.h"

namespace attn {

// Memory of an operand, in bytes: rows of `width`, by three dimensions (of an extent below
// 2^60 each), from `at` to `end`.
struct Rows {
    const char* name;
    uintptr_t at, end;
    long long width, stride[3];
    int n[3];
};

namespace host {

struct DeviceRef {
    void* state = nullptr;
    const attn_device_desc* desc = nullptr;
};

// Sets attn_last_error and returns code.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail_hip(hipError_t e, const char* what);
hipStream_t stream();
// The current device, gfx950 or an error.
int device(DeviceRef* out);
// The workspace of a call: the caller's, checked, or the stream's, with *lk held until the
// kernels that use it are enqueued.
int workspace(const DeviceRef& dev, size_t need, void* given, size_t given_bytes,
              std::unique_lock<std::mutex>* lk, void** out);
// One tensor of rows; written: its rows must not overlap.
int check_heads(const attn_heads* h, const char* name, int B, int S, int H, int d, bool written);
Rows heads_rows(const char* name, const attn_heads& h, int B, int S, int H, int d, int size);
// n0 rows of `row` values of `size` bytes, stride0 values apart
Rows plain_rows(const char* name, const void* p, int size, long long row, long long stride0 = 0,
                int n0 = 1);
// Results that share memory with each other or with an operand are refused.
int check_apart(const Rows* results, int n_results, const Rows* operands, int n_operands);

// No C++ exception leaves a C entry.
template <typename F>
auto guarded(F&& f) -> decltype(f()) {
    try {
        return f();
    } catch (const std::exception& e) {
        return host::fail(ATTN_ENOMEM, "host: %s", e.what());
    }
}

}  // namespace host
}  // namespace attn
