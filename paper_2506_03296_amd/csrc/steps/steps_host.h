// steps_host.h -- argument checks and workspaces shared by the entry points of
// libapex_steps.so.
#pragma once

#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <mutex>

#include "apex_steps.h"
#include "status.h"

namespace steps __attribute__((visibility("hidden"))) {

using apex::fail;

// Bytes of a block of 16 tokens' K of all kv-heads stay far below 2^32.
constexpr int kMostHeads = 1 << 16;

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// A buffer of a call, for the checks of what it writes against what it reads.
struct Extent {
    const char* name;
    const void* p;
    size_t bytes;
};

// APEX_OK, or an error if `written` (when not NULL) overlaps one of `others`.
int check_disjoint(const Extent& written, const Extent* others, int n);

// q-heads, kv-heads, head dim and scale of an attention over B requests with T
// rows in all, and the token strides (0: tight), which are set to what they stand for.
int check_attention(int B, int T, int Hq, int Hkv, int d, float scale, int64_t* q_stride, int64_t* kv_stride);

// Bytes from the first element of T rows to behind the last.
inline size_t rows_bytes(int T, int64_t stride, int heads, size_t element)
{
    return T <= 0 ? 0 : ((size_t)(T - 1) * (size_t)stride + (size_t)heads * 128) * element;
}

// The caller's workspace, checked.
int check_workspace(const void* given, size_t given_bytes, size_t bytes);

// The library's own workspace on the current device, at least `bytes` long.
// Under stream capture it is refused: a graph would keep an address that a later
// call may free.  The caller holds it (`hold`, locked here) until it has launched
// what uses it: another thread's call that grows or releases it waits for what
// has been launched and frees it.
using Hold = std::unique_lock<std::mutex>;
int library_workspace(size_t bytes, hipStream_t stream, Hold& hold, void** out);

// Compute units of the current device.
int compute_units(int* out);

// A launch's error as a status.
int launched(const char* what);

}  // namespace steps
