// kv4_host.h -- argument checks and workspaces shared by the entry points of
// libapex_kv4.so.
#pragma once

#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <mutex>

#include "apex_kv4.h"
#include "kv4_format.h"
#include "status.h"

namespace kv4 __attribute__((visibility("hidden"))) {

using apex::fail;

constexpr int kMaxDevices = 64;

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline bool overlaps(const void* a, size_t na, const void* b, size_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb && y < x + na;
}

// A buffer of a call, for the checks of what it writes against what it reads.
struct Extent {
    const char* name;
    const void* p;
    size_t bytes;
};

// APEX_OK, or an error if `written` (when not NULL) overlaps one of `others`.
int check_disjoint(const Extent& written, const Extent* others, int n);

// Shapes common to the calls; Hq = Hkv where a call has no q-heads.
int check_cache(int Hkv, int d, int block_size, int64_t num_blocks);
int check_batch(int B, int Hq, int Hkv, int d, int block_size, int64_t num_blocks, int64_t block_table_stride);

inline size_t cache_bytes(int Hkv, int64_t num_blocks) { return (size_t)num_blocks * Hkv * kSlabBytes; }
inline size_t slot_bytes(int Hkv, int64_t num_blocks) { return (size_t)num_blocks * Hkv * kBlockSize * 4; }

// The caller's workspace, checked.
int check_workspace(const void* given, size_t given_bytes, size_t bytes);

// One of the library's own buffers on the current device, at least `bytes`
// long; counters are zero when they are allocated.  Under stream capture it is
// refused: a graph would keep an address that a later call may free.
// The caller holds the buffers (`hold`, locked here) until it has launched what
// uses them: another thread's call that grows or releases them waits for what has
// been launched, and frees them then.
enum LibraryBuffer { kCounters = 0, kPartials = 1, kMasks = 2, kLibraryBuffers = 3 };
typedef std::unique_lock<std::mutex> Hold;
int library_buffer(LibraryBuffer kind, size_t bytes, hipStream_t stream, Hold& hold, void** out);

// Compute units of the current device.
int compute_units(int* out);

// A launch's error as a status.
int launched(const char* what);

}  // namespace kv4
