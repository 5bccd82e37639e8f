// kv4_host.cpp -- argument checks and workspaces of libapex_kv4.so.
#include "kv4_host.h"

namespace kv4 {

namespace {

struct Buffer {
    void* ptr = nullptr;
    size_t bytes = 0;
};

std::mutex g_mutex;         // of the buffers
Buffer g_buffers[kMaxDevices][kLibraryBuffers];
std::mutex g_units_mutex;
int g_units[kMaxDevices];

int current_device(int* dev)
{
    hipError_t e = hipGetDevice(dev);
    if (e != hipSuccess) return fail(APEX_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
    if (*dev < 0 || *dev >= kMaxDevices) return fail(APEX_ERR_HIP, "device ordinal %d out of range", *dev);
    return APEX_OK;
}

}  // namespace

int check_disjoint(const Extent& written, const Extent* others, int n)
{
    if (!written.p) return APEX_OK;
    for (int i = 0; i < n; ++i)
        if (others[i].p && overlaps(written.p, written.bytes, others[i].p, others[i].bytes))
            return fail(APEX_ERR_INVALID_ARG, "%s overlaps %s", written.name, others[i].name);
    return APEX_OK;
}

int check_cache(int Hkv, int d, int block_size, int64_t num_blocks)
{
    if (Hkv <= 0) return fail(APEX_ERR_INVALID_ARG, "Hkv = %d must be positive", Hkv);
    if (d != kHeadDim) return fail(APEX_ERR_UNSUPPORTED, "head dim %d unsupported (only 128)", d);
    if (block_size != kBlockSize) return fail(APEX_ERR_UNSUPPORTED, "block_size %d unsupported (only 16)", block_size);
    if (num_blocks < 0) return fail(APEX_ERR_INVALID_ARG, "num_blocks is negative");
    if (num_blocks > INT_MAX) return fail(APEX_ERR_UNSUPPORTED, "num_blocks exceeds 2^31 - 1");
    if (num_blocks > INT64_MAX / ((int64_t)Hkv * kSlabBytes))
        return fail(APEX_ERR_INVALID_ARG, "cache size overflows");
    return APEX_OK;
}

int check_batch(int B, int Hq, int Hkv, int d, int block_size, int64_t num_blocks, int64_t block_table_stride)
{
    if (B < 0) return fail(APEX_ERR_INVALID_ARG, "B = %d is negative", B);
    const int rc = check_cache(Hkv, d, block_size, num_blocks);
    if (rc != APEX_OK) return rc;
    if (Hq <= 0 || Hq % Hkv != 0)
        return fail(APEX_ERR_INVALID_ARG, "Hq = %d must be a positive multiple of Hkv = %d", Hq, Hkv);
    const int G = Hq / Hkv;
    if (G != 1 && G != 2 && G != 4 && G != 8)
        return fail(APEX_ERR_UNSUPPORTED, "group size Hq/Hkv = %d unsupported (1, 2, 4, 8)", G);
    if (block_table_stride < 0) return fail(APEX_ERR_INVALID_ARG, "block_table_stride is negative");
    if (block_table_stride >= INT_MAX / kBlockSize)
        return fail(APEX_ERR_UNSUPPORTED, "block_table_stride %lld reaches 2^27 - 1", (long long)block_table_stride);
    if ((int64_t)B * Hkv > (int64_t)INT_MAX / (block_table_stride + 64))
        return fail(APEX_ERR_UNSUPPORTED, "B * Hkv * (block_table_stride + 64) exceeds 2^31 - 1");
    return APEX_OK;
}

int check_workspace(const void* given, size_t given_bytes, size_t bytes)
{
    if (!aligned(given, 256)) return fail(APEX_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (given_bytes < bytes)
        return fail(APEX_ERR_OUT_OF_MEMORY, "caller workspace holds %zu bytes, %zu needed", given_bytes, bytes);
    return APEX_OK;
}

int library_buffer(LibraryBuffer kind, size_t bytes, hipStream_t stream, Hold& hold, void** out)
{
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    hipError_t e = hipStreamIsCapturing(stream, &st);
    if (e != hipSuccess || st != hipStreamCaptureStatusNone) {
        (void)hipGetLastError();
        return fail(APEX_ERR_INVALID_ARG, "a call under stream capture needs a workspace of its own");
    }
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != APEX_OK) return rc;
    if (!hold) hold = Hold(g_mutex);
    Buffer& w = g_buffers[dev][kind];
    if (w.bytes < bytes) {
        if (w.ptr) {
            e = hipDeviceSynchronize();
            if (e != hipSuccess) return fail(APEX_ERR_HIP, "hipDeviceSynchronize: %s", hipGetErrorString(e));
            (void)hipFree(w.ptr);
            w = Buffer();
        }
        const size_t want = align_up(bytes + bytes / 4, 1 << 20);
        void* p = nullptr;
        e = hipMalloc(&p, want);
        if (e != hipSuccess || !p) {
            (void)hipGetLastError();
            return fail(APEX_ERR_OUT_OF_MEMORY, "hipMalloc(%zu) for a workspace failed: %s", want, hipGetErrorString(e));
        }
        if (kind == kCounters) {
            e = hipMemset(p, 0, want);
            if (e == hipSuccess) e = hipDeviceSynchronize();   // zero before any stream's kernel runs
            if (e != hipSuccess) {
                (void)hipFree(p);
                return fail(APEX_ERR_HIP, "clearing the counters: %s", hipGetErrorString(e));
            }
        }
        w.ptr = p;
        w.bytes = want;
    }
    *out = w.ptr;
    return APEX_OK;
}

int compute_units(int* out)
{
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != APEX_OK) return rc;
    std::lock_guard<std::mutex> lock(g_units_mutex);
    if (g_units[dev] == 0) {
        int n = 0;
        hipError_t e = hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev);
        if (e != hipSuccess || n <= 0)
            return fail(APEX_ERR_HIP, "hipDeviceGetAttribute(CU count): %s", hipGetErrorString(e));
        g_units[dev] = n;
    }
    *out = g_units[dev];
    return APEX_OK;
}

int launched(const char* what)
{
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)APEX_OK : fail(APEX_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
}

}  // namespace kv4

extern "C" {

const char* apex_kv4_last_error(void) { return apex::last_error_message(); }

int apex_kv4_release_workspace(void)
{
    apex::clear_error();
    std::lock_guard<std::mutex> lock(kv4::g_mutex);
    int rc = APEX_OK;
    for (int d = 0; d < kv4::kMaxDevices; ++d) {
        for (auto& w : kv4::g_buffers[d]) {
            if (!w.ptr) continue;
            int prev = 0;
            (void)hipGetDevice(&prev);
            if (hipSetDevice(d) == hipSuccess && hipDeviceSynchronize() == hipSuccess) {
                (void)hipFree(w.ptr);
                w = kv4::Buffer();
            } else {
                rc = apex::fail(APEX_ERR_HIP, "could not release the workspaces of device %d", d);
            }
            (void)hipSetDevice(prev);
        }
    }
    return rc;
}

}  // extern "C"
