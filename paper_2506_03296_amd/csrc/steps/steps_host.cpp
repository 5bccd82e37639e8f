// steps_host.cpp -- argument checks and workspaces of libapex_steps.so.
#include "steps_host.h"

#include <math.h>

namespace steps {

namespace {

constexpr int kMaxDevices = 64;

struct Buffer {
    void* ptr = nullptr;
    size_t bytes = 0;
};

std::mutex g_mutex;         // of the workspaces
Buffer g_workspace[kMaxDevices];
std::mutex g_units_mutex;
int g_units[kMaxDevices];

int current_device(int* dev)
{
    hipError_t e = hipGetDevice(dev);
    if (e != hipSuccess) return fail(APEX_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
    if (*dev < 0 || *dev >= kMaxDevices) return fail(APEX_ERR_HIP, "device ordinal %d out of range", *dev);
    return APEX_OK;
}

int check_stride(const char* name, int64_t* stride, int64_t row)
{
    if (*stride == 0) *stride = row;
    if (*stride < row || *stride % 8 != 0)
        return fail(APEX_ERR_INVALID_ARG, "%s %lld must be 0 or a multiple of 8 and at least heads * d = %lld", name,
                    (long long)*stride, (long long)row);
    if (*stride > INT_MAX) return fail(APEX_ERR_UNSUPPORTED, "%s exceeds 2^31 - 1", name);
    return APEX_OK;
}

}  // namespace

int check_disjoint(const Extent& written, const Extent* others, int n)
{
    if (!written.p || !written.bytes) return APEX_OK;
    const uintptr_t x = (uintptr_t)written.p;
    for (int i = 0; i < n; ++i) {
        const uintptr_t y = (uintptr_t)others[i].p;
        if (others[i].p && others[i].bytes && x < y + others[i].bytes && y < x + written.bytes)
            return fail(APEX_ERR_INVALID_ARG, "%s overlaps %s", written.name, others[i].name);
    }
    return APEX_OK;
}

int check_attention(int B, int T, int Hq, int Hkv, int d, float scale, int64_t* q_stride, int64_t* kv_stride)
{
    if (B < 0 || T < 0) return fail(APEX_ERR_INVALID_ARG, "B = %d and T = %d must not be negative", B, T);
    if (Hkv <= 0) return fail(APEX_ERR_INVALID_ARG, "Hkv = %d must be positive", Hkv);
    if (Hq <= 0 || Hq % Hkv != 0)
        return fail(APEX_ERR_INVALID_ARG, "Hq = %d must be a positive multiple of Hkv = %d", Hq, Hkv);
    if (d != 128) return fail(APEX_ERR_UNSUPPORTED, "head dim %d unsupported (only 128)", d);
    if (Hq > kMostHeads) return fail(APEX_ERR_UNSUPPORTED, "Hq = %d exceeds %d", Hq, kMostHeads);
    if (((int64_t)T + 256) * Hq > INT_MAX / 2) return fail(APEX_ERR_UNSUPPORTED, "(T + 256) * Hq reaches 2^30");
    if (B > (1 << 22)) return fail(APEX_ERR_UNSUPPORTED, "B exceeds 2^22");
    if (((int64_t)B + (int64_t)(T / 32 + 1) * (Hq / Hkv)) * Hkv > INT_MAX / 2)
        return fail(APEX_ERR_UNSUPPORTED, "B * Hkv + T * Hq / 32 reaches 2^30");
    if (!isfinite(scale)) return fail(APEX_ERR_INVALID_ARG, "scale is not finite");
    const int rc = check_stride("q_token_stride", q_stride, (int64_t)Hq * d);
    return rc != APEX_OK ? rc : check_stride("kv_token_stride", kv_stride, (int64_t)Hkv * d);
}

int check_workspace(const void* given, size_t given_bytes, size_t bytes)
{
    if (!aligned(given, 256)) return fail(APEX_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (given_bytes < bytes)
        return fail(APEX_ERR_OUT_OF_MEMORY, "caller workspace holds %zu bytes, %zu needed", given_bytes, bytes);
    return APEX_OK;
}

int library_workspace(size_t bytes, hipStream_t stream, Hold& hold, void** out)
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
    hold = Hold(g_mutex);
    Buffer& w = g_workspace[dev];
    if (w.bytes < bytes) {
        if (w.ptr) {
            e = hipDeviceSynchronize();
            if (e != hipSuccess) return fail(APEX_ERR_HIP, "hipDeviceSynchronize: %s", hipGetErrorString(e));
            (void)hipFree(w.ptr);
            w = Buffer();
        }
        const size_t want = align_up(bytes, 1 << 20);
        void* p = nullptr;
        e = hipMalloc(&p, want);
        if (e != hipSuccess || !p) {
            (void)hipGetLastError();
            return fail(APEX_ERR_OUT_OF_MEMORY, "hipMalloc(%zu) for a workspace failed: %s", want, hipGetErrorString(e));
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

}  // namespace steps

extern "C" {

const char* apex_steps_last_error(void) { return apex::last_error_message(); }

int apex_steps_release_workspace(void)
{
    apex::clear_error();
    std::lock_guard<std::mutex> lock(steps::g_mutex);
    int rc = APEX_OK;
    for (int d = 0; d < steps::kMaxDevices; ++d) {
        steps::Buffer& w = steps::g_workspace[d];
        if (!w.ptr) continue;
        int prev = 0;
        (void)hipGetDevice(&prev);
        if (hipSetDevice(d) == hipSuccess && hipDeviceSynchronize() == hipSuccess) {
            (void)hipFree(w.ptr);
            w = steps::Buffer();
        } else {
            rc = apex::fail(APEX_ERR_HIP, "could not release the workspace of device %d", d);
        }
        (void)hipSetDevice(prev);
    }
    return rc;
}

}  // extern "C"
