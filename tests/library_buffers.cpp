// library_buffers.cpp -- a library's own workspaces under two threads, without a
// GPU (test_library_buffers.py).
//
// The program stands in for the HIP runtime: its functions are found before the
// runtime's.  One thread's call stops at its launch while another's grows or
// releases the workspaces; nothing may be freed before the launch has been made.
#include <dlfcn.h>
#include <hip/hip_runtime.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <chrono>
#include <condition_variable>
#include <mutex>
#include <set>
#include <thread>

#include "apex_decode.h"
#include "apex_kv4.h"

namespace {

std::mutex g_m;
std::condition_variable g_cv;
std::set<void*> g_live;
int g_frees = 0, g_launches = 0;
bool g_stop = false, g_stopped = false;   // the next launch stops; it has
int g_freed_meanwhile = 0;

}  // namespace

extern "C" {

hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipDeviceSynchronize(void) { return hipSuccess; }
hipError_t hipGetLastError(void) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "?"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipMemset(void* p, int v, size_t n) { memset(p, v, n); return hipSuccess; }
hipError_t hipModuleOccupancyMaxActiveBlocksPerMultiprocessor(int* n, hipFunction_t, int, size_t) { *n = 2; return hipSuccess; }
hipError_t hipOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void*, int, size_t) { *n = 2; return hipSuccess; }

hipError_t hipMalloc(void** p, size_t n)
{
    std::lock_guard<std::mutex> lock(g_m);
    *p = aligned_alloc(256, n);
    g_live.insert(*p);
    return hipSuccess;
}

hipError_t hipFree(void* p)
{
    std::lock_guard<std::mutex> lock(g_m);
    if (g_live.erase(p) != 1) abort();
    ++g_frees;
    g_cv.notify_all();
    free(p);
    return hipSuccess;
}

hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t)
{
    std::unique_lock<std::mutex> lock(g_m);
    ++g_launches;
    if (g_stop) {
        g_stop = false;
        g_stopped = true;
        const int before = g_frees;
        g_cv.notify_all();
        g_cv.wait_for(lock, std::chrono::milliseconds(300), [&] { return g_frees != before; });
        g_freed_meanwhile = g_frees - before;
    }
    return hipSuccess;
}

hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t) { return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream)
{
    *grid = *block = dim3(1);
    *lds = 0;
    *stream = nullptr;
    return hipSuccess;
}
void** __hipRegisterFatBinary(const void*) { static void* x; return &x; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}

}  // extern "C"

namespace {

void* g_lib;

template <typename F>
F* symbol(const char* name)
{
    void* f = dlsym(g_lib, name);
    if (!f) {
        fprintf(stderr, "%s: %s\n", name, dlerror());
        exit(2);
    }
    return (F*)f;
}

void* at(int i) { return (void*)(0x7f0000000000 + ((long)i << 36)); }

int attention(int B)
{
    return symbol<decltype(apex_kv4_attention)>("apex_kv4_attention")(at(0), at(1), (int32_t*)at(2), 10, (int32_t*)at(3), at(4),
                                                                      nullptr, B, 8, 8, 128, 16, 100, 0.1f, nullptr, 0, nullptr);
}

int evict(int B)
{
    return symbol<decltype(apex_kv4_evict)>("apex_kv4_evict")(at(0), (int32_t*)at(2), 10, (int32_t*)at(3), (float*)at(4),
                                                              (int32_t*)at(5), B, 8, 128, 16, 100, 64, 4, 16, nullptr, 0, nullptr);
}

int decode(int B)
{
    apex_decode_args a = {};
    a.q = at(0), a.k_cache = at(1), a.v_cache = at(2), a.block_table = (int32_t*)at(3), a.context_lens = (int32_t*)at(4);
    a.out = at(5), a.B = B, a.Hq = a.Hkv = 8, a.d = 128, a.block_size = 16, a.scale = 0.1f, a.block_table_stride = 10;
    return symbol<decltype(apex_decode_attention_ex)>("apex_decode_attention_ex")(&a);
}

}  // namespace

// library, call (attention, evict, decode), what the other thread does (grow,
// release)
int main(int argc, char** argv)
{
    if (argc != 4) return 2;
    g_lib = dlopen(argv[1], RTLD_NOW | RTLD_LOCAL);
    if (!g_lib) {
        fprintf(stderr, "%s\n", dlerror());
        return 2;
    }
    int (*const call)(int) = argv[2][0] == 'a' ? attention : argv[2][0] == 'e' ? evict : decode;
    int (*const release)() = symbol<int()>(argv[2][0] == 'd' ? "apex_decode_release_workspace" : "apex_kv4_release_workspace");
    const bool grow = argv[3][0] == 'g';
    if (call(4) != 0 || g_launches == 0 || g_live.empty()) return 2;   // the workspaces are there
    g_stop = true;
    int other = 0;
    std::thread a([&] {
        if (call(4) != 0) exit(2);
    });
    std::thread b([&] {
        {
            std::unique_lock<std::mutex> lock(g_m);
            g_cv.wait(lock, [] { return g_stopped; });
        }
        other = grow ? call(200000) : release();
    });
    a.join();
    b.join();
    printf("freed before the launch: %d, in all: %d\n", g_freed_meanwhile, g_frees);
    if (other != 0 || g_frees == 0) return 2;
    return g_freed_meanwhile == 0 ? 0 : 1;
}
