// steps_buffers.cpp -- the workspace of libapex_steps.so under two threads, without
// a GPU (test_steps_buffers.py): library_buffers.cpp's runtime, with a stop at the first
// or the second launch of a call.
#include <hip/hip_runtime.h>

#define hipLaunchKernel launch_one
#define main other_program
#include "library_buffers.cpp"
#undef main
#undef hipLaunchKernel

#include "apex_steps.h"

namespace {

int g_stop_at = 0;      // launches from here on until one stops

}  // namespace

extern "C" hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t stream)
{
    {
        std::lock_guard<std::mutex> lock(g_m);
        if (g_stop_at && --g_stop_at == 0) g_stop = true;
    }
    return launch_one(f, grid, block, args, lds, stream);
}

namespace {

int tree(int max_nodes)
{
    return symbol<decltype(apex_steps_tree_attention)>("apex_steps_tree_attention")(
        at(0), 0, at(1), at(2), 0, (int32_t*)at(3), (uint64_t*)at(4), at(5), at(6), (int32_t*)at(7), 10, (int32_t*)at(8), at(9), nullptr,
        4, 50, max_nodes, 32, 8, 128, 16, 100, 0.1f, nullptr, 0, nullptr);
}

}  // namespace

// library, the launch that stops (1, 2), what the other thread does (grow, release)
int main(int argc, char** argv)
{
    if (argc != 4) return 2;
    g_lib = dlopen(argv[1], RTLD_NOW | RTLD_LOCAL);
    if (!g_lib) {
        fprintf(stderr, "%s\n", dlerror());
        return 2;
    }
    const bool grow = argv[3][0] == 'g';
    if (tree(4) != 0 || g_launches != 2 || g_live.size() != 1) return 2;
    g_stop_at = atoi(argv[2]);
    int other = 0;
    std::thread a([&] {
        if (tree(4) != 0) exit(2);
    });
    std::thread b([&] {
        {
            std::unique_lock<std::mutex> lock(g_m);
            g_cv.wait(lock, [] { return g_stopped; });
        }
        other = grow ? tree(64) : symbol<int()>("apex_steps_release_workspace")();
    });
    a.join();
    b.join();
    printf("freed before the launch: %d, in all: %d, launches: %d\n", g_freed_meanwhile, g_frees, g_launches);
    if (other != 0 || g_frees != 1 || g_launches != (grow ? 6 : 4)) return 2;
    return g_freed_meanwhile == 0 ? 0 : 1;
}
