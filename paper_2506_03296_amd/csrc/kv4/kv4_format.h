// kv4_format.h -- layout of the 4-bit KV cache (include/apex_kv4.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kv4 {

constexpr int kHeadDim = 128;
constexpr int kBlockSize = 16;
constexpr int kSlabBytes = 2176;
constexpr int kVCodes = 1024;     // offset of the V codes in a slab
constexpr int kKScales = 2048;
constexpr int kVScales = 2112;
constexpr int kNanScale = 255;

// Offset of the 4 bytes that hold V's dims [8c, 8c + 8) of token t.
__host__ __device__ inline int v_code_offset(int t, int c) { return kVCodes + (t >> 2) * 256 + c * 16 + (t & 3) * 4; }

}  // namespace kv4
