// kv4_rows.hip -- rows into the 4-bit KV cache and back (include/apex_kv4.h).
//
// A row of 128 values is handled by 16 lanes, 8 values (16 bytes of fp16, 4 of
// codes) each, so a group of 32 is a quad of lanes and its largest value two
// quad permutes away.  A wave takes four consecutive tokens of one kv-head and
// a work group sixteen: where they lie in consecutive slots, as a prompt's do,
// a wave's codes are 256 contiguous bytes of K and of V, and the work group
// writes (or reads) whole slabs.  Bound by HBM for prompts (5.4 TB/s of reads
// and writes together; a large copy has 4.5-4.8), by the launch and two round trips
// for a decode step.
#include "kv4_host.h"

namespace {

using namespace kv4;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kRowLanes = 16;
// fp16 rows up to half the 256 MB Infinity Cache are read and written through
// it: they come out of a projection that has just written them, or go to a
// reader that comes next.  More would not stay there and goes past it (54 000
// tokens of 8 kv-heads, 224 MB: appended in 51 us, 58 through it, read back in
// 40, 49 through it).
constexpr size_t kCachedBytes = (size_t)128 << 20;
constexpr int kTokens = kThreads / kRowLanes;   // tokens of a work group at a time
constexpr int kRows = 2;                        // and how many times

__device__ inline f16x2 as_h2(unsigned u) { return __builtin_bit_cast(f16x2, u); }

// Max over a quad of lanes.
__device__ inline int quad_max(int x)
{
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, true));   // lanes 1, 0, 3, 2
    return max(x, __builtin_amdgcn_update_dpp(0, x, 0x4e, 0xf, 0xf, true));   // lanes 2, 3, 0, 1
}

// Codes and scale byte of a lane's 8 values, which share their group with the
// other lanes of the quad.  The scale's exponent comes from the bits of the
// largest value m: with m = 1.f 2^k it is k - 2 while 1.f <= 1.5 (m <= 6 2^(k-2)),
// else k - 1.  The conversion rounds to the nearest code, ties to the even one.
__device__ inline unsigned quantise(u32x4 x, int& scale)
{
    int m = 0;   // |value| bits, two to a word; NaN and infinity above all
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max((int)(x[i] & 0x7fff), (int)((x[i] >> 16) & 0x7fff)));
    m = quad_max(m);
    const float mf = (float)__builtin_bit_cast(_Float16, (unsigned short)m);   // (a subnormal becomes normal)
    scale = m == 0 ? 127 : (int)((__float_as_uint(mf) + 0x3fffffu) >> 23) - 2;
    unsigned codes = 0;
    if (m >= 0x7c00) {
        scale = kNanScale;
        return codes;
    }
    const float s = __uint_as_float((unsigned)scale << 23);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, as_h2(x[0]), s, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, as_h2(x[1]), s, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, as_h2(x[2]), s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, as_h2(x[3]), s, 3);
}

// The largest finite fp16 for what lies past it (an append can round 65504 up
// to 4 x 2^14).
__device__ inline unsigned saturate(f16x2 v)
{
    const f16x2 top = {(_Float16)65504.f, (_Float16)65504.f};
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_elementwise_min(v, top), -top));
}

__device__ inline u32x4 dequantise(unsigned codes, int scale)
{
    const float s = __uint_as_float((unsigned)scale << 23);
    u32x4 r;
    r[0] = saturate(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 0));
    r[1] = saturate(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 1));
    r[2] = saturate(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 2));
    r[3] = saturate(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 3));
    if (scale == kNanScale) r = u32x4{0x7e007e00u, 0x7e007e00u, 0x7e007e00u, 0x7e007e00u};
    return r;
}

struct RowShape {
    int T, Hkv;
    int64_t capacity;       // slots of the pool
    int64_t token_stride;   // bytes between tokens of the new rows
};

// A work group's tokens and head: heads fastest, so that the work groups of the
// same tokens run together.  A lane takes piece c of rows t, t + kTokens, ...
struct RowPlace {
    int64_t t;
    int g, c;
};

__device__ inline RowPlace row_place(const RowShape& s)
{
    const unsigned group = blockIdx.x, chunk = group / (unsigned)s.Hkv;
    return {(int64_t)chunk * (kTokens * kRows) + threadIdx.x / kRowLanes, (int)(group - chunk * (unsigned)s.Hkv),
            (int)(threadIdx.x % kRowLanes)};
}

// Slots of a lane's rows, -1 outside the pool: all are asked for before the
// first is needed, and rows only once their slot is known (padding costs its
// slot and nothing else).
__device__ inline void load_slots(const int64_t* slots, const RowShape& s, int64_t t, int64_t (&slot)[kRows])
{
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t at = t + i * kTokens;
        slot[i] = at < s.T ? slots[at] : -1;
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (slot[i] >= s.capacity) slot[i] = -1;
}

template <bool kStream>
__global__ __launch_bounds__(kThreads) void append_kernel(const char* __restrict__ k_new, const char* __restrict__ v_new,
                                                          char* __restrict__ cache, const int64_t* __restrict__ slots,
                                                          const int32_t* __restrict__ token_positions,
                                                          int32_t* __restrict__ positions, float* __restrict__ weights,
                                                          RowShape s)
{
    const RowPlace r = row_place(s);
    int64_t slot[kRows];
    load_slots(slots, s, r.t, slot);
    u32x4 k[kRows], v[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (slot[i] < 0) continue;   // (all 16 lanes of a row)
        const int64_t from = (r.t + i * kTokens) * s.token_stride + (int64_t)r.g * (kHeadDim * 2) + r.c * 16;
        k[i] = kStream ? __builtin_nontemporal_load((const u32x4*)(k_new + from)) : *(const u32x4*)(k_new + from);
        v[i] = kStream ? __builtin_nontemporal_load((const u32x4*)(v_new + from)) : *(const u32x4*)(v_new + from);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        if (slot[i] < 0) continue;
        int ks, vs;
        const unsigned kc = quantise(k[i], ks), vc = quantise(v[i], vs);
        const int64_t row = (slot[i] / kBlockSize) * s.Hkv + r.g;
        const int at = (int)(slot[i] % kBlockSize), c = r.c;
        char* slab = cache + row * kSlabBytes;
        *(unsigned*)(slab + at * 64 + c * 4) = kc;
        *(unsigned*)(slab + v_code_offset(at, c)) = vc;
        if ((c & 3) == 0) {
            slab[kKScales + at * 4 + (c >> 2)] = (char)ks;
            slab[kVScales + (c >> 2) * kBlockSize + at] = (char)vs;
        }
        if (positions && c == 1) positions[row * kBlockSize + at] = token_positions[r.t + i * kTokens];
        if (weights && c == 2) weights[row * kBlockSize + at] = 0.f;
    }
}

template <bool kStream>
__global__ __launch_bounds__(kThreads) void gather_kernel(const char* __restrict__ cache, const int64_t* __restrict__ slots,
                                                          char* __restrict__ k_out, char* __restrict__ v_out, RowShape s)
{
    const RowPlace r = row_place(s);
    int64_t slot[kRows];
    load_slots(slots, s, r.t, slot);
    unsigned kc[kRows], vc[kRows];
    int ks[kRows], vs[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        kc[i] = vc[i] = 0;
        ks[i] = vs[i] = 127;
        if (slot[i] < 0) continue;
        const char* slab = cache + ((slot[i] / kBlockSize) * s.Hkv + r.g) * kSlabBytes;
        const int at = (int)(slot[i] % kBlockSize), c = r.c;
        kc[i] = *(const unsigned*)(slab + at * 64 + c * 4);
        vc[i] = *(const unsigned*)(slab + v_code_offset(at, c));
        ks[i] = *(const unsigned char*)(slab + kKScales + at * 4 + (c >> 2));
        vs[i] = *(const unsigned char*)(slab + kVScales + (c >> 2) * kBlockSize + at);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t t = r.t + i * kTokens;
        if (t >= s.T) continue;
        const int64_t to = (t * s.Hkv + r.g) * (kHeadDim * 2) + r.c * 16;
        const u32x4 k = dequantise(kc[i], ks[i]), v = dequantise(vc[i], vs[i]);
        if (kStream) {
            __builtin_nontemporal_store(k, (u32x4*)(k_out + to));
            __builtin_nontemporal_store(v, (u32x4*)(v_out + to));
        } else {
            *(u32x4*)(k_out + to) = k;
            *(u32x4*)(v_out + to) = v;
        }
    }
}

// A launch holds fewer than 2^32 threads.
int check_rows(int T, int Hkv)
{
    if (T < 0) return fail(APEX_ERR_INVALID_ARG, "T = %d is negative", T);
    if (((int64_t)T + kTokens - 1) / kTokens * Hkv >= (1 << 24))
        return fail(APEX_ERR_UNSUPPORTED, "ceil(T / 16) * Hkv reaches 2^24 (T = %d, Hkv = %d)", T, Hkv);
    return APEX_OK;
}

dim3 row_grid(int T, int Hkv)
{
    return dim3((unsigned)(((int64_t)T + kTokens * kRows - 1) / (kTokens * kRows) * Hkv));
}

}  // namespace

extern "C" int apex_kv4_append(const void* k_new, const void* v_new, int64_t new_token_stride, void* kv_cache,
                               const int64_t* slot_mapping, const int32_t* token_positions, int32_t* positions,
                               float* weights, int T, int Hkv, int d, int block_size, int64_t num_blocks, void* stream)
{
    apex::clear_error();
    int rc = check_cache(Hkv, d, block_size, num_blocks);
    if (rc == APEX_OK) rc = check_rows(T, Hkv);
    if (rc != APEX_OK) return rc;
    const int64_t row = (int64_t)Hkv * d, stride = new_token_stride == 0 ? row : new_token_stride;
    if (stride < row || stride % 8 != 0 || stride > INT64_MAX / 4 / ((int64_t)T + 1))
        return fail(APEX_ERR_INVALID_ARG, "new_token_stride %lld must be 0 or a multiple of 8 >= Hkv * d",
                    (long long)new_token_stride);
    if ((positions != nullptr) != (token_positions != nullptr))
        return fail(APEX_ERR_INVALID_ARG, "positions and token_positions go together");
    if (T == 0 || num_blocks == 0) return APEX_OK;   // no row, or every slot is out of the pool
    if (!k_new || !v_new || !kv_cache || !slot_mapping) return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(kv_cache, 16) || !aligned(weights, 16))
        return fail(APEX_ERR_INVALID_ARG, "k_new, v_new, kv_cache and weights must be 16-byte aligned");
    if (!aligned(slot_mapping, 8) || !aligned(token_positions, 4) || !aligned(positions, 4))
        return fail(APEX_ERR_INVALID_ARG, "slot_mapping, token_positions or positions is misaligned");
    const size_t new_bytes = ((size_t)(T - 1) * stride + row) * 2, sb = slot_bytes(Hkv, num_blocks);
    const Extent in[] = {{"k_new", k_new, new_bytes},
                         {"v_new", v_new, new_bytes},
                         {"slot_mapping", slot_mapping, (size_t)T * 8},
                         {"token_positions", token_positions, (size_t)T * 4},
                         {"kv_cache", kv_cache, cache_bytes(Hkv, num_blocks)},
                         {"positions", positions, sb},
                         {"weights", weights, sb}};
    if ((rc = check_disjoint(in[4], in, 4)) != APEX_OK || (rc = check_disjoint(in[5], in, 5)) != APEX_OK ||
        (rc = check_disjoint(in[6], in, 6)) != APEX_OK)
        return rc;
    const RowShape s = {T, Hkv, num_blocks * kBlockSize, stride * 2};
    const auto kernel = 2 * (size_t)T * row * 2 > kCachedBytes ? append_kernel<true> : append_kernel<false>;
    kernel<<<row_grid(T, Hkv), kThreads, 0, (hipStream_t)stream>>>(
        (const char*)k_new, (const char*)v_new, (char*)kv_cache, slot_mapping, token_positions, positions, weights, s);
    return launched("kv4 append");
}

extern "C" int apex_kv4_gather(const void* kv_cache, const int64_t* slot_mapping, void* k_out, void* v_out, int T,
                               int Hkv, int d, int block_size, int64_t num_blocks, void* stream)
{
    apex::clear_error();
    int rc = check_cache(Hkv, d, block_size, num_blocks);
    if (rc == APEX_OK) rc = check_rows(T, Hkv);
    if (rc != APEX_OK || T == 0) return rc;
    if ((!kv_cache && num_blocks > 0) || !slot_mapping || !k_out || !v_out) return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(kv_cache, 16))
        return fail(APEX_ERR_INVALID_ARG, "kv_cache, k_out and v_out must be 16-byte aligned");
    if (!aligned(slot_mapping, 8)) return fail(APEX_ERR_INVALID_ARG, "slot_mapping must be 8-byte aligned");
    const size_t out_bytes = (size_t)T * Hkv * d * 2;
    const Extent all[] = {{"kv_cache", kv_cache, cache_bytes(Hkv, num_blocks)},
                          {"slot_mapping", slot_mapping, (size_t)T * 8},
                          {"k_out", k_out, out_bytes},
                          {"v_out", v_out, out_bytes}};
    if ((rc = check_disjoint(all[2], all, 2)) != APEX_OK || (rc = check_disjoint(all[3], all, 3)) != APEX_OK) return rc;
    const RowShape s = {T, Hkv, num_blocks * kBlockSize, 0};
    const auto kernel = 2 * out_bytes > kCachedBytes ? gather_kernel<true> : gather_kernel<false>;
    kernel<<<row_grid(T, Hkv), kThreads, 0, (hipStream_t)stream>>>((const char*)kv_cache, slot_mapping, (char*)k_out,
                                                                   (char*)v_out, s);
    return launched("kv4 gather");
}
