// kv4_evict.hip -- eviction from the 4-bit KV cache (include/apex_kv4.h).
//
// A token's key is 32 bits whose order is the order of keeping: all ones for a
// protected token, else its weight's bits made monotonic.  select_kernel finds,
// for one (request, kv-head) pair per work group, the key of the last token
// kept, digit by digit from the top (counts of a digit's values among the keys
// that agree so far), and writes a mask, one bit per slot.  move_kernel reads
// the masks only, so it may overwrite weights and positions: the i-th evicted
// slot below `keep` takes the i-th kept one from `keep` on.  Sources and targets
// are disjoint, so the moves need no order, and a cut by a few tokens moves a
// few rows.
#include "kv4_host.h"

namespace {

using namespace kv4;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048;
constexpr int kMoveThreads = 256;
constexpr int kMoves = 256;        // moves of a work group at a time

struct EvictParams {
    char* cache;
    const int32_t* bt;
    const int32_t* lens;
    float* weights;
    int32_t* positions;
    uint64_t* masks;       // [B][Hkv][words], bit i of word w: slot 64 w + i is kept
    int32_t* counts;       // [B][Hkv] tokens to move
    int64_t num_blocks;
    int Hkv, stride, words;
    int keep, sinks, recent;
};

__device__ inline int context(const EvictParams& p, int b)
{
    const int64_t row = (int64_t)p.stride * kBlockSize;
    const int L = p.lens[b];
    return L > row ? (int)row : L;
}

// Index of slot t of pair (b, g) in weights and positions; -1 for a block
// outside the pool.
__device__ inline int64_t slot_index(const EvictParams& p, const int32_t* row, int g, int t)
{
    const int id = row[t / kBlockSize];
    return id >= 0 && (int64_t)id < p.num_blocks ? ((int64_t)id * p.Hkv + g) * kBlockSize + t % kBlockSize : -1;
}

// Order-preserving bits of a weight; below every protected token's.
__device__ inline unsigned weight_key(float w)
{
    if (w != w) w = -INFINITY;
    const unsigned u = __float_as_uint(w + 0.f);   // (-0 becomes 0)
    return (u >> 31) ? ~u : u | 0x80000000u;
}

__device__ inline int wave_sum(int x)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
    return x;
}

// Inclusive sum over the lanes of a wave.
__device__ inline int wave_scan(int x, int lane)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int y = __shfl_up(x, m, 64);
        if (lane >= m) x += y;
    }
    return x;
}

__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictParams p)
{
    __shared__ unsigned s_bins[kBins];
    __shared__ int s_wave[kSelectWaves];
    __shared__ unsigned s_digit;
    __shared__ int s_above;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = (int)blockIdx.x / p.Hkv, g = (int)blockIdx.x - b * p.Hkv;
    const int L = context(p, b);
    if (L <= p.keep) {
        if (tid == 0) p.counts[blockIdx.x] = 0;
        return;
    }
    const int32_t* row = p.bt + (int64_t)b * p.stride;

    // the newest position
    int newest = INT_MIN;
    for (int t = tid; t < L; t += kSelectThreads) {
        const int64_t i = slot_index(p, row, g, t);
        if (i >= 0) newest = max(newest, p.positions[i]);
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) newest = max(newest, __shfl_xor(newest, m, 64));
    if (lane == 0) s_wave[wave] = newest;
    __syncthreads();
    for (int i = 0; i < kSelectWaves; ++i) newest = max(newest, s_wave[i]);
    const int64_t recent_from = (int64_t)newest - p.recent;

    auto key_of = [&](int t) -> unsigned {
        const int64_t i = slot_index(p, row, g, t);
        if (i < 0) return 0u;
        const int pos = p.positions[i];
        return pos < p.sinks || (int64_t)pos > recent_from ? 0xffffffffu : weight_key(p.weights[i]);
    };

    // the key of the keep-th token in the order of keeping: 11, 11 and 10 bits
    unsigned prefix = 0, mask = 0;
    int need = p.keep;   // tokens to keep among those that agree with prefix
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < kBins; i += kSelectThreads) s_bins[i] = 0;
        __syncthreads();
        for (int t = tid; t < L; t += kSelectThreads) {
            const unsigned k = key_of(t);
            if ((k & mask) == prefix) atomicAdd(&s_bins[(k >> shift) & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        // thread i has bins 2 i' and 2 i' + 1, from the top: counts above a bin
        const int top = kBins - 1 - 2 * tid;
        const int c0 = (int)s_bins[top], c1 = (int)s_bins[top - 1];
        int incl = wave_scan(c0 + c1, lane);
        if (lane == 63) s_wave[wave] = incl;
        __syncthreads();
        for (int i = 0; i < wave; ++i) incl += s_wave[i];
        const int above = incl - c0 - c1;
        if (above < need && need <= above + c0) {
            s_digit = (unsigned)top;
            s_above = above;
        } else if (above + c0 < need && need <= incl) {
            s_digit = (unsigned)top - 1;
            s_above = above + c0;
        }
        __syncthreads();
        prefix |= s_digit << shift;
        mask |= ((1u << bits) - 1) << shift;
        need -= s_above;
    }
    // kept: keys above prefix, and the first `need` (in slot order) that equal it
    uint64_t* out = p.masks + (int64_t)blockIdx.x * p.words;
    int equal_before = 0, moved = 0;
    for (int t0 = 0; t0 < L; t0 += kSelectThreads) {
        const int t = t0 + tid;
        const unsigned k = t < L ? key_of(t) : 0u;
        const bool eq = t < L && k == prefix;
        const uint64_t eqs = __ballot(eq);
        __syncthreads();
        if (lane == 0) s_wave[wave] = __popcll(eqs);
        __syncthreads();
        int before = equal_before;
        for (int i = 0; i < kSelectWaves; ++i) {
            before += i < wave ? s_wave[i] : 0;
            equal_before += s_wave[i];
        }
        const int rank = before + __popcll(eqs & ((1ull << lane) - 1));
        const bool kept = t < L && (k > prefix || (eq && rank < need));
        const uint64_t bits = __ballot(kept);
        moved += kept && t >= p.keep;
        if (lane == 0 && t < L) out[t >> 6] = bits;
    }
    moved = wave_sum(moved);
    __syncthreads();
    if (lane == 0) s_wave[wave] = moved;
    __syncthreads();
    if (tid == 0) {
        int n = 0;
        for (int i = 0; i < kSelectWaves; ++i) n += s_wave[i];
        p.counts[blockIdx.x] = n;
    }
}

// The slots with ranks [r0, r0 + kMoves) among the set bits of f(word), words
// [w0, w1), into list; every thread of the work group takes part.
template <typename F>
__device__ inline void list_slots(int w0, int w1, int r0, int* list, int* s_wave, F f)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (w1 - w0 + kMoveThreads - 1) / kMoveThreads;
    const int a = min(w1, w0 + tid * per), e = min(w1, a + per);
    int n = 0;
    for (int w = a; w < e; ++w) n += __popcll(f(w));
    int rank = wave_scan(n, lane);
    __syncthreads();
    if (lane == 63) s_wave[wave] = rank;
    __syncthreads();
    for (int i = 0; i < wave; ++i) rank += s_wave[i];
    rank -= n;
    for (int w = a; w < e && rank < r0 + kMoves; ++w) {
        uint64_t m = f(w);
        const int c = __popcll(m);
        if (rank + c <= r0) {
            rank += c;
            continue;
        }
        for (; m; m &= m - 1, ++rank)
            if (rank >= r0 && rank < r0 + kMoves) list[rank - r0] = w * 64 + __builtin_ctzll(m);
    }
}

__global__ __launch_bounds__(kMoveThreads) void move_kernel(EvictParams p)
{
    __shared__ int s_to[kMoves], s_from[kMoves];
    __shared__ int s_wave[kMoveThreads / 64];
    const int tid = threadIdx.x;
    const int pair = (int)blockIdx.x, b = pair / p.Hkv, g = pair - b * p.Hkv;
    const int n = p.counts[pair];
    const int L = context(p, b);
    const uint64_t* kept = p.masks + (int64_t)pair * p.words;
    const int32_t* row = p.bt + (int64_t)b * p.stride;
    for (int r0 = (int)blockIdx.y * kMoves; r0 < n; r0 += (int)gridDim.y * kMoves) {
        const int keep = p.keep;
        list_slots(0, (keep + 63) / 64, r0, s_to, s_wave, [&](int w) -> uint64_t {
            const int left = keep - w * 64;
            return ~kept[w] & (left >= 64 ? ~0ull : (1ull << left) - 1);
        });
        list_slots(keep / 64, (L + 63) / 64, r0, s_from, s_wave, [&](int w) -> uint64_t {
            const int skip = keep - w * 64;
            return kept[w] & (skip <= 0 ? ~0ull : ~0ull << skip);
        });
        __syncthreads();
        // 16 lanes a move: lane c has 4 bytes of K, dims [8c, 8c + 8) of V
        const int c = tid & 15, m1 = min(kMoves, n - r0);
        for (int m = tid >> 4; m < m1; m += kMoveThreads / 16) {
            const int64_t to = slot_index(p, row, g, s_to[m]), from = slot_index(p, row, g, s_from[m]);
            if (to < 0 || from < 0) continue;
            const int ti = (int)(to % kBlockSize), fi = (int)(from % kBlockSize);
            char* ts = p.cache + to / kBlockSize * kSlabBytes;
            const char* fs = p.cache + from / kBlockSize * kSlabBytes;
            const unsigned k = *(const unsigned*)(fs + fi * 64 + c * 4), v = *(const unsigned*)(fs + v_code_offset(fi, c));
            if (c < 4) {
                const char s = fs[kVScales + c * kBlockSize + fi];
                ts[kVScales + c * kBlockSize + ti] = s;
            } else if (c == 4) {
                *(unsigned*)(ts + kKScales + ti * 4) = *(const unsigned*)(fs + kKScales + fi * 4);
            } else if (c == 5) {
                p.weights[to] = p.weights[from];
            } else if (c == 6) {
                p.positions[to] = p.positions[from];
            }
            *(unsigned*)(ts + ti * 64 + c * 4) = k;
            *(unsigned*)(ts + v_code_offset(ti, c)) = v;
        }
        __syncthreads();
    }
}

int64_t mask_words(int64_t stride) { return (stride * kBlockSize + 63) / 64; }

size_t count_bytes(int B, int Hkv) { return align_up((size_t)B * Hkv * 4, 256); }

size_t need_bytes(int B, int Hkv, int64_t stride)
{
    return count_bytes(B, Hkv) + align_up((size_t)B * Hkv * mask_words(stride) * 8, 256);
}

}  // namespace

extern "C" size_t apex_kv4_evict_workspace_bytes(int B, int Hkv, int64_t block_table_stride)
{
    apex::clear_error();
    if (check_batch(B, Hkv, Hkv, kHeadDim, kBlockSize, 0, block_table_stride) != APEX_OK) return 0;
    return need_bytes(B, Hkv, block_table_stride);
}

extern "C" int apex_kv4_evict(void* kv_cache, const int32_t* block_table, int64_t block_table_stride,
                              const int32_t* context_lens, float* weights, int32_t* positions, int B, int Hkv, int d,
                              int block_size, int64_t num_blocks, int keep, int sinks, int recent, void* workspace,
                              size_t workspace_bytes, void* stream)
{
    apex::clear_error();
    int rc = check_batch(B, Hkv, Hkv, d, block_size, num_blocks, block_table_stride);
    if (rc != APEX_OK) return rc;
    if (keep <= 0 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > keep)
        return fail(APEX_ERR_INVALID_ARG, "keep = %d, sinks = %d, recent = %d: keep must be positive, sinks + recent at most keep",
                    keep, sinks, recent);
    if ((int64_t)B * Hkv >= 1 << 22) return fail(APEX_ERR_UNSUPPORTED, "B * Hkv = %lld reaches 2^22", (long long)B * Hkv);
    if (B == 0) return APEX_OK;
    if (!kv_cache || !block_table || !context_lens || !weights || !positions)
        return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!aligned(kv_cache, 16) || !aligned(weights, 16))
        return fail(APEX_ERR_INVALID_ARG, "kv_cache and weights must be 16-byte aligned");
    if (!aligned(positions, 4) || !aligned(block_table, 4) || !aligned(context_lens, 4))
        return fail(APEX_ERR_INVALID_ARG, "positions, block_table and context_lens must be 4-byte aligned");
    const size_t sb = slot_bytes(Hkv, num_blocks);
    const Extent in[] = {{"block_table", block_table, (size_t)B * block_table_stride * 4},
                         {"context_lens", context_lens, (size_t)B * 4},
                         {"kv_cache", kv_cache, cache_bytes(Hkv, num_blocks)},
                         {"weights", weights, sb},
                         {"positions", positions, sb},
                         {"workspace", workspace, workspace_bytes}};
    for (int i = 2; i < 6; ++i)
        if ((rc = check_disjoint(in[i], in, i)) != APEX_OK) return rc;
    const size_t need = need_bytes(B, Hkv, block_table_stride);
    rc = workspace ? check_workspace(workspace, workspace_bytes, need)
                   : library_buffer(kMasks, need, (hipStream_t)stream, &workspace);
    if (rc != APEX_OK) return rc;
    if (block_table_stride * kBlockSize <= keep) return APEX_OK;   // no request can be longer
    EvictParams p;
    p.cache = (char*)kv_cache;
    p.bt = block_table;
    p.lens = context_lens;
    p.weights = weights;
    p.positions = positions;
    p.counts = (int32_t*)workspace;
    p.masks = (uint64_t*)((char*)workspace + count_bytes(B, Hkv));
    p.num_blocks = num_blocks;
    p.Hkv = Hkv;
    p.stride = (int)block_table_stride;
    p.words = (int)mask_words(block_table_stride);
    p.keep = keep;
    p.sinks = sinks;
    p.recent = recent;
    const unsigned pairs = (unsigned)(B * Hkv);
    select_kernel<<<pairs, kSelectThreads, 0, (hipStream_t)stream>>>(p);
    if ((rc = launched("kv4 evict")) != APEX_OK) return rc;
    // at most min(keep, longest - keep) tokens of a pair move
    const int64_t longest = block_table_stride * kBlockSize, most = longest - keep < keep ? longest - keep : keep;
    int64_t groups = (most + kMoves - 1) / kMoves;
    if (groups * pairs > 4096) groups = 4096 / pairs > 0 ? 4096 / pairs : 1;
    move_kernel<<<dim3(pairs, (unsigned)groups), kMoveThreads, 0, (hipStream_t)stream>>>(p);
    return launched("kv4 evict");
}
