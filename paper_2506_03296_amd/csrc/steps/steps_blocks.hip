// steps_blocks.hip -- cache blocks of a batch's new tokens, and blocks given back
// (include/apex_steps.h).
//
// Both are sums over the requests in their order, with a few words moved per
// block and per token: bound by the launch and by round trips, not by bandwidth.
// extend takes 4.4 us for a decode step's 32 tokens and 7.8 for the 51 720 of 24
// prompts; release 6.4 us for 128 requests that drop a few tokens each and 20.4 for
// the 25 948 blocks of 32 requests.
#include <hip/hip_runtime.h>

#include "attend_tile.h"
#include "steps_host.h"

namespace steps {

namespace {

// Inclusive sums over a work group of kThreads, in 64 bits; `total` gets the sum
// of all.  `part` is LDS of a word per wave.
template <int kThreads>
__device__ inline int64_t group_scan(int64_t x, int64_t* part, int64_t* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int64_t y = __shfl_up(x, m);
        if (lane >= m) x += y;
    }
    __syncthreads();
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        before += w < wave ? part[w] : 0;
        all += part[w];
    }
    *total = all;
    return x + before;
}

// The last of n ascending sums that is not above x, counted from 0; n if all are
// not above: the request whose range [sum before it, its sum) holds x.
__device__ inline int find(const int64_t* upto, int n, int64_t x)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (upto[mid] <= x) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

struct ExtendArgs {
    const int32_t *lens, *news;
    int32_t* table;
    const int32_t* free_blocks;
    int32_t *state, *offsets, *totals;
    int64_t* slots;
    int32_t* positions;
    int64_t table_stride, num_blocks;
    int B, T, block_size;
};

constexpr int kExtendThreads = 256;
// A group's share, of a grid of at most kExtendGroups: four slots a thread.  The same
// sums in every group cost less than tokens that wait: 51 720 tokens, 256, 1024 and
// 4096 a group: 15.9, 16.0 and 17.7 us a call.
constexpr int kTokensPerGroup = 1024;
constexpr int kExtendGroups = 256;

// Every work group makes the sums over all requests and writes a share of the
// tokens' slots and of the table's new entries; nothing that it reads is written
// by another, but for the height of the stack, which the last one to end lowers.
__global__ __launch_bounds__(kExtendThreads) void extend_kernel(ExtendArgs a)
{
    constexpr int kThreads = kExtendThreads;
    __shared__ int64_t part[kThreads / 64];
    __shared__ int64_t tokens_upto[kThreads], blocks_upto[kThreads];
    __shared__ int32_t lens[kThreads];
    __shared__ uint8_t granted[kThreads];
    const int64_t height = min((int64_t)max(a.state[0], 0), a.num_blocks);
    const unsigned bs = (unsigned)a.block_size;
    const int64_t share = ((int64_t)a.T + gridDim.x - 1) / gridDim.x;
    const int64_t t0 = share * blockIdx.x, t1 = min(t0 + share, (int64_t)a.T);
    int64_t tokens = 0, blocks = 0, taken = 0;      // of the requests before these
    if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[0] = 0;
    for (int base = 0; base < a.B; base += kThreads) {
        const int b = base + (int)threadIdx.x, n_here = min(kThreads, a.B - base);
        int L = 0, n = 0;
        if (b < a.B) {
            L = max(a.lens[b], 0);
            n = max(a.news[b], 0);
        }
        int64_t all_tokens, all_blocks;
        const int64_t upto = tokens + group_scan<kThreads>(n, part, &all_tokens);
        const int64_t end = (int64_t)L + n;
        const int64_t have = ((unsigned)L + bs - 1) / bs, want = (end + bs - 1) / bs;
        const bool fits = b < a.B && upto <= a.T && end <= INT_MAX && want <= a.table_stride;
        const int64_t need = fits ? want - have : 0;
        const int64_t need_upto = blocks + group_scan<kThreads>(need, part, &all_blocks);
        const bool ok = fits && (need == 0 || need_upto <= height);
        int64_t taken_here;
        group_scan<kThreads>(ok ? need : 0, part, &taken_here);
        tokens_upto[threadIdx.x] = min(upto, (int64_t)a.T);
        blocks_upto[threadIdx.x] = need_upto;
        lens[threadIdx.x] = L;
        granted[threadIdx.x] = ok;
        __syncthreads();
        if (blockIdx.x == 0 && b < a.B) {
            a.offsets[b + 1] = (int32_t)min(upto, (int64_t)a.T);
            a.totals[b] = ok ? (int32_t)end : L;
        }
        // new entries of the table
        for (int64_t i = blocks + blockIdx.x * kThreads + threadIdx.x; i < blocks + taken_here; i += gridDim.x * kThreads) {
            const int r = find(blocks_upto, n_here, i);
            const int64_t first = r ? blocks_upto[r - 1] : blocks;
            const int64_t entry = ((unsigned)lens[r] + bs - 1) / bs + (i - first);
            a.table[(base + r) * a.table_stride + entry] = a.free_blocks[height - 1 - i];
        }
        // slots and positions
        const int64_t from = max(t0, min(tokens, (int64_t)a.T)), to = min(t1, tokens + all_tokens);
        for (int64_t t = from + threadIdx.x; t < to; t += kThreads) {
            const int r = find(tokens_upto, n_here, t);
            int64_t slot = -1;
            int32_t pos = 0;
            if (r < n_here && granted[r]) {
                pos = lens[r] + (int32_t)(t - (r ? tokens_upto[r - 1] : min(tokens, (int64_t)a.T)));
                const unsigned entry = (unsigned)pos / bs, held = ((unsigned)lens[r] + bs - 1) / bs;
                const int64_t first = r ? blocks_upto[r - 1] : blocks;
                const int id = entry < held ? a.table[(base + r) * a.table_stride + entry]
                                            : a.free_blocks[height - 1 - (first + entry - held)];
                if (id >= 0 && id < a.num_blocks) slot = (int64_t)id * bs + ((unsigned)pos - entry * bs);
            }
            a.slots[t] = slot;
            a.positions[t] = pos;
        }
        tokens += all_tokens;
        blocks += all_blocks;
        taken += taken_here;
        __syncthreads();
    }
    for (int64_t t = max(t0, min(tokens, (int64_t)a.T)) + threadIdx.x; t < t1; t += kThreads) {
        a.slots[t] = -1;
        a.positions[t] = 0;
    }
    if (threadIdx.x == 0) {
        // every group has its height before it counts itself here
        const bool last = gridDim.x == 1 || atomicAdd(&a.state[1], 1) == (int)gridDim.x - 1;
        if (last) {
            a.state[0] = (int32_t)(height - taken);
            if (gridDim.x > 1) a.state[1] = 0;
        }
    }
}

struct ReleaseArgs {
    const int32_t *lens, *keeps;
    int32_t *table, *free_blocks, *state;
    int64_t table_stride, num_blocks;
    int B, block_size;
};

constexpr int kReleaseThreads = 1024;
constexpr int kEntries = 8;      // of a thread at a time (16 and 24: 25.9 and 34.0 us a call for 24 on 25 948 blocks)

// One work group: where an id goes depends on how many of those before it count.
// It takes 8192 entries of the rows at a time, neighbouring lanes neighbouring
// entries, and ranks them by the waves' votes.  25 948 blocks: 20 us, 43 with every
// lane searching its row by halves.
__global__ __launch_bounds__(kReleaseThreads) void release_kernel(ReleaseArgs a)
{
    constexpr int kThreads = kReleaseThreads, kWaves = kThreads / 64, kVotes = kEntries * kWaves;
    static_assert(kVotes == 128, "two votes a lane");
    __shared__ int64_t part[kWaves];
    __shared__ int64_t upto[kThreads];
    __shared__ int32_t firsts[kThreads];
    __shared__ int votes[2][kVotes];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
    int64_t height = min((int64_t)max(a.state[0], 0), a.num_blocks);
    const unsigned bs = (unsigned)a.block_size;
    unsigned turn = 0;
    for (int base = 0; base < a.B; base += kThreads) {
        const int b = base + (int)threadIdx.x;
        int64_t first = 0, n = 0;
        if (b < a.B) {
            first = ((unsigned)max(a.keeps[b], 0) + bs - 1) / bs;
            const int64_t have = min((int64_t)(((unsigned)max(a.lens[b], 0) + bs - 1) / bs), a.table_stride);
            n = max(have - first, (int64_t)0);
        }
        int64_t all;
        upto[threadIdx.x] = group_scan<kThreads>(n, part, &all);
        firsts[threadIdx.x] = (int32_t)first;
        __syncthreads();
        const int64_t coarse = upto[16 * lane + 15];
        for (int64_t i0 = 0; i0 < all; i0 += kThreads * kEntries, turn ^= 1) {
            int32_t* at[kEntries];
            int32_t id[kEntries];
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                // the row of the wave's first entry, among the work group's 1024 in two
                // steps, and from there on the lane's own
                const int64_t i_wave = i0 + e * kThreads + wave * 64, i = i_wave + lane;
                at[e] = nullptr;
                id[e] = -1;
                if (i_wave >= all) continue;
                const int sixteen = 16 * __builtin_popcountll(__ballot(coarse <= i_wave));
                int r = sixteen + __builtin_popcountll(__ballot(lane < 16 && upto[min(sixteen + lane, kThreads - 1)] <= i_wave));
                if (i < all) {
                    for (int step = 0; step < 4 && upto[r] <= i; ++step) ++r;
                    if (upto[r] <= i) r += find(upto + r, kThreads - r, i);      // many rows with little or nothing to give
                    at[e] = a.table + (base + r) * a.table_stride + firsts[r] + (i - (r ? upto[r - 1] : 0));
                    id[e] = *at[e];
                }
            }
            uint64_t counts[kEntries];
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                counts[e] = __ballot(id[e] >= 0 && id[e] < a.num_blocks);
                if (lane == 0) votes[turn][e * kWaves + wave] = __builtin_popcountll(counts[e]);
            }
            __syncthreads();
            // votes before each of this wave's, two of all to a lane
            const int v0 = votes[turn][2 * lane], v1 = votes[turn][2 * lane + 1];
            const int sum = wave_scan(v0 + v1), before = sum - v0 - v1;
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                const int vote = e * kWaves + wave;
                const int ahead = __builtin_amdgcn_readlane(before, vote / 2) + (vote & 1 ? __builtin_amdgcn_readlane(v0, vote / 2) : 0);
                const int64_t to = height + ahead + __builtin_popcountll(counts[e] & ((1ull << lane) - 1));
                if (at[e]) *at[e] = -1;
                if ((counts[e] >> lane & 1) && to < a.num_blocks) a.free_blocks[to] = id[e];
            }
            height = min(height + __builtin_amdgcn_readlane(sum, 63), a.num_blocks);
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) a.state[0] = (int32_t)height;
}

int check_blocks(int B, int block_size, int64_t num_blocks, int64_t block_table_stride)
{
    if (B < 0) return fail(APEX_ERR_INVALID_ARG, "B = %d is negative", B);
    if (block_size <= 0) return fail(APEX_ERR_INVALID_ARG, "block_size = %d must be positive", block_size);
    if (num_blocks < 0 || block_table_stride < 0)
        return fail(APEX_ERR_INVALID_ARG, "num_blocks and block_table_stride must not be negative");
    if (B > (1 << 22)) return fail(APEX_ERR_UNSUPPORTED, "B exceeds 2^22");
    if (num_blocks > INT_MAX) return fail(APEX_ERR_UNSUPPORTED, "num_blocks exceeds 2^31 - 1");
    if (block_table_stride > INT_MAX) return fail(APEX_ERR_UNSUPPORTED, "block_table_stride exceeds 2^31 - 1");
    return APEX_OK;
}

}  // namespace

}  // namespace steps

extern "C" {

int apex_steps_extend(const int32_t* context_lens, const int32_t* new_lens, int32_t* block_table,
                      int64_t block_table_stride, const int32_t* free_blocks, int32_t* free_state,
                      int32_t* token_offsets, int32_t* total_lens, int64_t* slot_mapping, int32_t* token_positions,
                      int B, int T, int block_size, int64_t num_blocks, void* stream)
{
    using namespace steps;
    apex::clear_error();
    int rc = check_blocks(B, block_size, num_blocks, block_table_stride);
    if (rc != APEX_OK) return rc;
    if (T < 0) return fail(APEX_ERR_INVALID_ARG, "T = %d is negative", T);
    if (!free_state || !token_offsets || (B > 0 && (!context_lens || !new_lens || !total_lens)) ||
        (B > 0 && block_table_stride > 0 && !block_table) || (num_blocks > 0 && !free_blocks) ||
        (T > 0 && (!slot_mapping || !token_positions)))
        return fail(APEX_ERR_INVALID_ARG, "a pointer is NULL");
    const void* words[] = {context_lens, new_lens, block_table, free_blocks, free_state, token_offsets, total_lens, token_positions};
    for (const void* p : words)
        if (!aligned(p, 4)) return fail(APEX_ERR_INVALID_ARG, "an array is not aligned to its element");
    if (!aligned(slot_mapping, 8)) return fail(APEX_ERR_INVALID_ARG, "slot_mapping must be 8-byte aligned");
    const Extent all[] = {{"context_lens", context_lens, (size_t)B * 4},
                          {"new_lens", new_lens, (size_t)B * 4},
                          {"free_blocks", free_blocks, (size_t)num_blocks * 4},
                          {"block_table", block_table, (size_t)B * block_table_stride * 4},
                          {"free_state", free_state, 8},
                          {"token_offsets", token_offsets, ((size_t)B + 1) * 4},
                          {"total_lens", total_lens, (size_t)B * 4},
                          {"slot_mapping", slot_mapping, (size_t)T * 8},
                          {"token_positions", token_positions, (size_t)T * 4}};
    for (int i = 3; i < 9 && rc == APEX_OK; ++i) rc = check_disjoint(all[i], all, i);
    if (rc != APEX_OK) return rc;

    const ExtendArgs a = {context_lens, new_lens, block_table, free_blocks, free_state, token_offsets, total_lens,
                          slot_mapping, token_positions, block_table_stride, num_blocks, B, T, block_size};
    int groups = (int)(((int64_t)T + kTokensPerGroup - 1) / kTokensPerGroup);
    groups = groups < 1 ? 1 : groups > kExtendGroups ? kExtendGroups : groups;
    extend_kernel<<<groups, kExtendThreads, 0, (hipStream_t)stream>>>(a);
    return launched("extend");
}

int apex_steps_release(const int32_t* context_lens, const int32_t* keep_lens, int32_t* block_table,
                       int64_t block_table_stride, int32_t* free_blocks, int32_t* free_state, int B, int block_size,
                       int64_t num_blocks, void* stream)
{
    using namespace steps;
    apex::clear_error();
    int rc = check_blocks(B, block_size, num_blocks, block_table_stride);
    if (rc != APEX_OK) return rc;
    if (B == 0 || block_table_stride == 0 || num_blocks == 0) return APEX_OK;
    if (!context_lens || !keep_lens || !block_table || !free_blocks || !free_state)
        return fail(APEX_ERR_INVALID_ARG, "a pointer is NULL");
    const void* words[] = {context_lens, keep_lens, block_table, free_blocks, free_state};
    for (const void* p : words)
        if (!aligned(p, 4)) return fail(APEX_ERR_INVALID_ARG, "an array is not aligned to its element");
    const Extent all[] = {{"context_lens", context_lens, (size_t)B * 4},
                          {"keep_lens", keep_lens, (size_t)B * 4},
                          {"block_table", block_table, (size_t)B * block_table_stride * 4},
                          {"free_blocks", free_blocks, (size_t)num_blocks * 4},
                          {"free_state", free_state, 8}};
    for (int i = 2; i < 5 && rc == APEX_OK; ++i) rc = check_disjoint(all[i], all, i);
    if (rc != APEX_OK) return rc;

    const ReleaseArgs a = {context_lens, keep_lens, block_table, free_blocks, free_state, block_table_stride,
                           num_blocks, B, block_size};
    release_kernel<<<1, kReleaseThreads, 0, (hipStream_t)stream>>>(a);
    return launched("release");
}

}  // extern "C"
