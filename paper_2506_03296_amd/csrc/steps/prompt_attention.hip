// prompt_attention.hip -- causal attention of packed prompts (include/apex_steps.h).
#include "attend_tile.h"
#include "steps_host.h"

namespace steps {

namespace {

constexpr int kKeys = 64;                        // keys of a tile
constexpr int kTileBytes = kKeys * kRowBytes;    // of K or of V
constexpr int kSortedRequests = 64;              // requests a wave sorts, one a lane

struct PromptArgs {
    const char *q, *k, *v;
    const int32_t* offsets;
    char* out;
    float* lse;
    int64_t q_stride, kv_stride;   // bytes between tokens
    int B, T, Hq, Hkv, G;
    float c;                       // |scale| log2 e
    bool negate;
};

// One request's rows in the packed arrays, cut to [0, T].
__device__ inline void request_rows(const int32_t* offsets, int T, int b, int* first, int* n)
{
    const int lo = min(max(offsets[b], 0), T), hi = min(max(offsets[b + 1], lo), T);
    *first = lo;
    *n = hi - lo;
}

// The request and the tile of rows that work group `slot` takes; false: none.
// A tile's cost goes with its depth (its keys reach back to the request's first),
// so that the deepest are given out first, over all requests.  Up to 64 requests
// a lane counts one's tiles, and the depth of the slot-th tile in falling order
// is found by halving.  With more, requests have fixed ranges of slots, as many as
// their rows can fill (which needs no sums over other requests), deepest first;
// slots that are left over return.
template <int kRows>
__device__ bool find_tile(const PromptArgs& a, unsigned slot, unsigned slots, int* request, int* tile)
{
    const int lane = threadIdx.x & 63;
    if (a.B <= kSortedRequests) {
        int first, n = 0;
        if (lane < a.B) request_rows(a.offsets, a.T, lane, &first, &n);
        const int tiles = (int)(((int64_t)n * a.G + kRows - 1) / kRows);
        const int most = wave_max(tiles);
        int lo = 0, hi = most;    // more than slot tiles lie at depth lo or deeper; not so at hi
        if ((unsigned)wave_sum(tiles) <= slot) return false;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if ((unsigned)wave_sum(max(tiles - mid, 0)) > slot) lo = mid;
            else hi = mid;
        }
        unsigned at = slot - (unsigned)wave_sum(max(tiles - hi, 0));
        uint64_t have = __ballot(tiles > lo);
        while (at--) have &= have - 1;
        *request = __builtin_ctzll(have);
        *tile = lo;
        return true;
    }
    // request b's slots begin at offsets[b] G / kRows + b
    slot = slots - 1 - slot;
    int lo = 0, hi = a.B;        // begin(lo) <= slot < begin(hi)
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64;
        const int b = lo + lane * step;
        bool under = false;
        if (b < hi) under = (unsigned)((int64_t)min(max(a.offsets[b], 0), a.T) * a.G / kRows) + b <= slot;
        const int n = __builtin_popcountll(__ballot(under));
        if (n > 0) lo += (n - 1) * step;
        hi = min(hi, lo + step);
    }
    int first, n;
    request_rows(a.offsets, a.T, lo, &first, &n);
    *request = lo;
    *tile = (int)(slot - ((unsigned)((int64_t)first * a.G / kRows) + lo));
    return *tile < (int)(((int64_t)n * a.G + kRows - 1) / kRows);
}

template <int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void prompt_kernel(PromptArgs a, unsigned slots)
{
    constexpr int kThreads = 64 * kWaves, kRows = kWaveRows * kWaves;
    constexpr int kLoads = kTileBytes / (kThreads * 16);     // of K, and of V, that bring a tile
    __shared__ __attribute__((aligned(16))) char lds[2 * 2 * kTileBytes];

    const unsigned slot = blockIdx.x / (unsigned)a.Hkv, head = blockIdx.x - slot * (unsigned)a.Hkv;
    int request, tile;
    if (!find_tile<kRows>(a, slot, slots, &request, &tile)) return;
    request = __builtin_amdgcn_readfirstlane(request);
    tile = __builtin_amdgcn_readfirstlane(tile);
    int first, n;
    request_rows(a.offsets, a.T, request, &first, &n);
    const Group group = {a.G};
    const unsigned lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned rows = (unsigned)n * (unsigned)a.G;

    // this lane's row, and the positions of the wave's and the work group's rows
    const unsigned row = (unsigned)tile * kRows + wave * kWaveRows + (lane & 31);
    unsigned pos, in_group;
    group.split(min(row, rows - 1), &pos, &in_group);
    const int wave_lo = (int)(min((unsigned)tile * kRows + wave * kWaveRows, rows - 1) / (unsigned)a.G);
    const int wave_hi = (int)(min((unsigned)tile * kRows + wave * kWaveRows + 31, rows - 1) / (unsigned)a.G);
    const int all_hi = (int)(min((unsigned)tile * kRows + kRows - 1, rows - 1) / (unsigned)a.G);
    const bool live = row < rows, wave_live = (unsigned)tile * kRows + wave * kWaveRows < rows;
    const unsigned qhead = head * (unsigned)a.G + in_group;
    const int tiles = all_hi / kKeys + 1, own_tiles = wave_live ? wave_hi / kKeys + 1 : 0;

    Rows<2> r;
    r.start(0, live ? a.q + (int64_t)(first + (int)pos) * a.q_stride + qhead * kRowBytes : nullptr);
    if (a.negate) r.negate();
    r.clear();

    // A tile's rows: load j of a wave brings four keys, in LDS one behind the other,
    // and lane i the piece that belongs at i % 16 of key i / 16.  There are two
    // buffers: a tile is on its way while the one before it is worked on.
    const unsigned key0 = wave * 4 + (lane >> 4);
    constexpr unsigned kStep = 4 * kWaves;
    const int64_t request0 = (int64_t)first * a.kv_stride + head * kRowBytes;
    lds_char* const shared = (lds_char*)lds;
    const auto load = [&](int t) {
        const unsigned to = lds_address(shared) + (t & 1) * 2 * kTileBytes + wave * 1024;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const unsigned key = key0 + j * kStep;
            const int64_t at = request0 + (int64_t)(t * kKeys + (int)key) * a.kv_stride;
            const char* k = a.k + at + k_piece(key, lane & 15) * 16;
            const char* v = a.v + at + v_piece(key, lane & 15) * 16;
            if (t * kKeys + (int)key >= n) k = v = (const char*)kZeros;     // behind the request
            load_to_lds(k, to + j * kStep * kRowBytes);
            load_to_lds(v, to + kTileBytes + j * kStep * kRowBytes);
        }
    };
    load(0);
    int t = 0;
    for (; t < own_tiles; ++t) {
        arrived<0>();
        barrier();
        if (t + 1 < tiles) load(t + 1);
        const lds_char* kt = shared + (t & 1) * 2 * kTileBytes;
        f32x16 s[1][2];
        f16x8 p[1][4];
        r.scores(kt, s);
        if ((t + 1) * kKeys > wave_lo + 1) {
            const int seen = (int)pos - t * kKeys + 1;      // keys of the tile up to the row's own
            r.mask(s[0], seen >= 64 ? ~0ull : seen <= 0 ? 0ull : (1ull << seen) - 1);
        }
        r.weights(0, s[0], a.c, p[0]);
        r.add(kt + kTileBytes, p);
    }
    for (; t < tiles; ++t) {     // tiles that only other waves see
        arrived<0>();
        barrier();
        if (t + 1 < tiles) load(t + 1);
    }
    if (__builtin_expect(r.spoiled(), 0)) {
        r.clear();
#pragma nounroll
        for (int key = 0; key <= wave_hi; ++key) {
            const int64_t at = request0 + (int64_t)key * a.kv_stride;
            r.take_key(0, a.k + at, a.v + at, a.c, key <= (int)pos);
        }
    }

    const float sum = sum_of_halves(r.sum[0]);
    if (!live) return;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int64_t at = (int64_t)(first + (int)pos) * a.Hq + qhead;
    const unsigned half = lane >> 5;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x = {r.o[0][t][4 * i] * inv, r.o[0][t][4 * i + 1] * inv, r.o[0][t][4 * i + 2] * inv, r.o[0][t][4 * i + 3] * inv};
            *(f16x4*)(a.out + at * kRowBytes + t * 64 + i * 16 + half * 8) = __builtin_convertvector(x, f16x4);
        }
    if (a.lse && half == 0) a.lse[at] = (r.top[0] - kBias + __builtin_amdgcn_logf(sum)) * kLn2;
}

}  // namespace

}  // namespace steps

extern "C" int apex_steps_prompt_attention(const void* q, int64_t q_token_stride, const void* k, const void* v,
                                           int64_t kv_token_stride, const int32_t* token_offsets, void* out,
                                           float* lse_out, int B, int T, int Hq, int Hkv, int d, float scale,
                                           void* stream)
{
    using namespace steps;
    apex::clear_error();
    int rc = check_attention(B, T, Hq, Hkv, d, scale, &q_token_stride, &kv_token_stride);
    if (rc != APEX_OK) return rc;
    if (B == 0 || T == 0) return APEX_OK;
    if (!q || !k || !v || !token_offsets || !out) return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16))
        return fail(APEX_ERR_INVALID_ARG, "q, k, v and out must be 16-byte aligned");
    if (!aligned(token_offsets, 4) || !aligned(lse_out, 4))
        return fail(APEX_ERR_INVALID_ARG, "token_offsets and lse_out must be 4-byte aligned");
    const Extent inputs[] = {{"q", q, rows_bytes(T, q_token_stride, Hq, 2)},
                             {"k", k, rows_bytes(T, kv_token_stride, Hkv, 2)},
                             {"v", v, rows_bytes(T, kv_token_stride, Hkv, 2)},
                             {"token_offsets", token_offsets, ((size_t)B + 1) * 4},
                             {"lse_out", lse_out, (size_t)T * Hq * 4}};
    rc = check_disjoint({"out", out, (size_t)T * Hq * kRowBytes}, inputs, 5);
    if (rc == APEX_OK) rc = check_disjoint({"lse_out", lse_out, (size_t)T * Hq * 4}, inputs, 4);
    if (rc != APEX_OK) return rc;

    PromptArgs a;
    a.q = (const char*)q;
    a.k = (const char*)k;
    a.v = (const char*)v;
    a.offsets = token_offsets;
    a.out = (char*)out;
    a.lse = lse_out;
    a.q_stride = q_token_stride * 2;
    a.kv_stride = kv_token_stride * 2;
    a.B = B;
    a.T = T;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = Hq / Hkv;
    a.c = (scale < 0 ? -scale : scale) * kLog2e;
    a.negate = scale < 0;
    constexpr int kWaves = 8, kRows = kWaves * kWaveRows;
    const unsigned slots = (unsigned)((int64_t)T * a.G / kRows) + (unsigned)B;
    prompt_kernel<kWaves><<<slots * (unsigned)Hkv, 64 * kWaves, 0, (hipStream_t)stream>>>(a, slots);
    return launched("prompt_attention");
}
