// prompt_attention.hip -- causal attention of packed prompts (include/apex_steps.h).
//
// An item is one kv-head of one request and a tile of its rows, position by position
// the G q-heads of each: a work group walks over the keys up to its last row's in
// tiles of 64, in the one pass of attend_tile.h, and masks the tiles that its waves'
// diagonals cross (looking at their values first, see finite: 0.3 % of a long prompt,
// 2-3 % of batches of short ones).  A wave leaves out the tiles behind its own last row, and of its
// last tile the weights of a second half that it does not see (batches 0-2 % faster;
// leaving out its scores too needs a second copy of the loop, which spills).
//
// The matrix cores bound it from some 500 tokens on: 32768 tokens of 32 over 8 heads
// are 8.8 TFLOP and take 8.2 to 9.0 ms, 975-1070 TFLOP/s of the 1200 of a large
// library product; what holds a wave back is said in attend_tile.h.  One prompt has
// few items and its longest bounds it: 512 tokens 15.1 us, 1024 24.7, 2048 51, 4096 143,
// where the operations take 1.8, 7.2, 29 and 115 (512: the bytes 2.1).  Many short prompts are bound by
// their bytes and by items that fill few of their rows: 64, 128 and 512 prompts of
// 16-512 tokens take 116, 230 and 860 us, the bytes 66, 133 and 528.
//
// The tile: 256 rows read the 32 KB of 64 keys once from L2 (the 32768 tokens' reads
// are 1.41 GB, 3.5 times q, k and v).  Work groups of four waves, two a compute unit,
// and three buffers instead of two were no faster.
#include "attend_tile.h"
#include "steps_host.h"

namespace steps {

namespace {

constexpr int kWaves = 8;
constexpr int kPartKeys = 64;                    // keys of a tile that a wave takes
constexpr int kSortedRequests = 64;              // requests a wave sorts, one a lane

struct PromptArgs {
    const char *q, *k, *v;
    const int32_t* offsets;
    char* out;
    float* lse;
    int64_t q_stride, kv_stride;   // bytes between tokens
    int B, T, Hq;
    Divisor Hkv, G;
    QScale scale;
};

// One request's rows in the packed arrays, cut to [0, T].
__device__ inline void request_rows(const int32_t* offsets, int T, int b, int* first, int* n)
{
    const int lo = min(max(offsets[b], 0), T), hi = min(max(offsets[b + 1], lo), T);
    *first = lo;
    *n = hi - lo;
}

// A tile of a request's rows, for one kv-head.
struct Work {
    int first, n, tile;
    unsigned head;
};

// Which tile is the slot-th.  A tile's cost goes with its depth (its keys reach
// back to the request's first), so that the deepest are given out first, over all
// requests.  Up to 64 requests a lane counts one's tiles, and the depth of the
// slot-th tile in falling order is found by halving.  With more, requests have
// fixed ranges of slots, as many as their rows can fill (which needs no sums over
// other requests), deepest first; slots that are left over hold no tile.
template <int kRows>
struct Tiles {
    int first, n, count;      // of request `lane`, up to 64 requests
    __device__ void start(const PromptArgs& a)
    {
        const int lane = threadIdx.x & 63;
        first = n = 0;
        if (a.B <= kSortedRequests && lane < a.B) request_rows(a.offsets, a.T, lane, &first, &n);
        count = (int)(((int64_t)n * a.G.d + kRows - 1) / kRows);
    }

    __device__ bool find(const PromptArgs& a, unsigned slot, unsigned slots, Work& w) const
    {
        const int lane = threadIdx.x & 63;
        if (a.B <= kSortedRequests) {
            if ((unsigned)wave_sum(count) <= slot) return false;
            int lo = 0, hi = wave_max(count);    // more than slot tiles lie at depth lo or deeper; not so at hi
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if ((unsigned)wave_sum(max(count - mid, 0)) > slot) lo = mid;
                else hi = mid;
            }
            unsigned at = slot - (unsigned)wave_sum(max(count - hi, 0));
            uint64_t have = __ballot(count > lo);
            while (at--) have &= have - 1;
            const int b = __builtin_ctzll(have);
            w.first = __builtin_amdgcn_readlane(first, b);
            w.n = __builtin_amdgcn_readlane(n, b);
            w.tile = lo;
            return true;
        }
        // request b's slots begin at offsets[b] G / kRows + b
        slot = slots - 1 - slot;
        int lo = 0, hi = a.B;        // begin(lo) <= slot < begin(hi)
        while (hi - lo > 1) {
            const int step = (hi - lo + 63) / 64;
            const int b = lo + lane * step;
            bool under = false;
            if (b < hi) under = (unsigned)((int64_t)min(max(a.offsets[b], 0), a.T) * a.G.d / kRows) + b <= slot;
            const int m = __builtin_popcountll(__ballot(under));
            if (m > 0) lo += (m - 1) * step;
            hi = min(hi, lo + step);
        }
        lo = uniform(lo);
        request_rows(a.offsets, a.T, lo, &w.first, &w.n);
        w.tile = uniform((int)(slot - ((unsigned)((int64_t)w.first * a.G.d / kRows) + lo)));
        return w.tile >= 0 && w.tile < (int)(((int64_t)w.n * a.G.d + kRows - 1) / kRows);
    }
};

// The items, slots x kv-heads in falling order of their cost, go to work groups in
// two ways.  A work group a compute unit takes `rounds` of them, an even number of
// items that lie in the order w, 2 W - 1 - w, 2 W + w, ...: alike sums, and an item's
// first tile and rows are asked for before the item before it ends.  The cheapest
// items that remain have a work group each, which the hardware starts where the
// others end first.
//
// Eight waves: with one part they hold 32 rows each.  With two, four of them hold 128
// rows, and the other four the same rows for every second 64 keys; work groups are
// then one an item.
template <int kParts>
__global__ __launch_bounds__(64 * kWaves, 2) void prompt_kernel(PromptArgs a, unsigned slots, unsigned groups, unsigned rounds)
{
    constexpr int kRowWaves = kWaves / kParts, kRows = kWaveRows * kRowWaves;
    constexpr int kKeys = kParts * kPartKeys, kTileBytes = kKeys * kRowBytes;     // of a tile; of its K or V
    constexpr int kLoads = kTileBytes / (64 * kWaves * 16);     // of K, and of V, that bring a tile
    __shared__ __attribute__((aligned(16))) char lds[2 * 2 * kTileBytes + kRows * kRowBytes];

    const unsigned lane = threadIdx.x & 63, wave = (unsigned)uniform((int)(threadIdx.x >> 6));
    const unsigned row_wave = wave % kRowWaves, part = kParts == 1 ? 0 : wave / kRowWaves;
    Tiles<kRows> all;
    all.start(a);
    unsigned round = 0;
    const auto next = [&](Work& w) {                         // false: there are no more
        for (;; ++round) {
            if (round >= (blockIdx.x < groups ? rounds : 1)) return false;
            const unsigned id = blockIdx.x < groups ? round * groups + (round & 1 ? groups - 1 - blockIdx.x : blockIdx.x)
                                                    : rounds * groups + (blockIdx.x - groups);
            const unsigned slot = divide(id, a.Hkv);
            w.head = id - slot * a.Hkv.d;
            if (slot < slots && all.find(a, slot, slots, w)) {
                ++round;
                return true;
            }
        }
    };

    // A tile's rows: load j of a wave brings four keys, in LDS one behind the other,
    // and lane i the piece that belongs at i % 16 of key i / 16.  There are two
    // buffers: a tile is on its way while the one before it is worked on.
    lds_char* const shared = (lds_char*)lds;
    // Where a tile lies whole inside its request, a lane's offsets from its first row
    // are the same for all tiles (if a tile's rows span less than 2^31 bytes).
    const bool near = a.kv_stride < (int64_t)1 << 24;
    unsigned k_offset[kLoads], v_offset[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const unsigned key = wave * 4 + (lane >> 4) + j * 4 * kWaves, row = key * (unsigned)a.kv_stride;
        k_offset[j] = row + k_piece(key, lane & 15) * 16;
        v_offset[j] = row + v_piece(key, lane & 15) * 16;
    }
    const auto load = [&](const Work& w, int t, unsigned buffer) {
        const unsigned to = lds_address(shared) + buffer * 2 * kTileBytes + wave * 1024;
        const int64_t tile0 = (int64_t)(w.first + t * kKeys) * a.kv_stride + w.head * kRowBytes;
        if (near && (t + 1) * kKeys <= w.n) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                load_to_lds(a.k + tile0, k_offset[j], to + j * 4 * kWaves * kRowBytes);
                load_to_lds(a.v + tile0, v_offset[j], to + kTileBytes + j * 4 * kWaves * kRowBytes);
            }
            return;
        }
        const unsigned lane = lane_again();
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const unsigned key = wave * 4 + (lane >> 4) + j * 4 * kWaves;
            const int64_t at = tile0 + (int64_t)key * a.kv_stride;
            const char* k = a.k + at + k_piece(key, lane & 15) * 16;
            const char* v = a.v + at + v_piece(key, lane & 15) * 16;
            if (t * kKeys + (int)key >= w.n) k = v = (const char*)kZeros;     // behind the request
            load_to_lds(k, to + j * 4 * kWaves * kRowBytes);
            load_to_lds(v, to + kTileBytes + j * 4 * kWaves * kRowBytes);
        }
    };
    Rows<2, false> r;
    const auto row0 = [&](const Work& w) { return (unsigned)w.tile * kRows + row_wave * kWaveRows; };      // the wave's first row
    // The wave's rows of q and its results share a piece of LDS: rows of 256 bytes, laid out as K's.
    lds_char* const own = shared + 4 * kTileBytes + row_wave * kWaveRows * kRowBytes;
    const auto load_q = [&](const Work& w) {
        const unsigned n_rows = (unsigned)w.n * a.G.d, lane = lane_again();
#pragma unroll
        for (int j = 0; j < kWaveRows / 4; ++j) {
            const unsigned i = j * 4 + (lane >> 4), row = row0(w) + i, pos = divide(row, a.G);
            const char* q = a.q + (int64_t)(w.first + (int)pos) * a.q_stride + (w.head * a.G.d + row - pos * a.G.d) * kRowBytes
                            + k_piece(i, lane & 15) * 16;
            load_to_lds(row < n_rows ? q : (const char*)kZeros, lds_address(own) + j * 4 * kRowBytes);
        }
    };

    // With parts two waves have the same rows, once: straight from global memory.
    const auto rows = [&](const Work& w) {
        const unsigned row = row0(w) + (lane_again() & 31), pos = divide(row, a.G);
        r.start(row < (unsigned)w.n * a.G.d
                    ? a.q + (int64_t)(w.first + (int)pos) * a.q_stride + (w.head * a.G.d + row - pos * a.G.d) * kRowBytes
                    : nullptr);
    };

    // An item's results wait in LDS until the next one's first tile is worked on:
    // stores count among the loads that a wave waits for.
    float lse = 0.0f;
    const auto store = [&](const Work& w) {
        const unsigned n_rows = (unsigned)w.n * a.G.d, lane = lane_again();
        const auto at = [&](unsigned row) {
            const unsigned pos = divide(row, a.G);
            return (int64_t)(w.first + (int)pos) * a.Hq + w.head * a.G.d + row - pos * a.G.d;
        };
#pragma unroll
        for (int j = 0; j < kWaveRows / 4; ++j) {
            const unsigned i = j * 4 + (lane >> 4), row = row0(w) + i;
            const f32x4 x = *(const lds_f32x4*)(own + i * kRowBytes + k_piece(i, lane & 15) * 16);
            if (row < n_rows) *(f32x4*)(a.out + at(row) * kRowBytes + (lane & 15) * 16) = x;
        }
        const unsigned row = row0(w) + lane;
        if (a.lse && lane < 32 && row < n_rows) a.lse[at(row)] = lse;
    };

    Work w, ahead, before;
    bool have = next(w), stored = true;
    if (!have) return;
    if (kParts == 1) load_q(w);
    else rows(w);
    load(w, 0, 0);
    arrived<0>();
    if (kParts == 1) r.read_q(own);
    for (unsigned buffer = 0;;) {
        // the item's first tile and q have arrived; the results of the one before lie in `own`
        barrier();
        if (!stored && part == 0) store(before);
        if (!have) return;
        const bool more = kParts == 1 && next(ahead);
        // positions of the wave's and the work group's rows
        const unsigned last_row = (unsigned)w.n * a.G.d - 1;
        const int wave_lo = (int)divide(min(row0(w), last_row), a.G), wave_hi = (int)divide(min(row0(w) + 31, last_row), a.G);
        const int tiles = (int)divide(min((unsigned)w.tile * kRows + kRows - 1, last_row), a.G) / kKeys + 1;
        const int own_tiles = row0(w) <= last_row ? wave_hi / kKeys + 1 : 0;
        const int pos = (int)divide(min(row0(w) + (lane & 31), last_row), a.G);
        // what is brought while tile t is worked on: the next one, or the next item's first
        const auto bring = [&](int t) {
            const bool last = t + 1 == tiles;
            if (!last || more) load(last ? ahead : w, last ? 0 : t + 1, buffer ^ 1);
            if (last && more) {
                was_read();
                load_q(ahead);
            }
        };
        if (a.scale.sign != (_Float16)1) r.times(a.scale.sign);
        r.clear();
        int t = 0;
        for (; t < own_tiles; ++t) {
            bring(t);
            const lds_char* kt = shared + buffer * 2 * kTileBytes + part * kPartKeys * kRowBytes;
            const int own_t = t * kParts + (int)part;       // the wave's keys, in 64s
            if (kParts == 1 || own_t * kPartKeys <= wave_hi) {
                f32x16 s[2];
                r.scores(kt, s);
                int finite = 1;
                if ((own_t + 1) * kPartKeys > wave_lo + 1) {
                    const int seen = pos - own_t * kPartKeys + 1;       // of them, those up to the row's own
                    r.mask(s, seen >= 64 ? ~0ull : seen <= 0 ? 0ull : (1ull << seen) - 1);
                    finite = r.finite(kt + kTileBytes);
                }
                finite = uniform(finite);
                if (__builtin_expect(finite, 1)) r.take(s, a.scale.c, kt + kTileBytes, wave_hi < own_t * kPartKeys + 32);
                asm volatile("" : "+s"(finite));     // one branch, of both, spills the sums
                if (__builtin_expect(!finite, 0)) {
#pragma nounroll
                    for (int key = own_t * kPartKeys; key <= min(own_t * kPartKeys + kPartKeys - 1, wave_hi); ++key) {
                        const int64_t at = (int64_t)(w.first + key) * a.kv_stride + w.head * kRowBytes;
                        r.take_key(a.k + at, a.v + at, a.scale.c, key <= pos);
                    }
                }
            }
            buffer ^= 1;
            if (t + 1 < tiles) {
                arrived<0>();
                barrier();
            }
        }
        for (; t < tiles; ++t) {                            // tiles that only other waves see
            bring(t);
            buffer ^= 1;
            if (t + 1 < tiles) {
                arrived<0>();
                barrier();
            }
        }
        if (more) {
            arrived<0>();
            r.read_q(own);
        }
        float sum = sum_of_halves(r.sum);
        if (kParts == 2) {
            // the second part's sums to the first, by way of the buffer that the last
            // tile has left, in two rounds
            lds_char* const meet = shared + (buffer ^ 1) * 2 * kTileBytes;
            lds_char* const ends = meet + kRowWaves * 8 * 1024 + row_wave * 512;
            float f = 1.0f, g = 1.0f;
            barrier();
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (part == 1) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int d = 2 * half + i / 4, e = i % 4 * 4;
                        *(lds_f32x4*)(meet + ((row_wave * 8 + i) * 64 + lane) * 16) =
                            f32x4{r.o[d][e], r.o[d][e + 1], r.o[d][e + 2], r.o[d][e + 3]};
                    }
                    if (half == 0) *(lds_f32x2*)(ends + lane * 8) = f32x2{r.top, sum};
                }
                barrier();
                if (part == 0) {
                    if (half == 0) {
                        const f32x2 other = *(const lds_f32x2*)(ends + lane * 8);
                        const float top = fmaxf(r.top, other[0]);
                        f = r.top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(r.top - top);
                        g = other[0] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(other[0] - top);
                        sum = f * sum + g * other[1];
                        r.top = top;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int d = 2 * half + i / 4, e = i % 4 * 4;
                        const f32x4 z = *(const lds_f32x4*)(meet + ((row_wave * 8 + i) * 64 + lane) * 16);
#pragma unroll
                        for (int j = 0; j < 4; ++j) r.o[d][e + j] = f * r.o[d][e + j] + g * z[j];
                    }
                }
                if (half == 0) barrier();
            }
        }
        if (part == 0) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            lse = (r.top - kBias + __builtin_amdgcn_logf(sum)) * kLn2;
            const unsigned in = lane_again() & 31, upper = lane_again() >> 5;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 x = {r.o[d][4 * i] * inv, r.o[d][4 * i + 1] * inv, r.o[d][4 * i + 2] * inv, r.o[d][4 * i + 3] * inv};
                    *(lds_f16x4*)(own + in * kRowBytes + k_piece(in, 4 * d + i) * 16 + upper * 8) =
                        __builtin_convertvector(x, f16x4);
                }
        }
        stored = false;
        before = w;
        w = ahead;
        have = more;
    }
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
    a.Hkv = divisor((unsigned)Hkv);
    a.G = divisor((unsigned)(Hq / Hkv));
    a.scale = q_scale(scale);
    int units = 0;
    rc = compute_units(&units);
    if (rc != APEX_OK) return rc;
    const int64_t rows = (int64_t)T * a.G.d;
    // Parts pay where a prompt's own chain of tiles is what takes the time: few items,
    // not too short, or about two to a unit if they are long.  32 over 8 heads, parts
    // and none: one prompt of 256 tokens 11.3 us and 12.5, of 1024 24.7 and 32.8, of
    // 2048 51 and 61; but of 100 9.4 and 9.2, of 4096 165 and 143, four of 512 tokens
    // 25.6 and 22.5.
    const int64_t parts_items = (rows / 128 + B) * Hkv, mean = T / B;
    if (mean >= 256 && 4 * parts_items <= (mean >= 1024 ? 9 : 5) * (int64_t)units) {
        const unsigned items = (unsigned)parts_items;
        prompt_kernel<2><<<items, 64 * kWaves, 0, (hipStream_t)stream>>>(a, items / (unsigned)Hkv, items, 1);
        return launched("prompt_attention");
    }
    const unsigned slots = (unsigned)(rows / 256) + (unsigned)B, items = slots * (unsigned)Hkv,
                   groups = items < (unsigned)units ? items : (unsigned)units;
    // From eight items a work group on the sums are alike enough to deal them all out;
    // below, the cheapest are left.  34 batches of 1.4 to 23 items a work group (1-64
    // prompts of 16-8192 tokens, G of 1 and 4), each with 1 to 8 rounds and with all
    // dealt out: this rule is 2.1 % above the best of them in the mean (8.6 at most),
    // all dealt out 3.9, one round 7.1, two 5.2, four 3.2.  From 4.5 to 6.7 items: four
    // rounds 1.2 %, two 5.7, all 5.3; from eight on: all 2.5, four 4.0, one 9.2.
    const double ratio = (double)items / groups;
    const unsigned rounds = ratio >= 8 ? (unsigned)((items + groups - 1) / groups) : ratio < 2 ? 1 : ratio < 4.5 ? 2 : ratio < 6.7 ? 4 : 6;
    const unsigned alone = items > rounds * groups ? items - rounds * groups : 0;
    prompt_kernel<1><<<groups + alone, 64 * kWaves, 0, (hipStream_t)stream>>>(a, slots, groups, rounds);
    return launched("prompt_attention");
}
