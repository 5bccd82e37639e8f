// tree_attention.hip -- attention of drafted tokens over a paged cache and each
// other (include/apex_steps.h).
//
// A pair's rows, its G q-heads of all drafted tokens, read each K and V row once:
// below some 200 rows the cache's bytes bound it, above the matrix cores.  32
// requests of 4096-32768 tokens with 5-8 drafted ones, 32 over 8 heads, are 1.78 GB
// and take 283 us: 6.3 TB/s, and 6.6 inside the stream of units; the rest is the
// first loads (9 us with the launch), the ends of parts, and the join (5).  With
// more rows the work of a unit bounds it (attend_tile.h): 16 requests of 8000 tokens,
// 8, 16, 32 and 64 drafted ones: 90, 112, 157 and 254 us, where the bytes take 81 and
// the operations of 64 113.
#include "attend_tile.h"
#include "steps_host.h"

namespace steps {

namespace {

constexpr int kSlabBytes = kBlockSize * kRowBytes;

// A pair is one request, one kv-head and one tile of its rows.  Its keys are taken
// in units of `keys` tokens: the cached ones, then one unit of the drafted ones.
// All pairs' units lie in one row, each pair's behind kPairCost units that stand for
// its start (2, 4 and 6 were no better than 1); the work groups get equal shares of
// it, one unit at least (one request of 500 tokens, shares of at least 1, 2 and 4:
// 14.7, 15.2, 15.7 us).  A part of a pair leaves its sums in the workspace, for
// join_kernel, a launch of its own: 3.4 us for one short request, 5-6 for batches.  (The
// decode attention has the last part to come join the others, by coherent stores and
// a count, for 0.8-1.3 us a part; here that was not built.)
constexpr int kPairCost = 1;

struct TreeArgs {
    const char *q, *k_new, *v_new, *k_cache, *v_cache;
    const int32_t *offsets, *table, *lens;
    const uint64_t* mask;
    char* out;
    float* lse;
    float* sums;                   // [2 groups][rows][128] unnormalised results of parts of pairs
    float* tops;                   // [2 groups][rows][2] their M and sum
    int4* joins;                   // [groups] the pair that the group's last part opens
    int64_t q_stride, new_stride;  // bytes between tokens
    int64_t table_stride, num_blocks;
    int B, T, max_nodes, Hq, Hkv;
    Divisor G;
    QScale scale;
};

// The kernel's arguments, read again: what only the ends of a part need does not
// stay in registers between them.
using Arguments = const __attribute__((address_space(4))) TreeArgs*;
__device__ inline Arguments arguments()
{
    Arguments p = (Arguments)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
}

struct Request {
    int first, nodes, len;         // its first packed row, its drafted and its cached tokens
    int units, tiles;              // units of a pair, tiles of rows
};

template <int kTileRows, int kKeys, class Args>
__device__ inline Request read_request(const Args& a, int b)
{
    Request r;
    const int lo = min(max(a.offsets[b], 0), a.T), hi = min(max(a.offsets[b + 1], lo), a.T);
    r.first = lo;
    r.nodes = min(hi - lo, a.max_nodes);
    r.len = (int)min((int64_t)max(a.lens[b], 0), a.table_stride * kBlockSize);
    r.units = r.nodes ? (int)(((int64_t)r.len + kKeys - 1) / kKeys) + 1 : 0;
    r.tiles = (r.nodes * (int)a.G.d + kTileRows - 1) / kTileRows;
    return r;
}

// Units of all of a request's pairs.
template <class Args>
__device__ inline int request_cost(const Args& a, const Request& r)
{
    return r.nodes ? a.Hkv * r.tiles * (r.units + kPairCost) : 0;
}

// Eight waves, one work group a compute unit: kRowWaves of them hold 32 rows each,
// kParts of them share a row tile's keys, 32 kSub each of a unit.  (Two work groups of
// four waves, for up to 32 rows: 335 us for 319.)
constexpr int kWaves = 8;
template <int kRowWaves_, int kSub_>
struct Shape {
    static constexpr int kRowWaves = kRowWaves_, kSub = kSub_;
    static constexpr int kParts = kWaves / kRowWaves;
    static constexpr int kWaveKeys = 32 * kSub, kKeys = kParts * kWaveKeys;
    static constexpr int kTileRows = kRowWaves * kWaveRows;
    static constexpr int kBytes = kKeys * kRowBytes;             // of a unit's K or V
    // A wave brings the keys that it takes and no others, into one buffer, each half
    // of which it fills again as soon as it has read it (kOwn), or the work group's
    // waves bring a unit together, into one of two buffers.  (16 full trees over 32
    // heads, weights still in one part: 64 rows with a copy of the keys for each of the
    // two waves that take them, and no barrier, 95 us for 81; K brought one and a half
    // units ahead, with a second barrier a unit, 88.)
    static constexpr bool kOwn = kRowWaves == 1;
    static constexpr int kBuffers = kOwn ? 1 : 2, kLds = 2 * kBuffers * kBytes;
    static constexpr int kLoads = kKeys / (4 * kWaves);          // of K, and of V, by which a wave brings its share of a unit
    static constexpr int kPartBlocks = kWaveKeys / kBlockSize;   // blocks of a wave's keys
    // Parts' sums are joined by way of the buffer that the last unit has left (of
    // kOwn its half for V), in rounds.
    static constexpr int kRounds = kParts == 1 ? 1 : kWaves * kWaveRows * kHeadDim * 4 / ((kOwn ? 1 : 2) * kBytes);
    static_assert(kParts == 1 || kRounds == 1 || kRounds == 2 || kRounds == 4, "a round takes 128 / kRounds dims");
};

// A part of a pair that a work group takes: units [lo, hi) of it.
struct Segment {
    Request q;
    int b, pair_at, lo, hi, kv_head, tile, cached;
};

template <class S>
__global__ __launch_bounds__(64 * kWaves, 2) void tree_kernel(TreeArgs a)
{
    constexpr int kParts = S::kParts, kWaveKeys = S::kWaveKeys, kKeys = S::kKeys, kLoads = S::kLoads;
    constexpr int kTileRows = S::kTileRows, kBytes = S::kBytes, kSub = S::kSub;
    constexpr bool kOwn = S::kOwn;
    __shared__ __attribute__((aligned(16))) char lds[S::kLds];
    __shared__ float merge_top[kWaves][kWaveRows], merge_sum[kWaves][kWaveRows];

    const unsigned lane = threadIdx.x & 63, wave = (unsigned)uniform((int)(threadIdx.x >> 6));
    const unsigned half = lane >> 5;
    const int row_wave = (int)wave / kParts, part = (int)wave % kParts;
    const int from = part * kWaveKeys;                   // this wave's keys of a unit

    // the share of this work group: [begin, end) of `total` units
    if (threadIdx.x == 0) a.joins[2 * blockIdx.x] = int4{0, 0, 0, 0};
    Request mine = {};                                   // of request `lane`
    if ((int)lane < a.B) mine = read_request<kTileRows, kKeys>(a, lane);
    const int cost0 = request_cost(a, mine), upto0 = wave_scan(cost0);
    int total = __builtin_amdgcn_readlane(upto0, 63);
    for (int i = 64; i < a.B; i += 64)
        total += wave_sum(i + (int)lane < a.B ? request_cost(a, read_request<kTileRows, kKeys>(a, i + lane)) : 0);
    const int active = min((int)gridDim.x, total);
    if ((int)blockIdx.x >= active) return;
    const int share = uniform(total / active), longer = total - share * active;      // the first `longer` take one more
    const int begin = share * (int)blockIdx.x + min((int)blockIdx.x, longer);
    const int end = begin + share + ((int)blockIdx.x < longer ? 1 : 0);
    // the request that `begin` falls into, and where its pairs start
    int b = 0, base = 0;
    for (int i = 0; i < a.B; i += 64) {
        int cost = cost0, upto = upto0;
        if (i) {
            cost = i + (int)lane < a.B ? request_cost(a, read_request<kTileRows, kKeys>(a, i + lane)) : 0;
            upto = wave_scan(cost);
        }
        const uint64_t behind = __ballot(base + upto > begin);
        if (behind) {
            const int l = __builtin_ctzll(behind);
            b = i + l;
            base += __builtin_amdgcn_readlane(upto - cost, l);
            break;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
    }
    b = uniform(b);
    base = uniform(base);

    int x = begin;
    const auto next = [&](Segment& g) {                  // false: there are no more
        const Arguments f = arguments();
        while (x < end) {
            if (b < 64) {
                g.q.first = __builtin_amdgcn_readlane(mine.first, b);
                g.q.nodes = __builtin_amdgcn_readlane(mine.nodes, b);
                g.q.len = __builtin_amdgcn_readlane(mine.len, b);
                g.q.units = __builtin_amdgcn_readlane(mine.units, b);
                g.q.tiles = __builtin_amdgcn_readlane(mine.tiles, b);
            } else {
                g.q = read_request<kTileRows, kKeys>(*f, b);
            }
            const int cost = request_cost(*f, g.q);
            if (x >= base + cost) {
                base += cost;
                ++b;
                continue;
            }
            const int per_pair = g.q.units + kPairCost;
            const int pair = uniform((x - base) / per_pair);
            g.b = b;
            g.pair_at = base + pair * per_pair + kPairCost;      // the pair's unit 0
            g.lo = max(x - g.pair_at, 0);
            g.hi = min(end - g.pair_at, g.q.units);
            g.kv_head = g.q.tiles == 1 ? pair : uniform(pair / g.q.tiles);
            g.tile = pair - g.kv_head * g.q.tiles;
            g.cached = g.q.units - 1;                    // units of cached tokens
            x = g.pair_at + g.q.units;
            if (g.hi > g.lo) return true;
        }
        return false;
    };

    // A unit's rows: load j of a wave brings four keys, in LDS one behind the other,
    // and lane i the piece that belongs at i % 16 of key i / 16.
    lds_char* const shared = (lds_char*)lds;
    constexpr int kIds = kOwn ? kLoads / 4 : kLoads;
    int ids[kIds], part_ids[S::kPartBlocks];             // of the blocks of the unit that is asked for next
    const unsigned block_bytes = (unsigned)a.Hkv * kSlabBytes, num_blocks = (unsigned)a.num_blocks;
    const auto first_key = [&](int j) { return kOwn ? (int)wave * kWaveKeys + j * 4 : (j * kWaves + (int)wave) * 4; };
    const auto id_of = [&](const Segment& g, const int32_t* row, int u, int key) {
        const int e = u * (kKeys / kBlockSize) + key / kBlockSize;
        return u < g.cached && e * kBlockSize < g.q.len ? row[e] : -1;
    };
    const auto ask = [&](const Segment& g, int u) {
        const Arguments f = arguments();
        const int32_t* row = f->table + (int64_t)g.b * f->table_stride;
#pragma unroll
        for (int j = 0; j < kIds; ++j) ids[j] = id_of(g, row, u, first_key(kOwn ? 4 * j : j));
#pragma unroll
        for (int j = 0; j < S::kPartBlocks; ++j) part_ids[j] = id_of(g, row, u, from + j * kBlockSize);
    };
    const auto load = [&](const Segment& g, int u, int buffer, bool is_v) {
        const Arguments f = arguments();
        const char* const head = (is_v ? f->v_cache : f->k_cache) + (int64_t)g.kv_head * kSlabBytes;
        const unsigned to = lds_address(shared) + buffer * 2 * kBytes + (is_v ? kBytes : 0);
        const unsigned lane = lane_again(), quad = lane >> 4;      // the lane's key of a load's four
        const int left = u < g.cached ? g.q.len - u * kKeys : g.q.nodes;
        bool plain = first_key(kLoads - 1) + 4 <= left;
#pragma unroll
        for (int j = 0; j < kIds; ++j) plain = plain && (unsigned)ids[j] < num_blocks;
        if (plain) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                // of a block's 16 keys, the load's first
                const unsigned in_block = kOwn ? (j & 3) * 4 : (wave & 3) * 4;
                const unsigned offset = (in_block + quad) * kRowBytes
                                        + (is_v ? v_piece(quad, lane & 15) : k_piece(in_block + quad, lane & 15)) * 16;
                stream_to_lds(head + (int64_t)ids[kOwn ? j / 4 : j] * block_bytes, offset, to + first_key(j) * kRowBytes);
            }
            return;
        }
        if (u >= g.cached) {                             // drafted tokens
            const char* const fresh = (is_v ? f->v_new : f->k_new) + (int64_t)g.q.first * f->new_stride + g.kv_head * kRowBytes;
#pragma nounroll
            for (int j = 0; j < kLoads; ++j) {
                const int key = first_key(j) + (int)quad;
                const char* row = fresh + key * f->new_stride + (is_v ? v_piece(key, lane & 15) : k_piece(key, lane & 15)) * 16;
                if (key >= left) row = (const char*)kZeros;
                load_to_lds(row, to + first_key(j) * kRowBytes);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {               // a context's end, blocks outside the pool
            const unsigned in_block = (kOwn ? (j & 3) * 4 : (wave & 3) * 4) + quad;
            const int id = ids[kOwn ? j / 4 : j];
            const char* row = head + (int64_t)id * block_bytes + in_block * kRowBytes
                              + (is_v ? v_piece(quad, lane & 15) : k_piece(in_block, lane & 15)) * 16;
            if ((unsigned)id >= num_blocks || first_key(j) + (int)quad >= left) row = (const char*)kZeros;
            load_to_lds(row, to + first_key(j) * kRowBytes);
        }
    };
    // which blocks of the wave's part are in the pool
    const auto present = [&]() {
        unsigned bits = 0;
#pragma unroll
        for (int j = 0; j < S::kPartBlocks; ++j)
            if ((unsigned)part_ids[j] < num_blocks) bits |= 1u << j;
        return bits;
    };
    Rows<kSub, true> r;
    uint64_t tree;                                       // the drafted tokens that the lane's rows see
    const auto row_of = [&](const Segment& g) {
        return (unsigned)(g.tile * kTileRows + row_wave * kWaveRows) + (lane_again() & 31);
    };
    const auto rows = [&](const Segment& g) {
        const Arguments f = arguments();
        const unsigned row = row_of(g), G = f->G.d, node = divide(row, f->G);
        const bool live = (int)node < g.q.nodes;
        r.start(live ? f->q + (int64_t)(g.q.first + (int)node) * f->q_stride + (g.kv_head * G + row - node * G) * kRowBytes
                     : nullptr);
        tree = live ? f->mask[g.q.first + (int)node] : 0;
    };

    Segment g, ahead;
    if (!next(g)) return;
    ask(g, g.lo);
    rows(g);
    r.clear();
    unsigned there = present(), buffer = 0;
    load(g, g.lo, 0, false);
    load(g, g.lo, 0, true);
    if (a.scale.sign != (_Float16)1) r.times(a.scale.sign);
    const float c = a.scale.c;
    for (int u = g.lo;;) {
        // the unit that is brought while this one is worked on: the part's next, or
        // the first of the work group's next part
        const bool last = u + 1 == g.hi;
        bool more = true;
        if (last) more = next(ahead);
        else ahead = g;
        const int u_ahead = last ? ahead.lo : u + 1;
        if (more) ask(ahead, u_ahead);
        if (kOwn) {
            arrived<kLoads>();                           // K
        } else {
            arrived<0>();
            barrier();
            if (more) {
                load(ahead, u_ahead, buffer ^ 1, false);
                load(ahead, u_ahead, buffer ^ 1, true);
            }
        }
        lds_char* const kt = shared + (kOwn ? 0 : buffer * 2 * kBytes) + from * kRowBytes;
        // a wave without rows or keys leaves its SIMD to the others
        const int n = u < g.cached ? g.q.len - u * kKeys - from : g.q.nodes - from;      // the wave's keys
        const bool works = n > 0 && (kOwn || row_wave * kWaveRows < g.q.nodes * (int)a.G.d - g.tile * kTileRows);
        f32x16 s[kSub];
        if (works) r.scores(kt, s);
        if (kOwn && more) {
            was_read();
            load(ahead, u_ahead, 0, false);
        }
        if (kOwn) {
            if (more) arrived<kLoads>();                 // V; the next K is on its way
            else arrived<0>();
        }
        if (works) {
            int finite = 1;
            uint64_t allow = 0;                          // the keys that are there
            if (u < g.cached) {
#pragma unroll
                for (int j = 0; j < S::kPartBlocks; ++j)
                    if (there >> j & 1) allow |= 0xffffull << (16 * j);
                allow &= n >= 64 ? ~0ull : (1ull << n) - 1;
                if (allow != (kSub == 2 ? ~0ull : 0xffffffffull)) r.mask(s, allow);
            } else {
                r.mask(s, tree >> (from & 63) & (n >= 64 ? ~0ull : (1ull << n) - 1));
                finite = r.finite(kt + kBytes);
            }
            finite = uniform(finite);
            if (__builtin_expect(finite, 1)) r.take(s, c, kt + kBytes);
            asm volatile("" : "+s"(finite));     // one branch, of both, spills the sums
            if (__builtin_expect(!finite, 0)) {
                const Arguments f = arguments();
#pragma nounroll
                for (int i = 0; i < min(n, kWaveKeys); ++i) {
                    const int64_t at = (int64_t)(g.q.first + from + i) * f->new_stride + g.kv_head * kRowBytes;
                    r.take_key(f->k_new + at, f->v_new + at, c, tree >> (from + i) & 1);
                }
            }
        }
        if (kOwn && !last) {
            was_read();
            load(ahead, u_ahead, 0, true);
        }
        there = present();
        if (!last) {
            ++u;
            buffer ^= 1;
            continue;
        }

        // the part's end
        const Arguments out = arguments();
        if (more) rows(ahead);                           // on their way while the parts meet

        // the parts' sums together, each wave of a tile some of the dims
        lds_char* const meet = shared + (kOwn ? kBytes : buffer * 2 * kBytes);
        const bool whole = g.lo == 0 && g.hi == g.q.units;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (g.lo == 0 ? 1 : 0);
        float top = r.top, sum = sum_of_halves(r.sum), f[kParts];
        if (kParts > 1) {
            if (half == 0) {
                merge_top[wave][lane] = top;
                merge_sum[wave][lane] = sum;
            }
            barrier();
            top = -INFINITY;
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kParts; ++w) {
                f[w] = merge_top[row_wave * kParts + w][lane & 31];
                top = fmaxf(top, f[w]);
            }
#pragma unroll
            for (int w = 0; w < kParts; ++w) {
                f[w] = f[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(f[w] - top);
                sum = __builtin_fmaf(f[w], merge_sum[row_wave * kParts + w][lane & 31], sum);
            }
        }
        const unsigned row = row_of(g), G = out->G.d, node = divide(row, out->G);
        const bool live = (int)node < g.q.nodes;
        const int64_t to = (int64_t)(g.q.first + (int)node) * out->Hq + g.kv_head * G + row - node * G;
        const int64_t in_slot = slot * kTileRows + row_wave * kWaveRows + (lane & 31);
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int round = 0; round < S::kRounds; ++round) {
            constexpr int kQuads = 16 / S::kRounds;      // of 4 dims a lane, of a round
            if (kParts > 1) {
                if (round) barrier();
#pragma unroll
                for (int i = 0; i < kQuads; ++i) {
                    const int t = (round * kQuads + i) / 4, e = (round * kQuads + i) % 4 * 4;
                    *(lds_f32x4*)(meet + ((wave * kQuads + i) * 64 + lane) * 16) =
                        f32x4{r.o[t][e], r.o[t][e + 1], r.o[t][e + 2], r.o[t][e + 3]};
                }
                barrier();
            }
#pragma unroll
            for (int i = 0; i < kQuads; ++i) {
                if (kParts > 1 && i / (kQuads / kParts) != part) continue;
                const int t = (round * kQuads + i) / 4, e = (round * kQuads + i) % 4;
                f32x4 y = {r.o[t][4 * e], r.o[t][4 * e + 1], r.o[t][4 * e + 2], r.o[t][4 * e + 3]};
                if (kParts > 1) {
                    y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int w = 0; w < kParts; ++w) {
                        const f32x4 z = *(const lds_f32x4*)(meet + (((row_wave * kParts + w) * kQuads + i) * 64 + lane) * 16);
#pragma unroll
                        for (int j = 0; j < 4; ++j) y[j] = __builtin_fmaf(f[w], z[j], y[j]);
                    }
                }
                if (!live) continue;
                if (whole) {
                    y = f32x4{y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
                    *(f16x4*)(out->out + to * kRowBytes + t * 64 + e * 16 + half * 8) = __builtin_convertvector(y, f16x4);
                } else {
                    *(f32x4*)(out->sums + in_slot * kHeadDim + t * 32 + e * 8 + half * 4) = y;
                }
            }
        }
        if (live && part == 0 && half == 0) {
            if (!whole) *(f32x2*)(out->tops + in_slot * 2) = f32x2{top, sum};
            else if (out->lse) out->lse[to] = (top - kBias + __builtin_amdgcn_logf(sum)) * kLn2;
        }
        if (!whole && g.lo == 0 && threadIdx.x == 0) {
            // the parts: this one and those of the next work groups up to the pair's end
            const int to_end = g.pair_at + g.q.units - 1;         // the pair's last unit, and who takes it
            const int owner = to_end < longer * (share + 1) ? to_end / (share + 1) : longer + (to_end - longer * (share + 1)) / share;
            const int n_rows = min(kTileRows, g.q.nodes * (int)out->G.d - g.tile * kTileRows);
            out->joins[2 * blockIdx.x] = int4{n_rows, owner - (int)blockIdx.x + 1, g.q.first, g.kv_head};
            out->joins[2 * blockIdx.x + 1] = int4{g.tile * kTileRows, 0, 0, 0};
        }
        if (!more) return;
        if (kOwn) {
            barrier();                                   // all have met
            load(ahead, u_ahead, 0, true);
        }
        if (a.scale.sign != (_Float16)1) r.times(a.scale.sign);
        r.clear();
        g = ahead;
        u = g.lo;
        buffer ^= 1;
    }
}

// Joins the parts of the pair that work group x's last part opens; 8 rows a work
// group, 32 lanes a row.  Bound by its launch and two round trips, 3.4 us for small
// tiles, 6 for 128 rows; 16 to 64 rows a work group made 52 us of a chat batch 53-57.
__global__ __launch_bounds__(256) void join_kernel(TreeArgs a, int tile_rows)
{
    const int4 job = a.joins[2 * blockIdx.x];
    const int row = (int)blockIdx.y * 8 + (int)(threadIdx.x >> 5), i = threadIdx.x & 31;
    if (row >= job.x) return;
    const int at = a.joins[2 * blockIdx.x + 1].x + row;
    float top = -INFINITY, sum = 0.0f;
    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int p = 0; p < job.y; ++p) {
        const int64_t slot = p == 0 ? 2 * (int64_t)blockIdx.x + 1 : 2 * ((int64_t)blockIdx.x + p);
        const f32x2 ts = *(const f32x2*)(a.tops + (slot * tile_rows + row) * 2);
        const f32x4 z = *(const f32x4*)(a.sums + (slot * tile_rows + row) * kHeadDim + i * 4);
        const float to = fmaxf(top, ts[0]);
        const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - to);
        const float g = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ts[0] - to);
        sum = sum * f + ts[1] * g;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = y[j] * f + z[j] * g;
        top = to;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int G = (int)a.G.d, node = (int)divide((unsigned)at, a.G);
    const int64_t to = (int64_t)(job.z + node) * a.Hq + job.w * G + (at - node * G);
    y = f32x4{y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
    *(f16x4*)(a.out + to * kRowBytes + i * 8) = __builtin_convertvector(y, f16x4);
    if (a.lse && i == 0) a.lse[to] = (top - kBias + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Shapes by the most rows of a pair: the smallest that holds them, whose waves share
// the keys of a row among the most of them.  16 requests of 8000 tokens, 32 over
// 8 heads, in shapes of 32, 64, 128 and 256: 32 rows 90, 104, 111, 141 us; 64 rows 112,
// 118, 150; 128 rows 157, 175.  256 rows as one tile of 256 and as two of 128: 254 and
// 281 us, but 59 and 53 for 1000 tokens; 8 requests of 4096 tokens on 64 over 8 heads,
// 256 rows 84 and 91 us, 512 rows 141 and 153.  Their floors are 113, 17, 29 and
// 58 us: few units a work group, and ends of parts that are as long.
using Shape32 = Shape<1, 1>;
using Shape64 = Shape<2, 1>;
using Shape128 = Shape<4, 2>;
using Shape256 = Shape<8, 2>;

int tile_rows(int max_nodes, int G)
{
    const int64_t rows = (int64_t)max_nodes * G;
    return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256;
}

struct Workspace {
    size_t sums, tops, joins, bytes;
};

Workspace lay_out(int groups, int tile_rows)
{
    Workspace w;
    w.sums = 0;
    w.tops = align_up((size_t)2 * groups * tile_rows * kHeadDim * 4, 256);
    w.joins = w.tops + align_up((size_t)2 * groups * tile_rows * 8, 256);
    w.bytes = w.joins + align_up((size_t)groups * 32, 256);
    return w;
}

int check_nodes(int max_nodes)
{
    if (max_nodes < 1) return fail(APEX_ERR_INVALID_ARG, "max_nodes = %d must be positive", max_nodes);
    if (max_nodes > APEX_STEPS_MAX_NODES)
        return fail(APEX_ERR_UNSUPPORTED, "max_nodes = %d exceeds %d", max_nodes, APEX_STEPS_MAX_NODES);
    return APEX_OK;
}

}  // namespace

}  // namespace steps

extern "C" {

size_t apex_steps_tree_workspace_bytes(int max_nodes, int Hq, int Hkv)
{
    using namespace steps;
    apex::clear_error();
    int units = 0;
    if (Hkv <= 0 || Hq <= 0 || Hq % Hkv != 0 || Hq > kMostHeads || check_nodes(max_nodes) != APEX_OK ||
        compute_units(&units) != APEX_OK)
        return 0;
    return lay_out(units, tile_rows(max_nodes, Hq / Hkv)).bytes;
}

int apex_steps_tree_attention(const void* q, int64_t q_token_stride, const void* k_new, const void* v_new,
                              int64_t new_token_stride, const int32_t* token_offsets, const uint64_t* tree_mask,
                              const void* k_cache, const void* v_cache, const int32_t* block_table,
                              int64_t block_table_stride, const int32_t* context_lens, void* out, float* lse_out,
                              int B, int T, int max_nodes, int Hq, int Hkv, int d, int block_size,
                              int64_t num_blocks, float scale, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace steps;
    apex::clear_error();
    int rc = check_attention(B, T, Hq, Hkv, d, scale, &q_token_stride, &new_token_stride);
    if (rc == APEX_OK) rc = check_nodes(max_nodes);
    if (rc != APEX_OK) return rc;
    if (block_size != kBlockSize) return fail(APEX_ERR_UNSUPPORTED, "block_size %d unsupported (only 16)", block_size);
    if (num_blocks < 0 || block_table_stride < 0)
        return fail(APEX_ERR_INVALID_ARG, "num_blocks and block_table_stride must not be negative");
    constexpr int64_t kMost = (int64_t)1 << 27;
    if (num_blocks >= kMost || block_table_stride >= kMost)
        return fail(APEX_ERR_UNSUPPORTED, "num_blocks or block_table_stride reaches 2^27");
    const int G = Hq / Hkv;
    const int64_t tiles = ((int64_t)max_nodes * G + 127) / 128;
    if ((double)B * Hkv * tiles * (double)(block_table_stride + 64) >= 2147483648.0)
        return fail(APEX_ERR_UNSUPPORTED, "B * Hkv * row tiles * (block_table_stride + 64) reaches 2^31");
    if (B == 0 || T == 0) return APEX_OK;
    if (!q || !k_new || !v_new || !token_offsets || !tree_mask || !context_lens || !out)
        return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if ((num_blocks > 0 && (!k_cache || !v_cache)) || (block_table_stride > 0 && !block_table))
        return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_cache, 16) ||
        !aligned(v_cache, 16) || !aligned(out, 16))
        return fail(APEX_ERR_INVALID_ARG, "q, k_new, v_new, k_cache, v_cache and out must be 16-byte aligned");
    if (!aligned(token_offsets, 4) || !aligned(tree_mask, 8) || !aligned(block_table, 4) || !aligned(context_lens, 4) ||
        !aligned(lse_out, 4))
        return fail(APEX_ERR_INVALID_ARG, "an array is not aligned to its element");
    const size_t pool = (size_t)num_blocks * Hkv * kSlabBytes;
    const Extent inputs[] = {{"q", q, rows_bytes(T, q_token_stride, Hq, 2)},
                             {"k_new", k_new, rows_bytes(T, new_token_stride, Hkv, 2)},
                             {"v_new", v_new, rows_bytes(T, new_token_stride, Hkv, 2)},
                             {"token_offsets", token_offsets, ((size_t)B + 1) * 4},
                             {"tree_mask", tree_mask, (size_t)T * 8},
                             {"k_cache", k_cache, pool},
                             {"v_cache", v_cache, pool},
                             {"block_table", block_table, (size_t)B * block_table_stride * 4},
                             {"context_lens", context_lens, (size_t)B * 4},
                             {"lse_out", lse_out, (size_t)T * Hq * 4},
                             {"out", out, (size_t)T * Hq * kRowBytes}};
    rc = check_disjoint(inputs[10], inputs, 10);
    if (rc == APEX_OK) rc = check_disjoint(inputs[9], inputs, 9);
    if (rc != APEX_OK) return rc;

    if (workspace && !aligned(workspace, 256))
        return fail(APEX_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    int groups = 0;      // one on a compute unit
    rc = compute_units(&groups);
    if (rc != APEX_OK) return rc;
    const int rows = tile_rows(max_nodes, G);
    const Workspace w = lay_out(groups, rows);
    Hold hold;
    if (workspace) {
        rc = check_workspace(workspace, workspace_bytes, w.bytes);
        if (rc == APEX_OK) rc = check_disjoint({"workspace", workspace, w.bytes}, inputs, 11);
    } else {
        rc = library_workspace(w.bytes, (hipStream_t)stream, hold, &workspace);
    }
    if (rc != APEX_OK) return rc;

    TreeArgs a;
    a.q = (const char*)q;
    a.k_new = (const char*)k_new;
    a.v_new = (const char*)v_new;
    a.k_cache = (const char*)k_cache;
    a.v_cache = (const char*)v_cache;
    a.offsets = token_offsets;
    a.table = block_table;
    a.lens = context_lens;
    a.mask = tree_mask;
    a.out = (char*)out;
    a.lse = lse_out;
    a.sums = (float*)((char*)workspace + w.sums);
    a.tops = (float*)((char*)workspace + w.tops);
    a.joins = (int4*)((char*)workspace + w.joins);
    a.q_stride = q_token_stride * 2;
    a.new_stride = new_token_stride * 2;
    a.table_stride = block_table_stride;
    a.num_blocks = num_blocks;
    a.B = B;
    a.T = T;
    a.max_nodes = max_nodes;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = divisor((unsigned)G);
    a.scale = q_scale(scale);
    const hipStream_t on = (hipStream_t)stream;
    const auto kernel = rows == 32 ? tree_kernel<Shape32> : rows == 64 ? tree_kernel<Shape64>
                        : rows == 128 ? tree_kernel<Shape128> : tree_kernel<Shape256>;
    kernel<<<groups, 64 * kWaves, 0, on>>>(a);
    rc = launched("tree_attention");
    if (rc != APEX_OK) return rc;
    join_kernel<<<dim3(groups, rows / 8), 256, 0, on>>>(a, rows);
    return launched("tree_attention");
}

}  // extern "C"
