// tree_attention.hip -- attention of drafted tokens over a paged cache and each
// other (include/apex_steps.h).
#include "attend_tile.h"
#include "steps_host.h"

namespace steps {

namespace {

constexpr int kSlabBytes = kBlockSize * kRowBytes;

// A pair is one request, one kv-head and one tile of its rows.  Its keys are taken
// in units of `keys` tokens: the cached ones, then one unit of the drafted ones.
// All pairs' units lie in one row, each pair's behind kPairCost units that stand for
// its start; the work groups that take part get equal shares of it.
constexpr int kPairCost = 1;
constexpr int kLeastShare = 2;

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
    int B, T, max_nodes, Hq, Hkv, G;
    float c;
    bool negate;
};

struct Request {
    int first, nodes, len;         // its first packed row, its drafted and its cached tokens
    int units, tiles;              // units of a pair, tiles of rows
};

template <int kTileRows, int kKeys>
__device__ inline Request read_request(const TreeArgs& a, int b)
{
    Request r;
    const int lo = min(max(a.offsets[b], 0), a.T), hi = min(max(a.offsets[b + 1], lo), a.T);
    r.first = lo;
    r.nodes = min(hi - lo, a.max_nodes);
    r.len = (int)min((int64_t)max(a.lens[b], 0), a.table_stride * kBlockSize);
    r.units = r.nodes ? (int)(((int64_t)r.len + kKeys - 1) / kKeys) + 1 : 0;
    r.tiles = (r.nodes * a.G + kTileRows - 1) / kTileRows;
    return r;
}

// Units of all of a request's pairs.
__device__ inline int request_cost(const TreeArgs& a, const Request& r)
{
    return r.nodes ? a.Hkv * r.tiles * (r.units + kPairCost) : 0;
}

// kRowTiles waves hold a tile of rows each, kWaves / kRowTiles waves share a row
// tile's keys, 32 kSub each of a unit.
template <int kRowTiles, int kSub, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void tree_kernel(TreeArgs a)
{
    constexpr int kParts = kWaves / kRowTiles;
    constexpr int kWaveKeys = 32 * kSub, kKeys = kParts * kWaveKeys;
    constexpr int kTileRows = kRowTiles * kWaveRows;
    // A wave brings the keys that it takes and no others, into one buffer of its own
    // (kOwn), or the work group's waves bring a unit together, into one of two.
    constexpr bool kOwn = kRowTiles == 1;
    constexpr int kBuffers = kOwn ? 1 : 2;
    constexpr int kLoads = kKeys / (4 * kWaves);         // of K, and of V, by which a wave brings its share of a unit
    constexpr int kBlocks = kOwn ? kWaveKeys / kBlockSize : kKeys / kBlockSize;    // in which this share lies
    constexpr int kBytes = kKeys * kRowBytes;            // of K or of V
    static_assert(kParts == 1 || kWaves * kWaveRows * kHeadDim * 4 <= 2 * kBuffers * kBytes, "the sums pass through the buffers");
    static_assert(kOwn || kWaves == 4, "a wave's load brings four of a block's 16 keys");
    __shared__ __attribute__((aligned(16))) char lds[2 * kBuffers * kBytes];
    __shared__ float merge_top[kWaves][kWaveRows], merge_sum[kWaves][kWaveRows];

    const unsigned lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned half = lane >> 5;
    const int row_tile = (int)wave % kRowTiles, part = (int)wave / kRowTiles;

    // the share of this work group
    int64_t total = 0;
    for (int i = 0; i < a.B; i += 64) {
        int cost = 0;
        if (i + (int)lane < a.B) cost = request_cost(a, read_request<kTileRows, kKeys>(a, i + lane));
        total += wave_sum(cost);
    }
    const int64_t active = min((int64_t)gridDim.x, (total + kLeastShare - 1) / kLeastShare);
    if (threadIdx.x == 0) a.joins[2 * blockIdx.x] = int4{0, 0, 0, 0};
    if ((int64_t)blockIdx.x >= active) return;
    const int64_t begin = uniform((int64_t)(total * blockIdx.x / active));
    const int64_t end = uniform((int64_t)(total * (blockIdx.x + 1) / active));
    // the request that `begin` falls into, and where its pairs start
    int b = 0;
    int64_t base = 0;
    for (int i = 0; i < a.B; i += 64) {
        int cost = 0;
        if (i + (int)lane < a.B) cost = request_cost(a, read_request<kTileRows, kKeys>(a, i + lane));
        const int upto = wave_scan(cost);
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

    Rows<kSub> r;
    lds_char* const shared = (lds_char*)lds;
    for (int64_t x = begin; x < end;) {
        Request q = read_request<kTileRows, kKeys>(a, b);
        const int cost = request_cost(a, q);
        if (x >= base + cost) {
            base += cost;
            ++b;
            continue;
        }
        const int per_pair = q.units + kPairCost;
        const int pair = uniform((int)((x - base) / per_pair));
        const int64_t at = base + (int64_t)pair * per_pair + kPairCost;      // the pair's unit 0
        const int lo = (int)max(x - at, (int64_t)0), hi = (int)min(end - at, (int64_t)q.units);
        x = at + q.units;
        if (hi <= lo) continue;
        const int kv_head = pair / q.tiles, tile = pair - kv_head * q.tiles;
        const int cached = q.units - 1;                  // units of cached tokens
        const int rows = min(kTileRows, q.nodes * a.G - tile * kTileRows);

        const unsigned row = (unsigned)(tile * kTileRows + row_tile * kWaveRows) + (lane & 31);
        const bool live = (int)row < q.nodes * a.G;
        const unsigned node = min(row / (unsigned)a.G, (unsigned)q.nodes - 1);
        const unsigned qhead = (unsigned)kv_head * a.G + row % (unsigned)a.G;
        r.start(live ? a.q + (int64_t)(q.first + (int)node) * a.q_stride + qhead * kRowBytes : nullptr, a.negate);
        const uint64_t tree = a.mask[q.first + (int)node] & (q.nodes >= 64 ? ~0ull : (1ull << q.nodes) - 1);
        const int32_t* ids = a.table + (int64_t)b * a.table_stride;

        // A unit's rows: load j of a wave brings four keys, in LDS one behind the
        // other, and lane i the piece that belongs at i % 16 of key i / 16.  The ids of
        // the blocks are asked for a unit ahead.
        int ids_next[kBlocks];
        const auto ask = [&](int u) {
#pragma unroll
            for (int j = 0; j < kBlocks; ++j) {
                const int e = u * (kKeys / kBlockSize) + (kOwn ? (int)wave * kBlocks : 0) + j;
                ids_next[j] = u < cached && e * kBlockSize < q.len ? ids[e] : -1;
            }
        };
        unsigned there_next = 0;                         // blocks of ids_next that are in the pool
        const auto load = [&](int u, const char* cache, const char* fresh, bool is_v) {
            const unsigned to = lds_address(shared) + (u & (kBuffers - 1)) * 2 * kBytes + (is_v ? kBytes : 0);
            const int left = u < cached ? q.len - u * kKeys : q.nodes;
            there_next = 0;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int first_key = kOwn ? (int)wave * kWaveKeys + j * 4 : j * 16 + (int)wave * 4;
                const int key = first_key + (int)(lane >> 4), block = kOwn ? j / 4 : j;
                const unsigned piece = is_v ? v_piece(key, lane & 15) : k_piece(key, lane & 15);
                const char* from;
                if (u < cached) {
                    const int id = ids_next[block];
                    const bool in_pool = id >= 0 && id < (int)a.num_blocks;
                    if (in_pool) there_next |= 1u << block;
                    from = cache + ((int64_t)id * a.Hkv + kv_head) * kSlabBytes + (key % kBlockSize) * kRowBytes + piece * 16;
                    if (!in_pool || key >= left) from = (const char*)kZeros;
                } else {
                    from = fresh + (int64_t)(q.first + key) * a.new_stride + kv_head * kRowBytes + piece * 16;
                    if (key >= left) from = (const char*)kZeros;
                }
                load_to_lds(from, to + first_key * kRowBytes);
            }
        };
        const auto load_k = [&](int u) { load(u, a.k_cache, a.k_new, false); };
        const auto load_v = [&](int u) { load(u, a.v_cache, a.v_new, true); };
        const int from = part * kWaveKeys;               // this wave's keys of a unit
        ask(lo);
        barrier();                                       // the buffers are free
        load_k(lo);
        load_v(lo);
        for (int u = lo; u < hi; ++u) {
            const unsigned there = there_next;
            const bool more = u + 1 < hi;
            if (more) ask(u + 1);
            if (kOwn) {
                arrived<kLoads>();                       // K
            } else {
                arrived<0>();
                barrier();
                if (more) {
                    load_k(u + 1);
                    load_v(u + 1);
                }
            }
            uint64_t allow;                              // the keys that the lane's row sees
            bool all = false;
            if (u < cached) {
                allow = 0;
#pragma unroll
                for (int j = 0; j < kWaveKeys / kBlockSize; ++j)
                    if (there >> ((kOwn ? 0 : from / kBlockSize) + j) & 1) allow |= 0xffffull << (16 * j);
                const int n = q.len - u * kKeys - from;
                allow &= n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
                all = allow == (kSub == 2 ? ~0ull : 0xffffffffull);
            } else {
                allow = from < 64 ? tree >> from : 0;
            }
            const lds_char* kt = shared + (u & (kBuffers - 1)) * 2 * kBytes + from * kRowBytes;
            f32x16 s[kSub];
            f16x8 p[2 * kSub];
            r.scores(kt, s);
            if (kOwn && more) {
                was_read();
                load_k(u + 1);
            }
            if (!all) r.mask(s, allow);
            r.weights(s, a.c, p);
            if (kOwn) {
                if (more) arrived<kLoads>();             // V; the next K is on its way
                else arrived<0>();
            }
            r.add(kt + kBytes, p);
            if (kOwn && more) {
                was_read();
                load_v(u + 1);
            }
        }
        if (__builtin_expect(r.spoiled(), 0)) {
            r.clear();
#pragma nounroll
            for (int i = 0; i < (hi - lo) * kWaveKeys; ++i) {
                const int u = lo + i / kWaveKeys, key = from + i % kWaveKeys;
                const char *k = (const char*)kZeros, *v = k;
                bool sees = false;
                if (u < cached) {
                    const int token = u * kKeys + key;
                    const int id = token < q.len ? ids[token / kBlockSize] : -1;
                    if (id >= 0 && id < (int)a.num_blocks) {
                        const int64_t to = ((int64_t)id * a.Hkv + kv_head) * kSlabBytes + token % kBlockSize * kRowBytes;
                        k = a.k_cache + to;
                        v = a.v_cache + to;
                        sees = true;
                    }
                } else if (key < q.nodes) {
                    const int64_t to = (int64_t)(q.first + key) * a.new_stride + kv_head * kRowBytes;
                    k = a.k_new + to;
                    v = a.v_new + to;
                    sees = tree >> key & 1;
                }
                r.take_key(k, v, a.c, sees);
            }
        }

        // the parts' sums together: each wave of a row tile joins some of the dims
        float top = r.top, sum = sum_of_halves(r.sum), f[kParts];
        f[0] = 1.0f;
        if (kParts > 1) {
            barrier();
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(__attribute__((address_space(3))) f32x4*)(shared + ((wave * 16 + t * 4 + i) * 64 + lane) * 16) =
                        f32x4{r.o[t][4 * i], r.o[t][4 * i + 1], r.o[t][4 * i + 2], r.o[t][4 * i + 3]};
            if (half == 0) {
                merge_top[wave][lane] = top;
                merge_sum[wave][lane] = sum;
            }
            __syncthreads();
            float tp[kParts];
            top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kParts; ++w) {
                tp[w] = merge_top[w * kRowTiles + row_tile][lane & 31];
                top = fmaxf(top, tp[w]);
            }
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kParts; ++w) {
                f[w] = tp[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(tp[w] - top);
                const float sw = merge_sum[w * kRowTiles + row_tile][lane & 31];
                sum += f[w] * sw;
                // a part's NaN stays one also where the part has seen no score
                if (sw != sw) sum = sw;
            }
        }
        const bool whole = lo == 0 && hi == q.units;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (lo == 0 ? 1 : 0);
        const unsigned in_tile = row_tile * kWaveRows + (lane & 31);
        const int64_t to = (int64_t)(q.first + (int)node) * a.Hq + qhead;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (kParts > 1 && (t * 4 + i) / (16 / kParts) != part) continue;
                f32x4 y = {r.o[t][4 * i], r.o[t][4 * i + 1], r.o[t][4 * i + 2], r.o[t][4 * i + 3]};
                if (kParts > 1) {
                    y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int w = 0; w < kParts; ++w) {
                        const f32x4 z = *(const __attribute__((address_space(3))) f32x4*)(
                            shared + (((w * kRowTiles + row_tile) * 16 + t * 4 + i) * 64 + lane) * 16);
#pragma unroll
                        for (int j = 0; j < 4; ++j) y[j] = __builtin_fmaf(f[w], z[j], y[j]);
                    }
                }
                if (!live) continue;
                if (whole) {
                    y = f32x4{y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
                    *(f16x4*)(a.out + to * kRowBytes + t * 64 + i * 16 + half * 8) = __builtin_convertvector(y, f16x4);
                } else {
                    *(f32x4*)(a.sums + (slot * kTileRows + in_tile) * kHeadDim + t * 32 + i * 8 + half * 4) = y;
                }
            }
        }
        if (live && part == 0 && half == 0) {
            if (!whole) *(f32x2*)(a.tops + (slot * kTileRows + in_tile) * 2) = f32x2{top, sum};
            else if (a.lse) a.lse[to] = (top - kBias + __builtin_amdgcn_logf(sum)) * kLn2;
        }
        if (!whole && lo == 0 && threadIdx.x == 0) {
            // the parts: this one and those of the next work groups up to the pair's end
            const int64_t last = ((at + q.units) * active - 1) / total;
            a.joins[2 * blockIdx.x] = int4{rows, (int)(last - blockIdx.x) + 1, q.first, kv_head};
            a.joins[2 * blockIdx.x + 1] = int4{tile * kTileRows, 0, 0, 0};
        }
    }
}

// Joins the parts of the pair that work group x's last part opens; 8 rows a work
// group, 32 lanes a row.
__global__ __launch_bounds__(256) void join_kernel(TreeArgs a, int tile_rows)
{
    const int4 job = a.joins[2 * blockIdx.x];
    const int row = (int)blockIdx.y * 8 + (int)(threadIdx.x >> 5), i = threadIdx.x & 31;
    if (row >= job.x) return;
    const int at = a.joins[2 * blockIdx.x + 1].x + row;
    float top = -INFINITY, sum = 0.0f;
    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
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
    const int node = at / a.G;
    const int64_t to = (int64_t)(job.z + node) * a.Hq + job.w * a.G + (at - node * a.G);
    y = f32x4{y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv};
    *(f16x4*)(a.out + to * kRowBytes + i * 8) = __builtin_convertvector(y, f16x4);
    if (a.lse && i == 0) a.lse[to] = (top - kBias + __builtin_amdgcn_logf(sum)) * kLn2;
}

int row_tiles(int max_nodes, int G)
{
    const int rows = max_nodes * G;
    return rows <= kWaveRows ? 1 : rows <= 2 * kWaveRows ? 2 : 4;
}

// Work groups that a compute unit's LDS holds.
int groups_per_unit(int row_tiles) { return row_tiles == 1 ? 1 : 2; }

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
    if (Hkv <= 0 || Hq <= 0 || Hq % Hkv != 0 || Hq > INT_MAX / 1024 || check_nodes(max_nodes) != APEX_OK ||
        compute_units(&units) != APEX_OK)
        return 0;
    const int waves = row_tiles(max_nodes, Hq / Hkv);
    return lay_out(units * groups_per_unit(waves), waves * kWaveRows).bytes;
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
    int units = 0;
    rc = compute_units(&units);
    if (rc != APEX_OK) return rc;
    const int waves = row_tiles(max_nodes, G), tile_rows = waves * kWaveRows, groups = units * groups_per_unit(waves);
    const Workspace w = lay_out(groups, tile_rows);
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
    a.G = G;
    a.c = (scale < 0 ? -scale : scale) * kLog2e;
    a.negate = scale < 0;
    const auto kernel = waves == 1 ? tree_kernel<1, 1, 8> : waves == 2 ? tree_kernel<2, 1, 4> : tree_kernel<4, 2, 4>;
    kernel<<<groups, waves == 1 ? 512 : 256, 0, (hipStream_t)stream>>>(a);
    rc = launched("tree_attention");
    if (rc != APEX_OK) return rc;
    join_kernel<<<dim3(groups, tile_rows / 8), 256, 0, (hipStream_t)stream>>>(a, tile_rows);
    return launched("tree_attention");
}

}  // extern "C"
