// kv4_attention.hip -- decode attention over the 4-bit KV cache, and the
// accumulation of its attention weights (include/apex_kv4.h).
//
// Scores.  S^T = K Q^T runs on the block-scaled MFMA 16x16x128 (fp4 x fp8):
// K's codes and scale bytes go into it as they lie in the cache, 16 bytes and
// one byte per lane, and are never unpacked.  Its B operand holds 8-bit values,
// so a row of q is split into four digits: with 2^E <= max |q_i| < 2^(E + 1),
// q_i = 2^(E - 3) sum_p d_p 32^-p, the d_p integers with |d_p| <= 16, which
// fp8 holds exactly; the p-th digits of the G q-heads are columns 4p to 4p + 3
// of the operand, with the unit 2^(E - 3 - 5p) as their scale (G = 8: columns
// 0-7 and 8-15 hold two digits, a second MFMA the other two).  The last unit is
// 2^(E - 18): an element of at least 2^-8 of the row's largest binade is exact,
// a smaller one rounded by 2^-19 of it.  (fp8 digits with exponents of their
// own would be fewer, but the MFMA aligns its 128 products to a common
// exponent: 13 bits survive a wide range of exponents; sums of products of
// integers come out exact, and groups with different scales are joined to
// fp32 precision.)  The digits' columns are then added over lanes.
//
// Values.  O^T += V^T P^T runs on the bf16 MFMA 16x16x32.  A byte of V's codes
// holds two neighbouring dims of one token, and one conversion turns it, times
// the token's scale, into the two halves of an operand word.  The MFMA takes
// the halves as two k-indices, so k runs over (token, parity of the dim), the
// 16 rows over octets of dims, and B's columns are (head, parity): a column has
// the token's weight at its own parity and zero at the other.  That saves the
// byte permutes that a transpose in registers takes.  bf16 holds every
// value of the cache exactly (fp16 would not hold the largest); the fp32
// weights go in as two bf16 parts, in columns of their own (G = 8: in two passes):
// the first cut off, the rest rounded to nearest, so that a weight is within 2^-16
// of itself, to either side (the result's fp16 half step is 2^-11), while the
// normaliser sums them unrounded.
//
// Bound by HBM for long batches: 32 requests of 4096-32768 tokens, 8 kv-heads, G =
// 4, 452 MB in 79 us (5.7 TB/s; plain reads of slabs in the same pattern reach 6.8),
// one of 131071, 143 MB, in 29.4.  The difference is the launch, the first round trip
// (table, then slabs), the waves' uneven ends and the joining of split pairs, 6-8 us
// a call, which is most of a small batch's time (16 of 256-4096, 38 MB, 16.1 us).
#include <type_traits>

#include "kernels.h"
#include "kv4_host.h"

namespace {

using apex::f16;
using apex::f32x4;
using apex::u32x2;
using apex::u32x4;
using apex::uniform;
using kv4::fail;
using kv4::kBlockSize;
using kv4::kHeadDim;
using kv4::kSlabBytes;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Eight waves per work group and one work group per CU: they keep 4 blocks, 70
// KiB a CU, on their way, and 25 KiB saturate the memory.  More waves would need
// registers that the loop has not got (with 4 per SIMD it spills: 97 us for the
// 213 000 slabs of 32 requests of 4096-32768 tokens, 75 with 2).
constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;

struct Params {
    const f16* q;           // [B][Hq][128]
    const char* cache;      // [num_blocks][Hkv][kSlabBytes]
    const int32_t* bt;      // [B][stride]
    const int32_t* lens;
    unsigned num_blocks;
    int stride;
    int B, Hq, Hkv;
    int workers;            // work groups launched
    float scale_log2;       // |scale| log2(e)
    unsigned q_sign;        // 0x8000 to negate q (scale < 0)
    // attention
    f16* out;
    float* lse;             // may be null
    int32_t* counters;      // [B][Hkv] arrivals, zero between calls
    float* pacc;            // [2 workers][G][128] partial sums of the weighted values,
    float* pml;             // [2 workers][G][2] their maxima (log2 units) and sums of weights
    // accumulation of the weights
    const float* lse_in;    // [B][Hq]
    float* weights;         // [num_blocks][Hkv][16]
};

// --- partition ----------------------------------------------------------------
//
// Every wave derives the work group's share on its own from context_lens: a lane
// sums ceil(B / 64) consecutive requests, one scan joins them.  Three ways:
//   whole   many short pairs: a wave takes whole (request, kv-head) pairs;
//   parts   few pairs: each is cut into equal parts, a work group takes one part;
//   line    else: the line of plan_policy.h: every non-empty pair has kPairCost
//           positions, then its blocks; work group w takes the positions
//           [start(w), start(w + 1)).
// All positions are below 2^31 (the host checks the table's size).

// What a pair costs a work group besides its blocks, in blocks (0.08 us each): 32
// take 1.01 of the time over 30 batches, 1.16 at worst, 128 1.002, 1.04 at worst.
constexpr unsigned kPairCost = 64;
// Parts: the least, and the most that still goes better than the line (uneven
// last parts against pairs that begin and end inside a work group).  Over 50
// batches the line alone takes 1.16 of the time, 1.6 at worst (6 pairs of 20
// blocks 9.1 against 14.5 us, 192 of 20-54 10.1 against 15.7); parts of up to 128
// blocks 1.01, 1.5 at worst, of up to 1000 1.015, 1.34 at worst.
constexpr unsigned kMinPart = 32, kMaxPart = 320;
// Whole pairs by waves, where there are more pairs than work groups.  In blocks
// of a work group's time (0.08 us): the line takes (U + kPairCost pairs) / W; the
// waves stream U / W (uneven: an eighth more), or, with few blocks to a wave, are
// held up by its round trips, about 3 for each of the longest pairs in a row; and
// start once.  Measured, line against waves: 3200 pairs of 2-44 blocks 78 against
// 41 us, 2048 of 63 66 against 47, 1024 of 125 55 against 48; but 512 of 88-125 34
// against 44, 400 of 94 28 against 36.  Up to kWholeBlocks the waves always win
// (1080 pairs of 1-2 blocks 23.5 against 7.0 us); past kMostWhole the wave with the
// longest pairs ends alone (2400 pairs of 10-185 blocks 87 against 121 us).
constexpr unsigned kWholeBlocks = 32, kMostWhole = 128;

__device__ inline bool waves_take_pairs(unsigned U, unsigned pairs, unsigned longest, unsigned W)
{
    if (pairs <= W || longest > kMostWhole) return false;
    if (longest <= kWholeBlocks) return true;
    const unsigned per = U / W, rounds = (pairs + kWaves * W - 1) / (kWaves * W);
    return max(3 * longest * rounds, per + per / 8) + 32 < per + kPairCost * pairs / W;
}

struct Line {
    unsigned V, W, per, rest;   // positions, work groups; V = W per + rest
    __device__ inline void set(unsigned positions, unsigned groups)
    {
        V = positions;
        W = groups;
        per = W ? V / W : 0;
        rest = V - per * W;
    }
    __device__ inline unsigned start(unsigned w) const { return w * per + w * rest / W; }   // (w rest < W^2)
    __device__ inline unsigned owner(unsigned v) const
    {
        // at most one off the quotient of the reals
        unsigned w = (unsigned)((double)v * (double)W / (double)V);
        if (w >= W) w = W - 1;
        while (w + 1 < W && start(w + 1) <= v) ++w;
        while (start(w) > v) --w;
        return w;
    }
};

enum Way { kLine, kParts, kWhole };

struct Plan {
    Way way;
    Line line;
    unsigned v1;            // line: end of the work group's positions
    unsigned vf;            // line: position of the pair's block 0
    int b, g, blk, L;       // the first segment
    int take;               // its blocks; 0: none
    int first, last;        // parts: the work groups of the pair
    bool empty_rows;        // some request has no context
};

__device__ inline int context(const Params& p, int b)
{
    const int64_t row = (int64_t)p.stride * kBlockSize;
    const int L = p.lens[b];
    return L > row ? (int)row : L;
}

__device__ inline unsigned blocks(int L) { return L > 0 ? ((unsigned)L + kBlockSize - 1) / kBlockSize : 0u; }

// Blocks per part of a pair of nb; a long pair takes longer ones, since the last
// work group to finish reads all the parts' partials.
__device__ inline unsigned part_blocks(unsigned nb, unsigned least)
{
    const unsigned t = max(kMinPart, kMinPart / 2 + nb / 64);
    return max(t, least);
}

// Up to 64 requests (kFew) a lane holds one, and the plan reads the lengths once.
template <bool kAttention, bool kFew>
__device__ inline Plan plan_of(const Params& p, unsigned hk, unsigned K, unsigned w, int lane)
{
    const int R = kFew ? 1 : (p.B + 63) / 64;
    const int r0 = min(p.B, lane * R), r1 = min(p.B, r0 + R);
    const int own = r0 < r1 ? context(p, r0) : 0;   // the lane's only request's length (kFew)
    auto sum = [&](auto f) -> unsigned {            // of f(blocks) over the lane's requests
        if (kFew) return f(blocks(own));
        unsigned n = 0;
        for (int b = r0; b < r1; ++b) n += f(blocks(context(p, b)));
        return n;
    };
    auto length = [&](int b) -> int { return kFew ? apex::lane_value(own, b) : uniform(context(p, b)); };
    unsigned units = 0, count = 0, longest = 0;
    sum([&](unsigned nb) -> unsigned {
        units += nb;
        count += nb > 0;
        longest = max(longest, nb);
        return 0;
    });
    const unsigned cost = units + K * count;
    const unsigned hi = (unsigned)apex::wave_incl_sum((int)cost), lo = hi - cost;
    const unsigned total = (unsigned)apex::lane_value((int)hi, 63);
    const unsigned nonempty = kFew ? (unsigned)__popcll(__ballot(count > 0))
                                   : (unsigned)apex::lane_value(apex::wave_incl_sum((int)count), 63);
    longest = (unsigned)apex::lane_value(apex::wave_incl_max((int)longest), 63);
    Plan r;
    r.way = kLine;
    r.empty_rows = nonempty < (unsigned)p.B;
    r.v1 = r.vf = 0;
    r.b = r.g = r.blk = r.L = r.take = r.first = r.last = 0;
    const unsigned V = total * hk, pairs = nonempty * hk, U = V - K * pairs, W = (unsigned)p.workers;
    if (U == 0) return r;
    if (kAttention && waves_take_pairs(U, pairs, longest, W)) {
        r.way = kWhole;
        return r;
    }
    if (kAttention && pairs <= W) {
        const unsigned room = W - pairs;
        const unsigned least = longest <= 2 * kMinPart ? longest : room > 0 ? (U + room - 1) / room : U;
        if (least <= kMaxPart) {
            // the parts of the requests before a lane's, then the request of part w
            const unsigned parts = sum([&](unsigned nb) -> unsigned {
                const unsigned t = part_blocks(nb, least);
                return (nb + t - 1) / t;
            });
            r.way = kParts;
            const unsigned phi = (unsigned)apex::wave_incl_sum((int)parts), plo = phi - parts;
            const uint64_t hit = __ballot(plo * hk <= w && w < phi * hk);
            if (hit == 0) return r;
            const int ln = __builtin_ctzll(hit);
            unsigned rest = w - (unsigned)apex::lane_value((int)plo, ln) * hk;
            unsigned nb, t, c;
            for (int b = ln * R;; ++b) {
                r.b = b;
                r.L = length(b);
                nb = blocks(r.L);
                t = part_blocks(nb, least);
                c = (nb + t - 1) / t;
                if (rest < c * hk) break;
                rest -= c * hk;
            }
            r.g = (int)(rest / c);
            const unsigned part = rest - (unsigned)r.g * c;
            // equal parts (which may leave the last work groups of the pair without one)
            t = (nb + c - 1) / c;
            r.blk = (int)min(nb, part * t);
            r.take = (int)min(t, nb - (unsigned)r.blk);
            r.first = (int)(w - part);
            r.last = r.first + (int)((nb + t - 1) / t) - 1;
            return r;
        }
    }
    r.line.set(V, W);
    const unsigned v0 = r.line.start(w);
    r.v1 = r.line.start(w + 1);
    if (v0 >= r.v1) return r;
    // the lane whose requests hold v0, then the request
    const int ln = __builtin_ctzll(__ballot(lo * hk <= v0 && v0 < hi * hk));
    unsigned at = (unsigned)apex::lane_value((int)lo, ln) * hk;
    unsigned nb;
    for (int b = ln * R;; ++b) {
        r.b = b;
        r.L = length(b);
        nb = blocks(r.L);
        const unsigned span = nb > 0 ? (nb + K) * hk : 0u;
        if (v0 < at + span) break;
        at += span;
    }
    const unsigned off = v0 - at, len = nb + K;
    r.g = (int)(off / len);
    r.vf = at + (unsigned)r.g * len + K;
    r.blk = v0 > r.vf ? (int)(v0 - r.vf) : 0;
    if (r.vf + (unsigned)r.blk < r.v1) r.take = (int)min(nb - (unsigned)r.blk, r.v1 - (r.vf + (unsigned)r.blk));
    return r;
}

template <bool kAttention>
__device__ inline Plan make_plan(const Params& p, int heads, unsigned K, unsigned w, int lane)
{
    const unsigned hk = (unsigned)heads;
    return p.B <= 64 ? plan_of<kAttention, true>(p, hk, K, w, lane) : plan_of<kAttention, false>(p, hk, K, w, lane);
}

// Moves a line's plan to the work group's next segment; false when it has none.
__device__ inline bool next_segment(const Params& p, int heads, unsigned K, Plan& r)
{
    const unsigned nb = blocks(r.L);
    if ((unsigned)(r.blk + r.take) < nb) return false;   // the range ended inside the pair
    r.vf += nb + K;
    r.blk = 0;
    if (r.vf >= r.v1) return false;
    if (++r.g == heads) {
        r.g = 0;
        do {
            if (++r.b >= p.B) return false;
            r.L = uniform(context(p, r.b));
        } while (r.L <= 0);
    }
    r.take = (int)min(blocks(r.L), r.v1 - r.vf);
    return true;
}

// --- operands -----------------------------------------------------------------

// Digits of q as the B operand of the scores, and the column's scale byte.
// Lane (c, q) holds, for column c, dims 16q + [0, 16) and 64 + 16q + [0, 16) as
// bytes; the scale byte of block q of 32 dims is also lane (c, q)'s, and a row
// has one exponent, so all four are the same.
template <int G>
struct QueryOperand {
    i32x8 d[G == 8 ? 2 : 1];
    int scale[G == 8 ? 2 : 1];
};

// A lane's dims of its column's head, as they are.
struct QueryRow {
    u32x4 w[4];
};

template <int G>
__device__ inline void load_row(const Params& p, int b, int g, int lane, QueryRow& q)
{
    const int col = lane & 15;
    const int head = G == 8 ? col & 7 : (col & 3) & (G - 1);
    const f16* row = p.q + ((size_t)b * p.Hq + (size_t)g * G + head) * kHeadDim + 16 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) q.w[i] = *(const u32x4*)(row + (i >> 1) * 64 + (i & 1) * 8);
}

template <int G>
__device__ inline void split_query(unsigned q_sign, const QueryRow& row, int lane, QueryOperand<G>& op)
{
    const int col = lane & 15;
    u32x4 w[4] = {row.w[0], row.w[1], row.w[2], row.w[3]};
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[i][j] ^= q_sign * 0x10001u;
            m = max(m, max(w[i][j] & 0x7fffu, (w[i][j] >> 16) & 0x7fffu));
        }
    // as floats the bit patterns of non-negative values order alike; a NaN or
    // an infinity lies above every finite one
    m = max(m, (unsigned)__shfl_xor((int)m, 16, 64));
    m = max(m, (unsigned)__shfl_xor((int)m, 32, 64));
    const bool finite = m < 0x7c00u;
    const float mf = (float)__builtin_bit_cast(f16, (unsigned short)(m > 0 ? m : 1u));
    const int E = (int)(__float_as_uint(mf) >> 23) - 127;
#pragma unroll
    for (int s = 0; s < (G == 8 ? 2 : 1); ++s) {
        const int digit = G == 8 ? 2 * s + (col >> 3) : col >> 2;
        // q / unit of this digit, and of the one before it (0 for the first)
        const float hi = __uint_as_float((unsigned)(127 + 3 - E + 5 * digit) << 23);
        const float lo = digit > 0 ? hi * 0.03125f : 0.f;
        op.scale[s] = finite ? 127 + E - 3 - 5 * digit : kv4::kNanScale;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int bytes = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const apex::f16x2 h = apex::as_h2(w[i >> 1][(i & 1) * 2 + j]);
                const float x = (float)h[0], y = (float)h[1];
                const float dx = rintf(x * hi) - 32.f * rintf(x * lo), dy = rintf(y * hi) - 32.f * rintf(y * lo);
                bytes = j == 0 ? __builtin_amdgcn_cvt_pk_fp8_f32(dx, dy, bytes, false)
                               : __builtin_amdgcn_cvt_pk_fp8_f32(dx, dy, bytes, true);
            }
            op.d[s][i] = finite ? bytes : 0;
        }
    }
}

// One block of a pair: K's and V's codes and scales as a lane uses them.
struct Tile {
    u32x4 k, v;
    int ks;         // scale byte of token lane % 16, group lane / 16
    unsigned vs;    // scale bytes of tokens 4q .. 4q + 3, group (lane % 16) / 4
};

__device__ inline __amdgpu_buffer_rsrc_t slab_resource(const char* slab, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((void*)apex::uniform_ptr(slab), (short)0, bytes, apex::kRawBufferWord3);
}

// The attention reads K through the Infinity Cache: a step that accumulates its
// weights reads it again.  (Attention and accumulation of four caches in turn, 32
// requests of 8192 tokens, G = 4: 80 us a cache, 89 with K read past it; the
// attention alone is the same either way.)  V, and K in the accumulation, go past.
template <int kPolicy>
__device__ inline void load_keys(Tile& t, __amdgpu_buffer_rsrc_t r, int lane)
{
    const int c = lane & 15, q = lane >> 4;
    t.k = __builtin_amdgcn_raw_buffer_load_b128(r, c * 64 + q * 16, 0, kPolicy);
    t.ks = __builtin_amdgcn_raw_buffer_load_b8(r, kv4::kKScales + c * 4 + q, 0, kPolicy);
}

__device__ inline void load_values(Tile& t, __amdgpu_buffer_rsrc_t r, int lane)
{
    const int c = lane & 15, q = lane >> 4;
    t.v = __builtin_amdgcn_raw_buffer_load_b128(r, kv4::kVCodes + lane * 16, 0, apex::kStreamingLoad);
    t.vs = __builtin_amdgcn_raw_buffer_load_b32(r, kv4::kVScales + (c >> 2) * 16 + q * 4, 0, apex::kStreamingLoad);
}

// A value plus that of the lane 8 (or 4) columns on, within 16 lanes.
template <int kDpp>
__device__ inline float add_rotated(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kDpp, 0xf, 0xf, true));
}
constexpr int kRor4 = 0x124, kRor8 = 0x128;

// q . K of tokens 4q .. 4q + 3 with the lane's head.
template <int G>
__device__ inline f32x4 scores(const Tile& t, const QueryOperand<G>& op)
{
    const i32x8 a = {(int)t.k[0], (int)t.k[1], (int)t.k[2], (int)t.k[3], 0, 0, 0, 0};
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, op.d[0], s, 4, 0, 0, t.ks, 0, op.scale[0]);
    if constexpr (G == 8) s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, op.d[1], s, 4, 0, 0, t.ks, 0, op.scale[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = add_rotated<kRor8>(s[i]);
        if (G < 8) s[i] = add_rotated<kRor4>(s[i]);
    }
    return s;
}

// --- attention ------------------------------------------------------------------

// A wave's state: lane (col, q) has its head's running max m (log2 units) and
// sum l, and tile j's element i is the head's P.V at dim 8 (4q + i) + 2j +
// parity (for G < 8 of one part of the weights).
struct State {
    float m, l;
    f32x4 acc[4];
};

// The blocks of a wave in a segment: [first, first + n) of pair (b, g).
struct Span {
    const int32_t* bt;    // table entry of the first
    const char* pair;     // slab of kv-head g in block 0
    uint64_t step;        // bytes from a block to the next
    unsigned pool;        // blocks
    int first, n;
    int L;
};

// The wave's share of blocks [lo, hi), one of n (blocks are taken in twos).
__device__ inline Span wave_span(const Params& p, int b, int g, int L, int lo, int hi, int i, int n)
{
    Span s;
    const int per = (hi - lo + 2 * n - 1) / (2 * n) * 2;
    s.first = uniform(lo + i * per);
    s.n = uniform(max(0, min(hi, s.first + per) - s.first));
    s.bt = p.bt + (size_t)uniform(b) * (size_t)p.stride + (s.n > 0 ? s.first : 0);
    s.pair = apex::uniform_ptr(p.cache + (size_t)uniform(g) * kSlabBytes);
    s.step = (uint64_t)p.Hkv * kSlabBytes;
    s.pool = p.num_blocks;
    s.L = uniform(L);
    return s;
}

// Blocks of a wave are taken two at a time (a step), two steps in flight.
struct Step {
    Tile t[2];
    unsigned id[2];     // block ids of the tiles,
    unsigned next[2];   // and of those that refill them
};

struct Pipe {
    Step x[2];
    QueryRow q;
};

__device__ inline unsigned id_at(const Span& s, int i)
{
    // (an entry that is not the wave's is replaced, not read: s.bt[0] is readable)
    const unsigned id = *(const __attribute__((address_space(4))) uint32_t*)(s.bt + (i < s.n ? i : 0));
    return i < s.n ? id : 0xffffffffu;
}

// The slab of a block, with no extent (loads give zeros) outside the pool.
__device__ inline __amdgpu_buffer_rsrc_t slab_of(const Span& s, unsigned id)
{
    return slab_resource(s.pair + id * s.step, id < s.pool ? kSlabBytes : 0);
}

// Asks for the row of q and a span's first blocks.
template <int G>
__device__ inline void begin(const Params& p, int b, int g, const Span& s, int lane, Pipe& pipe)
{
    load_row<G>(p, b, g, lane, pipe.q);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        Step& x = pipe.x[i];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            x.id[j] = id_at(s, 2 * i + j);
            const auto r = slab_of(s, x.id[j]);
            load_keys<0>(x.t[j], r, lane);
            load_values(x.t[j], r, lane);
            x.next[j] = id_at(s, 4 + 2 * i + j);
        }
    }
}

// A wave's attention over its span, whose first blocks are on their way.
template <int G>
__device__ inline void attend(const Params& p, const Span& s, int lane, Pipe& pipe, State& st)
{
    const int col = lane & 15, q = lane >> 4;
    const int parity = G == 8 ? col >> 3 : (col >> 2) & 1;
    // bytes 2 and 3 of a weight to the half of its parity, zeros to the other
    const unsigned place = parity ? 0x03020c0cu : 0x0c0c0302u;
    const unsigned low_part = G < 8 && col >= 8 ? 0xffff0000u : 0u, round = G == 8 || col >= 8 ? 0x8000u : 0u;
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) st.acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // q's digits are worked out while the first blocks are on their way
    QueryOperand<G> op;
    split_query<G>(p.q_sign, pipe.q, lane, op);

    // blocks k and k + 1, in x; x is refilled with k + 4 and k + 5
    auto step = [&](Step& x, int k) {
        const bool good[2] = {x.id[0] < s.pool, x.id[1] < s.pool};
        const int tok = (s.first + k) * kBlockSize;
        const bool tail = !good[0] || !good[1] || tok > s.L - 2 * kBlockSize;
        float sc[8];
        {
            const f32x4 s0 = scores<G>(x.t[0], op), s1 = scores<G>(x.t[1], op);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sc[e] = s0[e];
                sc[4 + e] = s1[e];
            }
        }
        // a tile's registers are refilled as soon as they are read (in place: the
        // barrier keeps the scheduler from issuing the loads above the reads)
        __builtin_amdgcn_sched_barrier(0);
        __amdgpu_buffer_rsrc_t refill[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x.id[i] = x.next[i];
            refill[i] = slab_of(s, x.id[i]);
            load_keys<0>(x.t[i], refill[i], lane);
            x.next[i] = id_at(s, k + 8 + i);
        }
        bool live[8];
        if (tail) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                live[e] = good[e >> 2] && tok + (e >> 2) * kBlockSize + 4 * q + (e & 3) < s.L;
                sc[e] = live[e] ? sc[e] : -INFINITY;
            }
        }
        float bm = sc[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) bm = fmaxf(bm, sc[e]);
        bm = apex::rows_max4(bm);
        const float m = fmaxf(st.m, bm * p.scale_log2);
        const float ms = m == -INFINITY ? 0.f : m;   // no token so far
        const float alpha = apex::exp2_fast(st.m - ms);
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = apex::exp2_fast(fmaf(sc[e], p.scale_log2, -ms));
        if (tail) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = live[e] ? w[e] : 0.f;   // (a scale of 0 makes -inf a NaN)
        }
        st.l = fmaf(st.l, alpha, ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7])));
        st.m = m;
        if (alpha != 1.f) {
#pragma unroll
            for (int j = 0; j < 4; ++j) st.acc[j] *= alpha;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            // weights and values as operand words
            u32x4 hi, lo, a[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float we = w[4 * i + e];
                const unsigned u = __float_as_uint(we);
                if (G < 8) {
                    const unsigned part = __float_as_uint(we - __uint_as_float(u & low_part)) + round;
                    hi[e] = __builtin_amdgcn_perm(0u, part, place);
                } else {
                    hi[e] = __builtin_amdgcn_perm(0u, u, place);
                    lo[e] = __builtin_amdgcn_perm(0u, __float_as_uint(we - __uint_as_float(u & 0xffff0000u)) + round, place);
                }
            }
            const unsigned vs = x.t[i].vs;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float scale = __uint_as_float((e == 0 ? vs << 23 : e == 1 ? vs << 15 : e == 2 ? vs << 7 : vs >> 1) & 0x7f800000u);
                if (tail) scale = live[4 * i + e] ? scale : 1.f;   // (an unused slot may hold a NaN scale)
                const unsigned v = x.t[i].v[e];
                a[0][e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 0));
                a[1][e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 1));
                a[2][e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 2));
                a[3][e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, scale, 3));
            }
            __builtin_amdgcn_sched_barrier(0);
            load_values(x.t[i], refill[i], lane);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                st.acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[j]),
                                                                    __builtin_bit_cast(bf16x8, hi), st.acc[j], 0, 0, 0);
            if (G == 8) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    st.acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8, a[j]), __builtin_bit_cast(bf16x8, lo), st.acc[j], 0, 0, 0);
            }
        }
    };
    // pairs of steps, then an odd last one: straight code between the loads of
    // a step and its waits
    int k = 0;
    for (; k + 2 < s.n; k += 4) {
        step(pipe.x[0], k);
        step(pipe.x[1], k + 2);
    }
    if (k < s.n) step(pipe.x[0], k);
    st.l = apex::rows_sum4(st.l);
}

// A wave's state into LDS: sums [head][dim], maxima and sums of weights.
template <int G>
struct Shared {
    __attribute__((aligned(16))) float acc[kWaves][G * kHeadDim];
    float m[kWaves][G];
    float l[kWaves][G];
    int last;
};

template <int G>
__device__ inline void store_state(State& st, int wave, int lane, Shared<G>& sh)
{
    const int col = lane & 15, q = lane >> 4;
    if (G < 8) {
        // the two parts of the weights
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.acc[j][i] = add_rotated<kRor8>(st.acc[j][i]);
    }
    const int head = G == 8 ? col & 7 : col & 3, parity = G == 8 ? col >> 3 : (col >> 2) & 1;
    if (head < G && (G == 8 || col < 8)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) sh.acc[wave][head * kHeadDim + 8 * (4 * q + i) + 2 * j + parity] = st.acc[j][i];
    }
    if (col < G && q == 0) {
        sh.m[wave][col] = st.m;
        sh.l[wave][col] = st.l;
    }
}

// N consecutive elements of a head's row: numerators and denominator relative
// to 2^M.
template <int N>
struct Row {
    float M, den;
    float num[N];
};

template <int N>
__device__ inline void clear(Row<N>& r)
{
    r.M = -INFINITY;
    r.den = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) r.num[i] = 0.f;
}

// Rescales r to the running max of C more (max, sum) pairs, the first n of them
// given, and adds their sums; f gets their factors.
template <int N, int C>
__device__ inline void join_sums(const float (&m)[C], const float (&l)[C], int n, Row<N>& r, float (&f)[C])
{
    float M = r.M;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        f[j] = j < n ? m[j] : -INFINITY;
        M = fmaxf(M, f[j]);
    }
    const float Ms = M == -INFINITY ? 0.f : M;
    const float f0 = apex::exp2_fast(r.M - Ms);
    r.den *= f0;
#pragma unroll
    for (int i = 0; i < N; ++i) r.num[i] *= f0;
    r.M = M;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        f[j] = apex::exp2_fast(f[j] - Ms);
        if (j < n) r.den = fmaf(f[j], l[j], r.den);
    }
}

// The waves' states of head h at dims [dim, dim + N), joined.
template <int G, int N>
__device__ inline void join_waves(const Shared<G>& sh, int h, int dim, Row<N>& r)
{
    float m[kWaves], l[kWaves], f[kWaves];
#pragma unroll
    for (int j = 0; j < kWaves; ++j) {
        m[j] = sh.m[j][h];
        l[j] = sh.l[j][h];
    }
    clear(r);
    join_sums<N, kWaves>(m, l, kWaves, r, f);
#pragma unroll
    for (int j = 0; j < kWaves; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) r.num[i] = fmaf(f[j], sh.acc[j][h * kHeadDim + dim + i], r.num[i]);
}

// The result's elements: zeros and -inf where there was no token; NaNs stay.
// The cache can hold 65536 (65504 rounded up), whose half would be infinite: a
// larger result than 65504 becomes that.
template <int N>
__device__ inline void emit_row(const Params& p, int b, int head, int dim, const Row<N>& r)
{
    typename apex::vec_of<f16, N>::type o;
    const float inv = 1.f / r.den;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        // a quotient by the reciprocal, corrected once: within a rounding of the
        // division's, which takes three times the instructions
        const float y = r.num[i] * inv;
        const float x = r.den == 0.f ? 0.f : fmaf(fmaf(-y, r.den, r.num[i]), inv, y);
        o[i] = (f16)(__builtin_fabsf(x) > 65504.f ? __builtin_copysignf(65504.f, x) : x);
    }
    *(typename apex::vec_of<f16, N>::type*)&p.out[((size_t)b * p.Hq + head) * kHeadDim + dim] = o;
    if (p.lse && dim == 0)
        p.lse[(size_t)b * p.Hq + head] = r.den == 0.f ? -INFINITY : (r.M + __log2f(r.den)) * 0.69314718055994531f;
}

// Partials of a split pair, written and read device-coherently: contributor c
// (work group wf + c) has slot 2 (wf + c), the first one slot 2 wf + 1 (a work
// group has at most two: the end of one pair, the start of another).
__device__ inline int64_t partial_slot(int w, int wf) { return 2 * (int64_t)w + (w == wf); }

template <int G>
__device__ inline __amdgpu_buffer_rsrc_t partial_sums(const Params& p, int64_t slot, int n)
{
    return __builtin_amdgcn_make_buffer_rsrc((void*)apex::uniform_ptr(p.pacc + slot * (G * kHeadDim)), (short)0,
                                             n * 2 * G * kHeadDim * 4, apex::kRawBufferWord3);
}

template <int G>
__device__ inline __amdgpu_buffer_rsrc_t partial_maxima(const Params& p, int64_t slot, int n)
{
    return __builtin_amdgcn_make_buffer_rsrc((void*)apex::uniform_ptr(p.pml + slot * (G * 2)), (short)0, n * 2 * G * 8,
                                             apex::kRawBufferWord3);
}

template <int G, int N>
__device__ inline void store_partial(const Params& p, int64_t slot, int e0, int h, bool first, const Row<N>& r)
{
    const auto acc = partial_sums<G>(p, slot, 1);
    if constexpr (N == 1)
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(r.num[0]), acc, e0 * 4, 0, apex::kCoherent);
    else
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(r.num[0]), __float_as_uint(r.num[1])}, acc, e0 * 4, 0,
                                              apex::kCoherent);
    if (first) {
        const u32x2 v = {__float_as_uint(r.M), __float_as_uint(r.den)};
        __builtin_amdgcn_raw_buffer_store_b64(v, partial_maxima<G>(p, slot, 1), h * 8, 0, apex::kCoherent);
    }
}

// Contributors [c0, c1) of a pair joined into this wave's state in LDS.  A lane
// owns 2 G consecutive elements of the pair's rows and asks for kRows partials
// at once: what a combine takes is round trips.
template <int G>
__device__ inline void join_partials(const Params& p, int wf, int c0, int c1, int wave, int lane, Shared<G>& sh)
{
    constexpr int N = 2 * G, kRows = G == 8 ? 4 : 8, kVecs = G == 1 ? 1 : N / 4, kPer = N / kVecs;
    typedef typename apex::vec_of<unsigned, kPer>::type word;
    const int h = lane * N / kHeadDim, dim = lane * N % kHeadDim;
    Row<N> r;
    clear(r);
    for (; c0 < c1; c0 += kRows) {
        const int n = min(kRows, c1 - c0);
        const auto acc = partial_sums<G>(p, 2 * (int64_t)(wf + c0), n), ml = partial_maxima<G>(p, 2 * (int64_t)(wf + c0), n);
        float m[kRows], l[kRows], f[kRows];
        word a[kRows][kVecs];
#pragma unroll
        for (int j = 0; j < kRows; ++j) {   // (reads past n give zeros)
            const int slot = 2 * j + (j == 0 && c0 == 0);
            const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(ml, h * 8 + slot * (G * 8), 0, apex::kCoherent);
            m[j] = __uint_as_float(v[0]);
            l[j] = __uint_as_float(v[1]);
#pragma unroll
            for (int k = 0; k < kVecs; ++k) {
                const int off = lane * N * 4 + k * 16 + slot * (G * kHeadDim * 4);
                if constexpr (G == 1)
                    a[j][k] = __builtin_amdgcn_raw_buffer_load_b64(acc, off, 0, apex::kCoherent);
                else
                    a[j][k] = __builtin_amdgcn_raw_buffer_load_b128(acc, off, 0, apex::kCoherent);
            }
        }
        join_sums<N, kRows>(m, l, n, r, f);
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) r.num[i] = fmaf(f[j], __uint_as_float(a[j][i / kPer][i % kPer]), r.num[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sh.acc[wave][lane * N + i] = r.num[i];
    if (dim == 0) {
        sh.m[wave][h] = r.M;
        sh.l[wave][h] = r.den;
    }
}

template <int G>
__global__ __launch_bounds__(kThreads, 2) void attention_kernel(Params p)
{
    __shared__ Shared<G> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int w = (int)blockIdx.x;
    Plan plan = make_plan<true>(p, p.Hkv, kPairCost, (unsigned)w, lane);

    Pipe pipe;
    if (plan.way == kWhole) {
        // every wave takes whole pairs and writes their rows itself; the next
        // pair's first blocks are on their way meanwhile
        constexpr int N = 2 * G;
        const int h = lane * N / kHeadDim, dim = lane * N % kHeadDim;
        const int pairs = p.B * p.Hkv;
        struct Pair {
            int b, g, L;
        };
        auto start = [&](int i, Pair& x, Span& s) {
            x.b = uniform((int)((unsigned)i / (unsigned)p.Hkv));
            x.g = i - x.b * p.Hkv;
            x.L = uniform(context(p, x.b));
            s = wave_span(p, x.b, x.g, x.L, 0, (int)blocks(x.L), 0, 1);
            if (s.n > 0) begin<G>(p, x.b, x.g, s, lane, pipe);
        };
        Pair x;
        Span s;
        int i = wave * p.workers + w;
        if (i < pairs) start(i, x, s);
        while (i < pairs) {
            Row<N> r;
            clear(r);
            State st;
            if (s.n > 0) attend<G>(p, s, lane, pipe, st);
            const Pair done = x;
            const bool any = s.n > 0;
            i += kWaves * p.workers;
            if (i < pairs) start(i, x, s);
            if (any) {
                store_state<G>(st, wave, lane, sh);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                r.M = sh.m[wave][h];
                r.den = sh.l[wave][h];
#pragma unroll
                for (int e = 0; e < N; ++e) r.num[e] = sh.acc[wave][lane * N + e];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
            emit_row<N>(p, done.b, done.g * G + h, dim, r);
        }
        return;
    }

    constexpr int N = G == 8 ? 2 : 1;
    const int h = tid * N / kHeadDim, dim = tid * N % kHeadDim;
    const bool emits = h < G;
    bool more = plan.take > 0;
    Span s;
    auto start = [&]() {
        s = wave_span(p, plan.b, plan.g, plan.L, plan.blk, plan.blk + plan.take, wave, kWaves);
        begin<G>(p, plan.b, plan.g, s, lane, pipe);
    };
    if (more) start();
    while (more) {
        const int b = plan.b, g = plan.g, nb = (int)blocks(plan.L);
        State st;
        attend<G>(p, s, lane, pipe, st);
        // the pair's first and last work groups
        int wf = plan.first, wl = plan.last;
        if (plan.way == kLine) {
            wf = plan.blk == 0 ? w : uniform((int)plan.line.owner(plan.vf));
            wl = plan.blk + plan.take == nb ? w : uniform((int)plan.line.owner(plan.vf + (unsigned)nb - 1));
        }
        // the next segment's first blocks are on their way while this one is joined
        more = plan.way == kLine && next_segment(p, p.Hkv, kPairCost, plan);
        if (more) start();
        store_state<G>(st, wave, lane, sh);
        __syncthreads();
        if (emits) {
            Row<N> r;
            join_waves<G, N>(sh, h, dim, r);
            if (wf == wl)
                emit_row<N>(p, b, g * G + h, dim, r);
            else
                store_partial<G, N>(p, partial_slot(w, wf), tid * N, h, dim == 0, r);
        }
        if (wf != wl) {
            // the partials are written with device-coherent stores, complete
            // before the arrival is counted; the last to arrive reads them alike
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            if (tid == 0) {
                int32_t* cnt = &p.counters[(size_t)b * p.Hkv + g];
                const int old = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                const int last = old == wl - wf;
                if (last) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                sh.last = last;
            }
            __syncthreads();
            if (sh.last) {
                const int nc = wl - wf + 1, per = (nc + kWaves - 1) / kWaves;
                join_partials<G>(p, wf, wave * per, min(nc, wave * per + per), wave, lane, sh);
                __syncthreads();
                if (emits) {
                    Row<N> r;
                    join_waves<G, N>(sh, h, dim, r);
                    emit_row<N>(p, b, g * G + h, dim, r);
                }
            }
        }
        if (more) __syncthreads();
    }

    if (plan.empty_rows) {
        for (int b = w; b < p.B; b += (int)gridDim.x) {
            if (context(p, b) > 0) continue;
            Row<1> r;
            clear(r);
            for (int i = tid; i < p.Hq * kHeadDim; i += kThreads) emit_row<1>(p, b, i / kHeadDim, i % kHeadDim, r);
        }
    }
}

// --- accumulated weights ----------------------------------------------------------

// Every block is on its own: its K codes and scales, the scores, and 16 sums over
// the heads.  A wave collects the sums of kChunk blocks in LDS and adds them to
// the weights with one load and one store of all its lanes (four lanes to a
// block): a load and a store for every block, by four lanes each, put a store
// into the wait for every K tile, 37 us against 30 without the stores.
// Bound by HBM: 24 requests of 2048-16384 tokens, 8 kv-heads, G = 8, 143 MB, take 32.1
// us (4.5 TB/s, a fifth of it the weights' reads and writes), 16 of 256-4096 at G = 4
// 9.0.  For the two: 2 work groups a CU 34.1 and 8.7, 4 32.9 and 9.8; 2 tiles on
// their way 34.3 and 9.2, 8 33.0 and 9.9; a pair cost of 4 32.9 and 10.1, of 64 33.2
// and 9.6.
constexpr int kWeightThreads = 256;
constexpr int kWeightWaves = kWeightThreads / 64;
constexpr int kWeightGroupsPerCu = 3;
constexpr unsigned kWeightPairCost = 16;
constexpr int kChunk = 16, kAhead = 4;   // blocks; K tiles on their way

template <int G>
__device__ inline void accumulate(const Params& p, int b, int g, const Span& s, int lane, float* sums)
{
    const int col = lane & 15, q = lane >> 4;
    auto load = [&](Tile& t, unsigned id) { load_keys<apex::kStreamingLoad>(t, slab_of(s, id), lane); };
    // the lane's block of a chunk and its four tokens there
    const int own = lane >> 2, tok = 4 * (lane & 3);
    auto own_id = [&](int k) -> unsigned { return k + own < s.n ? (unsigned)s.bt[k + own] : 0xffffffffu; };
    unsigned lane_id = own_id(0);
    QueryRow row;
    load_row<G>(p, b, g, lane, row);
    Tile t[kAhead];
    unsigned next[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        load(t[i], id_at(s, i));
        next[i] = id_at(s, kAhead + i);
    }
    QueryOperand<G> op;
    split_query<G>(p.q_sign, row, lane, op);
    const int head = G == 8 ? col & 7 : (col & 3) & (G - 1);
    const float lse2 = p.lse_in[(size_t)b * p.Hq + (size_t)g * G + head] * 1.4426950408889634f;
    for (int k = 0; k < s.n; k += kChunk) {
        const bool live = lane_id < s.pool;
        f32x4* const to = (f32x4*)(p.weights + ((uint64_t)(live ? lane_id : 0) * p.Hkv + g) * kBlockSize + tok);
        f32x4 old = {0.f, 0.f, 0.f, 0.f};
        if (live) old = *to;
        lane_id = own_id(k + kChunk);
        // (surplus blocks of the last rounds have no extent, and no lane adds their sums)
#pragma unroll
        for (int j = 0; j < kChunk; j += kAhead) {
            if (k + j >= s.n) break;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                f32x4 w = scores<G>(t[i], op);
                __builtin_amdgcn_sched_barrier(0);
                load(t[i], next[i]);
                next[i] = id_at(s, k + j + 2 * kAhead + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] = apex::exp2_fast(fmaf(w[e], p.scale_log2, -lse2));
                    if (G >= 2) w[e] = add_rotated<0xb1>(w[e]);      // lanes 1, 0, 3, 2
                    if (G >= 4) w[e] = add_rotated<0x4e>(w[e]);      // lanes 2, 3, 0, 1
                    if (G == 8) w[e] = add_rotated<kRor4>(w[e]);
                }
                if (col == 0) *(f32x4*)&sums[(j + i) * kBlockSize + 4 * q] = w;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const f32x4 w = *(const f32x4*)&sums[own * kBlockSize + tok];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (live) {
            const int at = (s.first + k + own) * kBlockSize + tok;
#pragma unroll
            for (int e = 0; e < 4; ++e) old[e] = at + e < s.L ? old[e] + w[e] : old[e];
            *to = old;
        }
    }
}

template <int G>
__global__ __launch_bounds__(kWeightThreads, 3) void weights_kernel(Params p)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    // neighbouring heads of the same blocks on the waves of a work group
    __shared__ __attribute__((aligned(16))) float s_sums[kWeightWaves][kChunk * kBlockSize];
    const int together = p.Hkv % 4 == 0 ? 4 : p.Hkv % 2 == 0 ? 2 : 1;
    const int groups = p.Hkv / together;
    Plan plan = make_plan<false>(p, groups, kWeightPairCost, blockIdx.x, lane);
    bool more = plan.take > 0;
    while (more) {
        const int g = plan.g * together + wave % together;
        const Span s = wave_span(p, plan.b, g, plan.L, plan.blk, plan.blk + plan.take, wave / together, kWeightWaves / together);
        if (s.n > 0) accumulate<G>(p, plan.b, g, s, lane, s_sums[wave]);
        more = next_segment(p, groups, kWeightPairCost, plan);
    }
}

// --- host -------------------------------------------------------------------------

// A workspace: the partials at the size of the widest group, then the arrival
// counters, so that calls of any shapes find the counters where no call leaves
// partials.
size_t counter_bytes(int B, int Hkv) { return kv4::align_up((size_t)B * Hkv * sizeof(int32_t), 256); }

size_t acc_bytes(int workers) { return kv4::align_up(sizeof(float) * 2 * (size_t)workers * 8 * kHeadDim, 256); }

size_t partial_bytes(int workers)
{
    return acc_bytes(workers) + kv4::align_up(sizeof(float) * 4 * (size_t)workers * 8, 256);
}

template <typename F>
void with_group(int G, F f)
{
    switch (G) {
        case 1: f(std::integral_constant<int, 1>()); break;
        case 2: f(std::integral_constant<int, 2>()); break;
        case 4: f(std::integral_constant<int, 4>()); break;
        default: f(std::integral_constant<int, 8>()); break;
    }
}

// (an empty pool or table may be NULL)
int check_pointers(const void* q, const void* cache, int64_t num_blocks, const void* bt, int64_t stride, const void* lens,
                   const void* more, const char* name)
{
    if (!q || (!cache && num_blocks > 0) || (!bt && stride > 0) || !lens || !more)
        return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!kv4::aligned(q, 16) || !kv4::aligned(cache, 16))
        return fail(APEX_ERR_INVALID_ARG, "q and kv_cache must be 16-byte aligned");
    if (!kv4::aligned(bt, 4) || !kv4::aligned(lens, 4))
        return fail(APEX_ERR_INVALID_ARG, "block_table and context_lens must be 4-byte aligned");
    if (!kv4::aligned(more, 16)) return fail(APEX_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
    return APEX_OK;
}

Params fill(const void* q, const void* cache, const int32_t* bt, int64_t stride, const int32_t* lens, int B, int Hq,
            int Hkv, int64_t num_blocks, float scale, int workers)
{
    Params p = Params();
    p.q = (const f16*)q;
    p.cache = (const char*)cache;
    p.bt = bt;
    p.lens = lens;
    p.num_blocks = (unsigned)num_blocks;
    p.stride = (int)stride;
    p.B = B;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.workers = workers;
    p.scale_log2 = __builtin_fabsf(scale) * 1.4426950408889634f;
    p.q_sign = __builtin_signbit(scale) ? 0x8000u : 0u;
    return p;
}

}  // namespace

extern "C" {

size_t apex_kv4_attention_workspace_bytes(int B, int Hq, int Hkv)
{
    apex::clear_error();
    int cus = 0;
    if (kv4::check_batch(B, Hq, Hkv, kHeadDim, kBlockSize, 0, 0) != APEX_OK || kv4::compute_units(&cus) != APEX_OK)
        return 0;
    return partial_bytes(cus) + counter_bytes(B, Hkv);
}

int apex_kv4_attention(const void* q, const void* kv_cache, const int32_t* block_table, int64_t block_table_stride,
                       const int32_t* context_lens, void* out, float* lse_out, int B, int Hq, int Hkv, int d,
                       int block_size, int64_t num_blocks, float scale, void* workspace, size_t workspace_bytes,
                       void* stream)
{
    apex::clear_error();
    int rc = kv4::check_batch(B, Hq, Hkv, d, block_size, num_blocks, block_table_stride);
    if (rc != APEX_OK || B == 0) return rc;
    rc = check_pointers(q, kv_cache, num_blocks, block_table, block_table_stride, context_lens, out, "out");
    if (rc != APEX_OK) return rc;
    if (!kv4::aligned(lse_out, 4)) return fail(APEX_ERR_INVALID_ARG, "lse_out must be 4-byte aligned");
    const size_t qo = (size_t)B * Hq * d * 2;
    const kv4::Extent in[] = {{"q", q, qo},
                              {"kv_cache", kv_cache, kv4::cache_bytes(Hkv, num_blocks)},
                              {"block_table", block_table, (size_t)B * block_table_stride * 4},
                              {"context_lens", context_lens, (size_t)B * 4},
                              {"workspace", workspace, workspace_bytes},
                              {"out", out, qo},
                              {"lse_out", lse_out, (size_t)B * Hq * 4}};
    if ((rc = kv4::check_disjoint(in[4], in, 4)) != APEX_OK || (rc = kv4::check_disjoint(in[5], in, 5)) != APEX_OK ||
        (rc = kv4::check_disjoint(in[6], in, 6)) != APEX_OK)
        return rc;
    int cus = 0;
    rc = kv4::compute_units(&cus);
    if (rc != APEX_OK) return rc;
    const size_t cb = counter_bytes(B, Hkv), pb = partial_bytes(cus);
    void *partials = workspace, *counters = (char*)workspace + pb;
    kv4::Hold hold;
    if (workspace) {
        rc = kv4::check_workspace(workspace, workspace_bytes, pb + cb);
    } else {
        rc = kv4::library_buffer(kv4::kCounters, cb, (hipStream_t)stream, hold, &counters);
        if (rc == APEX_OK) rc = kv4::library_buffer(kv4::kPartials, pb, (hipStream_t)stream, hold, &partials);
    }
    if (rc != APEX_OK) return rc;
    Params p = fill(q, kv_cache, block_table, block_table_stride, context_lens, B, Hq, Hkv, num_blocks, scale, cus);
    p.out = (f16*)out;
    p.lse = lse_out;
    p.counters = (int32_t*)counters;
    p.pacc = (float*)partials;
    p.pml = (float*)((char*)partials + acc_bytes(cus));
    with_group(Hq / Hkv, [&](auto g) {
        attention_kernel<decltype(g)::value><<<(unsigned)cus, kThreads, 0, (hipStream_t)stream>>>(p);
    });
    return kv4::launched("kv4 attention");
}

int apex_kv4_accumulate_weights(const void* q, const void* kv_cache, const int32_t* block_table,
                                int64_t block_table_stride, const int32_t* context_lens, const float* lse,
                                float* weights, int B, int Hq, int Hkv, int d, int block_size, int64_t num_blocks,
                                float scale, void* stream)
{
    apex::clear_error();
    int rc = kv4::check_batch(B, Hq, Hkv, d, block_size, num_blocks, block_table_stride);
    if (rc != APEX_OK || B == 0) return rc;
    if (num_blocks == 0) return APEX_OK;   // no token is in the pool
    rc = check_pointers(q, kv_cache, num_blocks, block_table, block_table_stride, context_lens, weights, "weights");
    if (rc != APEX_OK) return rc;
    if (!lse) return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!kv4::aligned(lse, 4)) return fail(APEX_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    const kv4::Extent in[] = {{"q", q, (size_t)B * Hq * d * 2},
                              {"kv_cache", kv_cache, kv4::cache_bytes(Hkv, num_blocks)},
                              {"block_table", block_table, (size_t)B * block_table_stride * 4},
                              {"context_lens", context_lens, (size_t)B * 4},
                              {"lse", lse, (size_t)B * Hq * 4},
                              {"weights", weights, kv4::slot_bytes(Hkv, num_blocks)}};
    rc = kv4::check_disjoint(in[5], in, 5);
    if (rc != APEX_OK) return rc;
    int cus = 0;
    rc = kv4::compute_units(&cus);
    if (rc != APEX_OK) return rc;
    const int n = cus * kWeightGroupsPerCu;
    Params p = fill(q, kv_cache, block_table, block_table_stride, context_lens, B, Hq, Hkv, num_blocks, scale, n);
    p.lse_in = lse;
    p.weights = weights;
    with_group(Hq / Hkv, [&](auto g) {
        weights_kernel<decltype(g)::value><<<(unsigned)n, kWeightThreads, 0, (hipStream_t)stream>>>(p);
    });
    return kv4::launched("kv4 weights");
}

}  // extern "C"
