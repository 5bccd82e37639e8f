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
// weights go in as two bf16 parts, 16 bits, in columns of their own (G = 8: in
// two passes), while the normaliser sums them unrounded.
#include <type_traits>

#include "kernels.h"
#include "kv4_host.h"

namespace {

using apex::AttnParams;
using apex::f16;
using apex::f32x4;
using apex::kAttnThreads;
using apex::kStageFloats;
using apex::kWaves;
using apex::RowState;
using apex::u32x2;
using apex::u32x4;
using apex::uniform;
using kv4::fail;
using kv4::kBlockSize;
using kv4::kHeadDim;
using kv4::kSlabBytes;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Cost of starting and finishing a pair, in blocks.
constexpr int kPairCost = 24;

struct Kv4Params {
    const char* cache;      // [num_blocks][Hkv][kSlabBytes]
    const int32_t* bt;
    const int32_t* lens;
    int64_t num_blocks;
    int stride;             // entries per table row
    int workers;            // work groups that may get units
    float scale_log2;       // |scale| log2(e)
    unsigned q_sign;        // 0x8000 to negate q (scale < 0)
    const float* lse_in;    // accumulation of the weights: [B][Hq], and
    float* weights;         // [num_blocks][Hkv][16]
};

// --- partition ----------------------------------------------------------------
//
// The line of plan_policy.h: every non-empty (request, kv-head) pair has K cost
// positions, then its blocks; work group w takes positions [start(w),
// start(w + 1)).  Every wave derives it on its own from context_lens: a lane
// sums ceil(B / 64) consecutive requests, one scan joins them.  All positions
// are below 2^31 (the host checks the table's size).

struct Line {
    unsigned V, W, per, rest;   // positions, work groups; V = W per + rest
    __device__ inline unsigned start(unsigned w) const { return w * per + w * rest / W; }   // (w rest < W^2)
    __device__ inline unsigned owner(unsigned v) const
    {
        // w is at most one off the quotient of the reals
        unsigned w = (unsigned)((double)v * (double)W / (double)V);
        if (w >= W) w = W - 1;
        while (w + 1 < W && start(w + 1) <= v) ++w;
        while (start(w) > v) --w;
        return w;
    }
};

struct Plan {
    Line line;
    unsigned v0, v1;        // the work group's positions
    int b, g, blk, L;       // its first segment
    unsigned vf;            // position of the pair's block 0
    bool empty_rows;        // some request has no context
};

__device__ inline int cut_len(const Kv4Params& p, int L)
{
    const int64_t row = (int64_t)p.stride * kBlockSize;
    return L > row ? (int)row : L;
}

__device__ inline unsigned blocks(int L) { return L > 0 ? ((unsigned)L + kBlockSize - 1) / kBlockSize : 0u; }

__device__ inline Plan make_plan(const Kv4Params& p, int B, int Hkv, unsigned K, unsigned w, int lane)
{
    const int R = (B + 63) / 64;
    const int r0 = min(B, lane * R), r1 = min(B, r0 + R);
    unsigned cost = 0, count = 0;
    for (int b = r0; b < r1; ++b) {
        const unsigned nb = blocks(cut_len(p, p.lens[b]));
        count += nb > 0;
        cost += nb > 0 ? nb + K : 0u;
    }
    const unsigned hk = (unsigned)Hkv;
    const unsigned hi = (unsigned)apex::wave_incl_sum((int)cost), lo = hi - cost;
    const unsigned total = (unsigned)apex::lane_value((int)hi, 63);
    const unsigned nonempty = (unsigned)apex::lane_value(apex::wave_incl_sum((int)count), 63);
    Plan r;
    r.empty_rows = nonempty < (unsigned)B;
    r.v0 = r.v1 = r.vf = 0;
    r.b = r.g = r.blk = r.L = 0;
    const unsigned V = total * hk, pairs = nonempty * hk, U = V - K * pairs;
    unsigned W = U / 8;   // at least two blocks a wave
    W = W < pairs ? pairs : W;
    W = W < (unsigned)p.workers ? W : (unsigned)p.workers;
    r.line.V = V;
    r.line.W = W;
    if (V == 0 || w >= W) return r;
    r.line.per = V / W;
    r.line.rest = V - r.line.per * W;
    r.v0 = r.line.start(w);
    r.v1 = r.line.start(w + 1);
    // the lane whose requests hold v0, then the request
    const uint64_t hit = __ballot(lo * hk <= r.v0 && r.v0 < hi * hk);
    const int ln = __builtin_ctzll(hit);
    unsigned at = (unsigned)apex::lane_value((int)lo, ln) * hk;
    int b = ln * R;
    unsigned nb;
    while (true) {
        r.L = uniform(cut_len(p, p.lens[b]));
        nb = blocks(r.L);
        const unsigned span = nb > 0 ? (nb + K) * hk : 0u;
        if (r.v0 < at + span) break;
        at += span;
        ++b;
    }
    r.b = b;
    const unsigned off = r.v0 - at, len = nb + K;
    r.g = (int)(off / len);
    r.vf = at + (unsigned)r.g * len + K;
    r.blk = r.v0 > r.vf ? (int)(r.v0 - r.vf) : 0;
    return r;
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

template <int G>
__device__ inline void load_query(const AttnParams& p, unsigned q_sign, int b, int g, int lane, QueryOperand<G>& op)
{
    const int col = lane & 15, q = lane >> 4;
    const int head = G == 8 ? col & 7 : (col & 3) & (G - 1);
    const f16* row = p.q + ((size_t)b * p.Hq + (size_t)g * G + head) * kHeadDim + 16 * q;
    u32x4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = *(const u32x4*)(row + (i >> 1) * 64 + (i & 1) * 8);
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

template <bool kValues>
__device__ inline void load_tile(Tile& t, const char* slab, int bytes, int lane)
{
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)apex::uniform_ptr(slab), (short)0, bytes,
                                                                       apex::kRawBufferWord3);
    const int c = lane & 15, q = lane >> 4;
    t.k = __builtin_amdgcn_raw_buffer_load_b128(r, c * 64 + q * 16, 0, apex::kStreamingLoad);
    t.ks = __builtin_amdgcn_raw_buffer_load_b8(r, kv4::kKScales + c * 4 + q, 0, apex::kStreamingLoad);
    if (kValues) {
        t.v = __builtin_amdgcn_raw_buffer_load_b128(r, kv4::kVCodes + lane * 16, 0, apex::kStreamingLoad);
        t.vs = __builtin_amdgcn_raw_buffer_load_b32(r, kv4::kVScales + (c >> 2) * 16 + q * 4, 0, apex::kStreamingLoad);
    }
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
    int first, n;
    int L;
};

__device__ inline Span wave_span(const Kv4Params& p, int b, int g, int L, int lo, int hi, int wave)
{
    Span s;
    const int per = (hi - lo + kWaves - 1) / kWaves;
    s.first = uniform(lo + wave * per);
    s.n = uniform(max(0, min(hi, s.first + per) - s.first));
    s.bt = p.bt + (size_t)uniform(b) * (size_t)p.stride + (s.n > 0 ? s.first : 0);
    s.pair = apex::uniform_ptr(p.cache + (size_t)uniform(g) * kSlabBytes);
    s.L = uniform(L);
    return s;
}

constexpr int kDepth = 4;   // blocks in flight per wave

template <int G>
__device__ inline void attend(const Kv4Params& p, int Hkv, const Span& s, const QueryOperand<G>& op, int lane, State& st)
{
    const int col = lane & 15, q = lane >> 4;
    const int parity = G == 8 ? col >> 3 : (col >> 2) & 1;
    // bytes 2 and 3 of a weight to the half of its parity, zeros to the other
    const unsigned place = parity ? 0x03020c0cu : 0x0c0c0302u;
    const unsigned low_part = G < 8 && col >= 8 ? 0xffff0000u : 0u;
    const uint64_t step = (uint64_t)Hkv * kSlabBytes;

    auto id_at = [&](int i) -> int {
        return i < s.n ? *(const __attribute__((address_space(4))) int32_t*)(s.bt + i) : -1;
    };
    auto ok = [&](int id) -> bool { return id >= 0 && (int64_t)id < p.num_blocks; };
    auto load = [&](Tile& t, int id) {
        const bool good = ok(id);
        load_tile<true>(t, s.pair + (good ? (uint64_t)(uint32_t)id * step : 0), good ? kSlabBytes : 0, lane);
    };
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) st.acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};

    Tile tile[kDepth];
    int id[kDepth], next[kDepth];
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
        id[i] = id_at(i);
        load(tile[i], id[i]);
        next[i] = id_at(kDepth + i);
    }

    auto block = [&](Tile& t, int k, int& id, int& next) {
        const bool good = ok(id);
        const int tok = (s.first + k) * kBlockSize + 4 * q;
        const bool tail = !good || (s.first + k) * kBlockSize > s.L - kBlockSize;
        f32x4 sc = scores<G>(t, op);
        const u32x4 v = t.v;
        const unsigned vs = t.vs;
        id = next;
        next = id_at(k + 2 * kDepth);
        float vscale[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            vscale[e] = __uint_as_float((e == 0 ? vs << 23 : e == 1 ? vs << 15 : e == 2 ? vs << 7 : vs >> 1) & 0x7f800000u);
        }
        bool live[4];
        if (tail) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                live[e] = good && tok + e < s.L;
                sc[e] = live[e] ? sc[e] : -INFINITY;
                vscale[e] = live[e] ? vscale[e] : 1.f;   // (an unused slot may hold a NaN scale)
            }
        }
        const float bm = apex::rows_max4(fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])));
        const float m = fmaxf(st.m, bm * p.scale_log2);
        const float ms = m == -INFINITY ? 0.f : m;   // no token so far
        const float alpha = apex::exp2_fast(st.m - ms);
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = apex::exp2_fast(fmaf(sc[e], p.scale_log2, -ms));
        if (tail) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = live[e] ? w[e] : 0.f;   // (a scale of 0 makes -inf a NaN)
        }
        st.l = fmaf(st.l, alpha, (w[0] + w[1]) + (w[2] + w[3]));
        st.m = m;
        if (alpha != 1.f) {
#pragma unroll
            for (int j = 0; j < 4; ++j) st.acc[j] *= alpha;
        }
        // weights as operand words
        u32x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned u = __float_as_uint(w[e]);
            if (G < 8) {
                const unsigned part = __float_as_uint(w[e] - __uint_as_float(u & low_part));
                hi[e] = __builtin_amdgcn_perm(0u, part, place);
            } else {
                hi[e] = __builtin_amdgcn_perm(0u, u, place);
                lo[e] = __builtin_amdgcn_perm(0u, __float_as_uint(w[e] - __uint_as_float(u & 0xffff0000u)), place);
            }
        }
        u32x4 a[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[0][e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[e], vscale[e], 0));
            a[1][e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[e], vscale[e], 1));
            a[2][e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[e], vscale[e], 2));
            a[3][e] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v[e], vscale[e], 3));
        }
        // the tile is consumed
        __builtin_amdgcn_sched_barrier(0);
        load(t, id);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            st.acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[j]),
                                                                __builtin_bit_cast(bf16x8, hi), st.acc[j], 0, 0, 0);
        if (G == 8) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                st.acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[j]),
                                                                    __builtin_bit_cast(bf16x8, lo), st.acc[j], 0, 0, 0);
        }
    };
    for (int k = 0; k < s.n; k += kDepth) {
#pragma unroll
        for (int i = 0; i < kDepth; ++i)
            if (k + i < s.n) block(tile[i], k + i, id[i], next[i]);
    }
    st.l = apex::rows_sum4(st.l);
}

// A wave's state into LDS, [head][dim], to be merged with the other waves'.
template <int G>
__device__ inline void store_state(State& st, int wave, int lane, float (*s_acc)[kStageFloats], float (*s_m)[G],
                                   float (*s_l)[G])
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
            for (int j = 0; j < 4; ++j) s_acc[wave][head * kHeadDim + 8 * (4 * q + i) + 2 * j + parity] = st.acc[j][i];
    }
    if (col < G && q == 0) {
        s_m[wave][col] = st.m;
        s_l[wave][col] = st.l;
    }
}

// Rows of the pair's heads: zeros and -inf where there was no token; NaNs stay.
// The cache can hold 65536 (65504 rounded up), whose half would be infinite: a
// larger result than 65504 becomes that.
template <int N>
__device__ inline void emit_row(const AttnParams& p, int b, int head, int dim, const RowState<N>& r)
{
    typename apex::vec_of<f16, N>::type o;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = r.den == 0.f ? 0.f : r.num[i] / r.den;
        o[i] = (f16)(__builtin_fabsf(x) > 65504.f ? __builtin_copysignf(65504.f, x) : x);
    }
    *(typename apex::vec_of<f16, N>::type*)&p.out[((size_t)b * p.Hq + head) * kHeadDim + dim] = o;
    if (p.lse && dim == 0)
        p.lse[(size_t)b * p.Hq + head] = r.den == 0.f ? -INFINITY : (r.M + __log2f(r.den)) * 0.69314718055994531f;
}

// Walks the work group's segments: f(b, g, L, nb, blk, take, vf) for each.
template <typename F>
__device__ inline void for_segments(const Kv4Params& p, int B, int Hkv, unsigned K, const Plan& plan, F f)
{
    int b = plan.b, g = plan.g, blk = plan.blk, L = plan.L;
    unsigned vf = plan.vf;
    while (vf + (unsigned)blk < plan.v1) {
        const int nb = (int)blocks(L);
        const int take = (int)min((unsigned)(nb - blk), plan.v1 - (vf + (unsigned)blk));
        f(b, g, L, nb, blk, take, vf);
        if (blk + take < nb) return;
        vf += (unsigned)nb + K;
        blk = 0;
        if (++g == Hkv) {
            g = 0;
            do {
                if (++b >= B) return;
                L = uniform(cut_len(p, p.lens[b]));
            } while (L <= 0);
        }
    }
}

template <int G>
__global__ __launch_bounds__(kAttnThreads) void attention_kernel(AttnParams p, Kv4Params kp)
{
    __shared__ __align__(16) float s_acc[kWaves][kStageFloats];
    __shared__ float s_m[kWaves][G];
    __shared__ float s_l[kWaves][G];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const unsigned w = blockIdx.x;
    const Plan plan = make_plan(kp, p.B, p.Hkv, kPairCost, w, lane);
    constexpr int N = apex::kEmitElems<G>;
    const int h = tid * N / kHeadDim, dim = tid * N % kHeadDim;
    const bool emits = G >= 2 || tid < kHeadDim;

    for_segments(kp, p.B, p.Hkv, kPairCost, plan, [&](int b, int g, int L, int nb, int blk, int take, unsigned vf) {
        {
            QueryOperand<G> op;
            load_query<G>(p, kp.q_sign, b, g, lane, op);
            State st;
            attend<G>(kp, p.Hkv, wave_span(kp, b, g, L, blk, blk + take, wave), op, lane, st);
            store_state<G>(st, wave, lane, s_acc, s_m, s_l);
        }
        __syncthreads();
        // the pair's first and last work groups
        const int wf = blk == 0 ? (int)w : uniform((int)plan.line.owner(vf));
        const int wl = blk + take == nb ? (int)w : uniform((int)plan.line.owner(vf + (unsigned)nb - 1));
        if (emits) {
            const RowState<N> r = apex::merge_waves<G, N>(s_acc, s_m, s_l, h, dim);
            if (wf == wl)
                emit_row<N>(p, b, g * G + h, dim, r);
            else
                apex::store_partial<G, N>(p, apex::partial_slot(w, wf), tid * N, h, dim == 0, r);
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
                s_last = last;
            }
            __syncthreads();
            if (s_last) {
                const int nc = wl - wf + 1, per = (nc + kWaves - 1) / kWaves;
                const int c0 = wave * per;
                apex::combine_wave<G>(p, wf, c0, c0 + per < nc ? c0 + per : nc, wave, lane, s_acc, s_m, s_l);
                __syncthreads();
                if (emits) emit_row<N>(p, b, g * G + h, dim, apex::merge_waves<G, N>(s_acc, s_m, s_l, h, dim));
            }
        }
        __syncthreads();
    });

    if (plan.empty_rows) {
        for (int b = (int)w; b < p.B; b += (int)gridDim.x) {
            if (cut_len(kp, kp.lens[b]) > 0) continue;
            RowState<1> r;
            r.M = 0.f;
            r.den = 0.f;
            r.num = 0.f;
            for (int i = tid; i < p.Hq * kHeadDim; i += kAttnThreads)
                emit_row<1>(p, b, i / kHeadDim, i % kHeadDim, r);
        }
    }
}

// --- accumulated weights ----------------------------------------------------------

// Every block is on its own: its K codes and scales, the scores, the weights of
// 16 tokens added up over the heads, 64 bytes read and written.
template <int G>
__global__ __launch_bounds__(kAttnThreads) void weights_kernel(AttnParams p, Kv4Params kp)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int col = lane & 15, q = lane >> 4;
    const Plan plan = make_plan(kp, p.B, p.Hkv, kPairCost, blockIdx.x, lane);
    const uint64_t step = (uint64_t)p.Hkv * kSlabBytes;

    for_segments(kp, p.B, p.Hkv, kPairCost, plan, [&](int b, int g, int L, int, int blk, int take, unsigned) {
        QueryOperand<G> op;
        load_query<G>(p, kp.q_sign, b, g, lane, op);
        const int head = G == 8 ? col & 7 : (col & 3) & (G - 1);
        const float lse2 = kp.lse_in[(size_t)b * p.Hq + (size_t)g * G + head] * 1.4426950408889634f;
        const Span s = wave_span(kp, b, g, L, blk, blk + take, wave);
        for (int k = 0; k < s.n; ++k) {
            const int id = uniform(s.bt[k]);
            if (id < 0 || (int64_t)id >= kp.num_blocks) continue;
            Tile t;
            load_tile<false>(t, s.pair + (uint64_t)(uint32_t)id * step, kSlabBytes, lane);
            const f32x4 sc = scores<G>(t, op);
            f32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = apex::exp2_fast(fmaf(sc[e], kp.scale_log2, -lse2));
                if (G >= 2) x = add_rotated<0xb1>(x);      // lanes 1, 0, 3, 2
                if (G >= 4) x = add_rotated<0x4e>(x);      // lanes 2, 3, 0, 1
                if (G == 8) x = add_rotated<kRor4>(x);
                w[e] = x;
            }
            if (col == 0) {
                const int tok = (s.first + k) * kBlockSize + 4 * q;
                f32x4* to = (f32x4*)(kp.weights + ((uint64_t)(uint32_t)id * p.Hkv + g) * kBlockSize + 4 * q);
                f32x4 old = *to;
#pragma unroll
                for (int e = 0; e < 4; ++e) old[e] = tok + e < s.L ? old[e] + w[e] : old[e];
                *to = old;
            }
        }
    });
}

// --- host -------------------------------------------------------------------------

constexpr int kGroupsPerCu = 4;

int workers(int64_t* out)
{
    int cus = 0;
    const int rc = kv4::compute_units(&cus);
    *out = (int64_t)cus * kGroupsPerCu;
    return rc;
}

size_t counter_bytes(int B, int Hkv) { return kv4::align_up((size_t)B * Hkv * sizeof(int32_t), 256); }

size_t acc_bytes(int64_t workers, int G)
{
    return kv4::align_up(sizeof(float) * 2 * (size_t)workers * G * kHeadDim, 256);
}

size_t partial_bytes(int64_t workers, int G)
{
    return acc_bytes(workers, G) + kv4::align_up(sizeof(float) * 4 * (size_t)workers * G, 256);
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

int check_pointers(const void* q, const void* cache, const void* bt, const void* lens, const void* more, const char* name,
                   size_t align)
{
    if (!q || !cache || !bt || !lens || !more) return fail(APEX_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!kv4::aligned(q, 16) || !kv4::aligned(cache, 16))
        return fail(APEX_ERR_INVALID_ARG, "q and kv_cache must be 16-byte aligned");
    if (!kv4::aligned(bt, 4) || !kv4::aligned(lens, 4))
        return fail(APEX_ERR_INVALID_ARG, "block_table and context_lens must be 4-byte aligned");
    if (!kv4::aligned(more, align)) return fail(APEX_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
    return APEX_OK;
}

void fill(AttnParams& p, Kv4Params& kp, const void* q, const void* cache, const int32_t* bt, int64_t stride,
          const int32_t* lens, int B, int Hq, int Hkv, int64_t num_blocks, float scale, int64_t workers)
{
    p = AttnParams();
    p.q = (const f16*)q;
    p.B = B;
    p.Hq = Hq;
    p.Hkv = Hkv;
    kp = Kv4Params();
    kp.cache = (const char*)cache;
    kp.bt = bt;
    kp.lens = lens;
    kp.num_blocks = num_blocks;
    kp.stride = (int)stride;
    kp.workers = (int)workers;
    kp.scale_log2 = __builtin_fabsf(scale) * 1.4426950408889634f;
    kp.q_sign = __builtin_signbit(scale) ? 0x8000u : 0u;
}

}  // namespace

extern "C" {

size_t apex_kv4_attention_counter_bytes(int B, int Hkv)
{
    apex::clear_error();
    if (B < 0 || Hkv <= 0) {
        fail(APEX_ERR_INVALID_ARG, "B = %d or Hkv = %d", B, Hkv);
        return 0;
    }
    return counter_bytes(B, Hkv);
}

size_t apex_kv4_attention_workspace_bytes(int B, int Hq, int Hkv)
{
    apex::clear_error();
    int64_t n = 0;
    if (kv4::check_batch(B, Hq, Hkv, kHeadDim, kBlockSize, 0, 0) != APEX_OK || workers(&n) != APEX_OK) return 0;
    return counter_bytes(B, Hkv) + partial_bytes(n, Hq / Hkv);
}

int apex_kv4_attention(const void* q, const void* kv_cache, const int32_t* block_table, int64_t block_table_stride,
                       const int32_t* context_lens, void* out, float* lse_out, int B, int Hq, int Hkv, int d,
                       int block_size, int64_t num_blocks, float scale, void* workspace, size_t workspace_bytes,
                       void* stream)
{
    apex::clear_error();
    int rc = kv4::check_batch(B, Hq, Hkv, d, block_size, num_blocks, block_table_stride);
    if (rc != APEX_OK || B == 0) return rc;
    rc = check_pointers(q, kv_cache, block_table, context_lens, out, "out", 16);
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
    int64_t n = 0;
    rc = workers(&n);
    if (rc != APEX_OK) return rc;
    const int G = Hq / Hkv;
    const size_t cb = counter_bytes(B, Hkv), pb = partial_bytes(n, G);
    void *counters = workspace, *partials = (char*)workspace + cb;
    if (workspace) {
        rc = kv4::check_workspace(workspace, workspace_bytes, cb + pb);
    } else {
        rc = kv4::library_buffer(kv4::kCounters, cb, (hipStream_t)stream, &counters);
        if (rc == APEX_OK) rc = kv4::library_buffer(kv4::kPartials, pb, (hipStream_t)stream, &partials);
    }
    if (rc != APEX_OK) return rc;
    AttnParams p;
    Kv4Params kp;
    fill(p, kp, q, kv_cache, block_table, block_table_stride, context_lens, B, Hq, Hkv, num_blocks, scale, n);
    p.out = (f16*)out;
    p.lse = lse_out;
    p.counters = (int32_t*)counters;
    p.pacc = (float*)partials;
    p.pml = (float*)((char*)partials + acc_bytes(n, G));
    with_group(G, [&](auto g) {
        attention_kernel<decltype(g)::value><<<(unsigned)n, kAttnThreads, 0, (hipStream_t)stream>>>(p, kp);
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
    rc = check_pointers(q, kv_cache, block_table, context_lens, weights, "weights", 16);
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
    int64_t n = 0;
    rc = workers(&n);
    if (rc != APEX_OK) return rc;
    AttnParams p;
    Kv4Params kp;
    fill(p, kp, q, kv_cache, block_table, block_table_stride, context_lens, B, Hq, Hkv, num_blocks, scale, n);
    kp.lse_in = lse;
    kp.weights = weights;
    with_group(Hq / Hkv, [&](auto g) {
        weights_kernel<decltype(g)::value><<<(unsigned)n, kAttnThreads, 0, (hipStream_t)stream>>>(p, kp);
    });
    return kv4::launched("kv4 weights");
}

}  // extern "C"
