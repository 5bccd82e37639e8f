// attend_tile.h -- one wave's part of an attention: 32 query rows against tiles
// of keys that lie in LDS.
//
// A wave keeps 32 rows of q and their 32 x 128 sums in registers and takes the
// keys as they come, with the running maximum and sum of a softmax in one pass:
//     S^T = K Q^T          (keys down, queries across: v_mfma_f32_32x32x16_f16)
//     p   = 2^(c s - M)    (c = |scale| log2 e, M at most 2^kSlack below the row's maximum)
//     O^T += V^T P^T
// Transposed, a query is a lane's column in all three products: its maximum,
// sum and rescaling need no broadcast, only one exchange between the wave's
// halves (lanes n and n + 32 hold the same query's other keys).  The weights
// leave S^T in the order in which P^T takes them, but for the naming of the 16
// keys of a step; V^T is read in that naming too, so they stay where they are.
//
// Rounding: scores, maxima, sums and O are fp32.  The weights enter the second
// product as fp16, 2^kBias times what the softmax defines or more.
//   Prompts: one part, off by up to 2^-11 of a weight, at random, which the output's own
//   rounding to fp16 matches; below 2^-25 of the row's largest weight, among fp16's
//   subnormal numbers, by up to 2^-36 of the largest (2^-(25 + kBias)).  Against 64
//   bits the results are off by 2.3e-4 to 2.6e-4 relative, with fp32 weights 1.8e-4 to
//   2.1e-4.  A second part is half as many products again where products are what
//   takes the time: 8.2 ms would be 11.1 for 32768 tokens, 84 us 100 for a chat batch.
//   Trees (kFine): two parts, as the decode attention has them, since a drafted token's
//   row is to be what a decode step would give; off by up to 2^-21 of a weight, and by
//   2^-36 of the largest.  What is left is the output's own rounding.  Where the cache's
//   bytes are what takes the time it is free: up to 32 rows a pair 0-2 % (32 long
//   contexts 284 us either way), 64 rows 1-3 %; 128 rows cost 7-14 % (a chat batch 51.8
//   us and 56.1), 256 rows 9-20 %.
//
// What bounds it: the instructions of a wave.  64 keys are 32 matrix products, 1024
// cycles (48 with weights in two parts), and the conversions, maxima and exponentials of 2048 weights, which depend
// on the first half of the products and feed the second: a wave's own do not overlap
// much, so two waves of a SIMD have to fill each other's gaps.  Eight waves take a
// tile in 1.7 to 2.0 us, the matrix cores busy 53 % of it.  LDS has next to no bank conflicts.
// Other orders were measured and left: the products of the next 32 keys between the
// weights of these (5-10 % slower), half of the waves a phase behind the others
// (1-3 %), priorities around the products (0-1.5 %), two row tiles a wave with one
// wave a SIMD (132 us for 96 of a batch of trees).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace steps __attribute__((visibility("hidden"))) {

constexpr int kHeadDim = 128;
constexpr int kBlockSize = 16;
constexpr int kWaveRows = 32;      // query rows of a wave
constexpr int kRowBytes = kHeadDim * 2;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// M follows the running maximum only when that has passed it by 2^kSlack: the
// sums are rescaled on few tiles.  2^(kBias + kSlack) is an fp16 value.  A larger bias
// keeps more of small weights and rescales more often: 7 and 8, 11 and 4, 13 and 2, 14
// and 1 take 84.2, 84.4, 85.9, 87.3 us for a chat batch of prompts, 8.23, 8.19, 8.25, 8.31
// ms for 32768 tokens.
constexpr float kSlack = 4.0f;
constexpr float kBias = 11.0f;
// From here on c s and M are too coarse for 2^(c s - M) in one rounding, see nearer.
constexpr float kFar = 1048576.0f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) f16x8 lds_f16x8;
typedef __attribute__((address_space(3))) f16x4 lds_f16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
typedef __attribute__((address_space(3))) f32x2 lds_f32x2;

// Where 16-byte piece c of a key's row lies among the row's 16 pieces.  K is
// read with 32 neighbouring keys at one piece each: their pieces are spread over
// all banks.  V is read, transposed, as 4 neighbouring keys at four pieces each
// (64 bytes): each key's go to another quarter.
__device__ inline unsigned k_piece(unsigned key, unsigned c) { return c ^ (key & 15); }
__device__ inline unsigned v_piece(unsigned key, unsigned c) { return c ^ ((key & 3) << 2); }

// x of this lane and of the lane 32 away, in either order.
__device__ inline u32x2 both_halves(float x)
{
    const unsigned u = __float_as_uint(x);
    return __builtin_amdgcn_permlane32_swap(u, u, false, false);
}

__device__ inline float max_of_halves(float x)
{
    const u32x2 r = both_halves(x);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ inline float sum_of_halves(float x)
{
    const u32x2 r = both_halves(x);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The lane, computed anew: what hangs on it does not stay in registers from one
// use to the next.
__device__ inline unsigned lane_again()
{
    unsigned x = threadIdx.x & 63;
    asm volatile("" : "+v"(x));
    return x;
}

// A row of zeros, for rows that are not there.
__device__ __attribute__((aligned(16))) const unsigned int kZeros[kRowBytes / 4] = {0};

// 16 bytes of every lane from global memory to LDS, lane i's to `to` + 16 i (`to`
// the same in all lanes), past the registers; done when the wave has waited for
// its loads (arrived).
__device__ inline void load_to_lds(const char* from, unsigned to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane((int)to)), "v"(from) : "memory");
}

// The same from one address in all lanes and an offset of each.
__device__ inline void load_to_lds(const char* from, unsigned offset, unsigned to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane((int)to)),
                 "v"(offset), "s"(from) : "memory");
}

// The same, past the caches: what is read once (a batch of 32 long contexts: 282
// us, 315 by way of them).
__device__ inline void stream_to_lds(const char* from, unsigned offset, unsigned to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(__builtin_amdgcn_readfirstlane((int)to)),
                 "v"(offset), "s"(from) : "memory");
}

// Waits until all but the last n of the wave's loads have arrived and what it has
// read from LDS is there.
template <int n>
__device__ inline void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(n) : "memory");
}

// Waits until what the wave has read from LDS is there: loads may overwrite it.
__device__ inline void was_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Waits for the work group; LDS before it is LDS behind it.
__device__ inline void barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ inline unsigned lds_address(const lds_char* p) { return (unsigned)(uintptr_t)p; }

// One wave's 32 rows; kSub tiles of 32 keys are taken at a time.  kFine: the weights go
// in as two fp16 parts.
template <int kSub, bool kFine>
struct Rows {
    f16x8 q[8];          // lane n and n + 32: row n, dims 16 j + 8 (lane / 32) + 0..7 in q[j]
    f32x16 o[4];         // O^T, dims 32 t + 8 (i / 4) + 4 (lane / 32) + i % 4 in o[t][i], times 2^kBias
    float top;           // M
    float sum;           // of this lane's half of the keys
    bool far;            // M of some row of the wave's is kFar or more in magnitude

    // Row pointer of the lane's query, or NULL: a row of zeros.
    __device__ void start(const char* row)
    {
        const unsigned half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u32x4 x = {0u, 0u, 0u, 0u};
            if (row) x = *(const u32x4*)(row + j * 32 + half * 16);
            q[j] = __builtin_bit_cast(f16x8, x);
        }
    }

    // The lane's query out of rows in LDS that lie as K's.
    __device__ void read_q(const lds_char* rows)
    {
        const unsigned lane = lane_again(), row = lane & 31, half = lane >> 5;
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = *(const lds_f16x8*)(rows + row * kRowBytes + k_piece(row, 2 * j + half) * 16);
    }

    // The scale's sign, see QScale.
    __device__ void times(_Float16 sign)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] *= sign;
    }

    __device__ void clear()
    {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
        top = -INFINITY;
        sum = 0.0f;
        far = false;
    }

    // Scores of the tiles' keys: key 32 u + 8 (i / 4) + 4 (lane / 32) + i % 4 in s[u][i].
    __device__ void scores(const lds_char* k, f32x16 (&s)[kSub]) const
    {
        const unsigned lane = threadIdx.x & 63, key = lane & 31, half = lane >> 5;
        f16x8 a[kSub][8];
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                a[u][j] = *(const lds_f16x8*)(k + (key + 32 * u) * kRowBytes + k_piece(key, 2 * j + half) * 16);
        __builtin_amdgcn_sched_barrier(0);      // all reads are on their way before the first product waits
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int u = 0; u < kSub; ++u)
                s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[u][j], q[j], s[u], 0, 0, 0);
    }

    // Takes out the scores of keys that the lane's query does not see: bit j of
    // `allow` stands for key j.
    __device__ static void mask(f32x16 (&s)[kSub], uint64_t allow)
    {
        const unsigned half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const uint32_t bits = (uint32_t)(allow >> (32 * u)) >> (4 * half);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[u][i] = (bits >> (8 * (i / 4) + i % 4)) & 1 ? s[u][i] : -INFINITY;
        }
    }

    // The running maximum after these scores.
    __device__ void raise(const f32x16 (&s)[kSub], float c)
    {
        float m[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};      // four chains
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int i = u ? 0 : 4; i < 16; ++i) m[i & 3] = fmaxf(m[i & 3], s[u][i]);
        const float most = max_of_halves(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]))) * c;
        if (__builtin_expect(__any(most > top + kSlack), 0)) rescale(fmaxf(most, top));
    }

    // Weights of 32 keys' scores, as P^T's operands: keys 16 w + 4 half + 0..3 and + 8 in p[w].
    // kFine: p rounds towards 0, and `rest` has what is left.
    __device__ void weights(const f32x16& s, float c, float base, f16x8* p, f16x8* rest)
    {
        float part[2] = {0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                f32x2 e;
                e[0] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * w + j], c, -base));
                e[1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * w + j + 1], c, -base));
                part[0] += e[0];
                part[1] += e[1];
                f16x2 h = __builtin_convertvector(e, f16x2);
                if (kFine) {
                    h = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(e[0], e[1]));
                    const f32x2 d = {__builtin_fmaf((float)h[0], -1.0f, e[0]), __builtin_fmaf((float)h[1], -1.0f, e[1])};
                    const f16x2 l = __builtin_convertvector(d, f16x2);
                    rest[w][j] = l[0];
                    rest[w][j + 1] = l[1];
                }
                p[w][j] = h[0];
                p[w][j + 1] = h[1];
            }
        sum += part[0] + part[1];
    }

    __device__ void rescale(float to)
    {
        const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - to);
        sum *= f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] *= f;
        top = to;
        far = __any(fabsf(to) >= kFar && to != -INFINITY);
    }

    // M to take scores from: a row that has seen none yet keeps M = -inf, and 2^(-inf - 0)
    // is 0.
    __device__ float from() const { return top == -INFINITY ? 0.0f : top; }

    // Scores as their distance from M.  M is c times a score, rounded: c s - M in one
    // rounding is off by as much, and far from 0 that is whole powers of 2, so that the
    // largest weight itself would overflow or vanish.  With c s rounded as M was it is 0.
    __device__ void nearer(f32x16 (&s)[kSub], float c) const
    {
#pragma clang fp contract(off)
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = s[u][i] * c - from();
    }

    // V^T's operand: dims 32 t + lane % 32, the 16 keys of step w in P^T's order.
    __device__ static f16x8 v_operand(const lds_char* v, int w, int t)
    {
        const unsigned lane = threadIdx.x & 63, half = lane >> 5, in = lane & 15;
        const unsigned key = 4 * half + (in >> 2), quarter = (unsigned)t ^ (in >> 2);
        const unsigned at = key * kRowBytes + quarter * 64 + ((lane >> 4) & 1) * 32 + (in & 3) * 8;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v + at + w * 16 * kRowBytes));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v + at + (w * 16 + 8) * kRowBytes));
        return __builtin_bit_cast(f16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }

    // The operands of 32 keys, two steps.
    __device__ static void read_v(const lds_char* v, int u, f16x8 (&a)[2][4])
    {
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int t = 0; t < 4; ++t) a[w][t] = v_operand(v, 2 * u + w, t);
        __builtin_amdgcn_sched_barrier(0);
    }

    __device__ void add(const f16x8 (&a)[2][4], const f16x8* p)
    {
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int t = 0; t < 4; ++t) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[w][t], p[w], o[t], 0, 0, 0);
    }

    // False if a unit's values hold an infinity or a NaN.  A masked key has the weight
    // 0, but 0 x NaN is NaN: where rows differ in what they see, a row's last 64 keys at
    // most, a unit that is not finite is taken key by key (take_key).  Everywhere else
    // an infinity or a NaN is the rows' own.
    __device__ static bool finite(const lds_char* v)
    {
        const unsigned lane = lane_again();
        const f16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
        f16x8 x = zero;
#pragma unroll
        for (int i = 0; i < 8 * kSub; ++i) x = __builtin_elementwise_fma(*(const lds_f16x8*)(v + (i * 64 + lane) * 16), zero, x);
        const u32x4 bits = __builtin_bit_cast(u32x4, x);        // 0 x finite + 0 is +0
        return !__any((bits[0] | bits[1] | bits[2] | bits[3]) != 0);
    }

    // The weights of a unit's scores and their products with V: V's operands come
    // while weights are made, and the weights of 32 keys are made while the matrix
    // cores work on the 32 before them.  `half`: none of the second 32 is seen.
    __device__ void take(f32x16 (&s)[kSub], float c, const lds_char* v, bool half = false)
    {
        float base = 0.0f;
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            if (u && half) break;
            f16x8 a[2][4];
            read_v(v, u, a);
            if (u == 0) {
                raise(s, c);
                base = from() - kBias;
                if (__builtin_expect(far, 0)) {
                    nearer(s, c);
                    c = 1.0f;
                    base = -kBias;
                }
            }
            f16x8 p[2], rest[2];
            weights(s[u], c, base, p, rest);
            add(a, p);
            if (kFine) add(a, rest);
        }
    }

    // One key, by its rows in global memory (this kv-head's), for the queries that see it.
    __device__ void take_key(const char* k, const char* v, float c, bool sees)
    {
        const unsigned half = (threadIdx.x & 63) >> 5;
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const f16x8 x = *(const f16x8*)(k + j * 32 + half * 16);
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                dot = __builtin_amdgcn_fdot2(f16x2{x[i], x[i + 1]}, f16x2{q[j][i], q[j][i + 1]}, dot, false);
            asm volatile("" ::: "memory");      // one load at a time: this path may not cost the other registers
        }
        dot = sum_of_halves(dot);
        float at;
        {
#pragma clang fp contract(off)
            const float m = sees ? dot * c : -INFINITY;
            if (__any(m > top + kSlack)) rescale(fmaxf(m, top));
            at = m - from();
        }
        const float e = __builtin_amdgcn_exp2f(at + kBias);
        if (!sees) return;
        if (half == 0) sum += e;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f16x4 x = *(const f16x4*)(v + t * 64 + i * 16 + half * 8);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[t][4 * i + j] = __builtin_fmaf(e, (float)x[j], o[t][4 * i + j]);
                asm volatile("" ::: "memory");
            }
    }
};

// A scale as the kernels take it: q times `sign`, -1, 1 or 0, and c = |scale| log2 e.  For
// a scale of 0 the zeros go into q, and c is 1: a masked score, -inf, stays what it is.
struct QScale {
    float c;
    _Float16 sign;
};

inline QScale q_scale(float scale)
{
    return {scale == 0.0f ? 1.0f : (scale < 0.0f ? -scale : scale) * kLog2e, (_Float16)(scale == 0.0f ? 0 : scale < 0.0f ? -1 : 1)};
}

// Division by a number that the host knows, of numbers below 2^31: with s the
// least power of two that is not below d, floor((n m / 2^32 + n) / 2^s) for
// m = floor(2^32 (2^s - d) / d) + 1.
struct Divisor {
    unsigned d, m, s;
};

inline Divisor divisor(unsigned d)
{
    unsigned s = 0;
    while ((1ull << s) < d) ++s;
    return {d, (unsigned)((((1ull << s) - d) << 32) / d + 1), s};
}

template <class D>
__device__ inline unsigned divide(unsigned n, const D& by) { return (__umulhi(n, by.m) + n) >> by.s; }

// A value that is the same in all lanes, as the compiler cannot know.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

template <int kControl>
__device__ inline int moved(int x)      // within rows of 16 lanes; 0 comes in
{
    return __builtin_amdgcn_update_dpp(0, x, kControl, 0xf, 0xf, true);
}

// Sum over a wave's lanes.
__device__ inline int wave_sum(int x)
{
    x += moved<0xb1>(x);      // lane ^ 1
    x += moved<0x4e>(x);      // lane ^ 2
    x += moved<0x141>(x);     // the other four of eight
    x += moved<0x140>(x);     // the other eight of sixteen
    return __builtin_amdgcn_readlane(x, 0) + __builtin_amdgcn_readlane(x, 16) + __builtin_amdgcn_readlane(x, 32) +
           __builtin_amdgcn_readlane(x, 48);
}

// Largest of a wave's lanes.
__device__ inline int wave_max(int x)
{
    x = max(x, moved<0xb1>(x));
    x = max(x, moved<0x4e>(x));
    x = max(x, moved<0x141>(x));
    x = max(x, moved<0x140>(x));
    return max(max(__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 16)),
               max(__builtin_amdgcn_readlane(x, 32), __builtin_amdgcn_readlane(x, 48)));
}

// Inclusive sums over a wave's lanes.
__device__ inline int wave_scan(int x)
{
    x += moved<0x111>(x);     // from 1, 2, 4 and 8 lanes below
    x += moved<0x112>(x);
    x += moved<0x114>(x);
    x += moved<0x118>(x);
    const int a = __builtin_amdgcn_readlane(x, 15), b = a + __builtin_amdgcn_readlane(x, 31);
    const int c = b + __builtin_amdgcn_readlane(x, 47), row = (threadIdx.x & 63) >> 4;
    return x + (row == 0 ? 0 : row == 1 ? a : row == 2 ? b : c);
}

}  // namespace steps
