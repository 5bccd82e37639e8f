// kv4_evict.hip -- eviction from the 4-bit KV cache (include/apex_kv4.h).
//
// The order of keeping is the order of 64-bit numbers: a token's key (all ones
// for a protected token, else its weight's bits made monotonic) above its slot
// inverted, so no two are equal.  One work group per (request, kv-head) pair
// finds the keep-th of them: counts of the top digit's values among the
// candidates, the digit that holds it, the next digit among those, until few
// candidates are left, which are ranked against each other.  A thread keeps up to
// 32 keys in registers, so weights and positions are read once; longer pairs read
// them again for every digit, or, where pairs are few, are spread over work
// groups, with a launch for every step.
//
// What is kept goes into a mask, one bit per slot, and the moves are read off
// the masks only (they overwrite weights and positions): the i-th evicted slot
// of the first `keep` takes the i-th kept one behind them.  Sources and targets
// are disjoint, so the moves need no order, and a cut by a few tokens moves a few
// rows.
//
// Slots of blocks outside the pool are none of these: they have key 0, below every
// token's, the first `keep` slots end where the next one of the pool lies (at `keep`
// itself unless ids before it are outside the pool), and up to there such a slot's
// bit says "kept", so that nothing is moved to it.
//
// 256 pairs of 2048-32768 tokens cut to 4096 take 139 us: 39 to select (8 bytes a
// token, but three digits' counts, each with its barriers), 99 to move.  A row's
// values are 4-byte pieces over 256 bytes that it shares with three other tokens,
// so the moves read 230 MB and write 126 for 190 MB of rows, 3.6 TB/s (a large copy
// has 4.5).  Short pairs are bound by the launch and some ten round trips (128 of
// 1025-1088 tokens cut to 1024: 14 us).
#include <type_traits>

#include "kernels.h"
#include "kv4_host.h"

namespace {

using namespace kv4;
using apex::uniform;

constexpr int kBins = 2048;
// Candidates that are ranked directly.  Up to 64: the same times; up to 1024: 89 us
// where it is 60 (32 pairs of 30000 tokens cut to 15000).
constexpr int kFew = 256;
constexpr int kMostPerThread = 32;         // keys that a thread keeps
constexpr int kAgainPerThread = 16;        // and reads at a time where it keeps none
// Threads of a work group: the larger where a pair has more tokens than the smaller
// one's registers hold, but not with pairs for every CU several times over, whose
// work groups run beside each other.  256 against 1024 threads: 1024 pairs of 1056
// tokens 23 against 44 us, 2048 of 600 57 against 99; 64 of 13000 84 against 44.
constexpr int kSmall = 256, kLarge = 1024;
constexpr int kResident = kMostPerThread * kLarge;
// Up to so many tokens of a pair are moved by the work group that selects them; more
// are spread by a second launch.  128 pairs of 1025-1088 tokens cut to 1024 take 16.9
// us, 18.7 if all go to the second launch; 32 of 4000 cut to 2000 26.6, 61 if none
// do.
constexpr int kOwnMoves = 1024;
constexpr int kGaps = INT_MIN;             // beside a count of moves

// What is known of the keep-th key: its leading digits, and that it is the
// need-th from the top of those that have them.
struct Found {
    unsigned prefix;
    int need;
};

struct EvictParams {
    char* cache;
    const int32_t* bt;
    const int32_t* lens;
    float* weights;
    int32_t* positions;
    uint64_t* masks;       // [B][Hkv][words], bit i of word w: slot 64 w + i is kept
    int32_t* counts;       // [B][Hkv] tokens left to move; kGaps: its `keep` slots do not end at `keep`
    unsigned num_blocks;
    int Hkv, stride, words;
    int keep, sinks, recent;
    // of pairs that are spread over work groups
    int chunks;            // of the longest possible pair
    int2* newest;          // [B][Hkv][chunks] highest position, tokens in the pool
    Found* found;          // [B][Hkv][2] after the first and the second digit
    uint16_t* bins;        // [2][B][Hkv][chunks][kBins]: of digits 1 and 3, of digit 2
};

__device__ inline int context(const EvictParams& p, int b)
{
    const int64_t row = (int64_t)p.stride * kBlockSize;
    const int L = p.lens[b];
    return L > row ? (int)row : L;
}

// Index of a slot in weights and positions from its block id; -1 outside the pool.
__device__ inline int64_t slot_index(const EvictParams& p, int id, int g, int t)
{
    return (unsigned)id < p.num_blocks ? ((int64_t)id * p.Hkv + g) * kBlockSize + t % kBlockSize : -1;
}

// Order-preserving bits of a weight; below every protected token's.
__device__ inline unsigned weight_key(float w)
{
    if (w != w) w = -INFINITY;
    const unsigned u = __float_as_uint(w + 0.f);   // (-0 becomes 0)
    return (u >> 31) ? ~u : u | 0x80000000u;
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

// Where the slot of the pool lies that has `before` of its kind ahead of it among
// slots [first, last) of a row (first a multiple of the block); 0 if there is none.
template <int kT>
__device__ inline int pool_slot(const EvictParams& p, const int32_t* row, int first, int last, int before, int (&sums)[kT / 64],
                                int& found)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int e0 = first / kBlockSize, n = (last - first + kBlockSize - 1) / kBlockSize, per = (n + kT - 1) / kT;
    const int a = e0 + min(n, tid * per), e = e0 + min(n, (tid + 1) * per);
    auto slots = [&](int i) -> int { return (unsigned)row[i] < p.num_blocks ? min(kBlockSize, last - i * kBlockSize) : 0; };
    int sum = 0;
    for (int i = a; i < e; ++i) sum += slots(i);
    int incl = wave_scan(sum, lane);
    if (lane == 63) sums[wave] = incl;
    if (tid == 0) found = 0;
    __syncthreads();
    for (int i = 0; i < wave; ++i) incl += sums[i];
    int left = before - (incl - sum);
    if (left >= 0 && left < sum) {
        int i = a;
        for (int s = slots(i); left >= s; s = slots(i)) {
            left -= s;
            ++i;
        }
        found = i * kBlockSize + left;
    }
    __syncthreads();
    const int at = found;
    __syncthreads();   // (the caller may write both again)
    return at;
}

// --- moves ------------------------------------------------------------------------

template <int kN>
struct Moves {
    int64_t to[kN], from[kN];   // slot indexes
    int2 hole_words[kN], mover_words[kN];   // words with listed slots: index, rank of the first
    int holes[kN / 64], movers[kN / 64];
    int hole_n, mover_n;
};

// Moves r0 .. r0 + kN of a pair's n, by kN threads; its first `keep` slots end at
// slot `end`.
template <int kN>
__device__ inline void move_rows(const EvictParams& p, const int32_t* row, int g, const uint64_t* kept, int L, int end, int r0,
                                 int n, Moves<kN>& sh)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // a thread counts the holes (evicted below end) and movers (kept from end
    // on) of consecutive words and a scan ranks them; the words with any of the
    // kN looked for, at most kN, are put down, and a wave lists a word's slots, a
    // lane each
    const int words = (L + 63) / 64, per = (words + kN - 1) / kN;
    const int a = min(words, tid * per), e = min(words, a + per);
    auto hole_bits = [&](int w) -> uint64_t {
        const int left = end - w * 64;
        return ~kept[w] & (left <= 0 ? 0ull : left >= 64 ? ~0ull : (1ull << left) - 1);
    };
    auto mover_bits = [&](int w) -> uint64_t {
        const int skip = end - w * 64;
        return kept[w] & (skip <= 0 ? ~0ull : skip >= 64 ? 0ull : ~0ull << skip);
    };
    int holes = 0, movers = 0;
    for (int w = a; w < e; ++w) {
        holes += __popcll(hole_bits(w));
        movers += __popcll(mover_bits(w));
    }
    int hole = wave_scan(holes, lane), mover = wave_scan(movers, lane);
    if (lane == 63) {
        sh.holes[wave] = hole;
        sh.movers[wave] = mover;
    }
    if (tid == 0) sh.hole_n = sh.mover_n = 0;
    sh.to[tid] = sh.from[tid] = -1;
    __syncthreads();
    for (int i = 0; i < wave; ++i) {
        hole += sh.holes[i];
        mover += sh.movers[i];
    }
    hole -= holes + r0;
    mover -= movers + r0;
    for (int w = a; w < e; ++w) {
        const int h = __popcll(hole_bits(w)), m = __popcll(mover_bits(w));
        if (h > 0 && hole < kN && hole + h > 0) sh.hole_words[atomicAdd(&sh.hole_n, 1)] = make_int2(w, hole);
        if (m > 0 && mover < kN && mover + m > 0) sh.mover_words[atomicAdd(&sh.mover_n, 1)] = make_int2(w, mover);
        hole += h;
        mover += m;
    }
    __syncthreads();
    auto list = [&](const int2* from, int n, auto bits, int64_t* to) {
        for (int i = wave; i < n; i += kN / 64) {
            const int2 x = from[i];
            const uint64_t m = bits(x.x);
            const int rank = x.y + __popcll(m & ((1ull << lane) - 1));
            if ((m >> lane & 1) && rank >= 0 && rank < kN) to[rank] = x.x * 64 + lane;
        }
    };
    list(sh.hole_words, sh.hole_n, hole_bits, sh.to);
    list(sh.mover_words, sh.mover_n, mover_bits, sh.from);
    __syncthreads();
    // slots to indexes, one pair a thread
    const int64_t to_slot = sh.to[tid], from_slot = sh.from[tid];
    if (to_slot >= 0 && from_slot >= 0) {
        const int to_id = row[to_slot / kBlockSize], from_id = row[from_slot / kBlockSize];
        sh.to[tid] = slot_index(p, to_id, g, (int)to_slot);
        sh.from[tid] = slot_index(p, from_id, g, (int)from_slot);
    }
    __syncthreads();
    // 16 lanes a move, kAtOnce moves a thread on their way: lane c has 4 bytes of
    // K and dims [8c, 8c + 8) of V; lanes 0-3 V's scales, 4 K's, 5 and 6 weight
    // and position
    constexpr int kAtOnce = 4, kLanes = 16, kStep = kN / kLanes;
    const int c = tid % kLanes, m1 = min(kN, n - r0);
    for (int m0 = tid / kLanes; m0 < m1; m0 += kStep * kAtOnce) {
        unsigned k[kAtOnce], v[kAtOnce], x[kAtOnce];
        int64_t to[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int m = m0 + i * kStep;
            const int64_t from = m < m1 ? sh.from[m] : -1;
            to[i] = m < m1 && from >= 0 ? sh.to[m] : -1;
            if (to[i] < 0) continue;
            const int fi = (int)(from % kBlockSize);
            const char* fs = p.cache + from / kBlockSize * kSlabBytes;
            k[i] = *(const unsigned*)(fs + fi * 64 + c * 4);
            v[i] = *(const unsigned*)(fs + v_code_offset(fi, c));
            if (c < 4)
                x[i] = *(const unsigned char*)(fs + kVScales + c * kBlockSize + fi);
            else if (c < 7)
                x[i] = *(c == 4 ? (const unsigned*)(fs + kKScales + fi * 4)
                                : c == 5 ? (const unsigned*)p.weights + from : (const unsigned*)p.positions + from);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (to[i] < 0) continue;
            const int ti = (int)(to[i] % kBlockSize);
            char* ts = p.cache + to[i] / kBlockSize * kSlabBytes;
            *(unsigned*)(ts + ti * 64 + c * 4) = k[i];
            *(unsigned*)(ts + v_code_offset(ti, c)) = v[i];
            if (c < 4)
                *(unsigned char*)(ts + kVScales + c * kBlockSize + ti) = (unsigned char)x[i];
            else if (c < 7)
                *(c == 4 ? (unsigned*)(ts + kKScales + ti * 4)
                         : c == 5 ? (unsigned*)p.weights + to[i] : (unsigned*)p.positions + to[i]) = x[i];
        }
    }
}

__global__ __launch_bounds__(kSmall) void move_kernel(EvictParams p)
{
    __shared__ Moves<kSmall> sh;
    const int pair = (int)blockIdx.x, b = pair / p.Hkv, g = pair - b * p.Hkv;
    const int32_t* row = p.bt + (int64_t)b * p.stride;
    const int count = p.counts[pair], n = count & ~kGaps, L = context(p, b);
    if ((int)blockIdx.y * kSmall >= n) return;
    const int end = count & kGaps ? pool_slot<kSmall>(p, row, 0, L, p.keep, sh.holes, sh.hole_n) : p.keep;
    for (int r0 = (int)blockIdx.y * kSmall; r0 < n; r0 += (int)gridDim.y * kSmall) {
        move_rows<kSmall>(p, row, g, p.masks + (int64_t)pair * p.words, L, end, r0, n, sh);
        __syncthreads();
    }
}

// --- selection --------------------------------------------------------------------

// The digit that holds the need-th from the top.
template <int kT>
struct Digit {
    int wave[kT / 64];
    unsigned digit;
    int above, count;   // with higher digits, with this one
};

// A thread has kPer bins, counted down from the top: c[0] that of digit kBins - 1
// - kPer tid.
template <int kT, int kPer>
__device__ inline void find_need(const int (&c)[kPer], int need, Digit<kT>& sh)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += c[i];
    int incl = wave_scan(sum, lane);
    if (lane == 63) sh.wave[wave] = incl;
    __syncthreads();
    for (int i = 0; i < wave; ++i) incl += sh.wave[i];
    int above = incl - sum;
    if (above < need && need <= incl) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (above < need && need <= above + c[i]) {
                sh.digit = (unsigned)(kBins - 1 - kPer * tid - i);
                sh.above = above;
                sh.count = c[i];
            }
            above += c[i];
        }
    }
    __syncthreads();
}

template <int kT>
struct Select {
    // counts of a digit, in copies by the lane's number: weights have few leading
    // digits, and additions to one address wait for each other.  (256 pairs of
    // 2048-32768 tokens, 1024 threads: selected in 45.1 us with one copy, 39.2 with
    // two, 39.1 with four, which take twice the LDS; 128 of 1025-1088 with 256
    // threads, who clear and add up the copies, 13.3 us with one and 14.0 with two.)
    static constexpr int kCopies = kT == kLarge ? 2 : 1;
    unsigned bins[kBins][kCopies];
    uint64_t few[kFew];
    Digit<kT> found;
    int2 seen[kT / 64];   // of a wave's tokens: highest position, whether some lie outside the pool
    int few_n;
    uint64_t last;
};

// Keys of tokens first + kT i + tid, i < kN, in two steps: what is read, and
// (once the newest position is known) the keys.  A slot past L or of a block
// outside the pool reads slot 0's values and has key 0.
template <int kT, int kN>
struct Tokens {
    unsigned w[kN];     // weights' bits, then keys
    int pos[kN];
    unsigned live;      // bit i
    __device__ inline void load(const EvictParams& p, const int32_t* row, int g, int L, int first)
    {
        static_assert(kN <= 32, "a bit for every token");
        const int tid = (int)threadIdx.x;
        int id[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int t = first + i * kT + tid;
            id[i] = row[t < L ? t / kBlockSize : 0];
        }
        live = 0;
        const int64_t at0 = (int64_t)g * kBlockSize + tid % kBlockSize;   // (kT is a multiple of the block)
        const int64_t step = (int64_t)p.Hkv * kBlockSize;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const bool ok = first + i * kT + tid < L && (unsigned)id[i] < p.num_blocks;
            live |= ok ? 1u << i : 0u;
            const int64_t at = at0 + (ok ? id[i] : 0) * step;
            pos[i] = p.positions[at];
            w[i] = __float_as_uint(p.weights[at]);
        }
    }
    __device__ inline int newest() const
    {
        int n = INT_MIN;
#pragma unroll
        for (int i = 0; i < kN; ++i) n = max(n, live >> i & 1 ? pos[i] : INT_MIN);
        return n;
    }
    // whether some of the thread's tokens lie outside the pool
    __device__ inline bool gaps(int L, int first) const
    {
        const int n = L - first - (int)threadIdx.x;   // (kT tokens on, the thread's next)
        return __popc(live) < (n <= 0 ? 0 : min(kN, (n + kT - 1) / kT));
    }
    __device__ inline void keys(int sinks, int64_t recent_from)
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const bool safe = pos[i] < sinks || (int64_t)pos[i] > recent_from;
            w[i] = !(live >> i & 1) ? 0u : safe ? 0xffffffffu : weight_key(__uint_as_float(w[i]));
        }
    }
};

// Returns where the first `keep` slots end, 0 if the pair is left as it is.
template <int kT, int kN, bool kAgain>
__device__ inline int select_pair(const EvictParams& p, const int32_t* row, int g, int L, uint64_t* out, Select<kT>& sh)
{
    constexpr int kCopies = Select<kT>::kCopies;
    constexpr int kWaves = kT / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    Tokens<kT, kN> x;
    int newest = INT_MIN, gaps = 0;
    for (int first = 0; first == 0 || (kAgain && first < L); first += kN * kT) {
        x.load(p, row, g, L, first);
        newest = max(newest, x.newest());
        gaps |= x.gaps(L, first);
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) newest = max(newest, __shfl_xor(newest, m, 64));
    gaps = __ballot(gaps) != 0;
    if (lane == 0) sh.seen[wave] = make_int2(newest, gaps);
    __syncthreads();
    for (int i = 0; i < kWaves; ++i) {
        newest = max(newest, sh.seen[i].x);
        gaps |= sh.seen[i].y;
    }
    gaps = uniform(gaps);
    const int end = gaps ? pool_slot<kT>(p, row, 0, L, p.keep, sh.found.wave, sh.few_n) : p.keep;
    if (end == 0) return 0;   // no more than `keep` tokens
    const int64_t recent_from = (int64_t)newest - p.recent;
    if (!kAgain) x.keys(p.sinks, recent_from);
    // f(key, t, i) for every token, the i-th of its thread's batch, then g(first)
    // for the batch.  Slots past L take part: they have key 0 and come after every
    // token, so the keep-th is none of them.
    auto walk = [&](auto f, auto batch) {
        for (int first = 0; first == 0 || (kAgain && first < L); first += kN * kT) {
            if (kAgain) {
                x.load(p, row, g, L, first);
                x.keys(p.sinks, recent_from);
            }
#pragma unroll
            for (int i = 0; i < kN; ++i) f(x.w[i], first + i * kT + tid, i);
            batch(first);
        }
    };
    auto no_batch = [](int) {};
    // counts of a digit of the tokens that are `in`, then the digit that holds the
    // need-th from the top
    const int all = (L + kN * kT - 1) / (kN * kT) * (kN * kT);
    int need = p.keep, candidates = all;
    auto find_digit = [&](auto in, auto digit, auto of_keys) -> unsigned {
        for (int i = tid; i < kBins * kCopies; i += kT) sh.bins[0][i] = 0;
        __syncthreads();
        if (candidates < all && candidates > all / 2) {
            // most tokens share the digits so far, so mostly the next one too
            // (equal weights): a wave whose candidates have one digit counts once
            walk([&](unsigned key, int t, int) {
                const bool c = in(key, t);
                const unsigned d = digit(key, t);
                const uint64_t act = __ballot(c);
                const unsigned d0 = (unsigned)__builtin_amdgcn_readlane((int)d, act ? __builtin_ctzll(act) : 0);
                if (__ballot(c && d != d0) == 0) {
                    if (lane == 0 && act) atomicAdd(&sh.bins[d0][0], (unsigned)__popcll(act));
                } else if (c) {
                    atomicAdd(&sh.bins[d][lane % kCopies], 1u);
                }
            }, no_batch);
        } else {
            // protected tokens share every digit of the key, and often a wave
            constexpr bool kKeys = decltype(of_keys)::value;
            int safe = 0;
            walk([&](unsigned key, int t, int) {
                const bool c = in(key, t), top = kKeys && key == 0xffffffffu;
                if (kKeys) safe += __popcll(__ballot(c && top));
                if (c && !top) atomicAdd(&sh.bins[digit(key, t)][lane % kCopies], 1u);
            }, no_batch);
            if (kKeys && lane == 0 && safe > 0) atomicAdd(&sh.bins[digit(0xffffffffu, 0)][0], (unsigned)safe);
        }
        __syncthreads();
        constexpr int kPer = kBins / kT;
        int c[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            c[i] = 0;
#pragma unroll
            for (int j = 0; j < kCopies; ++j) c[i] += (int)sh.bins[kBins - 1 - kPer * tid - i][j];
        }
        find_need<kT, kPer>(c, need, sh.found);
        need -= sh.found.above;
        candidates = sh.found.count;
        return sh.found.digit;
    };

    // the keep-th key from the top, digit by digit: candidates have key >> shift
    // == prefix.  Should more than kFew have the whole key, the same for their
    // slots, inverted: last_slot >> slot_shift of the candidates
    static_assert(kN * kT > kFew, "a walk has more slots than are ranked");
    unsigned prefix = find_digit([](unsigned, int) -> bool { return true; }, [](unsigned key, int) -> unsigned { return key >> 21; }, std::true_type());
    unsigned slots = 0;
    int shift = 21, slot_shift = 32;   // (32: no digit of the slots yet)
    auto in_keys = [&](unsigned key, int) -> bool { return key >> shift == prefix; };
    auto in_slots = [&](unsigned key, int t) -> bool {
        return key == prefix && (slot_shift == 32 || ~(unsigned)t >> slot_shift == slots);
    };
    while (candidates > kFew && shift > 0) {
        const int to = shift == 21 ? 10 : 0;
        const unsigned dm = to == 0 ? 1023u : 2047u;
        const unsigned d = find_digit(in_keys, [&](unsigned key, int) -> unsigned { return key >> to & dm; }, std::true_type());
        prefix = prefix << (shift - to) | d;
        shift = to;
    }
    while (candidates > kFew) {   // (slots differ: it ends)
        const int to = slot_shift == 32 ? 21 : slot_shift == 21 ? 10 : 0;
        const unsigned dm = to == 0 ? 1023u : 2047u;
        const unsigned d = find_digit(in_slots, [&](unsigned, int t) -> unsigned { return ~(unsigned)t >> to & dm; }, std::false_type());
        slots = slot_shift == 32 ? d : slots << (slot_shift - to) | d;
        slot_shift = to;
    }
    // rank the candidates by key, then slot
    if (tid == 0) sh.few_n = 0;
    __syncthreads();
    walk([&](unsigned key, int t, int) {
        const bool c = slot_shift < 32 ? in_slots(key, t) : in_keys(key, t);
        if (c) sh.few[atomicAdd(&sh.few_n, 1)] = (uint64_t)key << 32 | ~(unsigned)t;
    }, no_batch);
    __syncthreads();
    for (int i = tid; i < candidates; i += kT) {
        const uint64_t o = sh.few[i];
        int r = 0;
        for (int j = 0; j < candidates; ++j) r += sh.few[j] > o;
        if (r == need - 1) sh.last = o;
    }
    __syncthreads();
    const unsigned last_key = (unsigned)(sh.last >> 32);
    const int last_t = (int)~(unsigned)sh.last;
    // lane i of a wave gets the mask of the wave's i-th 64 slots
    int moved = 0;
    unsigned lo = 0, hi = 0;
    walk([&](unsigned key, int t, int i) {
        uint64_t bits = __ballot(key > last_key || (key == last_key && t <= last_t));
        if (gaps) bits |= __ballot(key == 0 && t < end);
        lo = lane == i ? (unsigned)bits : lo;
        hi = lane == i ? (unsigned)(bits >> 32) : hi;
    }, [&](int first) {
        const int t = first + lane * kT + wave * 64;
        if (lane < kN && t < L) {
            const uint64_t bits = (uint64_t)hi << 32 | lo;
            out[t >> 6] = bits;
            const int skip = end - t;
            moved += __popcll(bits & (skip <= 0 ? ~0ull : skip >= 64 ? 0ull : ~0ull << skip));
        }
    });
    moved = wave_scan(moved, lane);
    if (lane == 63) sh.found.wave[wave] = moved;
    __syncthreads();
    return end;
}

// kLong: pairs of more than kResident tokens are left to spread_kernel.
template <int kT, bool kLong>
__global__ __launch_bounds__(kT, 4) void select_kernel(EvictParams p)
{
    __shared__ union {
        Select<kT> select;
        Moves<kT> moves;
    } sh;
    const int pair = (int)blockIdx.x, b = pair / p.Hkv, g = pair - b * p.Hkv;
    const int L = context(p, b);
    if (L <= p.keep) {
        if (threadIdx.x == 0) p.counts[pair] = 0;
        return;
    }
    if (kLong && L > kResident) return;
    const int32_t* row = p.bt + (int64_t)b * p.stride;
    uint64_t* out = p.masks + (int64_t)pair * p.words;
    int end = 0;
    if (L <= 2 * kT)
        end = select_pair<kT, 2, false>(p, row, g, L, out, sh.select);
    else if (L <= 8 * kT)
        end = select_pair<kT, 8, false>(p, row, g, L, out, sh.select);
    else if (L <= 16 * kT)
        end = select_pair<kT, 16, false>(p, row, g, L, out, sh.select);
    else if (L <= kMostPerThread * kT)
        end = select_pair<kT, kMostPerThread, false>(p, row, g, L, out, sh.select);
    else if (!kLong)
        end = select_pair<kT, kAgainPerThread, true>(p, row, g, L, out, sh.select);
    int n = 0;
    if (end > 0)
        for (int i = 0; i < kT / 64; ++i) n += sh.select.found.wave[i];
    const bool own = n <= kOwnMoves;
    if (threadIdx.x == 0) p.counts[pair] = own ? 0 : end == p.keep ? n : n | kGaps;
    if (!own) return;
    // (the masks are this work group's own: the barrier makes them visible)
    for (int r0 = 0; r0 < n; r0 += kT) {
        __syncthreads();
        move_rows<kT>(p, row, g, out, L, end, r0, n, sh.moves);
    }
}

// --- selection over several work groups ---------------------------------------------

constexpr int kChunkKeys = 8;                        // a thread
constexpr int kChunk = kChunkKeys * kLarge;          // tokens a work group

// A pair's tokens in chunks, a work group each, and a launch for every step that
// needs all of them: the newest position and the tokens in the pool (step 0), the counts of the three digits
// of the keys (1 to 3; a chunk's counts fit 16 bits, each work group adds up the
// chunks' and finds the digit itself), the masks (4).  Of the tokens with the last
// key the first by slot are kept: the chunks' counts of that digit tell how many
// come before.
template <int kStep>
__global__ __launch_bounds__(kLarge, 4) void spread_kernel(EvictParams p)
{
    constexpr int kWaves = kLarge / 64;
    __shared__ unsigned s_bins[kStep >= 1 && kStep <= 3 ? kBins : 1];
    __shared__ Digit<kLarge> s_found;
    __shared__ int s_equal[kChunkKeys * kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int pair = (int)blockIdx.x, chunk = (int)blockIdx.y, b = pair / p.Hkv, g = pair - b * p.Hkv;
    const int L = context(p, b);
    if (L <= kResident || L <= p.keep || (int64_t)chunk * kChunk >= L) return;
    if (kStep == 0 && chunk == 0 && tid == 0) p.counts[pair] = 0;
    const int chunks = (L - 1) / kChunk + 1, first = chunk * kChunk;
    int2* const newest = p.newest + (int64_t)pair * p.chunks;
    Tokens<kLarge, kChunkKeys> x;
    x.load(p, p.bt + (int64_t)b * p.stride, g, L, first);
    if (kStep == 0) {
        int high = x.newest(), live = __popc(x.live);
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) {
            high = max(high, __shfl_xor(high, m, 64));
            live += __shfl_xor(live, m, 64);
        }
        if (lane == 0) {
            s_found.wave[wave] = high;
            s_equal[wave] = live;
        }
        __syncthreads();
        live = 0;
        for (int i = 0; i < kWaves; ++i) {
            high = max(high, s_found.wave[i]);
            live += s_equal[i];
        }
        if (tid == 0) newest[chunk] = make_int2(high, live);
        return;
    }

    // the digit that the launch before counted (asked for before the tokens are
    // waited for, as the newest position is)
    Found f = {0, p.keep};
    const int64_t all_bins = (int64_t)gridDim.x * p.chunks * kBins;
    uint16_t* const bins = p.bins + (int64_t)pair * p.chunks * kBins;
    const uint16_t* const counted = bins + (kStep == 3 ? all_bins : 0);
    int c[2] = {0, 0};
    if (kStep >= 2) {
        if (kStep >= 3) f = p.found[(int64_t)pair * 2 + kStep - 3];
#pragma unroll 8
        for (int i = 0; i < chunks; ++i) {
            const unsigned two = ((const unsigned*)(counted + (int64_t)i * kBins))[kBins / 2 - 1 - tid];
            c[0] += (int)(two >> 16);
            c[1] += (int)(two & 0xffff);
        }
    }
    int high = INT_MIN, live = 0;
    for (int i = lane; i < chunks; i += 64) {
        const int2 of = newest[i];
        high = max(high, of.x);
        live += of.y;
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        high = max(high, __shfl_xor(high, m, 64));
        live += __shfl_xor(live, m, 64);
    }
    if (live <= p.keep) return;   // (the same for all of the pair's work groups)
    int before = 0;
    if (kStep >= 2) {
        find_need<kLarge, 2>(c, f.need, s_found);
        f.need -= s_found.above;
        f.prefix = f.prefix << (kStep == 4 ? 10 : 11) | s_found.digit;
        if (kStep < 4 && chunk == 0 && tid == 0) p.found[(int64_t)pair * 2 + kStep - 2] = f;
        if (kStep == 4) {
            for (int i = lane; i < chunk; i += 64) before += counted[(int64_t)i * kBins + s_found.digit];
#pragma unroll
            for (int m = 32; m >= 1; m >>= 1) before += __shfl_xor(before, m, 64);
        }
    }
    x.keys(p.sinks, (int64_t)high - p.recent);

    if (kStep <= 3) {
        constexpr int kAbove = kStep == 1 ? 32 : kStep == 2 ? 21 : 10, kTo = kStep == 1 ? 21 : kStep == 2 ? 10 : 0;
        for (int i = tid; i < kBins; i += kLarge) s_bins[i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kChunkKeys; ++i) {
            const bool in = kStep == 1 || x.w[i] >> (kAbove & 31) == f.prefix;
            const unsigned d = x.w[i] >> kTo & ((1u << (kAbove - kTo)) - 1);
            // the lanes of the first one's digit count once: protected tokens and
            // equal weights share theirs
            const uint64_t act = __ballot(in);
            const unsigned d0 = (unsigned)__builtin_amdgcn_readlane((int)d, act ? __builtin_ctzll(act) : 0);
            const int same = __popcll(__ballot(in && d == d0));
            if (lane == 0 && same > 0) atomicAdd(&s_bins[d0], (unsigned)same);
            if (in && d != d0) atomicAdd(&s_bins[d], 1u);
        }
        __syncthreads();
        uint16_t* const to = bins + (kStep == 2 ? all_bins : 0) + (int64_t)chunk * kBins;
        ((unsigned*)to)[tid] = s_bins[2 * tid] | s_bins[2 * tid + 1] << 16;
        return;
    }

    // where the first `keep` slots end: in the chunk that holds the next one of the pool
    int end = p.keep;
    if (live < L) {
        int ahead = 0, at = 0;
        for (;; at += 64) {   // (it is there: live > keep)
            const int of = at + lane < chunks ? newest[at + lane].y : 0, incl = wave_scan(of, lane);
            const uint64_t hit = __ballot(ahead + incl > p.keep);
            const int ln = hit ? __builtin_ctzll(hit) : 63;
            ahead += __shfl(hit ? incl - of : incl, ln, 64);
            if (hit) {
                at += ln;
                break;
            }
        }
        end = pool_slot<kLarge>(p, p.bt + (int64_t)b * p.stride, at * kChunk, min(L, (at + 1) * kChunk), p.keep - ahead,
                                s_found.wave, s_equal[0]);
        if (chunk == 0 && tid == 0 && end != p.keep) atomicAdd(&p.counts[pair], kGaps);
    }

    // words in the order of their slots: kWaves of every i
    uint64_t equal[kChunkKeys];
#pragma unroll
    for (int i = 0; i < kChunkKeys; ++i) {
        equal[i] = __ballot(x.w[i] == f.prefix);
        if (lane == 0) s_equal[i * kWaves + wave] = __popcll(equal[i]);
    }
    __syncthreads();
    static_assert(kChunkKeys * kWaves == 128, "two words a lane");
    const int e0 = s_equal[2 * lane], e1 = s_equal[2 * lane + 1];
    int base = before + wave_scan(e0 + e1, lane) - e0 - e1;
    if (wave & 1) base += e0;
    uint64_t own = 0;
#pragma unroll
    for (int i = 0; i < kChunkKeys; ++i) {
        const int rank = __shfl(base, (i * kWaves + wave) / 2, 64) + __popcll(equal[i] & ((1ull << lane) - 1));
        const uint64_t bits = __ballot(x.w[i] > f.prefix || (x.w[i] == f.prefix && rank < f.need) ||
                                       (x.w[i] == 0 && first + i * kLarge + tid < end));
        own = lane == i ? bits : own;
    }
    const int64_t t = (int64_t)first + lane * kLarge + wave * 64;
    int moved = 0;
    if (lane < kChunkKeys && t < L) {
        p.masks[(int64_t)pair * p.words + (t >> 6)] = own;
        const int64_t skip = end - t;
        moved = __popcll(own & (skip <= 0 ? ~0ull : skip >= 64 ? 0ull : ~0ull << skip));
    }
    moved = wave_scan(moved, lane);
    if (lane == 63 && moved > 0) atomicAdd(&p.counts[pair], moved);
}

int64_t mask_words(int64_t stride) { return (stride * kBlockSize + 63) / 64; }

size_t count_bytes(int B, int Hkv) { return align_up((size_t)B * Hkv * 4, 256); }

size_t mask_bytes(int B, int Hkv, int64_t stride) { return align_up((size_t)B * Hkv * mask_words(stride) * 8, 256); }

// Few pairs, of which some may be longer than a work group's registers, are spread.
// Measured, a work group a pair against a launch a step, pairs x tokens: 8 x 131072
// 242 against 88 us, 32 x 131072 366 against 240, 64 x 65536 247 against 221, 96 x
// 65536 315 against 311, 128 x 65536 380 against 402.  Where all are short after all
// the idle launches cost 1.5 us each: 8 x 4000 19 against 28 us.
constexpr int64_t kMostSpread = 64;
bool spread(int64_t pairs, int64_t stride) { return stride * kBlockSize > kResident && pairs <= kMostSpread; }

int64_t chunks_of(int64_t stride) { return (stride * kBlockSize + kChunk - 1) / kChunk; }

size_t need_bytes(int B, int Hkv, int64_t stride)
{
    const size_t pairs = (size_t)B * Hkv, chunks = (size_t)chunks_of(stride);
    const size_t base = count_bytes(B, Hkv) + mask_bytes(B, Hkv, stride);
    if (!spread((int64_t)pairs, stride)) return base;
    return base + align_up(pairs * chunks * sizeof(int2), 256) + align_up(pairs * 2 * sizeof(Found), 256) + 2 * pairs * chunks * kBins * 2;
}

// Slots and steps over them stay below 2^31, chunks and pairs within a grid.
int check_evict(int B, int Hkv, int d, int block_size, int64_t num_blocks, int64_t stride)
{
    const int rc = check_batch(B, Hkv, Hkv, d, block_size, num_blocks, stride);
    if (rc != APEX_OK) return rc;
    if (stride >= 1 << 24) return fail(APEX_ERR_UNSUPPORTED, "block_table_stride %lld reaches 2^24", (long long)stride);
    if ((int64_t)B * Hkv >= 1 << 22) return fail(APEX_ERR_UNSUPPORTED, "B * Hkv = %lld reaches 2^22", (long long)B * Hkv);
    return APEX_OK;
}

}  // namespace

extern "C" size_t apex_kv4_evict_workspace_bytes(int B, int Hkv, int64_t block_table_stride)
{
    apex::clear_error();
    if (check_evict(B, Hkv, kHeadDim, kBlockSize, 0, block_table_stride) != APEX_OK) return 0;
    return need_bytes(B, Hkv, block_table_stride);
}

extern "C" int apex_kv4_evict(void* kv_cache, const int32_t* block_table, int64_t block_table_stride,
                              const int32_t* context_lens, float* weights, int32_t* positions, int B, int Hkv, int d,
                              int block_size, int64_t num_blocks, int keep, int sinks, int recent, void* workspace,
                              size_t workspace_bytes, void* stream)
{
    apex::clear_error();
    int rc = check_evict(B, Hkv, d, block_size, num_blocks, block_table_stride);
    if (rc != APEX_OK) return rc;
    if (keep <= 0 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > keep)
        return fail(APEX_ERR_INVALID_ARG, "keep = %d, sinks = %d, recent = %d: keep must be positive, sinks + recent at most keep",
                    keep, sinks, recent);
    // no request can be longer than keep, no token is in the pool
    const int64_t longest = block_table_stride * kBlockSize;
    if (B == 0 || longest <= keep || num_blocks == 0) return APEX_OK;
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
    Hold hold;
    rc = workspace ? check_workspace(workspace, workspace_bytes, need)
                   : library_buffer(kMasks, need, (hipStream_t)stream, hold, &workspace);
    if (rc != APEX_OK) return rc;
    int cus = 0;
    rc = compute_units(&cus);
    if (rc != APEX_OK) return rc;
    EvictParams p = EvictParams();
    p.cache = (char*)kv_cache;
    p.bt = block_table;
    p.lens = context_lens;
    p.weights = weights;
    p.positions = positions;
    p.counts = (int32_t*)workspace;
    p.masks = (uint64_t*)((char*)workspace + count_bytes(B, Hkv));
    p.num_blocks = (unsigned)num_blocks;
    p.Hkv = Hkv;
    p.stride = (int)block_table_stride;
    p.words = (int)mask_words(block_table_stride);
    p.keep = keep;
    p.sinks = sinks;
    p.recent = recent;
    const int pairs = B * Hkv;
    // at most min(keep, longest - keep) tokens of a pair move
    const int64_t most = longest - keep < keep ? longest - keep : keep;
    const bool wide = spread(pairs, block_table_stride);
    if (longest <= kMostPerThread * kSmall || pairs >= 4 * cus)
        select_kernel<kSmall, false><<<(unsigned)pairs, kSmall, 0, (hipStream_t)stream>>>(p);
    else if (!wide)
        select_kernel<kLarge, false><<<(unsigned)pairs, kLarge, 0, (hipStream_t)stream>>>(p);
    else {
        select_kernel<kLarge, true><<<(unsigned)pairs, kLarge, 0, (hipStream_t)stream>>>(p);
        p.chunks = (int)chunks_of(block_table_stride);
        char* at = (char*)p.masks + mask_bytes(B, Hkv, block_table_stride);
        p.newest = (int2*)at;
        at += align_up((size_t)pairs * p.chunks * sizeof(int2), 256);
        p.found = (Found*)at;
        p.bins = (uint16_t*)(at + align_up((size_t)pairs * 2 * sizeof(Found), 256));
        const dim3 grid((unsigned)pairs, (unsigned)p.chunks);
        spread_kernel<0><<<grid, kLarge, 0, (hipStream_t)stream>>>(p);
        spread_kernel<1><<<grid, kLarge, 0, (hipStream_t)stream>>>(p);
        spread_kernel<2><<<grid, kLarge, 0, (hipStream_t)stream>>>(p);
        spread_kernel<3><<<grid, kLarge, 0, (hipStream_t)stream>>>(p);
        spread_kernel<4><<<grid, kLarge, 0, (hipStream_t)stream>>>(p);
    }
    if ((rc = launched("kv4 evict")) != APEX_OK || (!wide && most <= kOwnMoves)) return rc;
    int64_t groups = (most + kSmall - 1) / kSmall;
    if (groups * pairs > 4096) groups = 4096 / pairs > 0 ? 4096 / pairs : 1;
    move_kernel<<<dim3((unsigned)pairs, (unsigned)groups), kSmall, 0, (hipStream_t)stream>>>(p);
    return launched("kv4 evict");
}
