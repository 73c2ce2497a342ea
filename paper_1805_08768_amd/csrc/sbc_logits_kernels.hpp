// Kernels over rows of logits: a teacher's top logits, and the loss of a student against them with its
// gradient.
//
// A row starts at whatever address its leading dimension gives.  All of them read it as vectors of eight
// values at multiples of the vector's size: vector i of a row that starts `lead` values behind such a
// multiple holds the values 8 i - lead to 8 i - lead + 7, of which those outside the row count as -inf.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sbc_mxfp_kernels.hpp"

namespace sbc {

constexpr int kTopMax = 256;             // the most logits that are listed for a row (SBC_TOP_MAX)

template <typename T> struct Vec8 { typedef T type __attribute__((ext_vector_type(8), aligned(8 * sizeof(T)))); };

// Values of row `row` that lie before its first vector's start.
template <typename T> __device__ __forceinline__ uint32_t row_lead(const T* row) {
    return (uint32_t)(reinterpret_cast<uintptr_t>(row) / sizeof(T)) & 7u;
}

// A row and its vectors.
template <typename T> struct Row {
    const T* start;                      // where vector 0 starts (before the row, where `lead` is not 0)
    uint32_t lead, vecs;                 // values before the row, vectors with values of the row
    uint32_t from, upto;                 // the vectors that lie within the row as a whole
    uint32_t vocab;
    __device__ __forceinline__ Row(const T* row, uint32_t vocab_) : lead(row_lead(row)), vocab(vocab_) {
        start = row - lead;
        vecs = (uint32_t)(((uint64_t)vocab + lead + 7u) >> 3);
        from = lead ? 1u : 0u;
        upto = (uint32_t)(((uint64_t)vocab + lead) >> 3);
    }
    __device__ __forceinline__ typename Vec8<T>::type load(uint32_t vec) const {
        const T* const at = start + (size_t)vec * 8;
        if (vec >= from && vec < upto) return *reinterpret_cast<const typename Vec8<T>::type*>(at);
        typename Vec8<T>::type v;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t index = vec * 8u + i - lead;                  // (at least vocab for those before the row)
            v[i] = index < vocab ? at[i] : (T)-__builtin_inff();
        }
        return v;
    }
    // the same places of another row
    __device__ __forceinline__ void store(T* row, uint32_t vec, const float (&v)[8]) const {
        T* const at = row + ((int64_t)vec * 8 - lead);
        if (vec >= from && vec < upto) {
            store_as<T, 8>(at, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (vec * 8u + i - lead < vocab) at[i] = (T)v[i];
        }
    }
};

// The largest of three; a quiet NaN loses against a number, but a signalling one, as a type's bits may hold it, counts as a quiet
// one before the third is looked at, so that a larger number beside it is lost.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}
__device__ __forceinline__ float max8(const float (&v)[8]) { return max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[6], v[7], v[7])); }

// The same, where any NaN wins; and of numbers alone (-inf where there is none).
__device__ __forceinline__ float maximum3(float a, float b, float c) {
    float d;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}
__device__ __forceinline__ float maximum8(const float (&v)[8]) { return maximum3(maximum3(v[0], v[1], v[2]), maximum3(v[3], v[4], v[5]), maximum3(v[6], v[7], v[7])); }
__device__ __forceinline__ float number8(const float (&v)[8]) {
    float w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = v[j] == v[j] ? v[j] : -__builtin_inff();
    return max8(w);
}

// Reductions over a wavefront, all of whose lanes take part: rows of 16 lanes by exchanges within the row, then the
// four rows, the same order for every lane.
template <int ctrl> __device__ __forceinline__ uint32_t row_exchange(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false); }
template <int ctrl> __device__ __forceinline__ float row_exchange(float v) { return __uint_as_float(row_exchange<ctrl>(__float_as_uint(v))); }
template <int ctrl> __device__ __forceinline__ double row_exchange(double v) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(v);
    return __longlong_as_double((long long)(((unsigned long long)row_exchange<ctrl>((uint32_t)(b >> 32)) << 32) | row_exchange<ctrl>((uint32_t)b)));
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane)); }
__device__ __forceinline__ double lane_of(double v, int lane) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __longlong_as_double((long long)(((unsigned long long)hi << 32) | lo));
}
constexpr int kSwapOne = 0xB1, kSwapTwo = 0x4E, kMirrorEight = 0x141, kMirrorRow = 0x140;      // lane ^ 1, ^ 2, 7 - lane of 8, 15 - lane of 16

template <typename V, typename F> __device__ __forceinline__ V wave_fold(V v, F f) {
    v = f(v, row_exchange<kSwapOne>(v));
    v = f(v, row_exchange<kSwapTwo>(v));
    v = f(v, row_exchange<kMirrorEight>(v));
    v = f(v, row_exchange<kMirrorRow>(v));
    return f(f(lane_of(v, 0), lane_of(v, 16)), f(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ float wave_max(float v) { return wave_fold(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float v) { return wave_fold(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ double wave_sum(double v) { return wave_fold(v, [](double a, double b) { return a + b; }); }

// Sum of exp((x - base) / T) as a pair; base is -inf and the sum 0 (or NaN) where no value is above -inf.
struct ExpSum { float base, sum; };

__device__ __forceinline__ float exp_scaled(float diff, float c) { return __builtin_amdgcn_exp2f(diff * c); }
__device__ __forceinline__ float finite_base(float m) { return m == -__builtin_inff() ? 0.0f : m; }

// ... where an infinite value makes the sum infinite, not NaN (the log-sum-exp; a NaN still shows)
__device__ __forceinline__ float lse_base(float m) { return m == __builtin_inff() ? 3.4028235e38f : finite_base(m); }

template <bool kLse = false> __device__ __forceinline__ ExpSum wave_join(ExpSum a, float c) {
    const float m = wave_max(a.base);
    return {m, wave_sum(a.sum * exp_scaled(a.base - (kLse ? lse_base(m) : finite_base(m)), c))};
}

// All wavefronts' pairs as one, in the same order whoever asks; `room` holds a pair for each.
__device__ __forceinline__ ExpSum block_sum(const ExpSum* room, uint32_t waves, float c) {
    float m = -__builtin_inff();
    for (uint32_t w = 0; w < waves; ++w) m = fmaxf(m, room[w].base);
    float s = 0.0f;
    for (uint32_t w = 0; w < waves; ++w) s += room[w].sum * exp_scaled(room[w].base - finite_base(m), c);
    return {m, s};
}
__device__ __forceinline__ ExpSum block_join(ExpSum a, ExpSum* room, uint32_t waves, float c) {
    a = wave_join(a, c);
    if ((threadIdx.x & 63u) == 0) room[threadIdx.x >> 6] = a;
    __syncthreads();
    return block_sum(room, waves, c);
}

// ----------------------------------------------------------- top logits ----
//
// A key orders a row's entries: by value, equal ones by the lowest index first.  Entries of -inf and NaN are
// never listed and have no key.
__device__ __forceinline__ uint32_t top_order(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);       // (-0 counts as 0)
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float top_value(uint32_t order) {
    return __uint_as_float(order ^ ((order >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ unsigned long long top_key(float v, uint32_t index) {
    return ((unsigned long long)top_order(v) << 32) | (0xffffffffu - index);
}

constexpr uint32_t kTopKept = 512;       // keys that are ranked by counting, at the most

// Greatest number that at least `need` of the wavefront's orders reach, to the upper 16 bits (so for a little more
// than `need` of them); 0 if there are not so many.  Orders of what is not listed are 0.
template <int n> __device__ __forceinline__ uint32_t wave_floor(const uint32_t (&order)[n], uint32_t need) {
    uint32_t lo = 0;
#pragma unroll 1
    for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
        const uint32_t t = lo | bit;
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < n; ++i) c += __popcll(__ballot(order[i] >= t));
        if (c >= need) lo = t;
    }
    return lo;
}

// What the wavefronts of a workgroup tell one another: two sets of words used in turn, so that one barrier parts
// the writing of a set from its reading, and the other set's barrier that from its next writing.
template <int waves> struct Tally {
    uint32_t word[2][waves];
};
template <int waves> __device__ __forceinline__ uint32_t block_total(Tally<waves>& t, uint32_t& turn, uint32_t mine) {
    if ((threadIdx.x & 63u) == 0) t.word[turn][threadIdx.x >> 6] = mine;
    __syncthreads();
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < waves; ++w) sum += t.word[turn][w];
    turn ^= 1u;
    return sum;
}
template <int waves> __device__ __forceinline__ uint32_t block_least(Tally<waves>& t, uint32_t& turn, uint32_t mine) {
    if ((threadIdx.x & 63u) == 0) t.word[turn][threadIdx.x >> 6] = mine;
    __syncthreads();
    uint32_t least = t.word[turn][0];
#pragma unroll
    for (int w = 1; w < waves; ++w) least = min(least, t.word[turn][w]);
    turn ^= 1u;
    return least;
}

// An order that at least k of the workgroup's values reach, and at most `most` of them if there is one; lo is reached by k
// and more than `most`, hi by none.  count(o): how many reach o, the same answer for everybody.  Mostly a few steps: the
// search ends with the first order that will do.
template <typename F> __device__ __forceinline__ uint32_t top_bisect(uint32_t lo, uint32_t hi, uint32_t k, uint32_t most, uint32_t& found, F count) {
#pragma unroll 1
    while (found > most && hi - lo > 1u) {
        const uint32_t mid = lo + (hi - lo) / 2u, c = count(mid);
        if (c >= k) {
            lo = mid;
            found = c;
        } else {
            hi = mid;
        }
    }
    return lo;
}
constexpr uint32_t kTopBeyond = 0xff800001u;    // above the order of infinity

// Puts the k greatest of the workgroup's distinct keys (0: none) and perhaps some more, kTopKept at the most, into LDS;
// returns how many.  `least` is an order that k of them reach, 0 if there are not so many; *count is 0 before.  Ends
// with a barrier.
template <int waves, int per>
__device__ __forceinline__ uint32_t top_select(unsigned long long* keys, const unsigned long long (&mine)[per], const uint32_t (&order)[per], uint32_t least, uint32_t k,
                                               uint32_t* count, Tally<waves>& t, uint32_t& turn) {
    least = max(least, 1u);
    uint32_t some = 0;
#pragma unroll
    for (int i = 0; i < per; ++i) some += __popcll(__ballot(order[i] >= least));
    uint32_t have = block_total(t, turn, some);
    least = top_bisect(least, kTopBeyond, k, kTopKept, have, [&](uint32_t o) {
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < per; ++i) found += __popcll(__ballot(order[i] >= o));
        return block_total(t, turn, found);
    });
    unsigned long long from = (unsigned long long)least << 32;
    if (have > kTopKept) {
        // (equal values by the hundred) exactly: the greatest 64-bit number that k keys reach
        from = 0;
#pragma unroll 1
        for (unsigned long long bit = 1ull << 63; bit; bit >>= 1) {
            const unsigned long long next = from | bit;
            some = 0;
#pragma unroll
            for (int i = 0; i < per; ++i) some += __popcll(__ballot(mine[i] >= next));
            if (block_total(t, turn, some) >= k) from = next;
        }
        have = k;
    }
#pragma unroll
    for (int i = 0; i < per; ++i)
        if (mine[i] >= from) keys[atomicAdd(count, 1u) & (kTopKept - 1u)] = mine[i];
    __syncthreads();
    return have;
}

// Leaves of `have` distinct keys in LDS (at most per * threads) the k greatest and perhaps some more, kTopKept at
// most; returns how many.  Called and left with no access to `keys` outstanding.  (Ranking costs the square of the
// keys' number, this a fixed time, and mostly leaves little more than k.)
template <int threads, int per>
__device__ __forceinline__ uint32_t top_reduce(unsigned long long* keys, uint32_t have, uint32_t k, uint32_t* count, Tally<threads / 64>& t, uint32_t& turn) {
    constexpr int waves = threads / 64;
    if (have <= max(128u, 2u * k)) return have;
    unsigned long long mine[per];
    uint32_t order[per];
#pragma unroll
    for (int i = 0; i < per; ++i) {
        const uint32_t at = i * threads + threadIdx.x;
        mine[i] = at < have ? keys[at] : 0ull;
        order[i] = (uint32_t)(mine[i] >> 32);
    }
    if (threadIdx.x == 0) *count = 0;
    const uint32_t least = block_least(t, turn, wave_floor(order, (k + waves - 1) / waves));
    return top_select<waves>(keys, mine, order, least, k, count, t, turn);
}

// Hands the k greatest of `have` distinct keys in LDS to out(rank, key); a key's rank is the number of keys above it.  Up to
// 128 keys have eight lanes each, which count a share; more have a lane, and all lanes read the same two keys at a time.
typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
template <int threads, typename Out>
__device__ __forceinline__ void top_ranked(const unsigned long long* keys, uint32_t have, uint32_t k, Out out) {
    if (have > 128u) {
        for (uint32_t i = threadIdx.x; i < have; i += threads) {
            const unsigned long long mine = keys[i];
            uint32_t rank = 0;
#pragma unroll 8
            for (uint32_t j = 0; j + 1 < have; j += 2) {
                const u64x2 two = *reinterpret_cast<const u64x2*>(keys + j);
                rank += two[0] > mine;
                rank += two[1] > mine;
            }
            if (have & 1u) rank += keys[have - 1] > mine;
            if (rank < k) out(rank, mine);
        }
        return;
    }
    for (uint32_t i = threadIdx.x >> 3; i < have; i += threads / 8) {
        const unsigned long long mine = keys[i];
        uint32_t rank = 0;
#pragma unroll 4
        for (uint32_t j = threadIdx.x & 7u; j < have; j += 8u) rank += keys[j] > mine;
        rank += row_exchange<kSwapOne>(rank);
        rank += row_exchange<kSwapTwo>(rank);
        rank += row_exchange<kMirrorEight>(rank);
        if ((threadIdx.x & 7u) == 0 && rank < k) out(rank, mine);
    }
}

struct TopOut {
    int32_t* index;
    float* top;
    float* lse;
};

__device__ __forceinline__ float log_sum(ExpSum s, float inv_t) { return s.base == -__builtin_inff() && s.sum == 0.0f ? s.base : lse_base(s.base) * inv_t + logf(s.sum); }

template <int threads>
__device__ __forceinline__ void top_store(const unsigned long long* keys, uint32_t have, uint32_t k, int64_t row, const TopOut& out) {
    top_ranked<threads>(keys, have, k, [&](uint32_t rank, unsigned long long key) {
        out.index[row * k + rank] = (int32_t)(0xffffffffu - (uint32_t)key);
        out.top[row * k + rank] = top_value((uint32_t)(key >> 32));
    });
    for (uint32_t i = have + threadIdx.x; i < k; i += threads) {
        out.index[row * k + i] = -1;
        out.top[row * k + i] = -__builtin_inff();
    }
}

// A part of a row to a workgroup, in chunks of threads * n vectors that pass through registers once (the next one's
// loads go out before this one is looked at).  A vector whose largest value reaches `tau` has its number noted in LDS,
// one step for 64 of them; tau is a number that at least k values of the part are known to reach.  The first chunk
// gives it: every wavefront finds a floor that k / waves of its vectors' maxima reach, and so do as many values; the
// lowest floor holds for the workgroup.  For values in no particular order little more than k vectors pass in that chunk
// and in any other (k = 64: 70 to 130).  At the end, and where the notes would overflow, top_digest reads the noted
// vectors again and makes keys of the values that reach tau.
//
// Reading bounds long rows: 4096 x 50021 of 16 bits, k = 64, 98 us (410 MB, 4.2 TB/s), the log-sum-exp from the same
// registers.  A workgroup's fixed part, the floor's search (16 ballots), the notes' second reading and the ranking, is 5 us of
// steps that wait for one another and bounds short rows: 700 x 2025 8 us with k = 8, 11 with k = 64.  One row of 131072 of 32 bits in 33 parts: 8.3 us,
// and 5.7 for the join.
constexpr int kTopThreads = 256;         // of a workgroup of k_top, or 64 for many short rows
constexpr uint32_t kTopRoom = 1024;      // keys

template <int threads> struct TopShared {
    static constexpr int kWaves = threads / 64, kNotes = 8 * threads;            // (at least a chunk's vectors)
    alignas(16) unsigned long long keys[kTopRoom];
    unsigned long long notes[kNotes];            // order of the vector's maximum, its number
    Tally<kWaves> tally;
    uint32_t noted, count;
    ExpSum sums[kWaves];
};

// Makes the notes (`noted` of them) and the `have` keys so far into keys, kTopKept at the most, among them the k greatest of
// all; returns how many and raises tau if that is known to be allowed.  Starts and ends with a barrier.
template <int threads, typename T>
__device__ __forceinline__ uint32_t top_digest(TopShared<threads>& sh, const Row<T>& x, uint32_t noted, uint32_t have, uint32_t k, float& tau, uint32_t& turn) {
    constexpr int n = 1, kTopWaves = threads / 64;
    constexpr uint32_t kTopNotes = TopShared<threads>::kNotes;
    __syncthreads();
    if (threadIdx.x == 0) sh.count = have;
    if (noted > (uint32_t)threads) {
        // a tau from all notes leaves little more than k of them
        constexpr int per = kTopNotes / threads;
        unsigned long long mine[per];
        uint32_t order[per];
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const uint32_t at = i * threads + threadIdx.x;
            mine[i] = at < noted ? sh.notes[at] : 0ull;
            order[i] = (uint32_t)(mine[i] >> 32);
        }
        const uint32_t floor_ = block_least(sh.tally, turn, wave_floor(order, (k + kTopWaves - 1) / kTopWaves));
        if (floor_) {
            tau = fmaxf(tau, top_value(floor_));
            if (threadIdx.x == 0) sh.noted = 0;
            __syncthreads();
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < per; ++i) {
                some += __popcll(__ballot(order[i] >= floor_));
                if (order[i] >= floor_) sh.notes[atomicAdd(&sh.noted, 1u) & (kTopNotes - 1u)] = mine[i];
            }
            noted = block_total(sh.tally, turn, some);
        }
    }
    float after = tau;
    for (uint32_t from = 0; from < noted; from += n * threads) {
        float v[n][8];
        uint32_t at[n];
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const uint32_t note = from + i * threads + threadIdx.x;
            at[i] = note < noted ? (uint32_t)sh.notes[note] : 0u;
            const typename Vec8<T>::type in = x.load(at[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = note < noted ? (float)in[j] : -__builtin_inff();
        }
        const auto key_of = [&](int i, int j) { return top_key(v[i][j], at[i] * 8u + j - x.lead); };
        const auto counted = [&](auto test) {
            uint32_t found = 0;
#pragma unroll
            for (int i = 0; i < n; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) found += __popcll(__ballot(test(i, j)));
            return block_total(sh.tally, turn, found);
        };
        unsigned long long least = 0;
        float next = tau;
        uint32_t some = counted([&](int i, int j) { return v[i][j] >= tau; });
        if (have + some > kTopRoom) {
            uint32_t order[n];
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float m = max8(v[i]);         // (or less, beside a NaN: a floor all the same)
                order[i] = m >= tau ? top_order(m) : 0u;
            }
            const uint32_t floor_ = block_least(sh.tally, turn, wave_floor(order, (k + kTopWaves - 1) / kTopWaves));
            if (floor_) tau = next = fmaxf(tau, top_value(floor_));
            some = counted([&](int i, int j) { return v[i][j] >= tau; });
            if (have + some > kTopRoom) {
                have = top_reduce<threads, kTopRoom / threads>(sh.keys, have, k, &sh.count, sh.tally, turn);
                __syncthreads();
                if (threadIdx.x == 0) sh.count = have;
            }
            if (have + some > kTopRoom) {
                const auto order_of = [&](int i, int j) { return v[i][j] >= tau ? top_order(v[i][j]) : 0u; };
                const uint32_t kth = top_bisect(top_order(tau), kTopBeyond, k, kTopRoom - have, some,
                                                [&](uint32_t o) { return counted([&](int i, int j) { return order_of(i, j) >= o; }); });
                tau = next = fmaxf(tau, top_value(kth));
                if (have + some > kTopRoom) {
                    // (equal values by the hundred) the k-th is found: of its equals the lowest indexes
                    const uint32_t need = k - counted([&](int i, int j) { return order_of(i, j) > kth; });
                    uint32_t low = 0;
#pragma unroll 1
                    for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
                        const uint32_t t = low | bit;
                        if (counted([&](int i, int j) { return order_of(i, j) == kth && (uint32_t)key_of(i, j) >= t; }) >= need) low = t;
                    }
                    least = ((unsigned long long)kth << 32) | low;
                    some = k;
                    after = fmaxf(after, top_value(kth + 1u));   // (k values reach the k-th; equal ones in later chunks come after them)
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < n; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (v[i][j] >= tau && (least == 0 || key_of(i, j) >= least)) sh.keys[atomicAdd(&sh.count, 1u) & (kTopRoom - 1u)] = key_of(i, j);
        have += some;
        tau = next;
    }
    tau = fmaxf(tau, after);
    __syncthreads();
    have = top_reduce<threads, kTopRoom / threads>(sh.keys, have, k, &sh.count, sh.tally, turn);
    __syncthreads();
    return have;
}

template <typename T, int n, int threads>
__global__ __launch_bounds__(threads) void k_top(const T* __restrict__ logits, int64_t ld, uint32_t vocab, uint32_t k, uint32_t parts, uint32_t part_vecs,
                                                float inv_t, float c, TopOut out, unsigned long long* __restrict__ part_keys, ExpSum* __restrict__ part_sums) {
    constexpr int kTopWaves = threads / 64;
    constexpr uint32_t kTopNotes = TopShared<threads>::kNotes;
    static_assert(n * threads <= (int)kTopNotes, "a chunk's notes");
    __shared__ TopShared<threads> sh;
    const uint32_t lane = threadIdx.x & 63u;
    const int64_t row = blockIdx.x / parts;
    const uint32_t first = (blockIdx.x % parts) * part_vecs;            // vectors
    const Row<T> x(logits + row * ld, vocab);
    const uint32_t end = min(first + part_vecs, x.vecs);
    uint32_t turn = 0;
    if (threadIdx.x == 0) sh.noted = 0;
    __syncthreads();

    typename Vec8<T>::type raw[n];
    const auto load = [&](uint32_t from) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const uint32_t at = from + i * threads + threadIdx.x;
            if (at < end) raw[i] = x.load(at);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) raw[i][j] = (T)-__builtin_inff();
        }
    };
    load(first);
    float tau = -3.4028235e38f;          // (the lowest value: -inf and NaN do not reach it)
    uint32_t noted = 0, have = 0;
    ExpSum s = {-__builtin_inff(), 0.0f};
    for (uint32_t from = first; from < end; from += n * threads) {
        float v[n][8], most[n];
        float m = s.base;
        bool nan = false;
#pragma unroll
        for (int i = 0; i < n; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = (float)raw[i][j];
            most[i] = maximum8(v[i]);
            nan |= most[i] != most[i];
        }
        // (a NaN must not hide the numbers beside it, and there hardly is one)
        if (__any(nan)) {
#pragma unroll
            for (int i = 0; i < n; ++i) most[i] = number8(v[i]);
        }
#pragma unroll
        for (int i = 0; i < n; ++i) m = fmaxf(m, most[i]);
        if (from + n * threads < end) load(from + n * threads);
        if (out.lse) {
            const float b = lse_base(m);
            float sum = s.sum * exp_scaled(s.base - b, c);
#pragma unroll
            for (int i = 0; i < n; ++i) {
                float e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = exp_scaled(v[i][j] - b, c);
                sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
            }
            s = {m, sum};
        }
        const auto passing = [&] {
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < n; ++i) some += __popcll(__ballot(most[i] >= tau));
            return block_total(sh.tally, turn, some);
        };
        uint32_t some = passing();
        if (some > 2u * k + 64u) {
            // (for few slots a lane's one largest value will do: the floor is a little lower, its search a quarter as long)
            const uint32_t need = (k + kTopWaves - 1) / kTopWaves;
            uint32_t order[n], one[1] = {0u};
#pragma unroll
            for (int i = 0; i < n; ++i) {
                order[i] = most[i] >= tau ? top_order(most[i]) : 0u;
                one[0] = max(one[0], order[i]);
            }
            const uint32_t floor_ = block_least(sh.tally, turn, need <= 24u ? wave_floor(one, need) : wave_floor(order, need));
            if (floor_) tau = fmaxf(tau, top_value(floor_));
            some = passing();
        }
        if (some == 0) continue;
        if (noted + some > kTopNotes) {
            have = top_digest(sh, x, noted, have, k, tau, turn);
            if (threadIdx.x == 0) sh.noted = 0;
            noted = 0;
            some = passing();            // (fewer reach the new tau)
        }
#pragma unroll
        for (int i = 0; i < n; ++i)
            if (most[i] >= tau)
                sh.notes[atomicAdd(&sh.noted, 1u) & (kTopNotes - 1u)] = ((unsigned long long)top_order(most[i]) << 32) | (from + i * threads + threadIdx.x);
        noted += some;
    }
    have = top_digest(sh, x, noted, have, k, tau, turn);
    ExpSum whole = s;
    if (out.lse) {
        s = wave_join<true>(s, c);
        if (lane == 0) sh.sums[threadIdx.x >> 6] = s;
        __syncthreads();
        whole = sh.sums[0];
#pragma unroll
        for (int w = 1; w < kTopWaves; ++w) whole.base = fmaxf(whole.base, sh.sums[w].base);
        whole.sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kTopWaves; ++w) whole.sum += sh.sums[w].sum * exp_scaled(sh.sums[w].base - lse_base(whole.base), c);
    }
    if (parts == 1) {
        top_store<threads>(sh.keys, have, k, row, out);
        if (out.lse && threadIdx.x == 0) out.lse[row] = log_sum(whole, inv_t);
        return;
    }
    // the k greatest, none as 0
    unsigned long long* const to = part_keys + (size_t)blockIdx.x * k;
    top_ranked<threads>(sh.keys, have, k, [&](uint32_t rank, unsigned long long key) { to[rank] = key; });
    for (uint32_t i = have + threadIdx.x; i < k; i += threads) to[i] = 0;
    if (threadIdx.x == 0) part_sums[blockIdx.x] = whole;
}

// The parts of a row joined: their k keys each (0 for none), kJoinKeys at the most, pass through registers once.  33 x 64 keys
// 5.7 us: the search and the ranking again, on one compute unit.
constexpr int kJoinThreads = 512;
constexpr int kJoinPer = 8;
constexpr int kJoinKeys = kJoinThreads * kJoinPer;

__global__ __launch_bounds__(kJoinThreads) void k_top_join(uint32_t k, uint32_t parts, float inv_t, float c, TopOut out,
                                                           const unsigned long long* __restrict__ part_keys, const ExpSum* __restrict__ part_sums) {
    constexpr int waves = kJoinThreads / 64;
    __shared__ __attribute__((aligned(16))) unsigned long long keys[kTopKept];
    __shared__ Tally<waves> tally;
    __shared__ ExpSum sums[waves];
    __shared__ uint32_t count;
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
    const int64_t row = blockIdx.x;
    const uint32_t slots = parts * k;
    const unsigned long long* const from = part_keys + (size_t)row * slots;
    unsigned long long mine[kJoinPer];
    uint32_t order[kJoinPer];
#pragma unroll
    for (int i = 0; i < kJoinPer; ++i) {
        const uint32_t at = i * kJoinThreads + threadIdx.x;
        mine[i] = at < slots ? from[at] : 0ull;
    }
    ExpSum s = {-__builtin_inff(), 0.0f};
    if (out.lse)
        for (uint32_t p = threadIdx.x; p < parts; p += kJoinThreads) {
            const ExpSum q = part_sums[row * parts + p];
            const float m = fmaxf(s.base, q.base), b = lse_base(m);
            s = {m, s.sum * exp_scaled(s.base - b, c) + q.sum * exp_scaled(q.base - b, c)};
        }
    if (threadIdx.x == 0) count = 0;
#pragma unroll
    for (int i = 0; i < kJoinPer; ++i) order[i] = (uint32_t)(mine[i] >> 32);
    s = wave_join<true>(s, c);
    if (lane == 0) sums[wave] = s;
    uint32_t turn = 0;
    const uint32_t least = block_least(tally, turn, wave_floor(order, (k + waves - 1) / waves));
    const uint32_t have = top_select<waves>(keys, mine, order, least, k, &count, tally, turn);
    top_store<kJoinThreads>(keys, have, k, row, out);
    if (out.lse && threadIdx.x == 0) {
        ExpSum whole = sums[0];
        for (int w = 1; w < waves; ++w) whole.base = fmaxf(whole.base, sums[w].base);
        whole.sum = 0.0f;
        for (int w = 0; w < waves; ++w) whole.sum += sums[w].sum * exp_scaled(sums[w].base - lse_base(whole.base), c);
        out.lse[row] = log_sum(whole, inv_t);
    }
}

// --------------------------------------------------------- distillation ----
//
// Row r of the student's logits s, the teacher's slots j with index i_j and logit t_j; a slot counts if its
// index lies in the vocabulary and its logit is above -inf.  With T the temperature and q = softmax(s / T),
//     p_j   = exp(t_j / T) / sum over the slots          or, given the teacher's log-sum-exp L,
//     p_j   = exp(t_j / T - L),  p_rest = max(0, 1 - sum p_j),  q_rest = sum of q over what no slot lists
//     loss  = T^2 (sum p_j (log p_j - log q_{i_j}) + p_rest (log p_rest - log q_rest))
//     dloss/ds_v = T ((P + p_rest) q_v - sum of p_j with i_j = v - [v not listed] p_rest q_v / q_rest),  P = sum p_j
// (without L p_rest is 0; the rest's part is left out where the student has nothing above -inf outside the
// list).  A row whose weight is 0, that has no slot, or whose student has nothing above -inf counts for nothing.
//
// The sum over what is not listed is formed on its own (R, relative to its own largest value): as the difference
// of two sums it would be lost wherever the listed values make up nearly all.  So outside the list the gradient is
// one number per row times exp((s_v - base) / T), and the listed entries are stored after that.
struct DistillArgs {
    const int32_t* index;
    const float* top;
    const float* teacher_lse;            // or null
    const float* weight;                 // or null: 1 (the gradient call's is what came back for the losses)
    uint32_t k;
    float c, t;                          // log2(e) / T, T
    double inv_t;
};

// What the gradient of a row needs, besides its weight.  Listed entries: share * exp((s - top) / T) - p; a negative share:
// the row counts for nothing.  Others: scale * exp((s - base) / T), where, without the teacher's log-sum-exp, base is top
// and scale is share, and a and b are the two halves of log(sum over the slots of exp(t / T)); with it they are base and scale.
struct DistillStats {
    float a, b;
    float top, share;
    __device__ __forceinline__ float base(bool given) const { return given ? a : top; }
    __device__ __forceinline__ float scale(bool given) const { return given ? b : share; }
};

// The slots of a row, four to a lane of one wavefront.  What is made of them is in 64 bits: a loss is a small difference
// of logarithms of ten times its size, and these are k numbers of a row, not its vocabulary.
struct Slots {
    uint32_t index[4];                   // kNoSlot: does not count
    float t[4], s[4];                    // the teacher's and the student's logit
};
constexpr uint32_t kNoSlot = 0xffffffffu;

// (a logit of NaN is not above -inf)
__device__ __forceinline__ bool slot_counts(uint32_t index, float t, uint32_t vocab) { return index < vocab && t > -__builtin_inff(); }

template <typename T> __device__ __forceinline__ void slots_fetch(Slots& z, const DistillArgs& a, int64_t row, uint32_t vocab, const T* x) {
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t j = i * 64 + lane;
        z.index[i] = kNoSlot;
        z.t[i] = -__builtin_inff();
        if (j < a.k) {
            z.index[i] = (uint32_t)a.index[row * a.k + j];
            z.t[i] = a.top[row * a.k + j];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (!slot_counts(z.index[i], z.t[i], vocab)) z.index[i] = kNoSlot;
        z.s[i] = z.index[i] != kNoSlot ? (float)x[z.index[i]] : -__builtin_inff();
    }
}

// log(sum over the slots of exp(t / T)), or the teacher's own.
__device__ __forceinline__ double slots_norm(const Slots& z, const DistillArgs& a, int64_t row) {
    if (a.teacher_lse) return a.teacher_lse[row];
    float most = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (z.index[i] != kNoSlot) most = fmaxf(most, z.t[i]);
    const double shift = finite_base(wave_max(most));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * 64u < a.k && z.index[i] != kNoSlot) sum += exp(((double)z.t[i] - shift) * a.inv_t);
    return shift * a.inv_t + log(wave_sum(sum));
}

struct SlotRoom {
    uint32_t index[kTopMax];
    double p[kTopMax];
};

// Slots with the same index: which is the first of them, and the sum of their p.
__device__ __forceinline__ void slots_same(const Slots& z, const double (&p)[4], const DistillArgs& a, SlotRoom& room, bool (&first)[4], double (&sum)[4]) {
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        room.index[i * 64 + lane] = z.index[i];
        room.p[i * 64 + lane] = p[i];
        first[i] = z.index[i] != kNoSlot;
        sum[i] = 0.0;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 4
    for (uint32_t j = 0; j < a.k; ++j) {
        const uint32_t index = room.index[j];
        const double q = room.p[j];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i * 64u >= a.k) break;
            const bool same = z.index[i] == index;
            sum[i] += same ? q : 0.0;
            first[i] = first[i] && !(same && j < i * 64 + lane);
        }
    }
}

// What the list alone says, relative to its own largest logit: nothing here waits for the rest of the row.
struct ListSums {
    double norm, total, cross, listed;   // slots_norm; P; sum of p (log p - (s - peak) / T); sum over the listed entries of exp((s - peak) / T)
    float peak;                          // -inf where no slot counts
    bool any;
    double e[4], sum[4];                 // of a slot: exp((s - peak) / T), and if it is the first with its index the sum of their p
    bool first[4];
};

// `same`: some slots may have the same index.
__device__ __forceinline__ void list_sums(ListSums& l, const Slots& z, const DistillArgs& a, int64_t row, SlotRoom& room, bool same) {
    bool any = false;
    float peak = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        any |= z.index[i] != kNoSlot;
        peak = fmaxf(peak, z.s[i]);
    }
    l.any = __any(any);
    l.peak = wave_max(peak);
    l.norm = slots_norm(z, a, row);
    const double base = finite_base(l.peak);
    double p[4], total = 0.0, cross = 0.0, listed = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[i] = l.e[i] = 0.0;
        if (i * 64u >= a.k) continue;
        if (z.index[i] != kNoSlot) {
            const double y = ((double)z.s[i] - base) * a.inv_t, log_p = (double)z.t[i] * a.inv_t - l.norm;
            p[i] = exp(log_p);
            l.e[i] = exp(y);
            if (!(p[i] == 0.0)) cross += p[i] * (log_p - y);
        }
    }
    if (same) {
        slots_same(z, p, a, room, l.first, l.sum);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            l.first[i] = z.index[i] != kNoSlot;
            l.sum[i] = p[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        total += p[i];
        listed += l.first[i] ? l.e[i] : 0.0;
    }
    l.total = wave_sum(total);
    l.cross = wave_sum(cross);
    l.listed = wave_sum(listed);
}

// The row's loss (before its weight) and what its gradient needs, from the sum over what is not listed.  Even and odd lanes
// have one function each of two numbers worked out at a time.  (In 64 bits, for the weight may bring a loss that 32 do not hold,
// of a word masked by the lowest value, back among the numbers that they do.)
__device__ __forceinline__ double distill_row(const ListSums& l, ExpSum rest, const DistillArgs& a, DistillStats& st) {
    const bool odd = threadIdx.x & 1u;
    const float m = fmaxf(rest.base, l.peak), top = finite_base(m);
    const bool empty = rest.base == -__builtin_inff() && rest.sum == 0.0f;
    // (a list of nothing but -inf has no part in the sum: its exponential, of how far 0 lies above the others, may be infinite)
    const double below = l.peak == -__builtin_inff() ? 0.0 : ((double)l.peak - (double)top) * a.inv_t, rest_below = ((double)rest.base - (double)top) * a.inv_t;
    const double downs = exp(odd ? rest_below : below), down = empty ? 0.0 : lane_of(downs, 1);
    const double listed = l.listed * lane_of(downs, 0), r = rest.sum * down, sum = listed + r;
    const double logs = log(odd ? (double)rest.sum : sum), log_z = lane_of(logs, 0);
    double loss = l.cross + l.total * (log_z - below);
    const double of_sum = 1.0 / sum, share = listed * of_sum;          // (the latter is Q, of q)
    const double p_rest = a.teacher_lse ? fmax(1.0 - l.total, 0.0) : 0.0;
    const bool on = p_rest > 0.0 && !empty;
    st.top = top;
    if (a.teacher_lse) {
        st.a = finite_base(rest.base);
        if (on) {
            // (log q_rest and the difference q_rest - p_rest from the listed shares where these are the smaller part)
            const double ones = log1p(odd ? -l.total : -share);
            const double log_q = share < 0.5 ? lane_of(ones, 0) : lane_of(logs, 1) + rest_below - log_z;
            loss += p_rest * (lane_of(ones, 1) - log_q);
            st.b = (float)((share < 0.5 ? l.total - share : r * of_sum - p_rest) / rest.sum);
        } else {
            st.b = (float)(l.total * down * of_sum);
        }
    } else {
        st.a = (float)l.norm;
        st.b = (float)(l.norm - (double)st.a);
    }
    st.share = (float)((on ? l.total + p_rest : l.total) * of_sum);
    const bool none = !l.any || (m == -__builtin_inff() && sum == 0.0);
    if (none) st = {0.0f, 0.0f, 0.0f, -1.0f};
    return none ? 0.0 : loss * (double)a.t * (double)a.t;
}

// Gradient of the listed entries.
template <typename T>
__device__ __forceinline__ void store_list(const ListSums& l, const Slots& z, T* g, const DistillStats& st, float factor, const DistillArgs& a) {
    const double share = st.share * (l.peak == -__builtin_inff() ? 0.0 : exp(((double)l.peak - (double)st.top) * a.inv_t));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (l.first[i]) g[z.index[i]] = (T)(float)(factor * (share * l.e[i] - l.sum[i]));
}

// Marks the listed entries of the vectors [first, first + vecs) of a row, a byte to a vector, in words that have been
// cleared; by one wavefront.  Returns whether some slots have the same index.
__device__ __forceinline__ bool mark_listed(const Slots& z, uint32_t* marks, uint32_t lead, uint32_t first, uint32_t vecs) {
    bool same = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t at = z.index[i] + lead, vec = (at >> 3) - first, bit = 1u << ((vec & 3u) * 8u + (at & 7u));
        if (z.index[i] != kNoSlot && vec < vecs) same |= (atomicOr(&marks[vec >> 2], bit) & bit) != 0;
    }
    return __any(same);
}

// The values of a vector, -inf for those that are listed.
template <typename T> __device__ __forceinline__ void unlisted(float (&v)[8], const typename Vec8<T>::type& in, uint32_t mark) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)in[j];
    if (__any(mark))
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if ((mark >> j) & 1u) v[j] = -__builtin_inff();
}

constexpr int kAhead = 4;                // vectors of a thread whose loads are under way together

// Sum over the unlisted values of vectors [first, first + vecs) of a row.
template <typename T, int threads>
__device__ __forceinline__ ExpSum sum_unlisted(const Row<T>& x, uint32_t first, uint32_t vecs, const uint8_t* marks, float c) {
    ExpSum s = {-__builtin_inff(), 0.0f};
    for (uint32_t from = threadIdx.x; from < vecs; from += kAhead * threads) {
        typename Vec8<T>::type in[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) in[i] = x.load(first + min(from + i * threads, vecs - 1u));
        float v[kAhead][8], m = s.base;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t at = from + i * threads;
            unlisted<T>(v[i], in[i], at < vecs ? marks[at] : 0xffu);
            m = fmaxf(m, max8(v[i]));
        }
        const float b = finite_base(m);
        float sum = s.sum * exp_scaled(s.base - b, c);    // (a base of -inf goes with a sum of 0 or NaN)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = exp_scaled(v[i][j] - b, c);
            sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        }
        s = {m, sum};
    }
    return s;
}

// scale * exp((s - base) / T) for the vectors [first, first + vecs) of a row.
template <typename T, int threads>
__device__ __forceinline__ void store_unlisted(const Row<T>& x, T* g, uint32_t first, uint32_t vecs, float base, float scale, float c) {
    uint32_t from = threadIdx.x;
    for (; from + (kAhead - 1) * threads < vecs; from += kAhead * threads) {
        typename Vec8<T>::type in[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) in[i] = x.load(first + from + i * threads);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = scale * exp_scaled((float)in[i][j] - base, c);
            x.store(g, first + from + i * threads, v);
        }
    }
    for (; from < vecs; from += threads) {
        const typename Vec8<T>::type in = x.load(first + from);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = scale * exp_scaled((float)in[j] - base, c);
        x.store(g, first + from, v);
    }
}

template <typename T, int threads> __device__ __forceinline__ void store_zeros(const Row<T>& x, T* g, uint32_t first, uint32_t vecs) {
    const float v[8] = {};
    for (uint32_t i = threadIdx.x; i < vecs; i += threads) x.store(g, first + i, v);
}

constexpr int kRowThreads = 512, kRowWaves = kRowThreads / 64;      // of a long row
constexpr int kWindowVecs = 16384;       // vectors whose marks are held at once

struct DistillOut {
    float* loss;
    DistillStats* stats;                 // or null
};

__device__ __forceinline__ void leave_out(const DistillOut& out, int64_t row) {
    out.loss[row] = 0.0f;
    if (out.stats) out.stats[row] = {0.0f, 0.0f, 0.0f, -1.0f};
}

// A row of up to threads * n vectors to a workgroup, which reads it once: the values stay in registers, after the
// sum as their exponentials, which the gradient only scales.  One wavefront more than the row's looks after the
// list: it marks it before they need the marks, and its arithmetic (1 to 2 us of dependent steps in 64 bits) runs
// beside their sum.  (Row and list are kept apart down to the weight's test: with both under way across it 5555 x 10602
// took 84 registers instead of 80 and 69 us instead of 62.)  Memory bounds it where enough rows are under way: 700 x 10000 of
// 32 bits with the gradient 13.4 us (54 MB, 4.1 TB/s), 5555 x 10602 of 16 bits 60 us (228 MB, 3.8 TB/s; one row in 16 has
// weight 0 in these and the following figures, and is not read).
template <typename T, int n, int threads>
__global__ __launch_bounds__(threads + 64) void k_distill_row(const T* logits, int64_t ld, uint32_t vocab, DistillArgs a, DistillOut out, T* grad, int64_t ld_grad) {
    __shared__ __attribute__((aligned(16))) uint32_t marks[threads * n / 4];
    __shared__ SlotRoom room;
    __shared__ ExpSum sums[threads / 64];
    __shared__ DistillStats shared;
    const int64_t row = blockIdx.x;
    const Row<T> x(logits + row * ld, vocab);
    T* const g = grad ? grad + row * ld_grad : nullptr;
    const bool given = a.teacher_lse != nullptr;
    if (threadIdx.x >= threads) {
        Slots z;
        ListSums l;
        slots_fetch(z, a, row, vocab, logits + row * ld);       // (before the weight is known, as the row's loads below)
        const float weight = a.weight ? a.weight[row] : 1.0f;
        if (weight == 0.0f) {
            if (threadIdx.x == threads) leave_out(out, row);
            return;
        }
        for (uint32_t i = threadIdx.x & 63u; i < threads * n / 16u; i += 64u) reinterpret_cast<u32x4*>(marks)[i] = u32x4{0, 0, 0, 0};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const bool same = mark_listed(z, marks, x.lead, 0, x.vecs);
        __syncthreads();
        list_sums(l, z, a, row, room, same);
        __syncthreads();
        DistillStats st;
        const double loss = distill_row(l, block_sum(sums, threads / 64, a.c), a, st);
        if (threadIdx.x == threads) {
            out.loss[row] = (float)(weight * loss);
            if (out.stats) out.stats[row] = st;
            shared = st;
        }
        if (!g) return;
        __syncthreads();
        __syncthreads();
        if (!(st.share < 0.0f)) store_list(l, z, g, st, weight * a.t, a);
        return;
    }
    typename Vec8<T>::type in[n];
#pragma unroll
    for (int i = 0; i < n; ++i) in[i] = x.load(min(i * threads + threadIdx.x, x.vecs - 1u));
    const float weight = a.weight ? a.weight[row] : 1.0f;
    if (weight == 0.0f) {
        if (g) store_zeros<T, threads>(x, g, 0, x.vecs);
        return;
    }
    const float factor = weight * a.t;
    __syncthreads();
    float v[n][8], m = -__builtin_inff(), sum = 0.0f;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const uint32_t at = i * threads + threadIdx.x;
        unlisted<T>(v[i], in[i], at < x.vecs ? reinterpret_cast<const uint8_t*>(marks)[at] : 0xffu);
        m = fmaxf(m, max8(v[i]));
    }
    const float b = finite_base(m);
#pragma unroll
    for (int i = 0; i < n; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = exp_scaled(v[i][j] - b, a.c);
        sum += ((v[i][0] + v[i][1]) + (v[i][2] + v[i][3])) + ((v[i][4] + v[i][5]) + (v[i][6] + v[i][7]));
    }
    const ExpSum mine = wave_join({m, sum}, a.c);
    if ((threadIdx.x & 63u) == 0) sums[threadIdx.x >> 6] = mine;
    __syncthreads();
    if (!g) return;
    __syncthreads();
    const DistillStats st = shared;
    // (a row that counts for nothing has zeros whatever it holds; a thread of nothing but -inf has exponentials of 0 and
    // a base that says nothing)
    const bool none = st.share < 0.0f;
    const float f = none || m == -__builtin_inff() ? 0.0f : factor * st.scale(given) * exp_scaled(m - st.base(given), a.c);
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const uint32_t at = i * threads + threadIdx.x;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = none ? 0.0f : v[i][j] * f;
        if (at < x.vecs) x.store(g, at, v[i]);
    }
    __syncthreads();
}

// A longer row to a workgroup, read a second time for the gradient.  8192 x 131071 of 16 bits, the loss alone, 375 us (2.01 GB,
// 5.4 TB/s); with the gradient 1000 x 50000 61 us (194 MB from memory, the second reading from nearer caches).
template <typename T>
__global__ __launch_bounds__(kRowThreads) void k_distill(const T* logits, int64_t ld, uint32_t vocab, DistillArgs a, DistillOut out, T* grad, int64_t ld_grad) {
    __shared__ uint32_t marks[kWindowVecs / 4];
    __shared__ SlotRoom room;
    __shared__ ExpSum sums[kRowThreads / 64];
    __shared__ DistillStats shared;
    const int64_t row = blockIdx.x;
    const Row<T> x(logits + row * ld, vocab);
    const float weight = a.weight ? a.weight[row] : 1.0f;
    T* const g = grad ? grad + row * ld_grad : nullptr;
    if (weight == 0.0f) {
        if (threadIdx.x == 0) leave_out(out, row);
        if (g) store_zeros<T, kRowThreads>(x, g, 0, x.vecs);
        return;
    }
    Slots z;
    ListSums l;
    bool same = false;
    if (threadIdx.x < 64) slots_fetch(z, a, row, vocab, logits + row * ld);
    ExpSum s = {-__builtin_inff(), 0.0f};
    for (uint32_t first = 0; first < x.vecs; first += kWindowVecs) {
        const uint32_t some = min((uint32_t)kWindowVecs, x.vecs - first);
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < (some + 3u) / 4u; i += kRowThreads) marks[i] = 0;
        __syncthreads();
        if (threadIdx.x < 64) same |= mark_listed(z, marks, x.lead, first, some);
        __syncthreads();
        const ExpSum w = sum_unlisted<T, kRowThreads>(x, first, some, reinterpret_cast<const uint8_t*>(marks), a.c);
        const float m = fmaxf(s.base, w.base), b = finite_base(m);
        s = {m, s.sum * exp_scaled(s.base - b, a.c) + w.sum * exp_scaled(w.base - b, a.c)};
    }
    const ExpSum rest = block_join(s, sums, kRowWaves, a.c);
    if (threadIdx.x < 64) {
        list_sums(l, z, a, row, room, same);
        DistillStats st;
        const double loss = distill_row(l, rest, a, st);
        if (threadIdx.x == 0) {
            out.loss[row] = (float)(weight * loss);
            if (out.stats) out.stats[row] = st;
            shared = st;
        }
    }
    if (!g) return;
    __syncthreads();
    const DistillStats st = shared;
    if (st.share < 0.0f) {
        store_zeros<T, kRowThreads>(x, g, 0, x.vecs);
        return;
    }
    const bool given = a.teacher_lse != nullptr;
    const float factor = weight * a.t;
    store_unlisted<T, kRowThreads>(x, g, 0, x.vecs, st.base(given), factor * st.scale(given), a.c);
    __syncthreads();
    if (threadIdx.x < 64) store_list(l, z, g, st, factor, a);
}

// Few long rows: a part of a row to a workgroup, whose sum goes to part_sums (one row of 131072 with its gradient 17.7 us
// for the three launches, which bound it), ...
constexpr int kPartThreads = 256;
constexpr int kPartMost = 2048;          // vectors of a part

template <typename T>
__global__ __launch_bounds__(kPartThreads) void k_distill_part(const T* __restrict__ logits, int64_t ld, uint32_t vocab, DistillArgs a, uint32_t parts, uint32_t part_vecs,
                                                              ExpSum* __restrict__ part_sums) {
    __shared__ uint32_t marks[kPartMost / 4];
    __shared__ ExpSum sums[kPartThreads / 64];
    const int64_t row = blockIdx.x / parts;
    const Row<T> x(logits + row * ld, vocab);
    const uint32_t first = (blockIdx.x % parts) * part_vecs;
    if (a.weight && a.weight[row] == 0.0f) return;
    if (first >= x.vecs) {
        if (threadIdx.x == 0) part_sums[blockIdx.x] = {-__builtin_inff(), 0.0f};
        return;
    }
    const uint32_t vecs = min(part_vecs, x.vecs - first);
    for (uint32_t i = threadIdx.x; i < (vecs + 3u) / 4u; i += kPartThreads) marks[i] = 0;
    __syncthreads();
    if (threadIdx.x < a.k) {
        const uint32_t index = (uint32_t)a.index[row * a.k + threadIdx.x], at = index + x.lead, vec = (at >> 3) - first;
        if (slot_counts(index, a.top[row * a.k + threadIdx.x], vocab) && vec < vecs) atomicOr(&marks[vec >> 2], 1u << ((vec & 3u) * 8u + (at & 7u)));
    }
    __syncthreads();
    const ExpSum s = block_join(sum_unlisted<T, kPartThreads>(x, first, vecs, reinterpret_cast<const uint8_t*>(marks), a.c), sums, kPartThreads / 64, a.c);
    if (threadIdx.x == 0) part_sums[blockIdx.x] = s;
}

// ... a wavefront per row, which makes the loss of them, ...
template <typename T>
__global__ __launch_bounds__(64) void k_distill_join(const T* __restrict__ logits, int64_t ld, uint32_t vocab, DistillArgs a, uint32_t parts, const ExpSum* __restrict__ part_sums,
                                                     DistillOut out) {
    __shared__ SlotRoom room;
    const int64_t row = blockIdx.x;
    const float weight = a.weight ? a.weight[row] : 1.0f;
    if (weight == 0.0f) {
        if (threadIdx.x == 0) leave_out(out, row);
        return;
    }
    Slots z;
    slots_fetch(z, a, row, vocab, logits + row * ld);
    ExpSum s = {-__builtin_inff(), 0.0f};
    for (uint32_t p = threadIdx.x; p < parts; p += 64u) {
        const ExpSum q = part_sums[row * parts + p];
        const float m = fmaxf(s.base, q.base), b = finite_base(m);
        s = {m, s.sum * exp_scaled(s.base - b, a.c) + q.sum * exp_scaled(q.base - b, a.c)};
    }
    ListSums l;
    list_sums(l, z, a, row, room, true);
    DistillStats st;
    const double loss = distill_row(l, wave_join(s, a.c), a, st);
    if (threadIdx.x == 0) {
        out.loss[row] = (float)(weight * loss);
        if (out.stats) out.stats[row] = st;
    }
}

// ... and parts again for the gradient from what the loss left, in this call or a later one.  As in k_distill_row the list
// has a wavefront of its own, which has the values ready when the others have stored theirs.  8192 x 131071 of 16 bits 800 us
// (4.16 GB read and written, 5.2 TB/s: memory).
template <typename T>
__global__ __launch_bounds__(kPartThreads + 64) void k_distill_grad(const T* logits, int64_t ld, uint32_t vocab, DistillArgs a, const DistillStats* __restrict__ stats,
                                                                   uint32_t parts, uint32_t part_vecs, T* grad, int64_t ld_grad) {
    __shared__ __attribute__((aligned(16))) uint32_t marks[kPartMost / 4];
    __shared__ SlotRoom room;
    const int64_t row = blockIdx.x / parts;
    const Row<T> x(logits + row * ld, vocab);
    const uint32_t first = (blockIdx.x % parts) * part_vecs;
    if (first >= x.vecs) return;
    const uint32_t vecs = min(part_vecs, x.vecs - first);
    const float weight = a.weight ? a.weight[row] : 1.0f;
    const DistillStats st = stats[row];
    T* const g = grad + row * ld_grad;
    if (weight == 0.0f || st.share < 0.0f) {
        store_zeros<T, kPartThreads + 64>(x, g, first, vecs);
        return;
    }
    const bool given = a.teacher_lse != nullptr, in_place = logits == grad;
    const float factor = weight * a.t;
    if (threadIdx.x < kPartThreads) {
        if (in_place) __syncthreads();                          // (the listed logits of this part have been read)
        store_unlisted<T, kPartThreads>(x, g, first, vecs, st.base(given), factor * st.scale(given), a.c);
        __syncthreads();
        return;
    }
    Slots z;
    slots_fetch(z, a, row, vocab, logits + row * ld);
    for (uint32_t i = threadIdx.x & 63u; i < (vecs + 15u) / 16u; i += 64u) reinterpret_cast<u32x4*>(marks)[i] = u32x4{0, 0, 0, 0};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    bool here[4], same = mark_listed(z, marks, x.lead, first, vecs);
    const double norm = given ? (double)a.teacher_lse[row] : (double)st.a + (double)st.b;
    double p[4], sum[4];
    float own[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        here[i] = z.index[i] != kNoSlot && ((z.index[i] + x.lead) >> 3) - first < vecs;
        p[i] = i * 64u < a.k && here[i] ? exp((double)z.t[i] * a.inv_t - norm) : 0.0;
        own[i] = z.s[i];
        sum[i] = p[i];
    }
    if (in_place) __syncthreads();
    if (same) {
        bool stands[4];
        slots_same(z, p, a, room, stands, sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) here[i] = here[i] && stands[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * 64u < a.k && here[i]) own[i] = (float)(factor * ((double)st.share * exp(((double)own[i] - (double)st.top) * a.inv_t) - sum[i]));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (here[i]) g[z.index[i]] = (T)own[i];
}

}  // namespace sbc
