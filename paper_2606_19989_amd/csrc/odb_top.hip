// The most probable tokens of every position of a tile, with log-probabilities, entropy and the label's rank.
//
// One pass over a position's logits forms the largest, the sum of exponentials and, for the entropy, their
// weighted logs, as the label's log-probability does.  Beside it the k largest are found by a bound that only
// few logits pass: with k cells of columns whose largest reach it, the row's k-th largest does not fall below
// it.  A 16-byte group with a logit above the bound is set aside whole, in LDS, for about ten instructions;
// behind the pass the groups are looked at once, under the last and highest bound, which leaves 1 to 2 k keys.
// Their k largest are picked by the digits of the keys where they are many, and ordered by counting.
// A key holds the logit, mapped to a whole number that grows with it, above the complement of the column: keys
// are never equal, and of equal logits the first column's is the largest.
// Where the room does not do (rows in ascending order, or with thousands of equal logits at the bound), the row
// is gone through again, above the k-th largest key so far.
//
// Bound by the reads of the logits and, about as much, by the instructions: nine a logit as without the
// alternatives (an exponential counts four), one more for its group's largest.  4,096 positions of 151,936 bf16
// logits, k = 64: 203 us (5.9 TB/s of reads; 182 without alternatives).
#include <algorithm>

#include "odb_vocab.h"

namespace odb {

namespace {

typedef unsigned long long u64;

constexpr int kBins = 256;      // of a digit
// Alternatives from which on a wave's cells are half a group of a thread's, 512, and not its 64 threads.  k = 20 / 32
// / 40 / 56 of 36,621 positions of 8,192 bf16 logits: 130 / 135 / 151 / 464 us with threads, 170 / 177 / 182 / 190 with
// half groups; of 1,024 logits (131,072 positions) 157 / 186 / 238 / 365 and 215 / 232 / 241 / 283.
constexpr int kFine = 32;
constexpr float kNone = -HUGE_VALF;

template <typename T>
__device__ __forceinline__ float lowest_of();
template <>
__device__ __forceinline__ float lowest_of<float>() { return kLowest; }
template <>
__device__ __forceinline__ float lowest_of<bf16_t>() { return -3.38953138925153547590470800371487867e38f; }
template <>
__device__ __forceinline__ float lowest_of<fp16_t>() { return -65504.0f; }

// Logits to whole numbers of the same order; -0 is 0.
__device__ __forceinline__ uint32_t ordered(float f) {
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ u64 key_of(float f, int64_t v) { return (u64)ordered(f) << 32 | (uint32_t)~(uint32_t)v; }
__device__ __forceinline__ float logit_of(u64 key) { return unordered((uint32_t)(key >> 32)); }
__device__ __forceinline__ int32_t column_of(u64 key) { return (int32_t)~(uint32_t)key; }

struct TopArgs {
    odb_logits_t x;
    const int32_t* labels;
    int32_t* ids;
    float* top;
    float* logprob;
    int32_t* rank;
    float* stats;
    float* entropy;
    int32_t* status;
    int32_t k;
    int32_t parts;          // blocks of a position, where it is more than one
    int64_t part_len;       // their columns
    struct Part* part;      // [positions * parts]
    u64* part_key;          // [positions * parts * 2 k]
};

// What a block leaves of its part of a position's columns, beside its candidates.
struct Part {
    Acc acc;
    float zy;               // the label's logit
    uint32_t ahead;
    int32_t n;              // candidates, in any order
};

// A group's LDS.
template <int G>
struct Room {
    static constexpr int kWaves = G / kWave;
    static constexpr int kHits = G == kWave ? 192 : 1024;
    static constexpr int kKeys = G == kWave ? 256 : 512;            // all multiples of 8
    static constexpr int kFew = G == kWave ? 128 : 256;             // candidates that are ordered by counting
    static constexpr int kHold = kHits * 20 / 8 + kKeys;            // the second way's candidates
    static_assert(kHold >= ODB_LIST_MAX + G * 8 && kHold % 8 == 0, "k of them and a step's");
    union {
        struct {
            uint4 hit[kHits];           // groups of 16 bytes with a candidate in them
            uint32_t hit_at[kHits];     // their first columns
            u64 key[kKeys];             // candidates
        };
        u64 hold[kHold];
    };
    u64 few[kFew];
    u64 top[ODB_LIST_MAX];
    uint32_t bins[kBins];
    uint32_t bound[kWaves];
    Acc acc[kWaves];
    u64 differ;
    uint32_t hits, count, few_count, ahead;
};

// The largest whole number with its low 16 bits 0 that `kth` of the wave's C numbers a lane reach.
template <int C>
__device__ __forceinline__ uint32_t wave_kth(const uint32_t* o, int kth) {
    uint32_t r = 0;
#pragma unroll(C == 1 ? 16 : 1)
    for (int i = 31; i >= 16; --i) {
        const uint32_t bit = 1u << i;
        int n = 0;
#pragma unroll
        for (int j = 0; j < C; ++j) n += __builtin_popcountll(__ballot(o[j] >= (r | bit)));
        if (n >= kth) r |= bit;
    }
    return r;
}

// The k largest of a list's n keys, ordered, to s.top; fewer if n < k.  The list has room for n rounded up to
// eight.  The group has met before, and meets at the end.
template <int G>
__device__ __forceinline__ void pick(Room<G>& s, u64* list, int n, int k) {
    constexpr int kFew = Room<G>::kFew;
    const int t = threadIdx.x & (G - 1), lane = threadIdx.x & (kWave - 1);
    if (G > kWave && n > kFew) {
        // a bound as in the pass, with the threads' largest keys for cells (a wave has too few for many alternatives)
        uint32_t o = 0;
        for (int i = t; i < n; i += G) {
            const uint32_t high = (uint32_t)(list[i] >> 32);
            o = high > o ? high : o;
        }
        o = wave_kth<1>(&o, (k + Room<G>::kWaves - 1) / Room<G>::kWaves);
        if (t == 0) s.few_count = 0;
        if (lane == 0) s.bound[t / kWave] = o;
        group_sync<G>();
#pragma unroll
        for (int i = 0; i < Room<G>::kWaves; ++i) o = s.bound[i] < o ? s.bound[i] : o;
        for (int i = t; i < n; i += G) {
            const u64 key = list[i];
            if ((uint32_t)(key >> 32) < o) continue;
            const uint32_t to = atomicAdd(&s.few_count, 1u);
            if (to < (uint32_t)kFew) s.few[to] = key;
        }
        group_sync<G>();
    }
    const int cut = G > kWave && n > kFew ? (int)s.few_count : kFew + 1;
    if (cut <= kFew) {
        n = cut;
        list = s.few;
    } else if (n > kFew) {
        // digits of 8 bits from the highest bit that differs
        if (t == 0) s.differ = 0;
        group_sync<G>();
        const u64 first = list[0];
        u64 differ = 0;
        for (int i = t; i < n; i += G) differ |= list[i] ^ first;
#pragma unroll
        for (int d = kWave / 2; d > 0; d >>= 1) differ |= __shfl_xor(differ, d, kWave);
        if (lane == 0) atomicOr(&s.differ, differ);
        group_sync<G>();
        differ = s.differ;
        int top = 64 - __builtin_clzll(differ);       // n > 1 keys differ: 1 to 64 low bits are open
        u64 fixed = top == 64 ? 0 : first >> top << top;
        int above = 0;                                // candidates above the digits found so far
        for (;;) {
            const int low = top > 8 ? top - 8 : 0;
            for (int i = t; i < kBins; i += G) s.bins[i] = 0;
            group_sync<G>();
            const u64 mask = top == 64 ? 0 : ~0ull << top;
            for (int i = t; i < n; i += G) {
                const u64 key = list[i];
                if ((key & mask) == fixed) atomicAdd(&s.bins[(uint32_t)(key >> low) & (kBins - 1)], 1u);
            }
            group_sync<G>();
            // four bins a lane from the highest down: where do they reach k?
            int c[4], sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += c[j] = (int)s.bins[kBins - 1 - 4 * lane - j];
            int until = sum;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const int o = __shfl_up(until, d, kWave);
                if (lane >= d) until += o;
            }
            const int at = __builtin_ctzll(__ballot(above + until >= k));     // exists: n >= kFew >= k
            int before = above + until - sum, with = before + c[0], bin = kBins - 1 - 4 * lane;
#pragma unroll
            for (int j = 1; j < 4; ++j) {
                if (with < k) {
                    before = with;
                    with += c[j];
                    --bin;
                }
            }
            with = __shfl(with, at, kWave);
            above = __shfl(before, at, kWave);
            fixed |= (u64)__shfl(bin, at, kWave) << low;
            top = low;
            if (with <= kFew || low == 0) break;
            group_sync<G>();
        }
        if (t == 0) s.few_count = 0;
        group_sync<G>();
        for (int i = t; i < n; i += G) {
            const u64 key = list[i];
            if (key >= fixed) s.few[atomicAdd(&s.few_count, 1u)] = key;
        }
        group_sync<G>();
        n = (int)s.few_count;
        list = s.few;
    }
    // Whole steps of eight: keys of 0 are behind all others.  As many threads count one key's place as there are.
    if (t < 8 && n + t < ((n + 7) & ~7)) list[n + t] = 0;
    group_sync<G>();
    int by = 0;     // 2^by threads
    while (G > kWave && (n << (by + 1)) <= G && by < 3) ++by;
    for (int i = t >> by; i < n; i += G >> by) {
        const u64 mine = list[i];
        int place = 0;
        for (int j = 8 * (t & ((1 << by) - 1)); j < n; j += 8 << by) {
#pragma unroll
            for (int u = 0; u < 8; ++u) place += list[j + u] > mine;
        }
        for (int d = 0; d < by; ++d) place += __shfl_xor(place, 1 << d, kWave);
        if (place < k) s.top[place] = mine;
    }
    group_sync<G>();
}

// Columns [v0, v1) of a row: the joined triple, the columns ahead of the label (s.ahead), and in s.key the *n
// candidates, the k largest among them, or *n > kKeys.  All of the group's threads get the same.
template <typename T, bool ENT, bool RANK, bool FINE, int G>
__device__ __forceinline__ Acc scan(const T* z, int64_t v0, int64_t v1, int32_t y, float zy, int kk, float k, Room<G>& s,
                                    int* n) {
    constexpr int N = Vec<T>::N;
    constexpr int kWavesIn = G / kWave;
    const int t = threadIdx.x & (G - 1), lane = threadIdx.x & (kWave - 1);
    const uint32_t none = ordered(lowest_of<T>());
    const int share = (kk + kWavesIn - 1) / kWavesIn;      // cells of each wave that make k
    if (t == 0) s.hits = s.count = s.ahead = 0;
    group_sync<G>();
    Acc r{kLowest, 0.0f, 0.0f};
    int ahead = 0;
    const int64_t whole = v0 + (v1 - v0) / N * N;
    auto load = [&](Vec<T>* w, int64_t v) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) w[j] = load_vec<true>(z + at_most(v + j * G * N, whole - N));
    };
    // a 16-byte group: its sums, its place beside the label's, and its largest
    auto take = [&](const Vec<T>& w, int64_t v, float* cell) __attribute__((always_inline)) {
        float f[N], half[2] = {kNone, kNone};
#pragma unroll
        for (int e = 0; e < N; ++e) {
            f[e] = (float)w.v[e];
            half[2 * e / N] = fmaxf(half[2 * e / N], f[e]);
        }
        if (FINE) {
            cell[0] = fmaxf(cell[0], half[0]);
            cell[1] = fmaxf(cell[1], half[1]);
        }
        const float most = fmaxf(half[0], half[1]);
        if (most > r.m) acc_rescale<ENT>(r, most, k);
#pragma unroll
        for (int e = 0; e < N; ++e) acc_term<ENT>(r, f[e], k);
        if (RANK) {
            if (v > y) {
#pragma unroll
                for (int e = 0; e < N; ++e) ahead += f[e] > zy;
            } else if (v + N <= y) {
#pragma unroll
                for (int e = 0; e < N; ++e) ahead += f[e] >= zy;
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) ahead += f[e] > zy || (f[e] == zy && v + e < y);
            }
        }
        return most;
    };
    auto limit_of = [&](uint32_t o) __attribute__((always_inline)) {
        return o > none + 1 ? unordered(o - 1 - (o - 1 == 0x7fffffffu)) : unordered(none);
    };
    // The bound is what `share` cells of every wave reach, a cell being the largest that one half of one of a
    // thread's groups has held in any round, or, for few, a thread; candidates are above the number below it.
    // Until there is one the group meets behind every round; then the waves go on by
    // themselves and form it anew whenever their rounds have doubled, and in the last: what a wave has left is
    // true whenever another reads it.
    volatile uint32_t* const of = s.bound;
    uint32_t met = 0;
    float cell[2 * kAhead];
#pragma unroll
    for (int j = 0; j < 2 * kAhead; ++j) cell[j] = kNone;
    float limit = unordered(none);
    int rounds = 0;
    int64_t v = v0 + (int64_t)t * N;
    Vec<T> next[kAhead];
    if (v0 < whole) load(next, v);
    for (int64_t at = v0; at < whole; at += kAhead * G * N, v += kAhead * G * N) {     // uniform
        Vec<T> w[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) w[j] = next[j];
        const bool last = at + kAhead * G * N >= whole;
        if (!last) load(next, v + kAhead * G * N);     // under way beside this round
        float most[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) most[j] = v + j * G * N < whole ? take(w[j], v + j * G * N, cell + 2 * j) : kNone;
        ++rounds;
        const bool meet = met <= none;
        if (meet || last || (rounds & (rounds - 1)) == 0) {
            uint32_t o, c[2 * kAhead];
            if (FINE) {
#pragma unroll
                for (int j = 0; j < 2 * kAhead; ++j) c[j] = ordered(cell[j]);
                o = wave_kth<2 * kAhead>(c, share);
            } else {
                c[0] = ordered(r.m);
                o = wave_kth<1>(c, share);
            }
            if (G > kWave) {
                if (lane == 0) of[threadIdx.x / kWave] = o;
                if (meet) __syncthreads();
#pragma unroll
                for (int i = 0; i < kWavesIn; ++i) {
                    const uint32_t other = of[i];
                    o = other < o ? other : o;
                }
                if (meet) __syncthreads();
            }
            if (meet) met = o;
            limit = limit_of(o);
        }
        int found = 0;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) found += most[j] > limit;
        if (found) {
            uint32_t to = atomicAdd(&s.hits, (uint32_t)found);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (most[j] > limit) {
                    if (to < (uint32_t)Room<G>::kHits) {
                        __builtin_memcpy(&s.hit[to], &w[j], 16);
                        s.hit_at[to] = (uint32_t)(v + j * G * N);
                    }
                    ++to;
                }
            }
        }
    }
    if (whole + t < v1) {
        const float f = (float)z[whole + t];
        if (f > r.m) acc_rescale<ENT>(r, f, k);
        acc_term<ENT>(r, f, k);
        if (RANK) ahead += f > zy || (f == zy && whole + t < y);
        if (f > limit) {
            const uint32_t to = atomicAdd(&s.count, 1u);
            if (to < (uint32_t)Room<G>::kKeys) s.key[to] = key_of(f, whole + t);
        }
    }
    if (RANK) {
#pragma unroll
        for (int d = kWave / 2; d > 0; d >>= 1) ahead += __shfl_xor(ahead, d, kWave);
        if (lane == 0) atomicAdd(&s.ahead, (uint32_t)ahead);
    }
    r = group_join<ENT, G>(r, s.acc, k);
    group_sync<G>();
    // what of the groups is above the last bound
    uint32_t o = s.bound[0];
#pragma unroll
    for (int i = 1; i < kWavesIn; ++i) o = s.bound[i] < o ? s.bound[i] : o;
    if (G > kWave && v0 < whole) limit = limit_of(o);
    const int hits = (int)s.hits, found = hits <= Room<G>::kHits ? hits * N : 0;
    const T* const of_hits = reinterpret_cast<const T*>(s.hit);
    for (int i = t; i < found; i += G) {
        const float f = (float)of_hits[i];
        if (f > limit) {
            const uint32_t to = atomicAdd(&s.count, 1u);
            if (to < (uint32_t)Room<G>::kKeys) s.key[to] = key_of(f, s.hit_at[i / N] + i % N);
        }
    }
    group_sync<G>();
    *n = hits > Room<G>::kHits ? Room<G>::kKeys + 1 : (int)s.count;
    return r;
}

// The k largest of columns [v0, v1), ordered, to s.top, and how many there are, from a list of n candidates that
// scan left.  Where its room did not do, or fewer than k columns are above the type's lowest value, which masks
// columns and is no candidate there, the row is gone through again, a load a step, above the k-th largest so far.
template <typename T, int G>
__device__ __forceinline__ int largest(const T* z, int64_t v0, int64_t v1, int kk, int n, Room<G>& s) {
    constexpr int N = Vec<T>::N;
    constexpr int kFull = Room<G>::kHold - G * N;
    const int t = threadIdx.x & (G - 1);
    const bool again = n > Room<G>::kKeys || n < kk;
    const int64_t whole = v0 + (v1 - v0) / N * N;
    u64* const list = again ? s.hold : s.key;
    u64 least = 0;
    int64_t v = v0 + (int64_t)t * N, at = v0;
    if (again) n = 0;
    for (;;) {      // uniform: one round unless the row is gone through again
        if (again) {
            group_sync<G>();
            if (t == 0) s.count = n;
            Vec<T> next{};
            if (v < whole) next = load_vec<false>(z + v);
            while (at < v1 && n <= kFull) {
                const Vec<T> w = next;
                if (v + G * N < whole) next = load_vec<false>(z + v + G * N);
                group_sync<G>();
                float f[N];
                uint32_t on = 0;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[e] = v < whole ? (float)w.v[e] : v + e < v1 ? (float)z[v + e] : kNone;
                    on |= (uint32_t)(f[e] > kNone && key_of(f[e], v + e) > least) << e;
                }
                if (on) {
                    uint32_t to = atomicAdd(&s.count, (uint32_t)__builtin_popcount(on));
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        if (on >> e & 1) {
                            if (to < (uint32_t)Room<G>::kHold) s.hold[to] = key_of(f[e], v + e);     // always
                            ++to;
                        }
                    }
                }
                group_sync<G>();
                n = (int)s.count;
                at += G * N;
                v += G * N;
            }
            group_sync<G>();
        }
        pick(s, list, n, kk);
        if (n > kk) n = kk;
        if (!again || at >= v1) return n;
        for (int i = t; i < n; i += G) s.hold[i] = s.top[i];
        if (n == kk) least = s.top[kk - 1];
    }
}

// A token's outputs from the joined triple and the n <= k largest, ordered, in s.top.
template <bool ENT, bool RANK, int G>
__device__ __forceinline__ void leave(const TopArgs& A, int64_t q, const Acc& r, float zy, int n, const Room<G>& s) {
    const int t = threadIdx.x & (G - 1);
    const float a = (float)A.x.scale, lse = logf(r.s);
    const bool sound = r.s > 0.0f && r.s < HUGE_VALF;      // a NaN or +inf among the logits, or none above -inf
    for (int j = t; j < A.k; j += G) {
        const bool there = sound && j < n;
        const u64 key = there ? s.top[j] : 0;
        A.ids[q * A.k + j] = there ? column_of(key) : ODB_LABEL_IGNORE;
        A.top[q * A.k + j] = there ? (logit_of(key) - r.m) * a - lse : sound ? kNone : __builtin_nanf("");
    }
    if (t == 0) {
        if (A.logprob) A.logprob[q] = (zy - r.m) * a - lse;
        if (RANK) A.rank[q] = sound ? (int32_t)s.ahead : -1;
        if (A.stats) reinterpret_cast<float2*>(A.stats)[q] = make_float2(r.m, lse);
        if (ENT) A.entropy[q] = lse - r.t / r.s * kLn2;
    }
}

template <bool ENT, bool RANK, int G>
__device__ __forceinline__ void leave_none(const TopArgs& A, int64_t q) {
    const int t = threadIdx.x & (G - 1);
    for (int j = t; j < A.k; j += G) {
        A.ids[q * A.k + j] = ODB_LABEL_IGNORE;
        A.top[q * A.k + j] = kNone;
    }
    if (t == 0) {
        if (A.logprob) A.logprob[q] = 0.0f;
        if (RANK) A.rank[q] = -1;
        if (A.stats) reinterpret_cast<float2*>(A.stats)[q] = make_float2(0.0f, 0.0f);
        if (ENT) A.entropy[q] = 0.0f;
    }
}

// A group of G threads, a wave or a block, takes a position.
template <typename T, bool ENT, bool RANK, bool FINE, int G>
__global__ void __launch_bounds__(kBlock, 4) top_kernel(TopArgs A) {
    static_assert(G == kWave || G == kBlock, "a wave or a block");
    __shared__ Room<G> s_room[kBlock / G];
    Room<G>& s = s_room[threadIdx.x / G];
    const odb_logits_t& x = A.x;
    const int64_t n = x.rows * x.cols, V = x.vocab;
    const int t = threadIdx.x & (G - 1);
    const float k = (float)x.scale * kLog2e;
    for (int64_t q = (int64_t)blockIdx.x * (kBlock / G) + threadIdx.x / G; q < n;
         q += (int64_t)gridDim.x * (kBlock / G)) {   // uniform over a group
        const uint32_t i = (uint32_t)q / (uint32_t)x.cols, c = (uint32_t)q - i * (uint32_t)x.cols;
        const int32_t y = c < (uint32_t)x.shift ? -1 : A.labels ? read_label(A.labels, q, V, A.status, t == 0) : 0;
        if (y < 0) {
            leave_none<ENT, RANK, G>(A, q);
            continue;
        }
        const T* z = static_cast<const T*>(x.d_logits) + (int64_t)i * x.row_stride +
                     (int64_t)(c - (uint32_t)x.shift) * x.col_stride;
        const float zy = (float)z[y];
        int have;
        const Acc r = scan<T, ENT, RANK, FINE, G>(z, 0, V, y, zy, A.k, k, s, &have);
        have = largest(z, 0, V, A.k, have, s);
        leave<ENT, RANK, G>(A, q, r, zy, have, s);
        group_sync<G>();     // the next position writes where this one's are read
    }
}

// Few positions: a block takes one of a position's parts, and leaves what it found in the workspace.
template <typename T, bool ENT, bool RANK, bool FINE>
__global__ void __launch_bounds__(kBlock) top_part_kernel(TopArgs A) {
    __shared__ Room<kBlock> s;
    const odb_logits_t& x = A.x;
    const int64_t V = x.vocab;
    const int64_t q = blockIdx.x / A.parts;
    const int64_t v0 = (blockIdx.x - q * A.parts) * A.part_len, v1 = v0 + A.part_len < V ? v0 + A.part_len : V;
    const uint32_t i = (uint32_t)q / (uint32_t)x.cols, c = (uint32_t)q - i * (uint32_t)x.cols;
    const int32_t y =
        c < (uint32_t)x.shift ? -1 : A.labels ? read_label(A.labels, q, V, A.status, threadIdx.x == 0) : 0;
    if (y < 0) return;
    const T* z = static_cast<const T*>(x.d_logits) + (int64_t)i * x.row_stride +
                 (int64_t)(c - (uint32_t)x.shift) * x.col_stride;
    const float zy = (float)z[y];
    int n;
    const Acc r = scan<T, ENT, RANK, FINE, kBlock>(z, v0, v1, y, zy, A.k, (float)x.scale * kLog2e, s, &n);
    const u64* from = s.key;
    if (n < A.k || n > 2 * A.k) {
        n = largest(z, v0, v1, A.k, n, s);
        from = s.top;
    }
    u64* to = A.part_key + (int64_t)blockIdx.x * 2 * A.k;
    for (int j = threadIdx.x; j < n; j += kBlock) to[j] = from[j];
    if (threadIdx.x == 0) A.part[blockIdx.x] = {r, zy, s.ahead, n};
}

// A position from its parts, in their order.
template <bool ENT, bool RANK>
__global__ void __launch_bounds__(kBlock) top_join_kernel(TopArgs A) {
    __shared__ Room<kBlock> s;
    const odb_logits_t& x = A.x;
    const int64_t q = blockIdx.x;
    const uint32_t c = (uint32_t)q % (uint32_t)x.cols;
    const int32_t y = c < (uint32_t)x.shift ? -1 : A.labels ? read_label(A.labels, q, x.vocab, A.status, false) : 0;
    if (y < 0) return leave_none<ENT, RANK, kBlock>(A, q);
    const float k = (float)x.scale * kLog2e;
    const Part* part = A.part + q * A.parts;
    // a part a lane, in every wave; their candidates behind each other
    const int lane = threadIdx.x & (kWave - 1);
    Part w{{kLowest, 0.0f, 0.0f}, 0.0f, 0, 0};
    if (lane < A.parts) w = part[lane];
    const u64* from = A.part_key + q * A.parts * 2 * A.k;
    int n = w.n;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(n, d, kWave);
        if (lane >= d) n += o;
    }
    if (threadIdx.x < kWave) {
        s.bins[lane] = (uint32_t)(n - w.n);
        s.bins[kWave + lane] = (uint32_t)w.n;
    }
    n = __shfl(n, kWave - 1, kWave);
    const float zy = __shfl(w.zy, 0, kWave);
    const Acc r = group_join<ENT, kWave>(w.acc, nullptr, k);
#pragma unroll
    for (int d = kWave / 2; d > 0; d >>= 1) w.ahead += __shfl_xor(w.ahead, d, kWave);
    if (threadIdx.x == 0) s.ahead = w.ahead;
    __syncthreads();
    for (int i = threadIdx.x; i < A.parts * 2 * A.k; i += kBlock) {
        const int p = i / (2 * A.k), j = i - p * 2 * A.k;
        if (j < (int)s.bins[kWave + p]) s.hold[s.bins[p] + j] = from[i];
    }
    __syncthreads();
    pick(s, s.hold, n, A.k);
    leave<ENT, RANK, kBlock>(A, q, r, zy, n < A.k ? n : A.k, s);
}

template <typename T, bool ENT, bool RANK>
void launch(const TopArgs& a, hipStream_t s) {
    const int64_t n = a.x.rows * a.x.cols;
    if (a.parts > 1) {
        hipLaunchKernelGGL((a.k > kWave ? top_part_kernel<T, ENT, RANK, true> : top_part_kernel<T, ENT, RANK, false>),
                           dim3((unsigned)(n * a.parts)), dim3(kBlock), 0, s, a);
        hipLaunchKernelGGL((top_join_kernel<ENT, RANK>), dim3((unsigned)n), dim3(kBlock), 0, s, a);
        return;
    }
    // A wave or a block takes a position, by the bytes of its logits.  A wave leaves four positions to a block, so
    // that one's wait behind its pass is another's reading; a block of four waves has cells for more alternatives,
    // and needs 4 KB for all of its threads to have any.  us for 600 MB of bf16 logits, k = 5 / 20 / 64 / 128:
    //   logits a row    wave                        block
    //   1,024           272 / 314 /  631 / 1349     4815 / 4815 / 4823 / 5253
    //   2,048           177 / 199 /  369 /  783      690 /  711 /  865 / 1596
    //   4,096           139 / 152 /  277 /  566      366 /  377 /  459 /  812
    //   8,192           126 / 126 /  204 / 1123      207 /  214 /  254 /  425
    //   16,384          112 / 116 /  413 /  771      154 /  157 /  175 /  302
    //   32,768          117 / 123 /  381 /  609      123 /  124 /  136 /  214
    //   65,536          135 / 142 /  408 /  578      116 /  115 /  121 /  162
    const int64_t row = a.x.vocab * (int64_t)sizeof(T);
    const bool wave = row <= 4096 || (n > 2 * num_cus() && row <= (a.k <= kFine ? 32768 : a.k <= kWave ? 16384 : 8192));
    if (wave)
        hipLaunchKernelGGL((a.k > kFine ? top_kernel<T, ENT, RANK, true, kWave> : top_kernel<T, ENT, RANK, false, kWave>),
                           dim3(grid_for(n, kBlock / kWave)), dim3(kBlock), 0, s, a);
    else
        hipLaunchKernelGGL((a.k > kWave ? top_kernel<T, ENT, RANK, true, kBlock> : top_kernel<T, ENT, RANK, false, kBlock>),
                           dim3(grid_for(n, 1)), dim3(kBlock), 0, s, a);
}

template <typename T>
void launch(const TopArgs& a, hipStream_t s) {
    if (a.entropy)
        a.rank ? launch<T, true, true>(a, s) : launch<T, true, false>(a, s);
    else
        a.rank ? launch<T, false, true>(a, s) : launch<T, false, false>(a, s);
}

int check_top(const odb_logits_t* x, int32_t k) {
    ODB_TRY(check_logits(x));
    if (k < 1 || k > ODB_LIST_MAX) return set_error(ODB_E_INVALID_ARG, "k must be in [1, %d] (got %d)", ODB_LIST_MAX, k);
    return ODB_OK;
}

// Blocks of a position: for fewer positions than would fill the chip, as many as have a round of loads each, as
// far as their candidates go to one block's LDS.  The join costs what six rounds do, and the parts of many positions take
// turns: a position is split if it has more than six rounds and an eighth as many as there are positions (long lists,
// which a part cuts to 2 k before the join, a 32nd).  us in a graph with parts / with one block, 1 / 32 / 128 / 512
// positions of bf16 logits:
//   logits (rounds)    k = 20                                             k = 128
//   50,000 (6.1)       12.5/12.4  13.7/13.0  16.1/13.6  21.0/16.4         17.6/24.2  19.3/26.1  23.4/27.0  36.9/29.5
//   100,000 (12.2)     10.3/17.9  13.0/19.3  18.9/19.6  29.9/24.3         22.0/33.5  25.8/35.0  29.8/35.4  49.4/40.5
//   151,936 (18.5)     11.8/23.8  14.0/25.2  22.4/25.1  38.4/34.6         23.7/41.5  27.2/44.3  36.2/44.1  61.3/90.0
//   250,000 (30.5)     12.6/33.6  15.6/34.2  25.5/35.5  54.9/51.8         27.6/61.4  32.1/154   42.3/199   153/213
constexpr int64_t kFillBlocks = 1024;
int32_t parts_for(const odb_logits_t* x, int32_t k, int64_t* len) {
    const int64_t n = x->rows * x->cols, round = x->dtype == ODB_FLOAT32 ? 4096 : 8192;
    int64_t parts = n > 0 ? kFillBlocks / n : 1;
    if (x->vocab <= 6 * round || x->vocab * (k > kWave ? 32 : 8) < n * round) return 1;
    parts = std::min({parts, (x->vocab + round - 1) / round, (int64_t)(Room<kBlock>::kHold / (2 * k)), (int64_t)kWave});
    if (parts <= 1) return 1;
    *len = ((x->vocab + parts - 1) / parts + 7) & ~(int64_t)7;
    return (int32_t)((x->vocab + *len - 1) / *len);
}

struct TopLayout {
    int32_t parts;
    int64_t len;
    size_t key, total;
};

TopLayout top_layout(const odb_logits_t* x, int32_t k) {
    TopLayout L{};
    L.parts = parts_for(x, k, &L.len);
    const size_t all = L.parts > 1 ? (size_t)(x->rows * x->cols * L.parts) : 0;
    L.key = (sizeof(Part) * all + 255) & ~size_t(255);
    L.total = std::max(L.key + 16 * all * k, size_t(256));
    return L;
}

}  // namespace

}  // namespace odb

using namespace odb;

extern "C" size_t odb_token_top_workspace_size(const odb_logits_t* x, int32_t k) {
    if (check_top(x, k) != ODB_OK) return 0;
    return top_layout(x, k).total;
}

extern "C" int odb_token_top_logprobs(const odb_logits_t* x, const int32_t* d_labels, int32_t k, int32_t* d_top_ids,
                                      float* d_top_logprob, float* d_logprob, int32_t* d_rank, float* d_stats,
                                      float* d_entropy, int32_t* d_status, void* d_ws, size_t ws_bytes, void* stream) {
    ODB_TRY(check_top(x, k));
    if (!d_labels && (d_logprob || d_rank))
        return set_error(ODB_E_INVALID_ARG, "d_logprob and d_rank need d_labels");
    if (x->rows == 0 || x->cols == 0) return ODB_OK;
    ODB_TRY(check_tile(x, x->d_logits, x->row_stride, x->col_stride, "d_logits"));
    if (!d_top_ids || !d_top_logprob) return set_error(ODB_E_INVALID_ARG, "d_top_ids and d_top_logprob must not be NULL");
    if (reinterpret_cast<uintptr_t>(d_stats) & 7)
        return set_error(ODB_E_INVALID_ARG, "d_stats must be 8-byte aligned");
    if (!d_ws) return set_error(ODB_E_INVALID_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(d_ws) & 255)
        return set_error(ODB_E_INVALID_ARG, "workspace must be 256-byte aligned");
    const TopLayout L = top_layout(x, k);
    if (ws_bytes < L.total)
        return set_error(ODB_E_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, L.total);
    TopArgs a{};
    a.x = *x;
    a.labels = d_labels;
    a.ids = d_top_ids;
    a.top = d_top_logprob;
    a.logprob = d_logprob;
    a.rank = d_rank;
    a.stats = d_stats;
    a.entropy = d_entropy;
    a.status = d_status;
    a.k = k;
    a.parts = L.parts;
    a.part_len = L.len;
    a.part = ws_at<Part>(d_ws, 0);
    a.part_key = ws_at<u64>(d_ws, L.key);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (x->dtype == ODB_FLOAT32)
        launch<float>(a, s);
    else if (x->dtype == ODB_BFLOAT16)
        launch<bf16_t>(a, s);
    else
        launch<fp16_t>(a, s);
    ODB_LAUNCHED();
    return ODB_OK;
}
