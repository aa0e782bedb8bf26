// The most probable tokens of every position of a tile, with log-probabilities, entropy and the label's rank.
//
// One pass over a position's logits forms the largest, the sum of exponentials and, for the entropy, their
// weighted logs, as the label's log-probability does.  Beside it the k largest are found by a bound that
// only a few candidates pass: k threads' largest of the first round of loads are k logits, so the k-th
// of those is a bound that the row's k-th largest does not fall below.  What reaches it goes to a list in
// LDS; behind the pass the list's k largest are picked by the digits of their keys and ordered by counting.
// A key holds the logit, mapped to a whole number that grows with it, above the complement of the column:
// keys are never equal, and of equal logits the first column's is the largest.
// Where the list does not hold what passes (a first round far below the rest, rows of few different
// values), the row is gone through again, with an exact bound behind every step.
#include "odb_vocab.h"

namespace odb {

namespace {

typedef unsigned long long u64;

constexpr int kBins = 256;      // of a digit
constexpr float kNone = -HUGE_VALF;

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
};

// A group's LDS.  Enough candidates for k = 128 and a step of one load of (at most 256) threads.
template <int G>
struct Room {
    static constexpr int kLanes = G < 256 ? G : 256;        // threads that load in a step
    static constexpr int kHold = ODB_LIST_MAX + kLanes * 8;
    static constexpr int kFew = G < 256 ? 128 : 256;        // candidates that are ordered by counting
    u64 key[kHold];
    u64 few[kFew];
    u64 top[ODB_LIST_MAX];
    uint32_t bins[kBins];
    uint32_t bound[(G + kWave - 1) / kWave];
    Acc acc[(G + kWave - 1) / kWave];
    u64 differ;
    uint32_t count, few_count, ahead;
};

// The largest whole number with its low 16 bits 0 that `kth` of the wave's lanes reach.
__device__ __forceinline__ uint32_t wave_kth(uint32_t o, int kth) {
    uint32_t r = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t c = r | 1u << bit;
        if (__builtin_popcountll(__ballot(o >= c)) >= kth) r = c;
    }
    return r;
}

template <int G>
__device__ __forceinline__ void keep(Room<G>& s, u64 key) {
    const uint32_t at = atomicAdd(&s.count, 1u);
    if (at < Room<G>::kHold) s.key[at] = key;
}

// The k largest of the n candidates (n <= kHold), ordered, to s.top; fewer if n < k.  The group has met
// before, and meets at the end.
template <int G>
__device__ void pick(Room<G>& s, int n, int k) {
    constexpr int kFew = Room<G>::kFew;
    const int t = threadIdx.x & (G - 1), lane = threadIdx.x & (kWave - 1);
    const u64* list = s.key;
    if (n > kFew) {
        // digits of 8 bits from the highest bit that differs
        if (t == 0) s.differ = 0;
        group_sync<G>();
        const u64 first = s.key[0];
        u64 differ = 0;
        for (int i = t; i < n; i += G) differ |= s.key[i] ^ first;
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
                const u64 key = s.key[i];
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
            const u64 key = s.key[i];
            if (key >= fixed) s.few[atomicAdd(&s.few_count, 1u)] = key;
        }
        group_sync<G>();
        n = (int)s.few_count;
        list = s.few;
    }
    for (int i = t; i < n; i += G) {
        const u64 mine = list[i];
        int place = 0;
        for (int j = 0; j < n; ++j) place += list[j] > mine;
        if (place < k) s.top[place] = mine;
    }
    group_sync<G>();
}

// Goes through columns [v0, v1) of a row: the joined triple, the columns ahead of the label, and candidates
// for the k largest, of which there are n <= kHold.  All of the group's threads get the same.
template <typename T, bool ENT, bool RANK, int G>
__device__ __forceinline__ Acc scan(const T* z, int64_t v0, int64_t v1, int32_t y, float zy, int kk, float k, Room<G>& s,
                                    int* n) {
    constexpr int N = Vec<T>::N;
    constexpr int kWavesIn = G / kWave;
    const int t = threadIdx.x & (G - 1), lane = threadIdx.x & (kWave - 1);
    if (t == 0) s.count = s.ahead = 0;
    group_sync<G>();
    Acc r{kLowest, 0.0f, 0.0f};
    int ahead = 0;
    const int64_t whole = v0 + (v1 - v0) / N * N;
    float bound = kNone;
    // a 16-byte group: its sums, its place beside the label's, and its largest
    auto take = [&](const Vec<T>& w, int64_t v) {
        float f[N], most = kNone;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            f[e] = (float)w.v[e];
            most = fmaxf(most, f[e]);
        }
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
    auto load = [&](Vec<T>* w, int64_t v) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) w[j] = load_vec<true>(z + at_most(v + j * G * N, whole - N));
    };
    int64_t v = v0 + (int64_t)t * N;
    if (v0 < whole) {     // uniform
        Vec<T> w[kAhead];
        load(w, v);
        float most[kAhead], all = kNone;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            most[j] = kNone;
            if (v + j * G * N < whole) most[j] = take(w[j], v + j * G * N);
            all = fmaxf(all, most[j]);
        }
        // every wave gives its share of k threads, or one wave all of them
        uint32_t o = wave_kth(ordered(all), (kk + kWavesIn - 1) / kWavesIn);
        if (G > kWave) {
            if (lane == 0) s.bound[threadIdx.x / kWave] = o;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kWavesIn; ++i) o = s.bound[i] < o ? s.bound[i] : o;
        }
        bound = o > ordered(kNone) ? unordered(o) : kNone;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (most[j] >= bound && most[j] > kNone) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float f = (float)w[j].v[e];
                    if (f >= bound && f > kNone) keep(s, key_of(f, v + j * G * N + e));
                }
            }
        }
    }
    // behind the first round k columns before these have reached the bound: equal ones come after them
    for (v += kAhead * G * N; v < whole; v += kAhead * G * N) {
        Vec<T> w[kAhead];
        load(w, v);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (v + j * G * N >= whole) break;
            if (take(w[j], v + j * G * N) > bound) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float f = (float)w[j].v[e];
                    if (f > bound) keep(s, key_of(f, v + j * G * N + e));
                }
            }
        }
    }
    if (whole + t < v1) {
        const float f = (float)z[whole + t];
        if (f > r.m) acc_rescale<ENT>(r, f, k);
        acc_term<ENT>(r, f, k);
        if (RANK) ahead += f > zy || (f == zy && whole + t < y);
        if (f > bound) keep(s, key_of(f, whole + t));
    }
    if (RANK) {
#pragma unroll
        for (int d = kWave / 2; d > 0; d >>= 1) ahead += __shfl_xor(ahead, d, kWave);
        if (lane == 0) atomicAdd(&s.ahead, (uint32_t)ahead);
    }
    r = group_join<ENT, G>(r, s.acc, k);
    group_sync<G>();
    int have = (int)s.count;
    if (have > Room<G>::kHold) {
        // again, a load a step, above the k-th largest so far
        constexpr int kLanes = Room<G>::kLanes;
        group_sync<G>();
        u64 least = 0;
        have = 0;
        for (int64_t at = v0; at < v1; at += kLanes * N) {
            if (t == 0) s.count = have;
            group_sync<G>();
            const int64_t mine = at + (int64_t)t * N;
            for (int e = 0; t < kLanes && e < N && mine + e < v1; ++e) {
                const float f = (float)z[mine + e];
                const u64 key = key_of(f, mine + e);
                if (f > kNone && key > least) keep(s, key);
            }
            group_sync<G>();
            have = (int)s.count;
            if (have > kk) {
                pick(s, have, kk);
                for (int i = t; i < kk; i += G) s.key[i] = s.top[i];
                have = kk;
                least = s.top[kk - 1];
            }
            group_sync<G>();
        }
    }
    *n = have;
    return r;
}

// A token's outputs from the joined triple and the n <= k largest, ordered, in s.top.
template <bool ENT, bool RANK, int G>
__device__ __forceinline__ void leave(const TopArgs& A, int64_t q, const Acc& r, int32_t y, float zy, int n, uint32_t ahead,
                                      const Room<G>& s) {
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
        if (RANK) A.rank[q] = sound ? (int32_t)ahead : -1;
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
template <typename T, bool ENT, bool RANK, int G>
__global__ void __launch_bounds__(kBlock) top_kernel(TopArgs A) {
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
        const Acc r = scan<T, ENT, RANK, G>(z, 0, V, y, zy, A.k, k, s, &have);
        pick(s, have, A.k);
        leave<ENT, RANK, G>(A, q, r, y, zy, have < A.k ? have : A.k, s.ahead, s);
        group_sync<G>();     // the next position writes where this one's are read
    }
}

template <typename T, bool ENT, bool RANK>
void launch(const TopArgs& a, hipStream_t s) {
    const int64_t n = a.x.rows * a.x.cols;
    const int64_t row = a.x.vocab * (int64_t)sizeof(T);
    if (row <= 16384 && a.k <= kWave && n > 2 * num_cus())
        hipLaunchKernelGGL((top_kernel<T, ENT, RANK, kWave>), dim3(grid_for(n, kBlock / kWave)), dim3(kBlock), 0, s, a);
    else
        hipLaunchKernelGGL((top_kernel<T, ENT, RANK, kBlock>), dim3(grid_for(n, 1)), dim3(kBlock), 0, s, a);
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

size_t top_workspace(const odb_logits_t*, int32_t) { return 256; }

}  // namespace

}  // namespace odb

using namespace odb;

extern "C" size_t odb_token_top_workspace_size(const odb_logits_t* x, int32_t k) {
    if (check_top(x, k) != ODB_OK) return 0;
    return top_workspace(x, k);
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
    if (ws_bytes < top_workspace(x, k))
        return set_error(ODB_E_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, top_workspace(x, k));
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
