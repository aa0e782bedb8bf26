// Losses over a run of a plan's tiles, with their gradients: the clipped policy loss with a KL
// term (one number per slot) and the preference loss (one number per pair of rows).
//
// The run's elements are cut into chunks of equal length wherever slots and rows end, so any mix
// of tiles keeps every compute unit busy.  What a chunk adds to a slot (or a row) is a partial of
// its own: going through the chunks b in order, the slot k never falls, so b + k names each pair
// that occurs once and a slot's partials are neighbours.  They are summed in a fixed order, in 64
// bits, by whoever needs the sum: no atomics on sums, the same result from call to call.
//
// A mean's weight is known only after the labels have been read.  That pass leaves one bit per
// element (does it count?), which is all that the later ones read of them: 4 bytes become 1/8.
#include <algorithm>
#include <cmath>

#include "odb_internal.h"
#include "odb_tiles.h"

namespace odb {

namespace {

constexpr int kMinChunk = 1024, kMaxChunk = 8192;    // elements of a chunk
// Runs of few elements go through one launch of one block, whose time grows with each 1,024 elements where
// the passes' does not.  us in a graph, one block / passes:
//   elements    policy, token mean   policy, row mean    preference, by id   preference, by row
//   300          6.9 / 11.3           7.1 / 13.0         11.3 / 12.2          9.7 / 9.9
//   1,000        7.5 / 11.6           7.7 / 13.3         15.1 / 12.5         13.3 / 10.0
//   2,000        9.7 / 12.3          10.1 / 14.2         15.7 / 13.0         13.9 / 10.6
//   4,000       13.7 / 12.3          14.5 / 14.7         16.3 / 13.1         14.6 / 10.6
// With 1,024 threads: 12.6 / 13.0 (policy) at 4,000 elements, but 16.5 at 8,192, where the passes take 12.6.
constexpr int kOnePolicy = 4096;
constexpr int kOnePairs = 512;
static_assert(kOnePairs <= kMinChunk);
constexpr int kOneSlots = 4096;     // and few slots: an empty one, too, has its numbers to write
constexpr int kWaves = kBlock / kWave;
static_assert(kWaves == 4, "a wave takes a quarter of a chunk");
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLog2eLow = 1.92596299112661746887e-8f;   // log2 e - kLog2e
constexpr float kLn2 = 0.69314718055994530942f;

typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
typedef int int4u __attribute__((ext_vector_type(4), aligned(4)));

// Chunks of a run from which on a launch of its own folds what the chunks counted of a slot into its first 64
// chunks' counts, which is all that each block adds up then.  Without it a slot of C chunks is added up C times:
// 2^28 elements in one slot took 3.0 ms and 2^30 42.5 (mean over tokens), with it 0.98 and 4.0; in slots of 2^20
// 0.75 and 3.0.
constexpr int64_t kManyChunks = 1 << 15;
constexpr int kCheckBlocks = 256;   // blocks of a pass that look over the slots, at most

// ------------------------------------------------------------------ workspace
struct SlotPart {
    double sum[4];      // policy, KL, entropy, ratio
    int32_t clipped[3];
    int32_t counted;
};

// A row's sum and count where it lies in one part (a wave's quarter of a chunk), otherwise the parts
// that it touches, whose partials hold them.  No parts: a row of a contradicting slot.
struct RowInfo {
    double sum;
    int32_t count;
    int32_t parts, first;
    int32_t pad;
};

struct PairPart {
    double loss;
    int32_t pairs, right;
};

struct LossLayout {
    size_t bits, chunk_slot, slot_count, slot_part, row_sum, row_count, row_info, coef, pair_part, disorder, row_of;
    size_t total;
    int64_t chunks;
    int32_t chunk;
};

constexpr int64_t kMaxElems = (int64_t)1 << 36;    // 2^23 chunks: a grid's threads stay below 2^32

// Elements of a chunk, a power of two: as many chunks as keep the chip busy (it holds 2,048 blocks of 256
// threads), but not more, since each costs a search for its first slot and a reduction.  us of a whole call
// with chunks of 1,024 / 2,048 / 4,096 / 8,192 / 16,384, tiles of up to 32,768 tokens:
//   elements    policy, mean over tokens      preference by row, rows of about 480
//   2^17         18 /  19 /  21 /  28 /  38    16 /  16 /  18 /  23 /  32
//   2^20         25 /  23 /  24 /  29 /  40    21 /  20 /  21 /  25 /  36
//   2^21         39 /  32 /  30 /  36 /  50    32 /  26 /  27 /  31 /  41
//   2^22         60 /  47 /  40 /  42 /  55    46 /  36 /  32 /  37 /  49
//   2^23         99 /  72 /  59 /  54 /  63    75 /  52 /  46 /  48 /  58
//   2^25        317 / 220 / 162 / 150 / 150   244 / 154 / 123 / 117 / 124
//   2^28       2527 /1598 /1102 / 946 / 957  2027 /1274 /1036 / 934 / 941
int32_t chunk_for(int64_t elems) {
    int32_t chunk = kMinChunk;
    while (chunk < kMaxChunk && elems >= chunk * (int64_t)2048) chunk *= 2;
    return chunk;
}

int check_tiles(const odb_tiles_t* t) {
    if (!t) return set_error(ODB_E_INVALID_ARG, "tiles is NULL");
    if (t->num_slots < 0 || t->num_slots > INT32_MAX)
        return set_error(ODB_E_INVALID_ARG, "num_slots must be in [0, 2^31)");
    if (t->num_rows < 0 || t->num_rows > INT32_MAX) return set_error(ODB_E_INVALID_ARG, "num_rows must be in [0, 2^31)");
    if (t->num_elems < 0 || t->num_elems > kMaxElems)
        return set_error(ODB_E_INVALID_ARG, "num_elems must be in [0, 2^36]");
    if (t->shift != 0 && t->shift != 1) return set_error(ODB_E_INVALID_ARG, "shift must be 0 or 1 (got %d)", t->shift);
    if (t->reserved0 != 0) return set_error(ODB_E_INVALID_ARG, "tiles.reserved0 must be 0");
    return ODB_OK;
}

LossLayout loss_layout(const odb_tiles_t* t, int64_t num_ids) {
    LossLayout L;
    size_t o = 0;
    auto take = [&](int64_t bytes) {
        const size_t at = o;
        o = (o + (size_t)(bytes > 0 ? bytes : 1) + 255) & ~size_t(255);
        return at;
    };
    L.chunk = chunk_for(t->num_elems);
    L.chunks = (t->num_elems + L.chunk - 1) / L.chunk;
    const int64_t K = t->num_slots, R = t->num_rows;
    L.bits = take(L.chunks * (L.chunk / 8));
    L.chunk_slot = take(4 * L.chunks);
    L.slot_count = take(4 * (L.chunks + K));
    L.slot_part = take((int64_t)sizeof(SlotPart) * (L.chunks + K));
    L.row_sum = take(8 * (kWaves * L.chunks + R));
    L.row_count = take(4 * (kWaves * L.chunks + R));
    L.row_info = take((int64_t)sizeof(RowInfo) * R);
    L.coef = take(8 * R);
    L.pair_part = take((int64_t)sizeof(PairPart) * (R / kBlock + 1));
    L.disorder = take(4 * kCheckBlocks * kWaves);
    L.row_of = take(4 * num_ids);
    L.total = o;
    return L;
}

int check_loss_workspace(const LossLayout& L, const void* d_ws, size_t ws_bytes) {
    if (!d_ws) return set_error(ODB_E_INVALID_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(d_ws) & 255)
        return set_error(ODB_E_INVALID_ARG, "workspace must be 256-byte aligned");
    if (ws_bytes < L.total)
        return set_error(ODB_E_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, L.total);
    return ODB_OK;
}

// Blocks that look over K slots.
int64_t check_blocks(int64_t K) { return std::min((K + kBlock - 1) / kBlock, (int64_t)kCheckBlocks); }

// ------------------------------------------------------------------ shared by the passes
// Block b of `blocks` looks over its part of the run's slots: f(real, slot) for every one, called by whole waves
// (`real`: the lane has a slot).  A wave leaves a word: is one of its slots not ordered?  Then the passes' partials
// mean nothing, and who takes the sums has them as 0.  Blocks of the first pass behind those of the chunks do it,
// beside them (in front of a chunk it took 0.3 us of a call).
template <typename F>
__device__ __forceinline__ void check_slots(const odb_tiles_t& t, int64_t b, uint32_t* disorder, int64_t blocks,
                                            const F& f) {
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    uint32_t found = 0;
    for (int64_t first = b * kBlock + wave * kWave; first < t.num_slots; first += blocks * kBlock) {   // uniform
        const int64_t k = first + lane;
        const bool real = k < t.num_slots;
        const SlotView s = slot_view(t, real ? k : first, e_base, r_base);
        found |= !s.ordered;
        f(real, s);
    }
    found = __any(found);
    if (lane == 0) disorder[b * kWaves + wave] = found;
}

struct NoVisit {
    __device__ __forceinline__ void operator()(bool, const SlotView&) const {}
};

// A lane's part of those words, of which one that is set is asked for with __any: late, when other loads have
// been waited for as well.
__device__ __forceinline__ uint32_t disorder_words(const uint32_t* disorder, int64_t blocks) {
    const int lane = threadIdx.x & (kWave - 1), words = (int)blocks * kWaves;
    uint32_t found = lane < words ? disorder[lane] : 0;
    for (int i = lane + kWave; i < words; i += kWave) found |= disorder[i];    // more than 4,096 slots
    return found;
}

// Last slot from `from` on that starts at or before element e, 64 probes a step (one a lane; every lane of
// the wave must be active): two loads one after the other for up to 4,096 slots, where halving the range
// takes twelve.
__device__ __forceinline__ int64_t slot_at(const odb_tiles_t& t, int64_t e_base, int64_t from, int64_t e) {
    const int lane = threadIdx.x & (kWave - 1);
    return search_slot(from, t.num_slots, [&](int64_t lo, int64_t step, int64_t hi) {
        const int64_t at = lo + lane * step;
        const uint64_t before = __ballot(at < hi && offset_from(t.d_slot_tile_off[at < hi ? at : lo], e_base) <= e);
        return before == ~0ull ? kProbes : __builtin_ctzll(~before);
    });
}

__device__ __forceinline__ int64_t first_slot(const odb_tiles_t& t, int64_t e_base, int64_t c0) {
    return slot_at(t, e_base, 0, c0);
}

// The slots with elements in [c0, c1), from slot k0 on; every lane of the wave must be active.
template <typename F>
__device__ __forceinline__ void each_slot(const odb_tiles_t& t, int64_t e_base, int64_t r_base, int64_t k0, int64_t c0,
                                          int64_t c1, const F& f) {
    chunk_slots(t, e_base, r_base, k0, c0, c1, [&](int64_t from, int64_t e) { return slot_at(t, e_base, from, e); }, f);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_plus(double v) {
    const long long u = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)u, CTRL, ROWS, 0xf, true);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xf, true);
    return v + __longlong_as_double((long long)(((unsigned long long)hi << 32) | lo));
}

// Sum over the 64 lanes in a fixed order, on every lane; all lanes must be active.
__device__ __forceinline__ double wave_total(double v) {
    v = dpp_plus<0x111, 0xf>(v);
    v = dpp_plus<0x112, 0xf>(v);
    v = dpp_plus<0x114, 0xf>(v);
    v = dpp_plus<0x118, 0xf>(v);
    v = dpp_plus<0x142, 0xa>(v);
    v = dpp_plus<0x143, 0xc>(v);
    const long long u = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)u, kWave - 1);
    const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)(u >> 32), kWave - 1);
    return __longlong_as_double((long long)(((unsigned long long)hi << 32) | lo));
}

__device__ __forceinline__ int wave_total(int v) { return wave_last(wave_scan_dpp<OpAdd>(v)); }

template <typename T>
__device__ __forceinline__ T block_total(T v) {
    __shared__ T s_part[kWaves];
    v = wave_total(v);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) s_part[threadIdx.x / kWave] = v;
    __syncthreads();
    T sum = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) sum += s_part[i];
    return sum;
}

// Four values of an array from position o of a chunk on; what lies behind the array, whose last four are at
// `last`, holds any of its values.  SAFE, for where a group may end behind it: each value is read on its own,
// the last one for those behind.  Otherwise a position past `last` reads that one.  Either way there is no
// branch, so that loads of many groups go out together.
// What is read here is read once: past the caches' usual order, 67 M elements in 2,080 tiles take 260 us
// instead of 268 (policy) and 222 instead of 283 (preference).
template <typename V4, bool SAFE, typename T>
__device__ __forceinline__ V4 load4(const T* p, int o, int last) {
    if (SAFE) {
        V4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = p[o + j < last + 3 ? o + j : last + 3];
        return v;
    }
    const uint32_t at = 4u * (uint32_t)(o < last ? o : last);    // one 32-bit offset to the chunk's address
    return __builtin_nontemporal_load(reinterpret_cast<const V4*>(reinterpret_cast<const char*>(p) + at));
}

// Which of a group's elements count.
__device__ __forceinline__ uint32_t count_mask(Group q, const int4u& y, int maxlen, int shift) {
    uint32_t on = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        on |= (uint32_t)(y[j] != ODB_LABEL_IGNORE && q.col >= shift) << j;
        q.next(maxlen);
    }
    return on & q.mask;
}

__device__ __forceinline__ void store4(float* p, const Group& q, const float v[4]) {
    if (q.mask == 0xf) {
        const float4u x = {v[0], v[1], v[2], v[3]};
        *reinterpret_cast<float4u*>(p + q.o) = x;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (q.mask >> j & 1) p[q.o + j] = v[j];
    }
}

// A chunk's bits to LDS; the block meets before and after.
__device__ __forceinline__ void load_bits(uint32_t* s_bits, const uint32_t* bits, int64_t b, int chunk) {
    const int words = chunk / 32;
    __syncthreads();
    for (int i = threadIdx.x; i < words; i += kBlock) s_bits[i] = bits[b * words + i];
    __syncthreads();
}

// Position in a chunk of the arrays' last four elements, as far as a chunk's positions go; negative in
// a last chunk of fewer.  Whether a span's groups reach past them:
__device__ __forceinline__ int last_four(const odb_tiles_t& t, int64_t c0) {
    const int64_t n = t.num_elems - 4 - c0;
    return (int)(n < 2 * kMaxChunk ? n : 2 * kMaxChunk);
}

__device__ __forceinline__ bool at_end(int o1, int last) { return ((o1 + 3) & ~3) > last + 4; }

// ------------------------------------------------------------------ policy loss
struct PolicyArgs {
    odb_tiles_t t;
    const float* logprob;
    const float* old;
    const float* ref;
    const float* entropy;
    const float* advantage;
    const double* slot_weight;
    float* slot_loss;
    float* slot_means;
    int64_t* slot_counts;
    float* grad;
    float* grad_entropy;
    uint32_t* bits;
    int32_t* chunk_slot;        // first slot of every chunk, left by the first pass
    int32_t* slot_count;        // counted tokens (token mean) or complete rows with any (row mean)
    SlotPart* slot_part;
    int32_t* row_count;
    uint32_t* disorder;
    int32_t* status;
    int64_t chunks, check_blocks;
    int64_t counts;                     // chunks from a slot's first on that hold what all of them counted
    double at_low, at_high, at_dual;    // ln(1 - e_l), ln(1 + e_h), ln c
    double kl_coef, entropy_coef, loss_scale;
    float low, high, dual;              // 1 - e_l, 1 + e_h, c
    int32_t chunk, chunk_log2;
    bool token_advantage, on_policy;    // on_policy: no old log-probabilities, the ratio is 1
};

// Groups of a thread whose loads are under way together.
constexpr int kAhead = 4;

// Rows of a chunk that one block weighs in LDS; those of fewer elements than 8 may be more, and are weighed where
// they are met.  us a call for room for 512 / 1,024 / 4,096, which leaves fewer blocks on a compute unit (mean
// over rows, 67 M elements in rows of about 480): 319 / 319 / 344; 34 M in rows of 40: 208 / 204 / 214, of 5:
// 262 / 239 / 248; one tile of 1,000,000 x 3: 71 / 70 / 68.
constexpr int kLdsRows = 1024;

// Adds a group's counted elements to its rows, the first of them `row0`.
__device__ __forceinline__ void add_to_rows(int* s_rows, Group q, uint32_t on, int maxlen, int row0) {
    if (q.col <= maxlen - 4) {
        if (on) atomicAdd(&s_rows[q.row - row0], __builtin_popcount(on));
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (on >> j & 1) atomicAdd(&s_rows[q.row - row0], 1);
        q.next(maxlen);
    }
}

// First pass of a mean: the bits, and per chunk and slot the counted tokens, or (ROWS) per chunk and
// row the counted tokens and per chunk and slot the rows with any that lie wholly in the chunk.
// Bound by the reads of the labels: 67 M elements in 2,080 tiles take 59 us (5.1 TB/s).
template <bool ROWS>
__global__ void __launch_bounds__(kBlock) policy_count_kernel(PolicyArgs A) {
    __shared__ alignas(16) uint8_t s_nibble[kMaxChunk / 4];
    __shared__ int s_rows[ROWS ? kLdsRows : 1];
    const odb_tiles_t& t = A.t;
    if (blockIdx.x >= A.chunks) return check_slots(t, blockIdx.x - A.chunks, A.disorder, A.check_blocks, NoVisit{});
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    const int64_t b = blockIdx.x, c0 = b * A.chunk, c1 = c0 + A.chunk < total ? c0 + A.chunk : total;
    if (c0 >= c1) return;
    const int32_t* labels = t.d_labels + c0;
    const int last = last_four(t, c0);
    for (int i = threadIdx.x; i < A.chunk / 16; i += kBlock) reinterpret_cast<uint32_t*>(s_nibble)[i] = 0;
    const int64_t k0 = first_slot(t, e_base, c0);
    if (threadIdx.x == 0) A.chunk_slot[b] = (int32_t)k0;
    __syncthreads();
    each_slot(t, e_base, r_base, k0, c0, c1, [&](int64_t k, const SlotView& s, int64_t a0, int64_t a1) {
        const Span p(s, a0, a1, c0, kBlock);
        const int rows = (int)((a1 - 1 - s.lo) / s.maxlen) - p.row_a + 1;
        const bool lds = ROWS && rows <= kLdsRows;
        if (lds) {
            for (int i = threadIdx.x; i < rows; i += kBlock) s_rows[i] = 0;
            __syncthreads();
        }
        int count = 0;
        Group q = p.first((int)threadIdx.x);
        auto take = [&](const int4u& y) {
            const uint32_t on = count_mask(q, y, p.maxlen, t.shift);
            if (on) s_nibble[q.o / 4] |= (uint8_t)on;
            if (lds)
                add_to_rows(s_rows, q, on, p.maxlen, p.row_a);
            else
                count += __builtin_popcount(on);
            p.advance(&q);
        };
        if (at_end(p.o1, last)) {
            while (q.o < p.o1) take(load4<int4u, true>(labels, q.o, last));
        } else {
            for (int o = p.o0 & ~3; o < p.o1; o += kAhead * p.ahead) {     // uniform
                int4u y[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) y[i] = load4<int4u, false>(labels, q.o + i * p.ahead, last);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) take(y[i]);
            }
        }
        if (ROWS) {
            // a row counts here if it starts and ends here; the others are joined by who needs the slot's rows
            __syncthreads();
            count = 0;
            for (int i = threadIdx.x; i < rows; i += kBlock) {
                const int64_t start = s.lo + (int64_t)(p.row_a + i) * s.maxlen;
                int n = 0;
                if (lds) {
                    n = s_rows[i];
                } else {     // rows of a few elements
                    for (int64_t e = start > a0 ? start : a0; e < start + s.maxlen && e < a1; ++e)
                        n += s_nibble[(e - c0) / 4] >> ((e - c0) & 3) & 1;
                }
                A.row_count[b + s.row0 + p.row_a + i] = n;
                count += n > 0 && start >= c0 && start + s.maxlen <= c0 + A.chunk;
            }
        }
        count = block_total(count);
        if (threadIdx.x == 0) A.slot_count[b + k] = count;
        __syncthreads();
    });
    for (int i = threadIdx.x; i < A.chunk / 32; i += kBlock) {
        const uint2 w = reinterpret_cast<const uint2*>(s_nibble)[i];
        // eight bytes of four bits to one word
        uint32_t v = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v |= (w.x >> (8 * j) & 0xf) << (4 * j) | (w.y >> (8 * j) & 0xf) << (16 + 4 * j);
        A.bits[b * (A.chunk / 32) + i] = v;
    }
}

// exp(d) to about one rounding of fp32: the part of d log2 e that a product loses is put back.
__device__ __forceinline__ float exp_near(float d) {
    const float u = d * kLog2e;
    const float e = __builtin_amdgcn_exp2f(u);
    const float lost = fmaf(d, kLog2eLow, fmaf(d, kLog2e, -u));
    return u > -200.0f && u < 128.0f ? fmaf(e * lost, kLn2, e) : e;    // outside: 0 and infinity
}

// exp(d) - 1 - d: below 3/2 by its series (the next term is under 2^-31 of the sum), where the
// difference would cancel.
constexpr float kSeries = 1.5f;

__device__ __forceinline__ float less_line_series(float d) {
    float q = 1.0f / 87178291200.0f;
    q = fmaf(q, d, 1.0f / 6227020800.0f);
    q = fmaf(q, d, 1.0f / 479001600.0f);
    q = fmaf(q, d, 1.0f / 39916800.0f);
    q = fmaf(q, d, 1.0f / 3628800.0f);
    q = fmaf(q, d, 1.0f / 362880.0f);
    q = fmaf(q, d, 1.0f / 40320.0f);
    q = fmaf(q, d, 1.0f / 5040.0f);
    q = fmaf(q, d, 1.0f / 720.0f);
    q = fmaf(q, d, 1.0f / 120.0f);
    q = fmaf(q, d, 1.0f / 24.0f);
    q = fmaf(q, d, 1.0f / 6.0f);
    q = fmaf(q, d, 0.5f);
    return q * d * d;
}

__device__ __forceinline__ float less_line_far(float d) { return exp_near(d) - 1.0f - d; }

// The bounds on lp - old, rounded to fp32.
struct Bounds {
    float low, high, dual;
};

// A thread's part of a slot.
struct PolicySums {
    double sum[4] = {0, 0, 0, 0};
    int counted = 0;
    int clipped[3] = {0, 0, 0};
};

// The chunk's part of every array, and what does not change from group to group.
struct PolicyChunk {
    const float* logprob;
    const float* old;
    const float* ref;
    const float* entropy;
    const float* advantage;     // of the chunk (per token) or of the slot (per row)
    float* grad;
    float* grad_entropy;
    int last;
    float kl_coef, entropy_coef;
    Bounds bounds;
};

// A group's inputs on their way.  A group in which nothing counts reads the chunk's first elements
// instead, as all such do: no traffic, and no branch that parts the loads.
struct PolicyLoads {
    float4u lp, old, ref, H, adv;
    uint32_t on;
};

template <int KL, bool ENT, bool SAFE>
__device__ __forceinline__ PolicyLoads policy_load(const PolicyArgs& A, const PolicyChunk& C, Group q, uint32_t on,
                                                   int maxlen, int row_a) {
    PolicyLoads L;
    L.on = on;
    const int o = on ? q.o : 0;
    L.lp = load4<float4u, SAFE>(C.logprob, o, C.last);
    L.old = load4<float4u, SAFE>(C.old, o, C.last);
    if (KL != ODB_KL_NONE) L.ref = load4<float4u, SAFE>(C.ref, o, C.last);
    if (ENT) L.H = load4<float4u, SAFE>(C.entropy, o, C.last);
    if (A.token_advantage) {
        L.adv = load4<float4u, SAFE>(C.advantage, o, C.last);
    } else {
        L.adv[0] = C.advantage[on ? q.row : row_a];
        L.adv[1] = L.adv[2] = L.adv[3] = L.adv[0];
        if (on && q.col > maxlen - 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (on >> j & 1) L.adv[j] = C.advantage[q.row];
                q.next(maxlen);
            }
        }
    }
    return L;
}

// A group's part of the sums, and its gradients.  weight(row, &f, &gs) gives the weight of a row's
// token in the slot's mean and the factor of its gradient (ROWS: they differ from row to row).  What
// does not count has its inputs replaced by 0, which makes all but the ratio and the linear KL term's
// slope 0.  Terms are formed in fp32, weighed and added in 64 bits: where signs differ the sum may be far
// smaller than they are, and terms near the type's largest have a mean (67 M elements: 242 us with the sums
// of a group of four in fp32 239; row means, whose weights were rounded as well, 312 and 300).  A gradient is
// an fp32 slope times an fp32 factor.  Four tokens go through without a branch but the one of the rare cases.
template <int KL, bool ROWS, bool ENT, typename Weight>
__device__ __forceinline__ void policy_group(const PolicyArgs& A, const PolicyChunk& C, Group q, const PolicyLoads& L,
                                             int maxlen, const Weight& weight, PolicySums& S) {
    float g[4] = {0, 0, 0, 0}, ge[4] = {0, 0, 0, 0};
    if (__any(L.on != 0)) {
        float d[4], x[4], adv[4], kl[4], kl_slope[4];
        bool over[4], under[4], rare = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool live = L.on >> j & 1;
            const float lp = live ? L.lp[j] : 0.0f;
            adv[j] = live ? L.adv[j] : 0.0f;
            d[j] = lp - (live ? L.old[j] : 0.0f);
            d[j] = A.on_policy ? 0.0f : d[j];
            // neither bound for advantages of 0 and NaN: nothing is clipped
            const bool pos = adv[j] > 0.0f, neg = adv[j] < 0.0f;
            const float up = pos ? C.bounds.high : neg ? C.bounds.dual : INFINITY, low = neg ? C.bounds.low : -INFINITY;
            over[j] = d[j] > up;
            under[j] = d[j] < low;
            // rounding keeps order: the rounded difference decides unless it equals a rounded bound
            rare |= d[j] == up || d[j] == low;
            if (KL != ODB_KL_NONE) x[j] = lp - (live ? L.ref[j] : 0.0f);
            if (KL == ODB_KL_EXP) {
                kl[j] = less_line_series(-x[j]);
                kl_slope[j] = x[j] - kl[j];    // 1 - exp(-x)
                rare |= fabsf(x[j]) >= kSeries;
            }
        }
        if (__builtin_expect(rare, 0)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool live = L.on >> j & 1, pos = adv[j] > 0.0f, neg = adv[j] < 0.0f;
                const double z = A.on_policy || !live ? 0.0 : (double)L.lp[j] - (double)L.old[j];
                over[j] = z > (pos ? A.at_high : neg ? A.at_dual : HUGE_VAL);
                under[j] = neg && z < A.at_low;
                if (KL == ODB_KL_EXP && fabsf(x[j]) >= kSeries) {
                    // the slope without x, beside which it would be lost: a reference of no probability has 1
                    kl[j] = less_line_far(-x[j]);
                    kl_slope[j] = 1.0f - exp_near(-x[j]);
                }
            }
        }
        double f[4];
        float gs[4];
        if (!ROWS) {
            weight(0, &f[0], &gs[0]);
#pragma unroll
            for (int j = 1; j < 4; ++j) gs[j] = gs[0];
        } else {
            Group r = q;
            double w = 0.0;
            float k = 0.0f;
            int have = -1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if ((L.on >> j & 1) && r.row != have) {
                    weight(r.row, &w, &k);
                    have = r.row;
                }
                f[j] = w;
                gs[j] = k;
                r.next(maxlen);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool live = L.on >> j & 1, pos = adv[j] > 0.0f;
            const float ratio = exp_near(d[j]);
            float bound = over[j] ? (pos ? A.high : A.dual) : ratio;
            bound = under[j] ? A.low : bound;
            bound = adv[j] == 0.0f ? 0.0f : bound;   // an overflowing ratio must not make the term NaN
            const float policy = -bound * adv[j];
            const float slope = over[j] || under[j] ? 0.0f : policy;
            if (KL == ODB_KL_LINEAR) {
                kl[j] = x[j];
                kl_slope[j] = live ? 1.0f : 0.0f;
            } else if (KL == ODB_KL_SQUARE) {
                kl[j] = 0.5f * x[j] * x[j];
                kl_slope[j] = x[j];
            } else if (KL == ODB_KL_NONE) {
                kl[j] = kl_slope[j] = 0.0f;
            }
            const float terms[4] = {policy, kl[j], ENT && live ? L.H[j] : 0.0f, live ? ratio : 0.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((KL != ODB_KL_NONE || i != 1) && (ENT || i != 2))
                    S.sum[i] = ROWS ? fma(f[j], (double)terms[i], S.sum[i]) : S.sum[i] + (double)terms[i];
            S.clipped[0] += under[j];
            S.clipped[1] += over[j] && pos;
            S.clipped[2] += over[j] && !pos;
            // 0 where nothing counts, also times a factor that is not finite
            const float total = C.kl_coef != 0.0f ? fmaf(C.kl_coef, kl_slope[j], slope) : slope;
            g[j] = live ? gs[j] * total : 0.0f;
            if (ENT) ge[j] = live ? -C.entropy_coef * gs[j] : 0.0f;
        }
        S.counted += __builtin_popcount(L.on);
    }
    if (q.mask) {
        if (A.grad) store4(C.grad, q, g);
        if (A.grad_entropy) store4(C.grad_entropy, q, ge);
    }
}

// The block's part of a slot from its threads', on thread 0.
__device__ __forceinline__ SlotPart block_part(const PolicySums& S, double same) {
    __shared__ SlotPart s_part[kWaves];
    SlotPart p;
#pragma unroll
    for (int j = 0; j < 4; ++j) p.sum[j] = wave_total(S.sum[j]);
    p.counted = wave_total(S.counted);
#pragma unroll
    for (int j = 0; j < 3; ++j) p.clipped[j] = wave_total(S.clipped[j]);
    if ((threadIdx.x & (kWave - 1)) == 0) s_part[threadIdx.x / kWave] = p;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWaves; ++w) {
            for (int j = 0; j < 4; ++j) p.sum[j] += s_part[w].sum[j];
            for (int j = 0; j < 3; ++j) p.clipped[j] += s_part[w].clipped[j];
            p.counted += s_part[w].counted;
        }
        for (int j = 0; j < 4; ++j) p.sum[j] *= same;
    }
    __syncthreads();
    return p;
}

// A slot's numbers from its sums.
__device__ __forceinline__ void leave_slot(const PolicyArgs& A, int64_t k, const double sum[4], int64_t counted,
                                           const int64_t clipped[3]) {
    const double scale = A.loss_scale * (A.slot_weight ? A.slot_weight[k] : 1.0);
    const double kl = A.kl_coef != 0.0 ? A.kl_coef * sum[1] : 0.0;      // a term that is only watched may overflow
    const double bonus = A.entropy_coef != 0.0 ? A.entropy_coef * sum[2] : 0.0;
    A.slot_loss[k] = counted > 0 ? (float)(scale * (sum[0] + kl - bonus)) : 0.0f;
    for (int i = 0; i < 4; ++i) A.slot_means[4 * k + i] = (float)sum[i];
    A.slot_counts[4 * k] = counted;
    for (int i = 0; i < 3; ++i) A.slot_counts[4 * k + 1 + i] = clipped[i];
}

__device__ __forceinline__ PolicyChunk policy_chunk(const PolicyArgs& A, const SlotView& s, int64_t c0) {
    PolicyChunk C;
    C.logprob = A.logprob + c0;
    C.old = A.old + c0;
    C.ref = A.ref + c0;
    C.entropy = A.entropy + c0;
    C.advantage = A.advantage + (A.token_advantage ? c0 : s.row0);
    C.grad = A.grad + c0;
    C.grad_entropy = A.grad_entropy + c0;
    C.last = last_four(A.t, c0);
    C.kl_coef = (float)A.kl_coef;
    C.entropy_coef = (float)A.entropy_coef;
    C.bounds = Bounds{(float)A.at_low, (float)A.at_high, (float)A.at_dual};
    return C;
}

// The block's part of a slot: counted(group) tells which elements count.
template <int KL, bool ROWS, bool ENT, bool SAFE, typename Counted, typename Weight>
__device__ __forceinline__ void policy_span(const PolicyArgs& A, const PolicyChunk& C, const Span& p,
                                            const Counted& counted, const Weight& weight, PolicySums& S) {
    // uniform over the block: a wave's lanes stay together, those behind the slot with nothing to do
    Group q = p.first((int)threadIdx.x);
    for (int o = p.o0 & ~3; o < p.o1; o += p.ahead, p.advance(&q)) {
        const PolicyLoads L = policy_load<KL, ENT, SAFE>(A, C, q, q.mask ? counted(q) : 0, p.maxlen, p.row_a);
        policy_group<KL, ROWS, ENT>(A, C, q, L, p.maxlen, weight, S);
    }
}

// The chunks that a row touches.
struct RowChunks {
    int64_t first, last;

    __device__ __forceinline__ RowChunks(const PolicyArgs& A, const SlotView& s, int64_t row) {
        const int64_t start = s.lo + row * s.maxlen;
        first = start >> A.chunk_log2;
        last = (start + s.maxlen - 1) >> A.chunk_log2;
    }
};

// Chunks of a row from which on the wave counts it, and not a lane: with a lane alone the mean over two rows of
// 131,072 tokens takes 26 us, not 17.5; with the wave for all of them rows of 480 in one tile take 15.5, not 14.6.
constexpr int kLongRow = 8;

// Counted tokens of a row, over the chunks it touches, by a lane.
__device__ __forceinline__ double row_tokens(const PolicyArgs& A, const SlotView& s, int64_t row) {
    const RowChunks c(A, s, row);
    int n = 0;
    for (int64_t b = c.first; b <= c.last; ++b) n += A.row_count[b + s.row0 + row];
    return n;
}

// The same by the wave; every lane must be active.
__device__ __forceinline__ double long_row_tokens(const PolicyArgs& A, const SlotView& s, int64_t row,
                                                  const RowChunks& c) {
    double n = 0;
#pragma unroll 4
    for (int64_t b = c.first + (threadIdx.x & (kWave - 1)); b <= c.last; b += kWave) n += A.row_count[b + s.row0 + row];
    return wave_total(n);
}

// Whether a row has any, by a lane: found in its first chunks, unless all of the row before is a prompt.
__device__ __forceinline__ bool row_counts(const PolicyArgs& A, const SlotView& s, int64_t row) {
    const RowChunks c(A, s, row);
    for (int64_t b = c.first; b <= c.last; b += 2) {
        const int64_t next = b < c.last ? b + 1 : b;
        if (A.row_count[b + s.row0 + row] | A.row_count[next + s.row0 + row]) return true;
    }
    return false;
}

// What chunk j counted of a slot: tokens, or (ROWS) whole rows with any and the row that starts in it and goes on.
template <bool ROWS>
__device__ __forceinline__ int chunk_counted(const PolicyArgs& A, const SlotView& s, int64_t k, int64_t j) {
    int n = A.slot_count[j + k];
    if (ROWS) {
        const int64_t end = (j + 1) * A.chunk;
        if (end < s.hi && (end - s.lo) % s.maxlen) {
            const int64_t row = (end - s.lo) / s.maxlen;
            if (s.lo + row * s.maxlen >= j * A.chunk) n += row_counts(A, s, row);
        }
    }
    return n;
}

// A slot's count from its chunks', one a lane, on every lane: a whole number that may pass 2^31.
template <bool ROWS>
__device__ __forceinline__ double slot_counted(const PolicyArgs& A, const SlotView& s, int64_t k) {
    const int64_t first = s.lo >> A.chunk_log2, end = ((s.hi - 1) >> A.chunk_log2) + 1;
    const int64_t stop = end < first + A.counts ? end : first + A.counts;
    const bool folded = A.counts == kWave;
    double n = 0;
    for (int64_t j = first + (threadIdx.x & (kWave - 1)); j < stop; j += kWave)
        n += ROWS && !folded ? chunk_counted<true>(A, s, k, j) : A.slot_count[j + k];
    return wave_total(n);
}

// Folds the counts of slots of more than 64 chunks, a block a slot: at most 2^17 chunks into one, 2^30 tokens.
template <bool ROWS>
__global__ void __launch_bounds__(kBlock) policy_fold_kernel(PolicyArgs A) {
    __shared__ int s_count[kBlock];
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    for (int64_t k = blockIdx.x; k < t.num_slots; k += gridDim.x) {
        const SlotView s = slot_view(t, k, e_base, r_base);
        if (!s.ok || s.hi == s.lo) continue;     // uniform
        const int64_t first = s.lo >> A.chunk_log2, last = (s.hi - 1) >> A.chunk_log2;
        int n = 0;
        for (int64_t j = first + threadIdx.x; j <= last; j += kBlock) n += chunk_counted<ROWS>(A, s, k, j);
        s_count[threadIdx.x] = n;
        __syncthreads();
        if (threadIdx.x < kWave && first + threadIdx.x <= last) {
            n = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) n += s_count[w * kWave + threadIdx.x];
            A.slot_count[first + threadIdx.x + k] = n;
        }
        __syncthreads();
    }
}

// The loss and its gradient, the elements that count given by the bits (by the labels for a sum, which
// needs no weights and so no pass before).  67 M elements in 2,080 tiles, the exponential KL term, 3/4 of them
// counted: 201 us for 603 MB read and 270 MB written (4.3 TB/s).  Instructions (about 100 an element, a power
// and the KL term's series among them) and memory take about as long; the waves of other chunks hide one
// behind the other.  A variant of the kernel by KL term, reduction and entropies keeps the rest of the work
// and its registers out of it.
template <int KL, int REDUCE, bool ENT>
__global__ void __launch_bounds__(kBlock) policy_kernel(PolicyArgs A) {
    constexpr bool ROWS = REDUCE == ODB_REDUCE_ROW_MEAN, LABELS = REDUCE == ODB_REDUCE_SUM;
    __shared__ double s_weight[ROWS ? kLdsRows : 1];
    __shared__ uint32_t s_bits[LABELS ? 1 : kMaxChunk / 32];
    const odb_tiles_t& t = A.t;
    if (LABELS && blockIdx.x >= A.chunks)
        return check_slots(t, blockIdx.x - A.chunks, A.disorder, A.check_blocks, NoVisit{});
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    const int64_t b = blockIdx.x, c0 = b * A.chunk, c1 = c0 + A.chunk < total ? c0 + A.chunk : total;
    if (c0 >= c1) return;
    const int64_t k0 = LABELS ? first_slot(t, e_base, c0) : (int64_t)A.chunk_slot[b];
    if (!LABELS) load_bits(s_bits, A.bits, b, A.chunk);
    each_slot(t, e_base, r_base, k0, c0, c1, [&](int64_t k, const SlotView& s, int64_t a0, int64_t a1) {
        const Span p(s, a0, a1, c0, kBlock);
        const double scale = A.loss_scale * (A.slot_weight ? A.slot_weight[k] : 1.0);
        double same = 1.0;       // weight of every token, where rows have none of their own
        double rows = 0;         // of the slot, with a counted token
        const int here = (int)((a1 - 1 - s.lo) / s.maxlen) - p.row_a + 1;
        const bool lds = ROWS && here <= kLdsRows;
        if (!LABELS) {
            const double n = slot_counted<ROWS>(A, s, k);
            if (ROWS) rows = n;
            else same = n > 0 ? 1.0 / n : 0.0;
        }
        auto of_count = [&](double n) { return n > 0 ? 1.0 / (n * rows) : 0.0; };
        // of the rows here only the first and the last may be long; below 0: not
        double w_first = -1.0, w_last = -1.0;
        if (ROWS) {
            const RowChunks first(A, s, p.row_a), last(A, s, p.row_a + here - 1);
            if (first.last - first.first >= kLongRow) w_first = of_count(long_row_tokens(A, s, p.row_a, first));
            if (here > 1 && last.last - last.first >= kLongRow)
                w_last = of_count(long_row_tokens(A, s, p.row_a + here - 1, last));
        }
        auto row_weight = [&](int i) {
            const double w = i == 0 ? w_first : i == here - 1 ? w_last : -1.0;
            return w >= 0.0 ? w : of_count(row_tokens(A, s, p.row_a + i));
        };
        if (lds) {
            for (int i = threadIdx.x; i < here; i += kBlock) s_weight[i] = row_weight(i);
            __syncthreads();
        }
        const float factor = (float)(scale * same);
        auto weight = [&](int row, double* f, float* gs) {
            if (ROWS) {
                const double w = lds ? s_weight[row - p.row_a] : row_weight(row - p.row_a);
                *f = w;
                *gs = (float)(scale * w);
            } else {
                *f = 1.0;
                *gs = factor;
            }
        };
        const PolicyChunk C = policy_chunk(A, s, c0);
        auto from_bits = [&](const Group& q) { return s_bits[q.o / 32] >> (q.o & 31) & q.mask; };
        PolicySums S;
        if (at_end(p.o1, C.last)) {
            auto from_labels = [&](const Group& q) {
                return count_mask(q, load4<int4u, true>(t.d_labels + c0, q.o, C.last), p.maxlen, t.shift);
            };
            if (LABELS) policy_span<KL, ROWS, ENT, true>(A, C, p, from_labels, weight, S);
            else policy_span<KL, ROWS, ENT, true>(A, C, p, from_bits, weight, S);
        } else {
            auto from_labels = [&](const Group& q) {
                return count_mask(q, load4<int4u, false>(t.d_labels + c0, q.o, C.last), p.maxlen, t.shift);
            };
            if (LABELS) policy_span<KL, ROWS, ENT, false>(A, C, p, from_labels, weight, S);
            else policy_span<KL, ROWS, ENT, false>(A, C, p, from_bits, weight, S);
        }
        const SlotPart part = block_part(S, same);
        if (threadIdx.x == 0) A.slot_part[b + k] = part;
    });
}

// A run of few elements, in one launch of one block.  A slot that the walk misses for offsets out of order keeps
// the zeros written first.
template <int KL>
__global__ void __launch_bounds__(kBlock) policy_one_kernel(PolicyArgs A, int reduce) {
    __shared__ uint8_t s_nibble[kOnePolicy / 4];
    __shared__ int s_rows[kOnePolicy];
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t none[3] = {0, 0, 0};
    const double nothing[4] = {0, 0, 0, 0};
    for (int64_t k = threadIdx.x; k < t.num_slots; k += kBlock) {
        leave_slot(A, k, nothing, 0, none);
        if (A.status && !slot_view(t, k, e_base, r_base).ok) *A.status = kErrTiles;
    }
    __syncthreads();
    if (t.num_elems == 0) return;
    each_slot(t, e_base, r_base, first_slot(t, e_base, 0), 0, t.num_elems,
              [&](int64_t k, const SlotView& s, int64_t a0, int64_t a1) {
        const Span p(s, a0, a1, 0, kBlock);
        const PolicyChunk C = policy_chunk(A, s, 0);
        for (int i = threadIdx.x; i < s.rows; i += kBlock) s_rows[i] = 0;
        __syncthreads();
        int count = 0;
        for (Group q = p.first((int)threadIdx.x); q.o < p.o1; p.advance(&q)) {
            const uint32_t on = count_mask(q, load4<int4u, true>(t.d_labels, q.o, C.last), p.maxlen, t.shift);
            s_nibble[q.o / 4] = (uint8_t)on;
            count += __builtin_popcount(on);
            if (reduce == ODB_REDUCE_ROW_MEAN) add_to_rows(s_rows, q, on, p.maxlen, 0);
        }
        __syncthreads();
        if (reduce == ODB_REDUCE_ROW_MEAN) {
            count = 0;
            for (int i = threadIdx.x; i < s.rows; i += kBlock) count += s_rows[i] > 0;
        }
        count = block_total(count);
        const double scale = A.loss_scale * (A.slot_weight ? A.slot_weight[k] : 1.0);
        const double same = reduce == ODB_REDUCE_SUM ? 1.0 : count > 0 ? 1.0 / count : 0.0;
        auto weight = [&](int row, double* f, float* gs) {
            const double w = reduce == ODB_REDUCE_ROW_MEAN ? 1.0 / ((double)s_rows[row] * count) : same;
            *f = w;
            *gs = (float)(scale * w);
        };
        PolicySums S;
        auto counted = [&](const Group& q) { return (uint32_t)s_nibble[q.o / 4]; };
        if (A.entropy) policy_span<KL, true, true, true>(A, C, p, counted, weight, S);
        else policy_span<KL, true, false, true>(A, C, p, counted, weight, S);
        const SlotPart part = block_part(S, 1.0);
        if (threadIdx.x == 0) {
            const int64_t clipped[3] = {part.clipped[0], part.clipped[1], part.clipped[2]};
            leave_slot(A, k, part.sum, part.counted, clipped);
        }
    });
}

using PolicyOneKernel = void (*)(PolicyArgs, int);
const PolicyOneKernel policy_one_kernels[4] = {policy_one_kernel<0>, policy_one_kernel<1>, policy_one_kernel<2>,
                                               policy_one_kernel<3>};

using PolicyKernel = void (*)(PolicyArgs);
#define ODB_POLICY_KERNELS(KL) \
    {{policy_kernel<KL, 0, false>, policy_kernel<KL, 1, false>, policy_kernel<KL, 2, false>}, \
     {policy_kernel<KL, 0, true>, policy_kernel<KL, 1, true>, policy_kernel<KL, 2, true>}}
const PolicyKernel policy_kernels[4][2][3] = {ODB_POLICY_KERNELS(0), ODB_POLICY_KERNELS(1), ODB_POLICY_KERNELS(2),
                                              ODB_POLICY_KERNELS(3)};   // by odb_kl_t, entropies and odb_reduce_t
#undef ODB_POLICY_KERNELS

// The slots' numbers from their chunks' partials, a wave a slot: 5 us for 2,080 slots, waits for loads.
__global__ void __launch_bounds__(kBlock) policy_slots_kernel(PolicyArgs A) {
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int lane = threadIdx.x & (kWave - 1);
    const uint32_t disorder = disorder_words(A.disorder, A.check_blocks);
    for (int64_t k = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); k < t.num_slots;
         k += (int64_t)gridDim.x * kWaves) {
        const SlotView s = slot_view(t, k, e_base, r_base);
        double sum[4] = {0, 0, 0, 0};
        double n = 0, clipped[3] = {0, 0, 0};     // whole numbers below 2^41
        if (!s.ok) {
            if (A.status && lane == 0) *A.status = kErrTiles;
        } else if (s.hi > s.lo) {
            for (int64_t j = (s.lo >> A.chunk_log2) + lane; j <= (s.hi - 1) >> A.chunk_log2; j += kWave) {
                const SlotPart p = A.slot_part[j + k];
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += p.sum[i];
#pragma unroll
                for (int i = 0; i < 3; ++i) clipped[i] += p.clipped[i];
                n += p.counted;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = wave_total(sum[i]);
#pragma unroll
        for (int i = 0; i < 3; ++i) clipped[i] = wave_total(clipped[i]);
        n = wave_total(n);
        if (__any(disorder)) n = sum[0] = sum[1] = sum[2] = sum[3] = clipped[0] = clipped[1] = clipped[2] = 0.0;
        if (lane == 0) {
            const int64_t c[3] = {(int64_t)clipped[0], (int64_t)clipped[1], (int64_t)clipped[2]};
            leave_slot(A, k, sum, (int64_t)n, c);
        }
    }
}

// ------------------------------------------------------------------ preference loss
struct PairArgs {
    odb_tiles_t t;
    const float* logprob;
    const float* ref;
    const int32_t* row_ids;
    const int32_t* pair;
    int64_t num_ids;
    int32_t* row_of;
    int32_t* row_count;
    double* row_sum;
    RowInfo* row_info;
    double* coef;
    PairPart* part;
    uint32_t* bits;
    uint32_t* disorder;
    int32_t* chunk_slot;
    float* loss;
    float* row_loss;
    float* row_reward;
    int64_t* counts;
    float* grad;
    int32_t* status;
    int64_t chunks, check_blocks;
    double beta, margin, smoothing, loss_scale;
    int32_t kind, chunk, quarter_log2;
    bool normalize;
};

// Rows of tiles up to this width are taken several at a time.  us a call, 34 M elements, up to a width of
// 16 / 64 / 256: rows of about 12 533 / 518 / 520, 40 279 / 237 / 243, 100 200 / 170 / 181, 480 124 / 125 / 132.
constexpr int kShortRow = 64;
// Groups of a lane whose loads (two or three each) are under way together: with 1 / 2 / 4 the same takes 231 /
// 237 / 238 (rows of 40), 127 / 125 / 125 (480), 113 / 109 / 109 (2,000).
constexpr int kRowAhead = 2;

// What a wave leaves of a row in its quarter of a chunk, by its lane 0.
__device__ __forceinline__ void leave_row(const PairArgs& A, const SlotView& s, int64_t part, int64_t c0, int row,
                                          int count, double sum, int lane) {
    if (lane != 0) return;
    const int64_t at = s.row0 + row, start = s.lo + (int64_t)row * s.maxlen;
    const int64_t last = (start + s.maxlen - 1) >> A.quarter_log2;
    if (start >= c0) {   // the row starts here
        const bool whole = last == part;
        A.row_info[at] = RowInfo{whole ? sum : 0.0, whole ? count : 0, (int32_t)(last - part + 1), (int32_t)part, 0};
        if (whole) return;
    }
    A.row_count[part + at] = count;
    A.row_sum[part + at] = sum;
}

// The lowest n of four bits.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 4 ? 0xfu : (1u << n) - 1; }

// The wave's part of a slot with longer rows: positions [a0, a1) - c0 of its quarter.
template <bool REF, bool SAFE>
__device__ __forceinline__ void long_rows(const PairArgs& A, const SlotView& s, int64_t part, int64_t c0, int64_t a0,
                                          int64_t a1, int last, int lane, uint32_t* bits) {
    const int32_t* labels = A.t.d_labels + c0;
    const float* logprob = A.logprob + c0;
    const float* ref = A.ref + c0;
    const int o0 = (int)(a0 - c0), o1 = (int)(a1 - c0), shift = A.t.shift;
    int row = (int)((a0 - s.lo) / s.maxlen);
    // the current row's positions in the quarter; its start may lie before, its end behind
    int64_t ends = s.lo + ((int64_t)row + 1) * s.maxlen - c0;
    int begin = ends - s.maxlen >= 0 ? (int)(ends - s.maxlen) + shift : 0;
    int count = 0;          // of the lane
    double sum = 0.0;
    for (int o = o0 & ~3; o < o1; o += 4 * kWave * kRowAhead) {   // uniform
        int4u y[kRowAhead];
        float4u lp[kRowAhead], rf[kRowAhead];
#pragma unroll
        for (int i = 0; i < kRowAhead; ++i) {
            const int at = o + 4 * (kWave * i + lane);
            y[i] = load4<int4u, SAFE>(labels, at, last);
            lp[i] = load4<float4u, SAFE>(logprob, at, last);
            if (REF) rf[i] = load4<float4u, SAFE>(ref, at, last);
        }
#pragma unroll
        for (int i = 0; i < kRowAhead; ++i) {
            const int from = o + 4 * kWave * i, at = from + 4 * lane;
            if (from >= o1) break;     // uniform
            const int to = from + 4 * kWave < o1 ? from + 4 * kWave : o1;
            uint32_t real = 0, on = 0;
            double x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                real |= (uint32_t)(y[i][j] != ODB_LABEL_IGNORE) << j;
                x[j] = REF ? (double)lp[i][j] - (double)rf[i][j] : (double)lp[i][j];
            }
            for (;;) {     // the rows in these 256 elements; uniform
                const int z = ends < to ? (int)ends : to;
                const uint32_t mine = real & low_bits(z - at) & ~low_bits(begin - at);   // none behind the slot
                on |= mine;
                count += __builtin_popcount(mine);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += mine >> j & 1 ? x[j] : 0.0;
                if (ends > to || (ends == to && to == o1)) break;
                leave_row(A, s, part, c0, row, wave_total(count), wave_total(sum), lane);
                count = 0;
                sum = 0.0;
                ++row;
                begin = (int)ends + shift;
                ends += s.maxlen;
                if (begin - shift >= to) break;
            }
            if (on) atomicOr(&bits[at >> 5], on << (at & 31));
        }
    }
    leave_row(A, s, part, c0, row, wave_total(count), wave_total(sum), lane);
}

// The same with rows of up to 64 elements, taken by the smallest power of two of lanes that covers them
// four elements each.
template <bool REF>
__device__ __forceinline__ void short_rows(const PairArgs& A, const SlotView& s, int64_t part, int64_t c0, int64_t a0,
                                           int64_t a1, int last, int lane, uint32_t* bits) {
    const int row_a = (int)((a0 - s.lo) / s.maxlen), row_b = (int)((a1 - 1 - s.lo) / s.maxlen);
    const int o0 = (int)(a0 - c0), o1 = (int)(a1 - c0);
    int lanes = 1;
    while (4 * lanes < s.maxlen) lanes *= 2;
    const int sub = lane & (lanes - 1);
    // every group of lanes goes round as often as the first, so that none leaves a reduction alone
    for (int r0 = row_a; r0 <= row_b; r0 += kWave / lanes) {
        const int r = r0 + lane / lanes;
        int count = 0;
        double sum = 0.0;
        if (r <= row_b) {
            // positions in the quarter; a row's start may lie before it
            const int start = (int)(s.lo + (int64_t)r * s.maxlen - c0);
            const int x0 = start > o0 ? start : o0, x1 = start + s.maxlen < o1 ? start + s.maxlen : o1;
            const int o = x0 + 4 * sub, from = start + A.t.shift;
            if (o < x1) {
                uint32_t on = low_bits(x1 - o) & ~low_bits(from - o);
                int4u y;
                float4u p, q = {0, 0, 0, 0};
                if (o <= last) {
                    y = load4<int4u, false>(A.t.d_labels + c0, o, last);
                    p = load4<float4u, false>(A.logprob + c0, o, last);
                    if (REF) q = load4<float4u, false>(A.ref + c0, o, last);
                } else {
                    y = load4<int4u, true>(A.t.d_labels + c0, o, last);
                    p = load4<float4u, true>(A.logprob + c0, o, last);
                    if (REF) q = load4<float4u, true>(A.ref + c0, o, last);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (y[j] == ODB_LABEL_IGNORE) on &= ~(1u << j);
                    const double x = REF ? (double)p[j] - (double)q[j] : (double)p[j];
                    sum += on >> j & 1 ? x : 0.0;
                }
                count = __builtin_popcount(on);
                const uint64_t w = (uint64_t)on << (o & 31);
                if ((uint32_t)w) atomicOr(&bits[o >> 5], (uint32_t)w);
                if (w >> 32) atomicOr(&bits[(o >> 5) + 1], (uint32_t)(w >> 32));
            }
        }
        for (int d = lanes / 2; d > 0; d >>= 1) {
            count += __shfl_xor(count, d, kWave);
            sum += __shfl_xor(sum, d, kWave);
        }
        if (r <= row_b) leave_row(A, s, part, c0, r, count, sum, sub);
    }
}

// First pass: the bits, and per quarter of a chunk and row how many tokens count and the sum over
// them.  A wave takes a quarter.  Rows of more than 64 elements are summed across the wave as its 256
// elements at a time come in and are left where they end.  Bound by the reads: 67 M elements of labels and two
// log-probabilities, rows of about 480 with prompts, 157 us for 821 MB (5.3 TB/s).
template <bool REF>
__device__ __forceinline__ void row_sums(const PairArgs& A, uint32_t* s_bits) {
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    const int words = A.chunk / 32, quarter = A.chunk / kWaves;
    // (uniform over the wave, which the compiler does not see by itself)
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t b = blockIdx.x;
    if (A.row_of) {      // the ids' first rows, beside the tiles
        const int64_t rows = run_rows(t, r_base);
        for (int64_t i = b * kBlock + threadIdx.x; i < rows; i += (int64_t)gridDim.x * kBlock) {
            const int32_t id = A.row_ids[i];
            if (id >= 0 && id < A.num_ids) atomicMin(&A.row_of[id], (int32_t)i);
        }
    }
    if (b * A.chunk >= total) return;
    for (int i = threadIdx.x; i < words; i += kBlock) s_bits[i] = 0;
    __syncthreads();
    const int64_t part = b * kWaves + wave, c0 = part * quarter, c1 = c0 + quarter < total ? c0 + quarter : total;
    if (c0 < c1) {
        const int64_t k0 = first_slot(t, e_base, c0);
        if (threadIdx.x == 0) A.chunk_slot[b] = (int32_t)k0;     // the first wave's quarter starts the chunk
        const int last = last_four(t, c0);
        uint32_t* bits = s_bits + wave * (quarter / 32);
        each_slot(t, e_base, r_base, k0, c0, c1, [&](int64_t, const SlotView& s, int64_t a0, int64_t a1) {
            if (s.maxlen <= kShortRow)
                short_rows<REF>(A, s, part, c0, a0, a1, last, lane, bits);
            else if (at_end((int)(a1 - c0), last))
                long_rows<REF, true>(A, s, part, c0, a0, a1, last, lane, bits);
            else
                long_rows<REF, false>(A, s, part, c0, a0, a1, last, lane, bits);
        });
    }
    __syncthreads();
    for (int i = threadIdx.x; i < words; i += kBlock) A.bits[b * words + i] = s_bits[i];
}

// What a wave leaves of its lanes' slots: the status and the rows that the walk passes over.
struct MarkRows {
    const PairArgs& A;

    __device__ __forceinline__ void operator()(bool real, const SlotView& s) const {
        if (real && !s.ok && A.status) *A.status = kErrTiles;
        for (uint64_t bad = __ballot(real && !s.ok && s.ordered); bad; bad &= bad - 1) {
            const int of = __builtin_ctzll(bad);
            const int64_t row1 = __shfl(s.row1, of, kWave);
            for (int64_t i = __shfl(s.row0, of, kWave) + (threadIdx.x & (kWave - 1)); i < row1; i += kWave)
                A.row_info[i] = RowInfo{};
        }
    }
};

template <bool REF>
__global__ void __launch_bounds__(kBlock) row_sums_kernel(PairArgs A) {
    __shared__ uint32_t s_bits[kMaxChunk / 32];
    if (blockIdx.x >= A.chunks)
        check_slots(A.t, blockIdx.x - A.chunks, A.disorder, A.check_blocks, MarkRows{A});
    row_sums<REF>(A, s_bits);
}

// Clears the entries of the ids that have a row.  The others hold anything: an entry is believed
// only if the row that it names has the id.
__device__ __forceinline__ void clear_rows(const PairArgs& A) {
    const int64_t rows = run_rows(A.t, A.t.d_slot_row_off[0]);
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < rows; i += (int64_t)gridDim.x * kBlock) {
        const int32_t id = A.row_ids[i];
        if (id >= 0 && id < A.num_ids) A.row_of[id] = INT32_MAX;
    }
}

__global__ void __launch_bounds__(kBlock) clear_rows_kernel(PairArgs A) { clear_rows(A); }

// A lane's row's log ratio from its record (if `live`); nothing is read outside the partials whatever that
// holds.  Every lane of the wave must be active.  A lane reads its row's parts 4 at a time, or the wave those
// of its long rows one row after the other, 64 parts at a time: whichever takes fewer waits.  (Two rows of
// 131,072 tokens: 12 us a call by the wave, 91 with a lane reading one part at a time; 100 rows of 40,000: 37
// by the lanes, 94 by the wave.)
constexpr int kLaneParts = 16;

__device__ __forceinline__ double log_ratio(const PairArgs& A, int64_t row, const RowInfo& f, bool live, int* count) {
    constexpr int kLoads = 4;
    const int lane = threadIdx.x & (kWave - 1);
    const bool joined = live && f.parts > 1 && f.first >= 0 && (int64_t)f.first + f.parts <= kWaves * A.chunks;
    int n = live ? f.count : 0;
    double s = live ? f.sum : 0.0;
    uint64_t many = __ballot(joined && f.parts > kLaneParts);
    if (!__any(joined && f.parts >= kLaneParts * __builtin_popcountll(many))) many = 0;
    if (joined && !(many >> lane & 1)) {
        for (int b = 0; b < f.parts; b += kLoads) {
            int c[kLoads];
            double v[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int64_t at = f.first + row + (b + i < f.parts ? b + i : f.parts - 1);
                c[i] = A.row_count[at];
                v[i] = A.row_sum[at];
            }
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                n += b + i < f.parts ? c[i] : 0;
                s += b + i < f.parts ? v[i] : 0.0;
            }
        }
    }
    for (; many; many &= many - 1) {
        const int of = __builtin_ctzll(many);
        const int parts = __builtin_amdgcn_readlane(f.parts, of);
        const int64_t first = __shfl(f.first + row, of, kWave);
        int m = 0;
        double t = 0.0;
#pragma unroll 4
        for (int b = lane; b < parts; b += kWave) {
            m += A.row_count[first + b];
            t += A.row_sum[first + b];
        }
        m = wave_total(m);
        t = wave_total(t);
        if (lane == of) {
            n += m;
            s += t;
        }
    }
    *count = n;
    return n == 0 ? 0.0 : A.normalize ? s / n : s;
}

// Row of a row's partner (-1: none here), and whether the row is the chosen one.  What may be needed is
// loaded at once, from the first entry where there is none: two waits instead of five.
__device__ __forceinline__ int64_t partner_row(const PairArgs& A, int64_t row, int64_t rows, bool* chosen) {
    const int64_t id = A.row_ids ? A.row_ids[row] : row;
    *chosen = false;
    if (id < 0 || id >= A.num_ids) {
        if (A.status) *A.status = kErrPair;
        return -1;
    }
    const int64_t v = A.pair[id];
    if (v == 0) return -1;
    const int64_t other = (v < 0 ? -v : v) - 1;
    const int64_t at = other < A.num_ids ? other : 0;
    // written by atomics, in one block's case in this launch: read behind the first cache
    auto row_of = [&](int64_t i) {
        return (int64_t)__hip_atomic_load(&A.row_of[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    const int64_t back = A.pair[at], first = A.row_of ? row_of(id) : row;
    const int64_t j = A.row_of ? row_of(at) : at;
    if (other >= A.num_ids || back != (v < 0 ? id + 1 : -(id + 1))) {
        if (A.status) *A.status = kErrPair;
        return -1;
    }
    *chosen = v > 0;
    // a later row of an id that has one already, or a partner without a row
    if (first != row || j < 0 || j >= rows) return -1;
    return j;
}

// What a thread's rows add up to.
struct PairSums {
    double loss = 0.0;
    int pairs = 0, right = 0;
};

// Of a lane's row, if it is below `rows`: its loss (at the chosen row of a pair) and reward, if `out`, and the
// factor of its tokens' gradients; all 0 if slots are out of order (a word of `disorder` is set: the records may
// hold anything).  Every lane of the wave must be active.
__device__ __forceinline__ double pair_row(const PairArgs& A, int64_t row, int64_t rows, uint32_t disorder, bool out,
                                           PairSums* sums) {
    const bool live = row < rows;
    RowInfo mine{}, its{};
    bool chosen = false;
    int64_t j = -1;
    if (live) {
        mine = A.row_info[row];
        j = partner_row(A, row, rows, &chosen);
        its = A.row_info[j >= 0 ? j : row];
        if (mine.parts == 0 || its.parts == 0) j = -1;
        // an id's entry is believed only if the row that it names has the id
        if (j >= 0 && A.row_of) {
            const int64_t v = A.pair[A.row_ids[row]];
            if (A.row_ids[j] != (v < 0 ? -v : v) - 1) j = -1;
        }
    }
    const bool sound = !__any(disorder);
    if (!sound) j = -1;
    int n, m;
    const double S = log_ratio(A, row, mine, live && sound, &n), T = log_ratio(A, j, its, j >= 0, &m);
    double c = 0.0, loss = 0.0;
    if (j >= 0) {
        const double h = A.beta * (chosen ? S - T : T - S) - A.margin;
        double dh;
        if (A.kind == ODB_PREFERENCE_SIGMOID) {
            const double q = exp(-fabs(h)), soft = log1p(q);           // -ln s(|h|)
            const double far = 1.0 / (1.0 + q), near = q / (1.0 + q);  // s(|h|), s(-|h|)
            const double up = h >= 0 ? far : near, down = h >= 0 ? near : far;
            // no product of 0 and an infinite side: a rejected label at -inf makes h infinite
            loss = (A.smoothing < 1.0 ? (1.0 - A.smoothing) * (soft + (h < 0 ? -h : 0.0)) : 0.0) +
                   (A.smoothing > 0.0 ? A.smoothing * (soft + (h > 0 ? h : 0.0)) : 0.0);
            dh = A.smoothing * up - (1.0 - A.smoothing) * down;
        } else if (A.kind == ODB_PREFERENCE_HINGE) {
            // a NaN stays one: it is not below 1, and not at or above it either
            loss = h >= 1.0 ? 0.0 : 1.0 - h;
            dh = h >= 1.0 ? 0.0 : h < 1.0 ? -1.0 : h;
        } else {
            loss = (h - 0.5) / A.beta;
            dh = 2.0 * loss / A.beta;
            loss *= loss;
        }
        c = A.loss_scale * A.beta * (chosen ? dh : -dh);
        if (A.normalize) c /= n > 0 ? n : 1;
        loss = chosen ? A.loss_scale * loss : 0.0;
        sums->loss += loss;
        sums->pairs += chosen;
        sums->right += chosen && S > T;
    }
    if (out && live) {
        A.row_loss[row] = (float)loss;
        A.row_reward[row] = (float)(A.beta * S);
    }
    return c;
}

// The pairs, a thread a row: 13 us for 140,000 rows, 7 for 6,000: a chain of waits (row, partner's id, its row,
// its record) with nothing to do meanwhile.
__global__ void __launch_bounds__(kBlock) pairs_kernel(PairArgs A) {
    const odb_tiles_t& t = A.t;
    const int64_t rows = run_rows(t, t.d_slot_row_off[0]);
    const int64_t row = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    PairSums sums;
    const double c = pair_row(A, row, rows, disorder_words(A.disorder, A.check_blocks), true, &sums);
    if (row < rows) A.coef[row] = c;
    PairPart p;
    p.loss = block_total(sums.loss);
    p.pairs = block_total(sums.pairs);
    p.right = block_total(sums.right);
    if (threadIdx.x == 0) A.part[blockIdx.x] = p;
}

// The totals from the threads' sums (whole numbers below 2^31).
__device__ __forceinline__ void leave_totals(const PairArgs& A, double loss, double pairs, double right) {
    loss = block_total(loss);
    pairs = block_total(pairs);
    right = block_total(right);
    if (threadIdx.x == 0) {
        *A.loss = (float)loss;
        A.counts[0] = (int64_t)pairs;
        A.counts[1] = (int64_t)right;
    }
}

// Gradients of the block's chunk from the factors of the rows.
__device__ __forceinline__ void pairs_grad(const PairArgs& A, const double* coef, uint32_t* s_bits) {
    const odb_tiles_t& t = A.t;
    if (!A.grad) return;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    const int64_t b = blockIdx.x, c0 = b * A.chunk, c1 = c0 + A.chunk < total ? c0 + A.chunk : total;
    if (c0 >= c1) return;
    const int64_t k0 = A.chunk_slot[b];
    load_bits(s_bits, A.bits, b, A.chunk);
    each_slot(t, e_base, r_base, k0, c0, c1, [&](int64_t, const SlotView& s, int64_t a0, int64_t a1) {
        const Span p(s, a0, a1, c0, kBlock);
        const double* of_row = coef + s.row0;
        Group q = p.first((int)threadIdx.x);
#pragma unroll 4
        for (; q.o < p.o1; p.advance(&q)) {
            const uint32_t on = s_bits[q.o / 32] >> (q.o & 31) & q.mask;
            const float c = (float)of_row[q.row];
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = on >> j & 1 ? c : 0.0f;
            if (q.col > p.maxlen - 4) {
                Group r = q;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (on >> j & 1) v[j] = (float)of_row[r.row];
                    r.next(p.maxlen);
                }
            }
            store4(A.grad + c0, q, v);
        }
    });
}

// Gradients of the tiles; the first block also sums what the pairs left.  Bound by the writes: 67 M elements
// take 47 us for 269 MB (5.7 TB/s).
__global__ void __launch_bounds__(kBlock) pairs_grad_kernel(PairArgs A, int64_t parts) {
    __shared__ uint32_t s_bits[kMaxChunk / 32];
    if (blockIdx.x == 0) {
        double loss = 0.0, pairs = 0.0, right = 0.0;
        for (int64_t i = threadIdx.x; i < parts; i += kBlock) {
            loss += A.part[i].loss;
            pairs += A.part[i].pairs;
            right += A.part[i].right;
        }
        leave_totals(A, loss, pairs, right);
    }
    pairs_grad(A, A.coef, s_bits);
}

// Runs of at most kBlock rows and kFewChunks chunks: every block forms the factors of all rows instead of
// waiting for a kernel that does, and the first one leaves the rows' numbers.  us a call, this / the two
// kernels: 64 rows of 480 tokens (30 chunks) 10.4 / 12.0, 256 of 1,000 (250) 11.2 / 12.7, 256 of 2,000 (500)
// 14.3 / 14.3, 256 of 32,768 (1,024) 60 / 39.
constexpr int64_t kFewChunks = 256;

__global__ void __launch_bounds__(kBlock) few_rows_kernel(PairArgs A) {
    __shared__ double s_coef[kBlock];
    __shared__ uint32_t s_bits[kMaxChunk / 32];
    const int64_t rows = run_rows(A.t, A.t.d_slot_row_off[0]);
    PairSums sums;
    s_coef[threadIdx.x] = pair_row(A, threadIdx.x, rows, disorder_words(A.disorder, A.check_blocks), blockIdx.x == 0,
                                   &sums);
    if (blockIdx.x == 0) leave_totals(A, sums.loss, sums.pairs, sums.right);
    __syncthreads();
    pairs_grad(A, s_coef, s_bits);
}

__global__ void no_pairs_kernel(PairArgs A) {
    *A.loss = 0.0f;
    A.counts[0] = A.counts[1] = 0;
}

// A run of few elements, which are one chunk, in one launch of one block.
template <bool REF>
__global__ void __launch_bounds__(kBlock) pairs_one_kernel(PairArgs A) {
    __shared__ uint32_t s_bits[kMinChunk / 32];
    __shared__ uint32_t s_disorder[kWaves];
    if (A.row_of) {
        clear_rows(A);
        __threadfence();     // before the atomics on the same entries
        __syncthreads();
    }
    row_sums<REF>(A, s_bits);
    // behind the sums, which have the slots at hand
    check_slots(A.t, 0, s_disorder, 1, MarkRows{A});
    __syncthreads();
    const uint32_t disorder = s_disorder[0] | s_disorder[1] | s_disorder[2] | s_disorder[3];
    const int64_t rows = run_rows(A.t, A.t.d_slot_row_off[0]);
    PairSums sums;
    for (int64_t first = 0; first < rows; first += kBlock) {     // uniform
        const int64_t row = first + threadIdx.x;
        const double c = pair_row(A, row, rows, disorder, true, &sums);
        if (row < rows) A.coef[row] = c;
    }
    leave_totals(A, sums.loss, sums.pairs, sums.right);
    __syncthreads();
    pairs_grad(A, A.coef, s_bits);
}

int check_tile_arrays(const odb_tiles_t* t) {
    if (!t->d_slot_rows || !t->d_slot_maxlen || !t->d_slot_row_off || !t->d_slot_tile_off)
        return set_error(ODB_E_INVALID_ARG, "slot arrays must not be NULL");
    if (t->num_elems > 0 && !t->d_labels) return set_error(ODB_E_INVALID_ARG, "d_labels must not be NULL");
    return ODB_OK;
}

}  // namespace

}  // namespace odb

using namespace odb;

extern "C" size_t odb_loss_workspace_size(const odb_tiles_t* t, int64_t num_ids) {
    if (check_tiles(t) != ODB_OK) return 0;
    if (num_ids < 0 || num_ids > INT32_MAX) {
        set_error(ODB_E_INVALID_ARG, "num_ids must be in [0, 2^31)");
        return 0;
    }
    return loss_layout(t, num_ids).total;
}

extern "C" int odb_policy_loss(const odb_tiles_t* t, const odb_policy_params_t* p, const float* d_logprob,
                               const float* d_old_logprob, const float* d_ref_logprob, const float* d_entropy,
                               const float* d_advantage, const double* d_slot_weight, float* d_slot_loss,
                               float* d_slot_means, int64_t* d_slot_counts, float* d_grad_logprob,
                               float* d_grad_entropy, int32_t* d_status, void* d_ws, size_t ws_bytes, void* stream) {
    ODB_TRY(check_tiles(t));
    if (!p) return set_error(ODB_E_INVALID_ARG, "params is NULL");
    if (p->kl < ODB_KL_NONE || p->kl > ODB_KL_EXP) return set_error(ODB_E_INVALID_ARG, "unknown KL term %d", p->kl);
    if (p->reduce < ODB_REDUCE_TOKEN_MEAN || p->reduce > ODB_REDUCE_SUM)
        return set_error(ODB_E_INVALID_ARG, "unknown reduction %d", p->reduce);
    if (p->token_advantage != 0 && p->token_advantage != 1)
        return set_error(ODB_E_INVALID_ARG, "token_advantage must be 0 or 1");
    if (p->reserved0 != 0) return set_error(ODB_E_INVALID_ARG, "params.reserved0 must be 0");
    if (!(p->clip_low >= 0.0 && p->clip_low <= 1.0)) return set_error(ODB_E_INVALID_ARG, "clip_low must be in [0, 1]");
    if (!(p->clip_high >= 0.0)) return set_error(ODB_E_INVALID_ARG, "clip_high must be >= 0");
    if (!(p->dual_clip == 0.0 || (p->dual_clip > 1.0 && std::isfinite(p->dual_clip))))
        return set_error(ODB_E_INVALID_ARG, "dual_clip must be 0 or finite and > 1");
    // the gradients' coefficients are rounded to fp32
    if (!std::isfinite((float)p->kl_coef) || !std::isfinite((float)p->entropy_coef) || !std::isfinite(p->loss_scale))
        return set_error(ODB_E_INVALID_ARG, "kl_coef and entropy_coef must be finite in fp32, loss_scale finite");
    if (t->num_elems > 0 && !d_entropy && (p->entropy_coef != 0.0 || d_grad_entropy))
        return set_error(ODB_E_INVALID_ARG, "an entropy term needs d_entropy");
    if (t->num_slots == 0) return ODB_OK;
    ODB_TRY(check_tile_arrays(t));
    if (!d_slot_loss || !d_slot_means || !d_slot_counts)
        return set_error(ODB_E_INVALID_ARG, "d_slot_loss, d_slot_means and d_slot_counts must not be NULL");
    if (t->num_elems > 0 && (!d_logprob || !d_advantage || (p->kl != ODB_KL_NONE && !d_ref_logprob)))
        return set_error(ODB_E_INVALID_ARG, "d_logprob, d_advantage and, with a KL term, d_ref_logprob must not be NULL");
    const LossLayout L = loss_layout(t, 0);
    ODB_TRY(check_loss_workspace(L, d_ws, ws_bytes));

    hipStream_t s = static_cast<hipStream_t>(stream);
    PolicyArgs a{};
    a.t = *t;
    a.logprob = d_logprob;
    a.old = d_old_logprob ? d_old_logprob : d_logprob;
    a.on_policy = !d_old_logprob;
    a.ref = d_ref_logprob;
    a.entropy = d_entropy;
    a.advantage = d_advantage;
    a.slot_weight = d_slot_weight;
    a.slot_loss = d_slot_loss;
    a.slot_means = d_slot_means;
    a.slot_counts = d_slot_counts;
    a.grad = d_grad_logprob;
    a.grad_entropy = d_grad_entropy;
    a.bits = ws_at<uint32_t>(d_ws, L.bits);
    a.chunk_slot = ws_at<int32_t>(d_ws, L.chunk_slot);
    a.slot_count = ws_at<int32_t>(d_ws, L.slot_count);
    a.slot_part = ws_at<SlotPart>(d_ws, L.slot_part);
    a.row_count = ws_at<int32_t>(d_ws, L.row_count);
    a.disorder = ws_at<uint32_t>(d_ws, L.disorder);
    a.status = d_status;
    a.chunks = L.chunks;
    a.check_blocks = L.chunks > 0 ? check_blocks(t->num_slots) : 0;
    a.counts = L.chunks >= kManyChunks ? kWave : kMaxElems;
    a.chunk = L.chunk;
    a.chunk_log2 = __builtin_ctz((unsigned)L.chunk);
    a.at_low = std::log1p(-p->clip_low);
    a.at_high = std::log1p(p->clip_high);
    a.at_dual = p->dual_clip > 0.0 ? std::log(p->dual_clip) : HUGE_VAL;
    a.kl_coef = p->kl_coef;
    a.entropy_coef = p->entropy_coef;
    a.loss_scale = p->loss_scale;
    a.low = (float)(1.0 - p->clip_low);
    a.high = (float)(1.0 + p->clip_high);
    a.dual = (float)p->dual_clip;
    a.token_advantage = p->token_advantage;
    // at most 2^23 blocks and, in the first pass, those that look over the slots
    const dim3 grid((unsigned)L.chunks), first((unsigned)(L.chunks + a.check_blocks)), block(kBlock);
    if (t->num_elems <= kOnePolicy && t->num_slots <= kOneSlots) {
        hipLaunchKernelGGL(policy_one_kernels[p->kl], dim3(1), block, 0, s, a, (int)p->reduce);
        ODB_LAUNCHED();
        return ODB_OK;
    }
    if (L.chunks > 0 && p->reduce != ODB_REDUCE_SUM) {
        hipLaunchKernelGGL(p->reduce == ODB_REDUCE_ROW_MEAN ? policy_count_kernel<true> : policy_count_kernel<false>,
                           first, block, 0, s, a);
        ODB_LAUNCHED();
        if (a.counts == kWave) {
            hipLaunchKernelGGL(p->reduce == ODB_REDUCE_ROW_MEAN ? policy_fold_kernel<true> : policy_fold_kernel<false>,
                               dim3(grid_for(t->num_slots, 1)), block, 0, s, a);
            ODB_LAUNCHED();
        }
    }
    if (L.chunks > 0) {
        hipLaunchKernelGGL(policy_kernels[p->kl][d_entropy ? 1 : 0][p->reduce], p->reduce == ODB_REDUCE_SUM ? first : grid,
                           block, 0, s, a);
        ODB_LAUNCHED();
    }
    hipLaunchKernelGGL(policy_slots_kernel, dim3(grid_for(t->num_slots, kWaves)), block, 0, s, a);
    ODB_LAUNCHED();
    return ODB_OK;
}

extern "C" int odb_preference_loss(const odb_tiles_t* t, const odb_preference_params_t* p, const float* d_logprob,
                                   const float* d_ref_logprob, const int32_t* d_row_ids, int64_t num_ids,
                                   const int32_t* d_pair, float* d_loss, float* d_row_loss, float* d_row_reward,
                                   int64_t* d_counts, float* d_grad_logprob, int32_t* d_status, void* d_ws,
                                   size_t ws_bytes, void* stream) {
    ODB_TRY(check_tiles(t));
    if (!p) return set_error(ODB_E_INVALID_ARG, "params is NULL");
    if (p->kind < ODB_PREFERENCE_SIGMOID || p->kind > ODB_PREFERENCE_SQUARE)
        return set_error(ODB_E_INVALID_ARG, "unknown preference loss %d", p->kind);
    if (p->normalize != 0 && p->normalize != 1) return set_error(ODB_E_INVALID_ARG, "normalize must be 0 or 1");
    if (!(p->beta > 0.0 && std::isfinite(p->beta))) return set_error(ODB_E_INVALID_ARG, "beta must be finite and > 0");
    if (!std::isfinite(p->margin) || !std::isfinite(p->loss_scale))
        return set_error(ODB_E_INVALID_ARG, "margin and loss_scale must be finite");
    if (!(p->label_smoothing >= 0.0 && p->label_smoothing <= 1.0) ||
        (p->label_smoothing != 0.0 && p->kind != ODB_PREFERENCE_SIGMOID))
        return set_error(ODB_E_INVALID_ARG, "label_smoothing must be in [0, 1], and 0 unless the loss is the sigmoid");
    if (num_ids < 0 || num_ids > INT32_MAX) return set_error(ODB_E_INVALID_ARG, "num_ids must be in [0, 2^31)");
    if (!d_row_ids && num_ids != t->num_rows)
        return set_error(ODB_E_INVALID_ARG, "without d_row_ids num_ids must be num_rows");
    if (!d_loss || !d_counts) return set_error(ODB_E_INVALID_ARG, "d_loss and d_counts must not be NULL");
    if (t->num_slots > 0) ODB_TRY(check_tile_arrays(t));
    const bool any = t->num_slots > 0;
    if (any && ((t->num_elems > 0 && !d_logprob) || (t->num_rows > 0 && (!d_row_loss || !d_row_reward)) ||
                (num_ids > 0 && !d_pair)))
        return set_error(ODB_E_INVALID_ARG, "d_logprob, d_pair, d_row_loss and d_row_reward must not be NULL");
    const LossLayout L = loss_layout(t, d_row_ids ? num_ids : 0);
    ODB_TRY(check_loss_workspace(L, d_ws, ws_bytes));

    hipStream_t s = static_cast<hipStream_t>(stream);
    PairArgs a{};
    a.t = *t;
    a.logprob = d_logprob;
    a.ref = d_ref_logprob;
    a.row_ids = d_row_ids;
    a.pair = d_pair;
    a.num_ids = num_ids;
    a.row_of = d_row_ids ? ws_at<int32_t>(d_ws, L.row_of) : nullptr;
    a.row_count = ws_at<int32_t>(d_ws, L.row_count);
    a.row_sum = ws_at<double>(d_ws, L.row_sum);
    a.row_info = ws_at<RowInfo>(d_ws, L.row_info);
    a.coef = ws_at<double>(d_ws, L.coef);
    a.part = ws_at<PairPart>(d_ws, L.pair_part);
    a.bits = ws_at<uint32_t>(d_ws, L.bits);
    a.chunk_slot = ws_at<int32_t>(d_ws, L.chunk_slot);
    a.loss = d_loss;
    a.row_loss = d_row_loss;
    a.row_reward = d_row_reward;
    a.counts = d_counts;
    a.grad = d_grad_logprob;
    a.disorder = ws_at<uint32_t>(d_ws, L.disorder);
    a.status = d_status;
    a.chunks = L.chunks;
    a.check_blocks = check_blocks(t->num_slots);
    a.chunk = L.chunk;
    a.quarter_log2 = __builtin_ctz((unsigned)L.chunk) - 2;
    a.beta = p->beta;
    a.margin = p->margin;
    a.smoothing = p->label_smoothing;
    a.loss_scale = p->loss_scale;
    a.kind = p->kind;
    a.normalize = p->normalize;
    const dim3 block(kBlock);
    if (!any) {
        hipLaunchKernelGGL(no_pairs_kernel, dim3(1), dim3(1), 0, s, a);
        ODB_LAUNCHED();
        return ODB_OK;
    }
    if (t->num_elems <= kOnePairs && t->num_slots <= kOneSlots) {
        hipLaunchKernelGGL(d_ref_logprob ? pairs_one_kernel<true> : pairs_one_kernel<false>, dim3(1), block, 0, s, a);
        ODB_LAUNCHED();
        return ODB_OK;
    }
    const int64_t parts = (t->num_rows + kBlock - 1) / kBlock;
    if (a.row_of && parts > 0) {
        hipLaunchKernelGGL(clear_rows_kernel, dim3(grid_for(parts, 1)), block, 0, s, a);
        ODB_LAUNCHED();
    }
    // at most 2^23 blocks and those that look over the slots
    const dim3 sums((unsigned)(L.chunks + a.check_blocks));
    hipLaunchKernelGGL(d_ref_logprob ? row_sums_kernel<true> : row_sums_kernel<false>, sums, block, 0, s, a);
    ODB_LAUNCHED();
    // without gradients the first block is all that the last kernel has to do
    const dim3 grid((unsigned)(a.grad ? std::max(L.chunks, (int64_t)1) : 1));
    if (parts <= 1 && L.chunks <= kFewChunks) {
        hipLaunchKernelGGL(few_rows_kernel, grid, block, 0, s, a);
        ODB_LAUNCHED();
        return ODB_OK;
    }
    if (parts > 0) {
        hipLaunchKernelGGL(pairs_kernel, dim3((unsigned)parts), block, 0, s, a);
        ODB_LAUNCHED();
    }
    hipLaunchKernelGGL(pairs_grad_kernel, grid, block, 0, s, a, parts);
    ODB_LAUNCHED();
    return ODB_OK;
}
