// What the losses over a run of tiles share: its slots in chunks of its elements, the first pass over its labels,
// which counts a slot's (or its rows') tokens, and sums in a fixed order.
#pragma once

#include <cmath>

#include "odb_internal.h"
#include "odb_tiles.h"

namespace odb {

namespace {

constexpr int kMinChunk = 1024, kMaxChunk = 8192;    // elements of a chunk
constexpr int kWaves = kBlock / kWave;
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
inline int32_t chunk_for(int64_t elems) {
    int32_t chunk = kMinChunk;
    while (chunk < kMaxChunk && elems >= chunk * (int64_t)2048) chunk *= 2;
    return chunk;
}

inline int check_tiles(const odb_tiles_t* t) {
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

inline int check_tile_arrays(const odb_tiles_t* t) {
    if (!t->d_slot_rows || !t->d_slot_maxlen || !t->d_slot_row_off || !t->d_slot_tile_off)
        return set_error(ODB_E_INVALID_ARG, "slot arrays must not be NULL");
    if (t->num_elems > 0 && !t->d_labels) return set_error(ODB_E_INVALID_ARG, "d_labels must not be NULL");
    return ODB_OK;
}

// Blocks that look over K slots.
inline int64_t check_blocks(int64_t K) { return std::min((K + kBlock - 1) / kBlock, (int64_t)kCheckBlocks); }

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

// ------------------------------------------------------------------ counts of slots and rows
// Groups of a thread whose loads are under way together.
constexpr int kAhead = 4;

// What the first pass over a run's labels leaves of it, and what it goes by.
struct SlotCounts {
    odb_tiles_t t;
    uint32_t* bits;
    int32_t* chunk_slot;        // first slot of every chunk, left by the first pass
    int32_t* slot_count;        // counted tokens (token mean) or complete rows with any (row mean)
    int32_t* row_count;
    uint32_t* disorder;
    int32_t* status;
    int64_t chunks, check_blocks;
    int64_t counts;                     // chunks from a slot's first on that hold what all of them counted
    int32_t chunk, chunk_log2;
};

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
template <bool ROWS, bool BITS>
__global__ void __launch_bounds__(kBlock) slot_count_kernel(SlotCounts A) {
    constexpr bool kNibbles = ROWS || BITS;      // who reads them
    __shared__ alignas(16) uint8_t s_nibble[kNibbles ? kMaxChunk / 4 : 4];
    __shared__ int s_rows[ROWS ? kLdsRows : 1];
    const odb_tiles_t& t = A.t;
    if (blockIdx.x >= A.chunks) return check_slots(t, blockIdx.x - A.chunks, A.disorder, A.check_blocks, NoVisit{});
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    const int64_t b = blockIdx.x, c0 = b * A.chunk, c1 = c0 + A.chunk < total ? c0 + A.chunk : total;
    if (c0 >= c1) return;
    const int32_t* labels = t.d_labels + c0;
    const int last = last_four(t, c0);
    for (int i = threadIdx.x; kNibbles && i < A.chunk / 16; i += kBlock) reinterpret_cast<uint32_t*>(s_nibble)[i] = 0;
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
            if (kNibbles && on) s_nibble[q.o / 4] |= (uint8_t)on;
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
    for (int i = threadIdx.x; BITS && i < A.chunk / 32; i += kBlock) {
        const uint2 w = reinterpret_cast<const uint2*>(s_nibble)[i];
        // eight bytes of four bits to one word
        uint32_t v = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v |= (w.x >> (8 * j) & 0xf) << (4 * j) | (w.y >> (8 * j) & 0xf) << (16 + 4 * j);
        A.bits[b * (A.chunk / 32) + i] = v;
    }
}

// The chunks that a row touches.
struct RowChunks {
    int64_t first, last;

    __device__ __forceinline__ RowChunks(const SlotCounts& A, const SlotView& s, int64_t row) {
        const int64_t start = s.lo + row * s.maxlen;
        first = start >> A.chunk_log2;
        last = (start + s.maxlen - 1) >> A.chunk_log2;
    }
};

// Chunks of a row from which on the wave counts it, and not a lane: with a lane alone the mean over two rows of
// 131,072 tokens takes 26 us, not 17.5; with the wave for all of them rows of 480 in one tile take 15.5, not 14.6.
constexpr int kLongRow = 8;

// Counted tokens of a row, over the chunks it touches, by a lane.
__device__ __forceinline__ double row_tokens(const SlotCounts& A, const SlotView& s, int64_t row) {
    const RowChunks c(A, s, row);
    int n = 0;
    for (int64_t b = c.first; b <= c.last; ++b) n += A.row_count[b + s.row0 + row];
    return n;
}

// The same by the wave; every lane must be active.
__device__ __forceinline__ double long_row_tokens(const SlotCounts& A, const SlotView& s, int64_t row,
                                                  const RowChunks& c) {
    double n = 0;
#pragma unroll 4
    for (int64_t b = c.first + (threadIdx.x & (kWave - 1)); b <= c.last; b += kWave) n += A.row_count[b + s.row0 + row];
    return wave_total(n);
}

// Whether a row has any, by a lane: found in its first chunks, unless all of the row before is a prompt.
__device__ __forceinline__ bool row_counts(const SlotCounts& A, const SlotView& s, int64_t row) {
    const RowChunks c(A, s, row);
    for (int64_t b = c.first; b <= c.last; b += 2) {
        const int64_t next = b < c.last ? b + 1 : b;
        if (A.row_count[b + s.row0 + row] | A.row_count[next + s.row0 + row]) return true;
    }
    return false;
}

// What chunk j counted of a slot: tokens, or (ROWS) whole rows with any and the row that starts in it and goes on.
template <bool ROWS>
__device__ __forceinline__ int chunk_counted(const SlotCounts& A, const SlotView& s, int64_t k, int64_t j) {
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
__device__ __forceinline__ double slot_counted(const SlotCounts& A, const SlotView& s, int64_t k) {
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
__global__ void __launch_bounds__(kBlock) slot_fold_kernel(SlotCounts A) {
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

// exp(d) to about one rounding of fp32: the part of d log2 e that a product loses is put back.
__device__ __forceinline__ float exp_near(float d) {
    const float u = d * kLog2e;
    const float e = __builtin_amdgcn_exp2f(u);
    const float lost = fmaf(d, kLog2eLow, fmaf(d, kLog2e, -u));
    return u > -200.0f && u < 128.0f ? fmaf(e * lost, kLn2, e) : e;    // outside: 0 and infinity
}

}  // namespace

}  // namespace odb
