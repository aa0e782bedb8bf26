// Which slots a chunk of a run's elements touches, and which rows and columns its elements are of,
// apart from the kernels so that they can be checked on the host, with slot arrays that contradict
// each other and at any lengths.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "odb.h"

namespace odb {

// Slot k of a run: its elements [lo, hi) and its first row, counted from the run's first.
struct SlotView {
    int64_t lo, hi;
    int64_t row0, row1;
    int32_t rows, maxlen;
    bool ordered;    // its offsets do not fall and stay inside the run's lengths
    bool ok;         // and its arrays agree
};

// If every slot is ordered, a slot's offsets are where the one before it ends: the walk below then meets
// each ok slot whole, and no two slots share an element or a row.  If one is not, neither holds: the
// search goes by offsets that fall, and the walk ends at one that leaves the run.

// Differences of offsets that may hold anything.
__host__ __device__ __forceinline__ int64_t offset_from(int64_t a, int64_t base) {
    return (int64_t)((uint64_t)a - (uint64_t)base);
}

__host__ __device__ __forceinline__ SlotView slot_view(const odb_tiles_t& t, int64_t k, int64_t e_base,
                                                       int64_t r_base) {
    SlotView s;
    s.lo = offset_from(t.d_slot_tile_off[k], e_base);
    s.hi = offset_from(t.d_slot_tile_off[k + 1], e_base);
    s.row0 = offset_from(t.d_slot_row_off[k], r_base);
    s.row1 = offset_from(t.d_slot_row_off[k + 1], r_base);
    s.rows = t.d_slot_rows[k];
    s.maxlen = t.d_slot_maxlen[k];
    s.ordered = 0 <= s.lo && s.lo <= s.hi && s.hi <= t.num_elems && 0 <= s.row0 && s.row0 <= s.row1 &&
                s.row1 <= t.num_rows;
    s.ok = s.ordered && s.rows >= 0 && s.maxlen >= 0 && (s.rows == 0) == (s.maxlen == 0) &&
           s.row1 - s.row0 == s.rows && s.hi - s.lo == (int64_t)s.rows * s.maxlen;
    return s;
}

// Probes of one step of the search below, one a lane.
constexpr int kProbes = 64;

// Last slot of [lo, hi) that starts at or before an element (lo if there is none), whatever the
// offsets hold: probe(lo, step, hi) is the first i < kProbes whose slot lo + i * step does not or is
// not below hi, else kProbes.
template <typename Probe>
__host__ __device__ __forceinline__ int64_t search_slot(int64_t lo, int64_t hi, const Probe& probe) {
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kProbes - 1) / kProbes;
        const int n = probe(lo, step, hi);
        if (n > 1) lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    return lo;
}

// Elements of the run, never more than its arrays hold.
__host__ __device__ __forceinline__ int64_t run_elems(const odb_tiles_t& t, int64_t e_base) {
    const int64_t n = offset_from(t.d_slot_tile_off[t.num_slots], e_base);
    return n < 0 ? 0 : n < t.num_elems ? n : t.num_elems;
}

// Rows of the run, never more than its arrays hold.
__host__ __device__ __forceinline__ int64_t run_rows(const odb_tiles_t& t, int64_t r_base) {
    const int64_t n = offset_from(t.d_slot_row_off[t.num_slots], r_base);
    return n < 0 ? 0 : n < t.num_rows ? n : t.num_rows;
}

// Calls f(k, slot, a0, a1) for every sound slot k >= first with elements [a0, a1) in [c0, c1), in
// order, until one starts behind them.  last_at(from, e) is the last slot >= from that starts at or
// before element e: where many empty slots (idle ranks' steps) lie together it finds the one behind them.
template <typename LastAt, typename F>
__host__ __device__ __forceinline__ void chunk_slots(const odb_tiles_t& t, int64_t e_base, int64_t r_base,
                                                     int64_t first, int64_t c0, int64_t c1, const LastAt& last_at,
                                                     const F& f) {
    int64_t k = first;
    while (k < t.num_slots) {
        const SlotView s = slot_view(t, k, e_base, r_base);
        if (s.lo >= c1) break;
        if (s.ok && s.hi == s.lo) {
            const int64_t next = last_at(k, s.lo);
            k = next > k ? next : k + 1;
            continue;
        }
        if (s.ok && s.hi > c0) f(k, s, s.lo > c0 ? s.lo : c0, s.hi < c1 ? s.hi : c1);
        ++k;
    }
}

// A thread's group of four elements of a chunk, from position o (a multiple of 4) on: which of them
// lie in the slot, and row and column of the first.  The column is negative where the slot starts
// inside the group.
struct Group {
    int o;
    uint32_t mask;
    int row, col;

    // Walks one element on.
    __host__ __device__ __forceinline__ void next(int maxlen) {
        if (++col == maxlen) {
            col = 0;
            ++row;
        }
    }
};

// A slot's elements [a0, a1) of the chunk that starts at c0, as positions [o0, o1) in it; `threads`
// threads take its groups in turn.  Rows count from the slot's first.
struct Span {
    int o0, o1, maxlen;
    int row_a, col_a;               // of element a0
    int ahead, rows_by, cols_by;    // from a thread's group to its next

    __host__ __device__ __forceinline__ Span(const SlotView& s, int64_t a0, int64_t a1, int64_t c0, int threads)
        : o0((int)(a0 - c0)), o1((int)(a1 - c0)), maxlen(s.maxlen), row_a((int)((a0 - s.lo) / s.maxlen)),
          col_a((int)((a0 - s.lo) - (int64_t)row_a * s.maxlen)), ahead(4 * threads), rows_by(ahead / s.maxlen),
          cols_by(ahead - rows_by * s.maxlen) {}

    __host__ __device__ __forceinline__ uint32_t mask_at(int o) const {
        return (o0 > o ? 0xfu << (o0 - o) : 0xfu) & (o1 - o >= 4 ? 0xfu : 0xfu >> (4 - (o1 - o)));
    }

    // Row of position o >= o0.
    __host__ __device__ __forceinline__ int row_at(int o) const {
        return row_a + (int)(((uint32_t)col_a + (uint32_t)(o - o0)) / (uint32_t)maxlen);
    }

    // First group of a thread; its o may lie behind the span.
    __host__ __device__ __forceinline__ Group first(int thread) const {
        Group q;
        q.o = (o0 & ~3) + 4 * thread;
        const int x = q.o - o0;      // negative only in the group in which the slot starts, where col_a is 0
        q.row = row_a;
        q.col = x;
        if (x >= 0) {
            const uint32_t c = (uint32_t)col_a + (uint32_t)x, r = c / (uint32_t)maxlen;
            q.row += (int)r;
            q.col = (int)(c - r * (uint32_t)maxlen);
        }
        q.mask = q.o < o1 ? mask_at(q.o) : 0;
        return q;
    }

    __host__ __device__ __forceinline__ void advance(Group* q) const {
        q->o += ahead;
        q->row += rows_by;
        if (q->col >= maxlen - cols_by) {    // no sum of two columns: they may pass 2^31
            q->col -= maxlen - cols_by;
            ++q->row;
        } else {
            q->col += cols_by;
        }
        while (q->col < 0) {    // behind the group in which the slot starts, where a step is fewer than 3 columns
            q->col += maxlen;
            --q->row;
        }
        q->mask = q->o < o1 ? mask_at(q->o) : 0;
    }
};

}  // namespace odb
