// Which slots a chunk of a run's elements touches, apart from the kernels so that it can be
// checked on the host with slot arrays that contradict each other.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "odb.h"

namespace odb {

// Slot k of a run: its elements [lo, hi) and its first row, counted from the run's first.
struct SlotView {
    int64_t lo, hi;
    int64_t row0;
    int32_t rows, maxlen;
    bool ok;    // the arrays agree and stay inside the run's lengths
};

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
    const int64_t row1 = offset_from(t.d_slot_row_off[k + 1], r_base);
    s.rows = t.d_slot_rows[k];
    s.maxlen = t.d_slot_maxlen[k];
    s.ok = s.rows >= 0 && s.maxlen >= 0 && (s.rows == 0) == (s.maxlen == 0) && 0 <= s.lo && s.lo <= s.hi &&
           s.hi <= t.num_elems && 0 <= s.row0 && s.row0 <= row1 && row1 <= t.num_rows && row1 - s.row0 == s.rows &&
           s.hi - s.lo == (int64_t)s.rows * s.maxlen;
    return s;
}

// Probes of one step of the search below, one a lane.
constexpr int kProbes = 64;

// Last slot of [0, slots) that starts at or before an element (0 if there is none), whatever the
// offsets hold: probe(lo, step, hi) is the first i < kProbes whose slot lo + i * step does not or is
// not below hi, else kProbes.
template <typename Probe>
__host__ __device__ __forceinline__ int64_t search_slot(int64_t slots, const Probe& probe) {
    int64_t lo = 0, hi = slots;
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
// order, until one starts behind them.
template <typename F>
__host__ __device__ __forceinline__ void chunk_slots(const odb_tiles_t& t, int64_t e_base, int64_t r_base,
                                                     int64_t first, int64_t c0, int64_t c1, const F& f) {
    for (int64_t k = first; k < t.num_slots; ++k) {
        const SlotView s = slot_view(t, k, e_base, r_base);
        if (s.lo >= c1) break;
        if (!s.ok || s.hi <= c0 || s.hi == s.lo) continue;
        f(k, s, s.lo > c0 ? s.lo : c0, s.hi < c1 ? s.hi : c1);
    }
}

}  // namespace odb
