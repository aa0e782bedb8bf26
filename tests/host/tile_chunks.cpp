// Walks the chunks of runs of tiles as the loss kernels do, over slot arrays that are sound and
// over ones that contradict each other, and checks every index that follows from them against
// the arrays' lengths before it would be used; over sound arrays, that every element is met once
// that partials b + k are met once, and that rows and columns are those of plain division.  Prints one line per mistake, returns 1 if there was any.
#include <cstdio>
#include <random>
#include <vector>

#include "odb_tiles.h"

namespace {

constexpr int64_t kChunk = 64;
int bad = 0;

void fail(const char* what, int64_t a, int64_t b) {
    if (!bad) std::printf("%s: %lld %lld\n", what, (long long)a, (long long)b);
    bad = 1;
}

void walk(const odb_tiles_t& t, bool sound) {
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = odb::run_elems(t, e_base), chunks = (t.num_elems + kChunk - 1) / kChunk;
    if (total < 0 || total > t.num_elems) fail("elements", total, t.num_elems);
    if (odb::run_rows(t, r_base) < 0 || odb::run_rows(t, r_base) > t.num_rows) fail("rows", 0, t.num_rows);
    std::vector<int> met(t.num_elems, 0), part(chunks + t.num_slots, 0);
    for (int64_t b = 0; b < chunks; ++b) {
        const int64_t c0 = b * kChunk, c1 = c0 + kChunk < total ? c0 + kChunk : total;
        if (c0 >= c1) continue;
        auto last_at = [&](int64_t from, int64_t e) {
            return odb::search_slot(from, t.num_slots, [&](int64_t lo, int64_t step, int64_t hi) {
                for (int i = 0; i < odb::kProbes; ++i) {
                    const int64_t at = lo + i * step;
                    if (at >= hi) return i;
                    if (at < 0 || at >= t.num_slots) fail("probe", at, t.num_slots);
                    if (odb::offset_from(t.d_slot_tile_off[at], e_base) > e) return i;
                }
                return odb::kProbes;
            });
        };
        const int64_t first = last_at(0, c0);
        if (first < 0 || first >= t.num_slots) {
            fail("first slot", first, t.num_slots);
            continue;
        }
        odb::chunk_slots(t, e_base, r_base, first, c0, c1, last_at,
                         [&](int64_t k, const odb::SlotView& s, int64_t a0, int64_t a1) {
            if (k < 0 || k >= t.num_slots) return fail("slot", k, t.num_slots);
            if (b + k >= (int64_t)part.size()) return fail("partial", b, k);
            if (a0 < c0 || a1 > c1 || a0 >= a1 || a1 > t.num_elems) return fail("range", a0, a1);
            if (s.maxlen < 1 || s.rows < 1 || s.row0 < 0 || s.row0 + s.rows > t.num_rows) return fail("rows", s.row0, s.rows);
            const int64_t row_b = (a1 - 1 - s.lo) / s.maxlen;
            if (a0 < s.lo || row_b >= s.rows) return fail("row", row_b, s.rows);
            // the chunks that the slot's partials are summed over
            if (s.lo / kChunk > b || (s.hi - 1) / kChunk < b || (s.hi - 1) / kChunk >= chunks) return fail("span", s.lo, s.hi);
            part[b + k] += 1;
            // rows and columns as the threads of a block, or the lanes of a wave, walk them
            for (const int threads : {2, 8}) {
                const odb::Span p(s, a0, a1, c0, threads);
                int64_t seen = 0;
                for (int thread = 0; thread < threads; ++thread) {
                    for (odb::Group q = p.first(thread); q.o < p.o1; p.advance(&q)) {
                        odb::Group r = q;
                        for (int j = 0; j < 4; ++j) {
                            const int64_t e = c0 + q.o + j;
                            if (((q.mask >> j) & 1) != (uint32_t)(e >= a0 && e < a1)) return fail("mask", e, a0);
                            if (q.mask >> j & 1) {
                                ++seen;
                                if (r.row != (e - s.lo) / s.maxlen || r.col != (e - s.lo) % s.maxlen)
                                    return fail("row and column", r.row, r.col);
                            }
                            r.next(s.maxlen);
                        }
                    }
                }
                if (seen != a1 - a0) return fail("elements of a span", seen, a1 - a0);
            }
            for (int64_t e = a0; e < a1; ++e) met[e] += 1;
        });
    }
    if (!sound) return;
    for (int64_t e = 0; e < t.num_elems; ++e)
        if (met[e] != (e < total)) fail("element met", e, met[e]);
    for (int64_t i = 0; i < (int64_t)part.size(); ++i)
        if (part[i] > 1) fail("partial met", i, part[i]);
}

}  // namespace

int main() {
    std::mt19937_64 rng(11);
    auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
    for (int run = 0; run < 4200; ++run) {
        const bool sparse = run >= 4000;    // many idle slots between those with rows
        const int64_t K = sparse || run % 50 == 0 ? pick(60, 9000) : pick(1, 12);
        std::vector<int32_t> rows(K), maxlen(K);
        std::vector<int64_t> row_off(K + 1), tile_off(K + 1);
        row_off[0] = pick(0, 1000);
        tile_off[0] = pick(0, 1000);
        for (int64_t k = 0; k < K; ++k) {
            const bool idle = sparse ? pick(0, 400) > 0 : pick(0, 3) == 0;
            rows[k] = idle ? 0 : (int32_t)pick(1, 9);
            maxlen[k] = idle ? 0 : (int32_t)pick(1, run % 2 || K > 12 ? 9 : 200);
            row_off[k + 1] = row_off[k] + rows[k];
            tile_off[k + 1] = tile_off[k] + (int64_t)rows[k] * maxlen[k];
        }
        odb_tiles_t t{};
        t.num_slots = K;
        t.num_rows = row_off[K] - row_off[0] + pick(0, 3);
        t.num_elems = tile_off[K] - tile_off[0] + pick(0, 70);
        t.d_slot_rows = rows.data();
        t.d_slot_maxlen = maxlen.data();
        t.d_slot_row_off = row_off.data();
        t.d_slot_tile_off = tile_off.data();
        walk(t, true);
        // one to three entries that hold anything
        const int64_t odd[] = {INT64_MIN, INT64_MAX, -1, 0, 1, 1ll << 31, 1ll << 40, -(1ll << 40)};
        for (int64_t n = pick(1, 3); n > 0; --n) {
            const int64_t v = pick(0, 1) ? odd[pick(0, 7)] : pick(-300, 3000);
            switch (pick(0, 5)) {
                case 0: rows[pick(0, K - 1)] = (int32_t)v; break;
                case 1: maxlen[pick(0, K - 1)] = (int32_t)v; break;
                case 2: row_off[pick(0, K)] = v; break;
                case 3: tile_off[pick(0, K)] = v; break;
                case 4: t.num_elems = pick(0, t.num_elems); break;
                default: t.num_rows = pick(0, t.num_rows); break;
            }
        }
        walk(t, false);
    }
    return bad;
}
