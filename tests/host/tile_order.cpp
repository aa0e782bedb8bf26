// What the loss kernels make of slot arrays that contradict each other, on the host: as long as every
// slot's offsets are in order the walk over the chunks meets each sound slot whole and no other, and sound
// slots share neither elements nor rows.  Where one's are not, sound slots may be missed, as in the run of
// twelve slots at the end: the passes then have to know.  Prints a line and returns 1 on a mistake.
#include <cstdio>
#include <random>
#include <vector>

#include "odb_tiles.h"

namespace {

constexpr int64_t kChunk = 64;

struct Arrays {
    std::vector<int32_t> rows, maxlen;
    std::vector<int64_t> row_off, tile_off;
    odb_tiles_t t{};

    explicit Arrays(int64_t K) : rows(K), maxlen(K), row_off(K + 1), tile_off(K + 1) {}

    void finish() {
        t.num_slots = (int64_t)rows.size();
        t.d_slot_rows = rows.data();
        t.d_slot_maxlen = maxlen.data();
        t.d_slot_row_off = row_off.data();
        t.d_slot_tile_off = tile_off.data();
    }
};

bool all_ordered(const odb_tiles_t& t) {
    for (int64_t k = 0; k < t.num_slots; ++k)
        if (!odb::slot_view(t, k, t.d_slot_tile_off[0], t.d_slot_row_off[0]).ordered) return false;
    return true;
}

// Elements of every slot that the walk meets.
std::vector<int64_t> walk(const odb_tiles_t& t) {
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0], total = odb::run_elems(t, e_base);
    std::vector<int64_t> met(t.num_slots, 0);
    auto last_at = [&](int64_t from, int64_t e) {
        return odb::search_slot(from, t.num_slots, [&](int64_t lo, int64_t step, int64_t hi) {
            for (int i = 0; i < odb::kProbes; ++i)
                if (lo + i * step >= hi || odb::offset_from(t.d_slot_tile_off[lo + i * step], e_base) > e) return i;
            return odb::kProbes;
        });
    };
    for (int64_t c0 = 0; c0 < total; c0 += kChunk) {
        const int64_t c1 = c0 + kChunk < total ? c0 + kChunk : total;
        odb::chunk_slots(t, e_base, r_base, last_at(0, c0), c0, c1, last_at,
                         [&](int64_t k, const odb::SlotView&, int64_t a0, int64_t a1) { met[k] += a1 - a0; });
    }
    return met;
}

int fail(const char* what, int run, int64_t k) {
    std::printf("%s: run %d, slot %lld\n", what, run, (long long)k);
    return 1;
}

// Sound slots met whole, others not at all, nothing shared.
int check(const odb_tiles_t& t, int run) {
    const std::vector<int64_t> met = walk(t);
    std::vector<char> elem(t.num_elems, 0), row(t.num_rows, 0);
    for (int64_t k = 0; k < t.num_slots; ++k) {
        const odb::SlotView s = odb::slot_view(t, k, t.d_slot_tile_off[0], t.d_slot_row_off[0]);
        if (met[k] != (s.ok ? s.hi - s.lo : 0)) return fail("elements met", run, k);
        if (!s.ok) continue;
        for (int64_t e = s.lo; e < s.hi; ++e)
            if (elem[e]++) return fail("a shared element", run, k);
        for (int64_t i = s.row0; i < s.row1; ++i)
            if (row[i]++) return fail("a shared row", run, k);
    }
    return 0;
}

}  // namespace

int main() {
    std::mt19937_64 rng(13);
    auto pick = [&](int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); };
    int ordered = 0, not_ordered = 0;
    for (int run = 0; run < 6000; ++run) {
        const int64_t K = run % 40 == 0 ? pick(60, 3000) : pick(1, 12);
        Arrays a(K);
        a.row_off[0] = pick(0, 1000);
        a.tile_off[0] = pick(0, 1000);
        for (int64_t k = 0; k < K; ++k) {
            const bool idle = pick(0, 3) == 0;
            a.rows[k] = idle ? 0 : (int32_t)pick(1, 9);
            a.maxlen[k] = idle ? 0 : (int32_t)pick(1, run % 2 || K > 12 ? 9 : 200);
            a.row_off[k + 1] = a.row_off[k] + a.rows[k];
            a.tile_off[k + 1] = a.tile_off[k] + (int64_t)a.rows[k] * a.maxlen[k];
        }
        a.t.num_rows = a.row_off[K] - a.row_off[0] + pick(0, 3);
        a.t.num_elems = a.tile_off[K] - a.tile_off[0] + pick(0, 70);
        a.finish();
        if (!all_ordered(a.t)) return fail("sound offsets out of order", run, -1);
        if (check(a.t, run)) return 1;
        // up to three entries that hold anything
        const int64_t odd[] = {INT64_MIN, INT64_MAX, -1, 0, 1, 1ll << 31, 1ll << 40, -(1ll << 40)};
        for (int64_t n = pick(1, 3); n > 0; --n) {
            const int64_t v = pick(0, 1) ? odd[pick(0, 7)] : pick(-300, 3000);
            switch (pick(0, 5)) {
                case 0: a.rows[pick(0, K - 1)] = (int32_t)v; break;
                case 1: a.maxlen[pick(0, K - 1)] = (int32_t)v; break;
                case 2: a.row_off[pick(0, K)] = v; break;
                case 3: a.tile_off[pick(0, K)] = v; break;
                case 4: a.row_off[pick(0, K)] += pick(-3, 3); break;
                default: a.tile_off[pick(0, K)] += pick(-9, 9); break;
            }
        }
        if (!all_ordered(a.t)) {
            ++not_ordered;
            continue;
        }
        ++ordered;
        if (check(a.t, run)) return 1;
    }
    if (ordered < 1000 || not_ordered < 1000) return fail("too few of a kind", ordered, not_ordered);

    Arrays a(12);
    for (int64_t k = 0; k < 12; ++k) {
        a.rows[k] = 10;
        a.maxlen[k] = 70;
        a.row_off[k + 1] = 10 * (k + 1);
        a.tile_off[k + 1] = 700 * (k + 1);
    }
    a.t.num_rows = 120;
    a.t.num_elems = 8400;
    a.finish();
    for (const int64_t wrong : {(int64_t)1 << 40, (int64_t)9000, (int64_t)8400}) {
        a.tile_off[2] = wrong;
        if (all_ordered(a.t)) return fail("a wrong offset in order", (int)wrong, 2);
        int64_t missed = 0;
        for (int64_t k = 0; k < 12; ++k)
            missed += odb::slot_view(a.t, k, 0, 0).ok && walk(a.t)[k] != 700;
        std::printf("tile_off[2] = %lld: %lld sound slots are missed\n", (long long)wrong, (long long)missed);
    }
    return 0;
}
