// Distillation loss over a run of a plan's tiles, with its gradient: per counted token a divergence between the
// teacher's and the student's log-probabilities of the token's list, reduced and weighted per slot.
//
// A token's k entries lie on a group of L lanes, four each; what a token needs as a whole (sums of
// probabilities, the value, the sum of slopes) is joined by a butterfly over those lanes.  The run's
// elements are cut into pieces wherever slots end, a block each; what a piece adds to a slot is a partial of its
// own, named piece + slot as the chunks' partials are, and partials are summed in a fixed order in 64 bits.
// A mean's weight is known after a pass over the labels, the one that the policy loss makes.
//
// Bound by the reads of both lists and the writes of the gradient, 12 k bytes an element, and beside them by the
// powers, logarithms and series: some 40 to 150 instructions an entry, with the rest most, whose sums need powers in 64
// bits.  2.1 M elements of 32 entries (64% counted), the reverse divergence with the rest: 185 us for 620 MB
// (3.4 TB/s, instructions most of the time); 0.54 M of 27, the mixture, renormalised: 80 us for 172 MB; one
// tile of 16,384 of 64: 15 us, three launches one after the other, of which the lists' pass takes 8.
#include <algorithm>

#include "odb_slots.h"

namespace odb {

namespace {

constexpr float kNone = -HUGE_VALF;          // a teacher's entry that is none
constexpr double kRestLeast = 0x1p-24;       // of what a list leaves out
constexpr int kMaxPiece = 2048;              // elements of a piece; with 4,096 their weights leave too few blocks
constexpr int64_t kMaxDistillElems = (int64_t)1 << 32;     // 2^23 pieces: a grid's threads stay below 2^32

// Chunks of a run from which on what they counted is folded (kManyChunks), unless its slots are many and so, nearly
// all, short: here every piece adds up its slot's counts, four to sixteen times as often as the other losses' chunks.
// us a call without it and with it, one slot of 2^24 / 2^26 / 2^27 elements of 8 entries:
//   mean over tokens         524 / 3,264 /  8,898    365 / 1,405 / 2,790
//   over rows of 512         625 / 5,464 / 19,474    377 / 1,445 / 2,898
// and in slots of 2^20 elements 371 / 1,416 / 2,898, 365 / 1,411 / 2,873 and 393 / 1,501 / 3,049, 388 / 1,471 / 2,987.
constexpr int64_t kManyCounts = 2048;

struct DistillPart {
    double sum;
    int64_t counted;
};

// A mixture's weights, the teacher's w and the student's v, and its series (mixture_entry): with cumulants w v c_n,
//   K(d) = w d (1 + d log_by(d)),   d K' - K = w v d^2 term_by(d).
struct Mixture {
    float w, v;
    float log_by[7];      // of |d| < 1/2: what follows is below 2^-25 of the sum
    float term_by[8];
};

struct DistillArgs : SlotCounts {
    const float* student;
    const float* teacher;
    const double* slot_weight;
    float* slot_loss;
    float* slot_mean;
    int64_t* slot_counted;
    float* grad;
    DistillPart* part;
    int64_t pieces;
    double loss_scale;
    Mixture mix;
    int32_t piece, piece_log2;
    int32_t k, kind, reduce;
};

// ------------------------------------------------------------------ a token
typedef float float4a __attribute__((ext_vector_type(4), aligned(4)));

template <int CTRL>
__device__ __forceinline__ float dpp_of(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double dpp_of(double v) {
    const long long u = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)u, CTRL, 0xf, 0xf, true);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xf, 0xf, true);
    return __longlong_as_double((long long)(((unsigned long long)hi << 32) | lo));
}

// f over a group's L lanes, the same on each: neighbours, pairs, quads and eights exchange (the mirrors swap
// halves whose lanes hold the same by then).
template <int L, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, const F& f) {
    if (L > 1) v = f(v, dpp_of<0xb1>(v));       // quad_perm 1 0 3 2
    if (L > 2) v = f(v, dpp_of<0x4e>(v));       // quad_perm 2 3 0 1
    if (L > 4) v = f(v, dpp_of<0x141>(v));      // row_half_mirror
    if (L > 8) v = f(v, dpp_of<0x140>(v));      // row_mirror
    if (L > 16) v = f(v, __shfl_xor(v, 16, kWave));
    return v;
}
template <int L, typename T>
__device__ __forceinline__ T lanes_sum(T v) {
    return over_lanes<L>(v, [](T a, T b) { return a + b; });
}
template <int L>
__device__ __forceinline__ float lanes_max(float v) {
    return over_lanes<L>(v, [](float a, float b) { return fmaxf(a, b); });
}

// A lane's four entries of a list of k, 4 l and on; those from k on hold anything.
__device__ __forceinline__ void load_entries(const float* p, int k, int l, float v[4]) {
    if (k < 4) {        // uniform
#pragma unroll
        for (int i = 0; i < 3; ++i) v[i] = p[i < k ? i : k - 1];
        v[3] = v[2];
        return;
    }
    const int at = 4 * l < k - 4 ? 4 * l : k - 4, by = 4 * l - at;
    // lists whose fours share lines with their neighbours' are better kept near: 0.52 M lists of 27 take 71 us (mixture,
    // renormalised) and 41 (reverse, as they are), past the caches' usual order 80 and 57; 2.1 M of 32 219 and 217
    const float4a* const from = reinterpret_cast<const float4a*>(p + at);
    const float4a w = k & 3 ? *from : __builtin_nontemporal_load(from);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
    if (k & 3) {        // the last lane's four start up to three entries early
        if (by & 1) {
            v[0] = v[1];
            v[1] = v[2];
            v[2] = v[3];
        }
        if (by & 2) {
            v[0] = v[2];
            v[1] = v[3];
        }
    }
}

__device__ __forceinline__ void store_entries(float* p, int k, int l, const float v[4]) {
    if (4 * l + 4 <= k) {
        const float4a w = {v[0], v[1], v[2], v[3]};
        __builtin_nontemporal_store(w, reinterpret_cast<float4a*>(p + 4 * l));
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (4 * l + i < k) p[4 * l + i] = v[i];
    }
}

// exp(d) for d <= 16 as exp_near gives it; below e^-150 a number as good as 0.  A NaN stays.
__device__ __forceinline__ float exp_below(float d) {
    d = d < -150.0f ? -150.0f : d;
    const float u = d * kLog2e;
    const float e = __builtin_amdgcn_exp2f(u);
    return fmaf(e * fmaf(d, kLog2eLow, fmaf(d, kLog2e, -u)), kLn2, e);
}

// ln x of a normal number to three roundings of it, next to x = 1 too: the hardware's is right to two of itself there.
__device__ __forceinline__ float log_near(float x) { return __builtin_amdgcn_logf(x) * kLn2; }

// An entry's probabilities, and ln p - ln q.
struct Entry {
    float p, q, d;
};

// c[0] + c[1] d + ...
template <int N>
__device__ __forceinline__ float series(const float (&c)[N], float d) {
    float r = c[N - 1];
#pragma unroll
    for (int i = N - 2; i >= 0; --i) r = fmaf(r, d, c[i]);
    return r;
}

// With m = w p + v q and K(d) = ln (v + w e^d) = ln (m / q): the slope v q ln (q / m) is -v q K, and the term
// w p ln (p / m) + v q ln (q / m) is m (d K' - K).  Both come from numbers of d's size, which the term, of d^2's,
// would be the difference of; so for |d| < kNear they are series in d with the cumulants of a weight of w, right
// to themselves however near the student is.  Beyond, ln (m / p) or ln (m / q) is taken where m's other part has the
// smaller weight, in at most half of the distance, which gives the other; past kFar where it is the smaller part.
constexpr float kNear = 0.5f, kFar = 16.0f;
__device__ __forceinline__ void mixture_entry(const Mixture& m, const Entry& x, float* term, float* slope) {
    const float d = x.d, size = fabsf(d);
    // near
    const float near_q = m.w * d * fmaf(d, series(m.log_by, d), 1.0f);
    const float part = m.w * m.v * (d * d) * fmaf(m.w, x.p, m.v * x.q) * series(m.term_by, d);
    // far: from p's side, or from q's
    const bool from_p = size < kFar ? m.w >= 0.5f : d >= 0.0f;
    const float along = from_p ? -d : d, c = from_p ? m.v : m.w, rest = from_p ? m.w : m.v;
    const float power = exp_below(along), u = fmaf(c, power, rest);
    const float lost = fmaf(c, power, -c) - (u - 1.0f);      // of u, which counts where u is next to 1
    const float here = log_near(u) + (u < 2.0f ? lost : 0.0f);
    const float there = here - along;
    const float of_p = from_p ? here : there, of_q = from_p ? there : here;
    const bool near = size < kNear;
    *slope = x.q == 0.0f ? 0.0f : -m.v * x.q * (near ? near_q : of_q);
    *term = near ? part : (x.p == 0.0f ? 0.0f : -m.w * x.p * of_p) + *slope;
}

// ln (1 + x), |x| < 1/2: the logarithm of the rounded sum, and what that lost.
__device__ __forceinline__ float log_beside(float x) {
    const float u = 1.0f + x;
    return log_near(u) + (x - (u - 1.0f));
}

// Where a and b both sum to 1, sum a ln (a / b) is the sum of a ln (a / b) + b - a = a (e^r - 1 - r), r = ln (b / a):
// of none below 0, where the logs' own sum is the small difference of numbers of either sign.  Next to r = 0 a series,
// whose rest is below 2^-27 of it.  *rise: b - a, right to itself there.  Infinite where b has nothing (r = -inf),
// however little a has; past r = 200 a is 0 in 32 bits.
__device__ __forceinline__ float excess(float a, float b, float r, float* rise) {
    const float c[8] = {1.0f / 2, 1.0f / 6, 1.0f / 24, 1.0f / 120, 1.0f / 720, 1.0f / 5040, 1.0f / 40320, 1.0f / 362880};
    const float bend = r * r * series(c, r);
    const bool near = fabsf(r) < kNear;
    *rise = near ? a * (r + bend) : b - a;
    return near ? a * bend : r == -HUGE_VALF ? HUGE_VALF : (b - a) - a * fminf(r, 200.0f);
}

// exp of four numbers in 64 bits to 2^-46, for sums of probabilities that are taken from 1: 2^n exp(g),
// |g| <= ln 2 / 2, by the polynomial of degree 9 whose largest relative error there is least (the series needs degree
// 11: 186 us where this takes 184, 2.1 M lists of 32).  Together, so that a coefficient is there for all.
__device__ __forceinline__ void exp_sums(const float t[4], double e[4]) {
    double g[4];
    int n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = t[i] < -700.0f ? -700.0f : t[i];      // as good as 0; a NaN stays
        const float by = rintf(x * kLog2e);
        n[i] = (int)by;
        g[i] = fma((double)by, -0.69314718055994530942, (double)x);
        e[i] = 2.7482089332277467e-06;
    }
    const double c[9] = {2.4884117327236977e-05, 0.00019841597248962728, 0.0013888802604866363, 0.00833333300152798,
                         0.041666667033890305, 0.1666666666783302, 0.4999999999945516, 0.9999999999998921,
                         1.0000000000000129};
#pragma unroll
    for (int j = 0; j < 9; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = fma(e[i], g[i], c[j]);
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = ldexp(e[i], n[i]);
}

// A counted token's lists with what they leave out as one more entry.  1 - sum cancels, and so does the difference of
// the rests, which stands for the distance of their logs beside the teacher: both in 64 bits.
template <bool MIX, int L>
__device__ __forceinline__ double token_with_rest(const DistillArgs& A, const float t[4], const float s[4],
                                                  const bool there[4], float slope[4]) {
    const Mixture& m = A.mix;
    const bool forward = A.kind == ODB_DISTILL_FORWARD;
    double wide_p[4], wide_q[4], rp = 0.0, rq = 0.0;
    exp_sums(t, wide_p);
    exp_sums(s, wide_q);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        rp += wide_p[i];
        rq += wide_q[i];
    }
    rp = 1.0 - lanes_sum<L>(rp);
    rq = 1.0 - lanes_sum<L>(rq);
    const bool held = rq <= kRestLeast;
    double over = 0.0;      // by how much the teacher's sum is above 1, less the student's
    if (rp < kRestLeast) {      // a NaN stays
        over += kRestLeast - rp;
        rp = kRestLeast;
    }
    if (rq < kRestLeast) {
        over -= kRestLeast - rq;
        rq = kRestLeast;
    }
    Entry rest{(float)rp, (float)rq, 0.0f};
    const float over_q = __builtin_amdgcn_rcpf(rest.q), times = rest.p * over_q;     // 2^-24 to 2^24
    const float apart = (float)(rp - rq) * over_q;      // p / q - 1
    const bool beside = fabsf(apart) < kNear;
    rest.d = beside ? log_beside(apart) : log_near(times);
    float value = 0.0f, term, rise, q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Entry x{(float)wide_p[i], (float)wide_q[i], t[i] - s[i]};
        q[i] = x.q;
        if (MIX) {
            mixture_entry(m, x, &term, &slope[i]);
        } else if (forward) {
            term = excess(x.p, x.q, -x.d, &rise);
            // -p + q rp / rq, unless the student's rest is held
            slope[i] = beside && !held ? fmaf(x.q, apart, rise) : fmaf(x.q, held ? 0.0f : times, -x.p);
        } else {
            term = excess(x.q, x.p, x.d, &rise);
            slope[i] = x.q == 0.0f ? 0.0f : x.q * ((held ? 1.0f : rest.d) - x.d);
        }
        if (!there[i]) term = slope[i] = 0.0f;
        value += term;
    }
    value = lanes_sum<L>(value);
    if (MIX) {
        mixture_entry(m, rest, &term, &rise);
        const float moves = held ? 0.0f : rise * over_q;      // d rq = -q_j d s_j
#pragma unroll
        for (int i = 0; i < 4; ++i) slope[i] = there[i] ? fmaf(-q[i], moves, slope[i]) : 0.0f;
        return (double)value + (double)term;
    }
    term = forward ? excess(rest.p, rest.q, -rest.d, &rise) : excess(rest.q, rest.p, rest.d, &rise);
    return (double)value + (double)term + (forward ? over : -over);
}

// A counted token's lists, each divided by its sum.  The logs of the sums are off by roundings, and with them, beside the
// teacher, all of a token's distances d by the same much more than their own.  By how much, e, is what is left of the sum
// of p - q, which is 0, when one side comes from the other with these distances: the forward and the reverse divergence,
// as sums of their excess, are too large by e^2 / 2 then, their slopes have it taken off.  The mixture, whose
// terms do not show it, has the sums' distance from the sum of the entries' differences, to begin with.
template <bool MIX, int L>
__device__ __forceinline__ double token_renormalized(const DistillArgs& A, const float t[4], const float s[4],
                                                     const bool there[4], float slope[4]) {
    const bool forward = A.kind == ODB_DISTILL_FORWARD;
    const float mt = lanes_max<L>(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])));
    const float ms = lanes_max<L>(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
    Entry x[4];
    float sum_t = 0.0f, sum_s = 0.0f, more = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i].p = there[i] ? exp_below(t[i] - mt) : 0.0f;
        x[i].q = there[i] ? exp_below(s[i] - ms) : 0.0f;
        x[i].d = (t[i] - s[i]) - (mt - ms);
        sum_t += x[i].p;
        sum_s += x[i].q;
        if (MIX) {      // p - q; next to each other q (e^d - 1), the series to 2^-24 of it
            const float c[5] = {1.0f, 1.0f / 2, 1.0f / 6, 1.0f / 24, 1.0f / 120};
            more += fabsf(x[i].d) < 0.125f ? x[i].q * (x[i].d * series(c, x[i].d)) : x[i].p - x[i].q;
        }
    }
    sum_t = lanes_sum<L>(sum_t);      // 1 to k
    sum_s = lanes_sum<L>(sum_s);
    const float over_t = __builtin_amdgcn_rcpf(sum_t), over_s = __builtin_amdgcn_rcpf(sum_s);
    float by = log_near(sum_t * over_s);
    if (MIX) {
        const float apart = lanes_sum<L>(more) * over_s;
        if (fabsf(apart) < kNear) by = log_beside(apart);
    }
    float value = 0.0f, rises = 0.0f, term;      // MIX: rises are slopes
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i].p *= over_t;
        x[i].q *= over_s;
        x[i].d -= by;
        if (MIX)
            mixture_entry(A.mix, x[i], &term, &slope[i]);
        else
            term = excess(forward ? x[i].p : x[i].q, forward ? x[i].q : x[i].p, forward ? -x[i].d : x[i].d, &slope[i]);
        if (!there[i]) term = slope[i] = x[i].q = 0.0f;
        value += term;
        rises += slope[i];
    }
    value = lanes_sum<L>(value);
    rises = lanes_sum<L>(rises);
    if (!MIX) {
        value = fmaf(-0.5f * rises, rises, value);
        if (value < 0.0f) value = 0.0f;      // of no distance but e; a NaN stays
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (MIX || forward)
            slope[i] = fmaf(-x[i].q, rises, slope[i]);
        else
            slope[i] = x[i].q == 0.0f ? 0.0f : -x[i].q * ((x[i].d - rises) + value);
    }
    return value;
}

// A counted token: its value on every lane of the group, and this lane's slopes.
template <bool MIX, int SUPPORT, int L>
__device__ __forceinline__ double token(const DistillArgs& A, int64_t e, int l, float slope[4]) {
    float t[4], s[4];
    bool there[4];
    load_entries(A.teacher + e * A.k, A.k, l, t);
    load_entries(A.student + e * A.k, A.k, l, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        there[i] = 4 * l + i < A.k && t[i] != kNone;
        if (!there[i]) t[i] = s[i] = kNone;
    }
    if (SUPPORT == ODB_SUPPORT_REST) return token_with_rest<MIX, L>(A, t, s, there, slope);
    if (SUPPORT == ODB_SUPPORT_RENORMALIZED) return token_renormalized<MIX, L>(A, t, s, there, slope);
    float value = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Entry x{exp_near(t[i]), exp_near(s[i]), t[i] - s[i]};
        float term;
        if (MIX) {
            mixture_entry(A.mix, x, &term, &slope[i]);
        } else if (A.kind == ODB_DISTILL_FORWARD) {
            term = x.d == HUGE_VALF ? HUGE_VALF : x.p * x.d;      // p may be 0 in 32 bits
            slope[i] = -x.p;
        } else {
            term = x.q == 0.0f ? 0.0f : -x.q * x.d;
            slope[i] = x.q + term;
        }
        if (!there[i]) term = slope[i] = 0.0f;
        value += term;
    }
    return lanes_sum<L>(value);
}

// The block's tokens of a slot's elements [a0, a1): weight(row) gives a token's weight in the reduction and the
// factor of its gradient, by its row counted from the slot's first.
// Row of element e of a slot: a run has 2^32 elements at most.
__device__ __forceinline__ uint32_t row_in(const SlotView& s, int64_t e) {
    return (uint32_t)(e - s.lo) / (uint32_t)s.maxlen;
}

struct DistillSum {
    double sum;
    int counted;
};

template <bool MIX, int SUPPORT, int L, typename Weight>
__device__ __forceinline__ DistillSum distill_span(const DistillArgs& A, const SlotView& s, int64_t a0, int64_t a1,
                                                   const Weight& weight) {
    constexpr int kStep = kBlock / L;      // tokens of the block at once
    const int l = threadIdx.x & (L - 1);
    const uint32_t maxlen = (uint32_t)s.maxlen, row_a = row_in(s, a0), col_a = (uint32_t)(a0 - s.lo) - row_a * maxlen;
    const int n = (int)(a1 - a0);
    DistillSum S{0.0, 0};
    int o = threadIdx.x / L;
    int32_t y = o < n ? A.t.d_labels[a0 + o] : ODB_LABEL_IGNORE;
    // row and column of the thread's token, and from one to its next
    const uint32_t rows_by = kStep / maxlen, cols_by = kStep - rows_by * maxlen;
    uint32_t r = (col_a + (uint32_t)o) / maxlen, col = col_a + (uint32_t)o - r * maxlen;
    auto advance = [&]() {
        r += rows_by;
        col += cols_by;      // below 2 maxlen < 2^32
        if (col >= maxlen) {
            col -= maxlen;
            ++r;
        }
    };
    for (; o < n; o += kStep, advance()) {
        const int32_t label = y;
        if (o + kStep < n) y = A.t.d_labels[a0 + o + kStep];      // on its way beside this token
        const bool on = label != ODB_LABEL_IGNORE && col >= (uint32_t)A.t.shift;
        float g[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (on) {
            const double value = token<MIX, SUPPORT, L>(A, a0 + o, l, g);
            double f;
            float gs;
            weight((int)(row_a + r), &f, &gs);
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = g[i] == 0.0f ? 0.0f : g[i] * gs;      // no entry beside a weight of infinity
            if (l == 0) {
                S.sum += value * f;
                ++S.counted;
            }
        }
        if (A.grad) store_entries(A.grad + (a0 + o) * A.k, A.k, l, g);
    }
    return S;
}

__device__ __forceinline__ void leave_slot(const DistillArgs& A, int64_t k, double sum, int64_t counted) {
    const double scale = A.loss_scale * (A.slot_weight ? A.slot_weight[k] : 1.0);
    A.slot_loss[k] = counted > 0 ? (float)(scale * sum) : 0.0f;
    A.slot_mean[k] = (float)sum;
    A.slot_counted[k] = counted;
}

// ------------------------------------------------------------------ the passes
template <bool MIX, int SUPPORT, int L>
__global__ void __launch_bounds__(kBlock) distill_kernel(DistillArgs A) {
    __shared__ double s_weight[kMaxPiece];
    const odb_tiles_t& t = A.t;
    if (blockIdx.x >= A.pieces) return check_slots(t, blockIdx.x - A.pieces, A.disorder, A.check_blocks, NoVisit{});
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    const int64_t b = blockIdx.x, c0 = b << A.piece_log2, c1 = c0 + A.piece < total ? c0 + A.piece : total;
    if (c0 >= c1) return;
    each_slot(t, e_base, r_base, slot_at(t, e_base, A.reduce == ODB_REDUCE_SUM ? 0 : A.chunk_slot[c0 >> A.chunk_log2], c0),
              c0, c1, [&](int64_t k, const SlotView& s, int64_t a0, int64_t a1) {
        const double scale = A.loss_scale * (A.slot_weight ? A.slot_weight[k] : 1.0);
        const int row_a = (int)row_in(s, a0), here = (int)row_in(s, a1 - 1) - row_a + 1;
        double same = 1.0;       // weight of every token, where rows have none of their own
        if (A.reduce == ODB_REDUCE_TOKEN_MEAN) {
            const double n = slot_counted<false>(A, s, k);
            same = n > 0 ? 1.0 / n : 0.0;
        } else if (A.reduce == ODB_REDUCE_ROW_MEAN) {
            const double rows = slot_counted<true>(A, s, k);
            auto of_count = [&](double n) { return n > 0 ? 1.0 / (n * rows) : 0.0; };
            // only the first and the last of the rows here may be long; below 0: not
            double w_first = -1.0, w_last = -1.0;
            const RowChunks first(A, s, row_a), last(A, s, row_a + here - 1);
            if (first.last - first.first >= kLongRow) w_first = of_count(long_row_tokens(A, s, row_a, first));
            if (here > 1 && last.last - last.first >= kLongRow)
                w_last = of_count(long_row_tokens(A, s, row_a + here - 1, last));
            __syncthreads();      // the slot before this one has read its weights
            for (int i = threadIdx.x; i < here; i += kBlock) {
                const double w = i == 0 ? w_first : i == here - 1 ? w_last : -1.0;
                s_weight[i] = w >= 0.0 ? w : of_count(row_tokens(A, s, row_a + i));
            }
            __syncthreads();
        }
        const float factor = (float)(scale * same);
        const DistillSum S = distill_span<MIX, SUPPORT, L>(A, s, a0, a1, [&](int row, double* f, float* gs) {
            *f = same;
            *gs = factor;
            if (A.reduce == ODB_REDUCE_ROW_MEAN) {
                *f = s_weight[row - row_a];
                *gs = (float)(scale * *f);
            }
        });
        const double sum = block_total(S.sum);
        const int counted = block_total(S.counted);
        if (threadIdx.x == 0) A.part[b + k] = {sum, counted};
    });
}

// The slots' numbers from their pieces' partials, G threads a slot.
template <int G>
__global__ void __launch_bounds__(kBlock) distill_slots_kernel(DistillArgs A) {
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int i = threadIdx.x & (G - 1);
    const uint32_t disorder = disorder_words(A.disorder, A.check_blocks);
    for (int64_t k = (int64_t)blockIdx.x * (kBlock / G) + __builtin_amdgcn_readfirstlane(threadIdx.x / G); k < t.num_slots;
         k += (int64_t)gridDim.x * (kBlock / G)) {
        const SlotView s = slot_view(t, k, e_base, r_base);
        double sum = 0.0, n = 0.0;      // whole numbers below 2^41
        if (!s.ok) {
            if (A.status && i == 0) *A.status = kErrTiles;
        } else if (s.hi > s.lo) {
#pragma unroll 4
            for (int64_t j = (s.lo >> A.piece_log2) + i; j <= (s.hi - 1) >> A.piece_log2; j += G) {
                sum += A.part[j + k].sum;
                n += (double)A.part[j + k].counted;
            }
        }
        sum = G == kBlock ? block_total(sum) : wave_total(sum);
        n = G == kBlock ? block_total(n) : wave_total(n);
        if (__any(disorder)) sum = n = 0.0;
        if (i == 0) leave_slot(A, k, sum, (int64_t)n);
    }
}

// A run of few elements, in one launch of one block.
constexpr int kOneElems = 1024;
constexpr int kOneEntries = 8192;
constexpr int kOneSlots = 1024;

template <bool MIX, int SUPPORT, int L>
__global__ void __launch_bounds__(kBlock) distill_one_kernel(DistillArgs A) {
    __shared__ int s_rows[kOneElems];
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    for (int64_t k = threadIdx.x; k < t.num_slots; k += kBlock) {
        leave_slot(A, k, 0.0, 0);
        if (A.status && !slot_view(t, k, e_base, r_base).ok) *A.status = kErrTiles;
    }
    __syncthreads();
    if (t.num_elems == 0) return;
    each_slot(t, e_base, r_base, first_slot(t, e_base, 0), 0, t.num_elems,
              [&](int64_t k, const SlotView& s, int64_t a0, int64_t a1) {
        const double scale = A.loss_scale * (A.slot_weight ? A.slot_weight[k] : 1.0);
        int count = 0;
        if (A.reduce != ODB_REDUCE_SUM) {
            __syncthreads();      // the slot before this one has read its rows
            for (int i = threadIdx.x; i < s.rows; i += kBlock) s_rows[i] = 0;
            __syncthreads();
            for (int o = threadIdx.x; o < a1 - a0; o += kBlock) {
                const int r = o / s.maxlen;
                if (t.d_labels[a0 + o] != ODB_LABEL_IGNORE && o - r * s.maxlen >= t.shift) {
                    ++count;
                    if (A.reduce == ODB_REDUCE_ROW_MEAN) atomicAdd(&s_rows[r], 1);
                }
            }
            __syncthreads();
            if (A.reduce == ODB_REDUCE_ROW_MEAN) {
                count = 0;
                for (int i = threadIdx.x; i < s.rows; i += kBlock) count += s_rows[i] > 0;
            }
            count = block_total(count);
        }
        const double same = A.reduce == ODB_REDUCE_SUM ? 1.0 : count > 0 ? 1.0 / count : 0.0;
        const DistillSum S = distill_span<MIX, SUPPORT, L>(A, s, a0, a1, [&](int row, double* f, float* gs) {
            *f = A.reduce == ODB_REDUCE_ROW_MEAN ? 1.0 / ((double)s_rows[row] * count) : same;
            *gs = (float)(scale * *f);
        });
        const double sum = block_total(S.sum);
        const int counted = block_total(S.counted);
        if (threadIdx.x == 0) leave_slot(A, k, sum, counted);
    });
}

// ------------------------------------------------------------------ host
// Elements of a piece, a power of two: small ones fill the chip with few tokens, large ones cost fewer searches for
// their slots and fewer sums of their counts.  us in a graph (forward, renormalised; rows of 512 in slots of 32,768) with
// pieces of a 4,096th of the elements, and with larger ones while they have fewer than 4,096 entries and are 512 or more:
// 3.0e7 elements of 1 entry (mean over rows) 525 and 338, 2^22 of 4 72 and 61, 2^16 of 32 20.5 and 18.3, 2^17 of 7 (sum)
// 14.7 and 13.8, 2^17 of 11 (mean over rows) 24.1 and 26.1, 2^14 of 64 (mean over rows) 14.6 and 15.3.  Up to 2,048
// elements and not 512: 526 for the first, 72 for the second.
int32_t piece_for(int64_t elems, int32_t k) {
    int32_t piece = 32;
    while ((piece < 512 && elems / piece >= 4096) || (piece < kMaxPiece && piece * k < 4096 && elems / piece >= 512))
        piece *= 2;
    return piece;
}

// The cumulants of a weight w are w, w v, w v (1 - 2 w), ...: each is w v times the derivative by w of the one before,
// and c_n = (that) / (w v) a polynomial in w, c_{n+1} = (1 - 2 w) c_n + w v c_n'.
Mixture mixture_of(double w) {
    constexpr int kTerms = 9;      // c_2 to c_10
    Mixture m;
    const double v = 1.0 - w;
    m.w = (float)w;
    m.v = (float)v;
    double by[kTerms] = {1.0}, factorial = 1.0;      // c_n's coefficients, n!
    for (int n = 2; n < 10; ++n) {
        double c = 0.0, next[kTerms] = {};
        factorial *= n;
        for (int i = kTerms - 1; i >= 0; --i) c = c * w + by[i];
        if (n - 2 < 7) m.log_by[n - 2] = (float)(v * c / factorial);
        m.term_by[n - 2] = (float)(c * (n - 1) / factorial);
        for (int i = 0; i < n - 1; ++i) {      // (1 - 2 w) by + (w - w^2) by'
            next[i] += by[i] * (1 + i);
            next[i + 1] -= by[i] * (2 + i);
        }
        std::copy(next, next + kTerms, by);
    }
    return m;
}

struct DistillLayout {
    size_t chunk_slot, slot_count, row_count, part, disorder, total;
    int64_t chunks, pieces;
    int32_t chunk, piece;
};

DistillLayout distill_layout(const odb_tiles_t* t, int32_t k) {
    DistillLayout L;
    size_t o = 0;
    auto take = [&](int64_t bytes) {
        const size_t at = o;
        o = (o + (size_t)(bytes > 0 ? bytes : 1) + 255) & ~size_t(255);
        return at;
    };
    L.chunk = chunk_for(t->num_elems);
    L.chunks = (t->num_elems + L.chunk - 1) / L.chunk;
    L.piece = piece_for(t->num_elems, k);
    L.pieces = (t->num_elems + L.piece - 1) / L.piece;
    L.chunk_slot = take(4 * L.chunks);
    L.slot_count = take(4 * (L.chunks + t->num_slots));
    L.row_count = take(4 * (L.chunks + t->num_rows));
    L.part = take((int64_t)sizeof(DistillPart) * (L.pieces + t->num_slots));
    L.disorder = take(4 * kCheckBlocks * kWaves);
    L.total = o;
    return L;
}

int check_distill_tiles(const odb_tiles_t* t, int32_t k) {
    ODB_TRY(check_tiles(t));
    if (k < 1 || k > ODB_LIST_MAX) return set_error(ODB_E_INVALID_ARG, "k must be in [1, %d] (got %d)", ODB_LIST_MAX, k);
    if (t->num_elems > kMaxDistillElems)
        return set_error(ODB_E_INVALID_ARG, "num_elems must be at most 2^32 for lists");
    return ODB_OK;
}

using DistillKernel = void (*)(DistillArgs);
#define ODB_DISTILL_LANES(KERNEL, MIX, SUPPORT) \
    {KERNEL<MIX, SUPPORT, 1>, KERNEL<MIX, SUPPORT, 2>, KERNEL<MIX, SUPPORT, 4>, KERNEL<MIX, SUPPORT, 8>, \
     KERNEL<MIX, SUPPORT, 16>, KERNEL<MIX, SUPPORT, 32>}
#define ODB_DISTILL_KERNELS(KERNEL) \
    {{ODB_DISTILL_LANES(KERNEL, false, 0), ODB_DISTILL_LANES(KERNEL, false, 1), ODB_DISTILL_LANES(KERNEL, false, 2)}, \
     {ODB_DISTILL_LANES(KERNEL, true, 0), ODB_DISTILL_LANES(KERNEL, true, 1), ODB_DISTILL_LANES(KERNEL, true, 2)}}
// by mixture, odb_support_t and the log of a token's lanes
const DistillKernel distill_kernels[2][3][6] = ODB_DISTILL_KERNELS(distill_kernel);
const DistillKernel distill_one_kernels[2][3][6] = ODB_DISTILL_KERNELS(distill_one_kernel);
#undef ODB_DISTILL_KERNELS
#undef ODB_DISTILL_LANES

}  // namespace

}  // namespace odb

using namespace odb;

extern "C" size_t odb_distill_workspace_size(const odb_tiles_t* t, int32_t k) {
    if (check_distill_tiles(t, k) != ODB_OK) return 0;
    return distill_layout(t, k).total;
}

extern "C" int odb_distill_loss(const odb_tiles_t* t, const odb_distill_params_t* p, int32_t k, const float* d_student,
                                const float* d_teacher, const double* d_slot_weight, float* d_slot_loss,
                                float* d_slot_mean, int64_t* d_slot_count, float* d_grad_student, int32_t* d_status,
                                void* d_ws, size_t ws_bytes, void* stream) {
    ODB_TRY(check_distill_tiles(t, k));
    if (!p) return set_error(ODB_E_INVALID_ARG, "params is NULL");
    if (p->kind < ODB_DISTILL_FORWARD || p->kind > ODB_DISTILL_MIXTURE)
        return set_error(ODB_E_INVALID_ARG, "unknown divergence %d", p->kind);
    if (p->support < ODB_SUPPORT_LISTED || p->support > ODB_SUPPORT_REST)
        return set_error(ODB_E_INVALID_ARG, "unknown support %d", p->support);
    if (p->reduce < ODB_REDUCE_TOKEN_MEAN || p->reduce > ODB_REDUCE_SUM)
        return set_error(ODB_E_INVALID_ARG, "unknown reduction %d", p->reduce);
    if (p->reserved0 != 0) return set_error(ODB_E_INVALID_ARG, "params.reserved0 must be 0");
    const bool mix = p->kind == ODB_DISTILL_MIXTURE;
    // both weights are used in 32 bits, as normal numbers
    if (mix && !((float)p->mix >= 0x1p-126f && (float)(1.0 - p->mix) >= 0x1p-126f && p->mix < 1.0))
        return set_error(ODB_E_INVALID_ARG, "mix must be inside (0, 1)");
    if (!std::isfinite(p->loss_scale)) return set_error(ODB_E_INVALID_ARG, "loss_scale must be finite");
    if (t->num_slots == 0) return ODB_OK;
    ODB_TRY(check_tile_arrays(t));
    if (!d_slot_loss || !d_slot_mean || !d_slot_count)
        return set_error(ODB_E_INVALID_ARG, "d_slot_loss, d_slot_mean and d_slot_count must not be NULL");
    if (t->num_elems > 0 && (!d_student || !d_teacher))
        return set_error(ODB_E_INVALID_ARG, "d_student and d_teacher must not be NULL");
    if (!d_ws) return set_error(ODB_E_INVALID_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(d_ws) & 255)
        return set_error(ODB_E_INVALID_ARG, "workspace must be 256-byte aligned");
    const DistillLayout L = distill_layout(t, k);
    if (ws_bytes < L.total)
        return set_error(ODB_E_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, L.total);

    hipStream_t s = static_cast<hipStream_t>(stream);
    DistillArgs a{};
    a.t = *t;
    a.chunk_slot = ws_at<int32_t>(d_ws, L.chunk_slot);
    a.slot_count = ws_at<int32_t>(d_ws, L.slot_count);
    a.row_count = ws_at<int32_t>(d_ws, L.row_count);
    a.disorder = ws_at<uint32_t>(d_ws, L.disorder);
    a.status = d_status;
    a.chunks = L.chunks;
    a.check_blocks = L.chunks > 0 ? check_blocks(t->num_slots) : 0;
    a.counts = L.chunks >= kManyChunks || (L.chunks >= kManyCounts && t->num_slots <= L.chunks) ? kWave : kMaxElems;
    a.chunk = L.chunk;
    a.chunk_log2 = __builtin_ctz((unsigned)L.chunk);
    a.student = d_student;
    a.teacher = d_teacher;
    a.slot_weight = d_slot_weight;
    a.slot_loss = d_slot_loss;
    a.slot_mean = d_slot_mean;
    a.slot_counted = d_slot_count;
    a.grad = d_grad_student;
    a.part = ws_at<DistillPart>(d_ws, L.part);
    a.pieces = L.pieces;
    a.loss_scale = p->loss_scale;
    if (mix) a.mix = mixture_of(p->mix);
    a.piece = L.piece;
    a.piece_log2 = __builtin_ctz((unsigned)L.piece);
    a.k = k;
    a.kind = p->kind;
    a.reduce = p->reduce;
    int lanes = 0;
    while ((4 << lanes) < k) ++lanes;
    const dim3 block(kBlock);
    if (t->num_elems <= kOneElems && t->num_elems * k <= kOneEntries && t->num_slots <= kOneSlots) {
        hipLaunchKernelGGL(distill_one_kernels[mix][p->support][lanes], dim3(1), block, 0, s, a);
        ODB_LAUNCHED();
        return ODB_OK;
    }
    if (L.chunks > 0 && p->reduce != ODB_REDUCE_SUM) {
        hipLaunchKernelGGL((p->reduce == ODB_REDUCE_ROW_MEAN ? slot_count_kernel<true, false>
                                                              : slot_count_kernel<false, false>),
                           dim3((unsigned)(L.chunks + a.check_blocks)), block, 0, s, static_cast<const SlotCounts&>(a));
        ODB_LAUNCHED();
        if (a.counts == kWave) {
            hipLaunchKernelGGL(p->reduce == ODB_REDUCE_ROW_MEAN ? slot_fold_kernel<true> : slot_fold_kernel<false>,
                               dim3(grid_for(t->num_slots, 1)), block, 0, s, static_cast<const SlotCounts&>(a));
            ODB_LAUNCHED();
        }
    }
    if (L.pieces > 0) {     // at most 2^23 of them, and the blocks that look over the slots
        hipLaunchKernelGGL(distill_kernels[mix][p->support][lanes],
                           dim3((unsigned)(L.pieces + (p->reduce == ODB_REDUCE_SUM ? a.check_blocks : 0))), block, 0, s, a);
        ODB_LAUNCHED();
    }
    if (t->num_slots <= 4096)
        hipLaunchKernelGGL((distill_slots_kernel<kBlock>), dim3(grid_for(t->num_slots, 1)), block, 0, s, a);
    else
        hipLaunchKernelGGL((distill_slots_kernel<kWave>), dim3(grid_for(t->num_slots, kWaves)), block, 0, s, a);
    ODB_LAUNCHED();
    return ODB_OK;
}
