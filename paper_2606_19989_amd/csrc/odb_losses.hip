// Losses over a run of a plan's tiles, with their gradients: the clipped policy loss with a KL
// term (one number per slot) and the preference loss (one number per pair of rows).
//
// The run's elements are cut into chunks of equal length wherever slots and rows end, so any mix
// of tiles keeps every compute unit busy.  What a chunk adds to a slot (or a row) is a partial of
// its own: going through the chunks b in order, the slot k never falls, so b + k names each pair
// that occurs once and a slot's partials are neighbours.  They are summed in that order, in 64
// bits, by whoever needs the sum: no atomics, the same result from call to call.
//
// The first pass reads the labels and leaves one bit per element (does it count?), which is all
// that the later passes read of them: 4 bytes an element become 1/8.
#include <cmath>

#include "odb_internal.h"
#include "odb_tiles.h"

namespace odb {

namespace {

constexpr int kChunk = 4096;                   // elements of a chunk
constexpr int kChunkWords = kChunk / 32;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLog2eLow = 1.92596299112661746887e-8f;   // log2 e - kLog2e
constexpr float kLn2 = 0.69314718055994530942f;

typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
typedef int int4u __attribute__((ext_vector_type(4), aligned(4)));

// ------------------------------------------------------------------ workspace
struct SlotPart {
    double sum[4];      // policy, KL, entropy, ratio
    int32_t clipped[3];
    int32_t pad;
};

struct RowInfo {
    int32_t first;      // chunk in which the row starts
    int32_t chunks;     // chunks it touches
};

struct PairPart {
    double loss;
    int32_t pairs, right;
};

struct LossLayout {
    size_t bits, slot_count, slot_part, row_sum, row_count, row_info, row_scale, pair_part, row_of;
    size_t total;
    int64_t chunks;
};

constexpr int64_t kMaxElems = (int64_t)1 << 40;

int check_tiles(const odb_tiles_t* t) {
    if (!t) return set_error(ODB_E_INVALID_ARG, "tiles is NULL");
    if (t->num_slots < 0 || t->num_slots > INT32_MAX)
        return set_error(ODB_E_INVALID_ARG, "num_slots must be in [0, 2^31)");
    if (t->num_rows < 0 || t->num_rows > INT32_MAX) return set_error(ODB_E_INVALID_ARG, "num_rows must be in [0, 2^31)");
    if (t->num_elems < 0 || t->num_elems > kMaxElems)
        return set_error(ODB_E_INVALID_ARG, "num_elems must be in [0, 2^40]");
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
    L.chunks = (t->num_elems + kChunk - 1) / kChunk;
    const int64_t K = t->num_slots, R = t->num_rows;
    L.bits = take(L.chunks * kChunkWords * 4);
    L.slot_count = take(4 * (L.chunks + K));
    L.slot_part = take((int64_t)sizeof(SlotPart) * (L.chunks + K));
    L.row_sum = take(8 * (L.chunks + R));
    L.row_count = take(4 * (L.chunks + R));
    L.row_info = take((int64_t)sizeof(RowInfo) * R);
    L.row_scale = take(8 * R);
    L.pair_part = take((int64_t)sizeof(PairPart) * (R / kBlock + 1));
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

// ------------------------------------------------------------------ first pass: rows and the mask
// Per chunk and row: how many of its tokens count, and (SUM) the sum of logprob - ref over them.
// Per chunk and slot: how many count.  A row is taken by the smallest power of two of lanes that
// covers it four elements each, up to a wave; rows of more than 1,024 elements by the block.
struct RowsArgs {
    odb_tiles_t t;
    const float* logprob;
    const float* ref;
    uint32_t* bits;
    int32_t* slot_count;
    double* row_sum;
    int32_t* row_count;
    RowInfo* row_info;
    const int32_t* row_ids;
    int32_t* row_of;
    int64_t num_ids;
    int64_t chunks;
    int32_t* status;
    bool rows;          // leave row partials
};

constexpr int kLongRow = 1024;

__device__ __forceinline__ void mark(uint32_t* s_bits, int at, uint32_t nibble) {
    if (!nibble) return;
    const uint64_t w = (uint64_t)nibble << (at & 31);
    atomicOr(&s_bits[at >> 5], (uint32_t)w);
    if (w >> 32) atomicOr(&s_bits[(at >> 5) + 1], (uint32_t)(w >> 32));
}

// Elements [a, b) of the run, four a lane of the `lanes` that share a row: count and sum.
template <bool SUM>
__device__ __forceinline__ void row_run(const RowsArgs& A, int64_t a, int64_t b, int64_t first_counted, int lane,
                                        int lanes, int64_t c0, uint32_t* s_bits, int* count, double* sum) {
    for (int64_t e = a + 4 * lane; e < b; e += 4 * lanes) {
        uint32_t nibble = 0;
        if (e + 4 <= b) {
            const int4u y = *reinterpret_cast<const int4u*>(A.t.d_labels + e);
            float4u p = {0, 0, 0, 0}, r = {0, 0, 0, 0};
            if (SUM) {
                p = *reinterpret_cast<const float4u*>(A.logprob + e);
                if (A.ref) r = *reinterpret_cast<const float4u*>(A.ref + e);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool on = y[j] != ODB_LABEL_IGNORE && e + j >= first_counted;
                nibble |= (uint32_t)on << j;
                if (SUM && on) *sum += (double)p[j] - (double)r[j];
            }
        } else {
            for (int j = 0; j < 4 && e + j < b; ++j) {
                const bool on = A.t.d_labels[e + j] != ODB_LABEL_IGNORE && e + j >= first_counted;
                nibble |= (uint32_t)on << j;
                if (SUM && on) *sum += (double)A.logprob[e + j] - (A.ref ? (double)A.ref[e + j] : 0.0);
            }
        }
        *count += __builtin_popcount(nibble);
        mark(s_bits, (int)(e - c0), nibble);
    }
}

template <bool SUM>
__global__ void __launch_bounds__(kBlock) loss_rows_kernel(RowsArgs A) {
    __shared__ uint32_t s_bits[kChunkWords];
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    for (int64_t b = blockIdx.x; b < A.chunks; b += gridDim.x) {   // uniform
        const int64_t c0 = b * kChunk, c1 = c0 + kChunk < total ? c0 + kChunk : total;
        for (int i = threadIdx.x; i < kChunkWords; i += kBlock) s_bits[i] = 0;
        __syncthreads();
        chunk_slots(t, e_base, r_base, c0, c1, [&](int64_t k, const SlotView& s, int64_t a0, int64_t a1) {
            const int64_t row_a = (a0 - s.lo) / s.maxlen, row_b = (a1 - 1 - s.lo) / s.maxlen;
            int slot_count = 0;
            const bool wide = s.maxlen > kLongRow;
            int lanes = 1;
            while (lanes < kWave && 4 * lanes < s.maxlen) lanes *= 2;
            if (wide) lanes = kBlock;
            const int lane = threadIdx.x & (lanes - 1);
            const int step = kBlock / lanes;
            // every group goes round as often as the first, so that no lane leaves a shuffle alone
            for (int64_t r0 = row_a; r0 <= row_b; r0 += step) {
                const int64_t r = r0 + threadIdx.x / lanes;
                const bool live = r <= row_b;
                const int64_t start = s.lo + r * s.maxlen;
                int count = 0;
                double sum = 0.0;
                if (live) {
                    const int64_t x0 = start > a0 ? start : a0, x1 = start + s.maxlen < a1 ? start + s.maxlen : a1;
                    row_run<SUM>(A, x0, x1, start + t.shift, lane, lanes, c0, s_bits, &count, &sum);
                }
                for (int d = (wide ? kWave : lanes) / 2; d > 0; d >>= 1) {
                    count += __shfl_xor(count, d, kWave);
                    if (SUM) sum += __shfl_xor(sum, d, kWave);
                }
                if (wide) {
                    __shared__ int w_count[kBlock / kWave];
                    __shared__ double w_sum[kBlock / kWave];
                    const int w = threadIdx.x / kWave;
                    if ((threadIdx.x & (kWave - 1)) == 0) {
                        w_count[w] = count;
                        w_sum[w] = sum;
                    }
                    __syncthreads();
                    count = 0;
                    sum = 0.0;
#pragma unroll
                    for (int j = 0; j < kBlock / kWave; ++j) {
                        count += w_count[j];
                        sum += w_sum[j];
                    }
                    __syncthreads();
                }
                if (live && lane == 0) {
                    const int64_t row = s.row0 + r;
                    slot_count += count;
                    if (A.rows) {
                        A.row_count[b + row] = count;
                        if (SUM) A.row_sum[b + row] = sum;
                        if (start >= c0) {   // the row starts here
                            const int64_t last = (start + s.maxlen - 1) / kChunk;
                            A.row_info[row] = RowInfo{(int32_t)b, (int32_t)(last - b + 1)};
                            if (A.row_of) {
                                const int32_t id = A.row_ids[row];
                                if (id >= 0 && id < A.num_ids) atomicMin(&A.row_of[id], (int32_t)row);
                            }
                        }
                    }
                }
            }
            slot_count = block_sum(slot_count);
            if (threadIdx.x == 0) A.slot_count[b + k] = slot_count;
        });
        __syncthreads();
        for (int i = threadIdx.x; i < kChunkWords; i += kBlock) A.bits[b * kChunkWords + i] = s_bits[i];
        __syncthreads();
    }
    if (A.status)
        for (int64_t k = (int64_t)blockIdx.x * kBlock + threadIdx.x; k < t.num_slots; k += (int64_t)gridDim.x * kBlock)
            if (!slot_view(t, k, e_base, r_base).ok) *A.status = kErrTiles;
}

__global__ void __launch_bounds__(kBlock) fill_rows_kernel(int32_t* row_of, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock)
        row_of[i] = INT32_MAX;
}

// Sum of a row's partials; nothing is read outside them whatever the row's record holds.
__device__ __forceinline__ int row_total(const int32_t* row_count, const double* row_sum, const RowInfo* info,
                                         int64_t chunks, int64_t row, double* sum) {
    const RowInfo f = info[row];
    int count = 0;
    double s = 0.0;
    if (f.first >= 0 && f.chunks > 0 && (int64_t)f.first + f.chunks <= chunks) {
        for (int64_t b = f.first; b < (int64_t)f.first + f.chunks; ++b) {
            count += row_count[b + row];
            if (sum) s += row_sum[b + row];
        }
    }
    if (sum) *sum = s;
    return count;
}

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
    const uint32_t* bits;
    const int32_t* slot_count;
    SlotPart* slot_part;
    const int32_t* row_count;
    const RowInfo* row_info;
    double* row_scale;
    int64_t chunks;
    double at_low, at_high, at_dual;    // ln(1 - e_l), ln(1 + e_h), ln c
    double kl_coef, entropy_coef, loss_scale;
    float low, high, dual;              // 1 - e_l, 1 + e_h, c
    int32_t kl, reduce;
    bool token_advantage;
};

// Weight of a row's token under the mean of row means: 1 / (the row's tokens * the slot's rows).
__global__ void __launch_bounds__(kBlock) row_scale_kernel(PolicyArgs A) {
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    for (int64_t k = blockIdx.x; k < t.num_slots; k += gridDim.x) {
        const SlotView s = slot_view(t, k, e_base, r_base);
        if (!s.ok || s.rows == 0) continue;   // uniform
        int rows = 0;
        for (int i = threadIdx.x; i < s.rows; i += kBlock)
            rows += row_total(A.row_count, nullptr, A.row_info, A.chunks, s.row0 + i, nullptr) > 0;
        rows = block_sum(rows);
        for (int i = threadIdx.x; i < s.rows; i += kBlock) {
            const int n = row_total(A.row_count, nullptr, A.row_info, A.chunks, s.row0 + i, nullptr);
            A.row_scale[s.row0 + i] = n > 0 ? 1.0 / ((double)n * rows) : 0.0;
        }
    }
}

// exp(d) to about one rounding of fp32: the part of d log2 e that a product loses is put back.
__device__ __forceinline__ float exp_near(float d) {
    const float u = d * kLog2e;
    const float e = __builtin_amdgcn_exp2f(u);
    const float lost = fmaf(d, kLog2eLow, fmaf(d, kLog2e, -u));
    return fabsf(u) < 200.0f ? fmaf(e * lost, kLn2, e) : e;
}

// exp(d) - 1 - d: below 1 by its series (the next term is under 2^-31 of the sum), where the
// difference would cancel.
__device__ __forceinline__ float exp_less_line(float d) {
    if (fabsf(d) < 1.0f) {
        float q = 1.0f / 479001600.0f;
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
    return exp_near(d) - 1.0f - d;
}

struct TokenTerms {
    float policy, ratio, kl, grad, kl_grad;
    int clip;    // 0 none, 1 below, 2 above, 3 by the dual bound
};

__device__ __forceinline__ TokenTerms policy_token(const PolicyArgs& A, float lp, float old, float ref, float adv) {
    TokenTerms o;
    // the comparisons are made on the difference itself; its fp32 rounding is enough for the rest
    const double d = A.old ? (double)lp - (double)old : 0.0;
    o.ratio = A.old ? exp_near(lp - old) : 1.0f;
    o.clip = 0;
    float bound = o.ratio;
    if (adv > 0.0f) {
        if (d > A.at_high) {
            o.clip = 2;
            bound = A.high;
        }
    } else if (adv < 0.0f) {
        if (d < A.at_low) {
            o.clip = 1;
            bound = A.low;
        } else if (d > A.at_dual) {
            o.clip = 3;
            bound = A.dual;
        }
    }
    o.policy = adv == 0.0f ? 0.0f : -bound * adv;
    o.grad = o.clip ? 0.0f : o.policy;
    o.kl = o.kl_grad = 0.0f;
    if (A.kl != ODB_KL_NONE) {
        const float x = lp - ref;
        if (A.kl == ODB_KL_LINEAR) {
            o.kl = x;
            o.kl_grad = 1.0f;
        } else if (A.kl == ODB_KL_SQUARE) {
            o.kl = 0.5f * x * x;
            o.kl_grad = x;
        } else {
            o.kl = exp_less_line(-x);
            o.kl_grad = x - o.kl;    // 1 - exp(-x)
        }
    }
    return o;
}

__global__ void __launch_bounds__(kBlock) policy_kernel(PolicyArgs A) {
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    for (int64_t b = blockIdx.x; b < A.chunks; b += gridDim.x) {   // uniform
        const int64_t c0 = b * kChunk, c1 = c0 + kChunk < total ? c0 + kChunk : total;
        chunk_slots(t, e_base, r_base, c0, c1, [&](int64_t k, const SlotView& s, int64_t a0, int64_t a1) {
            double weight = 1.0;     // of a token in the slot's mean, where it is the same for all
            if (A.reduce == ODB_REDUCE_TOKEN_MEAN) {
                int64_t n = 0;
                for (int64_t j = s.lo / kChunk; j <= (s.hi - 1) / kChunk; ++j) n += A.slot_count[j + k];
                weight = n > 0 ? 1.0 / (double)n : 0.0;
            }
            const double scale = A.loss_scale * (A.slot_weight ? A.slot_weight[k] : 1.0);
            const int64_t row_a = (a0 - s.lo) / s.maxlen;
            const uint32_t col_a = (uint32_t)((a0 - s.lo) - row_a * s.maxlen);
            double sum[4] = {0, 0, 0, 0};
            int clipped[3] = {0, 0, 0};
            for (int64_t e = a0 + threadIdx.x; e < a1; e += kBlock) {
                const uint32_t x = col_a + (uint32_t)(e - a0);
                const int64_t row = s.row0 + row_a + x / (uint32_t)s.maxlen;
                const bool on = A.bits[e / 32] >> (e & 31) & 1;
                float g = 0.0f, ge = 0.0f;
                if (on) {
                    const float adv = A.advantage[A.token_advantage ? e : row];
                    const TokenTerms o = policy_token(A, A.logprob[e], A.old ? A.old[e] : 0.0f,
                                                      A.kl != ODB_KL_NONE ? A.ref[e] : 0.0f, adv);
                    const double w = A.reduce == ODB_REDUCE_ROW_MEAN ? A.row_scale[row] : weight;
                    sum[0] += w * o.policy;
                    sum[1] += w * o.kl;
                    if (A.entropy) sum[2] += w * A.entropy[e];
                    sum[3] += w * o.ratio;
                    clipped[0] += o.clip == 1;
                    clipped[1] += o.clip == 2;
                    clipped[2] += o.clip == 3;
                    g = (float)(scale * w * ((double)o.grad + A.kl_coef * (double)o.kl_grad));
                    ge = (float)(-A.entropy_coef * scale * w);
                }
                if (A.grad) A.grad[e] = g;
                if (A.grad_entropy) A.grad_entropy[e] = ge;
            }
            SlotPart p;
#pragma unroll
            for (int j = 0; j < 4; ++j) p.sum[j] = block_sum(sum[j]);
#pragma unroll
            for (int j = 0; j < 3; ++j) p.clipped[j] = block_sum(clipped[j]);
            p.pad = 0;
            if (threadIdx.x == 0) A.slot_part[b + k] = p;
        });
    }
}

// The slots' numbers from their chunks' partials, a thread a slot.
__global__ void __launch_bounds__(kBlock) policy_slots_kernel(PolicyArgs A) {
    const odb_tiles_t& t = A.t;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    for (int64_t k = (int64_t)blockIdx.x * kBlock + threadIdx.x; k < t.num_slots; k += (int64_t)gridDim.x * kBlock) {
        const SlotView s = slot_view(t, k, e_base, r_base);
        double sum[4] = {0, 0, 0, 0};
        int64_t n = 0, clipped[3] = {0, 0, 0};
        if (s.ok && s.hi > s.lo) {
            for (int64_t j = s.lo / kChunk; j <= (s.hi - 1) / kChunk; ++j) {
                const SlotPart p = A.slot_part[j + k];
                n += A.slot_count[j + k];
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += p.sum[i];
#pragma unroll
                for (int i = 0; i < 3; ++i) clipped[i] += p.clipped[i];
            }
        }
        const double scale = A.loss_scale * (A.slot_weight ? A.slot_weight[k] : 1.0);
        A.slot_loss[k] = n > 0 ? (float)(scale * (sum[0] + A.kl_coef * sum[1] - A.entropy_coef * sum[2])) : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) A.slot_means[4 * k + i] = (float)sum[i];
        A.slot_counts[4 * k] = n;
#pragma unroll
        for (int i = 0; i < 3; ++i) A.slot_counts[4 * k + 1 + i] = clipped[i];
    }
}

// ------------------------------------------------------------------ preference loss
struct PairArgs {
    odb_tiles_t t;
    const int32_t* row_ids;
    const int32_t* pair;
    int64_t num_ids;
    const int32_t* row_of;
    const int32_t* row_count;
    const double* row_sum;
    const RowInfo* row_info;
    double* coef;
    PairPart* part;
    const uint32_t* bits;
    float* loss;
    float* row_loss;
    float* row_reward;
    int64_t* counts;
    float* grad;
    int32_t* status;
    int64_t chunks;
    double beta, margin, smoothing, loss_scale;
    int32_t kind;
    bool normalize;
};

__device__ __forceinline__ double log_ratio(const PairArgs& A, int64_t row, int* count) {
    double s;
    const int n = row_total(A.row_count, A.row_sum, A.row_info, A.chunks, row, &s);
    *count = n;
    return n == 0 ? 0.0 : A.normalize ? s / n : s;
}

// Row of a row's partner (-1: none here), and whether the row is the chosen one.
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
    if (other >= A.num_ids || A.pair[other] != (v < 0 ? id + 1 : -(id + 1))) {
        if (A.status) *A.status = kErrPair;
        return -1;
    }
    *chosen = v > 0;
    if (!A.row_ids) return other < rows ? other : -1;
    if (A.row_of[id] != row) return -1;        // a later row of an id that has one already
    const int64_t j = A.row_of[other];
    return j < rows ? j : -1;
}

__global__ void __launch_bounds__(kBlock) pairs_kernel(PairArgs A) {
    const odb_tiles_t& t = A.t;
    const int64_t rows = run_rows(t, t.d_slot_row_off[0]);
    const int64_t row = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    double loss = 0.0;
    int pairs = 0, right = 0;
    if (row < rows) {
        int n, m;
        const double S = log_ratio(A, row, &n);
        bool chosen;
        const int64_t j = partner_row(A, row, rows, &chosen);
        double c = 0.0;
        if (j >= 0) {
            const double T = log_ratio(A, j, &m);
            const double h = A.beta * (chosen ? S - T : T - S) - A.margin;
            double dh;
            if (A.kind == ODB_PREFERENCE_SIGMOID) {
                const double q = exp(-fabs(h)), soft = log1p(q);       // -ln s(|h|)
                const double far = 1.0 / (1.0 + q), near = q / (1.0 + q);  // s(|h|), s(-|h|)
                const double up = h >= 0 ? far : near, down = h >= 0 ? near : far;
                loss = (1.0 - A.smoothing) * (soft + (h < 0 ? -h : 0.0)) + A.smoothing * (soft + (h > 0 ? h : 0.0));
                dh = A.smoothing * up - (1.0 - A.smoothing) * down;
            } else if (A.kind == ODB_PREFERENCE_HINGE) {
                loss = h < 1.0 ? 1.0 - h : 0.0;
                dh = h < 1.0 ? -1.0 : 0.0;
            } else {
                loss = (h - 0.5) / A.beta;
                dh = 2.0 * loss / A.beta;
                loss *= loss;
            }
            c = A.loss_scale * A.beta * (chosen ? dh : -dh);
            if (A.normalize) c /= n > 0 ? n : 1;
            loss *= A.loss_scale;
            if (chosen) {
                pairs = 1;
                right = S > T;
            } else {
                loss = 0.0;
            }
        }
        A.coef[row] = c;
        A.row_loss[row] = (float)loss;
        A.row_reward[row] = (float)(A.beta * S);
    }
    PairPart p;
    p.loss = block_sum(loss);
    p.pairs = block_sum(pairs);
    p.right = block_sum(right);
    if (threadIdx.x == 0) A.part[blockIdx.x] = p;
}

// Gradients of the tiles; the first block also sums what the pairs left.
__global__ void __launch_bounds__(kBlock) pairs_grad_kernel(PairArgs A, int64_t parts) {
    const odb_tiles_t& t = A.t;
    if (blockIdx.x == 0) {
        double loss = 0.0;
        int64_t pairs = 0, right = 0;
        for (int64_t i = threadIdx.x; i < parts; i += kBlock) {
            loss += A.part[i].loss;
            pairs += A.part[i].pairs;
            right += A.part[i].right;
        }
        loss = block_sum(loss);
        pairs = block_sum(pairs);
        right = block_sum(right);
        if (threadIdx.x == 0) {
            *A.loss = (float)loss;
            A.counts[0] = pairs;
            A.counts[1] = right;
        }
    }
    if (!A.grad || t.num_slots == 0) return;
    const int64_t e_base = t.d_slot_tile_off[0], r_base = t.d_slot_row_off[0];
    const int64_t total = run_elems(t, e_base);
    for (int64_t b = blockIdx.x; b < A.chunks; b += gridDim.x) {   // uniform
        const int64_t c0 = b * kChunk, c1 = c0 + kChunk < total ? c0 + kChunk : total;
        chunk_slots(t, e_base, r_base, c0, c1, [&](int64_t k, const SlotView& s, int64_t a0, int64_t a1) {
            const int64_t row_a = (a0 - s.lo) / s.maxlen;
            const uint32_t col_a = (uint32_t)((a0 - s.lo) - row_a * s.maxlen);
            for (int64_t e = a0 + threadIdx.x; e < a1; e += kBlock) {
                const uint32_t x = col_a + (uint32_t)(e - a0);
                const int64_t row = s.row0 + row_a + x / (uint32_t)s.maxlen;
                const bool on = A.bits[e / 32] >> (e & 31) & 1;
                A.grad[e] = on ? (float)A.coef[row] : 0.0f;
            }
        });
    }
}

int check_tile_arrays(const odb_tiles_t* t) {
    if (!t->d_slot_rows || !t->d_slot_maxlen || !t->d_slot_row_off || !t->d_slot_tile_off)
        return set_error(ODB_E_INVALID_ARG, "slot arrays must not be NULL");
    if (t->num_elems > 0 && !t->d_labels) return set_error(ODB_E_INVALID_ARG, "d_labels must not be NULL");
    return ODB_OK;
}

void rows_args(RowsArgs* r, const odb_tiles_t* t, const LossLayout& L, void* ws, int32_t* status) {
    *r = RowsArgs{};
    r->t = *t;
    r->bits = ws_at<uint32_t>(ws, L.bits);
    r->slot_count = ws_at<int32_t>(ws, L.slot_count);
    r->row_sum = ws_at<double>(ws, L.row_sum);
    r->row_count = ws_at<int32_t>(ws, L.row_count);
    r->row_info = ws_at<RowInfo>(ws, L.row_info);
    r->chunks = L.chunks;
    r->status = status;
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
    if (!std::isfinite(p->kl_coef) || !std::isfinite(p->entropy_coef) || !std::isfinite(p->loss_scale))
        return set_error(ODB_E_INVALID_ARG, "kl_coef, entropy_coef and loss_scale must be finite");
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
    RowsArgs r;
    rows_args(&r, t, L, d_ws, d_status);
    r.rows = p->reduce == ODB_REDUCE_ROW_MEAN;
    PolicyArgs a{};
    a.t = *t;
    a.logprob = d_logprob;
    a.old = d_old_logprob;
    a.ref = d_ref_logprob;
    a.entropy = d_entropy;
    a.advantage = d_advantage;
    a.slot_weight = d_slot_weight;
    a.slot_loss = d_slot_loss;
    a.slot_means = d_slot_means;
    a.slot_counts = d_slot_counts;
    a.grad = d_grad_logprob;
    a.grad_entropy = d_grad_entropy;
    a.bits = r.bits;
    a.slot_count = r.slot_count;
    a.slot_part = ws_at<SlotPart>(d_ws, L.slot_part);
    a.row_count = r.row_count;
    a.row_info = r.row_info;
    a.row_scale = ws_at<double>(d_ws, L.row_scale);
    a.chunks = L.chunks;
    a.at_low = std::log1p(-p->clip_low);
    a.at_high = std::log1p(p->clip_high);
    a.at_dual = p->dual_clip > 0.0 ? std::log(p->dual_clip) : HUGE_VAL;
    a.kl_coef = p->kl_coef;
    a.entropy_coef = p->entropy_coef;
    a.loss_scale = p->loss_scale;
    a.low = (float)(1.0 - p->clip_low);
    a.high = (float)(1.0 + p->clip_high);
    a.dual = (float)p->dual_clip;
    a.kl = p->kl;
    a.reduce = p->reduce;
    a.token_advantage = p->token_advantage;
    const dim3 chunks(grid_for(L.chunks, 1));
    hipLaunchKernelGGL(loss_rows_kernel<false>, chunks, dim3(kBlock), 0, s, r);
    ODB_LAUNCHED();
    if (r.rows) {
        hipLaunchKernelGGL(row_scale_kernel, dim3(grid_for(t->num_slots, 1)), dim3(kBlock), 0, s, a);
        ODB_LAUNCHED();
    }
    hipLaunchKernelGGL(policy_kernel, chunks, dim3(kBlock), 0, s, a);
    ODB_LAUNCHED();
    hipLaunchKernelGGL(policy_slots_kernel, dim3(grid_for(t->num_slots, kBlock)), dim3(kBlock), 0, s, a);
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
    RowsArgs r;
    rows_args(&r, t, L, d_ws, d_status);
    r.logprob = d_logprob;
    r.ref = d_ref_logprob;
    r.row_ids = d_row_ids;
    r.row_of = d_row_ids ? ws_at<int32_t>(d_ws, L.row_of) : nullptr;
    r.num_ids = num_ids;
    r.rows = true;
    PairArgs a{};
    a.t = *t;
    a.row_ids = d_row_ids;
    a.pair = d_pair;
    a.num_ids = num_ids;
    a.row_of = r.row_of;
    a.row_count = r.row_count;
    a.row_sum = r.row_sum;
    a.row_info = r.row_info;
    a.coef = ws_at<double>(d_ws, L.row_scale);
    a.part = ws_at<PairPart>(d_ws, L.pair_part);
    a.bits = r.bits;
    a.loss = d_loss;
    a.row_loss = d_row_loss;
    a.row_reward = d_row_reward;
    a.counts = d_counts;
    a.grad = any ? d_grad_logprob : nullptr;
    a.status = d_status;
    a.chunks = any ? L.chunks : 0;
    a.beta = p->beta;
    a.margin = p->margin;
    a.smoothing = p->label_smoothing;
    a.loss_scale = p->loss_scale;
    a.kind = p->kind;
    a.normalize = p->normalize;
    const int64_t parts = any ? (t->num_rows + kBlock - 1) / kBlock : 0;
    if (any) {
        if (d_row_ids && num_ids > 0) {
            hipLaunchKernelGGL(fill_rows_kernel, dim3(grid_for(num_ids, kBlock, (int64_t)num_cus() * 8)), dim3(kBlock),
                               0, s, r.row_of, num_ids);
            ODB_LAUNCHED();
        }
        hipLaunchKernelGGL(loss_rows_kernel<true>, dim3(grid_for(L.chunks, 1)), dim3(kBlock), 0, s, r);
        ODB_LAUNCHED();
        if (parts > 0) {
            hipLaunchKernelGGL(pairs_kernel, dim3((unsigned)parts), dim3(kBlock), 0, s, a);
            ODB_LAUNCHED();
        }
    }
    hipLaunchKernelGGL(pairs_grad_kernel, dim3(a.grad ? grid_for(L.chunks, 1) : 1), dim3(kBlock), 0, s, a, parts);
    ODB_LAUNCHED();
    return ODB_OK;
}
