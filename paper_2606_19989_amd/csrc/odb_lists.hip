// Log-probabilities of a list of tokens at every position of a tile, and their gradient.
//
// Forward: the largest logit and the sum of exponentials of a position in one pass, then
// (z_id - m) a - logsum for each of its k listed tokens.
// Backward: with G = sum_j g_j, every logit has -a G p_v, written in one pass; the listed tokens'
// a (sum_{j: id_j = v} g_j - G p_v) are formed before it, from logits that it may overwrite, and written
// behind it, each in one place and rounded once.
//
// Bound by the reads of the logits and the writes of their gradient, as the label's log-probability: the list adds
// a few loads a position and, for ids that are listed twice, k^2 comparisons over all of a block's threads.
// 3,928 of 4,096 positions of 151,936 bf16 logits, k = 64: forward 184 us (6.5 TB/s of reads), backward 462 us
// (5.3 TB/s, half reads and half writes; a copy of 4 GiB reaches 4.7).
#include "odb_vocab.h"

namespace odb {

namespace {

// Whether a token counts; without labels every one that some logits score.
__device__ __forceinline__ bool token_counts(const int32_t* labels, int64_t at, int64_t vocab, int32_t* status,
                                             bool report) {
    return !labels || read_label(labels, at, vocab, status, report) >= 0;
}

// Id j of a list, or -1 if there is none.
__device__ __forceinline__ int32_t read_id(const int32_t* ids, int j, int64_t vocab, int32_t* status) {
    return read_label(ids, j, vocab, status, true);
}

struct ListArgs {
    odb_logits_t x;
    const int32_t* labels;
    const int32_t* ids;
    float* logprob;             // forward
    float* stats;
    const float* grad_list;     // backward
    const float* read_stats;
    void* grad;
    int64_t grad_rs, grad_cs;
    int32_t* status;
    int32_t k;
};

template <typename T, int G>
__global__ void __launch_bounds__(G > kBlock ? G : kBlock) list_logprobs_kernel(ListArgs A) {
    constexpr int kThreads = G > kBlock ? G : kBlock;
    constexpr int N = Vec<T>::N;
    __shared__ Acc s_acc[kThreads / kWave];
    const odb_logits_t& x = A.x;
    const int64_t n = x.rows * x.cols;
    const int t = threadIdx.x & (G - 1);
    const float a = (float)x.scale, k = a * kLog2e;
    const int64_t V = x.vocab;
    for (int64_t q = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G; q < n;
         q += (int64_t)gridDim.x * (kThreads / G)) {   // uniform over a group
        const uint32_t i = (uint32_t)q / (uint32_t)x.cols, c = (uint32_t)q - i * (uint32_t)x.cols;
        const int32_t* ids = A.ids + q * A.k;
        float* out = A.logprob + q * A.k;
        if (c < (uint32_t)x.shift || !token_counts(A.labels, q, V, A.status, t == 0)) {
            for (int j = t; j < A.k; j += G) out[j] = 0.0f;
            if (t == 0 && A.stats) reinterpret_cast<float2*>(A.stats)[q] = make_float2(0.0f, 0.0f);
            continue;
        }
        const T* z = static_cast<const T*>(x.d_logits) + (int64_t)i * x.row_stride +
                     (int64_t)(c - (uint32_t)x.shift) * x.col_stride;
        // a thread's first entry is under way beside the row
        const int32_t id0 = t < A.k ? read_id(ids, t, V, A.status) : -1;
        const float z0 = id0 >= 0 ? (float)z[id0] : 0.0f;
        Acc r{kLowest, 0.0f, 0.0f};
        const int64_t whole = V / N * N;
        for (int64_t v = (int64_t)t * N; v < whole; v += kAhead * G * N) {
            Vec<T> w[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) w[j] = load_vec<true>(z + at_most(v + j * G * N, whole - N));
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (v + j * G * N < whole) acc_vec<T, false>(r, w[j], k);
        }
        if (whole + t < V) {
            const float f = (float)z[whole + t];
            if (f > r.m) acc_rescale<false>(r, f, k);
            acc_term<false>(r, f, k);
        }
        r = group_join<false, G>(r, s_acc, k);
        const float lse = logf(r.s);
        for (int j = t; j < A.k; j += G) {
            const int32_t id = j == t ? id0 : read_id(ids, j, V, A.status);
            const float f = j == t ? z0 : id >= 0 ? (float)z[id] : 0.0f;
            out[j] = id >= 0 ? (f - r.m) * a - lse : 0.0f;
        }
        if (t == 0 && A.stats) reinterpret_cast<float2*>(A.stats)[q] = make_float2(r.m, lse);
    }
}

// A position's list, in LDS.
struct List {
    int32_t* id;     // -1: none
    float* g;        // its gradient
    float* z;        // its logit, then the gradient of that logit
    int32_t* put;    // where that goes: its id, or -1 if an entry before it has the same
    int32_t* order;  // for few columns: the entries whose id is listed more than once, in their order
    uint32_t* seen;  // and a bit a column: listed
    uint32_t* again; // listed more than once
};

// Columns up to which a group of at most a wave looks for ids that are listed twice by a bit each.
constexpr int kSeen = 4096;

size_t list_bytes(int32_t k, int64_t vocab, int group) {
    return group <= kWave && vocab <= kSeen ? 20 * (size_t)k + ((size_t)vocab + 31) / 32 * 8 : 16 * (size_t)k;
}

// The lanes of a group, of a wave at most, that say so; of a larger one the wave's.
template <int G>
__device__ __forceinline__ uint64_t group_ballot(bool on) {
    const uint64_t all = __ballot(on);
    if (G >= kWave) return all;
    return all >> ((threadIdx.x & (kWave - 1)) & ~(G - 1)) & ((1ull << (G & (kWave - 1))) - 1);
}

// G is 8 at least, as in the forward call.
template <typename T, int G>
__global__ void __launch_bounds__(G > kBlock ? G : kBlock) list_logprobs_backward_kernel(ListArgs A, int bytes) {
    constexpr int kThreads = G > kBlock ? G : kBlock;
    constexpr int N = Vec<T>::N;
    extern __shared__ __align__(16) char s_lists[];
    const odb_logits_t& x = A.x;
    char* const room = s_lists + threadIdx.x / G * bytes;
    const List s{reinterpret_cast<int32_t*>(room), reinterpret_cast<float*>(room + 4 * A.k),
                 reinterpret_cast<float*>(room + 8 * A.k), reinterpret_cast<int32_t*>(room + 12 * A.k),
                 reinterpret_cast<int32_t*>(room + 16 * A.k), reinterpret_cast<uint32_t*>(room + 20 * A.k),
                 reinterpret_cast<uint32_t*>(room + 20 * A.k) + (x.vocab + 31) / 32};
    const int64_t n = x.rows * x.cols;
    const int t = threadIdx.x & (G - 1);
    const float a = (float)x.scale, k = a * kLog2e;
    const int64_t V = x.vocab;
    for (int64_t q = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G; q < n;
         q += (int64_t)gridDim.x * (kThreads / G)) {   // uniform over a group
        const uint32_t i = (uint32_t)q / (uint32_t)x.cols, c = (uint32_t)q - i * (uint32_t)x.cols;
        const int64_t at = q + x.shift;   // the token these logits score
        const bool counts = c + x.shift < x.cols && token_counts(A.labels, at, V, A.status, t == 0);
        const T* z = static_cast<const T*>(x.d_logits) + (int64_t)i * x.row_stride + (int64_t)c * x.col_stride;
        T* d = static_cast<T*>(A.grad) + (int64_t)i * A.grad_rs + (int64_t)c * A.grad_cs;
        const int head = head_of(d, V);    // the stores' alignment
        const int64_t whole = (V - head) / N * N;
        T* db = d + head;
        float sum = 0.0f;
        bool any = false;
        const bool bits = G <= kWave && V <= kSeen;
        int shared = bits ? 0 : A.k;      // entries that may share their id with another
        if (counts) {
            if (bits)
                for (int j = t; j < (int)((V + 31) / 32); j += G) s.seen[j] = s.again[j] = 0;
            for (int j = t; j < A.k; j += G) {
                const int32_t id = read_id(A.ids + at * A.k, j, V, A.status);
                s.id[j] = id;
                s.g[j] = id >= 0 ? A.grad_list[at * A.k + j] : 0.0f;
                s.z[j] = id >= 0 ? (float)z[id] : 0.0f;
                s.put[j] = id;
            }
            group_sync<G>();
            constexpr int kLanes = G < kWave ? G : kWave;
            for (int j = t & (kLanes - 1); j < A.k; j += kLanes) sum += s.g[j];
            bool more = false;
            for (int j = t & (kLanes - 1); j < A.k; j += kLanes) more |= s.g[j] != 0.0f;
            any = group_ballot<G>(more) != 0;
#pragma unroll
            for (int l = 1; l < kLanes; l <<= 1) sum += __shfl_xor(sum, l, kWave);
            if (bits) {
                for (int j = t; j < A.k; j += G) {
                    const int32_t id = s.id[j];
                    const uint32_t bit = 1u << (id & 31);
                    if (id >= 0 && (atomicOr(&s.seen[id >> 5], bit) & bit)) atomicOr(&s.again[id >> 5], bit);
                }
                group_sync<G>();
                for (int j = t; j < ((A.k + G - 1) & ~(G - 1)); j += G) {
                    const int32_t id = j < A.k ? s.id[j] : -1;
                    const bool on = id >= 0 && (s.again[id >> 5] >> (id & 31) & 1);
                    const uint64_t all = group_ballot<G>(on);
                    if (on) s.order[shared + __builtin_popcountll(all & ((1ull << t) - 1))] = j;
                    shared += __builtin_popcountll(all);
                }
                group_sync<G>();
            }
        }
        if (!any) {
            Vec<T> zero;
#pragma unroll
            for (int j = 0; j < N; ++j) zero.v[j] = (T)0.0f;
            if (t < head) d[t] = (T)0.0f;
            for (int64_t v = (int64_t)t * N; v < whole; v += G * N) store_vec(db + v, zero);
            if (head + whole + t < V) db[whole + t] = (T)0.0f;
            group_sync<G>();
            continue;
        }
        const float2 st = reinterpret_cast<const float2*>(A.read_stats)[at];
        const float m = st.x, inv = expf(-st.y), all = a * sum;
        auto prob = [&](float f) { return __builtin_amdgcn_exp2f((f - m) * k) * inv; };
        if (bits)
            for (int j = t; j < A.k; j += G) {
                const int32_t id = s.id[j];
                if (id >= 0 && !(s.again[id >> 5] >> (id & 31) & 1)) s.z[j] = a * fmaf(-prob(s.z[j]), sum, s.g[j]);
            }
        // Entries that share an id: its gradient is that of all of them, and the first has it written.  2^by threads
        // an entry, each with every 2^by-th of the others.
        int by = 0;
        while (by < 6 && (shared << (by + 1)) <= G && shared > 0) ++by;
        for (int i0 = t >> by; i0 < shared; i0 += G >> by) {
            const int j = bits ? s.order[i0] : i0;
            const int32_t id = s.id[j];
            float g = 0.0f;
            bool first = id >= 0;
            for (int o0 = t & ((1 << by) - 1); o0 < shared; o0 += 1 << by) {
                const int o = bits ? s.order[o0] : o0;
                if (s.id[o] == id) {
                    g += s.g[o];
                    first &= o >= j;
                }
            }
            for (int l = 0; l < by; ++l) {
                g += __shfl_xor(g, 1 << l, kWave);
                first &= (bool)__shfl_xor((int)first, 1 << l, kWave);
            }
            if ((t & ((1 << by) - 1)) == 0) {
                s.z[j] = a * fmaf(-prob(s.z[j]), sum, g);
                s.put[j] = first ? id : -1;
            }
        }
        if (t < head) d[t] = (T)(-prob((float)z[t]) * all);
        const T* zb = z + head;
        for (int64_t v = (int64_t)t * N; v < whole; v += kAhead * G * N) {
            Vec<T> w[kAhead];
            // in place: those past the row's end read what this thread has yet to write or another has written,
            // and drop it
#pragma unroll
            for (int j = 0; j < kAhead; ++j) w[j] = load_vec<false>(zb + at_most(v + j * G * N, whole - N));
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (v + j * G * N >= whole) break;
#pragma unroll
                for (int e = 0; e < N; ++e) w[j].v[e] = (T)(-prob((float)w[j].v[e]) * all);
                store_vec(db + v + j * G * N, w[j]);
            }
        }
        if (head + whole + t < V) db[whole + t] = (T)(-prob((float)zb[whole + t]) * all);
        group_sync<G>();    // behind the stores of the row, and every read of the list
        for (int j = t; j < A.k; j += G)
            if (s.put[j] >= 0) d[s.put[j]] = (T)s.z[j];
    }
}

// Threads of a position, as for the labels' log-probabilities; short rows with long lists take a wave, so that a
// thread has few entries.  us for 131,072 positions of 500 bf16 logits, k = 8 / 64 / 128, with 8 threads and with
// 64: forward 37 / 126 / 232 and 51 / 64 / 76, backward 81 / 330 / 1,370 and 90 / 132 / 272.
enum Group { kGroup8, kGroup32, kGroup64, kGroup256, kGroup512, kGroup1024 };

Group group_for(const odb_logits_t* x, int32_t k, bool backward) {
    const int64_t row = x->vocab * (x->dtype == ODB_FLOAT32 ? 4 : 2);
    if (x->rows * x->cols <= 2 * (int64_t)num_cus())
        return row <= 1024    ? kGroup64
               : row <= 32768 ? kGroup256
               : row <= (backward ? 49152 : 131072) ? kGroup512
                                                    : kGroup1024;
    if (row <= 1024 && k <= 16) return kGroup8;
    if (row <= 2048 && k <= 32) return kGroup32;
    if (!backward) return row <= 16384 ? kGroup64 : row <= 98304 ? kGroup256 : kGroup512;
    return row <= 8192 ? kGroup64 : row <= 24576 ? kGroup256 : row <= 49152 ? kGroup512 : kGroup1024;
}

template <typename T, int G>
void launch(const ListArgs& a, bool backward, hipStream_t s) {
    constexpr int kThreads = G > kBlock ? G : kBlock;
    const dim3 grid(grid_for(a.x.rows * a.x.cols, kThreads / G)), block(kThreads);
    if (backward) {
        const size_t bytes = list_bytes(a.k, a.x.vocab, G);
        hipLaunchKernelGGL((list_logprobs_backward_kernel<T, G>), grid, block, bytes * (kThreads / G), s, a, (int)bytes);
    } else
        hipLaunchKernelGGL((list_logprobs_kernel<T, G>), grid, block, 0, s, a);
}

template <typename T>
void launch(const ListArgs& a, bool backward, hipStream_t s) {
    switch (group_for(&a.x, a.k, backward)) {
        case kGroup8: return launch<T, 8>(a, backward, s);
        case kGroup32: return launch<T, 32>(a, backward, s);
        case kGroup64: return launch<T, 64>(a, backward, s);
        case kGroup256: return launch<T, 256>(a, backward, s);
        case kGroup512: return launch<T, 512>(a, backward, s);
        default: return launch<T, 1024>(a, backward, s);
    }
}

int run(const ListArgs& a, bool backward, hipStream_t s) {
    if (a.x.dtype == ODB_FLOAT32)
        launch<float>(a, backward, s);
    else if (a.x.dtype == ODB_BFLOAT16)
        launch<bf16_t>(a, backward, s);
    else
        launch<fp16_t>(a, backward, s);
    ODB_LAUNCHED();
    return ODB_OK;
}

int check_list(const odb_logits_t* x, int32_t k) {
    ODB_TRY(check_logits(x));
    if (k < 1 || k > ODB_LIST_MAX) return set_error(ODB_E_INVALID_ARG, "k must be in [1, %d] (got %d)", ODB_LIST_MAX, k);
    return ODB_OK;
}

}  // namespace

}  // namespace odb

using namespace odb;

extern "C" int odb_token_list_logprobs(const odb_logits_t* x, const int32_t* d_labels, int32_t k, const int32_t* d_ids,
                                       float* d_list_logprob, float* d_stats, int32_t* d_status, void* stream) {
    ODB_TRY(check_list(x, k));
    if (x->rows == 0 || x->cols == 0) return ODB_OK;
    ODB_TRY(check_tile(x, x->d_logits, x->row_stride, x->col_stride, "d_logits"));
    if (!d_ids || !d_list_logprob) return set_error(ODB_E_INVALID_ARG, "d_ids and d_list_logprob must not be NULL");
    if (reinterpret_cast<uintptr_t>(d_stats) & 7)
        return set_error(ODB_E_INVALID_ARG, "d_stats must be 8-byte aligned");
    ListArgs a{};
    a.x = *x;
    a.labels = d_labels;
    a.ids = d_ids;
    a.logprob = d_list_logprob;
    a.stats = d_stats;
    a.status = d_status;
    a.k = k;
    return run(a, false, static_cast<hipStream_t>(stream));
}

extern "C" int odb_token_list_logprobs_backward(const odb_logits_t* x, const int32_t* d_labels, int32_t k,
                                                const int32_t* d_ids, const float* d_stats, const float* d_grad_list,
                                                void* d_grad_logits, int64_t grad_row_stride, int64_t grad_col_stride,
                                                int32_t* d_status, void* stream) {
    ODB_TRY(check_list(x, k));
    if (grad_row_stride < 0 || grad_col_stride < 0)
        return set_error(ODB_E_INVALID_ARG, "gradient strides must be >= 0");
    if (x->rows == 0 || x->cols == 0) return ODB_OK;
    ODB_TRY(check_tile(x, x->d_logits, x->row_stride, x->col_stride, "d_logits"));
    ODB_TRY(check_grad_tile(x, d_grad_logits, grad_row_stride, grad_col_stride));
    if (!d_ids || !d_stats || !d_grad_list)
        return set_error(ODB_E_INVALID_ARG, "d_ids, d_stats and d_grad_list must not be NULL");
    if (reinterpret_cast<uintptr_t>(d_stats) & 7)
        return set_error(ODB_E_INVALID_ARG, "d_stats must be 8-byte aligned");
    ListArgs a{};
    a.x = *x;
    a.labels = d_labels;
    a.ids = d_ids;
    a.read_stats = d_stats;
    a.grad_list = d_grad_list;
    a.grad = d_grad_logits;
    a.grad_rs = grad_row_stride;
    a.grad_cs = grad_col_stride;
    a.status = d_status;
    a.k = k;
    return run(a, true, static_cast<hipStream_t>(stream));
}
