// Log-probabilities of a tile's labels from its logits, and their gradient.
//
// Forward: one pass over a position's V logits.  Every thread keeps the largest logit m it has
// met, s = sum exp(a (z - m)) and, for the entropy, t = sum e x with x = a (z - m) in base 2; a
// new largest logit rescales the two sums.  The threads' triples join in a tree:
// (m1, s1) + (m2, s2) = (M, s1 exp(a (m1 - M)) + s2 exp(a (m2 - M))), M = max(m1, m2).
// x is formed as (z - m) k, k = a log2 e: the difference first, so that rows whose logits are all
// the type's lowest value stay finite.
// Backward: p = exp(a (z - m)) exp(-logsum) needs no second pass, the forward call left both.
//
// Bound by the reads of the logits (and the writes of the gradient): 2 or 4 bytes against about
// ten instructions a logit, of which the exponential is a quarter-rate one.  Measured: 7,832 scored positions
// of 151,936 bf16 logits forward in 350 to 375 us (6.4 to 6.8 TB/s of reads), 3,928 of 4,096 backward in
// 440 to 450 us (5.5 TB/s, half reads and half writes; a copy reaches 5.0 to 5.2).  One position of 32,000:
// 5.3 us, the label's load, one round of the logits' and the reduction one after the other.
#include "odb_vocab.h"

namespace odb {

namespace {

// A group of G threads (a divisor of a wave or whole waves) takes a position; blocks of max(G, 256)
// threads.  G is 8 at least, so that a thread has at most one of the elements outside the 16-byte groups.
template <typename T, bool ENT, int G>
__global__ void __launch_bounds__(G > kBlock ? G : kBlock) token_logprobs_kernel(odb_logits_t x,
                                                                                const int32_t* __restrict__ labels,
                                                                                float* __restrict__ logprob,
                                                                                float* __restrict__ stats,
                                                                                float* __restrict__ entropy,
                                                                                int32_t* status) {
    constexpr int kThreads = G > kBlock ? G : kBlock;
    constexpr int N = Vec<T>::N;
    __shared__ Acc s_acc[kThreads / kWave];
    const int64_t n = x.rows * x.cols;
    const int t = threadIdx.x & (G - 1);
    const float a = (float)x.scale, k = a * kLog2e;
    const int64_t V = x.vocab;
    for (int64_t q = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G; q < n;
         q += (int64_t)gridDim.x * (kThreads / G)) {   // uniform over a group
        const uint32_t i = (uint32_t)q / (uint32_t)x.cols, c = (uint32_t)q - i * (uint32_t)x.cols;
        const int32_t y = c >= (uint32_t)x.shift ? read_label(labels, q, V, status, t == 0) : -1;
        if (y < 0) {
            if (t == 0) {
                logprob[q] = 0.0f;
                if (stats) reinterpret_cast<float2*>(stats)[q] = make_float2(0.0f, 0.0f);
                if (ENT) entropy[q] = 0.0f;
            }
            continue;
        }
        const T* z = static_cast<const T*>(x.d_logits) + (int64_t)i * x.row_stride +
                     (int64_t)(c - (uint32_t)x.shift) * x.col_stride;
        const float zy = (float)z[y];
        Acc r{kLowest, 0.0f, 0.0f};
        auto one = [&](float f) {
            if (f > r.m) acc_rescale<ENT>(r, f, k);
            acc_term<ENT>(r, f, k);
        };
        const int64_t whole = V / N * N;
        for (int64_t v = (int64_t)t * N; v < whole; v += kAhead * G * N) {
            Vec<T> w[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) w[j] = load_vec<true>(z + at_most(v + j * G * N, whole - N));
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (v + j * G * N < whole) acc_vec<T, ENT>(r, w[j], k);
        }
        if (whole + t < V) one((float)z[whole + t]);
#pragma unroll
        for (int d = (G < kWave ? G : kWave) / 2; d > 0; d >>= 1) {
            Acc o{__shfl_xor(r.m, d, kWave), __shfl_xor(r.s, d, kWave), ENT ? __shfl_xor(r.t, d, kWave) : 0.0f};
            r = acc_join<ENT>(r, o, k);
        }
        if (G > kWave) {
            const int w = threadIdx.x / kWave;
            if ((threadIdx.x & (kWave - 1)) == 0) s_acc[w] = r;
            __syncthreads();
            r = s_acc[0];
#pragma unroll
            for (int j = 1; j < kThreads / kWave; ++j) r = acc_join<ENT>(r, s_acc[j], k);
            __syncthreads();
        }
        if (t == 0) {
            const float lse = logf(r.s);
            logprob[q] = (zy - r.m) * a - lse;
            if (stats) reinterpret_cast<float2*>(stats)[q] = make_float2(r.m, lse);
            if (ENT) entropy[q] = lse - r.t / r.s * kLn2;
        }
    }
}

template <typename T, bool ENT, int G>
__global__ void __launch_bounds__(G > kBlock ? G : kBlock) token_logprobs_backward_kernel(
    odb_logits_t x, const int32_t* __restrict__ labels, const float* __restrict__ stats,
    const float* __restrict__ grad_logprob, const float* __restrict__ entropy, const float* __restrict__ grad_entropy,
    T* grad, int64_t grs, int64_t gcs, int32_t* status) {
    constexpr int kThreads = G > kBlock ? G : kBlock;
    constexpr int N = Vec<T>::N;
    const int64_t n = x.rows * x.cols;
    const int t = threadIdx.x & (G - 1);
    const float a = (float)x.scale, k = a * kLog2e;
    const int64_t V = x.vocab;
    for (int64_t q = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G; q < n;
         q += (int64_t)gridDim.x * (kThreads / G)) {
        const uint32_t i = (uint32_t)q / (uint32_t)x.cols, c = (uint32_t)q - i * (uint32_t)x.cols;
        const int64_t at = q + x.shift;   // the token these logits score
        const int32_t y = c + x.shift < x.cols ? read_label(labels, at, V, status, t == 0) : -1;
        float g = 0.0f, h = 0.0f;
        if (y >= 0) {
            g = grad_logprob[at];
            if (ENT) h = grad_entropy[at];
        }
        T* d = grad + (int64_t)i * grs + (int64_t)c * gcs;
        const int head = head_of(d, V);    // the stores' alignment: half a line written costs more than read
        const int64_t whole = (V - head) / N * N;
        T* db = d + head;
        if (y < 0 || (g == 0.0f && h == 0.0f)) {
            Vec<T> zero;
#pragma unroll
            for (int j = 0; j < N; ++j) zero.v[j] = (T)0.0f;
            if (t < head) d[t] = (T)0.0f;
            for (int64_t v = (int64_t)t * N; v < whole; v += G * N) store_vec(db + v, zero);
            if (head + whole + t < V) db[whole + t] = (T)0.0f;
            continue;
        }
        const T* z = static_cast<const T*>(x.d_logits) + (int64_t)i * x.row_stride + (int64_t)c * x.col_stride;
        const float2 st = reinterpret_cast<const float2*>(stats)[at];
        const float m = st.x, inv = expf(-st.y), ag = a * g;
        // a (g + h (ln p + H)) = c0 + c1 x,  x = log2 exp(a (z - m))
        const float c0 = ENT ? ag + a * h * (entropy[at] - st.y) : ag, c1 = ENT ? a * h * kLn2 : 0.0f;
        auto one = [&](float f) {
            const float u = (f - m) * k;
            const float p = __builtin_amdgcn_exp2f(u) * inv;
            return ENT ? -p * (c0 + c1 * fmaxf(u, kFarBelow)) : -p * c0;
        };
        auto store_one = [&](int64_t v) {
            float o = one((float)z[v]);
            if (v == y) o += ag;
            d[v] = (T)o;
        };
        if (t < head) store_one(t);
        const T* zb = z + head;
        const int64_t yb = y - head;
        auto store_group = [&](const Vec<T>& w, int64_t v) {
            float o[N];
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = one((float)w.v[e]);
            if ((uint64_t)(yb - v) < (uint64_t)N) {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (v + e == yb) o[e] += ag;
            }
            Vec<T> r;
#pragma unroll
            for (int e = 0; e < N; ++e) r.v[e] = (T)o[e];
            store_vec(db + v, r);
        };
        for (int64_t v = (int64_t)t * N; v < whole; v += kAhead * G * N) {
            Vec<T> w[kAhead];
            // in place: those past the row's end read what this thread has yet to write or another has written,
            // and drop it
#pragma unroll
            for (int j = 0; j < kAhead; ++j) w[j] = load_vec<false>(zb + at_most(v + j * G * N, whole - N));
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (v + j * G * N < whole) store_group(w[j], v + j * G * N);
        }
        if (head + whole + t < V) store_one(head + whole + t);
    }
}

// Threads of a position, by the bytes of its logits.  Too many leave the reduction and the label's load
// in front of too little work, too few leave loads unissued.  us for about 600 MB of logits (N positions
// of V; 2 x 600 MB for the gradient), and in a graph for 32 positions:
//   bytes of a row     forward 64 / 256 / 512 / 1,024 threads    backward 64 / 256 / 512 / 1,024
//   4 KB               109 / 246 / 463 / 1320                    198 / 325 / 567 / 1049
//   16 KB               95 / 122 / 189 /  412                    222 / 201 / 245 / 403
//   32 KB               98 /  96 / 123 /  267                    219 / 212 / 195 / 284
//   64 KB              103 /  98 / 110 /  207                    250 / 229 / 207 / 203
//   128 KB             120 / 101 /  97 /  147                    283 / 263 / 249 / 215
//   1 KB x 32          3.0 / 3.3 / 3.4 /  4.1                    3.0 / 3.0 / 2.9 / 2.9
//   4 KB x 32          3.4 / 3.4 / 3.5 /  4.1                    3.4 / 3.0 / 2.9 / 2.9
//   16 KB x 32         5.7 / 3.8 / 3.9 /  4.7                    5.7 / 3.6 / 3.3 / 3.7
//   32 KB x 32         9.1 / 4.6 / 4.3 /  5.0                    9.0 / 4.4 / 3.8 / 3.9
//   48 KB x 32        12.2 / 5.3 / 5.1 /  5.4                   12.0 / 5.1 / 4.7 / 4.3
//   64 KB x 32        15.7 / 6.1 / 5.4 /  5.9                   15.2 / 6.1 / 5.0 / 4.7
//   128 KB x 32       26.9 / 9.2 / 7.6 /  7.7                   27.8 / 9.2 / 7.5 / 6.9
//   304 KB x 32         81 /  23 /  17 /   15                     61 /  18 /  14 /  12
//   304 KB x 1          56 /  17 /  13 /   12                     55 /  17 /  13 /  12
// One position's are within 0.6 us of 32's up to 128 KB; 512 positions of up to 8 KB take up to 1.5 us more with
// 1,024 threads, with fewer 0.5.
// Rows of 128 bytes, 4.7 M: 1,682 with a wave a row, 245 with 8 threads; of 512 bytes 461 and 106; of
// 1 KB 240 and 99; of 2 KB 160, and 110 with 32.
enum Group { kGroup8, kGroup32, kGroup64, kGroup256, kGroup512, kGroup1024 };

Group group_for(const odb_logits_t* x, bool backward) {
    const int64_t row = x->vocab * (x->dtype == ODB_FLOAT32 ? 4 : 2);
    if (x->rows * x->cols <= 2 * (int64_t)num_cus())
        return row <= 1024    ? kGroup64
               : row <= 32768 ? kGroup256
               : row <= (backward ? 49152 : 131072) ? kGroup512
                                                    : kGroup1024;
    if (row <= 1024) return kGroup8;
    if (row <= 2048) return kGroup32;
    if (!backward) return row <= 16384 ? kGroup64 : row <= 98304 ? kGroup256 : kGroup512;
    return row <= 8192 ? kGroup64 : row <= 24576 ? kGroup256 : row <= 49152 ? kGroup512 : kGroup1024;
}

template <typename T, int G>
void launch_forward(const odb_logits_t* x, const int32_t* labels, float* logprob, float* stats, float* entropy,
                    int32_t* status, hipStream_t s) {
    constexpr int kThreads = G > kBlock ? G : kBlock;
    hipLaunchKernelGGL((entropy ? token_logprobs_kernel<T, true, G> : token_logprobs_kernel<T, false, G>),
                       dim3(grid_for(x->rows * x->cols, kThreads / G)), dim3(kThreads), 0, s, *x, labels, logprob, stats,
                       entropy, status);
}

template <typename T>
void forward(const odb_logits_t* x, const int32_t* labels, float* logprob, float* stats, float* entropy,
             int32_t* status, hipStream_t s) {
    switch (group_for(x, false)) {
        case kGroup8: return launch_forward<T, 8>(x, labels, logprob, stats, entropy, status, s);
        case kGroup32: return launch_forward<T, 32>(x, labels, logprob, stats, entropy, status, s);
        case kGroup64: return launch_forward<T, 64>(x, labels, logprob, stats, entropy, status, s);
        case kGroup256: return launch_forward<T, 256>(x, labels, logprob, stats, entropy, status, s);
        case kGroup512: return launch_forward<T, 512>(x, labels, logprob, stats, entropy, status, s);
        default: return launch_forward<T, 1024>(x, labels, logprob, stats, entropy, status, s);
    }
}

struct BackwardArgs {
    const int32_t* labels;
    const float* stats;
    const float* grad_logprob;
    const float* entropy;
    const float* grad_entropy;
    void* grad;
    int64_t row_stride, col_stride;
    int32_t* status;
};

template <typename T, int G>
void launch_backward(const odb_logits_t* x, const BackwardArgs& a, hipStream_t s) {
    constexpr int kThreads = G > kBlock ? G : kBlock;
    hipLaunchKernelGGL((a.entropy ? token_logprobs_backward_kernel<T, true, G>
                                  : token_logprobs_backward_kernel<T, false, G>),
                       dim3(grid_for(x->rows * x->cols, kThreads / G)), dim3(kThreads), 0, s, *x, a.labels, a.stats,
                       a.grad_logprob, a.entropy, a.grad_entropy, static_cast<T*>(a.grad), a.row_stride, a.col_stride,
                       a.status);
}

template <typename T>
void backward(const odb_logits_t* x, const BackwardArgs& a, hipStream_t s) {
    switch (group_for(x, true)) {
        case kGroup8: return launch_backward<T, 8>(x, a, s);
        case kGroup32: return launch_backward<T, 32>(x, a, s);
        case kGroup64: return launch_backward<T, 64>(x, a, s);
        case kGroup256: return launch_backward<T, 256>(x, a, s);
        case kGroup512: return launch_backward<T, 512>(x, a, s);
        default: return launch_backward<T, 1024>(x, a, s);
    }
}

}  // namespace

}  // namespace odb

using namespace odb;

extern "C" int odb_token_logprobs(const odb_logits_t* x, const int32_t* d_labels, float* d_logprob, float* d_stats,
                                  float* d_entropy, int32_t* d_status, void* stream) {
    ODB_TRY(check_logits(x));
    if (x->rows == 0 || x->cols == 0) return ODB_OK;
    ODB_TRY(check_tile(x, x->d_logits, x->row_stride, x->col_stride, "d_logits"));
    if (!d_labels || !d_logprob) return set_error(ODB_E_INVALID_ARG, "d_labels and d_logprob must not be NULL");
    if (reinterpret_cast<uintptr_t>(d_stats) & 7)
        return set_error(ODB_E_INVALID_ARG, "d_stats must be 8-byte aligned");
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (x->dtype == ODB_FLOAT32)
        forward<float>(x, d_labels, d_logprob, d_stats, d_entropy, d_status, s);
    else if (x->dtype == ODB_BFLOAT16)
        forward<bf16_t>(x, d_labels, d_logprob, d_stats, d_entropy, d_status, s);
    else
        forward<fp16_t>(x, d_labels, d_logprob, d_stats, d_entropy, d_status, s);
    ODB_LAUNCHED();
    return ODB_OK;
}

extern "C" int odb_token_logprobs_backward(const odb_logits_t* x, const int32_t* d_labels, const float* d_stats,
                                           const float* d_grad_logprob, const float* d_entropy,
                                           const float* d_grad_entropy, void* d_grad_logits, int64_t grad_row_stride,
                                           int64_t grad_col_stride, int32_t* d_status, void* stream) {
    ODB_TRY(check_logits(x));
    if (grad_row_stride < 0 || grad_col_stride < 0)
        return set_error(ODB_E_INVALID_ARG, "gradient strides must be >= 0");
    if (x->rows == 0 || x->cols == 0) return ODB_OK;
    ODB_TRY(check_tile(x, x->d_logits, x->row_stride, x->col_stride, "d_logits"));
    ODB_TRY(check_grad_tile(x, d_grad_logits, grad_row_stride, grad_col_stride));
    if (!d_labels || !d_stats || !d_grad_logprob)
        return set_error(ODB_E_INVALID_ARG, "d_labels, d_stats and d_grad_logprob must not be NULL");
    if (reinterpret_cast<uintptr_t>(d_stats) & 7)
        return set_error(ODB_E_INVALID_ARG, "d_stats must be 8-byte aligned");
    if (!d_entropy != !d_grad_entropy)
        return set_error(ODB_E_INVALID_ARG, "d_entropy and d_grad_entropy come together or not at all");
    hipStream_t s = static_cast<hipStream_t>(stream);
    const BackwardArgs a{d_labels, d_stats, d_grad_logprob, d_entropy, d_grad_entropy, d_grad_logits,
                         grad_row_stride, grad_col_stride, d_status};
    if (x->dtype == ODB_FLOAT32)
        backward<float>(x, a, s);
    else if (x->dtype == ODB_BFLOAT16)
        backward<bf16_t>(x, a, s);
    else
        backward<fp16_t>(x, a, s);
    ODB_LAUNCHED();
    return ODB_OK;
}
