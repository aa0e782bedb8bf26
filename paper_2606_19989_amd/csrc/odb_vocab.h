// What the operators over a tile's logits share: 16 bytes of a row at a time, the running largest logit and
// sum of exponentials, and the checks of a tile's descriptor.
#pragma once

#include <cmath>

#include "odb_internal.h"

namespace odb {

namespace {

constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kFarBelow = -16384.0f;   // base-2 exponent whose power is 0, finite for products with 0

typedef __bf16 bf16_t;
typedef _Float16 fp16_t;

// 16 bytes of logits: N values.  Rows of an odd vocabulary start at any element; global memory serves
// 16-byte accesses at any address.  The forward call makes use of that, so that a row's sums run in the
// same order wherever it lies.  The gradient is written in the alignment of its own rows: up to N - 1
// elements one by one, then 16 bytes at a time (2,545 positions of 65,537 bf16 logits, replayed in a graph:
// 79 us, 120 us without).
typedef unsigned u4a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u4a4 __attribute__((ext_vector_type(4), aligned(4)));
template <int ALIGN>
struct Words {
    typedef u4a2 type;
};
template <>
struct Words<4> {
    typedef u4a4 type;
};

template <typename T>
struct alignas(sizeof(T)) Vec {
    static constexpr int N = 16 / sizeof(T);
    T v[N];
};

template <bool ONCE, typename T>
__device__ __forceinline__ Vec<T> load_vec(const T* p) {
    const auto* q = reinterpret_cast<const typename Words<sizeof(T)>::type*>(p);
    const auto w = ONCE ? __builtin_nontemporal_load(q) : *q;
    Vec<T> r;
    __builtin_memcpy(&r, &w, 16);
    return r;
}

template <typename T>
__device__ __forceinline__ void store_vec(T* p, const Vec<T>& r) {
    typename Words<sizeof(T)>::type w;
    __builtin_memcpy(&w, &r, 16);
    __builtin_nontemporal_store(w, reinterpret_cast<typename Words<sizeof(T)>::type*>(p));
}

// Elements before the first 16-byte boundary of a row, at most n.
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int64_t n) {
    const int h = (int)(-reinterpret_cast<uintptr_t>(p) & 15) / (int)sizeof(T);
    return h < n ? h : (int)n;
}

constexpr int kAhead = 4;    // 16-byte loads of a thread that are under way together

__device__ __forceinline__ int64_t at_most(int64_t v, int64_t most) { return v < most ? v : most; }

struct Acc {
    float m, s, t;
};

template <bool ENT>
__device__ __forceinline__ void acc_rescale(Acc& a, float m, float k) {
    float x = (a.m - m) * k;
    if (ENT) {
        x = fmaxf(x, kFarBelow);
        a.t += a.s * x;
    }
    const float c = __builtin_amdgcn_exp2f(x);
    a.s *= c;
    if (ENT) a.t *= c;
    a.m = m;
}

template <bool ENT>
__device__ __forceinline__ void acc_term(Acc& a, float z, float k) {
    float x = (z - a.m) * k;
    const float e = __builtin_amdgcn_exp2f(x);
    a.s += e;
    if (ENT) a.t += e * fmaxf(x, kFarBelow);
}

template <typename T, bool ENT>
__device__ __forceinline__ void acc_vec(Acc& a, const Vec<T>& v, float k) {
    constexpr int N = Vec<T>::N;
    float f[N];
    float m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        f[i] = (float)v.v[i];
        m = fmaxf(m, f[i]);
    }
    if (m > a.m) acc_rescale<ENT>(a, m, k);
#pragma unroll
    for (int i = 0; i < N; ++i) acc_term<ENT>(a, f[i], k);
}

template <bool ENT>
__device__ __forceinline__ Acc acc_join(Acc a, Acc b, float k) {
    const float m = fmaxf(a.m, b.m);
    acc_rescale<ENT>(a, m, k);
    acc_rescale<ENT>(b, m, k);
    a.s += b.s;
    a.t += b.t;
    return a;
}

// The triples of a group's G threads as one, on every thread.  s_acc: a word a wave of the block, free again
// when the call returns.
template <bool ENT, int G>
__device__ __forceinline__ Acc group_join(Acc r, Acc* s_acc, float k) {
#pragma unroll
    for (int d = (G < kWave ? G : kWave) / 2; d > 0; d >>= 1) {
        Acc o{__shfl_xor(r.m, d, kWave), __shfl_xor(r.s, d, kWave), ENT ? __shfl_xor(r.t, d, kWave) : 0.0f};
        r = acc_join<ENT>(r, o, k);
    }
    if (G > kWave) {
        if ((threadIdx.x & (kWave - 1)) == 0) s_acc[threadIdx.x / kWave] = r;
        __syncthreads();
        Acc all{s_acc[0].m, s_acc[0].s, s_acc[0].t};
#pragma unroll
        for (int j = 1; j < G / kWave; ++j) all = acc_join<ENT>(all, Acc{s_acc[j].m, s_acc[j].s, s_acc[j].t}, k);
        __syncthreads();
        return all;
    }
    return r;
}

// Meeting of the G threads of a group, with what they have written to LDS and to memory.
template <int G>
__device__ __forceinline__ void group_sync() {
    if (G > kWave) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    }
}

// Label of a token, or -1 if it is not scored.
__device__ __forceinline__ int32_t read_label(const int32_t* labels, int64_t at, int64_t vocab, int32_t* status,
                                              bool report) {
    const int32_t y = labels[at];
    if (y == ODB_LABEL_IGNORE) return -1;
    if (y < 0 || y >= vocab) {
        if (report && status) *status = kErrLabel;
        return -1;
    }
    return y;
}

inline int check_logits(const odb_logits_t* x) {
    if (!x) return set_error(ODB_E_INVALID_ARG, "logits is NULL");
    if (x->dtype != ODB_FLOAT32 && x->dtype != ODB_BFLOAT16 && x->dtype != ODB_FLOAT16)
        return set_error(ODB_E_INVALID_ARG, "unknown logits type %d", x->dtype);
    if (x->shift != 0 && x->shift != 1) return set_error(ODB_E_INVALID_ARG, "shift must be 0 or 1 (got %d)", x->shift);
    if (x->rows < 0 || x->cols < 0 || x->rows > INT32_MAX || x->cols > INT32_MAX ||
        (x->cols > 0 && x->rows > INT32_MAX / x->cols))
        return set_error(ODB_E_INVALID_ARG, "rows and cols must be >= 0 and rows * cols < 2^31");
    if (x->vocab < 1 || x->vocab > INT32_MAX) return set_error(ODB_E_INVALID_ARG, "vocab must be in [1, 2^31)");
    if (x->row_stride < 0 || x->col_stride < 0) return set_error(ODB_E_INVALID_ARG, "strides must be >= 0");
    const float a = (float)x->scale;
    if (!(a > 0.0f) || !std::isfinite(a) || !std::isfinite(a * kLog2e))
        return set_error(ODB_E_INVALID_ARG, "scale must be finite and > 0 in fp32");
    return ODB_OK;
}

// Bytes from the first element of the tile to behind its last, or -1 if they pass 2^62.
inline int64_t tile_span(const odb_logits_t* x, int64_t rs, int64_t cs) {
    const size_t elt = x->dtype == ODB_FLOAT32 ? 4 : 2;
    const __int128 last = (__int128)(x->rows - 1) * rs + (__int128)(x->cols - 1) * cs + x->vocab;
    return last * elt > ((__int128)1 << 62) ? -1 : (int64_t)(last * elt);
}

inline int check_tile(const odb_logits_t* x, const void* p, int64_t rs, int64_t cs, const char* what) {
    if (!p) return set_error(ODB_E_INVALID_ARG, "%s must not be NULL", what);
    if (reinterpret_cast<uintptr_t>(p) % (x->dtype == ODB_FLOAT32 ? 4 : 2))
        return set_error(ODB_E_INVALID_ARG, "%s is not aligned to its element", what);
    if (tile_span(x, rs, cs) < 0) return set_error(ODB_E_INVALID_ARG, "%s: the strides pass the address space", what);
    return ODB_OK;
}

// The gradient of a tile's logits: memory of its own whose elements lie apart, or the logits' with their strides.
inline int check_grad_tile(const odb_logits_t* x, const void* d_grad_logits, int64_t grad_row_stride,
                           int64_t grad_col_stride) {
    ODB_TRY(check_tile(x, d_grad_logits, grad_row_stride, grad_col_stride, "d_grad_logits"));
    // rows of the vocabulary that lie apart, in either order of rows and columns
    const __int128 rs = grad_row_stride, cs = grad_col_stride, V = x->vocab;
    const bool by_rows = (x->cols == 1 || cs >= V) && (x->rows == 1 || rs >= (x->cols - 1) * cs + V);
    const bool by_cols = (x->rows == 1 || rs >= V) && (x->cols == 1 || cs >= (x->rows - 1) * rs + V);
    if (!by_rows && !by_cols) return set_error(ODB_E_INVALID_ARG, "gradient strides let elements overlap");
    if (d_grad_logits == x->d_logits && ((x->rows > 1 && grad_row_stride != x->row_stride) ||
                                         (x->cols > 1 && grad_col_stride != x->col_stride)))
        return set_error(ODB_E_INVALID_ARG, "a gradient in place needs the strides of the logits");
    return ODB_OK;
}

}  // namespace

}  // namespace odb
