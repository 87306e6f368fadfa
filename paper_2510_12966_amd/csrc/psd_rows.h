// What the operators on rows of logits share: rows of either type, read and written 16 bytes at a time, and their checks.
#pragma once
#include "psd_device.h"
#include "psd_host.h"

// Every fused multiply-add behind this line is written out: kernels that form the same sum in different surroundings round alike.
#pragma clang fp contract(off)

namespace psd {

constexpr int kMaxRows = 65535;       // rows of a call, as in psd_sample and psd_row_stats
constexpr int kMaxVocab = 1 << 27;    // keeps every index of a row, rounded up to whole chunks, inside 32 bits

// Sums of exponentials are kept with the largest logit of their range, sum 2^((z - max) c2): the difference first, so that rows whose
// every entry is the type's lowest value still have a distribution.  A range without an entry above -inf has the lowest finite maximum
// (differences with it are no NaN) and sum 0.
constexpr float kNoEntry = -3.402823466e38f;
__device__ inline float2 join_sums(float2 a, float2 b, float c2) {
    const float m = fmaxf(a.x, b.x);
    return make_float2(m, fmaf(a.y, fast_exp2((a.x - m) * c2), b.y * fast_exp2((b.x - m) * c2)));
}

// Rows start wherever their stride puts them, so 16 bytes are asked for at the alignment of one element; the hardware takes that,
// and a line that two lanes share is read once by either.
typedef uint32_t raw16 __attribute__((ext_vector_type(4)));
typedef uint32_t raw16_of_f32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t raw16_of_bf16 __attribute__((ext_vector_type(4), aligned(2)));

template <bool BF16>
struct Row;   // N: elements of 16 bytes
template <>
struct Row<false> {
    typedef float T;
    typedef raw16_of_f32 V;
    static constexpr int N = 4;
    static __device__ inline float get(const raw16& r, int i) { return __uint_as_float(r[i]); }
    static __device__ inline float one(const T* p) { return *p; }
    static __device__ inline void put_one(T* p, float v) { *p = v; }
    static __device__ inline raw16 pack(const float* v) { return raw16{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])}; }
};
template <>
struct Row<true> {
    typedef uint16_t T;
    typedef raw16_of_bf16 V;
    static constexpr int N = 8;
    static __device__ inline float get(const raw16& r, int i) { return __uint_as_float((i & 1) ? (r[i >> 1] & 0xffff0000u) : (r[i >> 1] << 16)); }
    static __device__ inline float one(const T* p) { return bf16_to_f32(*p); }
    static __device__ inline void put_one(T* p, float v) { *p = f32_to_bf16(v); }
    static __device__ inline raw16 pack(const float* v) {
        return raw16{f32x2_to_bf16(v[0], v[1]), f32x2_to_bf16(v[2], v[3]), f32x2_to_bf16(v[4], v[5]), f32x2_to_bf16(v[6], v[7])};
    }
};

// elements v .. v + N - 1 of a row of V > v; those at or beyond V read as -inf
template <bool BF16>
__device__ inline raw16 row_load(const void* row, int v, int V) {
    typedef Row<BF16> R;
    const typename R::T* p = (const typename R::T*)row + v;
    if (v + R::N <= V) return __builtin_nontemporal_load((const typename R::V*)p);
    float e[R::N];
#pragma unroll
    for (int i = 0; i < R::N; ++i) e[i] = R::one(p + min(i, V - 1 - v));   // loads that need not wait for each other (v < V)
#pragma unroll
    for (int i = 0; i < R::N; ++i) e[i] = v + i < V ? e[i] : -INFINITY;
    return R::pack(e);
}
template <bool BF16>
__device__ inline void row_store(void* row, int v, int V, const float* e) {
    typedef Row<BF16> R;
    typename R::T* p = (typename R::T*)row + v;
    if (v + R::N <= V) {
        __builtin_nontemporal_store((typename R::V)R::pack(e), (typename R::V*)p);
        return;
    }
#pragma unroll
    for (int i = 0; i < R::N; ++i)
        if (v + i < V) R::put_one(p + i, e[i]);
}

template <bool BF16>
struct None;   // 16 bytes of -inf
template <> struct None<false> { static constexpr uint32_t word = 0xff800000u; };
template <> struct None<true> { static constexpr uint32_t word = 0xff80ff80u; };
template <bool BF16>
__device__ inline raw16 none16() { return raw16{None<BF16>::word, None<BF16>::word, None<BF16>::word, None<BF16>::word}; }

template <bool BF16>
__device__ inline float vec_max(const raw16& r, float m) {
#pragma unroll
    for (int x = 0; x < Row<BF16>::N; ++x) m = fmaxf(m, Row<BF16>::get(r, x));
    return m;
}
template <bool BF16>
__device__ inline float vec_sum(const raw16& r, float m, float c2, float s) {
#pragma unroll
    for (int x = 0; x < Row<BF16>::N; ++x) s += fast_exp2((Row<BF16>::get(r, x) - m) * c2);
    return s;
}

inline int row_elem(int dtype) { return dtype == PSD_BF16 ? 2 : 4; }

// Two sets of rows are the same rows, or have no byte in common
inline bool rows_apart_or_same(const void* a, long long stride_a, const void* b, long long stride_b, long long n_rows, int vocab, int el) {
    if (a == b) return stride_a == stride_b || n_rows == 1;
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    const uintptr_t a1 = a0 + (uintptr_t)(((n_rows - 1) * stride_a + vocab) * el), b1 = b0 + (uintptr_t)(((n_rows - 1) * stride_b + vocab) * el);
    return a1 <= b0 || b1 <= a0;
}

// the part of the arguments that all operators on rows have
inline int rows_check(const char* who, const void* logits, int dtype, long long n_rows, int vocab, long long stride, char* err) {
    if (!logits) PSD_FAIL(PSD_EINVAL, err, "%s: null pointer", who);
    if (dtype != PSD_F32 && dtype != PSD_BF16) PSD_FAIL(PSD_EINVAL, err, "%s: dtype=%d", who, dtype);
    if (n_rows < 1 || n_rows > kMaxRows || vocab < 1 || vocab > kMaxVocab)
        PSD_FAIL(PSD_EINVAL, err, "%s: %lld rows of %d entries", who, n_rows, vocab);
    if (stride < vocab || stride > (1LL << 40)) PSD_FAIL(PSD_EINVAL, err, "%s: stride %lld of rows of %d entries", who, stride, vocab);
    if ((uintptr_t)logits % row_elem(dtype)) PSD_FAIL(PSD_EINVAL, err, "%s: misaligned logits", who);
    return PSD_OK;
}

// exponents are taken as differences times kLog2e / temperature, which has to be a number
inline bool temperature_fits(float temperature) { return temperature > 0.f && temperature <= 3.402823466e38f && kLog2e / temperature <= 3.402823466e38f; }

}  // namespace psd
