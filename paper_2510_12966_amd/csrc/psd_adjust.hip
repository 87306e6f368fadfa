// Adjusting rows of logits before they are judged or sampled: penalties for repeated tokens, biases, masks.
//
// One launch.  A workgroup takes one chunk of the vocabulary of one sequence and some of the sequence's rows.  It counts the
// occurrences of the chunk's tokens in the history (integer atomics in LDS: the counts do not depend on their order), finds the last bias
// given for each (an atomic maximum of places in the list), and then goes through its rows, adding one token of the window
// after each.  Bound: the bytes of the rows, read once and written once.
#include "psd_rows.h"

namespace psd {

constexpr int kAdjThreads = 256;
constexpr int kAdjChunk = 4096;         // vocabulary entries of a workgroup: 16 KB of counts and as much of biases
constexpr uint32_t kPromptOnly = 0x80000000u;   // a count word: occurrences that count for presence and frequency, and this bit where
                                                // the token stands in the uncounted part of the history: 0 means it never occurred

struct AdjustArgs {
    const void* in;
    void* out;
    int rows, V, group;   // group: rows of a sequence that one workgroup goes through
    long long in_stride, out_stride;
    psd_adjust a;
};

// the part lo .. hi - 1 of a concatenation of n entries that belongs to list s
__device__ inline void list_of(const int64_t* offsets, int s, int64_t n, int64_t& lo, int64_t& hi) {
    lo = offsets[s];
    hi = offsets[s + 1];
    lo = lo < 0 ? 0 : lo > n ? n : lo;
    hi = hi < lo ? lo : hi > n ? n : hi;
}

template <bool BF16>
__global__ __launch_bounds__(kAdjThreads) void adjust_rows(const AdjustArgs g) {
    typedef Row<BF16> R;
    constexpr int N = R::N, VEC = kAdjChunk / (N * kAdjThreads);   // vectors of a row that a thread has: 4 or 2
    __shared__ uint32_t count[kAdjChunk];
    __shared__ uint32_t bias[kAdjChunk];   // places in the list (from 1 on), then the biases themselves
    const psd_adjust& a = g.a;
    const int s = blockIdx.z, v0 = blockIdx.x * kAdjChunk, n = min(kAdjChunk, g.V - v0);
    const int j0 = blockIdx.y * g.group, j1 = min(g.rows, j0 + g.group);
    const int t = threadIdx.x;
    int64_t h0 = 0, h1 = 0, b0 = 0, b1 = 0;
    if (a.history) list_of(a.history_offsets, s, a.n_history, h0, h1);
    if (a.bias) list_of(a.bias_offsets, s, a.n_bias, b0, b1);
    for (int i = t; i < kAdjChunk; i += kAdjThreads) count[i] = 0, bias[i] = 0;
    __syncthreads();
    const int64_t counted = h0 + (a.n_prompt ? max(0, a.n_prompt[s]) : 0);
    for (int64_t i = h0 + t; i < h1; i += kAdjThreads) {
        const uint32_t u = (uint32_t)a.history[i] - (uint32_t)v0;
        if (u >= (uint32_t)n) continue;
        if (i >= counted) atomicAdd(&count[u], 1u);
        else atomicOr(&count[u], kPromptOnly);
    }
    const int32_t* window = a.window ? a.window + (int64_t)s * a.window_stride : nullptr;
    if (window)
        for (int i = t; i < j0; i += kAdjThreads) {
            const uint32_t u = (uint32_t)window[i] - (uint32_t)v0;
            if (u < (uint32_t)n) atomicAdd(&count[u], 1u);
        }
    for (int64_t i = b0 + t; i < b1; i += kAdjThreads) {
        const uint32_t u = (uint32_t)a.bias_tokens[i] - (uint32_t)v0;
        if (u < (uint32_t)n) atomicMax(&bias[u], (uint32_t)(i - b0) + 1u);
    }
    __syncthreads();
    if (b1 > b0) {
        for (int i = t; i < n; i += kAdjThreads) {
            const uint32_t at = bias[i];
            bias[i] = at ? __float_as_uint(a.bias[b0 + at - 1]) : 0u;
        }
        __syncthreads();
    }
    float rep = 1.f, presence = 0.f, frequency = 0.f;
    if (a.penalties) {
        rep = a.penalties[3 * s];
        presence = a.penalties[3 * s + 1];
        frequency = a.penalties[3 * s + 2];
        if (!(rep > 0.f)) rep = 1.f;
    }
    const int words = (g.V + 31) >> 5;
    for (int j = j0; j < j1; ++j) {
        const long long r = (long long)s * g.rows + j;
        const typename R::T* row = (const typename R::T*)g.in + r * g.in_stride;
        typename R::T* to = (typename R::T*)g.out + r * g.out_stride;
        const uint32_t* mask = nullptr;
        bool closed = false;
        if (a.mask_index) {
            const int m = a.mask_index[r];
            if (m >= 0 && m < a.n_masks) mask = a.masks + (long long)m * words;
            else closed = m != -1;
        }
        raw16 z[VEC];
        uint32_t open[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int v = v0 + N * (t + kAdjThreads * i);
            open[i] = closed ? 0u : 0xffffffffu;
            if (v < g.V) {
                z[i] = row_load<BF16>(row, v, g.V);
                if (mask) open[i] = mask[v >> 5] >> (v & 31);
            }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int u = N * (t + kAdjThreads * i), v = v0 + u;
            if (v >= g.V) continue;
            float e[N];
#pragma unroll
            for (int x = 0; x < N; ++x) {
                float y = R::get(z[i], x);
                const uint32_t c = count[u + x];
                if (c) {
                    y = y > 0.f ? y / rep : y * rep;
                    const uint32_t occurrences = c & ~kPromptOnly;
                    if (occurrences) y = y - fmaf((float)occurrences, frequency, presence);
                }
                y = y + __uint_as_float(bias[u + x]);
                e[x] = (open[i] >> x) & 1 ? y : -INFINITY;
            }
            row_store<BF16>(to, v, g.V, e);
        }
        if (window && j + 1 < j1) {
            __syncthreads();
            if (t == 0) {
                const uint32_t u = (uint32_t)window[j] - (uint32_t)v0;
                if (u < (uint32_t)n) count[u] += 1;
            }
            __syncthreads();
        }
    }
}

}  // namespace psd

using namespace psd;

extern "C" int psd_adjust_logits(const void* logits, void* out, int32_t dtype, int32_t n_seqs, int32_t rows, int32_t vocab,
                                 int64_t logits_stride, int64_t out_stride, const psd_adjust* adjust, void* stream) {
    char* err = tls_error();
    const char* who = "psd_adjust_logits";
    if (!out || !adjust) PSD_FAIL(PSD_EINVAL, err, "%s: null pointer", who);
    if (n_seqs < 1 || rows < 1) PSD_FAIL(PSD_EINVAL, err, "%s: n_seqs=%d rows=%d", who, n_seqs, rows);
    const long long n = (long long)n_seqs * rows;
    int rc = rows_check(who, logits, dtype, n, vocab, logits_stride, err);
    if (rc == PSD_OK) rc = rows_check(who, out, dtype, n, vocab, out_stride, err);
    if (rc != PSD_OK) return rc;
    if (!rows_apart_or_same(logits, logits_stride, out, out_stride, n, vocab, row_elem(dtype)))
        PSD_FAIL(PSD_EINVAL, err, "%s: out overlaps the logits", who);
    AdjustArgs g{logits, out, rows, vocab, rows, logits_stride, out_stride, *adjust};
    psd_adjust& a = g.a;
    if (a.n_history < 0 || a.n_bias < 0 || a.n_masks < 0 || a.n_masks > 0x7fffffffLL || a.n_bias > 0x7fffffffLL)
        PSD_FAIL(PSD_EINVAL, err, "%s: n_history=%lld n_bias=%lld n_masks=%lld", who, (long long)a.n_history, (long long)a.n_bias, (long long)a.n_masks);
    if (a.n_history > 0 && (!a.history || !a.history_offsets)) PSD_FAIL(PSD_EINVAL, err, "%s: a history needs its tokens and offsets", who);
    if (a.n_bias > 0 && (!a.bias || !a.bias_tokens || !a.bias_offsets)) PSD_FAIL(PSD_EINVAL, err, "%s: biases need their tokens and offsets", who);
    if (a.n_masks > 0 && !a.masks) PSD_FAIL(PSD_EINVAL, err, "%s: null masks", who);
    if ((a.masks != nullptr) != (a.mask_index != nullptr)) PSD_FAIL(PSD_EINVAL, err, "%s: masks and mask_index come together", who);
    if (a.window && a.window_stride < rows - 1) PSD_FAIL(PSD_EINVAL, err, "%s: window_stride %lld of windows of %d tokens", who, (long long)a.window_stride, rows - 1);
    if (((uintptr_t)a.history | (uintptr_t)a.n_prompt | (uintptr_t)a.window | (uintptr_t)a.penalties | (uintptr_t)a.bias_tokens | (uintptr_t)a.bias |
         (uintptr_t)a.masks | (uintptr_t)a.mask_index) & 3 || ((uintptr_t)a.history_offsets | (uintptr_t)a.bias_offsets) & 7)
        PSD_FAIL(PSD_EINVAL, err, "%s: misaligned lists", who);
    if (a.n_history == 0) a.history = nullptr;
    if (a.n_bias == 0) a.bias = nullptr;
    if (rows == 1) a.window = nullptr;
    const int chunks = (vocab + kAdjChunk - 1) / kAdjChunk;
    // Every workgroup goes through the history again, so a sequence's rows stay together, unless that leaves the chip short of workgroups
    while (g.group > 1 && (long long)chunks * n_seqs * ((rows + g.group - 1) / g.group) < 1024) g.group = (g.group + 1) / 2;
    const dim3 grid(chunks, (rows + g.group - 1) / g.group, n_seqs);
    if (dtype == PSD_BF16) adjust_rows<true><<<grid, kAdjThreads, 0, (hipStream_t)stream>>>(g);
    else adjust_rows<false><<<grid, kAdjThreads, 0, (hipStream_t)stream>>>(g);
    PSD_HIP(hipGetLastError(), err);
    return PSD_OK;
}
