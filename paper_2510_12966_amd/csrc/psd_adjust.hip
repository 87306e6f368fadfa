// Adjusting rows of logits before they are judged or sampled: penalties for repeated tokens, biases, masks.
//
// One launch.  A workgroup takes one chunk of the vocabulary of one sequence and some of the sequence's rows.  It counts the
// occurrences of the chunk's tokens in the history (integer atomics in LDS: the counts do not depend on their order), finds the last bias
// given for each (an atomic maximum of places in the list), and then goes through its rows, the next one on its way while one is written,
// adding one token of the window after each.  Bound: the bytes of the rows, read once and written once, where histories are short; every
// chunk's workgroups go through the whole history, which is why long ones get larger chunks.
#include "psd_rows.h"

namespace psd {

constexpr int kAdjPer = 16;             // entries of a row that a thread has
constexpr uint32_t kPromptOnly = 0x80000000u;   // a count word: occurrences that count for presence and frequency, and this bit where
                                                // the token stands in the uncounted part of the history: 0 means it never occurred

struct AdjustArgs {
    const void* in;
    void* out;
    int rows, V, group;    // group: rows of a sequence that one workgroup goes through
    int counts, biases;    // 0 or 1: whether there are counts and biases to keep
    long long in_stride, out_stride;
    psd_adjust a;
};

// the part lo .. hi - 1 of a concatenation of n entries that belongs to a list with these offsets
__device__ inline void clamp_list(int64_t& lo, int64_t& hi, int64_t n) {
    lo = lo < 0 ? 0 : lo > n ? n : lo;
    hi = hi < lo ? lo : hi > n ? n : hi;
}

typedef int32_t four_tokens __attribute__((ext_vector_type(4), aligned(4)));

struct Penalty { float repetition, inverse, presence, frequency; };   // inverse: 1 / repetition

// One logit.  The quotient comes from the rounded inverse and one correction by its remainder (exact in the fused multiply-add); one beyond
// the largest float has no remainder and stays infinite.
__device__ inline float adjusted(float z, uint32_t count, const Penalty& p) {
    const float q = z * p.inverse, corrected = fmaf(fmaf(-q, p.repetition, z), p.inverse, q), quotient = corrected == corrected ? corrected : q;
    const float y = z > 0.f ? quotient : z * p.repetition;
    const uint32_t occurrences = count & ~kPromptOnly;
    const float minus = occurrences ? fmaf((float)occurrences, p.frequency, p.presence) : 0.f;
    return count ? y - minus : z;
}

// Where a sequence's lists lie.  Asked for all together, before anything waits.
struct Lists {
    int64_t lo, hi, counted, b0, b1;   // history, the first of its tokens that count, biases
    int m0, m1, m2;                    // the masks of the group's first rows
};

// What the lists say about the n entries from v0 on: occurrences in the history and in the window's first j0 tokens, and biases.  All threads,
// after the counts and biases have been cleared; a barrier at its end.
template <int NT>
__device__ inline void read_lists(const AdjustArgs& g, const Lists& w, uint32_t* count, uint32_t* bias, const int32_t* window, int v0, int n, int j0) {
    constexpr int AHEAD = 4;
    const psd_adjust& a = g.a;
    const int t = threadIdx.x;
    const uint32_t spare = kAdjPer * NT + (t & 63);
    // the first of the biases (all of them, most of the time) set out first
    const int64_t b0 = w.b0, b1 = w.b1;
    int32_t btok = -1;
    float bval = 0.f;
    if (b0 + t < b1) btok = a.bias_tokens[b0 + t], bval = a.bias[b0 + t];
    if (w.lo < w.hi) {   // two parts of the history on their way, in registers that take turns
        constexpr int PART = 4 * NT * AHEAD;
        auto fetch = [&](int32_t (&tok)[AHEAD][4], int64_t i0) {
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) {
                const int64_t i = i0 + 4 * (t + NT * x);
                if (i + 4 <= w.hi) {
                    const four_tokens f = *reinterpret_cast<const four_tokens*>(a.history + i);
#pragma unroll
                    for (int y = 0; y < 4; ++y) tok[x][y] = f[y];
                } else {
#pragma unroll
                    for (int y = 0; y < 4; ++y) tok[x][y] = i + y < w.hi ? a.history[i + y] : -1;
                }
            }
        };
        auto enter = [&](const int32_t (&tok)[AHEAD][4], int64_t i0) {
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) {
                // tokens of other chunks add to words behind the table, for a branch costs more than an addition; a wave whose tokens all
                // count, or none of them, does one of the two
                if (i0 + 4 * ((t & ~63) + NT * x) >= w.hi) break;
                const int before = (int)min(max(w.counted - (i0 + 4 * (t + NT * x)), (int64_t)0), (int64_t)4);   // of this thread's tokens
                uint32_t* at[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) at[y] = count + min((uint32_t)tok[x][y] - (uint32_t)v0, spare);
                if (__ballot(before < 4))
#pragma unroll
                    for (int y = 0; y < 4; ++y) atomicAdd(y < before ? count + spare : at[y], 1u);
                if (__ballot(before > 0))
#pragma unroll
                    for (int y = 0; y < 4; ++y) atomicOr(y < before ? at[y] : count + spare, kPromptOnly);
            }
        };
        int32_t even[AHEAD][4], odd[AHEAD][4];
        fetch(even, w.lo);
        if (w.lo + PART < w.hi) fetch(odd, w.lo + PART);
        for (int64_t i0 = w.lo;; i0 += 2 * PART) {
            enter(even, i0);
            if (i0 + PART >= w.hi) break;
            if (i0 + 2 * PART < w.hi) fetch(even, i0 + 2 * PART);
            enter(odd, i0 + PART);
            if (i0 + 2 * PART >= w.hi) break;
            if (i0 + 3 * PART < w.hi) fetch(odd, i0 + 3 * PART);
        }
    }
    if (window)
        for (int i = t; i < j0; i += NT) {
            const uint32_t u = (uint32_t)window[i] - (uint32_t)v0;
            if (u < (uint32_t)n) atomicAdd(&count[u], 1u);
        }
    if (a.bias) {
        const uint32_t u = (uint32_t)btok - (uint32_t)v0;
        if (u < (uint32_t)n) atomicMax(&bias[u], (uint32_t)t + 1u);
        for (int64_t i = b0 + NT + t; i < b1; i += NT) {
            const uint32_t w = (uint32_t)a.bias_tokens[i] - (uint32_t)v0;
            if (w < (uint32_t)n) atomicMax(&bias[w], (uint32_t)(i - b0) + 1u);
        }
        __syncthreads();
        if (b1 - b0 <= NT) {   // the places' own threads put the values there, once all have looked
            const bool counts = u < (uint32_t)n && bias[u] == (uint32_t)t + 1u;
            __syncthreads();
            if (counts) bias[u] = __float_as_uint(bval);
        } else {
            for (int i = t; i < n; i += NT) {
                const uint32_t at = bias[i];
                if (at) bias[i] = __float_as_uint(a.bias[b0 + at - 1]);
            }
        }
    }
    __syncthreads();
}

// The rows j0 .. j1 - 1 of a chunk: WHOLE where it lies inside the vocabulary.  Two rows are on their way while one is written; their registers
// take turns (moving a row over would wait for it).
template <bool BF16, int NT, bool WHOLE>
__device__ inline void adjust_group(const AdjustArgs& g, const Lists& lists, uint32_t* count, uint32_t* bias, const Penalty& pen, int s, int v0, int j0, int j1) {
    typedef Row<BF16> R;
    typedef typename R::T T;
    constexpr int N = R::N, VEC = kAdjPer / N;
    const psd_adjust& a = g.a;
    const int t = threadIdx.x, words = (g.V + 31) >> 5, n = WHOLE ? kAdjPer * NT : g.V - v0;
    const long long row0 = (long long)s * g.rows;
    auto mask_of = [&](int j) { return a.mask_index && j < j1 ? a.mask_index[row0 + j] : -1; };   // asked for a row ahead of its use
    auto load = [&](int j, int m, raw16 (&z)[VEC], uint32_t (&open)[VEC]) {
        const T* row = (const T*)g.in + (row0 + j) * g.in_stride + v0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int u = N * (t + NT * i);
            if (WHOLE) z[i] = (raw16)__builtin_nontemporal_load((const typename R::V*)(row + u));
            else if (u < n) z[i] = row_load<BF16>(row, u, n);
        }
        const bool masked = m >= 0 && m < a.n_masks;
#pragma unroll
        for (int i = 0; i < VEC; ++i) open[i] = m == -1 ? 0xffffffffu : 0u;
        if (masked) {
            const uint32_t* mask = a.masks + (long long)m * words + (v0 >> 5);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int u = N * (t + NT * i);
                if (WHOLE || u < n) open[i] = mask[u >> 5];   // shifted at its use, which waits for it
            }
        }
    };
    raw16 even[VEC], odd[VEC];
    uint32_t open_even[VEC], open_odd[VEC];
    int j = j0, m_next = lists.m2;
    load(j0, lists.m0, even, open_even);
    if (j0 + 1 < j1) load(j0 + 1, lists.m1, odd, open_odd);
    const int32_t* window = a.window ? a.window + (int64_t)s * a.window_stride : nullptr;
    __syncthreads();
    read_lists<NT>(g, lists, count, bias, window, v0, n, j0);
    auto step = [&](raw16 (&z)[VEC], uint32_t (&open)[VEC]) {   // true: the last row
        T* to = (T*)g.out + (row0 + j) * g.out_stride + v0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int u = N * (t + NT * i);
            float e[N];
#pragma unroll
            for (int x = 0; x < N; ++x) e[x] = R::get(z[i], x);
            if (g.counts) {
#pragma unroll
                for (int q = 0; q < N; q += 4) {
                    const uint4 c = *reinterpret_cast<const uint4*>(&count[u + q]);
                    e[q] = adjusted(e[q], c.x, pen);
                    e[q + 1] = adjusted(e[q + 1], c.y, pen);
                    e[q + 2] = adjusted(e[q + 2], c.z, pen);
                    e[q + 3] = adjusted(e[q + 3], c.w, pen);
                }
            }
            if (g.biases) {
#pragma unroll
                for (int q = 0; q < N; q += 4) {
                    const float4 b = *reinterpret_cast<const float4*>(&bias[u + q]);
                    e[q] += b.x;
                    e[q + 1] += b.y;
                    e[q + 2] += b.z;
                    e[q + 3] += b.w;
                }
            }
            const uint32_t allowed = open[i] >> (u & 31);
#pragma unroll
            for (int x = 0; x < N; ++x) e[x] = (allowed >> x) & 1 ? e[x] : -INFINITY;
            if (WHOLE) __builtin_nontemporal_store((typename R::V)R::pack(e), (typename R::V*)(to + u));
            else if (u < n) row_store<BF16>(to, u, n, e);
        }
        if (j + 2 < j1) {
            load(j + 2, m_next, z, open);
            m_next = mask_of(j + 3);
        }
        if (j + 1 >= j1) return true;
        if (window) {
            const uint32_t u = (uint32_t)window[j] - (uint32_t)v0;
            if (u < (uint32_t)n) {   // the same for all threads
                __syncthreads();
                if (t == 0) count[u] += 1;
                __syncthreads();
            }
        }
        ++j;
        return false;
    };
    while (!step(even, open_even) && !step(odd, open_odd)) {}
}

template <bool BF16, int NT>
__global__ __launch_bounds__(NT, 4) void adjust_rows(const AdjustArgs g) {
    constexpr int CHUNK = kAdjPer * NT;
    extern __shared__ uint4 lds[];
    uint32_t* const count = reinterpret_cast<uint32_t*>(lds);
    uint32_t* const bias = count + (g.counts ? CHUNK + 64 : 0);   // places in the list (from 1 on), then the biases themselves
    // the sequence is the fastest index: workgroups go round the dies, and the chunks of one sequence read its history out of the same L2
    const int s = blockIdx.x, v0 = blockIdx.z * CHUNK, j0 = blockIdx.y * g.group, j1 = min(g.rows, j0 + g.group);
    // What there is of each list is looked up by loads that no branch keeps from setting out together: those of an absent list read the
    // arguments themselves.
    const psd_adjust& a = g.a;
    const uint64_t here = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    const auto* off = (const __attribute__((address_space(4))) int64_t*)(a.history ? (uint64_t)(a.history_offsets + s) : here);
    const auto* boff = (const __attribute__((address_space(4))) int64_t*)(a.bias ? (uint64_t)(a.bias_offsets + s) : here);
    const auto* prompt = (const __attribute__((address_space(4))) int32_t*)(a.n_prompt ? (uint64_t)(a.n_prompt + s) : here);
    const auto* mask = (const __attribute__((address_space(4))) int32_t*)(a.mask_index ? (uint64_t)(a.mask_index + (long long)s * g.rows + j0) : here);
    const auto* pens = (const __attribute__((address_space(4))) float*)(a.penalties ? (uint64_t)(a.penalties + 3 * (int64_t)s) : here);
    const int more = a.mask_index ? j1 - 1 - j0 : 0;
    Lists lists{off[0], off[1], prompt[0], boff[0], boff[1], mask[0], mask[min(1, more)], mask[min(2, more)]};
    Penalty pen{pens[0], 0.f, pens[1], pens[2]};
    for (int i = threadIdx.x; i < (g.counts + g.biases) * (CHUNK / 4) + 16 * g.counts; i += NT) lds[i] = make_uint4(0, 0, 0, 0);
    clamp_list(lists.lo, lists.hi, a.n_history);
    clamp_list(lists.b0, lists.b1, a.n_bias);
    lists.counted = a.n_prompt ? lists.lo + max((int64_t)0, lists.counted) : lists.lo;
    if (!a.history) lists.hi = lists.lo;
    if (!a.bias) lists.b1 = lists.b0;
    if (!a.mask_index) lists.m0 = lists.m1 = lists.m2 = -1;
    if (!a.penalties) pen = Penalty{1.f, 1.f, 0.f, 0.f};
    if (!(pen.repetition > 0.f)) pen.repetition = 1.f;
    pen.inverse = 1.f / pen.repetition;
    if (v0 + CHUNK <= g.V) adjust_group<BF16, NT, true>(g, lists, count, bias, pen, s, v0, j0, j1);
    else adjust_group<BF16, NT, false>(g, lists, count, bias, pen, s, v0, j0, j1);
}

template <bool BF16, int NT>
static void adjust_launch(AdjustArgs& g, int n_seqs, hipStream_t st) {
    const int chunks = (g.V + kAdjPer * NT - 1) / (kAdjPer * NT);
    const dim3 grid(n_seqs, (g.rows + g.group - 1) / g.group, chunks);
    adjust_rows<BF16, NT><<<grid, NT, (size_t)(g.counts + g.biases) * kAdjPer * NT * 4 + 256 * g.counts, st>>>(g);
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
    AdjustArgs g{logits, out, rows, vocab, rows, 0, 0, logits_stride, out_stride, *adjust};
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
    // without penalties occurrences change nothing
    if (!a.penalties) a.history = nullptr, a.window = nullptr;
    g.counts = a.history || a.window;
    g.biases = a.bias != nullptr;
    // Chunks of 4096 entries; of 16384 (a workgroup of 1024 threads per unit) where histories are long, for every chunk reads all of its
    // sequence's (us, 4096 / 16384; one bf16 row of 128256 for each of 64 sequences: 30000 tokens 33.9 / 20.8, 3000 tokens 15.1 / 15.7)
    const bool large = a.history && a.n_history / n_seqs > 4096;
    // Every group of rows reads the lists again and leaves a workgroup more: groups of one row as long as the chip is not full, larger ones then (us;
    // 32 rows of 32000 for 8 sequences: 1 / 2 / 5 rows a group 16.1 / 14.6 / 18.9; 9 rows of 128256 for 48: 98 / 93 / 91)
    const long long chunks = (vocab + (large ? 16383 : 4095)) / (large ? 16384 : 4096), most = (n * vocab * row_elem(dtype) < 64LL << 20 ? 1024 : 3072) / (large ? 4 : 1);
    long long groups = most / (chunks * n_seqs);
    groups = groups < 1 ? 1 : groups > rows ? rows : groups;
    g.group = (int)((rows + groups - 1) / groups);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == PSD_BF16) large ? adjust_launch<true, 1024>(g, n_seqs, st) : adjust_launch<true, 256>(g, n_seqs, st);
    else large ? adjust_launch<false, 1024>(g, n_seqs, st) : adjust_launch<false, 256>(g, n_seqs, st);
    PSD_HIP(hipGetLastError(), err);
    return PSD_OK;
}
