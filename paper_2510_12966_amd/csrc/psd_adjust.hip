// Adjusting rows of logits before they are judged or sampled: penalties for repeated tokens, biases, masks.
//
// One launch.  A workgroup takes one chunk of the vocabulary of one sequence and some of the sequence's rows.  It finds the last bias given
// for each of the chunk's tokens (an atomic maximum of places in the list), counts their occurrences in the history (integer atomics in LDS: the
// counts do not depend on their order), and then goes through its rows, the next one on its way while one is written, adding one token of the
// window after each.
// Bound: the bytes of the rows, read once and written once: 4.8 TB/s with 2000 tokens of history and 9 fp32 rows of 128255 for each of 48
// sequences (93 us), as a large copy has; bf16 rows have twice the entries per byte: 432 of 128256, 55 us, 4.1 TB/s.  Long histories: every
// chunk's workgroups go through all of it, out of their die's L2; 64 bf16 rows with 30000 tokens each (15000 to 45000) take 17 us, 10 without
// any history.  Few rows: one launch and three loads that wait for one another (where the lists lie, their tokens, what they count), 4.9 us for
// one row.
#include "psd_rows.h"

#include <algorithm>

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

struct Penalty { float repetition, divisor, up, inverse, presence, frequency; };   // divisor: repetition * up, inverse: 1 / divisor

// One logit.  The quotient comes from the rounded inverse and one correction by its remainder (exact in the fused multiply-add); one beyond
// the largest float has no remainder and stays infinite.  A repetition so small that its inverse is no float is taken 2^64 times as large, and the
// logit with it (where that passes the largest float, the quotient does as well).
__device__ inline float adjusted(float z, uint32_t count, const Penalty& p) {
    const float n = z * p.up, q = n * p.inverse, corrected = fmaf(fmaf(-q, p.divisor, n), p.inverse, q), quotient = corrected == corrected ? corrected : q;
    const float y = z > 0.f ? quotient : z * p.repetition;
    const uint32_t occurrences = count & ~kPromptOnly;
    const float minus = occurrences ? fmaf((float)occurrences, p.frequency, p.presence) : 0.f;
    return count ? y - minus : z;
}

// What a workgroup keeps of the lists.  Biases are few: a bit for every entry of the chunk that has one, and their values packed, those of 32
// entries from `first` on.
struct ChunkLds {
    uint32_t* count;    // [chunk + 64], the last 64 for tokens of other chunks
    uint32_t* biased;   // [chunk / 32]
    uint32_t* first;    // [chunk / 32], of words that are not 0
    float* value;
    uint32_t* total;
};
constexpr uint32_t kNoToken = 0xffffffffu;

// Where a sequence's lists lie.  Asked for all together, before anything waits.
struct Lists {
    int64_t lo, hi, counted, b0, b1;   // history, the first of its tokens that count, biases
    int m0, m1, m2;                    // the masks of the group's first rows
};

// What the lists say about the n entries from v0 on: occurrences in the history and in the window's first j0 tokens, and biases.  All threads,
// after the counts and biases have been cleared; a barrier at its end.
template <int NT, int PARTS>
__device__ inline void read_lists(const AdjustArgs& g, const Lists& w, const ChunkLds& l, const int32_t* window, int v0, int n, int j0) {
    constexpr int AHEAD = PARTS == 2 ? 2 : 4, CHUNK = kAdjPer * NT * PARTS;
    uint32_t* const count = l.count;
    const psd_adjust& a = g.a;
    const int t = threadIdx.x;
    const uint32_t spare = CHUNK + (t & 63);
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
    // the last bias of a token is the one whose place its word holds in the end; the first NT of the list stay with their threads
    const int many = (int)(w.b1 - w.b0);
    uint32_t u0 = kNoToken;
    float value0 = 0.f;
    auto fetch_bias = [&](int i, uint32_t& u, float& value) {
        u = (uint32_t)a.bias_tokens[w.b0 + i] - (uint32_t)v0;
        value = a.bias[w.b0 + i];
    };
    if (t < many) fetch_bias(t, u0, value0);
    int32_t even[AHEAD][4], odd[AHEAD][4];   // two parts of the history on their way, in registers that take turns
    if (w.lo < w.hi) fetch(even, w.lo);
    if (w.lo + PART < w.hi) fetch(odd, w.lo + PART);
    if (many > 0) {
        auto each = [&](auto&& f) {
            if (u0 < (uint32_t)n) f((uint32_t)t + 1u, u0, value0);
            for (int i = t + NT; i < many; i += NT) {
                uint32_t u;
                float value;
                fetch_bias(i, u, value);
                if (u < (uint32_t)n) f((uint32_t)i + 1u, u, value);
            }
        };
        each([&](uint32_t place, uint32_t u, float) {
            atomicMax(&count[u], place);
            atomicOr(&l.biased[u >> 5], 1u << (u & 31));
        });
        __syncthreads();
        for (int i = t; i < CHUNK / 32; i += NT)
            if (l.biased[i]) l.first[i] = atomicAdd(l.total, (uint32_t)__popc(l.biased[i]));
        __syncthreads();
        each([&](uint32_t place, uint32_t u, float value) {
            if (count[u] != place) return;
            count[u] = 0;
            l.value[l.first[u >> 5] + __popc(l.biased[u >> 5] & ((1u << (u & 31)) - 1u))] = value;
        });
        __syncthreads();
    }
    if (w.lo < w.hi)
        for (int64_t i0 = w.lo;; i0 += 2 * PART) {
            enter(even, i0);
            if (i0 + PART >= w.hi) break;
            if (i0 + 2 * PART < w.hi) fetch(even, i0 + 2 * PART);
            enter(odd, i0 + PART);
            if (i0 + 2 * PART >= w.hi) break;
            if (i0 + 3 * PART < w.hi) fetch(odd, i0 + 3 * PART);
        }
    if (window)
        for (int i = t; i < j0; i += NT) {
            const uint32_t u = (uint32_t)window[i] - (uint32_t)v0;
            if (u < (uint32_t)n) atomicAdd(&count[u], 1u);
        }
    __syncthreads();
}

// The rows j0 .. j1 - 1 of a chunk: WHOLE where it lies inside the vocabulary.  Two rows, or the PARTS = 2 of one, are on their way while one is
// written; their registers take turns (moving a row over would wait for it).
template <bool BF16, int NT, int PARTS, bool WHOLE>
__device__ inline void adjust_group(const AdjustArgs& g, const Lists& lists, const ChunkLds& l, const Penalty& pen, int s, int v0, int j0, int j1) {
    typedef Row<BF16> R;
    typedef typename R::T T;
    constexpr int N = R::N, VEC = kAdjPer / N, PART = kAdjPer * NT;
    const psd_adjust& a = g.a;
    const int t = threadIdx.x, words = (g.V + 31) >> 5, n = WHOLE ? PARTS * PART : g.V - v0;
    const long long row0 = (long long)s * g.rows;
    // entry `mine` + `ahead`, ahead the same for all threads and a multiple of 32: what depends on the thread is one address per table
    const int mine = N * t, mine_word = mine >> 5, mine_bit = mine & 31;
    auto mask_of = [&](int j) { return a.mask_index && j < j1 ? a.mask_index[row0 + j] : -1; };   // asked for a row ahead of its use
    auto load = [&](int j, int part, int m, raw16 (&z)[VEC], uint32_t (&open)[VEC]) {
        const T* row = (const T*)g.in + (row0 + j) * g.in_stride + v0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int ahead = N * NT * i + part * PART;
            if (WHOLE) z[i] = (raw16)__builtin_nontemporal_load((const typename R::V*)(row + ahead + mine));
            else if (mine < n - ahead) z[i] = row_load<BF16>(row, ahead + mine, n);
        }
        const bool masked = m >= 0 && m < a.n_masks;
#pragma unroll
        for (int i = 0; i < VEC; ++i) open[i] = m == -1 ? 0xffffffffu : 0u;
        if (masked) {
            const uint32_t* mask = a.masks + (long long)m * words + (v0 >> 5);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int ahead = N * NT * i + part * PART;
                if (WHOLE || mine < n - ahead) open[i] = (mask + ahead / 32)[mine_word];   // shifted at its use, which waits for it
            }
        }
    };
    raw16 even[VEC], odd[VEC];
    uint32_t open_even[VEC], open_odd[VEC];
    load(j0, 0, lists.m0, even, open_even);
    if (PARTS == 2) load(j0, 1, lists.m0, odd, open_odd);
    else if (j0 + 1 < j1) load(j0 + 1, 0, lists.m1, odd, open_odd);
    const int32_t* window = a.window ? a.window + (int64_t)s * a.window_stride : nullptr;
    __syncthreads();
    read_lists<NT, PARTS>(g, lists, l, window, v0, n, j0);
    auto put = [&](int j, int part, const raw16 (&z)[VEC], const uint32_t (&open)[VEC]) {
        T* to = (T*)g.out + (row0 + j) * g.out_stride + v0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int ahead = N * NT * i + part * PART;
            float e[N];
#pragma unroll
            for (int x = 0; x < N; ++x) e[x] = R::get(z[i], x);
            if (g.counts) {
#pragma unroll
                for (int q = 0; q < N; q += 4) {
                    const uint4 c = *reinterpret_cast<const uint4*>(&l.count[mine] + ahead + q);
                    e[q] = adjusted(e[q], c.x, pen);
                    e[q + 1] = adjusted(e[q + 1], c.y, pen);
                    e[q + 2] = adjusted(e[q + 2], c.z, pen);
                    e[q + 3] = adjusted(e[q + 3], c.w, pen);
                }
            }
            if (g.biases) {
                const uint32_t word = (&l.biased[mine_word])[ahead / 32], here = word >> mine_bit & ((1u << N) - 1u);
                if (here) {
                    const float* value = l.value + (&l.first[mine_word])[ahead / 32] + __popc(word & ((1u << mine_bit) - 1u));
#pragma unroll
                    for (int x = 0; x < N; ++x)
                        if ((here >> x) & 1) e[x] += *value++;
                }
            }
            const uint32_t allowed = open[i] >> mine_bit;
#pragma unroll
            for (int x = 0; x < N; ++x) e[x] = (allowed >> x) & 1 ? e[x] : -INFINITY;
            if (WHOLE) __builtin_nontemporal_store((typename R::V)R::pack(e), (typename R::V*)(to + ahead + mine));
            else if (mine < n - ahead) row_store<BF16>(to, ahead + mine, n, e);
            if (PARTS == 2) __builtin_amdgcn_sched_barrier(0);   // one vector's elements at a time
        }
    };
    auto next = [&](int j) {   // the row behind row j has one token more before it
        if (!window) return;
        const uint32_t u = (uint32_t)window[j] - (uint32_t)v0;
        if (u < (uint32_t)n) {   // the same for all threads
            __syncthreads();
            if (t == 0) l.count[u] += 1;
            __syncthreads();
        }
    };
    if constexpr (PARTS == 2) {
        for (int j = j0, m = lists.m1;; ++j) {
            const bool more = j + 1 < j1;
            put(j, 0, even, open_even);
            if (more) load(j + 1, 0, m, even, open_even);
            put(j, 1, odd, open_odd);
            if (!more) break;
            load(j + 1, 1, m, odd, open_odd);
            m = mask_of(j + 2);
            next(j);
        }
    } else {
        int j = j0, m = lists.m2;
        auto step = [&](raw16 (&z)[VEC], uint32_t (&open)[VEC]) {   // true: the last row
            put(j, 0, z, open);
            if (j + 2 < j1) {
                load(j + 2, 0, m, z, open);
                m = mask_of(j + 3);
            }
            if (j + 1 >= j1) return true;
            next(j++);
            return false;
        };
        while (!step(even, open_even) && !step(odd, open_odd)) {}
    }
}

template <bool BF16, int NT, int PARTS>
__global__ __launch_bounds__(NT, 4) void adjust_rows(const AdjustArgs g) {
    constexpr int CHUNK = kAdjPer * NT * PARTS;
    extern __shared__ uint4 lds[];
    uint32_t* const words = reinterpret_cast<uint32_t*>(lds);
    const ChunkLds l{words, words + CHUNK + 64, words + CHUNK + 64 + CHUNK / 32 + 4, reinterpret_cast<float*>(words + CHUNK + 64 + CHUNK / 16 + 4), words + CHUNK + 64 + CHUNK / 32};
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
    Penalty pen{pens[0], 1.f, 1.f, 1.f, pens[1], pens[2]};
    if (g.counts | g.biases)
        for (int i = threadIdx.x; i < (CHUNK + 64 + CHUNK / 32 + 4) / 4; i += NT) lds[i] = make_uint4(0, 0, 0, 0);
    clamp_list(lists.lo, lists.hi, a.n_history);
    clamp_list(lists.b0, lists.b1, a.n_bias);
    lists.counted = a.n_prompt ? lists.lo + max((int64_t)0, lists.counted) : lists.lo;
    if (!a.history) lists.hi = lists.lo;
    if (!a.bias) lists.b1 = lists.b0;
    if (!a.mask_index) lists.m0 = lists.m1 = lists.m2 = -1;
    if (!a.penalties) pen = Penalty{1.f, 1.f, 1.f, 1.f, 0.f, 0.f};
    if (!(pen.repetition > 0.f)) pen.repetition = 1.f;
    pen.up = pen.repetition < 0x1p-120f ? 0x1p64f : 1.f;
    pen.divisor = pen.repetition * pen.up;
    pen.inverse = 1.f / pen.divisor;
    if (v0 + CHUNK <= g.V) adjust_group<BF16, NT, PARTS, true>(g, lists, l, pen, s, v0, j0, j1);
    else adjust_group<BF16, NT, PARTS, false>(g, lists, l, pen, s, v0, j0, j1);
}

template <bool BF16, int NT, int PARTS>
static void adjust_launch(AdjustArgs& g, int n_seqs, hipStream_t st) {
    constexpr int CHUNK = kAdjPer * NT * PARTS;
    const dim3 grid(n_seqs, (g.rows + g.group - 1) / g.group, (g.V + CHUNK - 1) / CHUNK);
    const size_t words = (g.counts | g.biases ? CHUNK + 64 + CHUNK / 16 + 4 : 0) + (g.biases ? (size_t)std::min<int64_t>(g.a.n_bias, CHUNK) : 0);
    adjust_rows<BF16, NT, PARTS><<<grid, NT, words * 4, st>>>(g);
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
    if (a.n_history < 0 || a.n_bias < 0 || a.n_masks < 0 || a.n_masks > 0x7fffffffLL || a.n_bias > 1LL << 30)
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
    // Chunks of 4096 entries (a workgroup of 256 threads, four a unit with fp32 rows, five with bf16), or of 16384 (512 threads, two a unit; one where all
    // lists of biases together pass some 3500 entries, since the room in LDS is for them all: 64 bf16 rows with 30000 tokens, 40 / 60 biases
    // each 16.6 / 24.4 us): every chunk goes through all of
    // its sequence's history, so longer histories take larger chunks, the sooner the fuller the chip is without (us, 4096 / 16384; one row of 128256
    // for each sequence, fp32: 1 sequence with 12000 tokens 7.5 / 8.8, 30000: 11.0 / 11.1; 32 with 3000 8.8 / 9.8, 12000: 12.7 / 11.1; 64 with 500
    // 15.2 / 12.1, 30000: 37.8 / 18.7; 9 rows for each of 64: 500 tokens 114.5 / 117.5, 30000: 129.4 / 122.4)
    const long long units = (vocab + 4095LL) / 4096 * n_seqs, tokens = a.history ? a.n_history / n_seqs : 0;
    const bool large = a.history && (tokens > 16384 || (tokens > 4096 && units >= 1024) || (rows == 1 && units >= 2048));
    // Every group of rows reads the lists again and leaves a workgroup more: groups of few rows as long as the chip is not full, larger ones then
    // (us; 32 fp32 rows of 32000 for each of 8 sequences: 1 / 2 / 5 rows a group 16.9 / 16.6 / 21.7; 9 of 128256 for 8: 1 / 3 / 9 rows 18.6 / 15.2 / 24.3,
    // for 48: 96.2 / 92.2 / 89.1)
    const long long chunks = (vocab + (large ? 16383 : 4095)) / (large ? 16384 : 4096), most = (n * vocab * row_elem(dtype) < 64LL << 20 ? 1024 : 3 * 1024) / (large ? 4 : 1);
    long long groups = most / (chunks * n_seqs);
    groups = groups < 1 ? 1 : groups > rows ? rows : groups;
    g.group = (int)((rows + groups - 1) / groups);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == PSD_BF16) large ? adjust_launch<true, 512, 2>(g, n_seqs, st) : adjust_launch<true, 256, 1>(g, n_seqs, st);
    else large ? adjust_launch<false, 512, 2>(g, n_seqs, st) : adjust_launch<false, 256, 1>(g, n_seqs, st);
    PSD_HIP(hipGetLastError(), err);
    return PSD_OK;
}
