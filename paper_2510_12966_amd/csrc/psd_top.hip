// The k largest entries of every row of logits, with the row's log-sum-exp.
//
// A workgroup streams over a segment of a row, 4096 entries at a time, and keeps a list of candidates in LDS: entries not below a
// threshold that at least k entries of the segment are known to reach.  The first threshold is the k-th largest of the threads' own maxima in the
// first block; whenever the list is cut to its k largest, their smallest becomes the threshold, and later entries have to exceed it (an equal
// one has a higher token and comes behind).  Cuts are exact: radix selection, 8 bits a round, over 64-bit items (order-preserving image of
// the value, complement of the token), which all differ, so that equal values fall in the order of their tokens by themselves.
// Many rows: one segment each, one launch.  Few rows: several segments, whose lists a second launch merges.
// Bound: the bytes of the rows, read once.
#include "psd_rows.h"

namespace psd {

constexpr int kTopThreads = 256;
constexpr int kTopBlock = 4096;                       // entries between two looks at the list
constexpr int kTopPer = kTopBlock / kTopThreads;      // of one thread: 16
constexpr int kTopLow = 512;                          // a list longer than this is cut before the next block
constexpr int kTopList = kTopLow + kTopBlock;         // so every entry of a block finds a place in it
constexpr int kTopItems = kTopList / kTopThreads;     // 18

typedef unsigned long long u64;

// order-preserving image of a value; equal values (0 and -0 among them) have equal images; 0 is no value's
__device__ inline uint32_t rank_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(uint32_t r) { return __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r); }
__device__ inline u64 item_of(float z, int v) { return (u64)rank_of(z) << 32 | (uint32_t)~v; }

struct TopLds {
    u64 list[kTopList];
    uint32_t hist[3][256];   // one is filled, the next cleared, the last may still be read
    uint32_t maxima[kTopThreads];
    float2 part[kTopThreads / 64];
    int count;
    uint32_t least;
};

// Cuts a list of n items (k < n <= kTopList) to its k largest; returns the smallest of them.  All threads, n uniform.
__device__ inline u64 cut_to(TopLds& l, int n, int k) {
    const int t = threadIdx.x, lane = t & 63;
    u64 it[kTopItems];
#pragma unroll
    for (int i = 0; i < kTopItems; ++i) it[i] = t + kTopThreads * i < n ? l.list[t + kTopThreads * i] : 0;
    l.hist[0][t] = 0;
    __syncthreads();
    u64 least = 0;
    int need = k;
    for (int shift = 56, turn = 0; shift >= 0; shift -= 8, turn = turn == 2 ? 0 : turn + 1) {
        l.hist[turn == 2 ? 0 : turn + 1][t] = 0;
        const u64 above = shift == 56 ? 0 : ~0ull << (shift + 8);
#pragma unroll
        for (int i = 0; i < kTopItems; ++i)
            if (it[i] != 0 && (it[i] & above) == least) atomicAdd(&l.hist[turn][(uint32_t)(it[i] >> shift) & 255], 1u);
        __syncthreads();
        // every wave: lane x has bins 255 - 4x .. 252 - 4x; a scan over the lanes finds the bin in which the need-th largest lies
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = l.hist[turn][255 - 4 * lane - i];
        uint32_t sum = h[0] + h[1] + h[2] + h[3], upto = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int who = __ffsll(__ballot(upto >= (uint32_t)need)) - 1;   // there is one: the bins hold at least `need` items
        uint32_t before = upto - sum, bin = 0, size = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool here = before < (uint32_t)need && before + h[i] >= (uint32_t)need;
            if (here) bin = 255 - 4 * lane - i, size = h[i], sum = before;
            before += h[i];
        }
        bin = __shfl(bin, who);
        size = __shfl(size, who);
        need -= (int)__shfl(sum, who);
        least |= (u64)bin << shift;
        if ((uint32_t)need == size) break;   // the whole bin belongs to them
    }
    if (t == 0) l.count = 0;
    __syncthreads();
    u64 mine = ~0ull;
#pragma unroll
    for (int i = 0; i < kTopItems; ++i)
        if (it[i] != 0 && it[i] >= least) {
            l.list[atomicAdd(&l.count, 1)] = it[i];
            mine = min(mine, it[i]);
        }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) mine = min(mine, (u64)__shfl_xor((long long)mine, d));
    u64* smallest = reinterpret_cast<u64*>(l.maxima);
    if (lane == 0) smallest[t >> 6] = mine;
    __syncthreads();
    return min(min(smallest[0], smallest[1]), min(smallest[2], smallest[3]));
}

// The list's n <= k items in descending order into one row of the outputs
__device__ inline void put_sorted(const TopLds& l, int n, int k, float* values, int32_t* ids) {
    const int t = threadIdx.x;
    if (t < n) {
        const u64 mine = l.list[t];
        int at = 0;
        for (int i = 0; i < n; ++i) at += l.list[i] > mine;
        values[at] = value_of((uint32_t)(mine >> 32));
        ids[at] = (int32_t)~(uint32_t)mine;
    }
    if (t >= n && t < k) {
        values[t] = -INFINITY;
        ids[t] = -1;
    }
}

__device__ inline float lse_of(float2 p, float inv_temp) { return p.y > 0.f ? (float)((double)p.x * inv_temp + (double)logf(p.y)) : -INFINITY; }

struct TopArgs {
    const void* in;
    long long stride;
    int V, k, segs, seg_len;
    float inv_temp, c2;  // c2: logit -> base-2 exponent
    float* values;
    int32_t* ids;
    float* lse;          // may be null
    u64* lists;          // [rows][segs][k], several segments only
    float2* parts;       // [rows][segs]
};

template <bool BF16>
__global__ __launch_bounds__(kTopThreads) void top_segment(const TopArgs a) {
    typedef Row<BF16> R;
    constexpr int N = R::N, VEC = kTopPer / N;
    __shared__ TopLds l;
    const int t = threadIdx.x, lane = t & 63, row = blockIdx.y, seg = blockIdx.x;
    const typename R::T* p = (const typename R::T*)a.in + (long long)row * a.stride;
    const int v0 = seg * a.seg_len, v1 = min(a.V, v0 + a.seg_len);
    if (t == 0) l.count = 0, l.least = 0xffffffffu;
    float2 sum = make_float2(kNoEntry, 0.f);
    float from = kNoEntry;   // candidates are not below this: the lowest finite value shuts out -inf (and NaN)
    int n = 0, next_cut = 1;
    for (int b = v0, done = 0; b < v1; b += kTopBlock) {
        float z[kTopPer];
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int v = b + N * (t + kTopThreads * i);
            raw16 r;
            if (v < v1) r = row_load<BF16>(p, v, v1);
#pragma unroll
            for (int x = 0; x < N; ++x) {
                z[i * N + x] = v < v1 ? R::get(r, x) : -INFINITY;
                mx = fmaxf(mx, z[i * N + x]);
            }
        }
        if (a.lse) {
            const float m = fmaxf(sum.x, mx);
            float s = sum.y * fast_exp2((sum.x - m) * a.c2);
#pragma unroll
            for (int i = 0; i < kTopPer; ++i) s += fast_exp2((z[i] - m) * a.c2);
            sum = make_float2(m, s);
        }
        if (b == v0) {   // the k-th largest of the threads' maxima: k entries of this block at least reach it
            l.maxima[t] = mx > -INFINITY ? rank_of(mx) : 0;
            __syncthreads();
            const uint32_t mine = l.maxima[t];
            int above = 0;
#pragma unroll 16
            for (int i = 0; i < kTopThreads; ++i) above += l.maxima[i] > mine;
            if (above < a.k && mine != 0) atomicMin(&l.least, mine);
            __syncthreads();
            int entries = 0;   // where fewer threads than k have an entry at all, the smallest of their maxima is no bound
            for (int i = lane; i < kTopThreads; i += 64) entries += l.maxima[i] != 0;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) entries += __shfl_xor(entries, d);
            if (entries >= a.k) from = value_of(l.least);
        }
        if (mx >= from) {
#pragma unroll
            for (int i = 0; i < kTopPer; ++i)
                if (z[i] >= from) l.list[atomicAdd(&l.count, 1)] = item_of(z[i], b + N * (t + kTopThreads * (i / N)) + i % N);
        }
        __syncthreads();
        n = l.count;
        ++done;
        const bool last = b + kTopBlock >= v1;
        if (n > a.k && (n > kTopLow || done == next_cut || last)) {
            const u64 kth = cut_to(l, n, a.k);
            n = a.k;
            from = value_of((uint32_t)(kth >> 32) + 1u);
        }
        if (done == next_cut) next_cut *= 2;
        __syncthreads();   // the count has been read by all before the next block adds to it
    }
    if (a.lse) {
        const float m = wave_max_dpp(sum.x);
        const float s = wave_sum_dpp(sum.y * fast_exp2((sum.x - m) * a.c2));
        if (lane == 0) l.part[t >> 6] = make_float2(m, s);
        __syncthreads();
        if (t == 0) {
            float2 q = l.part[0];
            for (int i = 1; i < kTopThreads / 64; ++i) q = join_sums(q, l.part[i], a.c2);
            if (a.segs > 1) a.parts[(long long)row * a.segs + seg] = q;
            else a.lse[row] = lse_of(q, a.inv_temp);
        }
    }
    if (a.segs > 1) {
        u64* to = a.lists + ((long long)row * a.segs + seg) * a.k;
        if (t < a.k) to[t] = t < n ? l.list[t] : 0;
    } else {
        put_sorted(l, n, a.k, a.values + (long long)row * a.k, a.ids + (long long)row * a.k);
    }
}

// one workgroup per row: the lists of its segments (their unused places are 0)
__global__ __launch_bounds__(kTopThreads) void top_merge(const TopArgs a) {
    __shared__ TopLds l;
    const int t = threadIdx.x, row = blockIdx.x;
    const u64* from = a.lists + (long long)row * a.segs * a.k;
    if (t == 0) l.count = 0;
    __syncthreads();
    for (int i = t; i < a.segs * a.k; i += kTopThreads) {
        const u64 it = from[i];
        if (it) l.list[atomicAdd(&l.count, 1)] = it;
    }
    __syncthreads();
    int n = l.count;
    __syncthreads();
    if (n > a.k) {
        cut_to(l, n, a.k);
        n = a.k;
    }
    put_sorted(l, n, a.k, a.values + (long long)row * a.k, a.ids + (long long)row * a.k);
    if (a.lse && t == 0) {
        const float2* q = a.parts + (long long)row * a.segs;
        float2 s = q[0];
        for (int i = 1; i < a.segs; ++i) s = join_sums(s, q[i], a.c2);
        a.lse[row] = lse_of(s, a.inv_temp);
    }
}

// Segments of a row: one where the rows alone give the chip two rounds of workgroups, else as many as that takes, each of a block at
// least, and no more lists than one merging workgroup holds
static int top_segs(int n_rows, int vocab, int k) {
    const int blocks = (vocab + kTopBlock - 1) / kTopBlock;
    int segs = (1024 + n_rows - 1) / n_rows;
    if (segs > blocks) segs = blocks;
    if (segs > kTopList / k) segs = kTopList / k;
    const int len = (blocks + segs - 1) / segs;   // of equal length, in blocks
    return (blocks + len - 1) / len;
}

}  // namespace psd

using namespace psd;

extern "C" size_t psd_top_logits_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t k) {
    if (n_rows < 1 || n_rows > kMaxRows || vocab < 1 || vocab > kMaxVocab || k < 1 || k > PSD_MAX_TOP || k > vocab) return 0;
    const int segs = top_segs(n_rows, vocab, k);
    if (segs == 1) return 16;
    return align16((size_t)n_rows * segs * k * sizeof(u64)) + align16((size_t)n_rows * segs * sizeof(float2));
}

extern "C" int psd_top_logits(const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t stride, int32_t k,
                              float temperature, float* values, int32_t* ids, float* lse, void* workspace, size_t workspace_bytes,
                              void* stream) {
    char* err = tls_error();
    const char* who = "psd_top_logits";
    int rc = rows_check(who, logits, dtype, n_rows, vocab, stride, err);
    if (rc != PSD_OK) return rc;
    if (!values || !ids || !workspace) PSD_FAIL(PSD_EINVAL, err, "%s: null pointer", who);
    if (k < 1 || k > PSD_MAX_TOP || k > vocab) PSD_FAIL(PSD_EINVAL, err, "%s: k=%d of %d entries", who, k, vocab);
    if (!(temperature > 0.f)) PSD_FAIL(PSD_EINVAL, err, "%s: temperature=%g", who, temperature);
    if (((uintptr_t)values | (uintptr_t)ids | (uintptr_t)lse) & 3 || ((uintptr_t)workspace & 15))
        PSD_FAIL(PSD_EINVAL, err, "%s: misaligned outputs or workspace", who);
    if (workspace_bytes < psd_top_logits_workspace_bytes(n_rows, vocab, k))
        PSD_FAIL(PSD_ENOMEM, err, "%s: workspace %zu < %zu bytes", who, workspace_bytes, psd_top_logits_workspace_bytes(n_rows, vocab, k));
    const int segs = top_segs(n_rows, vocab, k), blocks = (vocab + kTopBlock - 1) / kTopBlock;
    TopArgs a{logits, stride, vocab, k, segs, (blocks + segs - 1) / segs * kTopBlock, 1.f / temperature, kLog2e / temperature, values, ids, lse, nullptr, nullptr};
    if (segs > 1) {
        a.lists = (u64*)workspace;
        a.parts = (float2*)((char*)workspace + align16((size_t)n_rows * segs * k * sizeof(u64)));
    }
    hipStream_t st = (hipStream_t)stream;
    if (dtype == PSD_BF16) top_segment<true><<<dim3(segs, n_rows), kTopThreads, 0, st>>>(a);
    else top_segment<false><<<dim3(segs, n_rows), kTopThreads, 0, st>>>(a);
    if (segs > 1) top_merge<<<n_rows, kTopThreads, 0, st>>>(a);
    PSD_HIP(hipGetLastError(), err);
    return PSD_OK;
}
