// The k largest entries of every row of logits, with the row's log-sum-exp.
//
// A workgroup streams over a segment of a row, 4096 entries at a time with the next ones on their way, and keeps a list of candidates in LDS:
// entries not below a threshold that at least k entries of the segment are known to reach.  The first threshold is one that k of the threads'
// own maxima in the first block reach.  Entries enter the list as they are; once enough have come they are counted in 256 bins by value, and the lower
// edge of the bin in which the k-th largest lies is the next threshold; a list that grows too long is freed of what lies below it.  So all but a few hundred entries of a
// row cost a maximum, an exponential and their load.  What is left at the end, or where the bins cannot tell values apart, is cut exactly: ranks
// come from comparing all pairs of at most 256 items, before that a longer list is filtered by the threads' maxima and, if that leaves too many, by
// radix selection, 8 bits a round.  Items are 64 bits (order-preserving image of the value, complement of the token) and all differ, so that
// equal values fall in the order of their tokens by themselves.
// Many rows: one segment each, one launch.  Few rows: several segments, whose lists a second launch merges.
// Bound: the bytes of the rows, read once: 6.1 TB/s (64 of 2048 fp32 rows of 128256, 174 us) against 6.6 of a kernel that does nothing else.
// Few rows: two launches that wait for one another (20 of one such row: 6.1 us for 32 segments, 4.4 for their merge), the larger k is the more
// the cuts of many candidates (230 of 49 fp32 rows of 65536: 22 us).  bf16 rows: the maxima, exponentials and comparisons of twice the entries per byte (64 of
// 2048 rows of 128256: 135 us, 3.9 TB/s).  Large k: the first threshold, reached by k of 256 threads' maxima, lets hundreds of entries of a block
// into the list, which is cut often (232 of 1629 bf16 rows of 65536: 103 us, 2.1 TB/s; 256 of 2048 bf16 rows of 128256: 355 us, 1.5 TB/s).
#include "psd_rows.h"

namespace psd {

constexpr int kTopThreads = 256;
constexpr int kTopBlock = 4096;                       // entries between two looks at the list
constexpr int kTopPer = kTopBlock / kTopThreads;      // of one thread: 16
constexpr int kTopLow = 480;                          // a list longer than this is cut before the next block
constexpr int kTopList = kTopLow + kTopBlock;         // so every entry of a block finds a place in it
constexpr int kTopItems = (kTopList + kTopThreads - 1) / kTopThreads;   // 18
static_assert(PSD_MAX_TOP <= kTopThreads && PSD_MAX_TOP <= kTopLow, "a thread, and a place in a cut list, per entry of the result");

typedef unsigned long long u64;

// order-preserving image of a value; equal values (0 and -0 among them) have equal images; 0 is no value's
__device__ inline uint32_t rank_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(uint32_t r) { return __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r); }

struct TopLds {
    union {
        alignas(16) u64 list[kTopList];
        uint2 fresh[kTopList];   // entries that are no items yet: complement of the token, value
    };
    alignas(16) uint32_t bins[256];
    union {   // (barriers lie between the uses of one and of the other)
        uint32_t hist[3][256];   // one is filled, the next cleared, the last may still be read
        alignas(16) uint32_t maxima[kTopThreads];
    };
    float2 part[kTopThreads / 64];
    alignas(16) uint4 least[kTopThreads / 64];
    int count;
};

// over a wave, every lane gets it
template <int CTRL>
__device__ inline uint32_t max_moved(uint32_t v) { return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true)); }
__device__ inline uint32_t wave_max_u32(uint32_t v) {
    v = max_moved<0xB1>(v);    // quad_perm [1,0,3,2]
    v = max_moved<0x4E>(v);    // quad_perm [2,3,0,1]
    v = max_moved<0x141>(v);   // row_half_mirror
    v = max_moved<0x140>(v);   // row_mirror
    {
        const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max(p[0], p[1]);
    }
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(p[0], p[1]);
}

// sum over the lanes up to and including each
template <int CTRL, int ROW_MASK>
__device__ inline int sum_moved(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROW_MASK, 0xf, false); }
__device__ inline int wave_scan(int v) {
    v = sum_moved<0x111, 0xf>(v);   // row_shr:1
    v = sum_moved<0x112, 0xf>(v);   // row_shr:2
    v = sum_moved<0x114, 0xf>(v);   // row_shr:4
    v = sum_moved<0x118, 0xf>(v);   // row_shr:8
    v = sum_moved<0x142, 0xa>(v);   // row_bcast15 into rows 1 and 3
    return sum_moved<0x143, 0xc>(v);   // row_bcast31 into rows 2 and 3
}

// An image that at least k of the threads' maxima reach (0: no entry; 1 where that many have none): in every wave a quarter of k, or half of k in
// two, or all k in one (short and masked rows leave waves without entries).  Every thread counts the larger ones of its own wave.  All threads;
// one barrier.
__device__ inline uint32_t reached_by(TopLds& l, uint32_t mine, int k) {
    const int t = threadIdx.x, w = t >> 6;
    l.maxima[t] = mine;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int above = 0;
#pragma unroll
    for (int i = 0; i < 64; i += 4) {
        const uint4 o = *reinterpret_cast<const uint4*>(&l.maxima[64 * w + i]);
        above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
    }
    uint32_t least[3];   // the wave's ceil(k / 4)-th, ceil(k / 2)-th and k-th largest, 0 where it has too few
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const int share = (k + (4 >> i) - 1) / (4 >> i);
        least[i] = share > 64 ? 0u : ~wave_max_u32(above < share ? ~mine : 0u);   // (a lane without an entry is among them where the wave has too few)
    }
    const uint32_t most = wave_max_u32(mine);
    if ((t & 63) == 0) l.least[w] = make_uint4(least[0], least[1], least[2], most);
    __syncthreads();
    const uint4 q0 = l.least[0], q1 = l.least[1], q2 = l.least[2], q3 = l.least[3];
    const uint32_t quarter = min(min(q0.x, q1.x), min(q2.x, q3.x)), one = max(max(q0.z, q1.z), max(q2.z, q3.z));
    const uint32_t half = max(max(min(q0.y, q1.y), min(q2.y, q3.y)), min(max(q0.y, q1.y), max(q2.y, q3.y)));   // the second largest
    return max(max(quarter, half), max(one, 1u));
}

// Radix selection among the items it[0 .. turns - 1] of all threads, of which more than k are not 0: the smallest of the k largest.  All threads.
__device__ inline u64 kth_item(TopLds& l, const u64 (&it)[kTopItems], int turns, int k) {
    const int t = threadIdx.x, lane = t & 63;
    l.hist[0][t] = 0;
    __syncthreads();
    u64 least = 0;
    int need = k;
    for (int shift = 56, turn = 0; shift >= 0; shift -= 8, turn = turn == 2 ? 0 : turn + 1) {
        l.hist[turn == 2 ? 0 : turn + 1][t] = 0;
        const u64 above = shift == 56 ? 0 : ~0ull << (shift + 8);
#pragma unroll
        for (int i = 0; i < kTopItems; ++i)
            if (i < turns && it[i] != 0 && (it[i] & above) == least) atomicAdd(&l.hist[turn][(uint32_t)(it[i] >> shift) & 255], 1u);
        __syncthreads();
        // every wave: lane x has bins 255 - 4x .. 252 - 4x; a scan over the lanes finds the bin in which the need-th largest lies
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = l.hist[turn][255 - 4 * lane - i];
        uint32_t sum = h[0] + h[1] + h[2] + h[3];
        const uint32_t upto = (uint32_t)wave_scan((int)sum);
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
    return least;
}

// Keeps the items of it[0 .. turns - 1] that are not below `least` in the list, in any order; their number.  All threads, after a barrier behind the last
// use of the list; two barriers.
__device__ inline int keep_from(TopLds& l, const u64 (&it)[kTopItems], int turns, u64 least) {
    if (threadIdx.x == 0) l.count = 0;
    __syncthreads();
    int keeps = 0;
#pragma unroll
    for (int i = 0; i < kTopItems; ++i)
        if (i < turns) keeps += it[i] != 0 && it[i] >= least;
    const int upto = wave_scan(keeps);
    int at = 0;
    if ((threadIdx.x & 63) == 63) at = atomicAdd(&l.count, upto);
    at = __builtin_amdgcn_readlane(at, 63) + upto - keeps;
#pragma unroll
    for (int i = 0; i < kTopItems; ++i)
        if (i < turns && it[i] != 0 && it[i] >= least) l.list[at++] = it[i];
    __syncthreads();
    return l.count;
}

// The bin in which the k-th largest of the counted entries lies.  Every wave for itself: lane x has bins 255 - 4x .. 252 - 4x.
__device__ inline int kth_bin(const TopLds& l, int k) {
    const int lane = threadIdx.x & 63;
    const uint4 q = *reinterpret_cast<const uint4*>(&l.bins[252 - 4 * lane]);
    const uint32_t h[4] = {q.w, q.z, q.y, q.x};
    const uint32_t sum = (h[0] + h[1]) + (h[2] + h[3]);
    const uint32_t upto = (uint32_t)wave_scan((int)sum);
    const uint64_t enough = __ballot(upto >= (uint32_t)k);
    if (enough == 0) return 0;
    uint32_t before = upto - sum;
    int bin = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (before < (uint32_t)k && before + h[i] >= (uint32_t)k) bin = 255 - 4 * lane - i;
        before += h[i];
    }
    return __shfl(bin, __builtin_ctzll(enough));
}

// The item of lane t ^ S of the wave
template <int S>
__device__ inline uint32_t from_lane(uint32_t v) {
    if constexpr (S == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true);   // quad_perm [1,0,3,2]
    if constexpr (S == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true);   // quad_perm [2,3,0,1]
    if constexpr (S == 4) return (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x101F);                    // xor 4
    if constexpr (S == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true);  // row_ror:8
    if constexpr (S == 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return threadIdx.x & 16 ? p[0] : p[1];
    }
    if constexpr (S == 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? p[0] : p[1];
    }
}
// one step of a bitonic network over a workgroup's items, descending in the end; strides of 64 and more go through the list
template <int SIZE, int STRIDE>
__device__ inline void bitonic_step(TopLds& l, u64& it) {
    const int t = threadIdx.x;
    u64 other;
    if constexpr (STRIDE >= 64) {
        __syncthreads();
        l.list[t] = it;
        __syncthreads();
        other = l.list[t ^ STRIDE];
    } else {
        other = (u64)from_lane<STRIDE>((uint32_t)(it >> 32)) << 32 | from_lane<STRIDE>((uint32_t)it);
    }
    const bool larger = ((t & STRIDE) == 0) == ((t & SIZE) == 0);
    it = (other > it) == larger ? other : it;
    if constexpr (STRIDE > 1) bitonic_step<SIZE, STRIDE / 2>(l, it);
}
template <int SIZE>
__device__ inline void bitonic_sort(TopLds& l, u64& it) {
    if constexpr (SIZE > 2) bitonic_sort<SIZE / 2>(l, it);
    bitonic_step<SIZE, SIZE / 2>(l, it);
}

// Brings the list's n <= 256 items into descending order and drops those behind the k-th; how many are left.  All threads.  A few items by
// counting the larger ones of each (7 n instructions a wave that has some), more by a bitonic network (about 400) where NET: its straight run pays
// once many workgroups have brought it into the instruction cache (a launch of one workgroup with 240 items: 8 us counting, 15.5 us)
template <bool NET>
__device__ inline int sort_list(TopLds& l, int n, int k) {
    const int t = threadIdx.x;
    u64 mine = t < n ? l.list[t] : 0;
    int at = t;
    if (!NET || n <= 64) {
        if (t >= n && t < ((n + 15) & ~15)) l.list[t] = 0;   // sixteen at a time: their reads need not wait for each other
        __syncthreads();
        if ((t & ~63) < n) {   // waves that have items
            at = 0;
#pragma unroll 1
            for (int i = 0; i < n; i += 16) {
                ulonglong2 o[8];
#pragma unroll
                for (int y = 0; y < 8; ++y) o[y] = *reinterpret_cast<const ulonglong2*>(&l.list[i + 2 * y]);
#pragma unroll
                for (int y = 0; y < 8; ++y) at += (o[y].x > mine) + (o[y].y > mine);
            }
        }
    } else if constexpr (NET) {
        bitonic_sort<256>(l, mine);
    }
    __syncthreads();
    if (t < n && at < k) l.list[at] = mine;
    if (t == 0) l.count = min(n, k);
    __syncthreads();
    return min(n, k);
}

// The list's n items into registers, 0 behind them; how many a thread has (the same for all)
__device__ inline int load_list(const TopLds& l, u64 (&it)[kTopItems], int t, int n) {
    const int turns = (n + kTopThreads - 1) / kTopThreads;
#pragma unroll
    for (int i = 0; i < kTopItems; ++i)
        if (i < turns) it[i] = t + kTopThreads * i < n ? l.list[t + kTopThreads * i] : 0;
    return turns;
}

// Frees a list of n <= kTopList items of those whose image is below `least`; how many are left.  All threads, n uniform, after a barrier.
__device__ inline int thin_list(TopLds& l, int n, uint32_t least) {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));   // else the caller's loop keeps every place's index in a register
    u64 it[kTopItems];
    const int turns = load_list(l, it, t, n);
    __syncthreads();
    return keep_from(l, it, turns, (u64)least << 32);
}

// The lower edge of bin `bin`, or a few units in the last place less: no entry counted in it may lie below
__device__ inline float edge_of(float base, float scale, int bin) {
    const float edge = base + (float)bin / scale;
    return edge - 1e-6f * (fabsf(edge) + fabsf(base));
}
__device__ inline int bin_of(float z, float base, float scale) { return min((int)((z - base) * scale), 255); }   // z >= base
__device__ inline float bin_scale(const TopLds& l, float base) {   // after reached_by: 256 bins up to the largest, 0 where there is nothing to tell apart
    const float width = value_of(max(max(l.least[0].w, l.least[1].w), max(l.least[2].w, l.least[3].w))) - base;
    return width > 1e-30f ? 255.f / width : 0.f;
}

// Puts the k largest of the items it[0 .. turns - 1] into the list, in descending order; how many there are.  All threads, after a barrier behind the last use of
// the list and the bins.
template <bool NET>
__device__ inline int cut_items(TopLds& l, const u64 (&it)[kTopItems], int turns, int k) {
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < kTopItems; ++i)
        if (i < turns) mx = max(mx, (uint32_t)(it[i] >> 32));
    const uint32_t bound = reached_by(l, mx, k);
    l.bins[threadIdx.x] = 0;
    int n = keep_from(l, it, turns, (u64)bound << 32);
    const float base = value_of(bound), scale = bound > 1 ? bin_scale(l, base) : 0.f;
    if (n > kTopThreads && scale > 0.f) {
#pragma unroll
        for (int i = 0; i < kTopItems; ++i)
            if (i < turns && (uint32_t)(it[i] >> 32) >= bound) atomicAdd(&l.bins[bin_of(value_of((uint32_t)(it[i] >> 32)), base, scale)], 1u);
        __syncthreads();
        n = keep_from(l, it, turns, (u64)max(bound, rank_of(edge_of(base, scale, kth_bin(l, k)))) << 32);
    }
    if (n > kTopThreads) {
        __syncthreads();   // the count has been read
        n = keep_from(l, it, turns, kth_item(l, it, turns, k));
    }
    return sort_list<NET>(l, n, k);
}

// Cuts a list of n <= kTopList items in the same way.  All threads, n uniform, after a barrier; spoils the bins.
template <bool NET>
__device__ inline int cut_list(TopLds& l, int n, int k) {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));   // as in thin_list
    if (n <= kTopThreads) return sort_list<NET>(l, n, k);
    u64 it[kTopItems];
    return cut_items<NET>(l, it, load_list(l, it, t, n), k);
}

// The list, sorted, into one row of the outputs
__device__ inline void put_list(const TopLds& l, int n, int k, float* values, int32_t* ids) {
    const int t = threadIdx.x;
    if (t >= k) return;
    const u64 it = t < n ? l.list[t] : 0;
    values[t] = t < n ? value_of((uint32_t)(it >> 32)) : -INFINITY;
    ids[t] = t < n ? (int32_t)~(uint32_t)it : -1;
}

__device__ inline float lse_of(float2 p, double inv_temp) { return p.y > 0.f ? (float)((double)p.x * inv_temp + (double)logf(p.y)) : -INFINITY; }

struct TopArgs {
    const void* in;
    long long stride;
    int V, k, segs, seg_len, slots;   // slots: places for the candidates of a segment, k or more
    double inv_temp;
    float c2;            // logit -> base-2 exponent
    float* values;
    int32_t* ids;
    float* lse;          // may be null
    u64* lists;          // [rows][segs][slots], several segments only
    float2* parts;       // [rows][segs]
};

template <bool BF16>
__global__ __launch_bounds__(kTopThreads, 4) void top_segment(const TopArgs a) {
    typedef Row<BF16> R;
    constexpr int N = R::N, VEC = kTopPer / N;
    __shared__ TopLds l;
    const int t = threadIdx.x, lane = t & 63, row = blockIdx.y, seg = blockIdx.x;
    const typename R::T* p = (const typename R::T*)a.in + (long long)row * a.stride;
    const int v0 = seg * a.seg_len, v1 = min(a.V, v0 + a.seg_len);
    if (t == 0) l.count = 0;
    l.bins[t] = 0;
    const raw16 none = none16<BF16>();
    auto load = [&](int b, raw16 (&r)[VEC]) {
        if (b + kTopBlock <= v1) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) r[i] = (raw16)__builtin_nontemporal_load((const typename R::V*)(p + b + N * (t + kTopThreads * i)));
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int v = b + N * (t + kTopThreads * i);
                r[i] = v < v1 ? row_load<BF16>(p, v, v1) : none;
            }
        }
    };
    float2 sum = make_float2(kNoEntry, 0.f);
    float from = kNoEntry;   // candidates are not below this: the lowest finite value shuts out -inf (and NaN)
    uint32_t least = 0;      // an image that k of the list's items reach, if it has so many (an exact cut leaves it below `from`)
    float base = kNoEntry, scale = 0.f;   // bins: (z - base) scale
    int n = 0, n_known = 0, n_items = 0, done = 0;   // n_items: those of the list that are items, not yet values and tokens
    // One block, then the load of the one after the next into the same registers: moving a block over would wait for it.  True: the last one.
    auto step = [&](raw16 (&r)[VEC]) {
        const int b = v0 + done * kTopBlock;
        const bool last = b + kTopBlock >= v1;
        ++done;
        float vm[VEC], mx = kNoEntry;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            vm[i] = vec_max<BF16>(r[i], kNoEntry);
            mx = fmaxf(mx, vm[i]);
        }
        if (a.lse) {
            const float m = fmaxf(sum.x, mx);
            float s = sum.y * fast_exp2((sum.x - m) * a.c2);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s = vec_sum<BF16>(r[i], m, a.c2, s);
            sum = make_float2(m, s);
        }
        if (done == 1) {
            // a thread without an entry above the lowest value counts as one without an entry: the bound only has to be reached by k others
            const uint32_t bound = reached_by(l, mx > kNoEntry ? rank_of(mx) : 0, a.k);
            if (bound > 1) {
                base = from = value_of(bound);
                least = bound;
                scale = bin_scale(l, base);
            }
        }
        if (__ballot(mx >= from)) {   // a wave takes its places in the list at once; which lanes bring an entry is a mask per element
            uint64_t in[VEC * N];
            int brings = 0;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    in[i * N + x] = __ballot(R::get(r[i], x) >= from);
                    brings += __popcll(in[i * N + x]);
                }
            int at = 0;
            if (lane == 0) at = atomicAdd(&l.count, brings);
            at = __builtin_amdgcn_readfirstlane(at);
            uint32_t first = ~(uint32_t)(b + N * t);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                asm volatile("" : "+v"(first));   // one vector's tokens at a time are registers enough
#pragma unroll
                for (int x = 0; x < N; ++x) {
                    const uint64_t who = in[i * N + x];
                    const float z = R::get(r[i], x);
                    if (z >= from) {
                        const uint32_t place = __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, at));
                        l.fresh[place].y = __float_as_uint(z);
                        __builtin_amdgcn_wave_barrier();   // two stores, or the row's registers would have to be halves of pairs
                        l.fresh[place].x = first - (uint32_t)(N * kTopThreads * i + x);
                    }
                    at += __popcll(who);
                }
            }
        }
        if (b + 2 * kTopBlock < v1) load(b + 2 * kTopBlock, r);
        __syncthreads();
        n = l.count;
        if (last || n > kTopLow || (n >= a.k && n >= n_known + 32)) {
            // the values that came since become items: here a thread has one each, above a whole wave goes through every element of it
            for (int i = n_items + t; i < n; i += kTopThreads) {
                const uint2 q = l.fresh[i];
                const float z = __uint_as_float(q.y);
                l.list[i] = (u64)rank_of(z) << 32 | q.x;
                if (scale > 0.f) atomicAdd(&l.bins[bin_of(z, base, scale)], 1u);
            }
            n_items = n;
            __syncthreads();
        }
        if (scale > 0.f && n >= a.k && (last ? n > kTopThreads : n >= n_known + 32)) {
            const float edge = edge_of(base, scale, kth_bin(l, a.k));
            from = fmaxf(from, edge);
            least = max(least, rank_of(edge));
            n_known = n;
        }
        if (last || n > kTopLow) {
            if (n > kTopThreads) n = n_known = thin_list(l, n, least);
            if (n > kTopThreads || (last && n > a.slots)) {
                __syncthreads();   // the count has been read
                if (n > kTopThreads) scale = 0.f;   // bins that cannot tell values apart have done their part
                n = n_known = cut_list<true>(l, n, a.k);
                if (n == a.k) {
                    least = (uint32_t)(l.list[a.k - 1] >> 32);
                    from = value_of(least + 1u);
                }
            }
            n_items = n;
        }
        __syncthreads();   // the count has been read by all before the next block adds to it
        return last;
    };
    raw16 even[VEC], odd[VEC];
    load(v0, even);
    if (v0 + kTopBlock < v1) load(v0 + kTopBlock, odd);
    while (!step(even) && !step(odd)) {}
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
        u64* to = a.lists + ((long long)row * a.segs + seg) * a.slots;
        if (t < a.slots) to[t] = t < n ? l.list[t] : 0;
    } else {
        put_list(l, n, a.k, a.values + (long long)row * a.k, a.ids + (long long)row * a.k);
    }
}

// one workgroup per row: the lists of its segments (their unused places are 0)
__global__ __launch_bounds__(kTopThreads) void top_merge(const TopArgs a) {
    __shared__ TopLds l;
    const int t = threadIdx.x, lane = t & 63, row = blockIdx.x, all = a.segs * a.slots;
    const u64* from = a.lists + (long long)row * all;
    // a run of places for every thread: the unused ones lie at the ends of the lists, and a thread that has none but them has no maximum
    const int per = (all + kTopThreads - 1) / kTopThreads;
    u64 it[kTopItems];
#pragma unroll
    for (int i = 0; i < kTopItems; ++i)
        if (i < per) it[i] = per * t + i < all ? from[per * t + i] : 0;
    float2 q = make_float2(kNoEntry, 0.f);
    if (a.lse && t < 64)
        for (int i = lane; i < a.segs; i += 64) q = join_sums(q, a.parts[(long long)row * a.segs + i], a.c2);
    const int n = cut_items<false>(l, it, per, a.k);
    put_list(l, n, a.k, a.values + (long long)row * a.k, a.ids + (long long)row * a.k);
    if (a.lse && t < 64) {
        const float m = wave_max_dpp(q.x);
        const float s = wave_sum_dpp(q.y * fast_exp2((q.x - m) * a.c2));
        if (t == 0) a.lse[row] = lse_of(make_float2(m, s), a.inv_temp);
    }
}

// Segments of a row: as many as make the call shortest, counted in blocks that pass one after the other.  1024 workgroups are on the chip at
// once; a workgroup's start and its last cut take as long as one and a half blocks, the merging launch as long as three (us by segments, fp32 rows
// of 128256: 1 row 1 / 4 / 16 / 32 segments 37.2 / 21.4 / 13.1 / 10.3; 300 rows 1 / 2 / 3 / 4: 55.8 / 44.1 / 40.7 / 47.3; 900 rows 1 / 2: 83.8 / 90.0).
static int top_slots(int k) { return k + k / 4 + 32 < kTopThreads ? k + k / 4 + 32 : kTopThreads; }   // what the first threshold lets in, usually
static int top_segs(int n_rows, int vocab, int k) {
    const int blocks = (vocab + kTopBlock - 1) / kTopBlock;
    int best = 1;
    double least = 1e30;
    for (int segs = 1; segs <= blocks && segs <= kTopList / top_slots(k) && segs <= 64; ++segs) {
        const int len = (blocks + segs - 1) / segs;
        if ((blocks + len - 1) / len != segs) continue;   // the same as fewer
        const double rounds = (double)(((long long)n_rows * segs + 1023) / 1024);
        const double cost = rounds * (len + 1.5) + (segs > 1 ? 3.0 : 0.0);
        if (cost < least) least = cost, best = segs;
    }
    return best;
}

}  // namespace psd

using namespace psd;

extern "C" size_t psd_top_logits_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t k) {
    if (n_rows < 1 || n_rows > kMaxRows || vocab < 1 || vocab > kMaxVocab || k < 1 || k > PSD_MAX_TOP || k > vocab) return 0;
    const int segs = top_segs(n_rows, vocab, k);
    if (segs == 1) return 16;
    return align16((size_t)n_rows * segs * top_slots(k) * sizeof(u64)) + align16((size_t)n_rows * segs * sizeof(float2));
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
    if (!temperature_fits(temperature)) PSD_FAIL(PSD_EINVAL, err, "%s: temperature=%g", who, temperature);
    if (((uintptr_t)values | (uintptr_t)ids | (uintptr_t)lse) & 3 || ((uintptr_t)workspace & 15))
        PSD_FAIL(PSD_EINVAL, err, "%s: misaligned outputs or workspace", who);
    if (workspace_bytes < psd_top_logits_workspace_bytes(n_rows, vocab, k))
        PSD_FAIL(PSD_ENOMEM, err, "%s: workspace %zu < %zu bytes", who, workspace_bytes, psd_top_logits_workspace_bytes(n_rows, vocab, k));
    const int segs = top_segs(n_rows, vocab, k), blocks = (vocab + kTopBlock - 1) / kTopBlock;
    TopArgs a{logits, stride, vocab, k, segs, (blocks + segs - 1) / segs * kTopBlock, segs > 1 ? top_slots(k) : 0, 1.0 / (double)temperature, kLog2e / temperature, values, ids, lse, nullptr, nullptr};
    if (segs > 1) {
        a.lists = (u64*)workspace;
        a.parts = (float2*)((char*)workspace + align16((size_t)n_rows * segs * top_slots(k) * sizeof(u64)));
    }
    hipStream_t st = (hipStream_t)stream;
    if (dtype == PSD_BF16) top_segment<true><<<dim3(segs, n_rows), kTopThreads, 0, st>>>(a);
    else top_segment<false><<<dim3(segs, n_rows), kTopThreads, 0, st>>>(a);
    if (segs > 1) top_merge<<<n_rows, kTopThreads, 0, st>>>(a);
    PSD_HIP(hipGetLastError(), err);
    return PSD_OK;
}
