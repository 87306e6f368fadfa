// Distillation from a teacher's top logits: the divergence between the record's K + 1 outcomes (its tokens, and all others together)
// and a student's row, and the gradient.
//
// Per row the student is needed as: its logits at the record's tokens, and the log-sum-exp of all other entries (its own maximum,
// so that it neither cancels against the record's mass nor underflows beside it).  From these the divergence and the gradient's K + 1
// coefficients follow: with g_b = q_b (dl/dq_b - sum_b q_b dl/dq_b) the gradient is g_i / T at a record's token and
// g_rest / T times softmax over the others at every other entry.  For KL g_b = q_b sum p - p_b, and the loss is a sum that needs
// nothing of the row but its two log-sum-exps once the record and its logits are known.
//   distill_pass   one workgroup per row, which passes by for the sums and once more, out of the caches, for the gradient
//   distill_row    one workgroup per row, which stays in registers and LDS between the two: read from memory once
//   distill_tail, distill_grad  (row, chunk): the sums of every chunk; then every chunk joins them, works out the coefficients and
//                  writes its part of the gradient (the logits read again)
// Bound: the rows' bytes, read once and written once: 5.0 TB/s (1024 rows of 128256 fp32 entries, 212 us) and 5.3 TB/s (4096 bf16 rows, a quarter of
// them padding, 348 us) against 4.7 of a large copy.  The loss alone of 777 bf16 rows of 50257 takes 22.7 us, 3.1 TB/s: an exponential and five
// more instructions per entry take about as long as the reads, and three workgroups a unit do not hide one behind the other altogether (two groups
// of vectors on their way, in registers that take turns: 25.2 us).
// The sums of the student's exponentials are fp32 (no entry passes through more than V / 256 + 96 additions), and so are
// its scaled differences, the record's p and the shares of JSD; the record's sums, the two log-sum-exps' logarithms, the losses and the coefficients are
// 64 bits.  Against 64 bits throughout: 1.5e-7 of the outputs' size, fp32, for the cases of perf/operators.py.
#include "psd_rows.h"

namespace psd {

constexpr int kPlaces = PSD_MAX_TOP;   // a thread of a workgroup's first four waves per place of the record
constexpr int kPlaceWaves = kPlaces / 64;
constexpr int kDisThreads = 256;
constexpr int kDisChunk = 8192;
constexpr int kDisPer = kDisChunk / kDisThreads;   // entries of a thread: 32
static_assert(kPlaces == 256 && kDisThreads >= kPlaces, "a thread per place of a record");
constexpr double kLn2d = 0.6931471805599453;

struct DistillArgs {
    const void* in;
    void* grad;
    long long stride, grad_stride;
    int V, k, chunks;
    float c2;                 // logit -> base-2 exponent
    double inv_temp;
    int divergence;
    const float* values;
    const int32_t* ids;
    const float* lse;
    const float* weights;
    float* loss;
    float2* parts;            // [rows][chunks]
    float* student;           // [rows][k]: the student's logits at the record's tokens
};

// What the workgroup keeps of a record: a thread of the first four waves ("place threads") has a place
struct PlaceLds {
    int2 list[kPlaces + 8];              // (token, place) of places that share 16 bytes of the row (or look as if), then kNowhere
    int n_list, n_found;
    float es[kPlaces];                   // student: 2^((z - z_max) c2), 0 where the place does not count
    float p[kPlaces];                    // teacher: probability times p_sum
    float z_max[kPlaceWaves], t_max[kPlaceWaves];
    int valid[kPlaceWaves], open[kPlaceWaves];
    double sums[5][kPlaceWaves];
    float lse;                           // of the teacher's row, 0 where the record is all of it
    float rest, rest_max;                // the others' gradient is rest * 2^((z - rest_max) c2)
    float2 tail;
};

// flags of a place: it counts (a token of the vocabulary that stands in no earlier place); no earlier place has a token of the same 16
// bytes of the row; which elements of those 16 bytes stand in the record
constexpr uint32_t kHere = 0x80000000u, kOwner = 0x40000000u;

// sums over a wave in a fixed order, in 64 bits; all lanes get it
template <int CTRL, int ROW_MASK, bool BOUND>
__device__ inline double dpp_move(double v) {
    const long long b = __double_as_longlong(v);
    const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROW_MASK, 0xf, BOUND), hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROW_MASK, 0xf, BOUND);
    return __longlong_as_double((long long)hi << 32 | (uint32_t)lo);
}
__device__ inline double wave_sum(double v) {
    v += dpp_move<0xB1, 0xf, true>(v);
    v += dpp_move<0x4E, 0xf, true>(v);
    v += dpp_move<0x141, 0xf, true>(v);
    v += dpp_move<0x140, 0xf, true>(v);
    v += dpp_move<0x142, 0xa, false>(v);
    v += dpp_move<0x143, 0xc, false>(v);
    const long long b = __double_as_longlong(v);
    const int lo = __builtin_amdgcn_readlane((int)b, 63), hi = __builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __longlong_as_double((long long)hi << 32 | (uint32_t)lo);
}
__device__ inline double sum_of(const double (&s)[kPlaceWaves]) { return (s[0] + s[1]) + (s[2] + s[3]); }
__device__ inline float max_of(const float (&s)[kPlaceWaves]) { return fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])); }
__device__ inline int sum_of(const int (&s)[kPlaceWaves]) { return (s[0] + s[1]) + (s[2] + s[3]); }
__device__ inline double x_times(double x, double y) { return x > 0.0 ? x * y : 0.0; }   // 0 ln 0 = 0

// e^x of a 64-bit x on the hardware's exponential: the argument as a rounded float and the rest.  0 where it is below 2^-126.
__device__ inline float exp_of(double x) {
    const double y = x * 1.4426950408889634;
    const float hi = (float)y;
    return y >= -126.0 ? fast_exp2(hi) * fmaf((float)(y - (double)hi), kLn2, 1.f) : 0.f;
}

// ln(2 x / (x + y)).  Near x = y by the odd series of 2 artanh(u) = ln((1 + u) / (1 - u)), u = (x - y) / (3 x + y), which loses nothing there
// (|u| < 1/3: nine terms are 2^-26 exact), else by the quotient.
__device__ inline double log_share(float x, float y) {
    const float s = x + y, u = (x - y) / fmaf(3.f, x, y);
    if (!(fabsf(u) < 0.33f)) return (double)(fast_log2(fmaxf(2.f * x / s, 1.2e-38f)) * kLn2);   // (a denormal quotient is none to the hardware)
    const float w = u * u;
    float c = 1.f / 17.f;
#pragma unroll
    for (int n = 15; n >= 1; n -= 2) c = fmaf(c, w, 1.f / (float)n);
    return (double)(2.f * u * c);
}

// Which places count.  A place enters a bit for its 16 bytes of the row into a table (`bit` in `word`, 0: it has no token) and learns
// whether another was there before; those that find one stand in a list, and so, a barrier later, does the place whose bit they found.  Only the
// list is searched, so that the usual row, whose tokens lie far apart, costs one atomic per place.  The outcome does not depend on who came first.
// Tokens of the same 16 bytes differ in the bits below N only; places that merely share a bit of the table drop out by their tokens.
constexpr int kNowhere = 1 << 30;   // differs from every token by more than N
// all threads, before a barrier
__device__ inline void place_clear(PlaceLds& l) {
    const int t = threadIdx.x;
    if (t < kPlaces) l.list[t] = make_int2(kNowhere, kPlaces);
    if (t < 8) l.list[kPlaces + t] = make_int2(kNowhere, kPlaces);
    if (t == 0) l.n_list = l.n_found = 0;
}
template <typename W>
__device__ inline bool place_enter(PlaceLds& l, int id, W* word, W bit) {
    if (!bit || !(atomicOr(word, bit) & bit)) return false;
    l.list[atomicAdd(&l.n_list, 1)] = make_int2(id, (int)threadIdx.x);
    return true;
}
// all threads, after a barrier; entered: in a place thread with a token, listed: place_enter's answer.  The flags of this place.
template <int N>
__device__ inline uint32_t place_flags(PlaceLds& l, int id, bool entered, bool listed) {
    const int t = threadIdx.x, n = l.n_list;
    uint32_t flags = entered ? kHere | kOwner | 1u << (id & (N - 1)) : 0u;
    if (n == 0) return flags;
    bool meets = false;
    if (entered && !listed)
        for (int i = 0; i < n; i += 8) {   // eight at a time: their reads need not wait for each other
            int o[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) o[y] = l.list[i + y].x;
#pragma unroll
            for (int y = 0; y < 8; ++y) meets |= ((uint32_t)o[y] ^ (uint32_t)id) < (uint32_t)N;
        }
    __syncthreads();   // nobody looks for the list's end any more
    if (meets) l.list[n + atomicAdd(&l.n_found, 1)] = make_int2(id, t);
    __syncthreads();
    if (listed || meets) {
        const int all = n + l.n_found;
        for (int i = 0; i < all; i += 8) {
            int2 o[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) o[y] = l.list[i + y];
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                const uint32_t x = (uint32_t)o[y].x ^ (uint32_t)id;
                flags |= x < (uint32_t)N ? 1u << (((uint32_t)id ^ x) & (N - 1)) : 0u;
                flags &= x < (uint32_t)N && o[y].y < t ? (x == 0 ? ~(kHere | kOwner) : ~kOwner) : ~0u;
            }
        }
    }
    return flags & kHere ? flags : 0u;
}

// The same for small vocabularies, where many places share bytes, from the first place of every token (kPlaces: none).
constexpr int kSmallVocab = 4096;
template <int N>
__device__ inline uint32_t place_flags_small(const int* first, int V, int id, bool entered) {
    if (!entered) return 0;
    const int t = threadIdx.x, v0 = id & ~(N - 1);
    uint32_t flags = first[id] == t ? kHere | kOwner : 0u;
#pragma unroll
    for (int x = 0; x < N; ++x) {
        const int f = v0 + x < V ? first[v0 + x] : kPlaces;
        if (f < kPlaces) flags |= 1u << x;
        if (f < t) flags &= ~kOwner;
    }
    return flags & kHere ? flags : 0u;
}

// their maxima and counts; z: the student's logit at the place's token
__device__ inline void place_first(const DistillArgs& a, PlaceLds& l, int id, uint32_t flags, float z, float value) {
    const int t = threadIdx.x, w = t >> 6;
    const float zm = wave_max_dpp(flags & kHere ? fmaxf(z, kNoEntry) : kNoEntry), tm = wave_max_dpp(flags & kHere ? fmaxf(value, kNoEntry) : kNoEntry);
    const int n = __popcll(__ballot((flags & kHere) != 0)), open = __popcll(__ballot(t < a.k && id < 0));
    if ((t & 63) == 0) l.z_max[w] = zm, l.t_max[w] = tm, l.valid[w] = n, l.open[w] = open;
}

// a barrier later: probabilities, and the sums of the student's, the teacher's, and the teacher's times ln p - ln q (but for what all ln p
// and all ln q have in common)
__device__ inline void place_second(const DistillArgs& a, PlaceLds& l, uint32_t flags, float z, float value, int row) {
    const int t = threadIdx.x, w = t >> 6;
    const float x = (z - max_of(l.z_max)) * a.c2;
    const float es = flags & kHere ? fast_exp2(x) : 0.f;
    const double lp = a.lse ? (double)value * a.inv_temp - (double)a.lse[row] : ((double)value - (double)max_of(l.t_max)) * a.inv_temp;
    const float p = flags & kHere ? exp_of(lp) : 0.f;
    if (t == 0) l.lse = a.lse ? a.lse[row] : 0.f;
    l.es[t] = es;
    l.p[t] = p;
    const double d = wave_sum(x_times(p, lp - (double)x * kLn2d));
    if ((t & 63) == 0) l.sums[2][w] = d;
    const double sp = wave_sum((double)p);
    if ((t & 63) == 0) l.sums[1][w] = sp;
    const double se = wave_sum((double)es);
    if ((t & 63) == 0) l.sums[0][w] = se;
}

// What follows from the sums once those of the other entries are known too; place i has q = es[i] * q_place and p = p[i] * p_place
struct RowSums {
    double total, q_place, q_rest, p_place, mass, p_rest;   // mass: sum of the places' p
    double scale;
    bool none;           // the student's row or the record is no distribution at all
    float z_shift;       // (z_max - m) c2 and (tail's maximum - m) c2 in base 2, m the larger of the two
    float tail_shift;
};
__device__ inline RowSums row_sums(const DistillArgs& a, const PlaceLds& l, float2 tail, float weight) {
    RowSums r;
    const float zm = max_of(l.z_max), m = fmaxf(zm, tail.x);
    r.z_shift = (zm - m) * a.c2;
    r.tail_shift = (tail.x - m) * a.c2;
    const double place = (double)fast_exp2(r.z_shift), others = (double)tail.y * fast_exp2(r.tail_shift);
    r.total = fma(sum_of(l.sums[0]), place, others);
    r.q_place = place / r.total;
    r.q_rest = others / r.total;
    const double s = sum_of(l.sums[1]);
    r.p_place = a.lse ? 1.0 : 1.0 / s;
    r.mass = a.lse ? s : 1.0;
    // A negative token: the teacher has no entries beside those of its record.  A record that just holds them all has none, and then 1 - s is
    // what the roundings leave (lse is a float, off by 2^-24 of itself, its logarithm and the p by a few 2^-24 more): a student without mass
    // beside them is not held to it, for whether a mask closes its entries by -inf or by a large negative number, that would cost it a remainder
    // of nothing times the logarithm of nothing.
    const bool noise = (tail.y == 0.f || r.tail_shift < -126.f) && 1.0 - s <= (2.0 + fabs((double)l.lse)) * 0x1p-22;
    r.p_rest = a.lse && sum_of(l.open) == 0 && sum_of(l.valid) < a.V && s < 1.0 && !noise ? 1.0 - s : 0.0;
    r.scale = (double)weight * a.inv_temp;
    r.none = !(r.total > 0.0) || !(a.lse || s > 0.0);
    return r;
}

// place threads: this place's part of the Jensen-Shannon sums
__device__ inline void jsd_sums(PlaceLds& l, const RowSums& r) {
    const int t = threadIdx.x, w = t >> 6;
    const float p = (float)(l.p[t] * r.p_place), q = (float)(l.es[t] * r.q_place);
    const double kq = x_times(q, log_share(q, p)), of_q = wave_sum(kq), both = wave_sum(x_times(p, log_share(p, q)) + kq);
    if ((t & 63) == 0) l.sums[3][w] = both, l.sums[4][w] = of_q;
}

// Place threads (a barrier after jsd_sums where that is the divergence): the gradient at this place's token; thread 0 leaves what the other
// entries and the loss need
__device__ inline float place_gradient(const DistillArgs& a, PlaceLds& l, const RowSums& r, float2 tail) {
    const int t = threadIdx.x;
    const double p = l.p[t] * r.p_place, q = l.es[t] * r.q_place;
    double g, g_rest;
    if (a.divergence == PSD_DIV_KL) {
        const double P = r.mass + r.p_rest;
        g_rest = fma(r.q_rest, P, -r.p_rest);
        g = fma(q, P, -p);
    } else {
        const float qr = (float)r.q_rest;
        const double kqr = x_times(qr, log_share(qr, (float)r.p_rest)), W = sum_of(l.sums[4]) + kqr;
        g_rest = 0.5 * fma(-r.q_rest, W, kqr);
        g = 0.5 * fma(-q, W, x_times((float)q, log_share((float)q, (float)p)));
    }
    if (t == 0) {
        l.rest = r.none ? NAN : tail.y > 0.f ? (float)(g_rest * r.scale / tail.y) : 0.f;
        l.rest_max = tail.x;
        l.tail = tail;
    }
    return r.none ? NAN : (float)(g * r.scale);
}

// one thread, after place_gradient
__device__ inline float row_loss(const DistillArgs& a, const PlaceLds& l, float weight) {
    const float2 tail = l.tail;
    const RowSums r = row_sums(a, l, tail, weight);
    double loss;
    if (a.divergence == PSD_DIV_KL) {
        const double log_total = log(r.total), lq_rest = (double)r.tail_shift * kLn2d + (double)logf(tail.y) - log_total;
        const double d = sum_of(l.sums[2]) * r.p_place + (a.lse ? 0.0 : log(r.p_place));
        loss = d - x_times(r.mass, (double)r.z_shift * kLn2d - log_total) + x_times(r.p_rest, (double)logf((float)r.p_rest) - lq_rest);
    } else {
        const float pr = (float)r.p_rest, qr = (float)r.q_rest;
        loss = 0.5 * (sum_of(l.sums[3]) + x_times(pr, log_share(pr, qr)) + x_times(qr, log_share(qr, pr)));
    }
    return r.none ? NAN : (float)(loss * weight);
}

// joins one (maximum, sum) per lane over the wave
__device__ inline float2 wave_join(float2 p, float c2) {
    const float m = wave_max_dpp(p.x);
    return make_float2(m, wave_sum_dpp(p.y * fast_exp2((p.x - m) * c2)));
}

// a vector with -inf in the places of the clear bits
template <bool BF16>
__device__ inline raw16 vec_only(const raw16& r, uint32_t on) {
    raw16 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) {
            const uint32_t lo = (on >> (2 * i)) & 1 ? r[i] & 0xffffu : 0xff80u, hi = (on >> (2 * i + 1)) & 1 ? r[i] & 0xffff0000u : 0xff800000u;
            o[i] = lo | hi;
        } else {
            o[i] = (on >> i) & 1 ? r[i] : None<false>::word;
        }
    }
    return o;
}

// the sums of a wave: (m, s) of each lane's vectors, and one vector more
template <bool BF16>
__device__ inline float2 wave_tail(float m, float s, const raw16& mine, float c2) {
    const float gm = wave_max_dpp(vec_max<BF16>(mine, m));
    return make_float2(gm, wave_sum_dpp(vec_sum<BF16>(mine, gm, c2, s * fast_exp2((m - gm) * c2))));
}

// ---- one workgroup per row, which holds it --------------------------------------------------------------
// A thread has HELD 16-byte vectors t, t + NT, t + 2 NT ... of the row, LDS of them in LDS and the others in registers, so that 512
// threads of 256 registers and 144 KB of LDS hold 504 KB, all but all of a compute unit.  Shorter rows take fewer threads or registers,
// and two or three workgroups share the unit, one reading while another computes or writes.  Besides the vectors a few values of the phases
// between do not fit: the compiler keeps 22 registers of <256, 32> in scratch memory and 4 of <256, 63> and of the fp32 <512, 63>.  A
// vector with tokens of the record is left out of the sums and of the stores (a bit per vector, a word per thread): the thread of its first place takes the vector's other elements
// and writes all of it.  The row's last, incomplete vector is the business of thread k (which has no place) in the same way.
template <bool BF16, int NT, int HELD, int LDS, int WAVES>
__global__ __launch_bounds__(NT, WAVES) void distill_row(const DistillArgs a) {
    typedef Row<BF16> R;
    typedef typename R::T T;
    constexpr int N = R::N, NW = NT / 64, REGS = HELD - LDS;
    constexpr int GROUP = HELD > 32 ? 3 : 4, FIRST = 8 / GROUP * GROUP;   // vectors whose sums go together; those asked for at once
    static_assert(HELD <= 64 && REGS % GROUP == 0 && LDS % GROUP == 0, "whole groups");
    __shared__ raw16 held[LDS ? LDS : 1][LDS ? NT : 1];
    __shared__ unsigned long long bits[NT];
    __shared__ float2 part[NW];
    __shared__ PlaceLds l;
    const int t = threadIdx.x, lane = t & 63, row = blockIdx.x;
    const T* p = (const T*)a.in + (long long)row * a.stride;
    T* to = (T*)a.grad + (long long)row * a.grad_stride;
    const float weight = a.weights ? a.weights[row] : 1.f;
    const int whole = a.V / N;   // complete vectors
    auto put_zero = [&]() {
        if (t == 0) a.loss[row] = 0.f;
        for (int w = t; w < whole; w += NT) __builtin_nontemporal_store((typename R::V)raw16{0, 0, 0, 0}, (typename R::V*)(to + (long long)w * N));
        if (t < a.V - whole * N) R::put_one(to + whole * N + t, 0.f);
    };
    int id = -1;
    float value = -INFINITY;
    if (t < a.k) id = a.ids[(long long)row * a.k + t], value = a.values[(long long)row * a.k + t];
    if (weight == 0.f) {
        put_zero();
        return;
    }
    bits[t] = 0;
    place_clear(l);
    __syncthreads();
    // The held vectors live across all phases.  `opaque` makes the compiler take a value as new, so that it neither keeps what an earlier
    // phase derived from it (unpacked elements, addresses, lane masks) nor runs out of registers for it.
    const auto opaque = [](auto& v) { asm volatile("" : "+v"(v)); };
    const uint32_t at = (uint32_t)t * 16u, end_at = (uint32_t)max(whole - 1, 0) * 16u;
    auto load = [&](int i) {   // past the end the last complete vector once more (it is masked out later)
        if (i * NT >= whole) return none16<BF16>();
        const uint32_t off = min(at + (uint32_t)i * NT * 16u, end_at);
        return (raw16)__builtin_nontemporal_load((const typename R::V*)((const char*)p + off));
    };
    // Loads come back in the order in which they are asked for: the vectors for LDS and the first group, then the record's tokens (known by
    // then), then the rest.  The sums follow them group by group, each with the thread's maximum so far.
    raw16 z[REGS];
    const bool entered = id >= 0 && id < a.V;
    bool listed = false;
    {
        raw16 h[LDS ? LDS : 1];
#pragma unroll
        for (int i = 0; i < LDS; ++i) h[i] = load(i);
#pragma unroll
        for (int i = 0; i < FIRST; ++i) z[i] = load(LDS + i);
        if (t < kPlaces) listed = place_enter(l, id, &bits[(uint32_t)id / N % NT], entered ? 1ull << (id / N / NT) : 0ull);
        __syncthreads();
        if constexpr (LDS > 0) {
#pragma unroll
            for (int i = 0; i < LDS; ++i) held[i][t] = h[i];
        }
    }
    const uint32_t flags = place_flags<N>(l, id, entered, listed);
    const bool tail = t == a.k && whole * N < a.V;
    float zp = -INFINITY;
    if (flags & kHere) zp = R::one(p + id);
    // what this thread takes beside its own vectors: a vector's elements that do not stand in the record (the bits of `flags`)
    const int beside = flags & kOwner ? id & ~(N - 1) : tail ? whole * N : a.V;
    raw16 mine = none16<BF16>();
    if (beside < a.V) mine = row_load<BF16>(p, beside, a.V);
#pragma unroll
    for (int i = FIRST; i < REGS; ++i) z[i] = load(LDS + i);
    const bool extra = (flags & kOwner) || (tail && !((bits[whole % NT] >> (whole / NT)) & 1));
    const int n_mine = whole > t ? (whole - t + NT - 1) / NT : 0;   // complete vectors of this thread
    unsigned long long live = (n_mine >= 64 ? ~0ull : (1ull << n_mine) - 1ull) & ~bits[t];   // those without a token of the record
    auto keep = [&](const raw16& r, int i) { return (live >> i) & 1 ? r : none16<BF16>(); };
    float m = kNoEntry, s = 0.f;   // of the other entries that this thread has
    auto rescale = [&](float to_m) {
        s *= fast_exp2((m - to_m) * a.c2);
        m = to_m;
    };
    auto add = [&](int i0) {   // a group in registers
        float gm = m;
#pragma unroll
        for (int i = i0; i < i0 + GROUP; ++i) {
            z[i] = keep(z[i], LDS + i);
            gm = vec_max<BF16>(z[i], gm);
            opaque(z[i]);
        }
        rescale(gm);
#pragma unroll
        for (int i = i0; i < i0 + GROUP; ++i) {
            s = vec_sum<BF16>(z[i], m, a.c2, s);
            opaque(z[i]);
            __builtin_amdgcn_sched_barrier(0);   // one vector's exponentials at a time are registers enough
        }
    };
    if constexpr (LDS > 0) {
#pragma unroll 1
        for (int i = 0; i < LDS; i += GROUP) {
            raw16 h[GROUP];
            float gm = m;
#pragma unroll
            for (int j = 0; j < GROUP; ++j) {
                h[j] = keep(held[i + j][t], i + j);
                gm = vec_max<BF16>(h[j], gm);
            }
            rescale(gm);
#pragma unroll
            for (int j = 0; j < GROUP; ++j) s = vec_sum<BF16>(h[j], m, a.c2, s);
        }
    }
#pragma unroll
    for (int i = 0; i < FIRST; i += GROUP) add(i);
    if (t < kPlaces) place_first(a, l, id, flags, zp, value);
    __syncthreads();
    if (sum_of(l.valid) == 0) {
        put_zero();
        return;
    }
    if (t < kPlaces) place_second(a, l, flags, zp, value, row);
#pragma unroll
    for (int i = FIRST; i < REGS; i += GROUP) add(i);
    const float2 q = wave_tail<BF16>(m, s, vec_only<BF16>(mine, extra ? ~flags : 0u), a.c2);
    if (lane == 0) part[t >> 6] = q;
    __syncthreads();
    float g = 0.f;
    if (t < kPlaces) {
        const float2 others = wave_join(lane < NW ? part[lane] : make_float2(kNoEntry, 0.f), a.c2);
        const RowSums r = row_sums(a, l, others, weight);
        if (a.divergence != PSD_DIV_KL) {
            jsd_sums(l, r);
            if (NT == kPlaces) __syncthreads();
        }
        if (NT == kPlaces || a.divergence == PSD_DIV_KL) g = place_gradient(a, l, r, others);
    }
    if (NT > kPlaces && a.divergence != PSD_DIV_KL) {
        __syncthreads();
        if (t < kPlaces) {
            const float2 others = wave_join(lane < NW ? part[lane] : make_float2(kNoEntry, 0.f), a.c2);
            g = place_gradient(a, l, row_sums(a, l, others, weight), others);
        }
    }
    __syncthreads();
    {
        const float rest = l.rest, rest_max = l.rest_max;
        if (extra) mine = row_load<BF16>(p, beside, a.V);   // again, rather than held all the while
        auto grad_at = [&](float y) { return rest * fast_exp2((y - rest_max) * a.c2); };
        auto store = [&](const raw16& v, int i) {
            if ((live >> i) & 1) __builtin_nontemporal_store((typename R::V)v, (typename R::V*)((char*)to + (at + (uint32_t)i * NT * 16u)));
        };
        auto grad_of = [&](const raw16& v) {
            float e[N];
#pragma unroll
            for (int x = 0; x < N; ++x) e[x] = grad_at(R::get(v, x));
            return R::pack(e);
        };
        constexpr int TURN = BF16 ? 2 : 4;   // vectors whose exponentials go side by side
#pragma unroll
        for (int i = 0; i < REGS; i += TURN) {
            opaque(live);
#pragma unroll
            for (int j = i; j < i + TURN && j < REGS; ++j) z[j] = grad_of(z[j]);
#pragma unroll
            for (int j = i; j < i + TURN && j < REGS; ++j) store(z[j], LDS + j);
        }
        if constexpr (LDS > 0)
#pragma unroll 2
            for (int i = 0; i < LDS; ++i) store(grad_of(held[i][t]), i);
        if (extra) {
#pragma unroll
            for (int x = 0; x < N; ++x)
                if (beside + x < a.V && !((flags >> x) & 1)) R::put_one(to + beside + x, grad_at(R::get(mine, x)));
        }
        if (flags & kHere) R::put_one(to + id, g);
    }
    if (t == 0) a.loss[row] = row_loss(a, l, weight);
}

// ---- one workgroup per row, which passes by --------------------------------------------------------------
// The same sums in the same order, a group of vectors on its way while one is added.  With GRAD the row passes a second time.  Short code:
// distill_row's long straight runs first have to come into the instruction cache (48 rows of 32000 fp32 entries: 17.6 us there, 9.4 here).
template <bool BF16, int NT, int GROUP, int WAVES, bool GRAD>
__global__ __launch_bounds__(NT, WAVES) void distill_pass(const DistillArgs a) {
    typedef Row<BF16> R;
    typedef typename R::T T;
    constexpr int N = R::N, NW = NT / 64;
    __shared__ unsigned long long bits[NT];
    __shared__ float2 part[NW];
    __shared__ PlaceLds l;
    __shared__ int first[kSmallVocab];
    const int t = threadIdx.x, lane = t & 63, row = blockIdx.x;
    const T* p = (const T*)a.in + (long long)row * a.stride;
    T* to = (T*)a.grad + (long long)row * a.grad_stride;
    const float weight = a.weights ? a.weights[row] : 1.f;
    const int whole = a.V / N;
    auto put_zero = [&]() {
        if (t == 0) a.loss[row] = 0.f;
        if (!GRAD) return;
        for (int w = t; w < whole; w += NT) __builtin_nontemporal_store((typename R::V)raw16{0, 0, 0, 0}, (typename R::V*)(to + (long long)w * N));
        if (t < a.V - whole * N) R::put_one(to + whole * N + t, 0.f);
    };
    int id = -1;
    float value = -INFINITY;
    if (t < a.k) id = a.ids[(long long)row * a.k + t], value = a.values[(long long)row * a.k + t];
    if (weight == 0.f) {
        put_zero();
        return;
    }
    bits[t] = 0;
    place_clear(l);
    const bool small = a.V <= kSmallVocab;
    if (small)
        for (int i = t; i < a.V; i += NT) first[i] = kPlaces;
    __syncthreads();
    const uint32_t at = (uint32_t)t * 16u, end_at = (uint32_t)max(whole - 1, 0) * 16u;
    auto load = [&](int i) {   // past the end the last complete vector once more (it is masked out later)
        const uint32_t off = min(at + (uint32_t)i * NT * 16u, end_at);
        if (whole <= 0) return none16<BF16>();
        if (GRAD) return (raw16) * (const typename R::V*)((const char*)p + off);
        return (raw16)__builtin_nontemporal_load((const typename R::V*)((const char*)p + off));
    };
    raw16 z[GROUP];
#pragma unroll
    for (int i = 0; i < GROUP; ++i) z[i] = load(i);
    const bool entered = id >= 0 && id < a.V;
    bool listed = false;
    if (small) {
        if (entered) atomicMin(&first[id], t), atomicOr(&bits[(uint32_t)id / N % NT], 1ull << (id / N / NT));
    } else if (t < kPlaces) {
        listed = place_enter(l, id, &bits[(uint32_t)id / N % NT], entered ? 1ull << (id / N / NT) : 0ull);
    }
    __syncthreads();
    const uint32_t flags = small ? place_flags_small<N>(first, a.V, id, entered) : place_flags<N>(l, id, entered, listed);
    const bool tail = t == a.k && whole * N < a.V;
    float zp = -INFINITY;
    if (flags & kHere) zp = R::one(p + id);
    // what this thread takes beside its own vectors: a vector's elements that do not stand in the record (the bits of `flags`)
    const int beside = flags & kOwner ? id & ~(N - 1) : tail ? whole * N : a.V;
    raw16 mine = none16<BF16>();
    if (beside < a.V) mine = row_load<BF16>(p, beside, a.V);
    const bool extra = (flags & kOwner) || (tail && !((bits[whole % NT] >> (whole / NT)) & 1));
    const int n_mine = whole > t ? (whole - t + NT - 1) / NT : 0;
    const unsigned long long live = (n_mine >= 64 ? ~0ull : (1ull << n_mine) - 1ull) & ~bits[t];
    float m = kNoEntry, s = 0.f;
    const int turns = (whole + NT * GROUP - 1) / (NT * GROUP);
#pragma unroll 1
    for (int j = 0; j < turns; ++j) {
        raw16 next[GROUP];
#pragma unroll
        for (int i = 0; i < GROUP; ++i) next[i] = load((j + 1) * GROUP + i);
        const uint32_t on = (uint32_t)(live >> (j * GROUP));
        float gm = m;
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            if (!((on >> i) & 1)) z[i] = none16<BF16>();
            gm = vec_max<BF16>(z[i], gm);
        }
        s *= fast_exp2((m - gm) * a.c2);
        m = gm;
#pragma unroll
        for (int i = 0; i < GROUP; ++i) s = vec_sum<BF16>(z[i], m, a.c2, s);
#pragma unroll
        for (int i = 0; i < GROUP; ++i) z[i] = next[i];
    }
    if (t < kPlaces) place_first(a, l, id, flags, zp, value);
    const float2 q = wave_tail<BF16>(m, s, vec_only<BF16>(mine, extra ? ~flags : 0u), a.c2);
    if (lane == 0) part[t >> 6] = q;
    __syncthreads();
    if (sum_of(l.valid) == 0) {
        put_zero();
        return;
    }
    if (t < kPlaces) place_second(a, l, flags, zp, value, row);
    __syncthreads();
    const float2 others = wave_join(lane < NW ? part[lane] : make_float2(kNoEntry, 0.f), a.c2);
    if (GRAD) {   // the first group of the second pass sets out
#pragma unroll
        for (int i = 0; i < GROUP; ++i) z[i] = load(i);
    }
    float g = 0.f;
    if (t < kPlaces && a.divergence != PSD_DIV_KL) jsd_sums(l, row_sums(a, l, others, weight));
    if (a.divergence != PSD_DIV_KL) __syncthreads();
    if (t < kPlaces) g = place_gradient(a, l, row_sums(a, l, others, weight), others);
    __syncthreads();
    if (GRAD) {
        const float rest = l.rest, rest_max = l.rest_max;
        auto grad_at = [&](float y) { return rest * fast_exp2((y - rest_max) * a.c2); };
#pragma unroll 1
        for (int j = 0; j < turns; ++j) {
            raw16 next[GROUP];
#pragma unroll
            for (int i = 0; i < GROUP; ++i) next[i] = load((j + 1) * GROUP + i);
            const uint32_t on = (uint32_t)(live >> (j * GROUP));
#pragma unroll
            for (int i = 0; i < GROUP; ++i) {
                float e[N];
#pragma unroll
                for (int x = 0; x < N; ++x) e[x] = grad_at(R::get(z[i], x));
                if ((on >> i) & 1) __builtin_nontemporal_store((typename R::V)R::pack(e), (typename R::V*)((char*)to + (at + (uint32_t)(j * GROUP + i) * NT * 16u)));
            }
#pragma unroll
            for (int i = 0; i < GROUP; ++i) z[i] = next[i];
        }
        if (extra) {
#pragma unroll
            for (int x = 0; x < N; ++x)
                if (beside + x < a.V && !((flags >> x) & 1)) R::put_one(to + beside + x, grad_at(R::get(mine, x)));
        }
        if (flags & kHere) R::put_one(to + id, g);
    }
    if (t == 0) a.loss[row] = row_loss(a, l, weight);
}

// ---- (row, chunk) -------------------------------------------------------------------------------------
template <bool BF16>
__global__ __launch_bounds__(kDisThreads) void distill_tail(const DistillArgs a) {
    typedef Row<BF16> R;
    constexpr int N = R::N, VEC = kDisPer / N;
    __shared__ uint32_t bits[kDisChunk / 32];   // the chunk's tokens that stand in the record
    __shared__ float2 part[kDisThreads / 64];
    const int t = threadIdx.x, lane = t & 63, row = blockIdx.y, chunk = blockIdx.x, v0 = chunk * kDisChunk;
    if (a.weights && a.weights[row] == 0.f) return;
    const typename R::T* p = (const typename R::T*)a.in + (long long)row * a.stride;
    int id = -1;
    if (t < a.k) id = a.ids[(long long)row * a.k + t];
    raw16 z[VEC];
    const raw16 none = none16<BF16>();
    if (v0 + kDisChunk <= a.V) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[i] = *(const typename R::V*)(p + v0 + N * (t + kDisThreads * i));
    } else {
#pragma unroll 1
        for (int i = 0; i < VEC; ++i) {
            const int v = v0 + N * (t + kDisThreads * i);
            const raw16 r = v < a.V ? row_load<BF16>(p, v, a.V) : none;
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (i == j) z[j] = r;
        }
    }
    for (int i = t; i < kDisChunk / 32; i += kDisThreads) bits[i] = 0;
    __syncthreads();
    const uint32_t u = (uint32_t)id - (uint32_t)v0;
    if (u < (uint32_t)kDisChunk && id < a.V) {
        atomicOr(&bits[u >> 5], 1u << (u & 31));
        a.student[(long long)row * a.k + t] = R::one(p + id);
    }
    __syncthreads();
    float m = kNoEntry;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int at = N * (t + kDisThreads * i);
        const uint32_t in_s = bits[at >> 5] >> (at & 31) & ((1u << N) - 1);
        if (in_s) {
            float e[N];
#pragma unroll
            for (int x = 0; x < N; ++x) e[x] = (in_s >> x) & 1 ? -INFINITY : R::get(z[i], x);
            z[i] = R::pack(e);
        }
        m = vec_max<BF16>(z[i], m);
    }
    m = wave_max_dpp(m);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < VEC; ++i) s = vec_sum<BF16>(z[i], m, a.c2, s);
    s = wave_sum_dpp(s);
    if (lane == 0) part[t >> 6] = make_float2(m, s);
    __syncthreads();
    if (t < 64) {
        const float2 q = wave_join(lane < kDisThreads / 64 ? part[lane] : make_float2(kNoEntry, 0.f), a.c2);
        if (t == 0) a.parts[(long long)row * a.chunks + chunk] = q;
    }
}

// without a gradient: one workgroup per row, the loss alone
template <bool BF16>
__global__ __launch_bounds__(kDisThreads) void distill_grad(const DistillArgs a) {
    typedef Row<BF16> R;
    typedef typename R::T T;
    constexpr int N = R::N, VEC = kDisPer / N;
    constexpr int kTable = 2 * kDisThreads;
    __shared__ uint32_t table[kTable];
    __shared__ PlaceLds l;
    const int t = threadIdx.x, lane = t & 63, row = blockIdx.y, chunk = blockIdx.x, v0 = chunk * kDisChunk;
    const T* p = (const T*)a.in + (long long)row * a.stride;
    T* to = (T*)a.grad + (long long)row * a.grad_stride;
    const float weight = a.weights ? a.weights[row] : 1.f;
    auto put_zero = [&]() {
        if (chunk == 0 && t == 0) a.loss[row] = 0.f;
        if (!a.grad) return;
        for (int v = v0 + t; v < min(a.V, v0 + kDisChunk); v += kDisThreads) R::put_one(to + v, 0.f);
    };
    if (weight == 0.f) {
        put_zero();
        return;
    }
    table[t] = table[t + kDisThreads] = 0;
    place_clear(l);
    __syncthreads();
    int id = -1;
    float value = -INFINITY, zp = -INFINITY;
    const long long base = (long long)row * a.k;
    if (t < a.k) {
        id = a.ids[base + t];
        value = a.values[base + t];
        if (id >= 0 && id < a.V) zp = a.student[base + t];
    }
    float2 tail = make_float2(kNoEntry, 0.f);
    for (int i = lane; i < a.chunks; i += 64) tail = join_sums(tail, a.parts[(long long)row * a.chunks + i], a.c2);
    const bool full = a.grad && v0 + kDisChunk <= a.V;
    raw16 z[VEC];
    if (full) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[i] = *(const typename R::V*)(p + v0 + N * (t + kDisThreads * i));
    }
    const bool entered = id >= 0 && id < a.V;
    const uint32_t at = (uint32_t)id / N % (32u * kTable);   // more tokens than the table has bits may meet in one
    const bool listed = place_enter(l, id, &table[at / 32], entered ? 1u << (at % 32) : 0u);
    __syncthreads();
    const uint32_t flags = place_flags<N>(l, id, entered, listed);
    place_first(a, l, id, flags, zp, value);
    __syncthreads();
    if (sum_of(l.valid) == 0) {
        put_zero();
        return;
    }
    place_second(a, l, flags, zp, value, row);
    tail = wave_join(tail, a.c2);
    __syncthreads();
    const RowSums r = row_sums(a, l, tail, weight);
    if (a.divergence != PSD_DIV_KL) {
        jsd_sums(l, r);
        __syncthreads();
    }
    const float g = place_gradient(a, l, r, tail);
    __syncthreads();
    if (chunk == 0 && t == 0) a.loss[row] = row_loss(a, l, weight);
    if (!a.grad) return;
    const float rest = l.rest, rest_max = l.rest_max;
    float e[N];
    if (full) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
#pragma unroll
            for (int x = 0; x < N; ++x) e[x] = rest * fast_exp2((R::get(z[i], x) - rest_max) * a.c2);
            *(typename R::V*)(to + v0 + N * (t + kDisThreads * i)) = (typename R::V)R::pack(e);
        }
    } else {
        for (int v = v0 + N * t; v < a.V; v += N * kDisThreads) {
            const raw16 q = row_load<BF16>(p, v, a.V);
#pragma unroll
            for (int x = 0; x < N; ++x) e[x] = rest * fast_exp2((R::get(q, x) - rest_max) * a.c2);
            row_store<BF16>(to, v, a.V, e);
        }
    }
    __syncthreads();   // the record's tokens last
    if ((flags & kHere) && id >= v0 && id < v0 + kDisChunk) R::put_one(to + id, g);
}

// How a call goes: in chunks, or its rows pass by a workgroup of 256, 512 or 1024 threads, or (with a gradient; else they pass by) they are held by
// one of 256 threads with 32 or 63 vectors each or of 512 with 63.  The loss takes the same sums in the same order with a gradient or without.
//   chunks   few long rows, which leave most units idle otherwise: 12 MB of them, 20 MB where a row has 256 KB (us, chunks / passing; 65536 fp32
//            entries: 64 rows 12.9 / 13.8, 89 rows 14.9 / 14.1; 128256: 29 rows 17.2 / 21.7, 48 rows 22.9 / 22.0; bf16: 64 rows 16.3 / 19.5, 89 rows
//            21.3 / 19.7; 65536 bf16: 64 rows 12.0 / 12.7, 108 rows 15.3 / 13.2; 49152 bf16: 32 rows 10.4 / 11.9, 100 rows 12.7 / 12.2; the loss alone
//            of 4 / 64 such rows 10.3 / 8.9 and 10.0 / 10.2), and rows over 1 MB
//   holding  rows from 96 KB, 240 MB of them in all: there the second pass comes from memory (passing / holding; 128256 fp32 entries: 800 rows
//            195 / 178, 300 rows, which pass, 76 / 73; bf16: 2000 rows 238 / 205, 800 rows 97 / 100; 50257 bf16: 3000 rows 196 / 170, 1200 rows 72 / 79).
//            Rows beyond 504 KB pass all the same (1024 rows of 129024 fp32 entries, held: 204, of 131072: 286), and with k = 256, where thread k of 256 has
//            a place, 512 threads hold a row (4096 bf16 rows of 128256, JSD: 422 with k = 255, 600)
//   passing  1024 threads for at most a row per unit, 512 for rows over 128 KB (65536 fp32 entries, 2000 rows: 237, with 256 threads 291), else 256
//            (50257 bf16, 800 rows: 55, with 512 threads 59; 4000 fp32 entries, 1000 rows: 11.7, with 1024 threads 25.5)
enum Way { PASS_256, PASS_512, PASS_1024, HOLD_128K, HOLD_252K, HOLD_504K, CHUNKS };
static Way way_of(int n_rows, int vocab, int el, int k) {
    const long long vectors = ((long long)vocab * el + 15) / 16, all = vectors * 16 * n_rows;
    if (vectors > 1024 * 64 || (vocab >= 49152 && all <= (vectors >= 16384 ? 20LL : 12LL) << 20)) return CHUNKS;
    if (n_rows <= 256 || vectors > 512 * 64) return PASS_1024;
    const bool narrow = k < kPlaces;   // thread k must have no place
    if (vectors >= 6144 && vectors <= 512 * 63 && all >= 240LL << 20) return narrow && vectors <= 256 * 32 ? HOLD_128K : narrow && vectors <= 256 * 63 ? HOLD_252K : HOLD_504K;
    return narrow && vectors <= 8192 ? PASS_256 : PASS_512;
}

template <bool BF16, bool GRAD>
static void distill_launch(const DistillArgs& a, int n_rows, Way way, hipStream_t st) {
    switch (way) {
        case PASS_256: distill_pass<BF16, 256, 4, 5, GRAD><<<n_rows, 256, 0, st>>>(a); break;
        case PASS_512: distill_pass<BF16, 512, 4, 4, GRAD><<<n_rows, 512, 0, st>>>(a); break;
        case PASS_1024: distill_pass<BF16, 1024, 4, 4, GRAD><<<n_rows, 1024, 0, st>>>(a); break;
        case HOLD_128K:
            if constexpr (GRAD) distill_row<BF16, 256, 32, 8, 3><<<n_rows, 256, 0, st>>>(a);
            else distill_pass<BF16, 256, 4, 5, false><<<n_rows, 256, 0, st>>>(a);
            break;
        case HOLD_252K:
            if constexpr (GRAD) distill_row<BF16, 256, 63, 18, 2><<<n_rows, 256, 0, st>>>(a);
            else distill_pass<BF16, 256, 3, 5, false><<<n_rows, 256, 0, st>>>(a);
            break;
        case HOLD_504K:
            if constexpr (GRAD) distill_row<BF16, 512, 63, 18, 2><<<n_rows, 512, 0, st>>>(a);
            else distill_pass<BF16, 512, 3, 4, false><<<n_rows, 512, 0, st>>>(a);
            break;
        case CHUNKS:
            distill_tail<BF16><<<dim3(a.chunks, n_rows), kDisThreads, 0, st>>>(a);
            distill_grad<BF16><<<dim3(GRAD ? a.chunks : 1, n_rows), kDisThreads, 0, st>>>(a);
    }
}

}  // namespace psd

using namespace psd;

extern "C" size_t psd_distill_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t k) {
    if (n_rows < 1 || n_rows > kMaxRows || vocab < 1 || vocab > kMaxVocab || k < 1 || k > PSD_MAX_TOP) return 0;
    const int chunks = (vocab + kDisChunk - 1) / kDisChunk;
    return align16((size_t)n_rows * chunks * sizeof(float2)) + align16((size_t)n_rows * k * sizeof(float));
}

extern "C" int psd_distill(const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t stride, const float* top_values,
                           const int32_t* top_ids, const float* top_lse, int32_t k, float temperature, int32_t divergence,
                           const float* row_weights, float* loss, void* grad, int64_t grad_stride, void* workspace,
                           size_t workspace_bytes, void* stream) {
    char* err = tls_error();
    const char* who = "psd_distill";
    int rc = rows_check(who, logits, dtype, n_rows, vocab, stride, err);
    if (rc == PSD_OK && grad) rc = rows_check(who, grad, dtype, n_rows, vocab, grad_stride, err);
    if (rc != PSD_OK) return rc;
    if (grad && !rows_apart_or_same(logits, stride, grad, grad_stride, n_rows, vocab, row_elem(dtype)))
        PSD_FAIL(PSD_EINVAL, err, "%s: grad overlaps the logits", who);
    if (!top_values || !top_ids || !loss || !workspace) PSD_FAIL(PSD_EINVAL, err, "%s: null pointer", who);
    if (k < 1 || k > PSD_MAX_TOP) PSD_FAIL(PSD_EINVAL, err, "%s: k=%d", who, k);
    if (!temperature_fits(temperature)) PSD_FAIL(PSD_EINVAL, err, "%s: temperature=%g", who, temperature);
    if (divergence != PSD_DIV_KL && divergence != PSD_DIV_JSD) PSD_FAIL(PSD_EINVAL, err, "%s: divergence=%d", who, divergence);
    if (((uintptr_t)top_values | (uintptr_t)top_ids | (uintptr_t)top_lse | (uintptr_t)row_weights | (uintptr_t)loss) & 3 || ((uintptr_t)workspace & 15))
        PSD_FAIL(PSD_EINVAL, err, "%s: misaligned record, weights, loss or workspace", who);
    if (workspace_bytes < psd_distill_workspace_bytes(n_rows, vocab, k))
        PSD_FAIL(PSD_ENOMEM, err, "%s: workspace %zu < %zu bytes", who, workspace_bytes, psd_distill_workspace_bytes(n_rows, vocab, k));
    const int chunks = (vocab + kDisChunk - 1) / kDisChunk;
    DistillArgs a{logits, grad, stride, grad_stride, vocab, k, chunks, kLog2e / temperature, 1.0 / (double)temperature, divergence,
                  top_values, top_ids, top_lse, row_weights, loss, (float2*)workspace,
                  (float*)((char*)workspace + align16((size_t)n_rows * chunks * sizeof(float2)))};
    const Way way = way_of(n_rows, vocab, row_elem(dtype), k);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == PSD_BF16) grad ? distill_launch<true, true>(a, n_rows, way, st) : distill_launch<true, false>(a, n_rows, way, st);
    else grad ? distill_launch<false, true>(a, n_rows, way, st) : distill_launch<false, false>(a, n_rows, way, st);
    PSD_HIP(hipGetLastError(), err);
    return PSD_OK;
}
