// Distillation from a teacher's top logits: the divergence between the record's K + 1 outcomes (its tokens, and all others together)
// and a student's row, and the gradient.
//
// Per row the student is needed as: its logits at the record's tokens, and the log-sum-exp of all other entries (its own maximum,
// so that it neither cancels against the record's mass nor underflows beside it).  From these the divergence and the gradient's K + 1
// coefficients follow: with g_b = q_b (dl/dq_b - sum_b q_b dl/dq_b) the gradient is g_i / T at a record's token and
// g_rest / T times softmax over the others at every other entry.
//   distill_tail  (row, chunk): maximum and sum of exponentials of the chunk without the record's tokens; their logits set aside
//   distill_grad  (row, chunk): joins the row's chunks, works out the coefficients, writes the chunk's part of the gradient
// Statistics, divergences and coefficients are formed from fp32 exponentials and logarithms, differences and sums in 64 bits.
#include "psd_rows.h"

namespace psd {

constexpr int kDisThreads = 256;
constexpr int kDisChunk = 8192;
constexpr int kDisPer = kDisChunk / kDisThreads;   // entries of a thread: 32
constexpr int kDisWaves = kDisThreads / 64;
static_assert(PSD_MAX_TOP <= kDisThreads, "a thread per place of a record");

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

struct DistillLds {
    alignas(16) int ids[PSD_MAX_TOP];
    uint32_t bits[kDisChunk / 32];   // the chunk's tokens that stand in the record
    float2 part[kDisWaves];
    double sums[4][kDisWaves];
};

__device__ inline double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// sum over the workgroup, in a fixed order; `slot` must not be in use by a sum that some thread may still read
__device__ inline double block_sum(double v, double* slot) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    return (slot[0] + slot[1]) + (slot[2] + slot[3]);
}
__device__ inline float block_max(float v, float2* slot) {
    v = wave_max_dpp(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6].x = v;
    __syncthreads();
    v = fmaxf(fmaxf(slot[0].x, slot[1].x), fmaxf(slot[2].x, slot[3].x));
    return v;
}

template <bool BF16>
__global__ __launch_bounds__(kDisThreads) void distill_tail(const DistillArgs a) {
    typedef Row<BF16> R;
    constexpr int N = R::N, VEC = kDisPer / N;
    __shared__ DistillLds l;
    const int t = threadIdx.x, row = blockIdx.y, chunk = blockIdx.x, v0 = chunk * kDisChunk;
    if (a.weights && a.weights[row] == 0.f) return;
    const typename R::T* p = (const typename R::T*)a.in + (long long)row * a.stride;
    raw16 z[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int v = v0 + N * (t + kDisThreads * i);
        if (v < a.V) z[i] = row_load<BF16>(p, v, a.V);
    }
    for (int i = t; i < kDisChunk / 32; i += kDisThreads) l.bits[i] = 0;
    __syncthreads();
    if (t < a.k) {
        const int id = a.ids[(long long)row * a.k + t];
        const uint32_t u = (uint32_t)id - (uint32_t)v0;
        if (u < (uint32_t)kDisChunk && id < a.V) {
            atomicOr(&l.bits[u >> 5], 1u << (u & 31));
            a.student[(long long)row * a.k + t] = R::one(p + id);
        }
    }
    __syncthreads();
    float mx = kNoEntry;
    float e[VEC][N];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int u = N * (t + kDisThreads * i);
        const uint32_t in_s = l.bits[u >> 5] >> (u & 31);
#pragma unroll
        for (int x = 0; x < N; ++x) {
            e[i][x] = v0 + u < a.V && !((in_s >> x) & 1) ? R::get(z[i], x) : -INFINITY;
            mx = fmaxf(mx, e[i][x]);
        }
    }
    mx = block_max(mx, l.part);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < VEC; ++i)
#pragma unroll
        for (int x = 0; x < N; ++x) s += fast_exp2((e[i][x] - mx) * a.c2);
    s = wave_sum_dpp(s);
    if ((t & 63) == 0) l.part[t >> 6].y = s;
    __syncthreads();
    if (t == 0) a.parts[(long long)row * a.chunks + chunk] = make_float2(mx, (l.part[0].y + l.part[1].y) + (l.part[2].y + l.part[3].y));
}

// What the row's gradient and loss come to.  here: place t of the record counts, and `g` is its gradient; the others' is
// rest * 2^((z - rest_max) c2)
struct RowResult {
    bool empty;      // weight 0 or no valid place
    bool here;
    float g, rest, rest_max;
    double loss;
};

__device__ inline double x_times(double x, double y) { return x > 0.0 ? x * y : 0.0; }   // 0 ln 0 = 0

// ln(2 x / (x + y)): near 1 by the difference, which loses nothing there, else by the quotient
__device__ inline double log_share(float x, float y) {
    const float s = x + y, d = (x - y) / s;
    return fabsf(d) < 0.5f ? log1pf(d) : logf(2.f * x / s);
}

__device__ inline RowResult finish_row(const DistillArgs& a, DistillLds& l, int row) {
    RowResult r{true, false, 0.f, 0.f, 0.f, 0.0};
    const float weight = a.weights ? a.weights[row] : 1.f;
    if (weight == 0.f) return r;
    const int t = threadIdx.x;
    const long long base = (long long)row * a.k;
    int id = -1;
    float value = -INFINITY, z = -INFINITY;
    if (t < a.k) id = a.ids[base + t], value = a.values[base + t];
    bool here = id >= 0 && id < a.V;
    if (here) z = a.student[base + t];
    l.ids[t] = id;
    // the others: the chunks' sums in order, by every thread alike
    const float2* parts = a.parts + (long long)row * a.chunks;
    float2 rest = parts[0];
    for (int c = 1; c < a.chunks; ++c) rest = join_sums(rest, parts[c], a.c2);
    __syncthreads();
    // the first place of a token counts; every thread reads all places, four at a time
    bool again = false;
#pragma unroll 8
    for (int i = 0; i < a.k; i += 4) {
        const int4 o = *reinterpret_cast<const int4*>(&l.ids[i]);
        again |= (o.x == id && i < t) | (o.y == id && i + 1 < t) | (o.z == id && i + 2 < t) | (o.w == id && i + 3 < t);
    }
    here = here && !again;
    const int n_valid = __syncthreads_count(here);
    const bool complete = __syncthreads_or(t < a.k && id < 0);   // the teacher has no entry beside those of its record
    if (n_valid == 0) return r;
    r.empty = false;
    r.here = here;
    // student
    const float m = block_max(fmaxf(here ? z : -INFINITY, rest.x), l.part);
    const float x = (z - m) * a.c2, es = here ? fast_exp2(x) : 0.f;
    const float rest_x = (rest.x - m) * a.c2;
    const double es_rest = (double)rest.y * fast_exp2(rest_x);
    const double total = block_sum(es, l.sums[0]) + es_rest;
    const double log_total = log(total);
    const double q = es / total, q_rest = es_rest / total;
    const double lq = (double)x * 0.6931471805599453 - log_total, lq_rest = (double)rest_x * 0.6931471805599453 + (double)logf(rest.y) - log_total;
    // teacher
    double p = 0.0, lp = -INFINITY, p_rest = 0.0, mass = 1.0;
    if (a.lse) {
        lp = (double)value * a.inv_temp - (double)a.lse[row];
        p = here ? (double)expf((float)lp) : 0.0;
        mass = block_sum(p, l.sums[1]);
        if (!complete && n_valid < a.V && mass < 1.0) p_rest = 1.0 - mass;
    } else {
        const float tm = block_max(here ? value : -INFINITY, l.part);
        lp = ((double)value - (double)tm) * a.inv_temp;
        p = here ? (double)expf((float)lp) : 0.0;
        const double sum = block_sum(p, l.sums[1]);
        p /= sum;
        lp -= log(sum);
    }
    const double lp_rest = (double)logf((float)p_rest);
    double g, g_rest, l_row;
    if (a.divergence == PSD_DIV_KL) {
        l_row = block_sum(here ? x_times(p, lp - lq) : 0.0, l.sums[2]) + x_times(p_rest, lp_rest - lq_rest);
        const double P = a.lse ? mass + p_rest : 1.0;
        g = q * P - p;
        g_rest = q_rest * P - p_rest;
    } else {
        const float fp = (float)p, fq = (float)q, fpr = (float)p_rest, fqr = (float)q_rest;
        const double kp = x_times(fp, log_share(fp, fq)), kq = x_times(fq, log_share(fq, fp));
        const double kpr = x_times(fpr, log_share(fpr, fqr)), kqr = x_times(fqr, log_share(fqr, fpr));
        l_row = 0.5 * (block_sum(kp + kq, l.sums[2]) + kpr + kqr);
        const double W = block_sum(kq, l.sums[3]) + kqr;
        g = 0.5 * (kq - q * W);
        g_rest = 0.5 * (kqr - q_rest * W);
    }
    if (!(total > 0.0)) l_row = g = g_rest = NAN;   // no distribution at all
    const double scale = (double)weight * a.inv_temp;
    r.loss = l_row * weight;
    r.g = (float)(g * scale);
    r.rest = rest.y > 0.f ? (float)(g_rest * scale / rest.y) : total > 0.0 ? 0.f : NAN;
    r.rest_max = rest.x;
    return r;
}

// gradient == nullptr: one workgroup per row, the loss alone
template <bool BF16>
__global__ __launch_bounds__(kDisThreads) void distill_grad(const DistillArgs a) {
    typedef Row<BF16> R;
    constexpr int N = R::N, VEC = kDisPer / N;
    __shared__ DistillLds l;
    const int t = threadIdx.x, row = blockIdx.y, chunk = blockIdx.x, v0 = chunk * kDisChunk;
    const RowResult r = finish_row(a, l, row);
    if (chunk == 0 && t == 0) a.loss[row] = (float)r.loss;
    if (!a.grad) return;
    const typename R::T* p = (const typename R::T*)a.in + (long long)row * a.stride;
    typename R::T* to = (typename R::T*)a.grad + (long long)row * a.grad_stride;
    float e[N];
    if (r.empty) {
#pragma unroll
        for (int x = 0; x < N; ++x) e[x] = 0.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int v = v0 + N * (t + kDisThreads * i);
            if (v < a.V) row_store<BF16>(to, v, a.V, e);
        }
        return;
    }
    raw16 z[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int v = v0 + N * (t + kDisThreads * i);
        if (v < a.V) z[i] = row_load<BF16>(p, v, a.V);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int v = v0 + N * (t + kDisThreads * i);
        if (v >= a.V) continue;
#pragma unroll
        for (int x = 0; x < N; ++x) e[x] = r.rest * fast_exp2((R::get(z[i], x) - r.rest_max) * a.c2);
        row_store<BF16>(to, v, a.V, e);
    }
    __syncthreads();   // the record's tokens last
    if (r.here) {
        const int id = l.ids[t];
        if (id >= v0 && id < v0 + kDisChunk) R::put_one(to + id, r.g);
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
    if (!(temperature > 0.f)) PSD_FAIL(PSD_EINVAL, err, "%s: temperature=%g", who, temperature);
    if (divergence != PSD_DIV_KL && divergence != PSD_DIV_JSD) PSD_FAIL(PSD_EINVAL, err, "%s: divergence=%d", who, divergence);
    if (((uintptr_t)top_values | (uintptr_t)top_ids | (uintptr_t)top_lse | (uintptr_t)row_weights | (uintptr_t)loss) & 3 || ((uintptr_t)workspace & 15))
        PSD_FAIL(PSD_EINVAL, err, "%s: misaligned record, weights, loss or workspace", who);
    if (workspace_bytes < psd_distill_workspace_bytes(n_rows, vocab, k))
        PSD_FAIL(PSD_ENOMEM, err, "%s: workspace %zu < %zu bytes", who, workspace_bytes, psd_distill_workspace_bytes(n_rows, vocab, k));
    const int chunks = (vocab + kDisChunk - 1) / kDisChunk;
    DistillArgs a{logits, grad, stride, grad_stride, vocab, k, chunks, kLog2e / temperature, 1.0 / (double)temperature, divergence,
                  top_values, top_ids, top_lse, row_weights, loss, (float2*)workspace,
                  (float*)((char*)workspace + align16((size_t)n_rows * chunks * sizeof(float2)))};
    hipStream_t st = (hipStream_t)stream;
    const dim3 all(chunks, n_rows), per_row(grad ? chunks : 1, n_rows);
    if (dtype == PSD_BF16) {
        distill_tail<true><<<all, kDisThreads, 0, st>>>(a);
        distill_grad<true><<<per_row, kDisThreads, 0, st>>>(a);
    } else {
        distill_tail<false><<<all, kDisThreads, 0, st>>>(a);
        distill_grad<false><<<per_row, kDisThreads, 0, st>>>(a);
    }
    PSD_HIP(hipGetLastError(), err);
    return PSD_OK;
}
