// distill.hip -- divergence of a student's logits from a teacher's top logits
// and its gradient.
//
// Forward: a block takes one slice of a row, marks the kept columns that lie
// in it in an LDS bitmap, and sums exp((z - m) / t) over the others, m their
// maximum in the slice.  The kept columns are left out of the sum rather than
// taken off it later: where they hold nearly all of q, the difference of two
// sums would lose q_rest.  One wave per row then joins the slices, reads the
// student's kept logits, and forms the loss in 64 bits from 32-bit
// exponentials (k of them against the slices' cols).
// Backward: q of every column from the saved maximum and sum, and the kept
// columns written again with their p.
#include <type_traits>

#include "launch.hpp"
#include "losses.hpp"

namespace dr {
namespace {

struct DistillArgs {
    Matrix m;
    Teacher t;
    Slices sl;
    const float *weight;
    float c;      // log2(e) / temperature
    float inv_t;  // 1 / temperature
    float2 *part;  // per row and slice: (maximum, sum of exponentials) of the columns not kept
    float *loss, *stats;
    const float *upstream;
    uint64_t upstream_stride;
    void *grad;
    uint64_t grad_stride;
};

// Marks the row's kept columns in [start, start + n) in the bitmap.
__device__ __forceinline__ void mark_kept(const Teacher &t, uint64_t row, uint32_t start, uint32_t n, uint32_t cols,
                                          uint32_t *bm) {
    for (uint32_t k = threadIdx.x; k < t.k; k += blockDim.x) {
        const uint32_t j = load_index(t.idx, row * t.idx_stride + k, t.idx_type, cols) - start;
        if (j < n) atomicOr(&bm[j >> 5], 1u << (j & 31u));
    }
}

// bits of vector i (VEC of them) in the bitmap
template <uint32_t VEC>
__device__ __forceinline__ uint32_t kept_bits(const uint32_t *bm, uint32_t i) {
    const uint32_t b = ((const uint8_t *)bm)[i * VEC / 8];
    return VEC == 8 ? b : (b >> (i * VEC % 8)) & 0xfu;
}

// (maximum, sum) of a slice's columns not kept, formed from x - m, by reading
// the slice again: where nothing is left, where all lies near the lowest
// number, or where a maximum of bits was no more than an estimate.
template <uint32_t TYPE>
__device__ __forceinline__ float2 slice_again(const typename Num<TYPE>::T *p, uint32_t n, uint64_t avail,
                                              const uint32_t *bm, float c, float (*red)[DIST_THREADS / 64]) {
    constexpr uint32_t VEC = Num<TYPE>::VEC, STEP = DIST_THREADS * VEC;
    float mx = F_NEG_INF, sum = 0.f;
#pragma unroll 1
    for (uint32_t pass = 0; pass < 2; ++pass) {
        const float ref = mx == F_NEG_INF ? 0.f : mx;
#pragma unroll 1
        for (uint32_t e0 = threadIdx.x * VEC; e0 < n; e0 += STEP) {
            const Vec<TYPE> v = load_vec<TYPE, false>(p, e0, n, avail);
            const uint32_t b = kept_bits<VEC>(bm, e0 / VEC);
#pragma unroll
            for (uint32_t e = 0; e < VEC; ++e) {
                const float x = b >> e & 1u ? F_NEG_INF : v.get(e);
                if (pass == 0)
                    mx = fmaxf(mx, x);
                else
                    sum += exp2_fast((x - ref) * c);
            }
        }
        if (pass == 0)
            mx = block_max_f<DIST_THREADS>(mx, red[0]);
        else
            sum = block_sum_f<DIST_THREADS>(sum, red[1]);
    }
    return make_float2(mx, sum);
}

template <uint32_t TYPE, int NV>
__global__ __launch_bounds__(DIST_THREADS) void k_distill_slice(DistillArgs a) {
    using N = Num<TYPE>;
    constexpr uint32_t VEC = N::VEC, CAP = DIST_THREADS * NV * VEC;
    __shared__ uint32_t bm[CAP / 32];
    __shared__ float red[4][DIST_THREADS / 64];
    const uint64_t row = blockIdx.x / a.sl.n;
    const uint32_t s = blockIdx.x % a.sl.n, start = s * a.sl.len, n = min(a.sl.len, a.m.cols - start);
    if (a.weight && a.weight[row] == 0.f) return;
    const auto *p = (const typename N::T *)a.m.p + row * a.m.stride + start;
    const uint64_t avail = row_avail(a.m, row) - start;
    Vec<TYPE> v[NV];
    load_slice<TYPE, DIST_THREADS>(v, p, n, avail);
    for (uint32_t i = threadIdx.x; i < CAP / 32; i += DIST_THREADS) bm[i] = 0;
    lds_barrier();
    mark_kept(a.t, row, start, n, a.m.cols, bm);
    lds_barrier();
    uint32_t bits = Vec<TYPE>::max_bits_none();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t b = kept_bits<VEC>(bm, i * DIST_THREADS + threadIdx.x);
        if (b) {
#pragma unroll
            for (uint32_t e = 0; e < VEC; ++e)
                if (b >> e & 1u) v[i].mask(e);
        }
        bits = v[i].max_bits(bits);
    }
    const float mx = block_max_f<DIST_THREADS>(Vec<TYPE>::max_value(bits), red[0]);
    const Base2 to2(mx, a.c);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) sum += to2(v[i].get(e));
    sum = block_sum_f<DIST_THREADS>(sum, red[1]);
    float2 x = make_float2(mx, sum * to2.to(mx));
    if (!sum_in_range(sum)) x = slice_again<TYPE>(p, n, avail, bm, a.c, red + 2);
    if (threadIdx.x == 0) a.part[row * a.sl.n + s] = x;
}

// x 2^((a - b) c) for a sum x relative to a, wanted relative to b >= a
__device__ __forceinline__ float rescale(float x, float a, float b, float c) {
    return x == 0.f ? 0.f : x * exp2_fast((a - b) * c);
}

// A row's result from its columns not kept (m_tail, tail: their maximum and
// sum) and its kept entries, one per lane and step: student's logit x, teacher's
// y, `there` telling whether there is one.  All lanes of a wave take part.
struct RowResult {
    double loss;  // not yet times the weight
    float stats[6];
};
template <int NK>
__device__ __forceinline__ RowResult row_result(float m_tail, double tail, const float (&x)[NK], const float (&y)[NK],
                                                const bool (&there)[NK], float rest, float c, float inv_t) {
    float m_p = rest, m = m_tail;
#pragma unroll
    for (int i = 0; i < NK; ++i)
        if (there[i]) {
            m = fmaxf(m, x[i]);
            m_p = fmaxf(m_p, y[i] * inv_t);
        }
    m = wave_max_f(m);
    m_p = wave_max_f(m_p);
    // sums relative to m and m_p; d: the teacher's logit less the student's
    double sum_q = 0.0, sum_p = 0.0, sum_d = 0.0;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
        if (!there[i]) continue;
        if (x[i] != F_NEG_INF) sum_q += exp2_fast((x[i] - m) * c);
        const float e = y[i] == F_NEG_INF ? 0.f : expf(y[i] * inv_t - m_p);
        if (e > 0.f) {
            sum_p += e;
            sum_d += e * (((double)y[i] - (double)x[i]) * (double)inv_t);
        }
    }
    const double tail_q = tail == 0.0 ? 0.0 : tail * exp2_fast((m_tail - m) * c);
    sum_q = wave_sum_f64(sum_q) + tail_q;
    sum_p = wave_sum_f64(sum_p);
    sum_d = wave_sum_f64(sum_d);
    const float e_rest = rest == F_NEG_INF ? 0.f : expf(rest - m_p);
    sum_p += e_rest;
    RowResult r;
    r.loss = 0.0;
    // the columns not kept have gradient (w / t) a_tail exp((z - m_tail) / t)
    double a_tail = 0.0;
    if (sum_p > 0.0) {
        if (sum_q == 0.0 || (e_rest > 0.f && tail == 0.0)) {
            r.loss = __builtin_inf();
        } else {
            if (e_rest > 0.f) sum_d += e_rest * ((double)rest - ((double)m_tail * inv_t + ln_sum(tail)));
            // the terms' mean, less ln of one normaliser over the other
            r.loss = sum_d / sum_p - ((m_p + ln_sum(sum_p)) - ((double)m * inv_t + ln_sum(sum_q)));
        }
        if (tail > 0.0) a_tail = (tail_q / sum_q - e_rest / sum_p) / tail;
    }
    r.stats[0] = m;
    r.stats[1] = sum_q > 0.0 ? (float)(1.0 / sum_q) : 0.f;
    r.stats[2] = m_tail;
    r.stats[3] = (float)a_tail;
    r.stats[4] = m_p;
    r.stats[5] = sum_p > 0.0 ? (float)(1.0 / sum_p) : 0.f;
    return r;
}

// One wave per row joins its slices; NK entries per lane.
template <uint32_t TYPE, int NK>
__global__ __launch_bounds__(DIST_THREADS) void k_distill_join(DistillArgs a) {
    const uint32_t lane = threadIdx.x & 63u;
    const uint64_t row = (uint64_t)blockIdx.x * (DIST_THREADS / 64) + (threadIdx.x >> 6);
    if (row >= a.m.rows) return;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (lane == 0) a.loss[row] = 0.f;
        if (a.stats && lane < STATS) a.stats[row * STATS + lane] = 0.f;
        return;
    }
    const auto *z = (const typename Num<TYPE>::T *)a.m.p + row * a.m.stride;
    float x[NK], y[NK];
    bool there[NK];
    uint32_t j[NK];
#pragma unroll
    for (int i = 0; i < NK; ++i) {
        const uint32_t k = i * 64 + lane;
        j[i] = k < a.t.k ? load_index(a.t.idx, row * a.t.idx_stride + k, a.t.idx_type, a.m.cols) : a.m.cols;
    }
    const float2 first = lane < a.sl.n ? a.part[row * a.sl.n + lane] : make_float2(F_NEG_INF, 0.f);
    const float rest = a.t.rest ? a.t.rest[row] : F_NEG_INF;
#pragma unroll
    for (int i = 0; i < NK; ++i) {
        there[i] = j[i] < a.m.cols;
        x[i] = y[i] = 0.f;
        if (there[i]) {
            x[i] = num_float<TYPE>(z[j[i]]);
            y[i] = load_num(a.t.val, row * a.t.val_stride + i * 64 + lane, a.t.val_type);
        }
    }
    float m_tail = first.x;
    for (uint32_t i = lane + 64; i < a.sl.n; i += 64) m_tail = fmaxf(m_tail, a.part[row * a.sl.n + i].x);
    m_tail = wave_max_f(m_tail);
    double tail = rescale(first.y, first.x, m_tail, a.c);
    for (uint32_t i = lane + 64; i < a.sl.n; i += 64) {
        const float2 p = a.part[row * a.sl.n + i];
        tail += rescale(p.y, p.x, m_tail, a.c);
    }
    tail = wave_sum_f64(tail);
    const RowResult r = row_result<NK>(m_tail, tail, x, y, there, rest, a.c, a.inv_t);
    if (lane == 0) a.loss[row] = (float)(w * r.loss);
    if (a.stats && lane < STATS) {
        float st = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < 6; ++i) st = lane == i ? r.stats[i] : st;
        a.stats[row * STATS + lane] = st;
    }
}

template <uint32_t TYPE, int NV>
__global__ __launch_bounds__(DIST_THREADS) void k_distill_grad(DistillArgs a) {
    using N = Num<TYPE>;
    using T = typename N::T;
    constexpr uint32_t VEC = N::VEC, PER = MAX_TEACHER / DIST_THREADS;
    const uint64_t row = blockIdx.x / a.sl.n;
    const uint32_t s = blockIdx.x % a.sl.n, start = s * a.sl.len, n = min(a.sl.len, a.m.cols - start);
    T *out = (T *)a.grad + row * a.grad_stride + start;
    const float w = (a.weight ? a.weight[row] : 1.f), u = a.upstream ? a.upstream[row * a.upstream_stride] : 1.f;
    if (w == 0.f || u == 0.f) {
        const float zero[VEC] = {};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t e = (i * DIST_THREADS + threadIdx.x) * VEC;
            if (e < n) store_vec<TYPE>(out, e, n, zero);
        }
        return;
    }
    const T *p = (const T *)a.m.p + row * a.m.stride + start;
    const uint64_t avail = row_avail(a.m, row) - start;
    Vec<TYPE> v[NV];
    load_slice<TYPE, DIST_THREADS>(v, p, n, avail);
    const float *st = a.stats + row * STATS;
    const float m = st[0] == F_NEG_INF ? 0.f : st[0], m_tail = st[2] == F_NEG_INF ? 0.f : st[2];
    const float scale = w * u * a.inv_t, q = scale * st[1], f = scale * st[3];
    // the kept columns of this slice: read before any thread writes, written after all have
    uint32_t at[PER];
    float g[PER];
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) {
        const uint32_t k = i * DIST_THREADS + threadIdx.x;
        at[i] = n;
        if (k >= a.t.k) continue;
        const uint32_t j = load_index(a.t.idx, row * a.t.idx_stride + k, a.t.idx_type, a.m.cols) - start;
        if (j >= n) continue;
        const float x = num_float<TYPE>(p[j]), y = load_num(a.t.val, row * a.t.val_stride + k, a.t.val_type);
        const float e = y == F_NEG_INF ? 0.f : expf(y * a.inv_t - st[4]) * st[5];
        at[i] = j;
        g[i] = q * exp2_fast((x - m) * a.c) - scale * e;
    }
    __syncthreads();
    const Base2 to2(m_tail, a.c);
    const bool low = fabsf(m_tail * a.c) >= 1e30f;  // all near the lowest number
    const float f2 = f * to2.to(m_tail);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t e0 = (i * DIST_THREADS + threadIdx.x) * VEC;
        float x[VEC];
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e)
            x[e] = low ? f * exp2_fast((v[i].get(e) - m_tail) * a.c) : f2 * to2(v[i].get(e));
        if (e0 < n) store_vec<TYPE>(out, e0, n, x);
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i)
        if (at[i] < n) out[at[i]] = num_round<TYPE>(g[i]);
}

Slices distill_slices(const Matrix &m) {
    return plan_slices(m.rows, m.cols, 16 / type_bytes(m.type), DIST_THREADS, DIST_NV);
}

DistillArgs distill_args(const Matrix &m, const Teacher &t, float temperature, const float *weight) {
    DistillArgs a = {};
    a.m = m;
    a.t = t;
    a.sl = distill_slices(m);
    a.weight = weight;
    a.c = (float)(1.4426950408889634074 / temperature);
    a.inv_t = (float)(1.0 / temperature);
    return a;
}

template <uint32_t TYPE>
void slice_kernel(const DistillArgs &a, hipStream_t s) {
    const uint32_t grid = (uint32_t)(a.m.rows * a.sl.n);
    switch (a.sl.nv) {
        case 1: k_distill_slice<TYPE, 1><<<grid, DIST_THREADS, 0, s>>>(a); break;
        case 2: k_distill_slice<TYPE, 2><<<grid, DIST_THREADS, 0, s>>>(a); break;
        case 4: k_distill_slice<TYPE, 4><<<grid, DIST_THREADS, 0, s>>>(a); break;
        default: k_distill_slice<TYPE, 8><<<grid, DIST_THREADS, 0, s>>>(a); break;
    }
    trace_mark(s, "k_distill_slice");
}

template <uint32_t TYPE>
void join_kernel(const DistillArgs &a, hipStream_t s) {
    const uint32_t per = DIST_THREADS / 64, grid = (uint32_t)((a.m.rows + per - 1) / per);
    if (a.t.k <= 64)
        k_distill_join<TYPE, 1><<<grid, DIST_THREADS, 0, s>>>(a);
    else if (a.t.k <= 256)
        k_distill_join<TYPE, 4><<<grid, DIST_THREADS, 0, s>>>(a);
    else
        k_distill_join<TYPE, 16><<<grid, DIST_THREADS, 0, s>>>(a);
    trace_mark(s, "k_distill_join");
}

template <uint32_t TYPE>
void grad_kernel(const DistillArgs &a, hipStream_t s) {
    const uint32_t grid = (uint32_t)(a.m.rows * a.sl.n);
    switch (a.sl.nv) {
        case 1: k_distill_grad<TYPE, 1><<<grid, DIST_THREADS, 0, s>>>(a); break;
        case 2: k_distill_grad<TYPE, 2><<<grid, DIST_THREADS, 0, s>>>(a); break;
        case 4: k_distill_grad<TYPE, 4><<<grid, DIST_THREADS, 0, s>>>(a); break;
        default: k_distill_grad<TYPE, 8><<<grid, DIST_THREADS, 0, s>>>(a); break;
    }
    trace_mark(s, "k_distill_grad");
}

template <typename F>
hipError_t by_type(uint32_t type, F f) {
    if (type == TYPE_F32)
        f(std::integral_constant<uint32_t, TYPE_F32>{});
    else if (type == TYPE_BF16)
        f(std::integral_constant<uint32_t, TYPE_BF16>{});
    else
        f(std::integral_constant<uint32_t, TYPE_F16>{});
    return hipGetLastError();
}

// the slices' results, then (a step's) saved numbers
size_t part_bytes(const Matrix &m) { return (m.rows * distill_slices(m).n * sizeof(float2) + 255) / 256 * 256; }

}  // namespace

size_t distill_ws_bytes(uint64_t rows, uint64_t cols, uint32_t type) {
    const Matrix m = {nullptr, rows, cols, (uint32_t)cols, type};
    return part_bytes(m) + rows * STATS * sizeof(float);
}

hipError_t launch_distill_forward(const Matrix &m, const Teacher &t, float temperature, const float *weight,
                                  float *loss_out, float *stats_out, uint8_t *ws, hipStream_t s) {
    DistillArgs a = distill_args(m, t, temperature, weight);
    a.part = (float2 *)ws;
    a.loss = loss_out;
    a.stats = stats_out;
    return by_type(m.type, [&](auto type) {
        slice_kernel<decltype(type)::value>(a, s);
        join_kernel<decltype(type)::value>(a, s);
    });
}

hipError_t launch_distill_backward(const Matrix &m, const Teacher &t, float temperature, const float *weight,
                                   const float *upstream, uint64_t upstream_stride, const float *stats, void *grad,
                                   uint64_t grad_stride, hipStream_t s) {
    DistillArgs a = distill_args(m, t, temperature, weight);
    a.stats = const_cast<float *>(stats);
    a.upstream = upstream;
    a.upstream_stride = upstream_stride;
    a.grad = grad;
    a.grad_stride = grad_stride;
    return by_type(m.type, [&](auto type) { grad_kernel<decltype(type)::value>(a, s); });
}

hipError_t launch_distill_step(const Matrix &m, const Teacher &t, float temperature, const float *weight,
                               float *loss_out, void *grad, uint64_t grad_stride, uint8_t *ws, hipStream_t s) {
    float *stats = (float *)(ws + part_bytes(m));
    hipError_t e = launch_distill_forward(m, t, temperature, weight, loss_out, stats, ws, s);
    if (e != hipSuccess) return e;
    return launch_distill_backward(m, t, temperature, weight, nullptr, 0, stats, grad, grad_stride, s);
}

}  // namespace dr
