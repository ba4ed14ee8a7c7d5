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

// bits of vector i (VEC of them) in the bitmap, in the low places
template <uint32_t VEC>
__device__ __forceinline__ uint32_t kept_bits(const uint32_t *bm, uint32_t i) {
    const uint32_t b = ((const uint8_t *)bm)[i * VEC / 8];
    return VEC == 8 ? b : (b >> (i * VEC % 8)) & 0xfu;
}

// (maximum, sum) of a slice's columns not kept, formed from x - m, by reading
// the slice again: where nothing is left, or where all lies near the lowest
// number or the largest.
template <uint32_t TYPE, uint32_t THREADS>
__device__ __forceinline__ float2 slice_again(const typename Num<TYPE>::T *p, uint32_t n, uint64_t avail,
                                              const uint32_t *bm, float c, float (*red)[THREADS / 64]) {
    constexpr uint32_t VEC = Num<TYPE>::VEC, STEP = THREADS * VEC;
    float mx = F_NEG_INF, sum = 0.f;
#pragma unroll 1
    for (uint32_t pass = 0; pass < 2; ++pass) {
        const float ref = mx == F_NEG_INF ? 0.f : mx;
#pragma unroll 1
        for (uint32_t e0 = threadIdx.x * VEC; e0 < n; e0 += STEP) {
            const Vec<TYPE> v = load_vec<TYPE, false>(p, e0, n, avail);
            const uint32_t b = kept_bits<VEC>(bm, e0 / VEC);
            float x[VEC];
#pragma unroll
            for (uint32_t e = 0; e < VEC; ++e) {
                x[e] = b >> e & 1u ? F_NEG_INF : v.get(e);
                if (pass == 0)
                    mx = fmaxf(mx, x[e]);
                else
                    x[e] = exp2_fast((x[e] - ref) * c);
            }
            if (pass != 0) add_fours(sum, x);
        }
        if (pass == 0)
            mx = block_max_f<THREADS>(mx, red[0]);
        else
            sum = block_sum_f<THREADS>(sum, red[1]);
    }
    return make_float2(mx, sum);
}

// One slice by one block, held in registers from one read: maximum, then sum.
// Bound by memory: 1500 x 100003 float16: 47 us, 6.4 TB/s; the vector
// instructions alone take 27.
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
    Largest<TYPE> most;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * DIST_THREADS * VEC >= n) break;
        const uint32_t b = kept_bits<VEC>(bm, i * DIST_THREADS + threadIdx.x);
        if (b) v[i].mask(b);
        v[i].keep_packed();
        most.add(v[i]);
    }
    most.complete(v);
    const float mx = block_max_f<DIST_THREADS>(most.value(), red[0]);
    const Base2 to2(mx, a.c);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * DIST_THREADS * VEC >= n) break;
        v[i].keep_packed();
        float x[VEC];
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) x[e] = to2(v[i].get(e));
        add_fours(sum, x);
        asm volatile("" : "+v"(sum));  // one vector's numbers after the other
    }
    sum = block_sum_f<DIST_THREADS>(sum, red[1]);
    float2 x = make_float2(mx, sum * to2.to(mx));
    if (!sum_in_range(sum)) x = slice_again<TYPE, DIST_THREADS>(p, n, avail, bm, a.c, red + 2);
    if (threadIdx.x == 0) a.part[row * a.sl.n + s] = x;
}

// x 2^((a - b) c) for a sum x relative to a, wanted relative to b >= a
__device__ __forceinline__ float rescale(float x, float a, float b, float c) {
    return x == 0.f ? 0.f : x * exp2_fast((a - b) * c);
}

// A largest logit over the temperature, as a finite float (-inf of none).
__device__ __forceinline__ float quotient(float y0, float inv_t) {
    return y0 == F_NEG_INF ? y0 : fminf(fmaxf(y0 * inv_t, F_LOWEST), -F_LOWEST);
}
// A teacher's reference from which on its rounding to a float is more than an
// exponent takes: the quotient is the float itself then, and entries are
// compared with the largest one before they are divided.
constexpr float FAR_REFERENCE = 16777216.f;

// A row's result from its columns not kept (m_tail, tail: a reference at least
// near their maximum, and their sum relative to it) and its kept entries:
// entry(i, x, y) gives the lane's i-th of n, the student's logit x and the
// teacher's y, or tells that there is none.  stats[3] is times 2^size.  All
// lanes of a wave take part.
struct RowResult {
    double loss;  // not yet times the weight
    float stats[6];
};
template <typename ENTRY>
__device__ __forceinline__ RowResult row_result(float m_tail, double tail, uint32_t n, ENTRY entry, float rest, float c,
                                                float inv_t, int size = 0) {
    float y0 = F_NEG_INF, m = m_tail, x, y;
#pragma unroll
    for (uint32_t i = 0; i < n; ++i)
        if (entry(i, x, y)) {
            m = fmaxf(m, x);
            y0 = fmaxf(y0, y);
        }
    m = wave_max_f(m);
    y0 = wave_max_f(y0);
    // Sums relative to y0 and m; d: the entry's ln of p over q but for the
    // sums.  Logits are taken off one another before anything else, so that
    // large ones, a mask's lowest number say, leave no error of their size.
    double sum_q = 0.0, sum_p = 0.0, sum_d = 0.0;
#pragma unroll
    for (uint32_t i = 0; i < n; ++i) {
        if (!entry(i, x, y)) continue;
        if (x != F_NEG_INF) sum_q += exp2_fast((x - m) * c);
        const float e = y == F_NEG_INF ? 0.f : exp2_fast((y - y0) * c);
        if (e > 0.f) {
            sum_p += e;
            sum_d += e * ((((double)y - (double)y0) - ((double)x - (double)m)) * (double)inv_t);
        }
    }
    const double tail_q = tail == 0.0 ? 0.0 : tail * exp2_fast((m_tail - m) * c);
    sum_q = wave_sum_f64(sum_q) + tail_q;
    sum_p = wave_sum_f64(sum_p);
    sum_d = wave_sum_f64(sum_d);
    // The teacher's reference: the largest logit over the temperature, or rest.
    const float y0_f = quotient(y0, inv_t), m_p = fmaxf(y0_f, rest);
    const double y0_t = fabsf(m_p) < FAR_REFERENCE ? (double)y0 * (double)inv_t : (double)y0_f;
    const float y0_p = y0 == F_NEG_INF ? 0.f : exp_below((float)(y0_t - m_p));  // and now relative to m_p
    sum_d = y0_p > 0.f ? y0_p * (sum_d + (y0_t - m_p) * sum_p) : 0.0;
    sum_p *= y0_p;
    const float e_rest = rest == F_NEG_INF ? 0.f : exp_below(rest - m_p);
    sum_p += e_rest;
    RowResult r;
    r.loss = 0.0;
    // the columns not kept have gradient (w / t) a_tail exp((z - m_tail) / t)
    double a_tail = 0.0;
    if (sum_p > 0.0) {
        if (sum_q == 0.0 || (e_rest > 0.f && tail == 0.0)) {
            r.loss = __builtin_inf();
        } else {
            if (e_rest > 0.f)
                sum_d += e_rest * (((double)rest - m_p) - (((double)m_tail - m) * (double)inv_t + ln_sum(tail)));
            // the terms' mean, less ln of one sum over the other
            r.loss = sum_d / sum_p - (ln_sum(sum_p) - ln_sum(sum_q));
        }
        if (tail > 0.0) a_tail = (tail_q / sum_q - e_rest / sum_p) / tail;
    }
    r.stats[0] = m;
    r.stats[1] = sum_q > 0.0 ? (float)(1.0 / sum_q) : 0.f;
    r.stats[2] = m_tail;
    r.stats[3] = (float)ldexp(a_tail, size);
    r.stats[4] = m_p;
    r.stats[5] = sum_p > 0.0 ? (float)(1.0 / sum_p) : 0.f;
    return r;
}

// p of an entry with the teacher's logit y of a row whose largest is y0 (read
// where the reference is far alone), from the saved numbers.
__device__ __forceinline__ float entry_p(float y, float y0, float inv_t, float c, const float *stats) {
    if (y == F_NEG_INF) return 0.f;
    const float m_p = stats[4];
    if (fabsf(m_p) < FAR_REFERENCE) return exp_below(fmaf(y, inv_t, -m_p)) * stats[5];
    return exp2_fast((y - y0) * c) * exp_below(quotient(y0, inv_t) - m_p) * stats[5];
}

// One wave per row joins its slices; NK entries per lane.  Bound by latency (an
// index, then the logit it names): 6.5 us for 1500 rows of 100 entries, 3.8 for 16.
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
    const auto entry = [&](uint32_t i, float &student, float &teacher) {
        student = x[i];
        teacher = y[i];
        return there[i];
    };
    const RowResult r = row_result(m_tail, tail, NK, entry, rest, a.c, a.inv_t);
    if (lane == 0) a.loss[row] = (float)(w * r.loss);
    if (a.stats && lane < STATS) {
        float st = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < 6; ++i) st = lane == i ? r.stats[i] : st;
        a.stats[row * STATS + lane] = st;
    }
}

// The gradient of one slice by one block: f exp2(z c - R) everywhere, then the
// kept columns.  Bound by memory: 2048 x 65536 bfloat16: 95 us, 5.6 TB/s read and
// written; the vector instructions alone take 23.
template <uint32_t TYPE, int NV>
__global__ __launch_bounds__(DIST_THREADS) void k_distill_grad(DistillArgs a) {
    using N = Num<TYPE>;
    using T = typename N::T;
    constexpr uint32_t VEC = N::VEC, PER = MAX_TEACHER / DIST_THREADS;
    __shared__ float red[DIST_THREADS / 64];
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
    // no gradient where the teacher's row is no distribution
    const float scale = w * u * a.inv_t, q = st[5] > 0.f ? scale * st[1] : 0.f, f = scale * st[3];
    float y0 = F_NEG_INF;  // the row's, of all slices
    if (!(fabsf(st[4]) < FAR_REFERENCE)) {
        for (uint32_t k = threadIdx.x; k < a.t.k; k += DIST_THREADS)
            if (load_index(a.t.idx, row * a.t.idx_stride + k, a.t.idx_type, a.m.cols) < a.m.cols)
                y0 = fmaxf(y0, load_num(a.t.val, row * a.t.val_stride + k, a.t.val_type));
        y0 = block_max_f<DIST_THREADS>(y0, red);
    }
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
        at[i] = j;
        g[i] = q * exp2_fast((x - m) * a.c) - scale * entry_p(y, y0, a.inv_t, a.c, st);
    }
    __syncthreads();
    const Base2 to2(m_tail, a.c);
    const float f2 = f * to2.to(m_tail);
    const bool far = !(fabsf(m_tail * a.c) < BASE2_FAR);  // a mask's numbers, say: from x - m_tail
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t s0 = i * DIST_THREADS * VEC, e0 = s0 + threadIdx.x * VEC;
        if (s0 >= n) break;
        float x[VEC];
        if (far) {
#pragma unroll
            for (uint32_t e = 0; e < VEC; ++e) x[e] = f * exp2_fast((v[i].get(e) - m_tail) * a.c);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < VEC; ++e) x[e] = f2 * to2(v[i].get(e));
        }
        if (s0 + DIST_THREADS * VEC <= n)
            store_run<TYPE>(out + s0, x);
        else if (e0 < n)
            store_vec<TYPE>(out, e0, n, x);
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i)
        if (at[i] < n) out[at[i]] = num_round<TYPE>(g[i]);
}

// A step (GRAD), or the forward pass of a row that THREADS threads hold, of one
// row by one block.  A step's first RES vectors of every thread stay in
// registers from the sum to the gradient.  What a longer row has beyond
// them is read twice, MORE vectors at a time, the second time mostly from L2:
// blocks of 1024 threads have a CU each, and the second halves of the 32 rows of
// 131072 16-bit numbers that an XCD's CUs then hold are the 4 MiB of its L2
// (1.11 GB are read beyond it of the 1.01 that have to be, with 0.50 read
// twice).  The sum is relative to the largest kept logit, which is known before
// the row has arrived.  Bound by memory: 4096 x 131072 bfloat16: 403 us, 5.2
// TB/s of the logits' and the gradient's bytes (in a profiler's trace 415 at
// least and 435 on average); the vector instructions alone take 173.  Short rows
// by their latency: 256 x 32000 fp32, one row per CU: 16 us.
constexpr int RES = 8;

// Adds a run's numbers but for the kept columns, relative to a reference, and
// (MAX) takes their maximum; vector i THREADS + thread lies at bit (first +
// i THREADS + thread) VEC.
template <uint32_t TYPE, uint32_t THREADS, bool MAX, int NV>
__device__ __forceinline__ float sum_run(Vec<TYPE> (&v)[NV], uint32_t n, uint32_t first, const uint32_t *bm,
                                         const Base2 &to2, float sum, Largest<TYPE> &most) {
    constexpr uint32_t VEC = Num<TYPE>::VEC;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * THREADS * VEC >= n) break;
        const uint32_t b = kept_bits<VEC>(bm, first + i * THREADS + threadIdx.x);
        if (b) v[i].mask(b);
        v[i].keep_packed();
        if (MAX) most.add(v[i]);
        float x[VEC];
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) x[e] = to2(v[i].get(e));
        add_fours(sum, x);
        asm volatile("" : "+v"(sum));  // one vector's numbers after the other
    }
    return sum;
}

// Writes a run's gradients f exp2(z c - R).
template <uint32_t TYPE, uint32_t THREADS, int NV>
__device__ __forceinline__ void grad_run(Vec<TYPE> (&v)[NV], typename Num<TYPE>::T *out, uint32_t n, const Base2 &to2,
                                         float f) {
    constexpr uint32_t VEC = Num<TYPE>::VEC, STEP = THREADS * VEC;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t e0 = i * STEP + threadIdx.x * VEC;
        if (i * STEP >= n) break;
        v[i].keep_packed();
        float x[VEC];
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) x[e] = f * to2(v[i].get(e));
        if ((i + 1) * STEP <= n)
            store_run<TYPE>(out + i * STEP, x);
        else if (e0 < n)
            store_vec<TYPE>(out, e0, n, x);
    }
}

// The bounds on waves per SIMD: a step's short rows spill ten registers at eight
// (16000 x 4000 bfloat16: 80 us, 70 at seven); 512 threads, of which three blocks
// share a CU, spill two of 16-bit rows.
template <uint32_t TYPE, uint32_t THREADS, bool GRAD>
__global__ __launch_bounds__(THREADS, !GRAD ? 8 : THREADS < 512 ? 7 : 6) void k_distill_row(DistillArgs a) {
    using N = Num<TYPE>;
    using T = typename N::T;
    constexpr uint32_t VEC = N::VEC, STEP = THREADS * VEC, CHUNK = RES * STEP;
    constexpr int MORE = THREADS < 512 ? 2 : 4;
    extern __shared__ uint32_t bm[];  // a bit per column, then the kept entries:
    const uint32_t words = row_bitmap_words(a.m.cols, STEP);
    float *const ex = (float *)(bm + words), *const ey = ex + a.t.k;  // student's logit, teacher's
    uint32_t *const ej = (uint32_t *)(ey + a.t.k);                    // and column
    __shared__ float red[4][THREADS / 64];
    __shared__ float row_stats[6];
    const uint64_t row = blockIdx.x;
    const uint32_t n = a.m.cols;
    T *out = (T *)a.grad + row * a.grad_stride;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        const float zero[VEC] = {};
        for (uint32_t e = threadIdx.x * VEC; GRAD && e < n; e += STEP) store_vec<TYPE>(out, e, n, zero);
        if (threadIdx.x == 0) a.loss[row] = 0.f;
        if (!GRAD && a.stats && threadIdx.x < STATS) a.stats[row * STATS + threadIdx.x] = 0.f;
        return;
    }
    const T *p = (const T *)a.m.p + row * a.m.stride;
    const uint64_t avail = row_avail(a.m, row);
    const uint32_t held = min(n, CHUNK);
    Vec<TYPE> v[RES];
    load_slice<TYPE, THREADS>(v, p, held, avail);
    for (uint32_t i = threadIdx.x; i < words; i += THREADS) bm[i] = 0;
    float top = F_NEG_INF;
    for (uint32_t k = threadIdx.x; k < a.t.k; k += THREADS) {
        const uint32_t j = load_index(a.t.idx, row * a.t.idx_stride + k, a.t.idx_type, n);
        ej[k] = j;
        if (j < n) {
            ex[k] = num_float<TYPE>(p[j]);
            ey[k] = load_num(a.t.val, row * a.t.val_stride + k, a.t.val_type);
            top = fmaxf(top, ex[k]);
        }
    }
    top = block_max_f<THREADS>(top, red[0]);
    for (uint32_t k = threadIdx.x; k < a.t.k; k += THREADS)
        if (ej[k] < n) atomicOr(&bm[ej[k] >> 5], 1u << (ej[k] & 31u));
    lds_barrier();
    float ref = top > F_NEG_INF ? top : 0.f;
    const Base2 by_top(ref, a.c);
    Largest<TYPE> most;
    float sum = sum_run<TYPE, THREADS, !GRAD>(v, held, 0, bm, by_top, 0.f, most);
#pragma unroll 1
    for (uint32_t e0 = CHUNK; GRAD && e0 < n; e0 += MORE * STEP) {
        Vec<TYPE> u[MORE];
        load_slice<TYPE, THREADS, MORE, false>(u, p + e0, n - e0, avail - e0);
        sum = sum_run<TYPE, THREADS, false>(u, n - e0, e0 / VEC, bm, by_top, sum, most);
    }
    sum = block_sum_f<THREADS>(sum, red[1]);
    if (!GRAD) {  // the saved numbers are relative to the largest logit not kept
        most.complete(v);
        const float mx = block_max_f<THREADS>(most.value(), red[0]);
        ref = mx > F_NEG_INF ? mx : ref;
    }
    float tail = sum * by_top.to(ref);
    // where nearly all lies far below the reference, numbers that count would be below a float's range
    if (!(sum > 1e-26f && sum < 1e30f && tail > 1e-30f && tail < 1e30f)) {
        const float2 x = slice_again<TYPE, THREADS>(p, n, avail, bm, a.c, red + 2);
        ref = x.x;
        tail = x.y;
    }
    // the tail's power of two: a step's gradients are relative to it, so that they have a float's whole range
    const int size = GRAD && tail > 0.f ? __builtin_amdgcn_frexp_expf(tail) : 0;
    if (threadIdx.x < 64) {
        const auto entry = [&](uint32_t i, float &student, float &teacher) {
            const uint32_t k = i * 64 + threadIdx.x;
            if (k >= a.t.k || ej[k] >= n) return false;
            student = ex[k];
            teacher = ey[k];
            return true;
        };
        const RowResult r = row_result(ref, tail, (a.t.k + 63) / 64, entry, a.t.rest ? a.t.rest[row] : F_NEG_INF, a.c,
                                       a.inv_t, size);
        if (threadIdx.x == 0) a.loss[row] = (float)(w * r.loss);
        if (GRAD || a.stats) {
            float st = 0.f;
#pragma unroll
            for (uint32_t i = 0; i < 6; ++i) st = threadIdx.x == i ? r.stats[i] : st;
            if (!GRAD && threadIdx.x < STATS) a.stats[row * STATS + threadIdx.x] = st;
            if (GRAD && threadIdx.x < 6) row_stats[threadIdx.x] = st;
        }
    }
    if constexpr (!GRAD) return;
    lds_barrier();
    const float m = row_stats[0] == F_NEG_INF ? 0.f : row_stats[0], scale = w * a.inv_t;
    const float q = row_stats[5] > 0.f ? scale * row_stats[1] : 0.f;  // no gradient without a teacher's distribution
    ref = ref == F_NEG_INF ? 0.f : ref;
    // f 2^(z c - R) with R larger by `size` and f, too, as far as R's rounding lets it
    Base2 to2(ref, a.c);
    const float r = to2.r, f = scale * row_stats[3];
    to2.r += (float)size;
    const float f2 = ldexpf(f * Base2(ref, a.c).to(ref), (int)(to2.r - r) - size);
    if (!(fabsf(ref * a.c) < BASE2_FAR)) {  // a mask's numbers, say: from x - ref
#pragma unroll 1
        for (uint32_t e0 = threadIdx.x * VEC; e0 < n; e0 += STEP) {
            const Vec<TYPE> u = load_vec<TYPE, false>(p, e0, n, avail);
            float x[VEC];
#pragma unroll
            for (uint32_t e = 0; e < VEC; ++e) x[e] = f * exp2_fast((u.get(e) - ref) * a.c - (float)size);
            store_vec<TYPE>(out, e0, n, x);
        }
    } else {
        grad_run<TYPE, THREADS>(v, out, held, to2, f2);
#pragma unroll 1
        for (uint32_t e0 = CHUNK; e0 < n; e0 += MORE * STEP) {
            Vec<TYPE> u[MORE];
            load_slice<TYPE, THREADS>(u, p + e0, n - e0, avail - e0);
            grad_run<TYPE, THREADS>(u, out + e0, n - e0, to2, f2);
        }
    }
    float y0 = F_NEG_INF;
    if (!(fabsf(row_stats[4]) < FAR_REFERENCE)) {
        for (uint32_t k = threadIdx.x; k < a.t.k; k += THREADS)
            if (ej[k] < n) y0 = fmaxf(y0, ey[k]);
        y0 = block_max_f<THREADS>(y0, red[0]);
    }
    __syncthreads();  // the kept columns are written again
    for (uint32_t k = threadIdx.x; k < a.t.k; k += THREADS) {
        if (ej[k] >= n) continue;
        const float p_k = entry_p(ey[k], y0, a.inv_t, a.c, row_stats);
        out[ej[k]] = num_round<TYPE>(q * exp2_fast((ex[k] - m) * a.c) - scale * p_k);
    }
}

constexpr uint64_t SLICES = 512;  // that a call is to have, if shorter ones make them
Slices distill_slices(const Matrix &m) {
    return plan_slices(m.rows, m.cols, 16 / type_bytes(m.type), DIST_THREADS, DIST_NV, SLICES);
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

// Whether a step takes its rows one by one: where they are many, or so short
// that a block is through with one as soon as it would be with a slice; and a
// row's bitmap must fit beside its entries.  131072 bfloat16 columns, one by
// one and by slices: 64 rows 18 and 15 us, 128 rows 20 and 21, 256 rows 29 and
// 40; 32 rows of 32000: 9.6 and 10.5.
constexpr uint32_t ROW_MAX_COLS = 1u << 18;
constexpr uint64_t row_bytes(uint32_t cols, uint32_t type) { return (uint64_t)cols * type_bytes(type); }
bool step_by_rows(const Matrix &m) {
    return m.cols <= ROW_MAX_COLS && (m.rows >= 128 || row_bytes(m.cols, m.type) <= 65536);
}
// A forward pass gains by rows of up to 256 threads' registers, being one
// launch (4000 rows of 8000 bfloat16 columns: 20 us one by one, 24 by slices;
// of 32000: 55 and 53, all on logits in the cache).
constexpr bool forward_by_rows(uint32_t cols, uint32_t type) { return row_bytes(cols, type) <= 256 * RES * 16; }
static_assert(!forward_by_rows(1u << 30, TYPE_F32) && !forward_by_rows((1u << 30) + 8192, TYPE_F32) &&
                  !forward_by_rows(1u << 30, TYPE_BF16) && !forward_by_rows(0x7fffffffu, TYPE_F16) &&
                  forward_by_rows(8192, TYPE_F32) && !forward_by_rows(16385, TYPE_F16),
              "rows by their bytes, also where these pass 32 bits");

// A thread of a row's block adds a number for four of the row's, 64 at most.
static_assert(ROW_MAX_COLS <= 64 * 1024 * 4 && 16384 <= 64 * 256 * 4, "longest sums");

// Threads per row: as many as hold it in RES vectors each, but 512 up to twice
// that, where three blocks share a CU and one of 1024 threads would have it for
// itself (2048 x 65536 bfloat16: 103 us, and 122 with 1024).  At 256, 512 and
// 1024 threads, 4096 x 131072 takes 494, 420 and 403 us; at 64, 128 and 256,
// 30000 x 2000 takes 68, 86 and 117.
uint32_t row_threads(const Matrix &m) {
    const uint32_t vec = 16 / type_bytes(m.type), vecs = (m.cols + vec - 1) / vec;
    for (uint32_t t = 64; t <= 256; t *= 2)
        if (vecs <= t * RES) return t;
    return vecs <= 2 * 512 * RES ? 512 : 1024;
}
// Every thread of a step, also one beyond the row, finds its bits in the bitmap.
constexpr bool bitmap_holds_steps(uint32_t n, uint32_t threads, uint32_t vec) {
    const uint32_t step = threads * vec, last = (n - 1) / step * threads + threads - 1;  // the last thread's vector
    return (last + 1) * vec <= 32 * row_bitmap_words(n, step);
}
static_assert(bitmap_holds_steps(1, 64, 8) && bitmap_holds_steps(512, 64, 8) && bitmap_holds_steps(513, 64, 8) &&
                  bitmap_holds_steps(1, 64, 4) && bitmap_holds_steps(257, 64, 4) && bitmap_holds_steps(2001, 128, 4) &&
                  bitmap_holds_steps(16383, 256, 8) && bitmap_holds_steps(32000, 512, 4) &&
                  bitmap_holds_steps(40001, 512, 8) && bitmap_holds_steps(262143, 1024, 8),
              "bits of a row's last step");
template <uint32_t TYPE, bool GRAD>
void row_kernel(const DistillArgs &a, hipStream_t s) {
    const uint32_t grid = (uint32_t)a.m.rows, threads = row_threads(a.m);
    const uint32_t lds = 4 * (row_bitmap_words(a.m.cols, threads * (16 / type_bytes(TYPE))) + 3 * a.t.k);
    if (threads == 64)
        k_distill_row<TYPE, 64, GRAD><<<grid, 64, lds, s>>>(a);
    else if (threads == 128)
        k_distill_row<TYPE, 128, GRAD><<<grid, 128, lds, s>>>(a);
    else if (!GRAD || threads == 256)
        k_distill_row<TYPE, 256, GRAD><<<grid, 256, lds, s>>>(a);
    else if (threads == 512)
        k_distill_row<TYPE, 512, true><<<grid, 512, lds, s>>>(a);
    else
        k_distill_row<TYPE, 1024, true><<<grid, 1024, lds, s>>>(a);
    trace_mark(s, "k_distill_row");
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

uint64_t distill_threads(const Matrix &m) {
    return m.rows * std::max<uint64_t>(row_threads(m), (uint64_t)distill_slices(m).n * DIST_THREADS);
}

// For as many rows and columns or fewer: fewer rows are cut into more slices
// each, down to 512 in all, so that there are the longest slices of all rows,
// or less than twice 512.
size_t distill_ws_bytes(uint64_t rows, uint64_t cols, uint32_t type) {
    const uint64_t longest = (uint64_t)DIST_THREADS * DIST_NV * (16 / type_bytes(type));
    const uint64_t slices = std::max<uint64_t>(rows * ((cols + longest - 1) / longest), 2 * SLICES);
    return slices * sizeof(float2) + 256 + rows * STATS * sizeof(float);
}

hipError_t launch_distill_forward(const Matrix &m, const Teacher &t, float temperature, const float *weight,
                                  float *loss_out, float *stats_out, uint8_t *ws, hipStream_t s) {
    DistillArgs a = distill_args(m, t, temperature, weight);
    a.part = (float2 *)ws;
    a.loss = loss_out;
    a.stats = stats_out;
    if (forward_by_rows(m.cols, m.type))
        return by_type(m.type, [&](auto type) { row_kernel<decltype(type)::value, false>(a, s); });
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
    if (step_by_rows(m)) {
        DistillArgs a = distill_args(m, t, temperature, weight);
        a.loss = loss_out;
        a.grad = grad;
        a.grad_stride = grad_stride;
        return by_type(m.type, [&](auto type) { row_kernel<decltype(type)::value, true>(a, s); });
    }
    float *stats = (float *)(ws + part_bytes(m));
    hipError_t e = launch_distill_forward(m, t, temperature, weight, loss_out, stats, ws, s);
    if (e != hipSuccess) return e;
    return launch_distill_backward(m, t, temperature, weight, nullptr, 0, stats, grad, grad_stride, s);
}

}  // namespace dr
