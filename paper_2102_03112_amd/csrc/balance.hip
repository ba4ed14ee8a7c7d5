// balance.hip -- per-expert counts and the balance loss of a router, and its
// gradient.
//
// A row of logits is shared by LANES lanes (a power of two) that hold its
// 16-byte vectors, so a wave takes 64 / LANES rows at a time and a softmax is
// a few exchanges between lanes.  A lane adds the probabilities of its columns
// over all rows it meets in registers; blocks own runs of rows within one
// group, and their sums are joined by a second launch in a fixed order.
// Counts are whole numbers, gathered by LDS atomics, whose order cannot show.
#include <type_traits>

#include "launch.hpp"
#include "losses.hpp"

namespace dr {
namespace {

constexpr uint32_t BT = 256, BW = BT / 64;

struct BalanceArgs {
    Matrix m;
    Routes r;
    uint32_t parts, part_rows;  // blocks per group, rows per block (but the last)
    float coef;
    // groups of several blocks, per block: sums of probabilities and choices (E each), valid rows
    float *psum;
    uint32_t *pcount, *prows;
    double *gloss;     // per group: sum_e f P
    uint32_t *done;    // groups joined so far
    int32_t *counts_out, *rows_out;
    float *prob_out, *loss_out;
    // backward
    const int32_t *counts, *count_rows, *rows_in;
    const float *upstream;
    void *grad;
    uint64_t grad_stride;
};

template <uint32_t LANES>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (uint32_t o = 1; o < LANES; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
template <uint32_t LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (uint32_t o = 1; o < LANES; o <<= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// x := softmax of the row that the LANES lanes share; 0 where all is -inf
template <uint32_t LANES, uint32_t N>
__device__ __forceinline__ void row_softmax(float (&x)[N]) {
    float mx = x[0];
#pragma unroll
    for (uint32_t i = 1; i < N; ++i) mx = fmaxf(mx, x[i]);
    mx = lanes_max<LANES>(mx);
    mx = mx == F_NEG_INF ? 0.f : mx;
    float s = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
        x[i] = exp2_fast((x[i] - mx) * LOG2E);
        s += x[i];
    }
    s = lanes_sum<LANES>(s);
    const float inv = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) x[i] *= inv;
}

// The block's group and rows [first, end).
struct Rows {
    uint32_t group;
    uint64_t first, end;
};
__device__ __forceinline__ Rows block_rows(const BalanceArgs &a) {
    Rows b;
    b.group = blockIdx.x / a.parts;
    const uint64_t g0 = (uint64_t)b.group * a.r.group_rows, g1 = min(g0 + a.r.group_rows, a.m.rows);
    b.first = min(g0 + (uint64_t)(blockIdx.x % a.parts) * a.part_rows, g1);
    b.end = min(b.first + a.part_rows, g1);
    return b;
}

// One row's columns of this lane: NI vectors, lane-contiguous per vector.
template <uint32_t TYPE, uint32_t LANES, uint32_t NI>
__device__ __forceinline__ void load_row(const Matrix &m, uint64_t row, bool valid, uint32_t sub,
                                         float (&x)[NI * Num<TYPE>::VEC]) {
    constexpr uint32_t VEC = Num<TYPE>::VEC;
#pragma unroll
    for (uint32_t i = 0; i < NI; ++i) {
        Vec<TYPE> v;
        if (valid)
            v = load_vec<TYPE, false>((const typename Num<TYPE>::T *)m.p + row * m.stride, (i * LANES + sub) * VEC, m.cols,
                               row_avail(m, row));
        else
            v.fill_neg_inf();
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) x[i * VEC + e] = v.get(e);
    }
}

// One expert's outputs at place i = group E + e; adds count P to the loss.
__device__ __forceinline__ void put_column(const BalanceArgs &a, uint64_t i, uint32_t count, double p, double &loss) {
    a.counts_out[i] = (int32_t)count;
    if (a.prob_out) a.prob_out[i] = (float)p;
    loss += (double)count * p;
}

// The block's sum of the threads' losses (valid on thread 0).
__device__ __forceinline__ double block_loss(double loss, double *red) {
    loss = wave_sum_f64(loss);
    if ((threadIdx.x & 63u) == 0) red[threadIdx.x >> 6] = loss;
    __syncthreads();
    for (uint32_t i = 1; threadIdx.x == 0 && i < BW; ++i) loss += red[i];
    return loss;
}

// A group's outputs from sum_e count P (f = E count / (k n)); the only group's
// loss is the call's.
__device__ __forceinline__ void put_group(const BalanceArgs &a, uint32_t g, uint32_t n, double loss) {
    loss *= n ? (double)a.m.cols / ((double)a.r.k * n) : 0.0;
    a.rows_out[g] = (int32_t)n;
    if (a.r.groups == 1)
        a.loss_out[0] = (float)(a.coef * loss);
    else
        __hip_atomic_store(&a.gloss[g], loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <uint32_t TYPE, uint32_t LANES, uint32_t NI>
__global__ __launch_bounds__(BT) void k_balance_rows(BalanceArgs a) {
    constexpr uint32_t VEC = Num<TYPE>::VEC, N = NI * VEC, RPW = 64 / LANES, COLS = LANES * N;
    __shared__ float sums[BW][COLS];
    __shared__ uint32_t hist[MAX_EXPERTS];
    __shared__ uint32_t rows;
    __shared__ double red[BW];
    const uint32_t E = a.m.cols, lane = threadIdx.x & 63u, w = threadIdx.x >> 6, sub = lane % LANES;
    const Rows b = block_rows(a);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;
    for (uint32_t e = threadIdx.x; e < E; e += BT) hist[e] = 0;
    if (threadIdx.x == 0) rows = 0;
    float acc[N] = {};
    uint32_t n = 0;
    for (uint64_t r = b.first + w * RPW + lane / LANES; r - lane / LANES < b.end; r += BW * RPW) {
        const bool valid = r < b.end && (!a.r.mask || a.r.mask[r]);
        n += valid && sub == 0;
        float x[N];
        load_row<TYPE, LANES, NI>(a.m, r, valid, sub, x);
        row_softmax<LANES>(x);
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) acc[i] += x[i];
    }
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {  // the wave's rows
#pragma unroll
        for (uint32_t o = LANES; o < 64; o <<= 1) acc[i] += __shfl_xor(acc[i], o, 64);
    }
    if (lane < LANES) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) sums[w][(i / VEC * LANES + sub) * VEC + i % VEC] = acc[i];
    }
    n = wave_sum(n);
    lds_barrier();
    if (lane == 0 && n) atomicAdd(&rows, n);
    const uint32_t K = a.r.k, choices = (uint32_t)(b.end - b.first) * K;
    for (uint32_t i = threadIdx.x; i < choices; i += BT) {
        const uint64_t r = b.first + i / K;
        if (a.r.mask && !a.r.mask[r]) continue;
        const uint32_t e = load_index(a.r.idx, r * a.r.idx_stride + i % K, a.r.idx_type, E);
        if (e < E) atomicAdd(&hist[e], 1u);
    }
    lds_barrier();
    const uint64_t at = (uint64_t)blockIdx.x * E;
    const double inv = rows ? 1.0 / rows : 0.0;
    double loss = 0.0;
    for (uint32_t e = threadIdx.x; e < E; e += BT) {
        float s = sums[0][e];
#pragma unroll
        for (uint32_t i = 1; i < BW; ++i) s += sums[i][e];
        if (a.parts > 1) {
            a.psum[at + e] = s;
            a.pcount[at + e] = hist[e];
        } else {
            put_column(a, at + e, hist[e], s * inv, loss);
        }
    }
    if (a.parts > 1) {
        if (threadIdx.x == 0) a.prows[blockIdx.x] = rows;
        return;
    }
    loss = block_loss(loss, red);
    if (threadIdx.x == 0) put_group(a, b.group, rows, loss);
}

// The mean of the groups' losses, by one block.
__device__ __forceinline__ void put_mean(const BalanceArgs &a, double *red) {
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < a.r.groups; i += BT)
        s += __hip_atomic_load(&a.gloss[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s = block_loss(s, red);
    if (threadIdx.x == 0) a.loss_out[0] = a.r.groups ? (float)(a.coef / (double)a.r.groups * s) : 0.f;
}

__global__ __launch_bounds__(BT) void k_balance_mean(BalanceArgs a) {
    __shared__ double red[BW];
    put_mean(a, red);
}

// Groups of several blocks: one block joins each, and the last one to finish
// adds the groups' losses in their order.
__global__ __launch_bounds__(BT) void k_balance_join(BalanceArgs a) {
    __shared__ double sums[BT];
    __shared__ uint32_t counts[BT];
    __shared__ uint32_t rows;
    __shared__ double red[BW], mean_red[BW];
    __shared__ bool last;
    const uint32_t E = a.m.cols, g = blockIdx.x;
    const uint64_t b0 = (uint64_t)g * a.parts;
    if (threadIdx.x == 0) rows = 0;
    __syncthreads();
    uint32_t n = 0;
    for (uint32_t i = threadIdx.x; i < a.parts; i += BT) n += a.prows[b0 + i];
    n = wave_sum(n);
    if ((threadIdx.x & 63u) == 0 && n) atomicAdd(&rows, n);
    __syncthreads();
    n = rows;
    const double inv = n ? 1.0 / n : 0.0;
    // `width` columns at a time, the blocks' sums shared by BT / width threads
    uint32_t width = 1;
    while (width < E && width < BT) width *= 2;
    const uint32_t ways = BT / width, way = threadIdx.x / width;
    double loss = 0.0;
    for (uint32_t e0 = 0; e0 < E; e0 += width) {
        const uint32_t e = e0 + threadIdx.x % width;
        double s = 0.0;
        uint32_t c = 0;
        if (e < E) {
            for (uint32_t i = way; i < a.parts; i += ways) {
                s += a.psum[(b0 + i) * E + e];
                c += a.pcount[(b0 + i) * E + e];
            }
        }
        sums[threadIdx.x] = s;
        counts[threadIdx.x] = c;
        __syncthreads();
        if (way == 0 && e < E) {
            for (uint32_t i = 1; i < ways; ++i) {
                s += sums[threadIdx.x + i * width];
                c += counts[threadIdx.x + i * width];
            }
            put_column(a, (uint64_t)g * E + e, c, s * inv, loss);
        }
        __syncthreads();
    }
    loss = block_loss(loss, red);
    if (threadIdx.x == 0) {
        put_group(a, g, n, loss);
        last = a.r.groups > 1 &&
               __hip_atomic_fetch_add(a.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == a.r.groups - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    put_mean(a, mean_red);
}

template <uint32_t TYPE, uint32_t LANES, uint32_t NI>
__global__ __launch_bounds__(BT) void k_balance_grad(BalanceArgs a) {
    constexpr uint32_t VEC = Num<TYPE>::VEC, N = NI * VEC, RPW = 64 / LANES;
    using T = typename Num<TYPE>::T;
    const uint32_t E = a.m.cols, lane = threadIdx.x & 63u, w = threadIdx.x >> 6, sub = lane % LANES;
    const Rows b = block_rows(a);
    const int32_t n = a.rows_in[b.group], cn = a.count_rows[b.group];
    const float u = a.upstream ? *a.upstream : 1.f;
    const float scale = n > 0 ? (float)((double)u * a.coef / ((double)a.r.groups * n)) : 0.f;
    const float per = cn > 0 ? (float)((double)E / ((double)a.r.k * cn)) : 0.f;
    float f[N];
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
        const uint32_t e = (i / VEC * LANES + sub) * VEC + i % VEC;
        f[i] = e < E ? a.counts[(uint64_t)b.group * E + e] * per : 0.f;
    }
    for (uint64_t r = b.first + w * RPW + lane / LANES; r - lane / LANES < b.end; r += BW * RPW) {
        const bool there = r < b.end, valid = there && (!a.r.mask || a.r.mask[r]);
        float x[N];
        load_row<TYPE, LANES, NI>(a.m, r, valid, sub, x);
        row_softmax<LANES>(x);
        float dot = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) dot += x[i] * f[i];
        dot = lanes_sum<LANES>(dot);
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) x[i] = valid ? scale * x[i] * (f[i] - dot) : 0.f;
        if (there) {
#pragma unroll
            for (uint32_t i = 0; i < NI; ++i) {
                const uint32_t e = (i * LANES + sub) * VEC;
                if (e < E) store_vec<TYPE, false>((T *)a.grad + r * a.grad_stride, e, E, x + i * VEC);
            }
        }
    }
}

// How a type's rows lie over lanes, and the blocks that a call takes.
struct Shape {
    uint32_t lanes, ni, parts, part_rows;
};
Shape plan_rows(uint64_t rows, uint32_t experts, uint32_t type, uint32_t group_rows) {
    Shape s;
    const uint32_t vec = 16 / type_bytes(type), vecs = (experts + vec - 1) / vec;
    s.lanes = 1;
    while (s.lanes < 64 && s.lanes < vecs) s.lanes *= 2;
    s.ni = (vecs + 63) / 64;
    const uint64_t groups = rows ? (rows + group_rows - 1) / group_rows : 0;
    const uint64_t own = std::min<uint64_t>(rows, group_rows), step = BW * (64 / s.lanes);
    // four blocks per CU in all, but two rounds of a block's waves at least
    uint64_t parts = std::max<uint64_t>(1, 1024 / std::max<uint64_t>(1, groups));
    parts = std::max<uint64_t>(1, std::min(parts, own / (2 * step)));
    const uint64_t per = own ? (own + parts - 1) / parts : 1;
    s.part_rows = (uint32_t)((per + step - 1) / step * step);
    s.parts = (uint32_t)std::max<uint64_t>(1, (own + s.part_rows - 1) / s.part_rows);
    return s;
}

template <uint32_t TYPE, bool GRAD, uint32_t LANES, uint32_t NI>
void rows_kernel(const BalanceArgs &a, uint32_t grid, hipStream_t s) {
    if (GRAD)
        k_balance_grad<TYPE, LANES, NI><<<grid, BT, 0, s>>>(a);
    else
        k_balance_rows<TYPE, LANES, NI><<<grid, BT, 0, s>>>(a);
    trace_mark(s, GRAD ? "k_balance_grad" : "k_balance_rows");
}

template <uint32_t TYPE, bool GRAD>
void rows_launch(const BalanceArgs &a, const Shape &sh, hipStream_t s) {
    const uint32_t grid = a.r.groups * sh.parts;
    switch (sh.lanes) {
        case 1: return rows_kernel<TYPE, GRAD, 1, 1>(a, grid, s);
        case 2: return rows_kernel<TYPE, GRAD, 2, 1>(a, grid, s);
        case 4: return rows_kernel<TYPE, GRAD, 4, 1>(a, grid, s);
        case 8: return rows_kernel<TYPE, GRAD, 8, 1>(a, grid, s);
        case 16: return rows_kernel<TYPE, GRAD, 16, 1>(a, grid, s);
        case 32: return rows_kernel<TYPE, GRAD, 32, 1>(a, grid, s);
    }
    if (sh.ni == 1) return rows_kernel<TYPE, GRAD, 64, 1>(a, grid, s);
    if (sh.ni == 2) return rows_kernel<TYPE, GRAD, 64, 2>(a, grid, s);
    if constexpr (TYPE == TYPE_F32) {  // up to MAX_EXPERTS of 4 a vector
        if (sh.ni == 3) return rows_kernel<TYPE, GRAD, 64, 3>(a, grid, s);
        return rows_kernel<TYPE, GRAD, 64, 4>(a, grid, s);
    }
}

template <bool GRAD>
hipError_t rows_dispatch(const BalanceArgs &a, const Shape &sh, hipStream_t s) {
    if (a.m.type == TYPE_F32)
        rows_launch<TYPE_F32, GRAD>(a, sh, s);
    else if (a.m.type == TYPE_BF16)
        rows_launch<TYPE_BF16, GRAD>(a, sh, s);
    else
        rows_launch<TYPE_F16, GRAD>(a, sh, s);
    return hipGetLastError();
}

BalanceArgs balance_args(const Matrix &m, const Routes &r, float coef, const Shape &sh) {
    BalanceArgs a = {};
    a.m = m;
    a.r = r;
    a.parts = sh.parts;
    a.part_rows = sh.part_rows;
    a.coef = coef;
    return a;
}

}  // namespace

// Results are kept per block where groups have several (at most 1024 blocks
// then), and a loss per group where there are several.
size_t balance_ws_bytes(uint64_t rows, uint64_t experts) {
    return 256 + 8 * rows + 1024 * (8 * experts + 4);
}

hipError_t launch_balance_forward(const Matrix &m, const Routes &r, float coef, int32_t *counts_out,
                                  int32_t *rows_out, float *prob_out, float *loss_out, uint8_t *ws, hipStream_t s) {
    const Shape sh = plan_rows(m.rows, m.cols, m.type, r.group_rows);
    BalanceArgs a = balance_args(m, r, coef, sh);
    const uint64_t blocks = (uint64_t)r.groups * sh.parts;
    a.done = (uint32_t *)ws;
    a.gloss = (double *)(ws + 256);
    a.psum = (float *)(a.gloss + r.groups);
    a.pcount = (uint32_t *)(a.psum + blocks * m.cols);
    a.prows = a.pcount + blocks * m.cols;
    a.counts_out = counts_out;
    a.rows_out = rows_out;
    a.prob_out = prob_out;
    a.loss_out = loss_out;
    if (r.groups) {
        hipError_t e = rows_dispatch<false>(a, sh, s);
        if (e != hipSuccess) return e;
    }
    if (sh.parts > 1) {
        k_balance_join<<<r.groups, BT, 0, s>>>(a);
        trace_mark(s, "k_balance_join");
    } else if (r.groups != 1) {
        k_balance_mean<<<1, BT, 0, s>>>(a);
        trace_mark(s, "k_balance_mean");
    }
    return hipGetLastError();
}

hipError_t launch_balance_backward(const Matrix &m, const Routes &r, float coef, const int32_t *counts,
                                   const int32_t *count_rows, const int32_t *rows_in, const float *upstream,
                                   void *grad, uint64_t grad_stride, hipStream_t s) {
    if (!r.groups) return hipSuccess;
    const Shape sh = plan_rows(m.rows, m.cols, m.type, r.group_rows);
    BalanceArgs a = balance_args(m, r, coef, sh);
    a.counts = counts;
    a.count_rows = count_rows;
    a.rows_in = rows_in;
    a.upstream = upstream;
    a.grad = grad;
    a.grad_stride = grad_stride;
    return rows_dispatch<true>(a, sh, s);
}

}  // namespace dr
