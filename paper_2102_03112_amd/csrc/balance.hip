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
    // groups of several blocks: (sum of probabilities, choices) per block and expert, valid rows per block
    uint2 *partial;
    uint32_t *prows;
    uint32_t col_blocks;  // joining blocks per group
    double *gloss;        // sum_e f P per group, or per joining block
    unsigned long long *total;  // not null: the sum of all joining blocks' and their number
    int32_t *counts_out, *rows_out;
    float *prob_out, *loss_out;
    // backward
    const int32_t *counts, *count_rows, *rows_in;
    const float *upstream;
    void *grad;
    uint64_t grad_stride;
};

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
    const float inv = s == 0.f ? 0.f : __builtin_amdgcn_rcpf(s);  // within 1 ulp
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

// A lane's columns of U rows, `apart` rows from one to the next: NI vectors a
// row.  All are loaded before any is used.
template <uint32_t TYPE, uint32_t LANES, uint32_t NI, uint32_t U>
struct RowBatch {
    static constexpr uint32_t VEC = Num<TYPE>::VEC;
    Vec<TYPE> v[U][NI];
    bool valid[U];

    __device__ __forceinline__ void load(const BalanceArgs &a, uint64_t row, uint64_t end, uint32_t apart,
                                         uint32_t sub) {
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint64_t r = row + u * apart;
            valid[u] = r < end && (!a.r.mask || a.r.mask[r]);
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint64_t r = row + u * apart;
#pragma unroll
            for (uint32_t i = 0; i < NI; ++i) {
                v[u][i].fill_neg_inf();
                if (valid[u])
                    v[u][i] = load_vec<TYPE>((const typename Num<TYPE>::T *)a.m.p + r * a.m.stride,
                                                    (i * LANES + sub) * VEC, a.m.cols, row_avail(a.m, r));
            }
        }
    }
    __device__ __forceinline__ void get(uint32_t u, float (&x)[NI * VEC]) const {
#pragma unroll
        for (uint32_t i = 0; i < NI * VEC; ++i) x[i] = v[u][i / VEC].get(i % VEC);
    }
};
// rows a lane holds at once: 12 or 16 registers
template <uint32_t NI>
constexpr uint32_t ROWS_AT_ONCE = NI == 1 ? 4 : NI == 2 ? 2 : 1;

// One expert's outputs at place i = group E + e; adds count P to the loss.
__device__ __forceinline__ void put_column(const BalanceArgs &a, uint64_t i, uint32_t count, double p, double &loss) {
    a.counts_out[i] = (int32_t)count;
    if (a.prob_out) a.prob_out[i] = (float)p;
    loss += (double)count * p;
}

// The block's sum of the threads' losses (valid on thread 0).
template <uint32_t THREADS>
__device__ __forceinline__ double block_loss(double loss, double *red) {
    loss = wave_sum_f64(loss);
    if ((threadIdx.x & 63u) == 0) red[threadIdx.x >> 6] = loss;
    __syncthreads();
    for (uint32_t i = 1; threadIdx.x == 0 && i < THREADS / 64; ++i) loss += red[i];
    return loss;
}

// sum_e f P from sum_e count P, with f = E count / (k n)
__device__ __forceinline__ double group_factor(const BalanceArgs &a, uint32_t n) {
    return n ? (double)a.m.cols / ((double)a.r.k * n) : 0.0;
}

// Sums and counts of a block's rows.  Bound by memory where rows are many: 131072
// x 256 fp32: 27 us, 5.1 TB/s; the vector instructions alone take 14.  Else by
// latency (load, softmax, counts in turn): 16384 x 64 bfloat16: 5.3 us.
// A lane adds up to FOLD rows in 32 bits; in blocks with more rows a lane (DEEP:
// of groups that are many and long) what each FOLD of them give is added in 64.
constexpr uint32_t FOLD = 64;
template <uint32_t TYPE, uint32_t LANES, uint32_t NI, bool DEEP>
__global__ __launch_bounds__(BT) void k_balance_rows(BalanceArgs a) {
    constexpr uint32_t VEC = Num<TYPE>::VEC, N = NI * VEC, RPW = 64 / LANES, COLS = LANES * N;
    constexpr uint32_t U = ROWS_AT_ONCE<NI>;
    using Sum = std::conditional_t<DEEP, double, float>;
    __shared__ Sum sums[BW][COLS];
    __shared__ uint32_t hist[MAX_EXPERTS];
    __shared__ uint32_t rows;
    __shared__ double red[BW];
    const uint32_t E = a.m.cols, lane = threadIdx.x & 63u, w = threadIdx.x >> 6, sub = lane % LANES;
    const Rows b = block_rows(a);
    for (uint32_t e = threadIdx.x; e < E; e += BT) hist[e] = 0;
    if (threadIdx.x == 0) rows = 0;
    if (blockIdx.x == 0 && a.total) {  // of the launch after this one
        if (threadIdx.x == 0) *a.total = 0;
        if (threadIdx.x < a.r.groups * a.col_blocks) a.gloss[threadIdx.x] = 0.0;
    }
    float acc[N] = {};
    uint32_t n = 0, added = 0;
    const auto fold = [&](bool first) {  // the wave's rows; a lane's own places
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) acc[i] = groups_sum<LANES>(acc[i]);
        if (lane < LANES) {
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) {
                Sum &s = sums[w][(i / VEC * LANES + sub) * VEC + i % VEC];
                s = first ? acc[i] : s + acc[i];
            }
        }
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) acc[i] = 0.f;
    };
    for (uint64_t r = b.first + w * RPW + lane / LANES; r - lane / LANES < b.end; r += U * BW * RPW) {
        RowBatch<TYPE, LANES, NI, U> rows_now;
        rows_now.load(a, r, b.end, BW * RPW, sub);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            if (r - lane / LANES + u * BW * RPW >= b.end) break;
            n += rows_now.valid[u] && sub == 0;
            float x[N];
            rows_now.get(u, x);
            row_softmax<LANES>(x);
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) acc[i] += x[i];
        }
        if constexpr (DEEP) {
            added += U;
            if (added % FOLD == 0) fold(added == FOLD);
        }
    }
    fold(added < FOLD);
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
        Sum s = sums[0][e];
#pragma unroll
        for (uint32_t i = 1; i < BW; ++i) s += sums[i][e];
        if (a.parts > 1) {
            a.partial[at + e] = make_uint2(__float_as_uint((float)s), hist[e]);
        } else {
            put_column(a, at + e, hist[e], s * inv, loss);
        }
    }
    if (a.parts > 1) {
        if (threadIdx.x == 0) a.prows[blockIdx.x] = rows;
        return;
    }
    loss = block_loss<BT>(loss, red);
    if (threadIdx.x == 0) {
        loss *= group_factor(a, rows);
        a.rows_out[b.group] = (int32_t)rows;
        if (a.r.groups == 1)
            a.loss_out[0] = (float)(a.coef * loss);
        else
            a.gloss[b.group] = loss;
    }
}

// Groups of several blocks: joined JOIN_COLS columns a block, so that the
// partial sums of a large batch (1024 blocks x 256 experts: 2 MiB) are read by
// many; every block counts the group's rows for itself.  One group of up to 256
// blocks and ONE_JOIN_COLS experts is joined by a single block, which has the
// loss, too (2048 x 64: 8.0 us for the forward pass, 8.7 by columns; 16384 x 64,
// 256 blocks: 9.4 and 9.4).  Bound by latency: 4.8 us.
constexpr uint32_t JOIN_COLS = 16, ONE_JOIN_COLS = 64;

// The loss from those of up to MAX_ADDING joining blocks, without a launch for
// it: added as whole numbers of 2^-LOSS_BITS, whose order cannot show, above two
// counts, of the blocks and of those that left their loss in a place of its
// own instead; one atomic operation adds a block's loss and tells the last block
// that it is.  A loss from 2^-13 on is then rounded by 2^-27 of itself at most;
// a smaller one, or one that is NaN, is left, in 64 bits, and the last block adds
// what was left in the blocks' order.  (Blocks of 16 experts: 64 blocks' groups
// times experts are 2^10 at most, and so is the sum of all f P, which takes 50
// bits.)  Leaving is an atomic operation, too, so that it takes place where
// every block sees it; it is done when it returns, and the count's operand is
// made from what it returned.  Each operation on the one word takes some 10 ns,
// so that more blocks leave their losses to a launch (131072 x 256: 16 blocks 4
// us less than with that launch, 512 blocks 5 us more).
constexpr uint32_t MAX_ADDING = 64, LOSS_BITS = 39, COUNT_BITS = 7;
__device__ __forceinline__ void add_losses(const BalanceArgs &a, double loss) {  // the first wave; loss: lane 0's
    constexpr double ONE = (double)(1ull << LOSS_BITS), SMALL = 1.0 / 8192;
    constexpr unsigned long long COUNT = (1ull << COUNT_BITS) - 1;
    auto *const left = (unsigned long long *)a.gloss;
    const uint32_t lane = threadIdx.x;
    unsigned long long sum = 0;
    uint32_t last = 0;  // 1: this block is the last one, 2: and others left their loss
    if (lane == 0) {
        unsigned long long add = 1;
        if (loss >= SMALL) {
            add |= (unsigned long long)(loss * ONE + 0.5) << 2 * COUNT_BITS;
        } else if (loss != 0.0) {
            const unsigned long long was = atomicExch(&left[blockIdx.x], __builtin_bit_cast(unsigned long long, loss));
            uint32_t one;
            asm volatile("v_mov_b32 %0, 1" : "=v"(one) : "v"((uint32_t)was));
            add = one << COUNT_BITS | one;
        }
        sum = atomicAdd(a.total, add) + add;
        if ((sum & COUNT) == gridDim.x) last = sum >> COUNT_BITS & COUNT ? 2 : 1;
    }
    last = __builtin_amdgcn_readfirstlane(last);
    if (last == 0) return;
    double more = 0.0;
    if (last == 2) {
        more = lane < gridDim.x ? __builtin_bit_cast(double, atomicAdd(&left[lane], 0ull)) : 0.0;
        more = wave_sum_f64(more);
    }
    if (lane == 0)
        a.loss_out[0] = (float)(a.coef / (double)a.r.groups * ((double)(sum >> 2 * COUNT_BITS) / ONE + more));
}

template <uint32_t JT, uint32_t JOIN_COLS>
__global__ __launch_bounds__(JT) void k_balance_join(BalanceArgs a) {
    constexpr uint32_t JOIN_WAYS = JT / JOIN_COLS;
    __shared__ double sums[JOIN_WAYS][JOIN_COLS];
    __shared__ uint32_t counts[JOIN_WAYS][JOIN_COLS];
    __shared__ uint32_t rows;
    __shared__ double red[JT / 64];
    const uint32_t E = a.m.cols, way = threadIdx.x / JOIN_COLS, col = threadIdx.x % JOIN_COLS;
    const uint32_t g = blockIdx.x / a.col_blocks, e = blockIdx.x % a.col_blocks * JOIN_COLS + col;
    const uint64_t b0 = (uint64_t)g * a.parts;
    if (threadIdx.x == 0) rows = 0;
    double s = 0.0;
    uint32_t c = 0, n = 0;
    for (uint32_t i = threadIdx.x; i < a.parts; i += JT) n += a.prows[b0 + i];
    if (e < E) {
#pragma unroll 4
        for (uint32_t i = way; i < a.parts; i += JOIN_WAYS) {
            const uint2 x = a.partial[(b0 + i) * E + e];
            s += __uint_as_float(x.x);
            c += x.y;
        }
    }
    sums[way][col] = s;
    counts[way][col] = c;
    __syncthreads();
    n = wave_sum(n);
    if ((threadIdx.x & 63u) == 0 && n) atomicAdd(&rows, n);
    __syncthreads();
    n = rows;
    double loss = 0.0;
    if (way == 0) {
        for (uint32_t i = 1; i < JOIN_WAYS; ++i) {
            s += sums[i][col];
            c += counts[i][col];
        }
        if (e < E) put_column(a, (uint64_t)g * E + e, c, n ? s / n : 0.0, loss);
    }
    loss = block_loss<JT>(loss, red) * group_factor(a, n);
    if (threadIdx.x == 0) {
        if (blockIdx.x % a.col_blocks == 0) a.rows_out[g] = (int32_t)n;
        if (gridDim.x == 1)
            a.loss_out[0] = (float)(a.coef * loss);
        else if (!a.total)
            a.gloss[blockIdx.x] = loss;
    }
    if (a.total && threadIdx.x < 64) add_losses(a, loss);
}

// The mean over groups, from n parts of their losses: a launch's 4.4 us.
__global__ __launch_bounds__(BT) void k_balance_mean(BalanceArgs a, uint32_t n) {
    __shared__ double red[BW];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += BT) s += a.gloss[i];
    s = block_loss<BT>(s, red);
    if (threadIdx.x == 0) a.loss_out[0] = a.r.groups ? (float)(a.coef / (double)a.r.groups * s) : 0.f;
}

// The gradient of a block's rows.  Bound by memory: 131072 x 256 fp32: 47 us, 5.7
// TB/s read and written; the vector instructions alone take 31.
template <uint32_t TYPE, uint32_t LANES, uint32_t NI>
__global__ __launch_bounds__(BT) void k_balance_grad(BalanceArgs a) {
    constexpr uint32_t VEC = Num<TYPE>::VEC, N = NI * VEC, RPW = 64 / LANES;
    constexpr uint32_t U = ROWS_AT_ONCE<NI>;
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
    for (uint64_t r0 = b.first + w * RPW + lane / LANES; r0 - lane / LANES < b.end; r0 += U * BW * RPW) {
        RowBatch<TYPE, LANES, NI, U> rows_now;
        rows_now.load(a, r0, b.end, BW * RPW, sub);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            const uint64_t r = r0 + u * BW * RPW;
            if (r - lane / LANES >= b.end) break;
            float x[N];
            rows_now.get(u, x);
            row_softmax<LANES>(x);
            float dot = 0.f;
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) dot += x[i] * f[i];
            dot = lanes_sum<LANES>(dot);
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) x[i] = rows_now.valid[u] ? scale * x[i] * (f[i] - dot) : 0.f;
            if (r < b.end) {
#pragma unroll
                for (uint32_t i = 0; i < NI; ++i) {
                    const uint32_t e = (i * LANES + sub) * VEC;
                    if (e < E) store_vec<TYPE>((T *)a.grad + r * a.grad_stride, e, E, x + i * VEC);
                }
            }
        }
    }
}

// How a type's rows lie over lanes, and the blocks that a call takes.
struct Shape {
    uint32_t lanes, ni, parts, part_rows;
};
constexpr uint32_t MAX_PARTS = 1024, MAX_GRAD_PARTS = 4096;
Shape plan_rows(uint64_t rows, uint32_t experts, uint32_t type, uint32_t group_rows, bool grad) {
    Shape s;
    const uint32_t vec = 16 / type_bytes(type), vecs = (experts + vec - 1) / vec;
    // Forward: eight lanes, a line of 128 bytes, for up to four vectors each, so
    // that exchanges between lanes serve several rows at once (262144 x 256
    // bfloat16: 41 us, 45 with a lane per vector).  Backward: a lane per vector up
    // to 64 (58 us, and 77 by eight lanes, whose stores come in more pieces).
    s.lanes = 1;
    while (grad ? s.lanes < 64 && s.lanes < vecs : s.lanes < 8 ? s.lanes < vecs : s.lanes * 4 < vecs) s.lanes *= 2;
    s.ni = (vecs + s.lanes - 1) / s.lanes;
    const uint64_t groups = rows ? (rows + group_rows - 1) / group_rows : 0;
    const uint64_t own = std::min<uint64_t>(rows, group_rows), step = BW * (64 / s.lanes);
    // Four blocks per CU in all, whose sums are to be joined, but two rounds of a
    // block's waves at least.  Backward, where there is nothing to join, up to four
    // times as many, which take turns to load and to store, if they have eight
    // rounds each, so that f is worth its reading (131072 x 256 fp32: 48 us, 57
    // with 1024 blocks; 65536 x 256 bfloat16: 17, and 27 as blocks of two rounds).
    const auto blocks = [&](uint64_t most, uint64_t rounds) {
        return std::max<uint64_t>(1, std::min(most / std::max<uint64_t>(1, groups), own / (rounds * step)));
    };
    const uint64_t parts = grad ? std::max(blocks(MAX_PARTS, 2), blocks(MAX_GRAD_PARTS, 8)) : blocks(MAX_PARTS, 2);
    const uint64_t per = own ? (own + parts - 1) / parts : 1;
    s.part_rows = (uint32_t)((per + step - 1) / step * step);
    s.parts = (uint32_t)std::max<uint64_t>(1, (own + s.part_rows - 1) / s.part_rows);
    return s;
}

template <uint32_t TYPE, bool GRAD, uint32_t LANES, uint32_t NI>
void rows_kernel(const BalanceArgs &a, uint32_t grid, hipStream_t s) {
    if constexpr (GRAD)
        k_balance_grad<TYPE, LANES, NI><<<grid, BT, 0, s>>>(a);
    else if (a.part_rows > FOLD * BW * (64 / LANES))
        k_balance_rows<TYPE, LANES, NI, true><<<grid, BT, 0, s>>>(a);
    else
        k_balance_rows<TYPE, LANES, NI, false><<<grid, BT, 0, s>>>(a);
    trace_mark(s, GRAD ? "k_balance_grad" : "k_balance_rows");
}

// MAX_EXPERTS of 16 bits are 128 vectors, of 32 bits 256
template <uint32_t TYPE, bool GRAD>
void rows_launch(const BalanceArgs &a, const Shape &sh, hipStream_t s) {
    const uint32_t grid = a.r.groups * sh.parts, shape = sh.lanes * 8 + sh.ni;
    switch (shape) {
        case 1 * 8 + 1: return rows_kernel<TYPE, GRAD, 1, 1>(a, grid, s);
        case 2 * 8 + 1: return rows_kernel<TYPE, GRAD, 2, 1>(a, grid, s);
        case 4 * 8 + 1: return rows_kernel<TYPE, GRAD, 4, 1>(a, grid, s);
        case 8 * 8 + 1: return rows_kernel<TYPE, GRAD, 8, 1>(a, grid, s);
    }
    if constexpr (GRAD) {
        switch (shape) {
            case 16 * 8 + 1: return rows_kernel<TYPE, true, 16, 1>(a, grid, s);
            case 32 * 8 + 1: return rows_kernel<TYPE, true, 32, 1>(a, grid, s);
            case 64 * 8 + 1: return rows_kernel<TYPE, true, 64, 1>(a, grid, s);
            case 64 * 8 + 2: return rows_kernel<TYPE, true, 64, 2>(a, grid, s);
        }
    } else {
        switch (shape) {
            case 8 * 8 + 2: return rows_kernel<TYPE, false, 8, 2>(a, grid, s);
            case 8 * 8 + 3: return rows_kernel<TYPE, false, 8, 3>(a, grid, s);
            case 8 * 8 + 4: return rows_kernel<TYPE, false, 8, 4>(a, grid, s);
            case 16 * 8 + 3: return rows_kernel<TYPE, false, 16, 3>(a, grid, s);
            case 16 * 8 + 4: return rows_kernel<TYPE, false, 16, 4>(a, grid, s);
            case 32 * 8 + 3: return rows_kernel<TYPE, false, 32, 3>(a, grid, s);
            case 32 * 8 + 4: return rows_kernel<TYPE, false, 32, 4>(a, grid, s);
        }
    }
    if constexpr (TYPE == TYPE_F32) {
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

// Results are kept per block where groups have several (at most MAX_PARTS
// blocks then), and losses per group or per joining block, behind their sum.
constexpr uint64_t LINE = 128;  // of the cache: a joining block's 16 columns are one, if they start one
size_t balance_ws_bytes(uint64_t rows, uint64_t experts) {
    const uint64_t joining = MAX_PARTS / 2 * ((experts + JOIN_COLS - 1) / JOIN_COLS);
    return 2 * LINE + 8 * std::max<uint64_t>(rows, joining) + MAX_PARTS * (8 * experts + 4);
}

uint64_t balance_threads(const Matrix &m, const Routes &r) {
    const uint64_t joining = (uint64_t)r.groups * ((m.cols + JOIN_COLS - 1) / JOIN_COLS) * 512;
    const Shape sh = plan_rows(m.rows, m.cols, m.type, r.group_rows, false);
    const Shape gr = plan_rows(m.rows, m.cols, m.type, r.group_rows, true);
    return std::max((uint64_t)r.groups * std::max(sh.parts, gr.parts) * BT, sh.parts > 1 ? joining : 0);
}

hipError_t launch_balance_forward(const Matrix &m, const Routes &r, float coef, int32_t *counts_out,
                                  int32_t *rows_out, float *prob_out, float *loss_out, uint8_t *ws, hipStream_t s) {
    const Shape sh = plan_rows(m.rows, m.cols, m.type, r.group_rows, false);
    BalanceArgs a = balance_args(m, r, coef, sh);
    const uint64_t blocks = (uint64_t)r.groups * sh.parts;
    a.gloss = (double *)(ws + LINE);
    const bool one = r.groups == 1 && m.cols <= ONE_JOIN_COLS && sh.parts <= 256;
    a.col_blocks = one ? 1 : (m.cols + JOIN_COLS - 1) / JOIN_COLS;
    const uint32_t losses = sh.parts > 1 ? r.groups * a.col_blocks : r.groups;
    a.total = sh.parts > 1 && losses > 1 && losses <= MAX_ADDING ? (unsigned long long *)ws : nullptr;
    a.partial = (uint2 *)(ws + LINE + (8ull * losses + LINE - 1) / LINE * LINE);
    a.prows = (uint32_t *)(a.partial + blocks * m.cols);
    a.counts_out = counts_out;
    a.rows_out = rows_out;
    a.prob_out = prob_out;
    a.loss_out = loss_out;
    if (r.groups) {
        hipError_t e = rows_dispatch<false>(a, sh, s);
        if (e != hipSuccess) return e;
    }
    if (sh.parts > 1) {
        if (one)
            k_balance_join<1024, ONE_JOIN_COLS><<<1, 1024, 0, s>>>(a);
        else
            k_balance_join<512, JOIN_COLS><<<losses, 512, 0, s>>>(a);
        trace_mark(s, "k_balance_join");
    }
    if (losses != 1 && !a.total) {
        k_balance_mean<<<1, BT, 0, s>>>(a, losses);
        trace_mark(s, "k_balance_mean");
    }
    return hipGetLastError();
}

hipError_t launch_balance_backward(const Matrix &m, const Routes &r, float coef, const int32_t *counts,
                                   const int32_t *count_rows, const int32_t *rows_in, const float *upstream,
                                   void *grad, uint64_t grad_stride, hipStream_t s) {
    if (!r.groups) return hipSuccess;
    const Shape sh = plan_rows(m.rows, m.cols, m.type, r.group_rows, true);
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
