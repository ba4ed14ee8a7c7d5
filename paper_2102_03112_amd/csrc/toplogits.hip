// toplogits.hip -- the K largest logits of each row, and the logarithm of the
// sum of exponentials over all others.
//
// A block holds one slice of a row in registers.  Its first look gives every
// thread's largest logit.  Each of the eight waves offers the ceil(K / 8)-th
// largest of its 64, and the largest offer that K threads reach bounds the
// slice's K-th largest logit from below; with numbers in no order only little
// more than K logits reach it.  The second look lists those
// in LDS and adds the exponentials of the others, so no sum is ever taken off
// another one.  A listed logit's rank is the number of listed ones before it
// (by value, then column), counted by one thread each; ranks from K on return
// to the sum.  Where too many logits reach the bound (equal ones, say), the
// exact K-th largest is found bit by bit instead.  Rows of several slices are
// joined list by list in further launches.
#include <type_traits>

#include "launch.hpp"
#include "losses.hpp"

namespace dr {
namespace {

// A slice's block of NT threads takes K up to NT / 2, and has room to list four
// times that; one wave may list all that it holds, or eight times an even share.
template <uint32_t NT>
constexpr uint32_t CAND = 2 * NT;
template <int NV>
constexpr uint32_t WAVE_CAND = NV == 1 ? 512 : 256;

// One row's payload, or one list of a join: `keys` hold the value's order key
// above the complement of the column, so a larger key comes first and no two
// are equal; 0 is no entry.
struct TopArgs {
    Matrix m;
    Slices sl;
    uint32_t k;
    float c;      // log2(e) / temperature
    float inv_t;  // 1 / temperature
    uint64_t *keys;  // lists out: k keys each; null: the row's outputs
    float2 *sums;    // and their (reference, sum of 2^((z - reference) c)) over what they leave out
    int32_t *idx_out;
    float *val_out, *rest_out;
    // join only
    const uint64_t *keys_in;
    const float2 *sums_in;
    uint32_t lists_in, fan;
};

__device__ __forceinline__ uint64_t top_key(float x, uint32_t col) {
    // -0 counts as +0; NaN comes before all others
    const uint32_t k = x != x ? 0xffffffffu : order_key(x + 0.f);
    return (uint64_t)k << 32 | (0xffffffffu - col);
}
__device__ __forceinline__ float key_value(uint64_t key) { return order_key_inv((uint32_t)(key >> 32)); }

// A float no larger than any whose order key has these upper 16 bits.
__device__ __forceinline__ float key16_floor(uint32_t k16) {
    return fmaxf(order_key_inv(k16 << 16), F_LOWEST);  // NaN patterns of -inf's neighbourhood become the lowest
}

// The n-th largest of the wave's 64 keys of 16 bits (1 <= n <= 64).
__device__ __forceinline__ uint32_t wave_nth16(uint32_t key, uint32_t n) {
    uint32_t t = 0;
#pragma unroll
    for (uint32_t b = 1u << 15; b != 0; b >>= 1)
        if (popc64(ballot(key >= (t | b))) >= n) t |= b;
    return t;
}

// The largest of the NW (up to 8) numbers that lane i % NW has of i, on every lane.
template <uint32_t NW>
__device__ __forceinline__ uint32_t lanes_max_u(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, DPP_XOR1, 0xf, 0xf, true));
    if constexpr (NW >= 4) v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, DPP_XOR2, 0xf, 0xf, true));
    if constexpr (NW >= 8) v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, DPP_MIRROR8, 0xf, 0xf, true));
    return __builtin_amdgcn_readfirstlane(v);
}
// The sum of lanes 0 .. i on lane i < 8.
__device__ __forceinline__ uint32_t first_lanes_scan(uint32_t v) {
    v += __builtin_amdgcn_mov_dpp(v, 0x111, 0xf, 0xf, true);  // shifts by 1, 2 and 4, 0 moving in
    v += __builtin_amdgcn_mov_dpp(v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_mov_dpp(v, 0x114, 0xf, 0xf, true);
    return v;
}

template <uint32_t NT>
struct TopShared {
    static constexpr uint32_t NW = NT / 64;
    alignas(16) uint64_t cand[CAND<NT>];
    uint64_t sorted[CAND<NT>];
    uint32_t rank[CAND<NT>];
    uint32_t count;
    uint32_t bound[NW], reached[NW], listed[NW];
    uint32_t scan[NW + 1];
    uint32_t bits[32];
    float red[3][NW];
};

// (sum relative to reference a) as one relative to b >= a
__device__ __forceinline__ float top_rescale(float x, float a, float b, float c) {
    return x == 0.f ? 0.f : x * exp2_fast((a - b) * c);
}

// How many of keys[0 .. n) are above `key`; n is a multiple of RANK_STEP.
constexpr uint32_t RANK_STEP = 4;
__device__ __forceinline__ uint32_t keys_above(const uint64_t *keys, uint32_t n, uint64_t key) {
    uint32_t r = 0;
#pragma unroll 1
    for (uint32_t j = 0; j < n; j += RANK_STEP) {
        const ulonglong2 a = *(const ulonglong2 *)(keys + j), b = *(const ulonglong2 *)(keys + j + 2);
        r += a.x > key ? 1u : 0u;
        r += a.y > key ? 1u : 0u;
        r += b.x > key ? 1u : 0u;
        r += b.y > key ? 1u : 0u;
    }
    return r;
}

// sorted[] := the n keys of in[] in descending order, by counting the keys
// before each, which the block's threads share where keys are few: as many
// threads as the keys (in whole waves) count in one run of them each, and the
// last run is filled up with 0, which is no key and above none.  in[] has room
// for that, being a multiple of RANK_STEP and twice the threads.
template <uint32_t THREADS>
__device__ __forceinline__ void rank_keys(uint64_t *in, uint32_t n, uint32_t *rank, uint64_t *sorted) {
    const uint32_t lanes = (n + 63u) & ~63u, ways = lanes && lanes < THREADS ? THREADS / lanes : 1u;
    const uint32_t run = ((n + ways - 1) / ways + RANK_STEP - 1) / RANK_STEP * RANK_STEP;
    for (uint32_t i = threadIdx.x; i < n; i += THREADS) rank[i] = 0;
    if (n + threadIdx.x < ways * run) in[n + threadIdx.x] = 0;
    __syncthreads();
    if (ways > 1) {
        const uint32_t way = threadIdx.x / lanes, i = threadIdx.x % lanes;
        if (way < ways && i < n) atomicAdd(&rank[i], keys_above(in + way * run, run, in[i]));
    } else {
        for (uint32_t i = threadIdx.x; i < n; i += THREADS) rank[i] = keys_above(in, run, in[i]);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += THREADS) sorted[rank[i]] = in[i];
    __syncthreads();
}

// The end of a slice or a join: n sorted keys, and (ref, sum) of everything
// else.  Writes the first K keys and returns the rest to the sum.
template <uint32_t THREADS>
__device__ __forceinline__ void top_finish(const TopArgs &a, uint64_t row, uint64_t list, const uint64_t *sorted,
                                           uint32_t n, float ref, float sum, float *red) {
    const uint32_t K = a.k;
    if (n > K) {  // sorted[K] is the largest of what returns
        const float first = key_value(sorted[K]), b = fmaxf(ref, first);
        float back = 0.f;
        for (uint32_t i = K + threadIdx.x; i < n; i += THREADS)
            back += exp2_fast((key_value(sorted[i]) - b) * a.c);
        back = wave_sum_f(back);
        if ((threadIdx.x & 63u) == 0) red[threadIdx.x >> 6] = back;
        lds_barrier();
        sum = top_rescale(sum, ref, b, a.c);
        for (uint32_t i = 0; i < THREADS / 64; ++i) sum += red[i];
        ref = b;
    }
    if (a.keys) {
        for (uint32_t i = threadIdx.x; i < K; i += THREADS) a.keys[list * K + i] = i < n ? sorted[i] : 0;
        if (threadIdx.x == 0) a.sums[list] = make_float2(ref, sum);
        return;
    }
    for (uint32_t i = threadIdx.x; i < K; i += THREADS) {
        const uint64_t key = i < n ? sorted[i] : 0;
        a.idx_out[row * K + i] = i < n ? (int32_t)(0xffffffffu - (uint32_t)key) : -1;
        a.val_out[row * K + i] = i < n ? key_value(key) : F_NEG_INF;
    }
    // finite where anything is left, also beyond a float's range: -inf would say that nothing is
    if (threadIdx.x == 0 && a.rest_out) {
        const double rest = (double)ref * (double)a.inv_t + ln_sum(sum);
        a.rest_out[row] = sum > 0.f ? (float)fmin(fmax(rest, (double)F_LOWEST), -(double)F_LOWEST) : F_NEG_INF;
    }
}

// A slice as the rare paths read it: again from memory, one vector per thread
// and step, so that they cost the usual path no registers.
template <uint32_t TYPE, uint32_t NT>
struct SliceView {
    const typename Num<TYPE>::T *p;
    uint64_t avail;
    uint32_t start, n;
    static constexpr uint32_t STEP = NT * Num<TYPE>::VEC;

    __device__ __forceinline__ Vec<TYPE> at(uint32_t e0) const {
        return load_vec<TYPE>(p, e0 + threadIdx.x * Num<TYPE>::VEC, n, avail);
    }
    __device__ __forceinline__ uint32_t col(uint32_t e0, uint32_t e) const {
        return start + e0 + threadIdx.x * Num<TYPE>::VEC + e;
    }
};

// For a slice with more than K logits above -inf: lists exactly K, those
// above the K-th largest, found bit by bit, and of those equal to it the ones
// of lowest column.  Returns the K-th largest; *equal receives how many are
// equal to it and not listed.
template <uint32_t TYPE, uint32_t NT>
__device__ __forceinline__ float top_exact(const SliceView<TYPE, NT> &sl, uint32_t K, TopShared<NT> &sh,
                                           uint32_t *equal) {
    constexpr uint32_t VEC = Num<TYPE>::VEC;
    if (threadIdx.x < 32) sh.bits[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    uint32_t t = 0;
#pragma unroll 1
    for (int b = 31; b >= 0; --b) {
        const uint32_t want = t | 1u << b;
        uint32_t n = 0;
#pragma unroll 1
        for (uint32_t e0 = 0; e0 < sl.n; e0 += sl.STEP) {
            const Vec<TYPE> v = sl.at(e0);
#pragma unroll
            for (uint32_t e = 0; e < VEC; ++e) {
                const uint32_t key = (uint32_t)(top_key(v.get(e), 0) >> 32);
                n += key >= want && key > KEY_NEG_INF ? 1u : 0u;
            }
        }
        n = wave_sum(n);
        if ((threadIdx.x & 63u) == 0 && n) atomicAdd(&sh.bits[b], n);
        __syncthreads();
        if (sh.bits[b] >= K) t = want;
    }
#pragma unroll 1
    for (uint32_t e0 = 0; e0 < sl.n; e0 += sl.STEP) {
        const Vec<TYPE> v = sl.at(e0);
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) {
            const uint64_t key = top_key(v.get(e), sl.col(e0, e));
            if ((uint32_t)(key >> 32) > t) sh.cand[atomicAdd(&sh.count, 1u)] = key;  // fewer than K
        }
    }
    __syncthreads();
    uint32_t have = sh.count, left = 0;
    __syncthreads();
#pragma unroll 1
    for (uint32_t e0 = 0; e0 < sl.n; e0 += sl.STEP) {  // columns ascend with the step, then the thread
        const Vec<TYPE> v = sl.at(e0);
        uint32_t n = 0, total;
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) n += (uint32_t)(top_key(v.get(e), 0) >> 32) == t;
        uint32_t at = have + block_excl_scan_n<NT>(n, sh.scan, &total);
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) {
            const uint64_t key = top_key(v.get(e), sl.col(e0, e));
            if ((uint32_t)(key >> 32) == t) {
                if (at < K) sh.cand[at] = key;
                ++at;
            }
        }
        const uint32_t take = min(total, K - have);
        have += take;
        left += total - take;
    }
    if (threadIdx.x == 0) sh.count = have;
    __syncthreads();
    *equal = left;
    return order_key_inv(t);
}

// (reference, sum) of a slice's logits below the bound, relative to their own
// largest; red: two sets of scratch.
template <uint32_t TYPE, uint32_t NT>
__device__ __forceinline__ float2 sum_below(const SliceView<TYPE, NT> &sl, float bound, float c,
                                            float (*red)[NT / 64]) {
    constexpr uint32_t VEC = Num<TYPE>::VEC;
    float mx = F_NEG_INF;
#pragma unroll 1
    for (uint32_t e0 = 0; e0 < sl.n; e0 += sl.STEP) {
        const Vec<TYPE> v = sl.at(e0);
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) mx = v.get(e) < bound ? fmaxf(mx, v.get(e)) : mx;
    }
    mx = block_max_f<NT>(mx, red[0]);
    const float ref = mx == F_NEG_INF ? 0.f : mx;
    float sum = 0.f;
#pragma unroll 1
    for (uint32_t e0 = 0; e0 < sl.n; e0 += sl.STEP) {
        const Vec<TYPE> v = sl.at(e0);
        float x[VEC];
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) x[e] = v.get(e) < bound ? exp2_fast((v.get(e) - ref) * c) : 0.f;
        add_fours(sum, x);
    }
    return make_float2(mx, block_sum_f<NT>(sum, red[1]));
}

// One slice by one block.  A number costs six issue slots (unpack, compare,
// multiply-add, an exponential at half rate, add), the slice itself (bound,
// list, ranks) some 300 instructions a wave: so slices are as long as registers
// allow (plan_top; blocks of 256 and 1024 threads were slower for long rows).
// Bound by vector issue beside memory: 2048 x 131072 bfloat16, K 64: 100 us, 5.4
// TB/s, of which the vector instructions alone take 84.  777 x 50001 fp32, K 100:
// 32 us, 4.9 TB/s, and 17: three blocks share a CU, and 18 of the 1554 are left to
// a third round.  8 x 32000: 8 us, one block's latency.
template <uint32_t TYPE, int NV, uint32_t NT>
__global__ __launch_bounds__(NT) void k_top_slice(TopArgs a) {
    using N = Num<TYPE>;
    constexpr uint32_t VEC = N::VEC, NW = NT / 64;
    __shared__ TopShared<NT> sh;
    __shared__ uint2 wave_cand[NW][WAVE_CAND<NV>];  // a listed logit and its column in the slice
    const uint64_t row = blockIdx.x / a.sl.n;
    const uint32_t s = blockIdx.x % a.sl.n, start = s * a.sl.len, n = min(a.sl.len, a.m.cols - start);
    const auto *p = (const typename N::T *)a.m.p + row * a.m.stride + start;
    const uint64_t avail = row_avail(a.m, row) - start;
    const SliceView<TYPE, NT> sl = {p, avail, start, n};
    Vec<TYPE> v[NV];
    load_slice<TYPE, NT>(v, p, n, avail);
    if (threadIdx.x < NW) sh.reached[threadIdx.x] = 0;
    Largest<TYPE> most;
#pragma unroll
    for (int i = 0; i < NV; ++i) most.add(v[i]);
    most.complete(v);
    // every wave's nth largest, then the largest of them that K threads reach
    const uint32_t key16 = order_key(most.value()) >> 16;
    const uint32_t w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    const uint32_t full = min(NW, n / (64 * VEC)), nth = full ? (a.k + full - 1) / full : 64u;
    const uint32_t own = wave_nth16(key16, min(nth, 64u));
    if (lane == 0) sh.bound[w] = own;
    lds_barrier();
    uint32_t reached = 0;  // on lane i: how many of the wave reach wave i's
#pragma unroll
    for (uint32_t i = 0; i < NW; ++i)
        asm("v_writelane_b32 %0, %1, m0" : "+v"(reached) : "s"(popc64(ballot(key16 >= sh.bound[i]))), "{m0}"(i));
    if (lane < NW) atomicAdd(&sh.reached[lane], reached);
    lds_barrier();
    const uint32_t low = lanes_max_u<NW>(sh.reached[lane % NW] >= a.k ? sh.bound[lane % NW] : 0);
    float bound = low ? key16_floor(low) : F_LOWEST;
    // list what reaches the bound, wave by wave, and add the others' exponentials
    const Base2 to2(bound, a.c);
    float ref = bound, sum = 0.f;
    uint32_t listed = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float x[VEC];
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) {
            x[e] = v[i].get(e);
            const bool reach = !(x[e] < bound);
            if (const uint64_t any = ballot(reach)) {
                uint32_t col = threadIdx.x * VEC;
                asm volatile("" : "+v"(col));  // a branch, which most waves pass over, and its columns stay in it
                const uint32_t at = listed + lanes_below(any);
                if (reach && at < WAVE_CAND<NV>)
                    wave_cand[w][at] = make_uint2(__float_as_uint(x[e]), col + (i * NT * VEC + e));
                x[e] = reach ? F_NEG_INF : x[e];
                listed += popc64(any);
            }
        }
#pragma unroll
        for (uint32_t e = 0; e < VEC; ++e) x[e] = to2(x[e]);
        add_fours(sum, x);
        asm volatile("" : "+v"(sum));  // now, not when all vectors' numbers are unpacked
    }
    if (lane == 0) sh.listed[w] = listed;
    __syncthreads();
    const uint32_t wave_listed = sh.listed[lane % NW], up_to = first_lanes_scan(wave_listed);
    uint32_t count = __builtin_amdgcn_readlane(up_to, NW - 1), equal = 0;
    const uint32_t before = __builtin_amdgcn_readlane(up_to, w) - listed;
    const bool exact = count > CAND<NT> || ballot(wave_listed > WAVE_CAND<NV>) != 0;
    if (!exact)
#pragma unroll 1
        for (uint32_t i = lane; i < listed; i += 64)
            sh.cand[before + i] = top_key(__uint_as_float(wave_cand[w][i].x), start + wave_cand[w][i].y);
    sum = block_sum_f<NT>(sum, sh.red[0]) * to2.to(bound);
    if (exact) {
        bound = top_exact<TYPE, NT>(sl, a.k, sh, &equal);
        count = sh.count;
    }
    // other logits than these are listed, or all that was added lies far below the bound
    if (exact || !(sum > 1e-20f && sum < 1e30f)) {
        const float2 x = sum_below<TYPE, NT>(sl, bound, a.c, sh.red + 1);
        ref = x.x;
        sum = x.y;
        if (equal) {
            sum = top_rescale(sum, ref, bound, a.c) + (float)equal;
            ref = bound;
        }
        __syncthreads();
    }
    rank_keys<NT>(sh.cand, count, sh.rank, sh.sorted);
    top_finish<NT>(a, row, (uint64_t)blockIdx.x, sh.sorted, count, ref, sum, sh.red[1]);
}

// `fan` sorted lists of a row into one, of at most ENTRIES keys in all.  Of F
// full lists the ceil(K / F)-th entries bound the K-th largest of all from
// below, as the threads' largest do in a slice: only what reaches the smallest
// of them is ranked.  512 keys are enough for the usual few lists, and their
// room lets eight blocks share a CU.  Bound by latency (reads, bound, ranks in
// turn): 8.8 us for 2048 rows of four lists of 64.
template <uint32_t JT, uint32_t ENTRIES>
__global__ __launch_bounds__(JT) void k_top_join(TopArgs a) {
    __shared__ alignas(16) uint64_t in[ENTRIES];
    __shared__ uint64_t sorted[ENTRIES];
    __shared__ uint32_t ranks[ENTRIES];
    __shared__ float red[3][JT / 64];
    __shared__ uint32_t full, entries;
    __shared__ uint64_t bound;
    const uint32_t groups = (a.lists_in + a.fan - 1) / a.fan, K = a.k;
    const uint64_t row = blockIdx.x / groups;
    const uint32_t first = blockIdx.x % groups * a.fan, lists = min(a.fan, a.lists_in - first);
    const uint64_t from = row * a.lists_in + first;
    if (threadIdx.x == 0) full = entries = 0, bound = ~0ull;
    const float2 mine = threadIdx.x < lists ? a.sums_in[from + threadIdx.x] : make_float2(F_NEG_INF, 0.f);
#pragma unroll
    for (uint32_t i = threadIdx.x; i < ENTRIES; i += JT)
        if (i < lists * K) sorted[i] = a.keys_in[from * K + i];
    float ref = mine.y > 0.f ? mine.x : F_NEG_INF;
    for (uint32_t i = threadIdx.x + JT; i < lists; i += JT) {
        const float2 x = a.sums_in[from + i];
        if (x.y > 0.f) ref = fmaxf(ref, x.x);
    }
    ref = block_max_f<JT>(ref, red[0]);
    for (uint32_t i = threadIdx.x; i < lists; i += JT)
        if (sorted[i * K + K - 1]) atomicAdd(&full, 1u);
    float sum = top_rescale(mine.y, mine.x, ref, a.c);
    for (uint32_t i = threadIdx.x + JT; i < lists; i += JT) {
        const float2 x = a.sums_in[from + i];
        sum += top_rescale(x.y, x.x, ref, a.c);
    }
    sum = block_sum_f<JT>(sum, red[1]);
    const uint32_t nth = full ? (K + full - 1) / full : 0;
    for (uint32_t i = threadIdx.x; nth && i < lists; i += JT)
        if (sorted[i * K + K - 1]) atomicMin((unsigned long long *)&bound, sorted[i * K + nth - 1]);
    __syncthreads();
    const uint64_t least = nth ? bound : 1;
    float left = 0.f;  // what does not reach the bound returns to the sum
    const float least_x = key_value(least);
    for (uint32_t i = threadIdx.x; i < lists * K; i += JT) {
        const uint64_t key = sorted[i];
        if (key >= least)
            in[atomicAdd(&entries, 1u)] = key;
        else if (key)
            left += exp2_fast((key_value(key) - least_x) * a.c);
    }
    __syncthreads();
    const uint32_t n = entries;
    left = block_sum_f<JT>(left, red[2]);
    float left_ref = least_x;
    if (!(left > 1e-20f)) {  // nothing, or all of it far below the bound: relative to its own largest then
        float mx = F_NEG_INF;
        for (uint32_t i = threadIdx.x; i < lists * K; i += JT)
            if (sorted[i] && sorted[i] < least) mx = fmaxf(mx, key_value(sorted[i]));
        left_ref = block_max_f<JT>(mx, red[0]);
        left = 0.f;
        for (uint32_t i = threadIdx.x; i < lists * K; i += JT)
            if (sorted[i] && sorted[i] < least) left += exp2_fast((key_value(sorted[i]) - left_ref) * a.c);
        left = block_sum_f<JT>(left, red[1]);
    }
    if (left > 0.f) {
        const float b = fmaxf(ref, left_ref);
        sum = top_rescale(sum, ref, b, a.c) + top_rescale(left, left_ref, b, a.c);
        ref = b;
    }
    rank_keys<JT>(in, n, ranks, sorted);
    top_finish<JT>(a, row, (uint64_t)blockIdx.x, sorted, n, ref, sum, red[0]);
}
constexpr uint32_t FEW_ENTRIES = 512;

template <uint32_t TYPE, uint32_t NT>
void slice_kernel(const TopArgs &a, hipStream_t s) {
    const uint32_t grid = (uint32_t)(a.m.rows * a.sl.n);
    switch (a.sl.nv) {
        case 1: k_top_slice<TYPE, 1, NT><<<grid, NT, 0, s>>>(a); break;
        case 2: k_top_slice<TYPE, 2, NT><<<grid, NT, 0, s>>>(a); break;
        case 3: k_top_slice<TYPE, 3, NT><<<grid, NT, 0, s>>>(a); break;
        case 4: k_top_slice<TYPE, 4, NT><<<grid, NT, 0, s>>>(a); break;
        case 6: k_top_slice<TYPE, 6, NT><<<grid, NT, 0, s>>>(a); break;
        case 8: k_top_slice<TYPE, 8, NT><<<grid, NT, 0, s>>>(a); break;
    }
    if constexpr (NT == 512) {
        switch (a.sl.nv) {
            case 10: k_top_slice<TYPE, 10, NT><<<grid, NT, 0, s>>>(a); break;
            case 12: k_top_slice<TYPE, 12, NT><<<grid, NT, 0, s>>>(a); break;
            case 16: k_top_slice<TYPE, 16, NT><<<grid, NT, 0, s>>>(a); break;
        }
    }
    trace_mark(s, "k_top_slice");
}

template <uint32_t TYPE>
void slice_kernel(const TopArgs &a, uint32_t threads, hipStream_t s) {
    if (threads == 128)
        slice_kernel<TYPE, 128>(a, s);
    else if (threads == 256)
        slice_kernel<TYPE, 256>(a, s);
    else
        slice_kernel<TYPE, 512>(a, s);
}

uint64_t list_bytes(uint64_t rows, uint64_t lists, uint32_t k) {
    return (rows * lists * (k * sizeof(uint64_t) + sizeof(float2)) + 255) / 256 * 256;
}

}  // namespace

TopPlan plan_top(uint64_t rows, uint64_t cols, uint32_t k, uint32_t type) {
    TopPlan p = {};
    // The fewest threads that hold a row and are twice K, if rows fill the chip.
    // Else slices as long as they go, also where rows are few: a slice costs a
    // block much the same whatever its length, and one slice needs no join (8 x
    // 32000 bfloat16, K 50: 7.7 us as one slice, 11.2 as eight).
    const uint32_t vec = 16 / type_bytes(type);
    p.threads = 512;
    for (uint32_t t = 128; t < 512; t *= 2)
        if (p.threads == 512 && rows >= 512 && 2 * k <= t && cols <= (uint64_t)t * TOP_NV * vec) p.threads = t;
    // Ten vectors a thread, at 58 registers, leave a SIMD its eight waves; sixteen,
    // at 80 and more, pay where a row is then one slice, without a join, and for
    // 32-bit numbers, of which they hold half as many (1000 x 50001 float16, K 200:
    // 49 us with sixteen, 65 with eight; 1000 x 40000 bfloat16: 21 with ten, 29 with
    // eight; 1024 x 131072 fp32: 94 and 101; but 2048 x 131072 bfloat16 by twelve
    // 109, by eight 101).
    const uint64_t whole = 512ull * 16 * vec;
    const uint32_t most = p.threads < 512 ? TOP_NV : type == TYPE_F32 || cols <= whole ? 16 : 10;
    p.sl = plan_slices(rows, cols, vec, p.threads, most, 1);
    // vectors that the slices need, of those that there are kernels for
    const uint32_t nv = (p.sl.len + p.threads * vec - 1) / (p.threads * vec);
    for (uint32_t n : {1, 2, 3, 4, 6, 8, 10, 12, 16})
        if (n >= nv) {
            p.sl.nv = n;
            break;
        }
    p.fan = std::max(2u, TOP_JOIN / k);
    p.lists[0] = p.sl.n > 1 ? p.sl.n : 0;
    p.lists[1] = p.sl.n > p.fan ? (p.sl.n + p.fan - 1) / p.fan : 0;
    p.bytes = list_bytes(rows, p.lists[0], k) + list_bytes(rows, p.lists[1], k);
    return p;
}

hipError_t launch_top(const Matrix &m, uint32_t k, float temperature, int32_t *idx_out, float *val_out,
                      float *rest_out, const TopPlan &p, uint8_t *ws, hipStream_t s) {
    TopArgs a = {};
    a.m = m;
    a.sl = p.sl;
    a.k = k;
    a.c = (float)(1.4426950408889634074 / temperature);
    a.inv_t = (float)(1.0 / temperature);
    a.idx_out = idx_out;
    a.val_out = val_out;
    a.rest_out = rest_out;
    uint64_t *keys[2];
    float2 *sums[2];
    for (int i = 0; i < 2; ++i) {
        keys[i] = (uint64_t *)(ws + (i ? list_bytes(m.rows, p.lists[0], k) : 0));
        sums[i] = (float2 *)(keys[i] + m.rows * p.lists[i] * k);
    }
    if (p.sl.n > 1) {
        a.keys = keys[0];
        a.sums = sums[0];
    }
    switch (m.type) {
        case TYPE_F32: slice_kernel<TYPE_F32>(a, p.threads, s); break;
        case TYPE_BF16: slice_kernel<TYPE_BF16>(a, p.threads, s); break;
        default: slice_kernel<TYPE_F16>(a, p.threads, s); break;
    }
    uint32_t lists = p.sl.n;
    for (int from = 0; lists > 1; from ^= 1) {
        const uint32_t groups = (lists + p.fan - 1) / p.fan;
        a.keys_in = keys[from];
        a.sums_in = sums[from];
        a.lists_in = lists;
        a.fan = p.fan;
        a.keys = groups > 1 ? keys[from ^ 1] : nullptr;
        a.sums = groups > 1 ? sums[from ^ 1] : nullptr;
        const uint32_t grid = (uint32_t)(m.rows * groups);
        if (std::min(lists, p.fan) * k <= FEW_ENTRIES)
            k_top_join<256, FEW_ENTRIES><<<grid, 256, 0, s>>>(a);
        else
            k_top_join<256, TOP_JOIN><<<grid, 256, 0, s>>>(a);
        trace_mark(s, "k_top_join");
        lists = groups;
    }
    return hipGetLastError();
}

}  // namespace dr
