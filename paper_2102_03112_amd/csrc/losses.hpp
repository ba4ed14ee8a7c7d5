// losses.hpp -- what the loss kernels share: number types and their 16-byte
// vectors, row slices, block reductions, and the host-side launchers.
//
// A row of logits is cut into slices, one block each: a slice is held in
// registers from one read, so that its maximum and its sum of exponentials
// take one pass over memory, and rows that are few still fill the chip.  The
// slices' results are joined in a second, small launch.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <stdint.h>

#include "dr_common.hpp"

namespace dr {

constexpr uint32_t TYPE_F32 = 0, TYPE_BF16 = 1, TYPE_F16 = 2;
constexpr uint32_t INDEX_I32 = 0, INDEX_I64 = 1;
constexpr uint32_t MAX_TOP = 256, MAX_TEACHER = 1024, MAX_EXPERTS = 1024;
constexpr uint32_t STATS = 8;  // floats saved per row by the distillation's forward pass
constexpr float LOG2E = 1.4426950408889634f;
constexpr float F_LOWEST = -3.4028234663852886e38f;
constexpr float F_NEG_INF = -__builtin_inff();
constexpr uint32_t KEY_NEG_INF = 0x007fffffu;  // order_key(-inf)

constexpr uint32_t type_bytes(uint32_t type) { return type == TYPE_F32 ? 4u : 2u; }

// A matrix of logits (or of gradients) as the kernels take it.
struct Matrix {
    const void *p;
    uint64_t rows, stride;
    uint32_t cols;
    uint32_t type;
};

// A number type: its storage, and how many a 16-byte vector holds.
template <uint32_t TYPE>
struct Num {
    using T = uint16_t;
    static constexpr uint32_t VEC = 8;
    static constexpr uint32_t NEG_INF = TYPE == TYPE_BF16 ? 0xff80u : 0xfc00u;
};
template <>
struct Num<TYPE_F32> {
    using T = uint32_t;
    static constexpr uint32_t VEC = 4;
    static constexpr uint32_t NEG_INF = 0xff800000u;
};

#if defined(__HIPCC__)

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf162_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));

// Maxima without the operation that quiets their operands first.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("v_pk_max_f16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_halves_signed(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("v_pk_max_i16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ uint32_t min_halves_unsigned(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("v_pk_min_u16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

template <uint32_t TYPE>
__device__ __forceinline__ float num_float(typename Num<TYPE>::T x) {
    if constexpr (TYPE == TYPE_F32)
        return __uint_as_float(x);
    else if constexpr (TYPE == TYPE_BF16)
        return __uint_as_float((uint32_t)x << 16);
    else
        return (float)__builtin_bit_cast(_Float16, x);
}

// round to nearest even
template <uint32_t TYPE>
__device__ __forceinline__ typename Num<TYPE>::T num_round(float x) {
    if constexpr (TYPE == TYPE_F32)
        return __float_as_uint(x);
    else if constexpr (TYPE == TYPE_BF16)
        return __builtin_bit_cast(uint16_t, (__bf16)x);
    else
        return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// One 16-byte vector of numbers in registers.
template <uint32_t TYPE>
struct Vec {
    using N = Num<TYPE>;
    using T = typename N::T;
    uint32_t w[4];

    __device__ __forceinline__ float get(uint32_t i) const {
        const uint32_t x = w[i * 4 / N::VEC];
        if constexpr (TYPE == TYPE_F32)
            return __uint_as_float(x);
        else if constexpr (TYPE == TYPE_BF16)
            return __uint_as_float(i & 1 ? x & 0xffff0000u : x << 16);
        else
            return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? x >> 16 : x));
    }
    // elements whose bit is set := -inf (by whole words: halves of their own
    // would take a register each)
    __device__ __forceinline__ void mask(uint32_t bits) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            if constexpr (TYPE == TYPE_F32) {
                w[i] = bits >> i & 1u ? N::NEG_INF : w[i];
            } else {
                const uint32_t lo = 0u - (bits >> (2 * i) & 1u), hi = 0u - (bits >> (2 * i + 1) & 1u);
                const uint32_t m = (lo & 0xffffu) | (hi << 16), inf = N::NEG_INF * 0x10001u;
                asm("v_bfi_b32 %0, %1, %2, %3" : "=v"(w[i]) : "v"(m), "v"(inf), "v"(w[i]));
            }
        }
    }
    // The numbers as a queue: push before the first one, take the first one off.
    __device__ __forceinline__ void push(T x) {
        if constexpr (TYPE == TYPE_F32) {
            w[3] = w[2], w[2] = w[1], w[1] = w[0], w[0] = x;
        } else {
            w[3] = w[3] << 16 | w[2] >> 16, w[2] = w[2] << 16 | w[1] >> 16, w[1] = w[1] << 16 | w[0] >> 16;
            w[0] = w[0] << 16 | x;
        }
    }
    __device__ __forceinline__ T pop() {
        const T x = (T)w[0];
        if constexpr (TYPE == TYPE_F32) {
            w[0] = w[1], w[1] = w[2], w[2] = w[3];
        } else {
            w[0] = w[0] >> 16 | w[1] << 16, w[1] = w[1] >> 16 | w[2] << 16, w[2] = w[2] >> 16 | w[3] << 16;
            w[3] >>= 16;
        }
        return x;
    }
    // Makes the next use unpack anew, instead of numbers unpacked before in
    // twice the registers.
    __device__ __forceinline__ void keep_packed() {
        if constexpr (TYPE != TYPE_F32) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) asm volatile("" : "+v"(w[i]));
        }
    }
    __device__ __forceinline__ void fill_neg_inf() {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) w[i] = TYPE == TYPE_F32 ? N::NEG_INF : N::NEG_INF * 0x10001u;
    }
    __device__ __forceinline__ void put(const float *x) {
        if constexpr (TYPE == TYPE_F32) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const float2_t f = {x[2 * i], x[2 * i + 1]};
                if constexpr (TYPE == TYPE_BF16)
                    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf162_t));
                else
                    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, half2_t));
            }
        }
    }
};

// The largest number of some vectors, kept as bits (-inf of none).  32-bit
// numbers: a float.  float16: two halves.  bfloat16: two halves as whole numbers,
// the largest of the bits with their sign; where a half of all vectors is
// negative, the smallest bits without it are the maximum, for which complete()
// goes over the vectors again.  (Read as float16, bfloat16 numbers from 2^121 on
// would be NaN, and the maximum of such halves no number of the vectors.)
template <uint32_t TYPE>
struct Largest {
    using N = Num<TYPE>;
    uint32_t w = TYPE == TYPE_F32 ? N::NEG_INF : N::NEG_INF * 0x10001u;

    __device__ __forceinline__ void add(const Vec<TYPE> &v) {
        if constexpr (TYPE == TYPE_F32) {
            const float f = max3(__uint_as_float(w), v.get(0), v.get(1));
            w = __float_as_uint(max3(f, v.get(2), v.get(3)));
        } else if constexpr (TYPE == TYPE_BF16) {
            w = max_halves_signed(max_halves_signed(w, v.w[0]),
                                  max_halves_signed(max_halves_signed(v.w[1], v.w[2]), v.w[3]));
        } else {
            w = max_halves(max_halves(w, v.w[0]), max_halves(max_halves(v.w[1], v.w[2]), v.w[3]));
        }
    }
    // after all of v, and no others, were added
    template <int NV>
    __device__ __forceinline__ void complete(const Vec<TYPE> (&v)[NV]) {
        if constexpr (TYPE == TYPE_BF16) {
            if (w & 0x80008000u) {
                uint32_t low = N::NEG_INF * 0x10001u;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    low = min_halves_unsigned(
                        min_halves_unsigned(low, v[i].w[0]),
                        min_halves_unsigned(min_halves_unsigned(v[i].w[1], v[i].w[2]), v[i].w[3]));
                w = (w & 0x8000u ? low & 0xffffu : w & 0xffffu) | (w >> 31 ? low & 0xffff0000u : w & 0xffff0000u);
            }
        }
    }
    __device__ __forceinline__ float value() const {
        using T = typename N::T;
        if constexpr (TYPE == TYPE_F32) {
            return __uint_as_float(w);
        } else {
            const float x = num_float<TYPE>((T)w), y = num_float<TYPE>((T)(w >> 16));
            return x > y ? x : y;
        }
    }
};

// 16 bytes at any address that suits a 16-bit number
typedef uint32_t vec_any __attribute__((ext_vector_type(4), aligned(2)));

template <uint32_t TYPE, bool NT>
__device__ __forceinline__ Vec<TYPE> load_whole(const typename Num<TYPE>::T *p) {
    const vec_any x = NT ? __builtin_nontemporal_load((const vec_any *)p) : *(const vec_any *)p;
    Vec<TYPE> v;
    __builtin_memcpy(v.w, &x, 16);
    return v;
}

// The vector at p[e .. e + VEC) with everything from element n on as -inf.
// `avail` numbers can be read from p on, so that a vector which only its last
// elements take out of the row is still one load; p is aligned to its type
// alone (the hardware loads 16 bytes at any address).  NT: numbers that are
// read once (reading 1 GiB: 6.1 TB/s without, 7.0 with; copying it: 5.4 with
// neither load nor store so, 6.3 with both).
template <uint32_t TYPE, bool NT = true>
__device__ __forceinline__ Vec<TYPE> load_vec(const typename Num<TYPE>::T *p, uint32_t e, uint32_t n, uint64_t avail) {
    constexpr uint32_t VEC = Num<TYPE>::VEC;
    Vec<TYPE> v;
    if (e >= n) {
        v.fill_neg_inf();
    } else if (e + VEC <= avail) {
        v = load_whole<TYPE, NT>(p + e);
        if (e + VEC > n) v.mask(~0u << (n - e));
    } else {  // the matrix ends in it: number by number, the last one first
        v.fill_neg_inf();
#pragma unroll 1
        for (uint32_t i = VEC; i-- > 0;) v.push(e + i < n ? p[e + i] : (typename Num<TYPE>::T)Num<TYPE>::NEG_INF);
    }
    return v;
}

// The calling thread's vector of a run of them that starts at p (the same on
// every lane: the address is a scalar base and one 32-bit offset for all runs).
template <uint32_t TYPE, bool NT>
__device__ __forceinline__ Vec<TYPE> load_run(const typename Num<TYPE>::T *p) {
    return load_whole<TYPE, NT>((const typename Num<TYPE>::T *)((const char *)p + threadIdx.x * 16u));
}
template <uint32_t TYPE, bool NT = true>
__device__ __forceinline__ void store_run(typename Num<TYPE>::T *p, const float *x) {
    Vec<TYPE> v;
    v.put(x);
    vec_any y;
    __builtin_memcpy(&y, v.w, 16);
    vec_any *at = (vec_any *)((char *)p + threadIdx.x * 16u);
    if (NT)
        __builtin_nontemporal_store(y, at);
    else
        *at = y;
}

// The NV vectors that a thread of a block of THREADS holds of n numbers:
// vector i THREADS + thread.
template <uint32_t TYPE, uint32_t THREADS, int NV, bool NT = true>
__device__ __forceinline__ void load_slice(Vec<TYPE> (&v)[NV], const typename Num<TYPE>::T *p, uint32_t n,
                                           uint64_t avail) {
    constexpr uint32_t VEC = Num<TYPE>::VEC;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if ((i + 1) * THREADS * VEC <= n)  // the whole block's
            v[i] = load_run<TYPE, NT>(p + i * THREADS * VEC);
        else
            v[i] = load_vec<TYPE, NT>(p, (i * THREADS + threadIdx.x) * VEC, n, avail);
    }
}

// p[e .. min(e + VEC, n)) := x
template <uint32_t TYPE, bool NT = true>
__device__ __forceinline__ void store_vec(typename Num<TYPE>::T *p, uint32_t e, uint32_t n, const float *x) {
    constexpr uint32_t VEC = Num<TYPE>::VEC;
    Vec<TYPE> v;
    v.put(x);
    if (e + VEC <= n) {
        vec_any y;
        __builtin_memcpy(&y, v.w, 16);
        if (NT)
            __builtin_nontemporal_store(y, (vec_any *)(p + e));
        else
            *(vec_any *)(p + e) = y;
    } else {
#pragma unroll 1
        for (; e < n; ++e) p[e] = v.pop();
    }
}

// numbers from row r's start to the end of the matrix
__device__ __forceinline__ uint64_t row_avail(const Matrix &m, uint64_t r) {
    return (m.rows - 1 - r) * m.stride + m.cols;
}

// A number or an index whose type is known at run time only.
__device__ __forceinline__ float load_num(const void *p, uint64_t i, uint32_t type) {
    if (type == TYPE_F32) return ((const float *)p)[i];
    const uint16_t x = ((const uint16_t *)p)[i];
    return type == TYPE_BF16 ? num_float<TYPE_BF16>(x) : num_float<TYPE_F16>(x);
}
// an index below n, or n for any other
__device__ __forceinline__ uint32_t load_index(const void *p, uint64_t i, uint32_t type, uint32_t n) {
    if (type == INDEX_I32) {
        const uint32_t x = ((const uint32_t *)p)[i];
        return x < n ? x : n;
    }
    const uint64_t x = ((const uint64_t *)p)[i];
    return x < n ? (uint32_t)x : n;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// exp of a number that is not above 0: an argument x is off by 2^-24 x, which
// takes at most 2e-8 of 1 from the result.
__device__ __forceinline__ float exp_below(float x) { return exp2_fast(x * LOG2E); }

// exp((x - m) / t) as 2^(x c - R) times 2^(R - m c), c = log2(e) / t and R the
// whole number next to m c: one fused operation per number, whose only
// rounding is that of a small result, and the second factor once.  Where m c is
// so large that a float's whole numbers are too far apart (from BASE2_FAR on
// R - m c would be beyond 4, and beyond all exponents soon), R = 0: such sums come
// out of range and are formed again from x - m.
constexpr float BASE2_FAR = 1e8f;
struct Base2 {
    float c, r;
    __device__ __forceinline__ Base2(float m, float c_) : c(c_) {
        const float x = rintf(m * c_);
        r = fabsf(x) < BASE2_FAR ? x : 0.f;
    }
    __device__ __forceinline__ float operator()(float x) const { return exp2_fast(fmaf(x, c, -r)); }
    __device__ __forceinline__ float to(float m) const { return exp2_fast(-fmaf(m, c, -r)); }
};
__device__ __forceinline__ bool sum_in_range(float s) { return s > 0.25f && s < 1e30f; }

// Adds a vector's numbers by fours, in pairs: as many additions as one after
// the other, of which a thread's sum meets one for four numbers, so that it is
// a chain of 64 at most.
template <uint32_t N>
__device__ __forceinline__ void add_fours(float &sum, const float (&x)[N]) {
#pragma unroll
    for (uint32_t i = 0; i < N; i += 4) sum += (x[i] + x[i + 1]) + (x[i + 2] + x[i + 3]);
}

// ln of a sum: the exponent apart, so that the logarithm's own error (of a
// number in [0.5, 1)) stays below 1e-7 however large the sum is
__device__ __forceinline__ double ln_sum(double x) {
    const int e = __builtin_amdgcn_frexp_exp(x);
    const float f = (float)__builtin_amdgcn_frexp_mant(x);
    return 0.6931471805599453 * ((double)e + (double)__builtin_amdgcn_logf(f));
}

// A value of another lane of the row of 16 (DPP control word CTRL).
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_MIRROR8 = 0x141, DPP_MIRROR16 = 0x140;

// Maximum and sum over each aligned group of LANES lanes (a power of two), on
// every lane of it, in one order: within four lanes, then with the mirrored
// four, eight, then with the neighbouring row and half of the wave.
template <uint32_t LANES, typename OP>
__device__ __forceinline__ float lanes_reduce(float v, OP op) {
    if constexpr (LANES >= 2) v = op(v, dpp<DPP_XOR1>(v));
    if constexpr (LANES >= 4) v = op(v, dpp<DPP_XOR2>(v));
    if constexpr (LANES >= 8) v = op(v, dpp<DPP_MIRROR8>(v));
    if constexpr (LANES >= 16) v = op(v, dpp<DPP_MIRROR16>(v));
    if constexpr (LANES >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if constexpr (LANES >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}
template <uint32_t LANES>
__device__ __forceinline__ float lanes_max(float v) {
    return lanes_reduce<LANES>(v, [](float a, float b) { return max3(a, b, b); });
}
template <uint32_t LANES>
__device__ __forceinline__ float lanes_sum(float v) {
    return lanes_reduce<LANES>(v, [](float a, float b) { return a + b; });
}
// Sum over the lanes of one place in every aligned group of LANES lanes: by
// rotations of the rows of 16, which keep a place, then over rows and halves.
template <uint32_t LANES>
__device__ __forceinline__ float groups_sum(float v) {
    if constexpr (LANES <= 8) v += dpp<0x128>(v);
    if constexpr (LANES <= 4) v += dpp<0x124>(v);
    if constexpr (LANES <= 2) v += dpp<0x122>(v);
    if constexpr (LANES <= 1) v += dpp<0x121>(v);
    if constexpr (LANES <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (LANES <= 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}
__device__ __forceinline__ float wave_max_f(float v) { return lanes_max<64>(v); }
__device__ __forceinline__ float wave_sum_f(float v) { return lanes_sum<64>(v); }

// Block-wide maximum and sum; scratch holds NT / 64 words.  The sum's order is
// fixed.  Every thread must call them; the scratch may be used again after the
// caller's next barrier.
template <uint32_t NT>
__device__ __forceinline__ float block_max_f(float v, float *scratch) {
    v = wave_max_f(v);
    if ((threadIdx.x & 63u) == 0) scratch[threadIdx.x >> 6] = v;
    lds_barrier();
    v = scratch[0];
#pragma unroll
    for (uint32_t i = 1; i < NT / 64; ++i) v = fmaxf(v, scratch[i]);
    return v;
}
template <uint32_t NT>
__device__ __forceinline__ float block_sum_f(float v, float *scratch) {
    v = wave_sum_f(v);
    if ((threadIdx.x & 63u) == 0) scratch[threadIdx.x >> 6] = v;
    lds_barrier();
    v = scratch[0];
#pragma unroll
    for (uint32_t i = 1; i < NT / 64; ++i) v += scratch[i];
    return v;
}

#endif  // __HIPCC__

// How a row of `cols` numbers is cut: slices of `len` numbers for blocks of
// NT threads that hold nv 16-byte vectors each.
struct Slices {
    uint32_t nv, len, n;
};
// The longest slices (fewest results to join) that give `blocks` blocks, and as
// few vectors as such a slice needs.
inline Slices plan_slices(uint64_t rows, uint64_t cols, uint32_t vec, uint32_t threads, uint32_t nv_max,
                          uint64_t blocks) {
    Slices s;
    uint64_t cap, n;
    for (s.nv = nv_max;; s.nv /= 2) {
        cap = (uint64_t)threads * s.nv * vec;
        n = (cols + cap - 1) / cap;
        if (rows * n >= blocks || s.nv == 1) break;
    }
    const uint64_t len = (cols + n - 1) / n;
    s.len = (uint32_t)std::min<uint64_t>(cap, (len + vec - 1) / vec * vec);
    s.n = (uint32_t)((cols + s.len - 1) / s.len);
    while (s.nv > 1 && (uint64_t)threads * (s.nv / 2) * vec >= s.len) s.nv /= 2;
    return s;
}

// A launch's threads are counted in 32 bits.
constexpr uint64_t MAX_THREADS = 0xffffffffull;

// toplogits.hip
constexpr uint32_t TOP_NV = 8;
constexpr uint32_t TOP_JOIN = 2048;  // list entries that one block joins
struct TopPlan {
    uint32_t threads;    // of a slice's block
    Slices sl;
    uint32_t fan;        // lists that one block joins
    uint64_t lists[2];   // most lists that the two buffers hold per row
    size_t bytes;
};
TopPlan plan_top(uint64_t rows, uint64_t cols, uint32_t k, uint32_t type);
hipError_t launch_top(const Matrix &m, uint32_t k, float temperature, int32_t *idx_out, float *val_out,
                      float *rest_out, const TopPlan &p, uint8_t *ws, hipStream_t s);

// distill.hip
struct Teacher {
    const void *idx, *val;
    const float *rest;
    uint64_t idx_stride, val_stride;
    uint32_t k, idx_type, val_type;
};
constexpr uint32_t DIST_THREADS = 256, DIST_NV = 8;
// Words of the bitmap of a row of n columns that a block reads `step` columns
// at a time: a bit for every place of every step, the last one's too.
constexpr uint32_t row_bitmap_words(uint32_t n, uint32_t step) { return (n + step - 1) / step * (step / 32); }
size_t distill_ws_bytes(uint64_t rows, uint64_t cols, uint32_t type);
uint64_t distill_threads(const Matrix &m);  // of the largest launch
hipError_t launch_distill_forward(const Matrix &m, const Teacher &t, float temperature, const float *weight,
                                  float *loss_out, float *stats_out, uint8_t *ws, hipStream_t s);
hipError_t launch_distill_backward(const Matrix &m, const Teacher &t, float temperature, const float *weight,
                                   const float *upstream, uint64_t upstream_stride, const float *stats, void *grad,
                                   uint64_t grad_stride, hipStream_t s);
hipError_t launch_distill_step(const Matrix &m, const Teacher &t, float temperature, const float *weight,
                               float *loss_out, void *grad, uint64_t grad_stride, uint8_t *ws, hipStream_t s);

// balance.hip
struct Routes {
    const void *idx;
    const uint8_t *mask;
    uint64_t idx_stride;
    uint32_t k, idx_type;
    uint32_t group_rows, groups;
};
size_t balance_ws_bytes(uint64_t rows, uint64_t experts);
uint64_t balance_threads(const Matrix &m, const Routes &r);  // of the largest launch
hipError_t launch_balance_forward(const Matrix &m, const Routes &r, float coef, int32_t *counts_out,
                                  int32_t *rows_out, float *prob_out, float *loss_out, uint8_t *ws, hipStream_t s);
hipError_t launch_balance_backward(const Matrix &m, const Routes &r, float coef, const int32_t *counts,
                                   const int32_t *count_rows, const int32_t *rows_in, const float *upstream,
                                   void *grad, uint64_t grad_stride, hipStream_t s);

}  // namespace dr
