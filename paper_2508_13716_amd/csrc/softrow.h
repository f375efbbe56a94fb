// What the row-wise softmax operators (answers.hip, distill.hip) share: loads, exponentials, reductions, the order of logits.
#pragma once

#include "common.h"

#include <cmath>

namespace capgnn {

// exp(d / T) = 2^(d * L): L and what its rounding to float leaves of log2(e) / T
struct TempScale {
    float L, L_lo, inv_T;
};

static inline TempScale temp_scale(float temperature) {
    const double l = 1.4426950408889634074 / static_cast<double>(temperature);
    TempScale t;
    t.L = static_cast<float>(l);
    t.L_lo = static_cast<float>(l - static_cast<double>(t.L));
    t.inv_T = static_cast<float>(1.0 / static_cast<double>(temperature));
    return t;
}

// T > 0, finite, and 1/T a finite float too
static inline bool good_temperature(float t) { return t > 1e-37f && t < 1e37f; }

template <bool BF16> __device__ __forceinline__ float ld_logit(const char *p, int64_t i) {
    if constexpr (BF16) return __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[i]) << 16);
    else return reinterpret_cast<const float *>(p)[i];
}

__device__ __forceinline__ uint32_t bf16_bits(float v) {        // round to nearest even; NaN stays NaN
    uint32_t u = __float_as_uint(v);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (u >> 16) | 0x40u;
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

template <bool BF16> __device__ __forceinline__ void st_grad(char *p, int64_t i, float v) {
    if constexpr (BF16) reinterpret_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(bf16_bits(v));
    else reinterpret_cast<float *>(p)[i] = v;
}

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// exp(d / T), d <= 0.  The product d * L loses up to |d L| 2^-24 of the exponent: what it loses is put back to first order.
__device__ __forceinline__ float exp_scaled(float d, const TempScale &t) {
    const float u = d * t.L;
    const float e = exp2_raw(u);
    const float lost = fmaf(d, t.L_lo, fmaf(d, t.L, -u));
    return e > 0.f ? fmaf(e, lost * 0.69314718f, e) : e;        // (d = -inf: lost is NaN, e is 0; a NaN d gives a NaN e)
}

// the larger of the two, a NaN never (the sum of the exponentials shows it)
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }

// the reference point of a row: 0 where every class is barred, so that -inf - -inf is never formed
__device__ __forceinline__ float safe_max(float m) { return m == -INFINITY ? 0.f : m; }

// Larger logit, then lower class: larger key.  NaN is the largest value; -0 and +0 are equal.  No key is 0 or all ones.
constexpr uint32_t ORDER_NAN = 0xfffffffeu;
__device__ __forceinline__ uint32_t logit_order(float z) {
    if (!(z == z)) return ORDER_NAN;
    const uint32_t u = __float_as_uint(z + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_logit(uint32_t o) {
    if (o == ORDER_NAN) return __uint_as_float(0x7fc00000u);
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t logit_key(float z, int k) {
    return static_cast<uint64_t>(logit_order(z)) << 32 | (0xffffffffu - static_cast<uint32_t>(k));
}

template <typename T, typename Op> __device__ __forceinline__ T wave_all(T v, Op op) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = op(v, __shfl_xor(v, off));
    return v;
}

// op over the workgroup, the same value in every thread; red: one T per wave.  Ends with a barrier before red may be used again.
template <int THREADS, typename T, typename Op> __device__ __forceinline__ T group_all(T v, T *red, Op op) {
    v = wave_all(v, op);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v = op(v, red[w]);
        __syncthreads();
    }
    return v;
}

struct OpMax { __device__ float operator()(float a, float b) const { return max_of(a, b); } };
struct OpSum {
    template <typename T> __device__ T operator()(T a, T b) const { return a + b; }
};
struct OpMaxKey { __device__ unsigned long long operator()(unsigned long long a, unsigned long long b) const { return a > b ? a : b; } };

// The number of masked rows (at least 1) on the device: norm_dev[0].  scratch: 512 doubles.  In ops.hip.
int launch_mask_count(int64_t n, const uint8_t *mask, float *norm_dev, double *scratch, hipStream_t stream);

static inline bool element_aligned(const void *p, int dtype) { return reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype) == 0; }

}  // namespace capgnn
