// Rows of elements at any pitch, vector by vector: what the row-wise operators of norm.hip, embed.hip and linear.hip share.
#pragma once

#include "softrow.h"

namespace capgnn {

// elements of a row that a lane takes at a time: 16 bytes of its type
template <bool BF16> constexpr int ROW_V = BF16 ? 8 : 4;

// V elements of a row from element j on (V: 4 or 8, or 1 for rows shorter than a vector); rows are shorter than 2^30 elements
template <bool BF16, int V> __device__ __forceinline__ void ld_row(const char *p, int j, float (&v)[V]) {
    if constexpr (V == 1) v[0] = ld_logit<BF16>(p, j);
    else ld_vector<BF16, V>(p, j, v);
}
template <bool BF16, int V> __device__ __forceinline__ void st_row(char *p, int j, const float (&v)[V]) {
    if constexpr (V == 1) st_grad<BF16>(p, j, v[0]);
    else st_vector<BF16, V>(p, j, v);
}
// the same where the type is known at run time (one branch for all lanes)
template <int V> __device__ __forceinline__ void ld_row_of(bool bf16, const char *p, int j, float (&v)[V]) {
    if (bf16) ld_row<true, V>(p, j, v);
    else ld_row<false, V>(p, j, v);
}
template <int V> __device__ __forceinline__ void st_row_of(bool bf16, char *p, int j, const float (&v)[V]) {
    if (bf16) st_row<true, V>(p, j, v);
    else st_row<false, V>(p, j, v);
}

// a vector of a row as it lies in memory, to be unpacked when it is used
template <bool BF16, int V> struct RawRow {
    raw16 r;
    __device__ __forceinline__ void clear() { r = raw16{0, 0, 0, 0}; }
    __device__ __forceinline__ void load(const char *p, int j) {
        static_assert(V == 1 || V == ROW_V<BF16>, "a vector is 16 bytes");
        if constexpr (V == 1) r[0] = __float_as_uint(ld_logit<BF16>(p, j));
        else r = Raw<BF16>::load(p, j);
    }
    __device__ __forceinline__ void arrive() { asm volatile("" : "+v"(r)); }    // what follows waits for the load
    __device__ __forceinline__ float get(int e) const { return V == 1 ? __uint_as_float(r[0]) : Raw<BF16>::get(r, e); }
};

// four floats to E4M3, nearest even, the first in the low byte; |v| <= 464 (what rounds to the largest value, 448) or NaN
__device__ __forceinline__ uint32_t e4m3_four(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true));
}
typedef uint32_t raw4_by1 __attribute__((aligned(1)));
typedef raw8 raw8_by1 __attribute__((aligned(1)));
template <int V> __device__ __forceinline__ void st_e4m3(char *p, int j, const float (&v)[V]) {
    if constexpr (V == 1) reinterpret_cast<uint8_t *>(p)[j] = static_cast<uint8_t>(e4m3_four(v[0], 0.f, 0.f, 0.f));
    else if constexpr (V == 4) *reinterpret_cast<raw4_by1 *>(p + static_cast<uint32_t>(j)) = e4m3_four(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<raw8_by1 *>(p + static_cast<uint32_t>(j)) = raw8{e4m3_four(v[0], v[1], v[2], v[3]), e4m3_four(v[4], v[5], v[6], v[7])};
}

static inline bool is_float_type(int dtype) { return dtype == CAPGNN_F32 || dtype == CAPGNN_BF16; }
static inline bool row_aligned(const void *p, int dtype) {
    return (reinterpret_cast<uintptr_t>(p) & (dtype == CAPGNN_F32 ? 3u : dtype == CAPGNN_BF16 ? 1u : 0u)) == 0;
}
static inline int pow2_at_least(int x) {
    int p = 1;
    while (p < x) p *= 2;
    return p;
}

}  // namespace capgnn
