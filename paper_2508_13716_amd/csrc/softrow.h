// What the row-wise softmax operators (answers.hip, distill.hip) share: loads, exponentials, reductions, the order of logits.
#pragma once

#include "common.h"

#include <cmath>

namespace capgnn {

// exp(d / T) = 2^(d * L): L and what its rounding to float leaves of log2(e) / T
struct TempScale {
    float L, L_lo, inv_T;
    float least;            // differences below this are taken for it: exp is 0 and every product with them finite
};

static inline TempScale temp_scale(float temperature) {
    const double l = 1.4426950408889634074 / static_cast<double>(temperature);
    TempScale t;
    t.L = static_cast<float>(l);
    t.L_lo = static_cast<float>(l - static_cast<double>(t.L));
    t.inv_T = static_cast<float>(1.0 / static_cast<double>(temperature));
    t.least = static_cast<float>(-1000.0 / l);
    return t;
}

// 2^-64 to 2^64: everything formed from T and a difference of logits that matters stays a finite float
static inline bool good_temperature(float t) { return t >= 5.421010862427522e-20f && t <= 1.8446744073709552e19f; }

template <bool BF16> __device__ __forceinline__ float ld_logit(const char *p, int64_t i) {
    if constexpr (BF16) return __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[i]) << 16);
    else return reinterpret_cast<const float *>(p)[i];
}

typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
typedef float float_pair __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_two(float a, float b) {        // (one instruction)
    const float_pair v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16_pair));
}

template <bool BF16> __device__ __forceinline__ void st_grad(char *p, int64_t i, float v) {
    if constexpr (BF16) reinterpret_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(bf16_two(v, 0.f));
    else reinterpret_cast<float *>(p)[i] = v;
}

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// the larger of the two; NaN if either is (one instruction, as the maximum that skips NaN)
__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// exp(d / T), d <= 0 and not below TempScale::least.  The product d * L loses up to |d L| 2^-24 of the exponent; EXACT puts what it loses back
// to first order (float results; a bf16 result's rounding is thousands of times as large).
template <bool EXACT = true> __device__ __forceinline__ float exp_scaled(float d, const TempScale &t) {
    const float u = d * t.L, e = exp2_raw(u);
    if constexpr (!EXACT) return e;
    return fmaf(e, fmaf(d, t.L_lo, fmaf(d, t.L, -u)) * 0.69314718f, e);
}
__device__ __forceinline__ float difference(float z, float m0, const TempScale &t) { return max_of(z - m0, t.least); }

// exp((a - b) / T), a <= b, without the rounding of a - b either (a teacher's probabilities: few, so the operations more do not count)
__device__ __forceinline__ float exp_difference(float a, float b, const TempScale &t) {
    const float d = a - b;
    if (d < t.least) return 0.f;
    const float back = d - a, rest = (a - (d - back)) + (-b - back);
    const float u = d * t.L, e = exp2_raw(u);
    return fmaf(e, fmaf(rest, t.L, fmaf(d, t.L_lo, fmaf(d, t.L, -u))) * 0.69314718f, e);
}

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

// 16 bytes of logits from any address that is aligned to its elements (one load instruction), V of them
typedef uint32_t raw16 __attribute__((ext_vector_type(4)));
typedef raw16 raw16_by2 __attribute__((aligned(2)));
typedef raw16 raw16_by4 __attribute__((aligned(4)));
template <bool BF16> struct Raw {
    static constexpr int V = BF16 ? 8 : 4;
    static constexpr uint32_t BARRED = BF16 ? 0xff80ff80u : 0xff800000u;

    // j >= 0; a row has 2^30 classes at most: its bytes are counted in 32 bits, and the row's address may stay in scalar registers
    static __device__ __forceinline__ raw16 load(const char *p, int j) {
        if constexpr (BF16) return *reinterpret_cast<const raw16_by2 *>(p + static_cast<uint32_t>(j) * 2u);
        else return *reinterpret_cast<const raw16_by4 *>(p + static_cast<uint32_t>(j) * 4u);
    }
    static __device__ __forceinline__ float get(raw16 r, int e) {
        if constexpr (BF16) return __uint_as_float(e & 1 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16);
        else return __uint_as_float(r[e]);
    }
    // Logits [j, j + V) of a row that ends at `end`.  Where fewer are left the row's last V are read, and those before j are
    // barred in the result (all of them for j >= end): what is returned starts at class `start`.  SHORT: the row may have fewer than V.
    template <bool SHORT = false> static __device__ __forceinline__ raw16 load_until(const char *p, int j, int end, int *start) {
        const int from = j + V <= end ? j : end - V;
        raw16 r;
        *start = from;
        if (SHORT && from < 0) {
            r = raw16{BARRED, BARRED, BARRED, BARRED};
            for (int k = 0; k < end; ++k) {
                const uint32_t b = __float_as_uint(ld_logit<BF16>(p, k));
                const int e = k - from, w = BF16 ? e / 2 : e;
                const uint32_t mask = !BF16 ? 0xffffffffu : e & 1 ? 0xffff0000u : 0xffffu, v = BF16 && !(e & 1) ? b >> 16 : b;
#pragma unroll
                for (int q = 0; q < 4; ++q) if (q == w) r[q] = (r[q] & ~mask) | (v & mask);
            }
        } else {
            r = load(p, from);
        }
        if (__any(from != j)) {
            const int out = j - from;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (BF16) r[w] = 2 * w + 1 < out ? BARRED : 2 * w < out ? (r[w] & 0xffff0000u) | (BARRED & 0xffffu) : r[w];
                else r[w] = w < out ? BARRED : r[w];
            }
        }
        return r;
    }
};

// V floats to the gradient row p, classes [j, j + V), in the widest stores there are; V is that of the logits' type
typedef uint32_t raw8 __attribute__((ext_vector_type(2)));
typedef raw8 raw8_by2 __attribute__((aligned(2)));
template <bool DBF16, int V> __device__ __forceinline__ void st_vector(char *p, int j, const float (&g)[V]) {
    if constexpr (DBF16) {
        if constexpr (V == 8)
            *reinterpret_cast<raw16_by2 *>(p + static_cast<uint32_t>(j) * 2u) =
                raw16{bf16_two(g[0], g[1]), bf16_two(g[2], g[3]), bf16_two(g[4], g[5]), bf16_two(g[6], g[7])};
        else
            *reinterpret_cast<raw8_by2 *>(p + static_cast<uint32_t>(j) * 2u) = raw8{bf16_two(g[0], g[1]), bf16_two(g[2], g[3])};
    } else {
#pragma unroll
        for (int h = 0; h < V; h += 4)
            *reinterpret_cast<raw16_by4 *>(p + static_cast<uint32_t>(j + h) * 4u) =
                raw16{__float_as_uint(g[h]), __float_as_uint(g[h + 1]), __float_as_uint(g[h + 2]), __float_as_uint(g[h + 3])};
    }
}
template <bool DBF16, int V> __device__ __forceinline__ void ld_vector(const char *p, int j, float (&g)[V]) {
    if constexpr (DBF16) {
        raw16 r = {0, 0, 0, 0};
        if constexpr (V == 8) {
            r = *reinterpret_cast<const raw16_by2 *>(p + static_cast<uint32_t>(j) * 2u);
        } else {
            const raw8 q = *reinterpret_cast<const raw8_by2 *>(p + static_cast<uint32_t>(j) * 2u);
            r[0] = q[0];
            r[1] = q[1];
        }
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = Raw<true>::get(r, e);
    } else {
#pragma unroll
        for (int h = 0; h < V; h += 4) {
            const raw16 r = *reinterpret_cast<const raw16_by4 *>(p + static_cast<uint32_t>(j + h) * 4u);
#pragma unroll
            for (int e = 0; e < 4; ++e) g[h + e] = __uint_as_float(r[e]);
        }
    }
}

// From here on the compiler knows nothing of r: what it has unpacked or derived from it before is not kept in registers for later, and
// work on one vector is not mixed with that on the next (which took twice the registers; other waves fill the gaps).
__device__ __forceinline__ void forget(raw16 &r) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" : "+v"(r));
}
// The thread's number, of which the compiler knows nothing: addresses and conditions formed from it are not kept for the next use.
__device__ __forceinline__ int thread_anew() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// The same for a value that all threads have: what one pass over a row's vectors has found out about their number is not carried into the next
// (code for every number of vectors, a kilobyte of scratch memory a thread; or a loop's conditions kept in spilled registers).
__device__ __forceinline__ int uniform_anew(int x) {
    x = __builtin_amdgcn_readfirstlane(x);
    asm volatile("" : "+s"(x));
    return x;
}

// Rows of at most NARROW_C classes: a wave takes 64 / G of them at a time through LDS, G lanes a row with at most 32 classes each, so that a
// row's sums need hardly any exchange between lanes (lane groups over registers spent four times the instructions at 47 classes:
// 612000 rows were bound by them, not by memory).  The next rows' loads are under way while a wave works on its own.  A row starts
// G * odd words after the one before it: lanes that read the same class of their rows at once hit different banks.  A lane reads its
// classes NARROW_BATCH at a time; what is behind a row's end holds -inf (narrow_ends).
// Up to NARROW_C classes it is the faster one throughout, against a wave a row, us: answers of 100000 rows with k = 8, 100 f32 25 / 218, 256 f32
// 44 / 581, bf16 93 / 615; their gradient, 256 f32 54 / 72, bf16 37 / 53; distillation with k = 16, 100 f32 63 / 135, 256 f32 89 / 139, bf16
// 66 / 146.  By a wave beyond: 257 classes, answers 134 f32, 139 bf16, gradient 89 and 57, distillation 158 and 150.
constexpr int NARROW_C = 256;
constexpr int NARROW_G = NARROW_C / 32;     // lanes of a row at most
constexpr int NARROW_BATCH = 8;
constexpr int NARROW_WAVES = 2;     // of a workgroup; each works for itself
struct NarrowShape {
    int C, lg;              // G = 1 << lg
    int rows, pitch;        // of a wave; words between rows in LDS
    int each;               // classes of a lane, whole batches
    int pieces, magic;      // loads of a row (16 bytes, or one logit where a row is shorter than 16 bytes); item / pieces = item * magic >> 16
    int items;              // rows * pieces <= 64 * NarrowLoad::MOST
    size_t lds_wave;        // bytes, without extra
};

static inline NarrowShape narrow_shape(int C, int dtype) {
    NarrowShape s;
    const int V = dtype == CAPGNN_BF16 ? 8 : 4;
    s.C = C;
    s.lg = 0;
    while ((32 << s.lg) < C) ++s.lg;
    const int G = 1 << s.lg;
    s.rows = 64 / G;
    s.each = ((C + G - 1) / G + NARROW_BATCH - 1) / NARROW_BATCH * NARROW_BATCH;
    s.pitch = G * (s.each | 1);
    s.pieces = C < V ? C : (C + V - 1) / V;
    s.magic = (65536 + s.pieces - 1) / s.pieces;
    s.items = s.rows * s.pieces;
    s.lds_wave = static_cast<size_t>(s.rows) * s.pitch * sizeof(float);
    return s;
}

// LDS written by other lanes of the wave may be read after this
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// workgroups: as many as the chip holds at once (lds: bytes of one), or fewer
static inline unsigned narrow_grid(const NarrowShape &s, int64_t n, size_t lds) {
    const int64_t held = static_cast<int64_t>(160 * 1024 / lds) < 10 ? static_cast<int64_t>(160 * 1024 / lds) : 10;
    const int64_t needed = (n + NARROW_WAVES * s.rows - 1) / (NARROW_WAVES * s.rows);
    return static_cast<unsigned>(needed < NUM_CU * held ? needed : NUM_CU * held);
}

// -inf behind the ends of the wave's rows; nothing writes there afterwards
__device__ __forceinline__ void narrow_ends(const NarrowShape &s, float *lds, int lane) {
    const int behind = s.pitch - s.C;
    for (int i = lane; i < s.rows * behind; i += 64) lds[i / behind * s.pitch + s.C + i % behind] = -INFINITY;
}

// rows so near to one another that a wave's offsets are products of 24-bit numbers (one instruction; a 64-bit product takes many)
__device__ __forceinline__ bool narrow_near(int64_t pitch_bytes) { return pitch_bytes < 1 << 24; }

template <bool BF16> struct NarrowLoad {
    static constexpr int MOST = BF16 ? 7 : 8;       // (bf16: 4 of 16 bytes, or up to 7 of one logit)
    raw16 q[MOST];

    // rows [row0, row0 + s.rows) from row0 < n on, those beyond the last one again the last one; row0: the same for all lanes
    __device__ __forceinline__ void fetch(const NarrowShape &s, const char *Z, int64_t ldz, int64_t n, int64_t row0) {
        typedef Raw<BF16> R;
        constexpr int ES = BF16 ? 2 : 4;
        const int lane = thread_anew() & 63, last = static_cast<int>(n - row0 < s.rows ? n - row0 : s.rows) - 1;
        const char *rows = Z + row0 * ldz * ES;
        const bool near = narrow_near(ldz * ES);
        const uint32_t pitch = static_cast<uint32_t>(ldz * ES);
        const int items = uniform_anew(s.items);
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            const int item = i * 64 + lane;
            if (i * 64 >= items) break;                 // (the same for all lanes)
            if (item < items) {
                int r = item * s.magic >> 16;
                const int v = item - __mul24(r, s.pieces);
                r = r < last ? r : last;
                const int j = s.C < R::V ? v : v * R::V + R::V <= s.C ? v * R::V : s.C - R::V;
                const char *p = near ? rows + __umul24(r, pitch) : rows + r * ldz * ES;
                if (s.C < R::V) q[i][0] = __float_as_uint(ld_logit<BF16>(p, j));
                else q[i] = R::load(p, j);
            }
        }
    }

    __device__ __forceinline__ void put(const NarrowShape &s, float *lds) {
        typedef Raw<BF16> R;
        const int lane = thread_anew() & 63, items = uniform_anew(s.items);
#pragma unroll
        for (int i = 0; i < MOST; ++i) {
            const int item = i * 64 + lane;
            if (i * 64 >= items) break;
            if (item < items) {
                const int r = item * s.magic >> 16, v = item - __mul24(r, s.pieces);
                float *row = lds + __mul24(r, s.pitch);
                if (s.C < R::V) {
                    row[v] = __uint_as_float(q[i][0]);
                } else {
                    const int j = v * R::V + R::V <= s.C ? v * R::V : s.C - R::V;
#pragma unroll
                    for (int e = 0; e < R::V; ++e) row[j + e] = R::get(q[i], e);
                }
            }
        }
    }
};

// The wave's rows of gradients, from LDS as NarrowLoad put the logits there; add: to what dZ holds.
template <bool BF16, bool DBF16>
__device__ __forceinline__ void narrow_store(const NarrowShape &s, const float *lds, char *dZ, int64_t lddz, int64_t n, int64_t row0, bool add) {
    constexpr int V = Raw<BF16>::V, ES = DBF16 ? 2 : 4;
    const int lane = thread_anew() & 63, there = static_cast<int>(n - row0 < s.rows ? n - row0 : s.rows);
    char *rows = dZ + row0 * lddz * ES;
    const bool near = narrow_near(lddz * ES);
    const uint32_t pitch = static_cast<uint32_t>(lddz * ES);
    const int items = uniform_anew(s.items);
#pragma unroll
    for (int i = 0; i < NarrowLoad<BF16>::MOST; ++i) {
        const int item = i * 64 + lane;
        if (i * 64 >= items) break;
        const int r = item * s.magic >> 16, v = item - __mul24(r, s.pieces);
        if (item < items && r < there) {
            char *p = near ? rows + __umul24(r, pitch) : rows + r * lddz * ES;
            const float *row = lds + __mul24(r, s.pitch);
            if (s.C < V || (add && v * V + V > s.C)) {          // one logit, or what is left of a row
                const int j = s.C < V ? v : v * V, end = s.C < V ? v + 1 : s.C;
                for (int k = j; k < end; ++k) st_grad<DBF16>(p, k, add ? ld_logit<DBF16>(p, k) + row[k] : row[k]);
            } else {
                const int j = v * V + V <= s.C ? v * V : s.C - V;        // (a row's last piece: some of what its neighbour writes, too)
                float g[V];
                if (add) ld_vector<DBF16>(p, j, g);
#pragma unroll
                for (int e = 0; e < V; ++e) g[e] = add ? g[e] + row[j + e] : row[j + e];
                st_vector<DBF16>(p, j, g);
            }
        }
    }
}

// v of the lane OFF before this one, round about in its 16 (no way through LDS)
template <int OFF, typename T> __device__ __forceinline__ T lane_before(T v) {
    static_assert(sizeof(T) % 4 == 0, "whole registers");
    struct Words { int w[sizeof(T) / 4]; } x = __builtin_bit_cast(Words, v);
#pragma unroll
    for (int &w : x.w) w = __builtin_amdgcn_update_dpp(w, w, 0x120 + OFF, 0xf, 0xf, false);
    return __builtin_bit_cast(T, x);
}
// op over the wave, in pairs of lanes 32, 16, 8, 4, 2 and 1 apart.  (Lanes 16, 8, ... apart hold the same by then: the one before is as good.)
template <typename T, typename Op> __device__ __forceinline__ T wave_all(T v, Op op) {
    v = op(v, __shfl_xor(v, 32));
    v = op(v, __shfl_xor(v, 16));
    v = op(v, lane_before<8>(v));
    v = op(v, lane_before<4>(v));
    v = op(v, lane_before<2>(v));
    return op(v, lane_before<1>(v));
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

constexpr int CLASSES_MOST = 1 << 30;       // class numbers plus a tile stay ints

// maximum and sum of exponentials of every thread, taken together: the same in every thread.  red: a pair per wave; a barrier has to
// pass before it is used again.
template <int THREADS> __device__ __forceinline__ void group_softmax(float &m, float &s, const TempScale &t, float2 *red) {
    const float M = wave_all(m, OpMax());
    s = wave_all(s * exp2_raw((m - safe_max(M)) * t.L), OpSum());
    m = M;
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_float2(m, s);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) m = max_of(m, red[w].x);
        const float ref = safe_max(m);
        s = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) s += red[w].y * exp2_raw((red[w].x - ref) * t.L);
    }
}

static inline bool element_aligned(const void *p, int dtype) { return reinterpret_cast<uintptr_t>(p) % elem_bytes(dtype) == 0; }

}  // namespace capgnn
