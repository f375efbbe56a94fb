// Products with an epilogue, Y = act(A W^T + bias) + R, and the epilogue's gradient.
//
// Both operands run along the reduction index, so a tile of either is the same thing whatever its type: rows of 128 bytes, 32 fp32,
// 64 bf16 or 128 e4m3 numbers of k.  LDS holds such tiles in units of 16 bytes, unit u of row r at place u ^ (r / 2 % 8): the units of the
// same k of sixteen rows lie in different banks (of eight rows only, u ^ (r % 8): 8192^3 bf16 4 % slower).  The matrix instructions take 32 x 32 results; which k a lane's bytes are does not matter as long as
// both operands agree, so a lane of the lower and one of the upper half take alternate units of their row.
//
// D layout of the 32 x 32 instructions: register r of lane l holds row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32.
//
// us (TFLOP/s), epilogue of activation and residual included: 8192^3 bf16 903 (1218; a library product alone reaches 1350), 8192 x 8192 x 4096
// e4m3 316 (1740; 2740), fp32 2403 (229; 154), 4096^3 bf16 111 (1240).  The matrix cores bound the wide ones, at the clock that power
// leaves them (8192^3 bf16: busy 68 % of the cycles, at 1.6 GHz); the 8-bit one spends a quarter of its time on results, whose
// arithmetic no other workgroup on the compute unit hides (busy 37 %, at 2.0 GHz).
#include "rows.h"
#include "linear_plan.h"

#include <algorithm>
#include <type_traits>
#include <utility>

namespace capgnn {

typedef float acc16 __attribute__((ext_vector_type(16)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef __bf16 half8 __attribute__((ext_vector_type(8)));

struct LinearArgs {
    int64_t M, N, K;
    const char *A, *W;
    int64_t lda, ldw;           // in bytes
    const float *a_scale, *w_scale, *bias;
    int act;
    const char *R;
    char *U, *Y;
    int64_t ldr, ldu, ldy;      // in bytes
    int out_bf16;
    float *part;                // sums of parts of the reduction, [parts][M][part_ld], or null
    int64_t part_ld;
    int64_t part_k;             // of a part: whole steps
};

// A's and W's part of the reduction that is workgroup row blockIdx.y's
struct Stretch {
    const char *A, *W;
    int64_t K;
};
template <int ES> __device__ __forceinline__ Stretch stretch_of(const LinearArgs &g) {
    if (!g.part) return {g.A, g.W, g.K};
    const int64_t k0 = g.part_k * blockIdx.y;
    return {g.A + k0 * ES, g.W + k0 * ES, min(g.part_k, g.K - k0)};
}

// ------------------------------------------------------------------ activations
// exp(-x) and 1 / x by the hardware's instructions, one unit in the last place each: what the formulas lose by that is a few EPS |u|.
__device__ __forceinline__ float exp_minus(float x) { return __builtin_amdgcn_exp2f(x * -1.4426950408889634f); }
__device__ __forceinline__ float logistic(float u) { return __builtin_amdgcn_rcpf(1.f + exp_minus(u)); }

// Phi(u), the normal distribution, and exp(-u^2 / 2): 1 - Phi(|u|) = t (a1 + t (a2 + ...)) exp(-u^2 / 2) / 2 with t = 1 / (1 + p |u| / 2^1/2),
// Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26: erf to 1.5e-7, Phi to 0.75e-7.  (erff takes two branches
// of polynomials, several times the operations.)
__device__ __forceinline__ float normal(float u, float *bell) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, fabsf(u), 1.f));
    const float e = exp_minus(0.5f * u * u);
    *bell = e;
    const float p = fmaf(fmaf(fmaf(fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f), t, 0.5f * 1.421413741f), t, 0.5f * -0.284496736f), t, 0.5f * 0.254829592f);
    const float tail = p * t * e;
    return u < 0.f ? tail : 1.f - tail;
}
template <int ACT> __device__ __forceinline__ float act_of(float u) {
    float bell;
    if constexpr (ACT == CAPGNN_ACT_RELU) return u <= 0.f ? 0.f : u;           // (a NaN stays one)
    else if constexpr (ACT == CAPGNN_ACT_GELU) return u * normal(u, &bell);
    else if constexpr (ACT == CAPGNN_ACT_SILU) return u * logistic(u);
    else return u;
}
template <int ACT> __device__ __forceinline__ float act_slope(float u) {
    if constexpr (ACT == CAPGNN_ACT_RELU) return u > 0.f ? 1.f : u <= 0.f ? 0.f : u;
    else if constexpr (ACT == CAPGNN_ACT_GELU) {
        float bell;
        const float phi = normal(u, &bell);
        return fmaf(u * 0.39894228040143268f, bell, phi);
    } else if constexpr (ACT == CAPGNN_ACT_SILU) {
        const float s = logistic(u);
        return s * fmaf(u, 1.f - s, 1.f);
    } else return 1.f;
}
// f(ACT) with the activation as a compile-time number
template <class F> __host__ __device__ __forceinline__ void with_act(int act, F f) {
    if (act == CAPGNN_ACT_GELU) f(std::integral_constant<int, CAPGNN_ACT_GELU>());
    else if (act == CAPGNN_ACT_SILU) f(std::integral_constant<int, CAPGNN_ACT_SILU>());
    else if (act == CAPGNN_ACT_RELU) f(std::integral_constant<int, CAPGNN_ACT_RELU>());
    else f(std::integral_constant<int, CAPGNN_ACT_NONE>());
}
template <int V> __device__ __forceinline__ void act_all(int act, float (&v)[V]) {
    with_act(act, [&](auto k) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = act_of<k.value>(v[e]);
    });
}

// V elements of which the first `count` are inside the matrix
template <int V> __device__ __forceinline__ void ld_some(bool bf16, const char *p, int count, float (&v)[V]) {
    if (count == V) return ld_row_of<V>(bf16, p, 0, v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = e < count ? bf16 ? ld_logit<true>(p, e) : ld_logit<false>(p, e) : 0.f;
}
template <int V> __device__ __forceinline__ void st_some(bool bf16, char *p, int count, const float (&v)[V]) {
    if (count == V) return st_row_of<V>(bf16, p, 0, v);
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < count) bf16 ? st_grad<true>(p, e, v[e]) : st_grad<false>(p, e, v[e]);
}

// V neighbouring sums of row i from column j on, the first `count` of them inside the matrix: the whole epilogue
template <int V> __device__ __forceinline__ void finish(const LinearArgs &g, int64_t i, int64_t j, int count, float (&v)[V]) {
    const int es = g.out_bf16 ? 2 : 4;
    if (g.a_scale) {
        const float s = g.a_scale[i];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] *= s;
    }
    float x[V];
    if (g.w_scale) {
        ld_some<V>(false, reinterpret_cast<const char *>(g.w_scale + j), count, x);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] *= x[e];
    }
    if (g.bias) {
        ld_some<V>(false, reinterpret_cast<const char *>(g.bias + j), count, x);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += x[e];
    }
    if (g.U) st_some<V>(g.out_bf16, g.U + i * g.ldu + j * es, count, v);
    act_all<V>(g.act, v);
    if (g.R) {
        ld_some<V>(g.out_bf16, g.R + i * g.ldr + j * es, count, x);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += x[e];
    }
    st_some<V>(g.out_bf16, g.Y + i * g.ldy + j * es, count, v);
}

// ------------------------------------------------------------------ the matrix instructions, on 16-byte units
constexpr int UNITS = 8;                // units of a tile's row

// e4m3 operands of a float result.  The 8-bit matrix instructions add the products of eight neighbouring k at a time and drop, toward zero,
// what lies below 2^-13 of the largest one's power of two (groups of eight are then added in float): less than 7 * 2^-13 of each group's largest
// product, 1.3e-5 of a sum's size with normally distributed operands.  Beside a bf16 result's rounding that is nothing (8192 x 8192 x 4096: 1.669e-3
// off float64, root mean square, with it and without; one result in 190 is rounded the other way), but a hundred times a float's.  So for float
// results the operands are widened to bf16, exactly, and take the bf16 instruction, at half the rate.
constexpr int E4M3_FINE = 3;
// fp32 operands cut into three bf16 numbers each, exactly; the six largest of the nine products go to the bf16 instruction, smallest first, and what
// is dropped is 2^-23 of a product at most.  Six instructions stand for eight fp32 ones of twice the time.
constexpr int F32_CUT = 4;
template <int DT> constexpr int BYTES = DT == CAPGNN_F32 || DT == F32_CUT ? 4 : DT == CAPGNN_BF16 ? 2 : 1;

__device__ __forceinline__ int unit_at(int row, int unit) { return row * UNITS + (unit ^ (row >> 1 & 7)); }

// half e (eight numbers) of a unit of e4m3, as bf16
__device__ __forceinline__ half8 widen8(raw16 u, int e) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * e], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * e], 1.f, true);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * e + 1], 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * e + 1], 1.f, true);
    return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 16 bytes of a row from element k on; elements from `end` on are zero and not read
template <int DT> __device__ __forceinline__ raw16 load_unit(const char *row, int64_t k, int64_t end) {
    constexpr int E = 16 / BYTES<DT>;
    typedef raw16 raw16_by1 __attribute__((aligned(1)));
    if (k + E <= end) return *reinterpret_cast<const raw16_by1 *>(row + k * BYTES<DT>);
    raw16 r = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (k + e < end) {
            if constexpr (BYTES<DT> == 4) r[e] = reinterpret_cast<const uint32_t *>(row)[k + e];
            else if constexpr (BYTES<DT> == 2) r[e / 2] |= uint32_t(reinterpret_cast<const uint16_t *>(row)[k + e]) << (e % 2 * 16);
            else r[e / 4] |= uint32_t(reinterpret_cast<const uint8_t *>(row)[k + e]) << (e % 4 * 8);
        }
    return r;
}

// a step's products are formed a slice of k at a time, one instruction's (of fp32: four) for each pair of tiles
template <int DT> constexpr int SLICES = DT == CAPGNN_E4M3 || DT == F32_CUT ? 2 : 4;

template <int DT, int T> struct Slice {                                 // a lane's operands of T tiles' rows
    static constexpr int U = 4 / SLICES<DT>;
    raw16 u[T][U];
    __device__ __forceinline__ void read(const raw16 *tile, int row, int half, int s) {
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int q = 0; q < U; ++q) u[i][q] = tile[unit_at(row + i * 32, (2 * s + half) * U + q)];
    }
};
__device__ __forceinline__ int8v join_units(raw16 lo, raw16 hi) {
    return int8v{int(lo[0]), int(lo[1]), int(lo[2]), int(lo[3]), int(hi[0]), int(hi[1]), int(hi[2]), int(hi[3])};
}
// eight floats as three times eight bf16
struct Cut {
    half8 p[3];
    __device__ __forceinline__ void operator()(raw16 lo, raw16 hi) {
        uint32_t w[3][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float x = __uint_as_float(k < 2 ? lo[2 * k] : hi[2 * k - 4]), y = __uint_as_float(k < 2 ? lo[2 * k + 1] : hi[2 * k - 3]);
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                w[q][k] = bf16_two(x, y);
                x -= __uint_as_float(w[q][k] << 16);
                y -= __uint_as_float(w[q][k] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) p[q] = __builtin_bit_cast(half8, raw16{w[q][0], w[q][1], w[q][2], w[q][3]});
    }
};
template <int TM, int TN>
__device__ __forceinline__ void multiply_cut(const Slice<F32_CUT, TM> &a, const Slice<F32_CUT, TN> &b, acc16 (&acc)[TM][TN]) {
    Cut cb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) cb[j](b.u[j][0], b.u[j][1]);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        Cut ca;
        ca(a.u[i][0], a.u[i][1]);
#pragma unroll
        for (int s = 3; s-- > 0;)       // pieces p of A and s - p of W, 2^-8s of the product each
#pragma unroll
            for (int p = 0; p < 3; ++p)
                if (p <= s) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ca.p[p], cb[j].p[s - p], acc[i][j], 0, 0, 0);
                }
    }
}

template <int DT, int TM, int TN>
__device__ __forceinline__ void multiply_slice(const Slice<DT, TM> &a, const Slice<DT, TN> &b, acc16 (&acc)[TM][TN]) {
    if constexpr (DT == F32_CUT) return multiply_cut<TM, TN>(a, b, acc);
    else
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            if constexpr (DT == CAPGNN_E4M3) {
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join_units(a.u[i][0], a.u[i][1]), join_units(b.u[j][0], b.u[j][1]), acc[i][j], 0, 0, 0,
                                                                            0x7f7f7f7f, 0, 0x7f7f7f7f);
            } else if constexpr (DT == CAPGNN_BF16) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(half8, a.u[i][0]), __builtin_bit_cast(half8, b.u[j][0]), acc[i][j], 0, 0, 0);
            } else if constexpr (DT == E4M3_FINE) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(a.u[i][0], e), widen8(b.u[j][0], e), acc[i][j], 0, 0, 0);
            } else if constexpr (DT == CAPGNN_F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.u[i][0][e]), __uint_as_float(b.u[j][0][e]), acc[i][j], 0, 0, 0);
            }
        }
}

// ------------------------------------------------------------------ tiles
// Where a wave's results leave through: 32 rows at a time, so that memory is read and written along the rows
template <int TN> constexpr int STAGE_PITCH = TN * 32 + 8;              // floats: four rows further lie in the other half of the banks
template <int WAVES, int TN> constexpr int STAGE_BYTES = WAVES * 32 * STAGE_PITCH<TN> * 4;

template <int... I, class F> __device__ __forceinline__ void repeat(std::integer_sequence<int, I...>, F f) { (f(std::integral_constant<int, I>()), ...); }

// 8 neighbouring results as they lie in memory
template <bool OB> struct RawOut {
    raw16 r[OB ? 1 : 2];
    __device__ __forceinline__ void load(const char *p) {
        if constexpr (OB) r[0] = *reinterpret_cast<const raw16_by2 *>(p);
        else {
            r[0] = *reinterpret_cast<const raw16_by4 *>(p);
            r[1] = *reinterpret_cast<const raw16_by4 *>(p + 16);
        }
    }
    __device__ __forceinline__ float get(int e) const { return OB ? Raw<true>::get(r[0], e) : __uint_as_float(r[OB ? 0 : e / 4][e % 4]); }
};

// OB: results in bf16.  A lane keeps its 8 columns, so their bias and scales are read once; the residual's rows are all asked for before the
// results of the 32 rows are on their way through LDS.
template <bool OB, int WR, int WC, int TM, int TN>
__device__ __forceinline__ void store_tile(const LinearArgs &g, raw16 *lds, int64_t m0, int64_t n0, const acc16 (&acc)[TM][TN]) {
    constexpr int PITCH = STAGE_PITCH<TN>, LANES = TN * 4, ROWS = 64 / LANES, PASSES = 32 / ROWS, ES = OB ? 2 : 4;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, half = lane / 32;
    float *stage = reinterpret_cast<float *>(lds) + wave * 32 * PITCH;
    const float *mine = stage + lane / LANES * PITCH + lane % LANES * 8;
    const int64_t col = n0 + lane % LANES * 8;
    const int count = static_cast<int>(max(min(g.N - col, int64_t(8)), int64_t(0)));
    if (g.part) {
        repeat(std::make_integer_sequence<int, TM>(), [&](auto at) __attribute__((always_inline)) {
            constexpr int i = at.value;
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int k = 0; k < 16; ++k) stage[(8 * (k / 4) + 4 * half + k % 4) * PITCH + j * 32 + lane % 32] = acc[i][j][k];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int64_t row = m0 + i * 32 + lane / LANES + p * ROWS;
                if (row < g.M && count) {               // (rows of parts are whole vectors of 8)
                    float v[8];
                    ld_row<false, 8>(reinterpret_cast<const char *>(mine + p * ROWS * PITCH), 0, v);
                    st_row<false, 8>(reinterpret_cast<char *>(g.part + (blockIdx.y * g.M + row) * g.part_ld + col), 0, v);
                }
            }
            __builtin_amdgcn_wave_barrier();
        });
        return;
    }
    float bias[8], scale[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        bias[e] = 0.f;
        scale[e] = 1.f;
    }
    if (count) {
        if (g.bias) ld_some<8>(false, reinterpret_cast<const char *>(g.bias + col), count, bias);
        if (g.w_scale) ld_some<8>(false, reinterpret_cast<const char *>(g.w_scale + col), count, scale);
    }
    // (one copy of the code per 32 rows, whatever its size: a loop over accumulators that is not unrolled would put them into memory)
    repeat(std::make_integer_sequence<int, TM>(), [&](auto at) __attribute__((always_inline)) {
        constexpr int i = at.value;
        const int64_t first = m0 + i * 32 + lane / LANES;               // the lane's rows: first + p * ROWS
        RawOut<OB> r[PASSES];
        if (g.R && count == 8) {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) r[p].load(g.R + min(first + p * ROWS, g.M - 1) * g.ldr + col * ES);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) stage[(8 * (k / 4) + 4 * half + k % 4) * PITCH + j * 32 + lane % 32] = acc[i][j][k];
        __builtin_amdgcn_wave_barrier();
        if (count == 8) {
            with_act(g.act, [&](auto act) {
#pragma unroll
                for (int p = 0; p < PASSES; ++p) {
                    const int64_t row = first + p * ROWS;
                    if (row >= g.M) continue;
                    float v[8];
                    ld_row<false, 8>(reinterpret_cast<const char *>(mine + p * ROWS * PITCH), 0, v);
                    if (g.a_scale) {                    // (one after the other: the scales' product may leave float's range where the result does not)
                        const float s = g.a_scale[row];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] *= s;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], scale[e], bias[e]);
                    if (g.U) st_row<OB, 8>(g.U + row * g.ldu + col * ES, 0, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[e] = act_of<act.value>(v[e]);
                        if (g.R) v[e] += r[p].get(e);
                    }
                    st_row<OB, 8>(g.Y + row * g.ldy + col * ES, 0, v);
                }
            });
        } else if (count) {
#pragma unroll 1
            for (int p = 0; p < PASSES; ++p) {
                if (first + p * ROWS >= g.M) break;
                float v[8];
                ld_row<false, 8>(reinterpret_cast<const char *>(mine + p * ROWS * PITCH), 0, v);
                finish<8>(g, first + p * ROWS, col, count, v);
            }
        }
        __builtin_amdgcn_wave_barrier();
    });
}

// Tile of a workgroup.  Workgroups go round the L2 domains one by one: each domain gets a stretch of tiles, in bands of 8 rows of tiles, so that
// what runs on it at a time shares rows of both operands.
__device__ __forceinline__ void tile_of(unsigned tiles_m, unsigned tiles_n, unsigned *m, unsigned *n) {
    const unsigned all = tiles_m * tiles_n, d = blockIdx.x % NUM_XCD, k = blockIdx.x / NUM_XCD;
    const unsigned t = all / NUM_XCD * d + min(d, all % NUM_XCD) + k;
    const unsigned band = t / (8 * tiles_n), first = band * 8, rows = min(8u, tiles_m - first), in = t - band * 8 * tiles_n;
    *m = first + in % rows;
    *n = in / rows;
}

// WR x WC waves with TM x TN accumulators of 32 x 32 each: a tile of WR TM 32 rows of A by WC TN 32 rows of W.
template <int DT, bool OB, int WR, int WC, int TM, int TN> __global__ __launch_bounds__(WR *WC * 64) void linear_tile_kernel(LinearArgs g) {
    constexpr int T = WR * WC * 64, BM = WR * TM * 32, BN = WC * TN * 32, STEP = 128 / BYTES<DT>;
    constexpr int PA = BM * UNITS / T, PB = BN * UNITS / T;             // units that a thread loads
    constexpr int STAGE = STAGE_BYTES<WR * WC, TN>, TILES = (BM + BN) * UNITS * 16;
    __shared__ raw16 lds[(STAGE > TILES ? STAGE : TILES) / 16];
    raw16 *As = lds, *Bs = lds + BM * UNITS;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, half = lane / 32;
    const int wm = wave / WC * TM * 32, wn = wave % WC * TN * 32;
    unsigned tm, tn;
    tile_of(static_cast<unsigned>((g.M + BM - 1) / BM), static_cast<unsigned>((g.N + BN - 1) / BN), &tm, &tn);
    const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
    const Stretch x = stretch_of<BYTES<DT>>(g);
    acc16 acc[TM][TN] = {};
    raw16 ra[PA], rb[PB];
    auto fetch = [&](int64_t k) {
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const int u = p * T + threadIdx.x;
            ra[p] = load_unit<DT>(x.A + min(m0 + u / UNITS, g.M - 1) * g.lda, k + u % UNITS * (16 / BYTES<DT>), x.K);
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int u = p * T + threadIdx.x;
            rb[p] = load_unit<DT>(x.W + min(n0 + u / UNITS, g.N - 1) * g.ldw, k + u % UNITS * (16 / BYTES<DT>), x.K);
        }
    };
    if (x.K > 0) fetch(0);
    for (int64_t k = 0; k < x.K; k += STEP) {
        __syncthreads();
#pragma unroll
        for (int p = 0; p < PA; ++p) As[unit_at((p * T + threadIdx.x) / UNITS, threadIdx.x % UNITS)] = ra[p];
#pragma unroll
        for (int p = 0; p < PB; ++p) Bs[unit_at((p * T + threadIdx.x) / UNITS, threadIdx.x % UNITS)] = rb[p];
        __syncthreads();
        if (k + STEP < x.K) fetch(k + STEP);
#pragma unroll
        for (int s = 0; s < SLICES<DT>; ++s) {
            Slice<DT, TM> a;
            Slice<DT, TN> b;
            a.read(As, wm + lane % 32, half, s);
            b.read(Bs, wn + lane % 32, half, s);
            multiply_slice<DT, TM, TN>(a, b, acc);
        }
    }
    __syncthreads();
    store_tile<OB, WR, WC, TM, TN>(g, lds, m0 + wm, n0 + wn, acc);
}

// The same for operands whose rows start on 4 bytes (what a load to LDS asks for) and need no check but at the last step: loads go straight to LDS, steps ahead, and the operands
// of a slice (half or a quarter of a step) are read while the one before is multiplied, across the barrier too: behind the last slice's
// reads the other buffer's loads are waited for, this one's are free to start, and the next step's first slice is read.
// The order of a slice: reads of the next one's operands, then loads to LDS, between its matrix instructions.  (Asked for all at once they
// keep the only wave of a SIMD from issuing matrix instructions for a fifth of a step.)
template <int MFMAS, int READS, int LOADS> __device__ __forceinline__ void interleave() {
    constexpr int BATCH = MFMAS > 32 ? MFMAS / 32 : 1, N = MFMAS / BATCH, HALF = LOADS ? N / 2 : N;     // loads follow the reads (the compiler
#pragma unroll                                                                                          // takes them for writes of what is read)
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, BATCH, 0);                  // matrix instructions
        constexpr auto due = [](int k, int n, int of) { return (k + 1) * n / of - k * n / of; };
        if (i < HALF) {
            if (due(i, READS, HALF) == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);            // reads of LDS
            if (due(i, READS, HALF) == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            if (due(i, READS, HALF) == 3) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
        } else {
            if (due(i - HALF, LOADS, N - HALF) == 1) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0); // loads
            if (due(i - HALF, LOADS, N - HALF) == 2) __builtin_amdgcn_sched_group_barrier(0x020, 2, 0);
        }
    }
}

// NB: steps that LDS holds
template <int DT, bool OB, int WR, int WC, int TM, int TN, int NB> __global__ __launch_bounds__(WR *WC * 64) void linear_direct_kernel(LinearArgs g) {
    constexpr int T = WR * WC * 64, BM = WR * TM * 32, BN = WC * TN * 32, STEP = 128 / BYTES<DT>, S = SLICES<DT>;
    constexpr int ROWS = T / UNITS;                                     // of a load of all waves
    constexpr int PA = BM / ROWS, PB = BN / ROWS, TILE = (BM + BN) * UNITS;
    static_assert(STAGE_BYTES<WR * WC, TN> <= NB * TILE * 16, "results leave through the tiles' memory");
    static_assert((NB - 2) * (PA + PB) < 64, "loads that a wave can wait for one by one");
    __shared__ raw16 lds[NB * TILE];
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, half = lane / 32;
    const int wm = wave / WC * TM * 32, wn = wave % WC * TN * 32;
    unsigned tm, tn;
    tile_of(static_cast<unsigned>((g.M + BM - 1) / BM), static_cast<unsigned>((g.N + BN - 1) / BN), &tm, &tn);
    const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
    const int rows_a = static_cast<int>(min(g.M - m0, int64_t(BM))), rows_b = static_cast<int>(min(g.N - n0, int64_t(BN)));
    const uint32_t lda = static_cast<uint32_t>(g.lda), ldw = static_cast<uint32_t>(g.ldw);
    const Stretch x = stretch_of<BYTES<DT>>(g);
    const uint32_t width = static_cast<uint32_t>(x.K * BYTES<DT>);
    const char *A = x.A + m0 * g.lda, *W = x.W + n0 * g.ldw;
    auto sa = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(A), 0, (rows_a - 1) * lda + width, 0x00027000);
    auto sb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(W), 0, (rows_b - 1) * ldw + width, 0x00027000);
    // A wave's load fills LDS in order (lane l has place l % 8 of row l / 8), and place p of a row holds unit p ^ (row / 2 % 8).
    // Rows behind the last one are the last one again: their results are not stored, and nothing depends on the buffer's bounds.
    const uint32_t row = threadIdx.x / UNITS, byte = threadIdx.x % UNITS * 16;
    uint32_t oa[PA], ob[PB];
#pragma unroll
    for (int p = 0; p < PA; ++p) oa[p] = min(row + p * ROWS, rows_a - 1u) * lda + (byte ^ (row + p * ROWS) / 2 % 8 * 16);
#pragma unroll
    for (int p = 0; p < PB; ++p) ob[p] = min(row + p * ROWS, rows_b - 1u) * ldw + (byte ^ (row + p * ROWS) / 2 % 8 * 16);
    const int steps = static_cast<int>(x.K / STEP), all = steps + (x.K % STEP ? 1 : 0);
    auto fill = [&](int t) __attribute__((always_inline)) {
        raw16 *As = lds + t % NB * TILE + wave * 64, *Bs = As + BM * UNITS;
#pragma unroll
        for (int p = 0; p < PA; ++p) __builtin_amdgcn_raw_ptr_buffer_load_lds(sa, As + p * T, 16, static_cast<int>(oa[p]), t * 128, 0, 0);
#pragma unroll
        for (int p = 0; p < PB; ++p) __builtin_amdgcn_raw_ptr_buffer_load_lds(sb, Bs + p * T, 16, static_cast<int>(ob[p]), t * 128, 0, 0);
    };
    auto fill_end = [&]() __attribute__((always_inline)) {              // what is left of the reduction, element by element at its end
        raw16 *As = lds + steps % NB * TILE;
        const int64_t k = int64_t(steps) * STEP + threadIdx.x % UNITS * (16 / BYTES<DT>);
#pragma unroll 1
        for (int r = threadIdx.x / UNITS; r < BM + BN; r += T / UNITS)
            As[unit_at(r, threadIdx.x % UNITS)] = r < BM ? load_unit<DT>(A + int64_t(min(r, rows_a - 1)) * g.lda, k, x.K)
                                                        : load_unit<DT>(W + int64_t(min(r - BM, rows_b - 1)) * g.ldw, k, x.K);
    };
    acc16 acc[TM][TN] = {};
    constexpr int MFMAS = TM * TN * (DT == CAPGNN_F32 ? 4 : DT == F32_CUT ? 6 : DT == E4M3_FINE ? 2 : 1), READS = (TM + TN) * Slice<DT, TM>::U;
    Slice<DT, TM> a[2];
    Slice<DT, TN> b[2];
    auto read = [&](int k, int t, int s) {
        const raw16 *As = lds + t % NB * TILE;
        a[k].read(As, wm + lane % 32, half, s);
        b[k].read(As + BM * UNITS, wn + lane % 32, half, s);
    };
    // everyone's loads to LDS but the last `later` are there, and everyone has read what he asked for
    auto arrived = [&](auto later) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(later.value) : "memory");
        __syncthreads();
    };
    using None = std::integral_constant<int, 0>;
    using Later = std::integral_constant<int, (NB - 2) * (PA + PB)>;
    auto most = [&](int t) __attribute__((always_inline)) {             // the slices of step t but the last
#pragma unroll
        for (int s = 0; s + 1 < S; ++s) {
            read((s + 1) & 1, t, s + 1);
            multiply_slice<DT, TM, TN>(a[s & 1], b[s & 1], acc);
            interleave<MFMAS, READS, 0>();
        }
    };
#pragma unroll 1
    for (int t = 0; t < min(steps, NB); ++t) fill(t);
    if (steps < NB && steps < all) fill_end();
    arrived(None());
    read(0, 0, 0);
    int t = 0;
    for (; t + NB < steps; ++t) {
        most(t);
        arrived(Later());               // step t + 1 is; t + 2 .. t + NB - 1 may be on their way
        read(0, t + 1, 0);
        fill(t + NB);
        multiply_slice<DT, TM, TN>(a[1], b[1], acc);
        interleave<MFMAS, READS, PA + PB>();
    }
    for (; t < all; ++t) {
        most(t);
        if (t + 1 < all) {
            arrived(None());
            if (t + NB == steps && steps < all) fill_end();
            read(0, t + 1, 0);
        }
        multiply_slice<DT, TM, TN>(a[1], b[1], acc);
    }
    __syncthreads();
    store_tile<OB, WR, WC, TM, TN>(g, lds, m0 + wm, n0 + wn, acc);
}

// The parts' sums, in order, and the epilogue: a thread 8 columns of a row
__global__ __launch_bounds__(256) void linear_join_kernel(LinearArgs g, int parts) {
    const int64_t across = g.part_ld / 8, at = int64_t(blockIdx.x) * 256 + threadIdx.x, row = at / across, col = at % across * 8;
    if (row >= g.M) return;
    float sum[8];
    ld_row<false, 8>(reinterpret_cast<const char *>(g.part + row * g.part_ld + col), 0, sum);
#pragma unroll 4
    for (int p = 1; p < parts; ++p) {
        float v[8];
        ld_row<false, 8>(reinterpret_cast<const char *>(g.part + (p * g.M + row) * g.part_ld + col), 0, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[e];
    }
    const int count = static_cast<int>(min(g.N - col, int64_t(8)));
    if (count > 0) finish<8>(g, row, col, count, sum);
}

// ------------------------------------------------------------------ a few rows of A
// The weights' bytes bound these: every row of W is read once, straight into the registers of the matrix instruction (16 x 16 results: lane l has
// row l % 16 of W, and of A, and every fourth 16-byte unit of it, from l / 16 on), by a workgroup per 16 rows, whose waves take lines of
// 128 bytes in turn.  Their sums meet in LDS, in wave order.  A stays in the caches.  8-bit operands are widened to bf16 whatever the result.
// 1 x 4096 x 4096 bf16 9.5 us (3.5 TB/s), e4m3 8, fp32 18.
// D layout of the 16 x 16 instructions: register r of lane l holds row 4 (l / 16) + r, column l % 16: 4 neighbouring columns of a row of Y, with W
// as the first operand.
typedef float acc4 __attribute__((ext_vector_type(4)));
template <int DT> __device__ __forceinline__ acc4 multiply16(raw16 w, raw16 a, acc4 acc) {
    if constexpr (DT == CAPGNN_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[e]), __uint_as_float(a[e]), acc, 0, 0, 0);
        return acc;
    } else if constexpr (DT == CAPGNN_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(half8, w), __builtin_bit_cast(half8, a), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w, 0), widen8(a, 0), acc, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w, 1), widen8(a, 1), acc, 0, 0, 0);
    }
}

constexpr int FEW_AHEAD = 8;            // units of a row on their way at a time, per lane

template <int DT> __global__ __launch_bounds__(FEW_WAVES * 64) void linear_few_kernel(LinearArgs g) {
    constexpr int E = 16 / BYTES<DT>;
    __shared__ acc4 sums[FEW_WAVES][64];
    const int wave = threadIdx.x / 64, waves = blockDim.x / 64, lane = threadIdx.x & 63;
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    const Stretch x = stretch_of<BYTES<DT>>(g);
    const char *w = x.W + min(n0 + lane % 16, g.N - 1) * g.ldw, *a = x.A + min(int64_t(lane % 16), g.M - 1) * g.lda;
    acc4 acc = {};
    // a wave's unit q: 16 bytes at k, of line q / 2 of its own
    auto at = [&](int64_t q) { return ((q / 2 * waves + wave) * 8 + q % 2 * 4 + lane / 16) * E; };
    const int64_t lines = (x.K + 8 * E - 1) / (8 * E), mine = lines > wave ? ((lines - wave - 1) / waves + 1) * 2 : 0;
    const int64_t sure = x.K / (8 * E), whole = sure > wave ? ((sure - wave - 1) / waves + 1) * 2 : 0;      // of lines that end inside the row
    int64_t q = 0;
    for (; q + FEW_AHEAD <= whole; q += FEW_AHEAD) {
        raw16 rw[FEW_AHEAD], ra[FEW_AHEAD];
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u) {
            typedef raw16 raw16_by1 __attribute__((aligned(1)));
            const int64_t k = at(q + u) * BYTES<DT>;
            rw[u] = *reinterpret_cast<const raw16_by1 *>(w + k);
            ra[u] = *reinterpret_cast<const raw16_by1 *>(a + k);
        }
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u) acc = multiply16<DT>(rw[u], ra[u], acc);
    }
    for (; q < mine; q += 2) {              // a line at a time, its end checked
        raw16 rw[2], ra[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            rw[u] = load_unit<DT>(w, at(q + u), x.K);
            ra[u] = load_unit<DT>(a, at(q + u), x.K);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) acc = multiply16<DT>(rw[u], ra[u], acc);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    acc4 s = sums[0][lane];
    for (int v = 1; v < waves; ++v) s += sums[v][lane];
    const int64_t row = lane % 16, col = n0 + lane / 16 * 4;
    const int count = static_cast<int>(min(g.N - col, int64_t(4)));
    if (row < g.M && count > 0) {
        float v[4] = {s[0], s[1], s[2], s[3]};
        if (g.part) st_row<false, 4>(reinterpret_cast<char *>(g.part + (blockIdx.y * g.M + row) * g.part_ld + col), 0, v);
        else finish<4>(g, row, col, count, v);
    }
}

// ------------------------------------------------------------------ the epilogue's gradient
struct ActGradArgs {
    int64_t M, N;
    const char *dY, *U;
    char *dU;
    int64_t lddy, ldu, lddu;    // in bytes
    float *part;                // [parts][N], or null
    int64_t rows;               // of a part
};

// Memory bounds it: 3001 x 1009 fp32 9.5 us (3.8 TB/s), and 4.6 for the join of the column sums.
// A workgroup: 64 columns' vectors by 4 rows at a time, `rows` rows in all.  What is left at a row's end is taken element by element: dU may be
// dY or U, and nothing else may be read where it is written.
template <bool BF16, int ACT> __global__ __launch_bounds__(256) void act_grad_kernel(ActGradArgs a) {
    constexpr int V = ROW_V<BF16>, ES = BF16 ? 2 : 4;
    __shared__ float s[4][64 * V];
    const int lane = threadIdx.x & 63, q = threadIdx.x / 64;
    const int64_t j = (int64_t(blockIdx.x) * 64 + lane) * V, end = min(a.M, (blockIdx.y + 1) * a.rows);
    const int count = static_cast<int>(max(min(a.N - j, int64_t(V)), int64_t(0)));
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    if (count == V) {
#pragma unroll 2
        for (int64_t i = blockIdx.y * a.rows + q; i < end; i += 4) {
            float d[V], u[V];
            ld_row<BF16, V>(a.dY + i * a.lddy + j * ES, 0, d);
            if constexpr (ACT != CAPGNN_ACT_NONE) {
                ld_row<BF16, V>(a.U + i * a.ldu + j * ES, 0, u);
#pragma unroll
                for (int e = 0; e < V; ++e) d[e] *= act_slope<ACT>(u[e]);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += d[e];
            if (a.dU) st_row<BF16, V>(a.dU + i * a.lddu + j * ES, 0, d);
        }
    } else if (count) {
        for (int64_t i = blockIdx.y * a.rows + q; i < end; i += 4) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < count) {
                    float d = ld_logit<BF16>(a.dY + i * a.lddy + j * ES, e);
                    if constexpr (ACT != CAPGNN_ACT_NONE) d *= act_slope<ACT>(ld_logit<BF16>(a.U + i * a.ldu + j * ES, e));
                    sum[e] += d;
                    if (a.dU) st_grad<BF16>(a.dU + i * a.lddu + j * ES, e, d);
                }
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int e = 0; e < V; ++e) s[q][e * 64 + lane] = sum[e];
    __syncthreads();
    if (q == 0) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < count) a.part[int64_t(blockIdx.y) * a.N + j + e] = (s[0][e * 64 + lane] + s[1][e * 64 + lane]) + (s[2][e * 64 + lane] + s[3][e * 64 + lane]);
    }
}

int launch_column_join(const float *part, int parts, int64_t F, float *sums, hipStream_t st);     // norm.hip

static int act_parts(int64_t M, int64_t N, int64_t *rows) {
    const int64_t across = (N + 255) / 256;         // workgroups side by side, at least
    const int64_t parts = M <= 32 ? 1 : std::max<int64_t>(1, std::min<int64_t>((M + 15) / 16, 2048 / std::min<int64_t>(across, 2048)));
    *rows = (M + parts - 1) / parts;
    return static_cast<int>((M + *rows - 1) / *rows);
}

}  // namespace capgnn

using namespace capgnn;

static bool bad_act(int act) { return act < CAPGNN_ACT_NONE || act > CAPGNN_ACT_SILU; }

// f(operands, results in bf16) as compile-time numbers
template <class F> static void with_types(int dtype, int out_dtype, bool cut, F f) {
    using Y = std::true_type;
    using N = std::false_type;
    const bool o = out_dtype == CAPGNN_BF16;
    if (cut) o ? f(std::integral_constant<int, F32_CUT>(), Y()) : f(std::integral_constant<int, F32_CUT>(), N());
    else if (dtype == CAPGNN_F32) o ? f(std::integral_constant<int, CAPGNN_F32>(), Y()) : f(std::integral_constant<int, CAPGNN_F32>(), N());
    else if (dtype == CAPGNN_BF16) o ? f(std::integral_constant<int, CAPGNN_BF16>(), Y()) : f(std::integral_constant<int, CAPGNN_BF16>(), N());
    else o ? f(std::integral_constant<int, CAPGNN_E4M3>(), Y()) : f(std::integral_constant<int, E4M3_FINE>(), N());
}

static int operand_bytes(int dtype) { return dtype == CAPGNN_E4M3 ? 1 : elem_bytes(dtype); }
static int64_t part_pitch(int64_t N) { return (N + 7) / 8 * 8; }

extern "C" size_t capgnn_linear_workspace_bytes(int64_t M, int64_t N, int64_t K, int dtype) {
    const int64_t most = int64_t(1) << 31;
    if (M <= 0 || N <= 0 || K <= 0 || M >= most || N >= most || K >= most || (!is_float_type(dtype) && dtype != CAPGNN_E4M3)) return 0;
    const LinearPlan p = linear_plan(M, N, K, operand_bytes(dtype));
    return p.parts > 1 ? align_up(sizeof(float) * p.parts * M * part_pitch(N), 256) : 0;
}

extern "C" int capgnn_linear(int64_t M, int64_t N, int64_t K, const void *A, int64_t lda, const float *a_scale, const void *W, int64_t ldw,
                             const float *w_scale, int dtype, const float *bias, int act, const void *R, int64_t ldr, void *U, int64_t ldu,
                             void *Y, int64_t ldy, int out_dtype, void *ws, size_t ws_bytes, void *stream) {
    if (!is_float_type(dtype) && dtype != CAPGNN_E4M3) CG_FAIL(CAPGNN_EINVAL, "linear: unknown dtype");
    if (!is_float_type(out_dtype)) CG_FAIL(CAPGNN_EINVAL, "linear: unknown out_dtype");
    if (bad_act(act)) CG_FAIL(CAPGNN_EINVAL, "linear: unknown activation");
    const int64_t most = int64_t(1) << 31;
    if (M < 0 || N < 0 || K < 0 || M >= most || N >= most || K >= most) CG_FAIL(CAPGNN_EINVAL, "linear: bad sizes");
    if (dtype != CAPGNN_E4M3 && (a_scale || w_scale)) CG_FAIL(CAPGNN_EINVAL, "linear: scales belong to 8-bit operands");
    if (M == 0 || N == 0) return CAPGNN_OK;
    if ((K > 0 && (!A || !W)) || !Y) CG_FAIL(CAPGNN_EINVAL, "linear: NULL operand");
    if ((K > 0 && (lda < K || ldw < K)) || ldy < N || (R && ldr < N) || (U && ldu < N)) CG_FAIL(CAPGNN_EINVAL, "linear: leading dimension smaller than the row");
    if ((K > 0 && (!row_aligned(A, dtype) || !row_aligned(W, dtype))) || !row_aligned(R, out_dtype) || !row_aligned(U, out_dtype) ||
        !row_aligned(Y, out_dtype) || !row_aligned(bias, CAPGNN_F32) || !row_aligned(a_scale, CAPGNN_F32) || !row_aligned(w_scale, CAPGNN_F32))
        CG_FAIL(CAPGNN_EINVAL, "linear: an operand is not aligned to its elements");
    if (Y == U || (R && U == R) || (Y == R && ldy != ldr)) CG_FAIL(CAPGNN_EINVAL, "linear: Y may be R with the same pitch; U is neither");
    if (K > 0 && (Y == A || Y == W || (U && (U == A || U == W)))) CG_FAIL(CAPGNN_EINVAL, "linear: Y and U must not be A or W");
    const int es = operand_bytes(dtype), os = elem_bytes(out_dtype);
    if (K * es >= most) CG_FAIL(CAPGNN_EINVAL, "linear: rows of 2^31 bytes and more");
    const size_t need = capgnn_linear_workspace_bytes(M, N, K, dtype);
    if (need && (!ws || ws_bytes < need)) CG_FAIL(CAPGNN_ENOMEM, "linear: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : size_t(0));
    if (need && reinterpret_cast<uintptr_t>(ws) & 255u) CG_FAIL(CAPGNN_EINVAL, "linear: workspace must be 256-byte aligned");
    const LinearPlan p = linear_plan(M, N, K, es);
    const LinearArgs g{M, N, K, static_cast<const char *>(A), static_cast<const char *>(W), lda * es, ldw * es, a_scale, w_scale, bias, act,
                       static_cast<const char *>(R), static_cast<char *>(U), static_cast<char *>(Y), ldr * os, ldu * os, ldy * os,
                       out_dtype == CAPGNN_BF16, p.parts > 1 ? static_cast<float *>(ws) : nullptr, part_pitch(N), p.part_k};
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uintptr_t at = reinterpret_cast<uintptr_t>(A) | reinterpret_cast<uintptr_t>(W) | uintptr_t(g.lda) | uintptr_t(g.ldw);
    const LinearWay way = linear_way(p, M, N, K, es, K > 0 && at % 4 == 0 && g.lda < most / 256 && g.ldw < most / 256);
    if (way.tile == 0) {
        if (N > int64_t(1) << 26) CG_FAIL(CAPGNN_EUNSUPPORTED, "linear: more than 2^26 results of a few rows");
        const dim3 grid(static_cast<unsigned>((N + 15) / 16), p.parts);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(way.waves * 64), 0, st, g); };
        if (dtype == CAPGNN_F32) go(linear_few_kernel<CAPGNN_F32>);
        else if (dtype == CAPGNN_BF16) go(linear_few_kernel<CAPGNN_BF16>);
        else go(linear_few_kernel<E4M3_FINE>);
    } else {
        const int tile = way.tile;
        const int64_t tiles = (M + tile - 1) / tile * ((N + tile - 1) / tile);
        if (tiles > int64_t(1) << 22) CG_FAIL(CAPGNN_EUNSUPPORTED, "linear: more than 2^22 tiles of results");
        const dim3 grid(static_cast<unsigned>(tiles), p.parts);
        with_types(dtype, out_dtype, way.cut, [&](auto d, auto o) {
            auto direct = [&](auto wr, auto wc, auto tm, auto tn, auto nb) {
                hipLaunchKernelGGL((linear_direct_kernel<d.value, o.value, wr.value, wc.value, tm.value, tn.value, nb.value>), grid,
                                   dim3(wr.value * wc.value * 64), 0, st, g);
            };
            constexpr std::integral_constant<int, 1> I1;
            constexpr std::integral_constant<int, 2> I2;
            constexpr std::integral_constant<int, 3> I3;
            constexpr std::integral_constant<int, 4> I4;
            // Eight waves of 128 x 64 fill one another's gaps; 8-bit operands, whose matrix instructions run twice as long, and fp32 ones, which
            // are cut on their way, do with half the reads of four waves of 128 x 128 (us, four / eight: 8192^3 bf16 908 / 855,
            // 8192 x 8192 x 16384 e4m3 831 / 858).  Tiles of 128 leave room for two workgroups a compute unit, those of 64 for three.
            // A load to LDS takes rows that start on 4 bytes; others go through registers, one step in LDS, in tiles of 64 alone (the row's pitch one
            // element more: 8192^3 bf16 831 -> 2713, 4096^3 110 -> 327, 8192 x 8192 x 4096 e4m3 245 -> 740).
            if (tile == 256) {
                if constexpr (d.value == CAPGNN_E4M3 || d.value == F32_CUT) direct(I2, I2, I4, I4, I2);
                else if constexpr (d.value != CAPGNN_F32) direct(I2, I4, I4, I2, I2);
            } else if (tile == 128) {
                if constexpr (d.value != CAPGNN_F32) direct(I2, I2, I2, I2, I2);
            } else {
                if constexpr (d.value != F32_CUT) {
                    if (!way.direct) hipLaunchKernelGGL((linear_tile_kernel<d.value, o.value, 2, 2, 1, 1>), grid, dim3(256), 0, st, g);
                }
                if (way.direct) direct(I2, I2, I1, I1, I3);
            }
        });
    }
    CG_HIP(hipGetLastError());
    if (p.parts > 1) {
        const int64_t jobs = M * (g.part_ld / 8);
        hipLaunchKernelGGL(linear_join_kernel, dim3(static_cast<unsigned>((jobs + 255) / 256)), dim3(256), 0, st, g, p.parts);
        CG_HIP(hipGetLastError());
    }
    return CAPGNN_OK;
}

extern "C" size_t capgnn_linear_act_bwd_workspace_bytes(int64_t M, int64_t N) {
    if (M <= 0 || N <= 0) return 0;
    int64_t rows;
    const int parts = act_parts(M, N, &rows);
    return parts > 1 ? align_up(sizeof(float) * N * parts, 256) : 0;
}

extern "C" int capgnn_linear_act_bwd(int64_t M, int64_t N, const void *dY, int64_t lddy, const void *U, int64_t ldu, int dtype, int act, void *dU,
                                     int64_t lddu, float *dbias, void *ws, size_t ws_bytes, void *stream) {
    if (!is_float_type(dtype)) CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: unknown dtype");
    if (bad_act(act)) CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: unknown activation");
    if (M < 0 || N < 0 || M >= int64_t(1) << 31 || N >= int64_t(1) << 31) CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: bad sizes");
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (N == 0) return CAPGNN_OK;
    if (!row_aligned(dbias, CAPGNN_F32)) CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: an operand is not aligned to its elements");
    if (M == 0) return dbias ? launch_column_join(nullptr, 0, N, dbias, st) : CAPGNN_OK;
    if (!dY || (act != CAPGNN_ACT_NONE && !U)) CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: NULL operand");
    if (lddy < N || (act != CAPGNN_ACT_NONE && ldu < N) || (dU && lddu < N)) CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: leading dimension smaller than the row");
    if (!row_aligned(dY, dtype) || (act != CAPGNN_ACT_NONE && !row_aligned(U, dtype)) || !row_aligned(dU, dtype))
        CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: an operand is not aligned to its elements");
    if (dU && ((dU == dY && lddu != lddy) || (act != CAPGNN_ACT_NONE && dU == U && lddu != ldu)))
        CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: dU may be dY or U only with the same pitch");
    const size_t need = dbias ? capgnn_linear_act_bwd_workspace_bytes(M, N) : 0;
    if (need && (!ws || ws_bytes < need)) CG_FAIL(CAPGNN_ENOMEM, "linear_act_bwd: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : size_t(0));
    if (need && reinterpret_cast<uintptr_t>(ws) & 255u) CG_FAIL(CAPGNN_EINVAL, "linear_act_bwd: workspace must be 256-byte aligned");
    if (!dU && !dbias) return CAPGNN_OK;
    const bool bf16 = dtype == CAPGNN_BF16;
    const int es = elem_bytes(dtype), V = bf16 ? ROW_V<true> : ROW_V<false>;
    int64_t rows;
    const int parts = act_parts(M, N, &rows);
    const ActGradArgs a{M, N, static_cast<const char *>(dY), static_cast<const char *>(U), static_cast<char *>(dU), lddy * es, ldu * es,
                        lddu * es, dbias && parts > 1 ? static_cast<float *>(ws) : dbias, rows};
    const dim3 grid(static_cast<unsigned>((N + 64 * V - 1) / (64 * V)), parts);
    with_act(act, [&](auto k) {
        if (bf16) hipLaunchKernelGGL((act_grad_kernel<true, k.value>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((act_grad_kernel<false, k.value>), grid, dim3(256), 0, st, a);
    });
    CG_HIP(hipGetLastError());
    return dbias && parts > 1 ? launch_column_join(a.part, parts, N, dbias, st) : CAPGNN_OK;
}
