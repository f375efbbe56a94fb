// Products with an epilogue, Y = act(A W^T + bias) + R, and the epilogue's gradient.
//
// Both operands run along the reduction index, so a tile of either is the same thing whatever its type: rows of 128 bytes, 32 fp32,
// 64 bf16 or 128 e4m3 numbers of k.  LDS holds such tiles in units of 16 bytes, unit u of row r at place u ^ (r % 8): eight rows' units of
// the same k lie in different banks.  The matrix instructions take 32 x 32 results; which k a lane's bytes are does not matter as long as
// both operands agree, so a lane of the lower and one of the upper half take alternate units of their row.
//
// D layout of the 32 x 32 instructions: register r of lane l holds row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32.
#include "rows.h"
#include "grid.h"

#include <algorithm>

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
};

// ------------------------------------------------------------------ activations
__device__ __forceinline__ float act_of(int act, float u) {
    if (act == CAPGNN_ACT_RELU) return u > 0.f ? u : 0.f;
    if (act == CAPGNN_ACT_GELU) return 0.5f * u * (1.f + erff(u * 0.70710678118654752f));
    if (act == CAPGNN_ACT_SILU) return u / (1.f + expf(-u));
    return u;
}
__device__ __forceinline__ float act_slope(int act, float u) {
    if (act == CAPGNN_ACT_RELU) return u > 0.f ? 1.f : 0.f;
    if (act == CAPGNN_ACT_GELU) return 0.5f * (1.f + erff(u * 0.70710678118654752f)) + u * expf(-0.5f * u * u) * 0.39894228040143268f;
    if (act == CAPGNN_ACT_SILU) {
        const float s = 1.f / (1.f + expf(-u));
        return s * (1.f + u * (1.f - s));
    }
    return 1.f;
}

// V neighbouring sums of row i from column j on, the first `count` of them inside the matrix: the whole epilogue
template <int V> __device__ __forceinline__ void finish(const LinearArgs &g, int64_t i, int64_t j, int count, float (&v)[V]) {
    const int es = g.out_bf16 ? 2 : 4;
    const float sa = g.a_scale ? g.a_scale[i] : 1.f;
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < count) {
            if (g.a_scale || g.w_scale) v[e] *= g.w_scale ? sa * g.w_scale[j + e] : sa;
            if (g.bias) v[e] += g.bias[j + e];
        }
    char *y = g.Y + i * g.ldy + j * es, *u = g.U + i * g.ldu + j * es;
    const char *r = g.R + i * g.ldr + j * es;
    if (count == V) {
        if (g.U) st_row_of<V>(g.out_bf16, u, 0, v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = act_of(g.act, v[e]);
        if (g.R) {
            float x[V];
            ld_row_of<V>(g.out_bf16, r, 0, x);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] += x[e];
        }
        st_row_of<V>(g.out_bf16, y, 0, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < count) {
                if (g.U) g.out_bf16 ? st_grad<true>(u, e, v[e]) : st_grad<false>(u, e, v[e]);
                v[e] = act_of(g.act, v[e]);
                if (g.R) v[e] += g.out_bf16 ? ld_logit<true>(r, e) : ld_logit<false>(r, e);
                g.out_bf16 ? st_grad<true>(y, e, v[e]) : st_grad<false>(y, e, v[e]);
            }
    }
}

// ------------------------------------------------------------------ the matrix instructions, on 16-byte units
constexpr int UNITS = 8;                // units of a tile's row

// e4m3 operands of a float result.  The 8-bit matrix instructions add the products of eight neighbouring k at a time and drop, toward zero,
// what lies below 2^-13 of the largest one's power of two (groups of eight are then added in float): 1.3e-5 of a sum's size, nothing
// beside a bf16 result's rounding, but a hundred times a float's.  So for float results the operands are widened to bf16, exactly, and
// take the bf16 instruction, at half the rate.
constexpr int E4M3_FINE = 3;
template <int DT> constexpr int BYTES = DT == CAPGNN_F32 ? 4 : DT == CAPGNN_BF16 ? 2 : 1;

__device__ __forceinline__ int unit_at(int row, int unit) { return row * UNITS + (unit ^ (row & 7)); }

// half e (eight numbers) of a unit of e4m3, as bf16
__device__ __forceinline__ half8 widen8(raw16 u, int e) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * e], 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * e], 1.f, true);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * e + 1], 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[2 * e + 1], 1.f, true);
    return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// the products of a tile's 128 bytes of k; a and b: the lane's rows in LDS (row % 32 is the lane's)
template <int DT, int TM, int TN>
__device__ __forceinline__ void multiply(const raw16 *As, const raw16 *Bs, int row_a, int row_b, int half, acc16 (&acc)[TM][TN]) {
    if constexpr (DT == CAPGNN_E4M3) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            int8v a[TM], b[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const raw16 lo = As[unit_at(row_a + i * 32, 4 * s + 2 * half)], hi = As[unit_at(row_a + i * 32, 4 * s + 2 * half + 1)];
                a[i] = int8v{int(lo[0]), int(lo[1]), int(lo[2]), int(lo[3]), int(hi[0]), int(hi[1]), int(hi[2]), int(hi[3])};
            }
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                const raw16 lo = Bs[unit_at(row_b + i * 32, 4 * s + 2 * half)], hi = Bs[unit_at(row_b + i * 32, 4 * s + 2 * half + 1)];
                b[i] = int8v{int(lo[0]), int(lo[1]), int(lo[2]), int(lo[3]), int(hi[0]), int(hi[1]), int(hi[2]), int(hi[3])};
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[i], b[j], acc[i][j], 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
        }
    } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            raw16 a[TM], b[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) a[i] = As[unit_at(row_a + i * 32, 2 * s + half)];
#pragma unroll
            for (int i = 0; i < TN; ++i) b[i] = Bs[unit_at(row_b + i * 32, 2 * s + half)];
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    if constexpr (DT == CAPGNN_BF16) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(half8, a[i]), __builtin_bit_cast(half8, b[j]), acc[i][j], 0, 0, 0);
                    } else if constexpr (DT == E4M3_FINE) {
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(a[i], e), widen8(b[j], e), acc[i][j], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i][e]), __uint_as_float(b[j][e]), acc[i][j], 0, 0, 0);
                    }
                }
        }
    }
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
            if constexpr (DT == CAPGNN_F32) r[e] = reinterpret_cast<const uint32_t *>(row)[k + e];
            else if constexpr (DT == CAPGNN_BF16) r[e / 2] |= uint32_t(reinterpret_cast<const uint16_t *>(row)[k + e]) << (e % 2 * 16);
            else r[e / 4] |= uint32_t(reinterpret_cast<const uint8_t *>(row)[k + e]) << (e % 4 * 8);
        }
    return r;
}

// ------------------------------------------------------------------ tiles
// WR x WC waves with TM x TN accumulators of 32 x 32 each: a tile of WR TM 32 rows of A by WC TN 32 rows of W.
template <int DT, int WR, int WC, int TM, int TN> __global__ __launch_bounds__(WR *WC * 64) void linear_tile_kernel(LinearArgs g) {
    constexpr int T = WR * WC * 64, BM = WR * TM * 32, BN = WC * TN * 32, STEP = 128 / BYTES<DT>;
    constexpr int PA = BM * UNITS / T, PB = BN * UNITS / T;             // units that a thread loads
    constexpr int PITCH = TN * 32 + 8;                                  // floats: four rows further lie in the other half of the banks
    constexpr int STAGE = WR * WC * 32 * PITCH * 4, TILES = (BM + BN) * UNITS * 16;
    __shared__ raw16 lds[(STAGE > TILES ? STAGE : TILES) / 16];
    raw16 *As = lds, *Bs = lds + BM * UNITS;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, half = lane / 32;
    const int wm = wave / WC * TM * 32, wn = wave % WC * TN * 32;
    const int64_t m0 = int64_t(blockIdx.x) * BM, n0 = int64_t(blockIdx.y) * BN;
    acc16 acc[TM][TN] = {};
    raw16 ra[PA], rb[PB];
    auto fetch = [&](int64_t k) {
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const int u = p * T + threadIdx.x;
            ra[p] = load_unit<DT>(g.A + min(m0 + u / UNITS, g.M - 1) * g.lda, k + u % UNITS * (16 / BYTES<DT>), g.K);
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int u = p * T + threadIdx.x;
            rb[p] = load_unit<DT>(g.W + min(n0 + u / UNITS, g.N - 1) * g.ldw, k + u % UNITS * (16 / BYTES<DT>), g.K);
        }
    };
    if (g.K > 0) fetch(0);
    for (int64_t k = 0; k < g.K; k += STEP) {
        __syncthreads();
#pragma unroll
        for (int p = 0; p < PA; ++p) As[unit_at((p * T + threadIdx.x) / UNITS, threadIdx.x % UNITS)] = ra[p];
#pragma unroll
        for (int p = 0; p < PB; ++p) Bs[unit_at((p * T + threadIdx.x) / UNITS, threadIdx.x % UNITS)] = rb[p];
        __syncthreads();
        if (k + STEP < g.K) fetch(k + STEP);
        multiply<DT, TM, TN>(As, Bs, wm + lane % 32, wn + lane % 32, half, acc);
    }
    __syncthreads();
    // 32 rows of a wave's results at a time through LDS, so that memory is read and written along the rows
    float *stage = reinterpret_cast<float *>(lds) + wave * 32 * PITCH;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) stage[(8 * (r / 4) + 4 * half + r % 4) * PITCH + j * 32 + lane % 32] = acc[i][j][r];
        __builtin_amdgcn_wave_barrier();
        constexpr int LANES = TN * 4;                                   // of a row, 8 columns each
#pragma unroll
        for (int r = lane / LANES; r < 32; r += 64 / LANES) {
            const int64_t row = m0 + wm + i * 32 + r, col = n0 + wn + lane % LANES * 8;
            float v[8];
            ld_row<false, 8>(reinterpret_cast<const char *>(stage + r * PITCH + lane % LANES * 8), 0, v);
            const int count = static_cast<int>(min(g.N - col, int64_t(8)));
            if (row < g.M && count > 0) finish<8>(g, row, col, count, v);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ------------------------------------------------------------------ the epilogue's gradient
struct ActGradArgs {
    int64_t M, N;
    const char *dY, *U;
    char *dU;
    int64_t lddy, ldu, lddu;    // in bytes
    int act, bf16;
    float *part;                // [parts][N], or null
    int64_t rows;               // of a part
};

// A workgroup: 64 columns' vectors by 4 rows at a time, `rows` rows in all.  What is left at a row's end is taken element by element: dU may be
// dY or U, and nothing else may be read where it is written.
template <bool BF16> __global__ __launch_bounds__(256) void act_grad_kernel(ActGradArgs a) {
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
            if (a.act != CAPGNN_ACT_NONE) {
                ld_row<BF16, V>(a.U + i * a.ldu + j * ES, 0, u);
#pragma unroll
                for (int e = 0; e < V; ++e) d[e] *= act_slope(a.act, u[e]);
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
                    if (a.act != CAPGNN_ACT_NONE) d *= act_slope(a.act, ld_logit<BF16>(a.U + i * a.ldu + j * ES, e));
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
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((M + 15) / 16, 2048 / std::min<int64_t>(across, 2048)));
    *rows = (M + parts - 1) / parts;
    return static_cast<int>((M + *rows - 1) / *rows);
}

}  // namespace capgnn

using namespace capgnn;

static bool bad_act(int act) { return act < CAPGNN_ACT_NONE || act > CAPGNN_ACT_SILU; }

extern "C" size_t capgnn_linear_workspace_bytes(int64_t, int64_t, int64_t, int) { return 0; }

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
    const int es = dtype == CAPGNN_E4M3 ? 1 : elem_bytes(dtype), os = elem_bytes(out_dtype);
    if (K * es >= most) CG_FAIL(CAPGNN_EINVAL, "linear: rows of 2^31 bytes and more");
    const LinearArgs g{M, N, K, static_cast<const char *>(A), static_cast<const char *>(W), lda * es, ldw * es, a_scale, w_scale, bias, act,
                       static_cast<const char *>(R), static_cast<char *>(U), static_cast<char *>(Y), ldr * os, ldu * os, ldy * os,
                       out_dtype == CAPGNN_BF16};
    hipStream_t st = static_cast<hipStream_t>(stream);
    (void)ws;
    (void)ws_bytes;
    const dim3 grid(static_cast<unsigned>((M + 63) / 64), static_cast<unsigned>((N + 63) / 64));
    if (dtype == CAPGNN_F32) hipLaunchKernelGGL((linear_tile_kernel<CAPGNN_F32, 2, 2, 1, 1>), grid, dim3(256), 0, st, g);
    else if (dtype == CAPGNN_BF16) hipLaunchKernelGGL((linear_tile_kernel<CAPGNN_BF16, 2, 2, 1, 1>), grid, dim3(256), 0, st, g);
    else if (out_dtype == CAPGNN_F32) hipLaunchKernelGGL((linear_tile_kernel<E4M3_FINE, 2, 2, 1, 1>), grid, dim3(256), 0, st, g);
    else hipLaunchKernelGGL((linear_tile_kernel<CAPGNN_E4M3, 2, 2, 1, 1>), grid, dim3(256), 0, st, g);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}

extern "C" size_t capgnn_linear_act_bwd_workspace_bytes(int64_t M, int64_t N) {
    if (M <= 0 || N <= 0) return 0;
    int64_t rows;
    return align_up(sizeof(float) * N * act_parts(M, N, &rows), 256);
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
                        lddu * es, act, bf16, dbias ? static_cast<float *>(ws) : nullptr, rows};
    const dim3 grid(static_cast<unsigned>((N + 64 * V - 1) / (64 * V)), parts);
    if (bf16) hipLaunchKernelGGL(act_grad_kernel<true>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(act_grad_kernel<false>, grid, dim3(256), 0, st, a);
    CG_HIP(hipGetLastError());
    return dbias ? launch_column_join(a.part, parts, N, dbias, st) : CAPGNN_OK;
}
