// Root-mean-square norm with the residual's addition, rows in 8 bits, and the norm's gradient.
//
//   h = x + r, s = (mean h^2 + eps)^-1/2, y = h s w;   dx = s g - h s^3 mean(g h) + dh with g = dy w;   dw = sum over rows of dy h s
//
// Memory bounds them: a row is read once, held in registers through its sums and written once.  A row belongs to a team: as many
// lanes of a wave as it has vectors of 16 bytes (a power of two), up to 64, or a workgroup for wide rows.  Where a row is no whole number
// of vectors its last lane takes the row's last V elements: those that the lane before it has, too, are left out of the sums (passed over, not
// multiplied by 0: one may be an infinity) and stored twice with the same value.  Every sum has a fixed order.
// us (of the bytes a pass cannot do without): 180000 x 602 fp32 with the residual 331 (5.2 TB/s), 16384 x 4096 bf16 gradient with dH and dw
// 112, and 7 for the join of dw's parts (4.5 TB/s), one row of 4096 into 8 bits 3.4.  16 elements per lane of the gradient at 1024
// threads and more (fp32 rows above 8192, bf16 rows above 16384) do not fit the registers: 36 bytes of scratch memory a thread for fp32 rows up to
// 16384, above that 536 (bf16 368).
#include "rows.h"

#include <algorithm>
#include <type_traits>

namespace capgnn {

struct NormArgs {
    int64_t n;
    int F, lanes;               // lanes of a team (waves only)
    const char *X, *R;
    int64_t ldx, ldr;           // in bytes
    char *H, *Y;
    int64_t ldh, ldy;
    const float *w;
    float eps, inv_F;
    int y_type, norm;           // norm 0: rows in 8 bits alone
    float *y_scale, *rstd;
};

__device__ __forceinline__ float team_sum(float v, int lanes) {
    for (int o = lanes >> 1; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ uint32_t team_max(uint32_t v, int lanes) {
    for (int o = lanes >> 1; o; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o)));
    return v;
}

// the elements of a row that a lane has: its vector i starts at from[i], the first skip[i] of which are another lane's too (V: none is its own)
template <int V, int K> struct Share {
    int from[K], skip[K];
    __device__ __forceinline__ Share(int lane, int lanes, int F) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int j = (lane + i * lanes) * V;
            from[i] = min(j, F - V);
            skip[i] = min(j - from[i], V);
        }
    }
};

// T: threads of a row's team, or 64 for teams of a.lanes lanes of a wave
template <bool BF16, int V, int K, int T> __global__ __launch_bounds__(T == 64 ? 256 : T) void rmsnorm_kernel(NormArgs a) {
    constexpr bool WIDE = T > 64;
    __shared__ float part[WIDE ? 2 * (T / 64) : 1];
    const int wave = threadIdx.x / 64, lanes = WIDE ? T : a.lanes;
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (lanes - 1);
    const int64_t per_wave = WIDE ? 1 : 64 / lanes;
    const int64_t row = WIDE ? blockIdx.x : (int64_t(blockIdx.x) * 4 + wave) * per_wave + (threadIdx.x & 63) / lanes;
    const bool live = row < a.n;
    const Share<V, K> s(lane, lanes, a.F);
    float h[K][V], sum = 0.f;
#pragma unroll
    for (int i = 0; i < K; ++i) {
#pragma unroll
        for (int e = 0; e < V; ++e) h[i][e] = 0.f;
        if (live && s.skip[i] < V) ld_row<BF16, V>(a.X + row * a.ldx, s.from[i], h[i]);
    }
    if (a.R) {
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (live && s.skip[i] < V) {
                float r[V];
                ld_row<BF16, V>(a.R + row * a.ldr, s.from[i], r);
#pragma unroll
                for (int e = 0; e < V; ++e) h[i][e] += r[e];
            }
    }
    float rstd = 1.f;
    if (a.norm) {
#pragma unroll
        for (int i = 0; i < K; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) sum = e < s.skip[i] ? sum : fmaf(h[i][e], h[i][e], sum);
        sum = team_sum(sum, WIDE ? 64 : lanes);
        if constexpr (WIDE) {
            if ((threadIdx.x & 63) == 0) part[wave] = sum;
            __syncthreads();
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < T / 64; ++i) sum += part[i];
        }
        rstd = 1.f / sqrtf(sum * a.inv_F + a.eps);
        if (live && lane == 0 && a.rstd) a.rstd[row] = rstd;
    }
    if (a.H) {
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (live && s.skip[i] < V) st_row<BF16, V>(a.H + row * a.ldh, s.from[i], h[i]);
    }
    if (a.norm) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            float w[V];
#pragma unroll
            for (int e = 0; e < V; ++e) w[e] = 1.f;
            if (a.w && s.skip[i] < V) ld_row<false, V>(reinterpret_cast<const char *>(a.w), s.from[i], w);
#pragma unroll
            for (int e = 0; e < V; ++e) h[i][e] = h[i][e] * rstd * w[e];
        }
    }
    if (a.y_type == CAPGNN_E4M3) {
        // magnitudes compare as their bits do, a NaN above everything: it becomes the scale, and with it the whole row's
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (s.skip[i] < V) {
#pragma unroll
                for (int e = 0; e < V; ++e) most = max(most, __float_as_uint(h[i][e]) & 0x7fffffffu);
            }
        most = team_max(most, WIDE ? 64 : lanes);
        if constexpr (WIDE) {
            uint32_t *p = reinterpret_cast<uint32_t *>(part) + T / 64;
            if ((threadIdx.x & 63) == 0) p[wave] = most;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < T / 64; ++i) most = max(most, p[i]);
        }
        const float scale = __uint_as_float(max(most, 0x0d800000u)) / 448.f;      // (2^-100)
        const float inverse = 1.f / scale;
        if (live && lane == 0) a.y_scale[row] = scale;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (live && s.skip[i] < V) {
#pragma unroll
                for (int e = 0; e < V; ++e) h[i][e] *= inverse;
                st_e4m3<V>(a.Y + row * a.ldy, s.from[i], h[i]);
            }
    } else {
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (live && s.skip[i] < V) st_row_of<V>(a.y_type == CAPGNN_BF16, a.Y + row * a.ldy, s.from[i], h[i]);
    }
}

struct NormGradArgs {
    int64_t n;
    int F, lanes, dy_bf16;
    const char *dY, *H, *dH;
    int64_t lddy, ldh, lddh;    // in bytes
    const float *w, *rstd;
    char *dX;
    int64_t lddx;
    float inv_F;
    float *part;                // [workgroups][F] parts of dw, or null
};

// A workgroup strides over the rows and keeps its part of dw in registers.  All of a row is asked for before its sum, dH too, which is
// used behind it.
template <bool BF16, int V, int K, int T> __global__ __launch_bounds__(T == 64 ? 256 : T) void rmsnorm_grad_kernel(NormGradArgs a) {
    constexpr bool WIDE = T > 64;
    __shared__ float part[WIDE ? 2 * (T / 64) : 4 * 64 * V * K];
    const int wave = threadIdx.x / 64, lanes = WIDE ? T : a.lanes;
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (lanes - 1);
    const int64_t rows = WIDE ? 1 : 4 * (64 / lanes), mine = WIDE ? 0 : threadIdx.x / lanes;
    const Share<V, K> s(lane, lanes, a.F);
    float acc[K][V];
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[i][e] = 0.f;
    int turn = 0;
    for (int64_t row0 = blockIdx.x * rows; row0 < a.n; row0 += gridDim.x * rows) {
        const int64_t row = row0 + mine;
        const bool live = row < a.n;
        const float rstd = live ? a.rstd[row] : 0.f;
        float h[K][V], g[K][V], sum = 0.f;
        RawRow<BF16, V> d[K];
#pragma unroll
        for (int i = 0; i < K; ++i) {
#pragma unroll
            for (int e = 0; e < V; ++e) h[i][e] = g[i][e] = 0.f;
            d[i].clear();
            if (live && s.skip[i] < V) {
                ld_row<BF16, V>(a.H + row * a.ldh, s.from[i], h[i]);
                ld_row_of<V>(a.dy_bf16, a.dY + row * a.lddy, s.from[i], g[i]);
                if (a.dH) d[i].load(a.dH + row * a.lddh, s.from[i]);
            }
        }
        // (dX may be dH: all of a row is here before any of it is stored, also what two lanes share)
#pragma unroll
        for (int i = 0; i < K; ++i) d[i].arrive();
#pragma unroll
        for (int i = 0; i < K; ++i) {
            float w[V];
#pragma unroll
            for (int e = 0; e < V; ++e) w[e] = 1.f;
            if (a.w && s.skip[i] < V) ld_row<false, V>(reinterpret_cast<const char *>(a.w), s.from[i], w);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float hat = h[i][e] * rstd;
                acc[i][e] = fmaf(g[i][e], hat, acc[i][e]);
                g[i][e] *= w[e];
                h[i][e] = hat;
                sum = e < s.skip[i] ? sum : fmaf(g[i][e], hat, sum);
            }
        }
        sum = team_sum(sum, WIDE ? 64 : lanes);
        if constexpr (WIDE) {           // (two sets of parts in turn: a wave may be a row ahead of the others)
            float *p = part + (turn ^= 1) * (T / 64);
            if ((threadIdx.x & 63) == 0) p[wave] = sum;
            __syncthreads();
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < T / 64; ++i) sum += p[i];
        }
        const float mean = sum * a.inv_F;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (live && s.skip[i] < V) {
                float x[V];
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = fmaf(rstd, fmaf(-mean, h[i][e], g[i][e]), d[i].get(e));
                st_row<BF16, V>(a.dX + row * a.lddx, s.from[i], x);
            }
    }
    if (!a.part) return;
    float *out = a.part + int64_t(blockIdx.x) * a.F;
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < K; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e >= s.skip[i]) out[s.from[i] + e] = acc[i][e];
    } else {
        // teams of a wave, then the waves
#pragma unroll
        for (int i = 0; i < K; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                for (int o = lanes; o < 64; o *= 2) acc[i][e] += __shfl_xor(acc[i][e], o);
                part[((wave * K + i) * V + e) * 64 + lane] = acc[i][e];
            }
        __syncthreads();
        if (threadIdx.x < lanes) {
#pragma unroll
            for (int i = 0; i < K; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float v = 0.f;
#pragma unroll
                    for (int q = 0; q < 4; ++q) v += part[((q * K + i) * V + e) * 64 + lane];
                    if (e >= s.skip[i]) out[s.from[i] + e] = v;
                }
        }
    }
}

// sums[j] = sum over the parts of column j: 16 columns a workgroup, 16 threads each with every 16th part, then their sums in order.
// Of rows of F columns it takes `columns`.
__global__ __launch_bounds__(256) void column_join_kernel(const float *part, int parts, int64_t F, int64_t columns, float *sums) {
    __shared__ float s[16][17];
    const int c = threadIdx.x & 15, q = threadIdx.x / 16;
    const int64_t j = int64_t(blockIdx.x) * 16 + c;
    float v = 0.f;
    if (j < columns) {
#pragma unroll 8
        for (int p = q; p < parts; p += 16) v += part[p * F + j];
    }
    s[q][c] = v;
    __syncthreads();
    if (q == 0 && j < columns) {
        for (int i = 1; i < 16; ++i) v += s[i][c];
        sums[j] = v;
    }
}
int launch_column_join(const float *part, int parts, int64_t F, float *sums, hipStream_t st) {
    constexpr int64_t most = int64_t(1) << 27;      // columns of a launch (fewer than 2^32 threads)
    for (int64_t j = 0; j < F; j += most) {
        const int64_t columns = std::min(F - j, most);
        hipLaunchKernelGGL(column_join_kernel, dim3(static_cast<unsigned>((columns + 15) / 16)), dim3(256), 0, st, part ? part + j : nullptr, parts, F, columns,
                           sums + j);
        CG_HIP(hipGetLastError());
    }
    return CAPGNN_OK;
}

// Team of a row: threads (64: lanes of a wave) and vectors per lane.  `held`: elements per lane, at most; of the widest team's 32.
struct NormShape {
    int V, K, T, lanes;
};
constexpr int NORM_HELD = 32, GRAD_HELD = 16;   // (the gradient holds h, dY, dH and the sums of dw)
static NormShape norm_shape(int F, bool bf16, int held) {
    const int V = bf16 ? ROW_V<true> : ROW_V<false>;
    if (F < V) return {1, 1, 64, pow2_at_least(F)};
    const int vectors = (F + V - 1) / V, most = (vectors <= 1024 * (held / V) ? held : 32) / V;
    const int T = vectors <= 64 * (held / V) ? 64 : vectors <= 256 * (held / V) ? 256 : 1024;
    int K = 1;
    while (K < most && vectors > T * K) K *= 2;
    return {V, K, T, T == 64 ? std::min(64, pow2_at_least((vectors + K - 1) / K)) : T};
}
// whether norm_shape gives a row of vectors of V elements K of them per lane of T
template <int HELD> constexpr bool has_shape(int V, int K, int T) {
    if (V == 1) return K == 1 && T == 64;
    const int most = HELD / V, narrower = T == 64 ? 0 : T == 256 ? 64 * most : 256 * most;      // vectors of the next narrower team
    return T * K > narrower && (K <= most || (T == 1024 && K * V == 32));
}

// f(type, V, K, T) as compile-time numbers
template <int HELD, class G> static void with_shape(const NormShape &s, bool bf16, G f) {
    auto one = [&](auto b, auto v, auto k, auto t) {
        if constexpr (has_shape<HELD>(v.value, k.value, t.value)) f(b, v, k, t);
    };
    auto threads = [&](auto b, auto v, auto k) {
        if (s.T == 64) one(b, v, k, std::integral_constant<int, 64>());
        else if (s.T == 256) one(b, v, k, std::integral_constant<int, 256>());
        else one(b, v, k, std::integral_constant<int, 1024>());
    };
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I4 = std::integral_constant<int, 4>;
    using I8 = std::integral_constant<int, 8>;
    if (s.V == 1) bf16 ? threads(std::true_type(), I1(), I1()) : threads(std::false_type(), I1(), I1());
    else if (bf16) s.K == 1 ? threads(std::true_type(), I8(), I1()) : s.K == 2 ? threads(std::true_type(), I8(), I2()) : threads(std::true_type(), I8(), I4());
    else
        s.K == 1 ? threads(std::false_type(), I4(), I1()) : s.K == 2 ? threads(std::false_type(), I4(), I2())
        : s.K == 4 ? threads(std::false_type(), I4(), I4()) : threads(std::false_type(), I4(), I8());
}

static int launch_norm(NormArgs a, bool bf16, hipStream_t st) {
    const NormShape s = norm_shape(a.F, bf16, NORM_HELD);
    a.lanes = s.lanes;
    const int64_t rows = s.T == 64 ? 4 * (64 / s.lanes) : 1;
    const int64_t most = int64_t(1) << 20;      // workgroups of a launch (fewer than 2^32 threads)
    for (int64_t done = 0; done < a.n; done += most * rows) {
        NormArgs b = a;
        b.n = std::min(a.n - done, most * rows);
        b.X += done * a.ldx;
        b.Y += done * a.ldy;
        if (b.R) b.R += done * a.ldr;
        if (b.H) b.H += done * a.ldh;
        if (b.y_scale) b.y_scale += done;
        if (b.rstd) b.rstd += done;
        const unsigned grid = static_cast<unsigned>((b.n + rows - 1) / rows);
        with_shape<NORM_HELD>(s, bf16, [&](auto t, auto v, auto k, auto th) {
            hipLaunchKernelGGL((rmsnorm_kernel<t.value, v.value, k.value, th.value>), dim3(grid), dim3(th.value == 64 ? 256 : th.value), 0, st, b);
        });
        CG_HIP(hipGetLastError());
    }
    return CAPGNN_OK;
}

// workgroups of the gradient: each has a part of dw
static int grad_groups(int64_t n, int F, bool bf16) {
    const NormShape s = norm_shape(F, bf16, GRAD_HELD);
    const int64_t rows = s.T == 64 ? 4 * (64 / s.lanes) : 1;
    return static_cast<int>(std::min<int64_t>((n + rows - 1) / rows, 1024));
}

}  // namespace capgnn

using namespace capgnn;

static int norm_width(const char *who, int F) {
    if (F <= 0) CG_FAIL(CAPGNN_EINVAL, "%s: bad sizes", who);
    if (F > CAPGNN_NORM_MAX) CG_FAIL(CAPGNN_EUNSUPPORTED, "%s: rows of %d elements, at most %d are supported", who, F, CAPGNN_NORM_MAX);
    return CAPGNN_OK;
}

extern "C" int capgnn_rmsnorm(int64_t n, int F, const void *X, int64_t ldx, const void *R, int64_t ldr, void *H, int64_t ldh, int dtype,
                              const float *w, float eps, void *Y, int64_t ldy, int y_dtype, float *y_scale, float *rstd, void *stream) {
    if (!is_float_type(dtype)) CG_FAIL(CAPGNN_EINVAL, "rmsnorm: unknown dtype");
    if (!is_float_type(y_dtype) && y_dtype != CAPGNN_E4M3) CG_FAIL(CAPGNN_EINVAL, "rmsnorm: unknown y_dtype");
    if (n < 0) CG_FAIL(CAPGNN_EINVAL, "rmsnorm: bad sizes");
    CG_TRY(norm_width("rmsnorm", F));
    if (!(eps >= 0.f) || !std::isfinite(eps)) CG_FAIL(CAPGNN_EINVAL, "rmsnorm: eps must be finite and not negative");
    if (n == 0) return CAPGNN_OK;
    if (!X || !Y) CG_FAIL(CAPGNN_EINVAL, "rmsnorm: NULL operand");
    if ((y_dtype == CAPGNN_E4M3) != (y_scale != nullptr)) CG_FAIL(CAPGNN_EINVAL, "rmsnorm: y_scale belongs to an 8-bit Y, and it to y_scale");
    if (ldx < F || ldy < F || (R && ldr < F) || (H && ldh < F)) CG_FAIL(CAPGNN_EINVAL, "rmsnorm: leading dimension smaller than the row");
    if (!row_aligned(X, dtype) || !row_aligned(R, dtype) || !row_aligned(H, dtype) || !row_aligned(Y, y_dtype) || !row_aligned(w, CAPGNN_F32) ||
        !row_aligned(y_scale, CAPGNN_F32) || !row_aligned(rstd, CAPGNN_F32))
        CG_FAIL(CAPGNN_EINVAL, "rmsnorm: an operand is not aligned to its elements");
    if ((H == X && ldh != ldx) || (H && H == R && ldh != ldr)) CG_FAIL(CAPGNN_EINVAL, "rmsnorm: H may be X or R only with the same pitch");
    if (Y == H || (Y == X && (ldy != ldx || y_dtype != dtype)) || (Y == R && (ldy != ldr || y_dtype != dtype)))
        CG_FAIL(CAPGNN_EINVAL, "rmsnorm: Y may be X or R only with the same type and pitch, and never H");
    const int es = elem_bytes(dtype), ys = y_dtype == CAPGNN_E4M3 ? 1 : elem_bytes(y_dtype);
    const NormArgs a{n, F, 0, static_cast<const char *>(X), static_cast<const char *>(R), ldx * es, ldr * es, static_cast<char *>(H),
                     static_cast<char *>(Y), ldh * es, ldy * ys, w, eps, 1.f / static_cast<float>(F), y_dtype, 1, y_scale, rstd};
    return launch_norm(a, dtype == CAPGNN_BF16, static_cast<hipStream_t>(stream));
}

extern "C" int capgnn_quantize_rows(int64_t n, int F, const void *X, int64_t ldx, int dtype, void *Q, int64_t ldq, float *q_scale, void *stream) {
    if (!is_float_type(dtype)) CG_FAIL(CAPGNN_EINVAL, "quantize_rows: unknown dtype");
    if (n < 0) CG_FAIL(CAPGNN_EINVAL, "quantize_rows: bad sizes");
    CG_TRY(norm_width("quantize_rows", F));
    if (n == 0) return CAPGNN_OK;
    if (!X || !Q || !q_scale) CG_FAIL(CAPGNN_EINVAL, "quantize_rows: NULL operand");
    if (ldx < F || ldq < F) CG_FAIL(CAPGNN_EINVAL, "quantize_rows: leading dimension smaller than the row");
    if (!row_aligned(X, dtype) || !row_aligned(q_scale, CAPGNN_F32)) CG_FAIL(CAPGNN_EINVAL, "quantize_rows: an operand is not aligned to its elements");
    if (Q == X) CG_FAIL(CAPGNN_EINVAL, "quantize_rows: Q must not be X");
    NormArgs a{};
    a.n = n;
    a.F = F;
    a.X = static_cast<const char *>(X);
    a.ldx = ldx * elem_bytes(dtype);
    a.Y = static_cast<char *>(Q);
    a.ldy = ldq;
    a.y_type = CAPGNN_E4M3;
    a.y_scale = q_scale;
    return launch_norm(a, dtype == CAPGNN_BF16, static_cast<hipStream_t>(stream));
}

extern "C" size_t capgnn_rmsnorm_bwd_workspace_bytes(int64_t n, int F) {
    if (n <= 0 || F <= 0 || F > CAPGNN_NORM_MAX) return 0;
    const int groups = std::max(grad_groups(n, F, false), grad_groups(n, F, true));
    return groups > 1 ? align_up(sizeof(float) * F * groups, 256) : 0;
}

extern "C" int capgnn_rmsnorm_bwd(int64_t n, int F, const void *dY, int64_t lddy, int dy_dtype, const void *H, int64_t ldh, int dtype,
                                  const float *w, const float *rstd, const void *dH, int64_t lddh, void *dX, int64_t lddx, float *dw, void *ws,
                                  size_t ws_bytes, void *stream) {
    if (!is_float_type(dtype) || !is_float_type(dy_dtype)) CG_FAIL(CAPGNN_EINVAL, "rmsnorm_bwd: unknown dtype or dy_dtype");
    if (n < 0) CG_FAIL(CAPGNN_EINVAL, "rmsnorm_bwd: bad sizes");
    CG_TRY(norm_width("rmsnorm_bwd", F));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (n == 0) {
        if (dw) return launch_column_join(nullptr, 0, F, dw, st);
        return CAPGNN_OK;
    }
    if (!dY || !H || !rstd || !dX) CG_FAIL(CAPGNN_EINVAL, "rmsnorm_bwd: NULL operand");
    if (lddy < F || ldh < F || lddx < F || (dH && lddh < F)) CG_FAIL(CAPGNN_EINVAL, "rmsnorm_bwd: leading dimension smaller than the row");
    if (!row_aligned(dY, dy_dtype) || !row_aligned(H, dtype) || !row_aligned(dH, dtype) || !row_aligned(dX, dtype) || !row_aligned(w, CAPGNN_F32) ||
        !row_aligned(rstd, CAPGNN_F32) || !row_aligned(dw, CAPGNN_F32))
        CG_FAIL(CAPGNN_EINVAL, "rmsnorm_bwd: an operand is not aligned to its elements");
    if ((dX == dY && (lddx != lddy || dtype != dy_dtype)) || (dX == H && lddx != ldh) || (dX == dH && lddx != lddh))
        CG_FAIL(CAPGNN_EINVAL, "rmsnorm_bwd: dX may be dY, H or dH only with the same type and pitch");
    const size_t need = dw ? capgnn_rmsnorm_bwd_workspace_bytes(n, F) : 0;
    if (need && (!ws || ws_bytes < need)) CG_FAIL(CAPGNN_ENOMEM, "rmsnorm_bwd: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : size_t(0));
    if (need && reinterpret_cast<uintptr_t>(ws) & 255u) CG_FAIL(CAPGNN_EINVAL, "rmsnorm_bwd: workspace must be 256-byte aligned");
    const bool bf16 = dtype == CAPGNN_BF16;
    const NormShape s = norm_shape(F, bf16, GRAD_HELD);
    const int groups = grad_groups(n, F, bf16);
    const int es = elem_bytes(dtype);
    const NormGradArgs a{n, F, s.lanes, dy_dtype == CAPGNN_BF16, static_cast<const char *>(dY), static_cast<const char *>(H),
                         static_cast<const char *>(dH), lddy * elem_bytes(dy_dtype), ldh * es, lddh * es, w, rstd, static_cast<char *>(dX),
                         lddx * es, 1.f / static_cast<float>(F), dw && groups > 1 ? static_cast<float *>(ws) : dw};
    with_shape<GRAD_HELD>(s, bf16, [&](auto t, auto v, auto k, auto th) {
        hipLaunchKernelGGL((rmsnorm_grad_kernel<t.value, v.value, k.value, th.value>), dim3(groups), dim3(th.value == 64 ? 256 : th.value), 0, st, a);
    });
    CG_HIP(hipGetLastError());
    return dw && groups > 1 ? launch_column_join(a.part, groups, F, dw, st) : CAPGNN_OK;
}
