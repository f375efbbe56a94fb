// The norm of many tensors' gradients together, their clipping, and the clipped update.
//
//   norm = (sum g^2)^1/2, c = min(1, max_norm / norm), g <- c g  or  W <- W - lr c g
//
// Memory bounds them: every gradient is read once for the norm, which all of them wait for, and once more when it is used.  The list of
// tensors is cut once, when it is made, into pieces of about equal size, so that a launch covers any number of tensors.  Squares are
// added in double: a float's square does not overflow there, and the sum's rounding is far below the result's; at one fused operation per
// 4 bytes that is a twentieth of the card's rate.  Every workgroup adds the first launch's sums itself, in one order: two launches in all.
// The second one takes the pieces from the last to the first: what the first has read last is what the caches still hold.
// us: 120 million fp32 gradients of bf16 weights in 300 tensors 273 (1.44 GB, 5.3 TB/s), 111 of them the norm; pieces of 32768
// elements 299, of 8192 272; 165 thousand in four tensors 3 and 4.4.
#include "rows.h"

#include <algorithm>
#include <exception>
#include <vector>

namespace capgnn {

struct alignas(16) ClipPiece {
    char *g, *p;
    uint32_t count, g_bf16, p_bf16, unused;
};
static_assert(sizeof(ClipPiece) == 32, "two 16-byte loads a piece");

constexpr unsigned CLIP_GROUPS = 4096;      // workgroups of a launch, and sums that the first one leaves
constexpr int CLIP_PIECE = 4096;            // elements of a piece (more where a list would have more than 2^22 of them)

// sum over a workgroup of 256, in every thread
__device__ __forceinline__ double group_sum(double v) {
    __shared__ double s[4];
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x / 64] = v;
    __syncthreads();
    return (s[0] + s[1]) + (s[2] + s[3]);
}

template <bool BF16> __device__ __forceinline__ double piece_squares(const char *g, int count) {
    constexpr int V = ROW_V<BF16>;
    double sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.0;
    int j = threadIdx.x * V;
    auto add = [&](const RawRow<BF16, V> &r) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = fma(static_cast<double>(r.get(e)), static_cast<double>(r.get(e)), sum[e]);
    };
    constexpr int U = 4;                // vectors on their way at a time
    for (; j + (U - 1) * 256 * V + V <= count; j += U * 256 * V) {
        RawRow<BF16, V> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u].load(g, j + u * 256 * V);
#pragma unroll
        for (int u = 0; u < U; ++u) add(r[u]);
    }
    for (; j + V <= count; j += 256 * V) {
        RawRow<BF16, V> r;
        r.load(g, j);
        add(r);
    }
    for (; j < count; ++j) {            // (one thread's: the others' j is behind the end by now)
        const double x = ld_logit<BF16>(g, j);
        sum[0] = fma(x, x, sum[0]);
    }
    double all = 0.0;
#pragma unroll
    for (int e = 0; e < V; ++e) all += sum[e];
    return all;
}

__global__ __launch_bounds__(256) void clip_squares_kernel(const ClipPiece *pieces, unsigned n, double *sums) {
    double sum = 0.0;
    ClipPiece ahead = pieces[blockIdx.x];
    for (unsigned k = blockIdx.x; k < n; k += gridDim.x) {
        const ClipPiece q = ahead;
        ahead = pieces[min(k + gridDim.x, n - 1)];
        sum += q.g_bf16 ? piece_squares<true>(q.g, q.count) : piece_squares<false>(q.g, q.count);
    }
    sum = group_sum(sum);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double whole_norm(const double *sums, unsigned groups) {
    double v = 0.0;
#pragma unroll
    for (unsigned i = 0; i < CLIP_GROUPS / 256; ++i) {
        const unsigned k = i * 256 + threadIdx.x;
        v += k < groups ? sums[k] : 0.0;
    }
    return sqrt(group_sum(v));
}

__global__ __launch_bounds__(256) void clip_norm_kernel(const double *sums, unsigned groups, float *norm_dev) {
    const double norm = whole_norm(sums, groups);
    if (threadIdx.x == 0) *norm_dev = static_cast<float>(norm);
}

// out = g * factor (STEP false), or out - factor * g
template <bool STEP, bool GB, bool PB> __device__ __forceinline__ void piece_apply(const ClipPiece &q, float factor) {
    constexpr int V = GB || PB ? 8 : 4;
    const int count = static_cast<int>(q.count);
    char *out = STEP ? q.p : q.g;
    int j = threadIdx.x * V;
#pragma unroll 2
    for (; j + V <= count; j += 256 * V) {
        float g[V], p[V];
        ld_row<GB, V>(q.g, j, g);
        if constexpr (STEP) ld_row<PB, V>(q.p, j, p);
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = STEP ? fmaf(-factor, g[e], p[e]) : factor * g[e];
        st_row<PB, V>(out, j, g);
    }
    for (; j < count; ++j) {
        const float g = ld_logit<GB>(q.g, j);
        st_grad<PB>(out, j, STEP ? fmaf(-factor, g, ld_logit<PB>(q.p, j)) : factor * g);
    }
}

// The same where a float has fewer bits of the factor, or none (a norm of 1e37 and a small limit): its product with a gradient of that size is
// an ordinary number.  Formed in double, rounded to float, then to the tensor's type.
template <bool STEP> __device__ __forceinline__ void piece_apply_small(const ClipPiece &q, double factor) {
    const int count = static_cast<int>(q.count);
    for (int j = threadIdx.x; j < count; j += 256) {
        const double g = q.g_bf16 ? ld_logit<true>(q.g, j) : ld_logit<false>(q.g, j);
        if constexpr (STEP) {
            const double p = q.p_bf16 ? ld_logit<true>(q.p, j) : ld_logit<false>(q.p, j);
            const float v = static_cast<float>(fma(-factor, g, p));
            q.p_bf16 ? st_grad<true>(q.p, j, v) : st_grad<false>(q.p, j, v);
        } else {
            const float v = static_cast<float>(factor * g);
            q.g_bf16 ? st_grad<true>(q.g, j, v) : st_grad<false>(q.g, j, v);
        }
    }
}

template <bool STEP> __global__ __launch_bounds__(256) void clip_apply_kernel(const ClipPiece *pieces, unsigned n, const double *sums,
                                                                              unsigned groups, float lr, float max_norm, float *norm_dev) {
    const double norm = whole_norm(sums, groups);
    const float shown = static_cast<float>(norm);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_dev = shown;
    if (!(shown <= 3.402823466e38f)) return;                 // infinity or NaN: nothing changes
    const bool clip = norm > static_cast<double>(max_norm);
    if (!STEP && !clip) return;
    const double c = clip ? static_cast<double>(max_norm) / norm : 1.0;
    const double whole = STEP ? static_cast<double>(lr) * c : c;
    const float factor = static_cast<float>(whole);
    const bool small = whole != 0.0 && fabs(whole) < 0x1p-126;
    if (blockIdx.x >= n) return;
    ClipPiece ahead = pieces[n - 1 - blockIdx.x];
    for (unsigned k = blockIdx.x; k < n; k += gridDim.x) {
        const ClipPiece q = ahead;
        ahead = pieces[n - 1 - min(k + gridDim.x, n - 1)];
        if (small) piece_apply_small<STEP>(q, whole);
        else if constexpr (STEP) {
            if (q.g_bf16) q.p_bf16 ? piece_apply<true, true, true>(q, factor) : piece_apply<true, true, false>(q, factor);
            else q.p_bf16 ? piece_apply<true, false, true>(q, factor) : piece_apply<true, false, false>(q, factor);
        } else {
            if (q.g_bf16) piece_apply<false, true, true>(q, factor);
            else piece_apply<false, false, false>(q, factor);
        }
    }
}

}  // namespace capgnn

using namespace capgnn;

struct capgnn_tensors {
    ClipPiece *pieces = nullptr;        // device
    unsigned n = 0;
    bool params = false;
};

extern "C" int capgnn_tensors_create(capgnn_tensors **t, int count, void *const *grads, const int32_t *grad_dtype, void *const *params,
                                     const int32_t *param_dtype, const int64_t *counts, void *stream) {
    if (!t) CG_FAIL(CAPGNN_EINVAL, "tensors_create: NULL handle");
    *t = nullptr;
    if (count < 0) CG_FAIL(CAPGNN_EINVAL, "tensors_create: bad sizes");
    if (count > 0 && (!grads || !grad_dtype || !counts || (params && !param_dtype))) CG_FAIL(CAPGNN_EINVAL, "tensors_create: NULL array");
    struct Span {
        uintptr_t from, to;
    };
    try {
        std::vector<Span> spans;
        std::vector<ClipPiece> pieces;
        int64_t total = 0;
        for (int i = 0; i < count; ++i) {
            if (counts[i] < 0 || counts[i] > int64_t(1) << 45) CG_FAIL(CAPGNN_EINVAL, "tensors_create: tensor %d has a bad size", i);
            if (!is_float_type(grad_dtype[i]) || (params && !is_float_type(param_dtype[i]))) CG_FAIL(CAPGNN_EINVAL, "tensors_create: tensor %d has an unknown type", i);
            if (counts[i] == 0) continue;
            if (!grads[i] || (params && !params[i])) CG_FAIL(CAPGNN_EINVAL, "tensors_create: tensor %d is NULL", i);
            if (!row_aligned(grads[i], grad_dtype[i]) || (params && !row_aligned(params[i], param_dtype[i])))
                CG_FAIL(CAPGNN_EINVAL, "tensors_create: tensor %d is not aligned to its elements", i);
            total += counts[i];
            if (total > int64_t(1) << 45) CG_FAIL(CAPGNN_EINVAL, "tensors_create: more than 2^45 elements");
            const uintptr_t g = reinterpret_cast<uintptr_t>(grads[i]);
            spans.push_back({g, g + static_cast<uintptr_t>(counts[i]) * elem_bytes(grad_dtype[i])});
            if (params) {
                const uintptr_t p = reinterpret_cast<uintptr_t>(params[i]);
                spans.push_back({p, p + static_cast<uintptr_t>(counts[i]) * elem_bytes(param_dtype[i])});
            }
        }
        std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.from < b.from; });
        for (size_t i = 1; i < spans.size(); ++i)
            if (spans[i].from < spans[i - 1].to) CG_FAIL(CAPGNN_EINVAL, "tensors_create: two tensors share memory");
        // pieces small enough that the workgroups of a launch work on one stretch of memory at a time, and few enough for the list
        int64_t size = CLIP_PIECE;
        while (total / size > int64_t(1) << 22) size *= 2;
        for (int i = 0; i < count; ++i)
            for (int64_t at = 0; at < counts[i]; at += size) {
                ClipPiece q{};
                q.g = static_cast<char *>(grads[i]) + at * elem_bytes(grad_dtype[i]);
                q.p = params ? static_cast<char *>(params[i]) + at * elem_bytes(param_dtype[i]) : nullptr;
                q.count = static_cast<uint32_t>(std::min(size, counts[i] - at));
                q.g_bf16 = grad_dtype[i] == CAPGNN_BF16;
                q.p_bf16 = params && param_dtype[i] == CAPGNN_BF16;
                pieces.push_back(q);
            }
        capgnn_tensors *h = new capgnn_tensors;
        h->n = static_cast<unsigned>(pieces.size());
        h->params = params != nullptr;
        if (h->n) {
            if (hipMalloc(reinterpret_cast<void **>(&h->pieces), pieces.size() * sizeof(ClipPiece)) != hipSuccess) {
                (void)hipGetLastError();
                delete h;
                CG_FAIL(CAPGNN_ENOMEM, "tensors_create: hipMalloc of %zu bytes failed", pieces.size() * sizeof(ClipPiece));
            }
            hipStream_t st = static_cast<hipStream_t>(stream);
            hipError_t e = hipMemcpyAsync(h->pieces, pieces.data(), pieces.size() * sizeof(ClipPiece), hipMemcpyHostToDevice, st);
            if (e == hipSuccess) e = hipStreamSynchronize(st);
            if (e != hipSuccess) {
                (void)hipFree(h->pieces);
                delete h;
                CG_FAIL(CAPGNN_EHIP, "tensors_create: %s", hipGetErrorString(e));
            }
        }
        *t = h;
    } catch (const std::exception &) {
        CG_FAIL(CAPGNN_ENOMEM, "tensors_create: out of host memory");
    }
    return CAPGNN_OK;
}

extern "C" int capgnn_tensors_destroy(capgnn_tensors *t) {
    if (!t) return CAPGNN_OK;
    if (t->pieces) (void)hipFree(t->pieces);
    delete t;
    return CAPGNN_OK;
}

extern "C" size_t capgnn_grad_workspace_bytes(const capgnn_tensors *t) {
    return t ? align_up(std::max(1u, std::min(t->n, CLIP_GROUPS)) * sizeof(double), 256) : 0;
}

static int clip_check(const char *who, const capgnn_tensors *t, const float *norm_dev, const void *ws, size_t ws_bytes) {
    if (!t) CG_FAIL(CAPGNN_EINVAL, "%s: NULL list", who);
    if (!norm_dev || !row_aligned(norm_dev, CAPGNN_F32)) CG_FAIL(CAPGNN_EINVAL, "%s: norm_dev must be a device float", who);
    const size_t need = capgnn_grad_workspace_bytes(t);
    if (!ws || ws_bytes < need) CG_FAIL(CAPGNN_ENOMEM, "%s: workspace of %zu bytes needed, %zu given", who, need, ws ? ws_bytes : size_t(0));
    if (reinterpret_cast<uintptr_t>(ws) & 255u) CG_FAIL(CAPGNN_EINVAL, "%s: workspace must be 256-byte aligned", who);
    return CAPGNN_OK;
}

// the first launch; *groups = how many sums it leaves
static int clip_squares(const capgnn_tensors *t, double *sums, unsigned *groups, hipStream_t st) {
    *groups = std::min(t->n, CLIP_GROUPS);
    if (*groups) hipLaunchKernelGGL(clip_squares_kernel, dim3(*groups), dim3(256), 0, st, t->pieces, t->n, sums);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}

extern "C" int capgnn_grad_norm(const capgnn_tensors *t, float *norm_dev, void *ws, size_t ws_bytes, void *stream) {
    CG_TRY(clip_check("grad_norm", t, norm_dev, ws, ws_bytes));
    hipStream_t st = static_cast<hipStream_t>(stream);
    double *sums = static_cast<double *>(ws);
    unsigned groups;
    CG_TRY(clip_squares(t, sums, &groups, st));
    hipLaunchKernelGGL(clip_norm_kernel, dim3(1), dim3(256), 0, st, sums, groups, norm_dev);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}

template <bool STEP> static int clip_apply(const capgnn_tensors *t, float lr, float max_norm, float *norm_dev, void *ws, hipStream_t st) {
    double *sums = static_cast<double *>(ws);
    unsigned groups;
    CG_TRY(clip_squares(t, sums, &groups, st));
    hipLaunchKernelGGL(clip_apply_kernel<STEP>, dim3(std::max(1u, groups)), dim3(256), 0, st, t->pieces, t->n, sums, groups, lr, max_norm, norm_dev);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}

extern "C" int capgnn_grad_clip(const capgnn_tensors *t, float max_norm, float *norm_dev, void *ws, size_t ws_bytes, void *stream) {
    CG_TRY(clip_check("grad_clip", t, norm_dev, ws, ws_bytes));
    if (!(max_norm >= 0.f)) CG_FAIL(CAPGNN_EINVAL, "grad_clip: max_norm must not be negative or NaN");
    return clip_apply<false>(t, 0.f, max_norm, norm_dev, ws, static_cast<hipStream_t>(stream));
}

extern "C" int capgnn_clipped_step(const capgnn_tensors *t, float lr, float max_norm, float *norm_dev, void *ws, size_t ws_bytes, void *stream) {
    CG_TRY(clip_check("clipped_step", t, norm_dev, ws, ws_bytes));
    if (!t->params) CG_FAIL(CAPGNN_EINVAL, "clipped_step: the list has no params");
    if (!std::isfinite(lr)) CG_FAIL(CAPGNN_EINVAL, "clipped_step: lr must be finite");
    if (!(max_norm >= 0.f)) CG_FAIL(CAPGNN_EINVAL, "clipped_step: max_norm must not be negative or NaN");
    return clip_apply<true>(t, lr, max_norm, norm_dev, ws, static_cast<hipStream_t>(stream));
}
