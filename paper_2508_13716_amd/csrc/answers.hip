// What a classifier answers with: log-probabilities of given classes, entropy, the most likely classes; and their gradient.
#include "softrow.h"

#include <algorithm>

namespace capgnn {

struct AnswerArgs {
    int64_t n;
    int C;
    const char *Z; int64_t ldz;
    TempScale t;
    const uint8_t *mask;
    const int32_t *ids; int64_t ldi; int m;
    float *logp; int64_t ldp;
    float *entropy, *stats;
    int k;
    int32_t *top_ids; float *top_logp; int64_t ldt;
};

// One workgroup per row: the largest logit, then the sums, then the k largest one after another.
template <bool BF16>
__global__ __launch_bounds__(256) void answers_kernel(AnswerArgs a) {
    __shared__ float red[4];
    __shared__ unsigned long long redk[4];
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const char *z = a.Z + row * a.ldz * (BF16 ? 2 : 4);
        if (a.mask && !a.mask[row]) {
            for (int i = threadIdx.x; i < a.m; i += 256) a.logp[row * a.ldp + i] = 0.f;
            for (int i = threadIdx.x; i < a.k; i += 256) {
                if (a.top_ids) a.top_ids[row * a.ldt + i] = -1;
                if (a.top_logp) a.top_logp[row * a.ldt + i] = 0.f;
            }
            if (threadIdx.x == 0) {
                if (a.entropy) a.entropy[row] = 0.f;
                if (a.stats) a.stats[2 * row] = a.stats[2 * row + 1] = 0.f;
            }
            continue;
        }
        float m = -INFINITY;
        for (int j = threadIdx.x; j < a.C; j += 256) m = max_of(m, ld_logit<BF16>(z, j));
        m = group_all<256>(m, red, OpMax());
        const float m0 = safe_max(m);
        float s = 0.f, e1 = 0.f;
        for (int j = threadIdx.x; j < a.C; j += 256) {
            const float d = ld_logit<BF16>(z, j) - m0, u = d * a.t.L, e = exp2_raw(u);
            s += e;
            e1 = fmaf(e, fmaxf(u, -160.f), e1);
        }
        s = group_all<256>(s, red, OpSum());
        e1 = group_all<256>(e1, red, OpSum());
        const bool empty = s == 0.f;
        const float ln_s = empty ? -INFINITY : logf(s);
        auto logp_of = [&](float v) { return empty ? -INFINITY : (v - m0) * a.t.inv_T - ln_s; };
        if (threadIdx.x == 0) {
            if (a.entropy) a.entropy[row] = empty ? 0.f : ln_s - e1 / s * 0.69314718f;
            if (a.stats) { a.stats[2 * row] = m; a.stats[2 * row + 1] = ln_s; }
        }
        for (int i = threadIdx.x; i < a.m; i += 256) {
            const int c = a.ids[row * a.ldi + i];
            a.logp[row * a.ldp + i] = c >= 0 && c < a.C ? logp_of(ld_logit<BF16>(z, c)) : 0.f;
        }
        unsigned long long last = ~0ull;
        for (int i = 0; i < a.k; ++i) {
            unsigned long long best = 0;
            for (int j = threadIdx.x; j < a.C; j += 256) {
                const unsigned long long key = logit_key(ld_logit<BF16>(z, j), j);
                if (key < last && key > best) best = key;
            }
            best = group_all<256>(best, redk, OpMaxKey());
            last = best;
            if (threadIdx.x == 0) {
                if (a.top_ids) a.top_ids[row * a.ldt + i] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(best));
                if (a.top_logp) a.top_logp[row * a.ldt + i] = logp_of(order_logit(static_cast<uint32_t>(best >> 32)));
            }
        }
    }
}

struct AnswerGradArgs {
    int64_t n;
    int C;
    const char *Z; int64_t ldz;
    TempScale t;
    const uint8_t *mask;
    const float *stats, *entropy;
    const int32_t *ids; int64_t ldi; int m;
    const float *dlogp; int64_t lddp;
    const float *dentropy;
    char *dZ; int64_t lddz;
};

// One workgroup per row: dz = -p (G + h (ln p + H)) everywhere, then the given classes get theirs from the thread that holds the first
// mention of the class.
template <bool BF16, bool DBF16>
__global__ __launch_bounds__(256) void answers_grad_kernel(AnswerGradArgs a) {
    __shared__ int32_t id[CAPGNN_GIVEN_MAX];
    __shared__ float g[CAPGNN_GIVEN_MAX];
    __shared__ float red[4];
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const char *z = a.Z + row * a.ldz * (BF16 ? 2 : 4);
        char *dz = a.dZ + row * a.lddz * (DBF16 ? 2 : 4);
        const bool on = !a.mask || a.mask[row];
        const float ln_s = on ? a.stats[2 * row + 1] : 0.f;
        if (!on || ln_s == -INFINITY) {
            for (int j = threadIdx.x; j < a.C; j += 256) st_grad<DBF16>(dz, j, 0.f);
            continue;
        }
        const float m0 = a.stats[2 * row], inv_s = expf(-ln_s);
        const float h = a.dentropy ? a.dentropy[row] : 0.f, H = a.dentropy ? a.entropy[row] : 0.f;
        float mine = 0.f, zc = 0.f;
        int c = -1;
        if (threadIdx.x < a.m) {
            c = a.ids[row * a.ldi + threadIdx.x];
            if (c < 0 || c >= a.C) c = -1;
            mine = c >= 0 ? a.dlogp[row * a.lddp + threadIdx.x] : 0.f;
            id[threadIdx.x] = c;
            g[threadIdx.x] = mine;
            if (c >= 0) zc = ld_logit<BF16>(z, c);
        }
        const float G = group_all<256>(mine, red, OpSum());
        auto base = [&](float v) {
            const float d = v - m0;
            const float p = exp_scaled(d, a.t) * inv_s;
            float f = G;
            if (a.dentropy && p != 0.f) f = fmaf(h, d * a.t.inv_T - ln_s + H, G);
            return -p * f;
        };
        for (int j = threadIdx.x; j < a.C; j += 256) st_grad<DBF16>(dz, j, base(ld_logit<BF16>(z, j)) * a.t.inv_T);
        __syncthreads();
        if (c >= 0) {
            bool first = true;
            float sum = 0.f;
            for (int i = 0; i < a.m; ++i)
                if (id[i] == c) {
                    if (i < static_cast<int>(threadIdx.x)) first = false;
                    sum += g[i];
                }
            if (first) st_grad<DBF16>(dz, c, (base(zc) + sum) * a.t.inv_T);
        }
        __syncthreads();
    }
}

}  // namespace capgnn

using namespace capgnn;

extern "C" size_t capgnn_logprobs_workspace_bytes(int64_t n, int C, int k) { (void)n; (void)C; (void)k; return 0; }

extern "C" int capgnn_logprobs(int64_t n, int C, const void *Z, int64_t ldz, int z_dtype, float temperature, const uint8_t *mask,
                               const int32_t *ids, int64_t ldi, int m, float *logp, int64_t ldp, float *entropy, float *stats,
                               int k, int32_t *top_ids, float *top_logp, int64_t ldt, void *ws, size_t ws_bytes, void *stream) {
    if (z_dtype != CAPGNN_F32 && z_dtype != CAPGNN_BF16) CG_FAIL(CAPGNN_EINVAL, "logprobs: unknown z_dtype");
    if (n < 0 || C <= 0) CG_FAIL(CAPGNN_EINVAL, "logprobs: bad sizes");
    if (m < 0 || m > CAPGNN_GIVEN_MAX) CG_FAIL(CAPGNN_EINVAL, "logprobs: m = %d, 0 to %d classes can be given per row", m, CAPGNN_GIVEN_MAX);
    if (k < 0 || k > CAPGNN_TOP_MAX || k > C) CG_FAIL(CAPGNN_EINVAL, "logprobs: k = %d, 0 to min(C, %d) expected", k, CAPGNN_TOP_MAX);
    if (!good_temperature(temperature)) CG_FAIL(CAPGNN_EINVAL, "logprobs: the temperature must be positive and finite");
    if (n == 0) return CAPGNN_OK;
    if (!Z || (m > 0 && (!ids || !logp)) || (k > 0 && !top_ids && !top_logp)) CG_FAIL(CAPGNN_EINVAL, "logprobs: NULL operand");
    if (ldz < C || (m > 0 && (ldi < m || ldp < m)) || (k > 0 && ldt < k)) CG_FAIL(CAPGNN_EINVAL, "logprobs: leading dimension smaller than the row");
    if (!element_aligned(Z, z_dtype)) CG_FAIL(CAPGNN_EINVAL, "logprobs: Z is not aligned to its elements");
    const size_t need = capgnn_logprobs_workspace_bytes(n, C, k);
    if (need && (!ws || ws_bytes < need)) CG_FAIL(CAPGNN_ENOMEM, "logprobs: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : size_t(0));
    if (need && reinterpret_cast<uintptr_t>(ws) & 255u) CG_FAIL(CAPGNN_EINVAL, "logprobs: workspace must be 256-byte aligned");
    hipStream_t st = static_cast<hipStream_t>(stream);
    AnswerArgs a{n, C, static_cast<const char *>(Z), ldz, temp_scale(temperature), mask, ids, ldi, m, logp, ldp, entropy, stats, k, top_ids,
                 top_logp, ldt};
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(n, 1 << 20));
    if (z_dtype == CAPGNN_BF16) hipLaunchKernelGGL(answers_kernel<true>, dim3(grid), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(answers_kernel<false>, dim3(grid), dim3(256), 0, st, a);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}

extern "C" int capgnn_logprobs_bwd(int64_t n, int C, const void *Z, int64_t ldz, int z_dtype, float temperature, const uint8_t *mask,
                                   const float *stats, const float *entropy, const int32_t *ids, int64_t ldi, int m, const float *dlogp,
                                   int64_t lddp, const float *dentropy, void *dZ, int64_t lddz, int dz_dtype, void *stream) {
    if ((z_dtype != CAPGNN_F32 && z_dtype != CAPGNN_BF16) || (dz_dtype != CAPGNN_F32 && dz_dtype != CAPGNN_BF16))
        CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: unknown z_dtype or dz_dtype");
    if (n < 0 || C <= 0) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: bad sizes");
    if (m < 0 || m > CAPGNN_GIVEN_MAX) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: m = %d, 0 to %d classes can be given per row", m, CAPGNN_GIVEN_MAX);
    if (!good_temperature(temperature)) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: the temperature must be positive and finite");
    if (n == 0) return CAPGNN_OK;
    if (!Z || !stats || !dZ || (m > 0 && (!ids || !dlogp)) || (dentropy && !entropy)) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: NULL operand");
    if (ldz < C || lddz < C || (m > 0 && (ldi < m || lddp < m))) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: leading dimension smaller than the row");
    if (!element_aligned(Z, z_dtype) || !element_aligned(dZ, dz_dtype)) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: Z or dZ is not aligned to its elements");
    if (dZ == Z && (lddz != ldz || dz_dtype != z_dtype)) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: dZ may be Z only with the same type and pitch");
    hipStream_t st = static_cast<hipStream_t>(stream);
    AnswerGradArgs a{n, C, static_cast<const char *>(Z), ldz, temp_scale(temperature), mask, stats, entropy, ids, ldi, m, dlogp, lddp,
                     dentropy, static_cast<char *>(dZ), lddz};
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(n, 1 << 20));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, st, a); };
    if (z_dtype == CAPGNN_BF16) dz_dtype == CAPGNN_BF16 ? go(answers_grad_kernel<true, true>) : go(answers_grad_kernel<true, false>);
    else dz_dtype == CAPGNN_BF16 ? go(answers_grad_kernel<false, true>) : go(answers_grad_kernel<false, false>);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}
