// Distillation from a teacher's top logits: the divergence of a row's softmax from the teacher's classes, and its gradient.
#include "softrow.h"

#include <algorithm>

namespace capgnn {

struct DistillArgs {
    int64_t n;
    int C;
    const char *Z; int64_t ldz;
    TempScale t;
    const uint8_t *mask;
    const int32_t *t_ids; const float *t_val; int64_t ldt; int k, rest;
    float weight;
    float norm_val; const float *norm_dev;
    double *part;                   // [gridDim.x]
    float *row_loss;
    char *dZ; int64_t lddz; int accumulate;
};

constexpr int SEEN_BITS = 32768;
constexpr float REST_LEAST = 9.5367431640625e-7f;       // 2^-20

// One workgroup per row; thread i holds the teacher's entry i.  What the teacher leaves (rest) is the small difference of numbers near 1: its
// exponentials and their sum are doubles.  The row's own probability outside the listed classes may be as small, so it is summed without
// them: a bit per class (modulo 32768) says which classes to look up in the list.
template <bool BF16, bool DBF16>
__global__ __launch_bounds__(256) void distill_kernel(DistillArgs a) {
    __shared__ int32_t id[CAPGNN_GIVEN_MAX];
    __shared__ float qs[CAPGNN_GIVEN_MAX];
    __shared__ float red[4];
    __shared__ double redd[4];
    __shared__ uint32_t seen[SEEN_BITS / 32];
    const float norm = a.norm_dev ? a.norm_dev[0] : a.norm_val;
    const float scale = a.weight / norm * a.t.inv_T;
    double loss = 0.0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const char *z = a.Z + row * a.ldz * (BF16 ? 2 : 4);
        char *dz = a.dZ ? a.dZ + row * a.lddz * (DBF16 ? 2 : 4) : nullptr;
        const bool on = !a.mask || a.mask[row];
        const int i = threadIdx.x;
        int c = -1;
        float v = 0.f;
        if (on && i < a.k) {
            c = a.t_ids[row * a.ldt + i];
            v = a.t_val[row * a.ldt + i];
            if (c < 0 || c >= a.C || v == -INFINITY) c = -1;
        }
        id[i] = c;
        const int entries = __syncthreads_count(c >= 0);
        float m = -INFINITY;
        if (on && entries) {
            for (int j = i; j < a.C; j += 256) m = max_of(m, ld_logit<BF16>(z, j));
            m = group_all<256>(m, red, OpMax());
        }
        const float m0 = safe_max(m);
        if (a.rest && on && entries) {
            for (int w = i; w < SEEN_BITS / 32; w += 256) seen[w] = 0;
            __syncthreads();
            if (c >= 0) atomicOr(&seen[c % SEEN_BITS / 32], 1u << (c % 32));
            __syncthreads();
        }
        bool first = c >= 0;
        for (int b = 0; b < i && first; ++b) first = id[b] != c;
        const float zc = first ? ld_logit<BF16>(z, c) : 0.f;
        const float ec = first ? exp_scaled(zc - m0, a.t) : 0.f;
        float others = 0.f, S = 0.f;        // the sum outside the listed classes (rest), the sum
        if (on && entries) {
            for (int j = i; j < a.C; j += 256) {
                const float e = exp_scaled(ld_logit<BF16>(z, j) - m0, a.t);
                bool out = true;
                if (a.rest && (seen[j % SEEN_BITS / 32] >> (j % 32) & 1u))
                    for (int b = 0; b < a.k && out; ++b) out = id[b] != j;
                others += out ? e : 0.f;
            }
            others = group_all<256>(others, red, OpSum());
            S = a.rest ? others + group_all<256>(ec, red, OpSum()) : others;
        }
        if (!on || !entries || S == 0.f) {
            if (a.row_loss && i == 0) a.row_loss[row] = 0.f;
            if (dz && !a.accumulate) for (int j = i; j < a.C; j += 256) st_grad<DBF16>(dz, j, 0.f);
            __syncthreads();
            continue;
        }
        // the teacher's distribution
        double q = 0.0;
        if (a.rest) {
            if (c >= 0) q = exp(static_cast<double>(v));
        } else {
            const float vm = group_all<256>(c >= 0 ? v : -INFINITY, red, OpMax());
            if (c >= 0) q = exp((static_cast<double>(v) - vm) * a.t.inv_T);
            const double Q = group_all<256>(q, redd, OpSum());
            q /= Q;
        }
        qs[i] = static_cast<float>(q);
        __syncthreads();
        float qc = 0.f;
        for (int b = i; b < a.k; ++b)
            if (id[b] == c) qc += qs[b];
        const double Q = group_all<256>(q, redd, OpSum());
        double r = a.rest ? 1.0 - Q : 0.0;
        if (r < REST_LEAST) r = 0.0;
        const float ln_s = logf(S), inv_s = 1.f / S;
        float term = 0.f;
        if (first && qc != 0.f) term = fmaf(-qc * (zc - m0), a.t.inv_T, qc * (logf(qc) + ln_s));   // (q d before 1/T: d / T may leave float's range)
        double kl = group_all<256>(static_cast<double>(term), redd, OpSum());
        if (r > 0.0) kl += r * (log(r) - (log(static_cast<double>(others)) - log(static_cast<double>(S))));
        if (i == 0) {
            loss += kl;
            if (a.row_loss) a.row_loss[row] = static_cast<float>(kl);
        }
        if (dz) {
            const float mass = static_cast<float>(a.rest ? Q + r : 1.0 + 0.0 * Q);
            const float away = r > 0.0 ? static_cast<float>((Q + r) - r * (static_cast<double>(S) / others)) : mass;
            float old = 0.f;
            if (first && a.accumulate) old = ld_logit<DBF16>(dz, c);
            __syncthreads();
            for (int j = i; j < a.C; j += 256) {
                const float p = exp_scaled(ld_logit<BF16>(z, j) - m0, a.t) * inv_s;
                const float g = p == 0.f ? 0.f : p * away * scale;
                st_grad<DBF16>(dz, j, a.accumulate ? ld_logit<DBF16>(dz, j) + g : g);
            }
            __syncthreads();
            if (first) st_grad<DBF16>(dz, c, old + (ec * inv_s * mass - qc) * scale);
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) a.part[blockIdx.x] = loss;
}

// loss = weight / norm * sum of part
__global__ __launch_bounds__(256) void distill_final_kernel(int parts, const double *part, float weight, float norm_val, const float *norm_dev,
                                                            float *loss_out) {
    __shared__ double red[4];
    double c = 0.0;
    for (int b = threadIdx.x; b < parts; b += 256) c += part[b];
    c = group_all<256>(c, red, OpSum());
    if (threadIdx.x == 0) loss_out[0] = static_cast<float>(c * weight / (norm_dev ? norm_dev[0] : norm_val));
}

constexpr size_t DISTILL_HEADER = 8192;     // [0] the normaliser, [256 ..] counts of the mask
constexpr int DISTILL_PARTS = 8192;

}  // namespace capgnn

using namespace capgnn;

extern "C" size_t capgnn_distill_workspace_bytes(int64_t n, int C) {
    (void)C;
    return DISTILL_HEADER + align_up(sizeof(double) * static_cast<size_t>(std::min<int64_t>(std::max<int64_t>(n, 1), DISTILL_PARTS)), 256);
}

extern "C" int capgnn_distill(int64_t n, int C, const void *Z, int64_t ldz, int z_dtype, const int32_t *teacher_ids,
                              const float *teacher_val, int64_t ldt, int k, int rest, float temperature, const uint8_t *mask,
                              double loss_norm, float weight, float *loss_dev, float *row_loss, void *dZ, int64_t lddz, int dz_dtype,
                              int accumulate, void *ws, size_t ws_bytes, void *stream) {
    if ((z_dtype != CAPGNN_F32 && z_dtype != CAPGNN_BF16) || (dz_dtype != CAPGNN_F32 && dz_dtype != CAPGNN_BF16))
        CG_FAIL(CAPGNN_EINVAL, "distill: unknown z_dtype or dz_dtype");
    if (n < 0 || C <= 0) CG_FAIL(CAPGNN_EINVAL, "distill: bad sizes");
    if (k < 1 || k > CAPGNN_GIVEN_MAX) CG_FAIL(CAPGNN_EINVAL, "distill: k = %d, 1 to %d classes of a teacher expected", k, CAPGNN_GIVEN_MAX);
    if (rest != 0 && rest != 1) CG_FAIL(CAPGNN_EINVAL, "distill: rest must be 0 or 1");
    if (!good_temperature(temperature)) CG_FAIL(CAPGNN_EINVAL, "distill: the temperature must be positive and finite");
    if (!std::isfinite(weight) || loss_norm != loss_norm) CG_FAIL(CAPGNN_EINVAL, "distill: weight or loss_norm is not a number");
    if (!loss_dev) CG_FAIL(CAPGNN_EINVAL, "distill: NULL operand");
    if (n > 0 && (!Z || !teacher_ids || !teacher_val)) CG_FAIL(CAPGNN_EINVAL, "distill: NULL operand");
    if (ldz < C || ldt < k || (dZ && lddz < C)) CG_FAIL(CAPGNN_EINVAL, "distill: leading dimension smaller than the row");
    if (!element_aligned(Z, z_dtype) || (dZ && !element_aligned(dZ, dz_dtype))) CG_FAIL(CAPGNN_EINVAL, "distill: Z or dZ is not aligned to its elements");
    if (n > 0 && dZ == Z && (lddz != ldz || dz_dtype != z_dtype || accumulate))
        CG_FAIL(CAPGNN_EINVAL, "distill: dZ may be Z only with the same type and pitch, and not to accumulate");
    const size_t need = capgnn_distill_workspace_bytes(n, C);
    if (!ws || ws_bytes < need) CG_FAIL(CAPGNN_ENOMEM, "distill: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : size_t(0));
    if (reinterpret_cast<uintptr_t>(ws) & 255u) CG_FAIL(CAPGNN_EINVAL, "distill: workspace must be 256-byte aligned");
    hipStream_t st = static_cast<hipStream_t>(stream);
    char *w = static_cast<char *>(ws);
    DistillArgs a{};
    a.n = n; a.C = C; a.Z = static_cast<const char *>(Z); a.ldz = ldz; a.t = temp_scale(temperature); a.mask = mask;
    a.t_ids = teacher_ids; a.t_val = teacher_val; a.ldt = ldt; a.k = k; a.rest = rest; a.weight = weight;
    a.row_loss = row_loss; a.dZ = static_cast<char *>(dZ); a.lddz = lddz; a.accumulate = accumulate;
    a.part = reinterpret_cast<double *>(w + DISTILL_HEADER);
    a.norm_val = 1.f;
    if (loss_norm > 0.0) a.norm_val = static_cast<float>(loss_norm);
    else if (n == 0 || !mask) a.norm_val = static_cast<float>(std::max<int64_t>(n, 1));
    else {
        CG_TRY(launch_mask_count(n, mask, reinterpret_cast<float *>(w), reinterpret_cast<double *>(w + 256), st));
        a.norm_dev = reinterpret_cast<const float *>(w);
    }
    const int grid = static_cast<int>(std::min<int64_t>(n, DISTILL_PARTS));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(grid)), dim3(256), 0, st, a); };
    if (grid > 0) {
        if (z_dtype == CAPGNN_BF16) dz_dtype == CAPGNN_BF16 ? go(distill_kernel<true, true>) : go(distill_kernel<true, false>);
        else dz_dtype == CAPGNN_BF16 ? go(distill_kernel<false, true>) : go(distill_kernel<false, false>);
    }
    hipLaunchKernelGGL(distill_final_kernel, dim3(1), dim3(256), 0, st, grid, a.part, weight, a.norm_val, a.norm_dev, loss_dev);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}
