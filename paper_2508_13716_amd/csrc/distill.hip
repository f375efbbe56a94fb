// capgnn_distill: checks, workspace, launches; the kernels without the teacher's remaining probability.
#include "distill.h"

#include <algorithm>

namespace capgnn {

// loss = weight / norm * sum of part
__global__ __launch_bounds__(1024) void distill_final_kernel(DistillArgs a, int parts, float *loss_out) {
    __shared__ double red[16];
    double c = 0.0;
    for (int b = threadIdx.x; b < parts; b += 8 * 1024) {       // (eight loads in flight)
        double v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = b + u * 1024 < parts ? a.part[b + u * 1024] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u) c += v[u];
    }
    const float norm = distill_norm(a);
    c = group_all<1024>(c, red, OpSum());
    if (threadIdx.x == 0) loss_out[0] = static_cast<float>(c * a.weight / norm);
}

constexpr size_t DISTILL_HEADER = 8192;     // [256 ..] counts of the mask

// Few long rows are cut into parts, about a thousand workgroups in all and at least DISTILL_PART_LEAST classes each; elsewhere
// one workgroup a row needs one launch less.  Parts against whole rows, us, k = 20: 1 x 24000 f32 15.2 / 12.8, 1 x 40000 f32 15.4 / 16.3,
// bf16 15.9 / 14.1, 1 x 65536 f32 14.9 / 21.8, bf16 15.0 / 16.1, 64 x 50000 bf16 19.8 / 17.0, 64 x 65536 f32 21.1 / 24.2, bf16 19.0 / 18.0,
// 128 x 150000 f32 47 / 53, bf16 33.9 / 35.3, 200 x 150000 f32 66 / 64, bf16 45 / 42, 300 x 9000 f32 20.0 / 13.1.
constexpr int DISTILL_PART_LEAST = 2048, DISTILL_WORKGROUPS = 1024;
constexpr int DISTILL_LONG = 49152, DISTILL_FEW = 1024;
static int distill_parts(int64_t n, int C, int *chunk) {
    if (C < DISTILL_LONG || C / DISTILL_FEW < n) { *chunk = C; return 1; }
    const int64_t parts = std::min<int64_t>(DISTILL_WORKGROUPS / std::max<int64_t>(n, 1), C / DISTILL_PART_LEAST);
    if (parts <= 1) { *chunk = C; return 1; }
    const int64_t c = ((C + parts - 1) / parts + 511) / 512 * 512;
    *chunk = static_cast<int>(c);
    return static_cast<int>((C + c - 1) / c);
}

}  // namespace capgnn

using namespace capgnn;

extern "C" size_t capgnn_distill_workspace_bytes(int64_t n, int C) {
    if (n < 0 || C <= 0) return 0;
    int chunk;
    const int parts = distill_parts(n, C, &chunk);
    return DISTILL_HEADER + sizeof(double) * DISTILL_GROUPS + (parts > 1 ? align_up((sizeof(float2) * parts + sizeof(float) * CAPGNN_GIVEN_MAX) * static_cast<size_t>(n), 256) : 0);
}

int capgnn::distill_check(int64_t n, int C, const void *Z, int64_t ldz, int z_dtype, const int32_t *teacher_ids, const float *teacher_val,
                          int64_t ldt, int k, int rest, float temperature, double loss_norm, float weight, const float *loss_dev,
                          const void *dZ, int64_t lddz, int dz_dtype, int accumulate) {
    if ((z_dtype != CAPGNN_F32 && z_dtype != CAPGNN_BF16) || (dz_dtype != CAPGNN_F32 && dz_dtype != CAPGNN_BF16))
        CG_FAIL(CAPGNN_EINVAL, "distill: unknown z_dtype or dz_dtype");
    if (n < 0 || C <= 0) CG_FAIL(CAPGNN_EINVAL, "distill: bad sizes");
    if (C > CLASSES_MOST) CG_FAIL(CAPGNN_EUNSUPPORTED, "distill: more than 2^30 classes");
    if (k < 1 || k > CAPGNN_GIVEN_MAX) CG_FAIL(CAPGNN_EINVAL, "distill: k = %d, 1 to %d classes of a teacher expected", k, CAPGNN_GIVEN_MAX);
    if (rest != 0 && rest != 1) CG_FAIL(CAPGNN_EINVAL, "distill: rest must be 0 or 1");
    if (!good_temperature(temperature)) CG_FAIL(CAPGNN_EINVAL, "distill: the temperature must lie between 2^-64 and 2^64");
    if (!std::isfinite(weight) || loss_norm != loss_norm) CG_FAIL(CAPGNN_EINVAL, "distill: weight or loss_norm is not a number");
    if (!loss_dev) CG_FAIL(CAPGNN_EINVAL, "distill: NULL operand");
    if (n > 0 && (!Z || !teacher_ids || !teacher_val)) CG_FAIL(CAPGNN_EINVAL, "distill: NULL operand");
    if (ldz < C || ldt < k || (dZ && lddz < C)) CG_FAIL(CAPGNN_EINVAL, "distill: leading dimension smaller than the row");
    if (!element_aligned(Z, z_dtype) || (dZ && !element_aligned(dZ, dz_dtype))) CG_FAIL(CAPGNN_EINVAL, "distill: Z or dZ is not aligned to its elements");
    if (n > 0 && dZ == Z && (lddz != ldz || dz_dtype != z_dtype || accumulate))
        CG_FAIL(CAPGNN_EINVAL, "distill: dZ may be Z only with the same type and pitch, and not to accumulate");
    return CAPGNN_OK;
}

extern "C" int capgnn_distill(int64_t n, int C, const void *Z, int64_t ldz, int z_dtype, const int32_t *teacher_ids,
                              const float *teacher_val, int64_t ldt, int k, int rest, float temperature, const uint8_t *mask,
                              double loss_norm, float weight, float *loss_dev, float *row_loss, void *dZ, int64_t lddz, int dz_dtype,
                              int accumulate, void *ws, size_t ws_bytes, void *stream) {
    CG_TRY(distill_check(n, C, Z, ldz, z_dtype, teacher_ids, teacher_val, ldt, k, rest, temperature, loss_norm, weight, loss_dev, dZ, lddz,
                         dz_dtype, accumulate));
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
        a.counts = reinterpret_cast<const double *>(w + 256);
        CG_TRY(launch_mask_counts(n, mask, reinterpret_cast<double *>(w + 256), &a.n_counts, st));
    }
    DistillParts p{};
    p.parts = distill_parts(n, C, &p.chunk);
    p.sums = reinterpret_cast<float2 *>(w + DISTILL_HEADER + sizeof(double) * DISTILL_GROUPS);
    p.listed = reinterpret_cast<float *>(p.sums + n * p.parts);
    int groups = 0;
    if (n > 0) {
        const bool zb = z_dtype == CAPGNN_BF16, db = dz_dtype == CAPGNN_BF16;
        const DistillLaunch run = rest ? distill_launch_rest(zb, db) : distill_launch_of<false>(zb, db);
        run(a, p, &groups, st);
    }
    hipLaunchKernelGGL(distill_final_kernel, dim3(1), dim3(1024), 0, st, a, groups, loss_dev);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}
