// The operators on rows behind the C boundary (include/gvhot.h): checks of their arguments, and the launches.
#include "gvhot.h"

#include <math.h>

#include <initializer_list>

#include "gv_host.hpp"
#include "gv_rows.hpp"

namespace {

using gv::fail_call;

constexpr uint64_t kMostRows = 1ull << 31, kMostStride = 1ull << 40, kMostQueries = 1ull << 16;

uint32_t size_of(int type) { return type == GV_F32 ? 4u : type == GV_I8 ? 1u : 2u; }

struct Matrix {
    const char *name;
    const void *at;
    uint64_t stride;
    int type;
};

int check_shape(const char *call, uint64_t rows, uint32_t cols, int type, bool bytes_too) {
    if (rows > kMostRows) return fail_call(GV_EINVAL, "%s: %llu rows: at most 2^31", call, (unsigned long long)rows);
    if (cols == 0 || cols > GV_MAX_ROW_COLS)
        return fail_call(GV_EINVAL, "%s: %u columns: 1..%u", call, cols, GV_MAX_ROW_COLS);
    if (type < GV_F32 || type > (bytes_too ? GV_I8 : GV_F16)) return fail_call(GV_EINVAL, "%s: bad type %d", call, type);
    return GV_OK;
}

int check_matrices(const char *call, uint32_t cols, std::initializer_list<Matrix> all) {
    for (const Matrix &m : all) {
        if (!m.at) return fail_call(GV_EINVAL, "%s: null %s", call, m.name);
        if ((uintptr_t)m.at % size_of(m.type)) return fail_call(GV_EINVAL, "%s: %s is not aligned to its values", call, m.name);
        if (m.stride < cols || m.stride > kMostStride)
            return fail_call(GV_EINVAL, "%s: stride %llu of %s: cols (%u)..2^40", call, (unsigned long long)m.stride, m.name, cols);
    }
    return GV_OK;
}

// float arrays and the like
int check_array(const char *call, const char *name, const void *at, uint32_t align) {
    if (!at) return fail_call(GV_EINVAL, "%s: null %s", call, name);
    if ((uintptr_t)at % align) return fail_call(GV_EINVAL, "%s: %s is not aligned to %u bytes", call, name, align);
    return GV_OK;
}

int drop_args(const char *call, double drop, uint64_t seed, uint64_t first_row, gv::DropArgs *out) {
    const double t = floor(65536.0 * drop + 0.5);
    if (!(drop >= 0.0) || !(t < 65536.0)) return fail_call(GV_EINVAL, "%s: drop %g: 0 or more, and less than 1 - 2^-17", call, drop);
    *out = gv::DropArgs{(uint32_t)t, (float)(65536.0 / (65536.0 - t)), seed, first_row};
    return GV_OK;
}

uint64_t workspace_of(uint64_t rows, uint32_t cols) {
    const uint32_t parts = gv::norm_grad_parts(rows, cols);
    return parts > 1 ? 4ull * parts * cols : 0;
}

int launched(const char *call, hipError_t e) {
    return e == hipSuccess ? GV_OK : fail_call(GV_EHIP, "%s: %s", call, hipGetErrorString(e));
}

}  // namespace

#define GV_TRY(expr) do { const int rc_ = (expr); if (rc_ != GV_OK) return rc_; } while (0)

extern "C" {

int gv_drop_rows(uint64_t rows, uint32_t cols, int type, const void *dev_x, uint64_t x_stride, double drop, uint64_t seed,
                 uint64_t first_row, void *dev_out, uint64_t out_stride, void *stream) {
    const char *call = "gv_drop_rows";
    GV_TRY(check_shape(call, rows, cols, type, false));
    gv::DropRowsArgs a{dev_x, dev_out, rows, x_stride, out_stride, cols, type, {}};
    GV_TRY(drop_args(call, drop, seed, first_row, &a.drop));
    if (rows == 0) return GV_OK;
    GV_TRY(check_matrices(call, cols, {{"x", dev_x, x_stride, type}, {"out", dev_out, out_stride, type}}));
    return launched(call, gv::launch_drop(a, (hipStream_t)stream));
}

int gv_norm_rows(uint64_t rows, uint32_t cols, int type, const void *dev_x, uint64_t x_stride, const void *dev_residual,
                 uint64_t residual_stride, const float *dev_gain, float eps, double drop, uint64_t seed, uint64_t first_row,
                 void *dev_sum, uint64_t sum_stride, int out_type, void *dev_out, uint64_t out_stride, float *dev_out_scale,
                 float *dev_rstd, void *stream) {
    const char *call = "gv_norm_rows";
    GV_TRY(check_shape(call, rows, cols, type, false));
    if (out_type != type && out_type != GV_I8) return fail_call(GV_EINVAL, "%s: out_type is type or GV_I8", call);
    if (!(eps >= 0.0f) || !isfinite(eps)) return fail_call(GV_EINVAL, "%s: eps %g: 0 or more, and finite", call, (double)eps);
    gv::NormArgs a{dev_x, dev_residual, dev_gain, dev_sum, dev_out, dev_out_scale, dev_rstd, rows, x_stride, residual_stride,
                   sum_stride, out_stride, cols, type, out_type, eps, {}};
    GV_TRY(drop_args(call, drop, seed, first_row, &a.drop));
    if (rows == 0) return GV_OK;
    GV_TRY(check_matrices(call, cols, {{"x", dev_x, x_stride, type}, {"out", dev_out, out_stride, out_type}}));
    if (dev_residual) GV_TRY(check_matrices(call, cols, {{"residual", dev_residual, residual_stride, type}}));
    if (dev_sum) GV_TRY(check_matrices(call, cols, {{"sum", dev_sum, sum_stride, type}}));
    GV_TRY(check_array(call, "gain", dev_gain, 4));
    if (out_type == GV_I8) GV_TRY(check_array(call, "out_scale", dev_out_scale, 4));
    if (dev_rstd) GV_TRY(check_array(call, "rstd", dev_rstd, 4));
    return launched(call, gv::launch_norm(a, (hipStream_t)stream));
}

int gv_norm_rows_workspace(uint64_t rows, uint32_t cols, uint64_t *bytes) {
    const char *call = "gv_norm_rows_workspace";
    GV_TRY(check_shape(call, rows, cols, GV_F32, false));
    if (!bytes) return fail_call(GV_EINVAL, "%s: null output", call);
    *bytes = workspace_of(rows, cols);
    return GV_OK;
}

int gv_norm_rows_backward(uint64_t rows, uint32_t cols, int type, const void *dev_grad_out, uint64_t grad_out_stride,
                          const void *dev_sum, uint64_t sum_stride, const float *dev_gain, const float *dev_rstd,
                          const void *dev_grad_sum, uint64_t grad_sum_stride, double drop, uint64_t seed, uint64_t first_row,
                          void *dev_grad_x, uint64_t grad_x_stride, void *dev_grad_residual, uint64_t grad_residual_stride,
                          float *dev_grad_gain, void *dev_workspace, uint64_t workspace_bytes, void *stream) {
    const char *call = "gv_norm_rows_backward";
    GV_TRY(check_shape(call, rows, cols, type, false));
    gv::NormGradArgs a{dev_grad_out, dev_sum, dev_grad_sum, dev_gain, dev_rstd, dev_grad_x, dev_grad_residual, dev_grad_gain,
                       (float *)dev_workspace, rows, grad_out_stride, sum_stride, grad_sum_stride, grad_x_stride,
                       grad_residual_stride, cols, type, {}};
    GV_TRY(drop_args(call, drop, seed, first_row, &a.drop));
    if (dev_grad_gain) {
        GV_TRY(check_array(call, "grad_gain", dev_grad_gain, 4));
        const uint64_t need = workspace_of(rows, cols);
        if (need > 0) GV_TRY(check_array(call, "workspace", dev_workspace, 16));
        if (workspace_bytes < need)
            return fail_call(GV_EINVAL, "%s: workspace of %llu bytes: %llu are needed", call, (unsigned long long)workspace_bytes,
                             (unsigned long long)need);
    }
    if (rows > 0) {
        GV_TRY(check_matrices(call, cols, {{"grad_out", dev_grad_out, grad_out_stride, type}, {"sum", dev_sum, sum_stride, type}}));
        if (dev_grad_sum) GV_TRY(check_matrices(call, cols, {{"grad_sum", dev_grad_sum, grad_sum_stride, type}}));
        if (dev_grad_x) GV_TRY(check_matrices(call, cols, {{"grad_x", dev_grad_x, grad_x_stride, type}}));
        if (dev_grad_residual)
            GV_TRY(check_matrices(call, cols, {{"grad_residual", dev_grad_residual, grad_residual_stride, type}}));
        GV_TRY(check_array(call, "gain", dev_gain, 4));
        GV_TRY(check_array(call, "rstd", dev_rstd, 4));
    }
    if (!dev_grad_gain && (rows == 0 || (!dev_grad_x && !dev_grad_residual))) return GV_OK;
    return launched(call, gv::launch_norm_grad(a, (hipStream_t)stream));
}

int gv_quantize_rows(uint64_t rows, uint32_t cols, int type, const void *dev_x, uint64_t x_stride, uint32_t group,
                     uint8_t *dev_codes, uint16_t *dev_scales, void *stream) {
    const char *call = "gv_quantize_rows";
    GV_TRY(check_shape(call, rows, cols, type, false));
    if (group != 32 && group != 64 && group != 128) return fail_call(GV_EINVAL, "%s: group %u: 32, 64 or 128", call, group);
    if (rows == 0) return GV_OK;
    GV_TRY(check_matrices(call, cols, {{"x", dev_x, x_stride, type}}));
    GV_TRY(check_array(call, "codes", dev_codes, 16));
    GV_TRY(check_array(call, "scales", dev_scales, 2));
    return launched(call, gv::launch_quantize({dev_x, dev_codes, dev_scales, rows, x_stride, cols, group, type}, (hipStream_t)stream));
}

int gv_score_rows(uint64_t rows, uint32_t cols, uint32_t group, const uint8_t *dev_codes, const uint16_t *dev_scales,
                  uint64_t queries, int type, const void *dev_x, uint64_t x_stride, const float *dev_x_scale, float *dev_out,
                  uint64_t out_stride, void *stream) {
    const char *call = "gv_score_rows";
    GV_TRY(check_shape(call, rows, cols, type, true));
    if (group != 32 && group != 64 && group != 128) return fail_call(GV_EINVAL, "%s: group %u: 32, 64 or 128", call, group);
    if (queries > kMostQueries) return fail_call(GV_EINVAL, "%s: %llu queries: at most 2^16", call, (unsigned long long)queries);
    if (rows == 0 || queries == 0) return GV_OK;
    GV_TRY(check_matrices(call, cols, {{"x", dev_x, x_stride, type}}));
    GV_TRY(check_array(call, "codes", dev_codes, 16));
    GV_TRY(check_array(call, "scales", dev_scales, 2));
    GV_TRY(check_array(call, "out", dev_out, 4));
    if (type == GV_I8) GV_TRY(check_array(call, "x_scale", dev_x_scale, 4));
    if (type != GV_I8 && dev_x_scale) return fail_call(GV_EINVAL, "%s: x_scale belongs to GV_I8 rows", call);
    if (out_stride < rows || out_stride > kMostStride)
        return fail_call(GV_EINVAL, "%s: stride %llu of out: rows (%llu)..2^40", call, (unsigned long long)out_stride,
                         (unsigned long long)rows);
    return launched(call, gv::launch_score({dev_codes, dev_scales, dev_x, dev_x_scale, dev_out, rows, queries, x_stride, out_stride,
                                            cols, group, type}, (hipStream_t)stream));
}

}  // extern "C"
