// The operators on rows behind the C boundary (include/gvhot.h): checks of their arguments, and the launches.
#include "gvhot.h"

#include <math.h>

#include <initializer_list>
#include <numeric>

#include "gv_host.hpp"
#include "gv_rows.hpp"

#define GV_TRY(expr) do { const int rc_ = (expr); if (rc_ != GV_OK) return rc_; } while (0)

namespace {

using gv::fail_call;

constexpr uint64_t kMostRows = 1ull << 31, kMostStride = 1ull << 40, kMostQueries = 1ull << 16;

uint32_t size_of(int type) { return type == GV_F32 || type == GV_I32 ? 4u : type == GV_I8 ? 1u : type == GV_I64 ? 8u : 2u; }

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

int check_index(const char *call, const gv::Index &index, uint64_t count, uint64_t rows) {
    if (count > kMostRows) return fail_call(GV_EINVAL, "%s: %llu indices: at most 2^31", call, (unsigned long long)count);
    if (rows > kMostRows) return fail_call(GV_EINVAL, "%s: %llu rows: at most 2^31", call, (unsigned long long)rows);
    if (index.type != GV_I32 && index.type != GV_I64)
        return fail_call(GV_EINVAL, "%s: index_type %d: GV_I32 or GV_I64", call, index.type);
    if (count == 0) return GV_OK;
    if (index.stride > kMostStride)
        return fail_call(GV_EINVAL, "%s: stride %llu of index: at most 2^40", call, (unsigned long long)index.stride);
    return check_array(call, "index", index.at, size_of(index.type));
}

// A matrix, as far as it goes.
struct Sized {
    Matrix matrix;
    uint64_t rows;
    uint32_t cols;
    uint64_t step() const { return rows > 1 ? matrix.stride * size_of(matrix.type) : 0; }  // bytes from row to row
    uint64_t width() const { return (uint64_t)cols * size_of(matrix.type); }
    unsigned __int128 end() const { return (unsigned __int128)(uintptr_t)matrix.at + (unsigned __int128)(rows - 1) * step() + width(); }
};

// Whether two matrices share values.  Those whose rows lie between each other's, as column slices of one buffer do, share none: what
// the steps from row to row have in common is a pattern that both repeat, and each has its own part of it.
bool overlap(const Sized &a, const Sized &b) {
    if (!a.matrix.at || !b.matrix.at || a.rows == 0 || b.rows == 0) return false;
    const uintptr_t a_at = (uintptr_t)a.matrix.at, b_at = (uintptr_t)b.matrix.at;
    if (a_at >= b.end() || b_at >= a.end()) return false;
    const uint64_t pattern = std::gcd(a.step(), b.step());
    if (pattern == 0) return true;  // one row each
    const uint64_t behind = b_at >= a_at ? (b_at - a_at) % pattern : (pattern - (a_at - b_at) % pattern) % pattern;
    return behind < a.width() || behind + b.width() > pattern;
}
// Whether an output is the very matrix of an input.
bool itself(const Sized &a, const Sized &b) {
    return a.matrix.at == b.matrix.at && a.rows == b.rows && a.cols == b.cols && a.matrix.type == b.matrix.type && a.step() == b.step();
}
int check_apart(const char *call, std::initializer_list<Sized> written, std::initializer_list<Sized> read) {
    for (const Sized &w : written)
        for (const Sized &r : read)
            if (overlap(w, r)) return fail_call(GV_EINVAL, "%s: %s overlaps %s", call, w.matrix.name, r.matrix.name);
    return GV_OK;
}

int check_workspace(const char *call, const void *workspace, uint64_t bytes, uint64_t need) {
    if (need > 0) GV_TRY(check_array(call, "workspace", workspace, 16));
    if (bytes < need)
        return fail_call(GV_EINVAL, "%s: workspace of %llu bytes: %llu are needed", call, (unsigned long long)bytes,
                         (unsigned long long)need);
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

int gv_lookup_rows(uint64_t count, const void *dev_index, uint64_t index_stride, int index_type, uint64_t rows, uint32_t cols, int type,
                   const void *dev_table, uint64_t table_stride, float scale, int out_type, void *dev_out, uint64_t out_stride,
                   void *stream) {
    const char *call = "gv_lookup_rows";
    const gv::Index index{dev_index, index_stride, index_type};
    if (type < GV_F32 || type > GV_I64) return fail_call(GV_EINVAL, "%s: bad type %d", call, type);
    GV_TRY(check_shape(call, rows, cols, GV_F32, false));
    if (type > GV_F16) {
        if (out_type != type || scale != 1.0f) return fail_call(GV_EINVAL, "%s: whole numbers are copied: out_type is type, scale 1", call);
    } else if (out_type < GV_F32 || out_type > GV_F16) {
        return fail_call(GV_EINVAL, "%s: bad out_type %d", call, out_type);
    }
    GV_TRY(check_index(call, index, count, rows));
    if (count == 0) return GV_OK;
    const Matrix table{"table", dev_table, table_stride, type}, out{"out", dev_out, out_stride, out_type};
    if (rows > 0) GV_TRY(check_matrices(call, cols, {table}));
    GV_TRY(check_matrices(call, cols, {out}));
    if (overlap({table, rows, cols}, {out, count, cols})) return fail_call(GV_EINVAL, "%s: out overlaps the table", call);
    const Sized result{out, count, cols}, indices{{"index", dev_index, index_stride, index_type}, count, 1};
    if (!itself(result, indices)) GV_TRY(check_apart(call, {result}, {indices}));
    return launched(call, gv::launch_lookup({index, dev_table, dev_out, count, table_stride, out_stride, (uint32_t)rows, cols, type, out_type,
                                             scale}, (hipStream_t)stream));
}

int gv_lookup_rows_workspace(uint64_t count, uint64_t rows, uint32_t cols, int add, uint64_t *bytes) {
    const char *call = "gv_lookup_rows_workspace";
    if (count > kMostRows) return fail_call(GV_EINVAL, "%s: %llu indices: at most 2^31", call, (unsigned long long)count);
    GV_TRY(check_shape(call, rows, cols, GV_F32, false));
    if (!bytes) return fail_call(GV_EINVAL, "%s: null output", call);
    *bytes = gv::lookup_grad_workspace(count, rows, cols, add != 0);
    return GV_OK;
}

int gv_lookup_rows_backward(uint64_t count, const void *dev_index, uint64_t index_stride, int index_type, uint64_t rows, uint32_t cols,
                            int type, const void *dev_grad, uint64_t grad_stride, float scale, int add, int out_type, void *dev_out,
                            uint64_t out_stride, void *dev_workspace, uint64_t workspace_bytes, void *stream) {
    const char *call = "gv_lookup_rows_backward";
    const gv::Index index{dev_index, index_stride, index_type};
    GV_TRY(check_shape(call, rows, cols, type, false));
    if (out_type < GV_F32 || out_type > GV_F16) return fail_call(GV_EINVAL, "%s: bad out_type %d", call, out_type);
    GV_TRY(check_index(call, index, count, rows));
    if (rows == 0 || (count == 0 && add)) return GV_OK;
    const Matrix grad{"grad", dev_grad, grad_stride, type}, out{"out", dev_out, out_stride, out_type};
    if (count > 0) GV_TRY(check_matrices(call, cols, {grad}));
    GV_TRY(check_matrices(call, cols, {out}));
    GV_TRY(check_apart(call, {{out, rows, cols}}, {{grad, count, cols}, {{"index", dev_index, index_stride, index_type}, count, 1}}));
    GV_TRY(check_workspace(call, dev_workspace, workspace_bytes, gv::lookup_grad_workspace(count, rows, cols, add != 0)));
    gv::LookupGradArgs a{};
    a.index = index, a.grad = dev_grad, a.out = dev_out, a.count = count, a.grad_stride = grad_stride, a.out_stride = out_stride;
    a.rows = (uint32_t)rows, a.cols = cols, a.type = type, a.out_type = out_type, a.scale = scale, a.add = add != 0;
    return launched(call, gv::launch_lookup_grad(a, dev_workspace, (hipStream_t)stream));
}

static int check_dense(const char *call, uint64_t rows, uint32_t cols, uint32_t outs, int type, int act) {
    GV_TRY(check_shape(call, rows, cols, type, false));
    if (outs == 0 || outs > GV_MAX_ROW_COLS) return fail_call(GV_EINVAL, "%s: %u columns of out: 1..%u", call, outs, GV_MAX_ROW_COLS);
    if (act < GV_ACT_NONE || act > GV_ACT_SILU) return fail_call(GV_EINVAL, "%s: bad activation %d", call, act);
    return GV_OK;
}

int gv_dense_rows_workspace(uint64_t rows, uint32_t cols, uint32_t outs, int type, uint64_t *bytes) {
    const char *call = "gv_dense_rows_workspace";
    GV_TRY(check_dense(call, rows, cols, outs, type, GV_ACT_NONE));
    if (!bytes) return fail_call(GV_EINVAL, "%s: null output", call);
    *bytes = gv::dense_workspace(rows, cols, outs, type);
    return GV_OK;
}

int gv_dense_rows(uint64_t rows, uint32_t cols, uint32_t outs, int type, const void *dev_x, uint64_t x_stride, const void *dev_weight,
                  uint64_t weight_stride, const void *dev_bias, int act, const void *dev_residual, uint64_t residual_stride,
                  void *dev_pre, uint64_t pre_stride, void *dev_out, uint64_t out_stride, void *dev_workspace, uint64_t workspace_bytes,
                  void *stream) {
    const char *call = "gv_dense_rows";
    GV_TRY(check_dense(call, rows, cols, outs, type, act));
    if (rows == 0) return GV_OK;
    const Sized x{{"x", dev_x, x_stride, type}, rows, cols}, weight{{"weight", dev_weight, weight_stride, type}, outs, cols};
    const Sized pre{{"pre", dev_pre, pre_stride, type}, rows, outs}, out{{"out", dev_out, out_stride, type}, rows, outs};
    GV_TRY(check_matrices(call, cols, {x.matrix, weight.matrix}));
    GV_TRY(check_matrices(call, outs, {out.matrix}));
    if (dev_bias) GV_TRY(check_array(call, "bias", dev_bias, size_of(type)));
    if (dev_residual) GV_TRY(check_matrices(call, outs, {{"residual", dev_residual, residual_stride, type}}));
    if (dev_pre) GV_TRY(check_matrices(call, outs, {pre.matrix}));
    const Sized residual{{"residual", dev_residual, residual_stride, type}, rows, outs}, bias{{"bias", dev_bias, outs, type}, 1, outs};
    GV_TRY(check_apart(call, {out, pre}, {x, weight}));
    GV_TRY(check_apart(call, {pre}, {out, residual}));
    if (!itself(out, residual)) GV_TRY(check_apart(call, {out}, {residual}));
    for (const Sized &written : {out, pre})
        if (!itself(written, bias)) GV_TRY(check_apart(call, {written}, {bias}));
    GV_TRY(check_workspace(call, dev_workspace, workspace_bytes, gv::dense_workspace(rows, cols, outs, type)));
    gv::DenseArgs a{};
    a.x = dev_x, a.weight = dev_weight, a.bias = dev_bias, a.residual = dev_residual, a.pre = dev_pre, a.out = dev_out;
    a.x_stride = x_stride, a.weight_stride = weight_stride, a.residual_stride = residual_stride, a.pre_stride = pre_stride;
    a.out_stride = out_stride, a.rows = (uint32_t)rows, a.cols = cols, a.outs = outs, a.type = type, a.act = act;
    return launched(call, gv::launch_dense(a, dev_workspace, (hipStream_t)stream));
}

int gv_dense_rows_backward_workspace(uint64_t rows, uint32_t cols, uint32_t outs, int type, int act, int grad_x, int grad_weight,
                                     int grad_bias, uint64_t *bytes) {
    const char *call = "gv_dense_rows_backward_workspace";
    GV_TRY(check_dense(call, rows, cols, outs, type, act));
    if (!bytes) return fail_call(GV_EINVAL, "%s: null output", call);
    *bytes = gv::dense_grad_workspace(rows, cols, outs, type, act, grad_x != 0, grad_weight != 0, grad_bias != 0);
    return GV_OK;
}

int gv_dense_rows_backward(uint64_t rows, uint32_t cols, uint32_t outs, int type, const void *dev_grad_out, uint64_t grad_out_stride,
                           const void *dev_x, uint64_t x_stride, const void *dev_weight, uint64_t weight_stride, int act,
                           const void *dev_pre, uint64_t pre_stride, void *dev_grad_x, uint64_t grad_x_stride, void *dev_grad_weight,
                           uint64_t grad_weight_stride, void *dev_grad_bias, void *dev_workspace, uint64_t workspace_bytes, void *stream) {
    const char *call = "gv_dense_rows_backward";
    GV_TRY(check_dense(call, rows, cols, outs, type, act));
    const Sized grad{{"grad_out", dev_grad_out, grad_out_stride, type}, rows, outs}, x{{"x", dev_x, x_stride, type}, rows, cols};
    const Sized weight{{"weight", dev_weight, weight_stride, type}, outs, cols}, pre{{"pre", dev_pre, pre_stride, type}, rows, outs};
    const Sized grad_x{{"grad_x", dev_grad_x, grad_x_stride, type}, rows, cols};
    const Sized grad_weight{{"grad_weight", dev_grad_weight, grad_weight_stride, type}, outs, cols};
    if (rows > 0) {
        GV_TRY(check_matrices(call, outs, {grad.matrix}));
        if (act != GV_ACT_NONE) GV_TRY(check_matrices(call, outs, {pre.matrix}));
        if (dev_grad_x) GV_TRY(check_matrices(call, cols, {weight.matrix, grad_x.matrix}));
        if (dev_grad_weight) GV_TRY(check_matrices(call, cols, {x.matrix}));
    }
    if (dev_grad_weight) GV_TRY(check_matrices(call, cols, {grad_weight.matrix}));
    if (dev_grad_bias) GV_TRY(check_array(call, "grad_bias", dev_grad_bias, size_of(type)));
    // of what the call reads
    const Sized none{}, bias{{"grad_bias", dev_grad_bias, outs, type}, 1, outs};
    const std::initializer_list<Sized> read = {grad, dev_grad_weight ? x : none, dev_grad_x && rows > 0 ? weight : none, act != GV_ACT_NONE ? pre : none};
    GV_TRY(check_apart(call, {grad_x, grad_weight}, read));
    GV_TRY(check_apart(call, {grad_x}, {grad_weight}));
    GV_TRY(check_workspace(call, dev_workspace, workspace_bytes,
                           gv::dense_grad_workspace(rows, cols, outs, type, act, dev_grad_x, dev_grad_weight, dev_grad_bias)));
    GV_TRY(check_apart(call, {bias}, read));
    GV_TRY(check_apart(call, {bias}, {grad_x, grad_weight}));
    gv::DenseGradArgs a{};
    a.grad = dev_grad_out, a.x = dev_x, a.weight = dev_weight, a.pre = dev_pre, a.grad_x = rows > 0 ? dev_grad_x : nullptr;
    a.grad_weight = dev_grad_weight, a.grad_bias = dev_grad_bias, a.rows = rows, a.grad_stride = grad_out_stride, a.x_stride = x_stride;
    a.weight_stride = weight_stride, a.pre_stride = pre_stride, a.grad_x_stride = grad_x_stride;
    a.grad_weight_stride = grad_weight_stride, a.cols = cols, a.outs = outs, a.type = type, a.act = act;
    return launched(call, gv::launch_dense_grad(a, dev_workspace, (hipStream_t)stream));
}

static int check_select(const char *call, uint64_t queries, uint64_t rows, uint32_t beams, uint32_t best) {
    if (queries > kMostQueries) return fail_call(GV_EINVAL, "%s: %llu queries: at most 2^16", call, (unsigned long long)queries);
    if (rows > kMostRows) return fail_call(GV_EINVAL, "%s: %llu rows: at most 2^31", call, (unsigned long long)rows);
    if (beams == 0 || beams > GV_MAX_BEAMS) return fail_call(GV_EINVAL, "%s: %u beams: 1..%u", call, beams, GV_MAX_BEAMS);
    if (queries % beams) return fail_call(GV_EINVAL, "%s: %llu queries are no groups of %u beams", call, (unsigned long long)queries, beams);
    if (best == 0 || best > GV_MAX_BEST) return fail_call(GV_EINVAL, "%s: the best %u: 1..%u", call, best, GV_MAX_BEST);
    return GV_OK;
}

int gv_select_rows_workspace(uint64_t queries, uint64_t rows, uint32_t beams, uint32_t best, uint64_t *bytes) {
    const char *call = "gv_select_rows_workspace";
    GV_TRY(check_select(call, queries, rows, beams, best));
    if (!bytes) return fail_call(GV_EINVAL, "%s: null output", call);
    *bytes = gv::select_workspace(queries, rows, beams, best);
    return GV_OK;
}

int gv_select_rows(uint64_t queries, uint64_t rows, int type, const void *dev_scores, uint64_t scores_stride, uint32_t beams,
                   const float *dev_totals, const uint8_t *dev_done, uint64_t end, int log_softmax, uint32_t best, int64_t *dev_parent,
                   int64_t *dev_row, float *dev_total, void *dev_workspace, uint64_t workspace_bytes, void *stream) {
    const char *call = "gv_select_rows";
    GV_TRY(check_select(call, queries, rows, beams, best));
    if (type < GV_F32 || type > GV_F16) return fail_call(GV_EINVAL, "%s: bad type %d", call, type);
    if (dev_done && end >= rows)
        return fail_call(GV_EINVAL, "%s: end %llu: a row of %llu", call, (unsigned long long)end, (unsigned long long)rows);
    if (queries == 0) return GV_OK;
    if (rows > 0) GV_TRY(check_array(call, "scores", dev_scores, size_of(type)));
    if (scores_stride < rows || scores_stride > kMostStride)
        return fail_call(GV_EINVAL, "%s: stride %llu of scores: rows (%llu)..2^40", call, (unsigned long long)scores_stride,
                         (unsigned long long)rows);
    if (dev_totals) GV_TRY(check_array(call, "totals", dev_totals, 4));
    GV_TRY(check_array(call, "parent", dev_parent, 8));
    GV_TRY(check_array(call, "row", dev_row, 8));
    GV_TRY(check_array(call, "total", dev_total, 4));
    GV_TRY(check_workspace(call, dev_workspace, workspace_bytes, gv::select_workspace(queries, rows, beams, best)));
    gv::SelectArgs a{};
    a.scores = dev_scores, a.totals = dev_totals, a.done = dev_done, a.parent = dev_parent, a.row = dev_row, a.total = dev_total;
    a.queries = queries, a.rows = rows, a.stride = scores_stride, a.beams = beams, a.best = best, a.end = (uint32_t)end, a.type = type;
    a.log_softmax = log_softmax != 0;
    return launched(call, gv::launch_select(a, dev_workspace, (hipStream_t)stream));
}

}  // extern "C"
