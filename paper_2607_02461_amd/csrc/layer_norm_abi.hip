// Entry points of the layer norms: argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "abi.h"
#include "device.h"
#include "internal.h"

using namespace orbit;

namespace {

constexpr int64_t kMaxReach = (int64_t)1 << 46;         // elements from a tensor's first to its last row
constexpr int64_t kMostThreads = (int64_t)UINT32_MAX;   // of a launch grid

bool is_type(int32_t t) { return t == ORBIT_OUT_F32 || t == ORBIT_OUT_BF16; }
int size_of(int32_t t) { return t == ORBIT_OUT_F32 ? 4 : 2; }
bool too_far(int64_t entries, int64_t stride) { return entries > 1 && (stride < 0 || stride > kMaxReach / (entries - 1)); }

orbit_status check_sizes(const char* who, int64_t B, int64_t L, int64_t N) {
    if (B < 0 || L < 0) return fail(ORBIT_EINVAL, "%s: negative B or L", who);
    if (N < 1) return fail(ORBIT_EINVAL, "%s: N=%lld must be positive", who, (long long)N);
    if (N > kNormMaxWidth) return fail(ORBIT_EUNSUPPORTED, "%s: N=%lld, up to %d is implemented", who, (long long)N, kNormMaxWidth);
    if (B > INT32_MAX || L > INT32_MAX || B * L > INT32_MAX) return fail(ORBIT_EUNSUPPORTED, "%s: more than 2^31 - 1 rows", who);
    return ORBIT_OK;
}

orbit_status check_rows(const char* who, const char* name, const orbit_rows* t, int64_t B, int64_t L, int64_t N, bool output, NormRows* out) {
    if (!t) return fail(ORBIT_EINVAL, "%s: %s is NULL", who, name);
    if (!is_type(t->dtype)) return fail(ORBIT_EINVAL, "%s: %s has the unknown type %d", who, name, t->dtype);
    if (B == 0 || L == 0) return ORBIT_OK;
    if (!t->data || !aligned(t->data, size_of(t->dtype))) return fail(ORBIT_EINVAL, "%s: %s is a null or misaligned device pointer", who, name);
    if (too_far(B, t->batch) || too_far(L, t->row)) return fail(ORBIT_EINVAL, "%s: %s has a stride out of range", who, name);
    out->p = t->data;
    out->batch = B > 1 ? t->batch : 0;
    out->row = L > 1 ? t->row : 0;
    if (!output) return ORBIT_OK;
    // batches behind each other, or between each other's rows
    const int64_t inner = L > 1 && B > 1 ? std::min(out->row, out->batch) : L > 1 ? out->row : out->batch;
    const int64_t outer = std::max(out->row, out->batch), many = inner == out->row ? L : B;
    if ((L > 1 || B > 1) && (inner < N || (L > 1 && B > 1 && outer < (many - 1) * inner + N)))
        return fail(ORBIT_EINVAL, "%s: %s's rows overlap", who, name);
    return ORBIT_OK;
}

// An output may replace an input row by row: its type and strides
orbit_status check_place(const char* who, const char* name, const NormRows& y, int32_t y_type, const NormRows& from, int32_t type) {
    if (!y.p || y.p != from.p || (y_type == type && y.batch == from.batch && y.row == from.row)) return ORBIT_OK;
    return fail(ORBIT_EINVAL, "%s: %s lies on an input that it does not replace row by row", who, name);
}

orbit_status check_weight(const char* who, const char* name, const void* w, int64_t batch, int64_t B, int64_t N, int32_t dtype) {
    if (!w) return ORBIT_OK;
    if (!is_type(dtype)) return fail(ORBIT_EINVAL, "%s: unknown type %d of the weights", who, dtype);
    if (!aligned(w, size_of(dtype))) return fail(ORBIT_EINVAL, "%s: misaligned %s", who, name);
    if (too_far(B, batch)) return fail(ORBIT_EINVAL, "%s: %s has a stride out of range", who, name);
    return ORBIT_OK;
}

// Whether the batches' rows follow each other at one stride
bool flat(const NormRows& t, int64_t B, int64_t L) { return B <= 1 || L == 0 || t.batch == L * t.row; }

// Groups of rows with weights of their own, and the rows of one
int groups_of(int64_t B, bool joined) { return joined ? 1 : (int)B; }
int64_t rows_of(int64_t B, int64_t L, bool joined) { return joined ? B * L : L; }

size_t workspace_bytes_of(int64_t B, int64_t L, int64_t N, bool joined, int cus) {
    if (B == 0 && !joined) return 0;
    const int groups = groups_of(B, joined);
    return (size_t)groups * layer_norm_parts(rows_of(B, L, joined), groups, N, false, cus) * 2 * N * sizeof(float);
}

}  // namespace

extern "C" {

orbit_status layer_norm(const orbit_rows* x, const orbit_rows* y, int64_t B, int64_t L, int64_t N, const void* weight, int64_t weight_batch,
                        const void* bias, int64_t bias_batch, int32_t w_dtype, int32_t modulate, float eps, void* stream) {
    const char* who = "layer_norm";
    clear_error();
    orbit_status st = check_sizes(who, B, L, N);
    NormParams p{};
    if (st == ORBIT_OK) st = check_rows(who, "x", x, B, L, N, false, &p.x);
    if (st == ORBIT_OK) st = check_rows(who, "y", y, B, L, N, true, &p.y);
    if (st == ORBIT_OK) st = check_place(who, "y", p.y, y->dtype, p.x, x->dtype);
    if (st == ORBIT_OK) st = check_weight(who, "weight", weight, weight_batch, B, N, w_dtype);
    if (st == ORBIT_OK) st = check_weight(who, "bias", bias, bias_batch, B, N, w_dtype);
    if (st != ORBIT_OK) return st;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(ORBIT_EINVAL, "%s: eps must be finite and at least 0", who);
    if (B == 0 || L == 0) return ORBIT_OK;
    int dev;
    DeviceInfo info;
    st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    p.w = weight;
    p.b = bias;
    p.w_batch = weight && B > 1 ? weight_batch : 0;
    p.b_batch = bias && B > 1 ? bias_batch : 0;
    p.w_f32 = w_dtype == ORBIT_OUT_F32;
    p.modulate = modulate != 0;
    p.N = (int)N;
    p.joined = p.w_batch == 0 && p.b_batch == 0;
    p.rows = rows_of(B, L, p.joined);
    p.L = L;
    p.eps = eps;
    const int groups = groups_of(B, p.joined);
    if (flat(p.x, B, L) && flat(p.y, B, L)) p.joined = 0;
    if ((int64_t)groups * 1024 > kMostThreads) return fail(ORBIT_EUNSUPPORTED, "%s: more than 2^22 - 1 batches with weights of their own", who);
    const hipError_t e = launch_layer_norm(p, groups, x->dtype == ORBIT_OUT_F32, y->dtype == ORBIT_OUT_F32, info.cus, (hipStream_t)stream);
    return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
}

orbit_status layer_norm_backward_workspace_size(int64_t B, int64_t L, int64_t N, int32_t per_batch, size_t* bytes) {
    const char* who = "layer_norm_backward_workspace_size";
    clear_error();
    if (!bytes) return fail(ORBIT_EINVAL, "%s: null output pointer", who);
    *bytes = 0;
    orbit_status st = check_sizes(who, B, L, N);
    if (st != ORBIT_OK) return st;
    int dev;
    DeviceInfo info;
    st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    *bytes = workspace_bytes_of(B, L, N, !per_batch, info.cus);
    return ORBIT_OK;
}

orbit_status layer_norm_backward(const orbit_rows* dy, const orbit_rows* x, const orbit_rows* dx, int64_t B, int64_t L, int64_t N, const void* weight,
                                 int64_t weight_batch, int32_t w_dtype, int32_t modulate, float eps, float* dweight, float* dbias,
                                 int32_t per_batch, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "layer_norm_backward";
    clear_error();
    orbit_status st = check_sizes(who, B, L, N);
    NormParams p{};
    if (st == ORBIT_OK) st = check_rows(who, "dy", dy, B, L, N, false, &p.g);
    if (st == ORBIT_OK) st = check_rows(who, "x", x, B, L, N, false, &p.x);
    if (st == ORBIT_OK) st = check_rows(who, "dx", dx, B, L, N, true, &p.y);
    if (st != ORBIT_OK) return st;
    if (dx->dtype != x->dtype) return fail(ORBIT_EINVAL, "%s: dx must have x's type", who);
    st = check_place(who, "dx", p.y, dx->dtype, p.x, x->dtype);
    if (st == ORBIT_OK) st = check_place(who, "dx", p.y, dx->dtype, p.g, dy->dtype);
    if (st == ORBIT_OK) st = check_weight(who, "weight", weight, weight_batch, B, N, w_dtype);
    if (st != ORBIT_OK) return st;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(ORBIT_EINVAL, "%s: eps must be finite and at least 0", who);
    if (!aligned(dweight, 4) || !aligned(dbias, 4)) return fail(ORBIT_EINVAL, "%s: misaligned gradient", who);
    if (weight && B > 1 && weight_batch && !per_batch && (dweight || dbias))
        return fail(ORBIT_EINVAL, "%s: batches with weights of their own have gradients of their own", who);
    if (B == 0 && per_batch) return ORBIT_OK;
    int dev;
    DeviceInfo info;
    st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    p.w = weight;
    p.w_batch = weight && B > 1 ? weight_batch : 0;
    p.w_f32 = w_dtype == ORBIT_OUT_F32;
    p.modulate = modulate != 0;
    p.N = (int)N;
    p.joined = !per_batch && p.w_batch == 0;
    p.rows = rows_of(B, L, p.joined);
    p.L = L;
    p.eps = eps;
    p.dw = dweight;
    p.db = dbias;
    const int groups = groups_of(B, p.joined);
    p.parts = layer_norm_parts(p.rows, groups, N, x->dtype == ORBIT_OUT_F32, info.cus);
    const size_t bytes = workspace_bytes_of(B, L, N, p.joined, info.cus);
    if (flat(p.x, B, L) && flat(p.y, B, L) && flat(p.g, B, L)) p.joined = 0;
    if ((int64_t)groups * std::max<int64_t>(1024 * p.parts, (N + 31) / 32 * 1024) > kMostThreads)
        return fail(ORBIT_EUNSUPPORTED, "%s: too many batches with gradients of their own for one launch", who);
    if (dweight || dbias) {
        if (!workspace || !aligned(workspace, 16) || workspace_bytes < bytes)
            return fail(ORBIT_EINVAL, "%s: takes a workspace of %zu bytes, aligned to 16", who, bytes);
        p.part = (float*)workspace;
    } else if (B == 0 || L == 0) {
        return ORBIT_OK;
    }
    const hipError_t e = launch_layer_norm_backward(p, groups, x->dtype == ORBIT_OUT_F32, dy->dtype == ORBIT_OUT_F32, info.cus, (hipStream_t)stream);
    return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
}

}  // extern "C"
