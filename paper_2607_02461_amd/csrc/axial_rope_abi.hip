// Entry points of the rotary positions and of the query and key norms: plans, argument checks, launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "abi.h"
#include "device.h"
#include "internal.h"

using namespace orbit;

namespace {

constexpr int32_t kMaxHeads = 1 << 30;        // indices of the heads that a wave's last step has beyond them fit 32 bits too
constexpr int64_t kMaxReach = (int64_t)1 << 50;  // elements from a dimension's first entry to its last: offsets fit 64 bits
constexpr int64_t kMaxTable = (int64_t)1 << 27;  // (cos, sin) pairs of a plan: their byte offsets and indices fit 32 bits

orbit_status rope_upload_dev(orbit_rope p, int dev) {
    std::lock_guard<std::mutex> lk(p->mu);
    if (p->dev_table[dev]) return ORBIT_OK;
    void* d = nullptr;
    const orbit_status st = upload_copy("rope_plan upload", p->table.data(), p->table.size() * sizeof(float), &d);
    p->dev_table[dev] = (float*)d;
    return st;
}

// angle(axis, position, j) fills the tables; the plan's other arguments are checked here.
template <typename F>
orbit_status make_plan(int32_t axes, const int32_t* dims, const int32_t* lengths, int32_t halves, orbit_rope* out, F angle) {
    if (!out) return fail(ORBIT_EINVAL, "rope_plan: out is NULL");
    *out = nullptr;
    if (axes < 1 || axes > kMaxAxes) return fail(ORBIT_EINVAL, "rope_plan: %d axes, 1..%d are possible", axes, kMaxAxes);
    if (!dims || !lengths) return fail(ORBIT_EINVAL, "rope_plan: dims or lengths is NULL");
    if (halves != 0 && halves != 1) return fail(ORBIT_EINVAL, "rope_plan: halves must be 0 or 1");
    int64_t sum = 0, entries = 0;
    for (int a = 0; a < axes; ++a) {
        if (dims[a] < 2 || dims[a] % 2 || dims[a] > kMaxHeadDim)
            return fail(ORBIT_EINVAL, "rope_plan: axis %d has %d values, an even number from 2 to %d is possible", a, dims[a], kMaxHeadDim);
        if (lengths[a] < 1) return fail(ORBIT_EINVAL, "rope_plan: axis %d has %d positions", a, lengths[a]);
        sum += dims[a];
        entries += (int64_t)lengths[a] * (dims[a] / 2);
    }
    if (sum % 8 || sum > kMaxHeadDim)
        return fail(ORBIT_EUNSUPPORTED, "rope_plan: the axes rotate %lld values of a head, a multiple of 8 up to %d is implemented",
                    (long long)sum, kMaxHeadDim);
    if (entries > kMaxTable) return fail(ORBIT_EUNSUPPORTED, "rope_plan: tables of %lld angles exceed %lld", (long long)entries, (long long)kMaxTable);
    orbit_rope p = new (std::nothrow) orbit_rope_s;
    if (!p) return fail(ORBIT_ENOMEM, "rope_plan: out of host memory");
    try {
        p->width.resize(axes);
        p->length.assign(lengths, lengths + axes);
        p->table.resize((size_t)entries * 2);
    } catch (...) {
        delete p;
        return fail(ORBIT_ENOMEM, "rope_plan: out of host memory");
    }
    p->axes = axes;
    p->pairs = (int32_t)(sum / 2);
    p->halves = halves != 0;
    float* at = p->table.data();
    for (int a = 0; a < axes; ++a) {
        p->width[a] = dims[a] / 2;
        for (int64_t i = 0; i < lengths[a]; ++i)
            for (int j = 0; j < dims[a] / 2; ++j, at += 2) {
                const double t = angle(a, i, j);
                if (!std::isfinite(t)) {
                    delete p;
                    return fail(ORBIT_EINVAL, "rope_plan: the angle of axis %d, position %lld, pair %d is not finite", a, (long long)i, j);
                }
                at[0] = (float)std::cos(t);
                at[1] = (float)std::sin(t);
            }
    }
    int dev;
    orbit_status st = device_for_upload(&dev);
    if (st == ORBIT_OK && dev >= 0) st = rope_upload_dev(p, dev);
    if (st != ORBIT_OK) {
        delete p;
        return st;
    }
    *out = p;
    return ORBIT_OK;
}

bool too_far(int64_t entries, int64_t stride) { return entries > 1 && (stride < 0 || stride > kMaxReach / (entries - 1)); }

bool is_type(int32_t t) { return t == ORBIT_OUT_F32 || t == ORBIT_OUT_BF16; }

// Rows of 16-byte groups: pointer and strides (of dimensions with more than one entry) multiples of 16 bytes.
orbit_status check_heads(const char* who, const char* name, const orbit_heads* t, int64_t B, int64_t L, int32_t heads, int32_t dtype,
                         HeadRows* out) {
    if (!t) return fail(ORBIT_EINVAL, "%s: %s is NULL", who, name);
    if (t->heads != heads) return fail(ORBIT_EINVAL, "%s: %s has %d heads, %d expected", who, name, t->heads, heads);
    if (t->dtype != dtype) return fail(ORBIT_EINVAL, "%s: %s has type %d, %d expected", who, name, t->dtype, dtype);
    if (heads < 1) return fail(ORBIT_EINVAL, "%s: %s has %d heads", who, name, heads);
    if (heads > kMaxHeads) return fail(ORBIT_EUNSUPPORTED, "%s: %s has more than %d heads", who, name, kMaxHeads);
    if (B <= 0 || L <= 0) return ORBIT_OK;
    if (!t->data) return fail(ORBIT_EINVAL, "%s: %s is a null device pointer", who, name);
    const int unit = dtype == ORBIT_OUT_F32 ? 4 : 8;
    if (!aligned(t->data, 16) || (B > 1 && t->batch % unit) || (L > 1 && t->token % unit) || (heads > 1 && t->head % unit))
        return fail(ORBIT_EINVAL, "%s: %s must be aligned to 16 bytes, its strides too", who, name);
    if (too_far(B, t->batch) || too_far(L, t->token) || too_far(heads, t->head))
        return fail(ORBIT_EINVAL, "%s: %s has a stride out of range", who, name);
    out->p = t->data;
    out->b = B > 1 ? t->batch : 0;
    out->l = L > 1 ? t->token : 0;
    out->h = heads > 1 ? t->head : 0;
    return ORBIT_OK;
}

// An output at an input's place has to be that input: its type and strides.  `from` may be another tensor's input, which an
// output never replaces.
orbit_status check_in_place(const char* who, const char* name, const HeadRows& y, const HeadRows& from, bool own) {
    if (!y.p || y.p != from.p || (own && y.b == from.b && y.l == from.l && y.h == from.h)) return ORBIT_OK;
    return fail(ORBIT_EINVAL, "%s: %s lies on an input that it does not replace row by row", who, name);
}

// The outputs against all inputs and each other.  Types: of x and y, and of g and y, equal or not.
orbit_status check_places(const char* who, const char* const* names, const RopeParams& p, bool x_type, bool g_type) {
    for (int i = 0; i < p.tensors; ++i)
        for (int j = 0; j < p.tensors; ++j) {
            orbit_status st = check_in_place(who, names[i], p.t[i].y, p.t[j].x, i == j && x_type);
            if (st == ORBIT_OK) st = check_in_place(who, names[i], p.t[i].y, p.t[j].g, i == j && g_type);
            if (st == ORBIT_OK && i != j) st = check_in_place(who, names[i], p.t[i].y, p.t[j].y, false);
            if (st != ORBIT_OK) return st;
        }
    return ORBIT_OK;
}

// Sizes, positions and the plan's tables, checked and written into p.  done: there is nothing to launch.
orbit_status common(const char* who, orbit_rope plan, int64_t B, int64_t L, int64_t D, const int32_t* pos, int64_t pos_batch, int heads,
                    RopeParams* p, DeviceInfo* info, bool* done) {
    *done = false;
    if (B < 0 || L < 0) return fail(ORBIT_EINVAL, "%s: negative B or L", who);
    if (D < 8 || D % 8 || D > kMaxHeadDim)
        return fail(ORBIT_EUNSUPPORTED, "%s: head size %lld, a multiple of 8 up to %d is implemented", who, (long long)D, kMaxHeadDim);
    if (plan && 2 * plan->pairs > D)
        return fail(ORBIT_EINVAL, "%s: the plan rotates %d values, a head has %lld", who, 2 * plan->pairs, (long long)D);
    if (pos_batch < 0 || too_far(B, pos_batch)) return fail(ORBIT_EINVAL, "%s: positions' batch stride out of range", who);
    if (B > INT32_MAX || L > INT32_MAX || B * L > INT32_MAX / heads)
        return fail(ORBIT_EUNSUPPORTED, "%s: more than 2^31 - 1 head rows", who);
    *done = B == 0 || L == 0;
    p->tokens = (uint32_t)(B * L);
    p->L = (uint32_t)L;
    p->D = (int)D;
    p->lanes = 1;
    while (p->lanes * 8 < D) p->lanes *= 2;
    p->inv_d = (float)(1.0 / (double)D);
    p->sign = 1.f;
    if (plan && !*done && (!pos || !aligned(pos, 4))) return fail(ORBIT_EINVAL, "%s: positions are null or misaligned", who);
    int dev;
    orbit_status st = current_device(&dev, info);
    if (st != ORBIT_OK || !plan) return st;
    {
        std::lock_guard<std::mutex> lk(plan->mu);
        p->table = plan->dev_table[dev];
    }
    if (!p->table)
        return fail(ORBIT_EINVAL, "%s: the plan has no tables on device %d: create it with that device current, or call "
                                  "rope_plan_upload there first", who, dev);
    p->pos = pos;
    p->pos_batch = pos_batch;
    p->axes = plan->axes;
    p->pairs = plan->pairs;
    p->halves = plan->halves;
    int first = 0, begin = 0;
    for (int a = 0; a < plan->axes; ++a) {
        p->first[a] = first;
        p->width[a] = plan->width[a];
        p->length[a] = plan->length[a];
        p->base[a] = begin - first;
        first += plan->width[a];
        begin += plan->width[a] * plan->length[a];
    }
    return ORBIT_OK;
}

orbit_status check_weight(const char* who, const void* w, int32_t w_dtype, RopeTensor* t) {
    if (!w) return ORBIT_OK;
    if (!is_type(w_dtype)) return fail(ORBIT_EINVAL, "%s: unknown type %d of the weights", who, w_dtype);
    if (!aligned(w, w_dtype == ORBIT_OUT_F32 ? 4 : 2)) return fail(ORBIT_EINVAL, "%s: misaligned weights", who);
    t->w = w;
    t->w_f32 = w_dtype == ORBIT_OUT_F32;
    return ORBIT_OK;
}

}  // namespace

extern "C" {

orbit_status rope_plan(int32_t axes, const int32_t* dims, const int32_t* lengths, double theta, int32_t halves, orbit_rope* out) {
    clear_error();
    if (!(theta > 0.0) || !std::isfinite(theta)) return fail(ORBIT_EINVAL, "rope_plan: theta must be finite and above 0");
    double freq[kMaxAxes][kMaxHeadDim / 2];
    if (axes >= 1 && axes <= kMaxAxes && dims)
        for (int a = 0; a < axes; ++a)
            for (int j = 0; j < dims[a] / 2 && j < kMaxHeadDim / 2; ++j) freq[a][j] = std::pow(theta, -2.0 * j / dims[a]);
    return make_plan(axes, dims, lengths, halves, out, [&](int a, int64_t i, int j) { return (double)i * freq[a][j]; });
}

orbit_status rope_plan_from_angles(int32_t axes, const int32_t* dims, const int32_t* lengths, const double* angles, int32_t halves,
                                   orbit_rope* out) {
    clear_error();
    if (!angles) return fail(ORBIT_EINVAL, "rope_plan_from_angles: angles is NULL");
    return make_plan(axes, dims, lengths, halves, out, [&](int, int64_t, int) { return *angles++; });
}

orbit_status rope_plan_upload(orbit_rope p) {
    clear_error();
    if (!p) return fail(ORBIT_EINVAL, "rope_plan_upload: plan is NULL");
    int dev;
    DeviceInfo info;
    const orbit_status st = current_device(&dev, &info);
    return st != ORBIT_OK ? st : rope_upload_dev(p, dev);
}

void rope_plan_destroy(orbit_rope p) {
    if (!p) return;
    free_per_device(p->dev_table);
    delete p;
}

orbit_status axial_rope(orbit_rope plan, const orbit_heads* x, const orbit_heads* y, int64_t B, int64_t L, int64_t D,
                        const int32_t* positions, int64_t pos_batch, int32_t inverse, void* stream) {
    const char* who = "axial_rope";
    clear_error();
    if (!plan) return fail(ORBIT_EINVAL, "%s: plan is NULL", who);
    if (!x) return fail(ORBIT_EINVAL, "%s: x is NULL", who);
    if (!is_type(x->dtype)) return fail(ORBIT_EINVAL, "%s: unknown type %d", who, x->dtype);
    if (inverse != 0 && inverse != 1) return fail(ORBIT_EINVAL, "%s: inverse must be 0 or 1", who);
    RopeParams p{};
    DeviceInfo info;
    bool done;
    orbit_status st = check_heads(who, "x", x, B, L, x->heads, x->dtype, &p.t[0].x);
    if (st == ORBIT_OK) st = check_heads(who, "y", y, B, L, x->heads, x->dtype, &p.t[0].y);
    p.tensors = 1;
    p.t[0].heads = x->heads;
    const char* const names[] = {"y"};
    if (st == ORBIT_OK) st = check_places(who, names, p, true, true);
    if (st == ORBIT_OK) st = common(who, plan, B, L, D, positions, pos_batch, x->heads, &p, &info, &done);
    if (st != ORBIT_OK || done) return st;
    p.sign = inverse ? -1.f : 1.f;
    const bool f32 = x->dtype == ORBIT_OUT_F32;
    const hipError_t e = launch_axial_rope(p, false, f32, f32, info.cus, (hipStream_t)stream);
    return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
}

orbit_status qk_norm_rope(orbit_rope plan, const orbit_heads* q, const orbit_heads* k, const orbit_heads* q_out, const orbit_heads* k_out,
                          int64_t B, int64_t L, int64_t D, const int32_t* positions, int64_t pos_batch, const void* q_weight,
                          const void* k_weight, int32_t w_dtype, float eps, void* stream) {
    const char* who = "qk_norm_rope";
    clear_error();
    if (!q || !q_out) return fail(ORBIT_EINVAL, "%s: q or q_out is NULL", who);
    if (!is_type(q->dtype) || !is_type(q_out->dtype)) return fail(ORBIT_EINVAL, "%s: unknown type", who);
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(ORBIT_EINVAL, "%s: eps must be finite and >= 0", who);
    if (!k != !k_out) return fail(ORBIT_EINVAL, "%s: k and k_out must both be given or both be NULL", who);
    if (!k && k_weight) return fail(ORBIT_EINVAL, "%s: a weight for k without k", who);
    const orbit_heads *in[2] = {q, k}, *to[2] = {q_out, k_out};
    const void* w[2] = {q_weight, k_weight};
    RopeParams p{};
    DeviceInfo info;
    bool done;
    int most = 0;
    for (int i = 0; i < 2 && in[i]; ++i) {
        RopeTensor& t = p.t[p.tensors++];
        orbit_status st = check_heads(who, i ? "k" : "q", in[i], B, L, in[i]->heads, q->dtype, &t.x);
        if (st == ORBIT_OK) st = check_heads(who, i ? "k_out" : "q_out", to[i], B, L, in[i]->heads, q_out->dtype, &t.y);
        if (st == ORBIT_OK) st = check_weight(who, w[i], w_dtype, &t);
        if (st != ORBIT_OK) return st;
        t.heads = in[i]->heads;
        most = t.heads > most ? t.heads : most;
    }
    const char* const names[] = {"q_out", "k_out"};
    orbit_status st = check_places(who, names, p, q->dtype == q_out->dtype, true);
    if (st == ORBIT_OK) st = common(who, plan, B, L, D, positions, pos_batch, most, &p, &info, &done);
    if (st != ORBIT_OK || done) return st;
    p.eps = eps;
    const hipError_t e = launch_axial_rope(p, true, q->dtype == ORBIT_OUT_F32, q_out->dtype == ORBIT_OUT_F32, info.cus, (hipStream_t)stream);
    return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
}

orbit_status qk_norm_rope_backward_workspace_size(int64_t D, size_t* bytes) {
    clear_error();
    if (!bytes) return fail(ORBIT_EINVAL, "qk_norm_rope_backward_workspace_size: null output pointer");
    *bytes = 0;
    if (D < 8 || D % 8 || D > kMaxHeadDim)
        return fail(ORBIT_EUNSUPPORTED, "qk_norm_rope_backward_workspace_size: head size %lld, a multiple of 8 up to %d is implemented",
                    (long long)D, kMaxHeadDim);
    int dev;
    DeviceInfo info;
    const orbit_status st = current_device(&dev, &info);
    if (st != ORBIT_OK) return st;
    *bytes = (size_t)2 * norm_rope_backward_groups(info.cus) * (size_t)D * sizeof(float);
    return ORBIT_OK;
}

orbit_status qk_norm_rope_backward(orbit_rope plan, const orbit_heads* dq, const orbit_heads* dk, const orbit_heads* q, const orbit_heads* k,
                                   const orbit_heads* q_grad, const orbit_heads* k_grad, int64_t B, int64_t L, int64_t D,
                                   const int32_t* positions, int64_t pos_batch, const void* q_weight, const void* k_weight, int32_t w_dtype,
                                   float eps, float* q_weight_grad, float* k_weight_grad, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    const char* who = "qk_norm_rope_backward";
    clear_error();
    if (!q || !dq || !q_grad) return fail(ORBIT_EINVAL, "%s: dq, q or q_grad is NULL", who);
    if (!is_type(q->dtype) || !is_type(dq->dtype)) return fail(ORBIT_EINVAL, "%s: unknown type", who);
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(ORBIT_EINVAL, "%s: eps must be finite and >= 0", who);
    if (!k != !dk || !k != !k_grad) return fail(ORBIT_EINVAL, "%s: dk, k and k_grad must all be given or all be NULL", who);
    if (!k && (k_weight || k_weight_grad)) return fail(ORBIT_EINVAL, "%s: a weight for k without k", who);
    const orbit_heads *in[2] = {q, k}, *grad[2] = {dq, dk}, *to[2] = {q_grad, k_grad};
    const void* w[2] = {q_weight, k_weight};
    float* dw[2] = {q_weight_grad, k_weight_grad};
    RopeParams p{};
    DeviceInfo info;
    bool done;
    int most = 0;
    for (int i = 0; i < 2 && in[i]; ++i) {
        RopeTensor& t = p.t[p.tensors++];
        orbit_status st = check_heads(who, i ? "k" : "q", in[i], B, L, in[i]->heads, q->dtype, &t.x);
        if (st == ORBIT_OK) st = check_heads(who, i ? "dk" : "dq", grad[i], B, L, in[i]->heads, dq->dtype, &t.g);
        if (st == ORBIT_OK) st = check_heads(who, i ? "k_grad" : "q_grad", to[i], B, L, in[i]->heads, q->dtype, &t.y);
        if (st == ORBIT_OK) st = check_weight(who, w[i], w_dtype, &t);
        if (st != ORBIT_OK) return st;
        if (dw[i] && (!w[i] || !aligned(dw[i], 4)))
            return fail(ORBIT_EINVAL, "%s: a weight's gradient is asked for without the weight, or is misaligned", who);
        t.heads = in[i]->heads;
        t.dw = dw[i];
        most = t.heads > most ? t.heads : most;
    }
    const char* const names[] = {"q_grad", "k_grad"};
    orbit_status st = check_places(who, names, p, true, q->dtype == dq->dtype);
    if (st == ORBIT_OK) st = common(who, plan, B, L, D, positions, pos_batch, most, &p, &info, &done);
    if (st != ORBIT_OK) return st;
    const size_t part = (size_t)norm_rope_backward_groups(info.cus) * (size_t)D;
    if ((q_weight_grad || k_weight_grad) && (!workspace || !aligned(workspace, 16) || workspace_bytes < 2 * part * sizeof(float)))
        return fail(ORBIT_EINVAL, "%s: weight gradients take a workspace of %zu bytes, aligned to 16", who, 2 * part * sizeof(float));
    for (int i = 0; i < p.tensors; ++i) p.t[i].dw_part = p.t[i].dw ? (float*)workspace + i * part : nullptr;
    p.eps = eps;
    const hipError_t e =
        launch_qk_norm_rope_backward(p, q->dtype == ORBIT_OUT_F32, dq->dtype == ORBIT_OUT_F32, info.cus, (hipStream_t)stream);
    return e == hipSuccess ? ORBIT_OK : hip_fail(e, who);
}

}  // extern "C"
