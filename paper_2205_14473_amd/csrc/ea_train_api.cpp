// ea_train_api.cpp -- the C ABI of the operators beside the round (declared in
// include/ea_train.h): argument checks and the tables that the launches carry.
// No entry point allocates memory or synchronizes.
#include "ea_train.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "ea_train.hpp"

namespace {

// Errors share the round's text: ea_last_error() gives the calling thread's
// buffer (512 bytes, not const where it is defined), of which these calls write
// the first half at most.
constexpr size_t kErrorBytes = 256;

__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(const_cast<char*>(ea_last_error()), kErrorBytes, fmt, ap);
    va_end(ap);
    return code;
}

int hip_status(hipError_t e, const char* what)
{
    if (e != hipSuccess) return fail(EA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    const_cast<char*>(ea_last_error())[0] = '\0';
    return EA_OK;
}

int check_t(int64_t t)
{
    if (t < 1 || t > (int64_t)0xFFFFFFFFLL) return fail(EA_ERR_ARG, "t must be in [1, 2^32-1] (got %lld)", (long long)t);
    return EA_OK;
}

struct PtrCheck {
    int rc = EA_OK;
    void need(const void* ptr, bool required, uintptr_t align, const char* name)
    {
        if (rc) return;
        if (!ptr) {
            if (required) rc = fail(EA_ERR_ARG, "%s is NULL", name);
            return;
        }
        if ((uintptr_t)ptr % align) rc = fail(EA_ERR_ALIGN, "%s is not %u-byte aligned", name, (unsigned)align);
    }
};

bool known_type(int32_t type)
{
    return type == EA_F32 || type == EA_BF16 || type == EA_F16;
}

uintptr_t type_bytes(int32_t type)
{
    return type == EA_F32 ? 4 : 2;
}

constexpr int64_t kMostElements = (int64_t)1 << 40;

// The list itself and each tensor's element count; `total` gets their sum.
int check_list(int32_t ntensors, const ea_tensor_t* tensors, int64_t* total)
{
    if (ntensors < 0) return fail(EA_ERR_ARG, "ntensors must be >= 0 (got %d)", ntensors);
    if (ntensors > ea::kMostTensors) return fail(EA_ERR_UNSUPPORTED, "more than 2^22 tensors in one call");
    if (ntensors > 0 && !tensors) return fail(EA_ERR_ARG, "tensors is NULL");
    *total = 0;
    for (int32_t i = 0; i < ntensors; ++i) {
        if (tensors[i].n < 0 || tensors[i].n >= kMostElements)
            return fail(EA_ERR_ARG, "tensor %d: n must be in [0, 2^40) (got %lld)", i, (long long)tensors[i].n);
        *total += tensors[i].n;
        if (*total >= kMostElements) return fail(EA_ERR_UNSUPPORTED, "2^40 elements or more in one call");
    }
    return EA_OK;
}

int need(const void* ptr, bool required, uintptr_t align, int32_t i, const char* name)
{
    if (!ptr) return required ? fail(EA_ERR_ARG, "tensor %d: %s is NULL", i, name) : EA_OK;
    if ((uintptr_t)ptr % align)
        return fail(EA_ERR_ALIGN, "tensor %d: %s is not %u-byte aligned", i, name, (unsigned)align);
    return EA_OK;
}

int check_adamw(const ea_adamw_t* c, int32_t ntensors, const ea_tensor_t* tensors, const float* gscale, int64_t* total)
{
    if (!c) return fail(EA_ERR_ARG, "config is NULL");
    if (!std::isfinite(c->lr) || c->lr < 0.0f) return fail(EA_ERR_ARG, "lr must be finite and >= 0");
    if (!(c->beta1 >= 0.0f && c->beta1 < 1.0f)) return fail(EA_ERR_ARG, "beta1 must be in [0, 1)");
    if (!(c->beta2 >= 0.0f && c->beta2 < 1.0f)) return fail(EA_ERR_ARG, "beta2 must be in [0, 1)");
    if (!std::isfinite(c->eps) || !(c->eps > 0.0f)) return fail(EA_ERR_ARG, "eps must be finite and > 0");
    if (!known_type(c->param_type)) return fail(EA_ERR_ARG, "unknown param_type %d", c->param_type);
    if (!known_type(c->grad_type)) return fail(EA_ERR_ARG, "unknown grad_type %d", c->grad_type);
    if (c->state_bits != 32 && c->state_bits != 8)
        return fail(EA_ERR_ARG, "state_bits must be 32 or 8 (got %d)", c->state_bits);
    if (c->rounding != EA_ROUND_NEAREST && c->rounding != EA_ROUND_STOCHASTIC)
        return fail(EA_ERR_ARG, "unknown rounding %d", c->rounding);
    if (c->state_bits == 32 && c->rounding != EA_ROUND_NEAREST)
        return fail(EA_ERR_ARG, "stochastic rounding is of the 8-bit states");
    int rc = check_list(ntensors, tensors, total);
    if (rc) return rc;
    const bool eight = c->state_bits == 8;
    const uintptr_t state = eight ? 1 : 4;
    for (int32_t i = 0; i < ntensors; ++i) {
        const ea_tensor_t& e = tensors[i];
        if (!std::isfinite(e.weight_decay) || e.weight_decay < 0.0f)
            return fail(EA_ERR_ARG, "tensor %d: weight_decay must be finite and >= 0", i);
        if (!std::isfinite(e.lr_scale) || e.lr_scale < 0.0f)
            return fail(EA_ERR_ARG, "tensor %d: lr_scale must be finite and >= 0", i);
        if (e.n == 0) continue;
        if ((rc = need(e.g, true, type_bytes(c->grad_type), i, "g"))) return rc;
        if ((rc = need(e.p, true, type_bytes(c->param_type), i, "p"))) return rc;
        if ((rc = need(e.m, true, state, i, "m"))) return rc;
        if ((rc = need(e.v, true, state, i, "v"))) return rc;
        if (eight && (rc = need(e.m_scale, true, 4, i, "m_scale"))) return rc;
        if (eight && (rc = need(e.v_scale, true, 4, i, "v_scale"))) return rc;
        if (e.master && c->param_type == EA_F32) return fail(EA_ERR_ARG, "tensor %d: a binary32 p has no master", i);
        if ((rc = need(e.master, false, 4, i, "master"))) return rc;
    }
    if (gscale && ((uintptr_t)gscale & 3u)) return fail(EA_ERR_ALIGN, "gscale is not 4-byte aligned");
    return EA_OK;
}

// `elements` of an array past ptr, for arrays of `bytes` an element.
template <class T>
T* past(T* ptr, int64_t elements, int64_t bytes)
{
    return ptr ? (T*)((uintptr_t)ptr + (uintptr_t)(elements * bytes)) : nullptr;
}

void set_scales(ea::Part32&, const ea_tensor_t&, int32_t, int64_t) {}

void set_scales(ea::Part8& p, const ea_tensor_t& e, int32_t i, int64_t at)
{
    p.m_scale = past(e.m_scale, at / EA_STATE_BLOCK, 4);
    p.v_scale = past(e.v_scale, at / EA_STATE_BLOCK, 4);
    p.place = ((uint32_t)i << ea::kPieceBits) | (uint32_t)(at / ea::kPartElements);
}

// The step over a checked list: launches of as many parts as a table holds.
template <class Args>
hipError_t adamw_launches(const ea_adamw_t& c, const ea_schedule_t* s, int64_t t, uint32_t* t_dev, int32_t ntensors,
                          const ea_tensor_t* tensors, int64_t total, const float* gscale, hipStream_t st)
{
    Args a{};
    a.lr = c.lr;
    a.beta1 = c.beta1;
    a.beta2 = c.beta2;
    a.eps = c.eps;
    a.t = (uint32_t)t;
    a.k0 = (uint32_t)c.seed;
    a.k1 = (uint32_t)(c.seed >> 32);
    a.gscale = gscale;
    a.t_dev = t_dev;
    if (!t_dev) a.root = ea::adamw_root(c.beta2, a.t);
    if (s) a.sched = *s;
    bool masters = false;
    for (int32_t i = 0; i < ntensors; ++i) masters |= tensors[i].master != nullptr;
    a.chunk = ea::adamw_chunk(c, total, masters);
    const int64_t state = c.state_bits / 8;
    const int64_t gb = (int64_t)type_bytes(c.grad_type), pb = (int64_t)type_bytes(c.param_type);
    hipError_t e = hipSuccess;
    for (int32_t i = 0; i < ntensors; ++i) {
        float keep = tensors[i].weight_decay, step = tensors[i].lr_scale;
        if (!t_dev) {
            const double lri = (double)c.lr * (double)step;
            keep = ea::adamw_keep(lri, tensors[i].weight_decay);
            step = ea::adamw_step_size(lri, c.beta1, a.t);
        }
        for (int64_t at = 0; at < tensors[i].n; at += ea::kPartElements) {
            const int64_t left = tensors[i].n - at, n = left < ea::kPartElements ? left : ea::kPartElements;
            const uint32_t groups = (uint32_t)((n + a.chunk - 1) / a.chunk);
            if (a.count == Args::kMost || a.first[a.count] + groups > ea::kMostGroups) {
                if ((e = ea::launch_adamw(a, c, st)) != hipSuccess) return e;
                a.count = 0;
            }
            auto& p = a.part[a.count];
            p.g = past(tensors[i].g, at, gb);
            p.p = past(tensors[i].p, at, pb);
            p.m = past(tensors[i].m, at, state);
            p.v = past(tensors[i].v, at, state);
            p.master = past(tensors[i].master, at, 4);
            p.n = (uint32_t)n;
            p.keep = keep;
            p.step = step;
            set_scales(p, tensors[i], i, at);
            a.first[a.count + 1] = a.first[a.count] + groups;
            ++a.count;
        }
    }
    return ea::launch_adamw(a, c, st);
}

int adamw_impl(const char* name, const ea_adamw_t* c, const ea_schedule_t* s, int64_t t, uint32_t* t_dev,
               int32_t ntensors, const ea_tensor_t* tensors, const float* gscale, void* stream)
{
    int64_t total = 0;
    const int rc = check_adamw(c, ntensors, tensors, gscale, &total);
    if (rc) return rc;
    const hipStream_t st = (hipStream_t)stream;
    hipError_t e = c->state_bits == 8
                       ? adamw_launches<ea::Adamw8Args>(*c, s, t, t_dev, ntensors, tensors, total, gscale, st)
                       : adamw_launches<ea::Adamw32Args>(*c, s, t, t_dev, ntensors, tensors, total, gscale, st);
    if (e == hipSuccess && t_dev) e = ea::launch_advance(t_dev, st);
    return hip_status(e, name);
}

// Workgroups of the norm over these tensors.
int64_t norm_groups(int32_t ntensors, const ea_tensor_t* tensors, int64_t chunk)
{
    int64_t groups = 0;
    for (int32_t i = 0; i < ntensors; ++i) groups += (tensors[i].n + chunk - 1) / chunk;
    return groups;
}

int check_embed(const ea_embed_t* c)
{
    if (!c) return fail(EA_ERR_ARG, "config is NULL");
    if (c->tokens < 0 || c->tokens >= (int64_t)1 << 30)
        return fail(EA_ERR_ARG, "tokens must be in [0, 2^30) (got %lld)", (long long)c->tokens);
    if (c->vocab < 1 || c->vocab >= ((int64_t)1 << 31) - 1)
        return fail(EA_ERR_ARG, "vocab must be in [1, 2^31 - 1) (got %lld)", (long long)c->vocab);
    if (c->dim < 1 || c->dim > (int64_t)1 << 20)
        return fail(EA_ERR_ARG, "dim must be in [1, 2^20] (got %lld)", (long long)c->dim);
    if (c->table_stride < c->dim || c->table_stride >= ((int64_t)1 << 32))
        return fail(EA_ERR_ARG, "table_stride must be in [dim, 2^32) (got %lld)", (long long)c->table_stride);
    if (c->x_stride < c->dim || c->x_stride >= ((int64_t)1 << 32))
        return fail(EA_ERR_ARG, "x_stride must be in [dim, 2^32) (got %lld)", (long long)c->x_stride);
    if (!std::isfinite(c->scale)) return fail(EA_ERR_ARG, "scale must be finite");
    if (!known_type(c->table_type)) return fail(EA_ERR_ARG, "unknown table_type %d", c->table_type);
    if (!known_type(c->x_type)) return fail(EA_ERR_ARG, "unknown x_type %d", c->x_type);
    if (c->index_bits != 32 && c->index_bits != 64)
        return fail(EA_ERR_ARG, "index_bits must be 32 or 64 (got %d)", c->index_bits);
    return EA_OK;
}

}  // namespace

extern "C" {

int ea_adamw_step(const ea_adamw_t* c, int64_t t, int32_t ntensors, const ea_tensor_t* tensors, const float* gscale,
                  void* stream)
{
    const int rc = check_t(t);
    if (rc) return rc;
    return adamw_impl("ea_adamw_step", c, nullptr, t, nullptr, ntensors, tensors, gscale, stream);
}

int ea_adamw_step_scheduled(const ea_adamw_t* c, const ea_schedule_t* s, uint32_t* t_dev, int32_t ntensors,
                            const ea_tensor_t* tensors, const float* gscale, void* stream)
{
    // the schedule's own checks, and its beta2 (the same at every step)
    ea_config_t at{};
    float lr = 0.0f, beta2 = 0.0f;
    const int rc = ea_schedule_at(&at, s, 1, &lr, &beta2);
    if (rc) return rc;
    if (!(beta2 < 1.0f)) return fail(EA_ERR_ARG, "schedule theta / T is too small: beta2 rounds to 1");
    if (!t_dev || ((uintptr_t)t_dev & 3u)) return fail(EA_ERR_ALIGN, "t_dev must be a 4-byte aligned device pointer");
    return adamw_impl("ea_adamw_step_scheduled", c, s, 1, t_dev, ntensors, tensors, gscale, stream);
}

int64_t ea_grad_norm_workspace_bytes(int32_t ntensors, const ea_tensor_t* tensors)
{
    int64_t total = 0;
    const int rc = check_list(ntensors, tensors, &total);
    if (rc) return rc;
    return norm_groups(ntensors, tensors, ea::norm_chunk(total)) * 8;
}

int ea_grad_norm(int32_t grad_type, int32_t ntensors, const ea_tensor_t* tensors, float scale, float max_norm,
                 float* norm, float* gscale, void* workspace, void* stream)
{
    if (!known_type(grad_type)) return fail(EA_ERR_ARG, "unknown grad_type %d", grad_type);
    if (!std::isfinite(scale) || !(scale > 0.0f)) return fail(EA_ERR_ARG, "scale must be finite and > 0");
    if (!(max_norm > 0.0f)) return fail(EA_ERR_ARG, "max_norm must be > 0");
    int64_t total = 0;
    int rc = check_list(ntensors, tensors, &total);
    if (rc) return rc;
    for (int32_t i = 0; i < ntensors; ++i)
        if (tensors[i].n > 0 && (rc = need(tensors[i].g, true, type_bytes(grad_type), i, "g"))) return rc;
    ea::NormArgs a{};
    a.chunk = ea::norm_chunk(total);
    const int64_t groups = norm_groups(ntensors, tensors, a.chunk);
    PtrCheck pc;
    pc.need(norm, true, 4, "norm");
    pc.need(gscale, false, 4, "gscale");
    pc.need(workspace, groups > 0, 8, "workspace");
    if (pc.rc) return pc.rc;
    const hipStream_t st = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    bool flushed = false;
    a.sums = (double*)workspace;
    for (int32_t i = 0; i < ntensors && e == hipSuccess; ++i) {
        if (tensors[i].n == 0) continue;
        if (a.count == ea::kNormParts) {
            e = ea::launch_norm(a, grad_type, st);
            a.sums += a.first[a.count];
            a.count = 0;
            flushed = true;
            if (e != hipSuccess) break;
        }
        a.part[a.count].g = tensors[i].g;
        a.part[a.count].n = tensors[i].n;
        a.first[a.count + 1] = a.first[a.count] + (uint32_t)((tensors[i].n + a.chunk - 1) / a.chunk);
        ++a.count;
    }
    if (e == hipSuccess && !flushed && ea::norm_in_one(a, total)) {
        e = ea::launch_norm_small(a, grad_type, scale, max_norm, norm, gscale, st);
    } else if (e == hipSuccess) {
        e = ea::launch_norm(a, grad_type, st);
        if (e == hipSuccess)
            e = ea::launch_norm_finish((const double*)workspace, groups, scale, max_norm, norm, gscale, st);
    }
    return hip_status(e, "ea_grad_norm");
}

int ea_embed_lookup(const ea_embed_t* c, const void* table, const void* ids, void* x, void* stream)
{
    const int rc = check_embed(c);
    if (rc) return rc;
    PtrCheck pc;
    pc.need(table, c->tokens > 0, type_bytes(c->table_type), "table");
    pc.need(ids, c->tokens > 0, (uintptr_t)c->index_bits / 8, "ids");
    pc.need(x, c->tokens > 0, type_bytes(c->x_type), "x");
    if (pc.rc) return pc.rc;
    return hip_status(ea::launch_embed_lookup(*c, table, ids, x, (hipStream_t)stream), "ea_embed_lookup");
}

int64_t ea_embed_workspace_bytes(const ea_embed_t* c)
{
    const int rc = check_embed(c);
    if (rc) return rc;
    return ea::embed_workspace_bytes(*c);
}

int ea_embed_grad(const ea_embed_t* c, const void* ids, const void* dx, void* dtable, int32_t accumulate,
                  void* workspace, void* stream)
{
    const int rc = check_embed(c);
    if (rc) return rc;
    if (accumulate != 0 && accumulate != 1) return fail(EA_ERR_ARG, "accumulate must be 0 or 1 (got %d)", accumulate);
    PtrCheck pc;
    pc.need(ids, c->tokens > 0, (uintptr_t)c->index_bits / 8, "ids");
    pc.need(dx, c->tokens > 0, type_bytes(c->x_type), "dx");
    pc.need(dtable, true, type_bytes(c->table_type), "dtable");
    pc.need(workspace, ea::embed_workspace_bytes(*c) > 0, 16, "workspace");
    if (pc.rc) return pc.rc;
    return hip_status(ea::launch_embed_grad(*c, ids, dx, dtable, accumulate == 1, workspace, (hipStream_t)stream),
                      "ea_embed_grad");
}

}  // extern "C"
