// ea_layer_api.cpp -- the C ABI of the layers' operators (declared in
// include/ea_layer.h): argument checks.  No entry point allocates memory or
// synchronizes.
#include "ea_layer.h"

#include <cmath>

#include "ea_check.hpp"
#include "ea_layer.hpp"

namespace {

int check_rows(int64_t rows, const char* name)
{
    if (rows < 0 || rows >= (int64_t)1 << 31)
        return fail(EA_ERR_ARG, "%s must be in [0, 2^31) (got %lld)", name, (long long)rows);
    return EA_OK;
}

int check_width(int64_t n, int bits, const char* name)
{
    if (n < 1 || n > (int64_t)1 << bits)
        return fail(EA_ERR_ARG, "%s must be in [1, 2^%d] (got %lld)", name, bits, (long long)n);
    return EA_OK;
}

int check_stride(int64_t stride, int64_t width, const char* name)
{
    if (stride < width || stride >= (int64_t)1 << 32)
        return fail(EA_ERR_ARG, "%s must be at least the row's width and under 2^32 (got %lld)", name, (long long)stride);
    return EA_OK;
}

int check_type(int32_t type, const char* name)
{
    return known_type(type) ? EA_OK : fail(EA_ERR_ARG, "unknown %s %d", name, type);
}

int check_layer_norm(const ea_layer_norm_t* c)
{
    if (!c) return fail(EA_ERR_ARG, "config is NULL");
    int rc;
    if ((rc = check_rows(c->rows, "rows")) || (rc = check_width(c->dim, 20, "dim")) ||
        (rc = check_stride(c->x_stride, c->dim, "x_stride")) || (rc = check_stride(c->y_stride, c->dim, "y_stride")) ||
        (rc = check_type(c->x_type, "x_type")) || (rc = check_type(c->y_type, "y_type")) ||
        (rc = check_type(c->w_type, "w_type")))
        return rc;
    if (!std::isfinite(c->eps) || !(c->eps > 0.0f)) return fail(EA_ERR_ARG, "eps must be finite and > 0");
    return EA_OK;
}

int check_dropout(const ea_dropout_t* c, int64_t t, const uint32_t* t_dev)
{
    if (!c) return fail(EA_ERR_ARG, "config is NULL");
    int rc;
    if ((rc = check_rows(c->rows, "rows")) || (rc = check_width(c->dim, 30, "dim")) ||
        (rc = check_stride(c->x_stride, c->dim, "x_stride")) || (rc = check_stride(c->y_stride, c->dim, "y_stride")) ||
        (rc = check_type(c->x_type, "x_type")) || (rc = check_type(c->y_type, "y_type")))
        return rc;
    if (!(c->p >= 0.0f && c->p <= 1.0f)) return fail(EA_ERR_ARG, "p must be in [0, 1]");
    if (!t_dev && (t < 0 || t > (int64_t)0xFFFFFFFFLL))
        return fail(EA_ERR_ARG, "t must be in [0, 2^32-1] (got %lld)", (long long)t);
    if ((uintptr_t)t_dev & 3u) return fail(EA_ERR_ALIGN, "t_dev is not 4-byte aligned");
    return EA_OK;
}

int check_recurrence(const ea_recurrence_t* c)
{
    if (!c) return fail(EA_ERR_ARG, "config is NULL");
    int rc;
    if ((rc = check_rows(c->batch, "batch")) || (rc = check_rows(c->length, "length")) ||
        (rc = check_width(c->dim, 20, "dim")) || (rc = check_stride(c->x_stride, c->dim, "x_stride")) ||
        (rc = check_stride(c->g_stride, c->dim, "g_stride")) || (rc = check_stride(c->y_stride, c->dim, "y_stride")) ||
        (rc = check_type(c->x_type, "x_type")) || (rc = check_type(c->g_type, "g_type")))
        return rc;
    if (c->gate != EA_GATE_PLAIN && c->gate != EA_GATE_SIGMOID) return fail(EA_ERR_ARG, "unknown gate %d", c->gate);
    if (c->reserved) return fail(EA_ERR_ARG, "reserved must be 0");
    if (c->batch * c->length >= (int64_t)1 << 31) return fail(EA_ERR_UNSUPPORTED, "2^31 rows or more in one call");
    // 64 channels of up to 128 steps of a sequence are a workgroup's: more than memory holds
    if (c->batch * (c->length / 128 + 1) * (c->dim / 64 + 1) >= (int64_t)1 << 31)
        return fail(EA_ERR_UNSUPPORTED, "batch, length and dim are too large for one call");
    return EA_OK;
}

int check_token_loss(const ea_token_loss_t* c)
{
    if (!c) return fail(EA_ERR_ARG, "config is NULL");
    int rc;
    if ((rc = check_rows(c->rows, "rows")) || (rc = check_width(c->vocab, 24, "vocab")) ||
        (rc = check_stride(c->logits_stride, c->vocab, "logits_stride")) ||
        (rc = check_stride(c->dlogits_stride, c->vocab, "dlogits_stride")) || (rc = check_type(c->type, "type")))
        return rc;
    if (!std::isfinite(c->scale)) return fail(EA_ERR_ARG, "scale must be finite");
    if (c->index_bits != 32 && c->index_bits != 64)
        return fail(EA_ERR_ARG, "index_bits must be 32 or 64 (got %d)", c->index_bits);
    if (c->reduction != EA_REDUCE_MEAN && c->reduction != EA_REDUCE_SUM)
        return fail(EA_ERR_ARG, "unknown reduction %d", c->reduction);
    return EA_OK;
}

// Whether `out` may take the place of `in`: it is another array, or the very same rows.
int check_same(const void* out, const void* in, bool alike, const char* names)
{
    return out && out == in && !alike ? fail(EA_ERR_ARG, "%s: one array needs one type and stride", names) : EA_OK;
}

}  // namespace

extern "C" {

int ea_layer_norm(const ea_layer_norm_t* c, const void* x, const void* weight, const void* bias, void* y, float* mean,
                  float* rstd, void* stream)
{
    int rc = check_layer_norm(c);
    if (rc) return rc;
    PtrCheck pc;
    pc.need(x, c->rows > 0, type_bytes(c->x_type), "x");
    pc.need(weight, false, type_bytes(c->w_type), "weight");
    pc.need(bias, false, type_bytes(c->w_type), "bias");
    pc.need(y, c->rows > 0, type_bytes(c->y_type), "y");
    pc.need(mean, false, 4, "mean");
    pc.need(rstd, false, 4, "rstd");
    if (pc.rc) return pc.rc;
    if ((rc = check_same(y, x, c->x_type == c->y_type && c->x_stride == c->y_stride, "y and x"))) return rc;
    return hip_status(ea::launch_layer_norm(*c, x, weight, bias, y, mean, rstd, (hipStream_t)stream), "ea_layer_norm");
}

int64_t ea_layer_norm_workspace_bytes(const ea_layer_norm_t* c)
{
    const int rc = check_layer_norm(c);
    if (rc) return rc;
    return ea::layer_norm_workspace_bytes(*c);
}

int ea_layer_norm_grad(const ea_layer_norm_t* c, const void* x, const void* dy, const void* weight, const float* mean,
                       const float* rstd, const void* add, void* dx, void* dweight, void* dbias, int32_t accumulate,
                       void* workspace, void* stream)
{
    int rc = check_layer_norm(c);
    if (rc) return rc;
    if (accumulate != 0 && accumulate != 1) return fail(EA_ERR_ARG, "accumulate must be 0 or 1 (got %d)", accumulate);
    const bool some = c->rows > 0;
    PtrCheck pc;
    pc.need(x, some, type_bytes(c->x_type), "x");
    pc.need(dy, some, type_bytes(c->y_type), "dy");
    pc.need(weight, false, type_bytes(c->w_type), "weight");
    pc.need(mean, some, 4, "mean");
    pc.need(rstd, some, 4, "rstd");
    pc.need(add, false, type_bytes(c->x_type), "add");
    pc.need(dx, some, type_bytes(c->x_type), "dx");
    pc.need(dweight, false, type_bytes(c->w_type), "dweight");
    pc.need(dbias, false, type_bytes(c->w_type), "dbias");
    pc.need(workspace, (dweight || dbias) && ea::layer_norm_workspace_bytes(*c) > 0, 16, "workspace");
    if (pc.rc) return pc.rc;
    if ((rc = check_same(dx, dy, c->x_type == c->y_type && c->x_stride == c->y_stride, "dx and dy"))) return rc;
    return hip_status(ea::launch_layer_norm_grad(*c, x, dy, weight, mean, rstd, add, dx, dweight, dbias, accumulate == 1,
                                                 workspace, (hipStream_t)stream),
                      "ea_layer_norm_grad");
}

int ea_dropout(const ea_dropout_t* c, int64_t t, const uint32_t* t_dev, const void* x, const void* residual, void* y,
               void* stream)
{
    int rc = check_dropout(c, t, t_dev);
    if (rc) return rc;
    PtrCheck pc;
    pc.need(x, c->rows > 0, type_bytes(c->x_type), "x");
    pc.need(residual, false, type_bytes(c->y_type), "residual");
    pc.need(y, c->rows > 0, type_bytes(c->y_type), "y");
    if (pc.rc) return pc.rc;
    if ((rc = check_same(y, x, c->x_type == c->y_type && c->x_stride == c->y_stride, "y and x"))) return rc;
    return hip_status(ea::launch_dropout(*c, false, (uint32_t)t, t_dev, x, residual, y, (hipStream_t)stream),
                      "ea_dropout");
}

int ea_dropout_grad(const ea_dropout_t* c, int64_t t, const uint32_t* t_dev, const void* dy, void* dx, void* stream)
{
    int rc = check_dropout(c, t, t_dev);
    if (rc) return rc;
    PtrCheck pc;
    pc.need(dy, c->rows > 0, type_bytes(c->y_type), "dy");
    pc.need(dx, c->rows > 0, type_bytes(c->x_type), "dx");
    if (pc.rc) return pc.rc;
    if ((rc = check_same(dx, dy, c->x_type == c->y_type && c->x_stride == c->y_stride, "dx and dy"))) return rc;
    return hip_status(ea::launch_dropout(*c, true, (uint32_t)t, t_dev, dy, nullptr, dx, (hipStream_t)stream),
                      "ea_dropout_grad");
}

int64_t ea_recurrence_states_bytes(const ea_recurrence_t* c)
{
    const int rc = check_recurrence(c);
    if (rc) return rc;
    return c->batch * ((c->length + EA_RECURRENCE_BLOCK - 1) / EA_RECURRENCE_BLOCK) * c->dim * 4;
}

int64_t ea_recurrence_workspace_bytes(const ea_recurrence_t* c)
{
    const int rc = check_recurrence(c);
    if (rc) return rc;
    return ea::recurrence_workspace_bytes(*c);
}

int ea_recurrence(const ea_recurrence_t* c, const void* g, const void* x, const float* h0, const int32_t* lengths,
                  void* y, float* states, float* h_last, void* workspace, void* stream)
{
    const int rc = check_recurrence(c);
    if (rc) return rc;
    const bool some = c->batch * c->length > 0;
    PtrCheck pc;
    pc.need(g, some, type_bytes(c->g_type), "g");
    pc.need(x, some, type_bytes(c->x_type), "x");
    pc.need(h0, false, 4, "h0");
    pc.need(lengths, false, 4, "lengths");
    pc.need(y, some, type_bytes(c->x_type), "y");
    pc.need(states, false, 4, "states");
    pc.need(h_last, false, 4, "h_last");
    pc.need(workspace, ea::recurrence_workspace_bytes(*c) > 0, 16, "workspace");
    if (pc.rc) return pc.rc;
    return hip_status(ea::launch_recurrence(*c, g, x, h0, lengths, y, states, h_last, workspace, (hipStream_t)stream),
                      "ea_recurrence");
}

int ea_recurrence_grad(const ea_recurrence_t* c, const void* g, const void* x, const float* states,
                       const int32_t* lengths, const void* dy, const float* dh_last, void* dg, void* dx, float* dh0,
                       void* workspace, void* stream)
{
    const int rc = check_recurrence(c);
    if (rc) return rc;
    const bool some = c->batch * c->length > 0;
    PtrCheck pc;
    pc.need(g, some, type_bytes(c->g_type), "g");
    pc.need(x, some, type_bytes(c->x_type), "x");
    pc.need(states, some, 4, "states");
    pc.need(lengths, false, 4, "lengths");
    pc.need(dy, some, type_bytes(c->x_type), "dy");
    pc.need(dh_last, false, 4, "dh_last");
    pc.need(dg, some, type_bytes(c->g_type), "dg");
    pc.need(dx, some, type_bytes(c->x_type), "dx");
    pc.need(dh0, false, 4, "dh0");
    pc.need(workspace, ea::recurrence_workspace_bytes(*c) > 0, 16, "workspace");
    if (pc.rc) return pc.rc;
    return hip_status(ea::launch_recurrence_grad(*c, g, x, states, lengths, dy, dh_last, dg, dx, dh0, workspace,
                                                 (hipStream_t)stream),
                      "ea_recurrence_grad");
}

int64_t ea_token_loss_workspace_bytes(const ea_token_loss_t* c)
{
    const int rc = check_token_loss(c);
    if (rc) return rc;
    return ea::token_loss_workspace_bytes(*c);
}

int ea_token_loss(const ea_token_loss_t* c, const void* logits, const void* targets, float* loss, float* total,
                  int32_t* count, void* dlogits, void* workspace, void* stream)
{
    int rc = check_token_loss(c);
    if (rc) return rc;
    const bool some = c->rows > 0;
    PtrCheck pc;
    pc.need(logits, some, type_bytes(c->type), "logits");
    pc.need(targets, some, (uintptr_t)c->index_bits / 8, "targets");
    pc.need(loss, false, 4, "loss");
    pc.need(total, true, 4, "total");
    pc.need(count, false, 4, "count");
    pc.need(dlogits, false, type_bytes(c->type), "dlogits");
    pc.need(workspace, ea::token_loss_workspace_bytes(*c) > 0, 16, "workspace");
    if (pc.rc) return pc.rc;
    if ((rc = check_same(dlogits, logits, c->logits_stride == c->dlogits_stride, "dlogits and logits"))) return rc;
    return hip_status(ea::launch_token_loss(*c, logits, targets, loss, total, count, dlogits, workspace,
                                            (hipStream_t)stream),
                      "ea_token_loss");
}

}  // extern "C"
