// C entry points of what surrounds an encoder's layers in training: argument
// checks on the host, then the launchers of norm.hip, dropout.hip, embedding.hip
// and loss.hip.
#include <math.h>

#include "extents.h"
#include "training.h"

using namespace gpic;

namespace {

constexpr int64_t kMostRows = 2147483647LL;

gpic_status check_sides(int64_t n, int64_t cols, const char *name, int32_t dtype)
{
    CHECK_ARG(dtype >= GPIC_F32 && dtype <= GPIC_BF16, "dtype %d is not F32 (0), F16 (1) or BF16 (2)",
              dtype);
    CHECK_ARG(n >= 0 && n <= kMostRows, "n = %lld out of range [0, 2^31-1]", (long long)n);
    CHECK_ARG(cols >= 1 && cols <= kMaxSide, "%s = %lld out of range [1, 2^20]", name,
              (long long)cols);
    return GPIC_OK;
}

gpic_status check_pitch(int64_t ld, int64_t cols, const char *name)
{
    CHECK_ARG(ld >= cols && ld <= kMaxPitch, "%s = %lld not in [%lld, 2^22]", name, (long long)ld,
              (long long)cols);
    return GPIC_OK;
}

gpic_status check_norm(const gpic_norm_params *p)
{
    CHECK_ARG(p != nullptr, "params is null");
    CHECK(check_sides(p->n, p->k, "k", p->dtype));
    CHECK(check_pitch(p->ldx, p->k, "ldx"));
    CHECK(check_pitch(p->ldy, p->k, "ldy"));
    CHECK_ARG(isfinite(p->eps) && p->eps >= 0.0f, "eps must be finite and >= 0");
    return GPIC_OK;
}

Norm norm_of(const gpic_norm_params *p)
{
    return Norm{p->n, p->k, p->ldx, p->ldy, p->eps, p->dtype};
}

gpic_status check_stats(const float *stats, bool nullable)
{
    CHECK_ARG(stats != nullptr || nullable, "stats is null");
    CHECK_ARG(aligned(stats, 8), "stats is not 8-byte aligned");
    return GPIC_OK;
}

// 2^16 p, rounded: a value stays where its bits are at least this
uint32_t limit_of(double p) { return (uint32_t)floor(p * 65536.0 + 0.5); }

gpic_status check_dropout(const gpic_dropout_params *p, bool residual)
{
    CHECK_ARG(p != nullptr, "params is null");
    CHECK(check_sides(p->n, p->m, "m", p->dtype));
    CHECK(check_pitch(p->ldx, p->m, "ldx"));
    CHECK(check_pitch(p->ldy, p->m, "ldy"));
    if (residual)
        CHECK(check_pitch(p->ldr, p->m, "ldr"));
    CHECK_ARG(p->p >= 0.0 && p->p <= 1.0 && limit_of(p->p) < 65536,
              "p = %g not in [0, 1 - 2^-17)", p->p);
    CHECK_ARG(p->reserved == 0, "reserved must be 0");
    return GPIC_OK;
}

gpic_status check_embedding(const gpic_embedding_params *p)
{
    CHECK_ARG(p != nullptr, "params is null");
    CHECK(check_sides(p->n, p->k, "k", p->dtype));
    CHECK_ARG(p->rows >= 1 && p->rows <= kMostRows, "rows = %lld out of range [1, 2^31-1]",
              (long long)p->rows);
    CHECK(check_pitch(p->ldt, p->k, "ldt"));
    CHECK(check_pitch(p->ldy, p->k, "ldy"));
    CHECK_ARG(isfinite(p->scale), "scale must be finite");
    CHECK_ARG(p->id_bytes == 4 || p->id_bytes == 8, "id_bytes must be 4 or 8");
    CHECK_ARG(p->accumulate == 0 || p->accumulate == 1, "accumulate must be 0 or 1");
    return GPIC_OK;
}

Embedding embedding_of(const gpic_embedding_params *p)
{
    return Embedding{p->n,     p->k,     p->rows,          p->ldt,
                     p->ldy,   p->scale, p->dtype,         p->id_bytes == 8,
                     p->accumulate != 0};
}

gpic_status check_gradient_fits(const gpic_embedding_params *p)
{
    if (!embedding_fits(embedding_of(p)))
        return fail(GPIC_ERR_UNSUPPORTED, "n = %lld, k = %lld: a gradient of more workgroups than "
                    "a launch takes", (long long)p->n, (long long)p->k);
    return GPIC_OK;
}

gpic_status check_ids(const void *ids, const char *name, int32_t bytes, bool nullable)
{
    CHECK_ARG(ids != nullptr || nullable, "%s is null", name);
    CHECK_ARG(aligned(ids, bytes), "%s is misaligned", name);
    return GPIC_OK;
}

Loss loss_of(const gpic_loss_params *p)
{
    return Loss{p->n,   p->k,     p->v,             p->ldx,
                p->ldw, p->dtype, p->id_bytes == 8, p->aligned16 != 0};
}

gpic_status check_loss(const gpic_loss_params *p, bool backward)
{
    CHECK_ARG(p != nullptr, "params is null");
    CHECK(check_sides(p->n, p->k, "k", p->dtype));
    CHECK_ARG(p->v >= 1 && p->v <= kMaxSide, "v = %lld out of range [1, 2^20]", (long long)p->v);
    CHECK(check_pitch(p->ldx, p->k, "ldx"));
    CHECK(check_pitch(p->ldw, p->k, "ldw"));
    CHECK_ARG(p->id_bytes == 4 || p->id_bytes == 8, "id_bytes must be 4 or 8");
    CHECK_ARG(p->aligned16 == 0 || p->aligned16 == 1, "aligned16 must be 0 or 1");
    CHECK_ARG(p->reserved == 0, "reserved must be 0");
    if (!loss_fits(loss_of(p), backward))
        return fail(GPIC_ERR_UNSUPPORTED, "n = %lld, k = %lld, v = %lld: a product of more "
                    "workgroups than a launch takes", (long long)p->n, (long long)p->k,
                    (long long)p->v);
    return GPIC_OK;
}

gpic_status check_floats(const float *x, const char *name, bool nullable)
{
    return check_matrix(x, name, GPIC_F32, nullable);
}

} // namespace

extern "C" {

gpic_status gpic_layer_norm(const gpic_norm_params *p, const void *X, const void *weight,
                            const void *bias, void *Y, float *stats, void *stream)
{
    CHECK(check_norm(p));
    const bool empty = p->n == 0;
    CHECK(check_matrix(X, "X", p->dtype, empty));
    CHECK(check_matrix(weight, "weight", p->dtype, true));
    CHECK(check_matrix(bias, "bias", p->dtype, true));
    CHECK(check_matrix(Y, "Y", p->dtype, empty));
    CHECK(check_stats(stats, true));
    const size_t e = size_of(p->dtype);
    const bool in_place = X == Y && (p->ldx == p->ldy || p->n == 1);
    const Extent out[] = {matrix("Y", Y, p->n, p->k, p->ldy, e), packed("stats", stats, p->n, 8)};
    const Extent in[] = {packed("weight", weight, p->k, e), packed("bias", bias, p->k, e),
                         matrix("X", in_place ? nullptr : X, p->n, p->k, p->ldx, e)};
    CHECK(check_apart(out, 2, in, 3));
    CHECK_HIP(run_norm(norm_of(p), X, weight, bias, Y, stats, (hipStream_t)stream), "layer norm");
    return GPIC_OK;
}

size_t gpic_layer_norm_workspace_bytes(const gpic_norm_params *p)
{
    return check_norm(p) == GPIC_OK ? norm_ws(norm_of(p)) : 0;
}

gpic_status gpic_layer_norm_backward(const gpic_norm_params *p, const void *dY, const void *X,
                                     const void *weight, const float *stats, void *dX, void *dW,
                                     void *db, void *ws, size_t ws_bytes, void *stream)
{
    CHECK(check_norm(p));
    const bool empty = p->n == 0;
    CHECK(check_matrix(dY, "dY", p->dtype, empty));
    CHECK(check_matrix(X, "X", p->dtype, empty));
    CHECK(check_matrix(weight, "weight", p->dtype, true));
    CHECK(check_stats(stats, empty));
    CHECK(check_matrix(dX, "dX", p->dtype, true));
    CHECK(check_matrix(dW, "dW", p->dtype, true));
    CHECK(check_matrix(db, "db", p->dtype, true));
    CHECK(check_ws(ws, ws_bytes, norm_ws(norm_of(p))));
    const size_t e = size_of(p->dtype);
    const Extent out[] = {packed("dX", dX, p->n * p->k, e), packed("dW", dW, p->k, e),
                          packed("db", db, p->k, e)};
    const Extent in[] = {matrix("dY", dY, p->n, p->k, p->ldy, e),
                         matrix("X", X, p->n, p->k, p->ldx, e), packed("weight", weight, p->k, e),
                         packed("stats", stats, p->n, 8)};
    CHECK(check_apart(out, 3, in, 4));
    CHECK_HIP(run_norm_backward(norm_of(p), dY, X, weight, stats, dX, dW, db, ws,
                                (hipStream_t)stream),
              "layer norm backward");
    return GPIC_OK;
}

gpic_status gpic_dropout(const gpic_dropout_params *p, const void *X, const void *residual,
                         const int64_t *step, void *Y, void *stream)
{
    CHECK(check_dropout(p, residual != nullptr));
    const bool empty = p->n == 0;
    CHECK(check_matrix(X, "X", p->dtype, empty));
    CHECK(check_matrix(residual, "residual", p->dtype, true));
    CHECK(check_matrix(Y, "Y", p->dtype, empty));
    CHECK_ARG(aligned(step, 8), "step is misaligned");
    const size_t e = size_of(p->dtype);
    const bool over_x = X == Y && (p->ldx == p->ldy || p->n == 1);
    const bool over_r = residual == Y && (p->ldr == p->ldy || p->n == 1);
    const Extent out = matrix("Y", Y, p->n, p->m, p->ldy, e);
    const Extent in[] = {matrix("X", over_x ? nullptr : X, p->n, p->m, p->ldx, e),
                         matrix("the residual", over_r ? nullptr : residual, p->n, p->m, p->ldr, e),
                         packed("step", step, 1, 8)};
    CHECK(check_apart(&out, 1, in, 3));
    const Dropout d{p->n,    p->m,      p->ldx,         p->ldr,  p->ldy,
                    p->seed, p->offset, limit_of(p->p), p->dtype};
    CHECK_HIP(run_dropout(d, X, residual, step, Y, (hipStream_t)stream), "dropout");
    return GPIC_OK;
}

gpic_status gpic_embedding(const gpic_embedding_params *p, const void *ids, const void *T, void *Y,
                           void *stream)
{
    CHECK(check_embedding(p));
    const bool empty = p->n == 0;
    CHECK(check_ids(ids, "ids", p->id_bytes, empty));
    CHECK(check_matrix(T, "T", p->dtype, empty));
    CHECK(check_matrix(Y, "Y", p->dtype, empty));
    const size_t e = size_of(p->dtype);
    const Extent out = matrix("Y", Y, p->n, p->k, p->ldy, e);
    const Extent in[] = {matrix("T", T, p->rows, p->k, p->ldt, e),
                         packed("ids", ids, p->n, p->id_bytes)};
    CHECK(check_apart(&out, 1, in, 2));
    CHECK_HIP(run_embedding(embedding_of(p), ids, T, Y, (hipStream_t)stream), "embedding");
    return GPIC_OK;
}

size_t gpic_embedding_workspace_bytes(const gpic_embedding_params *p)
{
    if (check_embedding(p) != GPIC_OK || check_gradient_fits(p) != GPIC_OK)
        return 0;
    return embedding_ws(embedding_of(p));
}

gpic_status gpic_embedding_backward(const gpic_embedding_params *p, const void *dY,
                                    const void *ids, void *dT, void *ws, size_t ws_bytes,
                                    void *stream)
{
    CHECK(check_embedding(p));
    CHECK(check_gradient_fits(p));
    const bool empty = p->n == 0;
    CHECK(check_matrix(dY, "dY", p->dtype, empty));
    CHECK(check_ids(ids, "ids", p->id_bytes, empty));
    CHECK(check_matrix(dT, "dT", p->dtype, false));
    CHECK(check_ws(ws, ws_bytes, embedding_ws(embedding_of(p))));
    const size_t e = size_of(p->dtype);
    const Extent out = matrix("dT", dT, p->rows, p->k, p->ldt, e);
    const Extent in[] = {matrix("dY", dY, p->n, p->k, p->ldy, e),
                         packed("ids", ids, p->n, p->id_bytes)};
    CHECK(check_apart(&out, 1, in, 2));
    CHECK_HIP(run_embedding_backward(embedding_of(p), dY, ids, dT, ws, (hipStream_t)stream),
              "embedding backward");
    return GPIC_OK;
}

size_t gpic_cross_entropy_workspace_bytes(int32_t backward, const gpic_loss_params *p)
{
    if (backward != 0 && backward != 1)
        return 0;
    return check_loss(p, backward != 0) == GPIC_OK ? loss_ws(loss_of(p), backward != 0) : 0;
}

gpic_status gpic_cross_entropy(const gpic_loss_params *p, const void *X, const void *W,
                               const void *bias, const void *targets, float *loss, float *lse,
                               void *ws, size_t ws_bytes, void *stream)
{
    CHECK(check_loss(p, false));
    const bool empty = p->n == 0, a16 = p->aligned16 != 0;
    CHECK(check_matrix(X, "X", p->dtype, empty, a16));
    CHECK(check_matrix(W, "W", p->dtype, false, a16));
    CHECK(check_matrix(bias, "bias", p->dtype, true));
    CHECK(check_ids(targets, "targets", p->id_bytes, empty));
    CHECK(check_floats(loss, "loss", empty));
    CHECK(check_floats(lse, "lse", true));
    CHECK(check_ws(ws, ws_bytes, loss_ws(loss_of(p), false)));
    const size_t e = size_of(p->dtype);
    const Extent out[] = {packed("loss", loss, p->n, 4), packed("lse", lse, p->n, 4)};
    const Extent in[] = {matrix("X", X, p->n, p->k, p->ldx, e),
                         matrix("W", W, p->v, p->k, p->ldw, e), packed("bias", bias, p->v, e),
                         packed("targets", targets, p->n, p->id_bytes)};
    CHECK(check_apart(out, 2, in, 4));
    CHECK_HIP(run_loss(loss_of(p), X, W, bias, targets, loss, lse, ws, (hipStream_t)stream),
              "cross entropy");
    return GPIC_OK;
}

gpic_status gpic_cross_entropy_backward(const gpic_loss_params *p, const float *dloss,
                                        const void *X, const void *W, const void *bias,
                                        const void *targets, const float *loss, const float *lse,
                                        void *dX, void *dW, void *db, void *ws, size_t ws_bytes,
                                        void *stream)
{
    CHECK(check_loss(p, true));
    const bool empty = p->n == 0, a16 = p->aligned16 != 0;
    CHECK(check_floats(dloss, "dloss", empty));
    CHECK(check_matrix(X, "X", p->dtype, empty, a16));
    CHECK(check_matrix(W, "W", p->dtype, empty, a16));
    CHECK(check_matrix(bias, "bias", p->dtype, true));
    CHECK(check_ids(targets, "targets", p->id_bytes, empty));
    CHECK(check_floats(loss, "loss", empty));
    CHECK(check_floats(lse, "lse", empty));
    CHECK(check_matrix(dX, "dX", p->dtype, true));
    CHECK(check_matrix(dW, "dW", p->dtype, true));
    CHECK(check_matrix(db, "db", p->dtype, true));
    CHECK(check_ws(ws, ws_bytes, loss_ws(loss_of(p), true)));
    const size_t e = size_of(p->dtype);
    const Extent out[] = {packed("dX", dX, p->n * p->k, e), packed("dW", dW, p->v * p->k, e),
                          packed("db", db, p->v, e)};
    const Extent in[] = {packed("dloss", dloss, p->n, 4), matrix("X", X, p->n, p->k, p->ldx, e),
                         matrix("W", W, p->v, p->k, p->ldw, e), packed("bias", bias, p->v, e),
                         packed("targets", targets, p->n, p->id_bytes),
                         packed("loss", loss, p->n, 4), packed("lse", lse, p->n, 4)};
    CHECK(check_apart(out, 3, in, 7));
    CHECK_HIP(run_loss_backward(loss_of(p), dloss, X, W, bias, targets, loss, lse, dX, dW, db, ws,
                                (hipStream_t)stream),
              "cross entropy backward");
    return GPIC_OK;
}

} // extern "C"
