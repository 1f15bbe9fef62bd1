// C entry points of the encoder operators: argument checks on the host,
// then the launchers of layers.hip and orthogonalize.hip.
#include <math.h>

#include "checks.h"
#include "encoder.h"

using namespace gpic;

namespace {

constexpr int64_t kMaxSide = 1 << 20;      // k, m (2 m), and the sides of an update
constexpr int64_t kMaxPitch = 1 << 22;     // 256 rows of it stay within 32-bit offsets

size_t size_of(int32_t dtype) { return dtype == GPIC_F32 ? 4 : 2; }

gpic_status check_layer(const gpic_layer_params *p, bool gated)
{
    CHECK_ARG(p != nullptr, "params is null");
    CHECK_ARG(p->dtype >= GPIC_F32 && p->dtype <= GPIC_BF16,
              "dtype %d is not F32 (0), F16 (1) or BF16 (2)", p->dtype);
    CHECK_ARG(p->activation >= GPIC_ACT_NONE && p->activation <= GPIC_ACT_SILU,
              "activation %d is not one of GPIC_ACT_*", p->activation);
    CHECK_ARG(p->aligned16 == 0 || p->aligned16 == 1, "aligned16 must be 0 or 1");
    CHECK_ARG(p->reserved == 0, "reserved must be 0");
    CHECK_ARG(p->n >= 0 && p->n <= 2147483647LL, "n = %lld out of range [0, 2^31-1]",
              (long long)p->n);
    CHECK_ARG(p->k >= 1 && p->k <= kMaxSide, "k = %lld out of range [1, 2^20]",
              (long long)p->k);
    CHECK_ARG(p->m >= 1 && p->m * (gated ? 2 : 1) <= kMaxSide,
              "m = %lld out of range (%s <= 2^20)", (long long)p->m, gated ? "2 m" : "m");
    CHECK_ARG(p->ldx >= p->k && p->ldx <= kMaxPitch, "ldx = %lld not in [k, 2^22]",
              (long long)p->ldx);
    CHECK_ARG(p->ldw >= p->k && p->ldw <= kMaxPitch, "ldw = %lld not in [k, 2^22]",
              (long long)p->ldw);
    CHECK_ARG(p->ldy >= p->m && p->ldy <= kMaxPitch, "ldy = %lld not in [m, 2^22]",
              (long long)p->ldy);
    if (gated) {
        // the gate's and the up projection's rows of one tile are addressed
        // from the gate's with 32-bit byte offsets
        const int64_t widest = p->ldw > split_ld(p->k) ? p->ldw : split_ld(p->k);
        if ((p->m + 256) * widest * 2 >= 0xfffffff0ll)
            return fail(GPIC_ERR_UNSUPPORTED, "gated weights of %lld x 2 rows of %lld: one half "
                        "must stay below 4 GiB", (long long)p->m, (long long)p->k);
    }
    return GPIC_OK;
}

gpic_status check_matrix(const void *x, const char *name, int32_t dtype, bool nullable,
                         bool aligned16 = false)
{
    if (x == nullptr) {
        if (nullable)
            return GPIC_OK;
        return fail(GPIC_ERR_INVALID_ARG, "%s is null", name);
    }
    CHECK_ARG(aligned(x, size_of(dtype)), "%s is misaligned", name);
    CHECK_ARG(!aligned16 || aligned(x, 16), "aligned16 is set and %s is not 16-byte aligned",
              name);
    return GPIC_OK;
}

gpic_status check_pre(const gpic_layer_params *p, bool gated)
{
    const int64_t width = gated ? 2 * p->m : p->m;
    CHECK_ARG(p->ldz >= width && p->ldz <= kMaxPitch, "ldz = %lld not in [%lld, 2^22]",
              (long long)p->ldz, (long long)width);
    return GPIC_OK;
}

// A matrix in memory: `rows` runs of `width` bytes, `pitch` bytes apart.
struct Extent {
    const char *name;
    const void *p;
    int64_t rows, width, pitch;
};

Extent matrix(const char *name, const void *p, int64_t rows, int64_t cols, int64_t ld, size_t size)
{
    return Extent{name, p, rows, cols * (int64_t)size, ld * (int64_t)size};
}

Extent packed(const char *name, const void *p, int64_t values, size_t size)
{
    return matrix(name, p, 1, values, values, size);
}

// Whether two matrices share a byte.  Columns of one table do not.
bool overlap(Extent a, Extent b)
{
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0)
        return false;
    const int64_t at = (int64_t)(uintptr_t)a.p, bt = (int64_t)(uintptr_t)b.p;
    if (at + (a.rows - 1) * a.pitch + a.width <= bt || bt + (b.rows - 1) * b.pitch + b.width <= at)
        return false;
    if (a.rows > 1 && b.rows > 1 && a.pitch == b.pitch) {
        int64_t d = (bt - at) % a.pitch;
        d = d < 0 ? d + a.pitch : d;
        return d < a.width || d + b.width > a.pitch;
    }
    if (a.rows > b.rows)
        return overlap(b, a);
    for (int64_t i = 0; i < a.rows; ++i) {
        // the first row of b that ends beyond this row's start
        const int64_t s = at + i * a.pitch, before = s - bt - b.width;
        const int64_t j = before < 0 ? 0 : (b.rows > 1 ? before / b.pitch + 1 : 1);
        if (j < b.rows && bt + j * b.pitch < s + a.width)
            return true;
    }
    return false;
}

// Results lie apart from what a call reads and from each other.
gpic_status check_apart(const Extent *out, int outs, const Extent *in, int ins)
{
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < ins; ++j)
            CHECK_ARG(!overlap(out[i], in[j]), "%s overlaps %s", out[i].name, in[j].name);
        for (int j = 0; j < i; ++j)
            CHECK_ARG(!overlap(out[i], out[j]), "%s overlaps %s", out[i].name, out[j].name);
    }
    return GPIC_OK;
}

Shape shape_of(const gpic_layer_params *p)
{
    Shape s;
    s.n = p->n;
    s.k = p->k;
    s.m = p->m;
    s.dtype = p->dtype;
    s.act = p->activation;
    s.ldx = p->ldx;
    s.ldw = p->ldw;
    s.ldr = p->ldr;
    s.ldy = p->ldy;
    s.ldz = p->ldz;
    s.aligned16 = p->aligned16 != 0;
    return s;
}

gpic_status check_fits(const gpic_layer_params *p, bool gated, bool backward)
{
    if (!layer_fits(shape_of(p), gated, backward))
        return fail(GPIC_ERR_UNSUPPORTED, "n = %lld, k = %lld, m = %lld: a product of more "
                    "workgroups than a launch takes", (long long)p->n, (long long)p->k,
                    (long long)p->m);
    return GPIC_OK;
}

// Largest |c1 s + c3 s^3 + c5 s^5| over [0, top]: the end or where the
// derivative c1 + 3 c3 s^2 + 5 c5 s^4 is zero.
double largest_odd(double c1, double c3, double c5, double top)
{
    auto at = [&](double s) { return fabs(s * (c1 + s * s * (c3 + s * s * c5))); };
    double most = at(top);
    auto consider = [&](double t) {
        if (t > 0.0 && t < top * top)
            most = fmax(most, at(sqrt(t)));
    };
    if (c5 == 0.0) {
        consider(c3 != 0.0 ? -c1 / (3.0 * c3) : 0.0);
        return most;
    }
    const double root = 9.0 * c3 * c3 - 20.0 * c5 * c1;
    if (root >= 0.0) {
        consider((-3.0 * c3 + sqrt(root)) / (10.0 * c5));
        consider((-3.0 * c3 - sqrt(root)) / (10.0 * c5));
    }
    return most;
}

// The iterates are held in halves times 1,024 (orthogonalize.hip): entries of
// A = X X^T are at most the square of X's largest singular value, those of
// b A + c A^2 at most |b s^2 + c s^4| there.  From 1 at the start, the bound of
// a step's singular values is the polynomial's largest over the step's before,
// and 1/256 for what is rounded.  The last step's result is no iterate.
gpic_status check_polynomial(const gpic_polar_params *p)
{
    const double a = p->a, b = p->b, c = p->c, limit = 60.0;     // 65,504 / 1,024 is 63.97
    double top = 1.0;
    for (int k = 0; k < p->steps; ++k) {
        double poly = fabs(top * top * (b + c * top * top));
        if (c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < top * top)
            poly = fmax(poly, b * b / (4.0 * fabs(c)));
        CHECK_ARG(top * top <= limit && poly <= limit,
                  "the polynomial takes singular values up to %g at step %d of %d: they must stay "
                  "below 7.7, and |b s^2 + c s^4| below 60 on them", top, k + 1, p->steps);
        top = largest_odd(a, b, c, top) * (1.0 + 1.0 / 256.0);
    }
    return GPIC_OK;
}

gpic_status check_polar(const gpic_polar_params *p)
{
    CHECK_ARG(p != nullptr, "params is null");
    CHECK_ARG(p->dtype >= GPIC_F32 && p->dtype <= GPIC_BF16,
              "dtype %d is not F32 (0), F16 (1) or BF16 (2)", p->dtype);
    CHECK_ARG(p->batch >= 0 && p->batch <= 65535, "batch = %lld out of range [0, 65535]",
              (long long)p->batch);
    CHECK_ARG(p->m >= 1 && p->m <= kMaxSide && p->n >= 1 && p->n <= kMaxSide,
              "m = %lld, n = %lld out of range [1, 2^20]", (long long)p->m, (long long)p->n);
    CHECK_ARG(p->steps >= 1 && p->steps <= 64, "steps = %d out of range [1, 64]", p->steps);
    CHECK_ARG(fabsf(p->a) <= 16.0f && fabsf(p->b) <= 16.0f && fabsf(p->c) <= 16.0f,
              "coefficients must be finite and at most 16 in magnitude");
    CHECK_ARG(isfinite(p->eps) && p->eps >= 0.0, "eps must be finite and >= 0");
    CHECK_ARG(p->reserved == 0, "reserved must be 0");
    return check_polynomial(p);
}

Polar polar_of(const gpic_polar_params *p)
{
    Polar q;
    q.batch = p->batch;
    q.m = p->m;
    q.n = p->n;
    q.dtype = p->dtype;
    q.steps = p->steps;
    q.a = p->a;
    q.b = p->b;
    q.c = p->c;
    q.eps = p->eps;
    return q;
}

#define CHECK(expr)                                                            \
    do {                                                                       \
        gpic_status st_ = (expr);                                              \
        if (st_ != GPIC_OK)                                                    \
            return st_;                                                        \
    } while (0)

} // namespace

extern "C" {

size_t gpic_layer_workspace_bytes(int32_t op, const gpic_layer_params *p)
{
    if (op < GPIC_LAYER_FORWARD || op > GPIC_GATED_BACKWARD)
        return 0;
    const bool gated = op >= GPIC_GATED_FORWARD;
    const bool backward = op == GPIC_LAYER_BACKWARD || op == GPIC_GATED_BACKWARD;
    if (check_layer(p, gated) != GPIC_OK)
        return 0;
    if (backward && (gated || p->activation != GPIC_ACT_NONE) && check_pre(p, gated) != GPIC_OK)
        return 0;
    if (check_fits(p, gated, backward) != GPIC_OK)
        return 0;
    return layer_ws(shape_of(p), gated, backward);
}

gpic_status gpic_linear(const gpic_layer_params *p, const void *X, const void *W,
                        const void *bias, const void *residual, void *Y, void *Z, void *ws,
                        size_t ws_bytes, void *stream)
{
    CHECK(check_layer(p, false));
    const bool empty = p->n == 0, a16 = p->aligned16 != 0;
    CHECK(check_matrix(X, "X", p->dtype, empty, a16));
    CHECK(check_matrix(W, "W", p->dtype, false, a16));
    CHECK(check_matrix(bias, "bias", p->dtype, true));
    CHECK(check_matrix(residual, "residual", p->dtype, true));
    CHECK(check_matrix(Y, "Y", p->dtype, empty));
    CHECK(check_matrix(Z, "Z", p->dtype, true));
    CHECK_ARG(residual == nullptr || (p->ldr >= p->m && p->ldr <= kMaxPitch),
              "ldr = %lld not in [m, 2^22]", (long long)p->ldr);
    if (Z != nullptr)
        CHECK(check_pre(p, false));
    CHECK(check_fits(p, false, false));
    CHECK(check_ws(ws, ws_bytes, layer_ws(shape_of(p), false, false)));
    {
        const size_t e = size_of(p->dtype);
        // Y may be the residual itself
        const bool in_place = residual == Y && (p->ldr == p->ldy || p->n == 1);
        const Extent out[] = {matrix("Y", Y, p->n, p->m, p->ldy, e),
                              matrix("Z", Z, p->n, p->m, p->ldz, e)};
        const Extent in[] = {matrix("X", X, p->n, p->k, p->ldx, e),
                             matrix("W", W, p->m, p->k, p->ldw, e), packed("bias", bias, p->m, e),
                             matrix("the residual", in_place ? nullptr : residual, p->n, p->m,
                                    p->ldr, e)};
        CHECK(check_apart(out, 2, in, 4));
    }
    CHECK_HIP(run_layer(shape_of(p), false, X, W, bias, residual, Y, Z, ws,
                        (hipStream_t)stream),
              "linear");
    return GPIC_OK;
}

gpic_status gpic_linear_backward(const gpic_layer_params *p, const void *dY, const void *X,
                                 const void *W, const void *Z, void *dX, void *dW, void *db,
                                 void *ws, size_t ws_bytes, void *stream)
{
    CHECK(check_layer(p, false));
    const bool empty = p->n == 0, a16 = p->aligned16 != 0;
    const bool act = p->activation != GPIC_ACT_NONE;
    CHECK(check_matrix(dY, "dY", p->dtype, empty, a16));
    CHECK(check_matrix(X, "X", p->dtype, empty || dW == nullptr, a16));
    CHECK(check_matrix(W, "W", p->dtype, dX == nullptr, a16));
    CHECK(check_matrix(Z, "Z", p->dtype, empty || !act));
    CHECK(check_matrix(dX, "dX", p->dtype, true));
    CHECK(check_matrix(dW, "dW", p->dtype, true));
    CHECK(check_matrix(db, "db", p->dtype, true));
    if (act)
        CHECK(check_pre(p, false));
    CHECK(check_fits(p, false, true));
    CHECK(check_ws(ws, ws_bytes, layer_ws(shape_of(p), false, true)));
    {
        const size_t e = size_of(p->dtype);
        const Extent out[] = {packed("dX", dX, p->n * p->k, e), packed("dW", dW, p->m * p->k, e),
                              packed("db", db, p->m, e)};
        const Extent in[] = {matrix("dY", dY, p->n, p->m, p->ldy, e),
                             matrix("X", dW ? X : nullptr, p->n, p->k, p->ldx, e),
                             matrix("W", dX ? W : nullptr, p->m, p->k, p->ldw, e),
                             matrix("Z", act ? Z : nullptr, p->n, p->m, p->ldz, e)};
        CHECK(check_apart(out, 3, in, 4));
    }
    CHECK_HIP(run_layer_backward(shape_of(p), false, dY, X, W, Z, dX, dW, db, ws,
                                 (hipStream_t)stream),
              "linear backward");
    return GPIC_OK;
}

gpic_status gpic_gated(const gpic_layer_params *p, const void *X, const void *W, void *H,
                       void *Z, void *ws, size_t ws_bytes, void *stream)
{
    CHECK(check_layer(p, true));
    const bool empty = p->n == 0, a16 = p->aligned16 != 0;
    CHECK(check_matrix(X, "X", p->dtype, empty, a16));
    CHECK(check_matrix(W, "W", p->dtype, false, a16));
    CHECK(check_matrix(H, "H", p->dtype, empty));
    CHECK(check_matrix(Z, "Z", GPIC_F32, true));
    if (Z != nullptr)
        CHECK(check_pre(p, true));
    CHECK(check_fits(p, true, false));
    CHECK(check_ws(ws, ws_bytes, layer_ws(shape_of(p), true, false)));
    {
        const size_t e = size_of(p->dtype);
        const Extent out[] = {matrix("H", H, p->n, p->m, p->ldy, e),
                              matrix("Z", Z, p->n, 2 * p->m, p->ldz, 4)};
        const Extent in[] = {matrix("X", X, p->n, p->k, p->ldx, e),
                             matrix("W", W, 2 * p->m, p->k, p->ldw, e)};
        CHECK(check_apart(out, 2, in, 2));
    }
    CHECK_HIP(run_layer(shape_of(p), true, X, W, nullptr, nullptr, H, Z, ws,
                        (hipStream_t)stream),
              "gated");
    return GPIC_OK;
}

gpic_status gpic_gated_backward(const gpic_layer_params *p, const void *dH, const void *X,
                                const void *W, const void *Z, void *dX, void *dW, void *ws,
                                size_t ws_bytes, void *stream)
{
    CHECK(check_layer(p, true));
    const bool empty = p->n == 0, a16 = p->aligned16 != 0;
    CHECK(check_matrix(dH, "dH", p->dtype, empty, a16));
    CHECK(check_matrix(X, "X", p->dtype, empty || dW == nullptr, a16));
    CHECK(check_matrix(W, "W", p->dtype, dX == nullptr, a16));
    CHECK(check_matrix(Z, "Z", GPIC_F32, empty));
    CHECK(check_matrix(dX, "dX", p->dtype, true));
    CHECK(check_matrix(dW, "dW", p->dtype, true));
    CHECK(check_pre(p, true));
    CHECK(check_fits(p, true, true));
    CHECK(check_ws(ws, ws_bytes, layer_ws(shape_of(p), true, true)));
    {
        const size_t e = size_of(p->dtype);
        const Extent out[] = {packed("dX", dX, p->n * p->k, e),
                              packed("dW", dW, 2 * p->m * p->k, e)};
        const Extent in[] = {matrix("dH", dH, p->n, p->m, p->ldy, e),
                             matrix("X", dW ? X : nullptr, p->n, p->k, p->ldx, e),
                             matrix("W", dX ? W : nullptr, 2 * p->m, p->k, p->ldw, e),
                             matrix("Z", Z, p->n, 2 * p->m, p->ldz, 4)};
        CHECK(check_apart(out, 2, in, 4));
    }
    CHECK_HIP(run_layer_backward(shape_of(p), true, dH, X, W, Z, dX, dW, nullptr, ws,
                                 (hipStream_t)stream),
              "gated backward");
    return GPIC_OK;
}

size_t gpic_polar_workspace_bytes(const gpic_polar_params *p)
{
    return check_polar(p) == GPIC_OK ? polar_ws(polar_of(p)) : 0;
}

gpic_status gpic_orthogonalize(const gpic_polar_params *p, const void *G, void *O, void *ws,
                               size_t ws_bytes, void *stream)
{
    CHECK(check_polar(p));
    const bool empty = p->batch == 0;
    CHECK(check_matrix(G, "G", p->dtype, empty));
    CHECK(check_matrix(O, "O", p->dtype, empty));
    CHECK(check_ws(ws, ws_bytes, polar_ws(polar_of(p))));
    {
        const int64_t values = p->batch * p->m * p->n;
        const Extent out = packed("O", O, values, size_of(p->dtype));
        const Extent in = packed("G", O == G ? nullptr : G, values, size_of(p->dtype));
        CHECK(check_apart(&out, 1, &in, 1));
    }
    CHECK_HIP(run_orthogonalize(polar_of(p), G, O, ws, (hipStream_t)stream), "orthogonalize");
    return GPIC_OK;
}

gpic_status gpic_muon_step(const gpic_polar_params *p, const gpic_muon_params *h, void *W,
                           const void *G, float *M, void *ws, size_t ws_bytes, void *stream)
{
    CHECK(check_polar(p));
    CHECK_ARG(h != nullptr, "the step's params are null");
    CHECK_ARG(isfinite(h->lr) && isfinite(h->momentum) && isfinite(h->weight_decay) &&
                  isfinite(h->scale),
              "lr, momentum, weight_decay and scale must be finite");
    CHECK_ARG(h->nesterov == 0 || h->nesterov == 1, "nesterov must be 0 or 1");
    CHECK_ARG(h->reserved == 0, "reserved must be 0");
    const bool empty = p->batch == 0;
    CHECK(check_matrix(W, "W", p->dtype, empty));
    CHECK(check_matrix(G, "G", p->dtype, empty));
    CHECK(check_matrix(M, "M", GPIC_F32, empty));
    CHECK(check_ws(ws, ws_bytes, polar_ws(polar_of(p))));
    {
        const int64_t values = p->batch * p->m * p->n;
        const Extent out[] = {packed("W", W, values, size_of(p->dtype)), packed("M", M, values, 4)};
        // (G is read before W is written)
        const Extent in = packed("G", G == W ? nullptr : G, values, size_of(p->dtype));
        CHECK(check_apart(out, 2, &in, 1));
    }
    MuonStep m;
    m.lr = h->lr;
    m.momentum = h->momentum;
    m.decay = h->weight_decay;
    m.scale = h->scale;
    m.nesterov = h->nesterov;
    CHECK_HIP(run_muon(polar_of(p), m, W, G, M, ws, (hipStream_t)stream), "muon step");
    return GPIC_OK;
}

} // extern "C"
