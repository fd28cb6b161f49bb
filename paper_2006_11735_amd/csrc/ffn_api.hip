// C boundary of the feed-forward operators in 8 bits: argument validation (host only, before any launch) and dispatch.
#include "../../include/icnn.h"
#include "ffn_common.h"

#include <cmath>

using namespace icnn;

namespace {

static_assert(kF32 == ICNN_F32 && kF16 == ICNN_F16 && kBf16 == ICNN_BF16, "types of a stream");

constexpr int64_t kMostRows = 0x7fff0000, kMostStride = (int64_t)1 << 40, kMostElements = (int64_t)1 << 44;      // (16 TiB of bytes)

int item_of(int dtype) { return dtype == ICNN_F32 ? 4 : 2; }

bool is_stream(int dtype) { return dtype == ICNN_F32 || dtype == ICNN_F16 || dtype == ICNN_BF16; }

int check_stride(const char *what, int64_t stride, int64_t least, int64_t rows)
{
    if (stride < least || stride > kMostStride)
        return fail(ICNN_E_SHAPE, "%s %lld must be in [%lld, 2^40]", what, (long long)stride, (long long)least);
    if (rows && stride > kMostElements / rows)
        return fail(ICNN_E_SHAPE, "%s %lld: %lld rows of it exceed 2^44 elements", what, (long long)stride, (long long)rows);
    return ICNN_OK;
}

// The bytes of a tensor: `rows` rows of `width` bytes, `pitch` apart
struct Rows {
    uintptr_t at, end;
    unsigned long long pitch, width;
};

Rows rows_of(const void *p, int64_t rows, int64_t stride, int64_t width, int item)
{
    Rows r;
    r.at = (uintptr_t)p;
    r.pitch = (unsigned long long)stride * item;
    r.width = (unsigned long long)width * item;
    r.end = r.at + (uintptr_t)(rows - 1) * r.pitch + r.width;
    return r;
}

// Do two tensors share a byte?  Column ranges of one buffer do not where they are disjoint; ranges that interleave with different pitches count as shared.
bool share(const Rows &a, const Rows &b)
{
    if (a.at >= b.end || b.at >= a.end) return false;
    if (a.pitch != b.pitch) return true;
    const unsigned long long d = b.at >= a.at ? (b.at - a.at) % a.pitch : (a.pitch - (a.at - b.at) % a.pitch) % a.pitch;
    return !(d >= a.width && d + b.width <= a.pitch);
}

bool same(const Rows &a, const Rows &b) { return a.at == b.at && a.pitch == b.pitch; }

bool aligned_to(const void *p, int item) { return ((uintptr_t)p & (uintptr_t)(item - 1)) == 0; }

int launched(hipError_t e, const char *what)
{
    return e == hipSuccess ? ICNN_OK : fail(ICNN_E_LAUNCH, "%s: %s", what, hipGetErrorString(e));
}

int check_rows_desc(const icnn_norm_desc *d)
{
    if (!d) return fail(ICNN_E_NULL, "descriptor is NULL");
    if (d->rows < 0 || d->rows > kMostRows) return fail(ICNN_E_SHAPE, "rows %lld must be in [0, 2^31 - 2^16]", (long long)d->rows);
    if (d->c < 1 || d->c > (1 << 20)) return fail(ICNN_E_SHAPE, "c %d must be in [1, 2^20]", d->c);
    if (!is_stream(d->dtype)) return fail(ICNN_E_PARAM, "dtype %d must be ICNN_F32, ICNN_F16 or ICNN_BF16", d->dtype);
    int rc = check_stride("x_stride", d->x_stride, d->c, d->rows);
    return rc ? rc : check_stride("q_stride", d->q_stride, d->c, d->rows);
}

int check_linear(const icnn_linear_desc *d)
{
    if (!d) return fail(ICNN_E_NULL, "descriptor is NULL");
    if (d->rows < 0 || d->rows > kMostRows) return fail(ICNN_E_SHAPE, "rows %lld must be in [0, 2^31 - 2^16]", (long long)d->rows);
    if (d->k < 1 || d->n < 1 || d->n > kMostRows) return fail(ICNN_E_SHAPE, "k and n must be >= 1, n at most 2^31 - 2^16");
    if (d->k > 131071) return fail(ICNN_E_SHAPE, "k = %d exceeds 131071: int32 accumulation not provably safe", d->k);
    if (!is_stream(d->dtype)) return fail(ICNN_E_PARAM, "dtype %d must be ICNN_F32, ICNN_F16 or ICNN_BF16", d->dtype);
    if (d->act < ICNN_ACT_NONE || d->act > ICNN_ACT_GELU_TANH) return fail(ICNN_E_PARAM, "unknown act %d", d->act);
    if (int rc = check_stride("x_stride", d->x_stride, d->k, d->rows)) return rc;
    if (int rc = check_stride("w_stride", d->w_stride, d->k, d->n)) return rc;
    return check_stride("y_stride", d->y_stride, d->n, d->rows);
}

struct Operand {
    const char *name;
    const void *p;
    Rows r;
};

void sizes_of(const icnn_linear_desc *d, LinearArgs &a)
{
    a.M = (int)d->rows;
    a.N = d->n;
    a.K = d->k;
    a.ldx = d->x_stride;
    a.ldw = d->w_stride;
    a.ldr = d->res_stride;
    a.ldy = d->y_stride;
    a.act = d->act;
    a.dtype = d->dtype;
}

// Everything behind the descriptor's own check; `a` holds the pointers.
int run_linear(const icnn_linear_desc *d, LinearArgs &a, void *workspace, void *stream, const char *what)
{
    const int item = item_of(d->dtype);
    if (a.res)
        if (int rc = check_stride("res_stride", d->res_stride, d->n, d->rows)) return rc;
    if (d->rows == 0) return ICNN_OK;
    if (!a.x || !a.xs || !a.w || !a.ws || !a.y) return fail(ICNN_E_NULL, "x, x_scale, w, w_scale and y must not be NULL");
    for (const void *p : {(const void *)a.xs, (const void *)a.ws, (const void *)a.ws2, (const void *)a.bias, (const void *)a.bias2})
        if (!aligned_to(p, 4)) return fail(ICNN_E_ALIGN, "scales and biases must be 4-byte aligned");
    if (!aligned_to(a.y, item) || !aligned_to(a.res, item)) return fail(ICNN_E_ALIGN, "y and residual must be aligned to their elements");
    if (!aligned_to(workspace, 16)) return fail(ICNN_E_ALIGN, "workspace must be 16-byte aligned");
    const Rows y = rows_of(a.y, d->rows, d->y_stride, d->n, item);
    const Operand in[] = {
        {"x", a.x, rows_of(a.x, d->rows, d->x_stride, d->k, 1)}, {"w", a.w, rows_of(a.w, d->n, d->w_stride, d->k, 1)},
        {"w_up", a.w2, rows_of(a.w2, d->n, d->w_stride, d->k, 1)}, {"x_scale", a.xs, rows_of(a.xs, 1, d->rows, d->rows, 4)},
        {"w_scale", a.ws, rows_of(a.ws, 1, d->n, d->n, 4)}, {"up_scale", a.ws2, rows_of(a.ws2, 1, d->n, d->n, 4)},
        {"bias", a.bias, rows_of(a.bias, 1, d->n, d->n, 4)}, {"up_bias", a.bias2, rows_of(a.bias2, 1, d->n, d->n, 4)},
        {"residual", a.res, rows_of(a.res, d->rows, d->res_stride, d->n, item)}};
    for (const Operand &o : in)
        if (o.p && share(y, o.r) && !(o.p == a.res && same(y, o.r))) return fail(ICNN_E_UNSUPPORTED, "y overlaps %s", o.name);
    sizes_of(d, a);
    a.workspace = workspace;
    return launched(launch_linear(a, (hipStream_t)stream), what);
}

int workspace_bytes(const icnn_linear_desc *desc, bool gated, size_t *bytes)
{
    if (int rc = check_linear(desc)) return rc;
    if (!bytes) return fail(ICNN_E_NULL, "bytes is NULL");
    LinearArgs a = {};
    sizes_of(desc, a);
    a.w2 = gated ? (const int8_t *)16 : nullptr;           // (whether there is one; never read)
    *bytes = desc->rows ? linear_workspace(a) : 0;
    return ICNN_OK;
}

}  // namespace

extern "C" {

int irms_norm_s8(const icnn_norm_desc *d, const void *x, const void *residual, const void *gamma, void *sum, void *q, float *scale, void *stream)
{
    if (int rc = check_rows_desc(d)) return rc;
    if (d->gamma_dtype != d->dtype && d->gamma_dtype != ICNN_F32)
        return fail(ICNN_E_PARAM, "gamma_dtype %d must be the stream's type or ICNN_F32", d->gamma_dtype);
    if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return fail(ICNN_E_PARAM, "eps must be finite and >= 0");
    if (residual)
        if (int rc = check_stride("res_stride", d->res_stride, d->c, d->rows)) return rc;
    if (sum)
        if (int rc = check_stride("sum_stride", d->sum_stride, d->c, d->rows)) return rc;
    if (d->rows == 0) return ICNN_OK;
    if (!x || !gamma || !q || !scale) return fail(ICNN_E_NULL, "x, gamma, q and scale must not be NULL");
    const int item = item_of(d->dtype), gitem = item_of(d->gamma_dtype);
    if (!aligned_to(x, item) || !aligned_to(residual, item) || !aligned_to(sum, item) || !aligned_to(gamma, gitem) || !aligned_to(scale, 4))
        return fail(ICNN_E_ALIGN, "x, residual, sum, gamma and scale must be aligned to their elements");
    const Rows rx = rows_of(x, d->rows, d->x_stride, d->c, item), rr = rows_of(residual, d->rows, d->res_stride, d->c, item),
               rs = rows_of(sum, d->rows, d->sum_stride, d->c, item), rq = rows_of(q, d->rows, d->q_stride, d->c, 1),
               rg = rows_of(gamma, 1, d->c, d->c, gitem), rc = rows_of(scale, 1, d->rows, d->rows, 4);
    bool bad = share(rq, rx) || share(rc, rx) || share(rq, rg) || share(rc, rg) || share(rq, rc);
    if (residual) bad = bad || share(rq, rr) || share(rc, rr);
    if (sum) {
        bad = bad || share(rs, rq) || share(rs, rc) || share(rs, rg) || (share(rs, rx) && !same(rs, rx));
        if (residual) bad = bad || (share(rs, rr) && !same(rs, rr));
    }
    if (bad) return fail(ICNN_E_UNSUPPORTED, "an output overlaps an input or another output");
    RowsArgs a;
    a.x = x; a.res = residual; a.gamma = gamma; a.sum = sum; a.q = (int8_t *)q; a.scale = scale;
    a.rows = d->rows; a.ldx = d->x_stride; a.ldr = d->res_stride; a.lds = d->sum_stride; a.ldq = d->q_stride;
    a.c = d->c; a.dtype = d->dtype; a.gamma_dtype = d->gamma_dtype; a.eps = d->eps;
    return launched(launch_rows(a, (hipStream_t)stream), "irms_norm_s8");
}

int iquantize_rows_s8(const icnn_norm_desc *d, const void *x, void *q, float *scale, void *stream)
{
    if (int rc = check_rows_desc(d)) return rc;
    if (d->rows == 0) return ICNN_OK;
    if (!x || !q || !scale) return fail(ICNN_E_NULL, "x, q and scale must not be NULL");
    const int item = item_of(d->dtype);
    if (!aligned_to(x, item) || !aligned_to(scale, 4)) return fail(ICNN_E_ALIGN, "x and scale must be aligned to their elements");
    const Rows rx = rows_of(x, d->rows, d->x_stride, d->c, item), rq = rows_of(q, d->rows, d->q_stride, d->c, 1),
               rc = rows_of(scale, 1, d->rows, d->rows, 4);
    if (share(rq, rx) || share(rc, rx) || share(rq, rc)) return fail(ICNN_E_UNSUPPORTED, "an output overlaps the input or the other output");
    RowsArgs a = {};
    a.x = x; a.q = (int8_t *)q; a.scale = scale;
    a.rows = d->rows; a.ldx = d->x_stride; a.ldq = d->q_stride;
    a.c = d->c; a.dtype = a.gamma_dtype = d->dtype;
    return launched(launch_rows(a, (hipStream_t)stream), "iquantize_rows_s8");
}

int ilinear_s8_workspace_bytes(const icnn_linear_desc *desc, size_t *bytes) { return workspace_bytes(desc, false, bytes); }

int igated_linear_s8_workspace_bytes(const icnn_linear_desc *desc, size_t *bytes) { return workspace_bytes(desc, true, bytes); }

int ilinear_s8(const icnn_linear_desc *desc, const void *x, const float *x_scale, const void *w, const float *w_scale, const float *bias,
               const void *residual, void *y, void *workspace, void *stream)
{
    if (int rc = check_linear(desc)) return rc;
    LinearArgs a = {};
    a.x = (const int8_t *)x; a.xs = x_scale;
    a.w = (const int8_t *)w; a.ws = w_scale; a.bias = bias;
    a.res = residual; a.y = y;
    return run_linear(desc, a, workspace, stream, "ilinear_s8");
}

int igated_linear_s8(const icnn_linear_desc *desc, const void *x, const float *x_scale, const void *w_gate, const float *gate_scale,
                     const float *gate_bias, const void *w_up, const float *up_scale, const float *up_bias, void *y, void *workspace, void *stream)
{
    if (int rc = check_linear(desc)) return rc;
    if (desc->rows && (!w_up || !up_scale)) return fail(ICNN_E_NULL, "w_up and up_scale must not be NULL");
    LinearArgs a = {};
    a.x = (const int8_t *)x; a.xs = x_scale;
    a.w = (const int8_t *)w_gate; a.ws = gate_scale; a.bias = gate_bias;
    a.w2 = (const int8_t *)w_up; a.ws2 = up_scale; a.bias2 = up_bias;
    a.y = y;
    return run_linear(desc, a, workspace, stream, "igated_linear_s8");
}

}  // extern "C"
