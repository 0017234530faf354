// Entry points of the products over groups of rows and of the 8-bit product: their checks, and the problem each is.
#include "grouped.h"
#include "ops.h"

namespace alt {
namespace {

struct Buffer {
    const char *name;
    const void *p;
    size_t align;
    bool used = true;
};

// What every call checks of its layer, dense strides filled in.
alt_status_t check_layer(alt_handle_t h, const char *call, const alt_grouped_desc_t *d, bool gradient, alt_grouped_desc_t *out)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "%s: null descriptor", call);
    *out = *d;
    if (d->rows < 0 || d->N < 1 || d->K < 1 || d->groups < 1 || d->lda < 0 || d->ldb < 0 || d->ldc < 0) return fail(h, ALT_INVALID_ARG, "%s: bad size", call);
    if (d->in_dtype != ALT_F32 && d->in_dtype != ALT_BF16 && d->in_dtype != ALT_I8) return fail(h, ALT_INVALID_ARG, "%s: bad in_dtype", call);
    if (d->out_dtype != ALT_F32 && d->out_dtype != ALT_BF16) return fail(h, ALT_INVALID_ARG, "%s: bad out_dtype", call);
    if (d->epilogue & ~(ALT_EPI_BIAS | ALT_EPI_RELU)) return fail(h, ALT_INVALID_ARG, "%s: unknown epilogue flag", call);
    if (!out->lda) out->lda = d->K;
    if (!out->ldb) out->ldb = d->K;
    if (!out->ldc) out->ldc = d->N;
    if (out->lda < d->K || out->ldb < d->K || out->ldc < d->N) return fail(h, ALT_SHAPE_MISMATCH, "%s: a row stride is shorter than a row", call);
    if (gradient && d->in_dtype == ALT_I8) return fail(h, ALT_UNSUPPORTED, "%s: 8-bit products have no gradients", call);
    if (d->in_dtype == ALT_F32 && d->out_dtype != ALT_F32) return fail(h, ALT_UNSUPPORTED, "%s: fp32 operands give fp32 results", call);
    if (d->rows > (1 << 30) || d->groups > (1 << 20) || out->lda > (1 << 22) || out->ldb > (1 << 22) || out->ldc > (1 << 22))
        return fail(h, ALT_UNSUPPORTED, "%s: more than 2^30 rows, 2^20 groups or 2^22 elements between rows", call);
    if (d->in_dtype == ALT_I8 && d->K > ALT_I8_MAX_K) return fail(h, ALT_UNSUPPORTED, "%s: 32-bit sums hold %d products of 8-bit numbers at most", call, ALT_I8_MAX_K);
    return ALT_OK;
}

alt_status_t check_buffers(alt_handle_t h, const char *call, std::initializer_list<Buffer> bufs)
{
    for (const Buffer &b : bufs) {
        if (!b.used) continue;
        if (!b.p) return fail(h, ALT_INVALID_ARG, "%s: %s is null", call, b.name);
        if ((uintptr_t)b.p % b.align) return fail(h, ALT_INVALID_ARG, "%s: %s is not aligned to its elements", call, b.name);
    }
    if (!h->has_gpu) return fail(h, ALT_HIP_ERROR, "no GPU device available");
    return ALT_OK;
}

size_t in_size(int dt) { return dt == ALT_I8 ? 1 : dtype_size(dt); }

alt_status_t run(alt_handle_t h, const char *call, int dtype, int form, GroupedParams &p, int64_t ldy_elems, hipStream_t st)
{
    const size_t os = p.flags & kGrpOutBf16 ? 2 : 4;
    p.ldy = ldy_elems * (int64_t)os;
    p.y_group *= (int64_t)os;
    p.places = h->compute_units;
    if (p.cols % (os == 2 ? 8 : 4) == 0) p.flags |= kGrpWhole;
    const hipError_t e = dtype == ALT_I8 ? grouped_run_i8(p, st) : dtype == ALT_BF16 ? grouped_run_bf16(form, p, st) : grouped_run_f32(form, p, st);
    if (e == hipErrorInvalidConfiguration) return fail(h, ALT_UNSUPPORTED, "%s: more output tiles than a launch holds", call);
    ALT_CHECK_HIP(h, e);
    return ALT_OK;
}

alt_status_t forward(alt_handle_t h, const char *call, const alt_grouped_desc_t &d, const void *a, const float *a_scale, const void *b, const float *b_scale,
                     const float *bias, const int32_t *offsets, void *y, void *stream)
{
    const size_t es = in_size(d.in_dtype);
    GroupedParams p{};
    p.a = a; p.b = b; p.y = y;
    p.a_scale = a_scale; p.b_scale = b_scale;
    p.bias = d.epilogue & ALT_EPI_BIAS ? bias : nullptr;
    p.offsets = offsets;
    p.lda = d.lda * (int64_t)es; p.ldb = d.ldb * (int64_t)es;
    p.b_group = d.N * p.ldb;
    p.rows = (int32_t)d.rows; p.cols = (int32_t)d.N; p.red = (int32_t)d.K; p.groups = d.groups;
    p.flags = (d.epilogue & ALT_EPI_RELU ? kGrpRelu : 0) | (d.out_dtype == ALT_BF16 ? kGrpOutBf16 : 0);
    return run(h, call, d.in_dtype, kForward, p, d.ldc, (hipStream_t)stream);
}

alt_status_t no_workspace(alt_handle_t h, const alt_grouped_desc_t *d, bool gradient, const char *call, size_t *bytes)
{
    alt_grouped_desc_t l;
    const alt_status_t s = check_layer(h, call, d, gradient, &l);
    if (s != ALT_OK) return s;
    if (!bytes) return fail(h, ALT_INVALID_ARG, "%s: null result", call);
    *bytes = 0;
    return ALT_OK;
}

// The 8-bit product as a layer of one group.
alt_grouped_desc_t one_group(const alt_gemm_i8_desc_t *d)
{
    alt_grouped_desc_t g{};
    g.rows = d->M; g.N = d->N; g.K = d->K;
    g.lda = d->lda; g.ldb = d->ldb; g.ldc = d->ldc;
    g.groups = 1;
    g.in_dtype = ALT_I8; g.out_dtype = d->out_dtype; g.epilogue = d->epilogue;
    return g;
}

}  // namespace
}  // namespace alt

using namespace alt;

extern "C" alt_status_t alt_gemm_grouped(alt_handle_t h, const alt_grouped_desc_t *d, const void *a, const float *a_scale, const void *b, const float *b_scale,
                                         const float *bias, const int32_t *offsets, void *y, void *workspace, size_t ws_bytes, void *stream)
{
    alt_grouped_desc_t l;
    alt_status_t s = check_layer(h, "alt_gemm_grouped", d, false, &l);
    if (s != ALT_OK) return s;
    (void)workspace; (void)ws_bytes;
    if (l.rows == 0) return ALT_OK;
    const size_t es = in_size(l.in_dtype);
    const bool scaled = l.in_dtype == ALT_I8;
    s = check_buffers(h, "alt_gemm_grouped", {{"a", a, es}, {"b", b, es}, {"offsets", offsets, 4}, {"y", y, dtype_size(l.out_dtype)}, {"a_scale", a_scale, 4, scaled},
                                              {"b_scale", b_scale, 4, scaled}, {"bias", bias, 4, (l.epilogue & ALT_EPI_BIAS) != 0}});
    if (s != ALT_OK) return s;
    return forward(h, "alt_gemm_grouped", l, a, a_scale, b, b_scale, bias, offsets, y, stream);
}

extern "C" alt_status_t alt_gemm_grouped_dx(alt_handle_t h, const alt_grouped_desc_t *d, const void *dy, const void *b, const void *relu_of, const int32_t *offsets,
                                            void *dx, void *workspace, size_t ws_bytes, void *stream)
{
    alt_grouped_desc_t l;
    alt_status_t s = check_layer(h, "alt_gemm_grouped_dx", d, true, &l);
    if (s != ALT_OK) return s;
    (void)workspace; (void)ws_bytes;
    if (l.epilogue & ALT_EPI_BIAS) return fail(h, ALT_INVALID_ARG, "alt_gemm_grouped_dx: a bias has no part in the gradient of x");
    if (l.rows == 0) return ALT_OK;
    const size_t es = in_size(l.in_dtype);
    s = check_buffers(h, "alt_gemm_grouped_dx", {{"dy", dy, es}, {"b", b, es}, {"offsets", offsets, 4}, {"dx", dx, dtype_size(l.out_dtype)},
                                                 {"relu_of", relu_of, es, (l.epilogue & ALT_EPI_RELU) != 0}});
    if (s != ALT_OK) return s;
    GroupedParams p{};
    p.a = dy; p.b = b; p.y = dx;
    p.mask = relu_of;
    p.offsets = offsets;
    p.lda = l.ldc * (int64_t)es; p.ldb = l.ldb * (int64_t)es; p.ldmask = l.lda * (int64_t)es;
    p.b_group = l.N * p.ldb;
    p.rows = (int32_t)l.rows; p.cols = (int32_t)l.K; p.red = (int32_t)l.N; p.groups = l.groups;
    p.flags = (l.epilogue & ALT_EPI_RELU ? kGrpMask : 0) | (l.out_dtype == ALT_BF16 ? kGrpOutBf16 : 0);
    return run(h, "alt_gemm_grouped_dx", l.in_dtype, kInput, p, l.lda, (hipStream_t)stream);
}

extern "C" alt_status_t alt_gemm_grouped_dw(alt_handle_t h, const alt_grouped_desc_t *d, const void *a, const void *dy, const int32_t *offsets, void *dw, float *dbias,
                                            void *workspace, size_t ws_bytes, void *stream)
{
    alt_grouped_desc_t l;
    alt_status_t s = check_layer(h, "alt_gemm_grouped_dw", d, true, &l);
    if (s != ALT_OK) return s;
    (void)workspace; (void)ws_bytes;
    if (l.epilogue & ALT_EPI_RELU) return fail(h, ALT_INVALID_ARG, "alt_gemm_grouped_dw: dy is the gradient before the ReLU");
    const size_t es = in_size(l.in_dtype);
    // (without rows the gradients are zeros, and a and dy need not exist)
    s = check_buffers(h, "alt_gemm_grouped_dw", {{"a", a, es, l.rows > 0}, {"dy", dy, es, l.rows > 0}, {"offsets", offsets, 4},
                                                 {"dw", dw, dtype_size(l.out_dtype)}, {"dbias", dbias, 4, (l.epilogue & ALT_EPI_BIAS) != 0}});
    if (s != ALT_OK) return s;
    GroupedParams p{};
    p.a = dy; p.b = a; p.y = dw;
    p.colsum = l.epilogue & ALT_EPI_BIAS ? dbias : nullptr;
    p.offsets = offsets;
    p.lda = l.ldc * (int64_t)es; p.ldb = l.lda * (int64_t)es;
    p.y_group = l.N * l.ldb;
    p.rows = (int32_t)l.N; p.cols = (int32_t)l.K; p.red = (int32_t)l.rows; p.groups = l.groups;
    p.flags = l.out_dtype == ALT_BF16 ? kGrpOutBf16 : 0;
    return run(h, "alt_gemm_grouped_dw", l.in_dtype, kWeights, p, l.ldb, (hipStream_t)stream);
}

extern "C" alt_status_t alt_gemm_grouped_workspace_size(alt_handle_t h, const alt_grouped_desc_t *d, size_t *bytes)
{
    return no_workspace(h, d, false, "alt_gemm_grouped_workspace_size", bytes);
}

extern "C" alt_status_t alt_gemm_grouped_dx_workspace_size(alt_handle_t h, const alt_grouped_desc_t *d, size_t *bytes)
{
    return no_workspace(h, d, true, "alt_gemm_grouped_dx_workspace_size", bytes);
}

extern "C" alt_status_t alt_gemm_grouped_dw_workspace_size(alt_handle_t h, const alt_grouped_desc_t *d, size_t *bytes)
{
    return no_workspace(h, d, true, "alt_gemm_grouped_dw_workspace_size", bytes);
}

extern "C" alt_status_t alt_gemm_i8(alt_handle_t h, const alt_gemm_i8_desc_t *d, const void *a, const float *a_scale, const void *b, const float *b_scale,
                                    const float *bias, void *y, void *workspace, size_t ws_bytes, void *stream)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "alt_gemm_i8: null descriptor");
    const alt_grouped_desc_t g = one_group(d);
    alt_grouped_desc_t l;
    alt_status_t s = check_layer(h, "alt_gemm_i8", &g, false, &l);
    if (s != ALT_OK) return s;
    (void)workspace; (void)ws_bytes;
    if (l.rows == 0) return ALT_OK;
    s = check_buffers(h, "alt_gemm_i8", {{"a", a, 1}, {"b", b, 1}, {"a_scale", a_scale, 4}, {"b_scale", b_scale, 4}, {"y", y, dtype_size(l.out_dtype)},
                                         {"bias", bias, 4, (l.epilogue & ALT_EPI_BIAS) != 0}});
    if (s != ALT_OK) return s;
    return forward(h, "alt_gemm_i8", l, a, a_scale, b, b_scale, bias, nullptr, y, stream);
}

extern "C" alt_status_t alt_gemm_i8_workspace_size(alt_handle_t h, const alt_gemm_i8_desc_t *d, size_t *bytes)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "alt_gemm_i8_workspace_size: null descriptor");
    const alt_grouped_desc_t g = one_group(d);
    return no_workspace(h, &g, false, "alt_gemm_i8_workspace_size", bytes);
}
