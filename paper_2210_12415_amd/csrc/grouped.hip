// Entry points of the products over groups of rows and of the 8-bit product: their checks, and the problem each is.
#include "adapters.h"
#include "ops.h"
#include "rows.h"

namespace alt {
namespace {

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

alt_status_t check_layer_buffers(alt_handle_t h, const char *call, std::initializer_list<RowsBuffer> bufs)
{
    const alt_status_t s = check_buffers(h, call, bufs);
    if (s != ALT_OK) return s;
    if (!h->has_gpu) return fail(h, ALT_HIP_ERROR, "no GPU device available");
    return ALT_OK;
}

size_t in_size(int dt) { return dt == ALT_I8 ? 1 : dtype_size(dt); }

// ---- operands whose rows are not whole 16-byte chunks, laid out anew -------------------------------------------------------------

// Rows of a matrix that are laid out anew: dst[r] = src[r] filled up with zeros to `dst_bytes` (a multiple of 16), in pieces of 32 bytes.
struct PackJob {
    const char *src;
    char *dst;
    int64_t ld;
    int bytes, dst_bytes;
    uint32_t pieces;
    FastDiv per_row;
};

// A thread moves a piece: the eight dwords it starts in and the one it ends in, shifted together; behind a row's last byte no dword is touched.
// Two matrices to a launch.  Bound by memory: two of 8191 rows of 8191 bytes in 42 us, 6.4 TB/s read and written.
__global__ __launch_bounds__(256) void grp_pack_kernel(const PackJob first, const PackJob second, uint32_t first_blocks)
{
    const bool is_first = blockIdx.x < first_blocks;
    const PackJob &j = is_first ? first : second;
    const uint32_t i = (blockIdx.x - (is_first ? 0u : first_blocks)) * 256u + threadIdx.x;
    if (i >= j.pieces) return;
    const uint32_t r = fast_div(i, j.per_row), at = (i - r * j.per_row.d) * 32u;
    const char *p = j.src + (int64_t)r * j.ld + at;
    char *d = j.dst + (int64_t)r * j.dst_bytes + at;
    const int exist = j.bytes - (int)at;
    GrpPair<false> w;
    if (exist >= 32) {
        w.load(p);
    } else {
        const char *dword = (const char *)((uintptr_t)p & ~(uintptr_t)3);
        uint32_t v[9];
#pragma unroll
        for (int q = 0; q < 9; ++q) v[q] = dword + q * 4 < p + exist ? *(const uint32_t *)(dword + q * 4) : 0u;
        w.lo = (u32x4_t){v[0], v[1], v[2], v[3]};
        w.hi = (u32x4_t){v[4], v[5], v[6], v[7]};
        w.more = v[8];
    }
    u32x4_t v[2] = {w.chunk(0, (uint32_t)(uintptr_t)p), w.chunk(1, (uint32_t)(uintptr_t)p)};
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const int left = exist - q * 4;                    // bytes of this dword that exist
        v[q / 4][q % 4] = left >= 4 ? v[q / 4][q % 4] : left > 0 ? v[q / 4][q % 4] & ((1u << left * 8) - 1u) : 0u;
    }
    *(u32x4_t *)d = v[0];
    if ((int)at + 16 < j.dst_bytes) *(u32x4_t *)(d + 16) = v[1];
}

struct Matrix {
    const void **p;                        // where the problem keeps it
    int64_t *ld;
    int64_t rows, bytes;                   // rows, and bytes of each that exist
    int64_t packed() const { return (bytes + 15) / 16 * 16; }
    int64_t size() const { return rows * packed(); }
    int64_t pieces() const { return rows * ((packed() + 31) / 32); }
    bool whole() const { return ((uint64_t)*p | (uint64_t)*ld | (uint64_t)bytes) % 16 == 0; }
};

// The operands as matrices of `form`.
void matrices(int form, int es, GroupedParams &p, Matrix &a, Matrix &b)
{
    a = {&p.a, &p.lda, form == kWeights ? p.red : p.rows, (int64_t)(form == kWeights ? p.rows : p.red) * es};
    b = {&p.b, &p.ldb, form == kWeights ? p.red : (int64_t)p.groups * (form == kForward ? p.cols : p.red), (int64_t)(form == kForward ? p.red : p.cols) * es};
}

// Bytes for operands laid out anew, 0 where that does not pay: the copy is held against what the kernels for whole chunks take for the reduction.  8191 x
// 8191 x 8191 in 8 bits takes 500 us so, 852 in the kernel for any alignment; 5000 rows of 5 experts, 2047 x 4095 bf16, by the rows 126 and 137
// (the copy 0.62 of the other's time, the forward product's 0.73: 145 and 147), 1497 x 3424 x 1117 (0.56) 40 and 32.  By the weights a group's length is
// the reduction, and uneven groups cost the kernel for any alignment more: 4685 rows of 24 experts, 91 x 2432, 17.6 and 23.1 (0.59); 5000 rows of 5
// 133 and 148 (0.45); 3424 x 1117 of 1497 rows 27.3 and 25.7 (0.28).
size_t pack_bytes(int form, int dtype, GroupedParams &p)
{
    if (dtype == ALT_F32 || p.rows == 0 || p.red == 0) return 0;
    if (form == kForward && grp_is_few(p, dtype == ALT_I8 ? 1 : 2)) return 0;
    if (form == kInput && grp_is_few_dx(p, 2)) return 0;
    const int es = dtype == ALT_I8 ? 1 : 2;
    Matrix a, b;
    matrices(form, es, p, a, b);
    size_t need = 0;
    double cost = 0;
    for (const Matrix *m : {&a, &b})
        if (!m->whole()) {
            if (m->packed() > (1 << 22) || m->rows > (1 << 30) || m->pieces() > (1 << 30)) return 0;
            need += (size_t)m->size();
            cost += 2.0 + 2.0 * (double)m->size() / 4.5e6;
        }
    GrpTime t;
    if (form == kForward) grp_choose<kForward>(p, es, &t);
    else if (form == kInput) grp_choose<kInput>(p, es, &t);
    else grp_choose<kWeights>(p, es, &t);
    return cost < (form == kWeights ? 0.8 : 0.55) * t.reduction ? need : 0;
}

hipError_t pack(Matrix &a, Matrix &b, char *to, hipStream_t st)
{
    PackJob jobs[2] = {};
    uint32_t blocks[2] = {0, 0};
    int n = 0;
    for (Matrix *m : {&a, &b})
        if (!m->whole()) {
            jobs[n] = {(const char *)*m->p, to, *m->ld, (int)m->bytes, (int)m->packed(), (uint32_t)m->pieces(), make_fastdiv((uint32_t)((m->packed() + 31) / 32))};
            blocks[n++] = ((uint32_t)m->pieces() + 255) / 256;
            *m->p = to;
            *m->ld = m->packed();
            to += m->size();
        }
    hipLaunchKernelGGL(grp_pack_kernel, dim3(blocks[0] + blocks[1]), dim3(256), 0, st, jobs[0], jobs[1], blocks[0]);
    return hipGetLastError();
}

// What the problem takes of its operands' and outputs' extents, strides in bytes.
GroupedParams problem(alt_handle_t h, const alt_grouped_desc_t &l, int form, const void *a, const void *b, void *y)
{
    const int64_t es = (int64_t)in_size(l.in_dtype), os = (int64_t)dtype_size(l.out_dtype), lda = l.lda * es, ldb = l.ldb * es, ldc = l.ldc * es;
    GroupedParams p{};
    p.a = a; p.b = b; p.y = y;
    p.groups = l.groups;
    p.places = h->compute_units;
    p.flags = l.out_dtype == ALT_BF16 ? kGrpOutBf16 : 0;
    p.rows = (int32_t)(form == kWeights ? l.N : l.rows);
    p.cols = (int32_t)(form == kForward ? l.N : l.K);
    p.red = (int32_t)(form == kForward ? l.K : form == kInput ? l.N : l.rows);
    p.lda = form == kForward ? lda : ldc;
    p.ldb = form == kWeights ? lda : ldb;
    p.ldy = (form == kForward ? l.ldc : form == kInput ? l.lda : l.ldb) * os;
    p.ldmask = form == kInput ? lda : 0;
    p.y_group = form == kWeights ? l.N * l.ldb * os : 0;
    if (p.cols % (os == 2 ? 8 : 4) == 0) p.flags |= kGrpWhole;
    return p;
}

alt_status_t run(alt_handle_t h, const char *call, int dtype, int form, GroupedParams &p, void *workspace, size_t ws_bytes, hipStream_t st)
{
    if (workspace && ws_bytes) {
        const uintptr_t ws = ((uintptr_t)workspace + 15) / 16 * 16;
        const size_t need = pack_bytes(form, dtype, p);
        if (need && need + (ws - (uintptr_t)workspace) <= ws_bytes) {
            Matrix a, b;
            matrices(form, dtype == ALT_I8 ? 1 : 2, p, a, b);
            ALT_CHECK_HIP(h, pack(a, b, (char *)ws, st));
            p.flags |= kGrpPacked;
        }
    }
    p.b_group = form == kWeights ? 0 : (int64_t)(form == kForward ? p.cols : p.red) * p.ldb;
    const hipError_t e = p.adapter ? (dtype == ALT_BF16 ? grouped_run_adapted_bf16(p, st) : grouped_run_adapted_f32(p, st)) : dtype == ALT_I8 ? grouped_run_i8(p, st) : dtype == ALT_BF16 ? grouped_run_bf16(form, p, st) : grouped_run_f32(form, p, st);
    if (e == hipErrorInvalidConfiguration) return fail(h, ALT_UNSUPPORTED, "%s: more output tiles than a launch holds", call);
    ALT_CHECK_HIP(h, e);
    return ALT_OK;
}

alt_status_t workspace_size(alt_handle_t h, const alt_grouped_desc_t *d, int form, bool one_group, const char *call, size_t *bytes)
{
    alt_grouped_desc_t l;
    const alt_status_t s = check_layer(h, call, d, form != kForward, &l);
    if (s != ALT_OK) return s;
    if (!bytes) return fail(h, ALT_INVALID_ARG, "%s: null result", call);
    // (buffers that start at whole chunks: what their rows do is known here)
    GroupedParams p = problem(h, l, form, nullptr, nullptr, nullptr);
    p.offsets = one_group ? nullptr : (const int32_t *)16;                  // (asked for, not read)
    if (p.places == 0) p.places = 256;
    const size_t need = pack_bytes(form, l.in_dtype, p);
    *bytes = need ? need + 16 : 0;                         // (a workspace may start anywhere)
    return ALT_OK;
}

alt_status_t forward(alt_handle_t h, const char *call, const alt_grouped_desc_t &l, const void *a, const float *a_scale, const void *b, const float *b_scale,
                     const float *bias, const int32_t *offsets, void *y, void *workspace, size_t ws_bytes, void *stream)
{
    GroupedParams p = problem(h, l, kForward, a, b, y);
    p.a_scale = a_scale;
    p.b_scale = b_scale;
    p.bias = l.epilogue & ALT_EPI_BIAS ? bias : nullptr;
    p.offsets = offsets;
    if (l.epilogue & ALT_EPI_RELU) p.flags |= kGrpRelu;
    return run(h, call, l.in_dtype, kForward, p, workspace, ws_bytes, (hipStream_t)stream);
}

// A product with adapters as a layer of one group.
alt_grouped_desc_t one_group(const alt_adapters_desc_t *d)
{
    alt_grouped_desc_t g{};
    g.rows = d->M; g.N = d->N; g.K = d->K;
    g.lda = d->lda; g.ldb = d->ldb; g.ldc = d->ldc;
    g.groups = 1;
    g.in_dtype = d->in_dtype; g.out_dtype = d->out_dtype; g.epilogue = d->epilogue;
    return g;
}

alt_status_t check_adapters(alt_handle_t h, const char *call, const alt_adapters_desc_t *d, alt_grouped_desc_t *out)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "%s: null descriptor", call);
    if (d->in_dtype == ALT_I8) return fail(h, ALT_INVALID_ARG, "%s: bad in_dtype", call);
    const alt_grouped_desc_t g = one_group(d);
    const alt_status_t s = check_layer(h, call, &g, false, out);
    if (s != ALT_OK) return s;
    if (d->adapters < 1 || d->rank < 1) return fail(h, ALT_INVALID_ARG, "%s: bad size", call);
    if (d->N > (1 << 24) || d->adapters > (1 << 20) || d->rank > ALT_ADAPTERS_MAX_RANK)
        return fail(h, ALT_UNSUPPORTED, "%s: more than 2^24 columns, 2^20 adapters or a rank over %d", call, ALT_ADAPTERS_MAX_RANK);
    return ALT_OK;
}

// A product with adapters as both of its parts see it, and the layout of its workspace: inner sums, where the product goes beside them its fp32 results, and
// operands laid out anew.
struct AdapterCall {
    GroupedParams product;
    AdapterParams adapters;
    size_t inner, base, pack;
};

AdapterCall adapter_call(alt_handle_t h, const alt_adapters_desc_t *d, const alt_grouped_desc_t &l, const void *x, const void *w, void *y)
{
    AdapterCall c{};
    GroupedParams &p = c.product;
    p = problem(h, l, kForward, x, w, y);
    if (p.places == 0) p.places = 256;
    AdapterParams &q = c.adapters;
    q.x = (const char *)x;
    q.w = (const char *)w;
    q.ldw = p.ldb;
    q.y = (char *)y;
    q.ldx = p.lda;
    q.ldy = p.ldy;
    q.rows = p.rows; q.cols = p.cols; q.K = p.red;
    q.rank = d->rank; q.adapters = d->adapters; q.places = p.places;
    q.relu = (l.epilogue & ALT_EPI_RELU) != 0;
    q.out_bf16 = l.out_dtype == ALT_BF16;
    adapters_plan(l.in_dtype, p, q);
    c.inner = adapters_inner_bytes(l.in_dtype, q);
    c.base = q.beside ? (size_t)q.base_slices * l.rows * l.N * 4 : 0;
    if (q.beside) {                                        // the product's results: dense fp32
        p.ldy = l.N * 4;
        p.flags = l.N % 4 == 0 ? kGrpWhole : 0;
    } else {
        p.rank = d->rank;
        p.adapters = d->adapters;
        p.inner_bytes = q.inner_bytes;
        if (q.relu) p.flags |= kGrpRelu;
    }
    c.pack = q.few ? 0 : pack_bytes(kForward, l.in_dtype, p);
    return c;
}

// What there is of the workspace beside operands that are laid out anew, which may be left as they are.
size_t adapters_need(const AdapterCall &c) { return c.inner + (c.base + 15) / 16 * 16 + 16; }

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
    if (l.rows == 0) return ALT_OK;
    const size_t es = in_size(l.in_dtype);
    const bool scaled = l.in_dtype == ALT_I8;
    s = check_layer_buffers(h, "alt_gemm_grouped", {{"a", a, es}, {"b", b, es}, {"offsets", offsets, 4}, {"y", y, dtype_size(l.out_dtype)}, {"a_scale", a_scale, 4, scaled},
                                              {"b_scale", b_scale, 4, scaled}, {"bias", bias, 4, (l.epilogue & ALT_EPI_BIAS) != 0}});
    if (s != ALT_OK) return s;
    return forward(h, "alt_gemm_grouped", l, a, a_scale, b, b_scale, bias, offsets, y, workspace, ws_bytes, stream);
}

extern "C" alt_status_t alt_gemm_grouped_dx(alt_handle_t h, const alt_grouped_desc_t *d, const void *dy, const void *b, const void *relu_of, const int32_t *offsets,
                                            void *dx, void *workspace, size_t ws_bytes, void *stream)
{
    alt_grouped_desc_t l;
    alt_status_t s = check_layer(h, "alt_gemm_grouped_dx", d, true, &l);
    if (s != ALT_OK) return s;
    if (l.epilogue & ALT_EPI_BIAS) return fail(h, ALT_INVALID_ARG, "alt_gemm_grouped_dx: a bias has no part in the gradient of x");
    if (l.rows == 0) return ALT_OK;
    const size_t es = in_size(l.in_dtype);
    s = check_layer_buffers(h, "alt_gemm_grouped_dx", {{"dy", dy, es}, {"b", b, es}, {"offsets", offsets, 4}, {"dx", dx, dtype_size(l.out_dtype)},
                                                 {"relu_of", relu_of, es, (l.epilogue & ALT_EPI_RELU) != 0}});
    if (s != ALT_OK) return s;
    GroupedParams p = problem(h, l, kInput, dy, b, dx);
    p.offsets = offsets;
    p.mask = relu_of;
    if (l.epilogue & ALT_EPI_RELU) p.flags |= kGrpMask;
    return run(h, "alt_gemm_grouped_dx", l.in_dtype, kInput, p, workspace, ws_bytes, (hipStream_t)stream);
}

extern "C" alt_status_t alt_gemm_grouped_dw(alt_handle_t h, const alt_grouped_desc_t *d, const void *a, const void *dy, const int32_t *offsets, void *dw, float *dbias,
                                            void *workspace, size_t ws_bytes, void *stream)
{
    alt_grouped_desc_t l;
    alt_status_t s = check_layer(h, "alt_gemm_grouped_dw", d, true, &l);
    if (s != ALT_OK) return s;
    if (l.epilogue & ALT_EPI_RELU) return fail(h, ALT_INVALID_ARG, "alt_gemm_grouped_dw: dy is the gradient before the ReLU");
    const size_t es = in_size(l.in_dtype);
    // (without rows the gradients are zeros, and a and dy need not exist)
    s = check_layer_buffers(h, "alt_gemm_grouped_dw", {{"a", a, es, l.rows > 0}, {"dy", dy, es, l.rows > 0}, {"offsets", offsets, 4},
                                                 {"dw", dw, dtype_size(l.out_dtype)}, {"dbias", dbias, 4, (l.epilogue & ALT_EPI_BIAS) != 0}});
    if (s != ALT_OK) return s;
    GroupedParams p = problem(h, l, kWeights, dy, a, dw);
    p.offsets = offsets;
    p.colsum = l.epilogue & ALT_EPI_BIAS ? dbias : nullptr;
    return run(h, "alt_gemm_grouped_dw", l.in_dtype, kWeights, p, workspace, ws_bytes, (hipStream_t)stream);
}

extern "C" alt_status_t alt_gemm_grouped_workspace_size(alt_handle_t h, const alt_grouped_desc_t *d, size_t *bytes)
{
    return workspace_size(h, d, kForward, false, "alt_gemm_grouped_workspace_size", bytes);
}

extern "C" alt_status_t alt_gemm_grouped_dx_workspace_size(alt_handle_t h, const alt_grouped_desc_t *d, size_t *bytes)
{
    return workspace_size(h, d, kInput, false, "alt_gemm_grouped_dx_workspace_size", bytes);
}

extern "C" alt_status_t alt_gemm_grouped_dw_workspace_size(alt_handle_t h, const alt_grouped_desc_t *d, size_t *bytes)
{
    return workspace_size(h, d, kWeights, false, "alt_gemm_grouped_dw_workspace_size", bytes);
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
    if (l.rows == 0) return ALT_OK;
    s = check_layer_buffers(h, "alt_gemm_i8", {{"a", a, 1}, {"b", b, 1}, {"a_scale", a_scale, 4}, {"b_scale", b_scale, 4}, {"y", y, dtype_size(l.out_dtype)},
                                         {"bias", bias, 4, (l.epilogue & ALT_EPI_BIAS) != 0}});
    if (s != ALT_OK) return s;
    return forward(h, "alt_gemm_i8", l, a, a_scale, b, b_scale, bias, nullptr, y, workspace, ws_bytes, stream);
}

extern "C" alt_status_t alt_gemm_i8_workspace_size(alt_handle_t h, const alt_gemm_i8_desc_t *d, size_t *bytes)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "alt_gemm_i8_workspace_size: null descriptor");
    const alt_grouped_desc_t g = one_group(d);
    return workspace_size(h, &g, kForward, true, "alt_gemm_i8_workspace_size", bytes);
}

extern "C" alt_status_t alt_gemm_adapters(alt_handle_t h, const alt_adapters_desc_t *d, const void *x, const void *w, const int32_t *adapter, const void *a, const void *b,
                                          const float *scale, const float *bias, void *y, void *workspace, size_t ws_bytes, void *stream)
{
    alt_grouped_desc_t l;
    alt_status_t s = check_adapters(h, "alt_gemm_adapters", d, &l);
    if (s != ALT_OK) return s;
    if (l.rows == 0) return ALT_OK;
    const size_t es = in_size(l.in_dtype);
    s = check_buffers(h, "alt_gemm_adapters", {{"x", x, es}, {"w", w, es}, {"adapter", adapter, 4}, {"a", a, es}, {"b", b, es}, {"scale", scale, 4, scale != nullptr},
                                               {"bias", bias, 4, (l.epilogue & ALT_EPI_BIAS) != 0}, {"y", y, dtype_size(l.out_dtype)}});
    if (s != ALT_OK) return s;
    AdapterCall c = adapter_call(h, d, l, x, w, y);
    s = check_workspace(h, "alt_gemm_adapters", workspace, ws_bytes, adapters_need(c));
    if (s == ALT_OK) s = check_device(h, "alt_gemm_adapters");
    if (s != ALT_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    char *ws = aligned_workspace(workspace);
    AdapterParams &q = c.adapters;
    GroupedParams &p = c.product;
    q.a = (const char *)a;
    q.b = (const char *)b;
    q.adapter = adapter;
    q.scale = scale;
    q.bias = l.epilogue & ALT_EPI_BIAS ? bias : nullptr;
    q.inner = ws;
    if (q.beside) {
        q.base = (float *)(ws + c.inner);
        p.y = ws + c.inner;
    } else {
        p.bias = q.bias;
        p.adapter = adapter;
        p.inner = ws;
        p.up = (const char *)b;
    }
    hipError_t e = q.few ? adapters_few(l.in_dtype, q, st) : adapters_down(l.in_dtype, q, st);
    if (e == hipSuccess && !q.few) {
        char *more = ws + c.inner + (c.base + 15) / 16 * 16;
        s = run(h, "alt_gemm_adapters", l.in_dtype, kForward, p, more, (size_t)((char *)workspace + ws_bytes - more), st);
        if (s != ALT_OK) return s;
    }
    if (e == hipSuccess && q.beside) e = adapters_up(l.in_dtype, q, st);
    if (e == hipErrorInvalidConfiguration) return fail(h, ALT_UNSUPPORTED, "alt_gemm_adapters: more workgroups than a launch holds");
    ALT_CHECK_HIP(h, e);
    return ALT_OK;
}

extern "C" alt_status_t alt_gemm_adapters_workspace_size(alt_handle_t h, const alt_adapters_desc_t *d, size_t *bytes)
{
    alt_grouped_desc_t l;
    const alt_status_t s = check_adapters(h, "alt_gemm_adapters_workspace_size", d, &l);
    if (s != ALT_OK) return s;
    if (!bytes) return fail(h, ALT_INVALID_ARG, "alt_gemm_adapters_workspace_size: null result");
    if (l.rows == 0) {
        *bytes = 0;
        return ALT_OK;
    }
    const AdapterCall c = adapter_call(h, d, l, nullptr, nullptr, nullptr);
    *bytes = adapters_need(c) + (c.pack ? c.pack + 16 : 0);
    return ALT_OK;
}
