// Rows from the tokens' order into the experts' and back, with the gradients.
//
//   dispatch  y[rows[t][j]] = x[t];   combine  y[t] = sum_j w[t][j] x[rows[t][j]]
//   gradients of combine  dx[rows[t][j]] = w[t][j] dy[t],  dw[t][j] = sum_c dy[t,c] x[rows[t][j],c]
//
// Bound by memory.  A workgroup has a token, so that the token's row is read or written once.
#include "common.h"
#include "rows.h"

namespace alt {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kMaxTop = ALT_ROUTE_MAX_TOP_K;

struct ExchangeParams {
    const char *x, *dy;
    const int32_t *rows;
    const float *weights;
    char *y;
    float *dweights;
    int64_t ldt, ldr;                      // bytes between rows of the tokens' order, of the experts'
    int32_t tokens, num, top_k, cols;              // num: rows of the experts' order
};

__device__ __forceinline__ int row_of(const ExchangeParams &p, int64_t slot)
{
    const int r = p.rows[slot];
    return r >= 0 && r < p.num ? r : -1;
}

template <int ES>
__global__ __launch_bounds__(kThreads) void dispatch_kernel(const ExchangeParams p)
{
    for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x)
    for (int c = threadIdx.x; c < p.cols; c += kThreads) {
        const float v = element<ES>(p.x + t * p.ldt + (int64_t)c * ES);
        for (int j = 0; j < p.top_k; ++j) {
            const int r = row_of(p, t * p.top_k + j);
            if (r >= 0) store_element<ES>(p.y + r * p.ldr + (int64_t)c * ES, v);
        }
    }
}

template <int ES>
__global__ __launch_bounds__(kThreads) void combine_kernel(const ExchangeParams p)
{
    for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x)
    for (int c = threadIdx.x; c < p.cols; c += kThreads) {
        float s = 0.f;
        for (int j = 0; j < p.top_k; ++j) {
            const int r = row_of(p, t * p.top_k + j);
            s += (p.weights ? p.weights[t * p.top_k + j] : 1.f) * (r >= 0 ? element<ES>(p.x + r * p.ldr + (int64_t)c * ES) : 0.f);
        }
        store_element<ES>(p.y + t * p.ldt + (int64_t)c * ES, s);
    }
}

template <int ES>
__global__ __launch_bounds__(kThreads) void combine_grad_kernel(const ExchangeParams p)
{
    __shared__ float part[kWaves];
    for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x)
    for (int j = 0; j < p.top_k; ++j) {
        const int64_t slot = t * p.top_k + j;
        const int r = row_of(p, slot);
        const float w = p.weights ? p.weights[slot] : 1.f;
        float s = 0.f;
        if (r >= 0)
            for (int c = threadIdx.x; c < p.cols; c += kThreads) {
                const float g = element<ES>(p.dy + t * p.ldt + (int64_t)c * ES);
                store_element<ES>(p.y + r * p.ldr + (int64_t)c * ES, w * g);
                if (p.dweights) s += g * element<ES>(p.x + r * p.ldr + (int64_t)c * ES);
            }
        if (!p.dweights) continue;
        s = wave_sum(s);
        __syncthreads();
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
        __syncthreads();
        if (threadIdx.x == 0) p.dweights[slot] = part[0] + part[1] + part[2] + part[3];
    }
}

alt_status_t check(alt_handle_t h, const char *call, const alt_exchange_desc_t *d, alt_exchange_desc_t *out)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "%s: null descriptor", call);
    *out = *d;
    if (d->tokens < 0 || d->rows < 0 || d->cols < 1 || d->token_stride < 0 || d->row_stride < 0 || d->top_k < 1) return fail(h, ALT_INVALID_ARG, "%s: bad size", call);
    if (d->dtype != ALT_F32 && d->dtype != ALT_BF16) return fail(h, ALT_INVALID_ARG, "%s: bad dtype", call);
    if (!out->token_stride) out->token_stride = d->cols;
    if (!out->row_stride) out->row_stride = d->cols;
    if (out->token_stride < d->cols || out->row_stride < d->cols) return fail(h, ALT_SHAPE_MISMATCH, "%s: a row stride is shorter than a row", call);
    if (d->top_k > kMaxTop) return fail(h, ALT_UNSUPPORTED, "%s: more than %d choices", call, kMaxTop);
    if (d->tokens > (1 << 30) / d->top_k || d->rows > (1 << 30) || d->cols > (1 << 24) || out->token_stride > 0x7fffffff || out->row_stride > 0x7fffffff)
        return fail(h, ALT_UNSUPPORTED, "%s: more than 2^30 choices or rows, 2^24 columns or a stride over 2^31", call);
    return ALT_OK;
}

ExchangeParams params(const alt_exchange_desc_t &d, const int32_t *rows, const float *weights)
{
    const int64_t es = (int64_t)dtype_size(d.dtype);
    ExchangeParams p{};
    p.rows = rows;
    p.weights = weights;
    p.ldt = d.token_stride * es;
    p.ldr = d.row_stride * es;
    p.num = (int32_t)d.rows;
    p.tokens = (int32_t)d.tokens;
    p.top_k = d.top_k;
    p.cols = (int32_t)d.cols;
    return p;
}

#define LAUNCH(kernel)                                                                                                                  \
    do {                                                                                                                                \
        if (d.dtype == ALT_F32) hipLaunchKernelGGL(kernel<4>, dim3((unsigned)std::min<int64_t>(d.tokens, 1 << 20)), dim3(kThreads), 0, (hipStream_t)stream, p);      \
        else hipLaunchKernelGGL(kernel<2>, dim3((unsigned)std::min<int64_t>(d.tokens, 1 << 20)), dim3(kThreads), 0, (hipStream_t)stream, p);                         \
        ALT_CHECK_HIP(h, hipGetLastError());                                                                                            \
    } while (0)

}  // namespace
}  // namespace alt

using namespace alt;

extern "C" alt_status_t alt_dispatch_rows(alt_handle_t h, const alt_exchange_desc_t *desc, const void *x, const int32_t *rows, void *y, void *stream)
{
    alt_exchange_desc_t d;
    alt_status_t s = check(h, "alt_dispatch_rows", desc, &d);
    if (s != ALT_OK) return s;
    if (d.tokens == 0 || d.rows == 0) return ALT_OK;
    const size_t es = dtype_size(d.dtype);
    s = check_buffers(h, "alt_dispatch_rows", {{"x", x, es}, {"rows", rows, 4}, {"y", y, es}});
    if (s == ALT_OK) s = check_device(h, "alt_dispatch_rows");
    if (s != ALT_OK) return s;
    ExchangeParams p = params(d, rows, nullptr);
    p.x = (const char *)x;
    p.y = (char *)y;
    LAUNCH(dispatch_kernel);
    return ALT_OK;
}

extern "C" alt_status_t alt_combine_rows(alt_handle_t h, const alt_exchange_desc_t *desc, const void *x, const int32_t *rows, const float *weights, void *y, void *stream)
{
    alt_exchange_desc_t d;
    alt_status_t s = check(h, "alt_combine_rows", desc, &d);
    if (s != ALT_OK) return s;
    if (d.tokens == 0) return ALT_OK;
    const size_t es = dtype_size(d.dtype);
    s = check_buffers(h, "alt_combine_rows", {{"x", x, es, d.rows > 0}, {"rows", rows, 4}, {"weights", weights, 4, weights != nullptr}, {"y", y, es}});
    if (s == ALT_OK) s = check_device(h, "alt_combine_rows");
    if (s != ALT_OK) return s;
    ExchangeParams p = params(d, rows, weights);
    p.x = (const char *)x;
    p.y = (char *)y;
    LAUNCH(combine_kernel);
    return ALT_OK;
}

extern "C" alt_status_t alt_combine_rows_grad(alt_handle_t h, const alt_exchange_desc_t *desc, const void *dy, const void *x, const int32_t *rows, const float *weights, void *dx,
                                              float *dweights, void *stream)
{
    alt_exchange_desc_t d;
    alt_status_t s = check(h, "alt_combine_rows_grad", desc, &d);
    if (s != ALT_OK) return s;
    if (d.tokens == 0) return ALT_OK;
    const size_t es = dtype_size(d.dtype);
    s = check_buffers(h, "alt_combine_rows_grad", {{"dy", dy, es}, {"x", x, es, d.rows > 0 && dweights}, {"rows", rows, 4}, {"weights", weights, 4, weights != nullptr},
                                                   {"dx", dx, es, d.rows > 0}, {"dweights", dweights, 4, dweights != nullptr}});
    if (s == ALT_OK) s = check_device(h, "alt_combine_rows_grad");
    if (s != ALT_OK) return s;
    ExchangeParams p = params(d, rows, weights);
    p.dy = (const char *)dy;
    p.x = (const char *)x;
    p.y = (char *)dx;
    p.dweights = dweights;
    LAUNCH(combine_grad_kernel);
    return ALT_OK;
}
