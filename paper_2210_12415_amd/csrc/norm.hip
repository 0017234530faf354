// Layer norm of rows and its gradients.
//
//   mean = sum_c x / cols,  rstd = 1 / sqrt(sum_c (x - mean)^2 / cols + eps),  u = (x - mean) rstd,  y = u gamma + beta
//   dx = rstd (g - mean_c(g) - u mean_c(g u))  with g = dy gamma,  dgamma = sum_m dy u,  dbeta = sum_m dy
//
// Bound by memory: forward reads x and writes y, backward reads dy and x and writes dx.
#include "common.h"
#include "rows.h"

namespace alt {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// The sum over a workgroup's threads, the same in all of them.
__device__ __forceinline__ float block_sum(float v, float (&part)[kWaves])
{
    v = wave_sum(v);
    __syncthreads();                                       // (the last sum is read)
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) v += part[i];
    return v;
}

template <int XS, int YS>
__global__ __launch_bounds__(kThreads) void norm_kernel(const char *x0, int64_t ldx, const float *gamma, const float *beta, char *y0, int64_t ldy, float *mean_out, float *rstd_out,
                                                        int64_t rows, int cols, float eps)
{
    __shared__ float part[kWaves];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const char *x = x0 + row * ldx;
    char *y = y0 + row * ldy;
    float s = 0.f;
    for (int c = threadIdx.x; c < cols; c += kThreads) s += element<XS>(x + (int64_t)c * XS);
    const float mean = block_sum(s, part) / (float)cols;
    s = 0.f;
    for (int c = threadIdx.x; c < cols; c += kThreads) {
        const float v = element<XS>(x + (int64_t)c * XS) - mean;
        s += v * v;
    }
    const float rstd = 1.f / sqrtf(block_sum(s, part) / (float)cols + eps);
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[row] = mean;
        if (rstd_out) rstd_out[row] = rstd;
    }
    for (int c = threadIdx.x; c < cols; c += kThreads)
        store_element<YS>(y + (int64_t)c * YS, (element<XS>(x + (int64_t)c * XS) - mean) * rstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f));
    }
}

template <int XS, int YS>
__global__ __launch_bounds__(kThreads) void norm_dx_kernel(const char *dy0, int64_t ldy, const char *x0, int64_t ldx, const float *mean_in, const float *rstd_in, const float *gamma,
                                                           char *dx0, int64_t rows, int cols)
{
    __shared__ float part[kWaves];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const char *dy = dy0 + row * ldy, *x = x0 + row * ldx;
    char *dx = dx0 + row * ldx;
    const float mean = mean_in[row], rstd = rstd_in[row];
    float sg = 0.f, sgu = 0.f;
    for (int c = threadIdx.x; c < cols; c += kThreads) {
        const float g = element<YS>(dy + (int64_t)c * YS) * (gamma ? gamma[c] : 1.f);
        sg += g;
        sgu += g * ((element<XS>(x + (int64_t)c * XS) - mean) * rstd);
    }
    sg = block_sum(sg, part) / (float)cols;
    sgu = block_sum(sgu, part) / (float)cols;
    for (int c = threadIdx.x; c < cols; c += kThreads) {
        const float g = element<YS>(dy + (int64_t)c * YS) * (gamma ? gamma[c] : 1.f), u = (element<XS>(x + (int64_t)c * XS) - mean) * rstd;
        store_element<XS>(dx + (int64_t)c * XS, rstd * (g - sg - u * sgu));
    }
    }
}

// dgamma and dbeta: a workgroup's columns over its share of the rows, then the shares one after another.
template <int XS, int YS>
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(const char *dy, int64_t ldy, const char *x, int64_t ldx, const float *mean, const float *rstd, float *part,
                                                                int64_t rows, int cols)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= cols) return;
    float dg = 0.f, db = 0.f;
    for (int64_t m = blockIdx.y; m < rows; m += gridDim.y) {
        const float v = element<YS>(dy + m * ldy + (int64_t)c * YS);
        dg += v * ((element<XS>(x + m * ldx + (int64_t)c * XS) - mean[m]) * rstd[m]);
        db += v;
    }
    part[(int64_t)blockIdx.y * 2 * cols + c] = dg;
    part[((int64_t)blockIdx.y * 2 + 1) * cols + c] = db;
}

__global__ __launch_bounds__(kThreads) void norm_join_kernel(const float *part, int shares, int cols, float *dgamma, float *dbeta)
{
    const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (c >= 2 * (int64_t)cols) return;
    float s = 0.f;
    for (int i = 0; i < shares; ++i) s += part[(int64_t)i * 2 * cols + c];
    float *to = c < cols ? dgamma : dbeta;
    if (to) to[c < cols ? c : c - cols] = s;
}

unsigned row_blocks(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 1 << 20); }
int column_shares(int64_t rows) { return (int)std::min<int64_t>(rows, 64); }

// What both directions check, dense strides filled in.
alt_status_t check(alt_handle_t h, const char *call, const alt_norm_desc_t *d, alt_norm_desc_t *out)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "%s: null descriptor", call);
    *out = *d;
    if (d->rows < 0 || d->cols < 1 || d->x_stride < 0 || d->y_stride < 0) return fail(h, ALT_INVALID_ARG, "%s: bad size", call);
    if (d->in_dtype != ALT_F32 && d->in_dtype != ALT_BF16) return fail(h, ALT_INVALID_ARG, "%s: bad in_dtype", call);
    if (d->out_dtype != ALT_F32 && d->out_dtype != ALT_BF16) return fail(h, ALT_INVALID_ARG, "%s: bad out_dtype", call);
    if (!(d->eps >= 0.f)) return fail(h, ALT_INVALID_ARG, "%s: eps is negative or NaN", call);
    if (!out->x_stride) out->x_stride = d->cols;
    if (!out->y_stride) out->y_stride = d->cols;
    if (out->x_stride < d->cols || out->y_stride < d->cols) return fail(h, ALT_SHAPE_MISMATCH, "%s: a row stride is shorter than a row", call);
    if (d->rows > (1 << 30) || d->cols > (1 << 24) || out->x_stride > 0x7fffffff || out->y_stride > 0x7fffffff)
        return fail(h, ALT_UNSUPPORTED, "%s: more than 2^30 rows, 2^24 columns or a stride over 2^31", call);
    return ALT_OK;
}

size_t grad_workspace(const alt_norm_desc_t &d) { return d.rows ? (size_t)column_shares(d.rows) * 2 * d.cols * 4 + 16 : 0; }

template <int XS, int YS>
void forward_run(const alt_norm_desc_t &d, const void *x, const float *gamma, const float *beta, void *y, float *mean, float *rstd, hipStream_t st)
{
    hipLaunchKernelGGL((norm_kernel<XS, YS>), dim3(row_blocks(d.rows)), dim3(kThreads), 0, st, (const char *)x, d.x_stride * XS, gamma, beta, (char *)y, d.y_stride * YS, mean,
                       rstd, d.rows, (int)d.cols, d.eps);
}

template <int XS, int YS>
void grad_run(const alt_norm_desc_t &d, const void *dy, const void *x, const float *mean, const float *rstd, const float *gamma, void *dx, float *dgamma, float *dbeta, float *part,
              hipStream_t st)
{
    if (d.rows)
        hipLaunchKernelGGL((norm_dx_kernel<XS, YS>), dim3(row_blocks(d.rows)), dim3(kThreads), 0, st, (const char *)dy, d.y_stride * YS, (const char *)x, d.x_stride * XS, mean, rstd,
                           gamma, (char *)dx, d.rows, (int)d.cols);
    if (!dgamma && !dbeta) return;
    const int shares = column_shares(d.rows);
    if (d.rows)
        hipLaunchKernelGGL((norm_columns_kernel<XS, YS>), dim3((unsigned)((d.cols + kThreads - 1) / kThreads), (unsigned)shares), dim3(kThreads), 0, st, (const char *)dy,
                           d.y_stride * YS, (const char *)x, d.x_stride * XS, mean, rstd, part, d.rows, (int)d.cols);
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)((2 * d.cols + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, part, shares, (int)d.cols, dgamma, dbeta);
}

}  // namespace
}  // namespace alt

using namespace alt;

extern "C" alt_status_t alt_layer_norm(alt_handle_t h, const alt_norm_desc_t *desc, const void *x, const float *gamma, const float *beta, void *y, float *mean, float *rstd,
                                       void *stream)
{
    alt_norm_desc_t d;
    alt_status_t s = check(h, "alt_layer_norm", desc, &d);
    if (s != ALT_OK) return s;
    if (d.rows == 0) return ALT_OK;
    s = check_buffers(h, "alt_layer_norm", {{"x", x, dtype_size(d.in_dtype)}, {"y", y, dtype_size(d.out_dtype)}, {"gamma", gamma, 4, gamma != nullptr},
                                            {"beta", beta, 4, beta != nullptr}, {"mean", mean, 4, mean != nullptr}, {"rstd", rstd, 4, rstd != nullptr}});
    if (s == ALT_OK) s = check_device(h, "alt_layer_norm");
    if (s != ALT_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    if (d.in_dtype == ALT_F32) {
        if (d.out_dtype == ALT_F32) forward_run<4, 4>(d, x, gamma, beta, y, mean, rstd, st);
        else forward_run<4, 2>(d, x, gamma, beta, y, mean, rstd, st);
    } else {
        if (d.out_dtype == ALT_F32) forward_run<2, 4>(d, x, gamma, beta, y, mean, rstd, st);
        else forward_run<2, 2>(d, x, gamma, beta, y, mean, rstd, st);
    }
    ALT_CHECK_HIP(h, hipGetLastError());
    return ALT_OK;
}

extern "C" alt_status_t alt_layer_norm_grad(alt_handle_t h, const alt_norm_desc_t *desc, const void *dy, const void *x, const float *mean, const float *rstd, const float *gamma,
                                            void *dx, float *dgamma, float *dbeta, void *workspace, size_t ws_bytes, void *stream)
{
    alt_norm_desc_t d;
    alt_status_t s = check(h, "alt_layer_norm_grad", desc, &d);
    if (s != ALT_OK) return s;
    const bool rows = d.rows > 0, columns = dgamma || dbeta;
    if (!rows && !columns) return ALT_OK;
    s = check_buffers(h, "alt_layer_norm_grad", {{"dy", dy, dtype_size(d.out_dtype), rows}, {"x", x, dtype_size(d.in_dtype), rows}, {"mean", mean, 4, rows}, {"rstd", rstd, 4, rows},
                                                 {"gamma", gamma, 4, gamma != nullptr}, {"dx", dx, dtype_size(d.in_dtype), rows}, {"dgamma", dgamma, 4, dgamma != nullptr},
                                                 {"dbeta", dbeta, 4, dbeta != nullptr}});
    if (s == ALT_OK && columns) s = check_workspace(h, "alt_layer_norm_grad", workspace, ws_bytes, grad_workspace(d));
    if (s == ALT_OK) s = check_device(h, "alt_layer_norm_grad");
    if (s != ALT_OK) return s;
    float *part = columns && rows ? (float *)aligned_workspace(workspace) : nullptr;
    const hipStream_t st = (hipStream_t)stream;
    if (d.in_dtype == ALT_F32) {
        if (d.out_dtype == ALT_F32) grad_run<4, 4>(d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
        else grad_run<4, 2>(d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
    } else {
        if (d.out_dtype == ALT_F32) grad_run<2, 4>(d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
        else grad_run<2, 2>(d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
    }
    ALT_CHECK_HIP(h, hipGetLastError());
    return ALT_OK;
}

extern "C" alt_status_t alt_layer_norm_grad_workspace_size(alt_handle_t h, const alt_norm_desc_t *desc, size_t *bytes)
{
    alt_norm_desc_t d;
    const alt_status_t s = check(h, "alt_layer_norm_grad_workspace_size", desc, &d);
    if (s != ALT_OK) return s;
    if (!bytes) return fail(h, ALT_INVALID_ARG, "alt_layer_norm_grad_workspace_size: null result");
    *bytes = grad_workspace(d);
    return ALT_OK;
}
