// Rows from the tokens' order into the experts' and back, with the gradients.
//
//   dispatch  y[rows[t][j]] = x[t];   combine  y[t] = sum_j w[t][j] x[rows[t][j]]
//   gradients of combine  dx[rows[t][j]] = w[t][j] dy[t],  dw[t][j] = sum_c dy[t,c] x[rows[t][j],c]
//
// Bound by memory.  A thread moves a chunk of eight columns of one token, whatever the row's length (the row's last chunk may be a part of one), so
// that a token's row is read or written once; where a gradient needs sums over the row, a wave or a workgroup has a token.
#include "common.h"
#include "rows.h"

namespace alt {
namespace {

constexpr int kThreads = 256, kMaxTop = ALT_ROUTE_MAX_TOP_K;
constexpr int kBatch = 4;                                  // choices whose rows are on their way at once

struct ExchangeParams {
    const char *x, *dy;
    const int32_t *rows;
    const float *weights;
    char *y;
    float *dweights;
    int64_t ldt, ldr;                      // bytes between rows of the tokens' order, of the experts'
    int32_t tokens, num, top_k, cols;      // num: rows of the experts' order
    uint32_t items;                        // chunks of all tokens of a launch
    FastDiv chunks;                        // of a row, with its last part
};

__device__ __forceinline__ int row_of(const ExchangeParams &p, int64_t slot)
{
    const int r = p.rows[slot];
    return r >= 0 && r < p.num ? r : -1;
}

__device__ __forceinline__ w4_t load16(const char *at)
{
    w4_t c;
    __builtin_memcpy(&c, at, 16);
    return c;
}

// Where in a row chunk c lies: the last one ends with the row and begins inside the chunk before it, whose bytes it moves again, the same ones (a row of
// 515 fp32 columns in elements behind its last whole chunk took 7.0 us for 1501 tokens, so 5.1).  Rows shorter than a chunk have one, at 0.
template <int ES>
__device__ __forceinline__ int64_t part_at(const ExchangeParams &p, uint32_t c)
{
    return max(min((int64_t)c * 16, (int64_t)p.cols * ES - 16), (int64_t)0);
}

// Rows and weights of the choices j0, j0 + 1, ... of a token; -1 and 0 behind the last.
__device__ __forceinline__ void choices(const ExchangeParams &p, int64_t t, int j0, int (&r)[kBatch], float (&w)[kBatch])
{
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
        const bool is = j0 + j < p.top_k;
        const int64_t slot = t * p.top_k + j0 + j;
        r[j] = is ? row_of(p, slot) : -1;
        w[j] = !is ? 0.f : p.weights ? p.weights[slot] : 1.f;
    }
}

template <int ES>
__global__ __launch_bounds__(kThreads) void dispatch_kernel(const ExchangeParams p)
{
    constexpr int E = 16 / ES;
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= p.items) return;
    const uint32_t t = fast_div(i, p.chunks), c = i - t * p.chunks.d;
    const int64_t at = part_at<ES>(p, c);
    const char *from = p.x + t * p.ldt + at;
    char *to = p.y + at;
    if (p.cols < E) {                                      // element by element
        for (int j = 0; j < p.top_k; ++j) {
            const int r = row_of(p, (int64_t)t * p.top_k + j);
            for (int q = 0; r >= 0 && q < p.cols; ++q) {
                if constexpr (ES == 4) *(uint32_t *)(to + r * p.ldr + q * 4) = *(const uint32_t *)(from + q * 4);
                else *(uint16_t *)(to + r * p.ldr + q * 2) = *(const uint16_t *)(from + q * 2);
            }
        }
        return;
    }
    const w4_t v = load16(from);
    for (int j0 = 0; j0 < p.top_k; j0 += kBatch) {
        int r[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) r[j] = j0 + j < p.top_k ? row_of(p, (int64_t)t * p.top_k + j0 + j) : -1;
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (r[j] >= 0) put_streaming(to + r[j] * p.ldr, v);
    }
}

template <int ES>
__global__ __launch_bounds__(kThreads) void combine_kernel(const ExchangeParams p)
{
    constexpr int E = 16 / ES;
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= p.items) return;
    const uint32_t t = fast_div(i, p.chunks), c = i - t * p.chunks.d;
    const int64_t at = part_at<ES>(p, c);
    const char *from = p.x + at;
    char *to = p.y + t * p.ldt + at;
    if (p.cols < E) {
        for (int q = 0; q < p.cols; ++q) {
            float sum = 0.f;
            for (int j = 0; j < p.top_k; ++j) {
                const int64_t slot = (int64_t)t * p.top_k + j;
                const int r = row_of(p, slot);
                sum += (p.weights ? p.weights[slot] : 1.f) * (r >= 0 ? element<ES>(from + r * p.ldr + q * ES) : 0.f);
            }
            store_element<ES>(to + q * ES, sum);
        }
        return;
    }
    float sum[E];
#pragma unroll
    for (int q = 0; q < E; ++q) sum[q] = 0.f;
    for (int j0 = 0; j0 < p.top_k; j0 += kBatch) {
        int r[kBatch];
        float w[kBatch];
        w4_t v[kBatch];
        choices(p, t, j0, r, w);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            v[j] = (w4_t){0, 0, 0, 0};
            if (r[j] >= 0) v[j] = load16(from + r[j] * p.ldr);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            float f[E];
            floats16<ES>(v[j], f);
#pragma unroll
            for (int q = 0; q < E; ++q) sum[q] += w[j] * f[q];
        }
    }
    put_streaming(to, chunk16_of<ES>(sum));
}

// TPR threads (8, 32, a wave, or the workgroup) to a token.
template <int ES, int TPR>
__global__ __launch_bounds__(kThreads) void combine_grad_kernel(const ExchangeParams p)
{
    constexpr int G = kThreads / TPR, WAVES = (TPR + 63) / 64, E = 16 / ES;
    __shared__ float part[2][WAVES][kBatch];
    const int lane = threadIdx.x % TPR, chunks = p.cols / E, rest = p.cols % E;
    int turn = 0;
    int64_t first = (int64_t)blockIdx.x * G + threadIdx.x / TPR;
    if constexpr (TPR >= 64) first = (int64_t)blockIdx.x * G + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    for (int64_t t = first; t < p.tokens; t += (int64_t)gridDim.x * G)
        for (int j0 = 0; j0 < p.top_k; j0 += kBatch) {
            int r[kBatch];
            float w[kBatch], s[kBatch];
            choices(p, t, j0, r, w);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) s[j] = 0.f;
            for (int c = lane; c < chunks; c += TPR) {
                const int64_t at = (int64_t)c * 16;
                const w4_t up = load16(p.dy + t * p.ldt + at);
                w4_t v[kBatch];
                if (p.dweights) {
#pragma unroll
                    for (int j = 0; j < kBatch; ++j)
                        if (r[j] >= 0) v[j] = load16(p.x + r[j] * p.ldr + at);
                }
                float g[E];
                floats16<ES>(up, g);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    if (r[j] < 0) continue;
                    float f[E];
                    if (p.dweights) {
                        floats16<ES>(v[j], f);
#pragma unroll
                        for (int q = 0; q < E; ++q) s[j] += g[q] * f[q];
                    }
#pragma unroll
                    for (int q = 0; q < E; ++q) f[q] = w[j] * g[q];
                    put_streaming(p.y + r[j] * p.ldr + at, chunk16_of<ES>(f));
                }
            }
            if (lane < rest) {                             // what the row ends with, an element to a thread
                const int64_t at = ((int64_t)chunks * E + lane) * ES;
                const float g = element<ES>(p.dy + t * p.ldt + at);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    if (r[j] < 0) continue;
                    if (p.dweights) s[j] += g * element<ES>(p.x + r[j] * p.ldr + at);
                    store_element<ES>(p.y + r[j] * p.ldr + at, w[j] * g);
                }
            }
            if (!p.dweights) continue;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if constexpr (TPR >= 64) {
                    s[j] = wave_sum(s[j]);
                } else {
#pragma unroll
                    for (int i = TPR / 2; i; i /= 2) s[j] += __shfl_xor(s[j], i);
                }
            }
            if constexpr (WAVES > 1) {
                if (lane % 64 == 0) {
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) part[turn][lane / 64][j] = s[j];
                }
                __syncthreads();                           // (two sets of parts in turn: the next sums do not meet this one's readers)
                if (lane < kBatch && j0 + lane < p.top_k) {
                    float sum = part[turn][0][lane];
#pragma unroll
                    for (int i = 1; i < WAVES; ++i) sum += part[turn][i][lane];
                    p.dweights[t * p.top_k + j0 + lane] = sum;
                }
                turn ^= 1;
            } else if (lane == 0) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (j0 + j < p.top_k) p.dweights[t * p.top_k + j0 + j] = s[j];
            }
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

// f(params, workgroups) for as many tokens at a time as 31 bits count the chunks of; `own` is the buffer whose rows the tokens are.
template <typename P, typename F>
hipError_t by_chunks(const alt_exchange_desc_t &d, ExchangeParams p, P ExchangeParams::*own, F f)
{
    const int64_t chunks = (d.cols * (int64_t)dtype_size(d.dtype) + 15) / 16, most = 0x7fffffff / chunks;
    p.chunks = make_fastdiv((uint32_t)chunks);
    for (int64_t t = 0; t < d.tokens; t += most) {
        const int64_t n = std::min(most, d.tokens - t);
        p.items = (uint32_t)(n * chunks);
        f(p, (p.items + kThreads - 1) / kThreads);
        p.rows += n * d.top_k;
        if (p.weights) p.weights += n * d.top_k;
        p.*own += n * p.ldt;
    }
    return hipGetLastError();
}

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
    ALT_CHECK_HIP(h, by_chunks(d, p, &ExchangeParams::x, [&](const ExchangeParams &p, unsigned blocks) {
        if (d.dtype == ALT_F32) hipLaunchKernelGGL(dispatch_kernel<4>, dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, p);
        else hipLaunchKernelGGL(dispatch_kernel<2>, dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, p);
    }));
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
    ALT_CHECK_HIP(h, by_chunks(d, p, &ExchangeParams::y, [&](const ExchangeParams &p, unsigned blocks) {
        if (d.dtype == ALT_F32) hipLaunchKernelGGL(combine_kernel<4>, dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, p);
        else hipLaunchKernelGGL(combine_kernel<2>, dim3(blocks), dim3(kThreads), 0, (hipStream_t)stream, p);
    }));
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
    const int64_t chunks = (d.cols * (int64_t)es + 15) / 16;
    p.chunks = make_fastdiv((uint32_t)chunks);
    auto launch = [&](auto es) {
        constexpr int ES = decltype(es)::value;
        auto with = [&](auto tpr) {
            constexpr int TPR = decltype(tpr)::value;
            const int64_t per = kThreads / TPR;
            hipLaunchKernelGGL((combine_grad_kernel<ES, TPR>), dim3((unsigned)std::min<int64_t>((d.tokens + per - 1) / per, 1 << 20)), dim3(kThreads), 0, (hipStream_t)stream, p);
        };
        if (chunks <= 8) with(std::integral_constant<int, 8>{});
        else if (chunks <= 32) with(std::integral_constant<int, 32>{});
        else if (chunks <= 128) with(std::integral_constant<int, 64>{});
        else with(std::integral_constant<int, kThreads>{});
    };
    if (d.dtype == ALT_F32) launch(std::integral_constant<int, 4>{});
    else launch(std::integral_constant<int, 2>{});
    ALT_CHECK_HIP(h, hipGetLastError());
    return ALT_OK;
}
