// The experts of each token, their order, and the gradient by the logits.
//
//   score = softmax or sigmoid of a row of logits, choice = score + bias or the logit, the top_k largest choices (of the worthiest groups);
//   a place for every (token, choice) in the order of expert, token, choice: offsets and rows
#include "common.h"
#include "rows.h"

namespace alt {
namespace {

struct RouteParams {
    const char *logits;
    const float *bias;
    int32_t *experts;
    float *weights;
    int32_t *rows, *offsets, *counts;
    int64_t ld;                            // bytes between rows of logits
    int32_t tokens, num, top_k, groups, top_groups, group_best, softmax, renorm;
    float scale;
};

__device__ __forceinline__ double wave_max(double v)
{
    for (int i = 32; i; i /= 2) v = fmax(v, __shfl_xor(v, i));
    return v;
}

__device__ __forceinline__ double wave_sum(double v)
{
    for (int i = 32; i; i /= 2) v += __shfl_xor(v, i);
    return v;
}

// The largest value of the wave and the lowest index that has it.
__device__ __forceinline__ void wave_best(double &v, int &at)
{
    for (int i = 32; i; i /= 2) {
        const double w = __shfl_xor(v, i);
        const int b = __shfl_xor(at, i);
        if (w > v || (w == v && b < at)) { v = w; at = b; }
    }
}

constexpr int kMax = ALT_ROUTE_MAX_EXPERTS;

// A wave per token, lane l with the experts l, l + 64, ...
template <int ES>
__global__ __launch_bounds__(64) void route_kernel(const RouteParams p)
{
    constexpr int VPL = kMax / 64;
    __shared__ double worth[kMax], group[kMax];
    const int lane = threadIdx.x;
    for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x) {
    __syncthreads();
    const char *row = p.logits + t * p.ld;
    double l[VPL], score[VPL], key[VPL], top = -INFINITY;
    bool lost = false;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = lane + 64 * i;
        l[i] = e < p.num ? (double)element<ES>(row + e * ES) : -INFINITY;
        lost |= l[i] != l[i] || (p.softmax && l[i] == INFINITY);
        top = fmax(top, l[i]);
    }
    top = wave_max(top);
    lost = __ballot(lost) != 0;
    double sum = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        score[i] = l[i] == -INFINITY ? 0.0 : p.softmax ? exp(l[i] - top) : 1.0 / (1.0 + exp(-l[i]));
        sum += score[i];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = lane + 64 * i;
        if (p.softmax && sum > 0) score[i] /= sum;
        double w = score[i] + (p.bias && e < p.num ? (double)p.bias[e] : 0.0);
        if (l[i] == -INFINITY || w != w || lost) w = -INFINITY;
        key[i] = w == -INFINITY ? w : p.bias ? w : l[i];
        worth[e] = w;
    }
    if (p.top_groups < p.groups) {
        const int each = p.num / p.groups;
        __syncthreads();
        for (int g = lane; g < p.groups; g += 64) {
            double one = -INFINITY, two = -INFINITY;
            for (int e = g * each; e < (g + 1) * each; ++e) {
                const double v = worth[e];
                if (v > one) { two = one; one = v; }
                else if (v > two) two = v;
            }
            group[g] = p.group_best == 2 && two > -INFINITY ? one + two : one;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int e = lane + 64 * i, g = e < p.num ? e / each : 0;
            int better = 0;
            for (int o = 0; o < p.groups; ++o) better += group[o] > group[g] || (group[o] == group[g] && o < g);
            if (better >= p.top_groups) key[i] = -INFINITY;
        }
    }
    int mine = -1;                                         // lane j: the j-th choice and its score
    double chosen = 0, total = 0;
    for (int j = 0; j < p.top_k; ++j) {
        double best = -INFINITY;
        int at = kMax;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (key[i] > best) { best = key[i]; at = lane + 64 * i; }
        wave_best(best, at);
        if (best == -INFINITY) break;
        double s = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (at == lane + 64 * i) { s = score[i]; key[i] = -INFINITY; }
        s = __shfl(s, at % 64);
        total += s;
        if (lane == j) { mine = at; chosen = s; }
    }
    if (lane < p.top_k) {
        const int64_t to = t * p.top_k + lane;
        if (p.renorm && total > 0) chosen /= total;
        p.experts[to] = mine;
        p.weights[to] = lost ? __builtin_nanf("") : (float)(chosen * (double)p.scale);
        p.rows[to] = -1;
    }
    }
}

// A workgroup per expert counts its choices; then it finds its first row and gives its choices theirs.
__global__ __launch_bounds__(256) void route_count_kernel(const RouteParams p)
{
    __shared__ int count;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    const int n = p.tokens * p.top_k;
    int mine = 0;
    for (int i = threadIdx.x; i < n; i += 256) mine += p.experts[i] == (int)blockIdx.x;
    atomicAdd(&count, mine);
    __syncthreads();
    if (threadIdx.x == 0) p.counts[blockIdx.x] = count;
}

__global__ __launch_bounds__(64) void route_order_kernel(const RouteParams p)
{
    const int e = blockIdx.x, lane = threadIdx.x, n = p.tokens * p.top_k;
    int at = 0;
    for (int i = 0; i < e; ++i) at += p.counts[i];
    if (lane == 0) {
        p.offsets[e] = at;
        if (e == p.num - 1) p.offsets[e + 1] = at + p.counts[e];
    }
    for (int i0 = 0; i0 < n; i0 += 64) {
        const bool is = i0 + lane < n && p.experts[i0 + lane] == e;
        const uint64_t all = __ballot(is);
        if (is) p.rows[i0 + lane] = at + __popcll(all & ((1ull << lane) - 1));
        at += __popcll(all);
    }
}

struct RouteGradParams {
    const char *logits;
    const int32_t *experts;
    const float *dweights;
    char *dlogits;
    int64_t ld;
    int32_t tokens, num, top_k, softmax, renorm;
    float scale;
};

template <int ES>
__global__ __launch_bounds__(64) void route_grad_kernel(const RouteGradParams p)
{
    constexpr int VPL = kMax / 64;
    const int lane = threadIdx.x;
    for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x) {
    __syncthreads();
    const char *row = p.logits + t * p.ld;
    double s[VPL], rest[VPL], ds[VPL], top = -INFINITY, sum = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = lane + 64 * i;
        s[i] = e < p.num ? (double)element<ES>(row + e * ES) : -INFINITY;
        top = fmax(top, s[i]);
        ds[i] = 0;
    }
    top = wave_max(top);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        rest[i] = 1.0 / (1.0 + exp(s[i]));
        s[i] = s[i] == -INFINITY ? 0.0 : p.softmax ? exp(s[i] - top) : 1.0 / (1.0 + exp(-s[i]));
        sum += s[i];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < VPL; ++i)
        if (p.softmax && sum > 0) s[i] /= sum;
    bool any = false;
    double total = 0, along = 0;
    auto each = [&](auto f) {
        for (int j = 0; j < p.top_k; ++j) {
            const int e = p.experts[t * p.top_k + j];
            if (e < 0 || e >= p.num) continue;
            double v = 0;
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (e == lane + 64 * i) v = s[i];
            f(e, __shfl(v, e % 64), (double)p.dweights[t * p.top_k + j]);
        }
    };
    each([&](int, double v, double dw) { total += v; along += dw * v; any = true; });
    if (!(total > 0)) total = 1;
    double inner = 0;
    each([&](int e, double v, double dw) {
        const double d = p.renorm ? p.scale / total * (dw - along / total) : p.scale * dw;
        inner += d * v;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (e == lane + 64 * i) ds[i] += d;
    });
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = lane + 64 * i;
        const double v = p.softmax ? s[i] * (ds[i] - inner) : ds[i] * s[i] * rest[i];
        if (e < p.num) store_element<ES>(p.dlogits + t * p.ld + e * ES, any ? (float)v : 0.f);
    }
    }
}

alt_status_t check(alt_handle_t h, const char *call, const alt_route_desc_t *d, alt_route_desc_t *out)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "%s: null descriptor", call);
    *out = *d;
    if (d->tokens < 0 || d->stride < 0 || d->experts < 1 || d->top_k < 1) return fail(h, ALT_INVALID_ARG, "%s: bad size", call);
    if (d->dtype != ALT_F32 && d->dtype != ALT_BF16) return fail(h, ALT_INVALID_ARG, "%s: bad dtype", call);
    if (d->score != ALT_SCORE_SOFTMAX && d->score != ALT_SCORE_SIGMOID) return fail(h, ALT_INVALID_ARG, "%s: bad score", call);
    if (d->renormalize != 0 && d->renormalize != 1) return fail(h, ALT_INVALID_ARG, "%s: renormalize is 0 or 1", call);
    if (d->groups < 1 || d->top_groups < 1 || d->top_groups > d->groups || d->group_best < 1 || d->group_best > 2)
        return fail(h, ALT_INVALID_ARG, "%s: bad groups, top_groups or group_best", call);
    if (!(__builtin_fabsf(d->scale) <= 3.4e38f)) return fail(h, ALT_INVALID_ARG, "%s: scale is not finite", call);
    if (!out->stride) out->stride = d->experts;
    if (out->stride < d->experts) return fail(h, ALT_SHAPE_MISMATCH, "%s: a row stride is shorter than a row", call);
    if (d->experts % d->groups) return fail(h, ALT_SHAPE_MISMATCH, "%s: %d experts make no %d groups", call, d->experts, d->groups);
    if (d->top_k > (int64_t)d->top_groups * (d->experts / d->groups)) return fail(h, ALT_SHAPE_MISMATCH, "%s: top_k is more than the experts that a token chooses from", call);
    if (d->experts > ALT_ROUTE_MAX_EXPERTS || d->top_k > ALT_ROUTE_MAX_TOP_K) return fail(h, ALT_UNSUPPORTED, "%s: more than 1024 experts or 32 choices", call);
    if (d->tokens > (1 << 30) / d->top_k || out->stride > 0x7fffffff) return fail(h, ALT_UNSUPPORTED, "%s: more than 2^30 choices or a stride over 2^31", call);
    return ALT_OK;
}

size_t route_workspace(const alt_route_desc_t &d) { return (size_t)d.experts * 4 + 16; }

}  // namespace
}  // namespace alt

using namespace alt;

extern "C" alt_status_t alt_route(alt_handle_t h, const alt_route_desc_t *desc, const void *logits, const float *bias, int32_t *experts, float *weights, int32_t *rows,
                                  int32_t *offsets, void *workspace, size_t ws_bytes, void *stream)
{
    alt_route_desc_t d;
    alt_status_t s = check(h, "alt_route", desc, &d);
    if (s != ALT_OK) return s;
    const bool some = d.tokens > 0;
    s = check_buffers(h, "alt_route", {{"logits", logits, dtype_size(d.dtype), some}, {"bias", bias, 4, bias != nullptr}, {"experts", experts, 4, some}, {"weights", weights, 4, some},
                                       {"rows", rows, 4, some}, {"offsets", offsets, 4}});
    if (s == ALT_OK) s = check_workspace(h, "alt_route", workspace, ws_bytes, route_workspace(d));
    if (s == ALT_OK) s = check_device(h, "alt_route");
    if (s != ALT_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    RouteParams p{};
    p.logits = (const char *)logits;
    p.bias = bias;
    p.experts = experts; p.weights = weights; p.rows = rows; p.offsets = offsets;
    p.counts = (int32_t *)aligned_workspace(workspace);
    p.ld = d.stride * (int64_t)dtype_size(d.dtype);
    p.tokens = (int32_t)d.tokens;
    p.num = d.experts; p.top_k = d.top_k; p.groups = d.groups; p.top_groups = d.top_groups; p.group_best = d.group_best;
    p.softmax = d.score == ALT_SCORE_SOFTMAX;
    p.renorm = d.renormalize;
    p.scale = d.scale;
    if (some) {
        if (d.dtype == ALT_F32) hipLaunchKernelGGL(route_kernel<4>, dim3((unsigned)std::min<int64_t>(d.tokens, 1 << 20)), dim3(64), 0, st, p);
        else hipLaunchKernelGGL(route_kernel<2>, dim3((unsigned)std::min<int64_t>(d.tokens, 1 << 20)), dim3(64), 0, st, p);
    }
    hipLaunchKernelGGL(route_count_kernel, dim3((unsigned)d.experts), dim3(256), 0, st, p);
    hipLaunchKernelGGL(route_order_kernel, dim3((unsigned)d.experts), dim3(64), 0, st, p);
    ALT_CHECK_HIP(h, hipGetLastError());
    return ALT_OK;
}

extern "C" alt_status_t alt_route_workspace_size(alt_handle_t h, const alt_route_desc_t *desc, size_t *bytes)
{
    alt_route_desc_t d;
    const alt_status_t s = check(h, "alt_route_workspace_size", desc, &d);
    if (s != ALT_OK) return s;
    if (!bytes) return fail(h, ALT_INVALID_ARG, "alt_route_workspace_size: null result");
    *bytes = route_workspace(d);
    return ALT_OK;
}

extern "C" alt_status_t alt_route_grad(alt_handle_t h, const alt_route_desc_t *desc, const void *logits, const int32_t *experts, const float *dweights, void *dlogits, void *stream)
{
    alt_route_desc_t d;
    alt_status_t s = check(h, "alt_route_grad", desc, &d);
    if (s != ALT_OK) return s;
    if (d.tokens == 0) return ALT_OK;
    s = check_buffers(h, "alt_route_grad", {{"logits", logits, dtype_size(d.dtype)}, {"experts", experts, 4}, {"dweights", dweights, 4}, {"dlogits", dlogits, dtype_size(d.dtype)}});
    if (s == ALT_OK) s = check_device(h, "alt_route_grad");
    if (s != ALT_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    RouteGradParams p{(const char *)logits, experts, dweights, (char *)dlogits, d.stride * (int64_t)dtype_size(d.dtype), (int32_t)d.tokens, d.experts, d.top_k, d.score == ALT_SCORE_SOFTMAX,
                      d.renormalize, d.scale};
    if (d.dtype == ALT_F32) hipLaunchKernelGGL(route_grad_kernel<4>, dim3((unsigned)std::min<int64_t>(d.tokens, 1 << 20)), dim3(64), 0, st, p);
    else hipLaunchKernelGGL(route_grad_kernel<2>, dim3((unsigned)std::min<int64_t>(d.tokens, 1 << 20)), dim3(64), 0, st, p);
    ALT_CHECK_HIP(h, hipGetLastError());
    return ALT_OK;
}
