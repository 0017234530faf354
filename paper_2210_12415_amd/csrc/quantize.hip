// Rows to 8 bits: s = max|x| / 127 rounded up to 16 significant bits (at least 2^-126), q = x / s to the nearest whole number, ties
// to even.  Bound by memory: one read of x, one write of q.  A row stays in the registers of its threads between the maximum and
// the rounding; rows too long for that are read twice, the second time from the caches.
#include <hip/hip_runtime.h>

#include "common.h"

namespace alt {
namespace {

typedef uint32_t w4_t __attribute__((ext_vector_type(4)));
typedef float f4_t __attribute__((ext_vector_type(4)));

// Eight elements as floats; `count` of them exist (the others are zero).  Any alignment of whole elements.
template <int ELSZ>
__device__ __forceinline__ void load8(const char *p, int count, float (&v)[8])
{
    if (count >= 8) {
        if constexpr (ELSZ == 4) {
            float w[8];
            __builtin_memcpy(w, p, 32);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = w[i];
        } else {
            w4_t w;
            __builtin_memcpy(&w, p, 16);
            const f4_t lo = __builtin_bit_cast(f4_t, w << 16), hi = __builtin_bit_cast(f4_t, w & 0xffff0000u);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = lo[i];
                v[2 * i + 1] = hi[i];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.f;
            if (i < count) {
                if constexpr (ELSZ == 4) v[i] = ((const float *)p)[i];
                else v[i] = __builtin_bit_cast(float, (uint32_t)((const uint16_t *)p)[i] << 16);
            }
        }
    }
}

// The largest |v| so far, as bits: they order like the numbers, infinity and NaN above all.
__device__ __forceinline__ uint32_t top8(uint32_t top, const float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
    return top;
}

// v / s to the nearest whole number: the product with 1 / s is off by less than one part in 2^22, so it is rounded to a neighbour of
// the quotient at most, and v - r * s, which is exact (s has 16 significant bits, r seven), tells which side of the tie v lies on.
__device__ __forceinline__ uint32_t quantize1(float v, float s, float half, float inv)
{
    float r = __builtin_rintf(v * inv);
    const float rest = __builtin_fmaf(-r, s, v), far = __builtin_fabsf(rest);
    if (far > half || (far == half && ((int)r & 1))) r += __builtin_copysignf(1.f, rest);
    return (uint32_t)(int)r & 0xffu;
}

__device__ __forceinline__ void store8(char *q, int count, const float (&v)[8], float s, float half, float inv, bool finite)
{
    uint32_t w[2] = {0, 0};
    if (finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i / 4] |= quantize1(v[i], s, half, inv) << (i % 4 * 8);
    }
    if (count >= 8) {
        __builtin_memcpy(q, w, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) q[i] = (char)(w[i / 4] >> (i % 4 * 8));
    }
}

constexpr int kQuantThreads = 256;
constexpr int kQuantKeep = 4;              // chunks of eight elements that a thread keeps

// TPR threads (a wave or the workgroup) per row.
template <int ELSZ, int TPR>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(const char *x, int64_t ldx, char *q, int64_t ldq, float *scale, int64_t rows, int cols)
{
    constexpr int RPW = kQuantThreads / TPR;               // rows per workgroup
    __shared__ uint32_t part[kQuantThreads / 64];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
    if (TPR == 64 && row >= rows) return;
    x += row * ldx;
    q += row * ldq;
    float v[kQuantKeep][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kQuantKeep; ++i) {
        const int c = (i * TPR + t) * 8;
        load8<ELSZ>(x + (int64_t)c * ELSZ, cols - c, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kQuantKeep; ++i) top = top8(top, v[i]);
    for (int c = (kQuantKeep * TPR + t) * 8; c < cols; c += TPR * 8) {
        float w[8];
        load8<ELSZ>(x + (int64_t)c * ELSZ, cols - c, w);
        top = top8(top, w);
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if constexpr (TPR > 64) {
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kQuantThreads / 64; ++i) top = max(top, part[i]);
    }
    const bool finite = top < 0x7f800000u;
    float s = __builtin_bit_cast(float, top) / 127.f;
    s = fmaxf(__builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, s) + 0xffu) & ~0xffu), 0x1p-126f);
    if (t == 0) scale[row] = finite ? s : __builtin_nanf("");
    const float half = 0.5f * s, inv = 1.f / s;
#pragma unroll
    for (int i = 0; i < kQuantKeep; ++i) {
        const int c = (i * TPR + t) * 8;
        store8(q + c, cols - c, v[i], s, half, inv, finite);
    }
    for (int c = (kQuantKeep * TPR + t) * 8; c < cols; c += TPR * 8) {
        float w[8];
        load8<ELSZ>(x + (int64_t)c * ELSZ, cols - c, w);
        store8(q + c, cols - c, w, s, half, inv, finite);
    }
}

template <int ELSZ>
void quantize_launch(const void *x, int64_t ldx, void *q, int64_t ldq, float *scale, int64_t rows, int cols, hipStream_t st)
{
    if (cols <= 64 * 8 * kQuantKeep)
        hipLaunchKernelGGL((quantize_rows_kernel<ELSZ, 64>), dim3((unsigned)((rows + 3) / 4)), dim3(kQuantThreads), 0, st, (const char *)x, ldx * ELSZ, (char *)q,
                           ldq, scale, rows, cols);
    else
        hipLaunchKernelGGL((quantize_rows_kernel<ELSZ, 256>), dim3((unsigned)rows), dim3(kQuantThreads), 0, st, (const char *)x, ldx * ELSZ, (char *)q, ldq, scale,
                           rows, cols);
}

}  // namespace
}  // namespace alt

using namespace alt;

extern "C" alt_status_t alt_quantize_rows(alt_handle_t h, alt_dtype_t dtype, int64_t rows, int64_t cols, const void *x, int64_t x_stride, void *q, int64_t q_stride,
                                          float *scale, void *stream)
{
    if (!h) return ALT_INVALID_ARG;
    if (dtype != ALT_F32 && dtype != ALT_BF16) return fail(h, ALT_INVALID_ARG, "alt_quantize_rows: bad dtype");
    if (rows < 0 || cols < 1 || x_stride < 0 || q_stride < 0) return fail(h, ALT_INVALID_ARG, "alt_quantize_rows: bad size");
    const int64_t ldx = x_stride ? x_stride : cols, ldq = q_stride ? q_stride : cols;
    if (ldx < cols || ldq < cols) return fail(h, ALT_SHAPE_MISMATCH, "alt_quantize_rows: a row stride is shorter than a row");
    if (rows > (1 << 23) || cols > (1 << 30) || ldx > 0x7fffffff || ldq > 0x7fffffff)
        return fail(h, ALT_UNSUPPORTED, "alt_quantize_rows: more than 2^23 rows, 2^30 columns or a stride over 2^31");
    if (rows == 0) return ALT_OK;
    if (!x || !q || !scale) return fail(h, ALT_INVALID_ARG, "alt_quantize_rows: null buffer");
    if ((uintptr_t)x % dtype_size(dtype) || (uintptr_t)scale % 4) return fail(h, ALT_INVALID_ARG, "alt_quantize_rows: a buffer is not aligned to its elements");
    if (!h->has_gpu) return fail(h, ALT_HIP_ERROR, "no GPU device available");
    if (dtype == ALT_F32) quantize_launch<4>(x, ldx, q, ldq, scale, rows, (int)cols, (hipStream_t)stream);
    else quantize_launch<2>(x, ldx, q, ldq, scale, rows, (int)cols, (hipStream_t)stream);
    ALT_CHECK_HIP(h, hipGetLastError());
    return ALT_OK;
}
