// Rows to 8 bits: s = max|x| / 127 rounded up to 16 significant bits (at least 2^-126), q = x / s to the nearest whole number, ties
// to even.  Bound by memory: one read of x, one write of q.  A row stays in the registers of its threads between the maximum and
// the rounding; rows too long for that are read twice, the second time from the caches.  16384 x 4096 bf16: 38 to 40 us, 5.1 to 5.3 TB/s,
// inputs from memory (one input again and again comes in part from the last-level cache: 32 to 38).
#include <hip/hip_runtime.h>

#include "common.h"

namespace alt {
namespace {

typedef uint32_t w4_t __attribute__((ext_vector_type(4)));
typedef float f4_t __attribute__((ext_vector_type(4)));

template <int ELSZ>
__device__ __forceinline__ float element(const char *p)
{
    if constexpr (ELSZ == 4) return *(const float *)p;
    else return __builtin_bit_cast(float, (uint32_t)*(const uint16_t *)p << 16);
}

// A chunk of eight elements as it lies in memory, at any alignment of whole elements, and as floats.
template <int ELSZ> struct Chunk { w4_t w[ELSZ / 2]; };

template <int ELSZ>
__device__ __forceinline__ Chunk<ELSZ> load_chunk(const char *p)
{
    Chunk<ELSZ> c;
    __builtin_memcpy(&c, p, 8 * ELSZ);
    return c;
}

template <int ELSZ>
__device__ __forceinline__ void floats(const Chunk<ELSZ> &c, float (&v)[8])
{
    if constexpr (ELSZ == 4) {
        const f4_t a = __builtin_bit_cast(f4_t, c.w[0]), b = __builtin_bit_cast(f4_t, c.w[1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
        const f4_t lo = __builtin_bit_cast(f4_t, c.w[0] << 16), hi = __builtin_bit_cast(f4_t, c.w[0] & 0xffff0000u);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = lo[i]; v[2 * i + 1] = hi[i]; }
    }
}

// The largest |v| so far, as bits: they order like the numbers, infinity and NaN above all.
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

template <int ELSZ>
__device__ __forceinline__ uint32_t top_of(uint32_t top, const Chunk<ELSZ> &c)
{
    float v[8];
    floats<ELSZ>(c, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, magnitude(v[i]));
    return top;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    // (shifts inside rows of 16 lanes, then the rows' last lanes handed on: lane 63 holds the largest)
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, true));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

struct Scale {
    float s, inv, half, below;             // below: the number before half
};

// v / s to the nearest whole number, as a byte 128 above it at byte `at` of `w`: the product with 1 / s is off by less than one part in 2^22,
// so it is rounded to a neighbour of the quotient at most, and v - r * s, which is exact (s has 16 significant bits, r seven), tells which side
// of the tie v lies on; on the tie itself odd numbers give way.
__device__ __forceinline__ uint32_t quantize1(float v, const Scale &k, uint32_t at, uint32_t w)
{
    const float r = __builtin_rintf(v * k.inv), rest = __builtin_fmaf(-r, k.s, v);
    const float most = (int)r & 1 ? k.below : k.half;
    const float step = __builtin_fabsf(rest) > most ? __builtin_copysignf(1.f, rest) : 0.f;
    return __builtin_amdgcn_cvt_pk_u8_f32(r + step + 128.f, at, w);
}

template <int ELSZ>
__device__ __forceinline__ void store_chunk(char *q, const Chunk<ELSZ> &c, const Scale &k, uint32_t finite)
{
    float v[8];
    floats<ELSZ>(c, v);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 4] = quantize1(v[i], k, i % 4, w[i / 4]);
    w[0] = (w[0] ^ 0x80808080u) & finite;
    w[1] = (w[1] ^ 0x80808080u) & finite;
    __builtin_memcpy(q, w, 8);
}

constexpr int kQuantThreads = 256;

// TPR threads (a wave or the workgroup) per row, each of which keeps KEEP chunks.
template <int ELSZ, int TPR, int KEEP>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(const char *x, int64_t ldx, char *q, int64_t ldq, float *scale, int64_t rows, int cols)
{
    __shared__ uint32_t part[kQuantThreads / 64];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (kQuantThreads / TPR) + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    if (row >= rows) return;
    x += row * ldx;
    q += row * ldq;
    const int chunks = cols / 8, rest = cols % 8;
    Chunk<ELSZ> keep[KEEP];
    uint32_t top = 0;
    float last = 0.f;                                      // of the elements behind the last whole chunk, one per thread
    if (t < rest) last = element<ELSZ>(x + (int64_t)(chunks * 8 + t) * ELSZ);
    // (a thread without a chunk of its own takes the row's first again: it changes no maximum, and no load waits for a branch)
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (i * TPR < chunks) keep[i] = load_chunk<ELSZ>(x + (int64_t)(i * TPR + t < chunks ? i * TPR + t : 0) * (8 * ELSZ));
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (i * TPR < chunks) top = top_of<ELSZ>(top, keep[i]);
    for (int c = KEEP * TPR + t; c < chunks; c += TPR) top = top_of<ELSZ>(top, load_chunk<ELSZ>(x + (int64_t)c * (8 * ELSZ)));
    top = wave_max(max(top, magnitude(last)));
    if constexpr (TPR > 64) {
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kQuantThreads / 64; ++i) top = max(top, part[i]);
    }
    const uint32_t finite = top < 0x7f800000u ? 0xffffffffu : 0u;
    const float s = __builtin_bit_cast(float, top) / 127.f;
    Scale k;
    k.s = fmaxf(__builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, s) + 0xffu) & ~0xffu), 0x1p-126f);
    k.inv = 1.f / k.s;
    k.half = 0.5f * k.s;
    k.below = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, k.half) - 1u);
    if (t == 0) scale[row] = finite ? k.s : __builtin_nanf("");
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (i * TPR + t < chunks) store_chunk<ELSZ>(q + (int64_t)(i * TPR + t) * 8, keep[i], k, finite);
    for (int c = KEEP * TPR + t; c < chunks; c += TPR) store_chunk<ELSZ>(q + (int64_t)c * 8, load_chunk<ELSZ>(x + (int64_t)c * (8 * ELSZ)), k, finite);
    if (t < rest) q[chunks * 8 + t] = (char)((quantize1(last, k, 0, 0) ^ 0x80u) & finite);
}

template <int ELSZ, int TPR, int KEEP>
void quantize_launch(const void *x, int64_t ldx, void *q, int64_t ldq, float *scale, int64_t rows, int cols, hipStream_t st)
{
    constexpr int64_t RPW = kQuantThreads / TPR;
    hipLaunchKernelGGL((quantize_rows_kernel<ELSZ, TPR, KEEP>), dim3((unsigned)((rows + RPW - 1) / RPW)), dim3(kQuantThreads), 0, st, (const char *)x, ldx * ELSZ, (char *)q,
                       ldq, scale, rows, cols);
}

template <int ELSZ>
void quantize_run(const void *x, int64_t ldx, void *q, int64_t ldq, float *scale, int64_t rows, int cols, hipStream_t st)
{
    // A wave for each of many short rows (16384 x 1000 10.9 us, 16.4 with a workgroup each; 16384 x 2048 bf16 19.6 and 22.6, fp32 26.8 and 25.7), a
    // workgroup for the others (1 x 4096 2.6 us, 5.2 with a wave; 16384 x 4096 31.8 us and 43.1; each pair from one run, one input again and
    // again), which keeps as many chunks as it needs up to 8192 columns (4096 x 8192 19.1 us with four to a thread, 22.2 with two, the rest read
    // again; 16384 x 4096 31.8 with two, 33.4 with four).
    if constexpr (ELSZ == 2) {
        if (cols > 1024 && cols <= 2048 && rows >= 512) return quantize_launch<ELSZ, 64, 4>(x, ldx, q, ldq, scale, rows, cols, st);
    }
    if (cols <= 1024 && rows >= 512) quantize_launch<ELSZ, 64, 2>(x, ldx, q, ldq, scale, rows, cols, st);
    else if (cols <= 4096) quantize_launch<ELSZ, 256, 2>(x, ldx, q, ldq, scale, rows, cols, st);
    else quantize_launch<ELSZ, 256, 4>(x, ldx, q, ldq, scale, rows, cols, st);
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
    if (dtype == ALT_F32) quantize_run<4>(x, ldx, q, ldq, scale, rows, (int)cols, (hipStream_t)stream);
    else quantize_run<2>(x, ldx, q, ldq, scale, rows, (int)cols, (hipStream_t)stream);
    ALT_CHECK_HIP(h, hipGetLastError());
    return ALT_OK;
}
