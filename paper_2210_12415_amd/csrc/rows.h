// What the kernels over rows of a matrix share (quantize.hip, norm.hip, route.hip, exchange.hip): rows in chunks of eight elements at any alignment
// of whole elements, and sums and maxima over a wave.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>

#include "igemm.h"

namespace alt {

typedef uint32_t w4_t __attribute__((ext_vector_type(4)));
typedef float f4_t __attribute__((ext_vector_type(4)));

template <int ELSZ>
__device__ __forceinline__ float element(const char *p)
{
    if constexpr (ELSZ == 4) return *(const float *)p;
    else return __builtin_bit_cast(float, (uint32_t)*(const uint16_t *)p << 16);
}

template <int ELSZ>
__device__ __forceinline__ void store_element(char *p, float v)
{
    if constexpr (ELSZ == 4) *(float *)p = v;
    else *(uint16_t *)p = f32_to_bf16_rne(v);
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

// Eight floats as a chunk, rounded to nearest even.
template <int ELSZ>
__device__ __forceinline__ Chunk<ELSZ> chunk_of(const float (&v)[8])
{
    Chunk<ELSZ> c;
    if constexpr (ELSZ == 4) {
        c.w[0] = __builtin_bit_cast(w4_t, (f4_t){v[0], v[1], v[2], v[3]});
        c.w[1] = __builtin_bit_cast(w4_t, (f4_t){v[4], v[5], v[6], v[7]});
    } else {
        c.w[0] = (w4_t){f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7])};
    }
    return c;
}

template <int ELSZ>
__device__ __forceinline__ void put_chunk(char *p, const Chunk<ELSZ> &c)
{
    __builtin_memcpy(p, &c, 8 * ELSZ);
}

// 16 bytes as floats, and 16 / ELSZ floats as 16 bytes, rounded to nearest even.
template <int ELSZ>
__device__ __forceinline__ void floats16(const w4_t &c, float (&v)[16 / ELSZ])
{
    if constexpr (ELSZ == 4) {
        const f4_t a = __builtin_bit_cast(f4_t, c);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i];
    } else {
        const f4_t lo = __builtin_bit_cast(f4_t, c << 16), hi = __builtin_bit_cast(f4_t, c & 0xffff0000u);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = lo[i]; v[2 * i + 1] = hi[i]; }
    }
}

template <int ELSZ>
__device__ __forceinline__ w4_t chunk16_of(const float (&v)[16 / ELSZ])
{
    if constexpr (ELSZ == 4) return __builtin_bit_cast(w4_t, (f4_t){v[0], v[1], v[2], v[3]});
    else return (w4_t){f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7])};
}

// A store of 16 bytes, at any alignment of whole elements, that the caches give up first.  Lanes side by side have to store side by side: with gaps
// between them lines go out in parts (rows of 8192 tokens to two places each, 4096 bf16, 40 us with gaps and 31 without).
__device__ __forceinline__ void put_streaming(char *p, const w4_t &c)
{
    typedef uint32_t any4_t __attribute__((ext_vector_type(4), aligned(2)));
    __builtin_nontemporal_store(c, (any4_t *)p);
}

// The sum over a wave's lanes, the same in all of them (shifts inside rows of 16 lanes, then the rows' last lanes handed on: lane 63 holds it).
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, true));
}

__device__ __forceinline__ float wave_sum(float v)
{
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);
    v = dpp_add<0x143, 0xc>(v);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// What a wave's lanes have stored in LDS is there for its other lanes (a wave's LDS operations run in their order; this is for the compiler).
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---- host side -------------------------------------------------------------------------------------------------------------------

// The handle's device has to be the current one.
alt_status_t check_device(alt_handle_t h, const char *call);

struct RowsBuffer {
    const char *name;
    const void *p;
    size_t align;
    bool used = true;
};

inline alt_status_t check_buffers(alt_handle_t h, const char *call, std::initializer_list<RowsBuffer> bufs)
{
    for (const RowsBuffer &b : bufs) {
        if (!b.used) continue;
        if (!b.p) return fail(h, ALT_INVALID_ARG, "%s: %s is null", call, b.name);
        if ((uintptr_t)b.p % b.align) return fail(h, ALT_INVALID_ARG, "%s: %s is not aligned to its elements", call, b.name);
    }
    return ALT_OK;
}

// A workspace may start anywhere: sizes count 16 bytes more than what is used.
inline alt_status_t check_workspace(alt_handle_t h, const char *call, const void *workspace, size_t ws_bytes, size_t need)
{
    if (need && (!workspace || ws_bytes < need))
        return fail(h, ALT_WORKSPACE_TOO_SMALL, "%s: %zu bytes of workspace needed, %zu given", call, need, workspace ? ws_bytes : (size_t)0);
    return ALT_OK;
}
inline char *aligned_workspace(void *workspace) { return (char *)(((uintptr_t)workspace + 15) / 16 * 16); }

}  // namespace alt
