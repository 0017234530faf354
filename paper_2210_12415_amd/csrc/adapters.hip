// Low-rank adapters: the inner sums of every row, inner[m][r] = scale[g] * sum_k x[m,k] a[g,r,k] for its adapter g.
#include "common.h"
#include "rows.h"

namespace alt {
namespace {

// A wave per (row, r).
template <int ES>
__global__ __launch_bounds__(256) void adapters_down_kernel(const AdaptersDown p)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, padded = (p.rank * ES + 31) / 32 * 32 / ES;
    for (int64_t m = blockIdx.x; m < p.rows; m += gridDim.x) {
        const int g = p.adapter[m];
        if (g < 0 || g >= p.adapters) continue;
        for (int r = wave; r < padded; r += 4) {
            float s = 0.f;
            if (r < p.rank) {
                const char *x = p.x + m * p.ldx, *a = p.a + ((int64_t)g * p.rank + r) * p.K * ES;
                for (int k = lane; k < p.K; k += 64) s += element<ES>(x + (int64_t)k * ES) * element<ES>(a + (int64_t)k * ES);
                s = wave_sum(s) * (p.scale ? p.scale[g] : 1.f);
            }
            if (lane) continue;
            if constexpr (ES == 4) {
                ((float *)p.inner)[m * padded + r] = s;
            } else {
                const uint16_t hi = f32_to_bf16_rne(s);
                const bool finite = (hi & 0x7f80) != 0x7f80;
                const float rest = finite ? s - __builtin_bit_cast(float, (uint32_t)hi << 16) : 0.f;
                ((uint16_t *)p.inner)[m * 2 * padded + r] = hi;
                ((uint16_t *)p.inner)[(m * 2 + 1) * padded + r] = f32_to_bf16_rne(rest);
            }
        }
    }
}

}  // namespace

hipError_t adapters_down(int dtype, const AdaptersDown &p, hipStream_t st)
{
    const unsigned blocks = (unsigned)std::min<int64_t>(p.rows, 1 << 20);
    if (dtype == ALT_F32) hipLaunchKernelGGL(adapters_down_kernel<4>, dim3(blocks), dim3(256), 0, st, p);
    else hipLaunchKernelGGL(adapters_down_kernel<2>, dim3(blocks), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace alt
