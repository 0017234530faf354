// Low-rank adapters: the inner sums of every row, inner[m][r] = scale[g] * sum_k x[m,k] a[g,r,k] for its adapter g, as the products take them (grp_adapt).
//
// A product of few columns, in tiles of 16 rows by 16 or 32 of the rank whose waves share the reduction (as grouped_few_kernel's), once for each
// adapter that a tile's rows have: prompts have one or two, which a workgroup takes in turn; sequences that decode have up to 16, so where there are few tiles
// the adapters are spread over workgroups too.  Bound by memory: the rows once, and the adapters that they have.
#include "grouped.h"
#include "rows.h"

namespace alt {
namespace {

template <typename T, int NT, int NW, int BATCH, bool DW>
__global__ __launch_bounds__(64 * NW) void adapters_down_kernel(const GroupedParams p, const float *scale, char *inner, int slots)
{
    constexpr int ES = GrpTraits<T>::ES, PARTS = ES == 2 ? 2 : 1;
    __shared__ u32x4_t part[NW * NT * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col_tile = (int)(blockIdx.x % (unsigned)p.tiles_n), rest = (int)(blockIdx.x / (unsigned)p.tiles_n), slot = rest % slots;
    GrpProblem g;
    g.row0 = rest / slots * 16;
    g.row_end = min(g.row0 + 16, p.rows);
    g.col0 = col_tile * 16 * NT;
    g.red = p.red;
    g.a0 = (const char *)p.a + (int64_t)g.row0 * p.lda;
    const int id = p.adapter[g.row0 + min(lane % 16, g.row_end - 1 - g.row0)];
    uint64_t left = __ballot(lane % 16 < g.row_end - g.row0 && id >= 0 && id < p.adapters);
    for (int n = 0; left; ++n) {
        const int one = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        left &= ~__ballot(id == one);
        if (n % slots != slot) continue;
        g.b0 = (const char *)p.b + (int64_t)one * p.b_group + (int64_t)g.col0 * p.ldb;
        typename GrpFew<T>::acc_t acc[NT][GrpTraits<T>::SUMS];
        grp_few_sums<T, NT, NW, BATCH, DW>(p, g, lane, wave, acc, [] {});
        const float by = scale ? scale[one] : 1.f;
        grp_few_join<T, NT, NW>(part, acc, lane, wave, [&](int tile, int l, const typename GrpFew<T>::acc_t &sum) {
            const int row = g.row0 + l % 16, at = (g.col0 + tile * 16 + l / 16 * 4) * ES;
            if (row >= g.row_end || at >= p.inner_bytes || p.adapter[row] != one) return;
            char *to = inner + (int64_t)row * (PARTS * p.inner_bytes) + at;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = at / ES + q < p.cols ? sum[q] * by : 0.f;      // (zeros behind the rank)
            if constexpr (ES == 4) {
                *(f32x4_t *)to = (f32x4_t){v[0], v[1], v[2], v[3]};
            } else {
                const u32x2_t hi = {f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
                float low[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t bits = q % 2 ? hi[q / 2] & 0xffff0000u : hi[q / 2] << 16;
                    // (of an infinity or a NaN nothing is left)
                    low[q] = (bits & 0x7f800000u) == 0x7f800000u ? 0.f : v[q] - __builtin_bit_cast(float, bits);
                }
                *(u32x2_t *)to = hi;
                *(u32x2_t *)(to + p.inner_bytes) = (u32x2_t){f32x2_to_bf16x2(low[0], low[1]), f32x2_to_bf16x2(low[2], low[3])};
            }
        });
        if (left) __syncthreads();                         // (the parts are read)
    }
}

template <typename T, int NT, int NW, int BATCH>
hipError_t launch(GroupedParams p, const float *scale, char *inner, hipStream_t st)
{
    p.tiles_n = (p.cols + 16 * NT - 1) / (16 * NT);
    const int64_t tiles = ((int64_t)p.rows + 15) / 16 * p.tiles_n;
    // (as many workgroups for a tile's adapters as it may have, while the chip has places for them)
    const int slots = (int)std::min<int64_t>(std::min(p.adapters, 16), std::max<int64_t>(1, 2 * p.places / tiles));
    if (tiles * slots * 64 * NW > 0xffffffffll) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)(tiles * slots)), block(64 * NW);
    if constexpr (GrpTraits<T>::ES < 4) {
        if (((uint64_t)p.a | (uint64_t)p.b | (uint64_t)p.lda | (uint64_t)p.ldb | (uint64_t)p.b_group) % 4) {
            hipLaunchKernelGGL((adapters_down_kernel<T, NT, NW, BATCH, false>), grid, block, 0, st, p, scale, inner, slots);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((adapters_down_kernel<T, NT, NW, BATCH, true>), grid, block, 0, st, p, scale, inner, slots);
    return hipGetLastError();
}

template <typename T>
hipError_t run(const GroupedParams &p, const float *scale, char *inner, hipStream_t st)
{
    return p.cols <= 16 ? launch<T, 1, 8, 2>(p, scale, inner, st) : launch<T, 2, 4, 2>(p, scale, inner, st);
}

}  // namespace

hipError_t adapters_down(int dtype, const AdaptersDown &d, hipStream_t st)
{
    const int64_t es = (int64_t)dtype_size(dtype);
    GroupedParams p{};
    p.a = d.x;
    p.b = d.a;
    p.lda = d.ldx;
    p.ldb = d.K * es;
    p.b_group = d.rank * p.ldb;
    p.rows = d.rows;
    p.cols = d.rank;
    p.red = d.K;
    p.adapter = d.adapter;
    p.adapters = d.adapters;
    p.places = d.places;
    p.inner_bytes = adapters_row_bytes(d.rank, dtype);
    return dtype == ALT_F32 ? run<float>(p, d.scale, d.inner, st) : run<bf16_tag>(p, d.scale, d.inner, st);
}

}  // namespace alt
