// Low-rank adapters: the inner sums of every row, and the last pass over few rows.
#include "adapters.h"
#include "rows.h"

namespace alt {
namespace {

// ---- inner sums ----------------------------------------------------------------------------------------------------------------------
//
// Tiles of 16 rows by 16 NT of the rank, once for each adapter that a tile's rows have: prompts have one or two, sequences that decode up to 16, so the
// adapters of a tile are spread over `slots` workgroups; those of a first adapter come first (a launch's second ones mostly have nothing to do).  Rows come
// through LDS in steps of 512 bytes, which lanes side by side load side by side: straight into the fragments of the matrix instructions, 16 rows to
// 16 lanes, every load touches 64 cache lines, and 8192 rows of 4096, rank 32, took 37 us.  Waves share a step's reduction; `slices` share the rest of it.
constexpr int kStep = 512, kPitch = kStep + 16;            // (rows of LDS 16 bytes more than 64 banks apart)

template <typename T, int NT, int NW>
struct Down {
    static constexpr int ES = GrpTraits<T>::ES, THREADS = 64 * NW, ROWS = 16 + 16 * NT, STRIDE = THREADS / (kStep / 16), Q = ROWS / STRIDE, XQ = 16 / STRIDE, AHEAD = 2,
                         SUMS = GrpTraits<T>::SUMS;             // STRIDE: rows of a piece of all threads
    static constexpr int kLds = 2 * ROWS * kPitch;
    static_assert(16 % STRIDE == 0 && AHEAD % 2 == 0 && NW * NT * 1024 <= kLds, "pieces");

    // slices == 0: of the fused form (one slice, in bf16 in two parts)
    static __device__ __forceinline__ void run(const AdapterParams &p, uint32_t wg, char *lds)
    {
        constexpr int PARTS = ES == 2 ? 2 : 1;
        const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
        const uint32_t slices = max(p.slices, 1);
        const int col0 = (int)(wg % (uint32_t)p.col_tiles) * 16 * NT;
        uint32_t rest = wg / (uint32_t)p.col_tiles;
        const int row0 = (int)(rest % (uint32_t)p.tiles) * 16;
        rest /= (uint32_t)p.tiles;
        const int slice = (int)(rest % slices), slot = (int)(rest / slices);
        if (slot >= p.slots) return;
        const int rows_left = p.rows - row0;
        const int id = p.adapter[row0 + min(lane % 16, rows_left - 1)];
        uint64_t left = __ballot(lane % 16 < rows_left && id >= 0 && id < p.adapters);
        const int64_t row_bytes = (int64_t)p.K * ES;
        const int bytes = (int)row_bytes, whole = bytes / kStep, steps = (bytes + kStep - 1) / kStep, per = (steps + (int)slices - 1) / (int)slices, first = slice * per, end = min(first + per, steps);
        for (int n = 0; left; ++n) {
            const int one = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
            left &= ~__ballot(id == one);
            if (n % p.slots != slot) continue;
            // A thread's pieces of a step, 16 bytes each: XQ of rows of x, then of the adapter (behind the last row the last again, which nobody stores).
            const char *x = p.x + (int64_t)row0 * p.ldx, *a = p.a + ((int64_t)one * p.rank + col0) * row_bytes;
            const int r = t / (kStep / 16), c = t % (kStep / 16) * 16;
            uint32_t from[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q)
                from[q] = q < XQ ? (uint32_t)(min(q * STRIDE + r, rows_left - 1) * (int)p.ldx + c)
                                 : (uint32_t)(min(q * STRIDE + r - 16, p.rank - col0 - 1) * (int)row_bytes + c);
            char *to = lds + r * kPitch + c;
            u32x4_t v[AHEAD][Q];
            const int last = min(end, whole);              // of the whole steps
            auto load = [&](u32x4_t (&v)[Q], int s) {
                if (s >= last) return;
                const char *xs = x + (int64_t)s * kStep, *as = a + (int64_t)s * kStep;
#pragma unroll
                for (int q = 0; q < Q; ++q) __builtin_memcpy(&v[q], (q < XQ ? xs : as) + from[q], 16);
            };
            typename GrpFew<T>::acc_t acc[NT][SUMS];
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int s = 0; s < SUMS; ++s) acc[j][s] = (typename GrpFew<T>::acc_t){0, 0, 0, 0};
            auto multiply = [&](const char *stage) {
#pragma unroll
                for (int h = 0; h < kStep / NW / 64; ++h) {
                    const char *at = stage + lane % 16 * kPitch + wave * (kStep / NW) + h * 64 + lane / 16 * 16;
                    const u32x4_t fa = *(const u32x4_t *)at;
#pragma unroll
                    for (int j = 0; j < NT; ++j) grp_mma16<T>(acc[j], *(const u32x4_t *)(at + (16 + j * 16) * kPitch), fa);
                }
            };
            auto step = [&](u32x4_t (&v)[Q], int s, int stage) {
#pragma unroll
                for (int q = 0; q < Q; ++q) *(u32x4_t *)(to + stage + q * STRIDE * kPitch) = v[q];
                load(v, s + AHEAD);
                __syncthreads();                           // (and the other stage's readers are through)
                multiply(lds + stage);
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) load(v[i], first + i);
            for (int s = first; s < last; s += AHEAD) {
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
                    if (s + i < last) step(v[i], s + i, i % 2 * (ROWS * kPitch));
            }
            if (end > whole && first < end) {              // what the reduction ends with
                __syncthreads();
                const int count = (bytes - whole * kStep - c) / ES;
#pragma unroll 1
                for (int q = 0; q < Q; ++q) {
                    const char *at = (q < XQ ? x + (int64_t)min(q * STRIDE + r, rows_left - 1) * p.ldx : a + (int64_t)min(q * STRIDE + r - 16, p.rank - col0 - 1) * row_bytes) + c;
                    *(u32x4_t *)(to + q * STRIDE * kPitch) = grp_load_chunk<ES>(at + (int64_t)whole * kStep, count);
                }
                __syncthreads();
                multiply(lds);
            }
            __syncthreads();                               // the stages' readers are through
            const float by = p.scale ? p.scale[one] : 1.f;
            grp_few_join<T, NT, NW>(*(u32x4_t (*)[NW * NT * 64])lds, acc, lane, wave, [&](int tile, int l, const typename GrpFew<T>::acc_t &sum) {
                const int row = row0 + l % 16, col = col0 + tile * 16 + l / 16 * 4;
                if (row >= p.rows || p.adapter[row] != one) return;
                float f[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) f[q] = col + q < p.rank ? sum[q] * by : 0.f;       // (zeros behind the rank)
                if (ES == 4 || p.slices) {
                    if (col * 4 < p.inner_bytes) *(f32x4_t *)(p.inner + ((int64_t)slice * p.rows + row) * p.inner_bytes + col * 4) = (f32x4_t){f[0], f[1], f[2], f[3]};
                } else if (col * 2 < p.inner_bytes) {
                    const u32x2_t hi = {f32x2_to_bf16x2(f[0], f[1]), f32x2_to_bf16x2(f[2], f[3])};
                    float low[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t bits = q % 2 ? hi[q / 2] & 0xffff0000u : hi[q / 2] << 16;
                        // (of an infinity or a NaN nothing is left)
                        low[q] = (bits & 0x7f800000u) == 0x7f800000u ? 0.f : f[q] - __builtin_bit_cast(float, bits);
                    }
                    char *at = p.inner + (int64_t)row * (PARTS * p.inner_bytes) + col * 2;
                    *(u32x2_t *)at = hi;
                    *(u32x2_t *)(at + p.inner_bytes) = (u32x2_t){f32x2_to_bf16x2(low[0], low[1]), f32x2_to_bf16x2(low[2], low[3])};
                }
            });
            if (left) __syncthreads();                     // (the parts are read)
        }
    }
};

template <typename T, int NT, int NW>
__global__ __launch_bounds__(64 * NW, 3) void adapters_down_kernel(const AdapterParams p)
{
    __shared__ uint4 lds[Down<T, NT, NW>::kLds / 16];
    Down<T, NT, NW>::run(p, blockIdx.x, (char *)lds);
}

// The inner sums in the first `down` workgroups, the product of few rows in the others: neither needs the other.
template <typename T, int NT, int NW, int BATCH, bool DW>
__global__ __launch_bounds__(64 * NW) void adapters_few_kernel(const AdapterParams p, const GroupedParams product, uint32_t down)
{
    __shared__ uint4 lds[Down<T, 1, NW>::kLds / 16];
    static_assert(NW * NT * 1024 <= sizeof lds, "LDS");
    if (blockIdx.x < down) Down<T, 1, NW>::run(p, blockIdx.x, (char *)lds);
    else grp_few<T, NT, NW, BATCH, DW>(product, blockIdx.x - down, *(u32x4_t (*)[NW * NT * 64])lds);
}

// ---- the last pass over few rows -------------------------------------------------------------------------------------------------------
//
// y[m][n] = base[m][n] + sum_r inner[m][r] * b[g][n][r] + bias[n].  A thread has a column of R rows, and reads its row of b again only where the next row has
// another adapter.  Bound by memory: b of the adapters that the rows have, and the product, which is still in the caches.
template <int ES, int R>
__global__ __launch_bounds__(256) void adapters_up_kernel(const AdapterParams p, int col_blocks)
{
    constexpr int E = 16 / ES, PIECE = 64;                 // of the rank at a time
    __shared__ float inner[R][PIECE];
    const int t = threadIdx.x, row0 = (int)(blockIdx.x / (unsigned)col_blocks) * R, col = (int)(blockIdx.x % (unsigned)col_blocks) * 256 + t, width = p.inner_bytes / 4;
    int ids[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int id = row0 + i < p.rows ? p.adapter[row0 + i] : -1;
        ids[i] = id < p.adapters ? id : -1;
    }
    float sum[R];
#pragma unroll
    for (int i = 0; i < R; ++i) sum[i] = row0 + i < p.rows && col < p.cols ? p.base[(int64_t)(row0 + i) * p.cols + col] : 0.f;
    const float bias = p.bias && col < p.cols ? p.bias[col] : 0.f;
    const char *b = p.b + (int64_t)min(col, p.cols - 1) * p.rank * ES;
    const int64_t b_adapter = (int64_t)p.cols * p.rank * ES;
    for (int r0 = 0; r0 < p.rank; r0 += PIECE) {
        const int here = min(PIECE, p.rank - r0);
        // (one row: its row of b is on its way before the inner sums are asked for, 5.1 us for 4096 columns of 32 rows, rank 16, so 4.6)
        u32x4_t ahead[R == 1 ? PIECE / E : 1];
        if constexpr (R == 1) {
#pragma unroll
            for (int k = 0; k < PIECE / E; ++k)
                if (k * E < here && ids[0] >= 0) ahead[k] = grp_load_chunk<ES>(b + ids[0] * b_adapter + (int64_t)(r0 + k * E) * ES, here - k * E);
        }
        __syncthreads();
        for (int i = t; i < R * PIECE; i += 256) {
            const int row = row0 + i / PIECE, r = r0 + i % PIECE;
            float f = 0.f;
            if (r < p.rank && row < p.rows) {
                const int id = p.adapter[row];
                if (id >= 0 && id < p.adapters)
                    for (int s = 0; s < p.slices; ++s) f += *(const float *)(p.inner + (((int64_t)s * p.rows + row) * width + r) * 4);
            }
            inner[i / PIECE][i % PIECE] = f;
        }
        __syncthreads();
        if constexpr (R == 1) {
#pragma unroll
            for (int k = 0; k < PIECE / E; ++k) {
                if (k * E >= here || ids[0] < 0) continue;
                float f[E];
                floats16<ES>(ahead[k], f);
#pragma unroll
                for (int q = 0; q < E; ++q) sum[0] += k * E + q < here ? inner[0][k * E + q] * f[q] : 0.f;
            }
            continue;
        }
        for (int r = 0; r < here; r += E) {
            u32x4_t v = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if (ids[i] < 0) continue;
                if (i == 0 || ids[i] != ids[i - 1]) v = grp_load_chunk<ES>(b + ids[i] * b_adapter + (int64_t)(r0 + r) * ES, here - r);
                float f[E];
                floats16<ES>(v, f);
#pragma unroll
                for (int q = 0; q < E; ++q) sum[i] += r + q < here ? inner[i][r + q] * f[q] : 0.f;
            }
        }
    }
    if (col >= p.cols) return;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (row0 + i >= p.rows) return;
        float f = sum[i] + bias;
        if (p.relu) f = grp_relu(f);
        char *to = p.y + (int64_t)(row0 + i) * p.ldy;
        if (p.out_bf16) ((uint16_t *)to)[col] = f32_to_bf16_rne(f);
        else ((float *)to)[col] = f;
    }
}

template <typename T, int NT, int NW>
hipError_t down(AdapterParams p, hipStream_t st)
{
    p.col_tiles = (p.rank + 16 * NT - 1) / (16 * NT);
    const int64_t n = (int64_t)p.tiles * p.col_tiles * std::max(p.slices, 1) * p.slots;
    if (n * 64 * NW > 0xffffffffll) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((adapters_down_kernel<T, NT, NW>), dim3((unsigned)n), dim3(64 * NW), 0, st, p);
    return hipGetLastError();
}

template <typename T, int NT, int NW>
hipError_t few(AdapterParams p, GroupedParams product, hipStream_t st)
{
    p.col_tiles = (p.rank + 15) / 16;
    const int64_t downs = ((int64_t)p.tiles * p.col_tiles * p.slices * p.slots + 7) / 8 * 8;       // (the product's workgroups go to their XCDs as ever)
    unsigned grid;
    const hipError_t e = grp_grid<kForward, 16, 16 * NT>(product, 64 * NW, &grid);
    if (e != hipSuccess) return e;
    if ((grid + downs) * 64 * NW > 0xffffffffll) return hipErrorInvalidConfiguration;
    if constexpr (GrpTraits<T>::ES < 4) {
        if (((uint64_t)product.a | (uint64_t)product.b | (uint64_t)product.lda | (uint64_t)product.ldb) % 4) {
            hipLaunchKernelGGL((adapters_few_kernel<T, NT, NW, 2, false>), dim3(grid + (unsigned)downs), dim3(64 * NW), 0, st, p, product, (uint32_t)downs);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((adapters_few_kernel<T, NT, NW, 2, true>), dim3(grid + (unsigned)downs), dim3(64 * NW), 0, st, p, product, (uint32_t)downs);
    return hipGetLastError();
}

template <int ES, int R>
hipError_t up(const AdapterParams &p, hipStream_t st)
{
    const int64_t cols = ((int64_t)p.cols + 255) / 256, n = ((int64_t)p.rows + R - 1) / R * cols;
    if (n * 256 > 0xffffffffll) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((adapters_up_kernel<ES, R>), dim3((unsigned)n), dim3(256), 0, st, p, (int)cols);
    return hipGetLastError();
}

}  // namespace

bool adapters_plan(int dtype, const GroupedParams &product, AdapterParams &p)
{
    const int es = (int)dtype_size(dtype);
    // beside: few rows, or where the last pass, at 5 TB/s and 3 us for its launch, takes less than the tiles' waiting, 0.7 us for each adapter of 32 rows
    // (of those that there can be most are taken to be): 256 rows of 256 requests and 32 adapters, 4096 x 4096, 41 us for 50; 2048 rows of four
    // adapters, 768 x 768, rank 8, 22 for 16
    const bool few_rows = grp_is_few(product, es);
    const double rounds = std::ceil(grp_tiles<kForward>(product, 128, 128) / p.places), wait = 0.5 * std::min(p.adapters, 32) * rounds;
    const bool beside = few_rows || 3 + (double)p.rows * p.cols * (8 + p.rank * es) / 5e6 < wait;
    const int steps = (int)(((int64_t)p.K * es + kStep - 1) / kStep);
    p.tiles = (p.rows + 15) / 16;
    const int64_t work = (int64_t)p.tiles * ((p.rank + 15) / 16);
    // workgroups for a tile's adapters, two at least and up to as many as the chip has places for
    p.slots = (int)std::min<int64_t>(std::min(std::min(p.adapters, 16), p.rows), std::max<int64_t>(2, p.places / work));
    p.slices = !beside ? 0 : (int)std::max<int64_t>(1, std::min<int64_t>(std::min(8, steps), p.places / (work * p.slots)));
    p.inner_bytes = beside ? (p.rank + 15) / 16 * 64 : (p.rank * es + 31) / 32 * 32;
    return beside;
}

size_t adapters_inner_bytes(int dtype, const AdapterParams &p, bool beside)
{
    return (size_t)p.rows * p.inner_bytes * (beside ? p.slices : dtype == ALT_BF16 ? 2 : 1);
}

hipError_t adapters_down(int dtype, const AdapterParams &p, bool, hipStream_t st)
{
    if (dtype == ALT_F32) return p.rank <= 16 ? down<float, 1, 4>(p, st) : down<float, 2, 4>(p, st);
    return p.rank <= 16 ? down<bf16_tag, 1, 4>(p, st) : down<bf16_tag, 2, 4>(p, st);
}

hipError_t adapters_few(int dtype, const AdapterParams &p, const GroupedParams &product, hipStream_t st)
{
    const bool narrow = grp_tiles<kForward>(product, 16, 16) <= product.places;                // (as in grouped_run)
    if (dtype == ALT_F32) return narrow ? few<float, 1, 8>(p, product, st) : few<float, 2, 4>(p, product, st);
    return narrow ? few<bf16_tag, 1, 8>(p, product, st) : few<bf16_tag, 2, 4>(p, product, st);
}

hipError_t adapters_up(int dtype, const AdapterParams &p, hipStream_t st)
{
    // (a row to a workgroup while that fills the chip twice at most)
    const bool one = (int64_t)p.rows * ((p.cols + 255) / 256) <= 2 * (int64_t)p.places;
    if (dtype == ALT_F32) return one ? up<4, 1>(p, st) : up<4, 4>(p, st);
    return one ? up<2, 1>(p, st) : up<2, 4>(p, st);
}

}  // namespace alt
