// Low-rank adapters: the inner sums of every row, and the last pass over few rows.
#include "adapters.h"
#include "rows.h"

namespace alt {
namespace {

// ---- products of few rows ------------------------------------------------------------------------------------------------------------
//
// Tiles of 16 RT rows by 16 NT columns whose operands, both with the reduction contiguous, come in pieces of 128 bytes a row, whole cache lines, the waves'
// in turn.  A wave takes its pieces through LDS of its own and waits for no other: 100 x 2048 x 2048 bf16 with 50 adapters of rank 16 14.6 us, where the waves
// shared all pieces at barriers 15.6.  (Straight into the fragments of the 16-row matrix instructions every load touches 64 cache lines: the inner sums of 8192
// rows of 4096, rank 32, took 37 us, so 24.)  AHEAD pieces are on their way in registers; four instead of two, eight waves instead of four and 32 rows
// instead of 16 took 25 to 30.  Chunk c of a piece of row r lies at c ^ (r % 8), so that 16 rows' chunks are at distinct banks.
constexpr int kPiece = 128, kWaves = 4, kStep = kWaves * kPiece;

template <typename T, int RT, int NT, int AHEAD>
struct Core {
    static constexpr int ES = GrpTraits<T>::ES, SUMS = GrpTraits<T>::SUMS, THREADS = 64 * kWaves, A = 16 * RT, ROWS = A + 16 * NT;
    static constexpr int Q = ROWS / 8, AQ = A / 8, kLds = ROWS * kStep;                                   // loads of a piece; of its rows of a
    static_assert(kWaves * RT * NT * 1024 <= kLds && kLds <= 64 * 1024, "LDS");
    typedef typename GrpFew<T>::acc_t acc_t;

    // This wave's sums of rows a (a_rows of them, lda bytes apart) by rows b, over the steps first .. end - 1 of kStep of `bytes` of each.  (Behind the last row
    // the last again, whose sums nobody stores.)
    static __device__ __forceinline__ void sums(const char *a, int64_t lda, int a_rows, const char *b, int64_t ldb, int b_rows, int bytes, int first, int end, char *lds,
                                                acc_t (&acc)[RT][NT][SUMS])
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane / 8, c = lane % 8;
        const int whole = bytes / kPiece, from_piece = first * kWaves + wave, n = max(0, (min(end * kWaves, whole) - from_piece + kWaves - 1) / kWaves);
        char *const stage = lds + wave * (ROWS * kPiece);
        uint32_t from[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) from[q] = (uint32_t)(q < AQ ? min(q * 8 + r, a_rows - 1) * (int)lda : min(q * 8 + r - A, b_rows - 1) * (int)ldb) + c * 16;
        u32x4_t v[AHEAD][Q];
        auto load = [&](u32x4_t (&v)[Q], int k) {
            const int64_t at = (int64_t)(from_piece + k * kWaves) * kPiece;
#pragma unroll
            for (int q = 0; q < Q; ++q) __builtin_memcpy(&v[q], (q < AQ ? a : b) + at + from[q], 16);
        };
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int s = 0; s < SUMS; ++s) acc[i][j][s] = (acc_t){0, 0, 0, 0};
        auto put = [&](const u32x4_t (&v)[Q]) {
#pragma unroll
            for (int q = 0; q < Q; ++q) *(u32x4_t *)(stage + q * (8 * kPiece) + r * kPiece + (c ^ r) * 16) = v[q];
        };
        auto multiply = [&] {
            wave_sync();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const char *at = stage + lane % 16 * kPiece + ((h * 4 + lane / 16) ^ (lane % 8)) * 16;
                u32x4_t fa[RT];
#pragma unroll
                for (int i = 0; i < RT; ++i) fa[i] = *(const u32x4_t *)(at + i * 16 * kPiece);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const u32x4_t fb = *(const u32x4_t *)(at + (A + j * 16) * kPiece);
#pragma unroll
                    for (int i = 0; i < RT; ++i) grp_mma16<T>(acc[i][j], fb, fa[i]);
                }
            }
            wave_sync();
        };
        auto step = [&](u32x4_t (&v)[Q], int k, auto MORE) {
            put(v);
            if (decltype(MORE)::value || k + AHEAD < n) load(v, k + AHEAD);
            multiply();
        };
        // (without branches around the loads while there are more, so that no piece waits for more of them than it needs; what there is none of is the last
        // again)
        if (n > 0) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) load(v[i], min(i, n - 1));
            int k = 0;
            for (; k + 2 * AHEAD <= n; k += AHEAD) {
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) step(v[i], k + i, std::true_type{});
            }
            for (; k < n; k += AHEAD) {
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
                    if (k + i < n) step(v[i], k + i, std::false_type{});
            }
        }
        if (bytes > whole * kPiece && whole >= from_piece && whole < end * kWaves && whole % kWaves == wave) {     // what the reduction ends with
            const int count = (bytes - whole * kPiece - c * 16) / ES;
            u32x4_t last[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) last[q] = grp_load_chunk<ES>((q < AQ ? a : b) + (int64_t)whole * kPiece + from[q], count);
            put(last);
            multiply();
        }
        __syncthreads();                                   // the stages' readers are through
    }

    // The waves' sums added in the waves' order: f(row, first of four columns, sum), of the tile.
    template <typename F>
    static __device__ __forceinline__ void join(char *lds, acc_t (&acc)[RT][NT][SUMS], F f)
    {
        u32x4_t *part = (u32x4_t *)lds;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if constexpr (SUMS == 4) acc[i][j][0] = (acc[i][j][0] + acc[i][j][1]) + (acc[i][j][2] + acc[i][j][3]);
                part[((wave * RT + i) * NT + j) * 64 + lane] = __builtin_bit_cast(u32x4_t, acc[i][j][0]);
            }
        __syncthreads();
        for (int s = threadIdx.x; s < RT * NT * 64; s += THREADS) {
            acc_t sum = __builtin_bit_cast(acc_t, part[s]);
#pragma unroll
            for (int w = 1; w < kWaves; ++w) sum += __builtin_bit_cast(acc_t, part[w * RT * NT * 64 + s]);
            f(s / 64 / NT * 16 + s % 16, s / 64 % NT * 16 + s % 64 / 16 * 4, sum);
        }
    }
};

// Steps of one of `slices` parts of a reduction.
__device__ __forceinline__ void slice_steps(int bytes, int slices, int slice, int &first, int &end)
{
    const int steps = (bytes + kStep - 1) / kStep, per = (steps + slices - 1) / slices;
    first = slice * per;
    end = min(first + per, steps);
}

// ---- inner sums: such a product once for each adapter that 16 rows have
//
// Prompts have one or two, sequences that decode up to 16, so the adapters of a tile are spread over `slots` workgroups, those of a first adapter before the
// others (which mostly have nothing to do).
template <typename T, int NT>
struct Down {
    using C = Core<T, 1, NT, 2>;
    static constexpr int ES = C::ES, ROWS = C::A, kLds = C::kLds;

    // slices == 0: of the fused form (one slice, in bf16 in two parts)
    static __device__ __forceinline__ void run(const AdapterParams &p, uint32_t wg, char *lds)
    {
        constexpr int PARTS = ES == 2 ? 2 : 1;
        const int lane = threadIdx.x & 63;
        const uint32_t slices = max(p.slices, 1);
        const int col0 = (int)(wg % (uint32_t)p.col_tiles) * 16 * NT;
        uint32_t rest = wg / (uint32_t)p.col_tiles;
        const int row0 = (int)(rest % (uint32_t)p.tiles) * ROWS;
        rest /= (uint32_t)p.tiles;
        const int slice = (int)(rest % slices), slot = (int)(rest / slices);
        if (slot >= p.slots) return;
        const int rows_left = p.rows - row0;
        const int id = p.adapter[row0 + min(lane % ROWS, rows_left - 1)];
        uint64_t left = __ballot(lane % ROWS < rows_left && id >= 0 && id < p.adapters);
        const int64_t row_bytes = (int64_t)p.K * ES;
        int first, end;
        slice_steps((int)row_bytes, (int)slices, slice, first, end);
        for (int n = 0; left; ++n) {
            const int one = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
            left &= ~__ballot(id == one);
            if (n % p.slots != slot) continue;
            typename C::acc_t acc[1][NT][C::SUMS];
            C::sums(p.x + (int64_t)row0 * p.ldx, p.ldx, rows_left, p.a + ((int64_t)one * p.rank + col0) * row_bytes, row_bytes, p.rank - col0, (int)row_bytes, first, end, lds, acc);
            const float by = p.scale ? p.scale[one] : 1.f;
            C::join(lds, acc, [&](int r, int at, const typename C::acc_t &sum) {
                const int row = row0 + r, col = col0 + at;
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

template <typename T, int NT>
__global__ __launch_bounds__(64 * kWaves) void adapters_down_kernel(const AdapterParams p, uint32_t begin)
{
    using D = Down<T, NT>;
    __shared__ uint4 lds[D::kLds / 16];
    D::run(p, begin + blockIdx.x, (char *)lds);
}

// The inner sums in the first `down` workgroups, the shared product in the others: neither needs the other.  Column tiles that run together are one XCD's
// (workgroups go to the XCDs in turn), rows first, so that a tile of w is read from memory once.
template <typename T, int RT, int NT>
__global__ __launch_bounds__(64 * kWaves) void adapters_few_kernel(const AdapterParams p, uint32_t begin, uint32_t down)
{
    using C = Core<T, RT, NT, 2>;
    constexpr int ES = C::ES;
    __shared__ uint4 lds[(C::kLds > Down<T, 1>::kLds ? C::kLds : Down<T, 1>::kLds) / 16];
    if (begin + blockIdx.x < down) {
        Down<T, 1>::run(p, begin + blockIdx.x, (char *)lds);
        return;
    }
    const uint32_t wg = begin + blockIdx.x - down, row_tiles = (uint32_t)(p.rows + 16 * RT - 1) / (16 * RT), col_tiles = (uint32_t)(p.cols + 16 * NT - 1) / (16 * NT);
    const uint32_t tiles = row_tiles * col_tiles * (uint32_t)p.base_slices, per = (tiles + 7) / 8, tile = (wg & 7) * per + (wg >> 3);
    if ((wg >> 3) >= per || tile >= tiles) return;
    const int row0 = (int)(tile % row_tiles) * 16 * RT, col0 = (int)(tile / row_tiles % col_tiles) * 16 * NT, slice = (int)(tile / row_tiles / col_tiles);
    int first, end;
    slice_steps(p.K * ES, p.base_slices, slice, first, end);
    typename C::acc_t acc[RT][NT][C::SUMS];
    C::sums(p.x + (int64_t)row0 * p.ldx, p.ldx, p.rows - row0, p.w + (int64_t)col0 * p.ldw, p.ldw, p.cols - col0, p.K * ES, first, end, (char *)lds, acc);
    float *base = p.base + (int64_t)slice * p.rows * p.cols;
    C::join((char *)lds, acc, [&](int r, int at, const typename C::acc_t &sum) {
        const int row = row0 + r, col = col0 + at;
        if (row >= p.rows || col >= p.cols) return;
        float *to = base + (int64_t)row * p.cols + col;
        if (p.cols % 4 == 0) {
            *(f32x4_t *)to = (f32x4_t){sum[0], sum[1], sum[2], sum[3]};
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (col + q < p.cols) to[q] = sum[q];
        }
    });
}

// ---- the last pass over few rows -------------------------------------------------------------------------------------------------------
//
// y[m][n] = base[m][n] + sum_r inner[m][r] * b[g][n][r] + bias[n].  A thread has a column of R rows, and reads its row of b again only where the next row has
// another adapter.  Bound by memory: b of the adapters that the rows have, and the product, which is still in the caches.
template <int ES, int R>
__global__ __launch_bounds__(256) void adapters_up_kernel(const AdapterParams p, uint32_t begin, uint32_t col_blocks)
{
    constexpr int E = 16 / ES, PIECE = 64;                 // of the rank at a time
    __shared__ float inner[R][PIECE];
    const uint32_t wg = begin + blockIdx.x;
    const int t = threadIdx.x, row0 = (int)(wg / col_blocks) * R, col = (int)(wg % col_blocks) * 256 + t, width = p.inner_bytes / 4;
    int ids[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int id = row0 + i < p.rows ? p.adapter[row0 + i] : -1;
        ids[i] = id < p.adapters ? id : -1;
    }
    float sum[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        sum[i] = 0.f;
        if (row0 + i < p.rows && col < p.cols)
            for (int s = 0; s < p.base_slices; ++s) sum[i] += p.base[((int64_t)s * p.rows + row0 + i) * p.cols + col];
    }
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

// f(begin, how many) of as many launches as n workgroups of 256 threads take: one has fewer than 2^32 threads.  (Whole eights, for the XCDs.)
template <typename F>
hipError_t in_launches(int64_t n, F f)
{
    static_assert(64 * kWaves == 256, "threads of a workgroup");
    constexpr int64_t most = (1 << 24) - 8;
    if (n > 0xffffffffll) return hipErrorInvalidConfiguration;
    for (int64_t begin = 0; begin < n; begin += most) f((uint32_t)begin, dim3((unsigned)std::min(n - begin, most)));
    return hipGetLastError();
}

template <typename T, int NT>
hipError_t down(AdapterParams p, hipStream_t st)
{
    p.col_tiles = (p.rank + 16 * NT - 1) / (16 * NT);
    const int64_t n = (int64_t)p.tiles * p.col_tiles * std::max(p.slices, 1) * p.slots;
    return in_launches(n, [&](uint32_t begin, dim3 grid) { hipLaunchKernelGGL((adapters_down_kernel<T, NT>), grid, dim3(64 * kWaves), 0, st, p, begin); });
}

template <typename T, int RT, int NT>
hipError_t few(AdapterParams p, hipStream_t st)
{
    p.col_tiles = (p.rank + 15) / 16;
    const int64_t downs = ((int64_t)p.tiles * p.col_tiles * p.slices * p.slots + 7) / 8 * 8;
    const int64_t tiles = ((int64_t)p.rows + 16 * RT - 1) / (16 * RT) * ((p.cols + 16 * NT - 1) / (16 * NT)) * p.base_slices;
    const int64_t n = downs + (tiles + 7) / 8 * 8;
    return in_launches(n, [&](uint32_t begin, dim3 grid) { hipLaunchKernelGGL((adapters_few_kernel<T, RT, NT>), grid, dim3(64 * kWaves), 0, st, p, begin, (uint32_t)downs); });
}

template <typename T>
hipError_t few(const AdapterParams &p, hipStream_t st)
{
    if (p.rows <= 16) return few<T, 1, 1>(p, st);
    return p.few_cols == 1 ? few<T, 2, 1>(p, st) : few<T, 2, 2>(p, st);
}

template <int ES, int R>
hipError_t up(const AdapterParams &p, hipStream_t st)
{
    const int64_t cols = ((int64_t)p.cols + 255) / 256, n = ((int64_t)p.rows + R - 1) / R * cols;
    return in_launches(n, [&](uint32_t begin, dim3 grid) { hipLaunchKernelGGL((adapters_up_kernel<ES, R>), grid, dim3(256), 0, st, p, begin, (uint32_t)cols); });
}

}  // namespace

void adapters_plan(int dtype, const GroupedParams &product, AdapterParams &p)
{
    const int es = (int)dtype_size(dtype);
    const double places = p.places;
    const int64_t steps = ((int64_t)p.K * es + kStep - 1) / kStep;
    const int64_t rt = p.rows <= 16 ? 1 : 2, row_tiles = (p.rows + 16 * rt - 1) / (16 * rt);
    p.few_cols = rt == 2 && row_tiles * ((p.cols + 31) / 32) >= p.places ? 2 : 1;
    const int64_t tiles = row_tiles * ((p.cols + 16 * p.few_cols - 1) / (16 * p.few_cols));
    // Times in us.  The last pass runs at 5 TB/s behind its launch.  The fused tiles wait for one adapter of 32 rows after another: 2048 x 4096 x 4096 92 with
    // one adapter, 120 with 8 and 196 with 32 in turn (beside 127, 145 and 166), 1.7 to 2 for each and each round; requests of many rows, which have one or two of
    // them there, wait far less, and 0.5 for each that there can be stands between the two.  The product of few rows takes its tiles' loads from the caches at 13
    // TB/s (fp32, whose matrix instructions take longer, at 7); others come after the launch of the inner sums.  bf16, rank 16, 32 adapters in turn: 128 x 4096 x
    // 4096 30 of few rows and 37 otherwise, 256 x 4096 x 4096 43 and 40, 256 x 1024 x 4096 20 and 39; taken on the slower side are 64 x 8192 x 8192 (57 and 61) and
    // 200 x 8192 x 2048 (few rows 40, beside 38, fused, as it goes, 48).  fp32 60 x 4096 x 4096 39 and 65.
    const double rounds = std::ceil(grp_tiles<kForward>(product, 128, 128) / places), wait = 0.5 * std::min(p.adapters, 32) * rounds;
    const double last = 3 + (double)p.rows * p.cols * (8 + p.rank * es) / 5e6, loads = (double)tiles * 16 * (rt + p.few_cols) * p.K * es;
    GrpTime t;
    (void)grp_choose<kForward>(product, es, &t);
    const double few = 4 + loads / (es == 4 ? 7e6 : 13e6) + last;
    const double other = 10 + (es == 4 ? 8 + 2.0 * p.rows * p.cols * p.K / 50e6 : t.fixed + t.reduction) + std::min(last, wait);
    p.few = p.rows <= 16 || few < other;
    p.beside = p.few || last < wait;
    // (as many workgroups as the chip has places for share a product's reduction, each with eight steps at least)
    p.base_slices = p.few ? (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(8, steps / 8), p.places / tiles)) : 1;
    p.tiles = (p.rows + 15) / 16;
    const int64_t work = (int64_t)p.tiles * ((p.rank + 15) / 16);
    // workgroups for a tile's adapters, two at least and up to as many as the chip has places for
    p.slots = (int)std::min<int64_t>(std::min(std::min(p.adapters, 16), p.rows), std::max<int64_t>(2, p.places / work));
    p.slices = !p.beside ? 0 : (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(8, steps), p.places / (work * p.slots)));
    p.inner_bytes = p.beside ? (p.rank + 15) / 16 * 64 : (p.rank * es + 31) / 32 * 32;
}

size_t adapters_inner_bytes(int dtype, const AdapterParams &p)
{
    return (size_t)p.rows * p.inner_bytes * (p.beside ? p.slices : dtype == ALT_BF16 ? 2 : 1);
}

hipError_t adapters_down(int dtype, const AdapterParams &p, hipStream_t st)
{
    if (dtype == ALT_F32) return p.rank <= 16 ? down<float, 1>(p, st) : down<float, 2>(p, st);
    return p.rank <= 16 ? down<bf16_tag, 1>(p, st) : down<bf16_tag, 2>(p, st);
}

hipError_t adapters_few(int dtype, const AdapterParams &p, hipStream_t st) { return dtype == ALT_F32 ? few<float>(p, st) : few<bf16_tag>(p, st); }

hipError_t adapters_up(int dtype, const AdapterParams &p, hipStream_t st)
{
    // (a row to a workgroup while that fills the chip twice at most)
    const bool one = (int64_t)p.rows * ((p.cols + 255) / 256) <= 2 * (int64_t)p.places;
    if (dtype == ALT_F32) return one ? up<4, 1>(p, st) : up<4, 4>(p, st);
    return one ? up<2, 1>(p, st) : up<2, 4>(p, st);
}

}  // namespace alt
