// Layer norm of rows and its gradients.
//
//   mean = sum_c x / cols,  rstd = 1 / sqrt(sum_c (x - mean)^2 / cols + eps),  u = (x - mean) rstd,  y = u gamma + beta
//   dx = rstd (g - mean_c(g) - u mean_c(g u))  with g = dy gamma,  dgamma = sum_m dy u,  dbeta = sum_m dy
//
// Bound by memory: forward reads x and writes y, backward reads dy and x and writes dx.  TPR threads (a wave, or a workgroup) have a row, in chunks
// that stay in registers from the first sum to the last store, and take one row after another: a thread's columns are the same in all
// of them, so gamma and beta are read once, dgamma and dbeta are summed in registers, and the next row is on its way while this one is reduced.  What the
// workgroups have of dgamma and dbeta goes to the workspace and is joined by a second launch, in the order of the workgroups.  Rows of more than 16384
// columns do not fit: they are read again for every sum.
#include "common.h"
#include "rows.h"

namespace alt {
namespace {

constexpr int kMostCols = 16384;                           // of a row in registers

// Columns of a chunk: what is 16 bytes of x and y, so that lanes side by side load and store side by side; eight where one is bf16 and the other fp32.
template <int XS, int YS> constexpr int kChunk = XS == 4 && YS == 4 ? 4 : 8;

template <int ES, int E>
__device__ __forceinline__ void chunk_floats(const char *p, float (&v)[E])
{
    if constexpr (E * ES == 16) {
        w4_t c;
        __builtin_memcpy(&c, p, 16);
        floats16<ES>(c, v);
    } else {
        floats<ES>(load_chunk<ES>(p), v);
    }
}

// A thread's part of a row: chunks t, t + TPR, ... of `chunks`, as they lie in memory, and one element of the `rest` behind them.  SHIFT: bf16 rows that may begin
// inside a dword; they are loaded from that dword on, with the one that they end in, and shifted when their values are asked for, as memory takes longer
// over addresses inside a dword (gradients of 16384 x 4096, rows 4097 apart, 106 us, so 90; where all rows begin at dwords 78, and 81 if they are looked at so).
template <int ES, int E, int TPR, int K, bool SHIFT>
struct Part {
    static_assert(!SHIFT || (ES == 2 && E == 8), "bf16");
    w4_t c[K][E * ES / 16];
    uint32_t more[SHIFT ? K : 1], shift;   // shift: bytes
    uint32_t bits;                         // of the element
    __device__ __forceinline__ void load(const char *row, int t, int chunks, int rest)
    {
        shift = SHIFT ? __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)row & 2u) : 0u;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i * TPR + t < chunks) {
                const char *at = row + (int64_t)(i * TPR + t) * (E * ES) - shift;
                __builtin_memcpy(&c[i], __builtin_assume_aligned(at, SHIFT ? 4 : ES), E * ES);
                if constexpr (SHIFT) {
                    if (shift) more[i] = *(const uint32_t *)(at + 16);
                }
            }
        bits = 0;
        if (t < rest) {
            const char *at = row + ((int64_t)chunks * E + t) * ES;
            if constexpr (ES == 4) bits = *(const uint32_t *)at;
            else bits = *(const uint16_t *)at;
        }
    }
    // (made of the bits when it is used: made when it is loaded it is waited for there, with all loads before it, 16384 x 4095 131 us for 77)
    __device__ __forceinline__ float last() const { return __builtin_bit_cast(float, ES == 4 ? bits : bits << 16); }
    __device__ __forceinline__ void values(int i, float (&v)[E]) const
    {
        if constexpr (SHIFT) {
            const w4_t w = c[i][0];
            floats16<2>((w4_t){__builtin_amdgcn_alignbyte(w.y, w.x, shift), __builtin_amdgcn_alignbyte(w.z, w.y, shift), __builtin_amdgcn_alignbyte(w.w, w.z, shift),
                               __builtin_amdgcn_alignbyte(more[i], w.w, shift)}, v);
        } else if constexpr (E * ES == 16) {
            floats16<ES>(c[i][0], v);
        } else {
            Chunk<ES> whole;
            __builtin_memcpy(&whole, &c[i], sizeof whole);
            floats<ES>(whole, v);
        }
    }
};

template <int ES, int E>
__device__ __forceinline__ void put_values(char *p, const float (&v)[E])
{
    if constexpr (E * ES == 16) put_streaming(p, chunk16_of<ES>(v));
    else put_chunk<ES>(p, chunk_of<ES>(v));
}

// fp32 values of a thread's columns: those of its chunks and the one behind them.
template <int E, int K>
struct Columns {
    float v[K][E], last;
    __device__ __forceinline__ void fill(float f)
    {
#pragma unroll
        for (int i = 0; i < K; ++i)
#pragma unroll
            for (int q = 0; q < E; ++q) v[i][q] = f;
        last = f;
    }
    template <int TPR>
    __device__ __forceinline__ void load(const float *p, int t, int chunks, int rest)
    {
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i * TPR + t < chunks) chunk_floats<4, E>((const char *)(p + (i * TPR + t) * E), v[i]);
        if (t < rest) last = p[chunks * E + t];
    }
};

// N sums over the TPR threads of a row, the same in all of them, for the G rows of a workgroup at once.  Two sets of parts in turn, so that one barrier a
// call is enough.
template <int TPR, int G, int N>
struct RowSum {
    static constexpr int WAVES = TPR / 64;
    typedef float Parts[2][G][WAVES][N];
    Parts *part;
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N])
    {
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
        if constexpr (WAVES > 1) {
            const int group = threadIdx.x / TPR;
            if (threadIdx.x % 64 == 0) {
#pragma unroll
                for (int n = 0; n < N; ++n) (*part)[turn][group][threadIdx.x % TPR / 64][n] = v[n];
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                v[n] = (*part)[turn][group][0][n];
#pragma unroll
                for (int i = 1; i < WAVES; ++i) v[n] += (*part)[turn][group][i][n];
            }
            turn ^= 1;
        }
    }
};

template <int E>
__device__ __forceinline__ void put_sums(float *p, const float (&v)[E])
{
    __builtin_memcpy(p, v, E * 4);
}

template <int TPR> constexpr int kThreadsOf = TPR < 256 ? 256 : TPR;

template <int XS, int YS, int TPR, int KEEP, bool SHIFT>
__global__ __launch_bounds__(kThreadsOf<TPR>) void norm_kernel(const char *x, int64_t ldx, const float *gamma, const float *beta, char *y, int64_t ldy, float *mean_out,
                                                               float *rstd_out, int64_t rows, int cols, float eps)
{
    constexpr int G = kThreadsOf<TPR> / TPR, E = kChunk<XS, YS>, K = KEEP * 8 / E;
    __shared__ typename RowSum<TPR, G, 1>::Parts part;
    RowSum<TPR, G, 1> sum{&part};
    const int t = threadIdx.x % TPR, chunks = cols / E, rest = cols % E;
    const int64_t step = (int64_t)gridDim.x * G;
    int64_t row = (int64_t)blockIdx.x * G + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    if (row >= rows) return;
    Part<XS, E, TPR, K, SHIFT> next;
    next.load(x + row * ldx, t, chunks, rest);
    Columns<E, K> g, b;
    g.fill(1.f);
    b.fill(0.f);
    if (gamma) g.template load<TPR>(gamma, t, chunks, rest);
    if (beta) b.template load<TPR>(beta, t, chunks, rest);
    const float n = (float)cols;
    for (; row < rows; row += step) {
        const Part<XS, E, TPR, K, SHIFT> mine = next;
        if (row + step < rows) next.load(x + (row + step) * ldx, t, chunks, rest);
        float v[K][E], s[1] = {mine.last()};
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i * TPR + t < chunks) {
                mine.values(i, v[i]);
#pragma unroll
                for (int q = 0; q < E; ++q) s[0] += v[i][q];
            }
        sum(s);
        const float mean = s[0] / n;
        s[0] = t < rest ? (mine.last() - mean) * (mine.last() - mean) : 0.f;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i * TPR + t < chunks) {
#pragma unroll
                for (int q = 0; q < E; ++q) {
                    v[i][q] -= mean;
                    s[0] += v[i][q] * v[i][q];
                }
            }
        sum(s);
        const float rstd = 1.f / sqrtf(s[0] / n + eps);
        if (t == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
        char *to = y + row * ldy;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i * TPR + t < chunks) {
#pragma unroll
                for (int q = 0; q < E; ++q) v[i][q] = v[i][q] * rstd * g.v[i][q] + b.v[i][q];
                put_values<YS, E>(to + (int64_t)(i * TPR + t) * (E * YS), v[i]);
            }
        if (t < rest) store_element<YS>(to + ((int64_t)chunks * E + t) * YS, (mine.last() - mean) * rstd * g.last + b.last);
    }
}

// dx, and this workgroup's part of dgamma and dbeta (`sums`: 2 x cols for each workgroup, or null).  G rows at once; with one chunk a thread
// keeps the next row on its way, with two there are no registers for that.
template <int XS, int YS, int TPR, int KEEP, int THREADS, bool SHIFT>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(const char *dy, int64_t ldy, const char *x, int64_t ldx, const float *mean, const float *rstd, const float *gamma,
                                                            char *dx, float *sums, int64_t rows, int cols)
{
    constexpr int G = THREADS / TPR, E = kChunk<XS, YS>, K = KEEP * 8 / E;
    constexpr bool AHEAD = KEEP == 1;
    __shared__ typename RowSum<TPR, G, 2>::Parts part;
    RowSum<TPR, G, 2> sum{&part};
    const int t = threadIdx.x % TPR, group = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR), chunks = cols / E, rest = cols % E;
    const int64_t step = (int64_t)gridDim.x * G;
    Part<XS, E, TPR, K, SHIFT> next_x;
    Part<YS, E, TPR, K, SHIFT> next_dy;
    float next_m = 0.f, next_r = 0.f;
    auto load = [&](int64_t row) {
        if (row >= rows) return;
        next_x.load(x + row * ldx, t, chunks, rest);
        next_dy.load(dy + row * ldy, t, chunks, rest);
        next_m = mean[row];
        next_r = rstd[row];
    };
    Columns<E, K> g, dg, db;
    g.fill(1.f);
    dg.fill(0.f);
    db.fill(0.f);
    if (AHEAD) load((int64_t)blockIdx.x * G + group);
    if (gamma) g.template load<TPR>(gamma, t, chunks, rest);
    const float n = (float)cols;
    // (all groups go round as often as the first, for the barriers of their sums)
    for (int64_t first = (int64_t)blockIdx.x * G; first < rows; first += step) {
        const int64_t row = first + group;
        const bool is = row < rows;
        if constexpr (!AHEAD) {
            load(row);
        }
        const Part<XS, E, TPR, K, SHIFT> mine_x = next_x;
        const Part<YS, E, TPR, K, SHIFT> mine_dy = next_dy;
        const float m = next_m, r = next_r;
        if (AHEAD) load(row + step);
        float u[K][E], w[K][E], s[2] = {0.f, 0.f}, last_u = 0.f, last_g = 0.f;
        auto values = [&](int i, float mean, float (&u)[E], float (&w)[E]) {
            mine_x.values(i, u);
            mine_dy.values(i, w);
#pragma unroll
            for (int q = 0; q < E; ++q) u[q] = (u[q] - mean) * r;
        };
        if (is) {
            last_u = t < rest ? (mine_x.last() - m) * r : 0.f;
            last_g = mine_dy.last() * g.last;
            s[0] = last_g;
            s[1] = last_g * last_u;
            dg.last += mine_dy.last() * last_u;
            db.last += mine_dy.last();
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (i * TPR + t < chunks) {
                    values(i, m, u[i], w[i]);
#pragma unroll
                    for (int q = 0; q < E; ++q) {
                        dg.v[i][q] += w[i][q] * u[i][q];
                        db.v[i][q] += w[i][q];
                        w[i][q] *= g.v[i][q];
                        s[0] += w[i][q];
                        s[1] += w[i][q] * u[i][q];
                    }
                }
        }
        sum(s);
        if (!is) continue;
        const float sg = s[0] / n, sgu = s[1] / n;
        char *to = dx + row * ldx;
        float again = m;
        if constexpr (!AHEAD) asm volatile("" : "+v"(again));              // (what the sums were made of is made again, not kept)
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i * TPR + t < chunks) {
                if constexpr (!AHEAD) {
                    values(i, again, u[i], w[i]);
#pragma unroll
                    for (int q = 0; q < E; ++q) w[i][q] *= g.v[i][q];
                }
#pragma unroll
                for (int q = 0; q < E; ++q) w[i][q] = r * (w[i][q] - sg - u[i][q] * sgu);
                put_values<XS, E>(to + (int64_t)(i * TPR + t) * (E * XS), w[i]);
            }
        if (t < rest) store_element<XS>(to + ((int64_t)chunks * E + t) * XS, r * (last_g - sg - last_u * sgu));
    }
    if (!sums) return;
    sums += (int64_t)blockIdx.x * 2 * cols;
    if constexpr (G > 1) {                                 // the groups' sums one after another, into the last group's registers
        __shared__ float to[2][K * E * TPR], ends[2][E];
        for (int k = 0; k < G; ++k) {
            __syncthreads();
            if (k != group) continue;
#pragma unroll
            for (int i = 0; i < K; ++i)
#pragma unroll
                for (int q = 0; q < E; ++q) {
                    const int at = (i * E + q) * TPR + t;
                    if (k) { dg.v[i][q] += to[0][at]; db.v[i][q] += to[1][at]; }
                    to[0][at] = dg.v[i][q];
                    to[1][at] = db.v[i][q];
                }
            if (t < rest) {
                if (k) { dg.last += ends[0][t]; db.last += ends[1][t]; }
                ends[0][t] = dg.last;
                ends[1][t] = db.last;
            }
        }
        if (group != G - 1) return;
    }
#pragma unroll
    for (int i = 0; i < K; ++i)
        if (i * TPR + t < chunks) {
            put_sums<E>(sums + (i * TPR + t) * E, dg.v[i]);
            put_sums<E>(sums + cols + (i * TPR + t) * E, db.v[i]);
        }
    if (t < rest) {
        sums[chunks * E + t] = dg.last;
        sums[cols + chunks * E + t] = db.last;
    }
}

// The workgroups' parts, in a fixed order: 32 columns to a workgroup, 32 threads to a column, each with eight of its parts on their way at once (four
// at once with eight threads to a column took longer than the rest: 2048 x 768 13.2 us for both launches).
constexpr int kJoinGroups = 32;

__global__ __launch_bounds__(32 * kJoinGroups) void norm_join_kernel(const float *sums, int shares, int cols, float *dgamma, float *dbeta)
{
    __shared__ float part[kJoinGroups][32];
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x % 32, width = 2 * (int64_t)cols;
    const int group = threadIdx.x / 32;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < width)
        for (int i0 = group; i0 < shares; i0 += 8 * kJoinGroups) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (i0 + q * kJoinGroups < shares) s[q] += sums[(i0 + q * kJoinGroups) * width + c];
        }
    part[group][threadIdx.x % 32] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    __syncthreads();
    if (group || c >= width) return;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kJoinGroups; ++k) sum += part[k][threadIdx.x];
    float *to = c < cols ? dgamma : dbeta;
    if (to) to[c < cols ? c : c - cols] = sum;
}

// ---- rows that registers do not hold ---------------------------------------------------------------------------------------------

constexpr int kThreads = 256;

template <int XS, int YS>
__global__ __launch_bounds__(kThreads) void norm_long_kernel(const char *x, int64_t ldx, const float *gamma, const float *beta, char *y, int64_t ldy, float *mean_out,
                                                             float *rstd_out, int64_t rows, int cols, float eps)
{
    __shared__ typename RowSum<kThreads, 1, 1>::Parts part;
    RowSum<kThreads, 1, 1> sum{&part};
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const char *from = x + row * ldx;
        char *to = y + row * ldy;
        float s[1] = {0.f};
        for (int c = threadIdx.x; c < cols; c += kThreads) s[0] += element<XS>(from + (int64_t)c * XS);
        sum(s);
        const float mean = s[0] / (float)cols;
        s[0] = 0.f;
        for (int c = threadIdx.x; c < cols; c += kThreads) {
            const float v = element<XS>(from + (int64_t)c * XS) - mean;
            s[0] += v * v;
        }
        sum(s);
        const float rstd = 1.f / sqrtf(s[0] / (float)cols + eps);
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
        for (int c = threadIdx.x; c < cols; c += kThreads)
            store_element<YS>(to + (int64_t)c * YS, (element<XS>(from + (int64_t)c * XS) - mean) * rstd * (gamma ? gamma[c] : 1.f) + (beta ? beta[c] : 0.f));
    }
}

template <int XS, int YS>
__global__ __launch_bounds__(kThreads) void norm_long_dx_kernel(const char *dy, int64_t ldy, const char *x, int64_t ldx, const float *mean, const float *rstd, const float *gamma,
                                                                char *dx, int64_t rows, int cols)
{
    __shared__ typename RowSum<kThreads, 1, 2>::Parts part;
    RowSum<kThreads, 1, 2> sum{&part};
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const char *from = x + row * ldx, *up = dy + row * ldy;
        const float m = mean[row], r = rstd[row];
        float s[2] = {0.f, 0.f};
        for (int c = threadIdx.x; c < cols; c += kThreads) {
            const float g = element<YS>(up + (int64_t)c * YS) * (gamma ? gamma[c] : 1.f);
            s[0] += g;
            s[1] += g * ((element<XS>(from + (int64_t)c * XS) - m) * r);
        }
        sum(s);
        const float sg = s[0] / (float)cols, sgu = s[1] / (float)cols;
        for (int c = threadIdx.x; c < cols; c += kThreads) {
            const float g = element<YS>(up + (int64_t)c * YS) * (gamma ? gamma[c] : 1.f), u = (element<XS>(from + (int64_t)c * XS) - m) * r;
            store_element<XS>(dx + row * ldx + (int64_t)c * XS, r * (g - sg - u * sgu));
        }
    }
}

template <int XS, int YS>
__global__ __launch_bounds__(kThreads) void norm_long_sums_kernel(const char *dy, int64_t ldy, const char *x, int64_t ldx, const float *mean, const float *rstd, float *sums,
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
    sums[(int64_t)blockIdx.y * 2 * cols + c] = dg;
    sums[((int64_t)blockIdx.y * 2 + 1) * cols + c] = db;
}

// ---- launches ----------------------------------------------------------------------------------------------------------------------

// Threads of a row, and its chunks in each thread.
struct Shape { int tpr, keep; };
Shape shape_of(int64_t cols)
{
    if (cols <= 1024) return {64, cols <= 512 ? 1 : 2};
    if (cols <= 4096) return {256, cols <= 2048 ? 1 : 2};
    return {cols <= 8192 ? 512 : 1024, 2};
}

// The gradients': one chunk to a thread (two behind 8192 columns), and a workgroup of 512 threads to a compute unit, which takes several rows at once
// where they are short: more of them keep no more of memory busy, but leave more sums to join (16384 x 4096 bf16 77 us, with two workgroups 82, with 1024
// threads 78, with four workgroups of 256 threads, two chunks each, 99).
constexpr int kGradThreads = 512;
int grad_tpr(int64_t cols)
{
    int tpr = 64;
    while (tpr < 1024 && tpr * 8 < cols) tpr *= 2;
    return tpr;
}
unsigned workgroups(alt_handle_t h, int64_t rows, int64_t cols)
{
    const int tpr = grad_tpr(cols), threads = std::max(tpr, kGradThreads);
    const int64_t per = threads / tpr, cus = h->compute_units > 0 ? h->compute_units : 256;
    return (unsigned)std::min<int64_t>((rows + per - 1) / per, cus);
}
int long_shares(int64_t rows) { return (int)std::min<int64_t>(rows, 64); }

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

int shares_of(alt_handle_t h, const alt_norm_desc_t &d) { return d.cols > kMostCols ? long_shares(d.rows) : (int)workgroups(h, d.rows, d.cols); }

size_t grad_workspace(alt_handle_t h, const alt_norm_desc_t &d) { return d.rows ? (size_t)shares_of(h, d) * 2 * d.cols * 4 + 16 : 0; }

// f(std::integral_constant TPR, KEEP) of a row's shape.
template <typename F>
void by_shape(int64_t cols, F f)
{
    const Shape s = shape_of(cols);
    using std::integral_constant;
    if (s.tpr == 64 && s.keep == 1) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (s.tpr == 64) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (s.tpr == 256 && s.keep == 1) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (s.tpr == 256) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (s.tpr == 512) f(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    else f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

template <typename F>
void grad_by_shape(int64_t cols, F f)
{
    using std::integral_constant;
    switch (grad_tpr(cols)) {
        case 64: f(integral_constant<int, 64>{}, integral_constant<int, 1>{}); break;
        case 128: f(integral_constant<int, 128>{}, integral_constant<int, 1>{}); break;
        case 256: f(integral_constant<int, 256>{}, integral_constant<int, 1>{}); break;
        case 512: f(integral_constant<int, 512>{}, integral_constant<int, 1>{}); break;
        default:
            if (cols <= 8192) f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
            else f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    }
}

// Whether bf16 rows begin inside dwords.
bool inside_dwords(const alt_norm_desc_t &d, const void *p, int64_t stride) { return (uintptr_t)p % 4 || (d.rows > 1 && stride % 2); }

template <int XS, int YS, bool SHIFT = false>
void forward_run(alt_handle_t h, const alt_norm_desc_t &d, const void *x, const float *gamma, const float *beta, void *y, float *mean, float *rstd, hipStream_t st)
{
    const int64_t ldx = d.x_stride * XS, ldy = d.y_stride * YS;
    const int cols = (int)d.cols;
    if (d.cols > kMostCols) {
        hipLaunchKernelGGL((norm_long_kernel<XS, YS>), dim3((unsigned)std::min<int64_t>(d.rows, 1 << 20)), dim3(kThreads), 0, st, (const char *)x, ldx, gamma, beta, (char *)y, ldy, mean,
                           rstd, d.rows, cols, d.eps);
        return;
    }
    by_shape(d.cols, [&](auto tpr, auto keep) {
        constexpr int TPR = decltype(tpr)::value;
        const int64_t per = kThreadsOf<TPR> / TPR, all = (d.rows + per - 1) / per;
        hipLaunchKernelGGL((norm_kernel<XS, YS, TPR, decltype(keep)::value, SHIFT>), dim3((unsigned)std::min<int64_t>(all, (int64_t)h->compute_units * (2048 / kThreadsOf<TPR>))),
                           dim3(kThreadsOf<TPR>), 0, st, (const char *)x, ldx, gamma, beta, (char *)y, ldy, mean, rstd, d.rows, cols, d.eps);
    });
}

template <int XS, int YS, bool SHIFT = false>
void grad_run(alt_handle_t h, const alt_norm_desc_t &d, const void *dy, const void *x, const float *mean, const float *rstd, const float *gamma, void *dx, float *dgamma,
              float *dbeta, float *sums, hipStream_t st)
{
    const int64_t ldx = d.x_stride * XS, ldy = d.y_stride * YS;
    const int cols = (int)d.cols, shares = d.rows ? shares_of(h, d) : 0;
    if (d.cols > kMostCols && d.rows) {
        hipLaunchKernelGGL((norm_long_dx_kernel<XS, YS>), dim3((unsigned)std::min<int64_t>(d.rows, 1 << 20)), dim3(kThreads), 0, st, (const char *)dy, ldy, (const char *)x, ldx, mean,
                           rstd, gamma, (char *)dx, d.rows, cols);
        if (sums)
            hipLaunchKernelGGL((norm_long_sums_kernel<XS, YS>), dim3((unsigned)((cols + kThreads - 1) / kThreads), (unsigned)shares), dim3(kThreads), 0, st, (const char *)dy, ldy,
                               (const char *)x, ldx, mean, rstd, sums, d.rows, cols);
    } else if (d.rows) {
        grad_by_shape(d.cols, [&](auto tpr, auto keep) {
            constexpr int TPR = decltype(tpr)::value, THREADS = TPR > kGradThreads ? TPR : kGradThreads;
            hipLaunchKernelGGL((norm_grad_kernel<XS, YS, TPR, decltype(keep)::value, THREADS, SHIFT>), dim3(workgroups(h, d.rows, d.cols)), dim3(THREADS), 0, st, (const char *)dy, ldy,
                               (const char *)x, ldx, mean, rstd, gamma, (char *)dx, sums, d.rows, cols);
        });
    }
    if (dgamma || dbeta)
        hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)((2 * d.cols + 31) / 32)), dim3(32 * kJoinGroups), 0, st, sums, shares, cols, dgamma, dbeta);
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
        if (d.out_dtype == ALT_F32) forward_run<4, 4>(h, d, x, gamma, beta, y, mean, rstd, st);
        else forward_run<4, 2>(h, d, x, gamma, beta, y, mean, rstd, st);
    } else {
        if (d.out_dtype == ALT_F32) forward_run<2, 4>(h, d, x, gamma, beta, y, mean, rstd, st);
        else if (inside_dwords(d, x, d.x_stride)) forward_run<2, 2, true>(h, d, x, gamma, beta, y, mean, rstd, st);
        else forward_run<2, 2>(h, d, x, gamma, beta, y, mean, rstd, st);
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
    if (s == ALT_OK && columns) s = check_workspace(h, "alt_layer_norm_grad", workspace, ws_bytes, grad_workspace(h, d));
    if (s == ALT_OK) s = check_device(h, "alt_layer_norm_grad");
    if (s != ALT_OK) return s;
    float *part = columns && rows ? (float *)aligned_workspace(workspace) : nullptr;
    const hipStream_t st = (hipStream_t)stream;
    if (d.in_dtype == ALT_F32) {
        if (d.out_dtype == ALT_F32) grad_run<4, 4>(h, d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
        else grad_run<4, 2>(h, d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
    } else {
        if (d.out_dtype == ALT_F32) grad_run<2, 4>(h, d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
        else if (inside_dwords(d, x, d.x_stride) || inside_dwords(d, dy, d.y_stride)) grad_run<2, 2, true>(h, d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
        else grad_run<2, 2>(h, d, dy, x, mean, rstd, gamma, dx, dgamma, dbeta, part, st);
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
    *bytes = grad_workspace(h, d);
    return ALT_OK;
}
