// Matrix products over groups of rows (the experts of a mixture, each with weights of its own), in bf16, fp32 and 8-bit
// integers, and the one 8-bit product, which is such a product with one group:
//
//   kForward   y[m][n]     = sum_k a[m][k] * b[e][n][k]     rows m of group e, a and b k-contiguous
//   kInput     dx[m][k]    = sum_n dy[m][n] * b[e][n][k]    the forward product's gradient by its rows
//   kWeights   dw[e][n][k] = sum_m dy[m][n] * a[m][k]       by its weights, m over the rows of group e
//
// Group e owns the rows [offsets[e], offsets[e + 1]); offsets lie on the device.  The kernels see one problem: `rows` x `cols`
// outputs, reduced over `red`, with a left operand (rows) and a right operand (columns).  An operand lies either with the
// reduction contiguous (one LDS row per operand row) or with its outer index contiguous (one LDS row per step of the
// reduction); fragments of the latter come out of LDS through the transpose read (bf16) or element by element (fp32).
//
// The matrix instructions of the three types take 16 bytes of the reduction per lane (bf16 32x32x16: 8 elements, i8 32x32x32:
// 16; fp32: four instructions of one float each), so tiles are laid out in bytes and one body serves all three.
#pragma once

#include "dconv.h"

namespace alt {

struct i8_tag {};
enum { kForward = 0, kInput = 1, kWeights = 2 };

struct GroupedParams {
    const void *a;             // left operand
    const void *b;             // right operand
    void *y;
    const float *bias;         // [groups][cols] (kForward)
    const float *a_scale;      // [rows] (8 bits)
    const float *b_scale;      // [groups][cols] (8 bits)
    const void *mask;          // output elements whose element here is not positive are zero (kInput), laid out by ldmask
    const int32_t *offsets;    // [groups + 1], or null: one group of all rows
    float *colsum;             // [groups][rows]: sums of the left operand over the reduction (kWeights), or null
    int64_t lda, ldb, ldy, ldmask;   // bytes between rows of the operands as they lie in memory
    int64_t b_group;           // bytes between the groups' right operands (kForward, kInput)
    int64_t y_group;           // bytes between the groups' outputs (kWeights)
    int32_t rows, cols, red;   // of one problem (kWeights: red = all rows of the tensors, of which a group takes its own)
    int32_t groups;
    int32_t tiles_n;           // column tiles
    int32_t flags;
};
enum { kGrpRelu = 1, kGrpOutBf16 = 2, kGrpVecOut = 4, kGrpMask = 8 };

template <typename T> struct GrpTraits;
template <> struct GrpTraits<bf16_tag> { static constexpr int ES = 2; typedef floatx16_t acc_t; };
template <> struct GrpTraits<float> { static constexpr int ES = 4; typedef floatx16_t acc_t; };
typedef int intx16_t __attribute__((ext_vector_type(16)));
template <> struct GrpTraits<i8_tag> { static constexpr int ES = 1; typedef intx16_t acc_t; };

template <typename T>
__device__ __forceinline__ void grp_mma(typename GrpTraits<T>::acc_t &c, const u32x4_t &first, const u32x4_t &second)
{
    if constexpr (std::is_same<T, bf16_tag>::value) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, first), __builtin_bit_cast(bf16x8_t, second), c, 0, 0, 0);
    } else if constexpr (std::is_same<T, i8_tag>::value) {
        typedef int i32x4v_t __attribute__((ext_vector_type(4)));
        c = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4v_t, first), __builtin_bit_cast(i32x4v_t, second), c, 0, 0, 0);
    } else {
        // (each instruction takes one float of each lane half, the same of both operands: any order of the reduction will do)
        const f32x4_t f = __builtin_bit_cast(f32x4_t, first), s = __builtin_bit_cast(f32x4_t, second);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(f[j], s[j], c, 0, 0, 0);
    }
}

// ---- which tile a workgroup computes ---------------------------------------------------------------------------------------

struct GrpTile {
    int group;                 // == groups: rows of no group, which are zero
    int row0, row_end;         // first output row and the end of the group's rows
    int col_tile;
};

__device__ __forceinline__ int grp_scan(int v, int lane)        // inclusive prefix sum over the wave
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(v, d);
        v += lane >= d ? o : 0;
    }
    return v;
}

// Rows of span s: group s, and as spans `groups` and `groups + 1` the rows behind the last group and before the first.
// (Clamped: whatever the offsets hold, rows stay inside the tensors.)
__device__ __forceinline__ void grp_span(const GroupedParams &p, int s, int &beg, int &end)
{
    beg = end = 0;
    if (s < p.groups + 2) {
        const int lo = s <= p.groups ? p.offsets[s] : 0, hi = s < p.groups ? p.offsets[s + 1] : s == p.groups ? p.rows : p.offsets[0];
        beg = min(max(lo, 0), p.rows);
        end = min(max(hi, beg), p.rows);
    }
}

// Tiles are numbered group by group, inside a group in panels of kPanel row tiles, rows fastest (tiles that run together share both
// operands in their XCD's L2), and each XCD gets a block of consecutive tiles: workgroups go to the XCDs in turn.
constexpr int kPanel = 8;

template <int BM>
__device__ __forceinline__ bool grp_find(const GroupedParams &p, int lane, uint32_t wg, GrpTile &t)
{
    int total = 0, upto = 0, beg = 0, end = 0;
    const int spans = p.offsets ? p.groups + 2 : 1;
    for (int s0 = 0; s0 < spans; s0 += 64) {
        if (p.offsets) grp_span(p, s0 + lane, beg, end);
        else { beg = 0; end = lane == 0 ? p.rows : 0; }
        upto = grp_scan((end - beg + BM - 1) / BM, lane);
        total += __builtin_amdgcn_readlane(upto, 63);
    }
    const uint32_t tiles = (uint32_t)total * (uint32_t)p.tiles_n, per = (tiles + 7) / 8;
    const uint32_t logical = (wg & 7) * per + (wg >> 3);
    if ((wg >> 3) >= per || logical >= tiles) return false;
    // the span that holds it
    int before = 0;
    for (int s0 = 0; s0 < spans; s0 += 64) {
        if (spans > 64) {
            grp_span(p, s0 + lane, beg, end);
            upto = grp_scan((end - beg + BM - 1) / BM, lane);
        }
        const uint64_t past = __ballot((uint32_t)(before + upto) * (uint32_t)p.tiles_n > logical);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int mt = (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(beg, l) + BM - 1) / BM;
            const int first = before + __builtin_amdgcn_readlane(upto, l) - mt;
            const int q = (int)(logical - (uint32_t)first * (uint32_t)p.tiles_n);
            const int panel = q / (kPanel * p.tiles_n), rest = q - panel * (kPanel * p.tiles_n);
            const int pm = min(kPanel, mt - panel * kPanel);
            t.group = min(s0 + l, p.groups);
            t.col_tile = rest / pm;
            t.row_end = __builtin_amdgcn_readlane(end, l);
            t.row0 = __builtin_amdgcn_readlane(beg, l) + (panel * kPanel + rest % pm) * BM;
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// ---- operands ----------------------------------------------------------------------------------------------------------------

// One operand's tile: OUTER rows (left) or columns (right) of the output by BKB bytes of the reduction.
//   RED  reduction contiguous: LDS row = outer index, BKB bytes; 16-byte chunk c of row r at chunk position c ^ ((r / RP) % CPR), so that
//        the 16 rows a fragment read touches together lie on distinct banks
//   !RED outer index contiguous: LDS row = step of the reduction, OUTER elements; chunks of rows that a transpose read touches
//        together (four consecutive ones; fp32: four apart) swap places
template <int ES, bool RED, int OUTER, int BKB>
struct GrpOperand {
    static constexpr int EPC = 16 / ES;                     // elements per chunk
    static constexpr int BK = BKB / ES;                     // reduction steps per stage
    static constexpr int BYTES = OUTER * BKB;
    static constexpr int CPR = RED ? BKB / 16 : OUTER / EPC;   // chunks per LDS row
    static constexpr int PITCH = CPR * 16;
    static __device__ __forceinline__ int swz(int row)
    {
        if constexpr (RED) return (row / (256 / BKB)) & (CPR - 1);
        else if constexpr (ES == 4) return ((row >> 2) & 1) * 8;
        else if constexpr (OUTER >= 128) return (row & 3) * 4;
        else return ((row >> 1) & 1) * 4;
    }

    // The chunk of slot s of a stage: its LDS row, and its first element inside that row's memory.
    static __device__ __forceinline__ void slot(int s, int &row, int &elem)
    {
        row = s / CPR;
        elem = ((s % CPR) ^ swz(row)) * EPC;
    }

    // LDS offset of the fragment of MFMA tile `tile0` (its first outer index) and k chunk kc, for this lane.
    static __device__ __forceinline__ uint32_t frag(int tile0, int kc, int lane)
    {
        if constexpr (RED) {
            const int r = tile0 + (lane & 31);
            return (uint32_t)(r * PITCH + (((kc * 2 + (lane >> 5)) ^ swz(r)) * 16));
        } else if constexpr (ES == 2) {
            // lane: group l / 16 = (k half, 16 outer elements), inside it row (l % 16) / 4 and four elements
            const int grp = lane >> 4, j4 = (lane & 15) >> 2, o = tile0 + (grp & 1) * 16 + (lane & 3) * 4;
            const int k = kc * 16 + (grp >> 1) * 8 + j4;
            return (uint32_t)(k * PITCH + (((o >> 3) ^ swz(k)) * 16) + (o & 7) * 2);
        } else {
            const int k = kc * 8 + (lane >> 5) * 4, o = tile0 + (lane & 31);
            return (uint32_t)(k * PITCH + (((o >> 2) ^ swz(k)) * 16) + (o & 3) * 4);
        }
    }
    static __device__ __forceinline__ u32x4_t read(const char *lds, uint32_t at)
    {
        if constexpr (RED) {
            return *(const u32x4_t *)(lds + at);
        } else if constexpr (ES == 2) {
            typedef short s16x4_t __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
            const u32x2_t lo = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(lds + at)));
            const u32x2_t hi = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(lds + at + 4 * PITCH)));
            return (u32x4_t){lo.x, lo.y, hi.x, hi.y};
        } else {
            u32x4_t v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *(const uint32_t *)(lds + at + j * PITCH);
            return v;
        }
    }
};

// The 16-byte chunk at p, of which the first `count` elements (0 .. EPC) exist; any alignment of whole elements.
template <int ES>
__device__ __forceinline__ u32x4_t grp_load_chunk(const char *p, int count)
{
    u32x4_t v = {0, 0, 0, 0};
    if (count * ES >= 16) {
        __builtin_memcpy(&v, p, 16);
    } else if (count > 0) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16 / ES; ++i) {
            if (i >= count) break;
            uint32_t e;
            if constexpr (ES == 4) e = *(const uint32_t *)(p + i * 4);
            else if constexpr (ES == 2) e = *(const uint16_t *)(p + i * 2);
            else e = *(const uint8_t *)(p + i);
            w[i * ES / 4] |= e << (i * ES % 4 * 8);
        }
        v = (u32x4_t){w[0], w[1], w[2], w[3]};
    }
    return v;
}

// The sum of a fragment's elements.  (Whole vectors are cast, not their elements: this toolchain reads the first element four times otherwise.)
template <int ES>
__device__ __forceinline__ float grp_sum(const u32x4_t &v)
{
    if constexpr (ES == 2) {
        const f32x4_t lo = __builtin_bit_cast(f32x4_t, v << 16), hi = __builtin_bit_cast(f32x4_t, v & 0xffff0000u);
        const f32x4_t s = lo + hi;
        return (s.x + s.y) + (s.z + s.w);
    } else {
        const f32x4_t s = __builtin_bit_cast(f32x4_t, v);
        return (s.x + s.y) + (s.z + s.w);
    }
}

// ---- epilogue ----------------------------------------------------------------------------------------------------------------

// Four consecutive columns of one output row.
template <typename T>
__device__ __forceinline__ void grp_store4(const GroupedParams &p, char *y_row, const char *mask_row, int col, const float *v)
{
    float o[4] = {v[0], v[1], v[2], v[3]};
    const bool whole = (p.flags & kGrpVecOut) && col + 4 <= p.cols;
    if (p.flags & kGrpMask) {
        constexpr int ES = GrpTraits<T>::ES;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (col + q >= p.cols) break;
            float m;
            if constexpr (ES == 4) m = ((const float *)mask_row)[col + q];
            else m = __builtin_bit_cast(float, (uint32_t)((const uint16_t *)mask_row)[col + q] << 16);
            o[q] = m > 0.f ? o[q] : 0.f;
        }
    }
    if (p.flags & kGrpRelu) {
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = o[q] < 0.f ? 0.f : o[q];           // (keeps NaN)
    }
    if (p.flags & kGrpOutBf16) {
        const uint32_t lo = f32x2_to_bf16x2(o[0], o[1]), hi = f32x2_to_bf16x2(o[2], o[3]);
        uint16_t *d = (uint16_t *)y_row + col;
        if (whole) {
            *(u32x2_t *)d = (u32x2_t){lo, hi};
        } else {
            if (col < p.cols) d[0] = (uint16_t)lo;
            if (col + 1 < p.cols) d[1] = (uint16_t)(lo >> 16);
            if (col + 2 < p.cols) d[2] = (uint16_t)hi;
            if (col + 3 < p.cols) d[3] = (uint16_t)(hi >> 16);
        }
    } else {
        float *d = (float *)y_row + col;
        if (whole) {
            *(f32x4_t *)d = (f32x4_t){o[0], o[1], o[2], o[3]};
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (col + q < p.cols) d[q] = o[q];
        }
    }
}

// ---- the tile kernel ---------------------------------------------------------------------------------------------------------

template <typename T, int FORM, int BM, int BN, int WGM, int WGN, int BKB>
__global__ __launch_bounds__(64 * WGM * WGN) void grouped_kernel(const GroupedParams p)
{
    constexpr int ES = GrpTraits<T>::ES;
    constexpr int THREADS = 64 * WGM * WGN;
    constexpr int WTM = BM / WGM, WTN = BN / WGN, TM = WTM / 32, TN = WTN / 32, NKC = BKB / 32;
    using A = GrpOperand<ES, FORM != kWeights, BM, BKB>;
    using B = GrpOperand<ES, FORM == kForward, BN, BKB>;
    constexpr int BK = A::BK, STAGE = A::BYTES + B::BYTES;
    constexpr int NLA = A::BYTES / 16 / THREADS, NLB = B::BYTES / 16 / THREADS;
    static_assert(NLA * THREADS * 16 == A::BYTES && NLB * THREADS * 16 == B::BYTES, "whole chunks per thread");

    extern __shared__ uint4 smem_u4[];
    char *lds = (char *)smem_u4;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave / WGN, wn = wave % WGN;

    // ---- the tile: rows [row0, row_end) of the output, columns from col0, reduction over `red` steps from the operands' bases
    int row0, row_end, col0, red, group;
    const char *a0, *b0;
    char *y = (char *)p.y;
    if constexpr (FORM == kWeights) {
        const int per = ((p.rows + BM - 1) / BM) * p.tiles_n;
        group = (int)(blockIdx.x / (unsigned)per);
        const int q = (int)(blockIdx.x % (unsigned)per);
        row0 = q / p.tiles_n * BM;
        row_end = p.rows;
        col0 = q % p.tiles_n * BN;
        const int beg = min(max(p.offsets[group], 0), p.red), end = min(max(p.offsets[group + 1], beg), p.red);
        red = end - beg;
        a0 = (const char *)p.a + (int64_t)beg * p.lda + (int64_t)row0 * ES;
        b0 = (const char *)p.b + (int64_t)beg * p.ldb + (int64_t)col0 * ES;
        y += (int64_t)group * p.y_group;
    } else {
        GrpTile tile;
        if (!grp_find<BM>(p, lane, blockIdx.x, tile)) return;
        group = tile.group;
        row0 = tile.row0;
        row_end = tile.row_end;
        col0 = tile.col_tile * BN;
        red = group < p.groups ? p.red : 0;
        a0 = (const char *)p.a + (int64_t)row0 * p.lda;
        b0 = (const char *)p.b + (int64_t)(group < p.groups ? group : 0) * p.b_group + (FORM == kForward ? (int64_t)col0 * p.ldb : (int64_t)col0 * ES);
    }
    const int rows_left = row_end - row0, cols_left = p.cols - col0;

    // ---- operand chunks through registers
    u32x4_t ra[NLA], rb[NLB];
    auto load = [&](int step) {
#pragma unroll
        for (int i = 0; i < NLA; ++i) {
            int r, e;
            A::slot(i * THREADS + t, r, e);
            if constexpr (FORM != kWeights) {
                const int k = step * BK + e;
                ra[i] = grp_load_chunk<ES>(a0 + (int64_t)r * p.lda + (int64_t)k * ES, r < rows_left ? red - k : 0);
            } else {
                const int k = step * BK + r;
                ra[i] = grp_load_chunk<ES>(a0 + (int64_t)k * p.lda + (int64_t)e * ES, k < red ? rows_left - e : 0);
            }
        }
#pragma unroll
        for (int i = 0; i < NLB; ++i) {
            int r, e;
            B::slot(i * THREADS + t, r, e);
            if constexpr (FORM == kForward) {
                const int k = step * BK + e;
                rb[i] = grp_load_chunk<ES>(b0 + (int64_t)r * p.ldb + (int64_t)k * ES, r < cols_left ? red - k : 0);
            } else {
                const int k = step * BK + r;
                rb[i] = grp_load_chunk<ES>(b0 + (int64_t)k * p.ldb + (int64_t)e * ES, k < red ? cols_left - e : 0);
            }
        }
    };
    auto store = [&](int stage) {
        char *d = lds + stage * STAGE;
#pragma unroll
        for (int i = 0; i < NLA; ++i) *(u32x4_t *)(d + (i * THREADS + t) * 16) = ra[i];
#pragma unroll
        for (int i = 0; i < NLB; ++i) *(u32x4_t *)(d + A::BYTES + (i * THREADS + t) * 16) = rb[i];
    };

    typename GrpTraits<T>::acc_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    float sums[TM];                                        // kWeights: of this lane's row of the left operand
#pragma unroll
    for (int i = 0; i < TM; ++i) sums[i] = 0.f;
    const bool take_sums = FORM == kWeights && p.colsum && col0 == 0 && wn == 0;

    const int steps = (red + BK - 1) / BK;
    if (steps > 0) {
        load(0);
        store(0);
    }
    for (int s = 0; s < steps; ++s) {
        __syncthreads();                                   // stage s is written, stage s + 1's last readers are through
        if (s + 1 < steps) load(s + 1);
        const char *d = lds + (s & 1) * STAGE;
#pragma unroll
        for (int kc = 0; kc < NKC; ++kc) {
            u32x4_t fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = A::read(d, A::frag(wm * WTM + i * 32, kc, lane));
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = B::read(d + A::BYTES, B::frag(wn * WTN + j * 32, kc, lane));
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) grp_mma<T>(acc[i][j], fb[j], fa[i]);
            if constexpr (FORM == kWeights) {
                if (take_sums) {
#pragma unroll
                    for (int i = 0; i < TM; ++i)
                        sums[i] += grp_sum<ES>(fa[i]);
                }
            }
        }
        if (s + 1 < steps) store((s + 1) & 1);
    }

    // ---- epilogue: lane = output row, registers = columns (the right operand is the instructions' first)
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int r = wm * WTM + i * 32 + (lane & 31);
        const bool row_ok = r < rows_left;
        if constexpr (FORM == kWeights) {
            if (take_sums) {
                const float s = sums[i] + __shfl_xor(sums[i], 32);
                if (lane < 32 && row_ok) p.colsum[(int64_t)group * p.rows + row0 + r] = s;
            }
        }
        if (!row_ok) continue;
        char *y_row = y + (int64_t)(row0 + r) * p.ldy;
        const char *mask_row = (const char *)p.mask + (int64_t)(row0 + r) * p.ldmask;
        float sa = 1.f;
        if constexpr (ES == 1) sa = group < p.groups ? p.a_scale[row0 + r] : 1.f;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = col0 + wn * WTN + j * 32 + g * 8 + (lane >> 5) * 4;
                if (col >= p.cols) continue;
                float v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v[q] = (float)acc[i][j][g * 4 + q];
                    if constexpr (FORM == kForward) {
                        if (group < p.groups && col + q < p.cols) {
                            const int64_t c = (int64_t)group * p.cols + col + q;
                            if constexpr (ES == 1) v[q] = v[q] * sa * p.b_scale[c];
                            if (p.bias) v[q] += p.bias[c];
                        }
                    }
                }
                grp_store4<T>(p, y_row, mask_row, col, v);
            }
    }
}

template <typename T, int FORM, int BM, int BN, int WGM, int WGN, int BKB>
hipError_t grouped_launch(const GroupedParams &p, unsigned grid, hipStream_t st)
{
    constexpr size_t lds = (size_t)2 * (BM + BN) * BKB;
    hipLaunchKernelGGL((grouped_kernel<T, FORM, BM, BN, WGM, WGN, BKB>), dim3(grid), dim3(64 * WGM * WGN), lds, st, p);
    return hipGetLastError();
}

// One product of `form` on the kernel that suits it (grouped_bf16.hip, grouped_f32.hip, grouped_i8.hip).
hipError_t grouped_run_bf16(int form, GroupedParams p, hipStream_t st);
hipError_t grouped_run_f32(int form, GroupedParams p, hipStream_t st);
hipError_t grouped_run_i8(GroupedParams p, hipStream_t st);

// Most tiles of BM rows that any offsets in order can make of p.rows rows: each span ends in one part tile at most.
inline int64_t grp_row_tiles(const GroupedParams &p, int BM)
{
    if (!p.offsets) return ((int64_t)p.rows + BM - 1) / BM;
    const int64_t spans = (int64_t)p.groups + 2;
    return p.rows / BM + (spans < p.rows ? spans : p.rows);
}

template <typename T, int FORM, int BM, int BN, int WGM, int WGN, int BKB>
hipError_t grouped_tiles(GroupedParams p, hipStream_t st)
{
    p.tiles_n = (p.cols + BN - 1) / BN;
    int64_t grid;
    if (FORM == kWeights) grid = (int64_t)((p.rows + BM - 1) / BM) * p.tiles_n * p.groups;
    else grid = (grp_row_tiles(p, BM) * p.tiles_n + 7) / 8 * 8;            // (a block of tiles for each XCD)
    if (grid <= 0) return hipSuccess;
    if (grid * (64 * WGM * WGN) > 0xffffffffll) return hipErrorInvalidConfiguration;   // (threads of a launch)
    return grouped_launch<T, FORM, BM, BN, WGM, WGN, BKB>(p, (unsigned)grid, st);
}

}  // namespace alt
