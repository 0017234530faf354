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

#include <algorithm>
#include <cmath>

#include "dconv.h"

namespace alt {

struct i8_tag {};
struct bf16_adapted_tag {};    // bf16 and fp32 products with low-rank adapters beside them (kForward)
struct f32_adapted_tag {};
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
    int32_t places;            // compute units
    FastDiv d_panel;           // of kPanel * tiles_n
    int32_t flags;
    // low-rank adapters beside the product (the adapted types below): each row's adapter, and its inner sums (grp_adapt says how they lie)
    const int32_t *adapter;
    const char *inner;
    const char *up;            // [adapters][cols][rank]
    int32_t adapters, rank, inner_bytes;
};
enum { kGrpRelu = 1, kGrpOutBf16 = 2, kGrpMask = 4, kGrpWhole = 8, kGrpPacked = 16 };
// (kGrpWhole: the columns are whole 16-byte chunks of the output, and whole fours; kGrpPacked: operand rows are filled up with zeros to whole chunks)

template <typename T> struct GrpTraits;
// (SUMS: sums per output and wave.  fp32 keeps four, each over every fourth product, added at the end: that halves their rounding error, 5.7e-7 to 2.9e-7
// of the result in the 2-norm at reductions of 1000; the kernel for any alignment keeps two.)
template <> struct GrpTraits<bf16_tag> { static constexpr int ES = 2, SUMS = 1; static constexpr bool ADAPT = false; typedef floatx16_t acc_t; };
template <> struct GrpTraits<float> { static constexpr int ES = 4, SUMS = 4; static constexpr bool ADAPT = false; typedef floatx16_t acc_t; };
typedef int intx16_t __attribute__((ext_vector_type(16)));
template <> struct GrpTraits<i8_tag> { static constexpr int ES = 1, SUMS = 1; static constexpr bool ADAPT = false; typedef intx16_t acc_t; };
template <> struct GrpTraits<bf16_adapted_tag> : GrpTraits<bf16_tag> { static constexpr bool ADAPT = true; };
template <> struct GrpTraits<f32_adapted_tag> : GrpTraits<float> { static constexpr bool ADAPT = true; };

template <typename T, int SUMS>
__device__ __forceinline__ void grp_mma(typename GrpTraits<T>::acc_t (&c)[SUMS], const u32x4_t &first, const u32x4_t &second)
{
    if constexpr (GrpTraits<T>::ES == 2) {
        c[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, first), __builtin_bit_cast(bf16x8_t, second), c[0], 0, 0, 0);
    } else if constexpr (std::is_same<T, i8_tag>::value) {
        typedef int i32x4v_t __attribute__((ext_vector_type(4)));
        c[0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4v_t, first), __builtin_bit_cast(i32x4v_t, second), c[0], 0, 0, 0);
    } else {
        // (each instruction takes one float of each lane half, the same of both operands: any order of the reduction will do)
        const f32x4_t f = __builtin_bit_cast(f32x4_t, first), s = __builtin_bit_cast(f32x4_t, second);
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j % SUMS] = __builtin_amdgcn_mfma_f32_32x32x2f32(f[j], s[j], c[j % SUMS], 0, 0, 0);
    }
}

// A wave's sums, TM x TN matrix tiles.
template <typename T, int TM, int TN, int SUMS = GrpTraits<T>::SUMS>
struct GrpSums {
    typename GrpTraits<T>::acc_t c[TM][TN][SUMS];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int s = 0; s < SUMS; ++s)
#pragma unroll
                    for (int e = 0; e < 16; ++e) c[i][j][s][e] = 0;
    }
    __device__ __forceinline__ void join()                 // into c[i][j][0]
    {
#pragma unroll
        for (int h = SUMS / 2; h > 0; h /= 2)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int s = 0; s < h; ++s)
#pragma unroll
                        for (int e = 0; e < 16; ++e) c[i][j][s][e] += c[i][j][s + h][e];
    }
};

// ---- which tile a workgroup computes ---------------------------------------------------------------------------------------

struct GrpTile {
    int group;                 // == groups: rows of no group, which are zero
    int row0, row_end;         // first output row and the end of the group's rows
    int col_tile;
};

__device__ __forceinline__ int grp_scan(int v)                  // inclusive prefix sum over the wave
{
    // (shifts inside rows of 16 lanes, then the rows' last lanes handed on)
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true);
    return v;
}

__device__ __forceinline__ int grp_scan_max(int v)              // inclusive prefix maximum over the wave, of values from 0 on
{
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true));
    return v;
}

// Rows of the spans s0 to s0 + 63, one per lane: span s is group s, and the spans `groups` and `groups + 1` are the rows behind the last group and
// before the first.  Offsets count as their running maximum, at most p.rows: whatever they hold, the spans are disjoint and together all rows, so that
// there are never more tiles than the launch counts on, and no sum of them wraps.  `past`: that maximum over the spans before s0 (0 at first).
__device__ __forceinline__ void grp_spans(const GroupedParams &p, int s0, int lane, int &past, int &beg, int &end)
{
    const int s = s0 + lane;
    if (!p.offsets) {
        beg = 0;
        end = s == 0 ? p.rows : 0;
        return;
    }
    const int lo = s <= p.groups ? p.offsets[s] : 0, hi = s < p.groups ? p.offsets[s + 1] : s == p.groups ? p.rows : s == p.groups + 1 ? p.offsets[0] : 0;
    const int top = max(grp_scan_max(min(max(lo, 0), p.rows)), past);
    past = __builtin_amdgcn_readlane(top, 63);
    beg = s <= p.groups ? top : 0;
    end = min(max(hi, beg), p.rows);
}

// Tiles are numbered group by group, inside a group in panels of kPanel row tiles, rows fastest (tiles that run together share both
// operands in their XCD's L2), and each XCD gets a block of consecutive tiles: workgroups go to the XCDs in turn.
constexpr int kPanel = 8;

__device__ __forceinline__ void grp_order(const GroupedParams &p, int q, int tiles_m, int &row_tile, int &col_tile)
{
    const int panel = (int)fast_div((uint32_t)q, p.d_panel), rest = q - panel * (kPanel * p.tiles_n);
    const int pm = min(kPanel, tiles_m - panel * kPanel);
    col_tile = pm == kPanel ? rest / kPanel : rest / pm;
    row_tile = panel * kPanel + rest - col_tile * pm;
}

// Of many groups no workgroup looks at every offset: each has a slot that may hold a row tile, and searches the offsets for its span, 64 probes at a time.
// Spans here lie in the order of their rows (0: before the first group, s: group s - 1, groups + 1: behind the last), span s from row b(s) on.  Where
// there are few rows each row is a slot, and its tile is the one that begins there; otherwise span s has the slots from b(s) / BM + s on, which are
// never fewer than its tiles.  Offsets out of order lead a search anywhere, but to rows inside the tensors, and each workgroup to one tile at most.
// A scan takes every workgroup two turns for each 64 groups, so that a launch grows with their square, and a search leaves slots empty, each of which takes a
// compute unit's time where a tile's LDS is most of it: 128 groups of 128 rows, 1024 x 1024 bf16, 86 us with the scan and 90 with the search, 200 of 82
// 127 and 118, 512 of 32 336 and 258; one row each, 64 x 64, 4096 groups 358 and 25, 65536 107 ms and 0.54, 2^20 9.0 ms with the search.
constexpr int kScanSpans = 192;

__host__ __device__ inline bool grp_searches(const GroupedParams &p) { return p.offsets && p.groups + 2 > kScanSpans; }
__host__ __device__ inline bool grp_slot_per_row(const GroupedParams &p, int BM) { return p.rows <= p.rows / BM + p.groups + 2; }

template <int BM>
__device__ __forceinline__ bool grp_search(const GroupedParams &p, int lane, uint32_t wg, GrpTile &t)
{
    const bool per_row = grp_slot_per_row(p, BM);
    const int spans = p.groups + 2, slots = per_row ? p.rows : p.rows / BM + spans;
    const uint32_t tiles = (uint32_t)slots * (uint32_t)p.tiles_n, per = (tiles + 7) / 8;
    const uint32_t logical = (wg & 7) * per + (wg >> 3);
    if ((wg >> 3) >= per || logical >= tiles) return false;
    const int slot = (int)(logical / (uint32_t)p.tiles_n);
    auto begin = [&](int s) { return s == 0 ? 0 : s < spans ? min(max(p.offsets[s - 1], 0), p.rows) : p.rows; };
    auto first_slot = [&](int s, int b) { return per_row ? b : b / BM + s; };
    // the last span that begins at or before the slot, among the `left` ones from `span` on, of which the first does
    int span = 0, left = spans;
    while (left > 1) {
        const int step = (left + 63) / 64, at = lane * step;
        const bool before = lane == 0 || (at < left && first_slot(span + at, begin(span + at)) <= slot);
        const int pick = (63 - __builtin_clzll(__ballot(before))) * step;
        span += pick;
        left = min(step, left - pick);
    }
    const int beg = begin(span), end = max(begin(span + 1), beg), mt = (end - beg + BM - 1) / BM, in = slot - first_slot(span, beg);
    const uint32_t q = logical - (uint32_t)(slot - in) * (uint32_t)p.tiles_n;      // of the span's first slot's tiles
    int row_tile;
    if (per_row) {
        if (in % BM || in >= end - beg) return false;
        row_tile = in / BM;
        t.col_tile = (int)(logical - (uint32_t)slot * (uint32_t)p.tiles_n);
    } else {
        if (q >= (uint32_t)mt * (uint32_t)p.tiles_n) return false;
        grp_order(p, (int)q, mt, row_tile, t.col_tile);
    }
    t.group = span == 0 ? p.groups : span - 1;             // (span groups + 1: group `groups`, too)
    t.row0 = beg + row_tile * BM;
    t.row_end = end;
    return true;
}

template <int BM>
__device__ __forceinline__ bool grp_find(const GroupedParams &p, int lane, uint32_t wg, GrpTile &t)
{
    if (grp_searches(p)) return grp_search<BM>(p, lane, wg, t);
    int total = 0, upto = 0, past_rows = 0, beg = 0, end = 0;
    const int spans = p.offsets ? p.groups + 2 : 1;
    for (int s0 = 0; s0 < spans; s0 += 64) {
        grp_spans(p, s0, lane, past_rows, beg, end);
        upto = grp_scan((end - beg + BM - 1) / BM);
        total += __builtin_amdgcn_readlane(upto, 63);
    }
    const uint32_t tiles = (uint32_t)total * (uint32_t)p.tiles_n, per = (tiles + 7) / 8;
    const uint32_t logical = (wg & 7) * per + (wg >> 3);
    if ((wg >> 3) >= per || logical >= tiles) return false;
    // the span that holds it
    int before = 0;
    past_rows = 0;
    for (int s0 = 0; s0 < spans; s0 += 64) {
        if (spans > 64) {
            grp_spans(p, s0, lane, past_rows, beg, end);
            upto = grp_scan((end - beg + BM - 1) / BM);
        }
        const uint64_t past = __ballot((uint32_t)(before + upto) * (uint32_t)p.tiles_n > logical);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int mt = (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(beg, l) + BM - 1) / BM;
            const int first = before + __builtin_amdgcn_readlane(upto, l) - mt;
            int row_tile;
            grp_order(p, (int)(logical - (uint32_t)first * (uint32_t)p.tiles_n), mt, row_tile, t.col_tile);
            t.group = min(s0 + l, p.groups);
            t.row_end = __builtin_amdgcn_readlane(end, l);
            t.row0 = __builtin_amdgcn_readlane(beg, l) + row_tile * BM;
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
    static constexpr bool kRed = RED;
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
    // From this lane's address of (RED) tile 0, chunk kc or (!RED) tile i, chunk 0 to that of tile i, chunk kc.
    static __device__ __forceinline__ constexpr int apart(int i, int kc) { return RED ? i * 32 * PITCH : kc * (32 / ES) * PITCH; }
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
            uint32_t e = 0;
            if (i < count) {
                if constexpr (ES == 4) e = *(const uint32_t *)(p + i * 4);
                else if constexpr (ES == 2) e = *(const uint16_t *)(p + i * 2);
                else e = *(const uint8_t *)(p + i);
            }
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

// W consecutive floats of a row, `count` of which exist (the others are zero).  Any alignment of whole elements.
template <int W>
__device__ __forceinline__ void grp_load_f(const float *p, int count, float (&v)[W])
{
    if (count >= W) {
        __builtin_memcpy(v, p, 4 * W);
    } else {
#pragma unroll
        for (int q = 0; q < W; ++q) v[q] = q < count ? p[q] : 0.f;
    }
}

// W elements (16 bytes of output, of type T) of the tensor that says which outputs stay, as far as `count` of them exist.
template <int ES, int W> struct GrpMask { uint32_t w[ES * W / 4]; };

// All bits where the element is positive (its sign and magnitude as a number of ES bytes; NaN is not).
template <int ES>
__device__ __forceinline__ bool grp_positive(uint32_t bits)
{
    const uint32_t f = ES == 4 ? bits : bits << 16;
    return f - 1u < 0x7f800000u;
}

__device__ __forceinline__ float grp_relu(float v) { return __builtin_elementwise_maximum(v, 0.f); }      // (keeps NaN)

// W (4 or 8) consecutive columns of one output row: ReLU, rounding.
template <int W>
__device__ __forceinline__ void grp_store(const GroupedParams &p, char *y_row, int col, float (&v)[W])
{
    const int count = p.cols - col;
    if (p.flags & kGrpRelu) {
#pragma unroll
        for (int q = 0; q < W; ++q) v[q] = grp_relu(v[q]);
    }
    if (p.flags & kGrpOutBf16) {
        uint32_t w[W / 2];
#pragma unroll
        for (int q = 0; q < W / 2; ++q) w[q] = f32x2_to_bf16x2(v[2 * q], v[2 * q + 1]);
        uint16_t *d = (uint16_t *)y_row + col;
        if (count >= W) {
            __builtin_memcpy(d, w, 2 * W);
        } else {
#pragma unroll
            for (int q = 0; q < W; ++q)
                if (q < count) d[q] = (uint16_t)(w[q / 2] >> (q % 2 * 16));
        }
    } else {
        float *d = (float *)y_row + col;
        if (count >= W) {
            __builtin_memcpy(d, v, 4 * W);
        } else {
#pragma unroll
            for (int q = 0; q < W; ++q)
                if (q < count) d[q] = v[q];
        }
    }
}

// ---- what the tile kernels share ---------------------------------------------------------------------------------------------

// One workgroup's tile: rows of the output from row0 on, a tile's number of them at most and up to row_end (where the group's end), columns from
// col0 on, reduced over `red` steps from a0 and b0.
struct GrpProblem {
    int row0, row_end, col0, red, group;
    const char *a0, *b0;
    char *y;
};

// kForward, kInput: the tile at row0 and col0 of a group's rows.
template <typename T, int FORM>
__device__ __forceinline__ void grp_at(const GroupedParams &p, int group, int row0, int row_end, int col0, GrpProblem &g)
{
    const bool owned = group < p.groups;
    g.group = group;
    g.row0 = row0;
    g.row_end = row_end;
    g.col0 = col0;
    g.red = owned ? p.red : 0;
    g.a0 = (const char *)p.a + (int64_t)row0 * p.lda;
    g.b0 = (const char *)p.b + (int64_t)(owned ? group : 0) * p.b_group + (FORM == kForward ? (int64_t)col0 * p.ldb : (int64_t)col0 * GrpTraits<T>::ES);
    g.y = (char *)p.y;
}

// Workgroups of one group of a kWeights launch: blocks of tiles for each XCD, where there are tiles enough for that.
__host__ __device__ inline int grp_weight_tiles(int tiles) { return tiles >= 64 ? (tiles + 7) / 8 * 8 : tiles; }

// The group that is `place`-th by its rows, the longest first (equal ones in order), of 64 at most.  A group's rows are the reduction of its tiles of a
// kWeights launch, so that the long ones begin first and the short ones fill the chip at the end: 1001 fp32 rows of 13 groups, 515 x 1030, 27 us for 26
// to 36 by where the longest group stands, 16384 rows of 8, 2048 x 4096 bf16, 286 for 294 in the mean.  (Finding it takes 0.8 us, more than it gives
// where all workgroups run at once.)
__device__ __forceinline__ int grp_by_length(const GroupedParams &p, int lane, int place)
{
    int rows = -1, before = 0;
    if (lane < p.groups) {
        const int beg = min(max(p.offsets[lane], 0), p.red);
        rows = min(max(p.offsets[lane + 1], beg), p.red) - beg;
    }
    for (int i = 0; i < p.groups; ++i) {
        const int other = __builtin_amdgcn_readlane(rows, i);
        before += other > rows || (other == rows && i < lane);
    }
    return __builtin_ctzll(__ballot(lane < p.groups && before == place));
}

template <typename T, int FORM, int BM, int BN>
__device__ __forceinline__ bool grp_problem(const GroupedParams &p, int lane, uint32_t wg, GrpProblem &g)
{
    constexpr int ES = GrpTraits<T>::ES;
    if constexpr (FORM == kWeights) {
        const int tiles_m = (p.rows + BM - 1) / BM, tiles = tiles_m * p.tiles_n, per = grp_weight_tiles(tiles);
        g.group = (int)(wg / (unsigned)per);
        if (p.groups <= 64 && gridDim.x > 2u * (unsigned)p.places) g.group = grp_by_length(p, lane, g.group);
        int q = (int)(wg % (unsigned)per), mt, nt;
        if (tiles >= 64) q = (q & 7) * (per / 8) + (q >> 3);
        if (q >= tiles) return false;
        grp_order(p, q, tiles_m, mt, nt);
        g.row0 = mt * BM;
        g.row_end = p.rows;
        g.col0 = nt * BN;
        const int beg = min(max(p.offsets[g.group], 0), p.red), end = min(max(p.offsets[g.group + 1], beg), p.red);
        g.red = end - beg;
        g.a0 = (const char *)p.a + (int64_t)beg * p.lda + (int64_t)g.row0 * ES;
        g.b0 = (const char *)p.b + (int64_t)beg * p.ldb + (int64_t)g.col0 * ES;
        g.y = (char *)p.y + (int64_t)g.group * p.y_group;
    } else {
        GrpTile tile;
        if (!grp_find<BM>(p, lane, wg, tile)) return false;
        grp_at<T, FORM>(p, tile.group, tile.row0, tile.row_end, tile.col_tile * BN, g);
    }
    return true;
}

// Stores a wave's tile, whose first row and column inside the workgroup's are wrow and wcol.  The matrix instructions leave lane = output row,
// registers = columns (the right operand is their first); 32 rows by 128 bytes at a time go through 4 KB of LDS of the wave's own and out as whole
// lines, 16 bytes per lane.  (Stored as they lie, a 256x256 tile took 13000 instructions, most of them branches at the edges.)  What the sums are
// combined with is asked for first.  The wave's earlier memory operations are complete when the first store goes out.
constexpr int kStageBytes = 4096;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t grp_buffer(const void *base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)bytes, 0x00020000);
}

// WHOLE: every chunk of an output row, and every four columns, exist or do not (no path for parts of them).  Rows and columns that do not exist
// lie outside the buffer descriptors: what is asked for there is zero, and what is stored there is dropped, without a branch.
template <typename T, int FORM, int TM, int TN, bool BF16, bool WHOLE, int SUMS>
__device__ __forceinline__ void grp_emit(const GroupedParams &p, const GrpProblem &g, const GrpSums<T, TM, TN, SUMS> &acc, char *stage, int wrow, int wcol, int lane)
{
    constexpr int ES = GrpTraits<T>::ES, OS = BF16 ? 2 : 4;
    constexpr int JB = BF16 && TN > 1 ? 2 : 1, CPB = BF16 ? 4 * JB : 8;      // column tiles and 16-byte chunks of a band's rows
    constexpr int W = 16 / OS, RPP = 64 / CPB, PASSES = 32 / RPP;             // columns of a chunk; rows per pass, passes per band
    constexpr int BANDS = TM * (TN / JB);
    const bool owned = g.group < p.groups, masked = FORM == kInput && (p.flags & kGrpMask), relu = FORM == kForward && (p.flags & kGrpRelu);
    const int col_in = g.col0 + wcol + (lane >> 5) * 4, col_out = g.col0 + wcol + lane % CPB * W;  // of the sums and of the chunks
    // From the tile's first row on; the last row is the last that is this wave's, so that a descriptor's size stays below kOutOfRange (rows are 16 MB
    // apart at most, 4 MB in tiles of more than 128).
    const int row_out = wrow + lane / CPB, last = min(g.row_end - g.row0, wrow + TM * 32) - 1;
    float sa[TM];
    f32x4_t scale[TN][4], bias[TN][4];
    auto columns = [&](f32x4_t (&v)[TN][4], const float *row, bool exist) {
        const __amdgpu_buffer_rsrc_t r = grp_buffer(row, exist ? (uint32_t)p.cols * 4u : 0u);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int at = (col_in + j * 32 + q4 * 8) * 4;
                if constexpr (WHOLE) {
                    v[j][q4] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[j][q4][q] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, at + q * 4, 0, 0));
                }
            }
    };
    if constexpr (FORM == kForward) {
        const int64_t at = (int64_t)(owned ? g.group : 0) * p.cols;
        if constexpr (ES == 1) {
            // (rows of no group: scales of zero columns, so that their zeros stay zeros)
#pragma unroll
            for (int i = 0; i < TM; ++i) sa[i] = owned ? p.a_scale[g.row0 + min(wrow + (lane & 31) + i * 32, last)] : 0.f;
            columns(scale, p.b_scale + at, owned);
        }
        columns(bias, p.bias ? p.bias + at : nullptr, p.bias && owned);
    }
    // A lane's chunk of row r lies at `at` + r * ld, outside everything where its columns do not exist.
    const __amdgpu_buffer_rsrc_t y_rsrc = grp_buffer(g.y + (int64_t)g.row0 * p.ldy, (uint32_t)last * (uint32_t)p.ldy + (uint32_t)(p.cols * OS));
    const __amdgpu_buffer_rsrc_t m_rsrc = grp_buffer((const char *)p.mask + (int64_t)g.row0 * p.ldmask, masked ? (uint32_t)last * (uint32_t)p.ldmask + (uint32_t)(p.cols * ES) : 0u);
    // (of two bands: the one that is stored and the one behind it)
    GrpMask<ES, W> mask[2][PASSES];
    auto load_mask = [&](int band) {
#pragma unroll
        for (int q = 0; q < PASSES; ++q) {
            const int col = col_out + band % (TN / JB) * JB * 32, at = (row_out + band / (TN / JB) * 32 + q * RPP) * (int)p.ldmask + col * ES;
            GrpMask<ES, W> &m = mask[band & 1][q];
            if constexpr (WHOLE && ES * W == 16) {
                const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(m_rsrc, col < p.cols ? at : (int)kOutOfRange, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) m.w[e % (ES * W / 4)] = v[e];
            } else if constexpr (WHOLE && ES * W == 8) {
                const u32x2_t v = __builtin_amdgcn_raw_buffer_load_b64(m_rsrc, col < p.cols ? at : (int)kOutOfRange, 0, 0);
                m.w[0] = v.x;
                m.w[1] = v.y;
            } else {
#pragma unroll
                for (int e = 0; e < ES * W / 4; ++e) m.w[e] = 0;
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const int o = col + e < p.cols ? at + e * ES : (int)kOutOfRange;
                    if constexpr (ES == 4) m.w[e % (ES * W / 4)] = __builtin_amdgcn_raw_buffer_load_b32(m_rsrc, o, 0, 0);
                    else if constexpr (ES == 2) m.w[e / 2] |= (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(m_rsrc, o, 0, 0) << (e % 2 * 16);
                }
            }
        }
    };
    if constexpr (FORM == kInput) {
        if (masked) load_mask(0);
    }
    wait_vmcnt<0>();
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; j += JB) {
            const int r_in = lane & 31, band = i * (TN / JB) + j / JB;
            if constexpr (FORM == kInput) {
                if (masked && band + 1 < BANDS) load_mask(band + 1);
            }
#pragma unroll
            for (int jj = 0; jj < JB; ++jj)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    f32x4_t f;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        f[q] = (float)acc.c[i][j + jj][0][q4 * 4 + q];
                        if constexpr (ES == 1) f[q] = __builtin_fmaf(f[q] * sa[i], scale[j + jj][q4][q], bias[j + jj][q4][q]);
                        else if constexpr (FORM == kForward) f[q] += bias[j + jj][q4][q];
                    }
                    if (relu) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) f[q] = grp_relu(f[q]);
                    }
                    if constexpr (BF16) {
                        const u32x2_t w = {f32x2_to_bf16x2(f.x, f.y), f32x2_to_bf16x2(f.z, f.w)};
                        *(u32x2_t *)(stage + r_in * (CPB * 16) + (((jj * 4 + q4) ^ (r_in & (CPB - 1))) * 16) + (lane >> 5) * 8) = w;
                    } else {
                        *(f32x4_t *)(stage + r_in * (CPB * 16) + (((q4 * 2 + (lane >> 5)) ^ (r_in & (CPB - 1))) * 16)) = f;
                    }
                }
            const int col = col_out + j * 32;
#pragma unroll
            for (int q = 0; q < PASSES; ++q) {
                const int r = lane / CPB + q * RPP;
                u32x4_t w = *(const u32x4_t *)(stage + r * (CPB * 16) + (((lane % CPB) ^ (r & (CPB - 1))) * 16));
                if constexpr (FORM == kInput) {
                    if (masked) {
                        const GrpMask<ES, W> &m = mask[band & 1][q];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if constexpr (!BF16) w[e] = grp_positive<ES>(ES == 4 ? m.w[e % (ES * W / 4)] : m.w[e / 2 % (ES * W / 4)] >> (e % 2 * 16)) ? w[e] : 0u;
                            else w[e] &= (grp_positive<2>(m.w[e] & 0xffffu) ? 0xffffu : 0u) | (grp_positive<2>(m.w[e] >> 16) ? 0xffff0000u : 0u);
                        }
                    }
                }
                const int at = (row_out + i * 32 + q * RPP) * (int)p.ldy + col * OS;
                if constexpr (WHOLE) {
                    __builtin_amdgcn_raw_buffer_store_b128(w, y_rsrc, col < p.cols ? at : (int)kOutOfRange, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        const int o = col + e < p.cols ? at + e * OS : (int)kOutOfRange;
                        if constexpr (BF16) __builtin_amdgcn_raw_buffer_store_b16((short)(w[e / 2] >> (e % 2 * 16)), y_rsrc, o, 0, 0);
                        else __builtin_amdgcn_raw_buffer_store_b32(w[e], y_rsrc, o, 0, 0);
                    }
                }
            }
        }
    }
}

// bf16 numbers, infinities and NaN among them zeros.
__device__ __forceinline__ u32x4_t grp_finite(const u32x4_t &v)
{
    typedef int16_t i16x2_t __attribute__((ext_vector_type(2)));
    u32x4_t out;
#pragma unroll
    for (int q = 0; q < 4; ++q) {                          // (an exponent of ones becomes its half's top bit)
        const i16x2_t all = __builtin_bit_cast(i16x2_t, (v[q] & 0x7f807f80u) + 0x00800080u) >> (int16_t)15;
        out[q] = v[q] & ~__builtin_bit_cast(uint32_t, all);
    }
    return out;
}

// The adapters' part of a wave's tile: c[row][col] += sum_r inner[row][r] * up[g][col][r] for the adapter g of the row, one adapter that its rows have
// after another, in registers: a product like the tile's own with `rank` more steps.  A row's inner sums lie one behind another, filled up to whole
// matrix instructions with zeros (inner_bytes), in bf16 as two such rows, the value rounded and what that left, so that the adapters' part is as exact as the
// tile's own.  Lanes hold rows: another adapter's rows take nothing of the sums, whatever they are.  What of `up` is not finite meets the first part alone, which
// makes of it what the whole sum would: beside it the second, zero or of another sign, would make NaN of infinities.
template <typename T, int TM, int TN, int SUMS>
__device__ __forceinline__ void grp_adapt(const GroupedParams &p, const GrpProblem &g, GrpSums<T, TM, TN, SUMS> &acc, int wrow, int wcol, int lane)
{
    constexpr int ES = GrpTraits<T>::ES, PARTS = ES == 2 ? 2 : 1, STEPS = 2;           // of which the loads go out together
    const int half = (lane >> 5) * 16;
    if (g.col0 + wcol >= p.cols) return;
    int ids[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = g.row0 + wrow + i * 32 + (lane & 31), id = p.adapter[min(row, g.row_end - 1)];
        ids[i] = row < g.row_end && id < p.adapters ? id : -1;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const char *inner = p.inner + (int64_t)min(g.row0 + wrow + i * 32 + (lane & 31), g.row_end - 1) * (PARTS * p.inner_bytes) + half;
        uint64_t left = __ballot(ids[i] >= 0);
        while (left) {
            const int one = __builtin_amdgcn_readlane(ids[i], __builtin_ctzll(left));
            const bool mine = ids[i] == one;
            left &= ~__ballot(mine);
            const char *up = p.up + ((int64_t)one * p.cols + g.col0 + wcol) * p.rank * ES + half;
            typename GrpTraits<T>::acc_t part[TN][1];
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) part[j][0][e] = 0;
            for (int at = 0; at < p.inner_bytes; at += 32 * STEPS) {
                u32x4_t fa[STEPS][PARTS], fb[STEPS][TN];
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const int from = at + s * 32;
                    const bool in = from < p.inner_bytes;
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) {
                        fa[s][q] = (u32x4_t){0, 0, 0, 0};
                        if (in) fa[s][q] = *(const u32x4_t *)(inner + q * p.inner_bytes + from);
                    }
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const int64_t col = min(j * 32 + (lane & 31), p.cols - 1 - g.col0 - wcol);
                        fb[s][j] = grp_load_chunk<ES>(up + col * p.rank * ES + from, p.rank - (from + half) / ES);
                    }
                }
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        grp_mma<T>(part[j], fb[s][j], fa[s][0]);
                        if constexpr (PARTS == 2) grp_mma<T>(part[j], grp_finite(fb[s][j]), fa[s][1]);
                    }
            }
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc.c[i][j][0][e] += mine ? part[j][0][e] : 0.f;
        }
    }
}

template <typename T, int FORM, int TM, int TN, int SUMS>
__device__ __forceinline__ void grp_epilogue(const GroupedParams &p, const GrpProblem &g, GrpSums<T, TM, TN, SUMS> &acc, char *stage, int wrow, int wcol,
                                             int lane)
{
    if constexpr (GrpTraits<T>::ADAPT) grp_adapt(p, g, acc, wrow, wcol, lane);
    const bool bf16 = GrpTraits<T>::ES < 4 && (p.flags & kGrpOutBf16);
    if ((p.flags & kGrpWhole) || g.col0 + wcol + TN * 32 <= p.cols) {
        if (bf16) grp_emit<T, FORM, TM, TN, (GrpTraits<T>::ES < 4), true>(p, g, acc, stage, wrow, wcol, lane);
        else grp_emit<T, FORM, TM, TN, false, true>(p, g, acc, stage, wrow, wcol, lane);
    } else {
        if (bf16) grp_emit<T, FORM, TM, TN, (GrpTraits<T>::ES < 4), false>(p, g, acc, stage, wrow, wcol, lane);
        else grp_emit<T, FORM, TM, TN, false, false>(p, g, acc, stage, wrow, wcol, lane);
    }
}

// kWeights: the sums of the left operand's rows, which lane and lane + 32 hold halves of.
template <int TM>
__device__ __forceinline__ void grp_store_sums(const GroupedParams &p, const GrpProblem &g, const float (&sums)[TM], int wrow, int lane)
{
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = g.row0 + wrow + i * 32 + (lane & 31);
        const float s = sums[i] + __shfl_xor(sums[i], 32);
        if (lane < 32 && row < g.row_end) p.colsum[(int64_t)g.group * p.rows + row] = s;
    }
}

// ---- the kernel for few rows per group: the weights stream through registers, once ---------------------------------------------
//
// Bound by the weights' bytes.  A tile is 16 rows by 16 * NT columns; the NW waves of a workgroup share its reduction, wave w taking units
// of 128 bytes w, w + NW, ... of every row, so that each line is read whole by one wave and the workgroup walks along the rows.  Fragments of the
// 16-row matrix instructions are 16 bytes of a row per lane; a lane takes both halves of 32 bytes (row lane % 16, quarter lane / 16 of the unit: both
// operands in the same order, so any order will do), straight from memory at any alignment; two batches of loads are in flight per wave.  The waves' sums meet in LDS and are added in the waves' order.
template <typename T> struct GrpFew;
template <> struct GrpFew<bf16_tag> { typedef f32x4_t acc_t; };
template <> struct GrpFew<float> { typedef f32x4_t acc_t; };
typedef int i32x4s_t __attribute__((ext_vector_type(4)));
template <> struct GrpFew<i8_tag> { typedef i32x4s_t acc_t; };

template <typename T>
__device__ __forceinline__ void grp_mma16(typename GrpFew<T>::acc_t (&c)[GrpTraits<T>::SUMS], const u32x4_t &first, const u32x4_t &second)
{
    if constexpr (GrpTraits<T>::ES == 2) {
        c[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, first), __builtin_bit_cast(bf16x8_t, second), c[0], 0, 0, 0);
    } else if constexpr (std::is_same<T, i8_tag>::value) {
        c[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4s_t, first), __builtin_bit_cast(i32x4s_t, second), c[0], 0, 0, 0);
    } else {
        const f32x4_t f = __builtin_bit_cast(f32x4_t, first), s = __builtin_bit_cast(f32x4_t, second);
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[j], s[j], c[j], 0, 0, 0);
    }
}

// 32 bytes at p, or the aligned dwords that hold them.  Memory takes more than twice as long over addresses inside a dword (16 x 6005 x 8192 in 8 bits
// 27.4 us, 14.3 at whole dwords), so where there are such (!DW) they are the eight dwords they start in and, if they start inside one, the dword they
// end in, shifted together.
template <bool DW>
struct GrpPair {
    u32x4_t lo, hi;
    uint32_t more;
    __device__ __forceinline__ void load(const char *p)
    {
        const char *first = DW ? p : (const char *)((uintptr_t)p & ~(uintptr_t)3);
        __builtin_memcpy(&lo, __builtin_assume_aligned(first, 4), 16);
        __builtin_memcpy(&hi, __builtin_assume_aligned(first + 16, 4), 16);
        if constexpr (!DW) more = *(const uint32_t *)(first + ((uintptr_t)p & 3 ? 32 : 28));
    }
    __device__ __forceinline__ u32x4_t chunk(int h, uint32_t address) const
    {
        const u32x4_t &v = h ? hi : lo;
        if constexpr (DW) {
            return v;
        } else {
            const uint32_t next = h ? more : hi.x;
            return (u32x4_t){__builtin_amdgcn_alignbyte(v.y, v.x, address), __builtin_amdgcn_alignbyte(v.z, v.y, address),
                             __builtin_amdgcn_alignbyte(v.w, v.z, address), __builtin_amdgcn_alignbyte(next, v.w, address)};
        }
    }
};

// This wave's sums of the tile `g`.
template <typename T, int NT, int NW, int BATCH, bool DW>
__device__ __forceinline__ void grp_few_sums(const GroupedParams &p, const GrpProblem &g, int lane, int wave, typename GrpFew<T>::acc_t (&acc)[NT][GrpTraits<T>::SUMS])
{
    constexpr int ES = GrpTraits<T>::ES, UNIT = 128;
    const int rows_left = g.row_end - g.row0, cols_left = p.cols - g.col0;

    // (rows and columns outside the tile's repeat its last one: their sums are never stored)
    const int at = lane / 16 * 32;
    const char *ap = g.a0 + (int64_t)min(lane % 16, rows_left - 1) * p.lda + at, *bp[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) bp[j] = g.b0 + (int64_t)min(j * 16 + lane % 16, cols_left - 1) * p.ldb + at;

    constexpr int SUMS = GrpTraits<T>::SUMS;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int s = 0; s < SUMS; ++s) acc[j][s] = (typename GrpFew<T>::acc_t){0, 0, 0, 0};

    struct Batch { GrpPair<DW> a[BATCH], b[BATCH][NT]; };
    const int bytes = g.red * ES, units = bytes / UNIT;    // whole units
    auto load = [&](Batch &f, int u) {                     // units u, u + NW, ... (past the last one the first again, which mma leaves out)
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            const int64_t off = (int64_t)(u + q * NW < units ? u + q * NW : 0) * UNIT;
#pragma unroll
            for (int j = 0; j < NT; ++j) f.b[q][j].load(bp[j] + off);
            f.a[q].load(ap + off);
        }
    };
    auto mma = [&](const Batch &f, int u) {
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            if (u + q * NW >= units) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4_t a = f.a[q].chunk(h, (uint32_t)(uintptr_t)ap);
#pragma unroll
                for (int j = 0; j < NT; ++j) grp_mma16<T>(acc[j], f.b[q][j].chunk(h, (uint32_t)(uintptr_t)bp[j]), a);
            }
        }
    };
    constexpr int STEP = NW * BATCH;
    if (wave < units) {
        Batch x, y;
        load(x, wave);
        for (int u = wave; u < units; u += 2 * STEP) {
            if (u + STEP < units) load(y, u + STEP);
            mma(x, u);
            if (u + 2 * STEP < units) load(x, u + 2 * STEP);
            if (u + STEP < units) mma(y, u + STEP);
        }
    }
    // what the reduction ends with: less than a unit
    if (bytes % UNIT && wave == units % NW) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = units * UNIT + h * 16, count = (bytes - k - at) / ES;
            const u32x4_t a = grp_load_chunk<ES>(ap + k, count);
#pragma unroll
            for (int j = 0; j < NT; ++j) grp_mma16<T>(acc[j], grp_load_chunk<ES>(bp[j] + k, count), a);
        }
    }
}

// The waves' sums added in the waves' order: f(tile, lane of it, sum) for each four columns (lane / 16 of the tile's) of a row (lane % 16).
template <typename T, int NT, int NW, typename F>
__device__ __forceinline__ void grp_few_join(u32x4_t (&part)[NW * NT * 64], typename GrpFew<T>::acc_t (&acc)[NT][GrpTraits<T>::SUMS], int lane, int wave, F f)
{
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        if constexpr (GrpTraits<T>::SUMS == 4) acc[j][0] = (acc[j][0] + acc[j][1]) + (acc[j][2] + acc[j][3]);
        part[(wave * NT + j) * 64 + lane] = __builtin_bit_cast(u32x4_t, acc[j][0]);
    }
    __syncthreads();
    for (int s = threadIdx.x; s < NT * 64; s += NW * 64) {
        typename GrpFew<T>::acc_t sum = __builtin_bit_cast(typename GrpFew<T>::acc_t, part[s]);
#pragma unroll
        for (int w = 1; w < NW; ++w) sum += __builtin_bit_cast(typename GrpFew<T>::acc_t, part[w * NT * 64 + s]);
        f(s / 64, s % 64, sum);
    }
}

// Workgroup `wg` of a launch; `part` is LDS.
template <typename T, int NT, int NW, int BATCH, bool DW>
__device__ __forceinline__ void grp_few(const GroupedParams &p, uint32_t wg, u32x4_t (&part)[NW * NT * 64])
{
    constexpr int ES = GrpTraits<T>::ES;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    GrpProblem g;
    if (!grp_problem<T, kForward, 16, 16 * NT>(p, lane, wg, g)) return;
    typename GrpFew<T>::acc_t acc[NT][GrpTraits<T>::SUMS];
    grp_few_sums<T, NT, NW, BATCH, DW>(p, g, lane, wave, acc);
    const bool owned = g.group < p.groups;
    grp_few_join<T, NT, NW>(part, acc, lane, wave, [&](int tile, int l, const typename GrpFew<T>::acc_t &sum) {
        const int row = g.row0 + l % 16, col = g.col0 + tile * 16 + l / 16 * 4;
        if (row >= g.row_end || col >= p.cols) return;
        float v[4], scale[4] = {1.f, 1.f, 1.f, 1.f}, bias[4] = {0.f, 0.f, 0.f, 0.f}, sa = 1.f;
        if (owned) {
            const int64_t c = (int64_t)g.group * p.cols + col;
            if constexpr (ES == 1) {
                sa = p.a_scale[row];
                grp_load_f<4>(p.b_scale + c, p.cols - col, scale);
            }
            if (p.bias) grp_load_f<4>(p.bias + c, p.cols - col, bias);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = (float)sum[q];
            if constexpr (ES == 1) v[q] = __builtin_fmaf(v[q] * sa, scale[q], bias[q]);
            else v[q] += bias[q];
        }
        grp_store<4>(p, g.y + (int64_t)row * p.ldy, col, v);
    });
}

template <typename T, int NT, int NW, int BATCH, bool DW>
__global__ __launch_bounds__(64 * NW) void grouped_few_kernel(const GroupedParams p)
{
    __shared__ u32x4_t part[NW * NT * 64];
    grp_few<T, NT, NW, BATCH, DW>(p, blockIdx.x, part);
}

// The same for the gradient by the rows, whose right operand has its columns contiguous: tiles of 16 rows by 64 columns.  A lane takes four consecutive
// columns (those of its lane % 16) of as many steps of the reduction as the matrix instruction takes of a lane (those of its lane / 16), so that each
// row of 64 columns is read whole; matrix tile j has the columns 4 c + j.  Units of 64 bytes of the left operand.  Bound by latency: 19 rows, 2538 x
// 128, fp32 17.7 us (two such units in flight: 22.2; sixteen waves: 20.4), 64 rows, 1024 x 4096, 10.9.
template <typename T, int NW>
__global__ __launch_bounds__(64 * NW) void grouped_few_dx_kernel(const GroupedParams p)
{
    constexpr int ES = GrpTraits<T>::ES, EPC = 16 / ES, UNIT = 4 * EPC, SUMS = GrpTraits<T>::SUMS;
    typedef uint32_t cols4_t __attribute__((ext_vector_type(ES)));             // four columns: 16 bytes, or 8
    __shared__ u32x4_t part[NW * 4 * 64];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    GrpProblem g;
    if (!grp_problem<T, kInput, 16, 64>(p, lane, blockIdx.x, g)) return;
    if (g.col0 + 64 > p.cols && p.cols >= 64) {            // (the last tile ends with the matrix)
        g.b0 -= (int64_t)(g.col0 + 64 - p.cols) * ES;
        g.col0 = p.cols - 64;
    }
    const bool narrow = p.cols < 64;
    const int step = lane / 16 * EPC, col = lane % 16 * 4; // this lane's first step of a unit and first column of the tile
    const char *ap = g.a0 + (int64_t)min(lane % 16, g.row_end - g.row0 - 1) * p.lda + step * ES;
    const char *bp = g.b0 + (int64_t)step * p.ldb + col * ES;

    typename GrpFew<T>::acc_t acc[4][SUMS];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < SUMS; ++q) acc[j][q] = (typename GrpFew<T>::acc_t){0, 0, 0, 0};

    auto mma = [&](const u32x4_t &a, const cols4_t (&b)[EPC]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4_t f;
            if constexpr (ES == 4) {
                f = (u32x4_t){b[0][j], b[1][j], b[2][j], b[3][j]};
            } else {
#pragma unroll
                for (int d = 0; d < 4; ++d) f[d] = __builtin_amdgcn_perm(b[2 * d + 1][j / 2], b[2 * d][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
            }
            grp_mma16<T>(acc[j], f, a);
        }
    };
    const int units = narrow ? 0 : g.red / UNIT;           // whole ones
    auto load = [&](u32x4_t &a, cols4_t (&b)[EPC], int u) {
        const int64_t n = (int64_t)u * UNIT;
#pragma unroll
        for (int i = 0; i < EPC; ++i) __builtin_memcpy(&b[i], bp + (n + i) * p.ldb, 4 * ES);
        __builtin_memcpy(&a, ap + n * ES, 16);
    };
    if (wave < units) {
        u32x4_t a[2];
        cols4_t b[2][EPC];
        load(a[0], b[0], wave);
        for (int u = wave; u < units; u += 2 * NW) {
            if (u + NW < units) load(a[1], b[1], u + NW);
            mma(a[0], b[0]);
            if (u + 2 * NW < units) load(a[0], b[0], u + 2 * NW);
            if (u + NW < units) mma(a[1], b[1]);
        }
    }
    // what is left: the reduction's end, or all of it for fewer than 64 columns
    for (int n = (units + (wave + NW - units % NW) % NW) * UNIT; n < g.red; n += NW * UNIT) {
        cols4_t b[EPC];
#pragma unroll
        for (int i = 0; i < EPC; ++i) {
            const u32x4_t v = grp_load_chunk<ES>(bp + (int64_t)(n + i) * p.ldb, n + step + i < g.red ? min(p.cols - g.col0 - col, 4) : 0);
            if constexpr (ES == 4) b[i] = v;
            else b[i] = (cols4_t){v.x, v.y};
        }
        mma(grp_load_chunk<ES>(ap + (int64_t)n * ES, g.red - n - step), b);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (SUMS == 4) acc[j][0] = (acc[j][0] + acc[j][1]) + (acc[j][2] + acc[j][3]);
        part[(wave * 4 + j) * 64 + lane] = __builtin_bit_cast(u32x4_t, acc[j][0]);
    }
    __syncthreads();
    // each thread: four columns of a row, which lie in the four tiles' sums of one lane
    const float *sums = (const float *)part;
    for (int i = t; i < 256; i += NW * 64) {
        const int r = i / 16, c = i % 16, row = g.row0 + r, first = g.col0 + c * 4;
        if (row >= g.row_end || first >= p.cols) continue;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) v[j] += sums[((w * 4 + j) * 64 + c / 4 * 16 + r) * 4 + c % 4];
        }
        if (p.flags & kGrpMask) {
            const char *m = (const char *)p.mask + (int64_t)row * p.ldmask + (int64_t)first * ES;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (first + j >= p.cols) break;
                const uint32_t e = ES == 4 ? *(const uint32_t *)(m + j * 4) : *(const uint16_t *)(m + j * 2);
                if (!grp_positive<ES>(e)) v[j] = 0.f;
            }
        }
        grp_store<4>(p, g.y + (int64_t)row * p.ldy, first, v);
    }
}

// ---- the kernel for any size, stride and alignment: operands go through registers --------------------------------------------
//
// Chunks of 16 bytes are loaded at whatever address they start at.  Rows and columns that do not exist repeat the tile's last ones (their sums are
// never stored), or, where the outer index is contiguous, the last tile is moved back to end with the matrix (what two tiles both compute they
// compute alike); so only the reduction's last step has chunks of which a part exists.  Loads are two steps ahead: those of step s + 2 go out
// before step s is computed, and reach LDS behind it a step later (four steps ahead: 12.4 us for 11.7 at 333 x 1001 x 2049 in 8 bits).  WGK = 2: twice
// the waves, halves of every step's chunks to each half of them, whose sums meet in LDS.  Bound in 8 and 16 bits by the issue of loads, LDS
// writes and reads (5000 rows of 5 groups, 2047 x 4095, bf16 132 to 147 us, 0.6 PFLOP/s), in fp32 by the matrix instructions (690 us, 122 TFLOP/s).
template <int ES, bool RED, int OUTER, int BKB, int THREADS>
struct GrpLoader {
    using Op = GrpOperand<ES, RED, OUTER, BKB>;
    static constexpr int NL = Op::BYTES / 16 / THREADS;
    static_assert(NL * THREADS * 16 == Op::BYTES, "whole chunks per thread");
    uint32_t voff[NL];
    int row[NL], elem[NL];
    const char *base;                      // of the step that is loaded next
    int64_t ld;
    int left, outer_left;                  // steps of the reduction from base on; outer indices from the tile's first on

    __device__ __forceinline__ void start(const char *p0, int64_t ld_, int outer, int red, int t)
    {
        base = p0;
        ld = ld_;
        left = red;
        outer_left = outer;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            Op::slot(i * THREADS + t, row[i], elem[i]);
            voff[i] = (uint32_t)(RED ? min(row[i], outer - 1) : row[i]) * (uint32_t)ld + (uint32_t)(elem[i] * ES);
        }
    }
    // Steps from `base` on that are whole.
    __device__ __forceinline__ int whole() const { return RED || outer_left >= OUTER ? max(left, 0) / Op::BK : 0; }
    __device__ __forceinline__ void next()
    {
        base += RED ? (int64_t)BKB : ld * Op::BK;
        left -= Op::BK;
    }
    __device__ __forceinline__ void load_whole(u32x4_t (&v)[NL])
    {
#pragma unroll
        for (int i = 0; i < NL; ++i) __builtin_memcpy(&v[i], base + voff[i], 16);
        next();
    }
    __device__ __forceinline__ void load(u32x4_t (&v)[NL])
    {
        if (left >= Op::BK && (RED || outer_left >= OUTER)) {
#pragma unroll
            for (int i = 0; i < NL; ++i) __builtin_memcpy(&v[i], base + voff[i], 16);
        } else if (left <= 0) {
#pragma unroll
            for (int i = 0; i < NL; ++i) v[i] = (u32x4_t){0, 0, 0, 0};
        } else if (!RED && outer_left >= OUTER) {
            // (rows behind the last: the last one's, cleared)
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                __builtin_memcpy(&v[i], base + (row[i] < left ? voff[i] : (uint32_t)(left - 1) * (uint32_t)ld + (uint32_t)(elem[i] * ES)), 16);
                if (row[i] >= left) v[i] = (u32x4_t){0, 0, 0, 0};
            }
        } else if (RED && left >= Op::EPC) {
            // (a chunk that ends behind the row is loaded to end with it, and shifted)
#pragma unroll
            for (int i = 0; i < NL; ++i) __builtin_memcpy(&v[i], base + voff[i] - (uint32_t)(max(elem[i] + Op::EPC - left, 0) * ES), 16);
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const int over = max(elem[i] + Op::EPC - left, 0);             // elements behind the end
                unsigned __int128 w = __builtin_bit_cast(unsigned __int128, v[i]);
                w = over >= Op::EPC ? 0 : w >> (over * ES * 8);
                v[i] = __builtin_bit_cast(u32x4_t, w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NL; ++i)
                v[i] = grp_load_chunk<ES>(base + voff[i], RED ? left - elem[i] : row[i] < left ? outer_left - elem[i] : 0);
        }
        next();
    }
};

// Registers 4 q to 4 q + 3 of a matrix tile's sums.
template <typename ACC>
__device__ __forceinline__ u32x4_t grp_quarter(const ACC &c, int q)
{
    const auto v = __builtin_shufflevector(c, c, 0, 1, 2, 3), w = __builtin_shufflevector(c, c, 4, 5, 6, 7), x = __builtin_shufflevector(c, c, 8, 9, 10, 11),
               y = __builtin_shufflevector(c, c, 12, 13, 14, 15);
    return __builtin_bit_cast(u32x4_t, q == 0 ? v : q == 1 ? w : q == 2 ? x : y);
}
template <typename ACC>
__device__ __forceinline__ void grp_add_quarter(ACC &c, int q, const u32x4_t &v)
{
    const auto w = __builtin_bit_cast(decltype(__builtin_shufflevector(c, c, 0, 1, 2, 3)), v);
#pragma unroll
    for (int e = 0; e < 4; ++e) c[q * 4 + e] += w[e];
}

template <typename T, int FORM, int BM, int BN, int WGM, int WGN, int WGK>
__global__ __launch_bounds__(64 * WGM * WGN * WGK) void grouped_any_kernel(const GroupedParams p)
{
    constexpr int ES = GrpTraits<T>::ES, BKB = 128, THREADS = 64 * WGM * WGN * WGK;
    constexpr int WTM = BM / WGM, WTN = BN / WGN, TM = WTM / 32, TN = WTN / 32, NKC = BKB / 32, TILES = WGM * WGN;
    using LA = GrpLoader<ES, FORM != kWeights, BM, BKB, THREADS>;
    using LB = GrpLoader<ES, FORM == kForward, BN, BKB, THREADS>;
    using A = typename LA::Op;
    using B = typename LB::Op;
    constexpr int STAGE = A::BYTES + B::BYTES;
    static_assert(TILES * kStageBytes <= 2 * STAGE && (WGK == 1 || (WGK == 2 && TM * TN == 1 && FORM != kWeights && TILES * 4096 <= 2 * STAGE)), "staging");

    extern __shared__ uint4 smem_u4[];
    char *lds = (char *)smem_u4;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wk = wave / TILES, tile = wave % TILES, wm = tile / WGN, wn = tile % WGN;
    GrpProblem g;
    if (!grp_problem<T, FORM, BM, BN>(p, lane, blockIdx.x, g)) return;
    if (FORM != kForward && g.col0 + BN > p.cols && p.cols >= BN) {
        g.b0 -= (int64_t)(g.col0 + BN - p.cols) * ES;
        g.col0 = p.cols - BN;
    }
    if (FORM == kWeights && g.row0 + BM > p.rows && p.rows >= BM) {
        g.a0 -= (int64_t)(g.row0 + BM - p.rows) * ES;
        g.row0 = p.rows - BM;
    }

    LA la;
    LB lb;
    la.start(g.a0, p.lda, g.row_end - g.row0, g.red, t);
    lb.start(g.b0, p.ldb, p.cols - g.col0, g.red, t);
    constexpr int PF = 2;
    u32x4_t ra[PF][LA::NL], rb[PF][LB::NL];
    auto store = [&](int stage, const u32x4_t (&va)[LA::NL], const u32x4_t (&vb)[LB::NL]) {
        char *d = lds + stage * STAGE;
#pragma unroll
        for (int i = 0; i < LA::NL; ++i) *(u32x4_t *)(d + (i * THREADS + t) * 16) = va[i];
#pragma unroll
        for (int i = 0; i < LB::NL; ++i) *(u32x4_t *)(d + A::BYTES + (i * THREADS + t) * 16) = vb[i];
    };

    // (two sums for fp32: four take the registers of a third wave, and 1001 rows of 13 groups, 515 x 1030, 34 us forward for 30.  Their error is 4.0e-7
    // at reductions of 1000, and with WGK = 2, which makes four of them, 2.9e-7)
    GrpSums<T, TM, TN, (ES == 4 ? 2 : 1)> acc;
    acc.clear();
    float sums[TM];                                        // kWeights: of this lane's row of the left operand
#pragma unroll
    for (int i = 0; i < TM; ++i) sums[i] = 0.f;
    const bool take_sums = FORM == kWeights && p.colsum && g.col0 == 0 && wn == 0;

    const int steps = (g.red + A::BK - 1) / A::BK;
    auto compute = [&](int stage) {
        const char *d = lds + stage * STAGE;
#pragma unroll
        for (int c = 0; c < NKC / WGK; ++c) {
            const int kc = wk * (NKC / WGK) + c;
            u32x4_t fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = A::read(d, A::frag(wm * WTM + i * 32, kc, lane));
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = B::read(d + A::BYTES, B::frag(wn * WTN + j * 32, kc, lane));
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) grp_mma<T>(acc.c[i][j], fb[j], fa[i]);
            if constexpr (FORM == kWeights) {
                if (take_sums) {
#pragma unroll
                    for (int i = 0; i < TM; ++i) sums[i] += grp_sum<ES>(fa[i]);
                }
            }
        }
    };
    // Step s in stage s & 1, its operands having come through registers s % PF.  WHOLE: steps s + PF and s + 1 exist, and s + PF is whole.
    auto step = [&](int s, auto PARITY, auto WHOLE) {
        constexpr int q = decltype(PARITY)::value;
        __syncthreads();                                   // stage s & 1 is written, the other stage's last readers are through
        if constexpr (decltype(WHOLE)::value) {
            la.load_whole(ra[q]);
            lb.load_whole(rb[q]);
        } else {
            la.load(ra[q]);
            lb.load(rb[q]);
        }
        compute(q & 1);
        if (decltype(WHOLE)::value || s + 1 < steps) store((q & 1) ^ 1, ra[(q + 1) % PF], rb[(q + 1) % PF]);
    };
    if (steps > 0) {
#pragma unroll
        for (int i = 0; i < PF; ++i) {
            la.load(ra[i]);
            lb.load(rb[i]);
        }
        store(0, ra[0], rb[0]);
    }
    const int whole = min(la.whole(), lb.whole());
    int s = 0;
    auto round = [&](auto WHOLE) {
        step(s, std::integral_constant<int, 0>{}, WHOLE);
        if (decltype(WHOLE)::value || s + 1 < steps) step(s + 1, std::integral_constant<int, 1>{}, WHOLE);
        s += PF;
    };
    // (without branches around the loads, so that no step waits for more of them than it needs)
    while (s + PF <= whole) round(std::true_type{});
    while (s < steps) round(std::false_type{});
    acc.join();
    __syncthreads();                                       // the last stage's readers are through
    if constexpr (WGK > 1) {
        char *mine = lds + tile * TM * TN * 4096;
        if (wk > 0) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) *(u32x4_t *)(mine + ((i * TN + j) * 4 + q) * 1024 + lane * 16) = grp_quarter(acc.c[i][j][0], q);
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) grp_add_quarter(acc.c[i][j][0], q, *(const u32x4_t *)(mine + ((i * TN + j) * 4 + q) * 1024 + lane * 16));
    }
    if (take_sums) grp_store_sums(p, g, sums, wm * WTM, lane);
    grp_epilogue<T, FORM, TM, TN>(p, g, acc, lds + tile * kStageBytes, wm * WTM, wn * WTN, lane);
}

// ---- the kernel for operands of whole 16-byte chunks: global memory straight into LDS -------------------------------------------

// An operand's loads: every lane's byte offset from the tile's base of step 0 is fixed; the base moves on from step to step, and the descriptor
// ends where the operand does, so that what lies behind the reduction or outside the tile reads zeros.
template <int ES, bool RED, int OUTER, int BKB, int NW>
struct GrpStream {
    using Op = GrpOperand<ES, RED, OUTER, BKB>;
    static constexpr int NL = Op::BYTES / 1024 / NW;       // wave loads per wave and step
    static_assert(NL * NW * 1024 == Op::BYTES && NL >= 1, "whole wave loads");
    static_assert(!RED || NW * 64 / Op::CPR % (256 / BKB * Op::CPR) == 0, "a lane's loads lie in one chunk column");
    uint32_t voff[NL];
    int chunk;                             // RED: this lane's chunk, as a byte offset inside a step
    uint64_t base;
    int left;                              // of the reduction from base on: bytes of a row (RED) or rows
    int ld, tail;                          // bytes between rows; RED: span of the rows before the last

    __device__ __forceinline__ void start(const char *p0, int64_t ld_, int outer_left, int red, int wave, int lane)
    {
        const uint64_t at = (uint64_t)p0;
        base = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
        ld = (int)ld_;
        left = __builtin_amdgcn_readfirstlane(RED ? (red * ES + 15) & ~15 : red);       // (rows are whole chunks)
        tail = __builtin_amdgcn_readfirstlane((min(max(outer_left, 1), OUTER) - 1) * ld);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            int r, e;
            Op::slot((i * NW + wave) * 64 + lane, r, e);
            const bool in = RED ? r < outer_left : e < outer_left;
            voff[i] = in ? (uint32_t)(r * ld + e * ES) : kOutOfRange;
            if (i == 0) chunk = e * ES;
        }
    }
    // (a step behind the operand's end has nothing left)
    __device__ __forceinline__ i32x4_t rsrc() const
    {
        const int bytes = RED ? left + tail : min(left, Op::BK) * ld;
        return make_rsrc((const void *)base, left > 0 ? (uint32_t)bytes : 0u);
    }
    // RED: this lane's chunk lies behind the reduction's end, which is not the descriptor's but in the last row
    __device__ __forceinline__ uint32_t past() const { return RED && chunk >= left ? kOutOfRange : 0u; }
    __device__ __forceinline__ void next()
    {
        base += RED ? (uint64_t)BKB : (uint64_t)((int64_t)ld * Op::BK);
        left -= RED ? BKB : Op::BK;
    }
};

// Tiles of 64x64, 128x64 and 128x128: a workgroup's operands run through a ring of NS stages in LDS.  At the barrier of step s the stages of steps s and
// s + 1 have landed and every wave has read stage s - 1 for the last time; then the loads of step s + NS - 1 go out into that stage, and each chunk's
// fragments are read three chunks before they are used, across the barrier too (a read takes about as long as four matrix instructions).  A wave issues
// in order, and a matrix instruction hides eight other instructions at most: behind each stand a few operand reads and loads, and the order is pinned.
// Bound by latency on small calls (the loads of three steps in flight are what hides it: 64 x 4096 x 4096 in 8 bits 9.6 us, 1.8 TB/s), by operand
// delivery into LDS above (2048 x 768 x 3072 in 8 bits, 192 tiles of 128x64, 13.0 us: steps of 24 KB in 0.33 us, 73 GB/s to a compute unit).
template <typename T, int FORM, int BM, int BN, int WGM, int WGN, int BKB, int NS>
struct GrpRing {
    using type = T;
    static constexpr int kForm = FORM, kBM = BM, kBN = BN, ES = GrpTraits<T>::ES;
    static constexpr int NW = WGM * WGN, THREADS = 64 * NW;
    static constexpr int WTM = BM / WGM, WTN = BN / WGN, TM = WTM / 32, TN = WTN / 32, NKC = BKB / 32;
    using SA = GrpStream<ES, FORM != kWeights, BM, BKB, NW>;
    using SB = GrpStream<ES, FORM == kForward, BN, BKB, NW>;
    using A = typename SA::Op;
    using B = typename SB::Op;
    static constexpr int BK = A::BK, STAGE = A::BYTES + B::BYTES, LPS = SA::NL + SB::NL;
    static constexpr int AHEAD = 3, NBUF = AHEAD + 1;
    static_assert(NS == 4 && NS * LPS < 60 && NKC % NBUF == 0, "ring");
    static constexpr int kLds = NS * STAGE;
    static_assert(NW * kStageBytes <= kLds, "staging");
    static_assert(kLds <= 160 * 1024, "LDS");

    static __device__ __forceinline__ void tile(const GroupedParams &p, const GrpProblem &g, char *lds)
    {
        const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave / WGN, wn = wave % WGN;
        SA sa;
        SB sb;
        sa.start(g.a0, p.lda, g.row_end - g.row0, g.red, wave, lane);
        sb.start(g.b0, p.ldb, p.cols - g.col0, g.red, wave, lane);
        i32x4_t rsa, rsb;
        uint32_t pasta, pastb, ldst = lds0 + wave * 1024;
        int lstage = 0;
        auto open_stage = [&]() { rsa = sa.rsrc(); rsb = sb.rsrc(); pasta = sa.past(); pastb = sb.past(); };
        auto issue_one = [&](int i) {
            if (i < SA::NL) dma_load16_s(rsa, sa.voff[i] | pasta, 0u, ldst + i * (NW * 1024));
            else dma_load16_s(rsb, sb.voff[i - SA::NL] | pastb, 0u, ldst + A::BYTES + (i - SA::NL) * (NW * 1024));
        };
        auto close_stage = [&]() {
            sa.next();
            sb.next();
            ++lstage;
            ldst += STAGE;
            if (lstage == NS) { lstage = 0; ldst -= NS * STAGE; }
        };
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) {
            open_stage();
#pragma unroll
            for (int i = 0; i < LPS; ++i) issue_one(i);
            close_stage();
        }

        // This lane's fragments in stage 0.  Where the reduction is contiguous, the wave's tiles are a fixed distance apart (whole swizzle periods)
        // and every chunk has an address of its own; otherwise the chunks are, and every tile has one.
        constexpr int NA = A::kRed ? NKC : TM, NB = B::kRed ? NKC : TN;
        uint32_t a_at[NA], b_at[NB];
#pragma unroll
        for (int i = 0; i < NA; ++i) a_at[i] = A::kRed ? A::frag(wm * WTM, i, lane) : A::frag(wm * WTM + i * 32, 0, lane);
#pragma unroll
        for (int i = 0; i < NB; ++i) b_at[i] = A::BYTES + (B::kRed ? B::frag(wn * WTN, i, lane) : B::frag(wn * WTN + i * 32, 0, lane));

        GrpSums<T, TM, TN> acc;
        acc.clear();
        float sums[TM];                                    // kWeights: of this lane's row of the left operand
#pragma unroll
        for (int i = 0; i < TM; ++i) sums[i] = 0.f;
        const bool take_sums = FORM == kWeights && p.colsum && g.col0 == 0 && wn == 0;

        u32x4_t fa[NBUF][TM], fb[NBUF][TN];
        auto read_one = [&](int buf, int r, uint32_t stage, int kc) {
            // (in the order in which the matrix instructions want them: the first row, all columns, the other rows)
            if (r == 0 || r > TN) {
                const int i = r == 0 ? 0 : r - TN;
                fa[buf][i] = A::read(lds, stage + a_at[A::kRed ? kc : i] + A::apart(i, kc));
            } else {
                fb[buf][r - 1] = B::read(lds, stage + b_at[B::kRed ? kc : r - 1] + B::apart(r - 1, kc));
            }
        };

        const int steps = (g.red + BK - 1) / BK;
        wait_vmcnt<(NS - 3) * LPS>();
        lds_barrier();
        uint32_t stage = 0;
#pragma unroll
        for (int c = 0; c < AHEAD; ++c)
#pragma unroll
            for (int r = 0; r < TM + TN; ++r) read_one(c, r, 0, c);
        for (int s = 0; s < steps; ++s) {
            if (s > 0) {
                wait_vmcnt<(NS - 3) * LPS>();
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("s_barrier" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
            }
            const uint32_t next_stage = stage + STAGE == NS * STAGE ? 0 : stage + STAGE;
            open_stage();
            constexpr int READS = TM + TN, LOADS = (LPS + NKC - 1) / NKC, PER = (READS + LOADS + TM * TN - 1) / (TM * TN);    // of a chunk
#pragma unroll
            for (int kc = 0; kc < NKC; ++kc) {
                const int buf = kc % NBUF, ahead = (kc + AHEAD) % NKC;
                const bool wraps = kc + AHEAD >= NKC;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        grp_mma<T>(acc.c[i][j], fb[buf][j], fa[buf][i]);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int q = (i * TN + j) * PER; q < (i * TN + j + 1) * PER; ++q) {
                            if (q < READS) read_one((kc + AHEAD) % NBUF, q, wraps ? next_stage : stage, ahead);
                            else if (q < READS + LOADS && kc * LOADS + q - READS < LPS) issue_one(kc * LOADS + q - READS);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if constexpr (FORM == kWeights) {
                        if (take_sums) sums[i] += grp_sum<ES>(fa[buf][i]);
                    }
                }
            }
            close_stage();
            stage = next_stage;
        }
        acc.join();
        wait_vmcnt<0>();                                   // (the stages behind the last step's)
        __syncthreads();                                   // the last stage's readers are through
        if (take_sums) grp_store_sums(p, g, sums, wm * WTM, lane);
        grp_epilogue<T, FORM, TM, TN>(p, g, acc, lds + wave * kStageBytes, wm * WTM, wn * WTN, lane);
    }
};

// Tiles of 256x256, eight waves of 128x64 each: 64 KB of operands for 128 bytes of the reduction.  A step takes whole cache lines (with steps of 64
// bytes each line comes to the L1 twice, and these requests are the bound: 8192 x 8192 x 8192 in bf16 870 us, so 780 us, 1.41 PFLOP/s, and a library's
// product 673; in 8 bits 470 and 428 us, 2.57 POP/s, the library's 441, where the chip's power is the bound: it runs at two thirds of its clock).  Two
// stages fit and a half, so the ring has five units of one operand each, A and B in turn.  One barrier a step stands before its last chunk, whose
// fragments every wave has read by then: the step's two units are free, the next step's have landed, and its first fragments are read behind the last
// chunk's matrix instructions.  Into the freed units go B of the step after next (which has one step to land) and A of the one behind it (which has
// two), the loads evenly behind the matrix instructions of this chunk and the next.
template <typename T, int FORM>
struct GrpWide {
    using type = T;
    static constexpr int kForm = FORM, kBM = 256, kBN = 256, ES = GrpTraits<T>::ES, BM = kBM, BN = kBN, BKB = 128;
    static constexpr int WGM = 2, WGN = 4, NW = WGM * WGN, THREADS = 64 * NW;
    static constexpr int WTM = BM / WGM, WTN = BN / WGN, TM = WTM / 32, TN = WTN / 32, NKC = BKB / 32;
    using SA = GrpStream<ES, FORM != kWeights, BM, BKB, NW>;
    using SB = GrpStream<ES, FORM == kForward, BN, BKB, NW>;
    using A = typename SA::Op;
    using B = typename SB::Op;
    static constexpr int BK = A::BK, UNIT = A::BYTES, UNITS = 5, NL = SA::NL;
    static_assert(A::BYTES == B::BYTES && SB::NL == NL && NKC == 4, "units");
    static constexpr int kLds = UNITS * UNIT;
    static_assert(kLds <= 160 * 1024 && NW * kStageBytes <= kLds, "LDS");

    static __device__ __forceinline__ void tile(const GroupedParams &p, const GrpProblem &g, char *lds)
    {
        const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wm = wave / WGN, wn = wave % WGN;
        SA sa;
        SB sb;
        sa.start(g.a0, p.lda, g.row_end - g.row0, g.red, wave, lane);
        sb.start(g.b0, p.ldb, p.cols - g.col0, g.red, wave, lane);
        i32x4_t rs;
        uint32_t past, fill = 0;                           // fill: the unit that is loaded next, as an offset
        auto after = [&](uint32_t unit) { return unit + UNIT == UNITS * UNIT ? 0u : unit + UNIT; };
        auto open_a = [&]() { rs = sa.rsrc(); past = sa.past(); };
        auto open_b = [&]() { rs = sb.rsrc(); past = sb.past(); };
        auto load_a = [&](int i) { dma_load16_s(rs, sa.voff[i] | past, 0u, lds0 + fill + wave * 1024 + i * (NW * 1024)); };
        auto load_b = [&](int i) { dma_load16_s(rs, sb.voff[i] | past, 0u, lds0 + fill + wave * 1024 + i * (NW * 1024)); };
        auto close_a = [&]() { sa.next(); fill = after(fill); };
        auto close_b = [&]() { sb.next(); fill = after(fill); };
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (u % 2 == 0) open_a(); else open_b();
#pragma unroll
            for (int i = 0; i < NL; ++i) { if (u % 2 == 0) load_a(i); else load_b(i); }
            if (u % 2 == 0) close_a(); else close_b();
        }

        constexpr int NA = A::kRed ? NKC : TM, NB = B::kRed ? NKC : TN;
        uint32_t a_at[NA], b_at[NB];
#pragma unroll
        for (int i = 0; i < NA; ++i) a_at[i] = A::kRed ? A::frag(wm * WTM, i, lane) : A::frag(wm * WTM + i * 32, 0, lane);
#pragma unroll
        for (int i = 0; i < NB; ++i) b_at[i] = B::kRed ? B::frag(wn * WTN, i, lane) : B::frag(wn * WTN + i * 32, 0, lane);

        GrpSums<T, TM, TN> acc;
        acc.clear();
        float sums[TM];                                    // kWeights: of this lane's row of the left operand
#pragma unroll
        for (int i = 0; i < TM; ++i) sums[i] = 0.f;
        const bool take_sums = FORM == kWeights && p.colsum && g.col0 == 0 && wn == 0;

        u32x4_t fa[2][TM], fb[2][TN];
        auto read_one = [&](int buf, int r, uint32_t unit_a, uint32_t unit_b, int kc) {
            // (in the order in which the matrix instructions want them: the first row, all columns, the other rows)
            if (r == 0 || r > TN) {
                const int i = r == 0 ? 0 : r - TN;
                fa[buf][i] = A::read(lds, unit_a + a_at[A::kRed ? kc : i] + A::apart(i, kc));
            } else {
                fb[buf][r - 1] = B::read(lds, unit_b + b_at[B::kRed ? kc : r - 1] + B::apart(r - 1, kc));
            }
        };

        const int steps = (g.red + BK - 1) / BK;
        wait_vmcnt<(UNITS - 2) * NL>();
        lds_barrier();
        uint32_t ua = 0, ub = UNIT;
#pragma unroll
        for (int r = 0; r < TM + TN; ++r) read_one(0, r, ua, ub, 0);
        constexpr int READS = TM + TN, SLOTS = TM * TN, PER = (READS + SLOTS - 1) / SLOTS;
        open_a();                                          // (nothing is loaded in the first step's first chunk: its units are the prologue's)
        for (int s = 0; s < steps; ++s) {
            const uint32_t na = after(ub), nb = after(na);
#pragma unroll
            for (int kc = 0; kc < NKC; ++kc) {
                const int buf = kc & 1;
                if (kc == NKC - 1) {
                    // this wave has read the step's last fragments, and the next step's units have landed but for A of the step behind
                    wait_vmcnt<NL>();
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __builtin_amdgcn_sched_barrier(0);
                    asm volatile("s_barrier" ::: "memory");
                    __builtin_amdgcn_sched_barrier(0);
                    open_b();
                }
#pragma unroll
                for (int i = 0; i < TM; ++i) {
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const int slot = i * TN + j;
                        grp_mma<T>(acc.c[i][j], fb[buf][j], fa[buf][i]);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int q = slot * PER; q < (slot + 1) * PER && q < READS; ++q)
                            read_one(buf ^ 1, q, kc + 1 < NKC ? ua : na, kc + 1 < NKC ? ub : nb, (kc + 1) % NKC);
                        if (kc == NKC - 1 || (kc == 0 && s > 0)) {
#pragma unroll
                            for (int l = 0; l < NL; ++l)
                                if ((l * SLOTS + SLOTS / 2) / NL == slot) {
                                    if (kc == 0) load_a(l); else load_b(l);
                                }
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if constexpr (FORM == kWeights) {
                        if (take_sums) sums[i] += grp_sum<ES>(fa[buf][i]);
                    }
                }
                if (kc == NKC - 1) {
                    close_b();
                    open_a();
                }
                if (kc == 0 && s > 0) close_a();
            }
            ua = na;
            ub = nb;
        }
        acc.join();
        wait_vmcnt<0>();                                   // (the units behind the last step's)
        __syncthreads();                                   // the last units' readers are through
        if (take_sums) grp_store_sums(p, g, sums, wm * WTM, lane);
        grp_epilogue<T, FORM, TM, TN>(p, g, acc, lds + wave * kStageBytes, wm * WTM, wn * WTN, lane);
    }
};

template <typename K>
__global__ __launch_bounds__(K::THREADS, K::kLds > 80 * 1024 ? (K::NW + 3) / 4 : 1) void grouped_kernel(const GroupedParams p)
{
    extern __shared__ uint4 smem_u4[];
    GrpProblem only;
    if (!grp_problem<typename K::type, K::kForm, K::kBM, K::kBN>(p, threadIdx.x & 63, blockIdx.x, only)) return;
    K::tile(p, only, (char *)smem_u4);
}

// ---- large tiles, and small ones where they end ------------------------------------------------------------------------------------
//
// Tiles of 256x256 need the fewest bytes per product, but they are coarse: of 16384 rows in eight groups and 2048 columns they make 2.1 rounds of
// the chip, which take as long as three, and a group that ends one row into a tile pays for the whole.  So a launch has tiles of two sizes, first
// all large ones, then small ones of 128x128 (a round of them counts 0.36 of a round of large ones): where a group's last tile would be half empty, and in
// place of the large tiles of the last round where those would leave most of the chip idle.  As many workgroups as compute units walk over them.
constexpr int kSmallCost = 36;                             // percent

struct GrpSchedule {
    int beg, end, upto_large, upto_small;                  // of this lane's span (spans 0 .. 63): rows; row tiles up to and with it
    int spans, large, cut, units;                          // tiles that stay large; tiles cut into four; small tiles in all
};

__device__ __forceinline__ void grp_rows(int len, int &large, int &small)
{
    const int rest = len & 255;
    large = (len >> 8) + (rest > 128);
    small = rest > 0 && rest <= 128;
}

__device__ __forceinline__ void grp_schedule(const GroupedParams &p, int lane, GrpSchedule &h)
{
    int large = 0, small = 0, past_rows = 0;
    h.spans = p.offsets ? p.groups + 2 : 1;
    for (int s0 = 0; s0 < h.spans; s0 += 64) {
        int beg, end, l, m;
        grp_spans(p, s0, lane, past_rows, beg, end);
        grp_rows(end - beg, l, m);
        l = grp_scan(l);
        m = grp_scan(m);
        if (s0 == 0) { h.beg = beg; h.end = end; h.upto_large = l; h.upto_small = m; }
        large += __builtin_amdgcn_readlane(l, 63);
        small += __builtin_amdgcn_readlane(m, 63);
    }
    const int tiles = large * p.tiles_n, rest = small * ((p.cols + 127) / 128), over = tiles % p.places;
    const int idle = over ? (p.places - over) * 2 : 0;     // small tiles that fit beside the last round's large ones
    const int whole = 100 + max(0, rest - idle + p.places - 1) / p.places * kSmallCost, cut = (4 * over + rest + p.places - 1) / p.places * kSmallCost;
    h.cut = over > 0 && cut < whole ? over : 0;
    h.large = tiles - h.cut;
    h.units = 4 * h.cut + rest;
}

// Row tile `q` of one size, counted over all spans: its span's rows and its place among the span's tiles of that size.
__device__ __forceinline__ bool grp_row_tile(const GroupedParams &p, const GrpSchedule &h, int lane, bool is_small, uint32_t q, uint32_t per_row, int &span, int &beg, int &end,
                                             int &first, int &count)
{
    int before = 0, past_rows = 0;
    for (int s0 = 0; s0 < h.spans; s0 += 64) {
        int b = h.beg, e = h.end, upto = is_small ? h.upto_small : h.upto_large;
        if (h.spans > 64) {
            int l, m;
            grp_spans(p, s0, lane, past_rows, b, e);
            grp_rows(e - b, l, m);
            upto = grp_scan(is_small ? m : l);
        }
        const uint64_t past = __ballot((uint32_t)(before + upto) * per_row > q);
        if (past) {
            const int at = __builtin_ctzll(past);
            span = s0 + at;
            beg = __builtin_amdgcn_readlane(b, at);
            end = __builtin_amdgcn_readlane(e, at);
            int l, m;
            grp_rows(end - beg, l, m);
            count = is_small ? m : l;
            first = before + __builtin_amdgcn_readlane(upto, at) - count;
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Large (or small) tile i of XCD x.  False: there is none.
template <typename T, int FORM, bool SMALL>
__device__ __forceinline__ bool grp_unit(const GroupedParams &p, const GrpSchedule &h, int lane, int x, int i, GrpProblem &g)
{
    const int all = SMALL ? h.units : h.large, per = (all + 7) / 8;
    int span, beg, end, first, count, q = x * per + i, sub = 0;
    if (i >= per || q >= all) return false;
    if (SMALL && q >= 4 * h.cut) {                         // the small tiles behind a group's large ones
        q -= 4 * h.cut;
        const int cols = (p.cols + 127) / 128;
        if (!grp_row_tile(p, h, lane, true, q, cols, span, beg, end, first, count)) return false;
        grp_at<T, FORM>(p, min(span, p.groups), beg + ((end - beg) & ~255), end, (q - first * cols) % cols * 128, g);
        return true;
    }
    if (SMALL) { sub = q & 3; q = h.large + (q >> 2); }
    if (!grp_row_tile(p, h, lane, false, q, p.tiles_n, span, beg, end, first, count)) return false;
    int mt, nt;
    grp_order(p, q - first * p.tiles_n, count, mt, nt);
    grp_at<T, FORM>(p, min(span, p.groups), beg + mt * 256 + (sub >> 1) * 128, end, nt * 256 + (sub & 1) * 128, g);
    if (g.col0 >= p.cols) g.red = 0;                       // (nothing is left of the large tile there)
    return true;
}

// The walk scans the offsets for every tile, 64 at a time, which pays up to some number of groups: 256 rows each, 512 x 512 bf16, 1024 groups 250 us, 315 in
// tiles of 128x128 that are searched for, 2048 594 and 619, 4096 1893 and 1269.
constexpr int kWalkGroups = 2048;

constexpr int kLargeThreads = 512;

template <typename T, int FORM> struct GrpLarge {
    using Large = GrpWide<T, FORM>;
    using Small = GrpRing<T, FORM, 128, 128, 2, 4, 128, 4>;
    static_assert(Large::THREADS == kLargeThreads && Small::THREADS == kLargeThreads, "threads");
    static constexpr int kLds = Large::kLds > Small::kLds ? Large::kLds : Small::kLds;
};

template <typename T, int FORM>
__global__ __launch_bounds__(kLargeThreads, 2) void grouped_large_kernel(const GroupedParams p)
{
    extern __shared__ uint4 smem_u4[];
    const int lane = threadIdx.x & 63;
    GrpSchedule h;
    grp_schedule(p, lane, h);
    const int x = blockIdx.x & 7, step = gridDim.x >> 3;
    for (int i = blockIdx.x >> 3;; i += step) {
        GrpProblem g;
        if (!grp_unit<T, FORM, false>(p, h, lane, x, i, g)) break;
        GrpLarge<T, FORM>::Large::tile(p, g, (char *)smem_u4);
        __syncthreads();                                   // the staging is read before the next tile's loads land there
    }
    // (two small tiles each for the workgroups that have no large one in the last round, then one for each in turn)
    const int slot = blockIdx.x >> 3, busy = (h.large + 7) / 8 % step, idle = busy ? step - busy : 0;
    for (int k = slot >= busy && idle ? 0 : 2;; ++k) {
        GrpProblem g;
        const int i = k < 2 ? slot - busy + k * idle : 2 * idle + slot + (k - 2) * step;
        if (!grp_unit<T, FORM, true>(p, h, lane, x, i, g)) break;
        GrpLarge<T, FORM>::Small::tile(p, g, (char *)smem_u4);
        __syncthreads();
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------------------

// One product of `form` on the kernel that suits it (grouped_bf16.hip, grouped_f32.hip, grouped_i8.hip).
hipError_t grouped_run_bf16(int form, const GroupedParams &p, hipStream_t st);
hipError_t grouped_run_f32(int form, const GroupedParams &p, hipStream_t st);
hipError_t grouped_run_i8(const GroupedParams &p, hipStream_t st);
hipError_t grouped_run_adapted_bf16(const GroupedParams &p, hipStream_t st);
hipError_t grouped_run_adapted_f32(const GroupedParams &p, hipStream_t st);

// Most tiles of BM rows that any offsets can make of p.rows rows: each span ends in one part tile at most, and each tile has a
// row.  (As many slots grp_search counts on.)
inline int64_t grp_row_tiles(const GroupedParams &p, int BM)
{
    if (!p.offsets) return ((int64_t)p.rows + BM - 1) / BM;
    return std::min<int64_t>(p.rows, p.rows / BM + (int64_t)p.groups + 2);
}

// Sets the column tiles and works out the workgroups of a launch (0: nothing to do).
template <int FORM, int BM, int BN>
hipError_t grp_grid(GroupedParams &p, int threads, unsigned *grid)
{
    p.tiles_n = (p.cols + BN - 1) / BN;
    p.d_panel = make_fastdiv((uint32_t)(kPanel * p.tiles_n));
    int64_t n;
    if (FORM == kWeights) n = (int64_t)grp_weight_tiles((p.rows + BM - 1) / BM * p.tiles_n) * p.groups;
    else n = (grp_row_tiles(p, BM) * p.tiles_n + 7) / 8 * 8;               // (a block of tiles for each XCD)
    if (n * threads > 0xffffffffll) return hipErrorInvalidConfiguration;   // (threads of a launch)
    *grid = (unsigned)n;
    return hipSuccess;
}

template <typename T, int FORM, int BM, int BN, int WGM, int WGN, int WGK>
hipError_t grouped_any(GroupedParams p, hipStream_t st)
{
    unsigned grid;
    const hipError_t e = grp_grid<FORM, BM, BN>(p, 64 * WGM * WGN * WGK, &grid);
    if (e != hipSuccess || !grid) return e;
    hipLaunchKernelGGL((grouped_any_kernel<T, FORM, BM, BN, WGM, WGN, WGK>), dim3(grid), dim3(64 * WGM * WGN * WGK), 2 * (BM + BN) * 128, st, p);
    return hipGetLastError();
}

template <typename T, int NT, int NW, int BATCH>
hipError_t grouped_few(GroupedParams p, hipStream_t st)
{
    unsigned grid;
    const hipError_t e = grp_grid<kForward, 16, 16 * NT>(p, 64 * NW, &grid);
    if (e != hipSuccess || !grid) return e;
    if constexpr (GrpTraits<T>::ES < 4) {
        if (((uint64_t)p.a | (uint64_t)p.b | (uint64_t)p.lda | (uint64_t)p.ldb | (uint64_t)p.b_group) % 4) {
            hipLaunchKernelGGL((grouped_few_kernel<T, NT, NW, BATCH, false>), dim3(grid), dim3(64 * NW), 0, st, p);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((grouped_few_kernel<T, NT, NW, BATCH, true>), dim3(grid), dim3(64 * NW), 0, st, p);
    return hipGetLastError();
}

template <typename T>
hipError_t grouped_few_dx(GroupedParams p, hipStream_t st)
{
    constexpr int NW = 8;
    unsigned grid;
    const hipError_t e = grp_grid<kInput, 16, 64>(p, 64 * NW, &grid);
    if (e != hipSuccess || !grid) return e;
    hipLaunchKernelGGL((grouped_few_dx_kernel<T, NW>), dim3(grid), dim3(64 * NW), 0, st, p);
    return hipGetLastError();
}

// Whether the direct loads take a product: whole chunks at whole addresses, and a tile's rows (or steps) within a descriptor.
template <typename T, int FORM>
bool grp_streams(const GroupedParams &p)
{
    constexpr int ES = GrpTraits<T>::ES;
    const uint64_t bits = (uint64_t)p.a | (uint64_t)p.b | (uint64_t)p.lda | (uint64_t)p.ldb | (uint64_t)p.b_group |
                          (FORM != kWeights ? (uint64_t)p.red * ES : (uint64_t)p.rows * ES) | (FORM == kForward ? 0 : (uint64_t)p.cols * ES);
    return (bits % 16 == 0 || (p.flags & kGrpPacked)) && p.lda <= (1 << 22) && p.ldb <= (1 << 22) && p.ldy <= (1 << 22) && p.ldmask <= (1 << 22);
}

template <typename K>
hipError_t grouped_tiles(GroupedParams p, hipStream_t st)
{
    unsigned grid;
    hipError_t e = grp_grid<K::kForm, K::kBM, K::kBN>(p, K::THREADS, &grid);
    if (e != hipSuccess || !grid) return e;
    auto kern = grouped_kernel<K>;
    static OncePerDevice lds_once;
    e = allow_lds(lds_once, (const void *)kern);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3(grid), dim3(K::THREADS), K::kLds, st, p);
    return hipGetLastError();
}

template <typename T, int FORM>
hipError_t grouped_large(GroupedParams p, hipStream_t st)
{
    p.tiles_n = (p.cols + 255) / 256;
    p.d_panel = make_fastdiv((uint32_t)(kPanel * p.tiles_n));
    if (grp_row_tiles(p, 256) * p.tiles_n * 4 > 0x7fffffff) return hipErrorInvalidConfiguration;
    auto kern = grouped_large_kernel<T, FORM>;
    static OncePerDevice lds_once;
    const hipError_t e = allow_lds(lds_once, (const void *)kern);
    if (e != hipSuccess) return e;
    constexpr int lds = GrpLarge<T, FORM>::kLds;
    hipLaunchKernelGGL(kern, dim3((p.places + 7) / 8 * 8), dim3(kLargeThreads), lds, st, p);
    return hipGetLastError();
}

// ---- which kernel a call runs ------------------------------------------------------------------------------------------------------
//
// Rows of each group: the offsets lie on the device, so the rule takes them as even.

// Tiles of BM x BN.
template <int FORM>
inline double grp_tiles(const GroupedParams &p, int BM, int BN)
{
    const int64_t cols = (p.cols + BN - 1) / BN;
    if (FORM == kWeights) return (double)((p.rows + BM - 1) / BM) * cols * p.groups;
    const int64_t spans = !p.offsets ? 1 : p.groups < p.rows ? p.groups : p.rows, each = (p.rows + spans - 1) / spans;
    return (double)spans * ((each + BM - 1) / BM) * cols;
}

// Time of a launch in us without what every launch costs: rounds of the chip's `places`, each a fixed part and a part for every 128 bytes of the
// reduction; a round that leaves places idle runs faster, the others having more of the caches and the clock to themselves.
struct GrpTime { double fixed, reduction; };
inline GrpTime grp_rounds(double tiles, double places, double units, double fixed, double per_unit)
{
    const double rounds = std::ceil(tiles / places);
    return {rounds * fixed, rounds * per_unit * units * (0.5 + 0.5 * tiles / (rounds * places))};
}

// Whether a forward product runs in tiles of 16 rows.  With up to 16 rows a group in the mean, even groups' weights are what there is to read, and they
// are read once: 16 x 4096 x 4096 in 8 bits 6.6 us.  A popular group's are read for every 16 of its rows, again from the caches, which takes about as
// long as the weights of as many groups from memory and far longer than large tiles would: 1000 rows of 64 groups, 4096 x 4096 bf16, even 441 us, half
// of them in one group 517, all in one 340 (that group alone, in larger tiles, 41); in 8 bits 225, 264 and 179 (25).  With more rows, where these tiles
// are so few that they all run at once, as the other kernels would leave most of the chip idle: 64 x 1024 x 4096 (256 tiles) 6.6 us for 12.8, 512 x 64 x
// 4096 6.4 for 12.8; 32 x 8192 x 8192 (1024) 25.1 for 16.4, 64 x 3000 x 2048 (752) 8.4 for 6.7.  In fp32 the others are slower and the line lies higher:
// 512 x 512 x 2048 (1024 tiles) 26.5 us for 42.8; 256 rows of 8 groups, 2048 x 2048 (2048), 51.5 for 47.2.
inline bool grp_is_few(const GroupedParams &p, int ES)
{
    const int64_t spans = !p.offsets ? 1 : p.groups < p.rows ? p.groups : p.rows;
    return p.rows <= 16 * spans || grp_tiles<kForward>(p, 16, 16) <= (ES == 4 ? 4 : 2) * p.places;
}

// The same for the gradient by the rows, in fp32 and where the direct loads do not take the operands (bf16 through those is as fast: 16 x 8192 x 8192
// 26.3 us, 28.6 so).  fp32: 316 rows, 1536 x 265 (100 tiles), 14.0 us for 30.0, 256 rows of 8 groups, 2048 x 2048 (512), 32.2 for 45.4, 1000 of 5, 1030 x 515
// (585), 30.9 for 24.6; bf16: one row, 3742 x 170, 12.9 for 17.1, 316 rows, 1536 x 265, 9.1 for 11.9.
inline bool grp_is_few_dx(const GroupedParams &p, int ES)
{
    const int64_t spans = !p.offsets ? 1 : p.groups < p.rows ? p.groups : p.rows;
    return p.rows <= 16 * spans || grp_tiles<kInput>(p, 16, 64) <= (ES == 4 ? 2 : 1) * p.places;
}

// Tiles of 64x64 with a deep ring (one to a compute unit) or a shallow one (two), of 128x64, of 128x128, of 256x256, for operands of 8 or 16 bits; the
// constants are those of 8-bit products of 32 .. 8192 rows, 768 .. 8192 columns and reductions of 512 .. 8192, which they give to 10 %; bf16 has the
// same tiles in bytes.  (128x64 for one round of the chip: 2048 x 1024 x 4096 17.2 us, 20.1 in tiles of 64x64, 19.9 of 128x128; the gradient by the rows
// gains nothing: 2000 rows of 8, 768 x 1024, 10.1 and 9.4.)
enum { kDeep, kShallow, kHalf, kMiddle, kLarge };
template <int FORM>
inline int grp_choose(const GroupedParams &p, int ES, GrpTime *time)
{
    const double places = p.places, units = std::ceil((double)p.red * ES / 128.0 / (FORM == kWeights ? p.groups : 1)), n64 = grp_tiles<FORM>(p, 64, 64);
    const GrpTime t[5] = {n64 <= places ? GrpTime{2.0, 0.21 * units} : GrpTime{1e30, 0.0}, grp_rounds(n64, 2 * places, units, 3.0, 0.43),
                          FORM == kForward ? grp_rounds(grp_tiles<FORM>(p, 128, 64), places, units, 2.3, 0.33) : GrpTime{1e30, 0.0},
                          grp_rounds(grp_tiles<FORM>(p, 128, 128), places, units, 3.3, 0.54), grp_rounds(grp_tiles<FORM>(p, 256, 256), places, units, 8.6, 1.57)};
    int best = 0;
    for (int i = 1; i < 5; ++i)
        if (t[i].fixed + t[i].reduction < t[best].fixed + t[best].reduction) best = i;
    *time = t[best];
    return best;
}

template <typename T, int FORM>
hipError_t grouped_run(const GroupedParams &p, hipStream_t st)
{
    constexpr int ES = GrpTraits<T>::ES;
    const double places = p.places;
    if constexpr (FORM == kForward && !GrpTraits<T>::ADAPT) {      // (few rows with adapters: adapters.hip)
        // (columns in twos, four waves, where that fills the chip, else one by one and eight waves to a reduction: 16 x 4096 x 4096 6.6 against 8.5 us,
        // 32 x 4096 x 4096 10.4 against 8.6)
        if (grp_is_few(p, ES))
            return grp_tiles<FORM>(p, 16, 16) <= places ? grouped_few<T, 1, 8, 2>(p, st) : grouped_few<T, 2, 4, 2>(p, st);
    }
    if constexpr (FORM == kInput) {
        if ((ES == 4 || !grp_streams<T, FORM>(p)) && grp_is_few_dx(p, ES)) return grouped_few_dx<T>(p, st);
    }
    if (!grp_streams<T, FORM>(p)) {
        // Tiles of 128x128 once they fill half the chip: 1500 x 1501 x 2049 in 8 bits (144 tiles) 21.8 us, in tiles of 64x64 27.2; 2048 x 770 x 3073 (112)
        // 28.0 and 26.0.  In fp32 the matrix cores are the bound, and small tiles leave none idle: 1001 rows of 13 groups, 515 x 1030, 25 against 72 us,
        // 5000 rows of 5 groups, 2047 x 4095, 708 against 760.
        if constexpr (ES < 4) {
            if (grp_tiles<FORM>(p, 128, 128) >= 0.5 * places) return grouped_any<T, FORM, 128, 128, 2, 4, 1>(p, st);
        }
        // While each compute unit has two tiles at most, twice the waves, which share every step's chunks: 333 x 1001 x 2049 in 8 bits 11.7 us for 13.1,
        // 1001 fp32 rows of 13 groups, 515 x 1030, 25.9 for 27.1; at 5000 rows, 2047 x 4095, 697 and 693.
        if constexpr (FORM != kWeights) {
            if (grp_tiles<FORM>(p, 64, 64) <= 2 * places) return grouped_any<T, FORM, 64, 64, 2, 2, 2>(p, st);
        }
        return grouped_any<T, FORM, 64, 64, 2, 2, 1>(p, st);
    }
    if constexpr (ES == 4) {
        // (as above; 5000 rows of 5 groups, 2048 x 4096: forward 695 us in tiles of 64x64, 762 of 128x128, by the weights 682 and 657)
        return FORM == kWeights && grp_tiles<FORM>(p, 128, 128) >= 4 * places ? grouped_tiles<GrpRing<T, FORM, 128, 128, 2, 4, 128, 4>>(p, st)
                                                                               : grouped_tiles<GrpRing<T, FORM, 64, 64, 2, 2, 128, 4>>(p, st);
    } else {
        GrpTime time;
        switch (grp_choose<FORM>(p, ES, &time)) {
            case kDeep: return grouped_tiles<GrpRing<T, FORM, 64, 64, 2, 2, 256, 4>>(p, st);
            case kShallow: return grouped_tiles<GrpRing<T, FORM, 64, 64, 2, 2, 128, 4>>(p, st);
            case kHalf:
                if constexpr (FORM == kForward) return grouped_tiles<GrpRing<T, FORM, 128, 64, 4, 2, 128, 4>>(p, st);
                break;                                     // (of the forward product only)
            case kMiddle: return grouped_tiles<GrpRing<T, FORM, 128, 128, 2, 4, 128, 4>>(p, st);
        }
        if constexpr (FORM == kWeights) return grouped_tiles<GrpWide<T, FORM>>(p, st);
        else if (p.offsets && p.groups > kWalkGroups) return grouped_tiles<GrpRing<T, FORM, 128, 128, 2, 4, 128, 4>>(p, st);
        else return grouped_large<T, FORM>(p, st);
    }
}

}  // namespace alt
