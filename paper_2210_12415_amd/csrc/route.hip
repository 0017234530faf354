// The experts of each token, their order, and the gradient by the logits.
//
//   score = softmax or sigmoid of a row of logits, choice = score + bias or the logit, the top_k largest choices (of the worthiest groups);
//   a place for every (token, choice) in the order of expert, token, choice: offsets and rows
//
// There is little to read: 16384 x 256 fp32 logits are 3 us of memory.  The time goes into launches and into the selection, about 100 instructions of a
// wave for each choice of its four rows, so lanes hold many experts and few lanes a row: with eight choices, biases and groups 23.4 us, 20.5 without groups,
// 16.3 without biases, and of them 7 for the ranks' two launches.  One launch chooses and ranks the choices inside each
// workgroup's tokens; where there is one workgroup that is all, else the ranks are moved by what the workgroups before have of each expert.
#include "common.h"
#include "rows.h"

namespace alt {
namespace {

constexpr int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64;

struct RouteParams {
    const char *logits;
    const float *bias;
    int32_t *experts;
    float *weights;
    int32_t *rows, *offsets;
    uint16_t *counts;                      // [workgroups][num]: choices of each expert
    int32_t *before;                       // [workgroups][num]: those of the workgroups before; then [num]: of all (route_scan_kernel)
    int64_t ld;                            // bytes between rows of logits
    int32_t tokens, num, top_k, groups, top_groups, group_best, softmax, renorm, chunks, size, listed;     // size: bytes of a logit; listed: choices of lists
    FastDiv each;                          // experts of a group
    float scale;
};

// ---- values of the lanes that share a row ------------------------------------------------------------------------------------------

template <int N, typename T>
__device__ __forceinline__ T rotated(T v)                  // of the lane N before, in turn inside 16 lanes
{
    if constexpr (sizeof(T) == 8) {
        const uint64_t w = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, 0x120 + N, 0xf, 0xf, true);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), 0x120 + N, 0xf, 0xf, true);
        return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
    } else {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, true));
    }
}

// f over the L (16, 32 or 64) lanes of a row, the same in all of them.
template <int L, typename T, typename F>
__device__ __forceinline__ T over_row(T v, F f)
{
    v = f(v, rotated<8>(v));
    v = f(v, rotated<4>(v));
    v = f(v, rotated<2>(v));
    v = f(v, rotated<1>(v));
    if constexpr (L >= 32) v = f(v, __shfl_xor(v, 16));
    if constexpr (L == 64) v = f(v, __shfl_xor(v, 32));
    return v;
}
// (of numbers: no NaN comes here)
__device__ __forceinline__ float larger(float a, float b) { return __builtin_fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return __builtin_fmax(a, b); }
__device__ __forceinline__ int larger(int a, int b) { return max(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return __builtin_fminf(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return __builtin_fmin(a, b); }
__device__ __forceinline__ int smaller(int a, int b) { return min(a, b); }
template <int L, typename T> __device__ __forceinline__ T row_max(T v) { return over_row<L>(v, [](T a, T b) { return larger(a, b); }); }
template <int L, typename T> __device__ __forceinline__ T row_min(T v) { return over_row<L>(v, [](T a, T b) { return smaller(a, b); }); }
template <int L, typename T> __device__ __forceinline__ T row_sum(T v) { return over_row<L>(v, [](T a, T b) { return a + b; }); }

// This lane's V logits, of the experts from e0 on; -inf behind the last.
template <int ES, int V>
__device__ __forceinline__ void load_logits(const char *row, int e0, int num, float (&l)[V])
{
    if (e0 + V <= num) {
        if constexpr (V * ES >= 16) {
#pragma unroll
            for (int i = 0; i < V * ES / 16; ++i) {
                w4_t c;
                float f[16 / ES];
                __builtin_memcpy(&c, row + (int64_t)e0 * ES + i * 16, 16);
                floats16<ES>(c, f);
#pragma unroll
                for (int q = 0; q < 16 / ES; ++q) l[i * (16 / ES) + q] = f[q];
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) l[i] = element<ES>(row + (int64_t)(e0 + i) * ES);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = e0 + i < num ? element<ES>(row + (int64_t)(e0 + i) * ES) : -INFINITY;
    }
}

__device__ __forceinline__ float exp_of(float v) { return expf(v); }
__device__ __forceinline__ double exp_of(double v) { return exp(v); }

// (by the exponential of what is negative: nothing overflows, and small results keep their digits)
template <typename F>
__device__ __forceinline__ F sigmoid_of(F v)
{
    const F e = exp_of(v < 0 ? v : -v);
    return (v < 0 ? e : (F)1) / (1 + e);
}

// A chosen expert's share of the chosen scores of its row: s, the sigmoid of v, to a lane (`is`: where there is one).  From -87 down exponentials lose digits in
// 32 bits and then all; where the scores are small, so that 1 + exp(v) is 1, their shares are those of a softmax, which keeps them.  (Scores that are zero in 64 bits are zero.)
template <int L>
__device__ __forceinline__ float sigmoid_share(float s, float v, bool is)
{
    const float sum = row_sum<L>(s);
    const bool small = sum < 0x1p-32f;
    float share = s / (sum > 0.f ? sum : 1.f);
    if (__ballot(is && small)) {
        const float top = row_max<L>(is ? v : -INFINITY), e = is && top > -745.13f ? expf(v - top) : 0.f, all = row_sum<L>(e);
        if (small) share = all > 0.f ? e / all : 0.f;
    }
    return share;
}

__device__ __forceinline__ float element_at(const char *row, int size, int e) { return size == 4 ? element<4>(row + (int64_t)e * 4) : element<2>(row + (int64_t)e * 2); }

// Sum over the lanes of the row up to and with this one.
template <int L>
__device__ __forceinline__ int row_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    if constexpr (L >= 32) v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true);
    if constexpr (L == 64) v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true);
    return v;
}

// ---- the choice --------------------------------------------------------------------------------------------------------------------

// What a row's lanes know of it: the largest logit, the sum of exp(logit - top), and whether it is lost to a NaN.
struct RowStats { float top, sum; bool lost; };

// Score and bias of an expert, by numbers of type F; -inf for one that is out.  `sum`: of the exponentials, in 32 bits its reciprocal.
template <typename F>
__device__ __forceinline__ F worth_of(const RouteParams &p, float l, float bias, const RowStats &st, F sum)
{
    F s;
    if constexpr (sizeof(F) == 4) {
        // (the hardware's base-2 exponential and reciprocal, each off by 2^-23 of itself: what is near is computed again anyway)
        const float x = p.softmax ? l - st.top : -__builtin_fabsf(l), e = __builtin_amdgcn_exp2f(x * 0x1.715476p+0f);
        s = p.softmax ? e * sum : (l < 0.f ? e : 1.f) * __builtin_amdgcn_rcpf(1.f + e);
    } else {
        s = p.softmax ? exp_of((F)l - (F)st.top) / sum : sigmoid_of((F)l);
    }
    const F w = s + (F)bias;
    return l == -INFINITY || w != w || st.lost ? (F)-INFINITY : w;
}

// (What is computed again is read again, in loops: all of it at once, from registers, takes scalar registers from what is always computed: 16384 tokens of 256
// experts, eight choices with biases, 23.2 us, so 20.6.)
template <int L, int V>
__device__ __forceinline__ double exact_sum(const RouteParams &p, const char *row, int e0, const RowStats &st)
{
    double sum = 0;
    if (!p.softmax) return sum;
#pragma unroll 4
    for (int i = 0; i < V; ++i) {
        const float l = e0 + i < p.num ? element_at(row, p.size, e0 + i) : -INFINITY;
        sum += l == -INFINITY ? 0.0 : exp((double)l - (double)st.top);
    }
    return row_sum<L>(sum);
}

// The worth in 64 bits of an expert that may be behind the last.
__device__ __forceinline__ double exact_worth(const RouteParams &p, const char *row, int e, const RowStats &st, double sum)
{
    const bool is = e < p.num;
    return worth_of<double>(p, is ? element_at(row, p.size, e) : -INFINITY, is && p.bias ? p.bias[e] : 0.f, st, sum);
}

template <typename F>
__device__ __forceinline__ void better_of(F v, F &one, F &two)
{
    two = v > one ? one : v > two ? v : two;
    one = v > one ? v : one;
}

// Which of a lane's V experts are of the row's worthiest groups, as bits.  In the row's LDS: the worths of the experts (or of each lane's two best, of
// `best_two`, where a lane's experts are of one group), in their place those of the groups, in the place of those which groups are kept.  `apart`: by how much the least
// worthy group that is kept is worth more than the worthiest that is not.
template <typename F, int L, int V, typename W, typename B>
__device__ __forceinline__ uint32_t kept_experts(const RouteParams &p, int sub, F *worth, W worth_at, B best_two, F &apart)
{
    const F none = -INFINITY, lowest = sizeof(F) == 4 ? (F)-__FLT_MAX__ : (F)-__DBL_MAX__;
    const int each = (int)p.each.d;
    const bool lanes = each % V == 0;
    const int per = lanes ? each / V * 2 : each;           // numbers of a group
    auto at = [](int i) { return i + (i >> 5); };          // (groups of 32 numbers begin at different banks)
    F one = none, two = none;
    if (lanes) {
        best_two(one, two);
        worth[at(sub * 2)] = one;
        worth[at(sub * 2 + 1)] = two;
    } else if constexpr (sizeof(F) == 8) {
#pragma unroll 2
        for (int i = 0; i < V; ++i) worth[at(sub * V + i)] = worth_at(i);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) worth[at(sub * V + i)] = worth_at(i);
    }
    wave_sync();
    for (int g = sub; g < p.groups; g += L) {
        one = two = none;
        for (int i = g * per; i < (g + 1) * per; ++i) better_of(worth[at(i)], one, two);
        // (a sum below the lowest number is not that of a group without experts; these numbers are this lane's alone)
        worth[at(g * per)] = p.group_best == 2 && two > none ? larger(one + two, lowest) : one;
    }
    wave_sync();
    uint32_t mine = 0;
    F least = INFINITY, most = none;
    for (int g = sub, i = 0; g < p.groups; g += L, ++i) {
        const F v = worth[at(g * per)];
        int better = 0;
#pragma unroll 8
        for (int o = 0; o < p.groups; ++o) {
            const F w = worth[at(o * per)];
            better += w > v || (w == v && o < g);
        }
        if (better < p.top_groups) {
            mine |= 1u << i;
            if (v > none) least = v < least ? v : least;
        } else {
            most = v > most ? v : most;
        }
    }
    wave_sync();
    for (int g = sub, i = 0; g < p.groups; g += L, ++i) worth[at(g * per)] = mine >> i & 1 ? (F)1 : (F)0;
    wave_sync();
    uint32_t kept = 0;
    if (lanes) {
        if (sub * V < p.num && worth[at((int)fast_div((uint32_t)(sub * V), p.each) * per)] != 0) kept = ~0u;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = sub * V + i;
            if (e < p.num && worth[at((int)fast_div((uint32_t)e, p.each) * per)] != 0) kept |= 1u << i;
        }
    }
    wave_sync();
    least = row_min<L>(least);
    most = row_max<L>(most);
    apart = most > none ? least - most : (F)INFINITY;
    return kept;
}

// ---- the largest numbers of a row ------------------------------------------------------------------------------------------------------
//
// A choice and its expert are one double: the choice, exactly, and in the bits that it leaves free the expert, so that of equal ones the lower is larger.
// Lists of the K largest, in order, are merged lane by lane: the larger of each number and its counterpart from the list's other end are the K
// largest of both, first up and then down, and a few exchanges order them.
constexpr double kNoChoice = -0x1p1000;                    // (what is below it is none)
// Five to eight choices come of lists where compute units have several waves to a vector unit, others one after another.  Of 256 experts, six choices and eight:
// 16384 tokens 19.5 and 19.6 us with lists of eight, 19.9 and 22.0 one after another (lists of four: four choices 18.1 for 19.0, one 18.2 for 16.7).  Eight choices
// with biases and groups: 64 tokens 13.6 and 16.4, but 32 tokens, eight waves, 12.6 and 11.7, 16 tokens 12.2 and 10.3: a wave alone waits for
// the longer way's instructions.
constexpr int kListed = 8;

__device__ __forceinline__ double choice_of(float key, int e)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, (double)(key + 0.f));               // (0 for -0)
    // infinities become 2^1023 and -2^1023: the positive numbers end there as signed integers, the negative ones as unsigned
    const uint32_t high = min((uint32_t)min((int)(bits >> 32), 0x7fe00000), 0xffe00000u), low = (uint32_t)bits | (uint32_t)(key < 0.f ? e : 1023 - e);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}

__device__ __forceinline__ int expert_of(double v)
{
    const int low = (int)(__builtin_bit_cast(uint64_t, v) & 1023);
    return v < kNoChoice ? -1 : v < 0 ? low : 1023 - low;
}

__device__ __forceinline__ void exchange(double &a, double &b)
{
    const double lo = smaller(a, b);
    a = larger(a, b);
    b = lo;
}

// Descending, of a list that goes up and then down (or the other way).
template <int K>
__device__ __forceinline__ void order_merged(double (&v)[K])
{
#pragma unroll
    for (int d = K / 2; d; d /= 2)
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (!(i & d)) exchange(v[i], v[i | d]);
}

// Descending, N at a time; then the K largest of all V (V < K: behind them nothing).
template <int K, int V>
__device__ __forceinline__ void order_own(const double (&v)[V], double (&list)[K])
{
    constexpr int N = V < K ? V : K;
#pragma unroll
    for (int at = 0; at < V; at += N) {
        double part[N];
#pragma unroll
        for (int i = 0; i < N; ++i) part[i] = v[at + i];
#pragma unroll
        for (int size = 2; size <= N; size *= 2)
#pragma unroll
            for (int d = size / 2; d; d /= 2)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (!(i & d)) {
                        if (i & size) exchange(part[i | d], part[i]);
                        else exchange(part[i], part[i | d]);
                    }
        if (at == 0) {
#pragma unroll
            for (int i = 0; i < K; ++i) list[i] = i < N ? part[i < N ? i : 0] : 2 * kNoChoice;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) list[i] = larger(list[i], part[N - 1 - i]);
            order_merged(list);
        }
    }
}

template <int CTRL>
__device__ __forceinline__ double moved(double v)
{
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CTRL, 0xf, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

template <int K, typename F>
__device__ __forceinline__ void merge_with(double (&v)[K], F other)
{
    double o[K];
#pragma unroll
    for (int i = 0; i < K; ++i) o[i] = other(v[i]);
#pragma unroll
    for (int i = 0; i < K; ++i) v[i] = larger(v[i], o[K - 1 - i]);
    order_merged(v);
}

// The row's K largest, the same in all of its lanes.
template <int L, int K, int V>
__device__ __forceinline__ void row_largest(const float (&key)[V], int e0, double (&list)[K])
{
    double own[V];
#pragma unroll
    for (int i = 0; i < V; ++i) own[i] = choice_of(key[i], e0 + i);
    order_own<K, V>(own, list);
    merge_with(list, [](double v) { return moved<0xb1>(v); });         // the lane beside; the other pair of four; the other four of eight; the other eight
    merge_with(list, [](double v) { return moved<0x4e>(v); });
    merge_with(list, [](double v) { return moved<0x141>(v); });
    merge_with(list, [](double v) { return moved<0x140>(v); });
    if constexpr (L >= 32) merge_with(list, [](double v) { return __shfl_xor(v, 16); });
    if constexpr (L == 64) merge_with(list, [](double v) { return __shfl_xor(v, 32); });
}

// Lane j's choice of the row's top_k <= K, the last of them, and whether two of them are so near that their order isn't sure.
template <int L, int K, int V>
__device__ __forceinline__ int choose_largest(const RouteParams &p, const float (&key)[V], float near, int sub, float &end, bool &sure)
{
    double list[K];
    row_largest<L, K, V>(key, sub * V, list);
    double mine = 2 * kNoChoice;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        if (i == sub) mine = list[i];
        if (i == p.top_k - 1 && list[i] > kNoChoice) end = (float)list[i];
        if (i + 1 < K && i + 1 < p.top_k && list[i + 1 < K ? i + 1 : i] > kNoChoice)
            sure &= list[i] - list[i + 1 < K ? i + 1 : i] > (double)near + __builtin_fabs(list[i]) * 0x1p-22;
    }
    return sub < p.top_k ? expert_of(mine) : -1;
}

// The choices of a row: lane j of it gets the j-th expert, or -1.
//
// Logits that are compared themselves are exact.  Scores in fp32 are not, and where two are nearer than what rounding can have moved them (`near`) they are
// computed again in 64 bits.  A sigmoid is off by 2^-22 (its exponential by (1.5 |x| + 2) 2^-24 of
// itself, which counts s (1 - s), the rest by 1.5 2^-23 s), a softmax by the roundings of its argument, sum and quotient, 2^-19 of the largest score
// of the row, which is 1 / sum; adding the bias rounds by 2^-24 of the choice; `near`, and what is added to it, is twice that of two of them.  In 64 bits go: the worths of the
// groups, where the last that is kept and the first that is not are near; the choices of the few experts, one to a lane, that are chosen or near the
// last chosen one; all of them, where those are more than a row has lanes.  There are such rows in every launch of thousands, and the launch ends with
// them, so they are short: 16384 tokens of 256 experts in eight groups took 5 us more where a near group had all its experts computed.
template <int L, int V>
__device__ __forceinline__ int choose(const RouteParams &p, const char *row, const float (&l)[V], const RowStats &st, int sub, char *lds)
{
    const float none = -INFINITY;
    const bool grouped = p.top_groups < p.groups, scored = p.bias || grouped;
    const int e0 = sub * V;
    float key[V], near = 0.f;
    uint32_t kept = ~0u;
    if (scored) {
        const float part = 1.f / st.sum;
        float bias[V];
#pragma unroll
        for (int i = 0; i < V; ++i) bias[i] = 0.f;
        if (p.bias) load_logits<4, V>((const char *)p.bias, e0, p.num, bias);
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = worth_of<float>(p, l[i], bias[i], st, part);
        near = (p.softmax ? 0x1.8p-17f * part : 0x1p-20f) + 0x1p-120f;
        if (grouped) {
            float apart, size = 0.f;
            float one = none, two = none;
#pragma unroll
            for (int i = 0; i < V; ++i) better_of(key[i], one, two);
            kept = kept_experts<float, L, V>(p, sub, (float *)lds, [&](int i) { return key[i]; }, [&](float &a, float &b) { a = one; b = two; }, apart);
#pragma unroll
            for (int i = 0; i < V; ++i) size = fmaxf(size, key[i] == none ? 0.f : __builtin_fabsf(key[i]));
            size = row_max<L>(size);
            if (__ballot(!(apart > 4.f * near + size * 0x1p-20f))) {
                const double sum = exact_sum<L, V>(p, row, e0, st);
                double exactly;
                // (a lane's two best are among those not below the second by more than `near`; where the second is infinite `from` is NaN and all are looked at)
                const float from = two == none ? none : two - (near + __builtin_fabsf(two) * 0x1p-22f);
                uint32_t few = 0;
#pragma unroll
                for (int i = 0; i < V; ++i) few |= key[i] != none && !(key[i] < from) ? 1u << i : 0u;
                kept = kept_experts<double, L, V>(
                    p, sub, (double *)lds, [&](int i) { return exact_worth(p, row, e0 + i, st, sum); },
                    [&](double &a, double &b) {
                        for (; few; few &= few - 1) {
                            better_of(exact_worth(p, row, e0 + __builtin_ctz(few), st, sum), a, b);
                        }
                    },
                    exactly);
            }
        }
    }
    if (!p.bias) {
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = st.lost || (scored && key[i] == none) ? none : l[i];
    }
    if (grouped) {
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = kept >> i & 1 ? key[i] : none;
    }
    int mine = -1;
    float end = none;                                      // the last chosen one
    bool sure = true;
    uint32_t few = 0;                                      // this lane's experts that are chosen or near the last chosen one
    if (p.listed) {
        mine = choose_largest<L, kListed, V>(p, key, near, sub, end, sure);
    } else {
        float last = INFINITY;                             // the pick before
        for (int picks = 0; picks < p.top_k; ++picks) {
            float best = key[0];
#pragma unroll
            for (int i = 1; i < V; ++i) best = larger(best, key[i]);
            const float top = row_max<L>(best);
            const bool is = top > none;
            if (!__ballot(is)) break;
            if (is && picks > 0 && !(last - top > near + __builtin_fabsf(last) * 0x1p-22f)) sure = false;
            last = top;
            if (picks == p.top_k - 1) end = top;
            int at = 0x7fffffff;
#pragma unroll
            for (int i = V - 1; i >= 0; --i) at = key[i] == top ? e0 + i : at;
            at = row_min<L>(is ? at : 0x7fffffff);
            if (sub == picks && is) mine = at;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (e0 + i == at) key[i] = none;
            }
            if (p.bias && at >= e0 && at < e0 + V) few |= 1u << (at - e0);
        }
    }
    if (!p.bias) return mine;
    const float from = end - (near + __builtin_fabsf(end) * 0x1p-22f);
#pragma unroll
    for (int i = 0; i < V; ++i) few |= key[i] != none && !(key[i] < from) ? 1u << i : 0u;
    const int own = __popc(few), count = row_sum<L>(own);
    if (__ballot(!sure || count > p.top_k)) {
        const double sum = exact_sum<L, V>(p, row, e0, st), out = -INFINITY;
        if (!__ballot(count > L)) {
            // the candidates' places, a candidate to a lane
            int *slot = (int *)lds, *chosen = slot + 3 * L;
            double *worth = (double *)(slot + L);
            slot[sub] = chosen[sub] = -1;
            wave_sync();
            for (int at = row_scan<L>(own) - own; few; few &= few - 1) slot[at++] = e0 + __builtin_ctz(few);
            wave_sync();
            const int e = slot[sub];
            const double v = e >= 0 ? exact_worth(p, row, e, st, sum) : out;
            worth[sub] = v;
            wave_sync();
            int place = 0;
            for (int o = 0; o < count; o += 8)
#pragma unroll
                for (int q = 0; q < 8; ++q) place += worth[o + q] > v || (worth[o + q] == v && slot[o + q] < e);
            if (e >= 0) chosen[place] = e;
            wave_sync();
            mine = chosen[sub];
        } else {
            // everything, in the row's LDS
            double *worth = (double *)lds;
#pragma unroll 2
            for (int i = 0; i < V; ++i) worth[i * L + sub] = kept >> i & 1 ? exact_worth(p, row, e0 + i, st, sum) : out;
            mine = -1;
            for (int j = 0; j < p.top_k; ++j) {
                double best = out;
                int at = 0x7fffffff, slot = 0;
                for (int i = 0; i < V; ++i) {
                    const double v = worth[i * L + sub];
                    if (v > best) { best = v; at = e0 + i; slot = i; }
                }
                const double top = row_max<L>(best);
                const int first = row_min<L>(best == top && top > out ? at : 0x7fffffff);
                if (sub == j && top > out) mine = first;
                if (at == first) worth[slot * L + sub] = out;              // (a lane without any: at = first = none, and its first number is -inf already)
            }
        }
    }
    return sub < p.top_k ? mine : -1;
}

// The sum of v over the threads before this one of the workgroup (`part`: one number for each wave).
__device__ __forceinline__ int before_thread(int v, int (&part)[kRouteWaves])
{
    const int upto = row_scan<64>(v), wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 63) part[wave] = upto;
    __syncthreads();
    int before = upto - v;
#pragma unroll
    for (int i = 0; i < kRouteWaves; ++i) before += i < wave ? part[i] : 0;
    return before;
}

// Bytes of LDS: the workgroup's choices and a row of counts for each wave, over the rows' group worths.
__host__ __device__ constexpr int route_slots(int L) { return kRouteThreads / L * (L == 16 ? 16 : ALT_ROUTE_MAX_TOP_K); }
template <int L> constexpr int kRowsOf = kRouteThreads / L;
__host__ __device__ constexpr int route_row_bytes(int experts) { return (experts + experts / 32) * 8; }
inline size_t route_lds(int L, int V, int num, bool scored)
{
    const size_t rank = (size_t)route_slots(L) * 2 + (size_t)kRouteWaves * num * 2, worth = scored ? (size_t)(kRouteThreads / L) * route_row_bytes(L * V) : 0;
    return (std::max(rank, worth) + 15) / 16 * 16;
}

// L lanes to a row, V experts to a lane.
template <int ES, int L, int V>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(const RouteParams p)
{
    extern __shared__ char route_smem[];
    __shared__ int part[kRouteWaves];
    constexpr int ROWS = kRowsOf<L>;
    const int t = threadIdx.x, sub = t % L, row_in = t / L, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64);
    const int64_t first = (int64_t)blockIdx.x * ROWS, token = first + row_in;
    const bool here = token < p.tokens;
    float l[V];
    if (here) {
        load_logits<ES, V>(p.logits + token * p.ld, sub * V, p.num, l);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = -INFINITY;
    }
    RowStats st;
    st.top = -INFINITY;
    int lost = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        lost |= l[i] != l[i];
        st.top = l[i] > st.top ? l[i] : st.top;
    }
    if (p.softmax) {
        st.top = row_max<L>(st.top);
        lost |= st.top == INFINITY;
    }
    st.lost = row_max<L>(lost) != 0;
    st.sum = 1.f;
    if (p.softmax && (!p.renorm || p.bias || p.top_groups < p.groups)) {
        st.sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) st.sum += l[i] == -INFINITY ? 0.f : expf(l[i] - st.top);
        st.sum = row_sum<L>(st.sum);
    }
    const int mine = choose<L, V>(p, p.logits + (here ? token : 0) * p.ld, l, st, sub, route_smem + (size_t)row_in * route_row_bytes(L * V));
    // weights, a choice to a lane
    if (here) {
        const bool is = mine >= 0;
        const float v = is ? element<ES>(p.logits + token * p.ld + (int64_t)mine * ES) : -INFINITY;
        float w;
        if (p.softmax) {
            // (renormalized: of the chosen ones alone, by the largest of them, which keeps what would be lost beside a larger one that was not chosen)
            const float top = p.renorm ? row_max<L>(v) : st.top;
            w = is ? expf(v - top) : 0.f;
            w = w / (p.renorm ? row_sum<L>(w) : st.sum);
        } else {
            w = is ? sigmoid_of(v) : 0.f;
            if (p.renorm) w = sigmoid_share<L>(w, v, is);
        }
        if (sub < p.top_k) {
            p.experts[token * p.top_k + sub] = mine;
            p.weights[token * p.top_k + sub] = st.lost ? __builtin_nanf("") : is ? w * p.scale : 0.f;
        }
    }
    // the choices of the workgroup's tokens, a choice to a thread: its place among those of its expert
    __syncthreads();                                       // (the group worths are read)
    int16_t *slot = (int16_t *)route_smem;
    uint16_t *count = (uint16_t *)(slot + route_slots(L));
    const int n = (int)min((int64_t)ROWS, p.tokens - first) * p.top_k, waves = (n + 63) / 64;
    if (sub < p.top_k && here) slot[row_in * p.top_k + sub] = (int16_t)mine;
    for (int i = t; i < waves * p.num; i += kRouteThreads) count[i] = 0;
    __syncthreads();
    const int e = t < n ? slot[t] : -1;
    int rank = 0;
    if (wave < waves) {
        uint64_t same = __ballot(e >= 0);
        for (int b = 1; b < p.num; b *= 2) {
            const uint64_t has = __ballot((e & b) != 0);
            same &= (e & b) ? has : ~has;
        }
        rank = __popcll(same & ((1ull << lane) - 1));
        if (e >= 0 && rank == 0) count[wave * p.num + e] = (uint16_t)__popcll(same);
    }
    __syncthreads();
    int all = 0;
    if (t < p.num)
        for (int w = 0; w < waves; ++w) {
            const int c = count[w * p.num + t];
            count[w * p.num + t] = (uint16_t)all;
            all += c;
        }
    int begin = 0;
    if (p.chunks == 1) {                                   // (the only workgroup)
        begin = before_thread(all, part);
        if (t < p.num) p.offsets[t] = begin;
        if (t == p.num - 1) p.offsets[p.num] = begin + all;
        __syncthreads();
        if (t < p.num)
            for (int w = 0; w < waves; ++w) count[w * p.num + t] += (uint16_t)begin;
    } else if (t < p.num) {
        p.counts[(int64_t)blockIdx.x * p.num + t] = (uint16_t)all;
    }
    __syncthreads();
    if (t < n) p.rows[first * p.top_k + t] = e >= 0 ? count[wave * p.num + e] + rank : -1;
}

// What the workgroups before have of each expert, and behind them what all have.  16 experts to a workgroup, 64 threads to an expert, each with a run of the
// workgroups.
__global__ __launch_bounds__(kRouteThreads) void route_scan_kernel(const RouteParams p)
{
    __shared__ int part[64][17];
    const int x = threadIdx.x % 16, run = threadIdx.x / 16, e = blockIdx.x * 16 + x, per = (p.chunks + 63) / 64, lo = run * per, hi = min(lo + per, p.chunks);
    int sum = 0;
    if (e < p.num) {
#pragma unroll 8
        for (int c = lo; c < hi; ++c) sum += p.counts[(int64_t)c * p.num + e];
    }
    part[run][x] = sum;
    __syncthreads();
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;            // a wave for each of the 16 experts
    const int upto = row_scan<64>(part[lane][wave]);
    __syncthreads();
    part[lane][wave] = upto;
    __syncthreads();
    int before = part[run][x] - sum;
    if (e >= p.num) return;
    if (run == 63) p.before[(int64_t)p.chunks * p.num + e] = before + sum;
#pragma unroll 8
    for (int c = lo; c < hi; ++c) {
        p.before[(int64_t)c * p.num + e] = before;
        before += p.counts[(int64_t)c * p.num + e];
    }
}

// Moves the ranks of a workgroup's choices to their rows.  COUNT: every workgroup adds up what those before it have, and all, itself.
template <int L, bool COUNT>
__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(const RouteParams p)
{
    __shared__ int part[kRouteWaves], base[kRouteThreads];
    const int t = threadIdx.x;
    const int64_t first = (int64_t)blockIdx.x * kRowsOf<L> * p.top_k, n = min((int64_t)kRowsOf<L> * p.top_k, (int64_t)p.tokens * p.top_k - first);
    static_assert(kRowsOf<L> * (L == 16 ? 16 : ALT_ROUTE_MAX_TOP_K) <= kRouteThreads, "a choice to a thread");
    const int e = t < n ? p.experts[first + t] : -1, rank = t < n ? p.rows[first + t] : 0;
    int all = 0, mine = 0;
    if constexpr (COUNT) {
        // a thread has an expert of every so many workgroups: lanes side by side have experts side by side
        __shared__ int sums[2][kRouteThreads];
        int width = 1;
        while (width < p.num) width *= 2;
        const int at = t & (width - 1), runs = kRouteThreads / width;
        int before = 0, total = 0;
        for (int c0 = t / width; c0 < p.chunks; c0 += 16 * runs) {
            int v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = p.counts[(int64_t)min(c0 + i * runs, p.chunks - 1) * p.num + min(at, p.num - 1)];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = c0 + i * runs;
                total += c < p.chunks ? v[i] : 0;
                before += c < (int)blockIdx.x ? v[i] : 0;
            }
        }
        for (int w = width; w < 64; w *= 2) {              // (the runs of a wave)
            total += __shfl_xor(total, w);
            before += __shfl_xor(before, w);
        }
        sums[0][t] = total;
        sums[1][t] = before;
        __syncthreads();
        if (t < p.num)
            for (int r = t; r < kRouteThreads; r += max(width, 64)) {
                all += sums[0][r];
                mine += sums[1][r];
            }
    } else if (t < p.num) {
        all = p.before[(int64_t)p.chunks * p.num + t];
        mine = p.before[(int64_t)blockIdx.x * p.num + t];
    }
    const int begin = before_thread(all, part);
    base[t] = begin + mine;
    if (blockIdx.x == 0) {
        if (t < p.num) p.offsets[t] = begin;
        if (t == p.num - 1) p.offsets[p.num] = begin + all;
    }
    __syncthreads();
    if (e >= 0) p.rows[first + t] = rank + base[e];
}

__global__ __launch_bounds__(kRouteThreads) void route_nothing_kernel(int32_t *offsets, int num)
{
    for (int i = threadIdx.x; i <= num; i += kRouteThreads) offsets[i] = 0;
}

// ---- the gradient ------------------------------------------------------------------------------------------------------------------

struct RouteGradParams {
    const char *logits;
    const int32_t *experts;
    const float *dweights;
    char *dlogits;
    int64_t ld;
    int32_t tokens, num, top_k, softmax, renorm;
    float scale;
};

constexpr int kGradThreads = 256;

// Four elements, at any alignment of whole elements.
template <int ES>
__device__ __forceinline__ void load_four(const char *at, float *f)
{
    if constexpr (ES == 4) {
        f4_t c;
        __builtin_memcpy(&c, at, 16);
#pragma unroll
        for (int q = 0; q < 4; ++q) f[q] = c[q];
    } else {
        uint32_t c[2];
        __builtin_memcpy(c, at, 8);
#pragma unroll
        for (int q = 0; q < 4; ++q) f[q] = __builtin_bit_cast(float, q % 2 ? c[q / 2] & 0xffff0000u : c[q / 2] << 16);
    }
}

template <int ES>
__device__ __forceinline__ void store_four(char *at, const float *f)
{
    if constexpr (ES == 4) {
        const f4_t c = {f[0], f[1], f[2], f[3]};
        __builtin_memcpy(at, &c, 16);
    } else {
        const uint32_t c[2] = {f32x2_to_bf16x2(f[0], f[1]), f32x2_to_bf16x2(f[2], f[3])};
        __builtin_memcpy(at, c, 8);
    }
}

// Bound by memory: it writes the row, and reads it where every expert's score has a part (softmax without renormalisation).  A lane has a choice, and
// then V experts, four side by side and the next four behind those of the other lanes (16384 x 256 fp32 7.0 us,
// where a lane has 16 side by side 11.4); the choices' gradients come to the experts' lanes through LDS.
template <int ES, int L, int V>
__global__ __launch_bounds__(kGradThreads) void route_grad_kernel(const RouteGradParams p)
{
    constexpr int ROWS = kGradThreads / L;
    __shared__ __attribute__((aligned(16))) float to[ROWS][L * V];
    __shared__ int chosen[ROWS][ALT_ROUTE_MAX_TOP_K];
    __shared__ float parts[ROWS][ALT_ROUTE_MAX_TOP_K];
    const int sub = threadIdx.x % L, row_in = threadIdx.x / L;
    auto first_of = [&](int i) { return (i * L + sub) * 4; };              // expert of the i-th four
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < p.tokens; first += (int64_t)gridDim.x * ROWS) {
        const int64_t token = first + row_in;
        const bool here = token < p.tokens;
        const char *row = p.logits + token * p.ld;
        float l[V], top = -INFINITY, sum = 1.f;
        const bool whole = p.softmax && !p.renorm;
        if (whole) {
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const int e0 = first_of(i);
                if (here && e0 + 4 <= p.num) {
                    load_four<ES>(row + (int64_t)e0 * ES, l + i * 4);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) l[i * 4 + q] = here && e0 + q < p.num ? element<ES>(row + (int64_t)(e0 + q) * ES) : -INFINITY;
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) top = l[i] > top ? l[i] : top;
            top = row_max<L>(top);
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                l[i] = l[i] == -INFINITY ? 0.f : expf(l[i] - top);
                sum += l[i];
            }
            sum = row_sum<L>(sum);
            sum = sum == 0.f ? 1.f : sum;
        }
        // a choice to a lane: its score (or share of the chosen scores) and dlogits = share * (dweight - mean) * rest
        int e = -1;
        float v = -INFINITY, dw = 0.f;
        if (here && sub < p.top_k) {
            e = p.experts[token * p.top_k + sub];
            if (e < 0 || e >= p.num) e = -1;
            if (e >= 0) {
                v = element<ES>(row + (int64_t)e * ES);
                dw = p.dweights[token * p.top_k + sub] * p.scale;
            }
        }
        const bool is = e >= 0 && v != -INFINITY;
        float s, rest = 1.f, mean = 0.f;
        if (p.softmax) {
            if (p.renorm) top = row_max<L>(v);
            s = is ? expf(v - top) : 0.f;
            if (p.renorm) {
                sum = row_sum<L>(s);
                sum = sum == 0.f ? 1.f : sum;
            }
            s /= sum;
        } else {
            s = is ? sigmoid_of(v) : 0.f;
            rest = is ? sigmoid_of(-v) : 0.f;
            if (p.renorm) s = sigmoid_share<L>(s, v, is);
        }
        if (p.renorm || p.softmax) mean = row_sum<L>(s * dw);
        const bool any = row_max<L>(e) >= 0;
        const float share = mean / sum;                    // (of an expert's exponential, where the whole row has a part)
        // (softmax without renormalisation: every expert has - score * mean, the chosen ones score * dweight beside it)
        const float mine = whole ? s * dw : s * (dw - mean) * rest;
        if (sub < p.top_k) {
            chosen[row_in][sub] = e;
            parts[row_in][sub] = e >= 0 ? mine : 0.f;
        }
#pragma unroll
        for (int i = 0; i < V / 4; ++i) *(f4_t *)&to[row_in][first_of(i)] = (f4_t){0.f, 0.f, 0.f, 0.f};
        wave_sync();
        if (e >= 0) {
            float total = 0.f;                             // (an expert that stands twice: every one of its choices stores both parts)
            for (int j = 0; j < p.top_k; ++j) total += chosen[row_in][j] == e ? parts[row_in][j] : 0.f;
            to[row_in][e] = total;
        }
        wave_sync();
        if (here) {
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const int e0 = first_of(i);
                const f4_t part = *(const f4_t *)&to[row_in][e0];
                float out[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    out[q] = part[q];
                    if (whole) out[q] -= l[i * 4 + q] * share;
                    if (!any) out[q] = 0.f;
                }
                char *at = p.dlogits + token * p.ld + (int64_t)e0 * ES;
                if (e0 + 4 <= p.num) {
                    store_four<ES>(at, out);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (e0 + q < p.num) store_element<ES>(at + q * ES, out[q]);
                }
            }
        }
        wave_sync();
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------------------------

// Lanes of a row and experts of a lane: as few lanes as hold the experts, 16 to a lane, and the choices (16384 tokens of 512 experts,
// eight choices: 32 lanes 30 us, 64 lanes 44).
struct Shape { int l, v; };
Shape shape_of(const alt_route_desc_t &d)
{
    if (d.top_k <= 16 && d.experts <= 256) return {16, d.experts <= 64 ? 4 : d.experts <= 128 ? 8 : 16};
    if (d.experts <= 512) return {32, d.experts <= 256 ? 8 : 16};
    return {64, 16};
}

template <typename F>
void by_shape(const alt_route_desc_t &d, F f)
{
    using std::integral_constant;
    const Shape s = shape_of(d);
    if (s.l == 16) {
        if (s.v == 4) f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
        else if (s.v == 8) f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
        else f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    } else {
        if (s.l == 64) f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
        else if (s.v == 8) f(integral_constant<int, 32>{}, integral_constant<int, 8>{});
        else f(integral_constant<int, 32>{}, integral_constant<int, 16>{});
    }
}

// Up to so many counts every workgroup reads them all, beyond them they have a launch of their own: 16384 tokens of 64 experts, two choices (16384 counts),
// 9.7 us the one way and 11.7 the other; 16384 of 256, eight choices (65536) 25.2 and 23.2, 32768 of 256 (131072) 44 and 25.
constexpr int64_t kCountsEach = 16384;
bool counts_each(int64_t chunks, int num) { return chunks * num <= kCountsEach; }

int64_t chunks_of(const alt_route_desc_t &d) { return (d.tokens + kRouteThreads / shape_of(d).l - 1) / (kRouteThreads / shape_of(d).l); }

template <int ES>
hipError_t route_run(const alt_route_desc_t &d, const RouteParams &p, hipStream_t st)
{
    hipError_t e = hipSuccess;
    by_shape(d, [&](auto l, auto v) {
        constexpr int L = decltype(l)::value, V = decltype(v)::value;
        const size_t lds = route_lds(L, V, p.num, p.bias || p.top_groups < p.groups);
        if (lds > 64 * 1024) {
            static OncePerDevice lds_once;
            e = allow_lds(lds_once, (const void *)route_kernel<ES, L, V>, 160 * 1024 - 256);
            if (e != hipSuccess) return;
        }
        hipLaunchKernelGGL((route_kernel<ES, L, V>), dim3((unsigned)p.chunks), dim3(kRouteThreads), lds, st, p);
        if ((e = hipGetLastError()) != hipSuccess || p.chunks == 1) return;
        if (counts_each(p.chunks, p.num)) {
            hipLaunchKernelGGL((route_place_kernel<L, true>), dim3((unsigned)p.chunks), dim3(kRouteThreads), 0, st, p);
        } else {
            hipLaunchKernelGGL(route_scan_kernel, dim3((unsigned)((p.num + 15) / 16)), dim3(kRouteThreads), 0, st, p);
            hipLaunchKernelGGL((route_place_kernel<L, false>), dim3((unsigned)p.chunks), dim3(kRouteThreads), 0, st, p);
        }
        e = hipGetLastError();
    });
    return e;
}

template <int ES>
void route_grad_run(const alt_route_desc_t &d, const RouteGradParams &p, hipStream_t st)
{
    by_shape(d, [&](auto l, auto v) {
        constexpr int L = decltype(l)::value, ROWS = kGradThreads / L;
        const int64_t blocks = ((int64_t)p.tokens + ROWS - 1) / ROWS;
        hipLaunchKernelGGL((route_grad_kernel<ES, L, decltype(v)::value>), dim3((unsigned)std::min<int64_t>(blocks, 1 << 20)), dim3(kGradThreads), 0, st, p);
    });
}

alt_status_t check(alt_handle_t h, const char *call, const alt_route_desc_t *d, alt_route_desc_t *out)
{
    if (!h) return ALT_INVALID_ARG;
    if (!d) return fail(h, ALT_INVALID_ARG, "%s: null descriptor", call);
    *out = *d;
    if (d->tokens < 0 || d->stride < 0 || d->experts < 1 || d->top_k < 1) return fail(h, ALT_INVALID_ARG, "%s: bad size", call);
    if (d->dtype != ALT_F32 && d->dtype != ALT_BF16) return fail(h, ALT_INVALID_ARG, "%s: bad dtype", call);
    if (d->score != ALT_SCORE_SOFTMAX && d->score != ALT_SCORE_SIGMOID) return fail(h, ALT_INVALID_ARG, "%s: bad score", call);
    if (d->renormalize != 0 && d->renormalize != 1) return fail(h, ALT_INVALID_ARG, "%s: renormalize is 0 or 1", call);
    if (d->groups < 1 || d->top_groups < 1 || d->top_groups > d->groups || d->group_best < 1 || d->group_best > 2)
        return fail(h, ALT_INVALID_ARG, "%s: bad groups, top_groups or group_best", call);
    if (!(__builtin_fabsf(d->scale) <= 3.4e38f)) return fail(h, ALT_INVALID_ARG, "%s: scale is not finite", call);
    if (!out->stride) out->stride = d->experts;
    if (out->stride < d->experts) return fail(h, ALT_SHAPE_MISMATCH, "%s: a row stride is shorter than a row", call);
    if (d->experts % d->groups) return fail(h, ALT_SHAPE_MISMATCH, "%s: %d experts make no %d groups", call, d->experts, d->groups);
    if (d->top_k > (int64_t)d->top_groups * (d->experts / d->groups)) return fail(h, ALT_SHAPE_MISMATCH, "%s: top_k is more than the experts that a token chooses from", call);
    if (d->experts > ALT_ROUTE_MAX_EXPERTS || d->top_k > ALT_ROUTE_MAX_TOP_K) return fail(h, ALT_UNSUPPORTED, "%s: more than 1024 experts or 32 choices", call);
    if (d->tokens > (1 << 25) || out->stride > 0x7fffffff) return fail(h, ALT_UNSUPPORTED, "%s: more than 2^25 tokens or a stride over 2^31", call);
    return ALT_OK;
}

// The workspace: what each workgroup counts, and, where that has a launch of its own, what those before have.
size_t counts_bytes(const alt_route_desc_t &d) { return ((size_t)chunks_of(d) * d.experts * 2 + 15) / 16 * 16; }
size_t route_workspace(const alt_route_desc_t &d)
{
    return counts_bytes(d) + (counts_each(chunks_of(d), d.experts) ? 0 : (size_t)(chunks_of(d) + 1) * d.experts * 4) + 16;
}

}  // namespace
}  // namespace alt

using namespace alt;

extern "C" alt_status_t alt_route(alt_handle_t h, const alt_route_desc_t *desc, const void *logits, const float *bias, int32_t *experts, float *weights, int32_t *rows,
                                  int32_t *offsets, void *workspace, size_t ws_bytes, void *stream)
{
    alt_route_desc_t d;
    alt_status_t s = check(h, "alt_route", desc, &d);
    if (s != ALT_OK) return s;
    const bool some = d.tokens > 0;
    s = check_buffers(h, "alt_route", {{"logits", logits, dtype_size(d.dtype), some}, {"bias", bias, 4, bias != nullptr}, {"experts", experts, 4, some}, {"weights", weights, 4, some},
                                       {"rows", rows, 4, some}, {"offsets", offsets, 4}});
    if (s == ALT_OK) s = check_workspace(h, "alt_route", workspace, ws_bytes, route_workspace(d));
    if (s == ALT_OK) s = check_device(h, "alt_route");
    if (s != ALT_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    RouteParams p{};
    p.logits = (const char *)logits;
    p.bias = bias;
    p.experts = experts; p.weights = weights; p.rows = rows; p.offsets = offsets;
    p.counts = (uint16_t *)aligned_workspace(workspace);
    p.before = (int32_t *)(aligned_workspace(workspace) + counts_bytes(d));
    p.ld = d.stride * (int64_t)dtype_size(d.dtype);
    p.tokens = (int32_t)d.tokens;
    p.num = d.experts; p.top_k = d.top_k; p.groups = d.groups; p.top_groups = d.top_groups; p.group_best = d.group_best;
    p.softmax = d.score == ALT_SCORE_SOFTMAX;
    p.renorm = d.renormalize;
    p.scale = d.scale;
    p.chunks = (int32_t)chunks_of(d);
    p.size = (int32_t)dtype_size(d.dtype);
    p.listed = d.top_k > 4 && d.top_k <= kListed && d.tokens * shape_of(d).l > 512;
    p.each = make_fastdiv((uint32_t)(d.experts / d.groups));
    if (!some) {
        hipLaunchKernelGGL(route_nothing_kernel, dim3(1), dim3(kRouteThreads), 0, st, offsets, (int)d.experts);
        ALT_CHECK_HIP(h, hipGetLastError());
        return ALT_OK;
    }
    ALT_CHECK_HIP(h, d.dtype == ALT_F32 ? route_run<4>(d, p, st) : route_run<2>(d, p, st));
    return ALT_OK;
}

extern "C" alt_status_t alt_route_workspace_size(alt_handle_t h, const alt_route_desc_t *desc, size_t *bytes)
{
    alt_route_desc_t d;
    const alt_status_t s = check(h, "alt_route_workspace_size", desc, &d);
    if (s != ALT_OK) return s;
    if (!bytes) return fail(h, ALT_INVALID_ARG, "alt_route_workspace_size: null result");
    *bytes = route_workspace(d);
    return ALT_OK;
}

extern "C" alt_status_t alt_route_grad(alt_handle_t h, const alt_route_desc_t *desc, const void *logits, const int32_t *experts, const float *dweights, void *dlogits, void *stream)
{
    alt_route_desc_t d;
    alt_status_t s = check(h, "alt_route_grad", desc, &d);
    if (s != ALT_OK) return s;
    if (d.tokens == 0) return ALT_OK;
    s = check_buffers(h, "alt_route_grad", {{"logits", logits, dtype_size(d.dtype)}, {"experts", experts, 4}, {"dweights", dweights, 4}, {"dlogits", dlogits, dtype_size(d.dtype)}});
    if (s == ALT_OK) s = check_device(h, "alt_route_grad");
    if (s != ALT_OK) return s;
    const hipStream_t st = (hipStream_t)stream;
    RouteGradParams p{(const char *)logits, experts, dweights, (char *)dlogits, d.stride * (int64_t)dtype_size(d.dtype), (int32_t)d.tokens, d.experts, d.top_k, d.score == ALT_SCORE_SOFTMAX,
                      d.renormalize, d.scale};
    if (d.dtype == ALT_F32) route_grad_run<4>(d, p, st);
    else route_grad_run<2>(d, p, st);
    ALT_CHECK_HIP(h, hipGetLastError());
    return ALT_OK;
}
