// What stands around the products of routed rows: the choice of k experts for every row with its weights and their gradient, the grouping
// of the chosen (row, place) pairs by expert, and the weighted sum of a row's results with its gradients.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cstdint>

#include "route.h"
#include "vbr_device.h"

namespace vbrk {
namespace {

constexpr int kRouteThreads = 256;     // 4 waves
constexpr int64_t kNarrowRows = 2048;  // rows from which on 16 lanes have one

template <int TY>
__device__ __forceinline__ float load_as_f32(const void *p, int64_t i)
{
    if constexpr (TY == VBR_F32) return static_cast<const float *>(p)[i];
    else if constexpr (TY == VBR_F16) return (float)static_cast<const _Float16 *>(p)[i];
    else return (float)static_cast<const __bf16 *>(p)[i];
}

template <int TY>
__device__ __forceinline__ void store_f32(void *p, int64_t i, float v)          // rounded to nearest, ties to even: the one rounding of a result
{
    if constexpr (TY == VBR_F32) static_cast<float *>(p)[i] = v;
    else if constexpr (TY == VBR_F16) static_cast<_Float16 *>(p)[i] = (_Float16)v;
    else static_cast<__bf16 *>(p)[i] = (__bf16)v;
}

// LP lanes have a row: all of them get the result.  16 lanes are one row of the vector unit.
template <int CTRL>
__device__ __forceinline__ uint32_t from_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true); }

template <int LP, class Op>
__device__ __forceinline__ uint32_t over_lanes(uint32_t x, Op op)
{
    x = op(x, from_lane<0xB1>(x));
    x = op(x, from_lane<0x4E>(x));
    x = op(x, from_lane<0x141>(x));
    x = op(x, from_lane<0x140>(x));
    if constexpr (LP == 64) {
        const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = op((uint32_t)a[0], (uint32_t)a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = op((uint32_t)b[0], (uint32_t)b[1]);
    }
    return x;
}
__device__ __forceinline__ uint32_t bits(float x) { return __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ float number(uint32_t x) { return __builtin_bit_cast(float, x); }
template <int LP>
__device__ __forceinline__ float row_max(float x) { return number(over_lanes<LP>(bits(x), [](uint32_t a, uint32_t b) { return bits(fmaxf(number(a), number(b))); })); }
template <int LP>
__device__ __forceinline__ float row_sum(float x) { return number(over_lanes<LP>(bits(x), [](uint32_t a, uint32_t b) { return bits(number(a) + number(b)); })); }
template <int LP>
__device__ __forceinline__ int row_min(int x) { return (int)over_lanes<LP>((uint32_t)x, [](uint32_t a, uint32_t b) { return a < b ? a : b; }); }     // none is negative
// over the whole wave, in 64 bits
template <int CTRL>
__device__ __forceinline__ double from_lane(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)from_lane<CTRL>((uint32_t)(b >> 32)) << 32 | from_lane<CTRL>((uint32_t)b));
}
__device__ __forceinline__ double wave_max(double x)
{
    x = fmax(x, from_lane<0xB1>(x));
    x = fmax(x, from_lane<0x4E>(x));
    x = fmax(x, from_lane<0x141>(x));
    x = fmax(x, from_lane<0x140>(x));
    auto swap = [&](auto f) {
        const uint64_t b = __builtin_bit_cast(uint64_t, x);
        const auto hi = f((uint32_t)(b >> 32)), lo = f((uint32_t)b);
        return fmax(__builtin_bit_cast(double, (uint64_t)(uint32_t)hi[0] << 32 | (uint32_t)lo[0]), __builtin_bit_cast(double, (uint64_t)(uint32_t)hi[1] << 32 | (uint32_t)lo[1]));
    };
    x = swap([](uint32_t h) { return __builtin_amdgcn_permlane16_swap(h, h, false, false); });
    return swap([](uint32_t h) { return __builtin_amdgcn_permlane32_swap(h, h, false, false); });
}
__device__ __forceinline__ double wave_sum(double x)
{
    for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
    return x;
}
__device__ __forceinline__ double of_lane(double x, int lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, lane));
}

// V consecutive experts of a row, the first of them e0; those that are not there are closed
template <int TY, int V>
__device__ __forceinline__ void load_row(const void *p, int64_t row, int e0, int n_experts, bool whole, float (&l)[V])
{
    constexpr int kBytes = V * (TY == VBR_F32 ? 4 : 2);
    if constexpr (kBytes >= 16) {
        if (whole) {
#pragma unroll
            for (int c = 0; c < kBytes / 16; ++c) {
                const uint4v w = reinterpret_cast<const uint4v *>(static_cast<const char *>(p) + (row + e0) * (TY == VBR_F32 ? 4 : 2))[c];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t x = w[j];
                    if constexpr (TY == VBR_F32) l[4 * c + j] = number(x);
                    else if constexpr (TY == VBR_BF16) { l[8 * c + 2 * j] = number(x << 16); l[8 * c + 2 * j + 1] = number(x & 0xFFFF0000u); }
                    else { l[8 * c + 2 * j] = (float)__builtin_bit_cast(_Float16, (uint16_t)x); l[8 * c + 2 * j + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(x >> 16)); }
                }
            }
            return;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = e0 + v < n_experts ? load_as_f32<TY>(p, row + e0 + v) : -INFINITY;
}

// A raw score as it counts: NaN closes the expert like -inf, +inf is the largest finite number.
__device__ __forceinline__ float raw_score(float l) { return l > -INFINITY ? fminf(l, FLT_MAX) : -INFINITY; }

struct TopkParams {
    const void *logits;
    const float *bias;
    int32_t *ids;
    float *weights;
    int64_t ld, n_rows;
    int32_t n_experts, top_k, n_groups, top_groups, group_size;
    int32_t lanes_a_group;                     // a power of two of whole lanes; 0: none
    uint32_t group_factor;                     // expert e is of group e group_factor >> 20
    int32_t sigmoid, renormalise, scored;      // scored: the keys are scores with their biases, not the raw scores
    int32_t whole, whole_bias;                 // rows are whole numbers of 16-byte pieces for each lane; the biases are
    float scale;
};

// Numbers as integers of the same order
__device__ __forceinline__ int ordered(float x)
{
    const int i = (int)bits(x + 0.f);                     // (-0 is 0)
    return i ^ (i >> 31 & INT_MAX);
}
__device__ __forceinline__ float of_ordered(int i) { return number((uint32_t)(i ^ (i >> 31 & INT_MAX))); }

template <int LP>
__device__ __forceinline__ int row_max_int(int x) { return (int)over_lanes<LP>((uint32_t)x, [](uint32_t a, uint32_t b) { return (uint32_t)((int)a > (int)b ? (int)a : (int)b); }); }
constexpr int kClosed = (int)0x807FFFFF;             // of -inf, and no number is as low

// The choice among the keys, V a lane of the wave, in 64 bits: lane j gets the j-th expert, -1 without one.  Of equal keys the lower index wins.
template <int V>
__device__ __forceinline__ int choose_exactly(const TopkParams &p, double (&key)[V], const float (&l)[V], double *lds, int sub)
{
    if (p.n_groups > p.top_groups) {
        double best = -INFINITY, second = -INFINITY;
        const int lanes = p.group_size / V;                // of a group, if a group is whole lanes, 1, 2, 4, 8 or 16 of them
        const bool by_lanes = lanes * V == p.group_size && lanes <= 16 && (lanes & (lanes - 1)) == 0;
        if (by_lanes) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                second = fmax(fmin(key[v], best), second);
                best = fmax(best, key[v]);
            }
            auto merge = [&](double b, double s) {
                second = fmax(fmin(best, b), fmax(second, s));
                best = fmax(best, b);
            };
            if (lanes >= 2) merge(from_lane<0xB1>(best), from_lane<0xB1>(second));
            if (lanes >= 4) merge(from_lane<0x4E>(best), from_lane<0x4E>(second));
            if (lanes >= 8) merge(from_lane<0x141>(best), from_lane<0x141>(second));
            if (lanes >= 16) merge(from_lane<0x140>(best), from_lane<0x140>(second));
        } else {
            // keys by way of LDS (one more place after every 16, or lanes meet in the same bank), a group a lane
#pragma unroll
            for (int v = 0; v < V; ++v) lds[(sub * V + v) + ((sub * V + v) >> 4)] = key[v];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (sub < p.n_groups) {
#pragma unroll 4
                for (int i = 0; i < p.group_size; ++i) {
                    const int e = sub * p.group_size + i;
                    const double x = lds[e + (e >> 4)];
                    second = fmax(fmin(x, best), second);
                    best = fmax(best, x);
                }
            }
        }
        const double mine = second > -INFINITY ? best + second : best;
        const int step = by_lanes ? lanes : 1;             // from a group's first lane to the next one's
        int ahead = 0;                                     // groups that come before this lane's
        for (int g = 0; g < p.n_groups; ++g) {
            const double other = of_lane(mine, g * step);
            ahead += (other > mine) | ((other == mine) & (g * step + step <= sub));
        }
        const bool stays = ahead < p.top_groups && mine > -INFINITY;
        if (by_lanes) {
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = stays ? key[v] : -INFINITY;
        } else {
            const uint64_t chosen = __ballot(stays);
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (sub * V + v < p.n_experts && !(chosen >> ((uint32_t)(sub * V + v) * p.group_factor >> 20) & 1)) key[v] = -INFINITY;
        }
    }
    // Rounded to 32 bits they keep their order, but for those that become equal: only these are compared in 64.
    int x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (p.bias == nullptr && key[v] > -INFINITY) key[v] = l[v];      // the same order, and exact
        x[v] = ordered((float)key[v]);
    }
    int my_id = -1;
    for (int j = 0; j < p.top_k; ++j) {
        int first = x[0];
#pragma unroll
        for (int v = 1; v < V; ++v) first = max(first, x[v]);
        const int most = row_max_int<64>(first);
        if (most <= kClosed) break;
        int n = 0, mine = 0;
        uint64_t lanes = 0;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) {
            const uint64_t have = __ballot(x[v] == most);
            n += __popcll(have);
            lanes |= have;
            mine = x[v] == most ? v : mine;
        }
        int at = __builtin_amdgcn_readlane(sub * V + mine, __builtin_ctzll(lanes));
        if (n > 1) {
            double top = -INFINITY;
#pragma unroll
            for (int v = V - 1; v >= 0; --v) {
                const bool as_high = x[v] == most && key[v] >= top;
                top = as_high ? key[v] : top;
                mine = as_high ? v : mine;
            }
            const double highest = wave_max(top);
            at = row_min<64>(first == most && top == highest ? sub * V + mine : INT_MAX);
        }
        if (sub == j) my_id = at;
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = at == sub * V + v ? kClosed : x[v];
    }
    return my_id;
}

// falling, by Batcher's odd-even merge sort: comparators that are known beforehand
template <int V>
__device__ __forceinline__ void sort_falling(int (&x)[V])
{
#pragma unroll
    for (int p = 1; p < V; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < V; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < V && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const int a = x[i + j], b = x[i + j + k];
                        x[i + j] = a > b ? a : b;
                        x[i + j + k] = a > b ? b : a;
                    }
}

// The same in 32 bits.  Keys are whole numbers in the order of the numbers, with an expert's place in its lane in the lowest bits, lower places first: a lane sorts
// its keys once, and a choice is the largest of the lanes' first ones.  The result says whether any difference that decides may be of the other sign.  A key is
// off by `bound` at most, and by kOff of its own size, and one without its lowest bits is lower by up to V steps: of two that differ the higher one is
// higher by at least the difference less what both are off by and V steps of the lower.  What a key can be at most rises with it, so that one further
// down than the next cannot come before the last chosen one if the next cannot.  Raw scores are what they are: those that differ without their lowest bits are in order.
// exact: the lowest bits were zero, and there is nothing to say.  Infinite keys (of biases) are all equal, and so are the sums of groups that have one; what an
// infinity is compared with is in doubt, but for another one in the order of their places.
constexpr float kOff = 0x1p-23f;
template <int LP, int V>
__device__ __forceinline__ bool choose(const TopkParams &p, const float (&key)[V], const float (&l)[V], float *lds, int sub, int &my_id, float bound, bool exact)
{
    bool unsure = false;              // (the same in every lane of the row)
    uint64_t chosen = ~0ull;          // groups
    bool stays = true;                // by lanes: this lane's is
    int x[V];
    auto pack = [&](const float (&from)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = (ordered(from[v]) & -V) | (V - 1 - v);
    };
    const bool by_raw = p.bias == nullptr;                // the same order, and exact
    const bool by_lanes = p.lanes_a_group && !by_raw;
    if (!by_raw) {
        pack(key);
        sort_falling(x);
    }
    if (p.n_groups > p.top_groups) {
        float mine, size, lower = 0.f;                    // half the sum of a group's two best keys (a sum may be beyond the type), of their sizes, and what it may be too low by
        int group = sub;
        if (by_lanes) {
            int best = x[0], second = V > 1 ? x[V > 1] : kClosed;
            auto merge = [&](int b, int s) {
                second = max(min(best, b), max(second, s));
                best = max(best, b);
            };
            if (p.lanes_a_group >= 2) merge((int)from_lane<0xB1>((uint32_t)best), (int)from_lane<0xB1>((uint32_t)second));
            if (p.lanes_a_group >= 4) merge((int)from_lane<0x4E>((uint32_t)best), (int)from_lane<0x4E>((uint32_t)second));
            if (p.lanes_a_group >= 8) merge((int)from_lane<0x141>((uint32_t)best), (int)from_lane<0x141>((uint32_t)second));
            const float a = best <= kClosed ? -INFINITY : 0.5f * of_ordered(best & -V), b = second <= kClosed ? 0.f : 0.5f * of_ordered(second & -V);
            mine = a + b;
            size = fabsf(a) + fabsf(b);
            lower = size * (V * 0x1p-23f);
            group = sub / p.lanes_a_group;
        } else {
            // by way of LDS (one more place after every 16, or lanes meet in the same bank), a group a lane
#pragma unroll
            for (int v = 0; v < V; ++v) lds[(sub * V + v) + ((sub * V + v) >> 4)] = key[v];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            float best = -INFINITY, second = -INFINITY;
            if (sub < p.n_groups) {
#pragma unroll 4
                for (int i = 0; i < p.group_size; ++i) {
                    const int e = sub * p.group_size + i;
                    const float y = lds[e + (e >> 4)];
                    second = fmaxf(fminf(y, best), second);
                    best = fmaxf(best, y);
                }
            }
            const float a = 0.5f * best, b = second > -INFINITY ? 0.5f * second : 0.f;
            mine = a + b;
            size = fabsf(a) + fabsf(b);
        }
        const float sum = mine, off = bound + 2 * kOff * size;               // (and rounded itself)
        if constexpr (LP == 16) {
            // By how many are before it; of equal ones that would be chosen together too many are, and the row is in doubt.
            int ahead = 0;
            static_for<15>([&](auto i) { ahead += number(from_lane<0x121 + i.value>(bits(mine))) > mine; });      // the other lanes, turned in the row
            const int wanted = p.top_groups * (by_lanes ? p.lanes_a_group : 1);
            stays = ahead < wanted && mine > -INFINITY;
            const uint32_t in = (uint32_t)(__ballot(stays) >> (threadIdx.x & 48)) & 0xFFFFu;
            unsure = __popc(in) > wanted;
            chosen = in;
        } else {
            chosen = 0;
            for (int i = 0; i < p.top_groups; ++i) {
                const float top = row_max<LP>(mine);
                const int at = row_min<LP>(mine == top && top > -INFINITY ? group : INT_MAX);
                if (at != INT_MAX) chosen |= 1ull << at;
                if (group == at) mine = -INFINITY;
            }
            stays = chosen >> group & 1;
        }
        // the least that one that stays can be, and the most that one that does not
        const float least = -row_max<LP>(stays ? off - sum : -INFINITY), most = row_max<LP>(!stays && sum > -INFINITY ? sum + off + lower : -INFINITY);
        unsure |= least <= most;
    }
    if (by_raw) {
        pack(l);
        if (p.n_groups > p.top_groups) {
#pragma unroll
            for (int v = 0; v < V; ++v) x[v] = chosen >> ((uint32_t)(sub * V + v) * p.group_factor >> 20) & 1 ? x[v] : kClosed;
        }
        sort_falling(x);
    } else if (by_lanes) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = stays ? x[v] : kClosed;
    } else if (p.n_groups > p.top_groups) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = chosen >> ((uint32_t)(sub * V + V - 1 - (x[v] & (V - 1))) * p.group_factor >> 20) & 1 ? x[v] : kClosed;
        sort_falling(x);
    }
    const float by = by_raw ? 0.f : 2 * bound, off = by_raw ? 0.f : kOff, lost = by_raw ? 0.f : kOff + V * 0x1p-23f;
    float before = INFINITY;
    for (int j = 0; j < p.top_k + (exact ? 0 : 1); ++j) {
        const int first = x[0] & -V, most = row_max_int<LP>(first), mine = sub * V + V - 1 - (x[0] & (V - 1));      // (places count among equal keys only)
        const int at = row_min<LP>(first == most && most > kClosed ? mine : INT_MAX);
        if (!exact) {
            const float now = of_ordered(most);
            unsure |= j > 0 && most > kClosed && before - now <= by + fabsf(before) * off + fabsf(now) * lost;
            before = now;
        }
        if (j < p.top_k && sub == j) my_id = at == INT_MAX ? -1 : at;
        const bool taken = at == mine;
#pragma unroll
        for (int v = 0; v + 1 < V; ++v) x[v] = taken ? x[v + 1] : x[v];
        x[V - 1] = taken ? kClosed : x[V - 1];
    }
    return unsure;
}

// The choice for one row in 64 bits, by a whole wave: lane j has the j-th expert.
template <int TY, int V>
__device__ __forceinline__ int choose_row_exactly(const TopkParams &p, int64_t row, int lane, double *lds)
{
    float l[V], bias[V], top = -INFINITY;
    load_row<TY, V>(p.logits, row * p.ld, lane * V, p.n_experts, false, l);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        l[v] = raw_score(l[v]);
        top = fmaxf(top, l[v]);
        bias[v] = p.bias && lane * V + v < p.n_experts ? p.bias[lane * V + v] : 0.f;
    }
    double key[V];
    if (p.scored) {
        const double most = fmaxf(row_max<64>(top), -FLT_MAX);
        double total = 0;
        // (without branches, so that the exponentials of several experts are on their way at once)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const double x = fmaxf(l[v], -FLT_MAX);
            key[v] = exp(p.sigmoid ? -x : x - most);
            total += l[v] > -INFINITY ? key[v] : 0.0;
        }
        if (!p.sigmoid) total = wave_sum(total);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            key[v] = (p.sigmoid ? 1.0 / (1.0 + key[v]) : key[v] / total) + (double)bias[v];
            if (!(l[v] > -INFINITY) || !(key[v] > -INFINITY)) key[v] = -INFINITY;
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = l[v];
    }
    return choose_exactly<V>(p, key, l, lds, lane);
}

// LP lanes a row, V experts a lane.  What decides between sums of scores and biases are differences that 32 bits may not tell: they are made in 32 bits, with a
// bound for what they are off by, and where a difference is within it, in 64 bits.  Raw scores are compared as they are: the score rises with them.
// 16384 rows, 8 of 256 in 4 of 8 groups, take 14.7 us: 8.2 are the issue of 1225 vector instructions for four rows, most of them the sorting of a lane's keys and the
// choice itself, 2.5 the launch, and the rows in doubt end about 4 after the others; 8192 rows, 8 of 128 by raw scores, 4.5.
template <int TY, int LP, int V>
__global__ void __launch_bounds__(kRouteThreads) route_topk_kernel(const TopkParams p)
{
    constexpr int kRows = kRouteThreads / LP;
    constexpr int kEachOf64 = LP * V < 64 ? 1 : LP * V / 64, kRowLds = LP * V + LP * V / 16, kWaveLds = std::max(64 / LP * kRowLds * 4, 64 * kEachOf64 * 17 / 16 * 8);
    __shared__ __attribute__((aligned(16))) char all_lds[kRouteThreads / 64][kWaveLds];
    char *lds = all_lds[threadIdx.x >> 6];
    const int sub = threadIdx.x % LP, in_wg = threadIdx.x / LP;
    float *row_lds = reinterpret_cast<float *>(lds) + in_wg % (64 / LP) * kRowLds;
    const int64_t wanted = (int64_t)blockIdx.x * kRows + in_wg, row = wanted < p.n_rows ? wanted : p.n_rows - 1;
    float l[V], key[V];
    load_row<TY, V>(p.logits, row * p.ld, sub * V, p.n_experts, p.whole && (sub + 1) * V <= p.n_experts, l);
    float top = -INFINITY, total = 1.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        l[v] = raw_score(l[v]);
        top = fmaxf(top, l[v]);
    }
    const bool softmax_sum = !p.sigmoid && (p.scored || !p.renormalise);
    if (softmax_sum) {
        top = row_max<LP>(top);
        total = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) total += exp_of(l[v] - top);                 // (0 of one that is closed)
        total = row_sum<LP>(total);
    }
    int my_id = -1;
    bool unsure;
    if (p.scored) {
        float bias[V];
        if (p.bias) {
            load_row<VBR_F32, V>(p.bias, 0, sub * V, p.n_experts, p.whole_bias && (sub + 1) * V <= p.n_experts, bias);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) bias[v] = 0.f;
        }
        const float one_of_total = 1.f / total;
        if (p.sigmoid) {
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = sigmoid_of(l[v]);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = exp_of(l[v] - top) * one_of_total;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float s = l[v] > -INFINITY ? key[v] + bias[v] : -INFINITY;
            key[v] = s > -INFINITY ? s : -INFINITY;                        // (NaN closes)
        }
        // A sigmoid is off by 8 half steps at 1 at most (exponential, sum, reciprocal, product), a softmax by those of the largest one, 1 / total, and what
        // V + 6 additions in a row leave in its sum; the sum with the bias by half a step of itself.
        unsure = choose<LP, V>(p, key, l, row_lds, sub, my_id, 0x1p-24f * (p.sigmoid ? 8.f : (18 + V) * one_of_total), false);
    } else {
        // numbers of 16 bits leave the lowest bits of 32 free, and nothing is lost
        unsure = choose<LP, V>(p, l, l, row_lds, sub, my_id, 0.f, TY != VBR_F32);
    }
    // rows in doubt, one after the other, by the whole wave
    for (uint64_t doubt = __ballot(unsure); doubt != 0;) {
        const int lane = threadIdx.x & 63, of_row = __builtin_ctzll(doubt) / LP;
        const int64_t at = (int64_t)blockIdx.x * kRows + (threadIdx.x >> 6) * (64 / LP) + of_row;
        const int id = choose_row_exactly<TY, kEachOf64>(p, at < p.n_rows ? at : p.n_rows - 1, lane, reinterpret_cast<double *>(lds));
        const int mine = __shfl(id, sub);
        if (lane / LP == of_row) my_id = mine;
        doubt &= LP == 64 ? 0 : ~(((1ull << (LP & 63)) - 1) << (of_row * LP));
    }
    // Renormalised, the scores are taken relative to the largest chosen one, so that no sum is zero however low they are.
    const float raw = my_id >= 0 ? raw_score(load_as_f32<TY>(p.logits, row * p.ld + my_id)) : -INFINITY;
    float w = 0.f;
    if (p.renormalise) {
        const float x = p.sigmoid ? fminf(raw, 0.f) : raw, most = row_max<LP>(x);
        if (my_id >= 0) {
            w = exp_of(x - most);
            if (p.sigmoid) w /= 1.f + exp_of(-fabsf(raw));
        }
        const float sum = row_sum<LP>(w);
        if (my_id >= 0) w /= sum;
    } else if (my_id >= 0) {
        w = p.sigmoid ? sigmoid_of(raw) : exp_of(raw - top) / total;
    }
    if (sub < p.top_k && wanted < p.n_rows) {
        p.ids[row * p.top_k + sub] = my_id;
        p.weights[row * p.top_k + sub] = w * p.scale;
    }
}

struct TopkGradParams {
    const void *logits;
    const int32_t *ids;
    const float *dweights;
    void *dlogits;
    int64_t ld, ldd, n_rows;
    int32_t n_experts, top_k, sigmoid, renormalise;
    int32_t whole, whole_out;
    float scale;
};

// The gradient to every raw score, the choice held fixed.  With r_j the chosen scores over their sum and c = sum_j dw_j r_j:
//   renormalised   dl = scale r_j (dw_j - c), times (1 - s_j) for sigmoids, at the chosen experts, zero elsewhere
//   sigmoid        dl = scale dw_j s_j (1 - s_j) at the chosen ones
//   softmax        dl = scale p_e (dw_e - sum_j dw_j p_j) everywhere
// Only the last one reads all raw scores.  Bound by what it writes and the launch: 8192 rows of 128 experts, choice and gradient, take 7.5 us.
template <int TY, int LP, int V>
__global__ void __launch_bounds__(kRouteThreads) route_topk_grad_kernel(const TopkGradParams p)
{
    constexpr int kRows = kRouteThreads / LP;
    const int sub = threadIdx.x % LP;
    const int64_t wanted = (int64_t)blockIdx.x * kRows + threadIdx.x / LP, row = wanted < p.n_rows ? wanted : p.n_rows - 1;
    int id = sub < p.top_k ? p.ids[row * p.top_k + sub] : -1;
    if (id >= p.n_experts) id = -1;
    const float raw = id >= 0 ? raw_score(load_as_f32<TY>(p.logits, row * p.ld + id)) : -INFINITY;
    const bool there = raw > -INFINITY, everywhere = !p.sigmoid && !p.renormalise;
    const float dw = there ? p.dweights[row * p.top_k + sub] : 0.f;
    float l[V], top = -INFINITY, total = 0.f;
    if (everywhere) {
        load_row<TY, V>(p.logits, row * p.ld, sub * V, p.n_experts, p.whole && (sub + 1) * V <= p.n_experts, l);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            l[v] = raw_score(l[v]);
            top = fmaxf(top, l[v]);
        }
        top = row_max<LP>(top);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            l[v] = exp_of(l[v] - top);                                         // (0 of one that is closed)
            total += l[v];
        }
        total = row_sum<LP>(total);
    }
    float mine = 0.f, common = 0.f;                 // this place's part of the gradient, and what every expert's has of the sum
    if (p.renormalise) {
        const float x = p.sigmoid ? fminf(raw, 0.f) : raw, most = row_max<LP>(x);
        float s = there ? exp_of(x - most) : 0.f, rest = 1.f;
        if (there && p.sigmoid) {
            const float e = exp_of(-fabsf(raw));
            s /= 1.f + e;
            rest = (raw > 0.f ? e : 1.f) / (1.f + e);           // 1 - sigmoid(raw)
        }
        const float sum = row_sum<LP>(s), r = there ? s / sum : 0.f;
        mine = p.scale * r * (dw - row_sum<LP>(dw * r)) * rest;
    } else if (p.sigmoid) {
        const float e = exp_of(-fabsf(raw));
        mine = there ? p.scale * dw * e / ((1.f + e) * (1.f + e)) : 0.f;
    } else {
        mine = there ? p.scale * dw * (exp_of(raw - top) / total) : 0.f;
        common = row_sum<LP>(mine);
    }
    float out[V];
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = everywhere && total > 0.f ? -common * (l[v] / total) : 0.f;
    for (int j = 0; j < p.top_k; ++j) {
        const int at = __shfl(id, j, LP) - sub * V;
        const float g = __shfl(mine, j, LP);
#pragma unroll
        for (int v = 0; v < V; ++v) out[v] += at == v ? g : 0.f;
    }
    if (wanted >= p.n_rows) return;
    constexpr int kBytes = V * (TY == VBR_F32 ? 4 : 2);
    if constexpr (kBytes >= 16) {
        if (p.whole_out && (sub + 1) * V <= p.n_experts) {
#pragma unroll
            for (int c = 0; c < kBytes / 16; ++c) {
                uint4v w;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (TY == VBR_F32) w[j] = bits(out[4 * c + j]);
                    else if constexpr (TY == VBR_BF16)
                        w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)out[8 * c + 2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)out[8 * c + 2 * j + 1]) << 16;
                    else
                        w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)out[8 * c + 2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)out[8 * c + 2 * j + 1]) << 16;
                }
                reinterpret_cast<uint4v *>(static_cast<char *>(p.dlogits) + (row * p.ldd + sub * V) * (TY == VBR_F32 ? 4 : 2))[c] = w;
            }
            return;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = sub * V + v;
        if (e < p.n_experts) store_f32<TY>(p.dlogits, row * p.ldd + e, out[v]);
    }
}

// ---- the grouping.  A workgroup owns consecutive pairs and each of its 16 waves a part of them, which it counts by expert in LDS.  With the counts of the
// workgroups and waves before it a wave knows where its first pair of every expert belongs, goes over its pairs again and puts them there: pairs of an
// expert stay in their order.  One workgroup needs no other's counts; of several, a first launch leaves them in the plan.
// Bound by its launches and the trips to memory and LDS that follow each other: 128 pairs of 64 experts take 4.7 us, 131072 of 256 10.8.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

__device__ __forceinline__ uint64_t same_id(int id, int bits)      // lanes with this lane's id
{
    uint64_t m = ~0ull;
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(id >> b & 1);
        m &= id >> b & 1 ? set : ~set;
    }
    return m;
}

__device__ __forceinline__ int expert_of(const int32_t *ids, int64_t at, int64_t end, int n_experts)     // n_experts: of no expert
{
    if (at >= end) return n_experts;
    const int id = ids[at];
    return id >= 0 && id < n_experts ? id : n_experts;
}

struct PlanParams {
    const int32_t *ids;
    int32_t *offsets, *order, *counts;             // counts [n_parts][n_experts]
    PlanTile *tiles;
    int64_t n_pairs, per_part, per_wave;           // pairs of a workgroup and of a wave, multiples of 64
    int32_t n_experts, bits, n_parts, tile_rows, n_tiles;
    int32_t lg_lanes;                              // 2^lg_lanes threads, at least as many as experts, have a part's counts
};

__global__ void __launch_bounds__(kPlanThreads) plan_count_kernel(const PlanParams p)
{
    extern __shared__ int32_t count[];
    for (int e = threadIdx.x; e < p.n_experts; e += kPlanThreads) count[e] = 0;
    __syncthreads();
    const int64_t first = blockIdx.x * p.per_part, end = first + p.per_part < p.n_pairs ? first + p.per_part : p.n_pairs;
    for (int64_t at = first + threadIdx.x; at < end; at += kPlanThreads) {
        const int id = expert_of(p.ids, at, end, p.n_experts);
        if (id < p.n_experts) atomicAdd(&count[id], 1);          // (whole numbers: in any order the same)
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.n_experts; e += kPlanThreads) p.counts[(int64_t)blockIdx.x * p.n_experts + e] = count[e];
}

// exclusive sums over the workgroup's threads of two numbers at once
__device__ __forceinline__ int2 scan_plan(int2 x, int2 *sums, int2 &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int2 up = x;
    for (int d = 1; d < 64; d <<= 1) {
        const int a = __shfl_up(up.x, d), b = __shfl_up(up.y, d);
        if (lane >= d) {
            up.x += a;
            up.y += b;
        }
    }
    if (lane == 63) sums[wave] = up;
    __syncthreads();
    int2 before = make_int2(0, 0);
    total = before;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        const int2 s = sums[w];
        if (w < wave) {
            before.x += s.x;
            before.y += s.y;
        }
        total.x += s.x;
        total.y += s.y;
    }
    return make_int2(before.x + up.x - x.x, before.y + up.y - x.y);
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanParams p)
{
    extern __shared__ int32_t next[];              // [wave][n_experts + 1], of no expert the last
    __shared__ int32_t all[kMaxExperts], before[kMaxExperts], tile_at[kMaxExperts + 1];
    __shared__ int2 sums[kPlanWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = p.n_experts + 1;
    for (int i = threadIdx.x; i < kPlanWaves * n; i += kPlanThreads) next[i] = 0;
    all[threadIdx.x] = 0;
    before[threadIdx.x] = 0;
    __syncthreads();
    const int64_t part_end = (blockIdx.x + 1) * p.per_part < p.n_pairs ? (blockIdx.x + 1) * p.per_part : p.n_pairs;
    const int64_t first = blockIdx.x * p.per_part + wave * p.per_wave, end = first + p.per_wave < part_end ? first + p.per_wave : part_end;
    int32_t *mine = next + wave * n;
    // (four loads at a time, or a wave waits for each)
    for (int64_t at = first; at < end; at += 256) {
        int id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) id[u] = expert_of(p.ids, at + 64 * u + lane, end, p.n_experts);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (at + 64 * u < end) atomicAdd(&mine[id[u]], 1);
    }
    if (p.n_parts > 1) {                           // the workgroups' counts: of all, and of those before this one
        const int e = threadIdx.x & ((1 << p.lg_lanes) - 1), step = kPlanThreads >> p.lg_lanes;
        if (e < p.n_experts) {
            int total = 0, lower = 0;
#pragma unroll 8
            for (int i = threadIdx.x >> p.lg_lanes; i < p.n_parts; i += step) {
                const int c = p.counts[(int64_t)i * p.n_experts + e];
                total += c;
                lower += i < (int)blockIdx.x ? c : 0;
            }
            atomicAdd(&all[e], total);
            atomicAdd(&before[e], lower);
        }
    }
    __syncthreads();
    const int e = threadIdx.x;
    int count = 0;
    if (e < p.n_experts) {
        if (p.n_parts > 1) {
            count = all[e];
        } else {
#pragma unroll
            for (int w = 0; w < kPlanWaves; ++w) count += next[w * n + e];
        }
    }
    const int tiles = (count + p.tile_rows - 1) / p.tile_rows;
    int2 total;
    const int2 start = scan_plan(make_int2(count, tiles), sums, total);
    if (e < p.n_experts) {
        all[e] = start.x;
        tile_at[e] = start.y;
        int at = start.x + (p.n_parts > 1 ? before[e] : 0);
#pragma unroll
        for (int w = 0; w < kPlanWaves; ++w) {
            const int here = next[w * n + e];
            next[w * n + e] = at;
            at += here;
        }
        if (blockIdx.x == 0) p.offsets[e] = start.x;
    }
    if (e == 0) {
        tile_at[p.n_experts] = total.y;
        if (blockIdx.x == 0) p.offsets[p.n_experts] = total.x;
    }
    __syncthreads();
    for (int64_t at = first; at < end; at += 256) {
        int id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) id[u] = expert_of(p.ids, at + 64 * u + lane, end, p.n_experts);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (at + 64 * u >= end) break;
            const uint64_t same = same_id(id[u], p.bits);
            const int earlier = __popcll(same & ((1ull << lane) - 1)), begin = mine[id[u]];
            if (id[u] < p.n_experts) p.order[begin + earlier] = (int32_t)(at + 64 * u + lane);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (earlier == 0) mine[id[u]] = begin + __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
    // the tiles, and what is behind the last pair, by all workgroups
    for (int64_t i = blockIdx.x * (int64_t)kPlanThreads + threadIdx.x; i < p.n_tiles; i += (int64_t)p.n_parts * kPlanThreads) {
        PlanTile t = {0, 0, 0, total.y};
        if (i < total.y) {
            int lo = 0, hi = p.n_experts;          // the last expert that begins at or before tile i and has one
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (tile_at[mid] <= i) lo = mid;
                else hi = mid;
            }
            const int expert_end = lo + 1 < p.n_experts ? all[lo + 1] : total.x;
            t.expert = lo;
            t.first = all[lo] + (int)(i - tile_at[lo]) * p.tile_rows;
            t.count = expert_end - t.first < p.tile_rows ? expert_end - t.first : p.tile_rows;
        }
        p.tiles[i] = t;
    }
    for (int64_t i = total.x + blockIdx.x * (int64_t)kPlanThreads + threadIdx.x; i < p.n_pairs; i += (int64_t)p.n_parts * kPlanThreads) p.order[i] = -1;
}

// ---- the weighted sum
struct CombineParams {
    const void *y, *dout;
    const int32_t *ids;
    const float *weights;
    void *out, *dy;
    float *dweights;
    int64_t ldy, ldo, lddy, n_rows;
    int32_t n_cols, top_k, n_experts, n_chunks;
    Divide by_chunks;
};

using Global = const __attribute__((address_space(1))) char *;
template <class T>
__device__ __forceinline__ T load_from(Global p) { return *(const __attribute__((address_space(1))) T *)p; }

template <int TY>
__device__ __forceinline__ void load8(Global p, float (&x)[8])
{
    if constexpr (TY == VBR_F32) {
        const float4v a = load_from<float4v>(p), b = load_from<float4v>(p + 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = a[j];
            x[j + 4] = b[j];
        }
    } else if constexpr (TY == VBR_F16) {
        const half8v a = load_from<half8v>(p);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)a[j];
    } else {
        const bf16x8v a = load_from<bf16x8v>(p);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)a[j];
    }
}
template <int TY>
__device__ __forceinline__ Global element(const void *p, int64_t i) { return (Global)p + i * (TY == VBR_F32 ? 4 : 2); }

template <int TY>
__device__ __forceinline__ void store8(void *p, int64_t i, const float (&x)[8])
{
    if constexpr (TY == VBR_F32) {
        *reinterpret_cast<float4v *>(static_cast<float *>(p) + i) = float4v{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<float4v *>(static_cast<float *>(p) + i + 4) = float4v{x[4], x[5], x[6], x[7]};
    } else if constexpr (TY == VBR_F16) {
        half8v a;
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = (_Float16)x[j];
        *reinterpret_cast<half8v *>(static_cast<_Float16 *>(p) + i) = a;
    } else {
        bf16x8v a;
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = (__bf16)x[j];
        *reinterpret_cast<bf16x8v *>(static_cast<__bf16 *>(p) + i) = a;
    }
}

// What is read in the place of a result whose pair has no expert, so that loads need no branch: such results are never read, and their rows need not be there.
__device__ const float4v nothing[2] = {};

// A thread owns eight columns of a row of out; the row's results are added in the order of their places.  Bound by what it reads: 4096 rows of 8 bf16 results of
// 2048 take 38 us, 4.0 TB/s, from memory (23 where they are in the cache behind the L2).  AT places are on their way at a time.
template <int TY, int TO, int AT>
__global__ void __launch_bounds__(kRouteThreads) route_combine_kernel(const CombineParams p)
{
    const uint32_t at = blockIdx.x * (uint32_t)kRouteThreads + threadIdx.x, row = p.by_chunks(at);
    const int col = (int)(at - row * (uint32_t)p.n_chunks) * 8;
    if (row >= p.n_rows) return;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    const int64_t first = (int64_t)row * p.top_k;
    for (int j0 = 0; j0 < p.top_k; j0 += AT) {
        bool there[AT];
        float w[AT], x[AT][8];
#pragma unroll
        for (int u = 0; u < AT; ++u) {
            const int64_t pair = j0 + u < p.top_k ? first + j0 + u : first;
            there[u] = (uint32_t)p.ids[pair] < (uint32_t)p.n_experts && j0 + u < p.top_k;
            w[u] = p.weights[pair];
        }
#pragma unroll
        for (int u = 0; u < AT; ++u) load8<TY>(there[u] ? element<TY>(p.y, (first + j0 + u) * p.ldy + col) : (Global)nothing, x[u]);
#pragma unroll
        for (int u = 0; u < AT; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = there[u] ? __builtin_fmaf(w[u], x[u][i], sum[i]) : sum[i];
    }
    store8<TO>(p.out, row * p.ldo + col, sum);
}

// A wave owns a pair: dy = w dout, dw = dout . y.  The k waves of a row read its dout from the caches.  Bound by what it reads and writes: for the rows above
// 49 us, 5.8 TB/s, part of it from the cache behind the L2.
template <int TY, int TO>
__global__ void __launch_bounds__(kRouteThreads) route_combine_grad_kernel(const CombineParams p)
{
    const int lane = threadIdx.x & 63;
    const int64_t pair = (int64_t)blockIdx.x * (kRouteThreads / 64) + (threadIdx.x >> 6);
    if (pair >= p.n_rows * p.top_k) return;
    const int64_t row = pair / p.top_k;
    const bool there = (uint32_t)p.ids[pair] < (uint32_t)p.n_experts;
    const float w = there ? p.weights[pair] : 0.f;
    float dot = 0.f;
    for (int col = lane * 8; col < p.n_cols; col += 512) {
        float g[8], x[8];
        load8<TO>(element<TO>(p.dout, row * p.ldo + col), g);
        if (there) {
            load8<TY>(element<TY>(p.y, pair * p.ldy + col), x);
#pragma unroll
            for (int i = 0; i < 8; ++i) dot = __builtin_fmaf(g[i], x[i], dot);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = there ? g[i] * w : 0.f;
        store8<TY>(p.dy, pair * p.lddy + col, g);
    }
    dot = row_sum<64>(dot);
    if (lane == 0) p.dweights[pair] = dot;
}

bool route_ok(const vbr_route_t *how)
{
    if (!how || how->n_experts < 1 || how->n_experts > kMaxExperts || how->top_k < 1 || how->top_k > kMaxTopK || how->top_k > how->n_experts) return false;
    if (how->score != VBR_SOFTMAX && how->score != VBR_SIGMOID) return false;
    if (how->n_groups < 1 || how->n_groups > kMaxGroups || how->n_experts % how->n_groups != 0) return false;
    if (how->top_groups < 1 || how->top_groups > how->n_groups || how->n_experts / how->n_groups * how->top_groups < how->top_k) return false;
    return how->scale - how->scale == 0.f;           // finite
}

bool float_type(int32_t t) { return t == VBR_F16 || t == VBR_BF16 || t == VBR_F32; }
int64_t up(int64_t x, int64_t q) { return (x + q - 1) / q * q; }

// Lanes of a row: 16 where they can hold the experts and there are many rows, four a wave, 64 elsewhere: one row of them is done sooner.  In us with 16 and 64,
// 8 of 256 experts in 8 groups: 1024 rows 9.5 and 6.0, 2048 9.8 and 9.4, 4096 9.9 and 12.9, 16384 17.1 and 27.8; 8 of 128: 512 5.5 and 5.9, 2048 4.2 and 4.6,
// 16384 5.9 and 13.4; 4 of 64: 1024 3.7 and 3.6, 2048 3.7 and 3.7, 16384 4.5 and 8.5.
struct Width {
    int32_t lanes, each;
};
Width route_width(int32_t n_experts, int32_t top_k, int32_t n_groups, int64_t n_rows)
{
    const int32_t lanes = n_rows >= kNarrowRows && n_experts <= 256 && top_k <= 16 && n_groups <= 16 ? 16 : 64;
    int32_t each = 1;
    while (lanes * each < n_experts) each *= 2;
    return {lanes, each};
}

#define ROUTE_LAUNCH(KERNEL, TY, LP, V) hipLaunchKernelGGL((KERNEL<TY, LP, V>), dim3(grid), dim3(kRouteThreads), 0, stream, p)
#define ROUTE_BY_EACH(KERNEL, TY, LP)                         \
    do {                                                      \
        if (width.each == 1) ROUTE_LAUNCH(KERNEL, TY, LP, 1);      \
        else if (width.each == 2) ROUTE_LAUNCH(KERNEL, TY, LP, 2); \
        else if (width.each == 4) ROUTE_LAUNCH(KERNEL, TY, LP, 4); \
        else if (width.each == 8) ROUTE_LAUNCH(KERNEL, TY, LP, 8); \
        else ROUTE_LAUNCH(KERNEL, TY, LP, 16);                \
    } while (0)
#define ROUTE_BY_WIDTH(KERNEL, TY)                            \
    do {                                                      \
        if (width.lanes == 16) ROUTE_BY_EACH(KERNEL, TY, 16);      \
        else ROUTE_BY_EACH(KERNEL, TY, 64);                   \
    } while (0)
#define ROUTE_BY_TYPE(KERNEL, type)                           \
    do {                                                      \
        if (type == VBR_F32) ROUTE_BY_WIDTH(KERNEL, VBR_F32);      \
        else if (type == VBR_F16) ROUTE_BY_WIDTH(KERNEL, VBR_F16); \
        else ROUTE_BY_WIDTH(KERNEL, VBR_BF16);                \
    } while (0)

bool whole_pieces(const void *rows, int64_t ld, uintptr_t size) { return aligned(rows, 16) && ld * (int64_t)size % 16 == 0; }

}  // namespace

// Rows of a tile of the products: by how many pairs an expert has if all have alike.  A tile reads its expert's matrix once, a larger one multiplies more rows
// that are not there.  In us, with tiles of 16, 32 and 64 rows, for 64 experts of 2816 x 2048 and 2048 x 1408 with
//   8 pairs each:  52 50 76 and 22 25 31     12:  55 50 76 and 29 25 32     16:  68 51 79 and 34 26 31
//   32:  100 68 81 and 56 31 32              48:  133 89 80 and 75 41 34    64:  163 106 95 and 97 46 49
int32_t plan_tile_rows(int64_t n_pairs, int32_t n_experts)
{
    const int64_t rows = n_pairs / n_experts;
    return rows <= 12 ? 16 : rows <= 32 ? 32 : 64;
}

// Tiles of tile_rows rows that any ids can need: an expert with c > 0 pairs has at most 1 + (c - 1) / tile_rows.
int64_t plan_max_tiles(int64_t n_pairs, int32_t n_experts, int32_t tile_rows)
{
    const int64_t most = n_pairs < n_experts ? n_pairs : n_experts;
    return most + (n_pairs - most) / tile_rows;
}

PlanParts plan_parts(int64_t n_pairs, int32_t n_experts)
{
    PlanParts q;
    q.tile_rows = plan_tile_rows(n_pairs, n_experts);
    q.n_tiles = plan_max_tiles(n_pairs, n_experts, q.tile_rows);
    // One workgroup needs one launch (4096 pairs of 64 experts 7.7 us, four workgroups 8.1; 8192 pairs 11.3, eight of them 8.0); of several each has at least kPlanPart
    // pairs (32768 of 256 experts 9.2 us, with 2048 each 10.8), and there are no more than compute units.
    q.n_parts = n_pairs <= kPlanAlone ? 1 : std::min<int64_t>(256, n_pairs / kPlanPart);
    q.per_wave = up((n_pairs + q.n_parts * kPlanWaves - 1) / (q.n_parts * kPlanWaves), 64);
    q.order = up(4 * ((int64_t)n_experts + 1), 256);
    q.tiles = up(q.order + 4 * n_pairs, 256);
    q.counts = up(q.tiles + (int64_t)sizeof(PlanTile) * q.n_tiles, 256);
    q.total = up(q.counts + 4 * q.n_parts * n_experts, 256);
    return q;
}

bool plan_sizes_ok(int64_t n_pairs, int32_t n_experts) { return n_pairs >= 0 && n_pairs <= kMaxPairs && n_experts >= 1 && n_experts <= kMaxExperts; }

}  // namespace vbrk

using namespace vbrk;

extern "C" int route_topk(const vbr_route_t *how, const void *logits_dev, int64_t ld, int32_t logits_type, const float *bias_dev, int64_t n_rows,
                          int32_t *ids_dev, float *weights_dev, void *hip_stream)
{
    if (!route_ok(how) || !float_type(logits_type) || n_rows < 0 || ld < how->n_experts) return VBR_EINVAL;
    if (n_rows > kMaxPairs / how->top_k) return VBR_EUNSUPPORTED;
    if (n_rows == 0) return VBR_OK;
    if (!logits_dev || !ids_dev || !weights_dev || !aligned(logits_dev, logits_type == VBR_F32 ? 4 : 2) || !aligned(bias_dev, 4) || !aligned(ids_dev, 4) || !aligned(weights_dev, 4)) return VBR_EINVAL;
    TopkParams p;
    p.logits = logits_dev;
    p.bias = bias_dev;
    p.ids = ids_dev;
    p.weights = weights_dev;
    p.ld = ld;
    p.n_rows = n_rows;
    p.n_experts = how->n_experts;
    p.top_k = how->top_k;
    p.n_groups = how->n_groups;
    p.top_groups = how->top_groups;
    p.group_size = how->n_experts / how->n_groups;
    p.group_factor = (uint32_t)((1 << 20) + p.group_size - 1) / (uint32_t)p.group_size;
    p.sigmoid = how->score == VBR_SIGMOID;
    p.renormalise = how->renormalise != 0;
    p.scored = bias_dev != nullptr || how->n_groups > 1;
    p.scale = how->scale;
    p.whole = whole_pieces(logits_dev, ld, logits_type == VBR_F32 ? 4 : 2);
    p.whole_bias = aligned(bias_dev, 16);
    const Width width = route_width(how->n_experts, how->top_k, how->n_groups, n_rows);
    const int32_t lanes_a_group = p.group_size / width.each;
    p.lanes_a_group = p.group_size % width.each == 0 && lanes_a_group <= 8 && (lanes_a_group & (lanes_a_group - 1)) == 0 ? lanes_a_group : 0;
    const int64_t workgroups = (n_rows + kRouteThreads / width.lanes - 1) / (kRouteThreads / width.lanes);
    if (workgroups > kMostThreads / kRouteThreads) return VBR_EUNSUPPORTED;
    const unsigned grid = (unsigned)workgroups;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ROUTE_BY_TYPE(route_topk_kernel, logits_type);
    return launched();
}

extern "C" int route_topk_grad(const vbr_route_t *how, const void *logits_dev, int64_t ld, int32_t logits_type, const int32_t *ids_dev, const float *dweights_dev,
                               int64_t n_rows, void *dlogits_dev, int64_t ldd, void *hip_stream)
{
    if (!route_ok(how) || !float_type(logits_type) || n_rows < 0 || ld < how->n_experts || ldd < how->n_experts) return VBR_EINVAL;
    if (n_rows > kMaxPairs / how->top_k) return VBR_EUNSUPPORTED;
    if (n_rows == 0) return VBR_OK;
    const uintptr_t size = logits_type == VBR_F32 ? 4 : 2;
    if (!logits_dev || !ids_dev || !dweights_dev || !dlogits_dev || !aligned(logits_dev, size) || !aligned(dlogits_dev, size) || !aligned(ids_dev, 4) || !aligned(dweights_dev, 4)) return VBR_EINVAL;
    TopkGradParams p;
    p.logits = logits_dev;
    p.ids = ids_dev;
    p.dweights = dweights_dev;
    p.dlogits = dlogits_dev;
    p.ld = ld;
    p.ldd = ldd;
    p.n_rows = n_rows;
    p.n_experts = how->n_experts;
    p.top_k = how->top_k;
    p.sigmoid = how->score == VBR_SIGMOID;
    p.renormalise = how->renormalise != 0;
    p.scale = how->scale;
    p.whole = whole_pieces(logits_dev, ld, size);
    p.whole_out = whole_pieces(dlogits_dev, ldd, size);
    const Width width = route_width(how->n_experts, how->top_k, 1, n_rows);
    const int64_t workgroups = (n_rows + kRouteThreads / width.lanes - 1) / (kRouteThreads / width.lanes);
    if (workgroups > kMostThreads / kRouteThreads) return VBR_EUNSUPPORTED;
    const unsigned grid = (unsigned)workgroups;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ROUTE_BY_TYPE(route_topk_grad_kernel, logits_type);
    return launched();
}

extern "C" int64_t route_plan_bytes(int64_t n_pairs, int32_t n_experts)
{
    return plan_sizes_ok(n_pairs, n_experts) ? plan_parts(n_pairs, n_experts).total : 0;
}

extern "C" int64_t route_plan_order(int64_t n_pairs, int32_t n_experts)
{
    return plan_sizes_ok(n_pairs, n_experts) ? plan_parts(n_pairs, n_experts).order : 0;
}

extern "C" int route_plan(const int32_t *ids_dev, int64_t n_pairs, int32_t n_experts, void *plan_dev, void *hip_stream)
{
    if (!plan_sizes_ok(n_pairs, n_experts) || !plan_dev || !aligned(plan_dev, 256) || (n_pairs > 0 && !ids_dev) || !aligned(ids_dev, 4)) return VBR_EINVAL;
    const PlanParts q = plan_parts(n_pairs, n_experts);
    char *d = static_cast<char *>(plan_dev);
    PlanParams p;
    p.ids = ids_dev;
    p.offsets = reinterpret_cast<int32_t *>(d);
    p.order = reinterpret_cast<int32_t *>(d + q.order);
    p.tiles = reinterpret_cast<PlanTile *>(d + q.tiles);
    p.counts = reinterpret_cast<int32_t *>(d + q.counts);
    p.n_pairs = n_pairs;
    p.n_experts = n_experts;
    p.bits = 32 - __builtin_clz((unsigned)n_experts);       // of 0 .. n_experts
    p.n_parts = (int32_t)q.n_parts;
    p.per_wave = q.per_wave;
    p.per_part = q.per_wave * kPlanWaves;
    p.tile_rows = q.tile_rows;
    p.n_tiles = (int32_t)q.n_tiles;
    p.lg_lanes = 32 - __builtin_clz((unsigned)n_experts) - ((n_experts & (n_experts - 1)) == 0 ? 1 : 0);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (q.n_parts > 1) hipLaunchKernelGGL(plan_count_kernel, dim3((unsigned)q.n_parts), dim3(kPlanThreads), 4 * (unsigned)n_experts, stream, p);
    hipLaunchKernelGGL(plan_kernel, dim3((unsigned)q.n_parts), dim3(kPlanThreads), 4 * kPlanWaves * ((unsigned)n_experts + 1), stream, p);
    return launched();
}

namespace {

int combine_args(int32_t y_type, int32_t out_type, int64_t n_cols, int64_t n_rows, int32_t top_k, int32_t n_experts, const void *const *rows, const int64_t *lds, int n)
{
    if (!float_type(y_type) || !float_type(out_type) || n_rows < 0 || top_k < 1 || top_k > kMaxTopK || n_experts < 1 || n_cols < 0 || n_cols % 8 != 0) return VBR_EINVAL;
    for (int i = 0; i < n; ++i)
        if (lds[i] < n_cols || lds[i] % 8 != 0 || !aligned(rows[i], 16)) return VBR_EINVAL;
    if (n_rows > kMaxPairs / top_k || n_cols > INT32_MAX / 2) return VBR_EUNSUPPORTED;
    return VBR_OK;
}

template <int TY, int TO>
constexpr auto route_combine_2 = route_combine_kernel<TY, TO, 2>;
template <int TY, int TO>
constexpr auto route_combine_8 = route_combine_kernel<TY, TO, 8>;

#define COMBINE_LAUNCH(KERNEL, TY, TO) hipLaunchKernelGGL((KERNEL<TY, TO>), dim3((unsigned)grid), dim3(kRouteThreads), 0, stream, p)
#define COMBINE_BY_OUT(KERNEL, TY)                                      \
    do {                                                                \
        if (out_type == VBR_F32) COMBINE_LAUNCH(KERNEL, TY, VBR_F32);      \
        else if (out_type == VBR_F16) COMBINE_LAUNCH(KERNEL, TY, VBR_F16); \
        else COMBINE_LAUNCH(KERNEL, TY, VBR_BF16);                      \
    } while (0)
#define COMBINE_BY_TYPES(KERNEL)                                        \
    do {                                                                \
        if (y_type == VBR_F32) COMBINE_BY_OUT(KERNEL, VBR_F32);            \
        else if (y_type == VBR_F16) COMBINE_BY_OUT(KERNEL, VBR_F16);       \
        else COMBINE_BY_OUT(KERNEL, VBR_BF16);                          \
    } while (0)

}  // namespace

extern "C" int route_combine(const void *y_dev, int64_t ldy, int32_t y_type, const int32_t *ids_dev, const float *weights_dev, int64_t n_rows, int32_t top_k, int32_t n_experts, int64_t n_cols,
                             void *out_dev, int64_t ldo, int32_t out_type, void *hip_stream)
{
    const void *rows[2] = {y_dev, out_dev};
    const int64_t lds[2] = {ldy, ldo};
    const int rc = combine_args(y_type, out_type, n_cols, n_rows, top_k, n_experts, rows, lds, 2);
    if (rc != VBR_OK || n_rows == 0 || n_cols == 0) return rc;
    if (!y_dev || !ids_dev || !weights_dev || !out_dev || !aligned(ids_dev, 4) || !aligned(weights_dev, 4)) return VBR_EINVAL;
    CombineParams p{};
    p.y = y_dev;
    p.ids = ids_dev;
    p.weights = weights_dev;
    p.out = out_dev;
    p.ldy = ldy;
    p.ldo = ldo;
    p.n_rows = n_rows;
    p.n_cols = (int32_t)n_cols;
    p.top_k = top_k;
    p.n_experts = n_experts;
    p.n_chunks = (int32_t)(n_cols / 8);
    p.by_chunks = Divide::by(p.n_chunks);
    const int64_t grid = (n_rows * p.n_chunks + kRouteThreads - 1) / kRouteThreads;
    if (grid > kMostThreads / 2 / kRouteThreads) return VBR_EUNSUPPORTED;          // (threads are divided by n_chunks in 31 bits)
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    // two places at a time, or eight where there are as many (in us, results in the cache; 16384 fp32 results of 2048 columns, 8 a row: 22.8, with two 22.9; 6 a row:
    // 24.0 and 23.9; one a row: 53.7 and 40.7)
    if (top_k < 8) COMBINE_BY_TYPES(route_combine_2);
    else COMBINE_BY_TYPES(route_combine_8);
    return launched();
}

extern "C" int route_combine_grad(const void *dout_dev, int64_t ldo, int32_t out_type, const void *y_dev, int64_t ldy, int32_t y_type, const int32_t *ids_dev, const float *weights_dev,
                                  int64_t n_rows, int32_t top_k, int32_t n_experts, int64_t n_cols, void *dy_dev, int64_t lddy, float *dweights_dev, void *hip_stream)
{
    const void *rows[3] = {y_dev, dout_dev, dy_dev};
    const int64_t lds[3] = {ldy, ldo, lddy};
    const int rc = combine_args(y_type, out_type, n_cols, n_rows, top_k, n_experts, rows, lds, 3);
    if (rc != VBR_OK || n_rows == 0) return rc;
    if (!ids_dev || !weights_dev || !dweights_dev || !aligned(ids_dev, 4) || !aligned(weights_dev, 4) || !aligned(dweights_dev, 4)) return VBR_EINVAL;
    if (n_cols > 0 && (!y_dev || !dout_dev || !dy_dev)) return VBR_EINVAL;
    CombineParams p{};
    p.y = y_dev;
    p.dout = dout_dev;
    p.ids = ids_dev;
    p.weights = weights_dev;
    p.dy = dy_dev;
    p.dweights = dweights_dev;
    p.ldy = ldy;
    p.ldo = ldo;
    p.lddy = lddy;
    p.n_rows = n_rows;
    p.n_cols = (int32_t)n_cols;
    p.top_k = top_k;
    p.n_experts = n_experts;
    const int64_t grid = (n_rows * top_k + kRouteThreads / 64 - 1) / (kRouteThreads / 64);
    if (grid > kMostThreads / kRouteThreads) return VBR_EUNSUPPORTED;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    COMBINE_BY_TYPES(route_combine_grad_kernel);
    return launched();
}
