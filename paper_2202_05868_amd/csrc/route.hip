// What stands around the products of routed rows: the choice of k experts for every row with its weights and their gradient, the grouping
// of the chosen (row, place) pairs by expert, and the weighted sum of a row's results with its gradients.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <climits>
#include <cstdint>

#include "route.h"
#include "vbr_device.h"
#include "vbr_host.h"

namespace vbrk {
namespace {

constexpr int kRouteThreads = 256;     // 4 waves

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

template <class T>
__device__ __forceinline__ T wave_max(T v)
{
    for (int m = 32; m; m >>= 1) {
        const T o = __shfl_xor(v, m);
        v = o > v ? o : v;
    }
    return v;
}

template <class T>
__device__ __forceinline__ T wave_sum(T v)
{
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// (key, index) of the largest key, of equal ones the lowest index, in every lane
__device__ __forceinline__ void wave_best(double &key, int &index)
{
    for (int m = 32; m; m >>= 1) {
        const double k = __shfl_xor(key, m);
        const int i = __shfl_xor(index, m);
        if (k > key || (k == key && i < index)) {
            key = k;
            index = i;
        }
    }
}

struct TopkParams {
    const void *logits;
    const float *bias;
    int32_t *ids;
    float *weights;
    int64_t ld, n_rows;
    int32_t n_experts, top_k, n_groups, top_groups, group_size;
    int32_t sigmoid, renormalise, scored;      // scored: the keys are scores with their biases, not the raw scores
    float scale;
};

// A raw score as it counts: NaN closes the expert like -inf, +inf is the largest finite number.
__device__ __forceinline__ float raw_score(float l) { return l > -INFINITY ? fminf(l, FLT_MAX) : -INFINITY; }

// One wave a row, V experts a lane.  Sums of scores and biases are compared in 64 bits: two of them that 32 bits cannot tell apart would let
// their order depend on how they were rounded.  Raw scores are compared as they are, since the score rises with them.
template <int TY, int V>
__global__ void __launch_bounds__(kRouteThreads) route_topk_kernel(const TopkParams p)
{
    __shared__ double keys[kRouteThreads / 64][64 * V];
    const int lane = threadIdx.x & 63, in_wg = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * (kRouteThreads / 64) + in_wg;
    if (row >= p.n_rows) return;
    float l[V];
    double key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane * V + v;
        l[v] = e < p.n_experts ? raw_score(load_as_f32<TY>(p.logits, row * p.ld + e)) : -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) top = fmaxf(top, l[v]);
    top = wave_max(top);
    double total = 0;
    if (!p.sigmoid && top > -INFINITY) {
#pragma unroll
        for (int v = 0; v < V; ++v) total += l[v] > -INFINITY ? exp((double)l[v] - (double)top) : 0.0;
        total = wave_sum(total);
    }
    auto score = [&](float x) { return p.sigmoid ? 1.0 / (1.0 + exp(-(double)x)) : exp((double)x - (double)top) / total; };
#pragma unroll
    for (int v = 0; v < V; ++v) {
        key[v] = -INFINITY;
        if (l[v] > -INFINITY) {
            if (p.scored) {
                key[v] = score(l[v]) + (p.bias ? (double)p.bias[lane * V + v] : 0.0);
                if (!(key[v] > -INFINITY)) key[v] = -INFINITY;
            } else {
                key[v] = (double)l[v];
            }
        }
    }
    if (p.n_groups > 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) keys[in_wg][lane * V + v] = key[v];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        double best = -INFINITY, second = -INFINITY;
        if (lane < p.n_groups) {
            for (int i = 0; i < p.group_size; ++i) {
                const double x = keys[in_wg][lane * p.group_size + i];
                if (x > best) {
                    second = best;
                    best = x;
                } else if (x > second) {
                    second = x;
                }
            }
        }
        double mine = second > -INFINITY ? best + second : best;
        uint64_t chosen = 0;
        for (int i = 0; i < p.top_groups; ++i) {
            double k = mine;
            int at = mine > -INFINITY ? lane : INT_MAX;
            wave_best(k, at);
            if (at == INT_MAX) break;
            chosen |= 1ull << at;
            if (lane == at) mine = -INFINITY;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = lane * V + v;
            if (e < p.n_experts && !(chosen >> (e / p.group_size) & 1)) key[v] = -INFINITY;
        }
    }
    // lane j keeps the j-th choice
    int my_id = -1;
    float my_raw = -INFINITY;
    if (!p.scored || p.bias == nullptr) {
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = key[v] > -INFINITY ? (double)l[v] : -INFINITY;
    }
    for (int j = 0; j < p.top_k; ++j) {
        double k = -INFINITY;
        int at = INT_MAX;
        float raw = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (key[v] > k) {
                k = key[v];
                at = lane * V + v;
            }
        }
        wave_best(k, at);
        if (at == INT_MAX) break;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (at == lane * V + v) {
                raw = l[v];
                key[v] = -INFINITY;
            }
        }
        raw = __shfl(raw, at / V);
        if (lane == j) {
            my_id = at;
            my_raw = raw;
        }
    }
    // Renormalised, the scores are taken relative to the largest chosen one, so that no sum is zero however low they are.
    double w = 0;
    if (p.renormalise) {
        const float x = p.sigmoid ? fminf(my_raw, 0.f) : my_raw;
        const float most = wave_max(my_id >= 0 ? x : -INFINITY);
        if (my_id >= 0) {
            w = exp((double)x - (double)most);
            if (p.sigmoid) w /= 1.0 + exp(-fabs((double)my_raw));
        }
        const double sum = wave_sum(w);
        if (my_id >= 0) w /= sum;
    } else if (my_id >= 0) {
        w = score(my_raw);
    }
    if (lane < p.top_k) {
        p.ids[row * p.top_k + lane] = my_id;
        p.weights[row * p.top_k + lane] = (float)(w * p.scale);
    }
}

struct TopkGradParams {
    const void *logits;
    const int32_t *ids;
    const float *dweights;
    void *dlogits;
    int64_t ld, ldd, n_rows;
    int32_t n_experts, top_k, sigmoid, renormalise;
    float scale;
};

// The gradient to every raw score, the choice held fixed.  With r_j the chosen scores over their sum and c = sum_j dw_j r_j:
//   renormalised   dl = scale r_j (dw_j - c), times (1 - s_j) for sigmoids, at the chosen experts, zero elsewhere
//   sigmoid        dl = scale dw_j s_j (1 - s_j) at the chosen ones
//   softmax        dl = scale p_e (dw_e - sum_j dw_j p_j) everywhere
template <int TY, int V>
__global__ void __launch_bounds__(kRouteThreads) route_topk_grad_kernel(const TopkGradParams p)
{
    const int lane = threadIdx.x & 63, in_wg = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * (kRouteThreads / 64) + in_wg;
    if (row >= p.n_rows) return;
    int id = lane < p.top_k ? p.ids[row * p.top_k + lane] : -1;
    if (id >= p.n_experts) id = -1;
    const float raw = id >= 0 ? raw_score(load_as_f32<TY>(p.logits, row * p.ld + id)) : -INFINITY;
    const bool there = raw > -INFINITY;
    const float dw = there ? p.dweights[row * p.top_k + lane] : 0.f;
    const bool everywhere = !p.sigmoid && !p.renormalise;
    float l[V];
    float top = -INFINITY, total = 0.f;
    if (everywhere) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = lane * V + v;
            l[v] = e < p.n_experts ? raw_score(load_as_f32<TY>(p.logits, row * p.ld + e)) : -INFINITY;
            top = fmaxf(top, l[v]);
        }
        top = wave_max(top);
#pragma unroll
        for (int v = 0; v < V; ++v) total += l[v] > -INFINITY ? expf(l[v] - top) : 0.f;
        total = wave_sum(total);
    }
    float s = 0.f, mine = 0.f, common = 0.f;        // this place's part of the gradient, and what every expert's has of the sum
    if (p.renormalise) {
        const float x = p.sigmoid ? fminf(raw, 0.f) : raw;
        const float most = wave_max(there ? x : -INFINITY);
        if (there) s = expf(x - most);
        float rest = 1.f;
        if (there && p.sigmoid) {
            const float e = expf(-fabsf(raw));
            s /= 1.f + e;
            rest = (raw > 0.f ? e : 1.f) / (1.f + e);           // 1 - sigmoid(raw)
        }
        const float sum = wave_sum(s), r = there ? s / sum : 0.f;
        mine = p.scale * r * (dw - wave_sum(dw * r)) * rest;
    } else if (p.sigmoid) {
        const float e = expf(-fabsf(raw));
        mine = there ? p.scale * dw * e / ((1.f + e) * (1.f + e)) : 0.f;
    } else {
        s = there ? expf(raw - top) / total : 0.f;
        mine = p.scale * s * dw;
        common = wave_sum(mine);
    }
    float out[V];
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = everywhere && l[v] > -INFINITY ? -common * (expf(l[v] - top) / total) : 0.f;
    for (int j = 0; j < p.top_k; ++j) {
        const int at = __shfl(id, j);
        const float g = __shfl(mine, j);
#pragma unroll
        for (int v = 0; v < V; ++v) out[v] += at == lane * V + v ? g : 0.f;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane * V + v;
        if (e < p.n_experts) store_f32<TY>(p.dlogits, row * p.ldd + e, out[v]);
    }
}

// ---- the grouping.  A wave owns a chunk of consecutive pairs and counts its experts; one workgroup turns the counts into every chunk's
// first positions; the waves go over their chunks again and put each pair where it belongs.  Pairs of an expert stay in their order.
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
    int32_t *offsets, *order, *counts;             // counts [n_chunks][n_experts]
    PlanTile *tiles;
    int64_t n_pairs;
    int32_t n_experts, bits, n_chunks, tile_rows, n_tiles;
};

__global__ void __launch_bounds__(64) plan_count_kernel(const PlanParams p)
{
    extern __shared__ int32_t hist[];
    const int lane = threadIdx.x;
    for (int e = lane; e <= p.n_experts; e += 64) hist[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kPlanChunk;
    const int64_t end = first + kPlanChunk < p.n_pairs ? first + kPlanChunk : p.n_pairs;
    for (int64_t at = first; at < end; at += 64) {
        const int id = expert_of(p.ids, at + lane, end, p.n_experts);
        const uint64_t same = same_id(id, p.bits);
        if (__builtin_ctzll(same) == lane) hist[id] += __popcll(same);
        __syncthreads();
    }
    for (int e = lane; e < p.n_experts; e += 64) p.counts[(int64_t)blockIdx.x * p.n_experts + e] = hist[e];
}

constexpr int kScanThreads = 1024;     // one a expert

__device__ __forceinline__ int scan_1024(int x, int *sums, int &total)      // exclusive sum over the workgroup's threads
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int up = x;
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(up, d);
        if (lane >= d) up += o;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = up;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < kScanThreads / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    return before + up - x;
}

__global__ void __launch_bounds__(kScanThreads) plan_scan_kernel(const PlanParams p)
{
    __shared__ int sums[kScanThreads / 64];
    const int e = threadIdx.x;
    int count = 0;
    if (e < p.n_experts)
        for (int c = 0; c < p.n_chunks; ++c) count += p.counts[(int64_t)c * p.n_experts + e];
    int total, n_tiles;
    const int start = scan_1024(count, sums, total);
    if (e < p.n_experts) {
        p.offsets[e] = start;
        int at = start;
        for (int c = 0; c < p.n_chunks; ++c) {
            int32_t *mine = p.counts + (int64_t)c * p.n_experts + e;
            const int here = *mine;
            *mine = at;
            at += here;
        }
    }
    if (e == 0) p.offsets[p.n_experts] = total;
    const int tiles = (count + p.tile_rows - 1) / p.tile_rows, tile = scan_1024(tiles, sums, n_tiles);
    for (int i = 0; i < tiles; ++i) {
        const int left = count - i * p.tile_rows;
        p.tiles[tile + i] = {e, start + i * p.tile_rows, left < p.tile_rows ? left : p.tile_rows, 0};
    }
    for (int i = n_tiles + e; i < p.n_tiles; i += kScanThreads) p.tiles[i] = {0, 0, 0, 0};
    for (int64_t i = total + (int64_t)e; i < p.n_pairs; i += kScanThreads) p.order[i] = -1;
}

__global__ void __launch_bounds__(64) plan_scatter_kernel(const PlanParams p)
{
    extern __shared__ int32_t next[];
    const int lane = threadIdx.x;
    for (int e = lane; e < p.n_experts; e += 64) next[e] = p.counts[(int64_t)blockIdx.x * p.n_experts + e];
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kPlanChunk;
    const int64_t end = first + kPlanChunk < p.n_pairs ? first + kPlanChunk : p.n_pairs;
    for (int64_t at = first; at < end; at += 64) {
        const int id = expert_of(p.ids, at + lane, end, p.n_experts);
        const uint64_t same = same_id(id, p.bits);
        const int before = __popcll(same & ((1ull << lane) - 1));
        if (id < p.n_experts) p.order[next[id] + before] = (int32_t)(at + lane);
        __syncthreads();
        if (id < p.n_experts && before == 0) next[id] += __popcll(same);
        __syncthreads();
    }
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
};

template <int TY>
__device__ __forceinline__ void load8(const void *p, int64_t i, float (&x)[8])
{
    if constexpr (TY == VBR_F32) {
        const float4v a = *reinterpret_cast<const float4v *>(static_cast<const float *>(p) + i), b = *reinterpret_cast<const float4v *>(static_cast<const float *>(p) + i + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = a[j];
            x[j + 4] = b[j];
        }
    } else if constexpr (TY == VBR_F16) {
        const half8v a = *reinterpret_cast<const half8v *>(static_cast<const _Float16 *>(p) + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)a[j];
    } else {
        const bf16x8v a = *reinterpret_cast<const bf16x8v *>(static_cast<const __bf16 *>(p) + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)a[j];
    }
}

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

// A thread owns eight columns of a row of out; the row's results are added in the order of their places.
template <int TY, int TO>
__global__ void __launch_bounds__(kRouteThreads) route_combine_kernel(const CombineParams p)
{
    const int64_t at = (int64_t)blockIdx.x * kRouteThreads + threadIdx.x;
    const int64_t row = at / p.n_chunks;
    const int col = (int)(at - row * p.n_chunks) * 8;
    if (row >= p.n_rows) return;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    for (int j = 0; j < p.top_k; ++j) {
        const int64_t pair = row * p.top_k + j;
        if ((uint32_t)p.ids[pair] >= (uint32_t)p.n_experts) continue;
        const float w = p.weights[pair];
        float x[8];
        load8<TY>(p.y, pair * p.ldy + col, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(w, x[i], sum[i]);
    }
    store8<TO>(p.out, row * p.ldo + col, sum);
}

// A wave owns a pair: dy = w dout, dw = dout . y.  The k waves of a row read its dout from the caches.
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
        load8<TO>(p.dout, row * p.ldo + col, g);
        if (there) {
            load8<TY>(p.y, pair * p.ldy + col, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) dot = __builtin_fmaf(g[i], x[i], dot);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = there ? g[i] * w : 0.f;
        store8<TY>(p.dy, pair * p.lddy + col, g);
    }
    dot = wave_sum(dot);
    if (lane == 0) p.dweights[pair] = dot;
}

int launched()
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        set_last_hip_error((int)e);
        return VBR_EHIP;
    }
    return VBR_OK;
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
bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
int64_t up(int64_t x, int64_t q) { return (x + q - 1) / q * q; }

#define ROUTE_LAUNCH(KERNEL, TY, V) hipLaunchKernelGGL((KERNEL<TY, V>), dim3(grid), dim3(kRouteThreads), 0, stream, p)
#define ROUTE_BY_WIDTH(KERNEL, TY)                        \
    do {                                                  \
        if (n_experts <= 64) ROUTE_LAUNCH(KERNEL, TY, 1);       \
        else if (n_experts <= 128) ROUTE_LAUNCH(KERNEL, TY, 2); \
        else if (n_experts <= 256) ROUTE_LAUNCH(KERNEL, TY, 4); \
        else if (n_experts <= 512) ROUTE_LAUNCH(KERNEL, TY, 8); \
        else ROUTE_LAUNCH(KERNEL, TY, 16);                \
    } while (0)
#define ROUTE_BY_TYPE(KERNEL, type)                       \
    do {                                                  \
        if (type == VBR_F32) ROUTE_BY_WIDTH(KERNEL, VBR_F32);      \
        else if (type == VBR_F16) ROUTE_BY_WIDTH(KERNEL, VBR_F16); \
        else ROUTE_BY_WIDTH(KERNEL, VBR_BF16);            \
    } while (0)

}  // namespace

// Rows of a tile of the products: by how many pairs an expert has if all have alike.
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
    q.n_chunks = (n_pairs + kPlanChunk - 1) / kPlanChunk;
    q.order = up(4 * ((int64_t)n_experts + 1), 256);
    q.tiles = up(q.order + 4 * n_pairs, 256);
    q.counts = up(q.tiles + (int64_t)sizeof(PlanTile) * q.n_tiles, 256);
    q.total = up(q.counts + 4 * q.n_chunks * n_experts, 256);
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
    p.sigmoid = how->score == VBR_SIGMOID;
    p.renormalise = how->renormalise != 0;
    p.scored = bias_dev != nullptr || how->n_groups > 1;
    p.scale = how->scale;
    const int n_experts = how->n_experts;
    const unsigned grid = (unsigned)((n_rows + kRouteThreads / 64 - 1) / (kRouteThreads / 64));
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
    const int n_experts = how->n_experts;
    const unsigned grid = (unsigned)((n_rows + kRouteThreads / 64 - 1) / (kRouteThreads / 64));
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
    p.n_chunks = (int32_t)q.n_chunks;
    p.tile_rows = q.tile_rows;
    p.n_tiles = (int32_t)q.n_tiles;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const unsigned lds = 4 * ((unsigned)n_experts + 1);
    if (n_pairs > 0) hipLaunchKernelGGL(plan_count_kernel, dim3((unsigned)q.n_chunks), dim3(64), lds, stream, p);
    hipLaunchKernelGGL(plan_scan_kernel, dim3(1), dim3(kScanThreads), 0, stream, p);
    if (n_pairs > 0) hipLaunchKernelGGL(plan_scatter_kernel, dim3((unsigned)q.n_chunks), dim3(64), lds, stream, p);
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
    const int64_t grid = (n_rows * p.n_chunks + kRouteThreads - 1) / kRouteThreads;
    if (grid > INT32_MAX) return VBR_EUNSUPPORTED;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    COMBINE_BY_TYPES(route_combine_kernel);
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
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    COMBINE_BY_TYPES(route_combine_grad_kernel);
    return launched();
}
