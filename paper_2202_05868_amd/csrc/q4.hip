// Products with matrices in 4 bits: Y = X W^T, W[n][k] = s[n][k / group] (c[n][k] - z[n][k / group]), c and z in 0 .. 15.
//
// The mathematics.  With the code in the upper bits of the mantissa, 16 + c is an fp16 or bf16 number as it stands: one rotation and one
// and-or make two of them.  The matrix units sum (16 + c) x over a group exactly as products, in fp32; with the sum of x over the group,
//   y = sum over groups s (sum_k (16 + c_k) x_k - (16 + z) sum_k x_k),
// so scale and zero point are applied to sums in fp32, once a group, and no weight is ever rounded.  sum_k x_k comes from the matrix units as well,
// as a product with ones.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>
#include <type_traits>

#include "route.h"
#include "vbr_device.h"

// A tile is 16 rows (of one half, if gated) and 128 columns: 1 KiB of codes, 16 bytes a lane.  Lane 16 q + n has row n; its word i has the
// columns 32 i + 8 q .. + 7, in the order that the rotations take them apart.  Tiles of a row follow each other; with a gate the tiles of 16
// gate rows stand before those of the 16 rows they gate.  Scales and zero points are [tile row][step][16 rows][groups of a step], a step being a tile's
// 128 columns, or a group where that is longer: one load each a lane and step.
struct q4 {
    int64_t n_mats = 0, n_rows = 0, n_cols = 0;
    int32_t group = 0, dtype = 0;
    bool zeros = false, gated = false;
    int64_t rows() const { return gated ? n_rows / 2 : n_rows; }                     // of a half
    int64_t tile_rows() const { return (rows() + 15) / 16 * (gated ? 2 : 1); }      // of a matrix
    int64_t k_tiles() const { return (n_cols + 127) / 128; }
    int64_t groups() const { return (n_cols + group - 1) / group; }
    int32_t groups_a_step() const { return group < 128 ? 128 / group : 1; }
    int64_t steps() const { return group < 128 ? k_tiles() : groups(); }
    int64_t kept() const { return n_mats * tile_rows() * steps() * 16 * groups_a_step(); }
    int64_t scales_at() const { return n_mats * tile_rows() * k_tiles() * 1024; }
    int64_t zeros_at() const { return scales_at() + 2 * kept(); }
    int64_t total() const { return (zeros_at() + (zeros ? kept() : 0) + 255) / 256 * 256; }
    void *dev = nullptr;
};

namespace vbrk {
namespace {

// ---- laying out
struct PackParams {
    const uint8_t *codes, *zeros;
    const uint16_t *scales;
    uint4v *tiles;
    uint16_t *kept_scales;
    uint8_t *kept_zeros;
    int64_t n_tiles, n_kept;
    int64_t n_rows, half, n_cols, tile_rows, k_tiles, groups, steps;
    int32_t gated, rotate, groups_a_step, words;      // words: rows of codes can be read 4 bytes at a time only
};

__device__ __forceinline__ int64_t source_row(const PackParams &p, int64_t tile_row, int n)       // in its matrix; -1: none
{
    const int64_t in_half = (p.gated ? tile_row / 2 : tile_row) * 16 + n;
    return in_half < p.half ? in_half + (p.gated && (tile_row & 1) ? p.half : 0) : -1;
}

// A wave turns tiles one after the other: lane 16 j + n reads the codes of columns 32 j .. 32 j + 31 of row n, four words, and the lanes of a row exchange
// them, so that lane 16 q + n has word q of each.
constexpr int kPackTiles = 8;          // of a wave
__global__ void __launch_bounds__(256) q4_pack_codes_kernel(const PackParams p)
{
    const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
    const int64_t first = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kPackTiles;
    int64_t row_of_all = first / p.k_tiles, t = first - row_of_all * p.k_tiles, mat = row_of_all / p.tile_rows, tile_row = row_of_all - mat * p.tile_rows;
    for (int64_t tile = first; tile < first + kPackTiles && tile < p.n_tiles; ++tile) {
        const int64_t row = source_row(p, tile_row, n), k = t * 128 + 32 * j;
        uint4v w = {0, 0, 0, 0};
        if (row >= 0 && k < p.n_cols) {
            const uint8_t *src = p.codes + (mat * p.n_rows + row) * (p.n_cols / 2) + k / 2;
            if (p.words) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const uint32_t *>(src)[i];
            } else {
                w = *reinterpret_cast<const uint4v *>(src);
            }
        }
        auto swap = [](auto a, auto b, auto f, uint4v &w) {
            const auto r = f(w[a.value], w[b.value]);
            w[a.value] = (uint32_t)r[0];
            w[b.value] = (uint32_t)r[1];
        };
        const auto far = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane32_swap(a, b, false, false); };
        const auto near = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane16_swap(a, b, false, false); };
        swap(constant<0>(), constant<2>(), far, w);
        swap(constant<1>(), constant<3>(), far, w);
        swap(constant<0>(), constant<1>(), near, w);
        swap(constant<2>(), constant<3>(), near, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t codes = w[i];
            uint32_t word = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) word |= (codes >> 8 * u & 15u) << 4 * u | (codes >> (8 * u + 4) & 15u) << (4 * u + 16);
            w[i] = word << p.rotate | word >> (32 - p.rotate);
        }
        p.tiles[tile * 64 + lane] = w;
        if (++t == p.k_tiles) {
            t = 0;
            if (++tile_row == p.tile_rows) {
                tile_row = 0;
                ++mat;
            }
        }
    }
}

__global__ void __launch_bounds__(256) q4_pack_scales_kernel(const PackParams p)
{
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < p.n_kept; at += (int64_t)gridDim.x * 256) {
        const int in_step = (int)(at % p.groups_a_step);
        const int64_t of_step = at / p.groups_a_step;
        const int n = of_step & 15;
        const int64_t g = (of_step >> 4) % p.steps * p.groups_a_step + in_step, row_of_all = (of_step >> 4) / p.steps, mat = row_of_all / p.tile_rows;
        const int64_t row = source_row(p, row_of_all - mat * p.tile_rows, n), from = (mat * p.n_rows + row) * p.groups + g;
        const bool there = row >= 0 && g < p.groups;
        p.kept_scales[at] = there ? p.scales[from] : 0;
        if (p.kept_zeros) p.kept_zeros[at] = there ? p.zeros[from] : 0;
    }
}

// ---- the products

struct MmParams {
    const uint4v *tiles;
    const char *scales, *zeros;
    const uint16_t *X;
    void *Y;
    int64_t ldx, ldy, n_rows;                  // rows of Y
    int64_t k_tiles, tile_rows, steps;
    uint32_t x_bytes, ldx_bytes;               // of X from its first element to its last; of a row to the next; 0 where that is beyond 32 bits
    int32_t half, k_chunks, lg_waves;          // k_chunks: columns / 32; lg_waves: of the waves of a workgroup that share the columns (of a pair)
    uint32_t step_divide;                      // tile t is of step t, or t step_divide >> 32 where that is not zero
    int32_t gated, f32, fours;                 // fours: four elements of Y from a multiple of four on are aligned to as much
    int32_t col_blocks;                        // of the launch: workgroup i has tile of rows i / col_blocks
    Divide by_col_blocks;
    int32_t follow;                            // of a plan's tiles: an XCD has some that follow each other
    // routed, or null
    const PlanTile *plan_tiles;
    int32_t lg_parts;                          // of a plan's tile: 2^lg_parts tiles of this product
    const int32_t *order;
    const int32_t *ids;                        // or, of pairs that each have a tile of their own, these and how many matrices there are
    int32_t n_mats;
    const float *weights;                      // of the pairs, of a sum over top_k of them in bf16 or not
    int32_t top_k, bf16;
    Divide by_places;                          // the pairs of a row of X
};

template <int DT>
__device__ __forceinline__ float as_f32(uint16_t x)
{
    if constexpr (DT == VBR_F16) return (float)__builtin_bit_cast(_Float16, x);
    else return __builtin_bit_cast(float, (uint32_t)x << 16);
}

// Eight numbers 16 + c out of a word.  One instruction takes a constant of this size from a scalar register and one from a vector register, and
// none from its own code: they are kept in registers.
template <int DT>
struct SixteenPlus {
    uint32_t mask = DT == VBR_F16 ? 0x03C003C0u : 0x00780078u, base = DT == VBR_F16 ? 0x4C004C00u : 0x41804180u;
    __device__ __forceinline__ SixteenPlus()
    {
        asm volatile("" : "+s"(mask));
        asm volatile("" : "+v"(base));
    }
    __device__ __forceinline__ short8v operator()(uint32_t w) const
    {
        uint4v r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = ((j ? __builtin_amdgcn_alignbit(w, w, 4 * j) : w) & mask) | base;
        return __builtin_bit_cast(short8v, r);
    }
};

// the scales and zero points of a lane's row of W for one step: N groups
template <int N>
struct Words {
    using Scales = std::conditional_t<N == 1, uint16_t, std::conditional_t<N == 2, uint32_t, uint64_t>>;
    using Zeros = std::conditional_t<N == 1, uint8_t, std::conditional_t<N == 2, uint16_t, uint32_t>>;
    Scales s;
    Zeros z;
    template <int DT>
    __device__ __forceinline__ float scale(int i) const { return as_f32<DT>((uint16_t)(s >> (N > 1 ? 16 * i : 0))); }
    __device__ __forceinline__ float minus_sixteen_plus_zero(int i) const { return -16.f - (float)(uint8_t)(z >> (N > 1 ? 8 * i : 0)); }
};
// x / (1 + exp(-x)) for any x, off by eight half steps of its size at most (three of the exponential, two of the reciprocal, one of the sum and of each product): x / (1 + e) or
// x e / (1 + e) with e = exp(-|x|), which does not overflow.  NaN stays NaN; below -87, where e is below the normal fp32 numbers, it may be zero.
__device__ __forceinline__ float silu(float x) { return x * sigmoid_of(x); }

template <int DT>
__device__ __forceinline__ void store_y(const MmParams &p, int64_t at, float y)
{
    if (p.f32) static_cast<float *>(p.Y)[at] = y;
    else if constexpr (DT == VBR_F16) static_cast<_Float16 *>(p.Y)[at] = (_Float16)y;
    else static_cast<__bf16 *>(p.Y)[at] = (__bf16)y;
}

// four columns of a row that begins at element `row`; they are stored together where that is a whole number of them
template <int DT>
__device__ __forceinline__ void store_4(const MmParams &p, int64_t row, int64_t col, float4v y)
{
    if (p.fours && col + 4 <= p.half) {
        if (p.f32) {
            *reinterpret_cast<float4v *>(static_cast<float *>(p.Y) + row + col) = y;
        } else if constexpr (DT == VBR_F16) {
            typedef _Float16 half4v __attribute__((ext_vector_type(4)));
            *reinterpret_cast<half4v *>(static_cast<_Float16 *>(p.Y) + row + col) = __builtin_convertvector(y, half4v);
        } else {
            typedef __bf16 bf16x4v __attribute__((ext_vector_type(4)));
            *reinterpret_cast<bf16x4v *>(static_cast<__bf16 *>(p.Y) + row + col) = __builtin_convertvector(y, bf16x4v);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < p.half) store_y<DT>(p, row + col + i, y[i]);
}

// rows first .. first + count - 1 (positions of the plan's order, if routed) of matrix mat
struct RowTile {
    int64_t mat, first;
    int32_t count;
};
__device__ __forceinline__ RowTile row_tile(const MmParams &p, int tile, int rows)      // count 0: none
{
    if (p.order) {
        const PlanTile t = p.plan_tiles[tile >> p.lg_parts];
        const int at = (tile & ((1 << p.lg_parts) - 1)) * rows, left = t.count - at;
        return {t.expert, t.first + at, left < 0 ? 0 : left < rows ? left : rows};
    }
    if (p.ids) {
        const int32_t id = p.ids[tile];
        return {id, tile, (uint32_t)id < (uint32_t)p.n_mats ? 1 : 0};
    }
    const int64_t first = (int64_t)tile * rows, left = p.n_rows - first;
    return {0, first, (int32_t)(left < rows ? left : rows)};
}
__device__ __forceinline__ int64_t x_row(const MmParams &p, int64_t y_row) { return p.order || p.ids ? (int64_t)p.by_places((uint32_t)y_row) : y_row; }
__device__ __forceinline__ uint32_t step_of(const MmParams &p, int t) { return p.step_divide ? __umulhi((uint32_t)t, p.step_divide) : (uint32_t)t; }

// The steps of a part of the columns, begun at another one in every workgroup: rows of X and W are powers of two apart more often than
// not, and what is read at the same time should not lie in the same channels.
struct Steps {
    int begin, count, turn, n_tiles;
    __device__ __forceinline__ Steps(const MmParams &p, int part, int lg_parts, uint32_t workgroup) : n_tiles((int)p.k_tiles)
    {
        begin = n_tiles * part >> lg_parts;
        count = (n_tiles * (part + 1) >> lg_parts) - begin;
        turn = (int)((workgroup * 40503u & 0xFFFFu) * (uint32_t)count >> 16);
    }
    __device__ __forceinline__ int operator()(int u) const        // the tile of step u; behind the last one that one; without any, one that is there
    {
        const int v = (u < count ? u : count > 0 ? count - 1 : 0) + turn, t = begin + (v < count ? v : v - count);
        return t < n_tiles ? t : n_tiles - 1;
    }
};
__device__ __forceinline__ int64_t y_row(const MmParams &p, int64_t at) { return p.order ? p.order[at] : at; }

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

template <int DT>
__device__ __forceinline__ float sum_of_8(uint4v x)
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t two = x[j];                           // (a bit cast of x[j] itself takes x[0])
        if constexpr (DT == VBR_F16) s = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, two), half2v{1, 1}, s, false);
        else s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2v, two), bf16x2v{1, 1}, s, false);
    }
    return s;
}

// What (16 + z) takes from a sum is a product itself, of the sums of x in a group and s (16 + z): four groups at a time it goes to the matrix units in
// fp32, so that the vector units have one multiplication and addition a sum and group.

__device__ __forceinline__ float sum_over_quarters(float x)           // of lanes n, 16 + n, 32 + n and 48 + n, in all four
{
    const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    const float y = __builtin_bit_cast(float, (uint32_t)a[0]) + __builtin_bit_cast(float, (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, y), false, false);
    return __builtin_bit_cast(float, (uint32_t)b[0]) + __builtin_bit_cast(float, (uint32_t)b[1]);
}

__device__ __forceinline__ float sum_over_halves(float x)             // of lanes n and 32 + n, in both
{
    const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return __builtin_bit_cast(float, (uint32_t)b[0]) + __builtin_bit_cast(float, (uint32_t)b[1]);
}

// sums [n_waves][NT][row][kSumRow], so that a lane's four are 16 bytes and rows fall on different banks; added in the waves' order and stored
constexpr int kSumRow = 20;
template <int DT, int NT, int ROWS>
__device__ __forceinline__ void store_sums(const MmParams &p, const RowTile &rt, int64_t r0, const float *sums, int n_waves)
{
    const int halves = p.gated ? 2 : 1, lg = (NT == 1 ? 2 : NT == 2 ? 3 : 4) - (p.gated ? 1 : 0);      // 2^lg threads have four columns each of a row
    const int h0 = (threadIdx.x >> 2 & ((1 << (lg - 2)) - 1)) * halves, c0 = (threadIdx.x & 3) * 4;
    const int64_t out_col = ((r0 + h0) >> (halves - 1)) * 16 + c0;
    for (int token = threadIdx.x >> lg; token < rt.count; token += blockDim.x >> lg) {
        auto sum = [&](int h) {
            float4v v = {0, 0, 0, 0};
            for (int k = 0; k < n_waves; ++k) v += *reinterpret_cast<const float4v *>(sums + ((k * NT + h) * ROWS + token) * kSumRow + c0);
            return v;
        };
        float4v v = sum(h0);
        if (p.gated) {
            const float4v up = sum(h0 + 1);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = silu(v[i]) * up[i];
        }
        store_4<DT>(p, y_row(p, rt.first + token) * p.ldy, out_col, v);
    }
}

// ---- up to 16 rows of X: a workgroup has them all and NT rows of tiles; its waves share the columns, each with a range of steps of its own, and nothing else
// before the end, where their sums are added in their order.  X comes from the L2 straight into registers, AHEAD_X steps ahead, W AHEAD_W.  CH: chunks of 32
// columns between applications of a scale (1, 2, or 4).
// Bound by the reading of W: 64 pairs that meet 40 of 64 matrices of 2816 x 2048 in groups of 64 take 25.8 us, 5.0 TB/s, which is what a large copy reaches.
// One row times 4096 x 4096 takes 4.6 us on the GPU, of which 2.5 are what any launch takes.

// The sums of the steps of tile_of: 16 rows of X times NT rows of tiles of a matrix from r0 on.  x_at: where this lane's row of X and its columns begin, or
// kNoRow of one that is not there, which is out of X's range, so that loads of it cost nothing.
constexpr uint32_t kNoRow = 0xFFFFF000u;
template <int DT, int CH, bool ZEROS, int NT, int AHEAD_W, int AHEAD_X>
__device__ __forceinline__ void split_sums(const MmParams &p, int64_t mat, int64_t r0, const Steps &tile_of, uint32_t x_at, int lane, float4v (&acc)[NT])
{
    constexpr int kGroups = 4 / CH;
    const int n = lane & 15, q = lane >> 4;
    const SixteenPlus<DT> sixteen_plus;
    const int64_t last = p.tile_rows - 1;
    const int further = (int)(last - r0 < NT ? last - r0 : NT - 1);
    const int64_t from = mat * p.tile_rows + r0;
    const char *w_at = reinterpret_cast<const char *>(p.tiles) + from * p.k_tiles * 1024;
    const char *s_at = p.scales + from * p.steps * (32 * kGroups), *z_at = p.zeros + from * p.steps * (16 * kGroups);
    const int n_tiles = tile_of.n_tiles, n_steps = tile_of.count;

    uint4v w[AHEAD_W][NT];
    Words<kGroups> sz[AHEAD_W][NT];
    short8v xf[AHEAD_X][4];
    auto fetch_w = [&](auto d, int h, int t) {
        const uint32_t hh = h < further ? h : further;
        w[d][h] = *reinterpret_cast<const uint4v *>(w_at + ((hh * (uint32_t)n_tiles + (uint32_t)t) * 1024u + (uint32_t)lane * 16u));
        const uint32_t at = (hh * (uint32_t)p.steps + step_of(p, t)) * 16u + (uint32_t)n;
        sz[d][h].s = *reinterpret_cast<const typename Words<kGroups>::Scales *>(s_at + at * (2u * kGroups));
        if constexpr (ZEROS) sz[d][h].z = *reinterpret_cast<const typename Words<kGroups>::Zeros *>(z_at + at * (uint32_t)kGroups);
    };
    static_for<AHEAD_W>([&](auto d) {
#pragma unroll
        for (int h = 0; h < NT; ++h) fetch_w(d, h, tile_of(d));
    });
    const __amdgpu_buffer_rsrc_t x_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(p.X), 0, (int)p.x_bytes, 0x00020000);
    auto fetch_x = [&](auto d, int t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int chunk = 4 * t + i < p.k_chunks ? 4 * t + i : p.k_chunks - 1;
            xf[d][i] = __builtin_bit_cast(short8v, __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, (int)x_at, 64 * chunk, 0));
        }
    };
    static_for<AHEAD_X>([&](auto d) { fetch_x(d, tile_of(d)); });

    float taken[NT], of_x = 0.f;                                       // -s (16 + z) and the sum of x of the q-th of four groups
#pragma unroll
    for (int h = 0; h < NT; ++h) {
        acc[h] = float4v{0, 0, 0, 0};
        taken[h] = 0.f;
    }
    auto take = [&]() {
#pragma unroll
        for (int h = 0; h < NT; ++h) {
            acc[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(of_x, taken[h], acc[h], 0, 0, 0);
            taken[h] = 0.f;
        }
    };
    auto step = [&](auto d, auto more_w, auto more_x, int u) {
        constexpr int dx = d.value % AHEAD_X;
        const int t = tile_of(u);
        if (4 * t + 4 > p.k_chunks) {                              // the last columns are fewer
#pragma unroll
            for (int i = 1; i < 4; ++i)
                if (4 * t + i >= p.k_chunks) xf[dx][i] = short8v{0, 0, 0, 0, 0, 0, 0, 0};
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int slot = ((AHEAD_W % 4 == 0 ? d.value : u) * kGroups + g) & 3;
            float sum = 0.f;
#pragma unroll
            for (int i = g * CH; i < (g + 1) * CH; ++i) sum += sum_of_8<DT>(__builtin_bit_cast(uint4v, xf[dx][i]));
            sum = sum_over_quarters(sum);
            of_x = q == slot ? sum : of_x;
#pragma unroll
            for (int h = 0; h < NT; ++h) {
                float4v part = float4v{0, 0, 0, 0};
#pragma unroll
                for (int i = g * CH; i < (g + 1) * CH; ++i) {
                    const short8v b = sixteen_plus(w[d][h][i]);
                    part = mfma16x16x32<DT>(xf[dx][i], b, part);
                }
                const float s = sz[d][h].template scale<DT>(g);
                if constexpr (CH == 1) {
                    if (g == 0) taken[h] = sz[d][h].template scale<DT>(q) * (ZEROS ? sz[d][h].minus_sixteen_plus_zero(q) : -24.f);
                } else {
                    taken[h] = q == slot ? s * (ZEROS ? sz[d][h].minus_sixteen_plus_zero(g) : -24.f) : taken[h];
                }
                if (more_w.value && g == kGroups - 1) fetch_w(d, h, tile_of(u + AHEAD_W));
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[h][i] = __builtin_fmaf(s, part[i], acc[h][i]);
            }
            if (g == kGroups - 1 && slot == 3) take();
        }
        if constexpr (more_x.value) fetch_x(constant<dx>(), tile_of(u + AHEAD_X));
    };
    // No load stands in a branch, so that every wait is for the oldest ones and not for all.
    int first = 0;
    for (; first + AHEAD_W < n_steps; first += AHEAD_W)
        static_for<AHEAD_W>([&](auto d) { step(d, constant<1>(), constant<1>(), first + d); });
    static_for<AHEAD_W>([&](auto d) {
        if (first + d < n_steps) step(d, constant<0>(), constant<(d.value + AHEAD_X < AHEAD_W)>(), first + d);
    });
    if constexpr (CH > 1) take();                                      // what is left of four groups; of the others taken is zero
}

template <int DT, int CH, bool ZEROS, int NT, int AHEAD_W, int AHEAD_X, int THREADS>
__global__ void __launch_bounds__(THREADS) q4_split_kernel(const MmParams p)
{
    constexpr int kRows = 16;
    extern __shared__ __attribute__((aligned(16))) float sums[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, q = lane >> 4;
    const uint32_t tile = p.by_col_blocks(blockIdx.x), col_block = blockIdx.x - tile * p.col_blocks;
    const RowTile rt = row_tile(p, tile, kRows);
    if (rt.count == 0) return;
    const int64_t r0 = (int64_t)col_block * NT;
    const uint32_t x_at = n < rt.count ? (uint32_t)x_row(p, y_row(p, rt.first + n)) * p.ldx_bytes + 16 * q : kNoRow;
    float4v acc[NT];
    split_sums<DT, CH, ZEROS, NT, AHEAD_W, AHEAD_X>(p, rt.mat, r0, Steps(p, wave, p.lg_waves, col_block), x_at, lane, acc);
    float *mine = sums + (int64_t)wave * NT * kRows * kSumRow;
#pragma unroll
    for (int h = 0; h < NT; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[(h * kRows + 4 * q + i) * kSumRow + n] = acc[h][i];
    __syncthreads();
    store_sums<DT, NT, kRows>(p, rt, r0, sums, 1 << p.lg_waves);
}

// ---- the products and the weighted sum behind them at once: a row of Y is the sum over a row's pairs of their weights times what their matrices give of the
// pairs' rows of X.  A workgroup has a row of tiles; each of its waves takes pairs, or parts of their columns where pairs are fewer than waves, and its sums are
// added in the waves' order.  A launch less, and no results on their way through memory: a layer for one row, 8 of 128 experts of 2 x 768 x 2048 and 2048 x 768,
// 12.0 us, 15.3 with a product and a sum.  What is left of it are two launches whose reads, 20 MB, take 4 us and follow the calls' latencies.
constexpr int kSumWaves = 8;
template <int DT, int CH, bool ZEROS>
__global__ void __launch_bounds__(64 * kSumWaves) q4_sum_kernel(const MmParams p)
{
    __shared__ float sums[kSumWaves][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t row = p.by_col_blocks(blockIdx.x), col_block = blockIdx.x - row * p.col_blocks;
    float sum = 0.f;                                                   // of column lane % 16
    for (int unit = wave; unit < p.top_k << p.lg_waves; unit += kSumWaves) {
        const int pair = (int)row * p.top_k + (unit >> p.lg_waves);
        const int32_t id = p.ids[pair];
        if ((uint32_t)id >= (uint32_t)p.n_mats) continue;
        float4v acc[1];
        split_sums<DT, CH, ZEROS, 1, 4, 2>(p, id, col_block, Steps(p, unit & ((1 << p.lg_waves) - 1), p.lg_waves, blockIdx.x),
                                           (lane & 15) == 0 ? (uint32_t)pair * p.ldx_bytes + 16 * (lane >> 4) : kNoRow, lane, acc);
        sum = __builtin_fmaf(p.weights[pair], acc[0][0], sum);         // the first of the sixteen rows, in the first sixteen lanes
    }
    if (lane < 16) sums[wave][lane] = sum;
    __syncthreads();
    const int64_t col = (int64_t)col_block * 16 + threadIdx.x;
    if (threadIdx.x >= 16 || col >= p.half) return;
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < kSumWaves; ++w) y += sums[w][threadIdx.x];
    const int64_t at = row * p.ldy + col;
    if (p.f32) static_cast<float *>(p.Y)[at] = y;
    else if (p.bf16) static_cast<__bf16 *>(p.Y)[at] = (__bf16)y;
    else static_cast<_Float16 *>(p.Y)[at] = (_Float16)y;
}

// ---- more rows than 16: by products of 32 rows with 32 rows of W, which the matrix units take at 1.4 times the rate of those with 16.  Two rows of tiles are
// side by side: lane 32 h + 16 b + n has row n of the b-th, and of its sixteen blocks of eight columns every second from the h-th on.
typedef float float16v __attribute__((ext_vector_type(16)));

template <int DT>
__device__ __forceinline__ float16v mfma32x32x16(short8v a, short8v b, float16v c)
{
    if constexpr (DT == VBR_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8v, a), __builtin_bit_cast(bf16x8v, b), c, 0, 0, 0);
}

// A wave's part of W: two pairs of rows of tiles from r0 on (behind the last one, that one), and the products with 32 MT rows of X.
template <int DT, int CH, bool ZEROS, int MT>
struct Pairs {
    static constexpr int kGroups = 4 / CH;
    uint4v w[2][2];
    Words<kGroups> sz[2];
    float16v acc[MT][2];
    float taken[2];                                              // -s (16 + z) of this half's one of two groups
    SixteenPlus<DT> sixteen_plus;
    const char *w_at[2], *s_at[2], *z_at[2];

    __device__ __forceinline__ Pairs(const MmParams &p, int64_t mat, int64_t r0, int lane)
    {
        const int64_t last = p.tile_rows - 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t r = r0 + 2 * h + (lane >> 4 & 1), row = mat * p.tile_rows + (r < last ? r : last);
            w_at[h] = reinterpret_cast<const char *>(p.tiles) + row * p.k_tiles * 1024 + ((lane & 15) + 16 * (lane >> 5)) * 16;
            s_at[h] = p.scales + (row * p.steps * 16 + (lane & 15)) * (2 * kGroups);
            z_at[h] = p.zeros + (row * p.steps * 16 + (lane & 15)) * kGroups;
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[m][h] = float16v{};
            taken[h] = 0.f;
        }
    }
    __device__ __forceinline__ void fetch(const MmParams &p, int h, int t)
    {
        w[h][0] = *reinterpret_cast<const uint4v *>(w_at[h] + (uint32_t)t * 1024u);
        w[h][1] = *reinterpret_cast<const uint4v *>(w_at[h] + (uint32_t)t * 1024u + 512);
        const uint32_t step = step_of(p, t);
        sz[h].s = *reinterpret_cast<const typename Words<kGroups>::Scales *>(s_at[h] + step * (32u * kGroups));
        if constexpr (ZEROS) sz[h].z = *reinterpret_cast<const typename Words<kGroups>::Zeros *>(z_at[h] + step * (16u * kGroups));
    }
    // Group g of step u (a tile in the order they are taken), and the fetch of the next one with the last group.  x(m, i): 32 rows and columns 16 i .. of
    // the tile; of_x(m, g): the sum of x of row m 32 + lane % 32 in this half's one of the groups g - 1 and g.
    template <class X, class Sums>
    __device__ __forceinline__ void group(const MmParams &p, int g, int u, int next, bool final, int half, X x, Sums of_x)
    {
        const int slot = (CH == 4 ? u : g) & 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float16v part[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) part[m] = float16v{};
#pragma unroll
            for (int i = 2 * CH * g; i < 2 * CH * (g + 1); ++i) {
                const short8v b = sixteen_plus(w[h][i & 1][i >> 1]);
#pragma unroll
                for (int m = 0; m < MT; ++m) part[m] = mfma32x32x16<DT>(x(m, i), b, part[m]);
            }
            const float s = sz[h].template scale<DT>(g);
            if constexpr (CH == 4) taken[h] = half == slot ? s * (ZEROS ? sz[h].minus_sixteen_plus_zero(0) : -24.f) : taken[h];
            else if (slot == 1) taken[h] = sz[h].template scale<DT>(g - 1 + half) * (ZEROS ? sz[h].minus_sixteen_plus_zero(g - 1 + half) : -24.f);
            if (g == kGroups - 1) fetch(p, h, next);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[m][h][i] = __builtin_fmaf(s, part[m][i], acc[m][h][i]);
        }
        if (slot == 1 || (CH == 4 && final)) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float sum = half <= slot ? of_x(m, g) : 0.f;
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[m][h] = __builtin_amdgcn_mfma_f32_32x32x2f32(sum, half <= slot ? taken[h] : 0.f, acc[m][h], 0, 0, 0);
            }
        }
    }
};

// 32 rows times 32 columns of sums, the ones of a product's accumulators, to Y: through LDS (32 * kSumRow32 floats that only this wave uses), so that a lane has
// four columns of a row.  token0: their first row in the tile of rows; y_at(token): where that row of Y begins; r: their first row of tiles.
constexpr int kSumRow32 = 36;
template <int DT, class At>
__device__ __forceinline__ void store_32(const MmParams &p, int count, int token0, int64_t r, float *lds, const float16v &v, int lane, At y_at)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) lds[(8 * (i >> 2) + 4 * (lane >> 5) + (i & 3)) * kSumRow32 + (lane & 31)] = v[i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (p.gated) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int token = 16 * j + (lane >> 2), c = 4 * (lane & 3);
            float4v g = *reinterpret_cast<const float4v *>(lds + token * kSumRow32 + c);
            const float4v u = *reinterpret_cast<const float4v *>(lds + token * kSumRow32 + 16 + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = silu(g[i]) * u[i];
            if (token0 + token < count && r < p.tile_rows) store_4<DT>(p, y_at(token0 + token), r / 2 * 16 + c, g);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int token = 8 * j + (lane >> 3), c = 4 * (lane & 7);
            const float4v y = *reinterpret_cast<const float4v *>(lds + token * kSumRow32 + c);
            if (token0 + token < count) store_4<DT>(p, y_at(token0 + token), r * 16 + c, y);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Few workgroups: the division of the work as above (192 rows times 4096 x 14336 in groups of 128: 38.7 us, 583 TFLOP/s; the waits for X and the unpacking, which
// is done once for each 64 rows, stand between it and the 880 to 970 of the kernel below), with X through a part of LDS that each wave has for itself.  A wave's load takes 256 bytes of four rows
// (the pieces of 32 bytes that the matrix units take are a part of a line each, and the rest is gone from the L1 before it is asked for).  The rows of a
// step are read into registers at once and those of the next step fetched into their place.
template <int DT, int CH, bool ZEROS, int MT>
__global__ void __launch_bounds__(512) q4_mid_kernel(const MmParams p)
{
    constexpr int kGroups = 4 / CH, kRows = 32 * MT;
    extern __shared__ __attribute__((aligned(16))) float sums[];
    __shared__ const char *row_lds[kRows];                             // where the rows of X begin
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_waves = 1 << p.lg_waves, half = lane >> 5;
    const uint32_t tile = p.by_col_blocks(blockIdx.x), col_block = blockIdx.x - tile * p.col_blocks;
    const RowTile rt = row_tile(p, tile, kRows);
    if (rt.count == 0) return;
    const int64_t r0 = (int64_t)col_block * 4;
    const Steps tile_of(p, wave, p.lg_waves, col_block);
    const int n_steps = tile_of.count;
    Pairs<DT, CH, ZEROS, MT> pairs(p, rt.mat, r0, lane);
    // rows behind the last one are the first again, and never stored
    if (threadIdx.x < kRows)
        row_lds[threadIdx.x] = reinterpret_cast<const char *>(p.X + x_row(p, y_row(p, rt.first + ((int)threadIdx.x < rt.count ? threadIdx.x : 0))) * p.ldx);
    __syncthreads();
    // chunk c of row r of this wave's part is at 16 (16 r + (c ^ r % 16)); lane l of load j takes what comes to row 4 j + l / 16, place l % 16
    uint4v *mine_x = reinterpret_cast<uint4v *>(sums) + wave * (kRows * 16);
    const uint32_t x_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4v *)mine_x;
    auto fetch_x = [&](int t) {
        const uint32_t left = (uint32_t)(p.k_chunks - 4 * t) * 4u - 1u;       // the last chunk that is there
        static_for<kRows / 4>([&](auto j) {
            uint32_t c = (uint32_t)(lane & 15) ^ (uint32_t)(4 * (j.value & 3) + (lane >> 4));
            c = c < left ? c : left;
            dma16(row_lds[4 * j.value + (lane >> 4)] + ((uint32_t)t * 256u + c * 16u), x_base + j.value * 1024);
        });
    };
    fetch_x(tile_of(0));
    pairs.fetch(p, 0, tile_of(0));
    pairs.fetch(p, 1, tile_of(0));
    float of_x[MT];                                                    // the sum of x in this half's one of two groups
#pragma unroll
    for (int m = 0; m < MT; ++m) of_x[m] = 0.f;
    for (int u = 0; u < n_steps; ++u) {
        const int t = tile_of(u), next = tile_of(u + 1);
        // X of this step is there when nothing but the four loads of codes behind it is on its way (with them go those of scales and zero points)
        wait_vmcnt<4>();
        short8v xf[MT][8];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 8; ++i) xf[m][i] = __builtin_bit_cast(short8v, mine_x[(32 * m + (lane & 31)) * 16 + ((2 * i + half) ^ (lane & 15))]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // read before it is written again
        fetch_x(next);
        if (4 * t + 4 > p.k_chunks) {                                  // the last columns are fewer
#pragma unroll
            for (int i = 2; i < 8; ++i)
                if (4 * t + i / 2 >= p.k_chunks) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) xf[m][i] = short8v{0, 0, 0, 0, 0, 0, 0, 0};
                }
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int slot = (CH == 4 ? u : g) & 1;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                float s = 0.f;
#pragma unroll
                for (int i = 2 * CH * g; i < 2 * CH * (g + 1); ++i) s += sum_of_8<DT>(__builtin_bit_cast(uint4v, xf[m][i]));
                s = sum_over_halves(s);
                of_x[m] = half == slot ? s : of_x[m];
            }
            pairs.group(p, g, u, next, u + 1 == n_steps, half, [&](int m, int i) { return xf[m][i]; }, [&](int m, int) { return of_x[m]; });
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // The waves' sums are added pairwise from the back: half of them write, the other half adds, until one is left.
    wait_vmcnt<0>();                                                   // (the last step fetched its own again)
    __syncthreads();
    for (int rest = n_waves >> 1; rest > 0; rest >>= 1) {
        float4v *place = reinterpret_cast<float4v *>(sums) + (int64_t)(wave % rest) * (MT * 2 * 4 * 64) + lane;
        if (wave >= rest && wave < 2 * rest) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        place[((m * 2 + h) * 4 + i) * 64] = float4v{pairs.acc[m][h][4 * i], pairs.acc[m][h][4 * i + 1], pairs.acc[m][h][4 * i + 2], pairs.acc[m][h][4 * i + 3]};
        }
        __syncthreads();
        if (wave < rest) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4v o = place[((m * 2 + h) * 4 + i) * 64];
#pragma unroll
                        for (int j = 0; j < 4; ++j) pairs.acc[m][h][4 * i + j] += o[j];
                    }
        }
        __syncthreads();
    }
    // the first wave has them all: it hands every wave a share to store
    if (wave == 0) {
        float4v *place = reinterpret_cast<float4v *>(sums) + lane;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    place[((m * 2 + h) * 4 + i) * 64] = float4v{pairs.acc[m][h][4 * i], pairs.acc[m][h][4 * i + 1], pairs.acc[m][h][4 * i + 2], pairs.acc[m][h][4 * i + 3]};
    }
    __syncthreads();
    float *own = sums + MT * 2 * 1024 + wave * (32 * kSumRow32);
    for (int part = wave; part < MT * 2; part += n_waves) {
        float16v v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4v o = reinterpret_cast<const float4v *>(sums)[(part * 4 + i) * 64 + lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = o[j];
        }
        store_32<DT>(p, rt.count, part / 2 * 32, r0 + part % 2 * 2, own, v, lane, [&](int token) { return y_row(p, rt.first + token) * p.ldy; });
    }
}

// Many workgroups: 32 MT rows of X times 16 rows of tiles, by four waves with four rows of tiles each.  X goes through LDS, which all waves read; W
// comes straight into registers, as it was laid out, and is turned into numbers there.
// Bound by the issue of instructions: beside each product of 32 x 32 x 16, which takes the place of about six vector instructions, stand for 64 rows 3.5 that make
// numbers of W (seven for two products), 2 that apply a scale (groups of 128) and the loads from LDS.  2048 rows times 8192 x 8192 reach 880 to 970 TFLOP/s with zero points
// and 920 to 1005 without, from card to card; a product of bf16 with bf16 of the library reaches 1186 at 8192 x 8192 x 8192.
template <int CTRL>
__device__ __forceinline__ float add_lane(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

template <int DT, int CH, bool ZEROS, int MT>
__global__ void __launch_bounds__(256, 2) q4_many_kernel(const MmParams p)
{
    constexpr int kRows = 32 * MT, kGroups = 4 / CH, kSums = CH == 1 ? 8 : 4, kLoads = kRows / 16;
    constexpr int kXBytes = 2 * kRows * 256, kOutBytes = 4 * 32 * kSumRow32 * 4;
    __shared__ __attribute__((aligned(16))) char lds[kXBytes > kOutBytes ? kXBytes : kOutBytes];
    __shared__ float sum_lds[kSums][kRows];                                      // of the groups of two tiles, or of four tiles
    __shared__ int64_t y_lds[kRows];                                             // where the rows of Y begin
    uint4v(*x_lds)[kRows * 16] = reinterpret_cast<uint4v(*)[kRows * 16]>(lds);   // chunk c of row r at r * 16 + (c ^ r % 16)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    // Workgroups go to the eight XCDs in turn.  Where an expert has few tiles, each XCD gets some that follow each other, whose rows of X, and of their expert's W,
    // its L2 then reads once.  Else each XCD has some columns of Y in turn, and their W.
    uint32_t place = blockIdx.x;
    if (p.follow) {
        const uint32_t work = ((uint32_t)p.plan_tiles[0].n_tiles << p.lg_parts) * (uint32_t)p.col_blocks, share = (work + 7) / 8;
        place = (blockIdx.x & 7) * share + (blockIdx.x >> 3);
        if (blockIdx.x >> 3 >= share || place >= work) return;
    }
    const uint32_t tile = p.by_col_blocks(place), col_block = place - tile * p.col_blocks;
    const RowTile rt = row_tile(p, tile, kRows);
    if (rt.count == 0) return;
    const int64_t r0 = ((int64_t)col_block * 4 + wave) * 4;
    Pairs<DT, CH, ZEROS, MT> pairs(p, rt.mat, r0, lane);
    pairs.fetch(p, 0, 0);
    pairs.fetch(p, 1, 0);

    // this thread's chunks of X: chunk c of rows xr + 16 j
    const int c = threadIdx.x & 15, xr = threadIdx.x >> 4;
    const uint16_t *src[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int64_t row = y_row(p, rt.first + (xr + 16 * j < rt.count ? xr + 16 * j : 0));
        if (c == 0) y_lds[xr + 16 * j] = row * p.ldy;
        src[j] = p.X + x_row(p, row) * p.ldx + 8 * c;
    }
    uint4v xv[kLoads];
    auto fetch_x = [&](int t) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            xv[j] = uint4v{0, 0, 0, 0};
            if (4 * t + (c >> 2) < p.k_chunks) xv[j] = *reinterpret_cast<const uint4v *>(src[j] + 128 * (int64_t)t);
        }
    };
    auto put_x = [&](int t) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            x_lds[t & 1][(xr + 16 * j) * 16 + (c ^ (xr & 15))] = xv[j];
            float s = sum_of_8<DT>(xv[j]);
            s = add_lane<0x4E>(add_lane<0xB1>(s));            // over four lanes, then eight, then sixteen
            if constexpr (CH >= 2) s = add_lane<0x141>(s);
            if constexpr (CH == 4) s = add_lane<0x140>(s);
            if (c % (4 * CH) == 0) sum_lds[(t * kGroups + c / (4 * CH)) % kSums][xr + 16 * j] = s;
        }
    };
    const int n_tiles = (int)p.k_tiles;
    fetch_x(0);
    put_x(0);
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
        const int next = t + 1 < n_tiles ? t + 1 : t;
        fetch_x(next);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            short8v xf[MT][2 * CH];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 2 * CH; ++i) xf[m][i] = __builtin_bit_cast(short8v, x_lds[t & 1][(32 * m + (lane & 31)) * 16 + ((2 * (g * 2 * CH + i) + half) ^ (lane & 15))]);
            pairs.group(p, g, t, next, t + 1 == n_tiles, half, [&](int m, int i) { return xf[m][i - g * 2 * CH]; },
                        [&](int m, int g) { return sum_lds[((CH == 4 ? t & ~1 : t * kGroups + g - 1) + half) % kSums][32 * m + (lane & 31)]; });
            __builtin_amdgcn_sched_barrier(0);                    // (groups taken up at once take registers that are not there)
        }
        if (t + 1 < n_tiles) put_x(t + 1);
        __syncthreads();
    }
    float *own = reinterpret_cast<float *>(lds) + wave * (32 * kSumRow32);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) store_32<DT>(p, rt.count, 32 * m, r0 + 2 * h, own, pairs.acc[m][h], lane, [&](int token) { return y_lds[token]; });
}

using MmKernel = void (*)(MmParams);
struct Variant {
    MmKernel kernel;
    int32_t tile_rows, threads, lds;                   // of a workgroup
};
template <int DT, int CH, bool ZEROS, int NT, int AHEAD_W, int AHEAD_X, int THREADS>
Variant split_variant(int waves)
{
    return {q4_split_kernel<DT, CH, ZEROS, NT, AHEAD_W, AHEAD_X, THREADS>, NT, 64 * waves, waves * NT * 16 * kSumRow * 4};
}
template <int DT, int CH, bool ZEROS, int MT>
Variant mid_variant(int waves)
{
    const int x = waves * 32 * MT * 256, halves = waves / 2 * MT * 2 * 4096, out = MT * 2 * 4096 + waves * 32 * kSumRow32 * 4;
    return {q4_mid_kernel<DT, CH, ZEROS, MT>, 4, 64 * waves, std::max(x, std::max(halves, out))};
}

// The variant for `rows` rows of a tile of rows (16, 32 or 64): nt rows of tiles a workgroup (16 of more than 16 rows: the kernel for many workgroups).
struct Choice {
    int32_t rows, nt, waves;
};
template <int DT, int CH, bool ZEROS>
Variant mm_variant(const Choice &c)
{
    if (c.rows == 16)
        return c.nt == 1 ? split_variant<DT, CH, ZEROS, 1, 4, 2, 512>(c.waves) : c.nt == 2 ? split_variant<DT, CH, ZEROS, 2, 1, 1, 512>(c.waves) : split_variant<DT, CH, ZEROS, 4, 2, 2, 256>(c.waves);
    if (c.nt == 4) return c.rows == 32 ? mid_variant<DT, CH, ZEROS, 1>(c.waves) : mid_variant<DT, CH, ZEROS, 2>(c.waves);
    return c.rows == 32 ? Variant{q4_many_kernel<DT, CH, ZEROS, 1>, 16, 256, 0} : Variant{q4_many_kernel<DT, CH, ZEROS, 2>, 16, 256, 0};
}
template <int DT>
Variant mm_variant(int32_t group, bool zeros, const Choice &c)
{
    if (group == 32) return zeros ? mm_variant<DT, 1, true>(c) : mm_variant<DT, 1, false>(c);
    if (group == 64) return zeros ? mm_variant<DT, 2, true>(c) : mm_variant<DT, 2, false>(c);
    return zeros ? mm_variant<DT, 4, true>(c) : mm_variant<DT, 4, false>(c);
}

template <int DT>
MmKernel sum_kernel(int32_t group, bool zeros)
{
    if (group == 32) return zeros ? q4_sum_kernel<DT, 1, true> : q4_sum_kernel<DT, 1, false>;
    if (group == 64) return zeros ? q4_sum_kernel<DT, 2, true> : q4_sum_kernel<DT, 2, false>;
    return zeros ? q4_sum_kernel<DT, 4, true> : q4_sum_kernel<DT, 4, false>;
}

// What both products ask of their operands; n_rows of Y
int mm_args(const q4_t *h, const void *X_dev, int64_t ldx, const void *Y_dev, int64_t ldy, int32_t y_type, int64_t n_rows)
{
    if (!h || (y_type != VBR_F32 && y_type != h->dtype) || n_rows < 0) return VBR_EINVAL;
    if (!h->dev) return VBR_ESTATE;
    if (n_rows == 0) return VBR_OK;
    if (!X_dev || !Y_dev || ldx < h->n_cols || ldx % 8 != 0 || ldy < h->rows() || !aligned(X_dev, 16) || !aligned(Y_dev, y_type == VBR_F32 ? 4 : 2)) return VBR_EINVAL;
    return VBR_OK;
}

MmParams mm_params(const q4_t *h, const void *X_dev, int64_t ldx, int64_t x_rows, void *Y_dev, int64_t ldy, int64_t n_rows)
{
    MmParams p{};
    const char *d = static_cast<const char *>(h->dev);
    p.tiles = reinterpret_cast<const uint4v *>(d);
    p.scales = d + h->scales_at();
    p.zeros = d + h->zeros_at();
    p.X = static_cast<const uint16_t *>(X_dev);
    p.Y = Y_dev;
    p.ldx = ldx;
    p.ldy = ldy;
    const int64_t x_bytes = b_bytes_of(x_rows, ldx, h->n_cols);
    p.x_bytes = x_bytes <= kNearBytes ? (uint32_t)x_bytes : 0;
    p.ldx_bytes = (uint32_t)(2 * ldx);
    p.n_rows = n_rows;
    p.k_tiles = h->k_tiles();
    p.tile_rows = h->tile_rows();
    p.steps = h->steps();
    p.half = (int32_t)h->rows();
    p.k_chunks = (int32_t)(h->n_cols / 32);
    const uint32_t tiles_a_step = h->group <= 128 ? 1 : (uint32_t)h->group / 128;
    p.step_divide = tiles_a_step == 1 ? 0 : (uint32_t)(((1ull << 32) + tiles_a_step - 1) / tiles_a_step);      // (tiles and tiles_a_step are below 2^16)
    p.gated = h->gated;
    return p;
}

// By how many workgroups there would be for the 256 compute units, in us (bf16, groups of 128, T rows times K x N):
//   more than 16 rows: the kernel for many workgroups from 256 of them on (T 512, 8192 x 8192, 256 workgroups: 98, the other 110; T 256, 4096 x 14336, 224: 53 and
//   51; T 256, 8192 x 8192, 128: 93 and 53).  Of a plan's tiles some are filled in part only, and which is not known here: taken to be one for every two
//   matrices beside the full ones, and 384 workgroups of them (16 experts of 4096 x 4096 with 64 rows each, 384: 78 and 80; with 48, 320: 74 and 68;
//   32 of 4096 x 1536 with 32, 288: 51 and 39; 64 of 1408 x 2048 with 14, 480: 26 and 30), or 224 where a wave of the other one has a single step
//   (128 of 512 x 512 with 48, 320: 16 and 22; with 14, 240: 9.5 and 12.5).  The other one with eight waves where a CU has one workgroup and each wave two steps (T 64, 8192 x 16384, 256
//   workgroups: 34, with four 42; T 256, 4096 x 8192, 512: 39 and 32; T 57, 704 x 12878: 10.7 and 10.0)
//   up to 16 rows: one row of tiles a workgroup and W four steps ahead while that is one workgroup for each CU (T 1, 4096 x 4096: 5.2, two rows 6.1; T 1,
//   8192 x 8192: 11.1 and 9.7).  Else two, and nothing ahead but the next step: then eight waves of a SIMD hide each other's waits (W four steps ahead
//   takes registers for that; T 1, 8192 x 16384: 15.2 and 21.3; 112 pairs of 28 experts, 576 x 1024: 5.4 and 7.1).  Four rows of tiles, for which X is
//   read half as often, with more than 8 rows of X and workgroups for every CU still (T 16, 8192 x 16384: 17.8, two 22.1; T 16, 4064 x 10999: 9.6 and 10.5; T 16,
//   8192 x 8192, 512 rows of tiles: 14.6 and 12.0; five tiles of rows, T 80, 14336 x 2048: 25.5 and 33.2), but with one tile of rows not for groups of 32, where the vector units
//   have more to do than to wait for X (T 16, 4064 x 10976: 12.9 and 11.5; T 9, 2048 x 16384: 9.3 and 7.9; T 48, 4096 x 4096: 12.3 and 12.8).
//   Eight waves where each has two steps or workgroups are few (T 1, 2048 x 14336: 6.3, four 6.4; T 8, 8192 x 8192: 9.9 and 13.2; 8 pairs, 2048 x 1536: 7.0 and
//   7.4), four where there are many (64 pairs of 64 experts, 2048 x 2816: 24.8, eight 25.5; 1408 x 2048: 14.9 and 16.2)
int64_t filled(const MmParams &p, int32_t rows, int64_t n_mats) { return p.n_rows / rows + n_mats / 2; }
bool many(const MmParams &p, int64_t row_tiles) { return row_tiles * ((p.tile_rows + 15) / 16) >= (p.order ? p.k_tiles <= 4 ? 224 : 384 : 256); }
Choice choose(const q4 *h, const MmParams &p, int32_t rows, int64_t row_tiles, int64_t rows_each)
{
    const int64_t tiles = row_tiles * p.tile_rows;
    if (rows > 16) {
        if (many(p, p.order ? filled(p, rows, h->n_mats) : row_tiles)) return {rows, 16, 4};
        return {rows, 4, row_tiles * ((p.tile_rows + 3) / 4) <= 256 && p.k_tiles >= 16 ? 8 : 4};
    }
    if (tiles <= 256 && !p.gated) return {16, 1, p.k_tiles >= 32 ? 8 : 4};
    if (tiles >= 640 && rows_each > 8 && (h->group > 32 || row_tiles > 1)) return {16, 4, 4};
    return {16, 2, (p.k_tiles >= 16 && tiles < 2048) || (p.k_tiles >= 8 && tiles < 1024) ? 8 : 4};
}

void set_y(MmParams &p, int32_t y_type)
{
    p.f32 = y_type == VBR_F32;
    p.fours = p.ldy % 4 == 0 && aligned(p.Y, p.f32 ? 16 : 8);
}

// Rows of a tile of one matrix's product.  Large ones make numbers of W less often, small ones fill the GPU sooner.  In us with tiles of 16, 32 and 64 rows:
//   16 where that makes up to 1024 pieces of 16 x 16: 64 rows, 4096 x 1024 (256 pieces) 7.4 10.9 16.0; 128 rows, 1024 x 1024 (512) 4.5 6.5 8.6; 32 rows, 8192 x 8192
//   (1024) 16.7 17.7; 64 rows, 4096 x 4096 (1024) 10.0 11.6 16.4; 80 rows (1280) 15.2 11.7 16.5
//   32 where that makes up to 256 workgroups of 32 x 64, one a CU, or 512 and either 64 rows make more than 256 too or columns are few: 128 rows, 4096 x 4096 (256) 15.7
//   12.4 16.8; 160 rows, 4096 x 6144 (480, and 288) 26.6 17.6 25.2; 512 rows, 2048 x 2048 (512, and 256) 16.9 11.5 13.0; 192 rows, 14336 x 4096 (384, and
//   192) - 46.9 41.6; 128 rows, 8192 x 8192 (512, and 256) 47 31 29; 192 rows, 4096 x 6144 (576) 32 22.7 25.3; 128 rows, 4096 x 14336 (896) 46 31 27
//   and for 65 to 96 rows, of which 64 would make 128: 80 rows, 4096 x 14336 (672) 33 22.9 26.5; 96 rows, 2048 x 32768 (1536) 41 27.8 29.5
int32_t mm_tile_rows(const MmParams &p, int64_t n_rows)
{
    const auto tiles = [n_rows](int32_t rows) { return (n_rows + rows - 1) / rows; };
    if (p.x_bytes != 0 && (n_rows <= 16 || tiles(16) * p.tile_rows <= 1024)) return 16;      // (an X of 4 GiB and more: the other kernels have 64-bit addresses)
    const int64_t side = (p.tile_rows + 3) / 4, of_32 = tiles(32) * side, of_64 = tiles(64) * side;
    if (n_rows <= 32 || (n_rows > 64 && n_rows <= 96) || of_32 <= 256 || (of_32 <= 512 && (of_64 > 256 || p.k_tiles <= 32))) return 32;
    return 64;
}

// Of a plan's product: by the same (16, 32 and 64 rows: 4 experts of 320 x 1280 with 48 rows each 5.5 7.9 10.5; 8 of 1024 x 1024 with 100 11.7 9.0 9.6), tiles that are
// filled in part counted as for choose(), and no more than a plan's tile has.  And 32 where that makes as many workgroups as the kernel for many wants, and 64 does not:
// 64 experts of 512 x 512 with 64 rows 10.6 and 15.3; 16 of 1024 x 2048 with 200 28.6 and 33.9; 32 of 1536 x 4096 with 48 49.5 and 46.9.
int32_t plan_rows(const MmParams &p, int32_t most, int64_t n_mats)
{
    if (most == 16 || (p.x_bytes != 0 && filled(p, 16, n_mats) * p.tile_rows <= 1024)) return 16;
    if (most == 32 || filled(p, 32, n_mats) * ((p.tile_rows + 3) / 4) <= 512) return 32;
    return many(p, filled(p, 32, n_mats)) && !many(p, filled(p, 64, n_mats)) ? 32 : 64;
}

int launch_mm(const q4 *h, MmParams &p, int32_t rows, int64_t row_tiles, int64_t rows_each, void *hip_stream)
{
    if (rows == 16 && p.x_bytes == 0) rows = 32;       // (of a plan's tiles, or of rows one by one: there are as many)
    const Choice c = choose(h, p, rows, row_tiles, rows_each);
    const Variant v = h->dtype == VBR_F16 ? mm_variant<VBR_F16>(h->group, h->zeros, c) : mm_variant<VBR_BF16>(h->group, h->zeros, c);
    p.col_blocks = (int32_t)((p.tile_rows + v.tile_rows - 1) / v.tile_rows);
    p.by_col_blocks = Divide::by(p.col_blocks);
    p.lg_waves = __builtin_ctz(v.threads / 64);
    // Tiles that follow each other, in us: 64 experts of 2816 x 2048 with 48 rows each 79, in turn 86, with 128 169 and 177; of 2048 x 1408 with 128 93 and 94;
    // 128 of 1536 x 2048 with 64 106 and 112; 16 of 4096 x 4096 with 256 194 and 196; 8 of 14336 x 4096 with 512 615 and 588
    p.follow = p.order && c.nt == 16 && rows_each <= 256;
    const int64_t work = row_tiles * p.col_blocks, grid = p.follow ? (work + 7) / 8 * 8 : work;
    if (grid > kMostThreads / v.threads || grid > INT32_MAX) return VBR_EUNSUPPORTED;
    hipLaunchKernelGGL(v.kernel, dim3((unsigned)grid), dim3(v.threads), v.lds, static_cast<hipStream_t>(hip_stream), p);
    return launched();
}

}  // namespace
}  // namespace vbrk

using namespace vbrk;

extern "C" int q4_create(int64_t n_mats, int64_t n_rows, int64_t n_cols, int32_t group, int32_t dtype, int32_t zeros, int32_t gated, q4_t **out)
{
    if (!out) return VBR_EINVAL;
    *out = nullptr;
    if (n_mats < 1 || n_rows < 1 || n_cols < 32 || n_cols % 32 != 0 || (dtype != VBR_F16 && dtype != VBR_BF16)) return VBR_EINVAL;
    if (group != 32 && group != 64 && (group < 128 || group % 128 != 0)) return VBR_EINVAL;
    if (gated && n_rows % 2 != 0) return VBR_EINVAL;
    if (n_mats > kMaxExperts || n_rows > 1 << 22 || n_cols > 1 << 22) return VBR_EUNSUPPORTED;
    q4 *h = new (std::nothrow) q4();
    if (!h) return VBR_ENOMEM;
    h->n_mats = n_mats;
    h->n_rows = n_rows;
    h->n_cols = n_cols;
    h->group = group;
    h->dtype = dtype;
    h->zeros = zeros != 0;
    h->gated = gated != 0;
    *out = h;
    return VBR_OK;
}

extern "C" int64_t q4_device_bytes(const q4_t *h) { return h ? h->total() : 0; }

extern "C" int q4_upload(q4_t *h, const void *codes_dev, const void *scales_dev, const void *zeros_dev, void *buf_dev, void *hip_stream)
{
    if (!h || !codes_dev || !scales_dev || !buf_dev || (h->zeros && !zeros_dev) || !aligned(codes_dev, 4) || !aligned(scales_dev, 2) || !aligned(buf_dev, 256)) return VBR_EINVAL;
    PackParams p{};
    char *d = static_cast<char *>(buf_dev);
    p.codes = static_cast<const uint8_t *>(codes_dev);
    p.scales = static_cast<const uint16_t *>(scales_dev);
    p.zeros = static_cast<const uint8_t *>(zeros_dev);
    p.tiles = reinterpret_cast<uint4v *>(d);
    p.kept_scales = reinterpret_cast<uint16_t *>(d + h->scales_at());
    p.kept_zeros = h->zeros ? reinterpret_cast<uint8_t *>(d + h->zeros_at()) : nullptr;
    p.n_tiles = h->scales_at() / 1024;
    p.words = !aligned(codes_dev, 16);
    p.n_kept = h->kept();
    p.n_rows = h->n_rows;
    p.half = h->rows();
    p.n_cols = h->n_cols;
    p.tile_rows = h->tile_rows();
    p.k_tiles = h->k_tiles();
    p.groups = h->groups();
    p.steps = h->steps();
    p.groups_a_step = h->groups_a_step();
    p.gated = h->gated;
    p.rotate = h->dtype == VBR_F16 ? 6 : 3;
    const int64_t workgroups = (p.n_tiles + 4 * kPackTiles - 1) / (4 * kPackTiles);
    if (workgroups > kMostThreads / 256) return VBR_EUNSUPPORTED;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipLaunchKernelGGL(q4_pack_codes_kernel, dim3((unsigned)workgroups), dim3(256), 0, stream, p);
    hipLaunchKernelGGL(q4_pack_scales_kernel, dim3((unsigned)std::min<int64_t>((p.n_kept + 255) / 256, 1 << 20)), dim3(256), 0, stream, p);
    const int rc = launched();
    if (rc != VBR_OK) return rc;
    const hipError_t e = hipStreamSynchronize(stream);
    if (e != hipSuccess) {
        set_last_hip_error((int)e);
        return VBR_EHIP;
    }
    h->dev = buf_dev;
    return VBR_OK;
}

extern "C" int q4_mm(const q4_t *h, const void *X_dev, int64_t ldx, void *Y_dev, int64_t ldy, int32_t y_type, int64_t n_rows, void *hip_stream)
{
    const int rc = mm_args(h, X_dev, ldx, Y_dev, ldy, y_type, n_rows);
    if (rc != VBR_OK) return rc;
    if (h->n_mats != 1) return VBR_EINVAL;
    if (n_rows == 0) return VBR_OK;
    MmParams p = mm_params(h, X_dev, ldx, n_rows, Y_dev, ldy, n_rows);
    set_y(p, y_type);
    const int32_t rows = mm_tile_rows(p, n_rows);
    return launch_mm(h, p, rows, (n_rows + rows - 1) / rows, n_rows, hip_stream);
}

// plan_dev, or ids_dev: a tile for each pair
static int mm_pairs(const q4_t *h, const void *plan_dev, const int32_t *ids_dev, int64_t n_pairs, const void *X_dev, int64_t ldx, int64_t n_rows, void *Y_dev, int64_t ldy, int32_t y_type,
                    void *hip_stream)
{
    const int rc = mm_args(h, X_dev, ldx, Y_dev, ldy, y_type, n_pairs);
    if (rc != VBR_OK) return rc;
    if (!plan_sizes_ok(n_pairs, (int32_t)h->n_mats)) return VBR_EUNSUPPORTED;
    if (n_pairs == 0) return VBR_OK;
    if (n_rows < 1 || n_pairs % n_rows != 0 || (!ids_dev && (!plan_dev || !aligned(plan_dev, 256)))) return VBR_EINVAL;
    MmParams p = mm_params(h, X_dev, ldx, n_rows, Y_dev, ldy, n_pairs);
    p.by_places = Divide::by(n_pairs / n_rows);
    set_y(p, y_type);
    if (ids_dev) {
        p.ids = ids_dev;
        p.n_mats = (int32_t)h->n_mats;
        return launch_mm(h, p, 16, n_pairs, 1, hip_stream);
    }
    const PlanParts parts = plan_parts(n_pairs, (int32_t)h->n_mats);
    const char *d = static_cast<const char *>(plan_dev);
    p.order = reinterpret_cast<const int32_t *>(d + parts.order);
    p.plan_tiles = reinterpret_cast<const PlanTile *>(d + parts.tiles);
    const int32_t rows = plan_rows(p, parts.tile_rows, h->n_mats);
    p.lg_parts = __builtin_ctz(parts.tile_rows / rows);
    return launch_mm(h, p, rows, parts.n_tiles << p.lg_parts, n_pairs / h->n_mats, hip_stream);
}

extern "C" int q4_mm_routed(const q4_t *h, const void *plan_dev, int64_t n_pairs, const void *X_dev, int64_t ldx, int64_t n_rows, void *Y_dev, int64_t ldy, int32_t y_type, void *hip_stream)
{
    return mm_pairs(h, plan_dev, nullptr, n_pairs, X_dev, ldx, n_rows, Y_dev, ldy, y_type, hip_stream);
}

namespace {

constexpr int64_t kAgain = 32 << 20;          // bytes read again that cost what the grouping does
struct Work {
    int64_t h, y, total;           // byte offsets in the work buffer, behind a plan
};
bool experts_ok(const q4_t *up, const q4_t *down, int64_t n_rows, int32_t top_k)
{
    if (!up || !down || !up->gated || down->gated || up->rows() != down->n_cols || up->n_mats != down->n_mats || up->dtype != down->dtype || down->n_rows % 8 != 0) return false;
    return n_rows >= 0 && top_k >= 1 && top_k <= kMaxTopK && n_rows <= kMaxPairs / top_k;
}
Work experts_work(const q4_t *up, const q4_t *down, int64_t n_pairs)
{
    Work w;
    w.h = plan_parts(n_pairs, (int32_t)up->n_mats).total;
    w.y = (w.h + n_pairs * up->rows() * 2 + 255) / 256 * 256;
    w.total = w.y + n_pairs * down->n_rows * 4;
    return w;
}

// Few pairs are not grouped: each is a tile of its own.  That saves two launches and reads a matrix again for every further pair of it, of which there are
// k^2 T (T - 1) / 2 E if no expert is chosen more often than others.  In us, grouped and not, where that is so many bytes:
//   8 of 128 experts of 2048 x 768: 2 rows, 1 MB: 23.5 and 14.9; 6, 17 MB: 36.2 and 30.9; 8, 33 MB: 41.1 and 38.8; 10, 52 MB: 45.2 and 46.5
//   8 of 256 of 2048 x 512: 12 rows, 26 MB: 43.2 and 39.4; 16, 46 MB: 49.9 and 50.7      2 of 8 of 4096 x 14336: 2 rows, 43 MB: 74.1 and 77.7
//   6 of 64 of 512 x 256, which stay in the cache: 24 rows, 30 MB: 17.5 and 14.7; 32, 54 MB: 17.6 and 17.4
// 256 pairs are as many as were measured (8 of 512 of 512 x 256, 12 MB: 26.5 and 18.9).
bool ungrouped(const q4_t *up, const q4_t *down, int64_t n_rows, int32_t top_k)
{
    const int64_t n_pairs = n_rows * top_k;
    if (n_rows == 1) return true;
    return n_pairs <= 256 && n_pairs * (n_pairs - top_k) / 2 * ((up->total() + down->total()) / up->n_mats) <= kAgain * up->n_mats;
}

int sum_pairs(const q4_t *h, const int32_t *ids_dev, const float *weights_dev, int64_t n_rows, int32_t top_k, const void *X_dev, void *Y_dev, int64_t ldy, int32_t y_type, void *hip_stream)
{
    MmParams p = mm_params(h, X_dev, h->n_cols, n_rows * top_k, Y_dev, ldy, n_rows);
    p.ids = ids_dev;
    p.n_mats = (int32_t)h->n_mats;
    p.weights = weights_dev;
    p.top_k = top_k;
    p.f32 = y_type == VBR_F32;
    p.bf16 = y_type == VBR_BF16;
    while (top_k << p.lg_waves < kSumWaves) ++p.lg_waves;
    p.col_blocks = (int32_t)p.tile_rows;
    p.by_col_blocks = Divide::by(p.col_blocks);
    const int64_t grid = n_rows * p.col_blocks;
    if (grid > kMostThreads / (64 * kSumWaves) || grid > INT32_MAX) return VBR_EUNSUPPORTED;
    const MmKernel kernel = h->dtype == VBR_F16 ? sum_kernel<VBR_F16>(h->group, h->zeros) : sum_kernel<VBR_BF16>(h->group, h->zeros);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kSumWaves), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched();
}

}  // namespace

extern "C" int64_t experts_work_bytes(const q4_t *up, const q4_t *down, int64_t n_rows, int32_t top_k)
{
    return experts_ok(up, down, n_rows, top_k) ? experts_work(up, down, n_rows * top_k).total : 0;
}

extern "C" int experts_forward(const q4_t *up, const q4_t *down, const void *X_dev, int64_t ldx, int64_t n_rows, const int32_t *ids_dev, const float *weights_dev, int32_t top_k,
                               void *out_dev, int64_t ldo, int32_t out_type, void *work_dev, void *hip_stream)
{
    if (!experts_ok(up, down, n_rows, top_k)) return VBR_EINVAL;
    if (!up->dev || !down->dev) return VBR_ESTATE;
    if (n_rows == 0) return VBR_OK;
    if (!ids_dev || !weights_dev || !out_dev || !work_dev || !aligned(work_dev, 256) || !aligned(ids_dev, 4) || !aligned(weights_dev, 4)) return VBR_EINVAL;
    // (operands are refused before anything is launched; products of more workgroups than a launch can have, by themselves)
    if ((out_type != VBR_F16 && out_type != VBR_BF16 && out_type != VBR_F32) || ldo < down->n_rows || ldo % 8 != 0 || !aligned(out_dev, 16)) return VBR_EINVAL;
    const int64_t n_pairs = n_rows * top_k;
    const Work w = experts_work(up, down, n_pairs);
    char *d = static_cast<char *>(work_dev);
    int rc = mm_args(up, X_dev, ldx, d + w.h, up->rows(), up->dtype, n_pairs);
    if (rc != VBR_OK) return rc;
    const int32_t *direct = ungrouped(up, down, n_rows, top_k) ? ids_dev : nullptr;
    if (!direct) rc = route_plan(ids_dev, n_pairs, (int32_t)up->n_mats, work_dev, hip_stream);
    if (rc == VBR_OK) rc = mm_pairs(up, work_dev, direct, n_pairs, X_dev, ldx, n_rows, d + w.h, up->rows(), up->dtype, hip_stream);
    if (direct) return rc == VBR_OK ? sum_pairs(down, ids_dev, weights_dev, n_rows, top_k, d + w.h, out_dev, ldo, out_type, hip_stream) : rc;
    if (rc == VBR_OK) rc = mm_pairs(down, work_dev, nullptr, n_pairs, d + w.h, up->rows(), n_pairs, d + w.y, down->n_rows, VBR_F32, hip_stream);
    if (rc == VBR_OK) rc = route_combine(d + w.y, down->n_rows, VBR_F32, ids_dev, weights_dev, n_rows, top_k, (int32_t)up->n_mats, down->n_rows, out_dev, ldo, out_type, hip_stream);
    return rc;
}

extern "C" void q4_free(q4_t *h) { delete h; }
