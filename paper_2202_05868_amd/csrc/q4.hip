// Products with matrices in 4 bits: Y = X W^T, W[n][k] = s[n][k / group] (c[n][k] - z[n][k / group]), c and z in 0 .. 15.
//
// The mathematics.  With the code in the upper bits of the mantissa, 16 + c is an fp16 or bf16 number as it stands: one rotation and one
// and-or make two of them.  The matrix units sum (16 + c) x over a group exactly as products, in fp32; with the sum of x over the group,
//   y = sum over groups s (sum_k (16 + c_k) x_k - (16 + z) sum_k x_k),
// so scale and zero point are applied to sums in fp32, once a group, and no weight is ever rounded.  sum_k x_k comes from the matrix units as well,
// as a product with ones.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>
#include <type_traits>

#include "route.h"
#include "vbr_device.h"
#include "vbr_host.h"

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
    uint32_t *tiles;
    uint16_t *kept_scales;
    uint8_t *kept_zeros;
    int64_t n_words, n_kept;
    int64_t n_rows, half, n_cols, tile_rows, k_tiles, groups, steps;
    int32_t gated, rotate, groups_a_step;
};

__device__ __forceinline__ int64_t source_row(const PackParams &p, int64_t tile_row, int n)       // in its matrix; -1: none
{
    const int64_t in_half = (p.gated ? tile_row / 2 : tile_row) * 16 + n;
    return in_half < p.half ? in_half + (p.gated && (tile_row & 1) ? p.half : 0) : -1;
}

__global__ void __launch_bounds__(256) q4_pack_codes_kernel(const PackParams p)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= p.n_words) return;
    const int i = at & 3, n = at >> 2 & 15, q = at >> 6 & 3;
    const int64_t tile = at >> 8, t = tile % p.k_tiles, row_of_all = tile / p.k_tiles, mat = row_of_all / p.tile_rows;
    const int64_t row = source_row(p, row_of_all - mat * p.tile_rows, n), k = t * 128 + 32 * i + 8 * q;
    uint32_t word = 0;
    if (row >= 0 && k < p.n_cols) {
        const uint32_t codes = *reinterpret_cast<const uint32_t *>(p.codes + (mat * p.n_rows + row) * (p.n_cols / 2) + k / 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) word |= (codes >> 8 * j & 15u) << 4 * j | (codes >> (8 * j + 4) & 15u) << (4 * j + 16);
    }
    p.tiles[at] = word << p.rotate | word >> (32 - p.rotate);
}

__global__ void __launch_bounds__(256) q4_pack_scales_kernel(const PackParams p)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= p.n_kept) return;
    const int in_step = (int)(at % p.groups_a_step);
    const int64_t of_step = at / p.groups_a_step;
    const int n = of_step & 15;
    const int64_t g = (of_step >> 4) % p.steps * p.groups_a_step + in_step, row_of_all = (of_step >> 4) / p.steps, mat = row_of_all / p.tile_rows;
    const int64_t row = source_row(p, row_of_all - mat * p.tile_rows, n), from = (mat * p.n_rows + row) * p.groups + g;
    const bool there = row >= 0 && g < p.groups;
    p.kept_scales[at] = there ? p.scales[from] : 0;
    if (p.kept_zeros) p.kept_zeros[at] = there ? p.zeros[from] : 0;
}

// ---- the products
struct MmParams {
    const uint4v *tiles;
    const char *scales, *zeros;
    const uint16_t *X;
    void *Y;
    int64_t ldx, ldy, n_rows;                  // rows of Y
    int64_t k_tiles, tile_rows, steps;
    int32_t half, k_chunks, tiles_a_step;      // k_chunks: columns / 32
    int32_t gated, f32;
    int32_t col_blocks, row_tiles;             // of the launch; row_tiles: at most so many, if routed
    // routed, or null
    const PlanTile *plan_tiles;
    const int32_t *order;
    uint32_t divide;                           // the row of X of pair i is i divide >> divide_shift
    int32_t divide_shift;
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
template <int N, bool ZEROS>
__device__ __forceinline__ Words<N> load_words(const MmParams &p, int64_t row, int64_t step, int n)
{
    const int64_t at = (row * p.steps + step) * 16 + n;
    Words<N> w{};
    w.s = reinterpret_cast<const typename Words<N>::Scales *>(p.scales)[at];
    if constexpr (ZEROS) w.z = reinterpret_cast<const typename Words<N>::Zeros *>(p.zeros)[at];
    return w;
}

// x / (1 + exp(-x)).  exp(-x) is 2^t (1 + r), r what rounding took from t = -x log2(e): a relative error of a few steps however large x is.
__device__ __forceinline__ float silu(float x)
{
    constexpr float log2e = 1.44269502f, rest = 1.92596299e-8f, ln2 = 0.693147181f;      // log2(e) in two numbers
    const float t = -x * log2e, r = __builtin_fmaf(-x, rest, __builtin_fmaf(-x, log2e, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    return x * __builtin_amdgcn_rcpf(1.f + __builtin_fmaf(e, r * ln2, e));
}

template <int DT>
__device__ __forceinline__ void store_y(const MmParams &p, int64_t at, float y)
{
    if (p.f32) static_cast<float *>(p.Y)[at] = y;
    else if constexpr (DT == VBR_F16) static_cast<_Float16 *>(p.Y)[at] = (_Float16)y;
    else static_cast<__bf16 *>(p.Y)[at] = (__bf16)y;
}

// rows first .. first + count - 1 (positions of the plan's order, if routed) of matrix mat
struct RowTile {
    int64_t mat, first;
    int32_t count;
};
__device__ __forceinline__ RowTile row_tile(const MmParams &p, int tile, int rows)      // count 0: none
{
    if (p.order) {
        const PlanTile t = p.plan_tiles[tile];
        return {t.expert, t.first, t.count};
    }
    const int64_t first = (int64_t)tile * rows, left = p.n_rows - first;
    return {0, first, (int32_t)(left < rows ? left : rows)};
}
__device__ __forceinline__ int64_t x_row(const MmParams &p, int64_t y_row) { return p.order ? (int64_t)((uint64_t)y_row * p.divide >> p.divide_shift) : y_row; }
__device__ __forceinline__ int64_t y_row(const MmParams &p, int64_t at) { return p.order ? p.order[at] : at; }

// ---- few rows: 16 of them times two rows of tiles, by four waves that share the columns.  The sums of the waves are added in their order.
// CH: steps of 32 columns between applications of a scale (1, 2, or 4)
constexpr int kFewWaves = 4;

template <int DT, int CH, bool ZEROS>
__global__ void __launch_bounds__(64 * kFewWaves) q4_few_kernel(const MmParams p)
{
    __shared__ float sums[kFewWaves][2][16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, q = lane >> 4;
    const RowTile rt = row_tile(p, blockIdx.x / p.col_blocks, 16);
    if (rt.count == 0) return;
    const SixteenPlus<DT> sixteen_plus;
    const int col_block = blockIdx.x % p.col_blocks;
    const int64_t last = p.tile_rows - 1, r0 = 2 * (int64_t)col_block, r1 = r0 < last ? r0 + 1 : r0;
    const int64_t row[2] = {rt.mat * p.tile_rows + r0, rt.mat * p.tile_rows + r1};
    const uint16_t *x = p.X + (n < rt.count ? x_row(p, y_row(p, rt.first + n)) : 0) * p.ldx + 8 * q;

    float4v acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    const float4v none = {0, 0, 0, 0};
    const short one = DT == VBR_F16 ? 0x3C00 : 0x3F80;
    const short8v ones = {one, one, one, one, one, one, one, one};
    const int begin = (int)(p.k_tiles * wave / kFewWaves), end = (int)(p.k_tiles * (wave + 1) / kFewWaves);
    for (int t = begin; t < end; ++t) {
        uint4v w[2];
        Words<4 / CH> sz[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            w[h] = p.tiles[(row[h] * p.k_tiles + t) * 64 + lane];
            sz[h] = load_words<4 / CH, ZEROS>(p, row[h], t / p.tiles_a_step, n);
        }
        short8v xf[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xf[i] = short8v{0, 0, 0, 0, 0, 0, 0, 0};
            if (n < rt.count && 4 * t + i < p.k_chunks) xf[i] = *reinterpret_cast<const short8v *>(x + 128 * (int64_t)t + 32 * i);
        }
#pragma unroll
        for (int c = 0; c < 4; c += CH) {
            float4v of_x = none, part[2] = {none, none};
#pragma unroll
            for (int i = c; i < c + CH; ++i) {
                of_x = mfma16x16x32<DT>(xf[i], ones, of_x);
#pragma unroll
                for (int h = 0; h < 2; ++h) part[h] = mfma16x16x32<DT>(xf[i], sixteen_plus(w[h][i]), part[h]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float s = sz[h].template scale<DT>(c / CH), z = ZEROS ? sz[h].minus_sixteen_plus_zero(c / CH) : -24.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[h][i] = __builtin_fmaf(s, __builtin_fmaf(z, of_x[i], part[h][i]), acc[h][i]);
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][h][4 * q + i][n] = acc[h][i];
    __syncthreads();
    const int outs = p.gated ? 1 : 2;
    for (int at = threadIdx.x; at < outs * 256; at += 64 * kFewWaves) {
        const int col = at & 15, token = at >> 4 & 15, h = at >> 8;
        const int64_t out_col = (p.gated ? col_block : r0 + h) * 16 + col;
        if (token >= rt.count || out_col >= p.half || (!p.gated && r0 + h > last)) continue;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) v += sums[k][h][token][col];
        if (p.gated) {
            float u = 0.f;
#pragma unroll
            for (int k = 0; k < kFewWaves; ++k) u += sums[k][1][token][col];
            v = silu(v) * u;
        }
        store_y<DT>(p, y_row(p, rt.first + token) * p.ldy + out_col, v);
    }
}

// ---- many rows: 16 MT of them times 16 rows of tiles, by four waves with four rows of tiles each.  A step is a tile's 128 columns: X goes through LDS,
// which all waves read; W comes straight into registers, as it was laid out, and is turned into numbers there.
constexpr int kManyRows = 4;           // rows of tiles a wave

template <int CTRL>
__device__ __forceinline__ float add_lane(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

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
template <int DT, int CH, bool ZEROS, int MT>
__global__ void __launch_bounds__(256, 2) q4_many_kernel(const MmParams p)
{
    constexpr int kRows = 16 * MT, kGroups = 4 / CH, NT = kManyRows;
    __shared__ __attribute__((aligned(16))) uint4v x_lds[2][kRows * 16];         // chunk c of row r at r * 16 + (c ^ r % 16)
    __shared__ float sum_lds[2][4][kRows];                                       // of four groups in turn
    __shared__ int64_t y_lds[kRows];                                             // where the rows of Y begin
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, q = lane >> 4;
    const RowTile rt = row_tile(p, blockIdx.x / p.col_blocks, kRows);
    if (rt.count == 0) return;
    const SixteenPlus<DT> sixteen_plus;
    const int64_t last = p.tile_rows - 1, r0 = ((int64_t)(blockIdx.x % p.col_blocks) * 4 + wave) * NT;
    // W from the wave's first row of tiles on (behind the last one, that one), 32-bit offsets from there
    const int64_t from = rt.mat * p.tile_rows + (r0 < last ? r0 : last);
    const int further = (int)(last - r0 < 0 ? 0 : last - r0 < NT ? last - r0 : NT - 1);
    const char *w_at = reinterpret_cast<const char *>(p.tiles) + from * p.k_tiles * 1024;
    const char *s_at = p.scales + from * p.steps * (32 * kGroups), *z_at = p.zeros + from * p.steps * (16 * kGroups);
    uint32_t w_row[NT], s_row[NT];
#pragma unroll
    for (int h = 0; h < NT; ++h) {
        w_row[h] = (uint32_t)((h < further ? h : further) * p.k_tiles) * 1024u;
        s_row[h] = (uint32_t)((h < further ? h : further) * p.steps) * 16u;
    }

    uint4v w[NT];
    Words<kGroups> sz[NT];
    auto fetch_w = [&](int h, int t) {
        w[h] = *reinterpret_cast<const uint4v *>(w_at + (w_row[h] + (uint32_t)t * 1024u + (uint32_t)lane * 16u));
        const uint32_t at = s_row[h] + (uint32_t)(t / p.tiles_a_step) * 16u + (uint32_t)n;
        sz[h].s = *reinterpret_cast<const typename Words<kGroups>::Scales *>(s_at + at * (2u * kGroups));
        if constexpr (ZEROS) sz[h].z = *reinterpret_cast<const typename Words<kGroups>::Zeros *>(z_at + at * (uint32_t)kGroups);
    };
#pragma unroll
    for (int h = 0; h < NT; ++h) fetch_w(h, 0);

    // this thread's chunks of X: chunk c of rows xr + 16 j
    const int c = threadIdx.x & 15, xr = threadIdx.x >> 4;
    const uint16_t *src[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) {
        const int64_t row = y_row(p, rt.first + (xr + 16 * j < rt.count ? xr + 16 * j : 0));
        if (c == 0) y_lds[xr + 16 * j] = row * p.ldy;
        src[j] = p.X + x_row(p, row) * p.ldx + 8 * c;
    }
    uint4v xv[MT];
    auto fetch_x = [&](int t) {
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            xv[j] = uint4v{0, 0, 0, 0};
            if (4 * t + (c >> 2) < p.k_chunks) xv[j] = *reinterpret_cast<const uint4v *>(src[j] + 128 * (int64_t)t);
        }
    };
    auto put_x = [&](int t) {
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            x_lds[t & 1][(xr + 16 * j) * 16 + (c ^ (xr & 15))] = xv[j];
            float s = sum_of_8<DT>(xv[j]);
            s = add_lane<0x4E>(add_lane<0xB1>(s));            // over four lanes, then eight, then sixteen
            if constexpr (CH >= 2) s = add_lane<0x141>(s);
            if constexpr (CH == 4) s = add_lane<0x140>(s);
            const int g = t * kGroups + c / (4 * CH);
            if (c % (4 * CH) == 0) sum_lds[g >> 2 & 1][g & 3][xr + 16 * j] = s;
        }
    };
    float4v acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < NT; ++h) acc[m][h] = float4v{0, 0, 0, 0};
    float taken[NT];                                              // -s (16 + z) of the q-th of four groups
#pragma unroll
    for (int h = 0; h < NT; ++h) taken[h] = 0.f;
    const int n_tiles = (int)p.k_tiles;
    fetch_x(0);
    put_x(0);
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
        const int next = t + 1 < n_tiles ? t + 1 : t;
        fetch_x(next);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int slot = (t * kGroups + g) & 3;
            short8v xf[MT][CH];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < CH; ++i) xf[m][i] = __builtin_bit_cast(short8v, x_lds[t & 1][(16 * m + n) * 16 + ((4 * (g * CH + i) + q) ^ n)]);
#pragma unroll
            for (int h = 0; h < NT; ++h) {
                float4v part[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) part[m] = float4v{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const short8v b = sixteen_plus(w[h][g * CH + i]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) part[m] = mfma16x16x32<DT>(xf[m][i], b, part[m]);
                }
                const float s = sz[h].template scale<DT>(g);
                if constexpr (CH == 1) {
                    if (g == 0) taken[h] = sz[h].template scale<DT>(q) * (ZEROS ? sz[h].minus_sixteen_plus_zero(q) : -24.f);
                } else {
                    taken[h] = q == slot ? s * (ZEROS ? sz[h].minus_sixteen_plus_zero(g) : -24.f) : taken[h];
                }
                if (g == kGroups - 1) fetch_w(h, next);           // a step ahead, into the registers just read
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][h][i] = __builtin_fmaf(s, part[m][i], acc[m][h][i]);
            }
            if (g == kGroups - 1 && (slot == 3 || t + 1 == n_tiles)) {
                const int four = (t * kGroups + g) >> 2 & 1;
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const float of_x = q <= slot ? sum_lds[four][q][16 * m + n] : 0.f;
#pragma unroll
                    for (int h = 0; h < NT; ++h) acc[m][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(of_x, taken[h], acc[m][h], 0, 0, 0);
                }
#pragma unroll
                for (int h = 0; h < NT; ++h) taken[h] = 0.f;
            }
            __builtin_amdgcn_sched_barrier(0);                    // (groups taken up at once take registers that are not there)
        }
        if (t + 1 < n_tiles) put_x(t + 1);
        __syncthreads();
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int token = 16 * m + 4 * q + i;
            if (token >= rt.count) continue;
            const int64_t at = y_lds[token];
            if (p.gated) {
#pragma unroll
                for (int h = 0; h < NT; h += 2) {
                    const int64_t col = (r0 + h) / 2 * 16 + n;
                    if (r0 + h < last && col < p.half) store_y<DT>(p, at + col, silu(acc[m][h][i]) * acc[m][h + 1][i]);
                }
            } else {
#pragma unroll
                for (int h = 0; h < NT; ++h) {
                    const int64_t col = (r0 + h) * 16 + n;
                    if (col < p.half) store_y<DT>(p, at + col, acc[m][h][i]);
                }
            }
        }
}

using MmKernel = void (*)(MmParams);
template <int DT, int CH, bool ZEROS>
MmKernel mm_kernel(int32_t rows)
{
    return rows == 16 ? q4_few_kernel<DT, CH, ZEROS> : rows == 32 ? q4_many_kernel<DT, CH, ZEROS, 2> : q4_many_kernel<DT, CH, ZEROS, 4>;
}
template <int DT>
MmKernel mm_kernel(int32_t group, bool zeros, int32_t rows)
{
    if (group == 32) return zeros ? mm_kernel<DT, 1, true>(rows) : mm_kernel<DT, 1, false>(rows);
    if (group == 64) return zeros ? mm_kernel<DT, 2, true>(rows) : mm_kernel<DT, 2, false>(rows);
    return zeros ? mm_kernel<DT, 4, true>(rows) : mm_kernel<DT, 4, false>(rows);
}

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int launched()
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        set_last_hip_error((int)e);
        return VBR_EHIP;
    }
    return VBR_OK;
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

MmParams mm_params(const q4_t *h, const void *X_dev, int64_t ldx, void *Y_dev, int64_t ldy, int64_t n_rows)
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
    p.n_rows = n_rows;
    p.k_tiles = h->k_tiles();
    p.tile_rows = h->tile_rows();
    p.steps = h->steps();
    p.half = (int32_t)h->rows();
    p.k_chunks = (int32_t)(h->n_cols / 32);
    p.tiles_a_step = h->group < 128 ? 1 : h->group / 128;
    p.gated = h->gated;
    return p;
}

int launch_mm(const q4 *h, MmParams &p, int32_t rows, int64_t row_tiles, void *hip_stream)
{
    const int64_t block = rows == 16 ? 2 : 4 * kManyRows;      // rows of tiles of a workgroup
    p.col_blocks = (int32_t)((p.tile_rows + block - 1) / block);
    const int64_t grid = row_tiles * p.col_blocks;
    if (grid > INT32_MAX) return VBR_EUNSUPPORTED;
    const MmKernel kernel = h->dtype == VBR_F16 ? mm_kernel<VBR_F16>(h->group, h->zeros, rows) : mm_kernel<VBR_BF16>(h->group, h->zeros, rows);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
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
    p.tiles = reinterpret_cast<uint32_t *>(d);
    p.kept_scales = reinterpret_cast<uint16_t *>(d + h->scales_at());
    p.kept_zeros = h->zeros ? reinterpret_cast<uint8_t *>(d + h->zeros_at()) : nullptr;
    p.n_words = h->scales_at() / 4;
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
    if ((p.n_words + 255) / 256 > INT32_MAX) return VBR_EUNSUPPORTED;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipLaunchKernelGGL(q4_pack_codes_kernel, dim3((unsigned)((p.n_words + 255) / 256)), dim3(256), 0, stream, p);
    hipLaunchKernelGGL(q4_pack_scales_kernel, dim3((unsigned)((p.n_kept + 255) / 256)), dim3(256), 0, stream, p);
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
    MmParams p = mm_params(h, X_dev, ldx, Y_dev, ldy, n_rows);
    p.f32 = y_type == VBR_F32;
    const int32_t rows = n_rows <= 16 ? 16 : n_rows <= 32 ? 32 : 64;
    return launch_mm(h, p, rows, (n_rows + rows - 1) / rows, hip_stream);
}

extern "C" int q4_mm_routed(const q4_t *h, const void *plan_dev, int64_t n_pairs, const void *X_dev, int64_t ldx, int64_t n_rows, void *Y_dev, int64_t ldy, int32_t y_type, void *hip_stream)
{
    const int rc = mm_args(h, X_dev, ldx, Y_dev, ldy, y_type, n_pairs);
    if (rc != VBR_OK) return rc;
    if (!plan_sizes_ok(n_pairs, (int32_t)h->n_mats)) return VBR_EUNSUPPORTED;
    if (n_pairs == 0) return VBR_OK;
    if (!plan_dev || !aligned(plan_dev, 256) || n_rows < 1 || n_pairs % n_rows != 0) return VBR_EINVAL;
    MmParams p = mm_params(h, X_dev, ldx, Y_dev, ldy, n_pairs);
    const PlanParts parts = plan_parts(n_pairs, (int32_t)h->n_mats);
    const char *d = static_cast<const char *>(plan_dev);
    p.order = reinterpret_cast<const int32_t *>(d + parts.order);
    p.plan_tiles = reinterpret_cast<const PlanTile *>(d + parts.tiles);
    // i / d for i below 2^31: 2^(31 + l) / d rounded up, l the bits of d - 1
    const int64_t d_rows = n_pairs / n_rows;
    const int l = d_rows > 1 ? 64 - __builtin_clzll((unsigned long long)d_rows - 1) : 0;
    p.divide = (uint32_t)(((1ull << (31 + l)) + d_rows - 1) / d_rows);
    p.divide_shift = 31 + l;
    p.f32 = y_type == VBR_F32;
    return launch_mm(h, p, parts.tile_rows, parts.n_tiles, hip_stream);
}

extern "C" void q4_free(q4_t *h) { delete h; }
