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

#include "route.h"
#include "vbr_device.h"
#include "vbr_host.h"

// A tile is 16 rows (of one half, if gated) and 128 columns: 1 KiB of codes, 16 bytes a lane.  Lane 16 q + n has row n; its word i has the
// columns 32 i + 8 q .. + 7, in the order that the rotations take them apart.  Tiles of a row follow each other; with a gate the tiles of 16
// gate rows stand before those of the 16 rows they gate.  Scales and zero points are [tile row][group][16 rows].
struct q4 {
    int64_t n_mats = 0, n_rows = 0, n_cols = 0;
    int32_t group = 0, dtype = 0;
    bool zeros = false, gated = false;
    int64_t rows() const { return gated ? n_rows / 2 : n_rows; }                     // of a half
    int64_t tile_rows() const { return (rows() + 15) / 16 * (gated ? 2 : 1); }      // of a matrix
    int64_t k_tiles() const { return (n_cols + 127) / 128; }
    int64_t groups() const { return (n_cols + group - 1) / group; }
    int64_t groups_kept() const { return (k_tiles() * 128 + group - 1) / group; }   // up to the end of the last tile
    int64_t scales_at() const { return n_mats * tile_rows() * k_tiles() * 1024; }
    int64_t zeros_at() const { return scales_at() + n_mats * tile_rows() * groups_kept() * 32; }
    int64_t total() const { return (zeros_at() + (zeros ? n_mats * tile_rows() * groups_kept() * 16 : 0) + 255) / 256 * 256; }
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
    int64_t n_rows, half, n_cols, tile_rows, k_tiles, groups, groups_kept;
    int32_t gated, rotate;
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
    const int n = at & 15;
    const int64_t g = (at >> 4) % p.groups_kept, row_of_all = (at >> 4) / p.groups_kept, mat = row_of_all / p.tile_rows;
    const int64_t row = source_row(p, row_of_all - mat * p.tile_rows, n), from = (mat * p.n_rows + row) * p.groups + g;
    const bool there = row >= 0 && g < p.groups;
    p.kept_scales[at] = there ? p.scales[from] : 0;
    if (p.kept_zeros) p.kept_zeros[at] = there ? p.zeros[from] : 0;
}

// ---- the product
struct MmParams {
    const uint4v *tiles;
    const uint16_t *scales;
    const uint8_t *zeros;
    const uint16_t *X;
    void *Y;
    int64_t ldx, ldy, n_rows;                  // rows of Y
    int64_t k_tiles, tile_rows, groups_kept;
    int32_t half, n_cols, k_chunks, tiles_a_group;     // k_chunks: columns / 32; tiles_a_group: group / 128, at least 1
    // routed
    const int2 *plan_tiles;
    const int32_t *offsets, *order;
    int32_t divide;                            // pairs of a row of X
};

constexpr int kMmWaves = 4;
constexpr int kTokens = 16;

template <int DT>
__device__ __forceinline__ float as_f32(uint16_t x)
{
    if constexpr (DT == VBR_F16) return (float)__builtin_bit_cast(_Float16, x);
    else return __builtin_bit_cast(float, (uint32_t)x << 16);
}

// eight numbers 16 + c out of a word
template <int DT>
__device__ __forceinline__ short8v sixteen_plus(uint32_t w)
{
    constexpr uint32_t mask = DT == VBR_F16 ? 0x03C003C0u : 0x00780078u, base = DT == VBR_F16 ? 0x4C004C00u : 0x41804180u;
    uint4v r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = ((j ? __builtin_amdgcn_alignbit(w, w, 4 * j) : w) & mask) | base;
    return __builtin_bit_cast(short8v, r);
}

__device__ __forceinline__ float silu(float x) { return x / (1.f + expf(-x)); }

// One workgroup: 16 rows of X (of one matrix) times two rows of tiles, four waves that share the columns.  The sums of the waves are added in their order.
// CH: steps of 32 columns between applications of a scale (1, 2, or 4)
template <int DT, int CH, bool ZEROS, bool GATED, bool ROUTED, bool F32>
__global__ void __launch_bounds__(64 * kMmWaves) q4_mm_kernel(const MmParams p)
{
    __shared__ float sums[kMmWaves][2][kTokens][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, q = lane >> 4;
    int64_t first = (int64_t)blockIdx.y * kTokens, mat = 0;
    int count;
    if constexpr (ROUTED) {
        const int2 tile = p.plan_tiles[blockIdx.y];
        if (tile.x < 0) return;
        mat = tile.x;
        first = tile.y;
        const int left = p.offsets[tile.x + 1] - tile.y;
        count = left < kTokens ? left : kTokens;
    } else {
        count = p.n_rows - first < kTokens ? (int)(p.n_rows - first) : kTokens;
    }
    const int64_t last = p.tile_rows - 1, r0 = 2 * (int64_t)blockIdx.x, r1 = r0 < last ? r0 + 1 : r0;
    const int64_t row[2] = {mat * p.tile_rows + r0, mat * p.tile_rows + r1};
    int64_t x_row = 0;
    if (n < count) x_row = ROUTED ? p.order[first + n] / p.divide : first + n;
    const uint16_t *x = p.X + x_row * p.ldx + 8 * q;

    float4v acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    const float4v none = {0, 0, 0, 0};
    const short one = DT == VBR_F16 ? 0x3C00 : 0x3F80;
    const short8v ones = {one, one, one, one, one, one, one, one};
    const int begin = (int)(p.k_tiles * wave / kMmWaves), end = (int)(p.k_tiles * (wave + 1) / kMmWaves);
    for (int t = begin; t < end; ++t) {
        uint4v w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = p.tiles[(row[h] * p.k_tiles + t) * 64 + lane];
        short8v xf[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xf[i] = short8v{0, 0, 0, 0, 0, 0, 0, 0};
            if (n < count && 4 * t + i < p.k_chunks) xf[i] = *reinterpret_cast<const short8v *>(x + 128 * (int64_t)t + 32 * i);
        }
#pragma unroll
        for (int c = 0; c < 4; c += CH) {
            const int64_t g = CH < 4 ? (int64_t)t * (4 / CH) + c / CH : t / p.tiles_a_group;
            float4v of_x = none, part[2] = {none, none};
#pragma unroll
            for (int i = c; i < c + CH; ++i) {
                of_x = mfma16x16x32<DT>(xf[i], ones, of_x);
#pragma unroll
                for (int h = 0; h < 2; ++h) part[h] = mfma16x16x32<DT>(xf[i], sixteen_plus<DT>(w[h][i]), part[h]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t at = (row[h] * p.groups_kept + g) * 16 + n;
                const float s = as_f32<DT>(p.scales[at]), z = ZEROS ? 16.f + (float)p.zeros[at] : 24.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[h][i] = __builtin_fmaf(s, __builtin_fmaf(-z, of_x[i], part[h][i]), acc[h][i]);
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][h][4 * q + i][n] = acc[h][i];
    __syncthreads();
    constexpr int kOut = GATED ? 1 : 2;
    for (int at = threadIdx.x; at < kOut * 16 * kTokens; at += 64 * kMmWaves) {
        const int col = at & 15, h = GATED ? 0 : at >> 4 & 1, token = at / (16 * kOut);
        const int64_t out_col = (GATED ? blockIdx.x : r0 + h) * 16 + col;
        if (token >= count || out_col >= p.half || (!GATED && r0 + h > last)) continue;
        float v[2];
#pragma unroll
        for (int u = 0; u < (GATED ? 2 : 1); ++u) {
            v[u] = 0;
            for (int k = 0; k < kMmWaves; ++k) v[u] += sums[k][GATED ? u : h][token][col];
        }
        const float y = GATED ? silu(v[0]) * v[1] : v[0];
        const int64_t y_row = ROUTED ? p.order[first + token] : first + token;
        if constexpr (F32) static_cast<float *>(p.Y)[y_row * p.ldy + out_col] = y;
        else if constexpr (DT == VBR_F16) static_cast<_Float16 *>(p.Y)[y_row * p.ldy + out_col] = (_Float16)y;
        else static_cast<__bf16 *>(p.Y)[y_row * p.ldy + out_col] = (__bf16)y;
    }
}

using MmKernel = void (*)(MmParams);
template <int DT, int CH, bool ZEROS, bool GATED>
MmKernel mm_kernel(bool routed, bool f32)
{
    return routed ? (f32 ? q4_mm_kernel<DT, CH, ZEROS, GATED, true, true> : q4_mm_kernel<DT, CH, ZEROS, GATED, true, false>)
                  : (f32 ? q4_mm_kernel<DT, CH, ZEROS, GATED, false, true> : q4_mm_kernel<DT, CH, ZEROS, GATED, false, false>);
}
template <int DT, int CH>
MmKernel mm_kernel(bool zeros, bool gated, bool routed, bool f32)
{
    return zeros ? (gated ? mm_kernel<DT, CH, true, true>(routed, f32) : mm_kernel<DT, CH, true, false>(routed, f32))
                 : (gated ? mm_kernel<DT, CH, false, true>(routed, f32) : mm_kernel<DT, CH, false, false>(routed, f32));
}
MmKernel mm_kernel(int32_t dtype, int32_t group, bool zeros, bool gated, bool routed, bool f32)
{
    if (dtype == VBR_F16)
        return group == 32 ? mm_kernel<VBR_F16, 1>(zeros, gated, routed, f32) : group == 64 ? mm_kernel<VBR_F16, 2>(zeros, gated, routed, f32) : mm_kernel<VBR_F16, 4>(zeros, gated, routed, f32);
    return group == 32 ? mm_kernel<VBR_BF16, 1>(zeros, gated, routed, f32) : group == 64 ? mm_kernel<VBR_BF16, 2>(zeros, gated, routed, f32) : mm_kernel<VBR_BF16, 4>(zeros, gated, routed, f32);
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
    p.scales = reinterpret_cast<const uint16_t *>(d + h->scales_at());
    p.zeros = reinterpret_cast<const uint8_t *>(d + h->zeros_at());
    p.X = static_cast<const uint16_t *>(X_dev);
    p.Y = Y_dev;
    p.ldx = ldx;
    p.ldy = ldy;
    p.n_rows = n_rows;
    p.k_tiles = h->k_tiles();
    p.tile_rows = h->tile_rows();
    p.groups_kept = h->groups_kept();
    p.half = (int32_t)h->rows();
    p.n_cols = (int32_t)h->n_cols;
    p.k_chunks = (int32_t)(h->n_cols / 32);
    p.tiles_a_group = h->group < 128 ? 1 : h->group / 128;
    return p;
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
    p.n_kept = h->n_mats * h->tile_rows() * h->groups_kept() * 16;
    p.n_rows = h->n_rows;
    p.half = h->rows();
    p.n_cols = h->n_cols;
    p.tile_rows = h->tile_rows();
    p.k_tiles = h->k_tiles();
    p.groups = h->groups();
    p.groups_kept = h->groups_kept();
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
    const MmParams p = mm_params(h, X_dev, ldx, Y_dev, ldy, n_rows);
    const int64_t y = (n_rows + kTokens - 1) / kTokens, x = (p.tile_rows + 1) / 2;
    if (y > 65535) return VBR_EUNSUPPORTED;
    hipLaunchKernelGGL(mm_kernel(h->dtype, h->group, h->zeros, h->gated, false, y_type == VBR_F32), dim3((unsigned)x, (unsigned)y), dim3(64 * kMmWaves), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched();
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
    p.offsets = reinterpret_cast<const int32_t *>(d);
    p.order = reinterpret_cast<const int32_t *>(d + parts.order);
    p.plan_tiles = reinterpret_cast<const int2 *>(d + parts.tiles);
    p.divide = (int32_t)(n_pairs / n_rows);
    const int64_t x = (p.tile_rows + 1) / 2;
    if (parts.n_tiles > 65535) return VBR_EUNSUPPORTED;
    hipLaunchKernelGGL(mm_kernel(h->dtype, h->group, h->zeros, h->gated, true, y_type == VBR_F32), dim3((unsigned)x, (unsigned)parts.n_tiles), dim3(64 * kMmWaves), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched();
}

extern "C" void q4_free(q4_t *h) { delete h; }
