// Device helpers that the kernels share.
#pragma once

#include <cstdint>
#include <type_traits>

#include "vbr_spmm.h"

namespace vbrk {
namespace {

typedef short short8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

template <int DT>
__device__ __forceinline__ float4v mfma16x16x32(short8v a, short8v b, float4v c)
{
    if constexpr (DT == VBR_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, a), __builtin_bit_cast(bf16x8v, b), c, 0, 0, 0);
}

// 16 bytes per active lane from global memory straight into LDS, no register staging: lane l's
// data lands at lds_base + 16 l (lds_base wave-uniform, passed in M0).  The load is counted in
// vmcnt like any vector load; the compiler does not see it, so the waits are placed by hand.
// Every wave must issue the same, fixed number of these per K-step (never with an empty lane mask).
__device__ __forceinline__ void dma16(const void *gptr, uint32_t lds_base)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(gptr),
                 "s"((uint32_t)__builtin_amdgcn_readfirstlane(lds_base)) : "memory");
}

// exp(x), x at most a little above 0, within three half steps: 2^t (1 + r), r what rounding took from t = x log2(e); 0 for -inf and NaN, which count as -200 like all
// that is lower (t and r of an infinity have no difference).  Not for numbers far above 0: of a power that overflows the last line takes infinity from infinity.
__device__ __forceinline__ float exp_of(float x)
{
    constexpr float log2e = 1.44269502f, rest = 1.92596299e-8f, ln2 = 0.693147181f;      // log2(e) in two numbers
    x = __builtin_fmaxf(x, -200.f);
    const float t = x * log2e, r = __builtin_fmaf(x, rest, __builtin_fmaf(x, log2e, -t)), e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, r * ln2, e);
}
__device__ __forceinline__ float sigmoid_of(float x)      // of a NaN: 1
{
    const float e = exp_of(-__builtin_fabsf(x)), d = __builtin_amdgcn_rcpf(1.f + e);
    return x < 0.f ? e * d : d;
}

template <int N>
__device__ __forceinline__ void wait_vmcnt()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int I>
__device__ __forceinline__ uint32_t row_lane(uint32_t x)     // lane I of every row of 16 lanes, to the whole row
{
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x150 + I, 0xf, 0xf, true);
}

template <int I>
using constant = std::integral_constant<int, I>;
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F f)               // f(0) .. f(N - 1), each a constant
{
    if constexpr (I < N) {
        f(constant<I>());
        static_for<N, I + 1>(f);
    }
}

}  // namespace
}  // namespace vbrk
