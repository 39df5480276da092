// What route.hip and q4.hip share: limits, the layout of a plan (route_plan), which the routed products read, and their launches' ends.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "vbr_host.h"

namespace vbrk {

constexpr int32_t kMaxExperts = 1024;              // one thread of a workgroup each, in the scan
constexpr int32_t kMaxTopK = 64, kMaxGroups = 64;  // one lane each
constexpr int64_t kMaxPairs = 1 << 30;             // positions are 32 bits
constexpr int64_t kPlanAlone = 4096;               // pairs up to which one workgroup groups them all
constexpr int64_t kPlanPart = 1024;                // pairs of a workgroup, at least, where there are several

constexpr int64_t kMostThreads = 0xFFFFFFFFll;     // of a launch

// i / d for i below 2^31: 2^(31 + l) / d rounded up, l the bits of d - 1, times i
struct Divide {
    uint32_t factor;
    int32_t shift;
    static Divide by(int64_t d)
    {
        const int l = d > 1 ? 64 - __builtin_clzll((unsigned long long)d - 1) : 0;
        return {(uint32_t)(((1ull << (31 + l)) + d - 1) / d), 31 + l};
    }
    __host__ __device__ uint32_t operator()(uint32_t i) const { return (uint32_t)((uint64_t)i * factor >> shift); }
};

inline bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline int launched()                              // what became of the last launch
{
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        set_last_hip_error((int)e);
        return VBR_EHIP;
    }
    return VBR_OK;
}

// Byte offsets in a plan: int32 offsets [n_experts + 1] at 0, int32 order [n_pairs], PlanTile tiles [n_tiles],
// int32 counts [n_parts][n_experts].
struct PlanTile {
    int32_t expert, first, count, n_tiles;         // positions first .. first + count - 1 of the order; count 0: no tile; how many there are
};
struct PlanParts {
    int64_t order, tiles, counts, total;
    int64_t n_tiles, n_parts, per_wave;
    int32_t tile_rows;
};
PlanParts plan_parts(int64_t n_pairs, int32_t n_experts);
bool plan_sizes_ok(int64_t n_pairs, int32_t n_experts);

}  // namespace vbrk
