// What the attention kernels over 16- or 32-bit and over 4-bit caches share: how a call is cut into chunks, and their joining.
#pragma once

#include "cache_device.h"

namespace paep {

static constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;

struct AttendPlan {
    int G, head_blocks;          // query heads of a key-value head, blocks of 16 of them
    int chunk, S;                // positions of a workgroup, chunks of the longest sequence
    int rows;                    // B * Hkv
    float* o;                    // [rows][S][G][Dv] outputs of the chunks, each over its own sum (S > 1)
    float2* ml;                  // [rows][S][G] the maxima of their scores, and their sums (S > 1 or mass)
    float* scores;               // [rows][S][G][chunk] (mass)
};

// the part of a sequence that is looked at: positions start .. len, counted in chunks from start rounded down to a multiple of 16
struct Range { int start, first, len, chunks; };
__device__ __forceinline__ Range range_of(const int32_t* lengths, const int32_t* starts, int b, int max_len, int chunk)
{
    Range r;
    r.len = clamped_length(lengths, b, max_len);
    r.start = starts && starts[b] > 0 ? starts[b] : 0;
    r.first = r.start & ~15;
    r.chunks = r.start < r.len ? (int)(((uint32_t)(r.len - r.first) + (uint32_t)chunk - 1) / (uint32_t)chunk) : 0;
    return r;
}

// Of differences of scores only: a score in units of log2 may be past the largest number where the score itself is not.
__device__ __forceinline__ float exp_(float v) { return __builtin_amdgcn_exp2f(v * LOG2E); }
// the reference point of exponentials whose maximum is m: 0 where nothing was above -infinity
__device__ __forceinline__ float origin(float m) { return m == -__builtin_inff() ? 0.0f : m; }

// How the positions are cut: workgroups aimed at, the fewest positions of a chunk, what its size is a multiple of, and the most
// positions where there is one sequence and where there are several.
struct AttendCut { int target, least, step, most_alone, most_several; };
AttendPlan attend_plan(const AttendArgs& a, const AttendCut& cut);
bool attend_plan_fits(const AttendArgs& a, const AttendCut& cut);
size_t attend_plan_workspace(const AttendArgs& a, const AttendCut& cut);
// the plan with its places in the workspace
AttendPlan attend_plan_placed(const AttendArgs& a, const AttendCut& cut);
// joins the chunks, and adds up the weights where there is a mass output
hipError_t launch_attend_join(const AttendArgs& a, const AttendPlan& pl);

}  // namespace paep
