// es_lanes.h -- sums and maxima over groups of a wave's lanes by register moves (no LDS).
#ifndef ES_SPMM_LANES_H
#define ES_SPMM_LANES_H

#include "es_common.h"

namespace {

// v as the lanes of the DPP pattern CTRL hand it over (a move inside rows of 16 lanes)
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_move(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ __forceinline__ float dpp_move(float v) { return __uint_as_float(dpp_move<CTRL>(__float_as_uint(v))); }

// Swaps the odd rows of 16 lanes of a with the even rows of b (ROWS16), or the upper half of a with the
// lower half of b: afterwards a holds both registers' even rows (lower halves) and b their odd rows (upper halves).
template <bool ROWS16>
__device__ __forceinline__ void lane_swap(uint32_t& a, uint32_t& b)
{
    if constexpr (ROWS16) {
        const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        a = r[0]; b = r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
        a = r[0]; b = r[1];
    }
}
template <bool ROWS16>
__device__ __forceinline__ void lane_swap(float& a, float& b)
{
    uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    lane_swap<ROWS16>(x, y);
    a = __uint_as_float(x); b = __uint_as_float(y);
}

// op over every aligned group of TEAM lanes; every lane of the group gets the result.  Inside 16 lanes:
// neighbours, pairs of a quad, then mirrored halves (whose lanes already agree).
template <int TEAM, class T, class Op>
__device__ __forceinline__ T team_reduce(T v, Op&& op)
{
    static_assert(TEAM == 1 || TEAM == 2 || TEAM == 4 || TEAM == 8 || TEAM == 16 || TEAM == 32 || TEAM == 64, "");
    if constexpr (TEAM >= 2) v = op(v, dpp_move<0xB1>(v));        // quad_perm [1, 0, 3, 2]
    if constexpr (TEAM >= 4) v = op(v, dpp_move<0x4E>(v));        // quad_perm [2, 3, 0, 1]
    if constexpr (TEAM >= 8) v = op(v, dpp_move<0x141>(v));       // row_half_mirror
    if constexpr (TEAM >= 16) v = op(v, dpp_move<0x140>(v));      // row_mirror
    if constexpr (TEAM >= 32) { T w = v; lane_swap<true>(v, w); v = op(v, w); }
    if constexpr (TEAM >= 64) { T w = v; lane_swap<false>(v, w); v = op(v, w); }
    return v;
}

}  // namespace

#endif  // ES_SPMM_LANES_H
