// Sums over neighbouring lanes of a wave.
#pragma once
#include <hip/hip_runtime.h>

namespace lp {

// v of another lane: what DPP reaches within a row of 16 lanes.
template <int CONTROL>
__device__ __forceinline__ float from_lane(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true));
}
// Sums over groups of `lanes` neighbouring lanes, for all of them.  Each step adds what the lanes of the other half have: of pairs and fours by
// permutations of four lanes, of eight and 16 by mirrors (all lanes of a half hold the same by then), of 32 and 64 by swaps of rows.
// (By shuffles through LDS a step takes some 100 cycles instead of 10, and the four to six sums of a position follow one another.)
template <int K>
__device__ __forceinline__ void lane_sums(float (&v)[K], int lanes)
{
    auto each = [&](auto&& f) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = f(v[k]);
    };
    if (lanes >= 2) each([](float a) { return a + from_lane<0xb1>(a); });    // quad_perm 1, 0, 3, 2
    if (lanes >= 4) each([](float a) { return a + from_lane<0x4e>(a); });    // quad_perm 2, 3, 0, 1
    if (lanes >= 8) each([](float a) { return a + from_lane<0x141>(a); });   // row_half_mirror
    if (lanes >= 16) each([](float a) { return a + from_lane<0x140>(a); });  // row_mirror
    if (lanes >= 32)
        each([](float a) {
            const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, a), false, false);
            return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
        });
    if (lanes >= 64)
        each([](float a) {
            const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, a), false, false);
            return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
        });
}

}  // namespace lp
