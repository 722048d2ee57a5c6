// Reductions over groups of 2^lg neighbouring lanes of a wave (lg <= 6), in
// registers: the first four steps by the exchanges inside a row of 16 lanes,
// the last two by swapping rows.  Every lane ends with the same bits.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace taurus {

template <int CTRL>
__device__ inline uint32_t lane_move(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
// v combined with that of the group's lanes: op(op(...)), op commutative
template <typename T, typename Op>
__device__ inline T lanes_all(T v, int lg, Op&& op) {
    static_assert(sizeof(T) == 4, "one register");
    auto bits = [](T x) { return __builtin_bit_cast(uint32_t, x); };
    auto value = [](uint32_t x) { return __builtin_bit_cast(T, x); };
    if (lg > 0) v = op(v, value(lane_move<0xb1>(bits(v))));   // lanes 1 0 3 2
    if (lg > 1) v = op(v, value(lane_move<0x4e>(bits(v))));   // 2 3 0 1
    if (lg > 2) v = op(v, value(lane_move<0x141>(bits(v))));  // mirrored in 8
    if (lg > 3) v = op(v, value(lane_move<0x140>(bits(v))));  // mirrored in 16
    if (lg > 4) {
        const auto s = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
        v = op(value((uint32_t)s[0]), value((uint32_t)s[1]));
    }
    if (lg > 5) {
        const auto s = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
        v = op(value((uint32_t)s[0]), value((uint32_t)s[1]));
    }
    return v;
}
__device__ inline float lanes_sum(float v, int lg) {
    return lanes_all(v, lg, [](float a, float b) { return a + b; });
}
__device__ inline float lanes_max(float v, int lg) {
    return lanes_all(v, lg, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline int lanes_min(int v, int lg) {
    return lanes_all(v, lg, [](int a, int b) { return min(a, b); });
}
__device__ inline float lane_value(float v, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

}  // namespace taurus
