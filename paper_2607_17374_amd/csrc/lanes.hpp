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
// Step K of a reduction: v combined with that of the lane 2^K away (or one
// that holds the same), op commutative.
template <int K, typename T, typename Op>
__device__ inline T lane_step(T v, Op&& op) {
    static_assert(sizeof(T) == 4, "one register");
    auto bits = [](T x) { return __builtin_bit_cast(uint32_t, x); };
    auto value = [](uint32_t x) { return __builtin_bit_cast(T, x); };
    if constexpr (K == 0) return op(v, value(lane_move<0xb1>(bits(v))));        // lanes 1 0 3 2
    else if constexpr (K == 1) return op(v, value(lane_move<0x4e>(bits(v))));   // 2 3 0 1
    else if constexpr (K == 2) return op(v, value(lane_move<0x141>(bits(v))));  // mirrored in 8
    else if constexpr (K == 3) return op(v, value(lane_move<0x140>(bits(v))));  // mirrored in 16
    else if constexpr (K == 4) {
        const auto s = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
        return op(value((uint32_t)s[0]), value((uint32_t)s[1]));
    } else {
        const auto s = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
        return op(value((uint32_t)s[0]), value((uint32_t)s[1]));
    }
}
template <int LG, typename T, typename Op>
__device__ inline T lanes_of(T v, Op&& op) {
    if constexpr (LG > 0) v = lane_step<LG - 1>(lanes_of<LG - 1>(v, op), op);
    return v;
}
// v over the 2^lg lanes; lg is the same for all lanes
template <typename T, typename Op>
__device__ inline T lanes_all(T v, int lg, Op&& op) {
    switch (lg) {
        case 0: return v;
        case 1: return lanes_of<1>(v, op);
        case 2: return lanes_of<2>(v, op);
        case 3: return lanes_of<3>(v, op);
        case 4: return lanes_of<4>(v, op);
        case 5: return lanes_of<5>(v, op);
        default: return lanes_of<6>(v, op);
    }
}
__device__ inline float lanes_sum(float v, int lg) {
    return lanes_all(v, lg, [](float a, float b) { return a + b; });
}
// two sums, step by step beside one another
__device__ inline float2 lanes_sum2(float2 v, int lg) {
    auto add = [](float a, float b) { return a + b; };
    switch (lg) {
        case 0: return v;
        case 1: return {lanes_of<1>(v.x, add), lanes_of<1>(v.y, add)};
        case 2: return {lanes_of<2>(v.x, add), lanes_of<2>(v.y, add)};
        case 3: return {lanes_of<3>(v.x, add), lanes_of<3>(v.y, add)};
        case 4: return {lanes_of<4>(v.x, add), lanes_of<4>(v.y, add)};
        case 5: return {lanes_of<5>(v.x, add), lanes_of<5>(v.y, add)};
        default: return {lanes_of<6>(v.x, add), lanes_of<6>(v.y, add)};
    }
}
__device__ inline float lanes_max(float v, int lg) {
    return lanes_all(v, lg, [](float a, float b) { return fmaxf(a, b); });
}
// the sum over lanes that agree in their low lg bits (the same columns of a
// wave's groups)
__device__ inline float groups_sum(float v, int lg) {
    auto add = [](float a, float b) { return a + b; };
    if (lg < 3)
        for (int o = 1 << lg; o < 8; o <<= 1) v += __shfl_xor(v, o, 64);
    if (lg < 4) v = add(v, __uint_as_float(lane_move<0x128>(__float_as_uint(v))));  // 8 round in 16
    if (lg < 5) v = lane_step<4>(v, add);
    if (lg < 6) v = lane_step<5>(v, add);
    return v;
}
__device__ inline float lane_value(float v, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

}  // namespace taurus
