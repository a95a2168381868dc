// Reductions over groups of 1, 2, 4, ..., 64 neighbouring lanes, and the element types of score matrices and gradients.
#pragma once
#include "common.hpp"

namespace grouter {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_move(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

// The value that the lane's partner in step `STEP` of a butterfly over its group holds.  After the steps before it, all lanes of
// STEP neighbours hold the same value, so mirrors of 8 and 16 lanes do what an exchange at distance 4 and 8 would.
template <int STEP>
__device__ __forceinline__ uint32_t partner(uint32_t v) {
    if constexpr (STEP == 1) return dpp_move<0xB1>(v);          // quad_perm [1,0,3,2]
    else if constexpr (STEP == 2) return dpp_move<0x4E>(v);     // quad_perm [2,3,0,1]
    else if constexpr (STEP == 4) return dpp_move<0x141>(v);    // row_half_mirror
    else if constexpr (STEP == 8) return dpp_move<0x140>(v);    // row_mirror
    else if constexpr (STEP == 16) return (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x401F);   // lane ^ 16
    else return (uint32_t)__shfl_xor((int)v, 32);
}

// Every lane of a group of L gets the group's result; all lanes of the wave have to be active.
template <int L, int STEP = 1>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
    if constexpr (STEP >= L) return v;
    else return group_max<L, 2 * STEP>(max(v, partner<STEP>(v)));
}
template <int L, int STEP = 1>
__device__ __forceinline__ float group_max(float v) {
    if constexpr (STEP >= L) return v;
    else return group_max<L, 2 * STEP>(fmaxf(v, __uint_as_float(partner<STEP>(__float_as_uint(v)))));
}
template <int L, int STEP = 1>
__device__ __forceinline__ float group_sum(float v) {
    if constexpr (STEP >= L) return v;
    else return group_sum<L, 2 * STEP>(v + __uint_as_float(partner<STEP>(__float_as_uint(v))));
}

struct Fp32 {
    typedef float stored;
    static __device__ __forceinline__ float widen(float v) { return v; }
    static __device__ __forceinline__ float narrow(float v) { return v; }
};
struct Bf16 {
    typedef uint16_t stored;
    static constexpr uint16_t kInf = 0x7f80;
    static __device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t narrow(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }   // to nearest, ties to even
};
struct Fp16 {
    typedef uint16_t stored;
    static constexpr uint16_t kInf = 0x7c00;
    static __device__ __forceinline__ float widen(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ uint16_t narrow(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

}  // namespace grouter
