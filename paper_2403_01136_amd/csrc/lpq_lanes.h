// Exchanges between the lanes of a wave, and the pointer types of the global-to-LDS loads: what the attention kernels share.
#pragma once
#include "lpq_device.h"

namespace lpq {

constexpr float LOG2E = 1.4426950408889634f;

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

// ---- lane exchanges without LDS: DPP inside 16 lanes, the row / half swaps above them -----------
template <int CTRL>
__device__ __forceinline__ float dpp_move(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// {v of lane % 32, v of lane % 32 + 32}, and the same for lanes 16 apart within 32.  The results go through scalars: a
// bit cast of a vector's element reads element 0 whichever is named.
__device__ __forceinline__ f2 both_halves(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = t[0], b = t[1];
    return f2{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ f2 both_rows(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto t = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a = t[0], b = t[1];
    return f2{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
// v <- op(v, v of a partner lane), doubling the group that shares the result: 2, 4, 8, 16 lanes by DPP
// (quad_perm [1,0,3,2], quad_perm [2,3,0,1], row_half_mirror, row_mirror), 32 and 64 by the swaps
template <int LANES, typename Op>
__device__ __forceinline__ float group_reduce(float v, Op op)
{
    if constexpr (LANES >= 2) v = op(v, dpp_move<0xB1>(v));
    if constexpr (LANES >= 4) v = op(v, dpp_move<0x4E>(v));
    if constexpr (LANES >= 8) v = op(v, dpp_move<0x141>(v));
    if constexpr (LANES >= 16) v = op(v, dpp_move<0x140>(v));
    if constexpr (LANES >= 32) { const f2 t = both_rows(v); v = op(t[0], t[1]); }
    if constexpr (LANES >= 64) { const f2 t = both_halves(v); v = op(t[0], t[1]); }
    return v;
}
struct OpAdd { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct OpMax { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

}  // namespace lpq
