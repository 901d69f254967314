// Sums and maxima over lanes side by side, in a fixed order.
#pragma once
#include <hip/hip_runtime.h>

namespace mpcnn {

// The sum over 16 lanes side by side, in all of them
template <int CTRL>
__device__ __forceinline__ float add_moved(float s)
{
    return s + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, s), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum16(float s)
{
    s = add_moved<0x128>(s);   // row_ror:8, 4, 2, 1
    s = add_moved<0x124>(s);
    s = add_moved<0x122>(s);
    return add_moved<0x121>(s);
}
__device__ __forceinline__ float sum64(float s)
{
    s = sum16(s);
    s += __shfl_xor(s, 16, 64);
    return s + __shfl_xor(s, 32, 64);
}

// The wave's largest value (all lanes active), largest64 in a scalar register; a NaN is passed over
template <int CTRL, int ROWS>
__device__ __forceinline__ float larger_moved(float m)
{
    const int o = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, m), __builtin_bit_cast(int, m), CTRL, ROWS, 0xf, false);
    return fmaxf(m, __builtin_bit_cast(float, o));
}
__device__ __forceinline__ float largest16(float m)        // of 16 lanes side by side, in all of them
{
    m = larger_moved<0x128, 0xf>(m);   // row_ror:8, 4, 2, 1
    m = larger_moved<0x124, 0xf>(m);
    m = larger_moved<0x122, 0xf>(m);
    return larger_moved<0x121, 0xf>(m);
}
__device__ __forceinline__ float largest_of16s(float m)    // of what 16 lanes have each
{
    m = larger_moved<0x142, 0xa>(m);   // row_bcast:15 into rows 1 and 3,
    m = larger_moved<0x143, 0xc>(m);   // row_bcast:31 into rows 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, m), 63));
}
__device__ __forceinline__ float largest64(float m) { return largest_of16s(largest16(m)); }

// The largest of 4 lanes side by side, in all of them
__device__ __forceinline__ unsigned largest4(unsigned m)
{
    const unsigned a = (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true);   // quad_perm:[1,0,3,2]
    m = a > m ? a : m;
    const unsigned b = (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true);   // quad_perm:[2,3,0,1]
    return b > m ? b : m;
}

}  // namespace mpcnn
