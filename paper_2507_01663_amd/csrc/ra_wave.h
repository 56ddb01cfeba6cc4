// Sums over the lanes of a wave, inside the vector unit (no LDS trip).
#pragma once
#include <hip/hip_runtime.h>

namespace ra {

// What a lane gets from another (CTRL), in the rows of sixteen lanes that ROWS names, and `none` where there is no other.  A sum goes by
// steps inside rows, then from the last lane of a row to the next row, then from the lower half to the upper.
template <int CTRL, int ROWS> __device__ __forceinline__ int from_lane(int x, int none) { return __builtin_amdgcn_update_dpp(none, x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS> __device__ __forceinline__ double from_lane(double x)
{
    const int2 w = {__double2loint(x), __double2hiint(x)};
    return __hiloint2double(from_lane<CTRL, ROWS>(w.y, 0), from_lane<CTRL, ROWS>(w.x, 0));
}
__device__ __forceinline__ double wave_scan(double x)           // the sum up to this lane, itself included
{
    x += from_lane<0x111, 0xf>(x);
    x += from_lane<0x112, 0xf>(x);
    x += from_lane<0x114, 0xf>(x);
    x += from_lane<0x118, 0xf>(x);
    x += from_lane<0x142, 0xa>(x);
    x += from_lane<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ int wave_scan(int x)
{
    x += from_lane<0x111, 0xf>(x, 0);
    x += from_lane<0x112, 0xf>(x, 0);
    x += from_lane<0x114, 0xf>(x, 0);
    x += from_lane<0x118, 0xf>(x, 0);
    x += from_lane<0x142, 0xa>(x, 0);
    x += from_lane<0x143, 0xc>(x, 0);
    return x;
}

} // namespace ra
