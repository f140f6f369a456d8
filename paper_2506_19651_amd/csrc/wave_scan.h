// Inclusive scans over a wavefront in vector registers.
#pragma once
#include <hip/hip_runtime.h>

namespace pevlm {

// x of the lane that the DPP control names, 0 where there is none or the row is not in row_mask
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int32_t from_lane(int32_t x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}

// inclusive scan over the wavefront: within rows of 16 lanes, then the rows' last lanes on to the rows behind
template <class T, class Add>
__device__ __forceinline__ T wave_scan(T x, Add add)
{
    const auto step = [&](int32_t y) { x = add(x, __builtin_bit_cast(T, y)); };
    step(from_lane<0x111>(__builtin_bit_cast(int32_t, x)));  // row_shr:1
    step(from_lane<0x112>(__builtin_bit_cast(int32_t, x)));
    step(from_lane<0x114>(__builtin_bit_cast(int32_t, x)));
    step(from_lane<0x118>(__builtin_bit_cast(int32_t, x)));
    step(from_lane<0x142, 0xa>(__builtin_bit_cast(int32_t, x)));  // row_bcast:15
    step(from_lane<0x143, 0xc>(__builtin_bit_cast(int32_t, x)));  // row_bcast:31
    return x;
}

}  // namespace pevlm
