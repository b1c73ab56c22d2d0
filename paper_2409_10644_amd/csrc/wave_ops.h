// What the kernels that share out their own work do across a wavefront.
#pragma once
#include <hip/hip_runtime.h>

namespace {

// Inclusive sum and maximum over the wavefront's lanes (numbers >= 0).
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_scan(int v)
{
    v += from_lane<0x111, 0xf>(v);   // from 1, 2, 4, 8 lanes below within 16, then the sums of 16 and 32
    v += from_lane<0x112, 0xf>(v);
    v += from_lane<0x114, 0xf>(v);
    v += from_lane<0x118, 0xf>(v);
    v += from_lane<0x142, 0xa>(v);
    v += from_lane<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ int wave_max(int v)
{
    v = max(v, from_lane<0x111, 0xf>(v));
    v = max(v, from_lane<0x112, 0xf>(v));
    v = max(v, from_lane<0x114, 0xf>(v));
    v = max(v, from_lane<0x118, 0xf>(v));
    v = max(v, from_lane<0x142, 0xa>(v));
    v = max(v, from_lane<0x143, 0xc>(v));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_last(int v) { return __builtin_amdgcn_readlane(v, 63); }
// n / d for 0 <= n < 2^30, d > 0 and a quotient below 2^20: rounded to 24 bits twice it is off by less than one.
__device__ __forceinline__ int small_div(int n, int d)
{
    const int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d)), r = n - q * d;
    return q + (r >= d) - (r < 0);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

}  // namespace
