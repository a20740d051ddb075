// Pieces of rows: the low half of an fp32 value, and 16 bytes of a row at any alignment.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace mnnb {

// lo = v - trunc(v) (no number for an infinity, which makes its sums none either: they are taken again)
__device__ __forceinline__ float low_half(float v) { return v - __uint_as_float(__float_as_uint(v) & 0xffffe000u); }
__device__ __forceinline__ float4 low_half(float4 v) { return make_float4(low_half(v.x), low_half(v.y), low_half(v.z), low_half(v.w)); }

// The 16 bytes at `at` of the tensor [begin, end), of which the first `valid` are wanted, the others zero.
template <int EB>
__device__ __forceinline__ uint4 load_piece(const char* at, int valid, const char* begin, const char* end)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(at);
    const char* lo = at - (a & 15u);
    if (valid >= 16 && (a & 15u) == 0) return __ldg(reinterpret_cast<const uint4*>(at));
    if (valid >= 16 && lo >= begin && lo + 32 <= end) {
        const uint4 p = __ldg(reinterpret_cast<const uint4*>(lo)), q = __ldg(reinterpret_cast<const uint4*>(lo) + 1);
        uint32_t u0 = p.x, u1 = p.y, u2 = p.z, u3 = p.w, u4 = q.x, u5 = q.y, u6 = q.z;
        if (a & 8u) { u0 = u2; u1 = u3; u2 = u4; u3 = u5; u4 = u6; u5 = q.w; u6 = 0; }
        if (a & 4u) { u0 = u1; u1 = u2; u2 = u3; u3 = u4; u4 = u5; }
        if (EB == 2 && (a & 2u)) {
            u0 = __funnelshift_r(u0, u1, 16);
            u1 = __funnelshift_r(u1, u2, 16);
            u2 = __funnelshift_r(u2, u3, 16);
            u3 = __funnelshift_r(u3, u4, 16);
        }
        return make_uint4(u0, u1, u2, u3);
    }
    uint32_t u[4] = {0, 0, 0, 0};
    if (EB == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j * 4 < valid) u[j] = __ldg(reinterpret_cast<const uint32_t*>(at) + j);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j * 2 < valid) u[j >> 1] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(at) + j) << ((j & 1) * 16);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

}  // namespace mnnb
