// Pieces of rows: the low half of an fp32 value, and 16 bytes of a row at any alignment.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace mnnb {

// lo = v - trunc(v), exact, and half a unit of the 11 bits that the tensor core reads of it, which so rounds what it cuts off.  (What has no
// finite value may have any low half: its high one is not finite either, and its sums are taken again.)
__device__ __forceinline__ float low_half(float v)
{
    const float lo = v - __uint_as_float(__float_as_uint(v) & 0xffffe000u);
    return __uint_as_float(__float_as_uint(lo) + 0x1000u);
}
__device__ __forceinline__ float4 low_half(float4 v) { return make_float4(low_half(v.x), low_half(v.y), low_half(v.z), low_half(v.w)); }

// 16 bytes that start `by` bytes into the 32 of p and q; by < 16, a multiple of EB.
template <int EB>
__device__ __forceinline__ uint4 shift_pieces(const uint4& p, const uint4& q, uint32_t by)
{
    uint32_t u0 = p.x, u1 = p.y, u2 = p.z, u3 = p.w, u4 = q.x, u5 = q.y, u6 = q.z;
    if (by & 8u) { u0 = u2; u1 = u3; u2 = u4; u3 = u5; u4 = u6; u5 = q.w; u6 = 0; }
    if (by & 4u) { u0 = u1; u1 = u2; u2 = u3; u3 = u4; u4 = u5; }
    if (EB == 2 && (by & 2u)) {
        u0 = __funnelshift_r(u0, u1, 16);
        u1 = __funnelshift_r(u1, u2, 16);
        u2 = __funnelshift_r(u2, u3, 16);
        u3 = __funnelshift_r(u3, u4, 16);
    }
    return make_uint4(u0, u1, u2, u3);
}

// The 16 bytes at `at` of the tensor [begin, end), of which the first `valid` are wanted, the others zero.
template <int EB>
__device__ __forceinline__ uint4 load_piece(const char* at, int valid, const char* begin, const char* end)
{
    const uint32_t by = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15u);
    const char* lo = at - by;
    if (valid >= 16 && by == 0) return __ldg(reinterpret_cast<const uint4*>(at));
    if (valid >= 16 && lo >= begin && lo + 32 <= end)
        return shift_pieces<EB>(__ldg(reinterpret_cast<const uint4*>(lo)), __ldg(reinterpret_cast<const uint4*>(lo) + 1), by);
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

// A warp's pass over the pieces of a row of `bytes` bytes at `row` of the tensor [begin, end): take(index, piece), with the loads of four
// pieces in flight per lane.  The pieces whose aligned neighbours all lie in the tensor go without checks.
template <int EB, typename Take>
__device__ __forceinline__ void for_pieces(const char* row, int bytes, const char* begin, const char* end, int lane, Take&& take)
{
    const int whole = bytes >> 4, pieces = (bytes + 15) >> 4;
    const uint32_t by = (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u);
    const uint4* const lo = reinterpret_cast<const uint4*>(row - by);
    // [first, last): pieces i whose lo[i] and, where the row is not aligned, lo[i + 1] lie in the tensor
    const int first = row - by >= begin ? 0 : 1;
    const int last = by == 0 ? whole : (int)min((long long)whole, (long long)((end - reinterpret_cast<const char*>(lo)) >> 4) - 1);
    if (lane < first) take(lane, load_piece<EB>(row + lane * 16ll, min(16, bytes - lane * 16), begin, end));
    int i = first + lane;
    for (; i + 96 < last; i += 128) {
        uint4 p[4], q[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) p[s] = __ldg(lo + i + 32 * s);
        if (by) {
#pragma unroll
            for (int s = 0; s < 4; ++s) q[s] = __ldg(lo + i + 32 * s + 1);
#pragma unroll
            for (int s = 0; s < 4; ++s) p[s] = shift_pieces<EB>(p[s], q[s], by);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) take(i + 32 * s, p[s]);
    }
    for (; i < pieces; i += 32) take(i, load_piece<EB>(row + i * 16ll, min(16, bytes - i * 16), begin, end));
}

}  // namespace mnnb
