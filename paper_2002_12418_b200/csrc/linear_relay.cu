// Ahead of the matrix product on pairs of SMs, or on tiles of rows that TMA cannot copy: operands laid into the workspace in the form that its copies need, a warp
// per row (several where rows are few).
//   rows that do not start on 16-byte boundaries -> the same values in rows that do
//   fp32, for pairs -> two halves in FP16: the row is scaled by a power of two that brings its largest finite value to [2^14, 2^15), then
//     hi = rn(v), lo = rn(v - hi).  hi + lo is v to 2^-24 of it down to 2^-16 of the row's largest value, and to 2^-39 of the
//     largest below (FP16's own smallest step); the scaling is exact and undone in the product's epilogue.
// One launch for both operands.  Bound by HBM bandwidth; small beside the product that it serves.
#include <cuda_fp16.h>

#include "linear.h"
#include "linear_piece.cuh"
#include "kernels.h"
#include "umma.cuh"

namespace mnnb {

namespace {

constexpr int kWarps = 8;

struct RelayParams {
    LinearRelayed t[2];
    int K, share;                    // share: warps of a CTA per row
    long long ld_out;                // elements
};

// EB: bytes of an element; HALVES: fp32 values to their halves, else copied
template <int EB, bool HALVES>
__global__ void __launch_bounds__(32 * kWarps)
linear_relay_kernel(RelayParams p)
{
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per_cta = kWarps / p.share;
    const int group = warp / p.share, slice = warp - group * p.share;
    const int bytes = p.K * EB, part = ((bytes + 15) / 16 + p.share - 1) / p.share;        // this warp's part of a row, in pieces of 16 bytes
    const int at0 = min(slice * part, (bytes + 15) / 16), some = min(part * 16, bytes - min(at0 * 16, bytes));
    __shared__ uint32_t part_most[kWarps];
    const long long all = p.t[0].rows + p.t[1].rows;
    for (long long r0 = (long long)blockIdx.x * per_cta; r0 < all; r0 += (long long)gridDim.x * per_cta) {
        const bool there = r0 + group < all;                         // (a warp without a row goes along to the barriers)
        const long long r = there ? r0 + group : r0;
        const bool second = r >= p.t[0].rows;
        const LinearRelayed& t = second ? p.t[1] : p.t[0];
        const long long row = second ? r - p.t[0].rows : r;
        const char* const begin = static_cast<const char*>(t.src);
        const char* const end = begin + ((t.rows - 1) * t.ld + p.K) * EB;
        const char* const src = begin + row * t.ld * EB + at0 * 16;
        if (HALVES) {
            uint32_t most = 0;
            if (some > 0) for_pieces<EB>(src, some, begin, end, lane, [&](int, const uint4& v) {
                const uint32_t u[4] = {v.x & 0x7fffffffu, v.y & 0x7fffffffu, v.z & 0x7fffffffu, v.w & 0x7fffffffu};
#pragma unroll
                for (int j = 0; j < 4; ++j) most = max(most, u[j] < 0x7f800000u ? u[j] : 0u);
            });
            most = __reduce_max_sync(0xffffffffu, most);
            if (p.share > 1) {
                if (lane == 0) part_most[warp] = most;
                __syncthreads();
                for (int i = 0; i < p.share; ++i) most = max(most, part_most[group * p.share + i]);
                __syncthreads();
            }
            if (!there) continue;
            const int up = min(14 - ((int)(most >> 23) - 127), 127);                 // -113..127
            const float scale = __uint_as_float((uint32_t)(up + 127) << 23);
            __half* const hi = static_cast<__half*>(t.same) + row * p.ld_out + at0 * 4;
            __half* const lo = static_cast<__half*>(t.low) + row * p.ld_out + at0 * 4;
            if (some > 0) for_pieces<EB>(src, some, begin, end, lane, [&](int i, const uint4& v) {
                const float f[4] = {__uint_as_float(v.x) * scale, __uint_as_float(v.y) * scale, __uint_as_float(v.z) * scale, __uint_as_float(v.w) * scale};
                __half h[4], l[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    h[j] = __float2half_rn(f[j]);
                    l[j] = __float2half_rn(f[j] - __half2float(h[j]));
                }
                *reinterpret_cast<uint2*>(hi + i * 4) = *reinterpret_cast<const uint2*>(h);
                *reinterpret_cast<uint2*>(lo + i * 4) = *reinterpret_cast<const uint2*>(l);
            });
            if (lane == 0 && slice == 0) t.up[row] = up;
        } else {
            uint4* const out = reinterpret_cast<uint4*>(static_cast<char*>(t.same) + row * p.ld_out * EB) + at0;
            if (there && some > 0) for_pieces<EB>(src, some, begin, end, lane, [&](int i, const uint4& v) { out[i] = v; });
        }
    }
}

}  // namespace

cudaError_t launch_linear_relay(const LinearRelayed& x, const LinearRelayed& w, int K, int elem_bytes, long long ld_out, int num_sms, cudaStream_t stream)
{
    RelayParams p = {};
    p.t[0] = x;
    p.t[1] = w;
    p.K = K;
    p.ld_out = ld_out;
    // several warps to a row where rows are few (5 x 12009 x 94 fp32, this and its product: 42 us with a warp each, 32), and for halves
    // where they are long, so that the second pass finds in L2 what the first one read (4728 x 11520 x 400: 309 us with a warp each, 261)
    const long long rows = x.rows + w.rows, row_bytes = (long long)K * elem_bytes;
    p.share = 1;
    while (p.share < kWarps && ((rows * p.share < 16ll * num_sms && row_bytes >= 2048ll * p.share) || (x.low && row_bytes >= 8192ll * p.share))) p.share *= 2;
    const long long blocks = (rows * p.share + kWarps - 1) / kWarps, most = 16ll * num_sms;
    auto kern = elem_bytes == 2 ? linear_relay_kernel<2, false> : x.low ? linear_relay_kernel<4, true> : linear_relay_kernel<4, false>;
    return launch_overlapped(kern, dim3((unsigned)(blocks < most ? blocks : most)), dim3(32 * kWarps), 0, stream, p);
}

}  // namespace mnnb
