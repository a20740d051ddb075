// The matrix product over rows of linear.cu for groups of up to four rows of x: every byte of w is used for a handful of multiply-adds, so
// the kernel is a stream of w.  A warp takes two features (one where that leaves too few warps), its lanes 16-byte pieces of both
// rows of w and of the rows of x (which stay in L1), and sums in fp32; where few features leave too few warps, several warps of a
// CTA share the K loop and add up in shared memory, in warp order.  No tensor map, barrier pipeline or tensor memory has to be
// set up.  Bound by HBM (or L2) bandwidth and, below a few MB, by latency.
#include "linear_epilogue.cuh"
#include "linear_piece.cuh"
#include "kernels.h"
#include "umma.cuh"

namespace mnnb {

namespace {

constexpr int kWarps = 8;

struct FewParams {
    int M, N, K, share;              // share: warps of a CTA per group of features
    const void *x, *w;
    long long ldx, ldw;
    LinearEpilogue epi;
};

template <int TYPE> struct Wide;     // 16 bytes as fp32 values
template <> struct Wide<MNN_TYPE_FP32> {
    static constexpr int kNum = 4;
    static __device__ __forceinline__ void get(const uint4& q, float (&v)[4])
    {
        v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
    }
};
template <> struct Wide<MNN_TYPE_BF16> {
    static constexpr int kNum = 8;
    static __device__ __forceinline__ void get(const uint4& q, float (&v)[8])
    {
        const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
};
template <> struct Wide<MNN_TYPE_FP16> {
    static constexpr int kNum = 8;
    static __device__ __forceinline__ void get(const uint4& q, float (&v)[8])
    {
        const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
};

// ROWS: rows of x in a group; FEATS: features of a warp; ALIGNED: all rows start on 16-byte boundaries, else their pieces are
// shifted together from aligned ones (the second of which the neighbouring lane has brought into L1).
template <int TYPE, int ROWS, int FEATS, bool ALIGNED>
__global__ void __launch_bounds__(32 * kWarps)
linear_few_kernel(FewParams p)
{
    typedef typename Elem<TYPE>::T T;
    constexpr int NUM = Wide<TYPE>::kNum;
    // pieces of a row that a lane has in flight (8 for 4, 1 x 2048 x 8192 BF16 7.6 -> 6.2 us, 1 x 4096 x 4096 8.4 -> 7.5; fp32, where a warp's
    // rows are twice as long, 1 x 4096 x 16384 43 -> 48)
    constexpr int STEP = !ALIGNED || ROWS * FEATS > 4 ? 2 : TYPE != MNN_TYPE_FP32 && ROWS * FEATS <= 2 ? 8 : 4;
    constexpr int EB = sizeof(T);
    __shared__ float part[kWarps][ROWS * FEATS];
    const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31;
    const int groups = kWarps / p.share;                 // groups of features in this CTA
    const int group = warp / p.share, slice = warp - group * p.share;
    const long long f0 = ((long long)blockIdx.x * groups + group) * FEATS;
    const int m0 = blockIdx.y * ROWS;                    // first row of x

    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();

    float sum[ROWS][FEATS];
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
#pragma unroll
        for (int f = 0; f < FEATS; ++f) sum[m][f] = 0.0f;
    // rows behind the last one read the last one again; their sums are not stored
    const T *wr[FEATS], *xr[ROWS];
#pragma unroll
    for (int f = 0; f < FEATS; ++f) wr[f] = static_cast<const T*>(p.w) + min(f0 + f, (long long)p.N - 1) * p.ldw;
#pragma unroll
    for (int m = 0; m < ROWS; ++m) xr[m] = static_cast<const T*>(p.x) + (long long)min(m0 + m, p.M - 1) * p.ldx;
    const int pieces = p.K / NUM;
    const int begin = (int)((long long)pieces * slice / p.share), end = (int)((long long)pieces * (slice + 1) / p.share);
    const char *xb = static_cast<const char*>(p.x), *wb = static_cast<const char*>(p.w);
    const char *xe = xb + ((p.M - 1) * p.ldx + p.K) * EB, *we = wb + ((p.N - 1) * p.ldw + p.K) * EB;
    auto w_piece = [&](const T* row, int i) -> uint4 {
        if (ALIGNED) return __ldg(reinterpret_cast<const uint4*>(row) + i);
        return load_piece<EB>(reinterpret_cast<const char*>(row) + i * 16ll, 16, wb, we);
    };
    auto x_piece = [&](const T* row, int i) -> uint4 {
        if (ALIGNED) return __ldg(reinterpret_cast<const uint4*>(row) + i);
        return load_piece<EB>(reinterpret_cast<const char*>(row) + i * 16ll, 16, xb, xe);
    };
    auto take = [&](const uint4 (&wq)[FEATS], const uint4 (&xq)[ROWS]) {
        float wv[FEATS][NUM];
#pragma unroll
        for (int f = 0; f < FEATS; ++f) Wide<TYPE>::get(wq[f], wv[f]);
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
            float xv[NUM];
            Wide<TYPE>::get(xq[m], xv);
#pragma unroll
            for (int f = 0; f < FEATS; ++f)
#pragma unroll
                for (int j = 0; j < NUM; ++j) sum[m][f] = fmaf(xv[j], wv[f][j], sum[m][f]);
        }
    };
    int i = begin + lane;
    for (; i + 32 * (STEP - 1) < end; i += 32 * STEP) {
        uint4 wq[STEP][FEATS], xq[STEP][ROWS];
#pragma unroll
        for (int s = 0; s < STEP; ++s)
#pragma unroll
            for (int f = 0; f < FEATS; ++f) wq[s][f] = w_piece(wr[f], i + 32 * s);
#pragma unroll
        for (int s = 0; s < STEP; ++s)
#pragma unroll
            for (int m = 0; m < ROWS; ++m) xq[s][m] = x_piece(xr[m], i + 32 * s);
#pragma unroll
        for (int s = 0; s < STEP; ++s) take(wq[s], xq[s]);
    }
    for (; i < end; i += 32) {
        uint4 wq[FEATS], xq[ROWS];
#pragma unroll
        for (int f = 0; f < FEATS; ++f) wq[f] = w_piece(wr[f], i);
#pragma unroll
        for (int m = 0; m < ROWS; ++m) xq[m] = x_piece(xr[m], i);
        take(wq, xq);
    }
    // the elements behind the last whole piece
    const int rest = pieces * NUM + lane;
    if (slice == 0 && rest < p.K) {
#pragma unroll
        for (int m = 0; m < ROWS; ++m)
#pragma unroll
            for (int f = 0; f < FEATS; ++f) sum[m][f] = fmaf(Elem<TYPE>::load(xr[m] + rest), Elem<TYPE>::load(wr[f] + rest), sum[m][f]);
    }
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
#pragma unroll
        for (int f = 0; f < FEATS; ++f)
#pragma unroll
            for (int o = 16; o; o >>= 1) sum[m][f] += __shfl_xor_sync(0xffffffffu, sum[m][f], o);
    // lane m * FEATS + f stores one result
    float mine = 0.0f;
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
#pragma unroll
        for (int f = 0; f < FEATS; ++f)
            if (lane == m * FEATS + f) mine = sum[m][f];
    if (p.share > 1) {
        if (lane < ROWS * FEATS) part[warp][lane] = mine;
        __syncthreads();
        if (slice != 0) return;
        mine = 0.0f;
        if (lane < ROWS * FEATS)
            for (int s = 0; s < p.share; ++s) mine += part[warp + s][lane];
    }
    const int m = lane / FEATS;
    const long long n = f0 + (lane - m * FEATS);
    if (m0 + m < p.M && m < ROWS && n < p.N) {
        LinearStore<TYPE, 1> out;
        out.fetch(p.epi, m0 + m, 1, (int)n, true);
        float s[1] = {mine};
        out.store(p.epi, s, linear_bias<TYPE>(p.epi, (int)n, true), m0 + m, 1, (int)n, true);
    }
}

template <int TYPE, int ROWS>
cudaError_t run_rows(const FewParams& p, int feats, bool aligned, cudaStream_t stream)
{
    const long long per_cta = (long long)kWarps / p.share * feats, grid = (p.N + per_cta - 1) / per_cta;
    auto kern = feats == 2 ? (aligned ? linear_few_kernel<TYPE, ROWS, 2, true> : linear_few_kernel<TYPE, ROWS, 2, false>)
                           : (aligned ? linear_few_kernel<TYPE, ROWS, 1, true> : linear_few_kernel<TYPE, ROWS, 1, false>);
    return launch_overlapped(kern, dim3((unsigned)grid, (unsigned)((p.M + ROWS - 1) / ROWS)), dim3(32 * kWarps), 0, stream, p);
}

template <int TYPE>
cudaError_t run_few(const FewParams& p, int feats, bool aligned, cudaStream_t stream)
{
    return p.M == 1   ? run_rows<TYPE, 1>(p, feats, aligned, stream)
           : p.M == 2 ? run_rows<TYPE, 2>(p, feats, aligned, stream)
                      : run_rows<TYPE, 4>(p, feats, aligned, stream);
}

}  // namespace

cudaError_t launch_linear_few(const LinearShape& s, const LinearTiling& t, const void* x, const void* w, const LinearEpilogue& epi, cudaStream_t stream)
{
    FewParams p = {};
    p.M = s.M; p.N = s.N; p.K = s.K;
    p.share = t.split;
    p.x = x; p.w = w; p.ldx = s.ldx; p.ldw = s.ldw;
    p.epi = epi;
    const int eb = s.type == MNN_TYPE_FP32 ? 4 : 2;
    const bool aligned = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(w)) & 15u) == 0 && (s.ldx * eb) % 16 == 0 && (s.ldw * eb) % 16 == 0;
    switch (s.type) {
        case MNN_TYPE_FP32: return run_few<MNN_TYPE_FP32>(p, t.feats, aligned, stream);
        case MNN_TYPE_BF16: return run_few<MNN_TYPE_BF16>(p, t.feats, aligned, stream);
        default: return run_few<MNN_TYPE_FP16>(p, t.feats, aligned, stream);
    }
}

}  // namespace mnnb
