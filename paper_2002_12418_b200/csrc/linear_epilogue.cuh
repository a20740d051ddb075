// What the kernels of the matrix product over rows share: element types, activations, and the order of work items.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/mnn_conv.h"
#include "cluster.cuh"
#include "linear.h"
#include "umma.cuh"

namespace mnnb {

template <int TYPE> struct Elem;
template <> struct Elem<MNN_TYPE_FP32> {
    typedef float T;
    static __device__ __forceinline__ float load(const T* p) { return *p; }
    static __device__ __forceinline__ T round(float v) { return v; }
};
template <> struct Elem<MNN_TYPE_BF16> {
    typedef __nv_bfloat16 T;
    static __device__ __forceinline__ float load(const T* p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ T round(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<MNN_TYPE_FP16> {
    typedef __half T;
    static __device__ __forceinline__ float load(const T* p) { return __half2float(*p); }
    static __device__ __forceinline__ T round(float v) { return __float2half_rn(v); }
};

// v / (1 + e^-t): with the fast exponential and division where the result is rounded to 16 bits, with the exact ones in fp32.  The fast
// exponential's error grows with |t|, by some 2^-23 of the result per unit: below 2^-16 at |t| = 88, where it leaves fp32's range, so it vanishes
// in a rounding of 2^-9; FP16's results are zero from |t| of some 20 on, with errors below 2^-18 up to there.  (Where e^-t passes 2^126 the result,
// then below 2^-119 in size, may come out as zero.)
template <int TYPE>
__device__ __forceinline__ float times_logistic(float v, float t)
{
    return TYPE == MNN_TYPE_FP32 ? v / (1.0f + expf(-t)) : __fdividef(v, 1.0f + __expf(-t));
}

// v (1 + erf(v / sqrt 2)) / 2 = v times the normal distribution's tail h = erfc(|v| / sqrt 2) / 2, or 1 - h above zero: 1 + erf would cancel
// below zero (4 % off at -5, nothing left at -5.6).  h = e^(-v^2/2) q(t), t = 1 / (1 + c |v|), with q minimax (by the exchange algorithm) in
// relative error: degree 6 and 1.9e-6 where the result is rounded to 16 bits, degree 8 and 3.1e-8 in fp32.  All errors together: below
// (1.5 v^2 + 20) 2^-24 of the result in fp32 (the square's, times its size, and 20 of t's two roundings, q's and e's), 52 for 16 bits.
// So, by erfcf and with 1 + erff, us: 2048 x 512 x 8192 BF16 46, 78 and 54, fp32 100, 127 and 106, 402 x 66 x 82722 fp32 251, 327 and 235.
template <int TYPE>
__device__ __forceinline__ float gelu(float v)
{
    float t, e, h;
    const float a = TYPE == MNN_TYPE_FP32 ? fminf(fabsf(v), 1e18f) : fabsf(v), d = fmaf(a, TYPE == MNN_TYPE_FP32 ? 0.295f : 0.3f, 1.0f);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(d));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * v * -0.72134752044448170f));
    if (TYPE == MNN_TYPE_FP32) {
        t = fmaf(t, fmaf(-d, t, 1.0f), t);
        h = 0.039721813f;
        h = fmaf(h, t, -0.18476456f);
        h = fmaf(h, t, 0.27361652f);
        h = fmaf(h, t, -0.11981790f);
        h = fmaf(h, t, 0.16803710f);
        h = fmaf(h, t, 0.084059909f);
        h = fmaf(h, t, 0.12186044f);
        h = fmaf(h, t, 0.11726858f);
        h = fmaf(h, t, 1.8129702e-5f);
    } else {
        h = -0.084593246f;
        h = fmaf(h, t, 0.24057280f);
        h = fmaf(h, t, -0.048644457f);
        h = fmaf(h, t, 0.16476454f);
        h = fmaf(h, t, 0.10670450f);
        h = fmaf(h, t, 0.12127471f);
        h = fmaf(h, t, -7.9789934e-5f);
    }
    h *= e;
    return v * (v < 0.0f ? h : 1.0f - h);
}

// The activations keep a NaN a NaN (ReLU too, unlike fmaxf).
template <int TYPE, int NUM>
__device__ __forceinline__ void activate(float (&v)[NUM], int act)
{
    if (act == MNN_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < NUM; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];
    } else if (act == MNN_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < NUM; ++j) v[j] = gelu<TYPE>(v[j]);
    } else if (act == MNN_ACT_GELU_TANH) {
        // (1 + tanh z) / 2 = 1 / (1 + e^-2z),  2 z = 2 sqrt(2/pi) (v + 0.044715 v^3)
#pragma unroll
        for (int j = 0; j < NUM; ++j) v[j] = times_logistic<TYPE>(v[j], 1.5957691216057308f * v[j] * fmaf(0.044715f * v[j], v[j], 1.0f));
    } else if (act == MNN_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < NUM; ++j) v[j] = times_logistic<TYPE>(v[j], v[j]);
    }
}

// Sums of NUM rows m0.. of x for one feature n -> y.  `rows` of them exist.  In a warp the lanes are 32 consecutive features,
// so that every load of the residual and every store of y is one contiguous run of 32 elements, whatever the alignment.
template <int TYPE, int NUM>
struct LinearStore {
    typedef typename Elem<TYPE>::T T;
    typename Elem<TYPE>::T r[NUM];
    __device__ __forceinline__ void fetch(const LinearEpilogue& e, long long m0, int rows, int n, bool n_ok)
    {
        if (e.res_mode == MNN_RESIDUAL_NONE || !n_ok) return;
        const T* p = static_cast<const T*>(e.residual) + m0 * e.ldr + n;
#pragma unroll
        for (int j = 0; j < NUM; ++j)
            if (j < rows) r[j] = p[j * e.ldr];
    }
    __device__ __forceinline__ void store(const LinearEpilogue& e, float (&v)[NUM], float bias, long long m0, int rows, int n, bool n_ok)
    {
        if (!n_ok) return;
#pragma unroll
        for (int j = 0; j < NUM; ++j) v[j] += bias;
        if (e.res_mode == MNN_RESIDUAL_BEFORE) {
#pragma unroll
            for (int j = 0; j < NUM; ++j)
                if (j < rows) v[j] += Elem<TYPE>::load(&r[j]);
        }
        activate<TYPE>(v, e.act);
        if (e.res_mode == MNN_RESIDUAL_AFTER) {
#pragma unroll
            for (int j = 0; j < NUM; ++j)
                if (j < rows) v[j] += Elem<TYPE>::load(&r[j]);
        }
        T* q = static_cast<T*>(e.y) + m0 * e.ldy + n;
#pragma unroll
        for (int j = 0; j < NUM; ++j)
            if (j < rows) q[j * e.ldy] = Elem<TYPE>::round(v[j]);
    }
};

// fp32: sums without a finite value are taken again, term by term (an infinity's low half is no number).  The loop is kept out of
// line and behind one branch: inlined, the compiler ran all of it under predicates for every sum (28 us of 54 at K = 1024).
// A thread may do this for 64 sums while other roles wait for its accumulator, longer than their waits last (256 x 256 sums on a pair:
// some 26 us per term): it counts `alive` up, in each of the CTAS whose roles wait, every kRetakeTick terms.  (By whole warps, 32 terms of
// one sum at a time, it took a quarter of that, but the call then cost sums without an infinity more registers: 3136 x 1024 x 1024 39 -> 42 us.)
constexpr int kRetakeTick = 8192;
template <int CTAS>
static __device__ __noinline__ float retake_sum(const float* x, const float* w, int K, int* alive)
{
    float t = 0.0f;
    int k = 0;
    for (; k + 8 <= K && t == t; k += 8) {           // (a NaN stays one)
        if ((k & (kRetakeTick - 1)) == 0) {
            if (CTAS == 1) atomicAdd(alive, 1);
            else
                for (uint32_t r = 0; r < CTAS; ++r)
                    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], 1;" ::"r"(ptx::map_to_rank(ptx::smem_u32(alive), r)) : "memory");
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) t = fmaf(x[k + j], w[k + j], t);
    }
    for (; k < K && t == t; ++k) t = fmaf(x[k], w[k], t);
    return t;
}
template <int CTAS, int NUM>
__device__ __forceinline__ void retake_sums(float (&s)[NUM], int rows, long long m0, int n, const float* x, long long ldx, const float* w, long long ldw, int K, int* alive)
{
    bool any = false;
#pragma unroll
    for (int j = 0; j < NUM; ++j) any = any || (j < rows && !isfinite(s[j]));
    if (!any) return;
#pragma unroll
    for (int j = 0; j < NUM; ++j)
        if (j < rows && !isfinite(s[j])) s[j] = retake_sum<CTAS>(x + (m0 + j) * ldx, w + (long long)n * ldw, K, alive);
}

template <int TYPE>
__device__ __forceinline__ float linear_bias(const LinearEpilogue& e, int n, bool n_ok)
{
    return e.bias && n_ok ? Elem<TYPE>::load(static_cast<const typename Elem<TYPE>::T*>(e.bias) + n) : 0.0f;
}

// Work items in groups of eight feature blocks, the feature block running fastest within a group: the items that run at one time
// cover a compact rectangle of the result, and their operands are read from L2 by several of them.
__device__ __forceinline__ void linear_item(long long item, int n_fblocks, int n_mblocks, int* fb, int* mb)
{
    const long long per_group = 8ll * n_mblocks;
    const int g = (int)(item / per_group);
    const int rem = (int)(item - g * per_group);
    const int width = min(8, n_fblocks - g * 8);
    *mb = rem / width;
    *fb = g * 8 + (rem - *mb * width);
}

}  // namespace mnnb
