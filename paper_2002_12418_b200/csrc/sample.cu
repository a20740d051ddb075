// Sampling: one token per row of logits l, from a given uniform number u per row.
//     w_i = exp((l_i - max l) / T)
// The candidates in the order of falling logits (ties: lower index first) are cut to a prefix by top-k (the first k), by top-p
// (those before which less than p of the mass of the k lies) and by min-p (w_i >= min_p); the token is the lowest index at which
// the running mass of what is kept, in index order, exceeds u times the whole.
//
// Every decision compares sums of weights with a border, so the sums have to be exact to below one weight and must not
// depend on the order in which threads add.  A weight is therefore evaluated in fp64 (relative error 5e-11) and held as an
// integer in units of 2^-scale (scale = 62 - log2 of the vocabulary, at most 45): the sums are of these integers, in any order, and no
// atomic changes a result.  The rounding to units makes them off by vocab / 2 units at most (by the root of that where roundings are
// independent; equals round alike).  A border of top-p lies at weights of at least (1 - p) / vocab, so that is below one weight unless
// 1 - p < vocab^2 2^-scale / 2.  (110674 values in steps of 0.5, T 0.29, p = 1 - 3.6e-7: one element of 1e-10 more than 11974 stays.)
//
// A cluster of CTAs holds a row in shared memory (read once from HBM).  No sort: the border of a prefix is one value of l.
//   top-k: a histogram of counts over 1024 bins of m - l (16 octaves of 64 bins, so that the bulk of a row spreads over many bins
//     whatever its scale, and an outlier or a mask of the type's lowest value costs nothing) gives the bin that holds it.
//   top-p: the same counts, each times the weight in the middle of its bin, tell within a few bins where the border must lie.
//     One pass then evaluates every weight once: those above that window are summed in registers, those inside go to 1024 finer
//     bins.  (Only where the border turns out to lie elsewhere, a histogram of all masses is taken.)
//   The few elements of the crossing bin are collected and ranked against each other; where there are many (ties by the thousand),
//     histograms over the range of their keys narrow it down to one value.
// Among equal values at the border the first ones by index are kept.
//
// Shared memory adds 32-bit integers in one instruction and 64-bit ones in a loop that retries, so masses are kept in three
// planes of 15 bits of the weight: a CTA holds at most 2^17 elements, and no plane's sum passes 32 bits.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/mnn_conv.h"
#include "cluster.cuh"
#include "kernels.h"
#include "linear.h"
#include "sample.h"
#include "umma.cuh"

namespace mnnb {

namespace {

typedef unsigned long long u64;

constexpr int kBins = 1024;
constexpr int kMaxWarps = 16;
constexpr int kMaxCtas = 8;
constexpr int kMaxSteps = 24;            // steps of 32 pieces of 16 bytes in a run: at most kMostBytes / 16 / 512, and one of rounding up
constexpr int kWindowRun = 256;          // elements of a warp from which on top-p counts first (64 rows of 32000 fp32 40.8 -> 32.9 us)
constexpr int kGather = 128;             // candidates that are ranked against each other instead of binned again
constexpr int kMaxScale = 45;
constexpr int kMostBytes = 176 * 1024;   // of a row's logits in one CTA: the largest vocabulary in fp32 over eight CTAs, and a step of rounding up

template <int TYPE> struct Logit { typedef float T; static constexpr int kVec = 4; };
template <> struct Logit<MNN_TYPE_FP16> { typedef __half T; static constexpr int kVec = 8; };
template <> struct Logit<MNN_TYPE_BF16> { typedef __nv_bfloat16 T; static constexpr int kVec = 8; };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }

// An integer that orders as the values do.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __float_as_uint(v);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of_key(uint32_t k) { return __uint_as_float(k >> 31 ? k ^ 0x80000000u : ~k); }

__device__ __forceinline__ uint32_t ld_cluster(const uint32_t* mine, uint32_t rank)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(ptx::map_to_rank(ptx::smem_u32(mine), rank)) : "memory");
    return v;
}
__device__ __forceinline__ u64 ld_cluster(const u64* mine, uint32_t rank)
{
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(ptx::map_to_rank(ptx::smem_u32(mine), rank)) : "memory");
    return v;
}

__device__ __forceinline__ void st_cluster(uint32_t* mine, uint32_t v, uint32_t rank)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ptx::map_to_rank(ptx::smem_u32(mine), rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(u64* mine, u64 v, uint32_t rank)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(ptx::map_to_rank(ptx::smem_u32(mine), rank)), "l"(v) : "memory");
}
// Lane r of a whole warp gives what lane 0 or 31 (`from`) holds to CTA r, in this CTA's place there.  What has few values is given before a
// barrier and not fetched behind it: a trip to another CTA's shared memory takes some 800 cycles, and a store is not waited for.
template <typename V>
__device__ __forceinline__ void give_all(V (&place)[kMaxCtas], V v, int from, uint32_t rank, uint32_t n_ctas, int lane)
{
    v = __shfl_sync(0xffffffffu, v, from);
    if (lane < (int)n_ctas) st_cluster(&place[rank], v, (uint32_t)lane);
}

// A value that was read from another CTA's shared memory has to be here before this thread arrives at the barrier behind which that
// memory is written again or its CTA is gone, and a use of it behind the barrier alone does not see to that.  So it decides a
// branch with a store that is never taken: the largest integer is no mass and no key.
__device__ __forceinline__ void landed(u64 v, uint32_t* never)
{
    if (v == ~0ull) *reinterpret_cast<volatile uint32_t*>(never) = 1;
}
// The same for what a row was given, by one sum of all of it.  (Whatever the values are: nothing reads what is stored.)  In a row without a
// candidate nothing else asks for these values before the last barrier.
__device__ __forceinline__ void landed(float temperature, float top_p, float min_p, float u, int top_k, uint32_t* never)
{
    const uint32_t sum = __float_as_uint(temperature) + __float_as_uint(top_p) + __float_as_uint(min_p) + __float_as_uint(u) + (uint32_t)top_k;
    if (sum == ~0u) *reinterpret_cast<volatile uint32_t*>(never) = 1;
}

// One value of every CTA, all reads in flight together; 0 for CTAs that are not there.
template <typename V>
__device__ __forceinline__ void ld_all(const V* mine, uint32_t n_ctas, V (&v)[kMaxCtas])
{
#pragma unroll
    for (uint32_t r = 0; r < kMaxCtas; ++r) v[r] = r < n_ctas ? ld_cluster(mine, r) : (V)0;
}
template <typename V>
__device__ __forceinline__ V sum_all(const V* mine, uint32_t n_ctas)
{
    V v[kMaxCtas], sum = 0;
    ld_all(mine, n_ctas, v);
#pragma unroll
    for (int r = 0; r < kMaxCtas; ++r) sum += v[r];
    return sum;
}

__device__ __forceinline__ u64 warp_sum(u64 v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename V>
__device__ __forceinline__ V warp_scan(V v, int lane)       // inclusive
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// 2^(d slope) with d slope <= 0, as an integer in units of 2^-scale, rounded to nearest.  2^r on [-1/2, 1/2] by 1 + r q(r) with q
// of degree 6 (minimax by the exchange algorithm, relative error 4.7e-11); additions of 1.5 * 2^52 round to integers.  Every
// operation is a named one: the sums of several passes are compared with each other, and a multiplication and an addition that
// the compiler joins in one place and not in another would make two weights of one value.
__device__ __forceinline__ double exp2_scaled(double d, double slope, int scale)      // 2^(d slope + scale)
{
    constexpr double kRound = 6755399441055744.0;
    const double y = __dmul_rn(d, slope);
    const double t = __dadd_rn(y, kRound);
    const double r = __dsub_rn(y, __dsub_rn(t, kRound));
    double q = 1.5196158527772698e-05;
    q = __fma_rn(q, r, 0.00015466756251326735);
    q = __fma_rn(q, r, 0.0013333935047106663);
    q = __fma_rn(q, r, 0.009618038132306056);
    q = __fma_rn(q, r, 0.05550410366001406);
    q = __fma_rn(q, r, 0.24022651066559253);
    q = __fma_rn(q, r, 0.6931471807045294);
    q = __fma_rn(q, r, 1.0);
    // times 2^(n + scale): an addition to the exponent
    return __hiloint2double(__double2hiint(q) + ((__double2loint(t) + scale) << 20), __double2loint(q));
}
__device__ __forceinline__ u64 exp2_units(double d, double slope, int scale)                  // rounded; below 2^46
{
    return (u64)__double_as_longlong(__dadd_rn(exp2_scaled(d, slope, scale), 4503599627370496.0)) & 0xfffffffffffffull;
}

// The element of a step of 32 * VEC: in one lane the index of its element at which the running mass exceeds `left`, in the others -1.
// `ties` equals of the border still count in this step; what lies above the border weighs `kept`.
template <int VEC, typename Kept>
__device__ __forceinline__ int draw_element(const float (&l)[VEC], u64 left, u64 ties, float border_value, bool equals_count, u64 border_w, int lane, Kept&& kept)
{
    uint32_t eq = 0;
#pragma unroll
    for (int j = 0; j < VEC; ++j) eq += equals_count && l[j] == border_value ? 1u : 0u;
    const uint32_t eq_incl = warp_scan(eq, lane);
    u64 t = ties > eq_incl - eq ? ties - (eq_incl - eq) : 0;         // this lane's equals that still count
    u64 w[VEC], sum = 0;
#pragma unroll
    for (int j = 0; j < VEC; ++j) w[j] = kept(l[j]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        if (!(l[j] > border_value)) {
            const bool e = equals_count && l[j] == border_value && t > 0;
            w[j] = e ? border_w : 0;
            t -= e ? 1 : 0;
        }
        sum += w[j];
    }
    const u64 incl = warp_scan(sum, lane);
    const unsigned hit = __ballot_sync(0xffffffffu, incl > left);
    int at = -1;
    if (hit && lane == __ffs(hit) - 1) {
        u64 rest = left - (incl - sum);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (at < 0 && rest < w[j]) at = j;
            rest -= w[j];
        }
    }
    return at;
}

// What a row was given.  One CTA of the cluster reads it and the others take it from there: their ways through the kernel hang on
// it, and must be one way even where a caller's program writes these arrays at the wrong time.
struct RowGiven {
    float temperature, top_p, min_p, u;
    int top_k;
    __device__ void load(const SampleArgs& a, int row)
    {
        temperature = a.temperature ? a.temperature[row] : 1.0f;
        top_p = a.top_p ? a.top_p[row] : 1.0f;
        min_p = a.min_p ? a.min_p[row] : 0.0f;
        u = a.u[row];
        top_k = a.top_k ? a.top_k[row] : 0;
    }
};
__device__ __forceinline__ float ld_cluster_float(const float* v) { return __uint_as_float(ld_cluster(reinterpret_cast<const uint32_t*>(v), 0)); }

struct Shared {
    RowGiven row;
    uint32_t count[kBins];
    uint32_t plane[3][kBins];        // masses by 15 bits: W & 0x7fff, (W >> 15) & 0x7fff, W >> 30
    // merged over the cluster: running sums through the bins of this CTA's share
    u64 run_mass[kBins];
    uint32_t run_count[kBins];
    u64 share_mass[kMaxCtas];        // of every CTA
    uint32_t share_count[kMaxCtas];
    u64 scan_mass[kMaxWarps];
    uint32_t scan_count[kMaxWarps];
    float scan_estimate[kMaxWarps];
    // sums of the warps' runs and of the CTAs
    u64 warp_mass[kMaxWarps], warp_above[kMaxWarps];
    uint32_t warp_count[kMaxWarps];
    u64 cta_whole[kMaxCtas], cta_above[kMaxCtas], cta_mass[kMaxCtas];        // of every CTA
    uint32_t cta_count[kMaxCtas];
    float warp_max[kMaxWarps];
    float max;                       // of this CTA
    uint32_t key_min, key_max;       // of this CTA
    uint32_t n_list;
    uint32_t list[kGather];          // keys of this CTA's candidates that are to be ranked
    uint32_t from_n[kMaxCtas], from[kMaxCtas][kGather];      // of every CTA's
    uint32_t all[kGather];           // the same in a row
    u64 all_mass[kGather];
    // what one warp found, for all
    uint32_t never;
    u64 found_mass, found_whole;
    uint32_t found_count, found_key, found_equal;
    int found_bin;
    u64 ties_kept[kMaxWarps];
    u64 step_mass[kMaxSteps];        // of 32 pieces each of the run that holds the token
    uint32_t step_count[kMaxSteps];
};

struct SampleParams {
    int rows, vocab, run, scale_log2, n_warps;
    long long ld, ld_probs;
    SampleArgs a;
};

template <int TYPE>
__global__ void __launch_bounds__(32 * kMaxWarps, 2)
sample_kernel(SampleParams p)
{
    typedef typename Logit<TYPE>::T T;
    constexpr int VEC = Logit<TYPE>::kVec;
    union Piece {
        uint4 v;
        T e[VEC];
        __device__ Piece() {}
    };
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ Shared sh;
    T* const held = reinterpret_cast<T*>(smem_raw);

    const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31, n_threads = blockDim.x;
    const uint32_t rank = ptx::cluster_ctarank();
    uint32_t n_ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ctas));
    const int row = blockIdx.x / n_ctas;
    auto sync_row = [&]() {
        __syncwarp();                                                // (the cluster's barrier takes whole warps)
        if (n_ctas > 1) ptx::cluster_sync_all();
        else __syncthreads();
    };
    auto clear = [&](bool masses) {
        for (int i = threadIdx.x; i < kBins; i += n_threads) {
            sh.count[i] = 0;
            if (masses) sh.plane[0][i] = sh.plane[1][i] = sh.plane[2][i] = 0;
        }
    };

    ptx::grid_launch_dependents();
    clear(true);
    if (threadIdx.x == 0) sh.n_list = 0;
    ptx::grid_dependency_wait();

    // ---- load.  Positions count from the 16-byte boundary at or before the row's first element; every warp holds a run of them.
    const int warp0 = warp * p.run;                                  // this warp's run in the CTA
    const int cta0 = (int)rank * p.run * p.n_warps;                  // this CTA in the row
    const T* const row_ptr = static_cast<const T*>(p.a.logits) + (long long)row * p.ld;
    const int shift = (int)((reinterpret_cast<uintptr_t>(row_ptr) & 15u) / sizeof(T));
    float top = -INFINITY;
    {
        const T* const base = row_ptr - shift;
        const int first = shift, last = shift + p.vocab;             // positions [first, last) are the row
        auto keep = [&](int i, const Piece& q) {
            *reinterpret_cast<uint4*>(held + warp0 + i) = q.v;
#pragma unroll
            for (int j = 0; j < VEC; ++j) top = fmaxf(top, widen(q.e[j]));       // fmaxf passes a NaN over
        };
        int i = lane * VEC;
        if (cta0 + warp0 >= first && cta0 + warp0 + p.run <= last)   // a run within the row: no checks, four loads in flight
            for (; i + 96 * VEC < p.run; i += 128 * VEC) {
                Piece q[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) q[j].v = __ldg(reinterpret_cast<const uint4*>(base + cta0 + warp0 + i + j * 32 * VEC));
#pragma unroll
                for (int j = 0; j < 4; ++j) keep(i + j * 32 * VEC, q[j]);
            }
        for (; i < p.run; i += 32 * VEC) {
            const int at = cta0 + warp0 + i;
            Piece q;
            if (at >= first && at + VEC <= last) {
                q.v = __ldg(reinterpret_cast<const uint4*>(base + at));
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) q.e[j] = at + j >= first && at + j < last ? base[at + j] : (T)(-INFINITY);
            }
            keep(i, q);
        }
    }
    if (threadIdx.x == 0 && rank == 0) sh.row.load(p.a, row);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) sh.warp_max[warp] = top;
    __syncthreads();
    if (warp == 0) {
        top = lane < p.n_warps ? sh.warp_max[lane] : -INFINITY;
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) sh.max = top;
    }
    sync_row();
    float m = -INFINITY;
    {
        uint32_t tops[kMaxCtas];
        ld_all(reinterpret_cast<const uint32_t*>(&sh.max), n_ctas, tops);
#pragma unroll
        for (uint32_t r = 0; r < kMaxCtas; ++r)
            if (r < n_ctas) m = fmaxf(m, __uint_as_float(tops[r]));
    }
    m += 0.0f;                                                       // (one zero)
    const float temperature = ld_cluster_float(&sh.row.temperature), top_p = ld_cluster_float(&sh.row.top_p), min_p = ld_cluster_float(&sh.row.min_p);
    const int top_k = (int)ld_cluster(reinterpret_cast<const uint32_t*>(&sh.row.top_k), 0);
    const float u_row = ld_cluster_float(&sh.row.u);
    landed(temperature, top_p, min_p, u_row, top_k, &sh.never);
    const bool one = !(temperature > 0.0f) || top_k == 1;            // the first largest alone
    const bool by_count = !one && top_k > 0 && top_k < p.vocab, by_mass = !one && top_p < 1.0f;
    const bool some = m > -INFINITY;

    // ---- weights.  Below `floor_l` they round to zero; with an infinite largest logit, or none but the first largest kept, all
    // but its equals do.  (No branch: evaluations for several elements are to overlap.)
    const bool m_inf = m == INFINITY;
    const double slope = one ? 0.0 : 1.4426950408889634074 / (double)temperature;         // log2(e) / T
    const float floor_l = m_inf || one ? m : m - (float)(p.scale_log2 + 3) * 0.6931472f * temperature;
    const double m_wide = (double)m;
    const u64 unit = 1ull << p.scale_log2;
    auto weight = [&](float l) -> u64 {
        const double d = l == m ? 0.0 : __dsub_rn((double)fmaxf(l, floor_l), m_wide);
        const u64 w = exp2_units(d, slope, p.scale_log2);
        return l < floor_l ? 0 : w;
    };
    auto key = [&](float l) { return key_of(l + 0.0f); };            // (one key for both zeros)
    // every element that this warp holds; what is no candidate is -infinity or NaN, and every test below is false for it
    auto for_each = [&](auto&& f) {
        for (int i = lane * VEC; i < p.run; i += 32 * VEC) {
            Piece q;
            q.v = *reinterpret_cast<const uint4*>(held + warp0 + i);
#pragma unroll
            for (int j = 0; j < VEC; ++j) f(widen(q.e[j]));
        }
    };
    // the same by whole pieces, so that what is evaluated for several elements overlaps
    auto for_each_piece = [&](auto&& f) {
        for (int i = lane * VEC; i < p.run; i += 32 * VEC) {
            Piece q;
            q.v = *reinterpret_cast<const uint4*>(held + warp0 + i);
            float l[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) l[j] = widen(q.e[j]);
            f(l);
        }
    };
    // 16 octaves of 64 bins of m - l, from 2^-10 to 2^6; what is nearer or further goes to the first or last bin
    constexpr int kFirstBin = (127 - 10) << 6;                       // the bits of 2^-10, over 2^17
    auto distance = [&](float l) { return l == m ? 0.0f : m - l; };
    auto bin_of = [&](float l) { return min(max((int)(__float_as_uint(distance(l)) >> 17) - kFirstBin, 0), kBins - 1); };
    auto add_mass = [&](int b, u64 w) {
        const uint32_t w0 = (uint32_t)w & 0x7fffu, w1 = (uint32_t)(w >> 15) & 0x7fffu, w2 = (uint32_t)(w >> 30);
        atomicAdd(&sh.plane[0][b], w0);
        if (w1) atomicAdd(&sh.plane[1][b], w1);
        if (w2) atomicAdd(&sh.plane[2][b], w2);
    };

    // What lies above the border that is being looked for, and the number of elements in the bin that holds it.
    u64 above_mass = 0;
    uint32_t above_count = 0, bin_count = 0;
    int bin = -1;
    // Sums the CTAs' histograms: each CTA takes a share of the bins.  Leaves them zeroed (for all after the next barrier).
    const int log_share = 10 - (31 - __clz((int)n_ctas)), share = 1 << log_share;
    auto merge = [&](bool masses) {
        sync_row();
        const int b0 = (int)rank * share, per = (share + n_threads - 1) / n_threads;
        u64 sum_m = 0;
        uint32_t sum_c = 0;
        for (int j = 0; j < per; ++j) {
            const int b = b0 + threadIdx.x * per + j;
            if (b < b0 + share) {
                if (n_ctas == 1) {
                    sum_c += sh.count[b];
                    if (masses) sum_m += (u64)sh.plane[0][b] + ((u64)sh.plane[1][b] << 15) + ((u64)sh.plane[2][b] << 30);
                } else {
                    sum_c += sum_all(&sh.count[b], n_ctas);
                }
                if (masses && n_ctas > 1) {                          // (a plane's sum over the cluster may pass 32 bits)
                    uint32_t w0[kMaxCtas], w1[kMaxCtas], w2[kMaxCtas];
                    ld_all(&sh.plane[0][b], n_ctas, w0);
                    ld_all(&sh.plane[1][b], n_ctas, w1);
                    ld_all(&sh.plane[2][b], n_ctas, w2);
#pragma unroll
                    for (int r = 0; r < kMaxCtas; ++r) sum_m += (u64)w0[r] + ((u64)w1[r] << 15) + ((u64)w2[r] << 30);
                }
                sh.run_mass[b] = sum_m;                              // (running within this thread; the rest is added below)
                sh.run_count[b] = sum_c;
            }
        }
        const u64 scan_m = masses ? warp_scan(sum_m, lane) : 0;
        const uint32_t scan_c = warp_scan(sum_c, lane);
        if (lane == 31) {
            sh.scan_mass[warp] = scan_m;
            sh.scan_count[warp] = scan_c;
        }
        __syncthreads();
        u64 base_m = scan_m - sum_m;
        uint32_t base_c = scan_c - sum_c;
        for (int i = 0; i < warp; ++i) {
            base_m += sh.scan_mass[i];
            base_c += sh.scan_count[i];
        }
        for (int j = 0; j < per; ++j) {
            const int b = b0 + threadIdx.x * per + j;
            if (b < b0 + share) {
                sh.run_mass[b] += base_m;
                sh.run_count[b] += base_c;
            }
        }
        if (warp == p.n_warps - 1) {                                 // this share's sums, to all
            give_all(sh.share_mass, base_m + sum_m, 31, rank, n_ctas, lane);
            give_all(sh.share_count, base_c + sum_c, 31, rank, n_ctas, lane);
        }
        sync_row();                                                  // (all have read this CTA's histograms)
        clear(masses);
    };
    // The first bin at which the running count (or mass) reaches `target`: found by one warp of each CTA, told to all.
    auto cross = [&](bool use_mass, u64 target) {
        if (warp == 0) {
            // the CTA whose share holds the target
            const u64 s_m = lane < (int)n_ctas ? sh.share_mass[lane] : 0;
            const uint32_t s_c = lane < (int)n_ctas ? sh.share_count[lane] : 0;
            const u64 i_m = above_mass + warp_scan(s_m, lane);
            const uint32_t i_c = above_count + warp_scan(s_c, lane);
            const unsigned in = __ballot_sync(0xffffffffu, use_mass ? i_m >= target : (u64)i_c >= target);
            const int r_lane = in ? __ffs(in) - 1 : 31;
            u64 base_m = __shfl_sync(0xffffffffu, i_m - s_m, r_lane);
            uint32_t base_c = __shfl_sync(0xffffffffu, i_c - s_c, r_lane), count = 0;
            int found = -1;
            if (in) {
                // every step-th place through the share, then the bins between two of them (a step is at most 32)
                const uint32_t r = (uint32_t)r_lane;
                const int b0 = (int)r * share, step = share >> 5;
                u64 bm = 0;                                          // running sums before the first place that reaches the target
                uint32_t bc = 0, cc = 0;
                auto first = [&](int at) {
                    const u64 rm = ld_cluster(&sh.run_mass[b0 + at], r);
                    const uint32_t rc = ld_cluster(&sh.run_count[b0 + at], r);
                    const unsigned hit = __ballot_sync(0xffffffffu, use_mass ? base_m + rm >= target : (u64)base_c + rc >= target);
                    const int src = hit ? __ffs(hit) - 1 : 31;
                    const u64 pm = __shfl_sync(0xffffffffu, rm, max(src - 1, 0));
                    const uint32_t pc = __shfl_sync(0xffffffffu, rc, max(src - 1, 0));
                    bm = src ? pm : bm;
                    bc = src ? pc : bc;
                    cc = __shfl_sync(0xffffffffu, rc, src);
                    return src;
                };
                const int lo = first((lane + 1) * step - 1) * step;
                found = b0 + (step > 1 ? lo + min(first(lo + min(lane, step - 1)), step - 1) : lo);
                count = cc - bc;
                base_m += bm;
                base_c += bc;
            }
            if (lane == 0) {
                sh.found_bin = found;
                sh.found_mass = base_m;
                sh.found_count = base_c;
                sh.found_equal = count;
            }
        }
        __syncthreads();
        bin = sh.found_bin;
        if (bin >= 0) {
            above_mass = sh.found_mass;
            above_count = sh.found_count;
            bin_count = sh.found_equal;
        }
        __syncthreads();
    };
    // Collects the keys of the n elements that `take` takes, in every CTA, with their weights if asked; their sum is returned.
    auto collect = [&](int n, bool masses, auto&& take) -> u64 {
        for_each([&](float l) {
            if (take(l)) sh.list[atomicAdd(&sh.n_list, 1u)] = key(l);
        });
        __syncthreads();
        const int mine = (int)sh.n_list;
        for (int i = threadIdx.x; i < mine * (int)n_ctas; i += n_threads) st_cluster(&sh.from[rank][i / (int)n_ctas], sh.list[i / (int)n_ctas], (uint32_t)(i % (int)n_ctas));
        if (threadIdx.x < n_ctas) st_cluster(&sh.from_n[rank], (uint32_t)mine, threadIdx.x);
        sync_row();
        u64 sum = 0;
        uint32_t have[kMaxCtas];
#pragma unroll
        for (uint32_t c = 0; c < kMaxCtas; ++c) have[c] = c < n_ctas ? sh.from_n[c] : 0;
        for (int at = threadIdx.x; at < n; at += n_threads) {
            int i = at;
            uint32_t r = 0;
#pragma unroll
            for (uint32_t c = 0; c + 1 < kMaxCtas; ++c)
                if (r == c && c + 1 < n_ctas && i >= (int)have[c]) {
                    i -= (int)have[c];
                    r = c + 1;
                }
            const uint32_t k = sh.from[r][i];
            const u64 w = masses ? weight(value_of_key(k)) : 0;
            sh.all[at] = k;
            sh.all_mass[at] = w;
            sum += w;
        }
        if (masses) {
            sum = warp_sum(sum);
            if (lane == 0) sh.scan_mass[warp] = sum;
        }
        __syncthreads();                                             // (before another collection there is a barrier of the cluster)
        if (threadIdx.x == 0) sh.n_list = 0;
        if (masses) {
            sum = 0;
            for (int i = 0; i < p.n_warps; ++i) sum += sh.scan_mass[i];
        }
        return sum;
    };
    uint32_t border_key = 0, border_equal = 0;                       // the border, and how many elements are equal to it
    // Of the n collected ones, the key at which the running count (or mass) reaches `target`.
    auto ranked = [&](int n, bool use_mass, bool masses, u64 target) {
        // 2^g threads of a warp per key
        int g = 0;
        while (g < 5 && n << (g + 1) <= n_threads) ++g;
        const int part = threadIdx.x & ((1 << g) - 1);
        for (int i0 = 0; i0 < n; i0 += n_threads >> g) {
            const int i = i0 + (threadIdx.x >> g);
            const uint32_t k = sh.all[min(i, n - 1)];
            u64 more = 0;
            uint32_t more_c = 0, equal = 0;
            for (int j = part; j < n; j += 1 << g) {
                const uint32_t other = sh.all[j];
                if (masses) more += other > k ? sh.all_mass[j] : 0;
                more_c += other > k ? 1u : 0u;
                equal += other == k ? 1u : 0u;
            }
            for (int o = 1 << g >> 1; o; o >>= 1) {
                if (masses) more += __shfl_xor_sync(0xffffffffu, more, o);
                more_c += __shfl_xor_sync(0xffffffffu, more_c, o);
                equal += __shfl_xor_sync(0xffffffffu, equal, o);
            }
            const u64 before = use_mass ? above_mass + more : (u64)above_count + more_c;
            const u64 here = use_mass ? (u64)equal * sh.all_mass[min(i, n - 1)] : (u64)equal;
            if (part == 0 && i < n && before < target && before + here >= target) {  // (equals write the same)
                sh.found_key = k;
                sh.found_equal = equal;
                sh.found_mass = above_mass + more;
                sh.found_count = above_count + more_c;
            }
        }
        __syncthreads();
        above_mass = sh.found_mass;
        above_count = sh.found_count;
        border_key = sh.found_key;
        border_equal = sh.found_equal;
        __syncthreads();
    };
    // The border within the crossing bin, whose elements `in` takes.
    auto narrow = [&](bool use_mass, u64 target, auto&& in) {
        if (bin_count <= (uint32_t)kGather) {
            const int n = (int)bin_count;
            collect(n, use_mass, in);
            ranked(n, use_mass, use_mass, target);
            return;
        }
        // many: the range of their keys, and a histogram over it, until one key is left
        uint32_t lo = 0, hi = 0;
        auto range = [&](auto&& take) {
            uint32_t mn = 0xffffffffu, mx = 0;
            if (threadIdx.x == 0) {
                sh.key_min = mn;
                sh.key_max = mx;
            }
            __syncthreads();
            for_each([&](float l) {
                if (take(l)) {
                    mn = min(mn, key(l));
                    mx = max(mx, key(l));
                }
            });
            mn = __reduce_min_sync(0xffffffffu, mn);
            mx = __reduce_max_sync(0xffffffffu, mx);
            if (lane == 0) {
                atomicMin(&sh.key_min, mn);
                atomicMax(&sh.key_max, mx);
            }
            sync_row();
            lo = 0xffffffffu;
            hi = 0;
            for (uint32_t r = 0; r < n_ctas; ++r) {
                lo = min(lo, ld_cluster(&sh.key_min, r));
                hi = max(hi, ld_cluster(&sh.key_max, r));
            }
            landed((u64)lo << 32 | hi, &sh.never);
            sync_row();
        };
        range(in);
        for (int level = 0; level < 4 && lo < hi; ++level) {          // (each divides the range by 1024)
            const int drop = max(0, 22 - __clz(hi - lo));            // (hi - key) >> drop < 1024
            const float v_lo = value_of_key(lo), v_hi = value_of_key(hi);
            for_each([&](float l) {
                if (l >= v_lo && l <= v_hi) {
                    const int b = (int)((hi - key(l)) >> drop);
                    atomicAdd(&sh.count[b], 1u);
                    if (use_mass) add_mass(b, weight(l));
                }
            });
            merge(use_mass);
            cross(use_mass, target);
            const uint32_t top_key = hi - ((uint32_t)max(bin, 0) << drop);
            if (drop == 0 || bin < 0) {
                lo = hi = top_key;
            } else {
                const float t_lo = value_of_key(max(lo, top_key - ((1u << drop) - 1u))), t_hi = value_of_key(top_key);
                range([&](float l) { return l >= t_lo && l <= t_hi; });
            }
        }
        border_key = lo;
        border_equal = bin_count;
    };

    // ---- the border: everything above its value is kept, and the first `ties` equal to it
    bool cut = some && one;
    u64 ties = 1;
    if (cut) border_key = key(m);
    u64 run_above = 0;                                               // mass of what lies above `window_top` in this warp's run
    float window_top = INFINITY;
    const bool by_window = by_mass && p.run >= kWindowRun;
    int n_listed = 0;                                                // elements that top-k's search left collected
    if (some && (by_count || by_window)) {
        for_each([&](float l) {
            if (l > -INFINITY) atomicAdd(&sh.count[bin_of(l)], 1u);
        });
        merge(false);
        if (by_count) {
            cross(false, (u64)top_k);
            if (bin >= 0) {                                          // else fewer candidates than k: all are kept
                const int b = bin;
                if (above_count + bin_count <= (uint32_t)kGather) {  // all down to the crossing bin are few: top-p can use them too
                    n_listed = (int)(above_count + bin_count);
                    collect(n_listed, by_mass, [&](float l) { return l > -INFINITY && bin_of(l) <= b; });
                    above_count = 0;
                    ranked(n_listed, false, by_mass, (u64)top_k);
                } else {
                    narrow(false, (u64)top_k, [&](float l) { return l > -INFINITY && bin_of(l) == b; });
                }
                ties = (u64)top_k - above_count;
                cut = true;
            }
        }
    }
    if (some && by_mass) {
        // kept while the mass before < p * whole: up to where the running mass reaches ceil(p * whole)
        auto border_target = [&](u64 whole) { return max(1ull, min((u64)ceil((double)fmaxf(top_p, 0.0f) * (double)whole), whole)); };
        u64 target = 0;
        bool done = false;
        if (n_listed) {                                              // few are left by top-k
            target = border_target(above_mass + ties * weight(value_of_key(border_key)));
            above_mass = 0;
            above_count = 0;
            ranked(n_listed, true, true, target);
            done = true;
        } else if (by_window && !cut) {
            // where the border must lie, by the counts and the weights in the middle of the bins
            const float s = (float)slope;
            auto middle = [&](int b) { return b == 0 ? 1.0f : exp2f(-s * __uint_as_float((uint32_t)((b + kFirstBin) << 17) + (1u << 16))); };
            auto estimate = [&](int b) {
                const uint32_t r = (uint32_t)(b >> log_share), c = ld_cluster(&sh.run_count[b], r);
                return (float)(c - (b & (share - 1) ? ld_cluster(&sh.run_count[b - 1], r) : 0u)) * middle(b);
            };
            const int per = kBins / n_threads;
            float part = 0.0f;
            for (int j = 0; j < per; ++j) part += estimate(threadIdx.x * per + j);
            float run = warp_scan(part, lane);
            if (lane == 31) sh.scan_estimate[warp] = run;
            if (threadIdx.x == 0) sh.found_bin = kBins - 1;
            __syncthreads();
            run -= part;
            float guess = 0.0f;
            for (int i = 0; i < p.n_warps; ++i) {
                if (i < warp) run += sh.scan_estimate[i];
                guess += sh.scan_estimate[i];
            }
            guess *= fmaxf(top_p, 0.0f);
            if (run <= guess && run + part > guess)
                for (int j = 0; j < per; ++j) {
                    run += estimate(threadIdx.x * per + j);
                    if (run > guess || j + 1 == per) {
                        atomicMin(&sh.found_bin, (int)threadIdx.x * per + j);        // (two neighbours may claim it by their rounding)
                        break;
                    }
                }
            __syncthreads();
            const int w0 = max(sh.found_bin - 1, 0), w1 = min(sh.found_bin + 2, kBins - 1);
            const uint32_t bits0 = (uint32_t)(w0 + kFirstBin) << 17;
            const float d0 = w0 ? __uint_as_float(bits0) : 0.0f;
            const float d1 = w1 == kBins - 1 ? INFINITY : __uint_as_float((uint32_t)(w1 + 1 + kFirstBin) << 17);
            // 1024 finer bins over the window of four
            auto fine = [&](float d) { return min(max((int)(__float_as_uint(d) - bits0) >> 9, 0), kBins - 1); };
            u64 sum_above = 0, sum = 0;
            for_each_piece([&](const float (&l)[VEC]) {
                u64 w[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[j] = weight(l[j]);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float d = distance(l[j]);
                    const bool counts = l[j] >= floor_l && l[j] > -INFINITY;
                    const u64 here = counts ? w[j] : 0;
                    sum += here;
                    sum_above += d < d0 ? here : 0;
                    if (counts && d >= d0 && d < d1) {
                        const int b = fine(d);
                        atomicAdd(&sh.count[b], 1u);
                        add_mass(b, here);
                    }
                }
            });
            run_above = warp_sum(sum_above);
            sum = warp_sum(sum);
            if (lane == 0) {
                sh.warp_above[warp] = run_above;
                sh.warp_mass[warp] = sum;
            }
            __syncthreads();
            if (warp == 0) {
                const u64 a = warp_sum(lane < p.n_warps ? sh.warp_above[lane] : 0), b = warp_sum(lane < p.n_warps ? sh.warp_mass[lane] : 0);
                give_all(sh.cta_above, a, 0, rank, n_ctas, lane);
                give_all(sh.cta_whole, b, 0, rank, n_ctas, lane);
            }
            merge(true);
            u64 whole = 0;
            above_mass = 0;
            above_count = 0;
            for (uint32_t r = 0; r < n_ctas; ++r) {
                above_mass += sh.cta_above[r];
                whole += sh.cta_whole[r];
            }
            target = border_target(whole);
            if (above_mass < target) {
                cross(true, target);
                done = bin >= 0;
            }
            if (done) {
                window_top = d0;
                // the fine bin as an interval of distances
                const float b0 = bin ? __uint_as_float(bits0 + ((uint32_t)bin << 9)) : d0;
                const float b1 = bin < kBins - 1 ? __uint_as_float(bits0 + ((uint32_t)(bin + 1) << 9)) : d1;
                narrow(true, target, [&](float l) {
                    const float d = distance(l);
                    return l >= floor_l && d >= b0 && d < b1;
                });
            } else {
                sync_row();                                          // (the histograms are zero again for all)
            }
        }
        if (!done) {                                                 // a histogram of all masses from top-k's border on
            const float from = cut ? value_of_key(border_key) : -INFINITY;
            const u64 surplus = cut ? (u64)(above_count + border_equal) - (u64)top_k : 0;      // equals of that border that do not count
            for_each([&](float l) {
                if (l >= from && l > -INFINITY) {
                    const int b = bin_of(l);
                    atomicAdd(&sh.count[b], 1u);
                    add_mass(b, weight(l));
                }
            });
            merge(true);
            u64 whole = 0;
            for (uint32_t r = 0; r < n_ctas; ++r) whole += sh.share_mass[r];
            if (surplus) whole -= surplus * weight(from);
            target = border_target(whole);
            above_mass = 0;
            above_count = 0;
            cross(true, target);
            const int b = bin;
            narrow(true, target, [&](float l) { return l >= from && l > -INFINITY && bin_of(l) == b; });
        }
        const u64 w = weight(value_of_key(border_key));
        ties = (target - above_mass + w - 1) / w;
        cut = true;
    }

    // ---- draw: masses of the warps' runs, then the run that holds the border, then the element
    const float border_value = cut ? value_of_key(border_key) : -INFINITY;
    const u64 least = min_p > 0.0f ? max(1ull, (u64)ceil((double)fminf(min_p, 1.0f) * (double)unit)) : 0;
    const u64 border_w = cut ? weight(border_value) : 0;
    const bool equals_count = cut && border_w >= least;
    auto kept_above = [&](float l) -> u64 {                          // the weight of an element above the border, if min-p keeps it
        const u64 w = weight(l);
        return w >= least ? w : 0;
    };
    u64 mass = 0;
    uint32_t equals = 0;
    if (window_top < INFINITY && equals_count) {                     // what lies above the window is summed already, and min-p keeps it
        mass = lane == 0 ? run_above : 0;
        for_each_piece([&](const float (&l)[VEC]) {
            bool any = false;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                any = any || (l[j] > border_value && distance(l[j]) >= window_top);
                equals += l[j] == border_value ? 1u : 0u;
            }
            if (any) {
                u64 w[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[j] = weight(l[j]);
#pragma unroll
                for (int j = 0; j < VEC; ++j) mass += l[j] > border_value && distance(l[j]) >= window_top ? w[j] : 0;
            }
        });
    } else if (some) {
        const float from = fmaxf(border_value, floor_l);
        for_each_piece([&](const float (&l)[VEC]) {
            bool any = false;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                any = any || l[j] >= from;
                equals += equals_count && l[j] == border_value ? 1u : 0u;
            }
            if (any) {
                u64 w[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[j] = kept_above(l[j]);
#pragma unroll
                for (int j = 0; j < VEC; ++j) mass += l[j] >= from && l[j] > border_value ? w[j] : 0;
            }
        });
    }
    mass = warp_sum(mass);
    equals = __reduce_add_sync(0xffffffffu, equals);
    if (lane == 0) {
        sh.warp_mass[warp] = mass;
        sh.warp_count[warp] = equals;
    }
    __syncthreads();
    u64 run_mass = 0, run_count = 0;                                 // lane i of warp 0: of warp i's run
    if (warp == 0) {
        run_mass = lane < p.n_warps ? sh.warp_mass[lane] : 0;
        run_count = lane < p.n_warps ? sh.warp_count[lane] : 0;
        const u64 a = warp_sum(run_mass), b = warp_sum(run_count);
        give_all(sh.cta_mass, a, 0, rank, n_ctas, lane);
        give_all(sh.cta_count, (uint32_t)b, 0, rank, n_ctas, lane);
    }
    sync_row();                                                      // nothing of another CTA is touched behind this: the others may leave
    auto share_of = [&](float l, double per_whole) {                 // weight / kept mass
        const double d = l == m ? 0.0 : (double)l - m_wide;
        return m_inf && l != m ? 0.0f : (float)(exp2_scaled(fmax(d * slope, -1000.0), 1.0, 0) * per_whole);
    };
    u64 total = 0, before0 = 0, seen0 = 0, left = 0, ties_left = 0;
    int found_run = -1;
    if (warp == 0) {
        // the CTAs' sums, with as many equals as still count
        const u64 c_m = lane < (int)n_ctas ? sh.cta_mass[lane] : 0;
        const u64 c_c = lane < (int)n_ctas ? sh.cta_count[lane] : 0;
        const u64 cta_seen = warp_scan(c_c, lane) - c_c;
        const u64 c_v = c_m + (cta_seen < ties ? min(c_c, ties - cta_seen) : 0) * border_w;
        const u64 c_incl = warp_scan(c_v, lane);
        total = __shfl_sync(0xffffffffu, c_incl, 31);
        seen0 = __shfl_sync(0xffffffffu, cta_seen, (int)rank);
        before0 = __shfl_sync(0xffffffffu, c_incl - c_v, (int)rank);
        // this CTA's runs
        const u64 seen = seen0 + warp_scan(run_count, lane) - run_count;
        const u64 ties_run = seen < ties ? min(run_count, ties - seen) : 0;
        const u64 v = run_mass + ties_run * border_w;
        const u64 before = before0 + warp_scan(v, lane) - v;
        if (lane < p.n_warps) sh.ties_kept[lane] = ties_run;
        if (lane == 0) sh.found_whole = total;
        if (total == 0) {                                            // no candidate
            if (rank == 0 && lane == 0) {
                p.a.token[row] = -1;
                if (p.a.prob) p.a.prob[row] = 0.0f;
            }
        } else {
            const float u = u_row > 0.0f ? fminf(u_row, 0.99999994f) : 0.0f;     // (a NaN counts as 0)
            const u64 target = min((u64)((double)u * (double)total), total - 1);
            const unsigned owner = __ballot_sync(0xffffffffu, target >= before && target < before + v);
            if (owner) {                                             // one run of the cluster
                found_run = __ffs(owner) - 1;
                left = target - __shfl_sync(0xffffffffu, before, found_run);
                ties_left = __shfl_sync(0xffffffffu, ties_run, found_run);
            }
        }
        if (lane == 0) sh.found_bin = found_run;
    }
    __syncthreads();
    const int drawn_run = sh.found_bin;
    if (drawn_run >= 0) {                                            // this CTA holds the token: the run's steps by all warps
        const int run0 = drawn_run * p.run, steps = p.run / (32 * VEC);
        auto elements = [&](int step, float (&l)[VEC]) {
            Piece q;
            q.v = *reinterpret_cast<const uint4*>(held + run0 + (step * 32 + lane) * VEC);
#pragma unroll
            for (int j = 0; j < VEC; ++j) l[j] = widen(q.e[j]);
        };
        for (int step = warp; step < steps; step += p.n_warps) {
            float l[VEC];
            elements(step, l);
            u64 w[VEC], sum = 0;
            uint32_t eq = 0;
#pragma unroll
            for (int j = 0; j < VEC; ++j) w[j] = kept_above(l[j]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                sum += l[j] > border_value ? w[j] : 0;
                eq += equals_count && l[j] == border_value ? 1u : 0u;
            }
            sum = warp_sum(sum);
            eq = __reduce_add_sync(0xffffffffu, eq);
            if (lane == 0) {
                sh.step_mass[step] = sum;
                sh.step_count[step] = eq;
            }
        }
        __syncthreads();
        if (warp == 0) {
            const u64 s_m = lane < steps ? sh.step_mass[lane] : 0, s_c = lane < steps ? sh.step_count[lane] : 0;
            const u64 s_seen = warp_scan(s_c, lane) - s_c;
            const u64 s_ties = s_seen < ties_left ? min(s_c, ties_left - s_seen) : 0;
            const u64 s_v = s_m + s_ties * border_w, s_incl = warp_scan(s_v, lane);
            const unsigned in = __ballot_sync(0xffffffffu, left < s_incl);
            const int step = in ? __ffs(in) - 1 : 0;
            float l[VEC];
            elements(step, l);
            const int at = draw_element<VEC>(l, left - __shfl_sync(0xffffffffu, s_incl - s_v, step), __shfl_sync(0xffffffffu, s_ties, step), border_value,
                                             equals_count, border_w, lane, kept_above);
            if (at >= 0) {
                const int index = run0 + (step * 32 + lane) * VEC + at;
                p.a.token[row] = cta0 + index - shift;
                if (p.a.prob) p.a.prob[row] = share_of(widen(held[index]), (double)unit / (double)total);
            }
        }
    }
    if (p.a.probs) {                                                 // the whole filtered distribution
        __syncthreads();
        float* const out = p.a.probs + (long long)row * p.ld_probs;
        ties_left = sh.ties_kept[warp];
        const double whole = (double)sh.found_whole, per_whole = (double)unit / whole;
        for (int i = lane; i < p.run; i += 32) {
            const int at = cta0 + warp0 + i - shift;
            const float l = widen(held[warp0 + i]);
            const bool eq = equals_count && l == border_value;
            const unsigned eqs = __ballot_sync(0xffffffffu, eq);
            const bool keep = l > border_value ? (least == 0 || weight(l) >= least) : eq && (u64)__popc(eqs & ((1u << lane) - 1u)) < ties_left;
            if (at >= 0 && at < p.vocab) out[at] = keep && whole > 0.0 ? share_of(l, per_whole) : 0.0f;
            const u64 n = (u64)__popc(eqs);
            ties_left = ties_left > n ? ties_left - n : 0;
        }
    }
}

// ---- BF16 rows: by values (long ones of which top-p, or very long ones of which top-k, may cut something)
//
// BF16 logits have few values: below a largest logit of 10, 1568 down to 2^-9.  A bin per value makes counts enough: its mass is
// the count times one weight, so weights are evaluated once per value and not once per element (the row's passes were bound by
// that evaluation, some 75 instructions), the bin that a border crosses is the border, and a CTA's kept mass follows from its own
// counts.  Only the CTA whose part of the row holds the drawn token looks at its elements again.
// The bins count values down from the largest logit by their bits.  What lies within 2^-9 of zero shares one bin, and so does what
// is more than 4094 values below the largest: in these two, weights are summed element by element, and a border that falls there
// is found by halving the range of keys.
constexpr int kValues = 4096;
constexpr int kNearZero = 0x3b00;        // the bits of 2^-9
constexpr int kLongByCount = 32768;      // logits of a row from which on top-k alone goes by values (launch_sample)

struct SharedValues {
    RowGiven row;
    float warp_max[kMaxWarps];
    float max;                       // of this CTA
    uint32_t special[2][3];          // planes of the masses of the two shared bins, of this CTA
    u64 share_mass[kMaxCtas];        // of every CTA
    uint32_t share_count[kMaxCtas];
    u64 scan_mass[kMaxWarps];
    uint32_t scan_count[kMaxWarps];
    u64 warp_mass[kMaxWarps];
    uint32_t warp_count[kMaxWarps];
    u64 cta_mass[kMaxCtas];          // of every CTA
    uint32_t cta_count[kMaxCtas];
    uint32_t key_min, key_max;       // of this CTA
    u64 half_mass;                   // of this CTA, while a range is halved
    uint32_t half_count;
    uint32_t never;
    u64 found_mass, found_whole;
    uint32_t found_count, found_equal;
    int found_bin;
    u64 ties_kept[kMaxWarps];
    u64 step_mass[kMaxWarps][kMaxSteps];     // of 256 elements each of a run
    uint32_t step_count[kMaxWarps][kMaxSteps];
};

__global__ void __launch_bounds__(32 * kMaxWarps, 2)
sample_values_kernel(SampleParams p)
{
    typedef __nv_bfloat16 T;
    constexpr int VEC = 8;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    __shared__ SharedValues sh;

    const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31, n_threads = blockDim.x;
    const uint32_t rank = ptx::cluster_ctarank();
    uint32_t n_ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ctas));
    const int row = blockIdx.x / n_ctas;
    const int share = kValues / (int)n_ctas;                         // bins that this CTA sums over the cluster
    // the row's part, its counts, and running sums through this CTA's share of the bins
    uint32_t* const held = reinterpret_cast<uint32_t*>(smem_raw);    // two logits each
    uint32_t* const count = reinterpret_cast<uint32_t*>(smem_raw + (size_t)p.run * p.n_warps * 2);
    u64* const run_mass = reinterpret_cast<u64*>(count + kValues);
    uint32_t* const run_count = reinterpret_cast<uint32_t*>(run_mass + share);
    auto sync_row = [&]() {
        __syncwarp();                                                // (the cluster's barrier takes whole warps)
        if (n_ctas > 1) ptx::cluster_sync_all();
        else __syncthreads();
    };

    ptx::grid_launch_dependents();
    for (int i = threadIdx.x; i < kValues / 4; i += n_threads) reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x < 6) sh.special[threadIdx.x / 3][threadIdx.x % 3] = 0;
    ptx::grid_dependency_wait();

    // ---- load (positions and runs as above)
    const int warp0 = warp * p.run, cta0 = (int)rank * p.run * p.n_warps;
    const T* const row_ptr = static_cast<const T*>(p.a.logits) + (long long)row * p.ld;
    const int shift = (int)((reinterpret_cast<uintptr_t>(row_ptr) & 15u) / sizeof(T));
    float top = -INFINITY;
    {
        const unsigned short* const base = reinterpret_cast<const unsigned short*>(row_ptr) - shift;
        const int first = shift, last = shift + p.vocab;
        auto keep = [&](int i, const uint4& q) {
            *reinterpret_cast<uint4*>(held + ((warp0 + i) >> 1)) = q;
            const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(__uint_as_float(u[j] << 16), __uint_as_float(u[j] & 0xffff0000u)));
        };
        int i = lane * VEC;
        if (cta0 + warp0 >= first && cta0 + warp0 + p.run <= last)
            for (; i + 96 * VEC < p.run; i += 128 * VEC) {
                uint4 q[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) q[j] = __ldg(reinterpret_cast<const uint4*>(base + cta0 + warp0 + i + j * 32 * VEC));
#pragma unroll
                for (int j = 0; j < 4; ++j) keep(i + j * 32 * VEC, q[j]);
            }
        for (; i < p.run; i += 32 * VEC) {
            const int at = cta0 + warp0 + i;
            uint4 q;
            if (at >= first && at + VEC <= last) {
                q = __ldg(reinterpret_cast<const uint4*>(base + at));
            } else {
                uint32_t u[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t a = at + 2 * j >= first && at + 2 * j < last ? base[at + 2 * j] : 0xff80u;
                    const uint32_t b = at + 2 * j + 1 >= first && at + 2 * j + 1 < last ? base[at + 2 * j + 1] : 0xff80u;
                    u[j] = a | (b << 16);
                }
                q = make_uint4(u[0], u[1], u[2], u[3]);
            }
            keep(i, q);
        }
    }
    if (threadIdx.x == 0 && rank == 0) sh.row.load(p.a, row);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) sh.warp_max[warp] = top;
    __syncthreads();
    if (warp == 0) {
        top = lane < p.n_warps ? sh.warp_max[lane] : -INFINITY;
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) sh.max = top;
    }
    sync_row();
    float m = -INFINITY;
    {
        uint32_t tops[kMaxCtas];
        ld_all(reinterpret_cast<const uint32_t*>(&sh.max), n_ctas, tops);
#pragma unroll
        for (uint32_t r = 0; r < kMaxCtas; ++r)
            if (r < n_ctas) m = fmaxf(m, __uint_as_float(tops[r]));
    }
    m += 0.0f;                                                       // (one zero)
    const float temperature = ld_cluster_float(&sh.row.temperature), top_p = ld_cluster_float(&sh.row.top_p), min_p = ld_cluster_float(&sh.row.min_p);
    const int top_k = (int)ld_cluster(reinterpret_cast<const uint32_t*>(&sh.row.top_k), 0);
    const float u_row = ld_cluster_float(&sh.row.u);
    landed(temperature, top_p, min_p, u_row, top_k, &sh.never);
    const bool one = !(temperature > 0.0f) || top_k == 1;            // the first largest alone
    const bool by_count = !one && top_k > 0 && top_k < p.vocab, by_mass = !one && top_p < 1.0f;
    const bool some = m > -INFINITY;

    // ---- weights, as above
    const bool m_inf = m == INFINITY;
    const double slope = one ? 0.0 : 1.4426950408889634074 / (double)temperature;         // log2(e) / T
    const float floor_l = m_inf || one ? m : m - (float)(p.scale_log2 + 3) * 0.6931472f * temperature;
    const double m_wide = (double)m;
    const u64 unit = 1ull << p.scale_log2;
    auto weight = [&](float l) -> u64 {
        const double d = l == m ? 0.0 : __dsub_rn((double)fmaxf(l, floor_l), m_wide);
        const u64 w = exp2_units(d, slope, p.scale_log2);
        return l < floor_l ? 0 : w;
    };
    auto key = [&](float l) { return key_of(l + 0.0f); };

    // ---- bins: rank_of counts values up from -largest through the shared one at 0
    auto rank_of = [](float l) {
        const int bits = (int)(__float_as_uint(l) >> 16), a = max((bits & 0x7fff) - kNearZero, 0);
        return bits & 0x8000 ? -a : a;
    };
    const int rank_m = rank_of(m), zero_bin = min(rank_m, kValues - 1);
    // (a largest logit below the shared values has no bin for them; its own rank is negative then)
    auto bin_of = [&](float l) { return min(rank_m - rank_of(l), kValues - 1); };
    auto is_shared = [&](int b) { return b == zero_bin || b == kValues - 1; };
    auto value_of_bin = [&](int b) {                                 // of a bin that holds one value
        const int r = rank_m - b;
        return __uint_as_float((uint32_t)(r > 0 ? r + kNearZero : 0x8000 | (kNearZero - r)) << 16);
    };
    auto for_each = [&](auto&& f) {
        for (int i = lane * VEC; i < p.run; i += 32 * VEC) {
            const uint4 q = *reinterpret_cast<const uint4*>(held + ((warp0 + i) >> 1));
            const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f(__uint_as_float(u[j] << 16));
                f(__uint_as_float(u[j] & 0xffff0000u));
            }
        }
    };
    if (some)
        for_each([&](float l) {
            if (l > -INFINITY) {
                const int b = bin_of(l);
                atomicAdd(&count[b], 1u);
                if (is_shared(b) && l >= floor_l) {                  // rare
                    const u64 w = weight(l);
                    const int s = b == kValues - 1 ? 1 : 0;
                    atomicAdd(&sh.special[s][0], (uint32_t)w & 0x7fffu);
                    atomicAdd(&sh.special[s][1], (uint32_t)(w >> 15) & 0x7fffu);
                    atomicAdd(&sh.special[s][2], (uint32_t)(w >> 30));
                }
            }
        });
    auto special_mass = [&](int b, uint32_t r) {
        const uint32_t* const s = sh.special[b == kValues - 1 ? 1 : 0];
        return (u64)ld_cluster(s, r) + ((u64)ld_cluster(s + 1, r) << 15) + ((u64)ld_cluster(s + 2, r) << 30);
    };

    u64 above_mass = 0;
    uint32_t above_count = 0, bin_count = 0;
    int bin = -1;
    auto merge = [&](bool masses) {
        sync_row();
        const int b0 = (int)rank * share, per = (share + n_threads - 1) / n_threads;
        u64 sum_m = 0;
        uint32_t sum_c = 0;
        for (int j = 0; j < per; ++j) {
            const int at = threadIdx.x * per + j, b = b0 + at;
            if (at < share) {
                uint32_t c = 0;
                c = n_ctas == 1 ? count[b] : sum_all(&count[b], n_ctas);
                if (masses && c) {
                    if (is_shared(b)) {
                        for (uint32_t r = 0; r < n_ctas; ++r) sum_m += special_mass(b, r);
                    } else {
                        sum_m += c * weight(value_of_bin(b));
                    }
                }
                sum_c += c;
                run_mass[at] = sum_m;                                // (running within this thread; the rest is added below)
                run_count[at] = sum_c;
            }
        }
        const u64 scan_m = masses ? warp_scan(sum_m, lane) : 0;
        const uint32_t scan_c = warp_scan(sum_c, lane);
        if (lane == 31) {
            sh.scan_mass[warp] = scan_m;
            sh.scan_count[warp] = scan_c;
        }
        __syncthreads();
        u64 base_m = scan_m - sum_m;
        uint32_t base_c = scan_c - sum_c;
        for (int i = 0; i < warp; ++i) {
            base_m += sh.scan_mass[i];
            base_c += sh.scan_count[i];
        }
        for (int j = 0; j < per; ++j) {
            const int at = threadIdx.x * per + j;
            if (at < share) {
                run_mass[at] += base_m;
                run_count[at] += base_c;
            }
        }
        if (warp == p.n_warps - 1) {                                 // this share's sums, to all
            give_all(sh.share_mass, base_m + sum_m, 31, rank, n_ctas, lane);
            give_all(sh.share_count, base_c + sum_c, 31, rank, n_ctas, lane);
        }
        sync_row();
    };
    // The first bin at which the running count (or mass) reaches `target`: found by one warp of each CTA, told to all.
    auto cross = [&](bool use_mass, u64 target) {
        if (warp == 0) {
            // the CTA whose share holds the target
            const u64 s_m = lane < (int)n_ctas ? sh.share_mass[lane] : 0;
            const uint32_t s_c = lane < (int)n_ctas ? sh.share_count[lane] : 0;
            const u64 i_m = warp_scan(s_m, lane);
            const uint32_t i_c = warp_scan(s_c, lane);
            const unsigned in = __ballot_sync(0xffffffffu, use_mass ? i_m >= target : (u64)i_c >= target);
            const int r_lane = in ? __ffs(in) - 1 : 31;
            u64 base_m = __shfl_sync(0xffffffffu, in ? i_m - s_m : i_m, r_lane);
            uint32_t base_c = __shfl_sync(0xffffffffu, in ? i_c - s_c : i_c, r_lane), here = 0;
            int found = -1;
            if (in) {
                const uint32_t r = (uint32_t)r_lane;
                // 32 places through the share, then the bins between two of them
                const int step = share >> 5;
                int lo = 0;
                for (int wide = step; found < 0; wide = 1) {
                    const int at = wide > 1 ? (lane + 1) * wide - 1 : lo + lane;
                    const u64 rm = at < share ? ld_cluster(&run_mass[at], r) : 0;
                    const uint32_t rc = at < share ? ld_cluster(&run_count[at], r) : 0;
                    const unsigned hit = __ballot_sync(0xffffffffu, at < share && (use_mass ? base_m + rm >= target : (u64)base_c + rc >= target));
                    const int src = hit ? __ffs(hit) - 1 : 31;
                    if (wide > 1) {
                        lo = src * wide;
                    } else if (hit || lo + 32 >= share) {
                        found = min(lo + src, share - 1);
                    } else {
                        lo += 32;
                    }
                }
                const u64 bm = found ? ld_cluster(&run_mass[found - 1], r) : 0;
                const uint32_t bc = found ? ld_cluster(&run_count[found - 1], r) : 0;
                here = ld_cluster(&run_count[found], r) - bc;
                base_m += bm;
                base_c += bc;
                found += (int)r * share;
            }
            if (lane == 0) {
                sh.found_bin = found;
                sh.found_mass = base_m;
                sh.found_count = base_c;
                sh.found_equal = here;
            }
        }
        __syncthreads();
        bin = sh.found_bin;
        above_mass = sh.found_mass;
        above_count = sh.found_count;
        bin_count = sh.found_equal;
        __syncthreads();
    };
    uint32_t border_key = 0, border_equal = 0;
    // The border in the crossing bin.
    auto narrow = [&](bool use_mass, u64 target) {
        if (!is_shared(bin)) {
            border_key = key(value_of_bin(bin));
            border_equal = bin_count;
            return;
        }
        // by halving the range of its keys: the largest at which the elements from it on reach the target
        const int b = bin;
        uint32_t mn = 0xffffffffu, mx = 0;
        if (threadIdx.x == 0) {
            sh.key_min = mn;
            sh.key_max = mx;
        }
        __syncthreads();
        for_each([&](float l) {
            if (l > -INFINITY && bin_of(l) == b) {
                mn = min(mn, key(l));
                mx = max(mx, key(l));
            }
        });
        mn = __reduce_min_sync(0xffffffffu, mn);
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0) {
            atomicMin(&sh.key_min, mn);
            atomicMax(&sh.key_max, mx);
        }
        sync_row();
        uint32_t lo = 0xffffffffu, hi = 0;
        for (uint32_t r = 0; r < n_ctas; ++r) {
            lo = min(lo, ld_cluster(&sh.key_min, r));
            hi = max(hi, ld_cluster(&sh.key_max, r));
        }
        // mass and number of the bin's elements with a key of at least k
        u64 mass_k = 0;
        uint32_t count_k = 0;
        auto from_key = [&](uint32_t k) {
            u64 s = 0;
            uint32_t c = 0;
            for_each([&](float l) {
                if (l > -INFINITY && bin_of(l) == b && key(l) >= k) {
                    ++c;
                    if (use_mass) s += weight(l);
                }
            });
            s = warp_sum(s);
            c = __reduce_add_sync(0xffffffffu, c);
            if (lane == 0) {
                sh.warp_mass[warp] = s;
                sh.warp_count[warp] = c;
            }
            __syncthreads();
            if (warp == 0) {
                const u64 a = warp_sum(lane < p.n_warps ? sh.warp_mass[lane] : 0);
                const uint32_t n = __reduce_add_sync(0xffffffffu, lane < p.n_warps ? sh.warp_count[lane] : 0u);
                if (lane == 0) {
                    sh.half_mass = a;
                    sh.half_count = n;
                }
            }
            sync_row();
            mass_k = 0;
            count_k = 0;
            for (uint32_t r = 0; r < n_ctas; ++r) {
                mass_k += ld_cluster(&sh.half_mass, r);
                count_k += ld_cluster(&sh.half_count, r);
            }
            landed(mass_k + count_k, &sh.never);
            sync_row();
        };
        for (int step = 0; step < 32 && lo < hi; ++step) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            from_key(mid);
            if (use_mass ? above_mass + mass_k >= target : (u64)above_count + count_k >= target) lo = mid;
            else hi = mid - 1;
        }
        from_key(lo);
        const uint32_t with = count_k;
        from_key(lo + 1);                                            // (a key is never the last integer: that would be a NaN)
        above_mass += mass_k;
        above_count += count_k;
        border_equal = with - count_k;
        border_key = lo;
    };

    // ---- the border: everything above its value is kept, and the first `ties` equal to it
    bool cut = some && one;
    u64 ties = 1;
    if (cut) border_key = key(m);
    if (some && (by_count || by_mass)) {
        merge(by_mass);
        if (by_count) {
            cross(false, (u64)top_k);
            if (bin >= 0) {                                          // else fewer candidates than k: all are kept
                narrow(false, (u64)top_k);
                ties = (u64)top_k - above_count;
                cut = true;
            }
        }
        if (by_mass) {
            u64 whole = 0;
            if (cut && !is_shared(bin)) {
                whole = above_mass + ties * weight(value_of_key(border_key));
            } else if (cut) {                                        // the masses above a border in a shared bin were not summed
                const float from = value_of_key(border_key);
                u64 s = 0;
                for_each([&](float l) {
                    if (l > from) s += weight(l);
                });
                s = warp_sum(s);
                if (lane == 0) sh.warp_mass[warp] = s;
                __syncthreads();
                if (warp == 0) {
                    const u64 a = warp_sum(lane < p.n_warps ? sh.warp_mass[lane] : 0);
                    if (lane == 0) sh.half_mass = a;
                }
                sync_row();
                for (uint32_t r = 0; r < n_ctas; ++r) whole += ld_cluster(&sh.half_mass, r);
                landed(whole, &sh.never);
                sync_row();
                whole += ties * weight(from);
            } else {
                for (uint32_t r = 0; r < n_ctas; ++r) whole += sh.share_mass[r];
            }
            // kept while the mass before < p * whole: up to where the running mass reaches ceil(p * whole)
            const u64 target = max(1ull, min((u64)ceil((double)fmaxf(top_p, 0.0f) * (double)whole), whole));
            cross(true, target);
            narrow(true, target);
            const u64 w = weight(value_of_key(border_key));
            ties = (target - above_mass + w - 1) / w;
            cut = true;
        }
    } else {
        __syncthreads();                                             // (the counts are read below)
    }

    // ---- draw: what each CTA keeps, by its counts; then, in the CTA that holds the token, its runs and elements
    const float border_value = cut ? value_of_key(border_key) : -INFINITY;
    const u64 least = min_p > 0.0f ? max(1ull, (u64)ceil((double)fminf(min_p, 1.0f) * (double)unit)) : 0;
    const u64 border_w = cut ? weight(border_value) : 0;
    const bool equals_count = cut && border_w >= least;
    const float from = fmaxf(border_value, floor_l);                 // nothing below weighs anything
    auto kept_above = [&](float l) -> u64 {
        const u64 w = weight(l);
        return w >= least ? w : 0;
    };
    u64 mass = 0;
    uint32_t equals = 0;
    if (some) {
        const int last = cut ? bin_of(border_value) : kValues - 1;   // the border's bin
        for (int b = threadIdx.x; b <= last; b += n_threads) {
            const uint32_t c = count[b];
            if (!c) continue;
            if (!is_shared(b)) {
                const float l = value_of_bin(b);
                if (l > border_value) {
                    if (l >= from) mass += c * kept_above(l);
                } else if (equals_count && l == border_value) {
                    equals += c;
                }
            } else if (least == 0 && b != last) {                    // all of a shared bin
                mass += special_mass(b, rank);
            }
        }
        // a shared bin of which the border or min-p may keep a part: by elements
        const bool parts = (count[zero_bin < 0 ? kValues - 1 : zero_bin] && zero_bin >= 0 && zero_bin <= last && (least > 0 || zero_bin == last)) ||
                           (last == kValues - 1 && count[kValues - 1]);
        if (parts)
            for_each([&](float l) {
                if (l > -INFINITY) {
                    const int b = bin_of(l);
                    if (is_shared(b) && (least > 0 || b == last)) {
                        if (l > border_value) {
                            if (l >= from) mass += kept_above(l);
                        } else if (equals_count && l == border_value) {
                            ++equals;
                        }
                    }
                }
            });
    }
    mass = warp_sum(mass);
    equals = __reduce_add_sync(0xffffffffu, equals);
    if (lane == 0) {
        sh.warp_mass[warp] = mass;
        sh.warp_count[warp] = equals;
    }
    __syncthreads();
    if (warp == 0) {
        const u64 a = warp_sum(lane < p.n_warps ? sh.warp_mass[lane] : 0);
        const uint32_t n = __reduce_add_sync(0xffffffffu, lane < p.n_warps ? sh.warp_count[lane] : 0u);
        give_all(sh.cta_mass, a, 0, rank, n_ctas, lane);
        give_all(sh.cta_count, n, 0, rank, n_ctas, lane);
    }
    sync_row();                                                      // nothing of another CTA is touched behind this: the others may leave
    // every warp: the CTAs' sums, with as many equals as still count
    const u64 c_m = lane < (int)n_ctas ? sh.cta_mass[lane] : 0;
    const u64 c_c = lane < (int)n_ctas ? sh.cta_count[lane] : 0;
    const u64 c_seen = warp_scan(c_c, lane) - c_c;
    const u64 c_v = c_m + (c_seen < ties ? min(c_c, ties - c_seen) : 0) * border_w;
    const u64 c_incl = warp_scan(c_v, lane);
    const u64 total = __shfl_sync(0xffffffffu, c_incl, 31);
    const u64 seen0 = __shfl_sync(0xffffffffu, c_seen, (int)rank), before0 = __shfl_sync(0xffffffffu, c_incl - c_v, (int)rank), mine = __shfl_sync(0xffffffffu, c_v, (int)rank);
    const double whole_kept = (double)total, per_whole = (double)unit / whole_kept;
    auto share_of = [&](float l) {                                   // weight / kept mass
        const double d = l == m ? 0.0 : (double)l - m_wide;
        return m_inf && l != m ? 0.0f : (float)(exp2_scaled(fmax(d * slope, -1000.0), 1.0, 0) * per_whole);
    };
    u64 target = 0;
    bool holds = false;
    if (total == 0) {                                                // no candidate
        if (rank == 0 && threadIdx.x == 0) {
            p.a.token[row] = -1;
            if (p.a.prob) p.a.prob[row] = 0.0f;
        }
    } else {
        const float u = u_row > 0.0f ? fminf(u_row, 0.99999994f) : 0.0f;         // (a NaN counts as 0)
        target = min((u64)((double)u * whole_kept), total - 1);
        holds = target >= before0 && target < before0 + mine;        // this CTA's part holds the token
    }
    if (holds || p.a.probs) {
        // this CTA's runs, step by step: masses above the border, and equals
        auto elements = [&](int at, float (&l)[VEC]) {
            const uint4 q = *reinterpret_cast<const uint4*>(held + (at >> 1));
            const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < VEC; ++j) l[j] = __uint_as_float(j & 1 ? u[j >> 1] & 0xffff0000u : u[j >> 1] << 16);
        };
        const int steps = p.run / (32 * VEC);
        u64 run_m = 0;
        uint32_t run_c = 0;
        for (int step = 0; step < steps; ++step) {
            float l[VEC];
            elements(warp0 + (step * 32 + lane) * VEC, l);
            bool any = false;
            u64 sum = 0;
            uint32_t eq = 0;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                any = any || (l[j] >= from && l[j] > border_value);
                eq += equals_count && l[j] == border_value ? 1u : 0u;
            }
            if (any) {
                u64 w[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[j] = kept_above(l[j]);
#pragma unroll
                for (int j = 0; j < VEC; ++j) sum += l[j] >= from && l[j] > border_value ? w[j] : 0;
            }
            sum = warp_sum(sum);
            eq = __reduce_add_sync(0xffffffffu, eq);
            run_m += sum;
            run_c += eq;
            if (lane == 0) {
                sh.step_mass[warp][step] = sum;
                sh.step_count[warp][step] = eq;
            }
        }
        if (lane == 0) {
            sh.warp_mass[warp] = run_m;
            sh.warp_count[warp] = run_c;
        }
        __syncthreads();
        if (warp == 0) {
            run_m = lane < p.n_warps ? sh.warp_mass[lane] : 0;
            const u64 rc = lane < p.n_warps ? sh.warp_count[lane] : 0;
            const u64 seen = seen0 + warp_scan(rc, lane) - rc;
            const u64 ties_run = seen < ties ? min(rc, ties - seen) : 0;
            const u64 v = run_m + ties_run * border_w;
            const u64 before = before0 + warp_scan(v, lane) - v;
            if (lane < p.n_warps) sh.ties_kept[lane] = ties_run;
            const unsigned owner = __ballot_sync(0xffffffffu, holds && target >= before && target < before + v);
            if (owner) {                                             // the run, the step in it, the element
                const int src = __ffs(owner) - 1;
                u64 left = target - __shfl_sync(0xffffffffu, before, src), ties_left = __shfl_sync(0xffffffffu, ties_run, src);
                const u64 s_m = lane < steps ? sh.step_mass[src][lane] : 0, s_c = lane < steps ? sh.step_count[src][lane] : 0;
                const u64 s_seen = warp_scan(s_c, lane) - s_c;
                const u64 s_ties = s_seen < ties_left ? min(s_c, ties_left - s_seen) : 0;
                const u64 s_v = s_m + s_ties * border_w, s_incl = warp_scan(s_v, lane);
                const unsigned in = __ballot_sync(0xffffffffu, left < s_incl);
                const int step = in ? __ffs(in) - 1 : 0;
                left -= __shfl_sync(0xffffffffu, s_incl - s_v, step);
                ties_left = __shfl_sync(0xffffffffu, s_ties, step);
                const int at0 = src * p.run + (step * 32 + lane) * VEC;
                float l[VEC];
                elements(at0, l);
                const int at = draw_element<VEC>(l, left, ties_left, border_value, equals_count, border_w, lane, kept_above);
                if (at >= 0) {
                    float drawn = 0.0f;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) drawn = at == j ? l[j] : drawn;
                    p.a.token[row] = cta0 + at0 + at - shift;
                    if (p.a.prob) p.a.prob[row] = share_of(drawn);
                }
            }
        }
    }
    if (p.a.probs) {                                                 // the whole filtered distribution
        __syncthreads();
        float* const out = p.a.probs + (long long)row * p.ld_probs;
        u64 ties_left = sh.ties_kept[warp];
        for (int i = lane; i < p.run; i += 32) {
            const int at = cta0 + warp0 + i - shift;
            const uint32_t pair = held[(warp0 + i) >> 1];
            const float l = __uint_as_float(i & 1 ? pair & 0xffff0000u : pair << 16);
            const bool eq = equals_count && l == border_value;
            const unsigned eqs = __ballot_sync(0xffffffffu, eq);
            const bool keep = l > border_value ? (least == 0 || weight(l) >= least) : eq && (u64)__popc(eqs & ((1u << lane) - 1u)) < ties_left;
            if (at >= 0 && at < p.vocab) out[at] = keep && total ? share_of(l) : 0.0f;
            const u64 n = (u64)__popc(eqs);
            ties_left = ties_left > n ? ties_left - n : 0;
        }
    }
}

template <int TYPE>
cudaError_t run_sample(const SampleShape& s, const SampleTiling& t, const SampleParams& p, cudaStream_t stream)
{
    static unsigned long long done = 0;
    const int bytes = t.run * t.warps * (TYPE == MNN_TYPE_FP32 ? 4 : 2);
    cudaError_t e = allow_smem_once(reinterpret_cast<const void*>(sample_kernel<TYPE>), kMostBytes, &done);
    if (e != cudaSuccess) return e;
    return launch_cluster(t.ctas, sample_kernel<TYPE>, dim3((unsigned)(s.rows * t.ctas)), dim3(32 * t.warps), (size_t)bytes, stream, p);
}

cudaError_t run_values(const SampleShape& s, const SampleTiling& t, const SampleParams& p, cudaStream_t stream)
{
    static unsigned long long done = 0;
    const int bytes = t.run * t.warps * 2 + kValues * 4 + kValues / t.ctas * 12;
    cudaError_t e = allow_smem_once(reinterpret_cast<const void*>(sample_values_kernel), kMostBytes, &done);
    if (e != cudaSuccess) return e;
    return launch_cluster(t.ctas, sample_values_kernel, dim3((unsigned)(s.rows * t.ctas)), dim3(32 * t.warps), (size_t)bytes, stream, p);
}

}  // namespace

SampleTiling sample_tiling(const SampleShape& s, int num_sms)
{
    SampleTiling t;
    const int size = s.type == MNN_TYPE_FP32 ? 4 : 2, vec = 16 / size;
    const long long span = (long long)s.vocab + vec - 1;             // with the positions before an unaligned row
    // CTAs per row: as many as leave each a size at which two are resident per SM, and more while SMs idle and every CTA keeps
    // 4096 elements
    t.ctas = 1;
    while (t.ctas < kMaxCtas) {
        const long long logits = (span + t.ctas - 1) / t.ctas * size;
        const long long sums = s.type == MNN_TYPE_BF16 ? kValues * 4 + kValues * 12 / t.ctas : 33 * 1024;
        const bool idle = (long long)s.rows * t.ctas <= num_sms && span / (2 * t.ctas) >= 4096;
        if (logits + sums <= 100 * 1024 && !idle) break;
        t.ctas *= 2;
    }
    const long long per_cta = (span + t.ctas - 1) / t.ctas;
    t.warps = per_cta > 2048 ? 16 : 8;
    const int step = 32 * vec;
    t.run = (int)((per_cta + (long long)t.warps * step - 1) / ((long long)t.warps * step)) * step;
    int bits = 0;
    while ((1ll << bits) < s.vocab) ++bits;
    t.scale_log2 = 62 - bits < kMaxScale ? 62 - bits : kMaxScale;
    return t;
}

cudaError_t launch_sample(const SampleShape& s, const SampleTiling& t, const SampleArgs& a, cudaStream_t stream)
{
    SampleParams p = {};
    p.rows = s.rows; p.vocab = s.vocab;
    p.run = t.run; p.scale_log2 = t.scale_log2; p.n_warps = t.warps;
    p.ld = s.ld; p.ld_probs = s.ld_probs;
    p.a = a;
    switch (s.type) {
        case MNN_TYPE_FP32: return run_sample<MNN_TYPE_FP32>(s, t, p, stream);
        // By values where top-p is given and rows have more logits than there are bins; with top-k alone, whose counts cost either kernel the
        // same, where rows are long.  us, by values and not.  Top-p 0.9: 512 x 1000 76.6 and 28.0, 1 x 5000 18.0 and 19.8, 512 x 8000 52 and 57, 512 x
        // 32000 96 and 141, 512 x 131072 242 and 484 (with top-k 50 as well 512 x 8000 53 and 39, 512 x 32000 87 and 84, 512 x 131072 211 and 244; what
        // the arrays hold is not known here).  Top-k 50 alone: 512 x 5000 48 and 32, 512 x 16000 58 and 44, 512 x 32000 81 and 78, 1 x 32000 13.6 and
        // 13.9, 512 x 64000 134 and 150, 512 x 131072 198 and 231; top-k 1000 512 x 16000 63 and 51, 512 x 32000 94 and 93, 512 x 64000 156 and 191.
        // Neither, or arrays that cut nothing: 1 x 131072 17.1 and 12.5, 512 x 32000 74 and 53.
        case MNN_TYPE_BF16:
            return (a.top_p && s.vocab > kValues) || (a.top_k && s.vocab > kLongByCount) ? run_values(s, t, p, stream) : run_sample<MNN_TYPE_BF16>(s, t, p, stream);
        default: return run_sample<MNN_TYPE_FP16>(s, t, p, stream);
    }
}

}  // namespace mnnb
