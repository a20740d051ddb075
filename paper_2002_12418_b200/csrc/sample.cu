// Sampling: one token per row of logits l, from a given uniform number u per row.
//     w_i = exp((l_i - max l) / T)
// The candidates in the order of falling logits (ties: lower index first) are cut to a prefix by top-k (the first k), by top-p
// (those before which less than p of the mass of the k lies) and by min-p (w_i >= min_p); the token is the lowest index at which
// the running mass of what is kept, in index order, exceeds u times the whole.
//
// Every decision compares sums of weights with a border, so the sums have to be exact to well below one weight and must not
// depend on the order in which threads add.  A weight is therefore computed in fp64 and held as a 64-bit integer in units of
// 2^-scale (scale = 62 - log2 of the vocabulary, at most 52): sums are exact, in any order, and no atomic changes a result.
//
// A cluster of CTAs holds a row in shared memory (read once from HBM).  No sort: the border of a prefix is one value of l, found
// by a histogram of counts and masses over 1024 bins of m - l (16 octaves of 64 bins, so that the bulk of a row spreads over many
// bins whatever its scale and an outlier or a mask of the type's lowest value costs nothing), then, within the crossing bin, by
// histograms over the range of its keys until one value is left.  Among equal values at the border the first ones by index are
// kept.  The same histogram serves top-k (counts) and top-p (masses).
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

template <int TYPE> struct Logit { typedef float T; static constexpr int kVec = 4; };
template <> struct Logit<MNN_TYPE_BF16> { typedef __nv_bfloat16 T; static constexpr int kVec = 8; };
template <> struct Logit<MNN_TYPE_FP16> { typedef __half T; static constexpr int kVec = 8; };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }

// Two zeros are one value and a NaN is no candidate.
__device__ __forceinline__ float canonical(float v) { return v != v ? -INFINITY : v + 0.0f; }

// An integer that orders as the values do.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __float_as_uint(v);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}

template <typename T>
__device__ __forceinline__ T ld_cluster(const T* mine, uint32_t rank)
{
    const uint32_t a = ptx::map_to_rank(ptx::smem_u32(mine), rank);
    if (sizeof(T) == 8) {
        u64 v;
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
        return (T)v;
    }
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return (T)v;
}

__device__ __forceinline__ u64 warp_sum(u64 v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <typename T>
__device__ __forceinline__ T warp_scan(T v, int lane)       // inclusive
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}

struct Shared {
    u64 mass[kBins];
    uint32_t count[kBins];
    u64 warp_mass[kMaxWarps];        // of this CTA, read by all
    uint32_t warp_count[kMaxWarps];
    float warp_max[kMaxWarps];
    uint32_t key_min, key_max;       // of this CTA
    float max;                       // of this CTA
    // results of a step, for this CTA's threads
    u64 scan_mass[kMaxWarps + 1];
    u64 scan_count[kMaxWarps + 1];
    int bin;
    u64 above_mass, bin_mass;
    uint32_t above_count, bin_count;
};

// The border of a prefix: everything above `key`, and the first `ties` with this key.
struct Border {
    uint32_t key;
    u64 ties;
    u64 mass_above;
    uint32_t count_above;
    bool any;                        // false: no border, everything is kept
};

struct SampleParams {
    int rows, vocab, run, scale_log2, n_warps;
    long long ld, ld_probs;
    SampleArgs a;
};

template <int TYPE>
__global__ void __launch_bounds__(32 * kMaxWarps)
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

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_threads = blockDim.x;
    const uint32_t rank = ptx::cluster_ctarank();
    uint32_t n_ctas;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n_ctas));
    const int row = blockIdx.x / n_ctas;
    const int chunk = p.run * p.n_warps;

    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();

    // ---- load.  Positions count from the 16-byte boundary at or before the row's first element.
    const T* const row_ptr = static_cast<const T*>(p.a.logits) + (long long)row * p.ld;
    const int shift = (int)((reinterpret_cast<uintptr_t>(row_ptr) & 15u) / sizeof(T));
    const T* const base = row_ptr - shift;
    const int first = shift, last = shift + p.vocab;                 // positions [first, last) are the row
    const int cta0 = (int)rank * chunk, warp0 = warp * p.run;        // of this CTA in the row, of this warp in the CTA
    float top = -INFINITY;
#pragma unroll 4
    for (int i = lane * VEC; i < p.run; i += 32 * VEC) {
        const int at = cta0 + warp0 + i;
        Piece q;
        if (at >= first && at + VEC <= last) {
            q.v = __ldg(reinterpret_cast<const uint4*>(base + at));
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) q.e[j] = at + j >= first && at + j < last ? base[at + j] : (T)(-INFINITY);
        }
        *reinterpret_cast<uint4*>(held + warp0 + i) = q.v;
#pragma unroll
        for (int j = 0; j < VEC; ++j) top = fmaxf(top, widen(q.e[j]));           // fmaxf passes a NaN over
    }
    const float temperature = p.a.temperature ? p.a.temperature[row] : 1.0f;
    const int top_k = p.a.top_k ? p.a.top_k[row] : 0;
    const float top_p = p.a.top_p ? p.a.top_p[row] : 1.0f;
    const float min_p = p.a.min_p ? p.a.min_p[row] : 0.0f;
    const bool greedy = !(temperature > 0.0f);
    const bool by_count = greedy || (top_k > 0 && top_k < p.vocab), by_mass = !greedy && top_p < 1.0f;
    const u64 k_target = greedy ? 1 : (u64)top_k;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) sh.warp_max[warp] = top;
    for (int i = threadIdx.x; i < kBins; i += n_threads) {
        sh.mass[i] = 0;
        sh.count[i] = 0;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < p.n_warps; ++i) top = fmaxf(top, sh.warp_max[i]);
        sh.max = top;
    }
    ptx::cluster_sync_all();
    float m = -INFINITY;
    for (uint32_t r = 0; r < n_ctas; ++r) m = fmaxf(m, __uint_as_float(ld_cluster(reinterpret_cast<const uint32_t*>(&sh.max), r)));
    m += 0.0f;                                                       // (one zero)

    // ---- weights
    const double slope = greedy ? 0.0 : 1.4426950408889634074 / (double)temperature;      // log2(e) / T
    const float cut = greedy ? 0.0f : -(float)(p.scale_log2 + 2) * 0.6931472f * temperature;    // below it a weight rounds to 0
    auto exponent = [&](float l) { return ((double)l - (double)m) * slope; };              // log2 of the weight; l < m
    auto weight = [&](float l) -> u64 {
        if (l == m) return 1ull << p.scale_log2;
        if (m == INFINITY || !(l - m >= cut)) return 0;
        return (u64)__double2ull_rn(exp2(exponent(l) + (double)p.scale_log2));
    };
    auto value = [&](T e) { return canonical(widen(e)); };
    auto for_each = [&](auto&& f) {                                  // every element that this warp holds
        for (int i = lane * VEC; i < p.run; i += 32 * VEC) {
            Piece q;
            q.v = *reinterpret_cast<const uint4*>(held + warp0 + i);
#pragma unroll
            for (int j = 0; j < VEC; ++j) f(value(q.e[j]));
        }
    };
    // 16 octaves of 64 bins of m - l, from 2^-10 to 2^6; what is nearer or further goes to the first or last bin
    auto bin_of = [&](float l) {
        const float d = l == m ? 0.0f : m - l;
        return min(max((int)(__float_as_uint(d) >> 17) - ((127 - 10) << 6), 0), kBins - 1);
    };

    // Sums the CTAs' histograms and finds the first bin at which the running count (or mass) reaches `target`, adding to what
    // lies above.  Leaves the histograms zeroed.
    auto crossing = [&](bool use_mass, u64 target, uint32_t count_above, u64 mass_above) {
        ptx::cluster_sync_all();
        constexpr int kPer = kBins / (32 * kMaxWarps);               // bins a thread of a full CTA takes
        u64 bm[kPer * 8];
        uint32_t bc[kPer * 8];
        const int per = kBins / n_threads;                           // 2..8: CTAs have 4 to 16 warps
        u64 sum_m = 0;
        uint32_t sum_c = 0;
#pragma unroll
        for (int j = 0; j < kPer * 8; ++j) {
            if (j >= per) break;
            const int b = threadIdx.x * per + j;
            u64 tm = 0;
            uint32_t tc = 0;
            for (uint32_t r = 0; r < n_ctas; ++r) {
                tm += ld_cluster(&sh.mass[b], r);
                tc += ld_cluster(&sh.count[b], r);
            }
            bm[j] = tm;
            bc[j] = tc;
            sum_m += tm;
            sum_c += tc;
        }
        u64 scan_m = warp_scan(sum_m, lane);
        u64 scan_c = warp_scan((u64)sum_c, lane);
        if (lane == 31) {
            sh.scan_mass[warp + 1] = scan_m;
            sh.scan_count[warp + 1] = scan_c;
        }
        if (threadIdx.x == 0) {
            sh.scan_mass[0] = 0;
            sh.scan_count[0] = 0;
            sh.bin = -1;
        }
        __syncthreads();
        for (int i = 0; i <= warp; ++i) {
            scan_m += sh.scan_mass[i];
            scan_c += sh.scan_count[i];
        }
        u64 run_m = mass_above + scan_m - sum_m;
        u64 run_c = count_above + scan_c - sum_c;
#pragma unroll
        for (int j = 0; j < kPer * 8; ++j) {
            if (j >= per) break;
            const u64 before = use_mass ? run_m : run_c, after = before + (use_mass ? bm[j] : bc[j]);
            if (before < target && after >= target) {
                sh.bin = threadIdx.x * per + j;
                sh.above_mass = run_m;
                sh.above_count = (uint32_t)run_c;
                sh.bin_mass = bm[j];
                sh.bin_count = bc[j];
            }
            run_m += bm[j];
            run_c += bc[j];
        }
        ptx::cluster_sync_all();                                     // (also: all have read this CTA's histograms)
        for (int i = threadIdx.x; i < kBins; i += n_threads) {
            sh.mass[i] = 0;
            sh.count[i] = 0;
        }
    };
    // Smallest and largest key of the elements that `in` takes, over the cluster.
    auto key_range = [&](auto&& in, uint32_t* lo, uint32_t* hi) {
        uint32_t mn = 0xffffffffu, mx = 0;
        if (threadIdx.x == 0) {
            sh.key_min = mn;
            sh.key_max = mx;
        }
        __syncthreads();
        for_each([&](float l) {
            if (l > -INFINITY && in(l)) {
                const uint32_t k = key_of(l);
                mn = min(mn, k);
                mx = max(mx, k);
            }
        });
        mn = __reduce_min_sync(0xffffffffu, mn);
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0) {
            atomicMin(&sh.key_min, mn);
            atomicMax(&sh.key_max, mx);
        }
        ptx::cluster_sync_all();
        mn = 0xffffffffu;
        mx = 0;
        for (uint32_t r = 0; r < n_ctas; ++r) {
            mn = min(mn, ld_cluster(&sh.key_min, r));
            mx = max(mx, ld_cluster(&sh.key_max, r));
        }
        ptx::cluster_sync_all();
        *lo = mn;
        *hi = mx;
    };
    auto first_histogram = [&](bool masses) {
        for_each([&](float l) {
            if (!(l > -INFINITY)) return;
            const int b = bin_of(l);
            atomicAdd(&sh.count[b], 1u);
            if (masses) {
                const u64 w = weight(l);
                if (w) atomicAdd(&sh.mass[b], w);
            }
        });
    };
    // The border at which the running count (or mass) reaches `target`; the histogram of the first level is in place.
    auto find_border = [&](bool use_mass, bool masses, u64 target) {
        Border b;
        b.any = true;
        crossing(use_mass, target, 0, 0);
        uint32_t lo, hi;
        int bin = sh.bin;
        if (bin < 0) {                                               // fewer candidates than k: everything is kept
            b.any = false;
            return b;
        }
        key_range([&](float l) { return bin_of(l) == bin; }, &lo, &hi);
        while (lo != hi) {
            const uint32_t span = hi - lo;
            const int sh_bits = max(0, 32 - __clz(span) - 10);       // (hi - key) >> sh_bits < 1024
            for_each([&](float l) {
                const uint32_t k = key_of(l);
                if (l > -INFINITY && k >= lo && k <= hi) {
                    atomicAdd(&sh.count[(hi - k) >> sh_bits], 1u);
                    if (masses) {
                        const u64 w = weight(l);
                        if (w) atomicAdd(&sh.mass[(hi - k) >> sh_bits], w);
                    }
                }
            });
            const uint32_t above_c = sh.above_count;
            const u64 above_m = sh.above_mass;
            crossing(use_mass, target, above_c, above_m);
            bin = sh.bin;
            const uint32_t top_key = hi - ((uint32_t)bin << sh_bits);
            if (sh_bits == 0) {
                lo = hi = top_key;
            } else {
                const uint32_t b_lo = max(lo, top_key - ((1u << sh_bits) - 1u)), b_hi = top_key;
                key_range([&](float l) {
                    const uint32_t k = key_of(l);
                    return k >= b_lo && k <= b_hi;
                }, &lo, &hi);
            }
        }
        b.key = lo;
        b.mass_above = sh.above_mass;
        b.count_above = sh.above_count;
        b.ties = sh.bin_count;                                       // (all of them; the caller cuts)
        return b;
    };
    auto value_of_key = [](uint32_t k) { return __uint_as_float(k >> 31 ? k ^ 0x80000000u : ~k); };

    Border border;
    border.any = false;
    if (m > -INFINITY) {
        u64 whole = 0;                                               // mass of what top-k leaves
        if (by_count || by_mass) {
            __syncthreads();
            first_histogram(by_mass);
        }
        if (by_count) {
            border = find_border(false, by_mass, k_target);
            if (border.any) {
                const u64 ties = k_target - border.count_above;      // 1.. of the border's equals
                border.ties = ties;
                if (by_mass) whole = border.mass_above + ties * weight(value_of_key(border.key));
            }
            if (by_mass) {
                __syncthreads();
                first_histogram(true);                               // again: the search used the bins up
            }
        }
        if (by_mass) {
            if (!border.any) {                                       // the whole row's mass
                u64 sum = 0;
                ptx::cluster_sync_all();
                for (int i = threadIdx.x; i < kBins; i += n_threads)
                    for (uint32_t r = 0; r < n_ctas; ++r) sum += ld_cluster(&sh.mass[i], r);
                sum = warp_sum(sum);
                if (lane == 0) sh.warp_mass[warp] = sum;
                __syncthreads();
                for (int i = 0; i < p.n_warps; ++i) whole += sh.warp_mass[i];
            }
            // kept while the mass before < p * whole: up to where the running mass reaches ceil(p * whole)
            const double want = ceil((double)fmaxf(top_p, 0.0f) * (double)whole);
            const u64 target = max(1ull, min((u64)want, whole));
            border = find_border(true, true, target);
            const u64 w = weight(value_of_key(border.key));
            border.ties = (target - border.mass_above + w - 1) / w;
        }
    }

    // ---- draw: masses of the warps' runs, then the run that holds the border, then the element
    const float border_value = border.any ? value_of_key(border.key) : -INFINITY;
    const u64 least = min_p > 0.0f ? max(1ull, (u64)ceil((double)fminf(min_p, 1.0f) * (double)(1ull << p.scale_log2))) : 0;
    const bool border_counts = border.any && m > -INFINITY && weight(border_value) >= least;
    auto above = [&](float l) { return border.any ? l > border_value : l > -INFINITY; };
    u64 mass = 0;
    uint32_t equals = 0;
    if (m > -INFINITY)
        for_each([&](float l) {
            if (above(l)) {
                const u64 w = weight(l);
                if (w >= least) mass += w;
            }
            equals += border_counts && l == border_value ? 1u : 0u;
        });
    mass = warp_sum(mass);
    equals = __reduce_add_sync(0xffffffffu, equals);
    __syncthreads();                                                 // (warp_mass is read above)
    if (lane == 0) {
        sh.warp_mass[warp] = mass;
        sh.warp_count[warp] = equals;
    }
    ptx::cluster_sync_all();
    // every warp: prefix over the runs before its own, and the whole
    const u64 border_w = border_counts ? weight(border_value) : 0;
    u64 total = 0, before = 0, mine = 0, ties_mine = 0;
    {
        u64 seen = 0;                                                // equals so far
        const int runs = (int)n_ctas * p.n_warps, own = (int)rank * p.n_warps + warp;
        for (int i0 = 0; i0 < runs; i0 += 32) {
            const int i = i0 + lane;
            u64 rm = 0;
            u64 rc = 0;
            if (i < runs) {
                rm = ld_cluster(&sh.warp_mass[i % p.n_warps], i / p.n_warps);
                rc = ld_cluster(&sh.warp_count[i % p.n_warps], i / p.n_warps);
            }
            const u64 c_incl = warp_scan(rc, lane), c_before = seen + c_incl - rc;
            const u64 ties = border_counts && c_before < border.ties ? min(rc, border.ties - c_before) : 0;
            const u64 v = rm + ties * border_w;
            const u64 v_incl = warp_scan(v, lane);
            if (own >= i0 && own < i0 + 32) {
                before = total + __shfl_sync(0xffffffffu, v_incl - v, own - i0);
                mine = __shfl_sync(0xffffffffu, v, own - i0);
                ties_mine = __shfl_sync(0xffffffffu, ties, own - i0);
            }
            total += __shfl_sync(0xffffffffu, v_incl, 31);
            seen += __shfl_sync(0xffffffffu, c_incl, 31);
        }
    }
    const double whole_kept = (double)total;
    auto share = [&](float l) {                                      // weight / kept mass
        const double w = l == m ? 1.0 : m == INFINITY ? 0.0 : exp2(exponent(l));
        return (float)(ldexp(w, p.scale_log2) / whole_kept);
    };
    const float u_row = p.a.u[row];
    const float u = u_row > 0.0f ? fminf(u_row, 0.99999994f) : 0.0f; // (a NaN counts as 0)
    const u64 target = min((u64)((double)u * whole_kept), total - 1);
    if (total == 0) {                                                // no candidate
        if (rank == 0 && threadIdx.x == 0) {
            p.a.token[row] = -1;
            if (p.a.prob) p.a.prob[row] = 0.0f;
        }
    } else if (target >= before && target < before + mine) {         // one warp of the cluster
        u64 left = target - before, ties_left = ties_mine;
        for (int i = lane * VEC; i < p.run; i += 32 * VEC) {
            Piece q;
            q.v = *reinterpret_cast<const uint4*>(held + warp0 + i);
            uint32_t eq = 0;
#pragma unroll
            for (int j = 0; j < VEC; ++j) eq += border_counts && value(q.e[j]) == border_value ? 1u : 0u;
            const uint32_t eq_incl = warp_scan(eq, lane);
            u64 ties_lane = ties_left > eq_incl - eq ? ties_left - (eq_incl - eq) : 0;    // that may still be kept from here on
            u64 wv[VEC], sum = 0;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float l = value(q.e[j]);
                u64 w = 0;
                if (above(l)) {
                    w = weight(l);
                    if (w < least) w = 0;
                } else if (border_counts && l == border_value && ties_lane > 0) {
                    w = border_w;
                    --ties_lane;
                }
                wv[j] = w;
                sum += w;
            }
            const u64 incl = warp_scan(sum, lane);
            const unsigned hit = __ballot_sync(0xffffffffu, incl > left);
            if (hit) {
                if (lane == __ffs(hit) - 1) {
                    u64 rest = left - (incl - sum);
                    bool found = false;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        if (!found && rest < wv[j]) {
                            found = true;
                            p.a.token[row] = cta0 + warp0 + i + j - shift;
                            if (p.a.prob) p.a.prob[row] = share(value(q.e[j]));
                        }
                        rest -= wv[j];
                    }
                }
                break;
            }
            left -= __shfl_sync(0xffffffffu, incl, 31);
            const uint32_t eq_all = __shfl_sync(0xffffffffu, eq_incl, 31);
            ties_left = ties_left > eq_all ? ties_left - eq_all : 0;
        }
    }
    if (p.a.probs) {                                                 // the whole filtered distribution
        float* const out = p.a.probs + (long long)row * p.ld_probs;
        u64 ties_left = ties_mine;
        for (int i = lane; i < p.run; i += 32) {
            const int at = cta0 + warp0 + i - shift;
            const float l = value(held[warp0 + i]);
            const bool eq = border_counts && l == border_value;
            const unsigned eqs = __ballot_sync(0xffffffffu, eq);
            const bool keep = above(l) ? (least == 0 || weight(l) >= least) : eq && (u64)__popc(eqs & ((1u << lane) - 1u)) < ties_left;
            if (at >= 0 && at < p.vocab) out[at] = keep && total ? share(l) : 0.0f;
            const u64 n = (u64)__popc(eqs);
            ties_left = ties_left > n ? ties_left - n : 0;
        }
    }
    ptx::cluster_sync_all();                                         // nobody leaves while its sums are being read
}

template <int TYPE>
cudaError_t run_sample(const SampleShape& s, const SampleTiling& t, const SampleParams& p, cudaStream_t stream)
{
    static unsigned long long done = 0;
    const int bytes = t.run * t.warps * (TYPE == MNN_TYPE_FP32 ? 4 : 2);
    cudaError_t e = allow_smem_once(reinterpret_cast<const void*>(sample_kernel<TYPE>), 208 * 1024, &done);
    if (e != cudaSuccess) return e;
    return launch_cluster(t.ctas, sample_kernel<TYPE>, dim3((unsigned)(s.rows * t.ctas)), dim3(32 * t.warps), (size_t)bytes, stream, p);
}

}  // namespace

SampleTiling sample_tiling(const SampleShape& s, int num_sms)
{
    SampleTiling t;
    const int size = s.type == MNN_TYPE_FP32 ? 4 : 2, vec = 16 / size;
    const int capacity = 200 * 1024 / size;                          // elements a CTA holds
    const long long span = (long long)s.vocab + vec - 1;             // with the positions before an unaligned row
    // CTAs per row: as many as the row needs, and more while that leaves SMs idle and every CTA 4096 elements
    t.ctas = 1;
    while (t.ctas < kMaxCtas && ((span + t.ctas - 1) / t.ctas > capacity ||
                                 ((long long)s.rows * t.ctas * 2 <= 2ll * num_sms && span / (2 * t.ctas) >= 4096)))
        t.ctas *= 2;
    const long long per_cta = (span + t.ctas - 1) / t.ctas;
    t.warps = per_cta > 8192 ? 16 : per_cta > 2048 ? 8 : 4;
    const int step = 32 * vec;
    t.run = (int)((per_cta + (long long)t.warps * step - 1) / ((long long)t.warps * step)) * step;
    int bits = 0;
    while ((1ll << bits) < s.vocab) ++bits;
    t.scale_log2 = 62 - bits < 52 ? 62 - bits : 52;
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
        case MNN_TYPE_BF16: return run_sample<MNN_TYPE_BF16>(s, t, p, stream);
        default: return run_sample<MNN_TYPE_FP16>(s, t, p, stream);
    }
}

}  // namespace mnnb
