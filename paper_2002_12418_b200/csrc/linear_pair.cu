// The matrix product over rows of linear.cu for many rows of 16-bit operands, on PAIRS of SMs: two CTAs of a cluster work on
// 256 features x 256 rows of x per work item with tcgen05.mma.cta_group::2.  Each CTA stages its own 128 rows of w and HALF of
// the x tile (128 of the 256 rows); the tensor cores of both SMs read both halves, and each CTA's tensor memory receives its own
// 128 features x 256 rows.  A CTA therefore pulls 2 x 128 operand rows per block of K where a CTA on its own would pull
// 128 + 256 for the same product: 64 bytes a clock at the tensor core's rate instead of 96, more than L2 delivers to an SM.
//
// fp32 operands come as two FP16 halves each, scaled by rows (linear_relay.cu): hi*hi + lo*hi + hi*lo, the dropped lo*lo is 2^-24 of
// a product.  (Three products of TF32 halves take the tensor core twice as long, and its inputs twice the bytes: 8192 x 4096 x
// 8192 3.23 ms.)  The tensor core's additions cut their result off instead of rounding it, a bias of about 2^-25 per step; so the
// small products of a block go first, and after every two blocks the accumulator is added to fp32 registers, which round.
//
// Barriers as in contract_pair.cu: "operands landed" lives in the first CTA and counts the bytes of both CTAs' copies; "stage
// free" and "accumulator complete" are signalled in both CTAs by one multicast commit; "accumulator drained" lives in the first
// CTA and collects the epilogue warps of both.  No copy is multicast.  All waits are local and bounded; a CTA leaves only after
// a cluster barrier, so that nothing is signalled into shared memory that is gone.
#include "cluster.cuh"
#include "linear_epilogue.cuh"
#include "kernels.h"
#include "umma.cuh"

namespace mnnb {

namespace {

constexpr int kRows = 128;               // rows of w per CTA and stage
constexpr int kPairN = 256;              // columns of tensor memory per accumulator: at most so many rows of x per work item
constexpr int kSegment = 2;              // fp32: blocks of 64 elements of K between additions to the registers
// epilogue warps, two to a quarter of the lanes; four for fp32, whose sums stay in registers (128 to a thread were too many)
template <int TYPE> constexpr int kEpiWarps = TYPE == MNN_TYPE_FP32 ? 16 : 8;
template <int TYPE> constexpr int kThreads = 64 + 32 * kEpiWarps<TYPE>;
constexpr int kMaxStages = 6;
constexpr uint32_t kTileBytes = kRows * 128;
constexpr int kSmem = 200 * 1024;        // one CTA per SM
constexpr int kErrProducer = 61, kErrMmaFull = 62, kErrMmaTmem = 63, kErrEpilogue = 64;   // status codes

struct PairLinearParams {
    int M, N, K, bm, n_fblocks, n_mblocks, k_blocks, stages;         // bm: rows of x per work item, half of them staged by each CTA
    long long items;
    // fp32: for sums that are taken again, and the exponents of the rows' scales
    const float *x, *w;
    long long ldx, ldw;
    const int *x_up, *w_up;
    LinearEpilogue epi;
    int* status;
};

__device__ __forceinline__ void remote_arrive(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// Tiled copy into THIS CTA's shared memory whose bytes are counted on a barrier given by its cluster address.
__device__ __forceinline__ void pair_load_2d(uint32_t dst_smem, const CUtensorMap* map, uint32_t cluster_bar, int c0, int c1)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst_smem), "l"(reinterpret_cast<uint64_t>(map)), "r"(cluster_bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t desc_hi, uint32_t idesc, uint32_t accumulate)
{
    const uint32_t z = 0;
    asm volatile(
        "{\n\t.reg .b64 da, db;\n\t.reg .pred p;\n\t"
        "mov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, {%6, %6, %6, %6, %6, %6, %6, %6}, p;\n\t}" ::"r"(d_tmem), "r"(a_lo),
        "r"(b_lo), "r"(desc_hi), "r"(idesc), "r"(accumulate), "r"(z)
        : "memory");
}
// 2^i for i in [-127, 127]
__device__ __forceinline__ float power_of_two(int i) { return __uint_as_float(i < -126 ? 0x00400000u : (uint32_t)(i + 127) << 23); }
// Arrive on the barrier at this shared-memory offset in both CTAs once the MMAs issued so far have completed.
__device__ __forceinline__ void pair_commit(uint32_t bar)
{
    const unsigned short both = 3;
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(both)
                 : "memory");
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads<TYPE>, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                   const __grid_constant__ CUtensorMap map_x_low, const __grid_constant__ CUtensorMap map_w_low, PairLinearParams p)
{
    constexpr bool F32 = TYPE == MNN_TYPE_FP32;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kMaxStages];
    __shared__ __align__(8) uint64_t empty_bar[kMaxStages];
    __shared__ __align__(8) uint64_t tfull_bar[2];
    __shared__ __align__(8) uint64_t tempty_bar[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, alive;         // alive: counted up while sums are taken again, by both CTAs

    const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_ctarank();
    const long long pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    // stage: [A][B], for fp32 followed by [A low][B low]
    const uint32_t raw_bytes = kTileBytes + (uint32_t)(p.bm >> 1) * 128, stage_bytes = raw_bytes * (F32 ? 2 : 1);
    volatile int* abortp = &abort_flag;
    const volatile int* const alivep = F32 ? &alive : nullptr;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            ptx::mbar_init(ptx::smem_u32(&full_bar[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&empty_bar[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(ptx::smem_u32(&tfull_bar[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&tempty_bar[s]), 2 * kEpiWarps<TYPE>);
        }
        abort_flag = alive = 0;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&map_x);
        ptx::prefetch_tensormap(&map_w);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ptx::smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_sync_all();                  // both CTAs' barriers exist before anything is signalled across
    ptx::tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    auto failed = [&](int code) {             // called by one lane
        if (!*abortp) atomicCAS(p.status, 0, code);
        *abortp = 1;
    };

    if (warp == 0) {
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (long long item = pair; item < p.items && ok; item += n_pairs) {
            int fb, mb;
            linear_item(item, p.n_fblocks, p.n_mblocks, &fb, &mb);
            const int w_row = (fb * 2 + (int)rank) * kRows, x_row = mb * p.bm + (int)rank * (p.bm >> 1);
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                if (!ptx::mbar_wait_warp(ptx::smem_u32(&empty_bar[stage]), phase ^ 1u, abortp, alivep)) {
                    if (lane == 0) failed(kErrProducer);
                    ok = false;
                    break;
                }
                // the first CTA's barrier counts the bytes of both CTAs' copies
                const uint32_t bar = ptx::map_to_rank(ptx::smem_u32(&full_bar[stage]), 0);
                const uint32_t sbase = smem_base + stage * stage_bytes;
                if (ptx::elect_one()) {
                    if (rank == 0) ptx::mbar_expect_tx(ptx::smem_u32(&full_bar[stage]), 2u * stage_bytes);
                    pair_load_2d(sbase, &map_w, bar, kb * 64, w_row);
                    pair_load_2d(sbase + kTileBytes, &map_x, bar, kb * 64, x_row);
                    if (F32) {
                        pair_load_2d(sbase + raw_bytes, &map_w_low, bar, kb * 64, w_row);
                        pair_load_2d(sbase + raw_bytes + kTileBytes, &map_x_low, bar, kb * 64, x_row);
                    }
                }
                if (++stage == (uint32_t)p.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t idesc = ptx::mma_idesc(TYPE == MNN_TYPE_BF16 ? 1 : 0, 2 * kRows, p.bm);
            constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
            const uint32_t a_lo0 = ((smem_base & 0x3FFFFu) >> 4) | (1u << 16);
            uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
            bool ok = true;
            for (long long item = pair; item < p.items && ok; item += n_pairs)
                for (int seg = 0; seg < p.k_blocks && ok; seg += F32 ? kSegment : p.k_blocks) {
                    if (!ptx::mbar_wait_warp(ptx::smem_u32(&tempty_bar[acc]), acc_phase ^ 1u, abortp, alivep)) {
                        if (lane == 0) failed(kErrMmaTmem);
                        ok = false;
                        break;
                    }
                    ptx::tc_fence_after();
                    const uint32_t d_tmem = tmem_base + acc * (uint32_t)kPairN;
                    const int seg_end = F32 ? min(seg + kSegment, p.k_blocks) : p.k_blocks;
                    for (int kb = seg; kb < seg_end; ++kb) {
                        if (!ptx::mbar_wait_warp(ptx::smem_u32(&full_bar[stage]), phase, abortp, alivep)) {
                            if (lane == 0) failed(kErrMmaFull);
                            ok = false;
                            break;
                        }
                        ptx::tc_fence_after();
                        const uint32_t a = a_lo0 + stage * (stage_bytes >> 4), b = a + (kTileBytes >> 4);
                        if (ptx::elect_one()) {
                            const uint32_t go = kb != seg ? 1u : 0u;
                            if (F32) {             // the small products first: the fewer additions to a large sum, the better
#pragma unroll
                                for (int ks = 0; ks < 4; ++ks) {
                                    pair_mma(d_tmem, a + (raw_bytes >> 4) + ks * 2, b + ks * 2, kDescHi, idesc, ks ? 1u : go);
                                    pair_mma(d_tmem, a + ks * 2, b + (raw_bytes >> 4) + ks * 2, kDescHi, idesc, 1u);
                                }
                            }
#pragma unroll
                            for (int ks = 0; ks < 4; ++ks) pair_mma(d_tmem, a + ks * 2, b + ks * 2, kDescHi, idesc, F32 || ks ? 1u : go);
                            pair_commit(ptx::smem_u32(&empty_bar[stage]));         // the stage is free in both CTAs
                        }
                        if (++stage == (uint32_t)p.stages) {
                            stage = 0;
                            phase ^= 1u;
                        }
                    }
                    if (!ok) break;
                    if (ptx::elect_one()) pair_commit(ptx::smem_u32(&tfull_bar[acc]));               // accumulator complete, both CTAs
                    acc ^= 1u;
                    if (acc == 0) acc_phase ^= 1u;
                }
        }
    } else {
        const int q = warp & 3;                       // tensor-memory lane quarter this warp may read
        constexpr int kParts = kEpiWarps<TYPE> / 4;
        const int n_chunks = p.bm >> 4, per_part = (n_chunks + kParts - 1) / kParts;
        const int ch0 = ((warp - 2) >> 2) * per_part, ch1 = min(ch0 + per_part, n_chunks);         // its share of the chunks of 16 rows
        uint32_t acc = 0, acc_phase = 0;
        auto wait_acc = [&]() {
            int got = 1;
            if (lane == 0) got = ptx::mbar_wait_relaxed(ptx::smem_u32(&tfull_bar[acc]), acc_phase, abortp, alivep) ? 1 : 0;
            got = __shfl_sync(0xffffffffu, got, 0);
            if (!got && lane == 0) failed(kErrEpilogue);
            ptx::tc_fence_after();
            return got != 0;
        };
        auto release_acc = [&]() {
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) remote_arrive(ptx::map_to_rank(ptx::smem_u32(&tempty_bar[acc]), 0));
            acc ^= 1u;
            if (acc == 0) acc_phase ^= 1u;
        };
        bool ok = true;
        for (long long item = pair; item < p.items && ok; item += n_pairs) {
            int fb, mb;
            linear_item(item, p.n_fblocks, p.n_mblocks, &fb, &mb);
            const int n = (fb * 2 + (int)rank) * kRows + q * 32 + lane;
            const bool n_ok = n < p.N;
            const long long m_item = (long long)mb * p.bm;
            const float bias = linear_bias<TYPE>(p.epi, n, n_ok);
            LinearStore<TYPE, 16> out;
            auto rows_at = [&](int ch) { return (int)min(16ll, p.M - (m_item + ch * 16)); };
            if (F32) {
                const int w_up = n_ok ? __ldg(p.w_up + n) : 0;
                float sum[4][16];                     // at most 64 of the 256 columns belong to this warp
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c][j] = 0.0f;
                // the residual's lines come into L2 while the product runs (its values would take the sums' registers)
                if (p.epi.res_mode != MNN_RESIDUAL_NONE) {
                    const float* r = static_cast<const float*>(p.epi.residual) + min(n - lane, p.N - 1);
                    for (int j = ch0 * 16 + lane; j < ch1 * 16; j += 32)
                        if (m_item + j < p.M) asm volatile("prefetch.global.L2 [%0];" ::"l"(r + (m_item + j) * p.epi.ldr));
                }
                for (int seg = 0; seg < p.k_blocks; seg += kSegment) {
                    if (!wait_acc()) {
                        ok = false;
                        break;
                    }
                    const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * (uint32_t)kPairN;
#pragma unroll
                    for (int c = 0; c < 4; c += 2)
                        if (ch0 + c < ch1) {          // (an odd last chunk's partner is read too, and not used)
                            uint32_t va[16], vb[16];
                            ptx::tmem_ld16(taddr + (uint32_t)((ch0 + c) * 16), va);
                            ptx::tmem_ld16(taddr + (uint32_t)(min(ch0 + c + 1, n_chunks - 1) * 16), vb);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                sum[c][j] += __uint_as_float(va[j]);
                                sum[c + 1][j] += __uint_as_float(vb[j]);
                            }
                        }
                    release_acc();
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (ch0 + c < ch1) {
                        const long long m0 = m_item + (ch0 + c) * 16;
                        const int rows = rows_at(ch0 + c);
                        // the scales of x's and w's rows undone: in two steps, each within fp32's exponents.  (A lane reads one
                        // row's exponent and the others take it from there.)
                        const int ups = __ldg(p.x_up + min(m0 + (lane & 15), (long long)p.M - 1));
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const int down = -(w_up + __shfl_sync(0xffffffffu, ups, j)), half = down >> 1;
                            sum[c][j] = sum[c][j] * power_of_two(half) * power_of_two(down - half);
                        }
                        if (n_ok) retake_sums<2>(sum[c], rows, m0, n, p.x, p.ldx, p.w, p.ldw, p.K, &alive);
                        // (eight rows of the residual at a time, and after the call: more of them beside the sums went to local
                        // memory.  3136 x 1024 x 1024 with a residual 45 -> 39 us, without one 45 -> 33)
                        LinearStore<TYPE, 8> part;
#pragma unroll
                        for (int h = 0; h < 16; h += 8) {
                            float v[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) v[j] = sum[c][h + j];
                            part.fetch(p.epi, m0 + h, rows - h, n, n_ok);
                            part.store(p.epi, v, bias, m0 + h, rows - h, n, n_ok);
                        }
                    }
            } else {
                out.fetch(p.epi, m_item + ch0 * 16, rows_at(ch0), n, n_ok);
                if (!wait_acc()) {
                    ok = false;
                    break;
                }
                const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * (uint32_t)kPairN;
                uint32_t v[16];
                if (ch0 < ch1) ptx::tmem_ld16(taddr + (uint32_t)(ch0 * 16), v);
                for (int ch = ch0; ch < ch1; ++ch) {
                    ptx::tmem_ld_wait();
                    float s[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) s[j] = __uint_as_float(v[j]);
                    LinearStore<TYPE, 16> now = out;
                    if (ch + 1 < ch1) {
                        ptx::tmem_ld16(taddr + (uint32_t)((ch + 1) * 16), v);
                        out.fetch(p.epi, m_item + (ch + 1) * 16, rows_at(ch + 1), n, n_ok);
                    }
                    now.store(p.epi, s, bias, m_item + ch * 16, rows_at(ch), n, n_ok);
                }
                release_acc();
            }
        }
    }

    // Teardown.  After an aborted run give copies still in flight time to land; nobody leaves before both CTAs are here.
    __syncwarp();
    if (*abortp) __nanosleep(200000);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_sync_all();
    if (warp == 1) {
        __syncwarp();
        ptx::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

template <int TYPE>
cudaError_t run_pair(PairLinearParams& p, int num_sms, const CUtensorMap (&m)[4], cudaStream_t stream)
{
    static unsigned long long done = 0;
    auto kern = linear_pair_kernel<TYPE>;
    cudaError_t e = allow_smem_once(reinterpret_cast<const void*>(kern), kSmem, &done);
    if (e != cudaSuccess) return e;
    const int stage_bytes = (kRows + p.bm / 2) * 128 * (TYPE == MNN_TYPE_FP32 ? 2 : 1);
    p.stages = (kSmem - 1024) / stage_bytes;
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    const long long max_pairs = num_sms / 2, pairs = p.items < max_pairs ? p.items : max_pairs;
    return launch_cluster(2, kern, dim3((unsigned)(2 * pairs)), dim3(kThreads<TYPE>), (size_t)kSmem, stream, m[0], m[1], m[2], m[3], p);
}

}  // namespace

cudaError_t launch_linear_pair(const LinearShape& s, const LinearTiling& t, int num_sms, const void* x, const void* w,
                               const LinearEpilogue& epi, int* status, void* relay, cudaStream_t stream, const char** why)
{
    const bool f32 = s.type == MNN_TYPE_FP32;
    PairLinearParams p = {};
    p.M = s.M; p.N = s.N; p.K = s.K;
    p.bm = t.bm;
    p.n_fblocks = (s.N + 2 * kRows - 1) / (2 * kRows);
    p.n_mblocks = (s.M + t.bm - 1) / t.bm;
    p.k_blocks = (int)(((long long)s.K + 63) / 64);
    p.items = t.items;
    p.x = static_cast<const float*>(x); p.w = static_cast<const float*>(w); p.ldx = s.ldx; p.ldw = s.ldw;
    p.epi = epi;
    p.status = status;
    // what the copies read: the operands themselves or what is laid out of them
    const void *xs = x, *ws = w, *xl = nullptr, *wl = nullptr;
    long long ldx = s.ldx, ldw = s.ldw;
    if (t.relay) {
        char* at = static_cast<char*>(relay);
        const long long x_bytes = (long long)s.M * t.ld_relay * 2, w_bytes = (long long)s.N * t.ld_relay * 2;
        LinearRelayed rx = {x, s.M, s.ldx, at, nullptr, nullptr}, rw = {w, s.N, s.ldw, at + x_bytes, nullptr, nullptr};
        xs = rx.same;
        ws = rw.same;
        ldx = ldw = t.ld_relay;
        if (f32) {
            at += x_bytes + w_bytes;
            xl = rx.low = at;
            wl = rw.low = at + x_bytes;
            at += x_bytes + w_bytes;
            rx.up = reinterpret_cast<int*>(at);
            rw.up = rx.up + s.M;
            p.x_up = rx.up;
            p.w_up = rw.up;
        }
        cudaError_t e = launch_linear_relay(rx, rw, s.K, f32 ? 4 : 2, t.ld_relay, num_sms, stream);
        if (e != cudaSuccess) return e;
    }
    CUtensorMap m[4] = {};
    if (!encode_rows_map(&m[0], xs, 2, s.K, s.M, ldx, t.bm / 2) || !encode_rows_map(&m[1], ws, 2, s.K, s.N, ldw, kRows) ||
        (f32 && (!encode_rows_map(&m[2], xl, 2, s.K, s.M, ldx, t.bm / 2) || !encode_rows_map(&m[3], wl, 2, s.K, s.N, ldw, kRows)))) {
        *why = "cuTensorMapEncodeTiled failed or is unavailable";
        return cudaErrorInvalidValue;
    }
    switch (s.type) {
        case MNN_TYPE_FP32: return run_pair<MNN_TYPE_FP32>(p, num_sms, m, stream);
        case MNN_TYPE_BF16: return run_pair<MNN_TYPE_BF16>(p, num_sms, m, stream);
        default: return run_pair<MNN_TYPE_FP16>(p, num_sms, m, stream);
    }
}

}  // namespace mnnb
