// Matrix product over rows with its epilogue, y = act(x w^T + bias) with a residual, on single SMs:
//     s[m][n] = sum_k x[m][k] w[n][k]
// The same persistent, warp-specialised structure as the contraction of the convolutions (contract_umma.cu), with the roles of
// the two operands turned round: the MMA "M" dimension (128 lanes of tensor memory) is the output feature n, "N" (bm columns, 16
// to 256) the row m of x.  One kernel then serves a single row as well as thousands: with few rows nearly all bytes are weights,
// which stream through the 128-row side at full tile width, and only the columns shrink.  In the epilogue the 32 lanes of a warp
// are 32 consecutive features of one row: stores, residual and bias are contiguous whatever the row strides are.
//
// With few work items a cluster of `split` CTAs shares each item's K loop and adds its partial sums in rank order through
// distributed shared memory (cluster.cuh): deterministic, one launch, no workspace.
//
// 16-bit operands go to the tensor core as they are.  fp32 operands are cut in two: the tensor core reads the high 19 bits
// (TF32, dropping the low 13), and `converter` warps write lo = v - trunc(v) beside each tile, with half a unit added so that dropping ITS low bits
// rounds it; hi*hi goes to one accumulator, lo*hi + hi*lo to another.  What is lost of a product: 2^-22 at most by the rounding of either low half, and lo*lo,
// 2^-22 on average (2^-20 at most).  relL2 with N(0, 1) data 3.5e-7 at K = 96 and 4.2e-7 at 2048 to 8192 (low halves cut off: 5.6e-7 and 6.3e-7, and 4 % faster: 128 x
// 1024 x 32000 77 -> 80 us; fp32 products by a library 1.8e-7 at K = 96 and 7e-7 to 1.1e-6).  The tensor core's own additions cut their
// result off instead of rounding it, which over a long K loop grows to a bias of about 2^-25 per step; so after every kSegment
// blocks of K both accumulators are added to fp32 registers, which round.  Sums that this leaves without a finite value
// (an infinity's low half is no number) are taken again by their thread, term by term in fp32.
//
// Operands whose rows do not start on 16-byte boundaries cannot be copied by TMA: `copier` warps read aligned 16-byte pieces,
// shift neighbours together and write the swizzled tile themselves.
#include "cluster.cuh"
#include "linear_epilogue.cuh"
#include "linear_piece.cuh"
#include "kernels.h"
#include "umma.cuh"

namespace mnnb {

namespace {

constexpr int kTileF = 128;              // features per work item
constexpr int kEpiWarps = 8;
constexpr int kLinearSmem = 200 * 1024;
constexpr int kLinearMaxStages = 10;
constexpr int kSegment = 4;              // fp32: blocks of 32 elements of K between additions to the registers
constexpr int kErrProducer = 51, kErrMmaFull = 52, kErrMmaTmem = 53, kErrEpilogue = 54, kErrAux = 55;   // status codes

struct LinearParams {
    int M, N, K, bm, n_fblocks, n_mblocks, k_blocks, stages, tmem_cols, split;
    long long items;
    const void *x, *w;
    long long ldx, ldw;
    LinearEpilogue epi;
    int* status;
};

template <int TYPE, bool COPY>
struct Roles {
    // copier or converter warps; for fp32 as many as leave the epilogue 128 registers
    static constexpr int kAux = TYPE == MNN_TYPE_FP32 ? 6 : COPY ? 8 : 0;
    static constexpr int kGroups = 3;            // of converter warps: each takes every third block, for the latency of a block
    static constexpr int kThreads = 64 + 32 * (kEpiWarps + kAux);
};

__device__ __forceinline__ void fence_proxy_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// TYPE: MNN_TYPE_*; COPY: operands fetched by copier warps; SPLIT: clusters share K loops; KB: blocks of K (128 bytes a row) per
// stage.
template <int TYPE, bool COPY, bool SPLIT, int KB>
__global__ void __launch_bounds__(Roles<TYPE, COPY>::kThreads, 1)
linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, LinearParams p)
{
    constexpr bool F32 = TYPE == MNN_TYPE_FP32;
    constexpr int kAux = Roles<TYPE, COPY>::kAux;
    constexpr int EB = F32 ? 4 : 2;
    constexpr int kBlockElems = 128 / EB;
    static_assert(KB == 1 || (!F32 && !COPY), "only 16-bit stages copied by TMA hold two blocks");
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kLinearMaxStages];      // operands landed (or written by the copiers)
    __shared__ __align__(8) uint64_t low_bar[kLinearMaxStages];       // fp32 by TMA: low halves written
    __shared__ __align__(8) uint64_t empty_bar[kLinearMaxStages];
    __shared__ __align__(8) uint64_t tfull_bar[2];
    __shared__ __align__(8) uint64_t tempty_bar[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, alive;                                 // alive: counted up while sums are taken again

    const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31;
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t a_bytes = kTileF * 128, b_bytes = (uint32_t)p.bm * 128;
    // stage: [A] x KB [B] x KB, for fp32 followed by [B low][A low]: B and its low half lie together as one operand of 2 bm rows, so
    // that hi*hi and hi*lo are one instruction and A is read twice and not three times.  The loop is bound by shared memory's
    // 128 bytes a clock (64 rows of x: 56 KB read by the tensor core and 72 KB by copies and conversion, per block of K).
    const uint32_t raw_bytes = (a_bytes + b_bytes) * KB, stage_bytes = raw_bytes * (F32 ? 2 : 1), off_b = a_bytes * KB;
    volatile int* abortp = &abort_flag;
    const volatile int* const alivep = F32 ? &alive : nullptr;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            ptx::mbar_init(ptx::smem_u32(&full_bar[s]), COPY ? kAux : 1);
            ptx::mbar_init(ptx::smem_u32(&low_bar[s]), kAux ? kAux / Roles<TYPE, COPY>::kGroups : 1);
            ptx::mbar_init(ptx::smem_u32(&empty_bar[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(ptx::smem_u32(&tfull_bar[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&tempty_bar[s]), kEpiWarps);
        }
        abort_flag = alive = 0;
        ptx::fence_barrier_init();
        if (!COPY) {
            ptx::prefetch_tensormap(&map_x);
            ptx::prefetch_tensormap(&map_w);
        }
    }
    if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_u32(&tmem_slot), (uint32_t)p.tmem_cols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();

    const uint32_t rank = SPLIT ? ptx::cluster_ctarank() : 0u;
    const long long first_item = SPLIT ? blockIdx.x / (unsigned)p.split : blockIdx.x;
    const long long item_step = SPLIT ? gridDim.x / (unsigned)p.split : gridDim.x;
    const int kb0 = SPLIT ? (int)((long long)p.k_blocks * (int)rank / p.split) : 0;
    const int kb1 = SPLIT ? (int)((long long)p.k_blocks * ((int)rank + 1) / p.split) : p.k_blocks;
    auto failed = [&](int code) {                      // called by one lane
        if (!*abortp) atomicCAS(p.status, 0, code);
        *abortp = 1;
    };

    if (warp == 0) {
        if (!COPY) {
            uint32_t stage = 0, phase = 0;
            bool ok = true;
            for (long long item = first_item; item < p.items && ok; item += item_step) {
                int fb, mb;
                linear_item(item, p.n_fblocks, p.n_mblocks, &fb, &mb);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!ptx::mbar_wait_warp(ptx::smem_u32(&empty_bar[stage]), phase ^ 1u, abortp, alivep)) {
                        if (lane == 0) failed(kErrProducer);
                        ok = false;
                        break;
                    }
                    const uint32_t bar = ptx::smem_u32(&full_bar[stage]), sbase = smem_base + stage * stage_bytes;
                    if (ptx::elect_one()) {
                        ptx::mbar_expect_tx(bar, raw_bytes);
#pragma unroll
                        for (int h = 0; h < KB; ++h) {
                            const int ke = (kb * KB + h) * kBlockElems;
                            ptx::tma_load_2d(sbase + h * a_bytes, &map_w, bar, ke, fb * kTileF);
                            ptx::tma_load_2d(sbase + off_b + h * b_bytes, &map_x, bar, ke, mb * p.bm);
                        }
                    }
                    if (++stage == (uint32_t)p.stages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
        }
    } else if (warp == 1) {
        // instruction format: 2 = TF32, 1 = BF16, 0 = FP16
        const uint32_t idesc = ptx::mma_idesc(F32 ? 2 : TYPE == MNN_TYPE_BF16 ? 1 : 0, kTileF, p.bm);
        const uint32_t idesc2 = ptx::mma_idesc(2, kTileF, 2 * p.bm);
        constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);       // 8-row groups 1024 bytes apart, 128-byte swizzle
        uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
        bool ok = true;
        const uint32_t a_lo0 = ((smem_base & 0x3FFFFu) >> 4) | (1u << 16);
        for (long long item = first_item; item < p.items && ok; item += item_step) {
            for (int seg = kb0; seg < kb1 && ok; seg += F32 ? kSegment : kb1 - kb0) {
                if (!ptx::mbar_wait_warp(ptx::smem_u32(&tempty_bar[acc]), acc_phase ^ 1u, abortp, alivep)) {
                    if (lane == 0) failed(kErrMmaTmem);
                    ok = false;
                    break;
                }
                ptx::tc_fence_after();
                const uint32_t d_main = tmem_base + acc * (uint32_t)(p.bm * (F32 ? 2 : 1)), d_cross = d_main + (uint32_t)p.bm;
                const int seg_end = F32 ? min(seg + kSegment, kb1) : kb1;
                uint32_t accumulate = 0;
                for (int kb = seg; kb < seg_end; ++kb) {
                    if (!ptx::mbar_wait_warp(ptx::smem_u32(F32 && !COPY ? &low_bar[stage] : &full_bar[stage]), phase, abortp, alivep)) {
                        if (lane == 0) failed(kErrMmaFull);
                        ok = false;
                        break;
                    }
                    if (COPY || F32) ptx::tc_fence_after();
                    const uint32_t a0 = a_lo0 + stage * (stage_bytes >> 4), b0 = a0 + (off_b >> 4);
                    if (ptx::elect_one()) {
#pragma unroll
                        for (int h = 0; h < KB; ++h)
#pragma unroll
                            for (int ks = 0; ks < 4; ++ks) {
                                const uint32_t a = a0 + h * (a_bytes >> 4) + ks * 2, b = b0 + h * (b_bytes >> 4) + ks * 2;
                                const uint32_t go = h || ks ? 1u : accumulate;
                                ptx::mma_lo<F32 ? 0 : 1>(d_main, a, b, kDescHi, F32 ? idesc2 : idesc, go);     // fp32: into d_cross too
                                if (F32) ptx::mma_lo<0>(d_cross, a + ((raw_bytes + b_bytes) >> 4), b, kDescHi, idesc, 1u);
                            }
                        ptx::mma_commit(ptx::smem_u32(&empty_bar[stage]));
                    }
                    accumulate = 1u;
                    if (++stage == (uint32_t)p.stages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (!ok) break;
                if (ptx::elect_one()) ptx::mma_commit(ptx::smem_u32(&tfull_bar[acc]));
                acc ^= 1u;
                if (acc == 0) acc_phase ^= 1u;
            }
        }
    } else if (warp < 2 + kEpiWarps) {
        const int q = warp & 3;                        // tensor-memory lane quarter this warp may read
        const int part = (warp - 2) >> 2;              // which half of the columns
        const int n_chunks = p.bm >> 4, per_part = (n_chunks + 1) >> 1;
        const int ch0 = part * per_part, ch1 = min(ch0 + per_part, n_chunks);
        uint32_t acc = 0, acc_phase = 0;
        bool ok = true;
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
            if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&tempty_bar[acc]));
            acc ^= 1u;
            if (acc == 0) acc_phase ^= 1u;
        };
        for (long long item = first_item; item < p.items && ok; item += item_step) {
            int fb, mb;
            linear_item(item, p.n_fblocks, p.n_mblocks, &fb, &mb);
            const int n = fb * kTileF + q * 32 + lane;
            const bool n_ok = n < p.N;
            const long long m_item = (long long)mb * p.bm;
            const float bias = SPLIT ? 0.0f : linear_bias<TYPE>(p.epi, n, n_ok);
            // the finished sums of one chunk of 16 rows
            auto emit = [&](float (&s)[16], int ch, LinearStore<TYPE, 16>& out) {
                if (SPLIT) {                            // partial sums over the operand slots, which nothing uses any more
                    const uint32_t red = smem_base + (uint32_t)(ch * 16 * 128 + q * 32 + lane) * 4u;
#pragma unroll
                    for (int j = 0; j < 16; ++j) asm volatile("st.shared.f32 [%0], %1;" ::"r"(red + j * 512), "f"(s[j]) : "memory");
                    return;
                }
                const long long m0 = m_item + ch * 16;
                const int rows = (int)min(16ll, p.M - m0);
                if (F32 && n_ok) retake_sums<1>(s, rows, m0, n, static_cast<const float*>(p.x), p.ldx, static_cast<const float*>(p.w), p.ldw, p.K, &alive);
                out.store(p.epi, s, bias, m0, rows, n, n_ok);
            };
            if (F32) {
                float sum[4][16];                       // at most 64 of the 128 columns belong to this warp
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c][j] = 0.0f;
                for (int seg = kb0; seg < kb1; seg += kSegment) {
                    if (!wait_acc()) {
                        ok = false;
                        break;
                    }
                    const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * (uint32_t)(p.bm * 2);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (ch0 + c < ch1) {
                            uint32_t va[16], vb[16];
                            ptx::tmem_ld16(taddr + (uint32_t)((ch0 + c) * 16), va);
                            ptx::tmem_ld16(taddr + (uint32_t)(p.bm + (ch0 + c) * 16), vb);
                            ptx::tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) sum[c][j] += __uint_as_float(va[j]) + __uint_as_float(vb[j]);
                        }
                    release_acc();
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (ch0 + c < ch1) {
                        LinearStore<TYPE, 16> out;
                        const long long m0 = m_item + (ch0 + c) * 16;
                        if (!SPLIT) out.fetch(p.epi, m0, (int)min(16ll, p.M - m0), n, n_ok);
                        emit(sum[c], ch0 + c, out);
                    }
            } else {
                LinearStore<TYPE, 16> out;
                auto fetch = [&](int ch) {
                    const long long m0 = m_item + ch * 16;
                    if (!SPLIT && ch < ch1) out.fetch(p.epi, m0, (int)min(16ll, p.M - m0), n, n_ok);
                };
                fetch(ch0);
                if (!wait_acc()) {
                    ok = false;
                    break;
                }
                const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * (uint32_t)p.bm;
                uint32_t v[16];
                if (ch0 < ch1) ptx::tmem_ld16(taddr + (uint32_t)(ch0 * 16), v);
                for (int ch = ch0; ch < ch1; ++ch) {
                    ptx::tmem_ld_wait();
                    float s[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) s[j] = __uint_as_float(v[j]);
                    LinearStore<TYPE, 16> now = out;
                    if (ch + 1 < ch1) ptx::tmem_ld16(taddr + (uint32_t)((ch + 1) * 16), v);
                    fetch(ch + 1);
                    emit(s, ch, now);
                }
                release_acc();
            }
        }
    } else if (COPY) {
        // copiers: a row's eight 16-byte pieces by eight lanes, four rows at a time by each warp
        const int w = warp - 2 - kEpiWarps, piece = lane & 7, sub = lane >> 3;
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        uint8_t* const generic_base = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
        const char *xb = static_cast<const char*>(p.x), *wb = static_cast<const char*>(p.w);
        const char *xe = xb + ((p.M - 1) * p.ldx + p.K) * EB, *we = wb + ((p.N - 1) * p.ldw + p.K) * EB;
        for (long long item = first_item; item < p.items && ok; item += item_step) {
            int fb, mb;
            linear_item(item, p.n_fblocks, p.n_mblocks, &fb, &mb);
            for (int kb = kb0; kb < kb1; ++kb) {
                int got = 1;
                if (lane == 0) got = ptx::mbar_wait_bounded(ptx::smem_u32(&empty_bar[stage]), phase ^ 1u, abortp, alivep) ? 1 : 0;
                got = __shfl_sync(0xffffffffu, got, 0);
                if (!got) {
                    if (lane == 0) failed(kErrAux);
                    ok = false;
                    break;
                }
                uint8_t* const sbase = generic_base + stage * stage_bytes;
                const int k0 = kb * kBlockElems + piece * (16 / EB);
                const int valid = min(16, (p.K - k0) * EB);
                auto rows_of = [&](const char* base, const char* end, long long ld, int row0, int total, int rows, uint8_t* tile, uint32_t to_low) {
#pragma unroll 4
                    for (int r = w * 4 + sub; r < rows; r += 4 * kAux) {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (row0 + r < total && valid > 0) v = load_piece<EB>(base + ((long long)(row0 + r) * ld + k0) * EB, valid, base, end);
                        const uint32_t at = (uint32_t)r * 128u + (uint32_t)((piece ^ (r & 7)) << 4);
                        *reinterpret_cast<uint4*>(tile + at) = v;
                        if (F32) *reinterpret_cast<float4*>(tile + to_low + at) = low_half(make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)));
                    }
                };
                rows_of(wb, we, p.ldw, fb * kTileF, p.N, kTileF, sbase, raw_bytes + b_bytes);
                rows_of(xb, xe, p.ldx, mb * p.bm, p.M, p.bm, sbase + off_b, b_bytes);
                fence_proxy_async_smem();                      // the tensor core reads these through the async proxy
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&full_bar[stage]));
                if (++stage == (uint32_t)p.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
    } else if (F32) {
        // converters: the low halves of both tiles, in the same (swizzled) places
        constexpr int kPer = F32 ? kAux / Roles<TYPE, COPY>::kGroups : 1;     // warps of a group
        const int w = warp - 2 - kEpiWarps, group = w / kPer, t = (w - group * kPer) * 32 + lane;
        uint32_t stage = 0, phase = 0;
        int turn = 0;
        bool ok = true;
        uint8_t* const generic_base = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
        for (long long item = first_item; item < p.items && ok; item += item_step)
            for (int kb = kb0; kb < kb1; ++kb) {
                if (turn == group) {
                    int got = 1;
                    if (lane == 0) got = ptx::mbar_wait_bounded(ptx::smem_u32(&full_bar[stage]), phase, abortp, alivep) ? 1 : 0;
                    got = __shfl_sync(0xffffffffu, got, 0);
                    if (!got) {
                        if (lane == 0) failed(kErrAux);
                        ok = false;
                        break;
                    }
                    const float4* const raw = reinterpret_cast<const float4*>(generic_base + stage * stage_bytes);
                    float4* const low = reinterpret_cast<float4*>(generic_base + stage * stage_bytes + raw_bytes);
                    const int a_count = (int)(a_bytes >> 4), b_count = (int)(b_bytes >> 4), count = a_count + b_count;
#pragma unroll 4
                    for (int i = t; i < count; i += 32 * kPer) low[i < a_count ? i + b_count : i - a_count] = low_half(raw[i]);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&low_bar[stage]));
                }
                if (++turn == Roles<TYPE, COPY>::kGroups) turn = 0;
                if (++stage == (uint32_t)p.stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
    }

    if (SPLIT) {
        __syncwarp();
        ptx::cluster_sync_all();
        if (warp >= 2 && warp < 2 + kEpiWarps && !*abortp && first_item < p.items) {
            int fb, mb;
            linear_item(first_item, p.n_fblocks, p.n_mblocks, &fb, &mb);
            const int row = (warp & 3) * 32 + lane, n = fb * kTileF + row;
            const bool n_ok = n < p.N;
            const float bias = linear_bias<TYPE>(p.epi, n, n_ok);
            if (n_ok)
                ptx::cluster_reduce_columns(smem_base, p.bm, rank, p.split, row, (warp - 2) >> 2, kEpiWarps >> 2, [&](int c, float sum) {
                    const long long m = (long long)mb * p.bm + c;
                    if (m >= p.M) return;
                    LinearStore<TYPE, 1> out;
                    out.fetch(p.epi, m, 1, n, true);
                    float s[1] = {sum};
                    if (F32) retake_sums<1>(s, 1, m, n, static_cast<const float*>(p.x), p.ldx, static_cast<const float*>(p.w), p.ldw, p.K, &alive);
                    out.store(p.epi, s, bias, m, 1, n, true);
                });
        }
        __syncwarp();
        ptx::cluster_sync_all();                           // nobody leaves while its partial sums are being read
    }

    // Teardown.  After an aborted run give copies still in flight time to land before shared memory is released.
    if (*abortp) __nanosleep(200000);
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
    }
}

template <int TYPE, bool COPY, bool SPLIT, int KB>
cudaError_t run_variant(const LinearTiling& t, LinearParams& p, int num_sms, const CUtensorMap& mx, const CUtensorMap& mw, cudaStream_t stream)
{
    constexpr bool F32 = TYPE == MNN_TYPE_FP32;
    static unsigned long long done = 0;
    auto kern = linear_kernel<TYPE, COPY, SPLIT, KB>;
    cudaError_t e = allow_smem_once(reinterpret_cast<const void*>(kern), kLinearSmem, &done);
    if (e != cudaSuccess) return e;
    const int stage_bytes = (kTileF + p.bm) * 128 * KB * (F32 ? 2 : 1);
    p.stages = (kLinearSmem - 1024) / stage_bytes;
    if (p.stages > kLinearMaxStages) p.stages = kLinearMaxStages;
    p.k_blocks = (p.K + 128 / (F32 ? 4 : 2) * KB - 1) / (128 / (F32 ? 4 : 2) * KB);
    p.tmem_cols = 32;
    while (p.tmem_cols < p.bm * (F32 ? 4 : 2)) p.tmem_cols *= 2;
    const dim3 block(Roles<TYPE, COPY>::kThreads);
    // the full budget of shared memory, so that one CTA at most is resident per SM: a second one could block in its
    // tensor-memory allocation
    if (SPLIT) return launch_cluster(t.split, kern, dim3((unsigned)(t.items * t.split)), block, (size_t)kLinearSmem, stream, mx, mw, p);
    const long long grid = t.items < num_sms ? t.items : num_sms;
    return launch_overlapped(kern, dim3((unsigned)grid), block, (size_t)kLinearSmem, stream, mx, mw, p);
}

template <int TYPE, int KB>
cudaError_t run_type(const LinearTiling& t, LinearParams& p, int num_sms, const CUtensorMap& mx, const CUtensorMap& mw, cudaStream_t stream)
{
    if (t.form == MNN_LINEAR_COPIED) return t.split > 1 ? run_variant<TYPE, true, true, 1>(t, p, num_sms, mx, mw, stream) : run_variant<TYPE, true, false, 1>(t, p, num_sms, mx, mw, stream);
    return t.split > 1 ? run_variant<TYPE, false, true, KB>(t, p, num_sms, mx, mw, stream) : run_variant<TYPE, false, false, KB>(t, p, num_sms, mx, mw, stream);
}

}  // namespace

cudaError_t allow_smem_once(const void* kern, int bytes, unsigned long long* done)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev < 64 && (__atomic_load_n(done, __ATOMIC_ACQUIRE) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) __atomic_fetch_or(done, bit, __ATOMIC_RELEASE);
    return e;
}

LinearTiling linear_tiling(const LinearShape& s, bool unaligned, int num_sms)
{
    const bool f32 = s.type == MNN_TYPE_FP32;
    const int eb = f32 ? 4 : 2;
    const bool strides = (s.ldx * eb) % 16 != 0 || (s.ldw * eb) % 16 != 0, copy = unaligned || strides;
    LinearTiling t = {};
    const long long w_bytes = (long long)s.N * s.K * eb, groups = (s.M + 3) / 4, pairs_of_features = (s.N + 1) / 2;
    // (the most that w may have in bytes for one group of rows)
    const long long most = s.M <= 2 ? (strides || f32 ? 1ll << 40 : (s.M == 1 ? 64 : 24) << 20) : (f32 ? strides ? 128 : 48 : strides ? 16 : 6) << 20;
    if ((s.M <= 4 && w_bytes <= most) ||
        (groups * pairs_of_features <= 10ll * num_sms && (s.M <= 32 || w_bytes <= 64 << 10) && groups * w_bytes <= (f32 ? strides ? 20 : 8 : 2) << 20)) {
        // up to four rows, or several groups of four where the product is small (beyond 32 rows: and w stays in L1): a stream of w
        // (linear_few.cu); two features a warp, and one, and several warps per K loop, where that leaves fewer than 16 warps per SM.
        // The more rows, the sooner the sums cost more than the stream.  Here and on tiles, us: BF16 1 x 2048 x 8192 6.2 and 8.2, 1 x 4096 x
        // 16384 28.1 and 24.5, 1 x 1008 x 131072 61 and 44, 2 x 1024 x 8192 5.6 and 6.8, 2 x 4096 x 4096 11.7 and 8.3, 4 x 1024 x 1000 3.5 and
        // 5.1, 4 x 4096 x 4096 12.3 and 8.4; fp32, whose halves cost tiles more, 2 x 2048 x 65536 88 and 136, 4 x 1024 x 8192 13.8 and 16.3,
        // 4 x 8192 x 8192 82 and 75; rows that tiles have to lay out first: BF16 1 x 1001 x 131072 92 and 155, 2 x 4099 x 16384 53 and 73,
        // 4 x 1022 x 4314 11.0 and 14.3, 4 x 4097 x 4096 26 and 23, fp32 4 x 1023 x 20000 50 and 72.  Groups: fp32 100 x 256 x 48 2.8 and 7.2,
        // 8 x 1024 x 1000 6.8 and 7.9, 12 x 1024 x 1000 8.8 and 8.0, and 16 x 12009 x 94, which tiles have to lay out first, 20.5 and
        // 34.6; BF16 100 x 256 x 48 2.5 and 3.5, 6 x 512 x 512 2.9 and 5.1, 8 x 704 x 1472 6.7 and 5.3; and with many warps
        // 1000 x 64 x 64 7.8 and 3.3 (fp32 5.8 and 5.4).
        t.form = MNN_LINEAR_FEW;
        t.bm = s.M < 4 ? s.M : 4;
        t.feats = s.M > 2 || s.N / 2 >= 16ll * num_sms ? 2 : 1;
        t.items = (s.N + t.feats - 1) / t.feats * groups;
        t.split = 1;
        while (t.split < 8 && t.items * t.split < 16ll * num_sms && (long long)s.K * eb >= 1024ll * t.split) t.split *= 2;
        return t;
    }
    // Estimated clocks of the tile kernel: waves of CTAs, each its share of K blocks at the slower of the tensor core (4096
    // multiply-adds of 16 bits a clock; fp32: shared memory) and the delivery of the tiles (about 48 bytes a clock
    // and SM by TMA, 3 by copier warps), plus start and end.  Rows whose strides TMA cannot copy are laid out anew first, at
    // about 20 bytes a clock and SM; where only a tensor's start is not aligned no workspace is kept for that, and copier warps
    // fetch it (64 x 4097 x 4096 BF16: 79 us by them).
    t.form = copy && !strides ? MNN_LINEAR_COPIED : MNN_LINEAR_TILES;
    t.feats = kTileF;
    const long long fblocks = (s.N + kTileF - 1) / kTileF, kblocks = ((long long)s.K * eb + 127) / 128;
    const double operand_bytes = ((double)s.M + s.N) * s.K * eb;
    t.relay = strides;
    if (t.relay) {
        t.ld_relay = kblocks * 128 / eb;             // whole lines: a row's 128 bytes then lie in one
        t.relay_bytes = (s.M + (long long)s.N) * t.ld_relay * eb;
    }
    const double tile_relay = t.relay ? 3000.0 + 2.0 * operand_bytes / (20.0 * num_sms) : 0.0;
    double best = 0;
    for (int bm = 16; bm <= (f32 ? 128 : 256); bm *= 2) {
        if (bm > 16 && bm / 2 >= s.M) break;
        const long long items = fblocks * ((s.M + bm - 1) / bm);
        for (int split = 1; split <= 8; split *= 2) {
            // (clusters of eight: only as many as surely run at one time)
            if (split > 1 && (items * split > num_sms || kblocks < 2 * split || (split == 8 && items > 8))) break;
            const double mma = f32 ? 1050.0 + 9.0 * bm : 2.0 * bm, load = (kTileF + bm) * 128.0 / (t.form == MNN_LINEAR_COPIED ? 3.0 : 48.0);
            const long long waves = (items * split + num_sms - 1) / num_sms;
            const double clocks = waves * ((kblocks + split - 1) / split * (mma > load ? mma : load)) + 1500.0 + (f32 ? 55.0 : 8.0) * bm + (split > 1 ? 1200.0 + 6.0 * bm : 0.0) + tile_relay;
            if (best == 0 || clocks < best) {
                best = clocks;
                t.bm = bm;
                t.split = split;
                t.items = items;
            }
        }
    }
    // Pairs of SMs (linear_pair.cu): half the rows of x per CTA, so that the tensor core and not the delivery decides.  fp32 (as
    // two FP16 halves, three products) needs a pass over both operands first, as rows that are not aligned do.  Here and on tiles, fp32:
    // 1024 x 4096 x 1024 65 and 84 us, 1024 x 1024 x 1024 24 and 30, 384 x 2048 x 2048 39 and 50, 512 x 4096 x 1024 (32 items of four
    // CTAs) 61 and 46; a short K does not earn the pass: 12544 x 128 x 256 20.0 and 14.2.
    // Fewer rows only where tiles have to lay fp32 operands out as well: 80 x 1001 x 8000 37 and 45, but 128 x 1024 x 32000 98 and 80.
    const long long pairs = num_sms / 2;
    if (s.M < (f32 && strides ? 72 : 192) || t.form == MNN_LINEAR_COPIED || (f32 && s.K < 192) || pairs < 1) return t;
    const long long blocks = ((long long)s.K + 63) / 64, ld = blocks * 64;
    const double relay = strides || f32 ? 3000.0 + 2.0 * operand_bytes / (20.0 * num_sms) : 0.0;
    for (int bm = 256; bm >= 128; bm -= 32) {
        const long long items = ((s.N + 255) / 256) * (long long)((s.M + bm - 1) / bm);
        const double clocks = (double)((items + pairs - 1) / pairs) * (blocks * (f32 ? 11.0 : 2.6) * bm + (f32 ? 4000.0 : 1000.0)) + 3500.0 + relay;
        if (clocks < best) {
            best = clocks;
            t.form = MNN_LINEAR_PAIRS;
            t.feats = 256;
            t.bm = bm;
            t.split = 1;
            t.items = items;
            t.relay = strides || f32;
            t.ld_relay = ld;
            t.relay_bytes = t.relay ? (s.M + (long long)s.N) * (f32 ? 4 * ld + 4 : 2 * ld) : 0;
        }
    }
    return t;
}

cudaError_t launch_linear(const LinearShape& s, const LinearTiling& t, int num_sms, const void* x, const void* w,
                          const LinearEpilogue& epi, int* status, void* relay, cudaStream_t stream, const char** why)
{
    LinearParams p = {};
    p.M = s.M; p.N = s.N; p.K = s.K;
    p.bm = t.bm;
    p.n_fblocks = (s.N + kTileF - 1) / kTileF;
    p.n_mblocks = (s.M + t.bm - 1) / t.bm;
    p.split = t.split;
    p.items = t.items;
    p.x = x; p.w = w; p.ldx = s.ldx; p.ldw = s.ldw;
    p.epi = epi;
    p.status = status;
    const int eb = s.type == MNN_TYPE_FP32 ? 4 : 2;
    CUtensorMap mx = {}, mw = {};
    const void *xs = x, *ws = w;
    long long ldx = s.ldx, ldw = s.ldw;
    if (t.relay) {
        const LinearRelayed rx = {x, s.M, s.ldx, relay, nullptr, nullptr}, rw = {w, s.N, s.ldw, static_cast<char*>(relay) + s.M * t.ld_relay * eb, nullptr, nullptr};
        cudaError_t e = launch_linear_relay(rx, rw, s.K, eb, t.ld_relay, num_sms, stream);
        if (e != cudaSuccess) return e;
        xs = rx.same;
        ws = rw.same;
        ldx = ldw = t.ld_relay;
    }
    if (t.form != MNN_LINEAR_COPIED && (!encode_rows_map(&mx, xs, eb, s.K, s.M, ldx, t.bm) || !encode_rows_map(&mw, ws, eb, s.K, s.N, ldw, kTileF))) {
        *why = "cuTensorMapEncodeTiled failed or is unavailable";
        return cudaErrorInvalidValue;
    }
    // two blocks of K per stage where the loop is long enough (a wait and a commit cost the issuing thread more than the four
    // instructions of a block) and that leaves three stages
    const long long blocks = ((long long)s.K * eb + 127) / 128 / t.split;
    const bool two = blocks >= 4 && t.bm <= 128;
    switch (s.type) {
        case MNN_TYPE_FP32: return run_type<MNN_TYPE_FP32, 1>(t, p, num_sms, mx, mw, stream);
        case MNN_TYPE_BF16: return two ? run_type<MNN_TYPE_BF16, 2>(t, p, num_sms, mx, mw, stream) : run_type<MNN_TYPE_BF16, 1>(t, p, num_sms, mx, mw, stream);
        default: return two ? run_type<MNN_TYPE_FP16, 2>(t, p, num_sms, mx, mw, stream) : run_type<MNN_TYPE_FP16, 1>(t, p, num_sms, mx, mw, stream);
    }
}

}  // namespace mnnb
