// The matrix product over rows, y = act(x w^T + bias) with a residual, on the tensor cores: host-side description.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

namespace mnnb {

// What follows the sums s[m][n] = sum_k x[m][k] w[n][k]; types and enumerations as in mnn_conv.h.
struct LinearEpilogue {
    const void* bias;        // [N] or null
    const void* residual;    // [M][ldr], read where res_mode != 0
    void* y;                 // [M][ldy]
    long long ldr, ldy;
    int act, res_mode;
};

struct LinearShape {
    int M, N, K, type;               // type: MNN_TYPE_*
    long long ldx, ldw, ldy, ldr;    // elements between rows
};

// How a product is cut: decided from sizes and alignment alone, ahead of any run.
struct LinearTiling {
    int form;            // MNN_LINEAR_*
    int bm;              // rows of x per work item
    int feats;           // features per work item
    int split;           // CTAs of a cluster (MNN_LINEAR_FEW: warps of a CTA) that share a work item's K loop
    long long items;
    bool relay;          // the operands are laid out anew first (linear_relay.cu)
    long long ld_relay;  // elements between rows there (of halves: fp32 on pairs)
    long long relay_bytes;
};

// unaligned: x or w does not start on a 16-byte boundary.
LinearTiling linear_tiling(const LinearShape& s, bool unaligned, int num_sms);

// An operand that is laid out anew: src -> same; fp32 on pairs: src -> high halves (same), low halves and the exponents of the rows' scales.
struct LinearRelayed {
    const void* src;
    long long rows, ld;              // ld: elements between rows of src
    void *same, *low;
    int* up;
};

// `relay`: relay_bytes of device memory.
cudaError_t launch_linear(const LinearShape& s, const LinearTiling& t, int num_sms, const void* x, const void* w,
                          const LinearEpilogue& epi, int* status, void* relay, cudaStream_t stream, const char** why);
cudaError_t launch_linear_few(const LinearShape& s, const LinearTiling& t, const void* x, const void* w, const LinearEpilogue& epi, cudaStream_t stream);
cudaError_t launch_linear_pair(const LinearShape& s, const LinearTiling& t, int num_sms, const void* x, const void* w,
                               const LinearEpilogue& epi, int* status, void* relay, cudaStream_t stream, const char** why);
cudaError_t launch_linear_relay(const LinearRelayed& x, const LinearRelayed& w, int K, int elem_bytes, long long ld_out, int num_sms, cudaStream_t stream);

// 2-D map over rows of k_len elements, ld elements apart; box = box_rows rows of 128 bytes in the 128-byte swizzle; what lies
// outside reads as zero.
bool encode_rows_map(CUtensorMap* map, const void* base, int elem_bytes, long long k_len, long long rows, long long ld, int box_rows);

// Allows `kern` its shared memory on the current device; asked once per device and kernel (`done` has a bit for each device).
cudaError_t allow_smem_once(const void* kern, int bytes, unsigned long long* done);

}  // namespace mnnb
