// One token per row of logits with temperature, top-k, top-p and min-p: host-side description.
#pragma once
#include <cuda_runtime.h>

namespace mnnb {

struct SampleShape {
    int rows, vocab, type;           // type: MNN_TYPE_*
    long long ld;                    // elements between rows of logits
    long long ld_probs;              // elements between rows of probs
};

// How a row is cut: a cluster of `ctas` CTAs of `warps` warps holds it in shared memory, each warp a run of `run` elements.
struct SampleTiling {
    int ctas, warps, run;
    int scale_log2;                  // weights are integers in units of 2^-scale_log2
};

struct SampleArgs {
    const void* logits;
    const float* temperature;
    const int* top_k;
    const float *top_p, *min_p, *u;
    int* token;
    float *prob, *probs;
};

// The largest vocabulary that a cluster holds.
constexpr int kSampleMaxVocab = 320 * 1024;

SampleTiling sample_tiling(const SampleShape& s, int num_sms);
cudaError_t launch_sample(const SampleShape& s, const SampleTiling& t, const SampleArgs& a, cudaStream_t stream);

}  // namespace mnnb
