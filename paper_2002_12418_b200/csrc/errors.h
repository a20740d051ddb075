// The reason behind a status code, kept per thread for mnn_last_error (api.cu).
#pragma once
#include <cuda_runtime.h>

namespace mnnb {

int report_error(int code, const char* why);                   // returns code
int report_cuda_error(cudaError_t e, const char* where);       // returns MNN_ECUDA

}  // namespace mnnb
