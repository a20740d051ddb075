// C ABI of what follows a feature map: the matrix product over rows (linear.cu, linear_pair.cu) and sampling (sample.cu).
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>
#include <new>

#include "../../include/mnn_conv.h"
#include "errors.h"
#include "linear.h"
#include "planner.h"
#include "sample.h"

using namespace mnnb;

static_assert(kSampleMaxVocab == MNN_SAMPLE_MAX_VOCAB, "the header states what a cluster holds");

struct mnn_linear_plan_s {
    LinearShape s;
    int act, residual, num_sms;
    LinearTiling tiling;             // by the row strides
    LinearTiling unaligned;          // where a run's x or w does not start on a 16-byte boundary
    char* ws = nullptr;              // status word, then the operands laid out anew
    long long workspace_bytes = 0;
};

struct mnn_sample_plan_s {
    SampleShape s;
    SampleTiling tiling;
};

namespace {

constexpr long long kStatusBytes = 1024;   // head of the workspace: device status word

int type_bytes(int type) { return type == MNN_TYPE_FP32 ? 4 : 2; }
bool known_type(int type) { return type >= MNN_TYPE_FP32 && type <= MNN_TYPE_FP16; }
bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

// Whether two sets of rows share memory.  (Rows of one stride whose columns lie side by side, as in a concatenated buffer, do not.)
struct RowSet {
    const void* base;
    long long rows, row_bytes, stride_bytes;
};
bool overlap(const RowSet& a, const RowSet& b)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.base), b0 = reinterpret_cast<uintptr_t>(b.base);
    const uintptr_t a1 = a0 + (uintptr_t)((a.rows - 1) * a.stride_bytes + a.row_bytes), b1 = b0 + (uintptr_t)((b.rows - 1) * b.stride_bytes + b.row_bytes);
    if (a1 <= b0 || b1 <= a0) return false;
    if (a.stride_bytes != b.stride_bytes) return true;
    const long long stride = a.stride_bytes, off = b0 >= a0 ? (long long)((b0 - a0) % (uintptr_t)stride) : (stride - (long long)((a0 - b0) % (uintptr_t)stride)) % stride;
    return off < a.row_bytes || off + b.row_bytes > stride;
}

}  // namespace

extern "C" {

mnn_linear_plan_t mnn_linear_plan(int M, int N, int K, const mnn_linear_opts* opts)
{
    mnn_linear_opts o;
    std::memset(&o, 0, sizeof(o));
    if (opts) o = *opts;
    if (M <= 0 || N <= 0 || K <= 0) {
        report_error(MNN_EINVAL, "M, N and K must be positive");
        return nullptr;
    }
    if (!known_type(o.type) || o.act < MNN_ACT_NONE || o.act > MNN_ACT_SILU || o.residual < MNN_RESIDUAL_NONE || o.residual > MNN_RESIDUAL_BEFORE) {
        report_error(MNN_EINVAL, "an option is outside its range");
        return nullptr;
    }
    if (o.ldx == 0) o.ldx = K;
    if (o.ldw == 0) o.ldw = K;
    if (o.ldy == 0) o.ldy = N;
    if (o.ldr == 0) o.ldr = N;
    if (o.ldx < K || o.ldw < K || o.ldy < N || o.ldr < N) {
        report_error(MNN_EINVAL, "a row stride is smaller than the row");
        return nullptr;
    }
    if (M > (1 << 28) || N > (1 << 28) || K > (1 << 28)) {
        report_error(MNN_EUNSUPPORTED, "M, N and K may be up to 2^28");
        return nullptr;
    }
    const long long most = 1ll << 40;
    if (o.ldx >= most / M || o.ldw >= most / N || o.ldy >= most / M || o.ldr >= most / M) {
        report_error(MNN_EUNSUPPORTED, "tensor too large");
        return nullptr;
    }
    mnn_linear_plan_t p = new (std::nothrow) mnn_linear_plan_s();
    if (!p) {
        report_error(MNN_EINVAL, "out of host memory");
        return nullptr;
    }
    p->s = LinearShape{M, N, K, o.type, o.ldx, o.ldw, o.ldy, o.ldr};
    p->act = o.act;
    p->residual = o.residual;
    p->num_sms = (int)current_calibration().c[7];
    p->tiling = linear_tiling(p->s, false, p->num_sms);
    p->unaligned = linear_tiling(p->s, true, p->num_sms);
    p->workspace_bytes = kStatusBytes + (p->tiling.relay_bytes > p->unaligned.relay_bytes ? p->tiling.relay_bytes : p->unaligned.relay_bytes);
    return p;
}

int mnn_linear_plan_query(mnn_linear_plan_t p, mnn_linear_info* info)
{
    if (!p || !info) return report_error(MNN_EINVAL, "NULL plan or info");
    std::memset(info, 0, sizeof(*info));
    info->M = p->s.M; info->N = p->s.N; info->K = p->s.K;
    info->type = p->s.type; info->act = p->act; info->residual = p->residual;
    info->form = p->tiling.form;
    info->form_unaligned = p->unaligned.form;
    info->rows_per_item = p->tiling.bm;
    info->features_per_item = p->tiling.feats;
    info->split = p->tiling.split;
    info->launches_per_run = p->tiling.relay ? 2 : 1;
    info->items = p->tiling.items;
    info->workspace_bytes = p->workspace_bytes;
    return MNN_OK;
}

int mnn_linear_set_workspace(mnn_linear_plan_t p, void* workspace, long long bytes)
{
    if (!p) return report_error(MNN_EINVAL, "NULL plan");
    p->ws = nullptr;
    if (!workspace) return report_error(MNN_EWORKSPACE, "the plan needs a workspace");
    if (bytes < p->workspace_bytes) return report_error(MNN_EWORKSPACE, "workspace smaller than info.workspace_bytes");
    if (!aligned(workspace, 1024)) return report_error(MNN_EALIGN, "workspace must be 1024-byte aligned");
    cudaError_t e = cudaMemset(workspace, 0, sizeof(int));
    if (e != cudaSuccess) return report_cuda_error(e, "clearing the status word");
    p->ws = static_cast<char*>(workspace);
    return MNN_OK;
}

int mnn_linear_run(mnn_linear_plan_t p, const void* x, const void* w, const void* bias, const void* residual, void* y, void* stream)
{
    if (!p || !x || !w || !y) return report_error(MNN_EINVAL, "NULL argument");
    if ((p->residual != MNN_RESIDUAL_NONE) != (residual != nullptr))
        return report_error(MNN_EINVAL, p->residual ? "the plan has a residual and none was given" : "a residual was given and the plan has none");
    if (!p->ws) return report_error(MNN_EWORKSPACE, "call mnn_linear_set_workspace first");
    const int eb = type_bytes(p->s.type);
    if (!aligned(x, eb) || !aligned(w, eb) || !aligned(y, eb) || !aligned(bias, eb) || !aligned(residual, eb))
        return report_error(MNN_EALIGN, "a tensor is not aligned to its elements");
    const LinearShape& s = p->s;
    const RowSet out = {y, s.M, (long long)s.N * eb, s.ldy * eb};
    if (overlap(out, {x, s.M, (long long)s.K * eb, s.ldx * eb}) || overlap(out, {w, s.N, (long long)s.K * eb, s.ldw * eb}) ||
        (bias && overlap(out, {bias, 1, (long long)s.N * eb, (long long)s.N * eb})))
        return report_error(MNN_EINVAL, "y must not overlap x, w or bias");
    if (residual && !(residual == y && s.ldr == s.ldy) && overlap(out, {residual, s.M, (long long)s.N * eb, s.ldr * eb}))
        return report_error(MNN_EINVAL, "y must be the residual itself or not overlap it");
    const LinearTiling& t = aligned(x, 16) && aligned(w, 16) ? p->tiling : p->unaligned;
    const LinearEpilogue epi = {bias, residual, y, p->s.ldr, p->s.ldy, p->act, p->residual};
    const char* why = "launching the matrix product";
    int* const status = reinterpret_cast<int*>(p->ws);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = t.form == MNN_LINEAR_FEW     ? launch_linear_few(s, t, x, w, epi, st)
                    : t.form == MNN_LINEAR_PAIRS ? launch_linear_pair(s, t, p->num_sms, x, w, epi, status, p->ws + kStatusBytes, st, &why)
                                                 : launch_linear(s, t, p->num_sms, x, w, epi, status, p->ws + kStatusBytes, st, &why);
    return e == cudaSuccess ? MNN_OK : report_cuda_error(e, why);
}

int mnn_linear_device_status(mnn_linear_plan_t p, void* stream, int* code)
{
    if (!p || !code) return report_error(MNN_EINVAL, "NULL plan or code");
    *code = 0;
    if (!p->ws) return MNN_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaMemcpyAsync(code, p->ws, sizeof(int), cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return report_cuda_error(e, "reading the status word");
    if (*code != 0) {
        e = cudaMemsetAsync(p->ws, 0, sizeof(int), st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
        if (e != cudaSuccess) return report_cuda_error(e, "clearing the status word");
    }
    return MNN_OK;
}

void mnn_linear_destroy(mnn_linear_plan_t p) { delete p; }

mnn_sample_plan_t mnn_sample_plan(int rows, int vocab, const mnn_sample_opts* opts)
{
    mnn_sample_opts o;
    std::memset(&o, 0, sizeof(o));
    if (opts) o = *opts;
    if (rows <= 0 || vocab <= 0) {
        report_error(MNN_EINVAL, "rows and vocab must be positive");
        return nullptr;
    }
    if (!known_type(o.type)) {
        report_error(MNN_EINVAL, "an option is outside its range");
        return nullptr;
    }
    if (o.ld == 0) o.ld = vocab;
    if (o.ld_probs == 0) o.ld_probs = vocab;
    if (o.ld < vocab || o.ld_probs < vocab) {
        report_error(MNN_EINVAL, "a row stride is smaller than the row");
        return nullptr;
    }
    if (vocab > MNN_SAMPLE_MAX_VOCAB) {
        report_error(MNN_EUNSUPPORTED, "vocab is larger than MNN_SAMPLE_MAX_VOCAB");
        return nullptr;
    }
    if (rows > (1 << 27) || o.ld >= (1ll << 40) / rows || o.ld_probs >= (1ll << 40) / rows) {
        report_error(MNN_EUNSUPPORTED, "tensor too large");
        return nullptr;
    }
    mnn_sample_plan_t p = new (std::nothrow) mnn_sample_plan_s();
    if (!p) {
        report_error(MNN_EINVAL, "out of host memory");
        return nullptr;
    }
    p->s = SampleShape{rows, vocab, o.type, o.ld, o.ld_probs};
    p->tiling = sample_tiling(p->s, (int)current_calibration().c[7]);
    return p;
}

int mnn_sample_plan_query(mnn_sample_plan_t p, mnn_sample_info* info)
{
    if (!p || !info) return report_error(MNN_EINVAL, "NULL plan or info");
    info->rows = p->s.rows; info->vocab = p->s.vocab; info->type = p->s.type;
    info->ctas_per_row = p->tiling.ctas;
    info->threads = 32 * p->tiling.warps;
    info->scale_log2 = p->tiling.scale_log2;
    return MNN_OK;
}

int mnn_sample_run(mnn_sample_plan_t p, const void* logits, const float* u, const float* temperature, const int* top_k,
                   const float* top_p, const float* min_p, int* token, float* prob, float* probs, void* stream)
{
    if (!p || !logits || !u || !token) return report_error(MNN_EINVAL, "NULL argument");
    if (!aligned(logits, type_bytes(p->s.type)) || !aligned(u, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) ||
        !aligned(min_p, 4) || !aligned(token, 4) || !aligned(prob, 4) || !aligned(probs, 4))
        return report_error(MNN_EALIGN, "an array is not aligned to its elements");
    const SampleArgs a = {logits, temperature, top_k, top_p, min_p, u, token, prob, probs};
    cudaError_t e = launch_sample(p->s, p->tiling, a, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? MNN_OK : report_cuda_error(e, "launching the sampling kernel");
}

void mnn_sample_destroy(mnn_sample_plan_t p) { delete p; }

}  // extern "C"
