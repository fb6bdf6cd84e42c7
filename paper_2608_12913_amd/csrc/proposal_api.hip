// C ABI of the 8-bit proposal path: argument validation and the launches.
#include <math.h>

#include "../../include/dcd.h"
#include "proposal.h"

namespace dcd {
namespace {

constexpr size_t kAlign = 256;
constexpr long long kMaxRows = 1 << 24;
constexpr long long kMaxVocab = 1 << 30;
constexpr int kMaxHidden = 1 << 20;
// a launch counts its threads in 32 bits: workgroups of 256 threads take up to 64 row groups, or one block
constexpr long long kMaxRowGroups = (1LL << 30) - 64;
constexpr long long kMaxBlocks = (1LL << 24) - 1;

bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Makes the stream's device the current one for the length of a call.
class OnDeviceOf {
public:
    explicit OnDeviceOf(hipStream_t st) {
        if (!st) return;
        int dev = -1;
        ok_ = hipStreamGetDevice(st, &dev) == hipSuccess && hipGetDevice(&before_) == hipSuccess;
        if (!ok_ || dev == before_) return;
        ok_ = hipSetDevice(dev) == hipSuccess;
        moved_ = ok_;
    }
    ~OnDeviceOf() {
        if (moved_) (void)hipSetDevice(before_);
    }
    bool ok() const { return ok_; }

private:
    int before_ = -1;
    bool ok_ = true, moved_ = false;
};

bool logit_type(int dtype) { return dtype == DCD_F32 || dtype == DCD_BF16; }

int run_quantize(int64_t rows, int32_t cols, int32_t dtype, int32_t block_rows, const void *x, void *q, float *scale,
                 void *stream) {
    if (rows < 0 || cols < 1 || cols > kMaxHidden) return DCD_ERR_SHAPE;
    if (!logit_type(dtype) || (block_rows != 1 && block_rows != kGroup)) return DCD_ERR_PARAM;
    QuantProblem p{};
    p.rows = rows;
    p.cols = cols;
    p.groups = (cols + kGroup - 1) / kGroup;
    p.dtype = dtype == DCD_BF16 ? kBF16 : kF32;
    p.block_rows = block_rows;
    if (rows > kMaxVocab || (rows + block_rows - 1) / block_rows * p.groups > (block_rows == 1 ? kMaxRowGroups : kMaxBlocks))
        return DCD_ERR_SHAPE;
    if (cols % 16) return DCD_ERR_ALIGN;
    if (rows == 0) return DCD_OK;
    if (!x || !q || !scale) return DCD_ERR_NULL;
    if (!aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 4)) return DCD_ERR_ALIGN;
    p.x = x;
    p.q = (uint8_t *)q;
    p.scale = scale;
    const OnDeviceOf device((hipStream_t)stream);
    if (!device.ok()) return DCD_ERR_HIP;
    return launch_quantize(p, (hipStream_t)stream) == hipSuccess ? DCD_OK : DCD_ERR_HIP;
}

int run_logits(const dcd_fp8_problem *p, const dcd_fp8_inputs *in, void *logits, void *stream) {
    if (!p) return DCD_ERR_NULL;
    if (p->rows < 0 || p->vocab < 1 || p->hidden < 1) return DCD_ERR_SHAPE;
    if (p->rows > kMaxRows || p->vocab > kMaxVocab || p->hidden > kMaxHidden) return DCD_ERR_SHAPE;
    const int64_t stride = p->stride ? p->stride : p->vocab;
    if (stride < p->vocab || stride > kMaxVocab) return DCD_ERR_SHAPE;
    if (!logit_type(p->dtype)) return DCD_ERR_PARAM;
    // tiles of 256 tokens x at least 128 rows, 512 threads each, their total counted in 32 bits
    if (((int64_t)p->vocab / 256 + 9) * (p->rows / 128 + 1) >= 1 << 23) return DCD_ERR_SHAPE;
    if (p->hidden % 16) return DCD_ERR_ALIGN;
    if (p->rows == 0) return DCD_OK;
    if (!in || !in->h || !in->h_scale || !in->w || !in->w_scale || !logits) return DCD_ERR_NULL;
    if (!aligned(in->h, 16) || !aligned(in->w, 16) || !aligned(in->h_scale, 4) || !aligned(in->w_scale, 4) ||
        !aligned(in->bias, 4) || !aligned(logits, p->dtype == DCD_BF16 ? 2 : 4))
        return DCD_ERR_ALIGN;
    Fp8Problem P{};
    P.M = p->rows;
    P.N = p->vocab;
    P.K = p->hidden;
    P.groups = (p->hidden + kGroup - 1) / kGroup;
    P.dtype = p->dtype == DCD_BF16 ? kBF16 : kF32;
    P.stride = stride;
    P.h = (const uint8_t *)in->h;
    P.w = (const uint8_t *)in->w;
    P.hs = in->h_scale;
    P.ws = in->w_scale;
    P.bias = in->bias;
    P.out = logits;
    const OnDeviceOf device((hipStream_t)stream);
    if (!device.ok()) return DCD_ERR_HIP;
    return launch_logits_fp8(P, (hipStream_t)stream) == hipSuccess ? DCD_OK : DCD_ERR_HIP;
}

int make_sample(const dcd_sample_problem *p, SampleProblem &P) {
    if (!p) return DCD_ERR_NULL;
    if (p->rows < 0 || p->vocab < 1) return DCD_ERR_SHAPE;
    if (p->rows > kMaxRows || p->vocab > kMaxVocab) return DCD_ERR_SHAPE;
    const int64_t stride = p->stride ? p->stride : p->vocab;
    if (stride < p->vocab || stride > kMaxVocab) return DCD_ERR_SHAPE;
    if (!logit_type(p->dtype)) return DCD_ERR_PARAM;
    // a launch counts its threads in 32 bits: 512 per row, 256 per slice of at least 2,048 tokens
    if (p->rows >= 1 << 22 || ((int64_t)p->vocab / 2048 + 1) * p->rows >= 1 << 24) return DCD_ERR_SHAPE;
    P = SampleProblem{};
    P.R = p->rows;
    P.V = p->vocab;
    P.dtype = p->dtype == DCD_BF16 ? kBF16 : kF32;
    P.stride = stride;
    return DCD_OK;
}

int run_sample(const dcd_sample_problem *p, const dcd_sample_inputs *in, const dcd_sample_outputs *out, void *ws,
               size_t ws_bytes, void *stream) {
    SampleProblem P;
    const int rc = make_sample(p, P);
    if (rc) return rc;
    if (P.R == 0) return DCD_OK;
    if (!in || !out || !in->logits || !in->u || !out->tokens) return DCD_ERR_NULL;
    const void *four[] = {in->u,       in->temperature, in->top_k,    in->top_p, in->min_p,
                          out->tokens, out->probs,      out->logprob, out->kept};
    for (const void *q : four)
        if (!aligned(q, 4)) return DCD_ERR_ALIGN;
    if (!aligned(in->logits, p->dtype == DCD_BF16 ? 2 : 4)) return DCD_ERR_ALIGN;
    if (!ws || ws_bytes < sample_workspace(P) || !aligned(ws, kAlign)) return DCD_ERR_WORKSPACE;
    P.logits = in->logits;
    P.u = in->u;
    P.temperature = in->temperature;
    P.top_k = in->top_k;
    P.top_p = in->top_p;
    P.min_p = in->min_p;
    P.tokens = out->tokens;
    P.probs = out->probs;
    P.logprob = out->logprob;
    P.kept = out->kept;
    const OnDeviceOf device((hipStream_t)stream);
    if (!device.ok()) return DCD_ERR_HIP;
    return launch_sample(P, ws, (hipStream_t)stream) == hipSuccess ? DCD_OK : DCD_ERR_HIP;
}

}  // namespace
}  // namespace dcd

extern "C" {

int dcd_quantize_fp8(int64_t rows, int32_t cols, int32_t dtype, int32_t block_rows, const void *x, void *q,
                     float *scale, void *hip_stream) {
    return dcd::run_quantize(rows, cols, dtype, block_rows, x, q, scale, hip_stream);
}

int dcd_logits_fp8(const dcd_fp8_problem *p, const dcd_fp8_inputs *in, void *logits, void *hip_stream) {
    return dcd::run_logits(p, in, logits, hip_stream);
}

size_t dcd_sample_workspace_bytes(const dcd_sample_problem *p) {
    dcd::SampleProblem P;
    return dcd::make_sample(p, P) == DCD_OK ? dcd::sample_workspace(P) : 0;
}

int dcd_sample(const dcd_sample_problem *p, const dcd_sample_inputs *in, const dcd_sample_outputs *out,
               void *workspace, size_t workspace_bytes, void *hip_stream) {
    return dcd::run_sample(p, in, out, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
