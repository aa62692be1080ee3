// C interface of the worker's operators: argument checks, then the launches
// of layer_norm.hip and vocab_loss.hip.  Nothing here allocates, waits or
// throws, and a call that is refused has enqueued nothing.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdint>
#include <cstdio>

#include "kernels.hpp"
#include "phub.h"
#include "worker_ops.hpp"

namespace {

constexpr int64_t kMaxNormRows = (int64_t(1) << 30) - 1, kMaxNormCols = int64_t(1) << 20;
constexpr int64_t kMaxRows = int64_t(1) << 21, kMaxCols = int64_t(1) << 16;
constexpr int64_t kMaxVocab = int64_t(1) << 24, kMaxStride = int64_t(1) << 21;
constexpr int kMaxTop = 1024;
constexpr int64_t kMaxEntries = int64_t(1) << 30;
constexpr uintptr_t kWorkspaceAlign = 256;

// Sets the error message; without host memory for it the code alone is
// returned (nothing may be thrown across the C interface).
int report(int code, const char* text) {
    try {
        return phub::report_error(code, text);
    } catch (...) {
        return code;
    }
}

template <typename... A>
int refuse(const char* fmt, A... args) {
    char text[256];
    std::snprintf(text, sizeof text, fmt, args...);
    return report(PHUB_EINVAL, text);
}

int check_type(int type) {
    if (type < PHUB_F32 || type > PHUB_F16) return refuse("unknown element type %d", type);
    return PHUB_OK;
}

uintptr_t element_bytes(int type) { return type == PHUB_F32 ? 4 : 2; }

int check_size(const char* name, int64_t n, int64_t least, int64_t most) {
    if (n < least || n > most)
        return refuse("%s is %lld, outside [%lld, %lld]", name, (long long)n, (long long)least,
                      (long long)most);
    return PHUB_OK;
}

int check_pointer(const char* name, const void* p, uintptr_t align, bool needed) {
    if (!p && needed) return refuse("%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % align != 0)
        return refuse("%s is not aligned to %d bytes", name, int(align));
    return PHUB_OK;
}

int check_matrix(const char* name, const void* p, int64_t stride, int64_t cols, int64_t most,
                 uintptr_t align, bool needed) {
    if (int rc = check_pointer(name, p, align, needed)) return rc;
    if (p && (stride < cols || stride > most))
        return refuse("the rows of %s are %lld elements apart, outside [%lld, %lld]", name,
                      (long long)stride, (long long)cols, (long long)most);
    return PHUB_OK;
}

int check_workspace(const void* p, int64_t bytes, int64_t least) {
    if (least == 0) return PHUB_OK;
    if (int rc = check_pointer("workspace", p, kWorkspaceAlign, true)) return rc;
    if (bytes < least)
        return refuse("the workspace has %lld bytes, %lld are needed", (long long)bytes,
                      (long long)least);
    return PHUB_OK;
}

int launched(hipError_t e, const char* what) {
    if (e == hipSuccess) return PHUB_OK;
    char text[256];
    std::snprintf(text, sizeof text, "launch of %s failed: %s (%d)", what, hipGetErrorString(e),
                  int(e));
    return report(PHUB_EHIP, text);
}

int check_norm(int type, int64_t rows, int64_t cols) {
    if (int rc = check_type(type)) return rc;
    if (int rc = check_size("rows", rows, 0, kMaxNormRows)) return rc;
    return check_size("cols", cols, 1, kMaxNormCols);
}

constexpr int64_t kAnyStride = int64_t(1) << 40;

int64_t norm_bytes(int64_t rows, int64_t cols) {
    return 2 * phub::norm_strips(rows, cols) * cols * int64_t(sizeof(float));
}

// The checks that the losses share.  top 0: targets.
int check_vocab(const phub::VocabArgs& a, bool grad) {
    const bool any = a.rows > 0;
    if (int rc = check_type(a.type)) return rc;
    if (int rc = check_size("rows", a.rows, 0, kMaxRows)) return rc;
    if (int rc = check_size("cols", a.cols, 1, kMaxCols)) return rc;
    if (int rc = check_size("vocab", a.vocab, 1, kMaxVocab)) return rc;
    const uintptr_t element = element_bytes(a.type);
    if (int rc = check_matrix("x", a.x, a.x_stride, a.cols, kMaxStride, element, any)) return rc;
    if (int rc = check_matrix("w", a.w, a.w_stride, a.cols, kMaxStride, element, any)) return rc;
    if (int rc = check_pointer(a.top ? "index" : "target", a.target, 8, any)) return rc;
    if (a.top)
        if (int rc = check_pointer("logit", a.logit, 4, any)) return rc;
    if (int rc = check_pointer("lse", a.lse, 4, any)) return rc;
    if (!grad) return check_pointer("loss", a.loss, 4, any);
    if (int rc = check_pointer("dloss", a.dloss, 4, false)) return rc;
    if (int rc = check_matrix("dx", a.dx, a.dx_stride, a.cols, kMaxStride, element, false)) return rc;
    return check_matrix("dw", a.dw, a.dw_stride, a.cols, kMaxStride, 4, false);
}

int check_teacher(int64_t rows, int top, float temperature) {
    if (int rc = check_size("top", top, 1, kMaxTop)) return rc;
    if (int rc = check_size("rows", rows, 0, kMaxRows)) return rc;
    if (rows * top > kMaxEntries)
        return refuse("%lld rows of %d entries are more than 2^30", (long long)rows, top);
    if (!(temperature >= 1e-6f && temperature <= 1e6f))
        return refuse("temperature %g is outside [1e-6, 1e6]", double(temperature));
    return PHUB_OK;
}

// *piece: what the workspace is enough for.
int check_vocab_workspace(const phub::VocabArgs& a, bool grad, const void* p, int64_t bytes,
                          int64_t* piece) {
    if (int rc = check_pointer("workspace", p, kWorkspaceAlign, true)) return rc;
    *piece = phub::vocab_piece(a, grad, bytes);
    if (*piece > 0) return PHUB_OK;
    int64_t least = 0;
    phub::vocab_bytes(a, grad, &least, nullptr);
    return check_workspace(p, bytes, least);
}

int loss(const phub::VocabArgs& a, void* workspace, int64_t bytes, void* stream) {
    if (int rc = check_vocab(a, false)) return rc;
    if (a.rows == 0) return PHUB_OK;
    int64_t piece = 0;
    if (int rc = check_vocab_workspace(a, false, workspace, bytes, &piece)) return rc;
    return launched(phub::launch_vocab_loss(a, piece, workspace, static_cast<hipStream_t>(stream)),
                    "a loss over the vocabulary");
}

int loss_grad(const phub::VocabArgs& a, void* workspace, int64_t bytes, void* stream) {
    if (int rc = check_vocab(a, true)) return rc;
    if (!a.dx && !a.dw) return PHUB_OK;
    int64_t piece = 0;
    if (a.rows > 0)
        if (int rc = check_vocab_workspace(a, true, workspace, bytes, &piece)) return rc;
    return launched(
        phub::launch_vocab_loss_grad(a, piece, workspace, static_cast<hipStream_t>(stream)),
        "a loss's gradients over the vocabulary");
}

}  // namespace

int phub_layer_norm(int type, int64_t rows, int64_t cols, const void* x, int64_t x_stride,
                    const float* weight, const float* bias, float eps, void* y, int64_t y_stride,
                    float* mean, float* rstd, void* hip_stream) {
    if (int rc = check_norm(type, rows, cols)) return rc;
    const uintptr_t element = element_bytes(type);
    if (int rc = check_matrix("x", x, x_stride, cols, kAnyStride, element, rows > 0)) return rc;
    if (int rc = check_matrix("y", y, y_stride, cols, kAnyStride, element, rows > 0)) return rc;
    if (int rc = check_pointer("weight", weight, 4, false)) return rc;
    if (int rc = check_pointer("bias", bias, 4, false)) return rc;
    if (int rc = check_pointer("mean", mean, 4, false)) return rc;
    if (int rc = check_pointer("rstd", rstd, 4, false)) return rc;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return refuse("eps %g is not a number >= 0", double(eps));
    phub::NormArgs a{};
    a.type = type;
    a.rows = rows;
    a.cols = cols;
    a.x = x;
    a.x_stride = x_stride;
    a.weight = weight;
    a.bias = bias;
    a.eps = eps;
    a.y = y;
    a.y_stride = y_stride;
    a.mean = mean;
    a.rstd = rstd;
    return launched(phub::launch_layer_norm(a, static_cast<hipStream_t>(hip_stream)), "layer norm");
}

int phub_layer_norm_grad_bytes(int64_t rows, int64_t cols, int64_t* bytes) {
    if (int rc = check_norm(PHUB_F32, rows, cols)) return rc;
    if (int rc = check_pointer("bytes", bytes, 8, true)) return rc;
    *bytes = norm_bytes(rows, cols);
    return PHUB_OK;
}

int phub_layer_norm_grad(int type, int64_t rows, int64_t cols, const void* dy, int64_t dy_stride,
                         const void* x, int64_t x_stride, const float* weight, const float* mean,
                         const float* rstd, void* dx, int64_t dx_stride, float* dweight,
                         float* dbias, int accumulate, void* workspace, int64_t workspace_bytes,
                         void* hip_stream) {
    if (int rc = check_norm(type, rows, cols)) return rc;
    const bool any = rows > 0;
    const uintptr_t element = element_bytes(type);
    if (int rc = check_matrix("dy", dy, dy_stride, cols, kAnyStride, element, any)) return rc;
    if (int rc = check_matrix("x", x, x_stride, cols, kAnyStride, element, any)) return rc;
    if (int rc = check_pointer("weight", weight, 4, false)) return rc;
    if (int rc = check_pointer("mean", mean, 4, any)) return rc;
    if (int rc = check_pointer("rstd", rstd, 4, any)) return rc;
    if (int rc = check_matrix("dx", dx, dx_stride, cols, kAnyStride, element, false)) return rc;
    if (int rc = check_pointer("dweight", dweight, 4, false)) return rc;
    if (int rc = check_pointer("dbias", dbias, 4, false)) return rc;
    if (!dx && !dweight && !dbias) return PHUB_OK;
    if (dweight || dbias)
        if (int rc = check_workspace(workspace, workspace_bytes, norm_bytes(rows, cols))) return rc;
    phub::NormArgs a{};
    a.type = type;
    a.rows = rows;
    a.cols = cols;
    a.x = x;
    a.x_stride = x_stride;
    a.dy = dy;
    a.dy_stride = dy_stride;
    a.weight = weight;
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.y = dx;
    a.y_stride = dx_stride;
    a.dweight = dweight;
    a.dbias = dbias;
    a.accumulate = accumulate != 0;
    a.partial = static_cast<float*>(workspace);
    return launched(phub::launch_layer_norm_grad(a, static_cast<hipStream_t>(hip_stream)),
                    "layer norm's gradients");
}

int phub_vocab_bytes(int type, int64_t rows, int64_t cols, int64_t vocab, const void* x,
                     int64_t x_stride, const void* w, int64_t w_stride, int top, int grad,
                     int64_t* least, int64_t* best) {
    if (int rc = check_type(type)) return rc;
    if (int rc = check_size("rows", rows, 0, kMaxRows)) return rc;
    if (int rc = check_size("cols", cols, 1, kMaxCols)) return rc;
    if (int rc = check_size("vocab", vocab, 1, kMaxVocab)) return rc;
    if (int rc = check_size("top", top, 0, kMaxTop)) return rc;
    phub::VocabArgs a{};
    a.type = type;
    a.rows = rows;
    a.cols = cols;
    a.vocab = vocab;
    a.x = x;
    a.x_stride = x_stride;
    a.w = w;
    a.w_stride = w_stride;
    a.top = top;
    // both gradients: what one alone takes is less
    a.dx = a.dw = reinterpret_cast<float*>(16);
    phub::vocab_bytes(a, grad != 0, least, best);
    return PHUB_OK;
}

int phub_vocab_loss(int type, int64_t rows, int64_t cols, int64_t vocab, const void* x,
                    int64_t x_stride, const void* w, int64_t w_stride, const int64_t* target,
                    float* loss_out, float* lse, void* workspace, int64_t workspace_bytes,
                    void* hip_stream) {
    phub::VocabArgs a{};
    a.type = type;
    a.rows = rows;
    a.cols = cols;
    a.vocab = vocab;
    a.x = x;
    a.x_stride = x_stride;
    a.w = w;
    a.w_stride = w_stride;
    a.target = target;
    a.temperature = 1.0f;
    a.loss = loss_out;
    a.lse = lse;
    return loss(a, workspace, workspace_bytes, hip_stream);
}

int phub_vocab_loss_grad(int type, int64_t rows, int64_t cols, int64_t vocab, const void* x,
                         int64_t x_stride, const void* w, int64_t w_stride, const int64_t* target,
                         const float* lse, const float* dloss, void* dx, int64_t dx_stride,
                         float* dw, int64_t dw_stride, int accumulate, void* workspace,
                         int64_t workspace_bytes, void* hip_stream) {
    phub::VocabArgs a{};
    a.type = type;
    a.rows = rows;
    a.cols = cols;
    a.vocab = vocab;
    a.x = x;
    a.x_stride = x_stride;
    a.w = w;
    a.w_stride = w_stride;
    a.target = target;
    a.temperature = 1.0f;
    a.lse = const_cast<float*>(lse);
    a.dloss = dloss;
    a.dx = dx;
    a.dx_stride = dx_stride;
    a.dw = dw;
    a.dw_stride = dw_stride;
    a.accumulate = accumulate != 0;
    return loss_grad(a, workspace, workspace_bytes, hip_stream);
}

int phub_distill_loss(int type, int64_t rows, int64_t cols, int64_t vocab, const void* x,
                      int64_t x_stride, const void* w, int64_t w_stride, int top,
                      const int64_t* index, const float* logit, float temperature, float* loss_out,
                      float* lse, void* workspace, int64_t workspace_bytes, void* hip_stream) {
    if (int rc = check_teacher(rows, top, temperature)) return rc;
    phub::VocabArgs a{};
    a.type = type;
    a.rows = rows;
    a.cols = cols;
    a.vocab = vocab;
    a.x = x;
    a.x_stride = x_stride;
    a.w = w;
    a.w_stride = w_stride;
    a.top = top;
    a.target = index;
    a.logit = logit;
    a.temperature = temperature;
    a.loss = loss_out;
    a.lse = lse;
    return loss(a, workspace, workspace_bytes, hip_stream);
}

int phub_distill_loss_grad(int type, int64_t rows, int64_t cols, int64_t vocab, const void* x,
                           int64_t x_stride, const void* w, int64_t w_stride, int top,
                           const int64_t* index, const float* logit, float temperature,
                           const float* lse, const float* dloss, void* dx, int64_t dx_stride,
                           float* dw, int64_t dw_stride, int accumulate, void* workspace,
                           int64_t workspace_bytes, void* hip_stream) {
    if (int rc = check_teacher(rows, top, temperature)) return rc;
    phub::VocabArgs a{};
    a.type = type;
    a.rows = rows;
    a.cols = cols;
    a.vocab = vocab;
    a.x = x;
    a.x_stride = x_stride;
    a.w = w;
    a.w_stride = w_stride;
    a.top = top;
    a.target = index;
    a.logit = logit;
    a.temperature = temperature;
    a.lse = const_cast<float*>(lse);
    a.dloss = dloss;
    a.dx = dx;
    a.dx_stride = dx_stride;
    a.dw = dw;
    a.dw_stride = dw_stride;
    a.accumulate = accumulate != 0;
    return loss_grad(a, workspace, workspace_bytes, hip_stream);
}
