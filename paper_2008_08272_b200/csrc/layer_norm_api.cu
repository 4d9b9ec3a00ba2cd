// C-ABI entries of layer normalisation: argument checks and the launches behind them.  Nothing here allocates device memory or synchronises.
#include <cuda_runtime.h>

#include <cmath>

#include "layer_norm.h"
#include "views.h"

using namespace onnxb;
using namespace onnxb::views;

namespace {

// One row of weights (or of their gradients) for rows of X
onnxb_status check_weights(const onnxb_matrix *w, const onnxb_matrix *X) {
    CHECK(check_view(w));
    if (w->type != X->type && w->type != ONNXB_FLOAT) return ONNXB_ERR_ATTR;
    return has_size(w, 1, X->cols) ? ONNXB_OK : ONNXB_ERR_SHAPE;
}
bool misaligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace

extern "C" onnxb_status onnx_layer_normalization_run(const onnxb_matrix *X, const onnxb_matrix *scale, const onnxb_matrix *bias, float epsilon,
                                                     const onnxb_matrix *Y, float *mean, float *inv_std, void *cuda_stream) {
    CHECK(check_view(X));
    CHECK(check_view(Y));
    if (!is_float_type(X->type) || Y->type != X->type || !std::isfinite(epsilon) || epsilon < 0.f) return ONNXB_ERR_ATTR;
    if (!has_size(Y, X->rows, X->cols)) return ONNXB_ERR_SHAPE;
    CHECK(check_weights(scale, X));
    if (bias) {
        CHECK(check_weights(bias, X));
        if (bias->type != scale->type) return ONNXB_ERR_ATTR;
    }
    if (X->rows == 0) return ONNXB_OK;
    if ((mean != nullptr) != (inv_std != nullptr)) return ONNXB_ERR_NULL;
    if (misaligned(mean) || misaligned(inv_std) || (mean && mean == inv_std)) return ONNXB_ERR_UNSUPPORTED;
    for (const onnxb_matrix *in : {X, scale, bias})
        if (same_place(Y, in)) return ONNXB_ERR_UNSUPPORTED;
    if (begins_at(mean, {X, Y, scale, bias}) || begins_at(inv_std, {X, Y, scale, bias})) return ONNXB_ERR_UNSUPPORTED;
    const LayerNormProblem p{X->type, scale->type, (int)X->rows, (int)X->cols, operand(X), operand(Y), scale->data, bias ? bias->data : nullptr,
                             epsilon, mean, inv_std};
    return status_of(launch_layer_norm(p, (cudaStream_t)cuda_stream));
}

extern "C" size_t onnx_layer_normalization_backward_workspace_bytes(const onnxb_matrix *X, const onnxb_matrix *dScale, const onnxb_matrix *dBias) {
    if (!X || X->rows < 1 || X->cols < 1 || X->rows > kMostSize || X->cols > kMostSize) return 0;
    return layer_norm_grad_workspace((int)X->rows, (int)X->cols, dScale || dBias);
}

extern "C" onnxb_status onnx_layer_normalization_backward_run(const onnxb_matrix *dY, const onnxb_matrix *X, const onnxb_matrix *scale,
                                                              const float *mean, const float *inv_std, const onnxb_matrix *dX,
                                                              const onnxb_matrix *dScale, const onnxb_matrix *dBias, void *workspace,
                                                              size_t workspace_bytes, void *cuda_stream) {
    if (!dX && !dScale && !dBias) return ONNXB_ERR_NULL;
    CHECK(check_view(dY));
    CHECK(check_view(X));
    if (!is_float_type(X->type) || dY->type != X->type) return ONNXB_ERR_ATTR;
    if (!has_size(dY, X->rows, X->cols)) return ONNXB_ERR_SHAPE;
    if (dX) {
        CHECK(check_view(dX));
        if (dX->type != X->type) return ONNXB_ERR_ATTR;
        if (!has_size(dX, X->rows, X->cols)) return ONNXB_ERR_SHAPE;
        if (!scale) return ONNXB_ERR_NULL;
    }
    const onnxb_matrix *weights[3] = {dX ? scale : nullptr, dScale, dBias}, *first = nullptr;
    for (const onnxb_matrix *w : weights) {
        if (!w) continue;
        CHECK(check_weights(w, X));
        if (first && w->type != first->type) return ONNXB_ERR_ATTR;
        if (!first) first = w;
    }
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (dScale && dBias && same_place(dScale, dBias)) return ONNXB_ERR_UNSUPPORTED;
    if (X->rows == 0) {
        // no rows: the weights' gradients are sums of nothing
        for (int i = 1; i < 3; ++i)
            if (weights[i] && cudaMemsetAsync(weights[i]->data, 0, (size_t)weights[i]->cols * type_bytes(weights[i]->type), stream) != cudaSuccess)
                return ONNXB_ERR_CUDA;
        return ONNXB_OK;
    }
    if (!mean || !inv_std) return ONNXB_ERR_NULL;
    if (misaligned(mean) || misaligned(inv_std)) return ONNXB_ERR_UNSUPPORTED;
    const onnxb_matrix *outs[3] = {dX, dScale, dBias};
    for (int i = 0; i < 3; ++i) {
        for (const onnxb_matrix *in : {dY, X, weights[0]})
            if (same_place(outs[i], in)) return ONNXB_ERR_UNSUPPORTED;
        if (i > 0 && same_place(outs[i], dX)) return ONNXB_ERR_UNSUPPORTED;
    }
    if (begins_at(mean, {dX, dScale, dBias}) || begins_at(inv_std, {dX, dScale, dBias})) return ONNXB_ERR_UNSUPPORTED;
    CHECK(check_workspace(workspace, workspace_bytes, onnx_layer_normalization_backward_workspace_bytes(X, dScale, dBias),
                          {dX, dScale, dBias, dY, X, weights[0]}));
    if (workspace && (workspace == mean || workspace == inv_std) && (dScale || dBias)) return ONNXB_ERR_UNSUPPORTED;
    const LayerNormGradProblem p{X->type, first ? first->type : X->type, (int)X->rows, (int)X->cols, operand(dY), operand(X),
                                 dX ? operand(dX) : DenseOperand{nullptr, 0}, dX ? scale->data : nullptr, mean, inv_std,
                                 dScale ? dScale->data : nullptr, dBias ? dBias->data : nullptr, workspace};
    return status_of(launch_layer_norm_grad(p, stream));
}
