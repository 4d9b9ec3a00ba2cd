// Layer normalisation (onnx_layer_normalization_run and its gradients): the problem as the kernels take it.
#pragma once
#include <cuda_runtime.h>

#include "dense.h"

namespace onnxb {

struct LayerNormProblem {
    int type, weight_type;       // weight_type: `type` or ONNXB_FLOAT
    int M, K;
    DenseOperand X, Y;
    const void *scale, *bias;    // bias: may be NULL
    float epsilon;
    float *mean, *inv_std;       // both or neither
};
int launch_layer_norm(const LayerNormProblem &p, cudaStream_t stream);

struct LayerNormGradProblem {
    int type, weight_type;
    int M, K;
    DenseOperand dY, X, dX;      // dX.p: NULL where it is not wanted
    const void *scale;           // not read without dX
    const float *mean, *inv_std;
    void *d_scale, *d_bias;      // each may be NULL
    void *partial;               // layer_norm_grad_workspace bytes
};
size_t layer_norm_grad_workspace(int M, int K, bool weights);
int launch_layer_norm_grad(const LayerNormGradProblem &p, cudaStream_t stream);

}  // namespace onnxb
