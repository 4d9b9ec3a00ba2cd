// Products whose weights go by the group (expert) that a row belongs to: the problem as the kernels take it (onnx_grouped_gemm_run,
// onnx_grouped_gated_run and their gradients).
#pragma once
#include <cuda_runtime.h>

#include "dense.h"

namespace onnxb {

constexpr int kMostGroups = 1024;

enum GroupedMode {
    kGroupedPlain = 0,   // Y[0][i] = A[0][i] W[0][g]^T for the rows i of group g
    kGroupedGated = 1,   // G = A[0] W[0][g]^T, U = A[0] W[1][g]^T; Y[0] = act(G) U, Y[1] = G and Y[2] = U where they are kept
    kGroupedGrad = 2     // dX = Y[0]: the sum over the terms t of A[t] W[t][g]; D[t][g] = A[t]^T X over the group's rows; those that are not NULL
};

struct GroupedWeights {
    const void *p;
    long long ld, stride;        // elements between rows, and from one group's to the next's
};

struct GroupedProblem {
    int mode, type;
    int rows, groups, channels, width;       // W [groups][channels][width]
    const int *offsets;                      // [groups + 1], device
    DenseOperand A[2], X;                    // X: of the gradients of the weights
    GroupedWeights W[2];
    int terms;                               // kGroupedGrad: 1, or 2 (the gated block's)
    int activation;
    void *Y[3];
    long long y_ld[3];
    GroupedWeights D[2];                     // (written)
    void *planes;                            // tc_grouped_workspace bytes, at a multiple of 16
};

// The forward products of a few rows (grouped_few.cu): of up to 16, or 128 where the weights would have to be copied.  Operands' rows and groups may begin anywhere.
// (in_place: the weights begin where the tensor cores' kernel can read them)
bool grouped_few_fits(int rows, int groups, int width, bool in_place);
int launch_grouped_few(const GroupedProblem &p, cudaStream_t stream);
// Scratch that launch_tc_grouped needs, by `mode`, `rows`, `groups`, `channels`, `width` and `terms` alone, for results by row (dX, or a forward product) and so many
// weights' gradients
size_t tc_grouped_workspace(const GroupedProblem &p, bool rows, int weights);
// On the tensor cores (tc_grouped.cu).  Operands' rows and groups begin at multiples of 16 bytes.
int launch_tc_grouped(const GroupedProblem &p, cudaStream_t stream);

}  // namespace onnxb
