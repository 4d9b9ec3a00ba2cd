// Dense layers of 8- and 16-bit operands: the problem as the kernels take it (onnx_gemm_int8_run, onnx_gated_run and its
// gradients), and the kernels' host-side interface.
#pragma once
#include <cuda_runtime.h>

#include "common.h"

namespace onnxb {

// What is multiplied and what becomes of the sums
enum DenseMode {
    kDensePlain = 0,     // Y[0] = A[0] B[0]^T, scaled
    kDenseGated = 1,     // G = A[0] B[0]^T, U = A[0] B[1]^T; Y[0] = act(G) U, Y[1] = G and Y[2] = U where they are kept
    kDenseGrad = 2       // dX = Y[0] = A[0] B[0] + A[1] B[1], dWg = Y[1] = A[0]^T B[2], dWu = Y[2] = A[1]^T B[2]; those that are not NULL
};

struct DenseOperand {
    const void *p;
    long long ld;        // elements between rows of the tensor as it is stored
};

struct GradChoice {      // tile shape, and parts of dX's reduction
    int ctas, BN, parts;
};

struct DenseProblem {
    int mode;
    int type;            // of the operands
    int M, N, K;         // tokens; columns of the results; the other size (of the gradients: channels)
    DenseOperand A[2], B[3];
    const float *a_scale, *b_scale[2], *bias;      // 8-bit operands
    int relu, activation;
    int y_type;
    void *Y[3];
    long long y_ld[3];
    GradChoice grad;     // kDenseGrad: tc_grad_choice's
    void *partial;       // tc_grad_workspace bytes
    // kDenseGrad of a few tokens: A[0] and A[1] hold every token twice, the 16-bit numbers nearest to dG and dU and, M/2 rows on, those nearest
    // to what these leave of them; B[2] holds X twice; Y[0] is the sum of both.  (M: rows of A)
    int twins;
};

inline int type_bytes(int type) { return type == ONNXB_FLOAT ? 4 : type == ONNXB_INT8 ? 1 : 2; }

// A product as its size asks for: by the kernel for a few tokens (dense_few.cu) or the one for many (tc_dense.cu).
int launch_dense(const DenseProblem &p, cudaStream_t stream);
bool dense_few_fits(const DenseProblem &p);
int launch_dense_few(const DenseProblem &p, cudaStream_t stream);
// On the tensor cores (tc_dense.cu).  Operands' rows begin at multiples of 16 bytes.
int launch_tc_dense(const DenseProblem &p, cudaStream_t stream);
// Scratch that the gradients' products need (dX in parts of its long reduction, where there would be few tiles)
GradChoice tc_grad_choice(int rows, int channels, int width, bool dX, int weights);
size_t tc_grad_workspace(const GradChoice &choice, int rows, int width, bool dX, bool twins);

// Y[i,j] = the sum over s < parts of P[s * part_rows + i][j], in that order, and of twins that of P[s * part_rows + M + i][j] after each finite
// one, rounded to `type`; P's rows p_ld floats apart (a multiple of 4)
struct SumPartsProblem {
    int parts, part_rows, M, N, type, twins;
    const float *P;
    long long p_ld;
    void *Y;
    long long y_ld;
};
int launch_sum_parts(const SumPartsProblem &p, cudaStream_t stream);

// dG = dH U act'(G), dU = dH act(G), each [M,F]; all of one 16-bit type.  twins: what rounding leaves of them as well, M rows on, and X [M,K]
// (its p NULL where there is none) copied to `twice`, and again M rows on, zeros there where it is not finite.
struct GatedSlopeProblem {
    int type, activation, M, F;
    DenseOperand dH, G, U;
    void *dG, *dU;
    long long d_ld;
    int twins, K;
    DenseOperand X;
    void *twice;
    long long twice_ld;
};
int launch_gated_slope(const GatedSlopeProblem &p, cudaStream_t stream);

int launch_quantize_rows(int type, int M, int K, const void *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream);

// Up to three tensors' rows laid out anew: dst's row r = the row_bytes bytes of src's, rows dst_pitch apart (a multiple of 16, as dst is)
struct RepackJob {
    const uint8_t *src;
    long long src_pitch, row_bytes;
    int rows, element;       // bytes of one
    uint8_t *dst;
    long long dst_pitch;
    int group_rows;          // src's rows lie in groups of so many, group_pitch apart (0: in one)
    long long group_pitch;
    const int *offsets;      // or NULL: groups whose next offset is not above their own are left out
};
struct RepackProblem {
    RepackJob job[3];
    int count;
};
int launch_repack_rows(const RepackProblem &p, cudaStream_t stream);

}  // namespace onnxb
