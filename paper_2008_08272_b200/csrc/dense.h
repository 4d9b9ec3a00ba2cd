// Dense layers of 8- and 16-bit operands: the problem as the kernels take it (onnx_gemm_int8_run, onnx_gated_run and its
// gradients), and the kernels' host-side interface.
#pragma once
#include <cuda_runtime.h>

#include "common.h"

namespace onnxb {

// What is multiplied and what becomes of the sums.  "Rows" of an operand run along the output's rows (A) or columns (B); an operand is
// MN-major when they are the contiguous ones in memory, K-major when the reduction is.
enum DenseMode {
    kDensePlain = 0,     // Y[0] = A[0] B[0]^T, scaled
    kDenseGated = 1,     // G = A[0] B[0]^T, U = A[0] B[1]^T; Y[0] = act(G) U, Y[1] = G and Y[2] = U where they are kept
    kDenseGradX = 2,     // Y[0] = A[0] B[0] + A[1] B[1], B MN-major
    kDenseGradW = 3      // Y[z] = A[z]^T B[0], z = 0, 1 (of those that are not NULL), both MN-major
};

struct DenseOperand {
    const void *p;
    long long ld;        // elements between rows of the tensor as it is stored
};

struct DenseProblem {
    int mode;
    int type;            // of the operands
    int M, N, K;         // of one product
    DenseOperand A[2], B[2];
    const float *a_scale, *b_scale[2], *bias;      // 8-bit operands
    int relu, activation;
    int y_type;
    void *Y[3];
    long long y_ld[3];
};

inline int type_bytes(int type) { return type == ONNXB_FLOAT ? 4 : type == ONNXB_INT8 ? 1 : 2; }

// A product as its size asks for: by the kernel for a few tokens (dense_few.cu) or the one for many (tc_dense.cu).
int launch_dense(const DenseProblem &p, cudaStream_t stream);
bool dense_few_fits(const DenseProblem &p);
int launch_dense_few(const DenseProblem &p, cudaStream_t stream);
// On the tensor cores (tc_dense.cu).  Operands' rows begin at multiples of 16 bytes.
int launch_tc_dense(const DenseProblem &p, cudaStream_t stream);

// dG = dH U act'(G), dU = dH act(G), each [M,F]; all of one 16-bit type
struct GatedSlopeProblem {
    int type, activation, M, F;
    DenseOperand dH, G, U;
    void *dG, *dU;
    long long d_ld;
};
int launch_gated_slope(const GatedSlopeProblem &p, cudaStream_t stream);

int launch_quantize_rows(int type, int M, int K, const void *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream);

// dst[r] = the first row_bytes bytes of src's row r, rows dst_pitch apart (a multiple of 16, as dst is)
int launch_repack_rows(const void *src, long long src_pitch, int rows, long long row_bytes, void *dst, long long dst_pitch, cudaStream_t stream);

}  // namespace onnxb
