// C-ABI entries of the dense layers of 8- and 16-bit operands: argument checks and the launches behind them.  Nothing here
// allocates device memory or synchronises.
#include <cuda_runtime.h>

#include <cstdint>
#include <initializer_list>

#include "dense.h"
#include "views.h"

using namespace onnxb;
using namespace onnxb::views;

namespace {

constexpr int64_t kMostInt8Terms = 131071;       // 131071 * 128 * 128 < 2^31

}  // namespace

extern "C" onnxb_status onnx_quantize_rows_run(const onnxb_matrix *X, const onnxb_matrix *Q, float *scale, void *cuda_stream) {
    CHECK(check_view(X));
    CHECK(check_view(Q));
    if (!is_float_type(X->type) || Q->type != ONNXB_INT8) return ONNXB_ERR_ATTR;
    if (!has_size(Q, X->rows, X->cols)) return ONNXB_ERR_SHAPE;
    if (X->rows == 0) return ONNXB_OK;
    if (!scale) return ONNXB_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(scale) % 4 || same_place(X, Q) || begins_at(scale, {X, Q})) return ONNXB_ERR_UNSUPPORTED;
    const DenseOperand x = operand(X), q = operand(Q);
    return status_of(launch_quantize_rows(X->type, (int)X->rows, (int)X->cols, x.p, x.ld, static_cast<int8_t *>(const_cast<void *>(q.p)), q.ld,
                                          scale, (cudaStream_t)cuda_stream));
}

extern "C" size_t onnx_gemm_int8_workspace_bytes(const onnxb_matrix *A, const onnxb_matrix *B) {
    return copy_bytes(A) + copy_bytes(B);
}

extern "C" onnxb_status onnx_gemm_int8_run(const onnxb_matrix *A, const float *a_scale, const onnxb_matrix *B, const float *b_scale, const float *C,
                                           int fuse_relu, const onnxb_matrix *Y, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    CHECK(check_view(A));
    CHECK(check_view(B));
    CHECK(check_view(Y));
    if (A->type != ONNXB_INT8 || B->type != ONNXB_INT8 || !is_float_type(Y->type)) return ONNXB_ERR_ATTR;
    const int64_t M = A->rows, K = A->cols, N = B->rows;
    if (N < 1 || B->cols != K || !has_size(Y, M, N)) return ONNXB_ERR_SHAPE;
    if (K > kMostInt8Terms) return ONNXB_ERR_UNSUPPORTED;
    if (M == 0) return ONNXB_OK;
    if (!a_scale || !b_scale) return ONNXB_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(a_scale) | reinterpret_cast<uintptr_t>(b_scale) | reinterpret_cast<uintptr_t>(C)) % 4) return ONNXB_ERR_UNSUPPORTED;
    if (same_place(Y, A) || same_place(Y, B) || begins_at(a_scale, {Y}) || begins_at(b_scale, {Y}) || begins_at(C, {Y})) return ONNXB_ERR_UNSUPPORTED;
    DenseProblem d{};
    d.mode = kDensePlain;
    d.type = ONNXB_INT8;
    d.M = (int)M; d.N = (int)N; d.K = (int)K;
    d.a_scale = a_scale; d.b_scale[0] = b_scale; d.bias = C; d.relu = fuse_relu != 0;
    d.y_type = Y->type;
    d.Y[0] = Y->data; d.y_ld[0] = operand(Y).ld;
    CHECK(check_workspace(workspace, workspace_bytes, onnx_gemm_int8_workspace_bytes(A, B), {A, B, Y}));
    Placement placed(workspace);
    d.A[0] = placed(A);
    d.B[0] = placed(B);
    d.K = placed.reduction(K, 2, ONNXB_INT8);
    const int err = placed.run((cudaStream_t)cuda_stream);
    return status_of(err ? err : launch_dense(d, (cudaStream_t)cuda_stream));
}

extern "C" size_t onnx_gated_workspace_bytes(const onnxb_matrix *X, const onnxb_matrix *Wg, const onnxb_matrix *Wu) {
    return copy_bytes(X) + copy_bytes(Wg) + copy_bytes(Wu);
}

// What both types of operands share; *done: there is nothing to compute.
static onnxb_status gated_problem(const onnxb_matrix *X, const onnxb_matrix *Wg, const onnxb_matrix *Wu, int activation, const onnxb_matrix *H,
                                  DenseProblem &d, bool &done) {
    CHECK(check_view(X));
    CHECK(check_view(Wg));
    CHECK(check_view(Wu));
    CHECK(check_view(H));
    if (Wg->type != X->type || Wu->type != X->type || activation < ONNXB_SILU || activation > ONNXB_RELU) return ONNXB_ERR_ATTR;
    const int64_t M = X->rows, K = X->cols, F = Wg->rows;
    if (F < 1 || Wg->cols != K || !has_size(Wu, F, K) || !has_size(H, M, F)) return ONNXB_ERR_SHAPE;
    if (same_place(H, X) || same_place(H, Wg) || same_place(H, Wu)) return ONNXB_ERR_UNSUPPORTED;
    done = M == 0;
    d = DenseProblem{};
    d.mode = kDenseGated;
    d.type = X->type;
    d.M = (int)M; d.N = (int)F; d.K = (int)K;
    d.activation = activation;
    d.y_type = H->type;
    d.Y[0] = H->data; d.y_ld[0] = operand(H).ld;
    return ONNXB_OK;
}

static onnxb_status run_gated(DenseProblem &d, const onnxb_matrix *X, const onnxb_matrix *Wg, const onnxb_matrix *Wu, const onnxb_matrix *H,
                              const onnxb_matrix *G, const onnxb_matrix *U, void *workspace, size_t workspace_bytes, cudaStream_t stream) {
    CHECK(check_workspace(workspace, workspace_bytes, onnx_gated_workspace_bytes(X, Wg, Wu), {X, Wg, Wu, H, G, U}));
    Placement placed(workspace);
    d.A[0] = placed(X);
    d.B[0] = placed(Wg);
    d.B[1] = placed(Wu);
    d.K = placed.reduction(X->cols, 3, X->type);
    const int err = placed.run(stream);
    return status_of(err ? err : launch_dense(d, stream));
}

extern "C" onnxb_status onnx_gated_run(const onnxb_matrix *X, const onnxb_matrix *Wg, const onnxb_matrix *Wu, int activation, const onnxb_matrix *H,
                                       const onnxb_matrix *G, const onnxb_matrix *U, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    DenseProblem d;
    bool done = false;
    CHECK(gated_problem(X, Wg, Wu, activation, H, d, done));
    if (!is_float16_type(X->type) || H->type != X->type) return ONNXB_ERR_ATTR;
    if ((G != nullptr) != (U != nullptr)) return ONNXB_ERR_NULL;
    if (G) {
        CHECK(check_view(G));
        CHECK(check_view(U));
        if (G->type != X->type || U->type != X->type) return ONNXB_ERR_ATTR;
        if (!has_size(G, H->rows, H->cols) || !has_size(U, H->rows, H->cols)) return ONNXB_ERR_SHAPE;
        if (same_place(G, U) || same_place(G, H) || same_place(U, H)) return ONNXB_ERR_UNSUPPORTED;
        for (const onnxb_matrix *in : {X, Wg, Wu})
            if (same_place(G, in) || same_place(U, in)) return ONNXB_ERR_UNSUPPORTED;
        d.Y[1] = G->data; d.y_ld[1] = operand(G).ld;
        d.Y[2] = U->data; d.y_ld[2] = operand(U).ld;
    }
    if (done) return ONNXB_OK;
    return run_gated(d, X, Wg, Wu, H, G, U, workspace, workspace_bytes, (cudaStream_t)cuda_stream);
}

extern "C" onnxb_status onnx_gated_int8_run(const onnxb_matrix *A, const float *a_scale, const onnxb_matrix *Wg, const float *g_scale,
                                            const onnxb_matrix *Wu, const float *u_scale, int activation, const onnxb_matrix *H, void *workspace,
                                            size_t workspace_bytes, void *cuda_stream) {
    DenseProblem d;
    bool done = false;
    CHECK(gated_problem(A, Wg, Wu, activation, H, d, done));
    if (A->type != ONNXB_INT8 || !is_float_type(H->type)) return ONNXB_ERR_ATTR;
    if (A->cols > kMostInt8Terms) return ONNXB_ERR_UNSUPPORTED;
    if (done) return ONNXB_OK;
    if (!a_scale || !g_scale || !u_scale) return ONNXB_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(a_scale) | reinterpret_cast<uintptr_t>(g_scale) | reinterpret_cast<uintptr_t>(u_scale)) % 4) return ONNXB_ERR_UNSUPPORTED;
    if (begins_at(a_scale, {H}) || begins_at(g_scale, {H}) || begins_at(u_scale, {H})) return ONNXB_ERR_UNSUPPORTED;
    d.a_scale = a_scale; d.b_scale[0] = g_scale; d.b_scale[1] = u_scale;
    return run_gated(d, A, Wg, Wu, H, nullptr, nullptr, workspace, workspace_bytes, (cudaStream_t)cuda_stream);
}

// The gradients' workspace: dG and dU, their rows at multiples of 16 bytes; for few tokens all of these rows twice, and X twice.
// Rounding dG and dU to 16 bits makes the gradients' error 1.4 times that of rounding them alone, but of single tokens up to twice it,
// since so few roundings do not average.  Up to kMostTwins tokens what is left of them goes along as tokens of its own: the tensor
// cores have room for these rows anyway (64 of a K block, 128 of a tile), and what it costs is dX's sum of both in a launch of its own
// (16 tokens, 4096 x 10240: 73.7 -> 75.3 us; one, 64 x 64: 3.7 -> 4.9).
constexpr int64_t kMostTwins = 32;
static int64_t padded_pitch(int64_t cols) { return (cols + 7) / 8 * 8; }
static bool has_twins(int64_t M) { return M <= kMostTwins; }
static int64_t slope_rows(int64_t M) { return has_twins(M) ? 2 * M : M; }
static size_t slope_bytes(int64_t M, int64_t F) { return (size_t)(slope_rows(M) * padded_pitch(F) * 2); }
// X for dWg and dWu
static size_t tokens_bytes(const onnxb_matrix *X) {
    if (!X || X->rows < 1 || X->cols < 1 || X->rows > kMostSize || X->cols > kMostSize) return 0;
    return has_twins(X->rows) ? slope_bytes(X->rows, X->cols) : copy_bytes(X);
}

static size_t backward_bytes(const onnxb_matrix *dH, const onnxb_matrix *X, const onnxb_matrix *Wg, const onnxb_matrix *Wu, const onnxb_matrix *dX,
                             const onnxb_matrix *dWg, const onnxb_matrix *dWu, GradChoice &choice) {
    if (!dH || dH->rows < 1 || dH->cols < 1 || dH->rows > kMostSize || dH->cols > kMostSize) return 0;
    const onnxb_matrix *one = dX ? dX : dWg ? dWg : dWu;
    if (!one || one->cols < 1 || one->cols > kMostSize) return 0;
    const int rows = (int)slope_rows(dH->rows), width = (int)one->cols;
    choice = tc_grad_choice(rows, (int)dH->cols, width, dX != nullptr, (dWg != nullptr) + (dWu != nullptr));
    return 2 * slope_bytes(dH->rows, dH->cols) + (dX ? copy_bytes(Wg) + copy_bytes(Wu) : 0) + (dWg || dWu ? tokens_bytes(X) : 0) +
           tc_grad_workspace(choice, rows, width, dX != nullptr, has_twins(dH->rows));
}

extern "C" size_t onnx_gated_backward_workspace_bytes(const onnxb_matrix *dH, const onnxb_matrix *X, const onnxb_matrix *Wg, const onnxb_matrix *Wu,
                                                      const onnxb_matrix *dX, const onnxb_matrix *dWg, const onnxb_matrix *dWu) {
    GradChoice choice;
    return backward_bytes(dH, X, Wg, Wu, dX, dWg, dWu, choice);
}

extern "C" onnxb_status onnx_gated_backward_run(const onnxb_matrix *dH, const onnxb_matrix *X, const onnxb_matrix *Wg, const onnxb_matrix *Wu,
                                                const onnxb_matrix *G, const onnxb_matrix *U, int activation, const onnxb_matrix *dX,
                                                const onnxb_matrix *dWg, const onnxb_matrix *dWu, void *workspace, size_t workspace_bytes,
                                                void *cuda_stream) {
    const bool weights = dWg || dWu;
    if (!dX && !weights) return ONNXB_ERR_NULL;
    CHECK(check_view(dH));
    CHECK(check_view(G));
    CHECK(check_view(U));
    const int64_t M = dH->rows, F = dH->cols;
    int64_t K = 0;
    const onnxb_matrix *outs[3] = {dX, dWg, dWu};
    if (!is_float16_type(dH->type) || activation < ONNXB_SILU || activation > ONNXB_RELU) return ONNXB_ERR_ATTR;
    if (G->type != dH->type || U->type != dH->type) return ONNXB_ERR_ATTR;
    if (!has_size(G, M, F) || !has_size(U, M, F)) return ONNXB_ERR_SHAPE;
    // the width, from the first result; all else is compared with it
    K = dX ? dX->cols : dWg ? dWg->cols : dWu->cols;
    const onnxb_matrix *ins[3] = {weights ? X : nullptr, dX ? Wg : nullptr, dX ? Wu : nullptr};
    if ((weights && !X) || (dX && (!Wg || !Wu))) return ONNXB_ERR_NULL;
    for (int i = 0; i < 3; ++i)
        for (const onnxb_matrix *m : {ins[i], outs[i]}) {
            if (!m) continue;
            CHECK(check_view(m));
            if (m->type != dH->type) return ONNXB_ERR_ATTR;
            if (!has_size(m, i == 0 ? M : F, K)) return ONNXB_ERR_SHAPE;
        }
    const onnxb_matrix *all[9] = {dX, dWg, dWu, dH, G, U, ins[0], ins[1], ins[2]};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 9; ++j)
            if (same_place(all[i], all[j])) return ONNXB_ERR_UNSUPPORTED;

    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (M == 0) {
        // no tokens: the weights' gradients are sums of nothing
        for (int i = 1; i < 3; ++i)
            if (outs[i] && cudaMemset2DAsync(outs[i]->data, (size_t)operand(outs[i]).ld * 2, 0, (size_t)K * 2, (size_t)F, stream) != cudaSuccess)
                return ONNXB_ERR_CUDA;
        return ONNXB_OK;
    }
    DenseProblem d{};
    CHECK(check_workspace(workspace, workspace_bytes, backward_bytes(dH, X, Wg, Wu, dX, dWg, dWu, d.grad),
                          {dX, dWg, dWu, dH, G, U, ins[0], ins[1], ins[2]}));
    GatedSlopeProblem s{};
    s.type = dH->type; s.activation = activation;
    s.M = (int)M; s.F = (int)F;
    s.dH = operand(dH); s.G = operand(G); s.U = operand(U);
    s.d_ld = padded_pitch(F);
    char *ws = static_cast<char *>(workspace);
    s.dG = ws;
    s.dU = ws + slope_bytes(M, F);
    ws += 2 * slope_bytes(M, F);
    s.twins = has_twins(M);
    s.K = (int)K;
    if (s.twins && weights) {
        s.X = operand(X);
        s.twice = ws;
        s.twice_ld = padded_pitch(K);
        ws += tokens_bytes(X);
    }
    int err = launch_gated_slope(s, stream);
    d.mode = kDenseGrad;
    d.type = d.y_type = dH->type;
    d.M = (int)slope_rows(M); d.N = (int)K; d.K = (int)F;
    d.twins = s.twins;
    d.A[0] = DenseOperand{s.dG, s.d_ld};
    d.A[1] = DenseOperand{s.dU, s.d_ld};
    Placement placed(ws);
    if (dX) {
        d.B[0] = placed(Wg);
        d.B[1] = placed(Wu);
    }
    if (weights) d.B[2] = s.twins ? DenseOperand{s.twice, s.twice_ld} : placed(X);
    if (err == 0) err = placed.run(stream);
    for (int i = 0; i < 3; ++i) {
        d.Y[i] = outs[i] ? outs[i]->data : nullptr;
        d.y_ld[i] = outs[i] ? operand(outs[i]).ld : 0;
    }
    d.partial = placed.workspace;
    return status_of(err ? err : launch_tc_dense(d, stream));
}
