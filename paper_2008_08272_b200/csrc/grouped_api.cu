// C-ABI entries of the products whose weights go by the row's group: argument checks and the launches behind them.  Nothing here allocates device
// memory or synchronises.
#include <cuda_runtime.h>

#include "grouped.h"
#include "views.h"

using namespace onnxb;
using namespace onnxb::views;

namespace {

constexpr int64_t kMostStride = 1ll << 36, kMostRows = 2147483647ll;
// Terms of a reduction on the tensor cores, whose waits are bounded: a tile of so many takes a second at most
constexpr int64_t kMostTerms = 1ll << 27;

// What holds for groups' weights by themselves: sizes, no rows that overlap, in whichever order they lie
onnxb_status check_groups(const onnxb_matrices *m) {
    if (!m) return ONNXB_ERR_NULL;
    if (m->reserved != 0 || !is_float16_type(m->type)) return ONNXB_ERR_ATTR;
    if (m->count < 1 || m->rows < 1 || m->cols < 1 || (m->rows > 1 && m->ld < m->cols)) return ONNXB_ERR_SHAPE;
    if (m->count > kMostGroups || m->rows > kMostSize || m->cols > kMostSize || m->count * m->rows > kMostRows) return ONNXB_ERR_UNSUPPORTED;
    const int64_t ld = m->rows > 1 ? m->ld : m->cols;
    if (m->rows > 1 && ld > kMostPitch) return ONNXB_ERR_UNSUPPORTED;
    if (m->count > 1) {
        if (m->stride > kMostStride) return ONNXB_ERR_UNSUPPORTED;
        const bool after = m->stride >= (m->rows - 1) * ld + m->cols, between = m->stride >= m->cols && ld >= (m->count - 1) * m->stride + m->cols;
        if (m->stride < 1 || !(after || (between && m->rows > 1))) return ONNXB_ERR_SHAPE;
    }
    if (!m->data) return ONNXB_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(m->data) % 2) return ONNXB_ERR_UNSUPPORTED;
    return ONNXB_OK;
}
bool has_size(const onnxb_matrices *m, int64_t count, int64_t rows, int64_t cols) { return m->count == count && m->rows == rows && m->cols == cols; }
GroupedWeights weights(const onnxb_matrices *m) {
    const long long ld = m->rows > 1 ? (long long)m->ld : (long long)m->cols;
    return GroupedWeights{m->data, ld, m->count > 1 ? (long long)m->stride : ld * (long long)m->rows};
}
bool in_place(const onnxb_matrices *m) {
    return reinterpret_cast<uintptr_t>(m->data) % 16 == 0 && (m->rows <= 1 || m->ld % 8 == 0) && (m->count <= 1 || m->stride % 8 == 0);
}
int64_t copy_pitch(const onnxb_matrices *m) { return (m->cols * 2 + 127) / 128 * 128; }
size_t copy_bytes(const onnxb_matrices *m) {
    if (!m || m->count < 1 || m->count > kMostGroups || m->rows < 1 || m->cols < 1 || m->rows > kMostSize || m->cols > kMostSize || in_place(m)) return 0;
    return (size_t)(copy_pitch(m) * m->rows * m->count);
}
// Groups' weights as the kernels read them: where they lie, or copied to the workspace with the other operands
GroupedWeights place(Placement &placed, const onnxb_matrices *m, const int32_t *offsets) {
    const size_t bytes = copy_bytes(m);
    const GroupedWeights w = weights(m);
    if (bytes == 0) return w;
    placed.repack.job[placed.repack.count++] = RepackJob{static_cast<const uint8_t *>(m->data), w.ld * 2, m->cols * 2, (int)(m->count * m->rows), 2,
                                                         reinterpret_cast<uint8_t *>(placed.workspace), copy_pitch(m), (int)m->rows, w.stride * 2, offsets};
    const GroupedWeights copy{placed.workspace, copy_pitch(m) / 2, copy_pitch(m) / 2 * m->rows};
    placed.workspace += bytes;
    return copy;
}

bool same_place(const void *a, const void *b) { return a && a == b; }
const void *data_of(const onnxb_matrix *m) { return m && m->rows > 0 ? m->data : nullptr; }
const void *data_of(const onnxb_matrices *m) { return m ? m->data : nullptr; }
// Outputs (the first `outs` of `all`) in a place of their own; the workspace, where there is one, too
onnxb_status check_places(const void *const *all, int outs, int count, const void *workspace, size_t need) {
    for (int i = 0; i < outs; ++i)
        for (int j = i + 1; j < count; ++j)
            if (same_place(all[i], all[j])) return ONNXB_ERR_UNSUPPORTED;
    for (int i = 0; need && i < count; ++i)
        if (same_place(workspace, all[i])) return ONNXB_ERR_UNSUPPORTED;
    return ONNXB_OK;
}
onnxb_status check_offsets(const int32_t *offsets) {
    if (!offsets) return ONNXB_ERR_NULL;
    return reinterpret_cast<uintptr_t>(offsets) % 4 ? ONNXB_ERR_UNSUPPORTED : ONNXB_OK;
}
onnxb_status check_space(const void *workspace, size_t bytes, size_t need) { return check_workspace(workspace, bytes, need, {}); }

}  // namespace

static bool sizes_are_some(const onnxb_matrix *m) { return m && m->rows >= 1 && m->cols >= 1 && m->rows <= kMostSize && m->cols <= kMostSize; }
// (few rows are taken from wherever they and the weights begin: grouped_few_fits says how many)
static bool few(const onnxb_matrix *X, const onnxb_matrices *Wg, const onnxb_matrices *Wu) {
    if (!sizes_are_some(X) || !Wg || Wg->count < 1 || Wg->count > kMostGroups) return false;
    return grouped_few_fits((int)X->rows, (int)Wg->count, (int)X->cols, in_place(Wg) && (!Wu || in_place(Wu)));
}
// The reductions' parts (from the sizes alone)
static GroupedProblem sizes_of(int mode, const onnxb_matrix *rows, int64_t channels, int64_t width, int64_t groups, int terms) {
    GroupedProblem d{};
    d.mode = mode;
    d.rows = (int)rows->rows; d.groups = (int)groups; d.channels = (int)channels; d.width = (int)width;
    d.terms = terms;
    return d;
}
static bool groups_are_some(const onnxb_matrices *m) { return m && m->count >= 1 && m->count <= kMostGroups && m->rows >= 1 && m->rows <= kMostSize && m->cols >= 1 && m->cols <= kMostSize; }
extern "C" size_t onnx_grouped_gemm_workspace_bytes(const onnxb_matrix *X, const onnxb_matrices *W) {
    if (!sizes_are_some(X) || !groups_are_some(W) || few(X, W, nullptr)) return 0;
    return views::copy_bytes(X) + copy_bytes(W) + tc_grouped_workspace(sizes_of(kGroupedPlain, X, W->rows, W->cols, W->count, 0), true, 0);
}
extern "C" size_t onnx_grouped_gated_workspace_bytes(const onnxb_matrix *X, const onnxb_matrices *Wg, const onnxb_matrices *Wu) {
    if (!sizes_are_some(X) || !groups_are_some(Wg) || few(X, Wg, Wu)) return 0;
    return views::copy_bytes(X) + copy_bytes(Wg) + copy_bytes(Wu) + tc_grouped_workspace(sizes_of(kGroupedGated, X, Wg->rows, Wg->cols, Wg->count, 0), true, 0);
}

// Both forward products: Wu NULL for the plain one
static onnxb_status forward(const onnxb_matrix *X, const onnxb_matrices *Wg, const onnxb_matrices *Wu, bool gated, const int32_t *offsets, int activation,
                            const onnxb_matrix *H, const onnxb_matrix *G, const onnxb_matrix *U, void *workspace, size_t workspace_bytes, cudaStream_t stream) {
    CHECK(check_view(X));
    CHECK(check_groups(Wg));
    if (gated) CHECK(check_groups(Wu));
    CHECK(check_view(H));
    if (!is_float16_type(X->type) || Wg->type != X->type || (gated && Wu->type != X->type) || H->type != X->type) return ONNXB_ERR_ATTR;
    if (activation < ONNXB_SILU || activation > ONNXB_RELU) return ONNXB_ERR_ATTR;
    const int64_t R = X->rows, K = X->cols, N = Wg->rows, groups = Wg->count;
    if (Wg->cols != K || (gated && !has_size(Wu, groups, N, K)) || !views::has_size(H, R, N)) return ONNXB_ERR_SHAPE;
    if ((G != nullptr) != (U != nullptr)) return ONNXB_ERR_NULL;
    if (G) {
        CHECK(check_view(G));
        CHECK(check_view(U));
        if (G->type != X->type || U->type != X->type) return ONNXB_ERR_ATTR;
        if (!views::has_size(G, R, N) || !views::has_size(U, R, N)) return ONNXB_ERR_SHAPE;
    }
    CHECK(check_offsets(offsets));
    if (R == 0) return ONNXB_OK;
    if (!few(X, Wg, Wu) && K > kMostTerms) return ONNXB_ERR_UNSUPPORTED;
    const size_t need = gated ? onnx_grouped_gated_workspace_bytes(X, Wg, Wu) : onnx_grouped_gemm_workspace_bytes(X, Wg);
    CHECK(check_space(workspace, workspace_bytes, need));
    const void *all[7] = {data_of(H), data_of(G), data_of(U), data_of(X), data_of(Wg), data_of(Wu), offsets};
    CHECK(check_places(all, 3, 7, workspace, need));
    GroupedProblem d{};
    d.mode = gated ? kGroupedGated : kGroupedPlain;
    d.type = X->type;
    d.rows = (int)R; d.groups = (int)groups; d.channels = (int)N; d.width = (int)K;
    d.offsets = offsets;
    d.activation = activation;
    const onnxb_matrix *outs[3] = {H, G, U};
    for (int i = 0; i < 3 && outs[i]; ++i) { d.Y[i] = outs[i]->data; d.y_ld[i] = operand(outs[i]).ld; }
    if (few(X, Wg, Wu)) {
        d.A[0] = operand(X);
        d.W[0] = weights(Wg);
        if (gated) d.W[1] = weights(Wu);
        return status_of(launch_grouped_few(d, stream));
    }
    Placement placed(workspace);
    d.A[0] = placed(X);
    d.W[0] = place(placed, Wg, offsets);
    if (gated) d.W[1] = place(placed, Wu, offsets);
    d.planes = placed.workspace;
    const int err = placed.run(stream);
    return status_of(err ? err : launch_tc_grouped(d, stream));
}

extern "C" onnxb_status onnx_grouped_gemm_run(const onnxb_matrix *X, const onnxb_matrices *W, const int32_t *offsets, const onnxb_matrix *Y, void *workspace,
                                              size_t workspace_bytes, void *cuda_stream) {
    return forward(X, W, nullptr, false, offsets, ONNXB_SILU, Y, nullptr, nullptr, workspace, workspace_bytes, (cudaStream_t)cuda_stream);
}
extern "C" onnxb_status onnx_grouped_gated_run(const onnxb_matrix *X, const onnxb_matrices *Wg, const onnxb_matrices *Wu, const int32_t *offsets, int activation,
                                               const onnxb_matrix *H, const onnxb_matrix *G, const onnxb_matrix *U, void *workspace, size_t workspace_bytes,
                                               void *cuda_stream) {
    return forward(X, Wg, Wu, true, offsets, activation, H, G, U, workspace, workspace_bytes, (cudaStream_t)cuda_stream);
}

// dG and dU: rows at multiples of 16 bytes
static int64_t slope_pitch(int64_t channels) { return (channels + 7) / 8 * 8; }
static size_t slope_bytes(int64_t rows, int64_t channels) { return (size_t)(rows * slope_pitch(channels) * 2); }
// What the gradients' products need: the width and the groups, from the first result or weights that have them
static size_t planes_bytes(const onnxb_matrix *dY, const onnxb_matrices *const *W, const onnxb_matrix *dX, const onnxb_matrices *const *D, int terms) {
    const onnxb_matrices *one = dX ? W[0] : D[0] ? D[0] : D[1];
    if (!sizes_are_some(dY) || !groups_are_some(one)) return 0;
    return tc_grouped_workspace(sizes_of(kGroupedGrad, dY, dY->cols, one->cols, one->count, terms), dX != nullptr, (D[0] != nullptr) + (D[1] != nullptr));
}

extern "C" size_t onnx_grouped_gemm_backward_workspace_bytes(const onnxb_matrix *dY, const onnxb_matrix *X, const onnxb_matrices *W, const onnxb_matrix *dX,
                                                             const onnxb_matrices *dW) {
    const onnxb_matrices *w[2] = {W, nullptr}, *d[2] = {dW, nullptr};
    return views::copy_bytes(dY) + (dW ? views::copy_bytes(X) : 0) + (dX ? copy_bytes(W) : 0) + planes_bytes(dY, w, dX, d, 1);
}
extern "C" size_t onnx_grouped_gated_backward_workspace_bytes(const onnxb_matrix *dH, const onnxb_matrix *X, const onnxb_matrices *Wg, const onnxb_matrices *Wu,
                                                              const onnxb_matrix *dX, const onnxb_matrices *dWg, const onnxb_matrices *dWu) {
    if (!sizes_are_some(dH)) return 0;
    const onnxb_matrices *w[2] = {Wg, Wu}, *d[2] = {dWg, dWu};
    return 2 * slope_bytes(dH->rows, dH->cols) + (dWg || dWu ? views::copy_bytes(X) : 0) + (dX ? copy_bytes(Wg) + copy_bytes(Wu) : 0) + planes_bytes(dH, w, dX, d, 2);
}

// Both forms' gradients: of the plain product G and U are NULL, and W[1] and D[1].  `gated` says which.
static onnxb_status backward(const onnxb_matrix *dY, const onnxb_matrix *X, const onnxb_matrices *const *W, bool gated, const onnxb_matrix *G,
                             const onnxb_matrix *U, const int32_t *offsets, int activation, const onnxb_matrix *dX, const onnxb_matrices *const *D,
                             void *workspace, size_t workspace_bytes, size_t need, cudaStream_t stream) {
    const bool of_weights = D[0] || D[1];
    const int terms = gated ? 2 : 1;
    if (!dX && !of_weights) return ONNXB_ERR_NULL;
    CHECK(check_view(dY));
    if (!is_float16_type(dY->type) || activation < ONNXB_SILU || activation > ONNXB_RELU) return ONNXB_ERR_ATTR;
    const int64_t R = dY->rows, N = dY->cols;
    for (const onnxb_matrix *m : {G, U}) {
        if (!gated) break;
        CHECK(check_view(m));
        if (m->type != dY->type) return ONNXB_ERR_ATTR;
        if (!views::has_size(m, R, N)) return ONNXB_ERR_SHAPE;
    }
    if (of_weights && !X) return ONNXB_ERR_NULL;
    for (int i = 0; dX && i < terms; ++i)
        if (!W[i]) return ONNXB_ERR_NULL;
    // the width and the groups, from the first that has them; all else is compared with them
    const onnxb_matrices *first = dX ? W[0] : D[0] ? D[0] : D[1];
    CHECK(check_groups(first));
    const int64_t K = first->cols, groups = first->count;
    for (const onnxb_matrix *m : {dX, of_weights ? X : nullptr}) {
        if (!m) continue;
        CHECK(check_view(m));
        if (m->type != dY->type) return ONNXB_ERR_ATTR;
        if (!views::has_size(m, R, K)) return ONNXB_ERR_SHAPE;
    }
    for (int i = 0; i < terms; ++i)
        for (const onnxb_matrices *m : {dX ? W[i] : nullptr, D[i]}) {
            if (!m) continue;
            CHECK(check_groups(m));
            if (m->type != dY->type) return ONNXB_ERR_ATTR;
            if (!has_size(m, groups, N, K)) return ONNXB_ERR_SHAPE;
        }
    CHECK(check_offsets(offsets));
    const void *all[10] = {data_of(dX), data_of(D[0]), data_of(D[1]), data_of(dY), gated ? data_of(G) : nullptr, gated ? data_of(U) : nullptr,
                           of_weights ? data_of(X) : nullptr, dX ? data_of(W[0]) : nullptr, dX && gated ? data_of(W[1]) : nullptr, offsets};
    if (R == 0) {
        CHECK(check_places(all, 3, 10, nullptr, 0));
        // no rows: the weights' gradients are sums of nothing
        for (int i = 0; i < terms; ++i)
            for (int64_t g = 0; D[i] && g < groups; ++g) {
                const GroupedWeights w = weights(D[i]);
                if (cudaMemset2DAsync(static_cast<uint16_t *>(const_cast<void *>(w.p)) + g * w.stride, (size_t)w.ld * 2, 0, (size_t)K * 2, (size_t)N, stream) != cudaSuccess)
                    return ONNXB_ERR_CUDA;
            }
        return ONNXB_OK;
    }
    if ((of_weights && R > kMostTerms) || (dX && N > kMostTerms)) return ONNXB_ERR_UNSUPPORTED;
    CHECK(check_space(workspace, workspace_bytes, need));
    CHECK(check_places(all, 3, 10, workspace, need));
    GroupedProblem d{};
    d.mode = kGroupedGrad;
    d.type = dY->type;
    d.rows = (int)R; d.groups = (int)groups; d.channels = (int)N; d.width = (int)K;
    d.offsets = offsets;
    d.terms = terms;
    char *ws = static_cast<char *>(workspace);
    int err = 0;
    if (gated) {
        // dG and dU are rounded to 16 bits, as the tensor cores take them: the results' error is 1.4 times that of rounding the results alone (bf16 2.3e-3 instead of
        // 1.7e-3 in the norm).  What rounding leaves of them as rows of their own (as the dense block has of up to 32 tokens) would be twice the products.
        GatedSlopeProblem s{};
        s.type = dY->type; s.activation = activation;
        s.M = (int)R; s.F = (int)N;
        s.dH = operand(dY); s.G = operand(G); s.U = operand(U);
        s.d_ld = slope_pitch(N);
        s.dG = ws;
        s.dU = ws + slope_bytes(R, N);
        ws += 2 * slope_bytes(R, N);
        err = launch_gated_slope(s, stream);
        d.A[0] = DenseOperand{s.dG, s.d_ld};
        d.A[1] = DenseOperand{s.dU, s.d_ld};
    }
    Placement placed(ws);
    if (!gated) d.A[0] = placed(dY);
    if (of_weights) d.X = placed(X);
    for (int i = 0; i < terms; ++i) {
        if (dX) d.W[i] = place(placed, W[i], offsets);
        if (D[i]) d.D[i] = weights(D[i]);
    }
    if (dX) { d.Y[0] = dX->data; d.y_ld[0] = operand(dX).ld; }
    d.planes = placed.workspace;
    if (err == 0) err = placed.run(stream);
    return status_of(err ? err : launch_tc_grouped(d, stream));
}

extern "C" onnxb_status onnx_grouped_gemm_backward_run(const onnxb_matrix *dY, const onnxb_matrix *X, const onnxb_matrices *W, const int32_t *offsets,
                                                       const onnxb_matrix *dX, const onnxb_matrices *dW, void *workspace, size_t workspace_bytes,
                                                       void *cuda_stream) {
    const onnxb_matrices *w[2] = {W, nullptr}, *d[2] = {dW, nullptr};
    return backward(dY, X, w, false, nullptr, nullptr, offsets, ONNXB_SILU, dX, d, workspace, workspace_bytes,
                    onnx_grouped_gemm_backward_workspace_bytes(dY, X, W, dX, dW), (cudaStream_t)cuda_stream);
}
extern "C" onnxb_status onnx_grouped_gated_backward_run(const onnxb_matrix *dH, const onnxb_matrix *X, const onnxb_matrices *Wg, const onnxb_matrices *Wu,
                                                        const onnxb_matrix *G, const onnxb_matrix *U, const int32_t *offsets, int activation,
                                                        const onnxb_matrix *dX, const onnxb_matrices *dWg, const onnxb_matrices *dWu, void *workspace,
                                                        size_t workspace_bytes, void *cuda_stream) {
    const onnxb_matrices *w[2] = {Wg, Wu}, *d[2] = {dWg, dWu};
    return backward(dH, X, w, true, G, U, offsets, activation, dX, d, workspace, workspace_bytes,
                    onnx_grouped_gated_backward_workspace_bytes(dH, X, Wg, Wu, dX, dWg, dWu), (cudaStream_t)cuda_stream);
}
