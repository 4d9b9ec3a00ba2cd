// Host side of the operators whose tensors are views (onnxb_matrix, onnxb_matrices): the checks that hold for a view by itself, and operands as
// TMA can address them, where they lie or copied to the workspace.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <initializer_list>

#include "dense.h"

namespace onnxb {
namespace views {

constexpr int64_t kMostSize = 1ll << 30, kMostPitch = 2147483647ll;

inline bool is_float16_type(int t) { return t == ONNXB_FLOAT16 || t == ONNXB_BFLOAT16; }
inline bool is_float_type(int t) { return t == ONNXB_FLOAT || is_float16_type(t); }

// What holds for a view by itself.  An empty one has no data to point at.
inline onnxb_status check_view(const onnxb_matrix *m) {
    if (!m) return ONNXB_ERR_NULL;
    if (m->reserved != 0 || !(m->type == ONNXB_INT8 || is_float_type(m->type))) return ONNXB_ERR_ATTR;
    if (m->rows < 0 || m->cols < 1 || (m->rows > 1 && m->ld < m->cols)) return ONNXB_ERR_SHAPE;
    if (m->rows > kMostSize || m->cols > kMostSize || (m->rows > 1 && m->ld > kMostPitch)) return ONNXB_ERR_UNSUPPORTED;
    if (!m->data && m->rows > 0) return ONNXB_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(m->data) % type_bytes(m->type)) return ONNXB_ERR_UNSUPPORTED;
    return ONNXB_OK;
}
inline bool has_size(const onnxb_matrix *m, int64_t rows, int64_t cols) { return m->rows == rows && m->cols == cols; }
// (a single row has no pitch: its own length stands for it)
inline DenseOperand operand(const onnxb_matrix *m) { return DenseOperand{m->data, m->rows > 1 ? (long long)m->ld : (long long)m->cols}; }
inline bool same_place(const onnxb_matrix *a, const onnxb_matrix *b) { return a && b && a->rows > 0 && a->data == b->data; }
// Whether a vector (or NULL), or the workspace, begins where a view does that has rows
inline bool begins_at(const void *p, std::initializer_list<const onnxb_matrix *> views) {
    for (const onnxb_matrix *m : views)
        if (p && m && m->rows > 0 && m->data == p) return true;
    return false;
}

// Whether TMA can address a view's rows; what its copy in the workspace takes otherwise, rows at multiples of 128 bytes (of 16 would do, but
// 8-bit 1001 x 1536 x 777 then takes 7.0 us, 5.8 so).
inline int64_t copy_pitch(const onnxb_matrix *m) { return (m->cols * type_bytes(m->type) + 127) / 128 * 128; }
inline bool in_place(const onnxb_matrix *m) {
    return reinterpret_cast<uintptr_t>(m->data) % 16 == 0 && (m->rows <= 1 || m->ld * type_bytes(m->type) % 16 == 0);
}
inline size_t copy_bytes(const onnxb_matrix *m) {
    if (!m || m->rows < 1 || m->cols < 1 || m->rows > kMostSize || m->cols > kMostSize || in_place(m)) return 0;
    return (size_t)(copy_pitch(m) * m->rows);
}
inline onnxb_status check_workspace(const void *workspace, size_t bytes, size_t need, std::initializer_list<const onnxb_matrix *> views) {
    if (need == 0) return ONNXB_OK;
    if (!workspace || bytes < need) return ONNXB_ERR_WORKSPACE;
    return reinterpret_cast<uintptr_t>(workspace) % 16 || begins_at(workspace, views) ? ONNXB_ERR_UNSUPPORTED : ONNXB_OK;
}
// Operands as the kernels read them: where they lie, or copied to the workspace, all in one launch (run(), before their first use).
struct Placement {
    char *workspace;
    RepackProblem repack{};
    explicit Placement(void *ws) : workspace(static_cast<char *>(ws)) {}
    DenseOperand operator()(const onnxb_matrix *m) {
        const size_t bytes = copy_bytes(m);
        if (bytes == 0) return operand(m);
        const int element = type_bytes(m->type);
        repack.job[repack.count++] = RepackJob{static_cast<const uint8_t *>(m->data), operand(m).ld * element, m->cols * element, (int)m->rows, element,
                                               reinterpret_cast<uint8_t *>(workspace), copy_pitch(m), 0, 0, nullptr};
        const DenseOperand o{workspace, copy_pitch(m) / element};
        workspace += bytes;
        return o;
    }
    // The reduction's length for `operands` that all run along it: where every one is a copy, that with the zeros behind its rows, so that
    // the kernels have whole blocks of it.
    int reduction(int64_t K, int operands, int type) const {
        return repack.count == operands ? (int)((K * type_bytes(type) + 127) / 128 * 128 / type_bytes(type)) : (int)K;
    }
    int run(cudaStream_t stream) const { return repack.count ? launch_repack_rows(repack, stream) : 0; }
};

inline onnxb_status status_of(int cuda_error) { return cuda_error == 0 ? ONNXB_OK : ONNXB_ERR_CUDA; }

#define CHECK(expr)                                      \
    do {                                                 \
        const onnxb_status check_status_ = (expr);       \
        if (check_status_ != ONNXB_OK) return check_status_; \
    } while (0)

}  // namespace views
}  // namespace onnxb
