// onnx_quantize_rows_run: 8-bit integers and a scale for each row.
//
// One pass over X where a row fits the registers of the threads that share it (a warp for short rows, a block for longer ones; up to
// 16 pieces of 16 bytes each): the row is read, its largest magnitude agreed on, and what the registers hold is divided and stored.  Longer
// rows are read a second time, out of L2.  Bound by the bytes of X and Q.
#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

// The nearest integer to x / scale, of the exact quotient, ties to even, at most 127 in magnitude.  `inverse` is 1 / scale: x * inverse
// is within 2 roundings of the quotient, so its nearest integer is off by one at most, next to a half.  What is left of x then
// (exact: it has no more digits than x and scale together span) says which side of the half the quotient is on.
__device__ __forceinline__ int quantize(float x, float scale, float inverse) {
    float q = rintf(x * inverse);
    const float rest = fmaf(-q, scale, x), half = 0.5f * scale;
    // (only where rest is half the scale or more, next to a half: hardly ever)
    if (fabsf(rest) >= half) {
        const bool odd = ((int)q & 1) != 0;
        if (rest > half || (rest == half && odd)) q += 1.f;
        if (rest < -half || (rest == -half && odd)) q -= 1.f;
    }
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}

// What a row's values are multiplied by before they are divided, and its scale after that: where the scale is so small that its
// inverse or the halves of it would not be exact, both are taken 2^100 times as large.
__device__ __forceinline__ float magnify(float scale) { return scale < 0x1p-100f ? 0x1p100f : 1.f; }

struct Row {
    float by, large, inverse;
    bool some;               // there is a scale, and it is no zero
};
// From a row's largest magnitude, as bits (those of magnitudes are ordered as they are, infinity and NaN above all others)
__device__ __forceinline__ Row row_of(unsigned most, float *scale_out, bool writes) {
    const bool finite = most < 0x7F800000u;
    const float s = __fdiv_rn(__uint_as_float(most), 127.f);
    if (writes) *scale_out = finite ? s : __uint_as_float(0x7FC00000u);
    Row r;
    r.some = finite && s > 0.f;
    r.by = magnify(s);
    r.large = s * r.by;
    r.inverse = __fdiv_rn(1.f, r.large);
    return r;
}
__device__ __forceinline__ int quantize(float x, const Row &r) { return r.some ? quantize(x * r.by, r.large, r.inverse) : 0; }
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(fabsf(x)); }

// Several rows a block, a group of kThreads threads each
template <int kThreads>
__device__ __forceinline__ unsigned most_of_group(unsigned m) {
    m = __reduce_max_sync(0xffffffffu, m);
    if (kThreads > 32) {
        __shared__ unsigned of_warp[32];
        if (threadIdx.x % 32 == 0) of_warp[threadIdx.x / 32] = m;
        __syncthreads();
        constexpr int kWarps = kThreads / 32;
        m = __reduce_max_sync(0xffffffffu, of_warp[threadIdx.x % kWarps]);
    }
    return m;
}

template <typename T>
struct Piece {               // 16 bytes of X
    static constexpr int kCount = 16 / sizeof(T);
    uint4 v;
    __device__ __forceinline__ float at(int i) const { return to_float(reinterpret_cast<const T *>(&v)[i]); }
};

// Rows that begin at multiples of 16 bytes in X and of 8 (fp32: 4) in Q, and whose width is a multiple of a piece
template <typename T, int kThreads, int kPieces>
__global__ void __launch_bounds__(256) quantize_pieces_kernel(int M, int pieces, const T *X, long long x_ld, int8_t *Q, long long q_ld, float *scale) {
    constexpr int kRows = 256 / kThreads, kCount = Piece<T>::kCount;
    const long long i = (long long)blockIdx.x * kRows + threadIdx.x / kThreads;
    const int at = threadIdx.x % kThreads;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const bool in = i < M;
    const uint4 *x = reinterpret_cast<const uint4 *>(X + (in ? i : 0) * x_ld);
    Piece<T> v[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k) v[k].v = in && at + k * kThreads < pieces ? __ldg(x + at + k * kThreads) : make_uint4(0, 0, 0, 0);
    unsigned m = 0;
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
        for (int e = 0; e < kCount; ++e) m = max(m, magnitude(v[k].at(e)));
    m = most_of_group<kThreads>(m);
    if (!in) return;
    const Row r = row_of(m, scale + i, at == 0);
    int8_t *q = Q + i * q_ld;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        const int piece = at + k * kThreads;
        if (piece >= pieces) break;
        uint32_t w[kCount / 4];
#pragma unroll
        for (int e = 0; e < kCount; e += 4)
            w[e / 4] = (uint32_t)(quantize(v[k].at(e), r) & 255) | (uint32_t)(quantize(v[k].at(e + 1), r) & 255) << 8 |
                       (uint32_t)(quantize(v[k].at(e + 2), r) & 255) << 16 | (uint32_t)quantize(v[k].at(e + 3), r) << 24;
        if (kCount == 4) reinterpret_cast<uint32_t *>(q)[piece] = w[0];
        else reinterpret_cast<uint2 *>(q)[piece] = make_uint2(w[0], w[kCount / 4 - 1]);
    }
}

// Any row: an element at a time, twice
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(int K, const T *X, long long x_ld, int8_t *Q, long long q_ld, float *scale) {
    const long long i = blockIdx.x;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const T *x = X + i * x_ld;
    int8_t *q = Q + i * q_ld;
    unsigned m = 0;
#pragma unroll 4
    for (int k = threadIdx.x; k < K; k += 256) m = max(m, magnitude(to_float(x[k])));
    const Row r = row_of(most_of_group<256>(m), scale + i, threadIdx.x == 0);
#pragma unroll 4
    for (int k = threadIdx.x; k < K; k += 256) q[k] = (int8_t)quantize(to_float(x[k]), r);
}

template <typename T>
int launch(int M, int K, const void *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream) {
    constexpr int kCount = Piece<T>::kCount;
    const int pieces = K / kCount;
    const bool in_pieces = K % kCount == 0 && reinterpret_cast<uintptr_t>(X) % 16 == 0 && reinterpret_cast<uintptr_t>(Q) % kCount == 0 &&
                           (M == 1 || (x_ld % kCount == 0 && q_ld % kCount == 0)) && pieces <= 256 * 16;
    const T *x = static_cast<const T *>(X);
    auto pieces_of = [&](auto kernel, int rows) {
        return (int)tc_host::launch_pdl(kernel, dim3((unsigned)((M + rows - 1) / rows)), dim3(256), 0, stream, M, pieces, x, x_ld, Q, q_ld, scale);
    };
    if (!in_pieces) return (int)tc_host::launch_pdl(quantize_rows_kernel<T>, dim3(M), dim3(256), 0, stream, K, x, x_ld, Q, q_ld, scale);
    if (pieces <= 64) return pieces_of(quantize_pieces_kernel<T, 32, 2>, 8);
    if (pieces <= 128) return pieces_of(quantize_pieces_kernel<T, 32, 4>, 8);
    if (pieces <= 512) return pieces_of(quantize_pieces_kernel<T, 256, 2>, 1);
    if (pieces <= 1024) return pieces_of(quantize_pieces_kernel<T, 256, 4>, 1);
    if (pieces <= 2048) return pieces_of(quantize_pieces_kernel<T, 256, 8>, 1);
    return pieces_of(quantize_pieces_kernel<T, 256, 16>, 1);
}

}  // namespace

int launch_quantize_rows(int type, int M, int K, const void *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream) {
    const int err = type == ONNXB_FLOAT     ? launch<float>(M, K, X, x_ld, Q, q_ld, scale, stream)
                    : type == ONNXB_FLOAT16 ? launch<__half>(M, K, X, x_ld, Q, q_ld, scale, stream)
                                            : launch<__nv_bfloat16>(M, K, X, x_ld, Q, q_ld, scale, stream);
    count_launch();
    return err;
}

}  // namespace onnxb
