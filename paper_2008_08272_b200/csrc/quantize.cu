// onnx_quantize_rows_run: 8-bit integers and a scale for each row.
#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"

namespace onnxb {

namespace {

using namespace dense;

// The nearest integer to x / scale, of the exact quotient, ties to even, at most 127 in magnitude.  `inverse` is 1 / scale: x * inverse
// is within 2 roundings of the quotient, so its nearest integer is off by one at most, next to a half.  What is left of x then
// (exact: it has no more digits than x and scale together span) says which side of the half the quotient is on.
__device__ __forceinline__ int quantize(float x, float scale, float inverse) {
    float q = rintf(x * inverse);
    const float rest = fmaf(-q, scale, x), half = 0.5f * scale;
    const bool odd = ((int)q & 1) != 0;
    if (rest > half || (rest == half && odd)) q += 1.f;
    if (rest < -half || (rest == -half && odd)) q -= 1.f;
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}

// What a row's values are multiplied by before they are divided, and its scale after that: where the scale is so small that its
// inverse or the halves of it would not be exact, both are taken 2^100 times as large.
__device__ __forceinline__ float magnify(float scale) { return scale < 0x1p-100f ? 0x1p100f : 1.f; }

template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(int M, int K, const T *X, long long x_ld, int8_t *Q, long long q_ld, float *scale) {
    __shared__ float most[8];
    const long long i = blockIdx.x;
    const T *x = X + i * x_ld;
    int8_t *q = Q + i * q_ld;
    // (as integers: the bits of magnitudes are ordered as they are, with infinity and NaN above all others)
    unsigned m = 0;
    for (int k = threadIdx.x; k < K; k += 256) m = max(m, __float_as_uint(fabsf(to_float(x[k]))));
    m = __reduce_max_sync(0xffffffffu, m);
    if (threadIdx.x % 32 == 0) most[threadIdx.x / 32] = __uint_as_float(m);
    __syncthreads();
    for (int w = 0; w < 8; ++w) m = max(m, __float_as_uint(most[w]));
    const bool finite = m < 0x7F800000u;
    const float s = __fdiv_rn(__uint_as_float(m), 127.f);
    if (threadIdx.x == 0) scale[i] = finite ? s : __uint_as_float(0x7FC00000u);
    const bool some = finite && s > 0.f;
    const float by = magnify(s), large = s * by, inverse = __fdiv_rn(1.f, large);
    for (int k = threadIdx.x; k < K; k += 256) q[k] = some ? (int8_t)quantize(to_float(x[k]) * by, large, inverse) : (int8_t)0;
}

template <typename T>
void launch(int M, int K, const void *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream) {
    quantize_rows_kernel<T><<<M, 256, 0, stream>>>(M, K, static_cast<const T *>(X), x_ld, Q, q_ld, scale);
}

}  // namespace

int launch_quantize_rows(int type, int M, int K, const void *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream) {
    if (type == ONNXB_FLOAT) launch<float>(M, K, X, x_ld, Q, q_ld, scale, stream);
    else if (type == ONNXB_FLOAT16) launch<__half>(M, K, X, x_ld, Q, q_ld, scale, stream);
    else launch<__nv_bfloat16>(M, K, X, x_ld, Q, q_ld, scale, stream);
    count_launch();
    return (int)cudaGetLastError();
}

}  // namespace onnxb
