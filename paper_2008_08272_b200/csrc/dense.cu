// Dense layers of 8- and 16-bit operands, the simple form: 64 x 64 tiles of the output, sums in registers, any pitch.
#include <algorithm>

#include "dense.h"
#include "dense_math.cuh"

namespace onnxb {

namespace {

using namespace dense;

constexpr int kTile = 64, kStep = 16;

struct Params {
    DenseProblem d;
    int a_mn, b_mn;
};

template <typename T>
struct Sum { typedef float type; };
template <>
struct Sum<int8_t> { typedef int type; };
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ int widen(int8_t v) { return v; }

__device__ void store(void *Y, int type, long long at, float v) {
    if (type == ONNXB_FLOAT) static_cast<float *>(Y)[at] = v;
    else if (type == ONNXB_FLOAT16) static_cast<__half *>(Y)[at] = from_float<__half>(v);
    else static_cast<__nv_bfloat16 *>(Y)[at] = from_float<__nv_bfloat16>(v);
}

// One product's share of a tile: rows i0.., columns j0..
template <typename T, typename S>
__device__ void accumulate(const DenseOperand &A, int a_mn, const DenseOperand &B, int b_mn, int M, int N, int K, int i0, int j0, S (&acc)[4][4]) {
    __shared__ S as[kStep][kTile + 1], bs[kStep][kTile + 1];
    const T *a = static_cast<const T *>(A.p), *b = static_cast<const T *>(B.p);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (int k0 = 0; k0 < K; k0 += kStep) {
        for (int e = threadIdx.x; e < kTile * kStep; e += 256) {
            const int ra = a_mn ? e % kTile : e / kStep, ka = a_mn ? e / kTile : e % kStep;
            const int rb = b_mn ? e % kTile : e / kStep, kb = b_mn ? e / kTile : e % kStep;
            as[ka][ra] = i0 + ra < M && k0 + ka < K ? widen(a_mn ? a[(k0 + ka) * A.ld + i0 + ra] : a[(i0 + ra) * A.ld + k0 + ka]) : S(0);
            bs[kb][rb] = j0 + rb < N && k0 + kb < K ? widen(b_mn ? b[(k0 + kb) * B.ld + j0 + rb] : b[(j0 + rb) * B.ld + k0 + kb]) : S(0);
        }
        __syncthreads();
        for (int k = 0; k < kStep; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] += as[k][ty + 16 * i] * bs[k][tx + 16 * j];
        __syncthreads();
    }
}

template <typename T>
__global__ void __launch_bounds__(256) dense_kernel(const Params p) {
    typedef typename Sum<T>::type S;
    const DenseProblem &d = p.d;
    const int i0 = blockIdx.x * kTile, j0 = blockIdx.y * kTile, z = blockIdx.z;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    S g[4][4] = {}, u[4][4] = {};
    if (d.mode == kDenseGradW && !d.Y[z]) return;
    accumulate<T, S>(d.A[d.mode == kDenseGradW ? z : 0], p.a_mn, d.B[0], p.b_mn, d.M, d.N, d.K, i0, j0, g);
    if (d.mode == kDenseGradX) accumulate<T, S>(d.A[1], p.a_mn, d.B[1], p.b_mn, d.M, d.N, d.K, i0, j0, g);
    if (d.mode == kDenseGated) accumulate<T, S>(d.A[0], p.a_mn, d.B[1], p.b_mn, d.M, d.N, d.K, i0, j0, u);
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int i = i0 + ty + 16 * a, j = j0 + tx + 16 * b;
            if (i >= d.M || j >= d.N) continue;
            // (one factor after the other: the sum may be 0 and the factors' product infinite)
            float v = (float)g[a][b], w = (float)u[a][b];
            if (d.a_scale) {
                v = v * d.a_scale[i] * d.b_scale[0][j];
                if (d.mode == kDenseGated) w = w * d.a_scale[i] * d.b_scale[1][j];
            }
            if (d.bias) v += d.bias[j];
            if (d.mode == kDenseGated) {
                if (d.Y[1]) store(d.Y[1], d.y_type, i * d.y_ld[1] + j, v);
                if (d.Y[2]) store(d.Y[2], d.y_type, i * d.y_ld[2] + j, w);
                v = activate(d.activation, v) * w;
            }
            if (d.relu) v = v > 0.f ? v : 0.f;
            const int y = d.mode == kDenseGradW ? z : 0;
            store(d.Y[y], d.y_type, i * d.y_ld[y] + j, v);
        }
}

template <typename T>
__global__ void gated_slope_kernel(const GatedSlopeProblem p) {
    const long long n = (long long)p.M * p.F;
    for (long long e = blockIdx.x * 256ll + threadIdx.x; e < n; e += gridDim.x * 256ll) {
        const long long i = e / p.F, j = e % p.F;
        const float dh = to_float(static_cast<const T *>(p.dH.p)[i * p.dH.ld + j]);
        const float g = to_float(static_cast<const T *>(p.G.p)[i * p.G.ld + j]), u = to_float(static_cast<const T *>(p.U.p)[i * p.U.ld + j]);
        float value, slope;
        activate_with_slope(p.activation, g, value, slope);
        static_cast<T *>(p.dG)[i * p.d_ld + j] = from_float<T>(dh * u * slope);
        static_cast<T *>(p.dU)[i * p.d_ld + j] = from_float<T>(dh * value);
    }
}

}  // namespace

int launch_dense(const DenseProblem &d, cudaStream_t stream) {
    Params p{d, d.mode == kDenseGradW, d.mode == kDenseGradX || d.mode == kDenseGradW};
    const dim3 grid((d.M + kTile - 1) / kTile, (d.N + kTile - 1) / kTile, d.mode == kDenseGradW ? 2 : 1);
    if (d.type == ONNXB_INT8) dense_kernel<int8_t><<<grid, 256, 0, stream>>>(p);
    else if (d.type == ONNXB_FLOAT16) dense_kernel<__half><<<grid, 256, 0, stream>>>(p);
    else dense_kernel<__nv_bfloat16><<<grid, 256, 0, stream>>>(p);
    count_launch();
    return (int)cudaGetLastError();
}

int launch_gated_slope(const GatedSlopeProblem &p, cudaStream_t stream) {
    const int grid = (int)std::min<long long>(((long long)p.M * p.F + 255) / 256, 148 * 16);
    if (p.type == ONNXB_FLOAT16) gated_slope_kernel<__half><<<grid, 256, 0, stream>>>(p);
    else gated_slope_kernel<__nv_bfloat16><<<grid, 256, 0, stream>>>(p);
    count_launch();
    return (int)cudaGetLastError();
}

}  // namespace onnxb
