// The dense layers' choice of kernel, and their elementwise ones: rows laid out for TMA, and the gated block's gradients before its products.
#include <algorithm>

#include "dense.h"
#include "dense_math.cuh"

namespace onnxb {

namespace {

using namespace dense;

// Rows that TMA cannot address (they do not begin at multiples of 16 bytes) laid out so that it can, 16 bytes a thread: aligned 4-byte loads,
// put together across their borders, except at a row's ends, where they would reach into what is not the row's.
__global__ void __launch_bounds__(256) repack_rows_kernel(const uint8_t *src, long long src_pitch, long long chunks, long long total, long long row_bytes,
                                                          uint8_t *dst, long long dst_pitch) {
    for (long long e = blockIdx.x * 256ll + threadIdx.x; e < total; e += gridDim.x * 256ll) {
        const long long row = e / chunks, at = (e - row * chunks) * 16;
        const uint8_t *from = src + row * src_pitch + at;
        uint32_t w[4] = {0, 0, 0, 0};
        const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(from) & 3);
        if (at + 16 <= row_bytes && off == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const uint32_t *>(from)[i];
        } else if (at > 0 && at + 20 <= row_bytes) {
            const uint32_t *words = reinterpret_cast<const uint32_t *>(from - off);
            uint32_t low = words[0];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t high = words[i + 1];
                w[i] = __funnelshift_r(low, high, off * 8);
                low = high;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (at + i < row_bytes) w[i / 4] |= (uint32_t)from[i] << (i % 4 * 8);
        }
        *reinterpret_cast<uint4 *>(dst + row * dst_pitch + at) = make_uint4(w[0], w[1], w[2], w[3]);
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

int launch_dense(const DenseProblem &p, cudaStream_t stream) { return dense_few_fits(p) ? launch_dense_few(p, stream) : launch_tc_dense(p, stream); }

int launch_repack_rows(const void *src, long long src_pitch, int rows, long long row_bytes, void *dst, long long dst_pitch, cudaStream_t stream) {
    const long long chunks = dst_pitch / 16, total = chunks * rows;
    const int grid = (int)std::min<long long>((total + 255) / 256, 148 * 8);
    repack_rows_kernel<<<grid, 256, 0, stream>>>(static_cast<const uint8_t *>(src), src_pitch, chunks, total, row_bytes, static_cast<uint8_t *>(dst), dst_pitch);
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
