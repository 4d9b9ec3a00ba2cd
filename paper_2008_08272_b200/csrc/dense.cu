// The dense layers' choice of kernel, and their elementwise ones: rows laid out for TMA, and the gated block's gradients before its products.
#include <algorithm>

#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"
#include "tc_host.h"

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

// dG = dH U act'(G), dU = dH act(G): five tensors' bytes, and about 40 instructions an element.  A block has 8 rows by 32 pieces of 8
// elements (of 1 where rows do not begin at multiples of 16 bytes), so that nothing is divided to find a place.  4096 x 10240 of 16-bit floats: see
// launch_gated_slope.
template <typename T, int kCount>
__global__ void __launch_bounds__(256) gated_slope_kernel(const GatedSlopeProblem p) {
    struct alignas(kCount * sizeof(T)) Piece { T v[kCount]; };
    const long long j = ((long long)blockIdx.x * 32 + threadIdx.x % 32) * kCount;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if (j >= p.F) return;
    for (int i = blockIdx.y * 8 + threadIdx.x / 32; i < p.M; i += gridDim.y * 8) {
        const Piece dh = *reinterpret_cast<const Piece *>(static_cast<const T *>(p.dH.p) + i * p.dH.ld + j);
        const Piece g = *reinterpret_cast<const Piece *>(static_cast<const T *>(p.G.p) + i * p.G.ld + j);
        const Piece u = *reinterpret_cast<const Piece *>(static_cast<const T *>(p.U.p) + i * p.U.ld + j);
        Piece dg, du;
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
            float value, slope;
            const float d = to_float(dh.v[e]);
            activate_with_slope(p.activation, to_float(g.v[e]), value, slope);
            dg.v[e] = from_float<T>(d * to_float(u.v[e]) * slope);
            du.v[e] = from_float<T>(d * value);
        }
        *reinterpret_cast<Piece *>(static_cast<T *>(p.dG) + i * p.d_ld + j) = dg;
        *reinterpret_cast<Piece *>(static_cast<T *>(p.dU) + i * p.d_ld + j) = du;
    }
}

// Four columns a thread, 8 rows by 128 columns a block
template <typename T>
__global__ void __launch_bounds__(256) sum_parts_kernel(const SumPartsProblem p) {
    const int j = (blockIdx.x * 32 + threadIdx.x % 32) * 4;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if (j >= p.N) return;
    for (int i = blockIdx.y * 8 + threadIdx.x / 32; i < p.M; i += gridDim.y * 8) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int s = 0; s < p.parts; ++s) {
            const float4 w = __ldg(reinterpret_cast<const float4 *>(p.P + ((long long)s * p.part_rows + i) * p.p_ld + j));
            v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
        }
        T *y = static_cast<T *>(p.Y) + i * p.y_ld + j;
        alignas(8) const T out[4] = {from_float<T>(v.x), from_float<T>(v.y), from_float<T>(v.z), from_float<T>(v.w)};
        if (j + 4 <= p.N && reinterpret_cast<uintptr_t>(y) % 8 == 0) *reinterpret_cast<uint2 *>(y) = *reinterpret_cast<const uint2 *>(out);
        else
            for (int e = 0; e < 4; ++e)
                if (j + e < p.N) y[e] = out[e];
    }
}

template <typename T>
int launch_slope(const GatedSlopeProblem &p, cudaStream_t stream) {
    auto aligned = [&](const DenseOperand &o) { return reinterpret_cast<uintptr_t>(o.p) % 16 == 0 && (p.M == 1 || o.ld % 8 == 0); };
    const bool pieces = p.F % 8 == 0 && aligned(p.dH) && aligned(p.G) && aligned(p.U);
    const int count = pieces ? 8 : 1, across = (p.F + 32 * count - 1) / (32 * count);
    const dim3 grid(across, std::min(65535, (p.M + 7) / 8));
    return (int)(pieces ? tc_host::launch_pdl(gated_slope_kernel<T, 8>, grid, dim3(256), 0, stream, p)
                        : tc_host::launch_pdl(gated_slope_kernel<T, 1>, grid, dim3(256), 0, stream, p));
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

int launch_sum_parts(const SumPartsProblem &p, cudaStream_t stream) {
    const dim3 grid((p.N + 127) / 128, std::min(65535, (p.M + 7) / 8));
    const cudaError_t e = p.type == ONNXB_FLOAT16 ? tc_host::launch_pdl(sum_parts_kernel<__half>, grid, dim3(256), 0, stream, p)
                                                  : tc_host::launch_pdl(sum_parts_kernel<__nv_bfloat16>, grid, dim3(256), 0, stream, p);
    count_launch();
    return (int)e;
}

int launch_gated_slope(const GatedSlopeProblem &p, cudaStream_t stream) {
    const int err = p.type == ONNXB_FLOAT16 ? launch_slope<__half>(p, stream) : launch_slope<__nv_bfloat16>(p, stream);
    count_launch();
    return err;
}

}  // namespace onnxb
