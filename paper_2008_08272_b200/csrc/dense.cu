// The dense layers' choice of kernel, and their elementwise ones: rows laid out for TMA, and the gated block's gradients before its products.
#include <algorithm>

#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

// Rows that TMA cannot address (they do not begin at multiples of 16 bytes) laid out so that it can: a warp per row, 16 bytes a lane and
// step.  A block per 8 rows of a tensor, all tensors of a call in one launch.
__global__ void __launch_bounds__(256) repack_rows_kernel(const RepackProblem p) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const RepackJob &job = p.job[blockIdx.y];
    const int lane = threadIdx.x % 32;
    for (int row = blockIdx.x * 8 + threadIdx.x / 32; row < job.rows; row += gridDim.x * 8) {
        const uint8_t *src = job.src + row * job.src_pitch;
        uint8_t *dst = job.dst + row * job.dst_pitch;
        for (long long at = lane * 16; at < job.row_bytes; at += 32 * 16) *reinterpret_cast<uint4 *>(dst + at) = job.element == 2 ? load16_anywhere<2>(src, at, job.row_bytes) : load16_anywhere<1>(src, at, job.row_bytes);
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
            const float4 w = *reinterpret_cast<const float4 *>(p.P + ((long long)s * p.part_rows + i) * p.p_ld + j);
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

int launch_repack_rows(const RepackProblem &p, cudaStream_t stream) {
    int rows = 1;
    for (int i = 0; i < p.count; ++i) rows = std::max(rows, p.job[i].rows);
    const dim3 grid(std::min((rows + 7) / 8, 148 * 8), p.count);
    const cudaError_t e = tc_host::launch_pdl(repack_rows_kernel, grid, dim3(256), 0, stream, p);
    count_launch();
    return (int)e;
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
