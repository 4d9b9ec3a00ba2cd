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
// step, put together from the two aligned 16-byte pieces that hold them; byte by byte at a row's ends, where those pieces reach into
// what is not the row's.  A block per 8 rows of a tensor, all tensors of a call in one launch.  2 x 105 MB of 10229-byte rows: see DESIGN.
__global__ void __launch_bounds__(256) repack_rows_kernel(const RepackProblem p) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const RepackJob &job = p.job[blockIdx.y];
    const int lane = threadIdx.x % 32;
    for (int row = blockIdx.x * 8 + threadIdx.x / 32; row < job.rows; row += gridDim.x * 8) {
        const uint8_t *src = job.src + row * job.src_pitch;
        uint8_t *dst = job.dst + row * job.dst_pitch;
        const int off = (int)(reinterpret_cast<uintptr_t>(src) & 15), bits = (off & 3) * 8;
        for (long long at = lane * 16; at < job.row_bytes; at += 32 * 16) {
            uint32_t w[8] = {}, out[4];
            if ((at > 0 || off == 0) && at + (off ? 32 - off : 16) <= job.row_bytes) {
                const uint4 *pieces = reinterpret_cast<const uint4 *>(src + at - off);
                const uint4 a = __ldg(pieces), b = off ? __ldg(pieces + 1) : make_uint4(0, 0, 0, 0);
                w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
                w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
                // (the same for the whole warp)
                auto from = [&](int first) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) out[i] = __funnelshift_r(w[first + i], first + i < 7 ? w[first + i + 1] : 0u, bits);
                };
                if (off < 4) from(0);
                else if (off < 8) from(1);
                else if (off < 12) from(2);
                else from(3);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (at + i < job.row_bytes) w[i / 4] |= (uint32_t)src[at + i] << (i % 4 * 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i] = w[i];
            }
            *reinterpret_cast<uint4 *>(dst + at) = make_uint4(out[0], out[1], out[2], out[3]);
        }
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
