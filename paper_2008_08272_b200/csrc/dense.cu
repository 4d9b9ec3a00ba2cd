// The dense layers' choice of kernel, and their elementwise ones: rows laid out for TMA, and the gated block's gradients before its products.
#include <algorithm>

#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

// Rows that TMA cannot address (they do not begin at multiples of 16 bytes) laid out so that it can, zeros up to the next one: 16 bytes a lane
// and step, a warp per row, several where rows are few and long, or one for several rows of less than 32 steps.  All tensors of a call in
// one launch.  Groups without rows (offsets that do not rise) are left out: nobody reads their weights.
__global__ void __launch_bounds__(256) repack_rows_kernel(const RepackProblem p) {
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const RepackJob &job = p.job[blockIdx.y];
    const int per_row = job.dst_pitch >= 512 ? 32 : job.dst_pitch >= 256 ? 16 : 8, rows = 256 / per_row, lane = threadIdx.x % per_row;
    for (int row = blockIdx.x * rows + threadIdx.x / per_row; row < job.rows; row += gridDim.x * rows) {
        const int group = job.group_rows ? row / job.group_rows : 0;
        if (job.offsets && job.offsets[group + 1] <= job.offsets[group]) continue;
        const uint8_t *src = job.src + group * job.group_pitch + (row - group * job.group_rows) * job.src_pitch;
        uint8_t *dst = job.dst + row * job.dst_pitch;
        for (long long at = (long long)(blockIdx.z * per_row + lane) * 16; at < job.dst_pitch; at += (long long)gridDim.z * per_row * 16)
            *reinterpret_cast<uint4 *>(dst + at) = job.element == 2 ? load16_anywhere<2>(src, at, job.row_bytes) : load16_anywhere<1>(src, at, job.row_bytes);
    }
}

// What a 16-bit number leaves of v, as one; nothing where there is no such number
template <typename T>
__device__ __forceinline__ T remainder_of(float v, T nearest) {
    const float left = v - to_float(nearest);
    return from_float<T>(isfinite(left) ? left : 0.f);
}

// dG = dH U act'(G), dU = dH act(G), in 32 bits and rounded once, to what the tensor cores take: five tensors' bytes, and about 40 instructions an element.  A block has 8 rows by 32 pieces of 8
// elements (of 1 where rows do not begin at multiples of 16 bytes), so that nothing is divided to find a place.  4096 x 10240 of bf16: 65 us (6.5
// TB/s).  kTwins: see GatedSlopeProblem; the blocks from x_blocks on copy X.
template <typename T, int kCount, bool kTwins>
__global__ void __launch_bounds__(256) gated_slope_kernel(const GatedSlopeProblem p, int x_blocks) {
    struct alignas(kCount * sizeof(T)) Piece { T v[kCount]; };
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if (kTwins && (int)blockIdx.x >= x_blocks) {
        const long long j = ((long long)blockIdx.x - x_blocks) * 32 + threadIdx.x % 32;
        if (j >= p.K) return;
        for (int i = blockIdx.y * 8 + threadIdx.x / 32; i < p.M; i += gridDim.y * 8) {
            const T x = static_cast<const T *>(p.X.p)[i * p.X.ld + j];
            T *to = static_cast<T *>(p.twice) + i * p.twice_ld + j;
            to[0] = x;
            // (what is left of dG and dU adds nothing to an infinity or a NaN, and would make a NaN of an infinity)
            to[p.M * p.twice_ld] = isfinite(to_float(x)) ? x : from_float<T>(0.f);
        }
        return;
    }
    const long long j = ((long long)blockIdx.x * 32 + threadIdx.x % 32) * kCount;
    if (j >= p.F) return;
    for (int i = blockIdx.y * 8 + threadIdx.x / 32; i < p.M; i += gridDim.y * 8) {
        const Piece dh = *reinterpret_cast<const Piece *>(static_cast<const T *>(p.dH.p) + i * p.dH.ld + j);
        const Piece g = *reinterpret_cast<const Piece *>(static_cast<const T *>(p.G.p) + i * p.G.ld + j);
        const Piece u = *reinterpret_cast<const Piece *>(static_cast<const T *>(p.U.p) + i * p.U.ld + j);
        Piece dg, du, dg_rest, du_rest;
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
            float value, slope;
            const float d = to_float(dh.v[e]);
            activate_with_slope(p.activation, to_float(g.v[e]), value, slope);
            const float a = d * to_float(u.v[e]) * slope, b = d * value;
            dg.v[e] = from_float<T>(a);
            du.v[e] = from_float<T>(b);
            if (kTwins) {
                dg_rest.v[e] = remainder_of(a, dg.v[e]);
                du_rest.v[e] = remainder_of(b, du.v[e]);
            }
        }
        T *to_g = static_cast<T *>(p.dG) + i * p.d_ld + j, *to_u = static_cast<T *>(p.dU) + i * p.d_ld + j;
        *reinterpret_cast<Piece *>(to_g) = dg;
        *reinterpret_cast<Piece *>(to_u) = du;
        if (kTwins) {
            *reinterpret_cast<Piece *>(to_g + p.M * p.d_ld) = dg_rest;
            *reinterpret_cast<Piece *>(to_u + p.M * p.d_ld) = du_rest;
        }
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
            const float *from = p.P + ((long long)s * p.part_rows + i) * p.p_ld + j;
            const float4 w = *reinterpret_cast<const float4 *>(from);
            const float4 rest = p.twins ? *reinterpret_cast<const float4 *>(from + p.M * p.p_ld) : make_float4(0.f, 0.f, 0.f, 0.f);
            // (of infinite weights the twins' sum is the opposite infinity or NaN, where there is nothing to add any more)
            auto both = [](float sum, float own, float twin) { return sum + own + (isfinite(own) ? twin : 0.f); };
            v = make_float4(both(v.x, w.x, rest.x), both(v.y, w.y, rest.y), both(v.z, w.z, rest.z), both(v.w, w.w, rest.w));
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
    const dim3 grid(across + (p.twins && p.X.p ? (p.K + 31) / 32 : 0), std::min(65535, (p.M + 7) / 8));
    auto kernel = pieces ? (p.twins ? gated_slope_kernel<T, 8, true> : gated_slope_kernel<T, 8, false>)
                         : (p.twins ? gated_slope_kernel<T, 1, true> : gated_slope_kernel<T, 1, false>);
    return (int)tc_host::launch_pdl(kernel, grid, dim3(256), 0, stream, p, across);
}

}  // namespace

int launch_dense(const DenseProblem &p, cudaStream_t stream) { return dense_few_fits(p) ? launch_dense_few(p, stream) : launch_tc_dense(p, stream); }

int launch_repack_rows(const RepackProblem &p, cudaStream_t stream) {
    int blocks = 1;
    long long parts = 1;
    for (int i = 0; i < p.count; ++i) {
        parts = std::max(parts, (p.job[i].dst_pitch + 511) / 512);
        const int rows = p.job[i].dst_pitch >= 512 ? 8 : p.job[i].dst_pitch >= 256 ? 16 : 32;        // a block
        blocks = std::max(blocks, (p.job[i].rows + rows - 1) / rows);
    }
    blocks = std::min(blocks, 148 * 8);
    const dim3 grid(blocks, p.count, (unsigned)std::max(1ll, std::min(parts, 148ll * 16 / (blocks * p.count))));
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
