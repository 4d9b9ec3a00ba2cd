// Products by group for a few rows, those of single tokens first of all: every weight of a group that has a row is read once, and that is what bounds it.
//
// As in dense_few.cu a block has 16 channels (the gated block's: of both weights), its warps share the reduction and add their sums in shared memory in a fixed
// order, and the weights go from global memory straight into the registers of mma.sync, 16 bytes a lane and load, so that as many loads are in flight
// as there are warps.  What is its own: a block is one of a row, and goes on if that row is its group's first, with all of the group's rows, eight at a time.
// Which group that is it finds in the offsets: the first of them above the row ends the group, the largest before that begins it.  And weights and rows
// may begin anywhere: nothing is copied, where most groups' weights are not read at all.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdlib>

#include "dense_math.cuh"
#include "grouped.h"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

constexpr int kChannels = 16, kRows = 8, kWarps = 8;

struct Params {
    int rows, groups, channels;
    const int *offsets;
    long long row_bytes;             // of the reduction
    const uint8_t *X, *W[2];
    long long x_pitch, w_pitch[2], w_stride[2];      // bytes
    int activation, type;
    void *Y[3];
    long long y_ld[3];
};

// 16 bytes of a row, zeros past its end
template <bool kAligned, bool kWeight>
__device__ __forceinline__ uint4 load16(const uint8_t *row, long long at, long long row_bytes) {
    if (!kAligned) return at < row_bytes ? load16_anywhere<2>(row, at, row_bytes) : make_uint4(0, 0, 0, 0);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (at + 16 <= row_bytes) {
        // (weights, which nobody reads twice, not by way of L1)
        if (kWeight) asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + at));
        else v = *reinterpret_cast<const uint4 *>(row + at);
    } else if (at < row_bytes) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; i += 2)
            if (at + i < row_bytes) w[i / 4] |= (uint32_t)*reinterpret_cast<const uint16_t *>(row + at + i) << (i % 4 * 8);
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}

template <bool kBf16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (kBf16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <bool kBf16>
__device__ __forceinline__ void put(void *Y, long long at, float v) {
    if (kBf16) static_cast<__nv_bfloat16 *>(Y)[at] = from_float<__nv_bfloat16>(v);
    else static_cast<__half *>(Y)[at] = from_float<__half>(v);
}

template <bool kBf16, int kWeights, bool kAligned>
__global__ void __launch_bounds__(32 * kWarps, 3) grouped_few_kernel(const Params p) {
    constexpr int kChunks = kWeights == 2 ? 2 : 4;
    __shared__ float sums[kWarps][kWeights][kChannels][kRows + 1];
    __shared__ int found[2][kWarps];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const int n0 = blockIdx.x * kChannels, row = blockIdx.y;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    // The group of this block's row: the first offset above it is its end (offsets that do not rise count as the largest before them)
    int end = p.groups + 1;
    for (int i = threadIdx.x; i <= p.groups; i += 32 * kWarps)
        if (p.offsets[i] > row) end = min(end, i);
    end = __reduce_min_sync(0xffffffffu, end);
    if (lane == 0) found[0][warp] = end;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) end = min(end, found[0][w]);
    if (end == 0 || end > p.groups) return;              // of no group
    int first = 0;
    for (int i = threadIdx.x; i < end; i += 32 * kWarps) first = max(first, p.offsets[i]);
    first = __reduce_max_sync(0xffffffffu, first);
    if (lane == 0) found[1][warp] = first;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) first = max(first, found[1][w]);
    if (first != row) return;                            // not its first
    const int last = min(p.offsets[end], p.rows), group = end - 1;
    // (channels past the last: the last one again, whose sums nobody stores)
    const uint8_t *b[kWeights][2];
#pragma unroll
    for (int w = 0; w < kWeights; ++w)
#pragma unroll
        for (int h = 0; h < 2; ++h) b[w][h] = p.W[w] + group * p.w_stride[w] + min(n0 + g + 8 * h, p.channels - 1) * p.w_pitch[w];
    const long long share = (p.row_bytes + kWarps * 64 - 1) / (kWarps * 64) * 64, begin = warp * share, stop = min(begin + share, p.row_bytes);
    for (int m0 = first; m0 < last; m0 += kRows) {
        const bool in = m0 + g < last;
        const uint8_t *a = p.X + (in ? m0 + g : m0) * p.x_pitch;
        float acc[kWeights][4] = {};
        for (long long at0 = begin + t * 16; at0 - t * 16 < stop; at0 += kChunks * 64) {
            uint4 wv[kChunks][kWeights][2], xv[kChunks];
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int w = 0; w < kWeights; ++w)
#pragma unroll
                    for (int h = 0; h < 2; ++h) wv[c][w][h] = load16<kAligned, true>(b[w][h], at0 + c * 64, stop);
#pragma unroll
            for (int c = 0; c < kChunks; ++c) xv[c] = in ? load16<kAligned, false>(a, at0 + c * 64, stop) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int w = 0; w < kWeights; ++w) {
                    // (which terms the instruction takes a lane's words for is all the same, as long as both operands agree)
                    const uint4 u = wv[c][w][0], v = wv[c][w][1], x = xv[c];
                    mma<kBf16>(acc[w], u.x, v.x, u.y, v.y, x.x, x.y);
                    mma<kBf16>(acc[w], u.z, v.z, u.w, v.w, x.z, x.w);
                }
        }
        __syncthreads();                                 // (the sums before these have been read)
#pragma unroll
        for (int w = 0; w < kWeights; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[warp][w][g + e / 2 * 8][2 * t + e % 2] = acc[w][e];
        __syncthreads();
        const int r = threadIdx.x % kChannels, n = n0 + r, m = threadIdx.x / kChannels;
        if (threadIdx.x < kChannels * kRows && n < p.channels && m0 + m < last) {
            float v[kWeights];
#pragma unroll
            for (int w = 0; w < kWeights; ++w) {
                v[w] = 0.f;
#pragma unroll
                for (int k = 0; k < kWarps; ++k) v[w] += sums[k][w][r][m];
            }
            const long long i = m0 + m;
            if (kWeights == 2) {
                if (p.Y[1]) {
                    put<kBf16>(p.Y[1], i * p.y_ld[1] + n, v[0]);
                    put<kBf16>(p.Y[2], i * p.y_ld[2] + n, v[kWeights - 1]);
                }
                v[0] = activate(p.activation, v[0]) * v[kWeights - 1];
            }
            put<kBf16>(p.Y[0], i * p.y_ld[0] + n, v[0]);
        }
    }
}

template <bool kBf16, bool kAligned>
void (*kernel_for(bool gated))(const Params) {
    return gated ? grouped_few_kernel<kBf16, 2, kAligned> : grouped_few_kernel<kBf16, 1, kAligned>;
}

}  // namespace

// Up to 16 rows: 2 rows of 8 groups, gated block 4096 -> 10240, 54.7 us here and 60.6 on the tensor cores, 16 of 64 groups 4096 -> 1408 54.5 and 61.7, one row
// 8192 -> 1024 10.7 and 22.5, whose few tiles read one SM's share of the bandwidth each; but 32 of 64 groups 1408 -> 2048 34 and 26.4.
// ONNXB_GROUPED_FEW = the most rows pins it for A/B measurements and tests (at most 64).
bool grouped_few_fits(int rows) {
    int most = 16;
    if (const char *e = getenv("ONNXB_GROUPED_FEW")) most = std::min(64, atoi(e));
    return rows <= most;
}

int launch_grouped_few(const GroupedProblem &d, cudaStream_t stream) {
    const bool gated = d.mode == kGroupedGated;
    Params p{};
    p.rows = d.rows; p.groups = d.groups; p.channels = d.channels; p.offsets = d.offsets;
    p.row_bytes = (long long)d.width * 2;
    p.X = static_cast<const uint8_t *>(d.A[0].p); p.x_pitch = d.A[0].ld * 2;
    bool aligned = reinterpret_cast<uintptr_t>(p.X) % 16 == 0 && (d.rows == 1 || p.x_pitch % 16 == 0);
    for (int w = 0; w < (gated ? 2 : 1); ++w) {
        p.W[w] = static_cast<const uint8_t *>(d.W[w].p);
        p.w_pitch[w] = d.W[w].ld * 2;
        p.w_stride[w] = d.W[w].stride * 2;
        aligned = aligned && reinterpret_cast<uintptr_t>(p.W[w]) % 16 == 0 && (d.channels == 1 || p.w_pitch[w] % 16 == 0) && (d.groups == 1 || p.w_stride[w] % 16 == 0);
    }
    p.activation = d.activation;
    for (int i = 0; i < 3; ++i) { p.Y[i] = d.Y[i]; p.y_ld[i] = d.y_ld[i]; }
    const bool bf16 = d.type == ONNXB_BFLOAT16;
    const auto kernel = bf16 ? (aligned ? kernel_for<true, true>(gated) : kernel_for<true, false>(gated)) : aligned ? kernel_for<false, true>(gated) : kernel_for<false, false>(gated);
    const dim3 grid((unsigned)((d.channels + kChannels - 1) / kChannels), (unsigned)d.rows);
    const cudaError_t e = tc_host::launch_pdl(kernel, grid, dim3(32 * kWarps), 0, stream, p);
    count_launch();
    return (int)e;
}

}  // namespace onnxb
