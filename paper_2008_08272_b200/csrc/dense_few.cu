// Dense layers of 8- and 16-bit operands for a few tokens (single tokens first of all): every weight is read once and multiplied by
// up to 16 tokens, so the weights' bytes are what bounds it, and what counts is that enough loads are in flight on every SM.
//
// A block of 8 warps has 16 channels (the gated block: of both weights); its warps share the reduction in turns of kChunks x 64 bytes
// and add their sums in shared memory, in a fixed order.  The weights go from global memory straight into the registers of
// mma.sync (16 channels x 8 tokens), 16 bytes per lane and load: which terms of the reduction a lane's registers hold is up to the
// kernel as long as both operands agree, so a lane's four words are the terms that its 16 bytes hold, no matter which the
// instruction calls them.  (tcgen05 would want them in shared memory first, and its 128 rows for a few tokens.)
#include <cuda_runtime.h>

#include <algorithm>

#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

constexpr int kWarps = 8, kThreads = 32 * kWarps, kChannels = 16;

struct Params {
    int M, N;
    long long row_bytes;             // of the reduction
    const uint8_t *A, *B[2];
    long long a_pitch, b_pitch[2];   // bytes
    const float *a_scale, *b_scale[2], *bias;
    int relu, activation, y_type;
    void *Y[3];
    long long y_ld[3];
};

// 16 bytes of a row, zeros past its end
__device__ __forceinline__ uint4 load16(const uint8_t *row, long long at, long long row_bytes) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (at + 16 <= row_bytes) {
        asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + at));
    } else if (at < row_bytes) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (at + i < row_bytes) w[i / 4] |= (uint32_t)row[at + i] << (i % 4 * 8);
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}

template <int kType>
struct Of { typedef float Sum; };
template <>
struct Of<ONNXB_INT8> { typedef int Sum; };

__device__ __forceinline__ void mma(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <int kType>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (kType == ONNXB_BFLOAT16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <int kType>
__device__ __forceinline__ void mma(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    mma(d, a0, a1, a2, a3, b0, b1);
}

__device__ __forceinline__ void put(void *Y, int type, long long at, float v) {
    if (type == ONNXB_FLOAT) static_cast<float *>(Y)[at] = v;
    else if (type == ONNXB_FLOAT16) static_cast<__half *>(Y)[at] = from_float<__half>(v);
    else static_cast<__nv_bfloat16 *>(Y)[at] = from_float<__nv_bfloat16>(v);
}

// kTiles: of 8 tokens; kWeights: 2 for the gated block
template <int kType, int kTiles, int kWeights>
__global__ void __launch_bounds__(kThreads) dense_few_kernel(const Params p) {
    typedef typename Of<kType>::Sum Sum;
    constexpr int kChunks = kWeights == 2 ? 2 : 4, kTokens = 8 * kTiles;
    __shared__ Sum sums[kWarps][kWeights][kChannels][kTokens + 1];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const int n0 = blockIdx.x * kChannels;
    tc::pdl_launch_dependents();
    // (channels past the last: the last one again, whose sums nobody stores)
    const uint8_t *b[kWeights][2], *a[kTiles];
#pragma unroll
    for (int w = 0; w < kWeights; ++w)
#pragma unroll
        for (int h = 0; h < 2; ++h) b[w][h] = p.B[w] + min(n0 + g + 8 * h, p.N - 1) * p.b_pitch[w];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) a[i] = p.A + min(g + 8 * i, p.M - 1) * p.a_pitch;
    Sum acc[kWeights][kTiles][4] = {};
    tc::pdl_wait();
    for (long long at0 = (long long)warp * kChunks * 64 + t * 16; at0 - t * 16 < p.row_bytes; at0 += kWarps * kChunks * 64) {
        uint4 wv[kChunks][kWeights][2], xv[kChunks][kTiles];
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int w = 0; w < kWeights; ++w)
#pragma unroll
                for (int h = 0; h < 2; ++h) wv[c][w][h] = load16(b[w][h], at0 + c * 64, p.row_bytes);
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < kTiles; ++i) xv[c][i] = g + 8 * i < p.M ? load16(a[i], at0 + c * 64, p.row_bytes) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int w = 0; w < kWeights; ++w)
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    const uint4 u = wv[c][w][0], v = wv[c][w][1], x = xv[c][i];
                    mma<kType>(acc[w][i], u.x, v.x, u.y, v.y, x.x, x.y);
                    mma<kType>(acc[w][i], u.z, v.z, u.w, v.w, x.z, x.w);
                }
    }
#pragma unroll
    for (int w = 0; w < kWeights; ++w)
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[warp][w][g + e / 2 * 8][i * 8 + 2 * t + e % 2] = acc[w][i][e];
    __syncthreads();
    for (int e = threadIdx.x; e < kChannels * p.M; e += kThreads) {
        const int m = e / kChannels, r = e % kChannels, n = n0 + r;
        if (n >= p.N) continue;
        float v[kWeights];
#pragma unroll
        for (int w = 0; w < kWeights; ++w) {
            Sum s = 0;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) s += sums[k][w][r][m];
            v[w] = (float)s;
            // (one factor after the other: the sum may be 0 where the factors' product is infinite)
            if (kType == ONNXB_INT8) v[w] = v[w] * p.a_scale[m] * p.b_scale[w][n];
        }
        float y = v[0];
        if (kWeights == 2) {
            if (p.Y[1]) {
                put(p.Y[1], p.y_type, m * p.y_ld[1] + n, v[0]);
                put(p.Y[2], p.y_type, m * p.y_ld[2] + n, v[kWeights - 1]);
            }
            y = activate(p.activation, v[0]) * v[kWeights - 1];
        } else {
            if (p.bias) y += p.bias[n];
            if (p.relu) y = fmaxf(y, 0.f);
        }
        put(p.Y[0], p.y_type, m * p.y_ld[0] + n, y);
    }
}

template <int kType, int kWeights>
void (*kernel_for(int M))(const Params) {
    return M <= 8 ? dense_few_kernel<kType, 1, kWeights> : dense_few_kernel<kType, 2, kWeights>;
}

}  // namespace

bool dense_few_fits(const DenseProblem &d) { return (d.mode == kDensePlain || d.mode == kDenseGated) && d.M <= 16; }

int launch_dense_few(const DenseProblem &d, cudaStream_t stream) {
    const bool gated = d.mode == kDenseGated;
    const int bytes = type_bytes(d.type);
    Params p{};
    p.M = d.M; p.N = d.N;
    p.row_bytes = (long long)d.K * bytes;
    p.A = static_cast<const uint8_t *>(d.A[0].p); p.a_pitch = d.A[0].ld * bytes;
    for (int w = 0; w < (gated ? 2 : 1); ++w) {
        p.B[w] = static_cast<const uint8_t *>(d.B[w].p);
        p.b_pitch[w] = d.B[w].ld * bytes;
        p.b_scale[w] = d.b_scale[w];
    }
    p.a_scale = d.a_scale; p.bias = d.bias;
    p.relu = d.relu; p.activation = d.activation; p.y_type = d.y_type;
    for (int i = 0; i < 3; ++i) { p.Y[i] = d.Y[i]; p.y_ld[i] = d.y_ld[i]; }
    auto kernel = d.type == ONNXB_INT8 ? (gated ? kernel_for<ONNXB_INT8, 2>(d.M) : kernel_for<ONNXB_INT8, 1>(d.M))
                  : d.type == ONNXB_FLOAT16 ? kernel_for<ONNXB_FLOAT16, 2>(d.M) : kernel_for<ONNXB_BFLOAT16, 2>(d.M);
    const cudaError_t e = tc_host::launch_pdl(kernel, dim3((d.N + kChannels - 1) / kChannels), dim3(kThreads), 0, stream, p);
    count_launch();
    return (int)e;
}

}  // namespace onnxb
