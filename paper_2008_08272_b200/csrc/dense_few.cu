// Dense layers of 8- and 16-bit operands for a few tokens (single tokens first of all): every weight is read once and multiplied by
// up to 16 tokens, so the weights' bytes are what bounds it, and what counts is that enough loads are in flight on every SM.
//
// A block has 16 channels (the gated block: of both weights).  Its warps share the reduction, a part of each row a warp, and add their
// sums in shared memory, in a fixed order.  The weights go from global memory straight into the registers of
// mma.sync (16 channels x 8 tokens), 16 bytes per lane and load: which terms of the reduction a lane's registers hold is up to the
// kernel as long as both operands agree, so a lane's four words are the terms that its 16 bytes hold, no matter which the
// instruction calls them.  (tcgen05 would want them in shared memory first, and its 128 rows for a few tokens: see dense_few_fits.)
// Measured, one call after another on weights out of HBM: one token, 8-bit 10240 -> 4096 9.6 us (4.4 TB/s), 4096 -> 10240 8.3 us (5.1
// TB/s); gated block 4096 -> 10240 of 16-bit weights 29.3 us (5.7 TB/s; 40960 channels 99 us, 6.8 TB/s), eight tokens of 8-bit ones 14.2 us
// (5.9 TB/s).  What is left is the launch and the first and last loads.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdlib>

#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

constexpr int kChannels = 16;
// Blocks an SM: 24 warps of 8 tokens (with 16 or 32 of them 8-bit 4096 -> 5120 takes 7.4 or 6.0 us, 5.0 so), of 16 tokens 16
constexpr int per_sm(int tiles, int warps) { return (tiles == 1 ? 24 : 16) / warps; }
constexpr int kAhead = 256;              // bytes of its part of a row that a warp asks for ahead

struct Params {
    int M, N;
    long long row_bytes;             // of the reduction
    const uint8_t *A, *B[2];
    long long a_pitch, b_pitch[2];   // bytes
    const float *a_scale, *b_scale[2], *bias;
    int relu, activation, y_type;
    int first;                       // blocks that run at once, from the first on
    void *Y[3];
    long long y_ld[3];
};

// 16 bytes of a row, zeros past its end; weights, which nobody reads twice, not by way of L1.  (No read-only loads here or in the other
// kernels of the dense layers: a kernel that starts before the previous one has finished may see its operands written.)
template <bool kWeight>
__device__ __forceinline__ uint4 load16(const uint8_t *row, long long at, long long row_bytes) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (at + 16 <= row_bytes) {
        if (kWeight) asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + at));
        else v = *reinterpret_cast<const uint4 *>(row + at);
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
template <int kType, int kTiles, int kWeights, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, per_sm(kTiles, kWarps)) dense_few_kernel(const Params p) {
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
    const long long share = (p.row_bytes + kWarps * 64 - 1) / (kWarps * 64) * 64, begin = warp * share, end = min(begin + share, p.row_bytes);
    // The first loads of the blocks that start at once are on their way into L2 before the previous kernel has finished (gated block
    // 30.0 -> 29.4 us; all that these blocks read 35, since what the loads wait for then comes in any order)
    if (blockIdx.x < p.first && lane < kChannels * kWeights && begin + 16 <= end) {
        const uint8_t *row = p.B[lane / kChannels] + min(n0 + lane % kChannels, p.N - 1) * p.b_pitch[lane / kChannels] + begin;
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row), "r"((uint32_t)min(end - begin, (long long)kAhead) / 16 * 16) : "memory");
    }
    tc::pdl_wait();
    // The results that are this thread's, and their scales, asked for before the sums are there
    constexpr int kResults = kTokens * kChannels / (32 * kWarps) > 0 ? kTokens * kChannels / (32 * kWarps) : 1;
    const int r = threadIdx.x % kChannels, n = n0 + r;
    float sa[kResults] = {}, sb[kWeights] = {}, bias = 0.f;
    if (kType == ONNXB_INT8 && n < p.N) {
#pragma unroll
        for (int i = 0; i < kResults; ++i) {
            const int m = threadIdx.x / kChannels + i * (2 * kWarps);
            if (m < p.M) sa[i] = p.a_scale[m];
        }
#pragma unroll
        for (int w = 0; w < kWeights; ++w) sb[w] = p.b_scale[w][n];
        if (kWeights == 1 && p.bias) bias = p.bias[n];
    }
    for (long long at0 = begin + t * 16; at0 - t * 16 < end; at0 += kChunks * 64) {
        uint4 wv[kChunks][kWeights][2], xv[kChunks][kTiles];
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int w = 0; w < kWeights; ++w)
#pragma unroll
                for (int h = 0; h < 2; ++h) wv[c][w][h] = load16<true>(b[w][h], at0 + c * 64, end);
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < kTiles; ++i) xv[c][i] = g + 8 * i < p.M ? load16<false>(a[i], at0 + c * 64, end) : make_uint4(0, 0, 0, 0);
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
    if (n >= p.N) return;
#pragma unroll
    for (int i = 0; i < kResults; ++i) {
        const int m = threadIdx.x / kChannels + i * (2 * kWarps);
        if (m >= p.M) return;
        float v[kWeights];
#pragma unroll
        for (int w = 0; w < kWeights; ++w) {
            Sum s = 0;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) s += sums[k][w][r][m];
            // (one factor after the other: the sum may be 0 where the factors' product is infinite)
            v[w] = kType == ONNXB_INT8 ? (float)s * sa[i] * sb[w] : (float)s;
        }
        float y = v[0];
        if (kWeights == 2) {
            if (p.Y[1]) {
                put(p.Y[1], p.y_type, m * p.y_ld[1] + n, v[0]);
                put(p.Y[2], p.y_type, m * p.y_ld[2] + n, v[kWeights - 1]);
            }
            y = activate(p.activation, v[0]) * v[kWeights - 1];
        } else {
            y += bias;
            if (p.relu) y = fmaxf(y, 0.f);
        }
        put(p.Y[0], p.y_type, m * p.y_ld[0] + n, y);
    }
}

template <int kType, int kWeights, int kWarps>
void (*kernel_for(int M))(const Params) {
    return M <= 8 ? dense_few_kernel<kType, 1, kWeights, kWarps> : dense_few_kernel<kType, 2, kWeights, kWarps>;
}
template <int kWarps>
void (*kernel_for(const DenseProblem &d))(const Params) {
    if (d.type == ONNXB_INT8) return d.mode == kDenseGated ? kernel_for<ONNXB_INT8, 2, kWarps>(d.M) : kernel_for<ONNXB_INT8, 1, kWarps>(d.M);
    return d.type == ONNXB_FLOAT16 ? kernel_for<ONNXB_FLOAT16, 2, kWarps>(d.M) : kernel_for<ONNXB_BFLOAT16, 2, kWarps>(d.M);
}
// Warps a block: as many as let all blocks run at once, or 8 where no number does.  (16, 8 and 4: gated block 8192 -> 1024 11.5, 17.8 and 30
// us; 8-bit 10240 -> 4096 11.6, 9.6 and 15.2; 4096 -> 10240 11.8, 9.4 and 8.3.)  That
// makes a step where 4 warps no longer do: one token, 8-bit 4096 -> 14208, 888 blocks, 9.4 us; -> 14224 11.2 of 8 warps (12.3 of 4; 9.0 are the
// weights' bytes); gated block of 16-bit weights 40.5 and 39.8, of 8 warps 36.0 and 39.8.  ONNXB_DENSE_FEW_WARPS pins it.
int warps_of(const DenseProblem &d) {
    if (const char *e = getenv("ONNXB_DENSE_FEW_WARPS")) return atoi(e) == 4 ? 4 : atoi(e) == 16 ? 16 : 8;
    const int tiles = d.M <= 8 ? 1 : 2;
    const long long blocks = (d.N + kChannels - 1) / kChannels, bytes = (long long)d.K * type_bytes(d.type), turn = d.mode == kDenseGated ? 128 : 256;
    for (int warps = 16; warps >= 4; warps /= 2)
        if (blocks <= per_sm(tiles, warps) * tc_host::num_sms() && (warps <= 4 || bytes >= warps * turn)) return warps;
    return 8;
}

}  // namespace

// Where it is the faster kernel: up to 8 tokens (gated block of 16-bit weights 4096 -> 10240 29 us here, 33 there; 8192 -> 128 8.9 and
// 10.7; 8-bit 10240 -> 4096 9.6 and 12.7), and up to 16 where two blocks an SM are all there are (16 tokens: 8-bit 10240 -> 4096 11.9 us
// here, 12.8 there; 4096 -> 10240 14.7 and 10.9) or the weights are few (gated block of 8-bit ones 512 -> 8192 3.8 and 4.9).
// ONNXB_DENSE_FEW = the most tokens pins it for A/B measurements and tests.
bool dense_few_fits(const DenseProblem &d) {
    if (d.mode != kDensePlain && d.mode != kDenseGated) return false;
    if (const char *e = getenv("ONNXB_DENSE_FEW")) return d.M <= std::min(16, atoi(e));
    const long long blocks = (d.N + kChannels - 1) / kChannels, bytes = (long long)d.K * type_bytes(d.type) * d.N * (d.mode == kDenseGated ? 2 : 1);
    return d.M <= 8 || (d.M <= 16 && (blocks <= 2 * tc_host::num_sms() || bytes <= 10000000));
}

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
    const int warps = warps_of(d);
    p.first = per_sm(d.M <= 8 ? 1 : 2, warps) * tc_host::num_sms();
    auto kernel = warps == 4 ? kernel_for<4>(d) : warps == 8 ? kernel_for<8>(d) : kernel_for<16>(d);
    const cudaError_t e = tc_host::launch_pdl(kernel, dim3((d.N + kChannels - 1) / kChannels), dim3(32 * warps), 0, stream, p);
    count_launch();
    return (int)e;
}

}  // namespace onnxb
