// Products by group for a few rows, those of single tokens first of all: every weight of a group that has a row is read once, and that is what bounds it.
//
// As in dense_few.cu a block has 16 channels (the gated block's: of both weights), its warps share the reduction and add their sums in shared memory in a fixed
// order, and the weights go from global memory straight into the registers of mma.sync, 16 bytes a lane and load, so that as many loads are in flight
// as there are warps.  What is its own: a block is one of a group, or where there are fewer rows than groups of a row, and goes on if that row is its group's
// first, with all of the group's rows, eight at a time.  Which group that is it finds in the offsets: the first of them above the row ends the group, the
// largest before that begins it.  And weights and rows may begin anywhere: nothing is copied, where most groups' weights are not read at all.  Rows of weights that
// do not all begin at multiples of 16 bytes do so alike every eight channels, whatever their pitch: a block then has every eighth channel, reads their pieces
// of 16 bytes as they lie, and the rows of X as far into theirs.  (Each row's pieces put together from two: 72 rows of 86 groups, 633 -> 8166, 373 us, as by a copy.)
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
    int rows, groups, channels, by_group;
    int blocks;                      // of channels
    const int *offsets;
    long long row_bytes;             // of the reduction
    const uint8_t *X, *W[2];
    long long x_pitch, w_pitch[2], w_stride[2];      // bytes
    int activation, type;
    void *Y[3];
    long long y_ld[3];
};

// The 16 bytes from `at` on (a multiple of 16) of weights that begin `before` bytes into their first piece of 16 and end before `end`: a piece as it lies, zeros for what
// is not the row's.  Not by way of L1, since nobody reads them twice.
__device__ __forceinline__ uint4 weights16(const uint8_t *pieces, long long at, int before, long long end) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (at + 16 <= end && at >= before) {
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(pieces + at));
        return v;
    }
    if (at >= end) return v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(pieces + at));
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (at + 2 * i < before || at + 2 * i >= end) w[i / 2] &= i % 2 ? 0x0000FFFFu : 0xFFFF0000u;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The 16 bytes from `at` on (which may be negative) of a row of row_bytes, zeros where they are not the row's
template <bool kAligned>
__device__ __forceinline__ uint4 row16(const uint8_t *row, long long at, long long row_bytes) {
    if (at >= 0 && at + 16 <= row_bytes) {
        if (kAligned) return *reinterpret_cast<const uint4 *>(row + at);
        // (the two aligned pieces that hold them: either has some)
        const int off = (int)(reinterpret_cast<uintptr_t>(row + at) & 15), words = off / 4, bits = off % 4 * 8;
        const uint4 *from = reinterpret_cast<const uint4 *>(row + at - off);
        const uint4 a = from[0], b = off ? from[1] : make_uint4(0, 0, 0, 0);
        uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = words & 2 ? w[i + 2] : w[i];
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = words & 1 ? w[i + 1] : w[i];
        return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; i += 2)
        if (at + i >= 0 && at + i < row_bytes) w[i / 4] |= (uint32_t)*reinterpret_cast<const uint16_t *>(row + at + i) << (i % 4 * 8);
    return make_uint4(w[0], w[1], w[2], w[3]);
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
    const int row = blockIdx.y;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    // The group of this block's row: the first offset above it is its end (offsets that do not rise count as the largest before them)
    int end = p.by_group ? row + 1 : p.groups + 1;
    if (!p.by_group) {
        for (int i = threadIdx.x; i <= p.groups; i += 32 * kWarps)
            if (p.offsets[i] > row) end = min(end, i);
        end = __reduce_min_sync(0xffffffffu, end);
        if (lane == 0) found[0][warp] = end;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) end = min(end, found[0][w]);
        if (end == 0 || end > p.groups) return;          // of no group
    }
    int first = 0;
    for (int i = threadIdx.x; i < end; i += 32 * kWarps) first = max(first, p.offsets[i]);
    first = __reduce_max_sync(0xffffffffu, first);
    if (lane == 0) found[1][warp] = first;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) first = max(first, found[1][w]);
    if (!p.by_group && first != row) return;             // not its first
    const int last = min(p.offsets[end], p.rows), group = end - 1;
    int block = blockIdx.x;
    do {
        // Channels n0 to n0 + 15, or every eighth; those past the last: another of the block's, whose sums nobody stores
        constexpr int each = kAligned ? 1 : 8;
        const int n0 = kAligned ? block * kChannels : block / 8 * 8 * kChannels + block % 8;
        if (n0 >= p.channels) continue;
        const uint8_t *b[kWeights][2];
        int before[kWeights] = {};
#pragma unroll
        for (int w = 0; w < kWeights; ++w)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = n0 + (g + 8 * h) * each;
                b[w][h] = p.W[w] + group * p.w_stride[w] + (n < p.channels ? n : n0) * p.w_pitch[w];
                if (!kAligned) {
                    before[w] = (int)(reinterpret_cast<uintptr_t>(b[w][h]) & 15);
                    b[w][h] -= before[w];
                }
            }
        const long long span = p.row_bytes + (kAligned ? 0 : max(before[0], before[kWeights - 1]));
        const long long share = (span + kWarps * 64 - 1) / (kWarps * 64) * 64, begin = warp * share, stop = min(begin + share, span);
        for (int m0 = first; m0 < last; m0 += kRows) {
            const bool in = m0 + g < last;
            const uint8_t *a = p.X + (in ? m0 + g : m0) * p.x_pitch;
            float acc[kWeights][4] = {};
            for (long long at0 = begin + t * 16; at0 - t * 16 < stop; at0 += kChunks * 64) {
                uint4 wv[kChunks][kWeights][2], xv[kChunks][kAligned ? 1 : kWeights];
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int w = 0; w < kWeights; ++w)
#pragma unroll
                        for (int h = 0; h < 2; ++h) wv[c][w][h] = weights16(b[w][h], at0 + c * 64, before[w], kAligned ? stop : min(stop, p.row_bytes + before[w]));
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int w = 0; w < (kAligned ? 1 : kWeights); ++w)
                        xv[c][w] = in && at0 + c * 64 < stop ? row16<kAligned>(a, at0 + c * 64 - before[w], p.row_bytes) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int w = 0; w < kWeights; ++w) {
                        // (which terms the instruction takes a lane's words for is all the same, as long as both operands agree)
                        const uint4 u = wv[c][w][0], v = wv[c][w][1], x = xv[c][kAligned ? 0 : w];
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
            const int r = threadIdx.x % kChannels, n = n0 + r * each, m = threadIdx.x / kChannels;
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
    } while (!kAligned && (block += gridDim.x) < p.blocks);
}

template <bool kBf16, bool kAligned>
void (*kernel_for(bool gated))(const Params) {
    return gated ? grouped_few_kernel<kBf16, 2, kAligned> : grouped_few_kernel<kBf16, 1, kAligned>;
}

}  // namespace

// Up to 16 rows: 2 rows of 8 groups, gated block 4096 -> 10240, 54.7 us here and 60.6 on the tensor cores, 16 of 64 groups 4096 -> 1408 54.5 and 61.7, one row
// 8192 -> 1024 10.7 and 22.5, whose few tiles read one SM's share of the bandwidth each; but 32 of 64 groups 1408 -> 2048 34 and 26.4.  And where the tensor
// cores would have the weights copied first (they begin at other than multiples of 16 bytes), up to 128 rows, of 4 a group on average, that are long enough.  How the rows lie the
// host does not know: weights are read once for every eight rows of a group, so that rows all of one group cost what even ones gain.  Here and on the tensor cores, rows lying
// evenly and all in one group: 72 rows of 86 groups, 633 -> 8166, 305 and 544 us, 86 and 62; 128 of 128, 1409 -> 2048, 227 and 471, 80 and 33; 64 of 16, 4097 -> 4096, 139 and 326,
// 108 and 33; 128 of 1024, 513 -> 264, 31 and 63, 109 and 45.  More rows, 512 of 128, 1409 -> 2048: 233 and 473, 309 and 39; 4096 of 1024, 513 -> 264: 190 and 266, 3660 and 56.
// Shorter ones, 49 of 30 groups, gated block 197 -> 2176: 46 and 59, 115 and 18.
// ONNXB_GROUPED_FEW = the most rows pins it for A/B measurements and tests.
bool grouped_few_fits(int rows, int groups, int width, bool in_place) {
    if (const char *e = getenv("ONNXB_GROUPED_FEW")) return rows <= atoi(e);
    return rows <= 16 || (!in_place && rows <= std::min(128, 4 * groups) && width >= 512);
}

int launch_grouped_few(const GroupedProblem &d, cudaStream_t stream) {
    const bool gated = d.mode == kGroupedGated;
    Params p{};
    p.rows = d.rows; p.groups = d.groups; p.channels = d.channels; p.offsets = d.offsets;
    p.by_group = d.rows >= d.groups;
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
    p.blocks = aligned ? (d.channels + kChannels - 1) / kChannels : (d.channels + 8 * kChannels - 1) / (8 * kChannels) * 8;
    // (a block has several times 16 channels of short rows that begin anywhere, 64 KB of weights, so that finding its group costs less than these; as long as there
    // are blocks for all SMs.  72 rows of 86 groups, 633 -> 8166: 259 -> 220 us.)
    const int groups = std::min(d.rows, d.groups);
    const long long several = aligned ? 1 : std::max(1ll, std::min(65536 / (kChannels * p.row_bytes * (gated ? 2 : 1)), (long long)p.blocks * groups / (148 * 3)));
    const dim3 grid((unsigned)((p.blocks + several - 1) / several), (unsigned)groups);
    const cudaError_t e = tc_host::launch_pdl(kernel, grid, dim3(32 * kWarps), 0, stream, p);
    count_launch();
    return (int)e;
}

}  // namespace onnxb
