// onnx_layer_normalization_run and its gradients.
//
// Bound by the bytes of X and Y (of dY, X and dX), so every element is read once: a row fits the registers of the threads that share it (a warp
// for short rows, a block of up to 1024 threads for longer ones), which first agree on its sums and then compute from what they hold.
// The mean is taken away before the squares are added up, in 32 bits: a row far from zero loses nothing.  A block takes two rows at once, so that
// twice the loads are in flight, the weights are read once for both, and its threads wait for one another once.
//
// The weights' gradients are sums over the rows: a block's threads add up their columns over its rows (in registers, or in shared
// memory where a thread has many), each block leaves its sums in the workspace, and a second kernel adds those up, in their order.
// Longer rows than a block's registers hold are read again, out of L2.
#include <algorithm>

#include "dense_math.cuh"
#include "layer_norm.h"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

// What a thread reads at once: 16 bytes.  kAligned: rows of whole pieces that begin at multiples of 16 bytes in all tensors.  Else rows begin
// anywhere, and the last piece has less.
template <typename T, bool kAligned>
struct Piece {
    static constexpr int kCount = 16 / sizeof(T);
    uint4 bits;
    __device__ __forceinline__ void clear() { bits = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const T *row, int K, int i) {
        bits = kAligned ? reinterpret_cast<const uint4 *>(row)[i]
                        : load16_anywhere<sizeof(T)>(reinterpret_cast<const uint8_t *>(row), i * 16ll, K * (long long)sizeof(T));
    }
    __device__ __forceinline__ float at(int e) const { return to_float(reinterpret_cast<const T *>(&bits)[e]); }
    __device__ __forceinline__ void set(int e, float v) { reinterpret_cast<T *>(&bits)[e] = from_float<T>(v); }
    __device__ __forceinline__ void store(T *row, int K, int i) const {
        T *to = row + (long long)i * kCount;
        if (kAligned || (reinterpret_cast<uintptr_t>(to) % 16 == 0 && (i + 1ll) * kCount <= K)) {
            *reinterpret_cast<uint4 *>(to) = bits;
        } else {
#pragma unroll
            for (int e = 0; e < kCount; ++e)
                if ((long long)i * kCount + e < K) to[e] = reinterpret_cast<const T *>(&bits)[e];
        }
    }
    // Whether element e of piece i is the row's
    __device__ __forceinline__ static bool has(int K, int i, int e) { return kAligned || (long long)i * kCount + e < K; }
};

// kCount weights from the i-th piece's first on (zeros behind the last)
template <typename W, bool kAligned, int kCount>
__device__ __forceinline__ void load_weights(const W *w, int K, int i, float (&v)[kCount]) {
    if (kAligned) {
        constexpr int kEach = 16 / sizeof(W);
#pragma unroll
        for (int part = 0; part < kCount; part += kEach) {
            const uint4 bits = reinterpret_cast<const uint4 *>(w + (long long)i * kCount)[part / kEach];
#pragma unroll
            for (int e = 0; e < kEach; ++e) v[part + e] = to_float(reinterpret_cast<const W *>(&bits)[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
            const long long at = (long long)i * kCount + e;
            v[e] = at < K ? to_float(w[at]) : 0.f;
        }
    }
}

// Sums over a row's threads, a warp's or the whole block's, of kSums values each, which all of them get.  `shared`: kSums values for each of 32
// warps, in which nobody reads or writes anything else at the time.
template <int kThreads, int kSums>
__device__ __forceinline__ void sum_over_row(float (&v)[kSums], float (*shared)[32]) {
#pragma unroll
    for (int s = 0; s < kSums; ++s)
#pragma unroll
        for (int o = 16; o > 0; o /= 2) v[s] += __shfl_xor_sync(0xffffffffu, v[s], o);
    if (kThreads > 32) {
        constexpr int kWarps = kThreads / 32;
        if (threadIdx.x % 32 == 0)
#pragma unroll
            for (int s = 0; s < kSums; ++s) shared[s][threadIdx.x / 32] = v[s];
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kSums; ++s) {
            v[s] = shared[s][threadIdx.x % kWarps];
#pragma unroll
            for (int o = kWarps / 2; o > 0; o /= 2) v[s] += __shfl_xor_sync(0xffffffffu, v[s], o);
        }
    }
}

struct Forward {
    int M, K, pieces;
    const void *X, *scale, *bias;
    long long x_ld, y_ld;
    void *Y;
    float *mean, *inv_std;
    float epsilon, per_row;      // 1 / K
};

// kThreads threads a row, kPieces pieces a thread at most, kRows rows at once; a warp a row: 8 rows a block
template <typename T, typename W, bool kAligned, int kThreads, int kPieces, int kRows>
__global__ void __launch_bounds__(kThreads < 256 ? 256 : kThreads) layer_norm_kernel(const Forward p) {
    typedef Piece<T, kAligned> P;
    constexpr int kCount = P::kCount;
    static_assert(kThreads > 32 || kRows == 1, "a warp has one row");
    __shared__ float shared[2][kRows][32];
    const int at = threadIdx.x % kThreads;
    const long long i0 = kThreads == 32 ? (long long)blockIdx.x * 8 + threadIdx.x / 32 : (long long)blockIdx.x * kRows;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    P v[kRows][kPieces];
    float sum[kRows] = {}, squares[kRows] = {};
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            if (i0 + r < p.M && at + k * kThreads < p.pieces) v[r][k].load(static_cast<const T *>(p.X) + (i0 + r) * p.x_ld, p.K, at + k * kThreads);
            else v[r][k].clear();
        }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
            for (int e = 0; e < kCount; ++e) sum[r] += v[r][k].at(e);
    sum_over_row<kThreads, kRows>(sum, shared[0]);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        sum[r] *= p.per_row;
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
            if (at + k * kThreads < p.pieces)
#pragma unroll
                for (int e = 0; e < kCount; ++e) {
                    const float d = v[r][k].at(e) - sum[r];
                    if (P::has(p.K, at + k * kThreads, e)) squares[r] = fmaf(d, d, squares[r]);
                }
    }
    sum_over_row<kThreads, kRows>(squares, shared[1]);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        squares[r] = __frsqrt_rn(fmaf(squares[r], p.per_row, p.epsilon));
        if (at == 0 && i0 + r < p.M && p.mean) {
            p.mean[i0 + r] = sum[r];
            p.inv_std[i0 + r] = squares[r];
        }
    }
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        if (at + k * kThreads >= p.pieces) continue;
        float scale[kCount], bias[kCount] = {};
        load_weights<W, kAligned, kCount>(static_cast<const W *>(p.scale), p.K, at + k * kThreads, scale);
        if (p.bias) load_weights<W, kAligned, kCount>(static_cast<const W *>(p.bias), p.K, at + k * kThreads, bias);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (i0 + r >= p.M) continue;
            P y;
#pragma unroll
            for (int e = 0; e < kCount; ++e) y.set(e, fmaf((v[r][k].at(e) - sum[r]) * squares[r], scale[e], bias[e]));
            y.store(static_cast<T *>(p.Y) + (i0 + r) * p.y_ld, p.K, at + k * kThreads);
        }
    }
}

// Longer rows: read three times
template <typename T, typename W, bool kAligned>
__global__ void __launch_bounds__(1024) layer_norm_long_kernel(const Forward p) {
    typedef Piece<T, kAligned> P;
    constexpr int kCount = P::kCount;
    __shared__ float shared[2][1][32];
    const long long i = blockIdx.x;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const T *x = static_cast<const T *>(p.X) + i * p.x_ld;
    P v;
    float sum[1] = {}, squares[1] = {};
#pragma unroll 4
    for (int k = threadIdx.x; k < p.pieces; k += 1024) {
        v.load(x, p.K, k);
#pragma unroll
        for (int e = 0; e < kCount; ++e) sum[0] += v.at(e);
    }
    sum_over_row<1024, 1>(sum, shared[0]);
    const float mean = sum[0] * p.per_row;
#pragma unroll 4
    for (int k = threadIdx.x; k < p.pieces; k += 1024) {
        v.load(x, p.K, k);
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
            const float d = v.at(e) - mean;
            if (P::has(p.K, k, e)) squares[0] = fmaf(d, d, squares[0]);
        }
    }
    sum_over_row<1024, 1>(squares, shared[1]);
    const float inv_std = __frsqrt_rn(fmaf(squares[0], p.per_row, p.epsilon));
    if (threadIdx.x == 0 && p.mean) {
        p.mean[i] = mean;
        p.inv_std[i] = inv_std;
    }
#pragma unroll 2
    for (int k = threadIdx.x; k < p.pieces; k += 1024) {
        float scale[kCount], bias[kCount] = {};
        load_weights<W, kAligned, kCount>(static_cast<const W *>(p.scale), p.K, k, scale);
        if (p.bias) load_weights<W, kAligned, kCount>(static_cast<const W *>(p.bias), p.K, k, bias);
        v.load(x, p.K, k);
#pragma unroll
        for (int e = 0; e < kCount; ++e) v.set(e, fmaf((v.at(e) - mean) * inv_std, scale[e], bias[e]));
        v.store(static_cast<T *>(p.Y) + i * p.y_ld, p.K, k);
    }
}

struct Backward {
    int M, K, pieces;
    const void *dY, *X, *scale;
    long long dy_ld, x_ld, dx_ld;
    void *dX;
    const float *mean, *inv_std;
    float *partial;              // for each block its sums of dY n, then of dY; NULL where no weights' gradient is wanted
    long long pitch;             // floats of one of these
    float per_row;
};

// dX = inv_std (d - mean(d) - n mean(d n)), n = (x - mean) inv_std, d = dY scale.  kShared: the columns' sums are kept in shared memory.
template <typename T, typename W, bool kAligned, int kThreads, int kPieces, int kRows, bool kShared>
__global__ void __launch_bounds__(kThreads < 256 ? 256 : kThreads, kThreads <= 256 ? 2 : 1) layer_norm_grad_kernel(const Backward p) {
    typedef Piece<T, kAligned> P;
    constexpr int kCount = P::kCount, kBlock = kThreads < 256 ? 256 : kThreads, kGroups = kBlock / kThreads;      // rows that a block's warps have at once
    extern __shared__ float4 dynamic[];
    __shared__ float shared[2][2 * kRows][32];
    const int at = threadIdx.x % kThreads, group = threadIdx.x / kThreads;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    float by_n[kShared ? 1 : kPieces][kCount] = {}, plain[kShared ? 1 : kPieces][kCount] = {};
    float *kept = reinterpret_cast<float *>(dynamic);        // [2][pieces * kCount]
    if (kShared && p.partial) {
        for (int i = threadIdx.x; i < 2 * p.pieces * kCount; i += kBlock) kept[i] = 0.f;
        // (a thread's own columns are all that it reads of these until the end, but others have cleared them)
        __syncthreads();
    }
    int turn = 0;
    const long long step = (long long)gridDim.x * kRows * kGroups;
    // (a warp that has no row any more leaves the loop by itself; a block's threads share their rows and leave together)
    for (long long i0 = ((long long)blockIdx.x * kGroups + group) * kRows; i0 < p.M; i0 += step, turn ^= 1) {
        P dy[kRows][kPieces], x[kRows][kPieces];
        float mean[kRows], inv_std[kRows], sums[2 * kRows] = {};
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const bool in = i0 + r < p.M;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                dy[r][k].clear();
                x[r][k].clear();
                if (in && at + k * kThreads < p.pieces) {
                    dy[r][k].load(static_cast<const T *>(p.dY) + (i0 + r) * p.dy_ld, p.K, at + k * kThreads);
                    x[r][k].load(static_cast<const T *>(p.X) + (i0 + r) * p.x_ld, p.K, at + k * kThreads);
                }
            }
            mean[r] = in ? p.mean[i0 + r] : 0.f;
            inv_std[r] = in ? p.inv_std[i0 + r] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int piece = at + k * kThreads;
            if (piece >= p.pieces) continue;
            float scale[kCount] = {};
            if (p.dX) load_weights<W, kAligned, kCount>(static_cast<const W *>(p.scale), p.K, piece, scale);
            float a[kCount] = {}, b[kCount] = {};
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int e = 0; e < kCount; ++e) {
                    const float g = dy[r][k].at(e), n = (x[r][k].at(e) - mean[r]) * inv_std[r], d = g * scale[e];
                    sums[2 * r] += d;
                    // (behind a row's end n is no number of the row's, but d and g are zeros)
                    if (P::has(p.K, piece, e)) sums[2 * r + 1] = fmaf(d, n, sums[2 * r + 1]);
                    a[e] = fmaf(g, n, a[e]);
                    b[e] += g;
                }
            if (kShared) {
                if (p.partial) {
#pragma unroll
                    for (int e = 0; e < kCount; e += 4) {
                        float4 &to_n = *reinterpret_cast<float4 *>(kept + piece * kCount + e), &to = *reinterpret_cast<float4 *>(kept + (p.pieces + piece) * kCount + e);
                        to_n = make_float4(to_n.x + a[e], to_n.y + a[e + 1], to_n.z + a[e + 2], to_n.w + a[e + 3]);
                        to = make_float4(to.x + b[e], to.y + b[e + 1], to.z + b[e + 2], to.w + b[e + 3]);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < kCount; ++e) {
                    by_n[kShared ? 0 : k][e] += a[e];
                    plain[kShared ? 0 : k][e] += b[e];
                }
            }
        }
        if (!p.dX) continue;
        // (in turns: a warp may write the next rows' sums while another still reads these)
        sum_over_row<kThreads, 2 * kRows>(sums, shared[turn]);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int piece = at + k * kThreads;
            if (piece >= p.pieces) continue;
            float scale[kCount];
            load_weights<W, kAligned, kCount>(static_cast<const W *>(p.scale), p.K, piece, scale);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                if (i0 + r >= p.M) continue;
                const float level = sums[2 * r] * p.per_row, along = sums[2 * r + 1] * p.per_row;
                P dx;
#pragma unroll
                for (int e = 0; e < kCount; ++e) {
                    const float n = (x[r][k].at(e) - mean[r]) * inv_std[r];
                    dx.set(e, inv_std[r] * (fmaf(dy[r][k].at(e), scale[e], -level) - n * along));
                }
                dx.store(static_cast<T *>(p.dX) + (i0 + r) * p.dx_ld, p.K, piece);
            }
        }
    }
    if (!p.partial) return;
    float *out = p.partial + 2 * p.pitch * blockIdx.x;
    if (kGroups > 1) {
        // the warps' columns, added up in the warps' order
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
            for (int e = 0; e < kCount; ++e) {
                const int c = (k * kThreads + at) * kCount + e;
                kept[(group * 2 + 0) * (kThreads * kPieces * kCount) + c] = by_n[kShared ? 0 : k][e];
                kept[(group * 2 + 1) * (kThreads * kPieces * kCount) + c] = plain[kShared ? 0 : k][e];
            }
        __syncthreads();
        constexpr int kWide = kThreads * kPieces * kCount;
        for (int c = threadIdx.x; c < 2 * kWide; c += kBlock) {
            float sum = 0.f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) sum += kept[g * 2 * kWide + c];
            const int which = c / kWide, col = c % kWide;
            if (col < p.K) out[which * p.pitch + col] = sum;
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        const int piece = at + k * kThreads;
        if (piece >= p.pieces) continue;
#pragma unroll
        for (int e = 0; e < kCount; ++e)
            if (P::has(p.K, piece, e)) {
                out[piece * kCount + e] = kShared ? kept[piece * kCount + e] : by_n[kShared ? 0 : k][e];
                out[p.pitch + piece * kCount + e] = kShared ? kept[(p.pieces + piece) * kCount + e] : plain[kShared ? 0 : k][e];
            }
    }
}

// Longer rows: dX by a block a row, which reads it twice
template <typename T, typename W, bool kAligned>
__global__ void __launch_bounds__(1024) layer_norm_grad_long_kernel(const Backward p) {
    typedef Piece<T, kAligned> P;
    constexpr int kCount = P::kCount;
    __shared__ float shared[2][32];
    const long long i = blockIdx.x;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const T *g = static_cast<const T *>(p.dY) + i * p.dy_ld, *x = static_cast<const T *>(p.X) + i * p.x_ld;
    const float mean = p.mean[i], inv_std = p.inv_std[i];
    P dy, v;
    float sums[2] = {};
#pragma unroll 2
    for (int k = threadIdx.x; k < p.pieces; k += 1024) {
        float scale[kCount];
        load_weights<W, kAligned, kCount>(static_cast<const W *>(p.scale), p.K, k, scale);
        dy.load(g, p.K, k);
        v.load(x, p.K, k);
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
            const float d = dy.at(e) * scale[e];
            sums[0] += d;
            if (P::has(p.K, k, e)) sums[1] = fmaf(d, (v.at(e) - mean) * inv_std, sums[1]);
        }
    }
    sum_over_row<1024, 2>(sums, shared);
    const float level = sums[0] * p.per_row, along = sums[1] * p.per_row;
#pragma unroll 2
    for (int k = threadIdx.x; k < p.pieces; k += 1024) {
        float scale[kCount];
        load_weights<W, kAligned, kCount>(static_cast<const W *>(p.scale), p.K, k, scale);
        dy.load(g, p.K, k);
        v.load(x, p.K, k);
#pragma unroll
        for (int e = 0; e < kCount; ++e) {
            const float n = (v.at(e) - mean) * inv_std;
            dy.set(e, inv_std * (fmaf(dy.at(e), scale[e], -level) - n * along));
        }
        dy.store(static_cast<T *>(p.dX) + i * p.dx_ld, p.K, k);
    }
}
// and the columns' sums of some rows by blocks of 32 pieces by 8 rows
template <typename T, bool kAligned>
__global__ void __launch_bounds__(256) layer_norm_columns_kernel(const Backward p) {
    typedef Piece<T, kAligned> P;
    constexpr int kCount = P::kCount;
    __shared__ float sums[8][2][32 * kCount + 1];
    const int lane = threadIdx.x % 32, group = threadIdx.x / 32, piece = blockIdx.x * 32 + lane;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    float a[kCount] = {}, b[kCount] = {};
    if (piece < p.pieces) {
#pragma unroll 2
        for (long long i = blockIdx.y * 8 + group; i < p.M; i += gridDim.y * 8) {
            P dy, x;
            dy.load(static_cast<const T *>(p.dY) + i * p.dy_ld, p.K, piece);
            x.load(static_cast<const T *>(p.X) + i * p.x_ld, p.K, piece);
            const float mean = p.mean[i], inv_std = p.inv_std[i];
#pragma unroll
            for (int e = 0; e < kCount; ++e) {
                a[e] = fmaf(dy.at(e), (x.at(e) - mean) * inv_std, a[e]);
                b[e] += dy.at(e);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < kCount; ++e) {
        sums[group][0][lane * kCount + e] = a[e];
        sums[group][1][lane * kCount + e] = b[e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 64 * kCount; c += 256) {
        const int which = c / (32 * kCount), col = c % (32 * kCount);
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < 8; ++g) sum += sums[g][which][col];
        const long long at = (long long)blockIdx.x * 32 * kCount + col;
        if (at < p.K) p.partial[(2ll * blockIdx.y + which) * p.pitch + at] = sum;
    }
}

// What the blocks left, added up: 64 columns a block, four a thread, 32 groups of threads with a share of the blocks each.  dScale's columns
// first, then dB's.
template <typename W>
__global__ void __launch_bounds__(512) layer_norm_sums_kernel(int K, int blocks, const float *partial, long long pitch, W *d_scale, W *d_bias) {
    __shared__ float4 sums[32][16];
    const int lane = threadIdx.x % 16, group = threadIdx.x / 16, which = blockIdx.y;
    const long long c = ((long long)blockIdx.x * 16 + lane) * 4;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    W *out = which ? d_bias : d_scale;
    if (!out) return;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < pitch) {
#pragma unroll 4
        for (int b = group; b < blocks; b += 32) {
            const float4 v = *reinterpret_cast<const float4 *>(partial + (2ll * b + which) * pitch + c);
            sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
    }
    sums[group][lane] = sum;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const long long at = (long long)blockIdx.x * 64 + threadIdx.x;
    if (at >= K) return;
    float total = 0.f;
#pragma unroll
    for (int g = 0; g < 32; ++g) total += reinterpret_cast<const float *>(&sums[g][threadIdx.x / 4])[threadIdx.x % 4];
    out[at] = from_float<W>(total);
}

bool at_16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

template <typename T, typename W, bool kAligned>
int launch(const Forward &p, cudaStream_t stream) {
    auto run = [&](auto kernel, int threads, int rows) {
        return (int)tc_host::launch_pdl(kernel, dim3((unsigned)(((long long)p.M + rows - 1) / rows)), dim3(threads), 0, stream, p);
    };
    // (two rows at once where there are blocks for all SMs all the same)
    const bool two = p.M > 2 * 148;
    if (p.pieces <= 32) return run(layer_norm_kernel<T, W, kAligned, 32, 1, 1>, 256, 8);
    if (p.pieces <= 128) return run(layer_norm_kernel<T, W, kAligned, 32, 4, 1>, 256, 8);
    if (p.pieces <= 512) return two ? run(layer_norm_kernel<T, W, kAligned, 256, 2, 2>, 256, 2) : run(layer_norm_kernel<T, W, kAligned, 256, 2, 1>, 256, 1);
    if (p.pieces <= 1024) return two ? run(layer_norm_kernel<T, W, kAligned, 512, 2, 2>, 512, 2) : run(layer_norm_kernel<T, W, kAligned, 512, 2, 1>, 512, 1);
    if (p.pieces <= 2048) return run(layer_norm_kernel<T, W, kAligned, 1024, 2, 1>, 1024, 1);
    if (p.pieces <= 4096) return run(layer_norm_kernel<T, W, kAligned, 1024, 4, 1>, 1024, 1);
    return run(layer_norm_long_kernel<T, W, kAligned>, 1024, 1);
}

// How the gradients' kernel for rows of so many pieces is made: threads a block, rows that it takes at once, whether its columns' sums are in shared
// memory; and how many blocks there are, each of which leaves sums of all columns (from the sizes alone, since the workspace depends on it:
// a B200 has 148 SMs).
struct GradShape {
    int threads, rows, blocks;
    size_t smem;
    bool held;                   // false: longer rows
};
constexpr size_t kMostKept = 200 * 1024;
GradShape grad_shape(int element, int M, int K) {
    const int count = 16 / element, pieces = (K + count - 1) / count;
    GradShape s{};
    s.held = true;
    int most = 148;
    if (pieces <= 64) { s.threads = 256; s.rows = 8; most = 148 * 4; s.smem = (size_t)8 * 2 * 32 * (pieces <= 32 ? 1 : 2) * count * 4; }
    else if (pieces <= 256) { s.threads = 256; s.rows = 2; most = 148 * 4; }
    else if (pieces <= 512) { s.threads = 512; s.rows = 2; most = 148 * 2; }
    else if (pieces <= 1024) { s.threads = 1024; s.rows = 1; }
    else {
        s.threads = 1024;
        s.rows = 1;
        s.smem = (size_t)2 * pieces * count * 4;
        s.held = pieces <= 4096 && s.smem <= kMostKept;
    }
    if (!s.held) {
        s.blocks = std::max(1, std::min(64, (M + 63) / 64));
        return s;
    }
    // (a block's sums cost what a row does: four rows at least, unless SMs would have none)
    const int turns = (int)(((long long)M + s.rows - 1) / s.rows);
    s.blocks = std::max(1, std::min({turns, most, std::max(148, turns / 4)}));
    return s;
}
long long grad_pitch(int K) { return (K + 3ll) / 4 * 4; }

template <typename T, typename W, bool kAligned>
int launch(const Backward &p, const GradShape &s, cudaStream_t stream) {
    auto run = [&](auto kernel) {
        if (s.smem > 48 * 1024) {
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostKept);
            if (e != cudaSuccess) return (int)e;
        }
        return (int)tc_host::launch_pdl(kernel, dim3(s.blocks), dim3(s.threads), s.smem, stream, p);
    };
    if (s.held) {
        if (p.pieces <= 32) return run(layer_norm_grad_kernel<T, W, kAligned, 32, 1, 1, false>);
        if (p.pieces <= 64) return run(layer_norm_grad_kernel<T, W, kAligned, 32, 2, 1, false>);
        if (p.pieces <= 256) return run(layer_norm_grad_kernel<T, W, kAligned, 256, 1, 2, false>);
        if (p.pieces <= 512) return run(layer_norm_grad_kernel<T, W, kAligned, 512, 1, 2, false>);
        if (p.pieces <= 1024) return run(layer_norm_grad_kernel<T, W, kAligned, 1024, 1, 1, false>);
        if (p.pieces <= 2048) return run(layer_norm_grad_kernel<T, W, kAligned, 1024, 2, 1, true>);
        return run(layer_norm_grad_kernel<T, W, kAligned, 1024, 4, 1, true>);
    }
    int err = 0;
    if (p.dX) {
        err = (int)tc_host::launch_pdl(layer_norm_grad_long_kernel<T, W, kAligned>, dim3(p.M), dim3(1024), 0, stream, p);
        if (p.partial) count_launch();
    }
    if (err == 0 && p.partial) err = (int)tc_host::launch_pdl(layer_norm_columns_kernel<T, kAligned>, dim3((p.pieces + 31) / 32, s.blocks), dim3(256), 0, stream, p);
    return err;
}

template <typename W>
int launch_sums(int K, int blocks, const float *partial, void *d_scale, void *d_bias, cudaStream_t stream) {
    const long long pitch = grad_pitch(K);
    return (int)tc_host::launch_pdl(layer_norm_sums_kernel<W>, dim3((unsigned)((pitch + 63) / 64), 2), dim3(512), 0, stream, K, blocks, partial, pitch,
                                    static_cast<W *>(d_scale), static_cast<W *>(d_bias));
}

// f(a value of T, a value of W) for the types' codes
template <typename F>
int by_types(int type, int weight_type, F f) {
    if (type == ONNXB_FLOAT) return f(float(), float());
    if (type == ONNXB_FLOAT16) return weight_type == ONNXB_FLOAT ? f(__half(), float()) : f(__half(), __half());
    return weight_type == ONNXB_FLOAT ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
}

}  // namespace

int launch_layer_norm(const LayerNormProblem &p, cudaStream_t stream) {
    const int err = by_types(p.type, p.weight_type, [&](auto t, auto w) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        constexpr int kCount = 16 / sizeof(T);
        const Forward f{p.M, p.K, (p.K + kCount - 1) / kCount, p.X.p, p.scale, p.bias, p.X.ld, p.Y.ld, const_cast<void *>(p.Y.p), p.mean, p.inv_std, p.epsilon,
                        (float)(1.0 / p.K)};
        const bool aligned = p.K % kCount == 0 && at_16(p.X.p) && at_16(p.Y.p) && at_16(p.scale) && at_16(p.bias) &&
                             (p.M == 1 || (p.X.ld % kCount == 0 && p.Y.ld % kCount == 0));
        return aligned ? launch<T, W, true>(f, stream) : launch<T, W, false>(f, stream);
    });
    count_launch();
    return err;
}

size_t layer_norm_grad_workspace(int type, int M, int K, bool weights) {
    return weights ? (size_t)(grad_shape(type_bytes(type), M, K).blocks * 2 * grad_pitch(K)) * 4 : 0;
}

int launch_layer_norm_grad(const LayerNormGradProblem &p, cudaStream_t stream) {
    const GradShape s = grad_shape(type_bytes(p.type), p.M, p.K);
    const bool weights = p.d_scale || p.d_bias;
    int err = by_types(p.type, p.weight_type, [&](auto t, auto w) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        constexpr int kCount = 16 / sizeof(T);
        const Backward b{p.M, p.K, (p.K + kCount - 1) / kCount, p.dY.p, p.X.p, p.scale, p.dY.ld, p.X.ld, p.dX.ld, const_cast<void *>(p.dX.p), p.mean, p.inv_std,
                         weights ? static_cast<float *>(p.partial) : nullptr, grad_pitch(p.K), (float)(1.0 / p.K)};
        const bool aligned = p.K % kCount == 0 && at_16(p.dY.p) && at_16(p.X.p) && at_16(p.dX.p) && at_16(p.scale) &&
                             (p.M == 1 || (p.dY.ld % kCount == 0 && p.X.ld % kCount == 0 && p.dX.ld % kCount == 0));
        return aligned ? launch<T, W, true>(b, s, stream) : launch<T, W, false>(b, s, stream);
    });
    count_launch();
    if (err == 0 && weights) {
        err = p.weight_type == ONNXB_FLOAT     ? launch_sums<float>(p.K, s.blocks, static_cast<const float *>(p.partial), p.d_scale, p.d_bias, stream)
              : p.weight_type == ONNXB_FLOAT16 ? launch_sums<__half>(p.K, s.blocks, static_cast<const float *>(p.partial), p.d_scale, p.d_bias, stream)
                                               : launch_sums<__nv_bfloat16>(p.K, s.blocks, static_cast<const float *>(p.partial), p.d_scale, p.d_bias, stream);
        count_launch();
    }
    return err;
}

}  // namespace onnxb
