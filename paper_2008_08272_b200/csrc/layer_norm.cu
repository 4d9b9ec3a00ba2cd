// onnx_layer_normalization_run and its gradients.
//
// Bound by the bytes of X and Y (of dY, X and dX): every element is read once, and what counts is that enough of them are on their way while others are
// computed with.  The mean is taken away before the squares are added up, in 32 bits; what the mean of a row far from zero, a sum of 32 bits, is off by is the mean of
// what is left, added up beside the squares and taken away, too: such a row loses nothing but what rounding takes of the mean that is kept.
//
// Forward: a row is held in registers, by one warp up to 1024 elements of 16 bits, which then waits for nobody, and by 2 to 16 warps up to 32768 (4096: 4 warps,
// two rows at once); of few rows by as many threads as leave each two pieces or four.  The SM's other rows hide what one waits for.
//
// Gradients: a thread adds up its 8 or 16 columns over its block's rows, so all columns of a row have to be a block's (of long rows a cluster's).  The block
// brings its next rows by asynchronous bulk copies into a ring in shared memory, takes one or two of them into registers, agrees on their sums,
// and computes their dX.  Agreeing is most of the work beside the bytes: of 4 sums over a warp a lane ends up with one (6 exchanges instead of 20: 16384 x 4096
// of bf16 106 -> 76 us).  Each block leaves its columns' sums in the workspace, and a second kernel adds those up, in their order.
// Rows of any alignment are copied from the multiple of 16 bytes before to the one behind them; rows that are not all at such multiples are read from there,
// and written, element by element, neighbours by neighbouring threads.
// Products whose rounding could be left out are written as such (__fmul_rn): the compiler would do so in one branch and not in another, and a result
// is to be the same bit by bit whichever others are wanted.
#include <algorithm>
#include <type_traits>

#include "dense_math.cuh"
#include "layer_norm.h"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

// Two 16-bit numbers of a word, and a word of two
__device__ __forceinline__ float low(uint32_t w, __half) { return __low2float(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ float high(uint32_t w, __half) { return __high2float(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ float low(uint32_t w, __nv_bfloat16) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w, __nv_bfloat16) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t word(float a, float b, __half) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t word(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Two elements at once: Blackwell's additions and multiplications of pairs of 32-bit numbers, each rounded as the single ones are.  (An instruction less for
// every second element: these kernels would be bound by their instructions otherwise.)
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 add(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 mul(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }

// A thread's k-th part of a row of n parts: 16 bytes where rows are whole such pieces that begin at multiples of 16 bytes in all tensors.
// again(): what has been made of the bits until here is to be made anew, not kept.  (The compiler keeps every element as 32 bits otherwise, for which there are
// no registers: 171 of them for 16 parts of bf16, and one block an SM.)
template <typename T, bool kWhole, int kThreads>
struct Part {
    static constexpr int kCount = 16 / sizeof(T), kPairs = kCount / 2;
    uint32_t w[4];
    __device__ __forceinline__ static bool any(int at, int k, int n) { return at + k * kThreads < n; }
    __device__ __forceinline__ void load(const T *row, int at, int k, int) {
        const uint4 v = reinterpret_cast<const uint4 *>(row)[at + k * kThreads];
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
    __device__ __forceinline__ float2 pair(int i) const {
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        else return make_float2(low(w[i], T()), high(w[i], T()));
    }
    __device__ __forceinline__ void set(int i, float2 v) {
        if constexpr (sizeof(T) == 4) {
            w[2 * i] = __float_as_uint(v.x);
            w[2 * i + 1] = __float_as_uint(v.y);
        } else {
            w[i] = word(v.x, v.y, T());
        }
    }
    __device__ __forceinline__ static float2 own(float2 v, int, int, int) { return v; }
    __device__ __forceinline__ void again() { asm volatile("" : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])); }
    __device__ __forceinline__ void store(T *row, int at, int k, int) const { reinterpret_cast<uint4 *>(row)[at + k * kThreads] = make_uint4(w[0], w[1], w[2], w[3]); }
    // weights, and columns' sums
    template <typename W>
    __device__ __forceinline__ static void weights(const W *from, int at, int k, int, float2 (&v)[kPairs]) {
        from += (long long)(at + k * kThreads) * kCount;
        constexpr int kEach = 16 / sizeof(W);
#pragma unroll
        for (int part = 0; part < kCount / kEach; ++part) {
            const uint4 bits = reinterpret_cast<const uint4 *>(from)[part];
            const uint32_t b[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
            for (int i = 0; i < kEach / 2; ++i) {
                if constexpr (sizeof(W) == 4) v[part * 2 + i] = make_float2(__uint_as_float(b[2 * i]), __uint_as_float(b[2 * i + 1]));
                else v[part * 4 + i] = make_float2(low(b[i], W()), high(b[i], W()));
            }
        }
    }
    __device__ __forceinline__ static void sums(float *to, int at, int k, int, const float2 (&v)[kPairs]) {
        to += (long long)(at + k * kThreads) * kCount;
#pragma unroll
        for (int i = 0; i < kPairs; i += 2) *reinterpret_cast<float4 *>(to + 2 * i) = make_float4(v[i].x, v[i].y, v[i + 1].x, v[i + 1].y);
    }
};
// Else two single elements, neighbours of which are neighbouring threads'.  (Pieces that straddle the boundaries, put together from two, took 7550 x 1505 four
// times as long.)  n: elements.
template <typename T, int kThreads>
struct Part<T, false, kThreads> {
    static constexpr int kCount = 2, kPairs = 1;
    T a, b;
    __device__ __forceinline__ static int first(int at, int k) { return at + 2 * k * kThreads; }
    __device__ __forceinline__ static bool any(int at, int k, int n) { return first(at, k) < n; }
    __device__ __forceinline__ static bool two(int at, int k, int n) { return first(at, k) + kThreads < n; }
    __device__ __forceinline__ void load(const T *row, int at, int k, int n) {
        a = row[first(at, k)];
        b = two(at, k, n) ? row[first(at, k) + kThreads] : from_float<T>(0.f);
    }
    __device__ __forceinline__ float2 pair(int) const { return make_float2(to_float(a), to_float(b)); }
    __device__ __forceinline__ void set(int, float2 v) {
        a = from_float<T>(v.x);
        b = from_float<T>(v.y);
    }
    // v without what is not the row's
    __device__ __forceinline__ static float2 own(float2 v, int at, int k, int n) { return make_float2(v.x, two(at, k, n) ? v.y : 0.f); }
    __device__ __forceinline__ void again() {}
    __device__ __forceinline__ void store(T *row, int at, int k, int n) const {
        row[first(at, k)] = a;
        if (two(at, k, n)) row[first(at, k) + kThreads] = b;
    }
    template <typename W>
    __device__ __forceinline__ static void weights(const W *from, int at, int k, int n, float2 (&v)[1]) {
        v[0] = make_float2(to_float(from[first(at, k)]), two(at, k, n) ? to_float(from[first(at, k) + kThreads]) : 0.f);
    }
    __device__ __forceinline__ static void sums(float *to, int at, int k, int n, const float2 (&v)[1]) {
        to[first(at, k)] = v[0].x;
        if (two(at, k, n)) to[first(at, k) + kThreads] = v[0].y;
    }
};

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
// Threads a row -> threads a block, rows of a block (a warp each)
__host__ __device__ constexpr int block_of(int threads) { return threads == 32 ? 256 : threads; }
__host__ __device__ constexpr int teams_of(int threads) { return threads == 32 ? 8 : 1; }

// Of a row's squares and deviations, added up, the variance and what the mean was off by.  That is taken from rows four standard deviations from zero on: the
// deviations' sum has roundings of its own, which nearer to zero are no less than the mean's.  (Squares that are infinite stay so, and their row becomes the bias.)
__device__ __forceinline__ float2 variance_and_drift(float mean, float squares, float deviations, float per_row) {
    const float variance = squares * per_row, drift = mean * mean > 16.f * variance ? deviations * per_row : 0.f;
    return make_float2(drift != 0.f ? fmaxf(fmaf(-drift, drift, variance), 0.f) : variance, drift);
}

struct Forward {
    int M, K, parts;             // of a row: 16 bytes each, or single elements
    const void *X, *scale, *bias;
    long long x_ld, y_ld;
    void *Y;
    float *mean, *inv_std;
    float epsilon, per_row;      // 1 / K
};

// kThreads threads a row, kParts parts a thread at most, kRows rows at once
template <typename T, typename W, bool kWhole, int kThreads, int kParts, int kRows>
__global__ void __launch_bounds__(block_of(kThreads), 1024 / block_of(kThreads)) layer_norm_kernel(const Forward p) {
    typedef Part<T, kWhole, kThreads> P;
    constexpr int kPairs = P::kPairs;
    __shared__ float shared[3 * kRows][32];
    const int at = threadIdx.x % kThreads;
    const long long i0 = ((long long)blockIdx.x * teams_of(kThreads) + threadIdx.x / kThreads) * kRows;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    if (i0 >= p.M) return;                   // (a warp of a block of eight; a block has rows)
    P v[kRows][kParts];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int k = 0; k < kParts; ++k)
            if (i0 + r < p.M && P::any(at, k, p.parts)) v[r][k].load(static_cast<const T *>(p.X) + (i0 + r) * p.x_ld, at, k, p.parts);
    float mean[kRows], inv_std[kRows], shift[kRows], left[2 * kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        float2 sum = both(0.f);
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            if (i0 + r < p.M && P::any(at, k, p.parts))
#pragma unroll
                for (int e = 0; e < kPairs; ++e) sum = add(sum, v[r][k].pair(e));
            v[r][k].again();
        }
        mean[r] = sum.x + sum.y;
    }
    sum_over_row<kThreads, kRows>(mean, shared);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        float2 squares = both(0.f), deviations = both(0.f);
        mean[r] *= p.per_row;
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
            if (i0 + r < p.M && P::any(at, k, p.parts))
#pragma unroll
                for (int e = 0; e < kPairs; ++e) {
                    const float2 d = P::own(add(v[r][k].pair(e), both(-mean[r])), at, k, p.parts);
                    squares = fma(d, d, squares);
                    deviations = add(deviations, d);
                }
            v[r][k].again();
        }
        left[2 * r] = squares.x + squares.y;
        left[2 * r + 1] = deviations.x + deviations.y;
    }
    sum_over_row<kThreads, 2 * kRows>(left, shared + kRows);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const float2 of_row = variance_and_drift(mean[r], left[2 * r], left[2 * r + 1], p.per_row);
        inv_std[r] = __frsqrt_rn(of_row.x + p.epsilon);
        shift[r] = -of_row.y * inv_std[r];
        if (at == 0 && p.mean && i0 + r < p.M) {
            p.mean[i0 + r] = mean[r] + of_row.y;
            p.inv_std[i0 + r] = inv_std[r];
        }
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
        if (!P::any(at, k, p.parts)) continue;
        float2 scale[kPairs], bias[kPairs] = {};
        P::weights(static_cast<const W *>(p.scale), at, k, p.parts, scale);
        if (p.bias) P::weights(static_cast<const W *>(p.bias), at, k, p.parts, bias);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (i0 + r >= p.M) continue;
            P out;
#pragma unroll
            for (int e = 0; e < kPairs; ++e) out.set(e, fma(fma(add(v[r][k].pair(e), both(-mean[r])), both(inv_std[r]), both(shift[r])), scale[e], bias[e]));
            out.store(static_cast<T *>(p.Y) + (i0 + r) * p.y_ld, at, k, p.parts);
        }
    }
}

// Rows too long for a block's registers: read three times
template <typename T, typename W, bool kWhole>
__global__ void __launch_bounds__(1024) layer_norm_long_kernel(const Forward p) {
    typedef Part<T, kWhole, 1024> P;
    constexpr int kPairs = P::kPairs;
    __shared__ float shared[3][32];
    const long long i = blockIdx.x;
    const int at = threadIdx.x;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const T *x = static_cast<const T *>(p.X) + i * p.x_ld;
    P v;
    float2 sum = both(0.f), squares = both(0.f), deviations = both(0.f);
#pragma unroll 4
    for (int k = 0; P::any(at, k, p.parts); ++k) {
        v.load(x, at, k, p.parts);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) sum = add(sum, v.pair(e));
    }
    float all[1] = {sum.x + sum.y};
    sum_over_row<1024, 1>(all, shared);
    const float mean = all[0] * p.per_row;
#pragma unroll 4
    for (int k = 0; P::any(at, k, p.parts); ++k) {
        v.load(x, at, k, p.parts);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const float2 d = P::own(add(v.pair(e), both(-mean)), at, k, p.parts);
            squares = fma(d, d, squares);
            deviations = add(deviations, d);
        }
    }
    float left[2] = {squares.x + squares.y, deviations.x + deviations.y};
    sum_over_row<1024, 2>(left, shared + 1);
    const float2 of_row = variance_and_drift(mean, left[0], left[1], p.per_row);
    const float inv_std = __frsqrt_rn(of_row.x + p.epsilon), shift = -of_row.y * inv_std;
    if (at == 0 && p.mean) {
        p.mean[i] = mean + of_row.y;
        p.inv_std[i] = inv_std;
    }
#pragma unroll 2
    for (int k = 0; P::any(at, k, p.parts); ++k) {
        float2 scale[kPairs], bias[kPairs] = {};
        P::weights(static_cast<const W *>(p.scale), at, k, p.parts, scale);
        if (p.bias) P::weights(static_cast<const W *>(p.bias), at, k, p.parts, bias);
        v.load(x, at, k, p.parts);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) v.set(e, fma(fma(add(v.pair(e), both(-mean)), both(inv_std), both(shift)), scale[e], bias[e]));
        v.store(static_cast<T *>(p.Y) + i * p.y_ld, at, k, p.parts);
    }
}

// A team: the threads that have a row's columns (or of a cluster's a block's part of them), 8 or 16 each; a block has one, or eight of a warp each.  Rows that
// a team takes at once; blocks an SM.  (512 threads an SM of 128 registers, or 1024 of 64: 16384 x 4096 of bf16 76 and 88 us.)
constexpr int kMostStages = 16;
__host__ __device__ constexpr int rows_of(int element) { return element == 4 ? 1 : 2; }
__host__ __device__ constexpr int per_sm(int threads) { return 512 / block_of(threads); }

// Sums of N values (a power of 2) each over a warp: a lane has one of them in the end, that of index lane / (32 / N).  (Of values that it does not keep a lane
// sends its share to one that does: 6 exchanges for 4 values instead of 20.)
template <int N>
__device__ __forceinline__ float sum_each(float (&v)[N]) {
    const int lane = threadIdx.x % 32;
    int o = 16;
#pragma unroll
    for (int n = N; n > 1; n /= 2, o /= 2)
#pragma unroll
        for (int i = 0; i < n / 2; ++i) {
            const bool upper = lane & o;
            const float kept = upper ? v[n / 2 + i] : v[i];
            v[i] = kept + __shfl_xor_sync(0xffffffffu, upper ? v[i] : v[n / 2 + i], o);
        }
    float sum = v[0];
#pragma unroll
    for (; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}

// The ring of a team, in shared memory: stages of rows_of rows of dY and of X, `pitch` bytes apart unless they follow one another in memory
struct Ring {
    int stages, stage_bytes, pitch;
    int columns;                 // of a block: all, or of a cluster's each its part
    int blocks;                  // of a cluster
};
struct Source {
    const uint8_t *p;
    long long pitch;             // bytes
    int dense;                   // the rows follow one another
};

struct Backward {
    int M, K;
    const void *scale;
    Source dY, X;
    void *dX;
    long long dx_ld;
    const float *mean, *inv_std;
    float *partial;              // for each block (cluster) its sums of dY n, then of dY; NULL where no weights' gradient is wanted
    long long pitch;             // floats of one of these
    float per_row;
    Ring ring;
    unsigned int *err;
};

// dX = inv_std (d - mean(d) - n mean(d n)), n = (x - mean) inv_std, d = dY scale
template <typename T, typename W, bool kWhole, int kThreads, int kElements>
__global__ void __launch_bounds__(block_of(kThreads), per_sm(kThreads)) layer_norm_grad_kernel(const Backward p) {
    typedef Part<T, kWhole, kThreads> P;
    constexpr int kPairs = P::kPairs, kParts = kElements / P::kCount, kTeams = teams_of(kThreads), kRows = rows_of(sizeof(T)), kWarps = kThreads / 32;
    extern __shared__ __align__(16) uint8_t memory[];
    __shared__ uint64_t full_of[kTeams][kMostStages];
    constexpr int kSums = 2 * kRows, kGroup = 32 / kSums;        // a row's two sums, or two rows'; lanes that have the same one
    __shared__ float by_warp[2][kSums][kWarps];
    __shared__ float2 across[2][kRows][8];               // and by a cluster's blocks
    const int at = threadIdx.x % kThreads, team = threadIdx.x / kThreads, lane = threadIdx.x % 32;
    const int blocks = kThreads == 512 ? p.ring.blocks : 1, rank = blocks > 1 ? (int)tc::cluster_ctarank() : 0;
    if (threadIdx.x < kTeams * kMostStages) tc::mbar_init(&full_of[0][0] + threadIdx.x, 1);
    tc::mbar_fence_init();
    __syncthreads();
    if (blocks > 1) tc::cluster_sync_all();              // all are there before one writes to another
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const int begin = rank * p.ring.columns, columns = min(p.ring.columns, p.K - begin), parts = kWhole ? columns / P::kCount : columns;
    const int row_bytes = columns * (int)sizeof(T);
    uint64_t *full = full_of[team];
    uint8_t *stages = memory + (size_t)team * p.ring.stages * p.ring.stage_bytes;
    const uint8_t *sources[2] = {p.dY.p + (long long)begin * sizeof(T), p.X.p + (long long)begin * sizeof(T)};
    const int first = ((int)(blockIdx.x / blocks) * kTeams + team) * kRows, step = (int)(gridDim.x / blocks) * kTeams * kRows;

    // (by a warp) Rows from `row` on into a stage: one copy for each tensor, or for each row of each
    auto fill = [&](int stage, int row) {
        if (row >= p.M) return;
        const int rows = min(kRows, p.M - row), tensor = lane / kRows, r = lane % kRows;
        const bool dense = tensor ? p.X.dense : p.dY.dense;
        uint32_t bytes = 0;
        const uint8_t *src = (tensor ? sources[1] : sources[0]) + (long long)(row + r) * (tensor ? p.X.pitch : p.dY.pitch);
        const uint32_t before = (uint32_t)(reinterpret_cast<uintptr_t>(src) & 15);
        if (tensor < 2 && r < (dense ? 1 : rows)) bytes = (before + (uint32_t)(row_bytes * (dense ? rows : 1)) + 15) / 16 * 16;
        const uint32_t all = __reduce_add_sync(0xffffffffu, bytes);
        if (lane == 0) tc::mbar_arrive_expect_tx(full + stage, all);
        __syncwarp();
        if (bytes) tc::bulk_load_1d(stages + (size_t)stage * p.ring.stage_bytes + (tensor * kRows + r) * p.ring.pitch, src - before, bytes, full + stage);
    };
    // Row i + r of a stage that begins with row i: where its elements are in shared memory
    auto row_at = [&](int tensor, int stage, int i, int r) {
        const Source &s = tensor ? p.X : p.dY;
        const uint8_t *base = stages + (size_t)stage * p.ring.stage_bytes + tensor * kRows * p.ring.pitch;
        if (kWhole) return reinterpret_cast<const T *>(base + r * p.ring.pitch);
        const uint8_t *src = sources[tensor] + (long long)i * s.pitch;
        if (s.dense) return reinterpret_cast<const T *>(base + (reinterpret_cast<uintptr_t>(src) & 15) + r * row_bytes);
        return reinterpret_cast<const T *>(base + r * p.ring.pitch + (reinterpret_cast<uintptr_t>(src + r * s.pitch) & 15));
    };
    if (at < 32)
        for (int s = 0; s < p.ring.stages; ++s) fill(s, first + s * step);
    float2 by_n[kParts][kPairs] = {}, plain[kParts][kPairs] = {}, scale[kParts][kPairs] = {};
#pragma unroll
    for (int k = 0; k < kParts; ++k)
        if (p.dX && P::any(at, k, parts)) P::weights(static_cast<const W *>(p.scale) + begin, at, k, parts, scale[k]);
    // a turn's means, asked for a turn ahead
    float next_mean[kRows] = {}, next_inv[kRows] = {};
    auto ask = [&](int i) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (i + r < p.M) {
                next_mean[r] = p.mean[i + r];
                next_inv[r] = p.inv_std[i + r];
            }
    };
    ask(first);
    int stage = 0, turn = 0;
    uint32_t phase = 0;
    // (a warp that has no row any more leaves the loop by itself; a block's and a cluster's threads share their rows and leave together)
    for (int i = first; i < p.M; i += step, turn ^= 1) {
        P dy[kRows][kParts], x[kRows][kParts];
        float mean[kRows], inv_std[kRows], sum[kRows], along[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            mean[r] = next_mean[r];
            inv_std[r] = next_inv[r];
        }
        ask(i + step);
        tc::mbar_wait(full + stage, phase, p.err, 7);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float2 sum2 = both(0.f), along2 = both(0.f);
            if (i + r < p.M) {
                const T *from_dy = row_at(0, stage, i, r), *from_x = row_at(1, stage, i, r);
#pragma unroll
                for (int k = 0; k < kParts; ++k) {
                    if (!P::any(at, k, parts)) continue;
                    dy[r][k].load(from_dy, at, k, parts);
                    x[r][k].load(from_x, at, k, parts);
#pragma unroll
                    for (int e = 0; e < kPairs; ++e) {
                        const float2 g = dy[r][k].pair(e), n = mul(add(x[r][k].pair(e), both(-mean[r])), both(inv_std[r])), d = mul(g, scale[k][e]);
                        sum2 = add(sum2, d);
                        // (the second of two single elements may be behind the row's end, where n is no number of the row's)
                        along2 = fma(d, P::own(n, at, k, parts), along2);
                        by_n[k][e] = fma(g, n, by_n[k][e]);
                        plain[k][e] = add(plain[k][e], g);
                    }
                    dy[r][k].again();
                    x[r][k].again();
                }
            }
            sum[r] = sum2.x + sum2.y;
            along[r] = along2.x + along2.y;
        }
        // The rows' sums over the team: a warp's, then (in turns, since a warp may write the next rows' while another still reads these) the warps'
        float sums[kSums];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            sums[2 * r] = sum[r];
            sums[2 * r + 1] = along[r];
        }
        float mine = sum_each<kSums>(sums);
        if (kWarps > 1) {
            if (lane % kGroup == 0) by_warp[turn][lane / kGroup][at / 32] = mine;
            __syncthreads();
            mine = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; w += kGroup)
                if (kWarps >= kGroup || lane % kGroup < kWarps) mine += by_warp[turn][lane / kGroup][w + lane % kGroup];
#pragma unroll
            for (int o = kGroup / 2; o > 0; o /= 2) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            sum[r] = __shfl_sync(0xffffffffu, mine, 2 * r * kGroup);
            along[r] = __shfl_sync(0xffffffffu, mine, (2 * r + 1) * kGroup);
        }
        // Here all of the team have read the stage: it is filled again
        if (at < 32) fill(stage, i + p.ring.stages * step);
        if (++stage == p.ring.stages) { stage = 0; phase ^= 1; }
        if (blocks > 1) {
            // over the cluster's blocks, in their order
            if ((int)threadIdx.x < blocks)
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(tc::map_to_cta(tc::smem_u32(&across[turn][r][rank]), threadIdx.x)), "f"(sum[r]),
                                 "f"(along[r]) : "memory");
            tc::cluster_sync_all();
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                sum[r] = along[r] = 0.f;
                for (int b = 0; b < blocks; ++b) {
                    sum[r] += across[turn][r][b].x;
                    along[r] += across[turn][r][b].y;
                }
            }
        }
        if (!p.dX) continue;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (i + r >= p.M) continue;
            const float level = sum[r] * p.per_row, by = along[r] * p.per_row;
            T *to = static_cast<T *>(p.dX) + (long long)(i + r) * p.dx_ld + begin;
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
                if (!P::any(at, k, parts)) continue;
                P out;
#pragma unroll
                for (int e = 0; e < kPairs; ++e) {
                    const float2 n = mul(add(x[r][k].pair(e), both(-mean[r])), both(inv_std[r]));
                    out.set(e, mul(both(inv_std[r]), fma(n, both(-by), fma(dy[r][k].pair(e), scale[k][e], both(-level)))));
                }
                out.store(to, at, k, parts);
            }
        }
    }
    if (blocks > 1) tc::cluster_sync_all();              // no block leaves while another may still write to it
    if (!p.partial) return;
    float *out = p.partial + 2 * p.pitch * (blockIdx.x / blocks) + begin;
    if (kTeams == 1) {
#pragma unroll
        for (int k = 0; k < kParts; ++k)
            if (P::any(at, k, parts)) {
                P::sums(out, at, k, parts, by_n[k]);
                P::sums(out + p.pitch, at, k, parts, plain[k]);
            }
    } else {
        // the warps' columns, added up in the warps' order, where the rings were
        constexpr int kWide = kThreads * kElements;
        float *kept = reinterpret_cast<float *>(memory) + team * 2 * kWide;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kParts; ++k)
            if (P::any(at, k, parts)) {
                P::sums(kept, at, k, parts, by_n[k]);
                P::sums(kept + kWide, at, k, parts, plain[k]);
            }
        kept = reinterpret_cast<float *>(memory);
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * kWide; c += block_of(kThreads)) {
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < kTeams; ++t) sum += kept[t * 2 * kWide + c];
            const int which = c / kWide, col = c % kWide;
            if (col < p.K) out[which * p.pitch + col] = sum;
        }
    }
}

// Rows too long for a cluster: dX by a block a row, which reads it twice
struct LongBackward {
    int M, K, parts;
    const void *dY, *X, *scale;
    long long dy_ld, x_ld, dx_ld;
    void *dX;
    const float *mean, *inv_std;
    float *partial;
    long long pitch;
    float per_row;
};
template <typename T, typename W, bool kWhole>
__global__ void __launch_bounds__(1024) layer_norm_grad_long_kernel(const LongBackward p) {
    typedef Part<T, kWhole, 1024> P;
    constexpr int kPairs = P::kPairs;
    __shared__ float shared[2][32];
    const long long i = blockIdx.x;
    const int at = threadIdx.x;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const T *g = static_cast<const T *>(p.dY) + i * p.dy_ld, *x = static_cast<const T *>(p.X) + i * p.x_ld;
    const float mean = p.mean[i], inv_std = p.inv_std[i];
    P dy, v;
    float2 sum2 = both(0.f), along2 = both(0.f), scale[kPairs];
#pragma unroll 2
    for (int k = 0; P::any(at, k, p.parts); ++k) {
        P::weights(static_cast<const W *>(p.scale), at, k, p.parts, scale);
        dy.load(g, at, k, p.parts);
        v.load(x, at, k, p.parts);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const float2 d = mul(dy.pair(e), scale[e]);
            sum2 = add(sum2, d);
            along2 = fma(d, P::own(mul(add(v.pair(e), both(-mean)), both(inv_std)), at, k, p.parts), along2);
        }
    }
    float sums[2] = {sum2.x + sum2.y, along2.x + along2.y};
    sum_over_row<1024, 2>(sums, shared);
    const float level = sums[0] * p.per_row, by = sums[1] * p.per_row;
#pragma unroll 2
    for (int k = 0; P::any(at, k, p.parts); ++k) {
        P::weights(static_cast<const W *>(p.scale), at, k, p.parts, scale);
        dy.load(g, at, k, p.parts);
        v.load(x, at, k, p.parts);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
            const float2 n = mul(add(v.pair(e), both(-mean)), both(inv_std));
            dy.set(e, mul(both(inv_std), fma(n, both(-by), fma(dy.pair(e), scale[e], both(-level)))));
        }
        dy.store(static_cast<T *>(p.dX) + i * p.dx_ld, at, k, p.parts);
    }
}
// and the columns' sums of some rows by blocks of 32 columns by 8 rows
template <typename T>
__global__ void __launch_bounds__(256) layer_norm_columns_kernel(const LongBackward p) {
    __shared__ float sums[8][2][32];
    const int lane = threadIdx.x % 32, group = threadIdx.x / 32, column = blockIdx.x * 32 + lane;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    float a = 0.f, b = 0.f;
    if (column < p.K) {
#pragma unroll 4
        for (long long i = blockIdx.y * 8 + group; i < p.M; i += gridDim.y * 8) {
            const float g = to_float(static_cast<const T *>(p.dY)[i * p.dy_ld + column]);
            a = fmaf(g, __fmul_rn(to_float(static_cast<const T *>(p.X)[i * p.x_ld + column]) - p.mean[i], p.inv_std[i]), a);
            b += g;
        }
    }
    sums[group][0][lane] = a;
    sums[group][1][lane] = b;
    __syncthreads();
    if (threadIdx.x >= 64 || column >= p.K) return;
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g) sum += sums[g][group][lane];
    p.partial[(2ll * blockIdx.y + group) * p.pitch + column] = sum;
}

// What the blocks left, added up: 32 columns a block, four a thread, 64 groups of threads with a share of the blocks each, which is little enough to be on its
// way at once.  dScale's columns first, then dB's.
template <typename W>
__global__ void __launch_bounds__(512) layer_norm_sums_kernel(int K, int blocks, const float *partial, long long pitch, W *d_scale, W *d_bias) {
    __shared__ float4 sums[16][8];
    const int lane = threadIdx.x % 8, group = threadIdx.x / 8, which = blockIdx.y;
    const long long c = ((long long)blockIdx.x * 8 + lane) * 4;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    W *out = which ? d_bias : d_scale;
    if (!out) return;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < pitch) {
#pragma unroll 5
        for (int b = group; b < blocks; b += 64) {
            const float4 v = *reinterpret_cast<const float4 *>(partial + (2ll * b + which) * pitch + c);
            sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
    }
#pragma unroll
    for (int o = 8; o < 32; o *= 2) {
        sum.x += __shfl_xor_sync(0xffffffffu, sum.x, o);
        sum.y += __shfl_xor_sync(0xffffffffu, sum.y, o);
        sum.z += __shfl_xor_sync(0xffffffffu, sum.z, o);
        sum.w += __shfl_xor_sync(0xffffffffu, sum.w, o);
    }
    if (threadIdx.x % 32 < 8) sums[threadIdx.x / 32][lane] = sum;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    const long long at = (long long)blockIdx.x * 32 + threadIdx.x;
    if (at >= K) return;
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) total += reinterpret_cast<const float *>(&sums[w][threadIdx.x / 4])[threadIdx.x % 4];
    out[at] = from_float<W>(total);
}

bool at_16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Threads a row, parts a thread and rows at once of the forward kernel: the first shape that has room for a row's parts (16 bytes, or of single elements two
// a thread).  Several rows at once are several times the loads on their way, and the weights are read once for all of them.
struct RowShape {
    int threads, parts, rows;
};
constexpr int kShapes = 8;
constexpr RowShape kWholeRows[kShapes] = {{32, 1, 4}, {32, 2, 2}, {32, 4, 1}, {64, 4, 2}, {128, 4, 2}, {256, 4, 2}, {512, 4, 2}, {512, 8, 1}};
constexpr RowShape kSingleRows[kShapes] = {{32, 4, 2}, {32, 8, 1}, {32, 16, 1}, {128, 8, 2}, {256, 8, 2}, {512, 8, 2}, {512, 16, 1}, {0, 0, 0}};
// of few rows
constexpr RowShape kWholeFew[kShapes] = {{32, 1, 1}, {256, 2, 1}, {512, 4, 1}, {512, 8, 1}, {0, 0, 0}};
constexpr RowShape kSingleFew[kShapes] = {{32, 4, 1}, {256, 4, 1}, {512, 16, 1}, {0, 0, 0}};
// f(threads, parts, rows, all as types) for it; false where none has room
template <const RowShape (&kRows)[kShapes], bool kWhole, int kAt = 0, typename F>
bool with_shape(int parts, F f) {
    if constexpr (kAt == kShapes || kRows[kAt % kShapes].threads == 0) return false;
    else {
        constexpr RowShape s = kRows[kAt];
        if (parts > s.threads * s.parts * (kWhole ? 1 : 2)) return with_shape<kRows, kWhole, kAt + 1>(parts, f);
        f(std::integral_constant<int, s.threads>(), std::integral_constant<int, s.parts>(), std::integral_constant<int, s.rows>());
        return true;
    }
}

template <typename T, typename W, bool kWhole>
int launch(const LayerNormProblem &q, cudaStream_t stream) {
    const Forward p{q.M, q.K, kWhole ? q.K / (int)(16 / sizeof(T)) : q.K, q.X.p, q.scale, q.bias, q.X.ld, q.Y.ld, const_cast<void *>(q.Y.p), q.mean, q.inv_std,
                    q.epsilon, (float)(1.0 / q.K)};
    int err = 0;
    auto run = [&](auto threads, auto parts, auto rows) {
        constexpr int kEach = teams_of(threads) * rows;
        const unsigned blocks = (unsigned)(((long long)q.M + kEach - 1) / kEach);
        err = (int)tc_host::launch_pdl(layer_norm_kernel<T, W, kWhole, threads, parts, rows>, dim3(blocks), dim3(block_of(threads)), 0, stream, p);
    };
    // (few: four an SM)
    const bool held = q.M <= 148 * 4 ? with_shape<kWhole ? kWholeFew : kSingleFew, kWhole>(p.parts, run) : with_shape<kWhole ? kWholeRows : kSingleRows, kWhole>(p.parts, run);
    return held ? err : (int)tc_host::launch_pdl(layer_norm_long_kernel<T, W, kWhole>, dim3(q.M), dim3(1024), 0, stream, p);
}

// Threads of a team of the gradients' kernel, and a thread's columns, for rows (or a block's part of them) of so many: f(threads, elements, both as types).
// Fewer threads with more columns each wait less for one another, but few blocks an SM leave less in the workspace.  (128 x 8, 256 x 8, 256 x 16 and 512 x 8:
// 16384 x 1024 of bf16 28.6, 36, 43 and 61 us, x 2048 -, 44, 51 and 67, x 4096 -, -, 70 and 79, 8192 x 4096 of 32 bits -, -, 74 and 65.)
constexpr int kMostCluster = 8;
template <typename F>
int with_team(int columns, int element, F f) {
    if (columns <= 32 * 16) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 16>());
    if (columns <= 128 * 8) return f(std::integral_constant<int, 128>(), std::integral_constant<int, 8>());
    if (columns <= 256 * 8) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 8>());
    if (columns <= 512 * 8) {
        if (element == 4) return f(std::integral_constant<int, 512>(), std::integral_constant<int, 8>());
        return f(std::integral_constant<int, 256>(), std::integral_constant<int, 16>());
    }
    return f(std::integral_constant<int, 512>(), std::integral_constant<int, 16>());
}
constexpr int kMostColumns = 8192;
int cluster_of(int K) {
    int blocks = 1;
    while (blocks * kMostColumns < K) blocks *= 2;
    return blocks;
}
int columns_of(int K) {
    const int blocks = cluster_of(K);
    return blocks == 1 ? K : ((K + blocks - 1) / blocks + 7) / 8 * 8;
}
// The ring, as deep as an SM's shared memory allows (three stages at least: 200 KB for stages of 64 KB and a little, those of 8192 columns)
Ring ring_of(int K, int element, int threads, bool whole) {
    Ring r{};
    r.blocks = cluster_of(K);
    r.columns = columns_of(K);
    const int row = r.columns * element, budget = 200 * 1024 / (per_sm(threads) * teams_of(threads));
    r.pitch = whole ? row : (row + 15) / 16 * 16 + 16;
    r.stage_bytes = 2 * rows_of(element) * r.pitch;
    r.stages = std::min(kMostStages, budget / r.stage_bytes);
    return r;
}
Source source_of(const DenseOperand &o, int M, int K, int element, bool one_block) {
    const long long pitch = (M == 1 ? K : o.ld) * element;
    return Source{static_cast<const uint8_t *>(o.p), pitch, one_block && pitch == (long long)K * element};
}

// The most blocks (clusters) of the gradients' kernels, each of which leaves sums of all columns in the workspace (a B200 has 148 SMs)
constexpr int kMostBlocks = 148 * 4;
int most_blocks(int M) { return std::min(M, kMostBlocks); }
long long grad_pitch(int K) { return (K + 3ll) / 4 * 4; }

// blocks: those that left sums
template <typename T, typename W, bool kWhole>
int launch(const LayerNormGradProblem &q, int &blocks, cudaStream_t stream) {
    float *partial = q.d_scale || q.d_bias ? static_cast<float *>(q.partial) : nullptr;
    if (q.K > kMostCluster * kMostColumns) {
        const LongBackward p{q.M, q.K, kWhole ? q.K / (int)(16 / sizeof(T)) : q.K, q.dY.p, q.X.p, q.scale, q.dY.ld, q.X.ld, q.dX.ld, const_cast<void *>(q.dX.p),
                             q.mean, q.inv_std, partial, grad_pitch(q.K), (float)(1.0 / q.K)};
        blocks = std::max(1, std::min(64, (q.M + 63) / 64));
        int err = 0;
        if (p.dX) {
            err = (int)tc_host::launch_pdl(layer_norm_grad_long_kernel<T, W, kWhole>, dim3(q.M), dim3(1024), 0, stream, p);
            if (partial) count_launch();
        }
        if (err == 0 && partial) err = (int)tc_host::launch_pdl(layer_norm_columns_kernel<T>, dim3((q.K + 31) / 32, blocks), dim3(256), 0, stream, p);
        return err;
    }
    return with_team(columns_of(q.K), sizeof(T), [&](auto threads, auto elements) {
        const Ring ring = ring_of(q.K, sizeof(T), threads, kWhole);
        const Backward p{q.M, q.K, q.scale, source_of(q.dY, q.M, q.K, sizeof(T), ring.blocks == 1), source_of(q.X, q.M, q.K, sizeof(T), ring.blocks == 1),
                         const_cast<void *>(q.dX.p), q.dX.ld, q.mean, q.inv_std, partial, grad_pitch(q.K), (float)(1.0 / q.K), ring, device_status_ptr()};
        if (!p.err) return (int)cudaErrorUnknown;
        constexpr int kTeams = teams_of(threads);
        const int rows = rows_of(sizeof(T)) * kTeams;
        blocks = (int)std::min<long long>(((long long)q.M + rows - 1) / rows, std::max(1, std::min(kMostBlocks, 148 * per_sm(threads)) / ring.blocks));
        // (where the warps' sums are added up there is room for them)
        const size_t smem = std::max<size_t>((size_t)kTeams * ring.stages * ring.stage_bytes, kTeams > 1 ? kTeams * 2 * threads * elements * 4 : 0);
        const auto kernel = layer_norm_grad_kernel<T, W, kWhole, threads, elements>;
        if (smem > 32 * 1024) {
            const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return (int)e;
        }
        if (ring.blocks == 1) return (int)tc_host::launch_pdl(kernel, dim3(blocks), dim3(block_of(threads)), smem, stream, p);
        return (int)tc_host::launch_pdl_cluster(kernel, (unsigned)ring.blocks, dim3((unsigned)(blocks * ring.blocks)), dim3(block_of(threads)), smem, stream, p);
    });
}

template <typename W>
int launch_sums(int K, int blocks, const float *partial, void *d_scale, void *d_bias, cudaStream_t stream) {
    const long long pitch = grad_pitch(K);
    return (int)tc_host::launch_pdl(layer_norm_sums_kernel<W>, dim3((unsigned)((pitch + 31) / 32), 2), dim3(512), 0, stream, K, blocks, partial, pitch,
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
        const bool whole = p.K % kCount == 0 && at_16(p.X.p) && at_16(p.Y.p) && at_16(p.scale) && at_16(p.bias) &&
                           (p.M == 1 || (p.X.ld % kCount == 0 && p.Y.ld % kCount == 0));
        return whole ? launch<T, W, true>(p, stream) : launch<T, W, false>(p, stream);
    });
    count_launch();
    return err;
}

size_t layer_norm_grad_workspace(int M, int K, bool weights) { return weights ? (size_t)(most_blocks(M) * 2 * grad_pitch(K)) * 4 : 0; }

int launch_layer_norm_grad(const LayerNormGradProblem &p, cudaStream_t stream) {
    const bool weights = p.d_scale || p.d_bias;
    int blocks = 0;
    int err = by_types(p.type, p.weight_type, [&](auto t, auto w) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        constexpr int kCount = 16 / sizeof(T);
        const bool whole = p.K % kCount == 0 && at_16(p.dY.p) && at_16(p.X.p) && at_16(p.dX.p) && at_16(p.scale) &&
                           (p.M == 1 || (p.dY.ld % kCount == 0 && p.X.ld % kCount == 0 && p.dX.ld % kCount == 0));
        return whole ? launch<T, W, true>(p, blocks, stream) : launch<T, W, false>(p, blocks, stream);
    });
    count_launch();
    if (err == 0 && weights) {
        const float *partial = static_cast<const float *>(p.partial);
        err = p.weight_type == ONNXB_FLOAT     ? launch_sums<float>(p.K, blocks, partial, p.d_scale, p.d_bias, stream)
              : p.weight_type == ONNXB_FLOAT16 ? launch_sums<__half>(p.K, blocks, partial, p.d_scale, p.d_bias, stream)
                                               : launch_sums<__nv_bfloat16>(p.K, blocks, partial, p.d_scale, p.d_bias, stream);
        count_launch();
    }
    return err;
}

}  // namespace onnxb
