// onnx_quantize_rows_run: 8-bit integers and a scale for each row.
//
// One pass over X where a row fits the registers of the threads that share it (a warp for short rows, a block of up to 1024 threads for
// longer ones, four pieces of 16 bytes each): the row is read, its largest magnitude agreed on, and what the registers hold is
// divided and stored.  Longer rows are read a second time, out of L2.  Bound by the bytes of X and Q where these are many: 8192 x 4096 of 32 bits
// 25.5 us (6.6 TB/s), 8192 x 12288 of 16 bits 60.8 us (5.0 TB/s; 97 with a conversion, a compare and a clamp for every element), 7550 rows
// of 1505 that begin anywhere 16.3 us (2.1 TB/s, whose ends are read element by element); one token of 4096 1.3 us.
#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace dense;

// The nearest integer to x / scale, of the exact quotient, ties to even, at most 127 in magnitude.  `inverse` is 1 / scale: x * inverse
// is within 2 roundings of the quotient, so its nearest integer is off by one at most, next to a half.  What is left of x then
// (exact: it has no more digits than x and scale together span) says which side of the half the quotient is on.
__device__ __noinline__ int quantize_exactly(float x, float scale, float inverse) {
    float q = rintf(x * inverse);
    const float rest = fmaf(-q, scale, x), half = 0.5f * scale;
    const bool odd = ((int)q & 1) != 0;
    if (rest > half || (rest == half && odd)) q += 1.f;
    if (rest < -half || (rest == -half && odd)) q -= 1.f;
    return (int)fminf(fmaxf(q, -127.f), 127.f);
}

struct Row {
    float by, scale, inverse;    // values and scale are multiplied by `by` first
    bool some, plain;            // there is a scale, and it is no zero; it is large enough for quantize_four
};
// From a row's largest magnitude, as bits (those of magnitudes are ordered as they are, infinity and NaN above all others).  Where the
// scale is so small that its inverse or the halves of it would not be exact, values and scale are taken 2^100 times as large.
__device__ __forceinline__ Row row_of(unsigned most, float *scale_out, bool writes) {
    const bool finite = most < 0x7F800000u;
    const float s = __fdiv_rn(__uint_as_float(most), 127.f);
    if (writes) *scale_out = finite ? s : __uint_as_float(0x7FC00000u);
    Row r;
    r.some = finite && s > 0.f;
    r.plain = finite && s >= 0x1p-100f;
    r.by = r.plain ? 1.f : 0x1p100f;
    r.scale = s * r.by;
    r.inverse = __fdiv_rn(1.f, r.scale);
    return r;
}
__device__ __forceinline__ int quantize_one(float x, const Row &r) { return r.some ? quantize_exactly(x * r.by, r.scale, r.inverse) : 0; }

// Four values of a row whose scale is no tiny one, as a word of four bytes.  1.5 * 2^23 plus the quotient is the nearest integer to it in
// the low bits (ties to even), without a conversion; at most 127, since the scale is the largest magnitude's 127th part to 24 digits.
// Where a rest is not below half the scale, next to a half, that is worked out (hardly ever).
__device__ __forceinline__ uint32_t quantize_four(const float (&x)[4], const Row &r) {
    constexpr float kLift = 12582912.f;
    float t[4], worst = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t[i] = fmaf(x[i], r.inverse, kLift);
        worst = fmaxf(worst, fabsf(fmaf(-(t[i] - kLift), r.scale, x[i])));
    }
    if (worst >= 0.5f * r.scale) {
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = __uint_as_float((uint32_t)quantize_exactly(x[i], r.scale, r.inverse));
    }
    const uint32_t low = __byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040), high = __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040);
    return __byte_perm(low, high, 0x5410);
}

__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(fabsf(x)); }
// The larger of two pairs of 16-bit magnitudes
__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// What a thread reads at once: 16 bytes.  kAligned: rows of whole pieces, which begin at multiples of 16 bytes in X and of as many as
// a piece has elements in Q.  Else rows begin anywhere, and the last piece has less.
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
    __device__ __forceinline__ unsigned most() const {
        if (sizeof(T) == 4) {
            unsigned m = 0;
#pragma unroll
            for (int e = 0; e < kCount; ++e) m = max(m, magnitude(at(e)));
            return m;
        }
        constexpr uint32_t kAbs = 0x7FFF7FFFu;
        const uint32_t pair = max_pairs(max_pairs(bits.x & kAbs, bits.y & kAbs), max_pairs(bits.z & kAbs, bits.w & kAbs));
        const uint16_t one = (uint16_t)max(pair & 0xFFFFu, pair >> 16);
        return magnitude(to_float(*reinterpret_cast<const T *>(&one)));
    }
    __device__ __forceinline__ void store(int8_t *row, int K, int i, const Row &r) const {
        uint32_t w[kCount / 4];
#pragma unroll
        for (int e = 0; e < kCount; e += 4) {
            const float x[4] = {at(e), at(e + 1), at(e + 2), at(e + 3)};
            if (r.plain) {
                w[e / 4] = quantize_four(x, r);
            } else {
                w[e / 4] = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[e / 4] |= (uint32_t)(quantize_one(x[k], r) & 255) << (8 * k);
            }
        }
        int8_t *to = row + (long long)i * kCount;
        if (kAligned || (reinterpret_cast<uintptr_t>(to) % kCount == 0 && (i + 1ll) * kCount <= K)) {
            if (kCount == 4) *reinterpret_cast<uint32_t *>(to) = w[0];
            else *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[kCount / 4 - 1]);
        } else {
#pragma unroll
            for (int e = 0; e < kCount; ++e)
                if ((long long)i * kCount + e < K) to[e] = (int8_t)(w[e / 4] >> (e % 4 * 8));
        }
    }
};

// The largest of a row's threads: a warp's, or those of the whole block
template <int kThreads>
__device__ __forceinline__ unsigned most_of_row(unsigned m) {
    m = __reduce_max_sync(0xffffffffu, m);
    if (kThreads > 32) {
        __shared__ unsigned of_warp[32];
        if (threadIdx.x % 32 == 0) of_warp[threadIdx.x / 32] = m;
        __syncthreads();
        constexpr int kWarps = kThreads / 32;
        m = __reduce_max_sync(0xffffffffu, of_warp[threadIdx.x % kWarps]);
    }
    return m;
}

// kThreads threads a row, kPieces pieces a thread at most; a warp a row: 8 rows a block
template <typename T, bool kAligned, int kThreads, int kPieces>
__global__ void __launch_bounds__(kThreads < 256 ? 256 : kThreads) quantize_rows_kernel(int M, int K, int pieces, const T *X, long long x_ld, int8_t *Q,
                                                                                         long long q_ld, float *scale) {
    constexpr int kRows = kThreads < 256 ? 256 / kThreads : 1;
    static_assert(kRows == 1 || kThreads == 32, "a row has a warp, or the block");
    const long long i = (long long)blockIdx.x * kRows + threadIdx.x / kThreads;
    const int at = threadIdx.x % kThreads;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const bool in = i < M;
    const T *x = X + (in ? i : 0) * x_ld;
    Piece<T, kAligned> v[kPieces];
    unsigned m = 0;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        if (in && at + k * kThreads < pieces) v[k].load(x, K, at + k * kThreads);
        else v[k].clear();
    }
#pragma unroll
    for (int k = 0; k < kPieces; ++k) m = max(m, v[k].most());
    m = most_of_row<kThreads>(m);
    if (!in) return;
    const Row r = row_of(m, scale + i, at == 0);
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
        if (at + k * kThreads < pieces) v[k].store(Q + i * q_ld, K, at + k * kThreads, r);
}

// Longer rows: read twice
template <typename T, bool kAligned>
__global__ void __launch_bounds__(1024) quantize_long_rows_kernel(int K, int pieces, const T *X, long long x_ld, int8_t *Q, long long q_ld, float *scale) {
    const long long i = blockIdx.x;
    tc::pdl_launch_dependents();
    tc::pdl_wait();
    const T *x = X + i * x_ld;
    unsigned m = 0;
    Piece<T, kAligned> v;
#pragma unroll 4
    for (int k = threadIdx.x; k < pieces; k += 1024) {
        v.load(x, K, k);
        m = max(m, v.most());
    }
    const Row r = row_of(most_of_row<1024>(m), scale + i, threadIdx.x == 0);
#pragma unroll 2
    for (int k = threadIdx.x; k < pieces; k += 1024) {
        v.load(x, K, k);
        v.store(Q + i * q_ld, K, k, r);
    }
}

template <typename T, bool kAligned>
int launch(int M, int K, const T *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream) {
    constexpr int kCount = 16 / sizeof(T);
    const int pieces = (K + kCount - 1) / kCount;
    auto run = [&](auto kernel, int threads, int rows) {
        return (int)tc_host::launch_pdl(kernel, dim3((unsigned)(((long long)M + rows - 1) / rows)), dim3(threads), 0, stream, M, K, pieces, X, x_ld, Q, q_ld, scale);
    };
    if (pieces <= 32) return run(quantize_rows_kernel<T, kAligned, 32, 1>, 256, 8);
    if (pieces <= 128) return run(quantize_rows_kernel<T, kAligned, 32, 4>, 256, 8);
    if (pieces <= 512) return run(quantize_rows_kernel<T, kAligned, 256, 2>, 256, 1);
    if (pieces <= 1024) return run(quantize_rows_kernel<T, kAligned, 256, 4>, 256, 1);
    if (pieces <= 2048) return run(quantize_rows_kernel<T, kAligned, 512, 4>, 512, 1);
    if (pieces <= 4096) return run(quantize_rows_kernel<T, kAligned, 1024, 4>, 1024, 1);
    return (int)tc_host::launch_pdl(quantize_long_rows_kernel<T, kAligned>, dim3(M), dim3(1024), 0, stream, K, pieces, X, x_ld, Q, q_ld, scale);
}

template <typename T>
int launch(int M, int K, const void *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream) {
    constexpr int kCount = 16 / sizeof(T);
    const T *x = static_cast<const T *>(X);
    const bool aligned = K % kCount == 0 && reinterpret_cast<uintptr_t>(X) % 16 == 0 && reinterpret_cast<uintptr_t>(Q) % kCount == 0 &&
                         (M == 1 || (x_ld % kCount == 0 && q_ld % kCount == 0));
    return aligned ? launch<T, true>(M, K, x, x_ld, Q, q_ld, scale, stream) : launch<T, false>(M, K, x, x_ld, Q, q_ld, scale, stream);
}

}  // namespace

int launch_quantize_rows(int type, int M, int K, const void *X, long long x_ld, int8_t *Q, long long q_ld, float *scale, cudaStream_t stream) {
    const int err = type == ONNXB_FLOAT     ? launch<float>(M, K, X, x_ld, Q, q_ld, scale, stream)
                    : type == ONNXB_FLOAT16 ? launch<__half>(M, K, X, x_ld, Q, q_ld, scale, stream)
                                            : launch<__nv_bfloat16>(M, K, X, x_ld, Q, q_ld, scale, stream);
    count_launch();
    return err;
}

}  // namespace onnxb
