// Elementwise mathematics of the dense layers, in 32 bits: activations, their slopes, and conversions to and from the types that
// tensors are kept in.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "onnx_b200.h"

namespace onnxb {
namespace dense {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// The 16 bytes at `at` (a multiple of 16) of a row of row_bytes that begins anywhere, zeros past its end: put together from the two
// aligned 16-byte pieces that hold them, or element by element (of kElement bytes) at the row's ends, where those pieces reach into
// what is not the row's.
template <int kElement>
__device__ __forceinline__ uint4 load16_anywhere(const uint8_t *row, long long at, long long row_bytes) {
    const int off = (int)(reinterpret_cast<uintptr_t>(row) & 15), bits = (off & 3) * 8;
    uint32_t w[8] = {};
    if ((at > 0 || off == 0) && at + (off ? 32 - off : 16) <= row_bytes) {
        const uint4 *pieces = reinterpret_cast<const uint4 *>(row + at - off);
        const uint4 a = pieces[0], b = off ? pieces[1] : make_uint4(0, 0, 0, 0);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        // (`off` is the same for all of a row)
        auto from = [&](int first) {
            uint32_t out[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) out[i] = __funnelshift_r(w[first + i], first + i < 7 ? w[first + i + 1] : 0u, bits);
            return make_uint4(out[0], out[1], out[2], out[3]);
        };
        return off < 4 ? from(0) : off < 8 ? from(1) : off < 12 ? from(2) : from(3);
    }
#pragma unroll
    for (int i = 0; i < 16; i += kElement)
        if (at + i < row_bytes) {
            const uint8_t *e = row + at + i;                     // (nothing is read past the row)
            const uint32_t v = kElement == 4 ? *reinterpret_cast<const uint32_t *>(e) : kElement == 2 ? *reinterpret_cast<const uint16_t *>(e) : *e;
            w[i / 4] |= v << (i % 4 * 8);
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 1 / (1 + exp(-z)): exp(-z) is finite up to z = -88 and infinite below, where the quotient is 0 as it should be (to 1e-38)
__device__ __forceinline__ float logistic(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }
// sqrt(8/pi) (g + 0.044715 g^3): tanh's argument in the approximation of gelu, twice, since (1 + tanh(y)) / 2 = logistic(2y).
// (As tanh the factor would lose all its digits where it is small.)
__device__ __forceinline__ float gelu_argument(float g) { return 1.5957691216057308f * fmaf(0.044715f * g * g, g, g); }

// The normal distribution's value at g, and exp(-g^2 / 2).  Its tail beyond |g| is exp(-g^2 / 2) t P(t), t = 1 / (1 + 0.3 |g|), P of degree 7 fitted
// to it for |g| < 14.5 (largest relative error 1.7e-7, by reweighted least squares on Chebyshev points; in 32 bits 4e-6 at |g| = 13, where g^2 / 2 is
// rounded, 1.3e-6 below 6).  erfcf's 50 instructions an element were most of the epilogue: gated block 1597 x 384 x 1088 17.8 us with it.
__device__ __forceinline__ float normal_at(float g, float &density) {
    const float t = __fdividef(1.f, fmaf(0.3f, fabsf(g), 1.f));
    float p = 0.03542385995388031f;
    p = fmaf(p, t, -0.1561589390039444f);
    p = fmaf(p, t, 0.20455756783485413f);
    p = fmaf(p, t, -0.052034683525562286f);
    p = fmaf(p, t, 0.1276920884847641f);
    p = fmaf(p, t, 0.10017585754394531f);
    p = fmaf(p, t, 0.12071214616298676f);
    p = fmaf(p, t, 0.11963200569152832f);
    density = __expf(-0.5f * g * g);
    const float tail = density * t * p;
    return g >= 0.f ? 1.f - tail : tail;
}

// act(g)
__device__ __forceinline__ float activate(int kind, float g) {
    if (kind == ONNXB_SILU) return g * logistic(g);
    if (kind == ONNXB_GELU) {
        float density;
        return g * normal_at(g, density);
    }
    if (kind == ONNXB_GELU_TANH) return g * logistic(gelu_argument(g));
    return g > 0.f ? g : 0.f;
}

// act(g) and act'(g)
__device__ __forceinline__ void activate_with_slope(int kind, float g, float &value, float &slope) {
    if (kind == ONNXB_SILU) {
        const float p = logistic(g);
        value = g * p;
        slope = fmaf(value, 1.f - p, p);
    } else if (kind == ONNXB_GELU) {
        float density;
        const float p = normal_at(g, density);
        value = g * p;
        slope = fmaf(g * 0.39894228040143268f, density, p);
    } else if (kind == ONNXB_GELU_TANH) {
        const float p = logistic(gelu_argument(g));
        value = g * p;
        const float c = fminf(fmaxf(g, -30.f), 30.f);            // (p (1 - p) is 0 beyond; g^2 could be infinite)
        slope = fmaf(c * p * (1.f - p), 1.5957691216057308f * fmaf(0.134145f * c, c, 1.f), p);
    } else {
        value = g > 0.f ? g : 0.f;
        slope = g > 0.f ? 1.f : 0.f;
    }
}

}  // namespace dense
}  // namespace onnxb
