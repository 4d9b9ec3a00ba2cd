// Dense layers of 8- and 16-bit operands on the 5th-generation tensor cores: onnx_gemm_int8_run, onnx_gated_run (and of 8-bit
// operands) and the three products of its gradients (DenseMode in dense.h).
//
// The pipeline is that of tc_gemm.cu: a persistent CTA (or a pair of two on one tile) per SM, 320 threads,
//   warp 0    TMA producer, a ring of stages of 128 bytes along the reduction (64 16-bit or 128 8-bit terms);
//   warp 1    one thread issues tcgen05.mma kind::f16 or kind::i8 into one of two TMEM accumulators;
//   warps 2-9 epilogue: tcgen05.ld, the mathematics, 32-row blocks of 128 bytes staged in swizzled shared memory, TMA stores (plain ones
//             where Y's rows do not begin at multiples of 16 bytes).
// What is its own:
//   - The gated block is one product: half of a tile's B rows are Wg's, half Wu's of the same channels, so that an accumulator holds
//     a channel's gate in column j and its other factor in column BN/2 + j, in the same TMEM lane.  X is read once for both, and
//     the pair's form costs nothing: each CTA stages one of the two.
//   - dX = dG Wg + dU Wu is one sum: the reduction runs over dG's channels, then dU's, with the other tensor maps from there on.
//   - dWg and dWu = dG^T X and dU^T X take their operands as they lie, the reduction (tokens) along the rows: MN-major, 64 x 64 boxes.
//     The same for Wg and Wu in dX.  No transposed copy is made.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdlib>

#include "dense.h"
#include "dense_math.cuh"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace tc;
using namespace dense;

constexpr int kBM = 128;                           // rows of a CTA's part of a tile (TMEM lanes)
constexpr int kRowBytes = 128;                     // of the reduction per stage: one swizzle row
constexpr int kMaxBN = 256;
constexpr int kMaxStages = 32;
constexpr int kThreads = 320;
constexpr int kEpiWarps = 8;
constexpr int kABytes = kBM * kRowBytes;
constexpr int kBlockBytes = 32 * kRowBytes;        // what an epilogue warp stages: 32 rows of 128 bytes
constexpr int kStagingBytes = kEpiWarps * kBlockBytes;
constexpr int kBarrierBytes = 1024;
constexpr int kSmemLimit = 232448;

struct Params {
    int M, N;                  // of the output
    int BN, out_cols;          // columns of an accumulator; of the output per tile (half of them for the gated block)
    int tiles_m, tiles_n, band, total;
    int num_kb, seg_kb;        // stages of the reduction; those before the second segment
    int products, first;       // kDenseGradW: how many products, and the first one's index
    int num_stages;
    uint32_t idesc, stage_bytes, a_bytes;      // a_bytes: of A in a stage
    const float *a_scale, *b_scale0, *b_scale1, *bias;
    int relu, activation;
    int y_type, outs;          // outs: results of a tile (the gated block: H alone, or H, G and U)
    void *Y[3];
    long long y_ld[3];
    int y_tma[3];              // by TMA: 0 no, 1 whole blocks of columns, 2 all
    unsigned int *err;
};

struct Maps {
    CUtensorMap A[2], B[2], Y[3];
};

// Tiles in the order they are run in: product by product, in bands of `band` row tiles, a band's columns one after the other, so that
// the tiles in flight share their operands in L2 (of 148 SMs' 74 pairs at band 8: 8 row tiles and 9 column tiles).
struct TileAt {
    int z, tm, tn;
};
__device__ __forceinline__ TileAt tile_at(const Params &p, int t) {
    const int per = p.tiles_m * p.tiles_n;
    const int z = t / per, r = t - z * per;
    const int b = r / (p.band * p.tiles_n), rr = r - b * p.band * p.tiles_n;
    const int rows = min(p.band, p.tiles_m - b * p.band);
    const int tn = rr / rows;
    return TileAt{z, b * p.band + rr - tn * rows, tn};
}

// Two 32-bit results as one word of 16-bit ones
template <typename T2>
__device__ __forceinline__ uint32_t pack(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack<__half2>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <>
__device__ __forceinline__ uint32_t pack<__nv_bfloat162>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

template <int kCtas, bool kInt8, int kMode>
__global__ void __launch_bounds__(kThreads, 1) tc_dense_kernel(const __grid_constant__ Maps maps, const Params p) {
    constexpr bool kAMn = kMode == kDenseGradW, kBMn = kMode == kDenseGradW || kMode == kDenseGradX;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t *stages = smem;
    uint8_t *staging = smem + (size_t)p.num_stages * p.stage_bytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + kStagingBytes);
    uint64_t *full = bars, *empty = bars + kMaxStages;
    uint64_t *tmem_full = bars + 2 * kMaxStages, *tmem_empty = tmem_full + 2;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(tmem_empty + 2);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = kCtas == 2 ? (int)cluster_ctarank() : 0;
    const int first_tile = blockIdx.x / kCtas, tile_step = gridDim.x / kCtas;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.num_stages; ++s) {
            mbar_init(&full[s], 1);        // (of a pair: the even CTA's, which counts both CTAs' copies)
            mbar_init(&empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&tmem_full[a], 1);
            mbar_init(&tmem_empty[a], kEpiWarps * kCtas);
        }
        mbar_fence_init();
        prefetch_tmap(&maps.A[0]);
        prefetch_tmap(&maps.B[0]);
        if (kMode == kDenseGated) prefetch_tmap(&maps.B[1]);
        if (p.y_tma[0]) prefetch_tmap(&maps.Y[0]);
    }
    if (warp == 1) {
        tmem_alloc(tmem_holder, 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_holder;
    if (kCtas == 2) cluster_sync_all();     // the peer's barriers exist before anything arrives on them
    pdl_launch_dependents();

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer: every lane with a copy of its own per stage
        int stage = 0;
        uint32_t phase = 0;
        const uint32_t full_issuer = kCtas == 2 ? map_to_cta(smem_u32(&full[0]), 0) : 0u;
        const int bnh = p.BN / kCtas;                                   // B rows that this CTA stages
        const int na = kAMn ? kBM / 64 : 1;
        const int nb = kBMn ? bnh / 64 : kMode == kDenseGated && kCtas == 1 ? 2 : 1;
        const bool is_a = lane < na, active = lane < na + nb;
        const int piece = is_a ? lane : lane - na;
        const uint32_t dst_off = is_a ? (uint32_t)piece * (kABytes / na) : p.a_bytes + (uint32_t)piece * (uint32_t)(bnh * kRowBytes / nb);
        constexpr int kTerms = kInt8 ? kRowBytes : kRowBytes / 2;       // of the reduction per stage
        const bool mn = is_a ? kAMn : kBMn;
        const int step0 = mn ? 0 : kTerms, step1 = mn ? kTerms : 0;
        bool first = true;
        for (int t = first_tile; t < p.total; t += tile_step) {
            const TileAt at = tile_at(p, t);
            const int z = kMode == kDenseGradW ? p.first + at.z : 0;
            // the first of the rows that this copy brings
            int row;
            const CUtensorMap *map = is_a ? &maps.A[z] : &maps.B[0];
            if (is_a) {
                row = (at.tm * kCtas + rank) * kBM + piece * 64;        // (of MN-major pieces; else piece is 0)
            } else if (kMode == kDenseGated) {
                // a pair's CTA has one of the two weights, a lone CTA both
                row = at.tn * p.out_cols;
                map = &maps.B[kCtas == 2 ? rank : piece & 1];
            } else {
                row = at.tn * p.BN + rank * bnh + piece * 64;
            }
            int c0 = mn ? row : 0, c1 = mn ? 0 : row;
            if (first) pdl_wait();
            first = false;
            for (int kb = 0; kb < p.num_kb; ++kb) {
                mbar_wait(&empty[stage], phase ^ 1, p.err, 1);
                if (lane == 0 && rank == 0) mbar_arrive_expect_tx(&full[stage], p.stage_bytes * kCtas);
                __syncwarp();
                if (kMode == kDenseGradX && kb == p.seg_kb) {
                    map = is_a ? &maps.A[1] : &maps.B[1];
                    c0 = mn ? row : 0;
                    c1 = mn ? 0 : row;
                }
                uint8_t *dst = stages + (size_t)stage * p.stage_bytes + dst_off;
                if (active) {
                    if (kCtas == 2) tma_load_2d_pair(dst, map, full_issuer + (uint32_t)stage * 8u, c0, c1);
                    else tma_load_2d(dst, map, &full[stage], c0, c1);
                }
                c0 += step0;
                c1 += step1;
                if (++stage == p.num_stages) { stage = 0; phase ^= 1; }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (of a pair: the even CTA)
        if ((kCtas == 1 || rank == 0) && elect_one()) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            // K-major: 8-row groups 1024 bytes apart, an instruction 32 bytes further along the swizzled rows.  MN-major: blocks of 64
            // rows or columns 64 x 128 bytes apart, groups of 8 terms 1024 bytes apart, an instruction two of those further.
            const uint64_t k_tmpl = make_smem_desc(0, 16, 1024, kSwizzle128B), mn_tmpl = make_smem_desc(0, 64 * kRowBytes, 1024, kSwizzle128B);
            const uint64_t a_tmpl = kAMn ? mn_tmpl : k_tmpl, b_tmpl = kBMn ? mn_tmpl : k_tmpl;
            const uint32_t a_hi = (uint32_t)(a_tmpl >> 32), b_hi = (uint32_t)(b_tmpl >> 32);
            const uint32_t a_lo = (uint32_t)a_tmpl | ((smem_u32(stages) >> 4) & 0x3FFFu);
            const uint32_t b_lo = (uint32_t)b_tmpl | (((smem_u32(stages) + p.a_bytes) >> 4) & 0x3FFFu);
            const uint32_t stage16 = p.stage_bytes >> 4;
            constexpr uint32_t kA16 = (kAMn ? 2048u : 32u) >> 4, kB16 = (kBMn ? 2048u : 32u) >> 4;
            for (int t = first_tile; t < p.total; t += tile_step) {
                if (kCtas == 2) mbar_wait_cluster(&tmem_empty[acc], acc_phase ^ 1, p.err, 2);
                else mbar_wait(&tmem_empty[acc], acc_phase ^ 1, p.err, 2);
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + (uint32_t)acc * kMaxBN;
                uint32_t accumulate = 0;
                for (int kb = 0; kb < p.num_kb; ++kb) {
                    mbar_wait(&full[stage], phase, p.err, 3);
                    tc_fence_after_sync();
                    const uint32_t al = a_lo + (uint32_t)stage * stage16, bl = b_lo + (uint32_t)stage * stage16;
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        if (kInt8) {
                            if (kCtas == 2) mma_i8_lohi_pair(d_tmem, al + k * kA16, a_hi, bl + k * kB16, b_hi, p.idesc, accumulate);
                            else mma_i8_lohi(d_tmem, al + k * kA16, a_hi, bl + k * kB16, b_hi, p.idesc, accumulate);
                        } else {
                            if (kCtas == 2) mma_f16_lohi_pair(d_tmem, al + k * kA16, a_hi, bl + k * kB16, b_hi, p.idesc, accumulate);
                            else mma_f16_lohi(d_tmem, al + k * kA16, a_hi, bl + k * kB16, b_hi, p.idesc, accumulate);
                        }
                        accumulate = 1;
                    }
                    if (kCtas == 2) mma_commit_pair(&empty[stage]);
                    else mma_commit(&empty[stage]);
                    if (++stage == p.num_stages) { stage = 0; phase ^= 1; }
                }
                if (kCtas == 2) mma_commit_pair(&tmem_full[acc]);
                else mma_commit(&tmem_full[acc]);
                acc ^= 1;
                if (acc == 0) acc_phase ^= 1;
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue
        pdl_wait();
        const int q = warp & 3, half = (warp - 2) >> 2;
        uint8_t *buf = staging + (warp - 2) * kBlockBytes;
        const bool wide = p.y_type == ONNXB_FLOAT;
        const int block_cols = wide ? 32 : 64;                 // columns of 128 bytes
        int acc = 0;
        uint32_t acc_phase = 0;
        const uint32_t peer_tmem_empty = kCtas == 2 ? map_to_cta(smem_u32(&tmem_empty[0]), 0) : 0u;
        for (int t = first_tile; t < p.total; t += tile_step) {
            const TileAt at = tile_at(p, t);
            const int row0 = (at.tm * kCtas + rank) * kBM + q * 32, row = row0 + lane;
            const int n0 = at.tn * p.out_cols, cols = min(p.out_cols, p.N - n0);
            const int blocks = (cols + block_cols - 1) / block_cols;
            const int lo = half ? (blocks + 1) / 2 : 0, hi = half ? blocks : (blocks + 1) / 2;
            // Scales and addends: the row's, and this lane's column's of the chunk of 32 that comes next, asked for ahead of it
            const float sa = kInt8 && row < p.M ? __ldg(p.a_scale + row) : 0.f;
            float s0 = 0.f, s1 = 0.f;                          // (s1: Wu's scale, or the plain product's addend)
            auto fetch = [&](int col) {
                const bool in = col + lane < cols;
                s0 = in ? __ldg(p.b_scale0 + n0 + col + lane) : 0.f;
                s1 = !in ? 0.f : kMode == kDenseGated ? __ldg(p.b_scale1 + n0 + col + lane) : p.bias ? __ldg(p.bias + n0 + col + lane) : 0.f;
            };
            if (kInt8) fetch(lo * block_cols);
            mbar_wait(&tmem_full[acc], acc_phase, p.err, 4);
            tc_fence_after_sync();
            if (row0 < p.M) {
                const uint32_t tbase = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * kMaxBN);
                for (int which = 0; which < p.outs; ++which) {
                    const int y = kMode == kDenseGradW ? p.first + at.z : which;
#pragma unroll 1
                    for (int b = lo; b < hi; ++b) {
                        // (TMA writes whole pieces of 16 bytes: not where the last columns fill none, since what follows is not Y's)
                        const bool by_tma = p.y_tma[y] == 2 || (p.y_tma[y] && (b + 1) * block_cols <= cols);
                        if (lane == 0) tma_store_wait_read<0>();                // the buffer's last block has gone
                        __syncwarp();
#pragma unroll 1
                        for (int c = 0; c < block_cols && b * block_cols + c < p.out_cols; c += 32) {
                            const int col = b * block_cols + c;
                            uint32_t v[32];
                            float f[32];
                            if (kMode == kDenseGated) {
                                uint32_t w[32];
                                tmem_ld_32x32(tbase + (uint32_t)(which == 2 ? p.out_cols + col : col), v);
                                if (which == 0) tmem_ld_32x32(tbase + (uint32_t)(p.out_cols + col), w);
                                tmem_ld_wait();
                                const float c0 = s0, c1 = s1;
                                if (kInt8) {
                                    fetch(col + 32);
                                    // (one factor after the other: the sum may be 0 where the factors' product is infinite)
#pragma unroll
                                    for (int j = 0; j < 32; ++j) {
                                        f[j] = (float)(int)v[j] * sa * __shfl_sync(0xffffffffu, c0, j);
                                        w[j] = __float_as_uint((float)(int)w[j] * sa * __shfl_sync(0xffffffffu, c1, j));
                                    }
                                } else {
#pragma unroll
                                    for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]);
                                }
                                if (which == 0) {
#define ONNXB_GATE(kind) _Pragma("unroll") for (int j = 0; j < 32; ++j) f[j] = activate(kind, f[j]) * __uint_as_float(w[j])
                                    if (p.activation == ONNXB_SILU) { ONNXB_GATE(ONNXB_SILU); }
                                    else if (p.activation == ONNXB_GELU) { ONNXB_GATE(ONNXB_GELU); }
                                    else if (p.activation == ONNXB_GELU_TANH) { ONNXB_GATE(ONNXB_GELU_TANH); }
                                    else { ONNXB_GATE(ONNXB_RELU); }
#undef ONNXB_GATE
                                }
                            } else {
                                tmem_ld_32x32(tbase + (uint32_t)col, v);
                                tmem_ld_wait();
                                if (kInt8) {
                                    const float c0 = s0, c1 = s1;
                                    fetch(col + 32);
#pragma unroll
                                    for (int j = 0; j < 32; ++j) {
                                        f[j] = (float)(int)v[j] * sa * __shfl_sync(0xffffffffu, c0, j) + __shfl_sync(0xffffffffu, c1, j);
                                        if (p.relu) f[j] = fmaxf(f[j], 0.f);
                                    }
                                } else {
#pragma unroll
                                    for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]);
                                }
                            }
                            // the lane's row of the block, 16-byte piece i at position i ^ (lane % 8): the 128-byte swizzle
                            if (wide) {
#pragma unroll
                                for (int i = 0; i < 8; ++i)
                                    *reinterpret_cast<float4 *>(buf + lane * kRowBytes + ((i ^ (lane & 7)) << 4)) =
                                        make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
                            } else {
                                uint32_t h[16];
                                if (p.y_type == ONNXB_FLOAT16) {
#pragma unroll
                                    for (int i = 0; i < 16; ++i) h[i] = pack<__half2>(f[2 * i], f[2 * i + 1]);
                                } else {
#pragma unroll
                                    for (int i = 0; i < 16; ++i) h[i] = pack<__nv_bfloat162>(f[2 * i], f[2 * i + 1]);
                                }
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    *reinterpret_cast<uint4 *>(buf + lane * kRowBytes + (((c / 8 + i) ^ (lane & 7)) << 4)) =
                                        make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
                            }
                        }
                        const int col0 = n0 + b * block_cols;
                        if (by_tma) {
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) {
                                tma_store_2d(&maps.Y[y], buf, col0, row0);
                                tma_store_commit();
                            }
                        } else {
                            // rows that TMA cannot address: read back row by row, a word per lane
                            __syncwarp();
                            const int rows = min(32, p.M - row0), left = cols - b * block_cols;
                            for (int r = 0; r < rows; ++r) {
                                const uint32_t word = *reinterpret_cast<const uint32_t *>(buf + r * kRowBytes + ((((lane >> 2) ^ (r & 7)) << 4) | ((lane & 3) << 2)));
                                const long long at_row = (long long)(row0 + r) * p.y_ld[y] + col0;
                                if (wide) {
                                    if (lane < left) static_cast<uint32_t *>(p.Y[y])[at_row + lane] = word;
                                } else {
                                    uint16_t *out = static_cast<uint16_t *>(p.Y[y]) + at_row + 2 * lane;
                                    if (2 * lane < left) out[0] = (uint16_t)word;
                                    if (2 * lane + 1 < left) out[1] = (uint16_t)(word >> 16);
                                }
                            }
                            __syncwarp();
                        }
                    }
                }
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (kCtas == 2) mbar_arrive_remote(peer_tmem_empty + (uint32_t)acc * 8u);
                else mbar_arrive(&tmem_empty[acc]);
            }
            acc ^= 1;
            if (acc == 0) acc_phase ^= 1;
        }
        if (lane == 0) tma_store_wait_all<0>();
    }

    tc_fence_before_sync();
    __syncthreads();
    if (kCtas == 2) cluster_sync_all();     // no CTA leaves while its peer may still signal it
    if (warp == 1) {
        __syncwarp();
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, 512);
    }
}

typedef void (*Kernel)(const Maps, const Params);

template <int kCtas>
Kernel kernel_for(int mode, bool int8) {
    if (int8) return mode == kDenseGated ? tc_dense_kernel<kCtas, true, kDenseGated> : tc_dense_kernel<kCtas, true, kDensePlain>;
    return mode == kDenseGated   ? tc_dense_kernel<kCtas, false, kDenseGated>
           : mode == kDenseGradX ? tc_dense_kernel<kCtas, false, kDenseGradX>
                                 : tc_dense_kernel<kCtas, false, kDenseGradW>;
}

// CTA pairs that run at once, asked of the device's occupancy once (as for tc_gemm_kernel, whose shared memory and threads are the same)
int max_pairs() {
    static std::atomic<int> cached{-1};
    int n = cached.load(std::memory_order_acquire);
    if (n >= 0) return n;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * 148);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemLimit;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    n = 0;
    auto kernel = tc_dense_kernel<2, false, kDenseGated>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = tc_host::num_sms() / 2;
    }
    cached.store(n, std::memory_order_release);
    return n;
}

// Tile shapes: one CTA with 128 rows or a pair with 256, and BN accumulator columns.  A stage (128 bytes of the reduction) takes the
// tensor cores 2 BN cycles on either; its operands come out of L2 at some 50 bytes a cycle and SM, of which a pair needs (128 + BN/2) * 128
// and a lone CTA (128 + BN) * 128.  On top of that a tile's epilogue, which the next tile's products hide but for the last one.
struct Tile {
    int ctas, BN;
};
bool tile_allowed(const DenseProblem &d, Tile t) {
    const bool b_mn = d.mode == kDenseGradX || d.mode == kDenseGradW;
    if (t.BN < 32 * t.ctas || t.BN > kMaxBN || t.BN % (32 * t.ctas)) return false;
    if (d.mode == kDenseGated) return t.BN % 64 == 0 && (t.BN == 64 || t.BN % 128 == 0);
    return !b_mn || t.BN % (64 * t.ctas) == 0;
}
Tile pick_tile(const DenseProblem &d, int products, int num_kb) {
    if (const char *e = getenv("ONNXB_DENSE_TILE")) {          // "<CTAs>x<BN>" pins the shape for A/B measurements and tests
        const Tile t{e[0] - '0', e[0] && e[1] == 'x' ? atoi(e + 2) : 0};
        if ((t.ctas == 1 || t.ctas == 2) && tile_allowed(d, t)) return t;
    }
    Tile best{1, 64};
    double best_cost = 1e300;
    for (int ctas = 1; ctas <= 2; ++ctas)
        for (int bn = 32; bn <= kMaxBN; bn += 32) {
            const Tile t{ctas, bn};
            if (!tile_allowed(d, t)) continue;
            const int out_cols = d.mode == kDenseGated ? bn / 2 : bn;
            const long long tiles = (long long)((d.M + kBM * ctas - 1) / (kBM * ctas)) * ((d.N + out_cols - 1) / out_cols) * products;
            const int units = ctas == 2 ? max_pairs() : tc_host::num_sms();
            const double waves = (double)((tiles + units - 1) / units);
            const double stage = std::max(2.0 * bn, (128.0 + bn / ctas) * kRowBytes / 50.0) + 30.0;
            const double epilogue = 1000.0 + 12.0 * bn;
            const double cost = waves * std::max(num_kb * stage, epilogue) + epilogue;
            if (cost < best_cost * (1 - 1e-9)) {
                best_cost = cost;
                best = t;
            }
        }
    return best;
}

}  // namespace

int launch_tc_dense(const DenseProblem &d, cudaStream_t stream) {
    using namespace tc_host;
    const bool int8 = d.type == ONNXB_INT8, gated = d.mode == kDenseGated;
    const bool a_mn = d.mode == kDenseGradW, b_mn = a_mn || d.mode == kDenseGradX;
    const int bytes = type_bytes(d.type), terms = kRowBytes / bytes, y_bytes = type_bytes(d.y_type);
    Params p{};
    p.M = d.M; p.N = d.N;
    p.seg_kb = (d.K + terms - 1) / terms;
    p.num_kb = d.mode == kDenseGradX ? 2 * p.seg_kb : p.seg_kb;
    p.first = a_mn && !d.Y[0] ? 1 : 0;
    p.products = a_mn && d.Y[0] && d.Y[1] ? 2 : 1;
    const Tile tile = pick_tile(d, p.products, p.num_kb);
    p.BN = tile.BN;
    p.out_cols = gated ? p.BN / 2 : p.BN;
    p.tiles_m = (d.M + kBM * tile.ctas - 1) / (kBM * tile.ctas);
    p.tiles_n = (d.N + p.out_cols - 1) / p.out_cols;
    p.band = 8;
    const long long total = (long long)p.tiles_m * p.tiles_n * p.products;
    if (total > 0x7fffffffLL - 65536 || (long long)p.band * p.tiles_n > 0x7fffffffLL) return (int)cudaErrorInvalidValue;
    p.total = (int)total;
    const int bnh = p.BN / tile.ctas;
    // Few tokens: no more of A's rows than there are.  The tensor cores read 128 all the same, what lies behind being other operands'
    // (or the staging blocks'); those rows of the accumulator are nobody's, and the ring is as much deeper.
    const int a_rows = tile.ctas == 1 && !a_mn && d.M <= 64 ? (d.M <= 16 ? 16 : d.M <= 32 ? 32 : 64) : kBM;
    p.a_bytes = (uint32_t)(a_rows * kRowBytes);
    p.stage_bytes = p.a_bytes + (uint32_t)(bnh * kRowBytes);
    p.num_stages = std::min(kMaxStages, (kSmemLimit - 1024 - kBarrierBytes - kStagingBytes) / (int)p.stage_bytes);
    p.idesc = int8 ? make_idesc_s8(kBM * tile.ctas, p.BN) : make_idesc_f16(kBM * tile.ctas, p.BN, d.type == ONNXB_BFLOAT16, a_mn, b_mn);
    p.a_scale = d.a_scale; p.b_scale0 = d.b_scale[0]; p.b_scale1 = d.b_scale[1]; p.bias = d.bias;
    p.relu = d.relu; p.activation = d.activation;
    p.y_type = d.y_type;
    p.outs = gated && d.Y[1] ? 3 : 1;
    p.err = device_status_ptr();
    if (!p.err) return (int)cudaErrorUnknown;

    Maps maps;
    // An operand: (terms, rows) boxes of 128 bytes x `box` rows, or MN-major (rows, terms) boxes of 64 x 64
    auto operand = [&](CUtensorMap *m, const DenseOperand &o, bool mn, int rows, int box) {
        const uint64_t dims[2] = {(uint64_t)(mn ? rows : d.K), (uint64_t)(mn ? d.K : rows)};
        const uint64_t pitch = (uint64_t)((mn ? d.K : rows) > 1 ? o.ld * bytes : (o.ld * bytes + 15) / 16 * 16);
        const uint32_t boxes[2] = {mn ? 64u : (uint32_t)terms, mn ? 64u : (uint32_t)box};
        return make_tmap_of(bytes, m, o.p, 2, dims, &pitch, boxes, kTmapSwizzle128);
    };
    for (int i = 0; i < 2; ++i) {
        const DenseOperand &a = d.A[d.mode == kDenseGradX || a_mn ? i : 0], &b = d.B[d.mode == kDenseGradX || gated ? i : 0];
        if (!operand(&maps.A[i], a, a_mn, d.M, a_rows) || !operand(&maps.B[i], b, b_mn, d.N, gated ? p.out_cols : bnh)) return (int)cudaErrorInvalidValue;
    }
    for (int i = 0; i < 3; ++i) {
        maps.Y[i] = maps.A[0];                     // (never used where y_tma is not set)
        p.Y[i] = d.Y[i]; p.y_ld[i] = d.y_ld[i];
        const uint64_t pitch = (uint64_t)(d.M > 1 ? d.y_ld[i] * y_bytes : (d.y_ld[i] * y_bytes + 15) / 16 * 16);
        if (!d.Y[i] || pitch % 16 || reinterpret_cast<uintptr_t>(d.Y[i]) % 16 || p.out_cols * y_bytes % kRowBytes) continue;
        const uint64_t dims[2] = {(uint64_t)d.N, (uint64_t)d.M};
        const uint32_t box[2] = {(uint32_t)(kRowBytes / y_bytes), 32};
        if (make_tmap_of(y_bytes, &maps.Y[i], d.Y[i], 2, dims, &pitch, box, kTmapSwizzle128)) p.y_tma[i] = (long long)d.N * y_bytes % 16 == 0 ? 2 : 1;
    }
    const size_t smem = smem_with_tmem(1024 + (size_t)p.num_stages * p.stage_bytes + kStagingBytes + kBarrierBytes, 512);
    const Kernel kernel = tile.ctas == 2 ? kernel_for<2>(d.mode, int8) : kernel_for<1>(d.mode, int8);
    const cudaError_t attr_err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
    if (attr_err != cudaSuccess) return (int)attr_err;
    const int units = tile.ctas == 2 ? max_pairs() : num_sms();
    const int grid = (int)std::min<long long>(total, units) * tile.ctas;
    const cudaError_t e = tile.ctas == 2 ? launch_pdl_cluster(kernel, 2, dim3(grid), dim3(kThreads), smem, stream, maps, p)
                                         : launch_pdl(kernel, dim3(grid), dim3(kThreads), smem, stream, maps, p);
    count_launch();
    return (int)e;
}

}  // namespace onnxb
