// Dense layers of 8- and 16-bit operands on the 5th-generation tensor cores: onnx_gemm_int8_run, onnx_gated_run (and of 8-bit
// operands) and the three products of its gradients (DenseMode in dense.h).
//
// The pipeline is that of tc_gemm.cu: a persistent CTA (or a pair of two on one tile) per SM, 320 threads,
//   warp 0    TMA producer, a ring of stages of 128 bytes along the reduction (64 16-bit or 128 8-bit terms), or of 2 or 4 times
//             that where tiles are small, since a stage costs its two single threads 240 cycles, and 170 more for each block;
//   warp 1    one thread issues tcgen05.mma kind::f16 or kind::i8 into one of two TMEM accumulators;
//   warps 2-9 epilogue: tcgen05.ld, the mathematics, 32-row blocks of 128 bytes staged in swizzled shared memory, TMA stores (plain ones
//             where Y's rows do not begin at multiples of 16 bytes).
// What is its own:
//   - The gated block is one product: half of a tile's B rows are Wg's, half Wu's of the same channels, so that an accumulator holds
//     a channel's gate in column j and its other factor in column BN/2 + j, in the same TMEM lane.  X is read once for both, and
//     the pair's form costs nothing: each CTA stages one of the two.
//   - The gradients are one launch: dX's tiles, which are few and long, then those of dWg and dWu, handed out so that the units that got
//     one tile of dX less get as many more of the others as that one takes.
//   - dX = dG Wg + dU Wu is one sum: the reduction runs over dG's channels, then dU's, with the other tensor maps from there on.
//   - dWg = dG^T X and dWu = dU^T X take their operands as they lie, the reduction (tokens) along the rows: MN-major, boxes of 64
//     by 64 or, two K blocks a stage, 128.  The same for Wg and Wu in dX.  No transposed copy is made, and dG's map serves both uses: its
//     boxes are 64 terms by so many tokens, or 64 channels by so many terms.
//   - Few tiles with a long reduction share it: the CTAs of a cluster have a part each of one tile's, and every quarter of a block of
//     columns is added up by one of them, from what the others write into its shared memory, in the parts' order.
// Measured (a burst; under the power cap of a long run in brackets): gated block 4096 x 4096 x 10240 in bf16 with G and U kept 450 us, 1.53
// PFLOP/s (535), of 8-bit operands 203 us, 3.4 POP/s (247); 8-bit Gemm 4096 x 10240 x 4096 110 us, 3.1 POP/s (130); the three products of
// the gradients at the first size 880 us, 1.56 PFLOP/s: the tensor pipe is 90 to 96 % busy.  Small tiles are bound by a stage's
// 410 cycles (of one block), short reductions by the epilogue's latencies (two warps a scheduler), few tokens by the weights' bytes.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdlib>
#include <cstring>

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
    int num_kb;                // stages of the reduction
    int ks, full_kb;           // K blocks of 128 bytes per stage; stages whose blocks all lie inside the reduction
    int split, part_kb;        // CTAs that share a tile's, and the stages of each
    // kDenseGrad.  dX: row tiles, all tiles (of all parts of the reduction), stages (half of them of the first of its two terms), parts,
    // stages of a part, rows of a part's plane, whether dX's tiles go to planes of fp32.  dWg and dWu: row tiles, all tiles, stages, the first that is wanted, tiles that a
    // unit with one tile of dX less takes before the others.
    int x_tiles_m, x_tiles, x_kb, x_parts, x_part_kb, x_part_rows, x_planes;
    int channels, w_tiles_m, w_tiles, w_kb, w_first, w_before;
    uint32_t idesc_x;
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
    CUtensorMap A[2], B[3], Y[3];
    CUtensorMap A4, B4[2];     // (terms, rows, K block, 1) views for stages of several blocks, or (terms, 8 rows, K block, group of rows)
};

struct TileAt {
    int tm, tn, z;             // z: the product, or the part of dX's reduction
    int kb0, kb1;              // stages
    bool x;                    // a tile of dX
};
// Tiles of one product lie in bands of `band` row tiles, a band's columns one after the other, so that the tiles in flight share
// their operands in L2 (of 148 SMs' 74 pairs at band 8: 8 row tiles and 9 column tiles), and a band's rows stay there.
__device__ __forceinline__ void place(const Params &p, int tiles_m, int t, TileAt &at) {
    const int per = tiles_m * p.tiles_n;
    at.z = t / per;
    const int r = t - at.z * per, b = r / (p.band * p.tiles_n), rr = r - b * p.band * p.tiles_n;
    const int rows = min(p.band, tiles_m - b * p.band);
    at.tn = rr / rows;
    at.tm = b * p.band + rr - at.tn * rows;
}
// The n-th tile of a unit (a CTA or a pair) of `units`; false: there is none
template <int kMode, bool kSplit>
__device__ __forceinline__ bool nth_tile(const Params &p, int unit, int units, int n, TileAt &at) {
    at.x = false;
    if (kSplit) {              // a cluster has one
        place(p, p.tiles_m, unit, at);
        at.kb0 = (int)cluster_ctarank() * p.part_kb;
        at.kb1 = min(at.kb0 + p.part_kb, p.num_kb);
        return n == 0;
    }
    at.kb0 = 0;
    at.kb1 = kMode == kDenseGrad ? p.w_kb : p.num_kb;
    if (kMode != kDenseGrad) {
        const int t = unit + n * units;
        if (t >= p.total) return false;
        place(p, p.tiles_m, t, at);
        return true;
    }
    const int longer = p.x_tiles % units, own = p.x_tiles / units + (unit < longer);        // (units with one tile of dX more)
    if (n < own) {
        place(p, p.x_tiles_m, unit + n * units, at);
        at.x = true;
        at.kb0 = at.z * p.x_part_kb;
        at.kb1 = min(at.kb0 + p.x_part_kb, p.x_kb);
        return true;
    }
    const int m = n - own, before = longer && unit >= longer ? p.w_before : 0;
    int t;
    if (m < before) t = unit - longer + m * (units - longer);
    else t = (longer ? p.w_before * (units - longer) : 0) + (m - before) * units + (unit >= longer ? unit - longer : unit - longer + units);
    if (t >= p.w_tiles) return false;
    place(p, p.w_tiles_m, t, at);
    return true;
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

template <int kCtas, bool kInt8, int kMode, bool kSplit = false>
__global__ void __launch_bounds__(kThreads, 1) tc_dense_kernel(const __grid_constant__ Maps maps, const Params p) {
    constexpr bool kGrad = kMode == kDenseGrad;
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
    const int unit = blockIdx.x / (kSplit ? p.split : kCtas), units = gridDim.x / kCtas;
    TileAt at;

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
        // (of those that there are)
        const bool blocks = !kGrad && p.ks > 1 && p.full_kb > 0;
        prefetch_tmap(blocks ? &maps.A4 : &maps.A[0]);
        if (!kGrad || p.x_tiles) prefetch_tmap(blocks ? &maps.B4[0] : &maps.B[0]);
        if (kMode == kDenseGated) prefetch_tmap(blocks ? &maps.B4[1] : &maps.B[1]);
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
    // (kSplit: what the other CTAs send goes where the ring was, once all of them are done with theirs)
    const int part = kSplit ? (int)cluster_ctarank() : 0;
    pdl_launch_dependents();

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer: every lane with a copy of its own per stage
        int stage = 0;
        uint32_t phase = 0;
        const uint32_t full_issuer = kCtas == 2 ? map_to_cta(smem_u32(&full[0]), 0) : 0u;
        const int bnh = p.BN / kCtas;                                   // B rows that this CTA stages
        const int na = kGrad ? kBM / 64 : 1;
        const int nb = kGrad ? bnh / 64 : kMode == kDenseGated && kCtas == 1 ? 2 : 1;
        const bool is_a = lane < na, active = lane < na + nb;
        const int piece = is_a ? lane : lane - na;
        // (a piece of 64 columns has a block of the reduction after the other; the two pieces of dG are such, or for dX its rows')
        const uint32_t dst_off = is_a ? (uint32_t)(piece * p.ks) * (kABytes / na)
                                      : (uint32_t)p.ks * (p.a_bytes + (uint32_t)piece * (uint32_t)(bnh * kRowBytes / nb));
        constexpr int kTerms = kInt8 ? kRowBytes : kRowBytes / 2;       // of the reduction per stage
        for (int n = 0; nth_tile<kMode, kSplit>(p, unit, units, n, at); ++n) {
            // the first of the rows that this copy brings (along the output's rows or columns), and whether they lie along a row in memory
            int row = is_a ? (at.tm * kCtas + rank) * kBM : at.tn * p.BN + rank * bnh;
            const bool mn = kGrad && !(is_a && at.x);
            if (kGrad && (mn || p.ks == 1)) row += piece * 64;
            const CUtensorMap *map = is_a ? &maps.A[0] : &maps.B[0];
            int term = at.kb0 * kTerms * p.ks;
            const int ahead = kGrad && p.ks == 2 && !mn ? piece * kTerms : 0;          // (dX's two pieces of dG: a block each)
            if (kMode == kDenseGated && !is_a) {
                // a pair's CTA has one of the two weights, a lone CTA both
                row = at.tn * p.out_cols;
                map = &maps.B[kCtas == 2 ? rank : piece & 1];
            }
            if (kGrad && !at.x) map = is_a ? &maps.A[p.w_first + at.z] : &maps.B[2];
            if (kGrad && at.x && at.kb0 * 2 >= p.x_kb) {
                map += 1;
                term -= p.x_kb / 2 * kTerms * p.ks;
            }
            if (n == 0) pdl_wait();
            for (int kb = at.kb0; kb < at.kb1; ++kb) {
                mbar_wait(&empty[stage], phase ^ 1, p.err, 1);
                if (lane == 0 && rank == 0) mbar_arrive_expect_tx(&full[stage], p.stage_bytes * kCtas);
                __syncwarp();
                if (!kGrad && p.ks > 1) {
                    // Several blocks: in one copy per operand, or at the end of the reduction, past which the view would go on into
                    // the next row, block by block
                    uint8_t *at_stage = stages + (size_t)stage * p.stage_bytes;
                    const uint32_t bar = full_issuer + (uint32_t)stage * 8u;
                    const bool whole = kb < p.full_kb;
                    const int s = whole ? 0 : lane % p.ks, o = whole ? lane : lane / p.ks;       // block, operand
                    if (o <= nb) {
                        const bool a = o == 0;
                        const int w = kMode == kDenseGated && !a ? (kCtas == 2 ? rank : o - 1) : 0, rows = a ? (int)p.a_bytes / kRowBytes : bnh / nb;
                        uint8_t *to = at_stage + (a ? 0u : (uint32_t)p.ks * (p.a_bytes + (uint32_t)((o - 1) * rows * kRowBytes))) + (uint32_t)(s * rows * kRowBytes);
                        const int first = a ? (at.tm * kCtas + rank) * kBM : kMode == kDenseGated ? at.tn * p.out_cols : at.tn * p.BN + rank * bnh;
                        const int block = kb * p.ks + s;
                        if (whole) {
                            // (one instruction for all lanes: see tc_gemm.cu)
                            const bool groups = kMode == kDenseGated && kCtas == 1 && !a;
                            const int c1 = groups ? 0 : first, c3 = groups ? first / 8 : 0;
                            if (kCtas == 2) tma_load_4d_pair(to, a ? &maps.A4 : &maps.B4[w], bar, 0, c1, block, c3);
                            else tma_load_4d(to, a ? &maps.A4 : &maps.B4[w], &full[stage], 0, c1, block, c3);
                        } else {
                            if (kCtas == 2) tma_load_2d_pair(to, a ? &maps.A[0] : &maps.B[w], bar, block * kTerms, first);
                            else tma_load_2d(to, a ? &maps.A[0] : &maps.B[w], &full[stage], block * kTerms, first);
                        }
                    }
                    if (++stage == p.num_stages) { stage = 0; phase ^= 1; }
                    continue;
                }
                if (kGrad && at.x && kb > at.kb0 && kb * 2 == p.x_kb) {
                    map += 1;
                    term = 0;
                }
                uint8_t *dst = stages + (size_t)stage * p.stage_bytes + dst_off;
                if (active) {
                    const int c0 = mn ? row : term + ahead, c1 = mn ? term : row;
                    if (kCtas == 2) tma_load_2d_pair(dst, map, full_issuer + (uint32_t)stage * 8u, c0, c1);
                    else tma_load_2d(dst, map, &full[stage], c0, c1);
                }
                term += kTerms * p.ks;
                if (++stage == p.num_stages) { stage = 0; phase ^= 1; }
            }
        }
        if (kSplit) {
            __syncwarp();
            cluster_sync_all();
            cluster_sync_all();
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (of a pair: the even CTA)
        if ((kCtas == 1 || rank == 0) && elect_one()) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            // K-major: 8-row groups 1024 bytes apart, an instruction 32 bytes further along the swizzled rows.  MN-major: blocks of 64
            // rows or columns a stage's 64 or 128 terms of 128 bytes apart, groups of 8 terms 1024 bytes apart, an instruction two of those further.
            const uint64_t k_tmpl = make_smem_desc(0, 16, 1024, kSwizzle128B), mn_tmpl = make_smem_desc(0, 64u * kRowBytes * (uint32_t)p.ks, 1024, kSwizzle128B);
            // (Both weights of the gated block in a lone CTA's stage of several blocks: a block's 8-row groups lie as far apart as all blocks'
            // take, so that one weight's go on where the other's end)
            const bool groups = kMode == kDenseGated && kCtas == 1;
            const uint64_t b_tmpl = kGrad ? mn_tmpl : make_smem_desc(0, 16, groups ? 1024u * (uint32_t)p.ks : 1024u, kSwizzle128B);
            const uint32_t b_hi = (uint32_t)(b_tmpl >> 32);
            const uint32_t a_at = (smem_u32(stages) >> 4) & 0x3FFFu, b_lo = (uint32_t)b_tmpl | (((smem_u32(stages) + (uint32_t)p.ks * p.a_bytes) >> 4) & 0x3FFFu);
            const uint32_t stage16 = p.stage_bytes >> 4, b_block16 = (kGrad ? 64u * kRowBytes : groups ? 1024u : (uint32_t)(p.BN / kCtas * kRowBytes)) >> 4;
            constexpr uint32_t kK16 = 32u >> 4, kMn16 = 2048u >> 4, kB16 = kGrad ? kMn16 : kK16;
            for (int n = 0; nth_tile<kMode, kSplit>(p, unit, units, n, at); ++n) {
                const bool a_mn = kGrad && !at.x;
                const uint64_t a_tmpl = a_mn ? mn_tmpl : k_tmpl;
                const uint32_t a_hi = (uint32_t)(a_tmpl >> 32), a_lo = (uint32_t)a_tmpl | a_at, a16 = a_mn ? kMn16 : kK16;
                const uint32_t idesc = kGrad && at.x ? p.idesc_x : p.idesc, a_block16 = (a_mn ? 64u * kRowBytes : p.a_bytes) >> 4;
                if (kCtas == 2) mbar_wait_cluster(&tmem_empty[acc], acc_phase ^ 1, p.err, 2);
                else mbar_wait(&tmem_empty[acc], acc_phase ^ 1, p.err, 2);
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + (uint32_t)acc * kMaxBN;
                uint32_t accumulate = 0;
                for (int kb = at.kb0; kb < at.kb1; ++kb) {
                    mbar_wait(&full[stage], phase, p.err, 3);
                    tc_fence_after_sync();
                    uint32_t al = a_lo + (uint32_t)stage * stage16, bl = b_lo + (uint32_t)stage * stage16;
                    for (int s = 0; s < p.ks; ++s) {
                        // a block's four instructions
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) {
                            if (kInt8) {
                                if (kCtas == 2) mma_i8_lohi_pair(d_tmem, al + k * a16, a_hi, bl + k * kB16, b_hi, idesc, accumulate);
                                else mma_i8_lohi(d_tmem, al + k * a16, a_hi, bl + k * kB16, b_hi, idesc, accumulate);
                            } else {
                                if (kCtas == 2) mma_f16_lohi_pair(d_tmem, al + k * a16, a_hi, bl + k * kB16, b_hi, idesc, accumulate);
                                else mma_f16_lohi(d_tmem, al + k * a16, a_hi, bl + k * kB16, b_hi, idesc, accumulate);
                            }
                            accumulate = 1;
                        }
                        al += a_block16;
                        bl += b_block16;
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
        if (kSplit) {
            __syncwarp();
            cluster_sync_all();
            cluster_sync_all();
        }
    } else {
        // ------------------------------------------------------------ epilogue
        pdl_wait();
        const int q = warp & 3, half = (warp - 2) >> 2;
        uint8_t *buf = staging + (warp - 2) * kBlockBytes;
        int acc = 0;
        uint32_t acc_phase = 0;
        const uint32_t peer_tmem_empty = kCtas == 2 ? map_to_cta(smem_u32(&tmem_empty[0]), 0) : 0u;
        for (int n = 0; nth_tile<kMode, kSplit>(p, unit, units, n, at); ++n) {
            // 32-bit results: of 8-bit operands where asked for, and the parts of a dX whose reduction is shared
            const bool parts = kGrad && at.x && p.x_planes, wide = kGrad ? parts : p.y_type == ONNXB_FLOAT;
            const int block_cols = wide ? 32 : 64;             // columns of 128 bytes
            const int M = kGrad && !at.x ? p.channels : p.M;
            const int row0 = (at.tm * kCtas + rank) * kBM + q * 32, row = row0 + lane;
            const int n0 = at.tn * p.out_cols, cols = min(p.out_cols, p.N - n0);
            const int blocks = (cols + block_cols - 1) / block_cols;
            const int lo = half ? (blocks + 1) / 2 : 0, hi = half ? blocks : (blocks + 1) / 2;
            // Scales and addends: the row's, and this lane's column's of the chunk of 32 that comes next, asked for ahead of it
            const float sa = kInt8 && row < M ? p.a_scale[row] : 0.f;
            float s0 = 0.f, s1 = 0.f;                          // (s1: Wu's scale, or the plain product's addend)
            auto fetch = [&](int col) {
                const bool in = col + lane < cols;
                s0 = in ? p.b_scale0[n0 + col + lane] : 0.f;
                s1 = !in ? 0.f : kMode == kDenseGated ? p.b_scale1[n0 + col + lane] : p.bias ? p.bias[n0 + col + lane] : 0.f;
            };
            if (kInt8 && !kSplit) fetch(lo * block_cols);
            mbar_wait(&tmem_full[acc], acc_phase, p.err, 4);
            tc_fence_after_sync();
            const uint32_t tbase = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * kMaxBN);
            // kSplit: a quarter (32 rows) of a block of results is added up by one CTA of the cluster, where each other CTA's 32 x 32 values
            // of it have a place of their own: four columns of a row by 32 rows, eight times.
            auto owner = [&](int blk) { return (blk * 4 + q) % p.split; };
            auto place_of = [&](int col, int from, int to) {
                const int in = col % p.out_cols, blk = in / block_cols, chunks = block_cols / 32, per = kMode == kDenseGated ? 2 : 1;
                const int slot = ((blk * 4 + q) / p.split * chunks + in % block_cols / 32) * per + (col >= p.out_cols ? 1 : 0);
                return (uint32_t)((slot * (p.split - 1) + from - (from > to ? 1 : 0)) * kBlockBytes + lane * 16);
            };
            if (kSplit) {
                cluster_sync_all();
                if (row0 < M) {
#pragma unroll 1
                    for (int col = half * 32; col < p.BN; col += 64) {
                        const int to = owner(col % p.out_cols / block_cols);
                        if (to == part || col % p.out_cols >= cols) continue;
                        uint32_t v[32];
                        tmem_ld_32x32(tbase + (uint32_t)col, v);
                        tmem_ld_wait();
                        const uint32_t at_peer = map_to_cta(smem_u32(stages) + place_of(col, part, to), (uint32_t)to);
#pragma unroll
                        for (int j = 0; j < 32; j += 4) st_cluster_v4(at_peer + (uint32_t)(j * 128), v[j], v[j + 1], v[j + 2], v[j + 3]);
                    }
                }
                cluster_sync_all();
            }
            // 32 columns of the accumulator, of all parts
            auto load = [&](int col, uint32_t (&v)[32]) {
                tmem_ld_32x32(tbase + (uint32_t)col, v);
                if (!kSplit) return;
                tmem_ld_wait();
                uint32_t sum[32] = {};
#pragma unroll 1
                for (int s = 0; s < p.split; ++s) {
                    const uint8_t *from = stages + place_of(col, s, part);
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        uint4 x = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                        if (s != part) x = *reinterpret_cast<const uint4 *>(from + j * 128);
                        auto add = [](uint32_t a, uint32_t b) { return kInt8 ? a + b : __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); };
                        sum[j] = add(sum[j], x.x);
                        sum[j + 1] = add(sum[j + 1], x.y);
                        sum[j + 2] = add(sum[j + 2], x.z);
                        sum[j + 3] = add(sum[j + 3], x.w);
                    }
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = sum[j];
            };
            if (row0 < M) {
                // The two warps of a quarter share its blocks of all results in turns; of 8-bit operands, whose scales are fetched from
                // one to the next, a half each
#pragma unroll 1
                for (int item = kInt8 ? lo : half, items = kInt8 ? hi : blocks * p.outs; item < items; item += kInt8 ? 1 : 2) {
                    const int which = kInt8 || item < blocks ? 0 : item < 2 * blocks ? 1 : 2, b = item - which * blocks;
                    const int y = !kGrad ? which : at.x ? 0 : 1 + p.w_first + at.z;
                    if (kSplit && owner(b) != part) continue;
                    // (TMA writes whole blocks, and of those at Y's end whole pieces of 16 bytes: not where the tile ends inside a block, or
                    // the last columns fill no piece, since what follows is another tile's or not Y's)
                    const bool by_tma = p.y_tma[y] && (b + 1) * block_cols <= (p.y_tma[y] == 2 ? p.out_cols : cols);
                    if (lane == 0) tma_store_wait_read<0>();                // the buffer's last block has gone
                    __syncwarp();
#pragma unroll 1
                    for (int c = 0; c < block_cols && b * block_cols + c < p.out_cols; c += 32) {
                        const int col = b * block_cols + c;
                        uint32_t v[32];
                        float f[32];
                        if (kMode == kDenseGated) {
                            uint32_t w[32];
                            if (kInt8 && kSplit) fetch(col);
                            load(which == 2 ? p.out_cols + col : col, v);
                            if (which == 0) load(p.out_cols + col, w);
                            tmem_ld_wait();
                            const float c0 = s0, c1 = s1;
                            if (kInt8) {
                                if (!kSplit) fetch(col + 32);
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
                            if (kInt8 && kSplit) fetch(col);
                            load(col, v);
                            tmem_ld_wait();
                            if (kInt8) {
                                const float c0 = s0, c1 = s1;
                                if (!kSplit) fetch(col + 32);
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
                            tma_store_2d(&maps.Y[y], buf, col0, parts ? at.z * p.x_part_rows + row0 : row0);
                            tma_store_commit();
                        }
                    } else {
                        // Rows that TMA cannot address: read back row by row, 8 bytes a lane and two rows at a time where they begin at
                        // multiples of 8, else 4 bytes a lane.  Short loops: most launches run this once or twice, out of cold
                        // instruction memory (with four rows' reads first and odd 16-bit rows shifted to whole words gated block
                        // 333 x 1000 x 2741 takes 12.9 us, 11.7 so; 2736 channels, by TMA, 10.6).
                        __syncwarp();
                        const int rows = min(32, M - row0), element = wide ? 4 : 2, left = (cols - b * block_cols) * element;
                        char *out = static_cast<char *>(p.Y[y]) + ((long long)row0 * p.y_ld[y] + col0) * element;
                        const long long pitch = p.y_ld[y] * element;
                        if (((reinterpret_cast<uintptr_t>(out) | (unsigned long long)pitch) & 7) == 0) {
                            const int at = lane % 16 * 8;
#pragma unroll 4
                            for (int r = lane / 16; r < rows; r += 2) {
                                const uint2 v = *reinterpret_cast<const uint2 *>(buf + r * kRowBytes + (((at >> 4) ^ (r & 7)) << 4 | (at & 8)));
                                char *to = out + r * pitch + at;
                                if (at + 8 <= left) *reinterpret_cast<uint2 *>(to) = v;
                                else if (at < left) {
                                    if (at + 4 <= left) *reinterpret_cast<uint32_t *>(to) = v.x;
                                    if (left & 2) *reinterpret_cast<uint16_t *>(to + (left & 4)) = (uint16_t)(left & 4 ? v.y : v.x);
                                }
                            }
                        } else {
                            const int at = lane * 4;
#pragma unroll 4
                            for (int r = 0; r < rows; ++r) {
                                const uint32_t v = *reinterpret_cast<const uint32_t *>(buf + r * kRowBytes + (((at >> 4) ^ (r & 7)) << 4 | (at & 12)));
                                char *to = out + r * pitch + at;
                                if (wide) {
                                    if (at < left) *reinterpret_cast<uint32_t *>(to) = v;
                                } else {
                                    if (at < left) *reinterpret_cast<uint16_t *>(to) = (uint16_t)v;
                                    if (at + 2 < left) *reinterpret_cast<uint16_t *>(to + 2) = (uint16_t)(v >> 16);
                                }
                            }
                        }
                        __syncwarp();
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
    return mode == kDenseGated ? tc_dense_kernel<kCtas, false, kDenseGated> : tc_dense_kernel<kCtas, false, kDenseGrad>;
}
Kernel split_kernel_for(int mode, bool int8) {
    if (!int8) return tc_dense_kernel<1, false, kDenseGated, true>;
    return mode == kDenseGated ? tc_dense_kernel<1, true, kDenseGated, true> : tc_dense_kernel<1, true, kDensePlain, true>;
}

// The kernel's shared memory allowed for, once a device (`index`: the kernel's, below 12)
cudaError_t allow_shared_memory(Kernel kernel, int index) {
    static std::atomic<uint64_t> done[12];
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done[index].load(std::memory_order_acquire) & bit)) return cudaSuccess;
    const cudaError_t set = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
    if (set == cudaSuccess && dev < 64) done[index].fetch_or(bit, std::memory_order_release);
    return set;
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

// Tile shapes: one CTA with 128 rows or a pair with 256, BN accumulator columns, and for few tiles a reduction shared by a cluster.  The
// estimate, in SM cycles, fitted to single waves of 8-bit products 128 x 1024 x 2048 and 12288 and gated blocks of 16-bit ones:
//   - a stage of ks K blocks takes the tensor cores 2 BN ks + 50, its two single threads 240 + 170 ks (75 for each copy beyond two), and its
//     operands' way out of L2 their bytes at 90 a cycle, or at what 8100 a cycle for all SMs leave each;
//   - a tile's epilogue 1000 + 13 BN, which the next tile's products hide but for the last one;
//   - a shared reduction 2500 + 28 BN for two CTAs, and a third and a half as much again for four and eight.
struct Tile {
    int ctas, BN;
    int split;                 // CTAs that share a tile's reduction, in a cluster
};
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
int ceil_int(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) / (unsigned)b); }      // (32 bits: a choice makes dozens)
bool tile_allowed(int mode, Tile t) {
    if (t.BN < 32 * t.ctas || t.BN > kMaxBN || t.BN % (32 * t.ctas)) return false;
    if (mode == kDenseGated) return t.BN % 64 == 0;
    return mode != kDenseGrad || t.BN % (64 * t.ctas) == 0;
}
int ring_bytes() { return kSmemLimit - 1024 - kBarrierBytes - kStagingBytes; }
// Few tokens: no more of A's rows than there are.  The tensor cores read 128 all the same, what lies behind being other operands'
// (or the staging blocks'); those rows of the accumulator are nobody's, and the ring is as much deeper.
// (`most_ks`: the most K blocks per stage, which ONNXB_DENSE_KS = 1 or 2 pins; read once a call, since looking through the environment for
// every shape costs more host time than the rest of the choice)
struct Shape : DenseProblem {
    int most_ks;
    explicit Shape(const DenseProblem &d) : DenseProblem(d), most_ks(4) {
        if (const char *e = getenv("ONNXB_DENSE_KS")) most_ks = e[0] == '1' ? 1 : e[0] == '2' ? 2 : 4;
    }
};
int a_rows_of(const Shape &d, Tile t) {
    return t.ctas == 1 && d.mode != kDenseGrad && d.M <= 64 ? (d.M <= 16 ? 16 : d.M <= 32 ? 32 : 64) : kBM;
}
int block_bytes_of(const Shape &d, Tile t) { return (a_rows_of(d, t) + t.BN / t.ctas) * kRowBytes; }
// K blocks per stage: as many as leave four stages in the ring.  (Both weights in one CTA's stage: where their view in groups of 8 rows
// ends with the tensors.)
int blocks_per_stage(const Shape &d, Tile t) {
    if (d.mode == kDenseGated && t.ctas == 1 && (d.N % 8 || d.K % (kRowBytes / type_bytes(d.type)))) return 1;
    const int most = std::min(d.most_ks, ring_bytes() / 4 / block_bytes_of(d, t));
    return most >= 4 && d.mode != kDenseGrad ? 4 : most >= 2 ? 2 : 1;
}
int stages_of(const Shape &d, Tile t) { return std::min(kMaxStages, ring_bytes() / (block_bytes_of(d, t) * blocks_per_stage(d, t))); }
long long stages_along(const Shape &d, Tile t) { return ceil_div(d.K, (long long)(kRowBytes / type_bytes(d.type)) * blocks_per_stage(d, t)); }
// A shared reduction: every CTA has a part of it, all tiles run at once (of 148 SMs not every eight are a cluster's: 128), and what
// the others send has room where the ring was
constexpr long long kMostShared = 128;
bool split_allowed(const Shape &d, Tile t) {
    if (t.split == 1) return true;
    const long long num_kb = stages_along(d, t);
    if (t.ctas != 1 || d.mode == kDenseGrad || t.split > 8 || num_kb < 2 * t.split) return false;
    const int out_cols = d.mode == kDenseGated ? t.BN / 2 : t.BN, block_cols = d.y_type == ONNXB_FLOAT ? 32 : 64;
    const long long tiles = ceil_div(d.M, kBM) * ceil_div(d.N, out_cols), part = ceil_div(num_kb, t.split);
    const long long places = ceil_div(ceil_div(out_cols, block_cols) * 4, t.split) * (block_cols / 32) * (d.mode == kDenseGated ? 2 : 1) * (t.split - 1);
    return tiles * t.split <= kMostShared && part * (t.split - 1) < num_kb &&
           places * kBlockBytes <= (long long)stages_of(d, t) * block_bytes_of(d, t) * blocks_per_stage(d, t);
}
// "<CTAs>x<BN>" or "1x<BN>/<split>" in ONNXB_DENSE_TILE pins the shape for A/B measurements and tests
bool pinned_tile(int mode, Tile &t) {
    const char *e = getenv("ONNXB_DENSE_TILE");
    if (!e) return false;
    const char *slash = strchr(e, '/');
    t = Tile{e[0] - '0', e[0] && e[1] == 'x' ? atoi(e + 2) : 0, slash ? atoi(slash + 1) : 1};
    return (t.ctas == 1 || t.ctas == 2) && t.split >= 1 && tile_allowed(mode, t);
}
// (ctas: that run at once; bytes: of a K block of a CTA)
double stage_cycles(Tile t, int mode, int ks, int bytes, double ctas) {
    const int copies = mode == kDenseGrad ? 2 + t.BN / t.ctas / 64 : mode == kDenseGated && t.ctas == 1 ? 3 : 2;
    const double from_l2 = bytes / std::min(90.0, 8100.0 / ctas);
    return std::max({2.0 * t.BN * ks + 50.0, 240.0 + 170.0 * ks + 75.0 * (copies - 2), from_l2 * ks});
}
double epilogue_cycles(Tile t) { return 1000.0 + 13.0 * t.BN; }

// `outs`: results that a tile's epilogue stores, the further ones at twice the first one's time in all; most_split: the most CTAs to share a reduction
Tile pick_tile(const Shape &d, int outs, int most_split) {
    Tile best{1, 64, 1}, t;
    double best_cost = 1e300;
    const int terms = kRowBytes / type_bytes(d.type), y_bytes = type_bytes(d.y_type);
    for (t.ctas = 1; t.ctas <= 2; ++t.ctas) {
        const int units = t.ctas == 2 ? max_pairs() : tc_host::num_sms(), tiles_m = ceil_int(d.M, kBM * t.ctas);
        for (t.BN = 32 * t.ctas; t.BN <= kMaxBN; t.BN += 32) {
            if (!tile_allowed(d.mode, t)) continue;
            const int out_cols = d.mode == kDenseGated ? t.BN / 2 : t.BN, ks = blocks_per_stage(d, t), bytes = block_bytes_of(d, t);
            const long long tiles = (long long)tiles_m * ceil_int(d.N, out_cols);
            const int stages = ceil_int(d.K, terms * ks);
            // (columns that fill no blocks are stored plainly)
            const double epilogue = epilogue_cycles(t) * (out_cols * y_bytes % kRowBytes ? 2.0 : 1.0) * (outs > 1 ? 2.0 : 1.0);
            for (t.split = 1; t.split <= most_split; t.split *= 2) {
                if (t.split > 1 && tiles * t.split > kMostShared) break;
                if (t.split > 1 && !split_allowed(d, t)) continue;
                const long long at_once = std::min<long long>(tiles * t.split, units);
                const double stage = stage_cycles(t, d.mode, ks, bytes, (double)(at_once * t.ctas));
                const double main = (t.split == 1 ? stages : ceil_int(stages, t.split)) * stage;
                double cost = (double)(tiles * t.split <= units ? 1 : ceil_div(tiles, units)) * std::max(main, epilogue) + epilogue;
                if (t.split > 1) cost += (2500.0 + 28.0 * t.BN) * (t.split == 2 ? 1.0 : t.split == 4 ? 1.3 : 1.5);
                if (cost < best_cost * (1 - 1e-9)) {
                    best_cost = cost;
                    best = t;
                }
            }
        }
    }
    return best;
}
Tile pick_tile(const Shape &d) {
    Tile t;
    if (pinned_tile(d.mode, t) && split_allowed(d, t)) return t;
    // Whether and how a reduction is shared does not go by what else is stored: the gated block's H is the same bit by bit with G and U and without
    t = pick_tile(d, 1, 8);
    return t.split == 1 && d.mode == kDenseGated && d.Y[1] ? pick_tile(d, 3, 1) : t;
}

// The gradients' tiles, and the parts of dX's reduction, each with an fp32 plane that sum_parts_kernel adds up.  From the sizes alone (as a B200
// has 148 SMs), since the workspace depends on it.
struct GradPlan {
    Tile tile;
    int parts;
};
constexpr int kGradTerms = kRowBytes / 2;
// `like`: a plan whose parts this one has to have, with their borders (which lie at whole stages)
GradPlan search_grad_plan(int tokens, int channels, int width, bool dX, int weights, const GradPlan *like) {
    DenseProblem sizes{};
    sizes.mode = kDenseGrad;
    sizes.type = ONNXB_BFLOAT16;
    sizes.M = tokens; sizes.N = width; sizes.K = channels;
    const Shape shape(sizes);
    GradPlan best{{1, 64, 1}, 1};
    double best_cost = 1e300;
    Tile pinned;
    const bool pin = pinned_tile(kDenseGrad, pinned);
    const char *pin_parts = getenv("ONNXB_DENSE_PARTS");
    const int only = pin_parts ? atoi(pin_parts) : 0;
    for (int ctas = 1; ctas <= 2; ++ctas) {
        const int units = ctas == 2 ? 74 : 148, tiles_x = ceil_int(tokens, kBM * ctas), tiles_w = ceil_int(channels, kBM * ctas) * weights;
        for (int bn = 64 * ctas; bn <= kMaxBN; bn += 64 * ctas) {
            const Tile t{ctas, bn, 1};
            if (pin && (t.ctas != pinned.ctas || t.BN != pinned.BN)) continue;
            const int ks = blocks_per_stage(shape, t);
            if (like && like->parts > 1 && ks != blocks_per_stage(shape, like->tile)) continue;
            const int x_kb = 2 * ceil_int(channels, kGradTerms * ks), w_kb = ceil_int(tokens, kGradTerms * ks);
            const double across = ceil_int(width, bn), epilogue = epilogue_cycles(t), w_tiles = tiles_w * across;
            for (int parts = 1; parts <= 8; parts *= 2) {
                if (parts > 1 && (!dX || x_kb < 8 * parts)) break;
                if (like && parts != like->parts) continue;
                if (only && parts != only && (parts > 1 || (dX && x_kb >= 8 * only))) continue;
                const double x_tiles = dX ? tiles_x * across * parts : 0.0;
                const double stage = stage_cycles(t, kDenseGrad, ks, block_bytes_of(shape, t), ctas * std::min((double)units, x_tiles + w_tiles));
                const double x_cost = std::max(x_kb * stage / parts, epilogue), w_cost = std::max(w_kb * stage, epilogue);
                double cost = std::ceil(x_tiles / units) * x_cost;
                if (w_tiles > 0) cost = std::max(cost, x_tiles > 0 ? (x_tiles * x_cost + w_tiles * w_cost) / units + 0.5 * w_cost : std::ceil(w_tiles / units) * w_cost);
                cost += epilogue;
                // (a launch, and the planes out of L2)
                if (parts > 1) cost += 4000.0 + (4.0 * parts + 2.0) * tokens * width / 4000.0;
                if (cost < best_cost * (1 - 1e-9)) {
                    best_cost = cost;
                    best = GradPlan{t, parts};
                }
                if (x_tiles >= 4 * units) break;       // (enough tiles: parts are for few)
            }
        }
    }
    return best;
}
// dX is the same bit by bit whichever weights' gradients are wanted with it: its parts are those of the call that wants both, the tiles' shape
// that of the call.  (By itself dX of 256 x 10240 x 4096 would take 63 us in four parts and takes 82 in two, of 2048 x 10240 x 4096 310 in four and
// 250 in one; of 512 x 2816 x 1024 25.6 either way.)
GradPlan grad_plan(int tokens, int channels, int width, bool dX, int weights) {
    if (!dX || weights == 2) return search_grad_plan(tokens, channels, width, dX, weights, nullptr);
    const GradPlan both = search_grad_plan(tokens, channels, width, true, 2, nullptr);
    return search_grad_plan(tokens, channels, width, true, weights, &both);
}
// a part's plane: whole tiles of rows, rows of whole 16-byte pieces
long long part_rows(int tokens, Tile t) { return ceil_div(tokens, kBM * t.ctas) * kBM * t.ctas; }
long long part_pitch(int width) { return ceil_div(width, 4) * 4; }

// A's and B's maps; their rows begin at multiples of 16 bytes.  K-major: (terms, rows) boxes of 128 bytes x `box` rows.  The gradients': 64 x 64 ks.
bool operand_map(CUtensorMap *m, const DenseOperand &o, int bytes, long long rows, long long cols, int box) {
    const uint64_t pitch = (uint64_t)(rows > 1 ? o.ld * bytes : (o.ld * bytes + 15) / 16 * 16);
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows};
    const uint32_t boxes[2] = {(uint32_t)(kRowBytes / bytes), (uint32_t)box};
    return tc_host::make_tmap_of(bytes, m, o.p, 2, dims, &pitch, boxes, tc_host::kTmapSwizzle128);
}
// The views for stages of `blocks` K blocks: (terms of a block, rows, block, 1), or where `groups` (terms, 8 rows, block, group of 8 rows).  Of the
// whole blocks alone: the elements behind a row's last are not the row's.
bool blocks_map(CUtensorMap *m, const DenseOperand &o, int bytes, long long rows, long long cols, int box, int blocks, bool groups) {
    const uint64_t pitch = (uint64_t)(rows > 1 ? o.ld * bytes : (o.ld * bytes + 15) / 16 * 16), terms = kRowBytes / bytes;
    const uint64_t dims[4] = {terms, groups ? 8 : (uint64_t)rows, (uint64_t)cols / terms, groups ? (uint64_t)rows / 8 : 1};
    const uint64_t pitches[3] = {pitch, kRowBytes, groups ? 8 * pitch : (uint64_t)rows * pitch};
    const uint32_t boxes[4] = {(uint32_t)terms, groups ? 8u : (uint32_t)box, (uint32_t)blocks, groups ? (uint32_t)box / 8 : 1u};
    return tc_host::make_tmap_of(bytes, m, o.p, 4, dims, pitches, boxes, tc_host::kTmapSwizzle128);
}
// A result's map, where TMA can store it: Params' y_tma
int result_map(CUtensorMap *m, void *y, long long ld, int bytes, long long rows, long long cols) {
    const uint64_t pitch = (uint64_t)(rows > 1 ? ld * bytes : (ld * bytes + 15) / 16 * 16);
    if (!y || pitch % 16 || reinterpret_cast<uintptr_t>(y) % 16) return 0;
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows};
    const uint32_t box[2] = {(uint32_t)(kRowBytes / bytes), 32};
    if (!tc_host::make_tmap_of(bytes, m, y, 2, dims, &pitch, box, tc_host::kTmapSwizzle128)) return 0;
    return cols * bytes % 16 == 0 ? 2 : 1;
}

}  // namespace

GradChoice tc_grad_choice(int rows, int channels, int width, bool dX, int weights) {
    const GradPlan plan = grad_plan(rows, channels, width, dX, weights);
    return GradChoice{plan.tile.ctas, plan.tile.BN, plan.parts};
}
size_t tc_grad_workspace(const GradChoice &c, int rows, int width, bool dX, bool twins) {
    const GradPlan plan{{c.ctas, c.BN, 1}, c.parts};
    return plan.parts > 1 || (dX && twins) ? (size_t)(plan.parts * part_rows(rows, plan.tile) * part_pitch(width) * 4) : 0;
}

int launch_tc_dense(const DenseProblem &problem, cudaStream_t stream) {
    using namespace tc_host;
    const Shape d(problem);
    const bool int8 = d.type == ONNXB_INT8, gated = d.mode == kDenseGated, grad = d.mode == kDenseGrad;
    const int bytes = type_bytes(d.type), terms = kRowBytes / bytes;
    const int weights = grad ? (d.Y[1] != nullptr) + (d.Y[2] != nullptr) : 0;
    const int tokens = d.twins ? d.M / 2 : d.M;
    Params p{};
    p.M = d.M; p.N = d.N;
    const GradPlan plan = grad ? GradPlan{{d.grad.ctas, d.grad.BN, 1}, d.grad.parts} : GradPlan{pick_tile(d), 1};
    const Tile tile = plan.tile;
    p.ks = blocks_per_stage(d, tile);
    p.num_kb = (int)stages_along(d, tile);
    p.full_kb = d.K % terms == 0 ? p.num_kb : d.K / (terms * p.ks);      // (whole blocks past the end of the view are zeros)
    p.BN = tile.BN;
    p.out_cols = gated ? p.BN / 2 : p.BN;
    p.tiles_m = (int)ceil_div(d.M, kBM * tile.ctas);
    p.tiles_n = (int)ceil_div(d.N, p.out_cols);
    // Bands of at most a third of L2 of A's rows, all alike.  (4, 8, 16 and 32 tiles a band: gated block 4096 x 4096 x 10240 in bf16 548, 515,
    // 511 and 508 us under the power cap; the gradients, whose operands are larger, 1125, 1125, 1139 and 1155.)
    const int most = (int)std::max(4LL, std::min(32LL, 40000000LL / ((long long)kBM * tile.ctas * d.K * bytes)));
    p.band = grad ? 8 : ceil_int(p.tiles_m, ceil_int(p.tiles_m, most));
    long long total = (long long)p.tiles_m * p.tiles_n, x_tiles = 0, w_tiles = 0;
    if (grad) {
        p.channels = d.K;
        p.x_tiles_m = p.tiles_m;
        p.x_kb = 2 * p.num_kb;
        p.x_parts = plan.parts;
        p.x_part_kb = (int)ceil_div(p.x_kb, plan.parts);
        p.x_part_rows = (int)part_rows(d.M, tile);
        p.x_planes = d.Y[0] && (plan.parts > 1 || d.twins);
        x_tiles = d.Y[0] ? total * plan.parts : 0;
        p.w_tiles_m = (int)ceil_div(d.K, kBM * tile.ctas);
        p.w_kb = (int)ceil_div(d.M, terms * p.ks);
        p.w_first = d.Y[1] ? 0 : 1;
        w_tiles = (long long)p.w_tiles_m * p.tiles_n * weights;
        const double stage = stage_cycles(tile, kDenseGrad, p.ks, block_bytes_of(d, tile), 148), epilogue = epilogue_cycles(tile);
        p.w_before = (int)(std::max(p.x_part_kb * stage, epilogue) / std::max(p.w_kb * stage, epilogue));
        total = x_tiles + w_tiles;
        if (plan.parts * (long long)p.x_part_rows > 0x7fffffffLL) return (int)cudaErrorInvalidValue;
    }
    if (total > 0x7fffffffLL / 2 || (long long)p.band * p.tiles_n > 0x7fffffffLL) return (int)cudaErrorInvalidValue;
    p.total = (int)total;
    p.x_tiles = (int)x_tiles;
    p.w_tiles = (int)w_tiles;
    const int bnh = p.BN / tile.ctas, a_rows = a_rows_of(d, tile);
    p.a_bytes = (uint32_t)(a_rows * kRowBytes);
    p.stage_bytes = (uint32_t)(block_bytes_of(d, tile) * p.ks);
    p.num_stages = stages_of(d, tile);
    p.split = tile.split;
    p.part_kb = (int)ceil_div(p.num_kb, tile.split);
    const int bf16 = d.type == ONNXB_BFLOAT16;
    p.idesc = int8 ? make_idesc_s8(kBM * tile.ctas, p.BN) : make_idesc_f16(kBM * tile.ctas, p.BN, bf16, grad, grad);
    p.idesc_x = make_idesc_f16(kBM * tile.ctas, p.BN, bf16, 0, 1);
    p.a_scale = d.a_scale; p.b_scale0 = d.b_scale[0]; p.b_scale1 = d.b_scale[1]; p.bias = d.bias;
    p.relu = d.relu; p.activation = d.activation;
    p.y_type = d.y_type;
    p.outs = gated && d.Y[1] ? 3 : 1;
    p.err = device_status_ptr();
    if (!p.err) return (int)cudaErrorUnknown;

    Maps maps{};
    bool fine = true;
    // (maps that nobody uses are left as they are: zeros)
    if (grad) {
        for (int i = 0; i < 2; ++i) {
            fine = fine && operand_map(&maps.A[i], d.A[i], bytes, d.M, d.K, 64 * p.ks);
            if (d.Y[0]) fine = fine && operand_map(&maps.B[i], d.B[i], bytes, d.K, d.N, 64 * p.ks);
        }
    } else {
        // (block by block, and by stages of several; each where there is such a stage, since a map costs 0.4 us of host time)
        const int b_rows = gated ? p.out_cols : bnh, count = gated ? 2 : 1;
        if (p.ks == 1 || p.full_kb < p.num_kb) {
            fine = operand_map(&maps.A[0], d.A[0], bytes, d.M, d.K, a_rows);
            for (int i = 0; i < count; ++i) fine = fine && operand_map(&maps.B[i], d.B[i], bytes, d.N, d.K, b_rows);
        }
        if (p.ks > 1 && p.full_kb > 0) {
            fine = fine && blocks_map(&maps.A4, d.A[0], bytes, d.M, d.K, a_rows, p.ks, false);
            for (int i = 0; i < count; ++i) fine = fine && blocks_map(&maps.B4[i], d.B[i], bytes, d.N, d.K, b_rows, p.ks, gated && tile.ctas == 1);
        }
    }
    if (weights) fine = fine && operand_map(&maps.B[2], d.B[2], bytes, d.M, d.N, 64 * p.ks);
    if (!fine) return (int)cudaErrorInvalidValue;
    for (int i = 0; i < 3; ++i) {
        p.Y[i] = d.Y[i]; p.y_ld[i] = d.y_ld[i];
        p.y_tma[i] = result_map(&maps.Y[i], d.Y[i], d.y_ld[i], type_bytes(d.y_type), grad && i > 0 ? d.K : tokens, d.N);
    }
    if (p.x_planes) {
        p.y_tma[0] = result_map(&maps.Y[0], d.partial, part_pitch(d.N), 4, plan.parts * (long long)p.x_part_rows, part_pitch(d.N));
        if (p.y_tma[0] != 2) return (int)cudaErrorInvalidValue;
    }
    const size_t smem = smem_with_tmem(1024 + (size_t)p.num_stages * p.stage_bytes + kStagingBytes + kBarrierBytes, 512);
    const Kernel kernel = tile.split > 1 ? split_kernel_for(d.mode, int8) : tile.ctas == 2 ? kernel_for<2>(d.mode, int8) : kernel_for<1>(d.mode, int8);
    const cudaError_t attr_err = allow_shared_memory(kernel, (tile.split > 1 ? 2 : tile.ctas - 1) * 4 + (int8 ? 2 : 0) + (gated ? 1 : 0));
    if (attr_err != cudaSuccess) return (int)attr_err;
    const int units = tile.ctas == 2 ? max_pairs() : num_sms();
    const int cluster = std::max(tile.ctas, tile.split);
    const int grid = (int)(tile.split > 1 ? total : std::min<long long>(total, units)) * cluster;
    const cudaError_t e = cluster > 1 ? launch_pdl_cluster(kernel, (unsigned)cluster, dim3(grid), dim3(kThreads), smem, stream, maps, p)
                                         : launch_pdl(kernel, dim3(grid), dim3(kThreads), smem, stream, maps, p);
    count_launch();
    if (e != cudaSuccess || !p.x_planes) return (int)e;
    const SumPartsProblem sum{plan.parts, p.x_part_rows, tokens, d.N, d.y_type, d.twins, static_cast<const float *>(d.partial), part_pitch(d.N), d.Y[0], d.y_ld[0]};
    return launch_sum_parts(sum, stream);
}

}  // namespace onnxb
