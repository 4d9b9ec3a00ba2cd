// Products of 16-bit floats whose weights go by the row's group (expert), on the 5th-generation tensor cores: onnx_grouped_gemm_run,
// onnx_grouped_gated_run, and the products of their gradients.
//
// The pipeline is that of tc_dense.cu: a persistent CTA (or a pair of two on one tile) per SM,
//   warp 0    TMA producer, a ring of stages of 64 terms of the reduction, in boxes of 64 terms by 64 rows (8 KB) that are one lane's copy each;
//   warp 1    one thread issues tcgen05.mma kind::f16 into one of two TMEM accumulators;
//   warps 2-9 epilogue: tcgen05.ld, the mathematics, 32 x 64 blocks laid out in shared memory and stored by whole 128-byte rows;
//   warp 10   clears what a stage holds of the next group's rows (below).
// What is its own:
//   - Where the groups lie only the device knows: every CTA reads the offsets, makes them rise, and counts the groups' row tiles, in shared
//     memory; a tile's number is looked up there.  The grid is what the host knows to be enough, at most one CTA an SM, and the call waits for nothing.
//   - A tile has rows of one group.  Its copies may bring the next group's rows too: they are rows of the accumulator that nobody stores.  Weights
//     are three-dimensional tensors to TMA, so that what lies behind a group's last channel is zeros.
//   - The gradients of the weights sum over a group's rows, which end inside a stage.  There, rows of the next group would be terms of the sum, and if
//     they are not finite zeros on the other side would not help: warp 10 clears them on both sides, up to the next multiple of 16 rows, and the
//     stage's instructions end there.  Such a stage's copies complete on a barrier of this CTA's own, since of a pair each CTA clears what it holds.
//   - Groups without rows: their weights' gradients are zeros, stored without a product.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdlib>

#include "dense_math.cuh"
#include "grouped.h"
#include "tc_common.cuh"
#include "tc_host.h"

namespace onnxb {

namespace {

using namespace tc;
using namespace dense;

constexpr int kBM = 128;                           // rows of a CTA's part of a tile (TMEM lanes)
constexpr int kTerms = 64;                         // of the reduction per stage: a swizzle row of 128 bytes
constexpr int kRowBytes = 128;
constexpr int kBox = 64;                           // rows of a copy
constexpr int kBoxBytes = kBox * kRowBytes;
constexpr int kMaxBN = 256;
constexpr int kMaxStages = 24;
constexpr int kThreads = 352;
constexpr int kEpiWarps = 8;
constexpr int kBlockBytes = 32 * kRowBytes;        // what an epilogue warp lays out: 32 rows of 128 bytes
constexpr int kStagingBytes = kEpiWarps * kBlockBytes;
constexpr int kBarrierBytes = 1024;
constexpr int kSmemLimit = 232448;
static_assert((4 * kMaxStages + 5) * 8 <= kBarrierBytes, "barriers");

struct Params {
    int rows, groups;
    const int *offsets;
    int channels, width;
    int N;                         // columns of the output (of both products of the gradients: the width)
    int BN, out_cols;              // columns of an accumulator; of the output per tile (half of them for the gated block)
    int tiles_n, band;
    int num_kb;                    // stages of the reduction; of one term of dX's
    int a_rows, b_box;             // rows of A in a stage; of a box of B
    int terms, with_x;             // kGroupedGrad: terms; dX is wanted
    int w_tiles_m, w_total;        // row tiles of one weights' gradient; tiles of all of them
    int w_first, w_count;          // the first that is wanted; how many are
    int num_stages;
    uint32_t idesc, idesc_x, stage_bytes, a_bytes;
    int bf16, activation, outs;    // outs: results of a tile (the gated block: H alone, or H, G and U)
    void *Y[3];
    long long y_ld[3];
    int y_wide[3];                 // rows begin at multiples of 16 bytes
    void *D[2];
    long long d_ld[2], d_stride[2];
    int d_wide[2];
    unsigned int *err;
};

struct Maps {
    CUtensorMap A[2], W[2], X;
};

// The groups, in shared memory: the first row of each and behind the last, and how many row tiles the groups before each have
struct Groups {
    int *first, *tiles;
};
struct TileAt {
    int g, tm, tn, z;          // z: which of the weights' gradients
    int row0, row_end;         // the tile's first row, and where its group ends (gradients of weights: the group's first row)
    int kb;                    // stages
    bool x;                    // of rows: the forward products and dX
};
// Of `tiles_m` by tiles_n tiles the r-th, in bands of `band` row tiles, a band's columns one after the other: the tiles in flight share operands in L2
__device__ __forceinline__ void place(const Params &p, int tiles_m, int r, TileAt &at) {
    const int b = r / (p.band * p.tiles_n), rr = r - b * p.band * p.tiles_n, rows = min(p.band, tiles_m - b * p.band);
    at.tn = rr / rows;
    at.tm = b * p.band + rr - at.tn * rows;
}
template <int kCtas, int kMode>
__device__ __forceinline__ bool tile_at(const Params &p, const Groups &s, int t, TileAt &at) {
    constexpr bool kGrad = kMode == kGroupedGrad;
    const int of_rows = !kGrad || p.with_x ? s.tiles[p.groups] * p.tiles_n : 0;
    at.x = t < of_rows;
    at.z = 0;
    if (at.x) {
        const int q = t / p.tiles_n;
        int lo = 0, hi = p.groups;             // tiles[lo] <= q < tiles[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s.tiles[mid] <= q) lo = mid;
            else hi = mid;
        }
        at.g = lo;
        place(p, s.tiles[lo + 1] - s.tiles[lo], t - s.tiles[lo] * p.tiles_n, at);
        at.row0 = s.first[lo] + at.tm * kBM * kCtas;
        at.row_end = s.first[lo + 1];
        at.kb = kGrad ? p.terms * p.num_kb : p.num_kb;
        return true;
    }
    t -= of_rows;
    if (!kGrad || t >= p.w_total) return false;
    const int per = p.w_tiles_m * p.tiles_n;
    at.g = t / (per * p.w_count);
    const int r = t - at.g * per * p.w_count;
    at.z = r / per;
    place(p, p.w_tiles_m, r - at.z * per, at);
    at.row0 = s.first[at.g];
    at.row_end = s.first[at.g + 1];
    at.kb = (at.row_end - at.row0 + kTerms - 1) / kTerms;
    return true;
}

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

template <int kCtas, int kMode>
__global__ void __launch_bounds__(kThreads, 1) tc_grouped_kernel(const __grid_constant__ Maps maps, const Params p) {
    constexpr bool kGrad = kMode == kGroupedGrad, kGated = kMode == kGroupedGated;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t *stages = smem;
    uint8_t *staging = smem + (size_t)p.num_stages * p.stage_bytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + kStagingBytes);
    uint64_t *full = bars, *empty = bars + kMaxStages, *tail_full = bars + 2 * kMaxStages, *cleared = bars + 3 * kMaxStages;
    uint64_t *tmem_full = bars + 4 * kMaxStages, *tmem_empty = tmem_full + 2;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(tmem_empty + 2);
    Groups groups;
    groups.first = reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(bars) + kBarrierBytes);
    groups.tiles = groups.first + p.groups + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = kCtas == 2 ? (int)cluster_ctarank() : 0;
    const int unit = blockIdx.x / kCtas, units = gridDim.x / kCtas;
    TileAt at;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.num_stages; ++s) {
            mbar_init(&full[s], 1);        // (of a pair: the even CTA's, which counts both CTAs' copies)
            mbar_init(&empty[s], 1);
            mbar_init(&tail_full[s], 1);
            mbar_init(&cleared[s], kCtas);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&tmem_full[a], 1);
            mbar_init(&tmem_empty[a], kEpiWarps * kCtas);
        }
        mbar_fence_init();
        prefetch_tmap(&maps.A[0]);
        prefetch_tmap(kGrad && !p.with_x ? &maps.X : &maps.W[0]);
        if (kGated) prefetch_tmap(&maps.W[1]);
    }
    if (warp == 1) {
        tmem_alloc(tmem_holder, 512);
        tmem_relinquish();
    }
    pdl_launch_dependents();
    pdl_wait();
    // The groups' first rows, between 0 and the rows that there are, rising (an offset below the one before it counts as that), and their tiles
    for (int i = threadIdx.x; i <= p.groups; i += kThreads) groups.first[i] = min(max(p.offsets[i], 0), p.rows);
    __syncthreads();
    if (warp == 0) {
        int most = groups.first[0], count = 0;
        if (lane == 0) groups.tiles[0] = 0;
        for (int base = 0; base < p.groups; base += 32) {
            const int i = base + lane;
            int end = i < p.groups ? groups.first[i + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int other = __shfl_up_sync(0xffffffffu, end, o);
                if (lane >= o) end = max(end, other);
            }
            end = max(end, most);
            int before = __shfl_up_sync(0xffffffffu, end, 1);
            if (lane == 0) before = most;
            int tiles = i < p.groups ? (end - before + kBM * kCtas - 1) / (kBM * kCtas) : 0;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int other = __shfl_up_sync(0xffffffffu, tiles, o);
                if (lane >= o) tiles += other;
            }
            if (i < p.groups) {
                groups.first[i + 1] = end;
                groups.tiles[i + 1] = count + tiles;
            }
            most = __shfl_sync(0xffffffffu, end, 31);
            count += __shfl_sync(0xffffffffu, tiles, 31);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_holder;
    if (kCtas == 2) cluster_sync_all();     // the peer's barriers exist before anything arrives on them

    // Whether a tile's last stage ends inside the next group's rows, where it is not by 16 rows that it does
    auto has_tail = [&](const TileAt &t) { return kGrad && !t.x && ((t.row_end - t.row0) & 15) != 0; };

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer: every lane with a copy of its own per stage
        int stage = 0;
        uint32_t phase = 0;
        const uint32_t full_issuer = kCtas == 2 ? map_to_cta(smem_u32(&full[0]), 0) : 0u;
        const uint32_t tail_own = kCtas == 2 ? map_to_cta(smem_u32(&tail_full[0]), (uint32_t)rank) : 0u;
        const int bnh = p.BN / kCtas, nb = bnh / p.b_box;                  // B's rows that this CTA stages, and their boxes
        for (int n = unit; tile_at<kCtas, kMode>(p, groups, n, at); n += units) {
            // Boxes of A: those that hold a row of the group's (gradients of weights: both)
            const int a_box = min(kBox, p.a_rows);
            auto boxes_of = [&](int r) { return !at.x ? 2 : min(max((at.row_end - at.row0 - r * kBM + a_box - 1) / a_box, 0), p.a_rows / a_box); };
            const int na = boxes_of(rank);
            uint32_t bytes = (uint32_t)(boxes_of(0) * a_box + nb * p.b_box) * kRowBytes;
            const uint32_t own_bytes = (uint32_t)(na * a_box + nb * p.b_box) * kRowBytes;
            if (kCtas == 2) bytes += (uint32_t)(boxes_of(1) * a_box + nb * p.b_box) * kRowBytes;
            const bool is_a = lane < na, active = lane < na + nb;
            const int piece = is_a ? lane : lane - na;
            const uint32_t dst_off = is_a ? (uint32_t)(piece * a_box) * kRowBytes : p.a_bytes + (uint32_t)(piece * p.b_box) * kRowBytes;
            const CUtensorMap *map = is_a ? &maps.A[0] : &maps.W[0];
            // where the copy begins: along the tile (rows, channels or columns), and along the reduction
            int along;
            if (at.x) {
                if (is_a) along = at.row0 + rank * kBM + piece * a_box;
                else if (kGated) {
                    // a pair's CTA has one of the two weights, a lone CTA both, each with half of the boxes
                    const int per = kCtas == 2 ? nb : nb / 2, w = kCtas == 2 ? rank : piece / per;
                    map = &maps.W[w];
                    along = at.tn * p.out_cols + (piece - (kCtas == 2 ? 0 : w * per)) * p.b_box;
                } else {
                    along = at.tn * p.BN + rank * bnh + piece * p.b_box;
                }
            } else {
                along = is_a ? (at.tm * kCtas + rank) * kBM + piece * kBox : at.tn * p.BN + rank * bnh + piece * kBox;
                map = is_a ? &maps.A[p.w_first + at.z] : &maps.X;
            }
            const bool tail = has_tail(at);
            int term = at.x ? 0 : at.row0;
            for (int kb = 0; kb < at.kb; ++kb) {
                mbar_wait(&empty[stage], phase ^ 1, p.err, 1);
                const bool to_clear = tail && kb == at.kb - 1;
                if (lane == 0) {
                    if (to_clear) {
                        mbar_arrive_expect_tx(&tail_full[stage], own_bytes);
                        if (rank == 0) mbar_arrive(&full[stage]);
                    } else if (rank == 0) {
                        mbar_arrive_expect_tx(&full[stage], bytes);
                    }
                }
                __syncwarp();
                if (kGrad && at.x && kb == p.num_kb) {         // dX's second term
                    map += 1;
                    term = 0;
                }
                if (active) {
                    uint8_t *dst = stages + (size_t)stage * p.stage_bytes + dst_off;
                    const uint32_t bar = kCtas == 2 ? (to_clear ? tail_own : full_issuer) + (uint32_t)stage * 8u : 0u;
                    uint64_t *own = to_clear ? &tail_full[stage] : &full[stage];
                    // A K-major: (term, row); MN-major: (row, term).  Weights: (term, channel, group), or for dX (column, channel, group).
                    if (!at.x || is_a) {
                        const int c0 = at.x ? term : along, c1 = at.x ? along : term;
                        if (kCtas == 2) tma_load_2d_pair(dst, map, bar, c0, c1);
                        else tma_load_2d(dst, map, own, c0, c1);
                    } else {
                        const int c0 = kGrad ? along : term, c1 = kGrad ? term : along;
                        if (kCtas == 2) tma_load_3d_pair(dst, map, bar, c0, c1, at.g);
                        else tma_load_3d(dst, map, own, c0, c1, at.g);
                    }
                }
                term += kTerms;
                if (++stage == p.num_stages) { stage = 0; phase ^= 1; }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (of a pair: the even CTA)
        if ((kCtas == 1 || rank == 0) && elect_one()) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0, clear_phase = 0;        // (the last: a bit for each stage)
            // K-major: 8-row groups 1024 bytes apart, an instruction 32 bytes further along the swizzled rows.  MN-major: blocks of 64 rows or
            // columns a box apart, groups of 8 terms 1024 bytes apart, an instruction two of those further.
            const uint64_t k_tmpl = make_smem_desc(0, 16, 1024, kSwizzle128B), mn_tmpl = make_smem_desc(0, kBoxBytes, 1024, kSwizzle128B);
            const uint64_t b_tmpl = kGrad ? mn_tmpl : k_tmpl;
            const uint32_t b_hi = (uint32_t)(b_tmpl >> 32);
            const uint32_t a_at = (smem_u32(stages) >> 4) & 0x3FFFu, b_lo = (uint32_t)b_tmpl | (((smem_u32(stages) + p.a_bytes) >> 4) & 0x3FFFu);
            const uint32_t stage16 = p.stage_bytes >> 4;
            constexpr uint32_t kK16 = 32u >> 4, kMn16 = 2048u >> 4, kB16 = kGrad ? kMn16 : kK16;
            for (int n = unit; tile_at<kCtas, kMode>(p, groups, n, at); n += units) {
                if (at.kb == 0) continue;              // a group without rows
                const bool a_mn = kGrad && !at.x, tail = has_tail(at);
                const uint64_t a_tmpl = a_mn ? mn_tmpl : k_tmpl;
                const uint32_t a_hi = (uint32_t)(a_tmpl >> 32), a_lo = (uint32_t)a_tmpl | a_at, a16 = a_mn ? kMn16 : kK16;
                const uint32_t idesc = kGrad && at.x ? p.idesc_x : p.idesc;
                // instructions of the last stage
                const int last = a_mn ? (at.row_end - at.row0 - (at.kb - 1) * kTerms + 15) / 16 : 4;
                if (kCtas == 2) mbar_wait_cluster(&tmem_empty[acc], acc_phase ^ 1, p.err, 2);
                else mbar_wait(&tmem_empty[acc], acc_phase ^ 1, p.err, 2);
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + (uint32_t)acc * kMaxBN;
                uint32_t accumulate = 0;
                for (int kb = 0; kb < at.kb; ++kb) {
                    mbar_wait(&full[stage], phase, p.err, 3);
                    if (tail && kb == at.kb - 1) {
                        if (kCtas == 2) mbar_wait_cluster(&cleared[stage], (clear_phase >> stage) & 1u, p.err, 5);
                        else mbar_wait(&cleared[stage], (clear_phase >> stage) & 1u, p.err, 5);
                        clear_phase ^= 1u << stage;
                    }
                    tc_fence_after_sync();
                    const uint32_t al = a_lo + (uint32_t)stage * stage16, bl = b_lo + (uint32_t)stage * stage16;
                    const int instructions = kb == at.kb - 1 ? last : 4;
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        if (kGrad && (int)k >= instructions) break;
                        if (kCtas == 2) mma_f16_lohi_pair(d_tmem, al + k * a16, a_hi, bl + k * kB16, b_hi, idesc, accumulate);
                        else mma_f16_lohi(d_tmem, al + k * a16, a_hi, bl + k * kB16, b_hi, idesc, accumulate);
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
    } else if (warp == 2 + kEpiWarps) {
        // ------------------------------------------------------------ stages that end inside the next group's rows
        if (kGrad) {
            int stage = 0;
            uint32_t clear_phase = 0;
            const uint32_t cleared_issuer = kCtas == 2 ? map_to_cta(smem_u32(&cleared[0]), 0) : 0u;
            const int boxes = (int)(p.stage_bytes / kBoxBytes);
            for (int n = unit; tile_at<kCtas, kMode>(p, groups, n, at); n += units) {
                if (at.kb == 0) continue;
                stage += at.kb - 1;
                stage %= p.num_stages;
                if (has_tail(at)) {
                    mbar_wait(&tail_full[stage], (clear_phase >> stage) & 1u, p.err, 6);
                    clear_phase ^= 1u << stage;
                    // a box has a row of the group's, 64 columns of it, in 128 bytes (the swizzle moves pieces within them)
                    const int from = (at.row_end - at.row0) - (at.kb - 1) * kTerms, pieces = ((from + 15) / 16 * 16 - from) * 8;
                    uint8_t *first = stages + (size_t)stage * p.stage_bytes + from * kRowBytes;
                    for (int b = 0; b < boxes; ++b)
                        for (int i = lane; i < pieces; i += 32) *reinterpret_cast<uint4 *>(first + b * kBoxBytes + i * 16) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if (kCtas == 2) mbar_arrive_remote_release(cleared_issuer + (uint32_t)stage * 8u);
                        else mbar_arrive(&cleared[stage]);
                    }
                }
                if (++stage == p.num_stages) stage = 0;
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue
        const int q = warp & 3, half = (warp - 2) >> 2;
        uint8_t *buf = staging + (warp - 2) * kBlockBytes;
        int acc = 0;
        uint32_t acc_phase = 0;
        const uint32_t peer_tmem_empty = kCtas == 2 ? map_to_cta(smem_u32(&tmem_empty[0]), 0) : 0u;
        for (int n = unit; tile_at<kCtas, kMode>(p, groups, n, at); n += units) {
            const int n0 = at.tn * p.out_cols, cols = min(p.out_cols, p.N - n0), blocks = (cols + 63) / 64;
            // the first row of this warp's quarter, in its output, and how many of its 32 are the group's (gradients of weights: channels)
            const int quarter = rank * kBM + q * 32;
            const int row0 = at.x ? at.row0 + quarter : at.tm * kCtas * kBM + quarter;
            const int rows = min(32, (at.x ? at.row_end : p.channels) - row0);
            const bool some = at.kb > 0;
            if (some) {
                mbar_wait(&tmem_full[acc], acc_phase, p.err, 4);
                tc_fence_after_sync();
            }
            const uint32_t tbase = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * kMaxBN);
            if (rows > 0) {
                // the two warps of a quarter share its blocks of all results in turns
#pragma unroll 1
                for (int item = half; item < blocks * p.outs; item += 2) {
                    const int which = item < blocks ? 0 : item < 2 * blocks ? 1 : 2, b = item - which * blocks;
#pragma unroll 1
                    for (int c = 0; c < 64 && b * 64 + c < p.out_cols; c += 32) {
                        const int col = b * 64 + c;
                        uint32_t v[32];
                        float f[32];
                        if (some) {
                            tmem_ld_32x32(tbase + (uint32_t)(which == 2 ? p.out_cols + col : col), v);
                            if (kGated && which == 0) {
                                uint32_t w[32];
                                tmem_ld_32x32(tbase + (uint32_t)(p.out_cols + col), w);
                                tmem_ld_wait();
#define ONNXB_GATE(kind) _Pragma("unroll") for (int j = 0; j < 32; ++j) f[j] = activate(kind, __uint_as_float(v[j])) * __uint_as_float(w[j])
                                if (p.activation == ONNXB_SILU) { ONNXB_GATE(ONNXB_SILU); }
                                else if (p.activation == ONNXB_GELU) { ONNXB_GATE(ONNXB_GELU); }
                                else if (p.activation == ONNXB_GELU_TANH) { ONNXB_GATE(ONNXB_GELU_TANH); }
                                else { ONNXB_GATE(ONNXB_RELU); }
#undef ONNXB_GATE
                            } else {
                                tmem_ld_wait();
#pragma unroll
                                for (int j = 0; j < 32; ++j) f[j] = __uint_as_float(v[j]);
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j) f[j] = 0.f;
                        }
                        // the lane's row of the block, 16-byte piece i at position i ^ (lane % 8)
                        uint32_t h[16];
                        if (p.bf16) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) h[i] = pack<__nv_bfloat162>(f[2 * i], f[2 * i + 1]);
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) h[i] = pack<__half2>(f[2 * i], f[2 * i + 1]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *reinterpret_cast<uint4 *>(buf + lane * kRowBytes + (((c / 8 + i) ^ (lane & 7)) << 4)) =
                                make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
                    }
                    __syncwarp();
                    // Stored by rows, four at a time in pieces of 16 bytes, or one in pairs of elements
                    const int w = p.w_first + at.z, left = min(64, cols - b * 64);
                    const bool of_weights = kGrad && !at.x;
                    const long long ld = of_weights ? p.d_ld[w] : p.y_ld[which];
                    uint16_t *out = static_cast<uint16_t *>(of_weights ? p.D[w] : p.Y[which]) + (of_weights ? at.g * p.d_stride[w] : 0) + row0 * ld + n0 + b * 64;
                    if (of_weights ? p.d_wide[w] : p.y_wide[which]) {
                        const int piece = lane & 7, mine = left - piece * 8;
#pragma unroll 4
                        for (int r = lane >> 3; r < rows; r += 4) {
                            const uint4 v = *reinterpret_cast<const uint4 *>(buf + r * kRowBytes + ((piece ^ (r & 7)) << 4));
                            uint16_t *to = out + r * ld + piece * 8;
                            if (mine >= 8) *reinterpret_cast<uint4 *>(to) = v;
                            else if (mine > 0) {
                                const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int e = 0; e < 7; ++e)
                                    if (e < mine) to[e] = (uint16_t)(word[e / 2] >> (e % 2 * 16));
                            }
                        }
                    } else {
#pragma unroll 4
                        for (int r = 0; r < rows; ++r) {
                            const uint32_t v = *reinterpret_cast<const uint32_t *>(buf + r * kRowBytes + (((lane >> 2) ^ (r & 7)) << 4 | (lane & 3) * 4));
                            uint16_t *to = out + r * ld + lane * 2;
                            if (lane * 2 < left) to[0] = (uint16_t)v;
                            if (lane * 2 + 1 < left) to[1] = (uint16_t)(v >> 16);
                        }
                    }
                    __syncwarp();
                }
            }
            if (!some) continue;
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (kCtas == 2) mbar_arrive_remote(peer_tmem_empty + (uint32_t)acc * 8u);
                else mbar_arrive(&tmem_empty[acc]);
            }
            acc ^= 1;
            if (acc == 0) acc_phase ^= 1;
        }
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
Kernel kernel_for(int mode) {
    return mode == kGroupedPlain ? tc_grouped_kernel<kCtas, kGroupedPlain> : mode == kGroupedGated ? tc_grouped_kernel<kCtas, kGroupedGated> : tc_grouped_kernel<kCtas, kGroupedGrad>;
}

// The kernel's shared memory allowed for, once a device
cudaError_t allow_shared_memory(Kernel kernel, int index) {
    static std::atomic<uint64_t> done[6];
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done[index].load(std::memory_order_acquire) & bit)) return cudaSuccess;
    const cudaError_t set = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
    if (set == cudaSuccess && dev < 64) done[index].fetch_or(bit, std::memory_order_release);
    return set;
}

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

struct Tile {
    int ctas, BN;
};
bool tile_allowed(int mode, Tile t) {
    if (t.BN < 64 || t.BN > kMaxBN || t.BN % 64) return false;
    // boxes of 64 rows of B in each CTA, or of both weights of the gated block in a lone one (of 32 where these are few)
    return t.ctas == 2 ? t.BN % 128 == 0 : mode != kGroupedGated || t.BN != 192;
}
// CTA pairs that run at once, asked of the device's occupancy once
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
    const Kernel kernel = kernel_for<2>(kGroupedPlain);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = tc_host::num_sms() / 2;
    }
    cached.store(n, std::memory_order_release);
    return n;
}
Tile pick_tile(const GroupedProblem &d) {
    if (const char *e = getenv("ONNXB_GROUPED_TILE")) {
        const Tile t{e[0] - '0', e[0] && e[1] == 'x' ? atoi(e + 2) : 0};
        if ((t.ctas == 1 || t.ctas == 2) && tile_allowed(d.mode, t)) return t;
    }
    const long long per_group = d.rows / std::min(d.rows, d.groups);
    if (per_group > 128) return Tile{2, 256};
    return Tile{1, per_group >= 32 ? 256 : 128};
}

// Rows that begin at multiples of 16 bytes, as (terms, rows) in boxes of 64 by `box`
bool rows_map(CUtensorMap *m, const DenseOperand &o, long long rows, long long cols, int box) {
    const uint64_t pitch = (uint64_t)(rows > 1 ? o.ld * 2 : (o.ld * 2 + 15) / 16 * 16);
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows};
    const uint32_t boxes[2] = {kTerms, (uint32_t)box};
    return tc_host::make_tmap_of(2, m, o.p, 2, dims, &pitch, boxes, tc_host::kTmapSwizzle128);
}
bool weights_map(CUtensorMap *m, const GroupedWeights &w, long long groups, long long channels, long long width, int box) {
    const uint64_t pitch = (uint64_t)(channels > 1 ? w.ld * 2 : (width * 2 + 15) / 16 * 16);
    const uint64_t dims[3] = {(uint64_t)width, (uint64_t)channels, (uint64_t)groups};
    const uint64_t pitches[2] = {pitch, groups > 1 ? (uint64_t)w.stride * 2 : pitch};
    const uint32_t boxes[3] = {kTerms, (uint32_t)box, 1};
    return tc_host::make_tmap_of(2, m, w.p, 3, dims, pitches, boxes, tc_host::kTmapSwizzle128);
}
bool by_16(const void *p, long long ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }

}  // namespace

int launch_tc_grouped(const GroupedProblem &d, cudaStream_t stream) {
    using namespace tc_host;
    const bool gated = d.mode == kGroupedGated, grad = d.mode == kGroupedGrad;
    const Tile tile = pick_tile(d);
    Params p{};
    p.rows = d.rows; p.groups = d.groups; p.offsets = d.offsets;
    p.channels = d.channels; p.width = d.width;
    p.N = grad ? d.width : d.channels;
    p.BN = tile.BN;
    p.out_cols = gated ? p.BN / 2 : p.BN;
    p.tiles_n = (int)ceil_div(p.N, p.out_cols);
    p.band = 8;
    p.num_kb = (int)ceil_div(grad ? d.channels : d.width, kTerms);
    // Few rows: no more of A's than there are.  The tensor cores read 128 all the same, what lies behind being other operands'; those rows of the accumulator are nobody's.
    p.a_rows = tile.ctas == 1 && !grad && d.rows <= 64 ? (d.rows <= 16 ? 16 : d.rows <= 32 ? 32 : 64) : kBM;
    p.b_box = gated && tile.BN / 2 < kBox && tile.ctas == 1 ? 32 : kBox;
    p.terms = d.terms;
    p.with_x = grad && d.Y[0] ? 1 : 0;
    p.w_first = d.D[0].p ? 0 : 1;
    p.w_count = grad ? (d.D[0].p != nullptr) + (d.D[1].p != nullptr) : 0;
    p.w_tiles_m = (int)ceil_div(d.channels, kBM * tile.ctas);
    const long long w_total = (long long)d.groups * p.w_count * p.w_tiles_m * p.tiles_n;
    // row tiles: at most one of each group is not whole
    const long long row_tiles = grad && !p.with_x ? 0 : d.rows / (kBM * tile.ctas) + std::min(d.groups, d.rows), most = row_tiles * p.tiles_n + w_total;
    if (most > 0x7fffffffLL / 2 || (long long)p.band * p.tiles_n > 0x7fffffffLL) return (int)cudaErrorInvalidValue;
    p.w_total = (int)w_total;
    p.a_bytes = (uint32_t)(p.a_rows * kRowBytes);
    p.stage_bytes = p.a_bytes + (uint32_t)(p.BN / tile.ctas * kRowBytes);
    const int table = ((2 * d.groups + 2) * 4 + 15) / 16 * 16;
    p.num_stages = std::min(kMaxStages, (kSmemLimit - 1024 - kBarrierBytes - kStagingBytes - table) / (int)p.stage_bytes);
    const int bf16 = d.type == ONNXB_BFLOAT16;
    p.idesc = make_idesc_f16(kBM * tile.ctas, p.BN, bf16, grad, grad);
    p.idesc_x = make_idesc_f16(kBM * tile.ctas, p.BN, bf16, 0, 1);
    p.bf16 = bf16;
    p.activation = d.activation;
    p.outs = gated && d.Y[1] ? 3 : 1;
    for (int i = 0; i < 3; ++i) { p.Y[i] = d.Y[i]; p.y_ld[i] = d.y_ld[i]; p.y_wide[i] = by_16(d.Y[i], d.y_ld[i]); }
    for (int i = 0; i < 2; ++i) {
        p.D[i] = const_cast<void *>(d.D[i].p); p.d_ld[i] = d.D[i].ld; p.d_stride[i] = d.D[i].stride;
        p.d_wide[i] = by_16(d.D[i].p, d.D[i].ld) && d.D[i].stride % 8 == 0;
    }
    p.err = device_status_ptr();
    if (!p.err) return (int)cudaErrorUnknown;

    Maps maps{};
    bool fine = true;
    for (int i = 0; i < (grad ? d.terms : 1); ++i) fine = fine && rows_map(&maps.A[i], d.A[i], d.rows, grad ? d.channels : d.width, std::min(kBox, p.a_rows));
    for (int i = 0; i < (gated ? 2 : grad ? d.terms : 1); ++i)
        if (!grad || p.with_x) fine = fine && weights_map(&maps.W[i], d.W[i], d.groups, d.channels, d.width, p.b_box);
    if (p.w_count) fine = fine && rows_map(&maps.X, d.X, d.rows, d.width, kBox);
    if (!fine) return (int)cudaErrorInvalidValue;

    const size_t smem = smem_with_tmem(1024 + (size_t)p.num_stages * p.stage_bytes + kStagingBytes + kBarrierBytes + table, 512);
    const Kernel kernel = tile.ctas == 2 ? kernel_for<2>(d.mode) : kernel_for<1>(d.mode);
    const cudaError_t attr_err = allow_shared_memory(kernel, (tile.ctas - 1) * 3 + d.mode);
    if (attr_err != cudaSuccess) return (int)attr_err;
    const int units = tile.ctas == 2 ? max_pairs() : num_sms(), grid = (int)std::min<long long>(most, units) * tile.ctas;
    const cudaError_t e = tile.ctas == 2 ? launch_pdl_cluster(kernel, 2u, dim3(grid), dim3(kThreads), smem, stream, maps, p)
                                         : launch_pdl(kernel, dim3(grid), dim3(kThreads), smem, stream, maps, p);
    count_launch();
    return (int)e;
}

}  // namespace onnxb
