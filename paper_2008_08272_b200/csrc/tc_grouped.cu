// Products of 16-bit floats whose weights go by the row's group (expert), on the 5th-generation tensor cores: onnx_grouped_gemm_run,
// onnx_grouped_gated_run, and the products of their gradients.
//
// The pipeline is that of tc_dense.cu: a persistent CTA (or a pair of two on one tile) per SM,
//   warp 0    TMA producer, a ring of stages of one K block or, of forward products, two (64 terms of the reduction each): a stage costs its two single threads 240 cycles, and
//             170 more for each block;
//   warp 1    one thread issues tcgen05.mma kind::f16 into one of two TMEM accumulators;
//   warps 2-9 epilogue: tcgen05.ld, the mathematics, stores;
//   warp 10   clears what a stage holds of the next group's rows (below).
// What is its own:
//   - Where the groups lie only the device knows: every CTA reads the offsets, makes them rise, and counts the groups' tiles, in shared memory; a tile's
//     number is looked up there.  The grid has a CTA (pair) for every tile that the host cannot rule out, and the call waits for nothing.
//   - Tiles take different times (groups' rows differ), so none is anybody's beforehand: a CTA that has begun to load one asks for another CTA of the grid
//     that has not been launched, computes its tile in its place, and tells its warps (of a pair, both CTAs') by a ring of tile numbers.
//   - Products of rows (the forward ones and dX) have the weights as the instruction's 128 or 256 rows and the group's rows as its columns, of which there
//     may be any multiple of 16 up to 256: a group's last tile then costs what it has, where 256 rows a tile would be half empty in groups of some
//     hundred.  A group's tiles are made as alike as multiples of 16 allow.  The accumulator is the result's transpose: a lane has a channel of 32 rows, and
//     trades every other one with its neighbour, so that both store two channels of 16 rows, 64 bytes of each row a warp.
//   - The gated block is one such product: of a CTA's 128 rows of weights 64 are Wg's and 64 Wu's of the same channels, so that a channel's gate and other
//     factor are lanes of two warps, each of which gives the other half of its rows and computes the other half's results.  (Two products side by side in the
//     accumulator instead, of up to 128 rows each, read 40 KB for what takes 32 so: 16384 x 2048 x 1408 of 64 groups 223 us, L2 at its limit.)
//   - A copy of a group's last rows may bring the next group's too: they are columns of the accumulator that nobody stores.  Weights are three-dimensional
//     tensors to TMA, so that what lies behind a group's last channel is zeros.
//   - The gradients of the weights sum over a group's rows, which end inside a stage.  There, rows of the next group would be terms of the sum, and if
//     they are not finite zeros on the other side would not help: warp 10 clears them on both sides, up to the next multiple of 16 rows, and the
//     stage's instructions end there.  Such a stage's copies complete on a barrier of this CTA's own, since of a pair each CTA clears what it holds.
//   - Groups without rows: their weights' gradients are zeros, stored without a product.
//   - Where a product of rows or the weights' gradients have few tiles and a long reduction, tiles have parts of it, whose sums go to planes of fp32 that a second kernel adds
//     up (73 rows of 17 groups, 6912 -> 64: 20.2 -> 11.8 us; gradients of 10272 rows of one group, 3712 x 72, 53.9 -> 36.7).
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <array>
#include <atomic>
#include <cstdlib>
#include <cstring>
#include <type_traits>

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
constexpr int kStagingBytes = kEpiWarps * kBlockBytes;         // (not of plain forward products)
constexpr int kABytes = kBM * kRowBytes;           // of a block of A
constexpr int kBarrierBytes = 1024;
constexpr int kSlots = 4;                          // tiles that the warps are told of ahead
constexpr int kSmemLimit = 232448;
static_assert((4 * kMaxStages + 5 + 2 * kSlots + 1) * 8 + 16 + 16 * kSlots <= kBarrierBytes, "barriers");

struct Params {
    int rows, groups;
    const int *offsets;
    int channels, width;
    int most_rows;                 // of a tile of rows: columns of an accumulator
    int tiles_n, band;             // of the results' columns, 128 or 256 of them a tile (half as many of the gated block's)
    int num_kb;                    // stages of the reduction; of one term of dX's
    int b_box;                     // rows of a small copy of rows
    int terms, with_x;             // kGroupedGrad: terms; dX is wanted
    int BN;                        // columns of a tile of the weights' gradients
    int w_tiles_m, w_tiles_n, w_total;     // row and column tiles of one weights' gradient; tiles of all of them
    int w_first, w_count;          // the first that is wanted; how many are
    int x_parts, w_parts;          // of the reductions of tiles of rows, and of the weights' gradients; where they are several,
    float *x_planes, *w_planes;    // each with a plane of fp32 of its own
    long long x_pitch, w_pitch;    // floats of their rows
    int num_stages;
    uint32_t idesc_x, idesc_w;     // (of tiles of rows without their columns)
    int ks;                        // K blocks of a stage (of gradients one)
    uint32_t stage_bytes, b_at;    // where B begins in a stage
    int b_block;                   // bytes from a block's rows to the next's
    int bf16, activation, outs;    // outs: results of a tile (the gated block: H alone, or H, G and U)
    void *Y[3];
    long long y_ld[3];
    int y_pairs[3];                // rows begin at multiples of 4 bytes
    void *D[2];
    long long d_ld[2], d_stride[2];
    int d_wide[2];                 // rows begin at multiples of 16 bytes
    unsigned int *err;
};

struct Maps {
    CUtensorMap W[2];              // weights, boxes of 128 channels (of 64 where a stage has two)
    CUtensorMap R[2], R_small[2];  // rows (X, or dY or dG and dU), boxes of 128 and of b_box rows
    CUtensorMap D[2], X;           // rows as terms of the weights' gradients, boxes of 64
};

// The groups, in shared memory: the first row of each and behind the last, and how many tiles of rows the groups before each have
struct Groups {
    int *first, *tiles;
};
// Rows of a tile of a group that has so many: as alike as multiples of 16 allow
__device__ __forceinline__ int rows_per_tile(int rows, int most) {
    const int tiles = (rows + most - 1) / most;
    return tiles > 0 ? ((rows + tiles - 1) / tiles + 15) / 16 * 16 : 16;
}
struct TileAt {
    int g, tm, tn, z;          // z: which of the weights' gradients
    int row0, rows;            // the tile's rows (gradients of weights: the group's)
    int part, kb0, kb;         // of the reduction; its first stage, and how many
    bool ends;                 // with the reduction's last
    bool x;                    // of rows: the forward products and dX
};
// Of `tiles_m` by `tiles_n` tiles the r-th, in bands of `band` row tiles, a band's columns one after the other: the tiles in flight share operands in L2
__device__ __forceinline__ void place(int band, int tiles_m, int tiles_n, int r, TileAt &at) {
    const int b = r / (band * tiles_n), rr = r - b * band * tiles_n, rows = min(band, tiles_m - b * band);
    at.tn = rr / rows;
    at.tm = b * band + rr - at.tn * rows;
}
// Tiles of rows; all of a call, of the weights' gradients too
template <int kMode, bool kParts>
__device__ __forceinline__ int row_tiles(const Params &p, const Groups &s) {
    return kMode != kGroupedGrad || p.with_x ? s.tiles[p.groups] * p.tiles_n * (kParts ? p.x_parts : 1) : 0;
}
template <int kMode, bool kParts>
__device__ __forceinline__ int all_tiles(const Params &p, const Groups &s) {
    return row_tiles<kMode, kParts>(p, s) + (kMode == kGroupedGrad ? p.w_total * (kParts ? p.w_parts : 1) : 0);
}
template <int kMode, bool kParts>
__device__ __forceinline__ void tile_at(const Params &p, const Groups &s, int t, TileAt &at) {
    constexpr bool kGrad = kMode == kGroupedGrad;
    const int of_rows = row_tiles<kMode, kParts>(p, s);
    at.x = t < of_rows;
    at.z = 0;
    t = at.x ? t : t - of_rows;
    at.part = 0;
    const int parts = !kParts ? 1 : at.x ? p.x_parts : p.w_parts;
    if (kParts) {
        // a tile's parts one after the other
        const int q = t / parts;
        at.part = t - q * parts;
        t = q;
    }
    auto share = [&](int stages) {
        const int each = kParts ? (stages + parts - 1) / parts : stages;
        at.kb0 = kParts ? min(at.part * each, stages) : 0;
        at.kb = kParts ? min(each, stages - at.kb0) : stages;
        at.ends = !kParts || (at.kb > 0 && at.kb0 + at.kb == stages);      // (parts behind the last stage have none)
    };
    if (at.x) {
        const int q = t / p.tiles_n;
        int lo = 0, hi = p.groups;             // tiles[lo] <= q < tiles[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s.tiles[mid] <= q) lo = mid;
            else hi = mid;
        }
        at.g = lo;
        place(p.band, s.tiles[lo + 1] - s.tiles[lo], p.tiles_n, t - s.tiles[lo] * p.tiles_n, at);
        const int all = s.first[lo + 1] - s.first[lo], per = rows_per_tile(all, p.most_rows);
        at.row0 = s.first[lo] + at.tm * per;
        at.rows = min(per, all - at.tm * per);
        share(kGrad ? p.terms * p.num_kb : p.num_kb);
        return;
    }
    if (!kGrad) return;
    const int per = p.w_tiles_m * p.w_tiles_n;
    at.g = t / (per * p.w_count);
    const int r = t - at.g * per * p.w_count;
    at.z = r / per;
    place(p.band, p.w_tiles_m, p.w_tiles_n, r - at.z * per, at);
    at.row0 = s.first[at.g];
    at.rows = s.first[at.g + 1] - at.row0;
    share((at.rows + kTerms - 1) / kTerms);
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

template <int kCtas, int kMode, bool kParts>
__global__ void __launch_bounds__(kThreads, 1) tc_grouped_kernel(const __grid_constant__ Maps maps, const Params p) {
    constexpr bool kGrad = kMode == kGroupedGrad, kGated = kMode == kGroupedGated;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t *stages = smem;
    uint8_t *staging = smem + (size_t)p.num_stages * p.stage_bytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(staging + (kMode != kGroupedPlain ? kStagingBytes : 0));
    uint64_t *full = bars, *empty = bars + kMaxStages, *tail_full = bars + 2 * kMaxStages, *cleared = bars + 3 * kMaxStages;
    uint64_t *tmem_full = bars + 4 * kMaxStages, *tmem_empty = tmem_full + 2;
    uint64_t *slot_full = tmem_empty + 2, *slot_empty = slot_full + kSlots, *answer_here = slot_empty + kSlots;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(answer_here + 1);
    uint4 *slots = reinterpret_cast<uint4 *>(reinterpret_cast<uint8_t *>(bars) + kBarrierBytes) - kSlots, *answer = slots - 1;
    Groups groups;
    groups.first = reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(bars) + kBarrierBytes);
    groups.tiles = groups.first + p.groups + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = kCtas == 2 ? (int)cluster_ctarank() : 0;
    const int ks = kGrad ? 1 : p.ks;
    int unit = blockIdx.x / kCtas;
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
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(&slot_full[i], 1);
            // (the even CTA's, which counts all that are told: epilogue, clearing warp, MMA issuer, the other CTA's producer)
            mbar_init(&slot_empty[i], (kEpiWarps + (kGrad ? 1 : 0)) * kCtas + kCtas);
        }
        mbar_init(answer_here, 1);
        mbar_fence_init();
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
            const int per = rows_per_tile(end - before, p.most_rows);
            int tiles = i < p.groups ? (end - before + per - 1) / per : 0;
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

    // Another CTA of the grid taken over, and its number or -1 (by the even CTA's warp 0)
    int left = (int)gridDim.x;
    uint32_t answer_phase = 0;
    auto ask = [&]() {
        if (lane == 0) {
            fence_proxy_async_smem();              // (the last answer has been read)
            mbar_arrive_expect_tx(answer_here, 16);
            ask_for_block(answer, answer_here);
        }
        __syncwarp();
    };
    auto granted = [&]() {
        mbar_wait(answer_here, answer_phase, p.err, 9);
        answer_phase ^= 1;
        const int block = granted_block(answer);
        __syncwarp();
        return block < 0 || --left <= 0 ? -1 : block / kCtas;
    };
    // There may be CTAs behind the last tile, for groups' tiles that might have been.  Which CTAs are granted goes by no order: such are passed over until there
    // are none to ask for.  One that is such itself does as much at once, and has the tile that it finds for its own (of a pair both have).
    const int tiles = all_tiles<kMode, kParts>(p, groups);
    if (unit >= tiles) {
        int *found = reinterpret_cast<int *>(tmem_holder + 1);
        if (warp == 0 && rank == 0) {
            do {
                ask();
                unit = granted();
            } while (unit >= tiles);
            if (lane == 0) *found = unit;
            if (kCtas == 2 && lane == 0)
                asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(map_to_cta(smem_u32(found), 1)), "r"(unit) : "memory");
        }
        __syncthreads();
        if (kCtas == 2) cluster_sync_all();
        unit = *reinterpret_cast<volatile int *>(found);
    }

    // Whether a tile's last stage ends inside the next group's rows, where it is not by 16 rows that it does
    auto has_tail = [&](const TileAt &t) { return kGrad && !t.x && t.ends && (t.rows & 15) != 0; };

    // The tile after this one, as the even CTA's producer says it; -1: none.  (By a warp's lanes, or the one that issues MMAs.  Nobody has more tiles than
    // there are: that ends the loops where a wait has run out, too.)
    const uint32_t told_back = kCtas == 2 ? map_to_cta(smem_u32(&slot_empty[0]), 0) : 0u;
    int slot = 0;
    uint32_t slot_phase = 0;
    auto next_tile = [&](bool by_warp) {
        if (kCtas == 2) mbar_wait_cluster(&slot_full[slot], slot_phase, p.err, 8);
        else mbar_wait(&slot_full[slot], slot_phase, p.err, 8);
        const int t = *reinterpret_cast<volatile int *>(&slots[slot]);
        if (by_warp) __syncwarp();
        if (!by_warp || lane == 0) {
            if (kCtas == 2) mbar_arrive_remote(told_back + (uint32_t)slot * 8u);
            else mbar_arrive(&slot_empty[slot]);
        }
        if (++slot == kSlots) { slot = 0; slot_phase ^= 1; }
        return --left > 0 ? t : -1;
    };

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer: every lane with a copy of its own per stage
        int stage = 0;
        uint32_t phase = 0;
        const uint32_t full_issuer = kCtas == 2 ? map_to_cta(smem_u32(&full[0]), 0) : 0u;
        const uint32_t tail_own = kCtas == 2 ? map_to_cta(smem_u32(&tail_full[0]), (uint32_t)rank) : 0u;
        const int bnh = p.BN / kCtas;
        int t = unit;
        while (t >= 0) {
            tile_at<kMode, kParts>(p, groups, t, at);
            if (rank == 0) ask();
            // Tiles of rows: the weights in one copy, or in two of 64 (the gated block's channels of each, dX's columns); then this CTA's rows, in one copy or
            // where they are few in one or two small ones.  Gradients of weights: copies of 64 channels and 64 columns by a stage's terms.  Where a stage has two
            // blocks a copy brings both, but for those whose rows would not follow one another then: the gated block's weights, and small ones.
            const int half_rows = ((at.rows + 15) / 16 * 16) / kCtas;
            const bool small = at.x && half_rows <= 2 * p.b_box;
            const int a_boxes = kMode == kGroupedPlain ? 1 : 2, b_boxes = !at.x ? bnh / kBox : small ? (half_rows + p.b_box - 1) / p.b_box : 1;
            const int na = kGated ? a_boxes * ks : a_boxes, nb = small ? b_boxes * ks : b_boxes;
            const int a_box_bytes = kMode != kGroupedPlain ? kBoxBytes : kABytes, b_box_bytes = !at.x ? kBoxBytes : (small ? p.b_box : kBM) * kRowBytes;
            const uint32_t bytes = (uint32_t)(ks * (a_boxes * a_box_bytes + b_boxes * b_box_bytes));
            const bool is_a = lane < na, active = lane < na + nb;
            const int piece = is_a ? lane : lane - na, boxes = is_a ? a_boxes : b_boxes, box = piece % boxes, block = piece / boxes;
            const uint32_t dst_off = !is_a ? p.b_at + (uint32_t)(small ? block * p.b_block + box * b_box_bytes : box * b_box_bytes * ks)
                                     : kGated ? (uint32_t)(block * kABytes + box * kBoxBytes) : (uint32_t)(box * a_box_bytes * ks);
            // The map, and where the copy begins: along a K-major reduction by the term, or by the block (the third) in stages of two; weights (term, channel,
            // block, group), for dX (column, channel, 0, group); rows (term, row, block, 0), or as terms themselves (channel or column, row, 0, 0).
            // From stage to stage one of the first three moves on.
            const CUtensorMap *map;
            int c0 = 0, c1, c2 = 0, c3 = 0;
            const bool second = at.x ? kGrad && is_a : true, by_block = !second && ks > 1;
            if (at.x) {
                map = !is_a ? (small ? &maps.R_small[0] : &maps.R[0]) : &maps.W[kGated ? box : 0];
                c1 = !is_a ? at.row0 + rank * half_rows + box * p.b_box : (at.tn * kCtas + rank) * (kGated ? kBox : kBM);
                if (second) {
                    c0 = c1 + box * kBox;
                    c1 = 0;
                } else {
                    c2 = block;
                }
                c3 = is_a ? at.g : 0;
            } else {
                map = is_a ? &maps.D[p.w_first + at.z] : &maps.X;
                c0 = is_a ? (at.tm * kCtas + rank) * kBM + box * kBox : at.tn * p.BN + rank * bnh + box * kBox;
                c1 = at.row0;
            }
            const int d0 = second || by_block ? 0 : kTerms, d1 = second ? kTerms : 0, d2 = by_block ? ks : 0;
            const bool tail = has_tail(at);
            uint8_t *dst = stages + dst_off;
            auto load = [&](uint32_t cluster_bar, uint64_t *own) {
                if (active) {
                    if (kCtas == 2) tma_load_4d_pair(dst + (size_t)stage * p.stage_bytes, map, cluster_bar + (uint32_t)stage * 8u, c0, c1, c2, c3);
                    else tma_load_4d(dst + (size_t)stage * p.stage_bytes, map, own + stage, c0, c1, c2, c3);
                }
                c0 += d0;
                c1 += d1;
                c2 += d2;
                if (++stage == p.num_stages) { stage = 0; phase ^= 1; }
            };
            auto load_whole = [&](int stages_of_it) {
                for (int kb = 0; kb < stages_of_it; ++kb) {
                    mbar_wait(&empty[stage], phase ^ 1, p.err, 1);
                    if (lane == 0 && rank == 0) mbar_arrive_expect_tx(&full[stage], bytes * kCtas);
                    __syncwarp();
                    load(full_issuer, full);
                }
            };
            auto move = [&](int by) {
                c0 += by * d0;
                c1 += by * d1;
                c2 += by * d2;
            };
            // (dX's second term: the same stages again of the other tensors)
            const int whole = at.kb - (tail ? 1 : 0), of_term = kGrad && at.x ? p.num_kb : whole;
            const bool second_term = kParts && kGrad && at.x && at.kb0 >= of_term;
            if (second_term) map += 1;
            if (kParts) move(second_term ? at.kb0 - of_term : at.kb0);
            const int now = kParts && kGrad && at.x && !second_term ? min(whole, of_term - at.kb0) : kParts ? whole : of_term;
            load_whole(now);
            if (kGrad && now < whole) {
                map += 1;
                move(-of_term);
                load_whole(whole - now);
            }
            if (tail) {
                mbar_wait(&empty[stage], phase ^ 1, p.err, 1);
                if (lane == 0) {
                    mbar_arrive_expect_tx(&tail_full[stage], bytes);
                    if (rank == 0) mbar_arrive(&full[stage]);
                }
                __syncwarp();
                load(tail_own, tail_full);
            }
            // The next tile
            if (rank == 0) {
                if (kCtas == 2) mbar_wait_cluster(&slot_empty[slot], slot_phase ^ 1, p.err, 10);
                else mbar_wait(&slot_empty[slot], slot_phase ^ 1, p.err, 10);
                t = granted();
                while (t >= tiles) {
                    ask();
                    t = granted();
                }
                if (lane == 0) {
                    if (kCtas == 2) {
                        mbar_arrive_expect_tx(&slot_full[slot], 16);
                        for (uint32_t r = 0; r < 2; ++r)
                            st_async_v4(map_to_cta(smem_u32(&slots[slot]), r), (uint32_t)t, 0u, 0u, 0u, map_to_cta(smem_u32(&slot_full[slot]), r));
                    } else {
                        *reinterpret_cast<volatile int *>(&slots[slot]) = t;
                        mbar_arrive(&slot_full[slot]);
                    }
                }
                __syncwarp();
                if (++slot == kSlots) { slot = 0; slot_phase ^= 1; }
            } else {
                if (lane == 0) mbar_arrive_expect_tx(&slot_full[slot], 16);
                __syncwarp();
                t = next_tile(true);
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (of a pair: the even CTA)
        if ((kCtas == 1 || rank == 0) && elect_one()) {
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0, clear_phase = 0;        // (the last: a bit for each stage)
            // K-major: 8-row groups 1024 bytes apart, an instruction 32 bytes further along the swizzled rows, a block as far on as its rows take.  MN-major: blocks of
            // 64 rows or columns 64 terms of 128 bytes apart, groups of 8 terms 1024 bytes apart, an instruction two of those further.
            const uint64_t k_tmpl = make_smem_desc(0, 16, 1024, kSwizzle128B), mn_tmpl = make_smem_desc(0, (uint32_t)kBoxBytes, 1024, kSwizzle128B);
            const uint64_t a_tmpl = kGrad ? mn_tmpl : k_tmpl;
            const uint32_t a_hi = (uint32_t)(a_tmpl >> 32), a_lo = (uint32_t)a_tmpl | ((smem_u32(stages) >> 4) & 0x3FFFu);
            const uint32_t b_base = ((smem_u32(stages) + p.b_at) >> 4) & 0x3FFFu, stage16 = p.stage_bytes >> 4;
            constexpr uint32_t kK16 = 32u >> 4, kMn16 = 2048u >> 4, kA16 = kGrad ? kMn16 : kK16, kABlock16 = (kGrad ? kBoxBytes : kABytes) >> 4;
            for (int t = unit; t >= 0; t = next_tile(false)) {
                tile_at<kMode, kParts>(p, groups, t, at);
                if (at.kb == 0) continue;              // a group without rows
                const bool b_mn = kGrad && !at.x, tail = has_tail(at);
                const uint64_t b_tmpl = b_mn ? mn_tmpl : k_tmpl;
                const uint32_t b_hi = (uint32_t)(b_tmpl >> 32), b_lo = (uint32_t)b_tmpl | b_base, b16 = b_mn ? kMn16 : kK16, b_block16 = (uint32_t)(b_mn ? kBoxBytes : p.b_block) >> 4;
                const uint32_t idesc = b_mn ? p.idesc_w : p.idesc_x | ((uint32_t)((at.rows + 15) / 16 * 2) << 17);
                // instructions of the last stage, where they are not four a block; stages before it
                const int most = 4 * ks, last = b_mn && (!kParts || at.ends) ? (at.rows - (at.kb0 + at.kb - 1) * kTerms + 15) / 16 : most, whole = last == most && !tail ? at.kb : at.kb - 1;
                if (kCtas == 2) mbar_wait_cluster(&tmem_empty[acc], acc_phase ^ 1, p.err, 2);
                else mbar_wait(&tmem_empty[acc], acc_phase ^ 1, p.err, 2);
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + (uint32_t)acc * kMaxBN;
                uint32_t accumulate = 0;
                auto multiply = [&](uint32_t s, uint32_t k) {
                    const uint32_t al = a_lo + (uint32_t)stage * stage16 + s * kABlock16 + k * kA16, bl = b_lo + (uint32_t)stage * stage16 + s * b_block16 + k * b16;
                    if (kCtas == 2) mma_f16_lohi_pair(d_tmem, al, a_hi, bl, b_hi, idesc, accumulate);
                    else mma_f16_lohi(d_tmem, al, a_hi, bl, b_hi, idesc, accumulate);
                    accumulate = 1;
                };
                auto done = [&]() {
                    if (kCtas == 2) mma_commit_pair(&empty[stage]);
                    else mma_commit(&empty[stage]);
                    if (++stage == p.num_stages) { stage = 0; phase ^= 1; }
                };
                for (int kb = 0; kb < whole; ++kb) {
                    mbar_wait(&full[stage], phase, p.err, 3);
                    tc_fence_after_sync();
                    for (uint32_t s = 0; s < (uint32_t)ks; ++s)
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) multiply(s, k);
                    done();
                }
                if (kGrad && whole < at.kb) {
                    mbar_wait(&full[stage], phase, p.err, 3);
                    if (tail) {
                        if (kCtas == 2) mbar_wait_cluster(&cleared[stage], (clear_phase >> stage) & 1u, p.err, 5);
                        else mbar_wait(&cleared[stage], (clear_phase >> stage) & 1u, p.err, 5);
                        clear_phase ^= 1u << stage;
                    }
                    tc_fence_after_sync();
#pragma unroll 1
                    for (uint32_t k = 0; k < (uint32_t)last; ++k) multiply(0, k);
                    done();
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
            const int boxes = kBM / kBox + p.BN / kCtas / kBox;
            for (int t = unit; t >= 0; t = next_tile(true)) {
                tile_at<kMode, kParts>(p, groups, t, at);
                if (at.kb == 0) continue;
                stage += at.kb - 1;
                stage %= p.num_stages;
                if (has_tail(at)) {
                    mbar_wait(&tail_full[stage], (clear_phase >> stage) & 1u, p.err, 6);
                    clear_phase ^= 1u << stage;
                    // a box has a row of the group's, 64 columns of it, in 128 bytes (the swizzle moves pieces within them)
                    const int from = at.rows - (at.kb0 + at.kb - 1) * kTerms, pieces = ((from + 15) / 16 * 16 - from) * 8;
                    uint8_t *first = stages + (size_t)stage * p.stage_bytes + from * kRowBytes;
                    for (int b = 0; b < boxes; ++b) {
                        uint8_t *box = first + b * kBoxBytes;
                        for (int i = lane; i < pieces; i += 32) *reinterpret_cast<uint4 *>(box + i * 16) = make_uint4(0, 0, 0, 0);
                    }
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
        int acc = 0, turn = 0;                         // turn: the half of a buffer that the gated block's next exchange takes, from tile to tile
        uint32_t acc_phase = 0;
        const uint32_t peer_tmem_empty = kCtas == 2 ? map_to_cta(smem_u32(&tmem_empty[0]), 0) : 0u;
        for (int t = unit; t >= 0; t = next_tile(true)) {
            tile_at<kMode, kParts>(p, groups, t, at);
            const bool some = at.kb > 0;
            if (some) {
                mbar_wait(&tmem_full[acc], acc_phase, p.err, 4);
                tc_fence_after_sync();
            }
            const uint32_t tbase = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * kMaxBN);
            auto words_of = [&](const float (&lo)[16], const float (&hi)[16], uint32_t (&h)[16]) {
                if (p.bf16) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) h[i] = pack<__nv_bfloat162>(lo[i], hi[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) h[i] = pack<__half2>(lo[i], hi[i]);
                }
            };
            // Stores rows `first` to first + kRows - 1 of the tile (those that there are) of a result, 32 channels a warp from channel0 on; `value`: a lane's channel's.
            // Of rows 2 i and 2 i + 1 an even lane keeps the first and an odd one the second, each of its own channel and its neighbour's.
            auto store = [&](int which, int first, int channel0, int all, auto rows_of_value, auto value) {
                constexpr int kPairs = decltype(rows_of_value)::value / 2;
                const int odd = lane & 1, mine = channel0 + (lane & ~1), rows = at.rows - first - odd;
                uint32_t h[kPairs];
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float a = value(2 * i), b = value(2 * i + 1), other = __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
                    const float lo = odd ? other : a, hi = odd ? b : other;
                    h[i] = p.bf16 ? pack<__nv_bfloat162>(lo, hi) : pack<__half2>(lo, hi);
                }
                const long long ld = p.y_ld[which];
                uint16_t *out = static_cast<uint16_t *>(p.Y[which]) + (at.row0 + first + odd) * ld + mine;
                if (p.y_pairs[which]) {
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        if (2 * i >= rows || mine >= all) continue;
                        if (mine + 1 < all) *reinterpret_cast<uint32_t *>(out + 2 * i * ld) = h[i];
                        else out[2 * i * ld] = (uint16_t)h[i];
                    }
                } else if (mine < all) {
                    // (as words, one lane's second channel with its neighbour's first where rows begin between two: 12345 rows of 1105 41 us instead of 24)
#pragma unroll
                    for (int i = 0; i < kPairs; ++i)
                        if (2 * i < rows) {
                            out[2 * i * ld] = (uint16_t)h[i];
                            if (mine + 1 < all) out[2 * i * ld + 1] = (uint16_t)(h[i] >> 16);
                        }
                }
            };
            // A part of the reduction: the tile's rows from `first` on as they are, 128 bytes of a row a warp
            auto store_part = [&](int plane, int first, int channel0, int all) {
                uint32_t v[32];
                if (some) {
                    tmem_ld_32x32(tbase + (uint32_t)first, v);
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = 0u;
                }
                const int rows = at.rows - first;
                float *out = p.x_planes + ((long long)plane * p.rows + at.row0 + first) * p.x_pitch + channel0 + lane;
                if (channel0 + lane < all)
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (j < rows) out[j * p.x_pitch] = __uint_as_float(v[j]);
            };
            if (kGated && kParts) {
                // (as below; the gate's planes and the other factor's in turns)
                const int channel0 = (at.tn * kCtas + rank) * kBox + (q & 1) * 32, blocks = channel0 < p.channels ? (at.rows + 31) / 32 : 0;
#pragma unroll 1
                for (int b = half; b < blocks; b += 2) store_part(at.part * 2 + (q >> 1), b * 32, channel0, p.channels);
            } else if (kGated) {
                // Lanes are channels, 64 of the gate and the same 64 of the other factor, columns rows.  The two warps that have the same 32 channels' go through
                // the blocks of 32 rows together; of every quarter two share them in turns.
                const int channel0 = (at.tn * kCtas + rank) * kBox + (q & 1) * 32, blocks = channel0 < p.channels ? (at.rows + 31) / 32 : 0;
                const bool up = q >= 2;
                const std::integral_constant<int, 32> kAll;
                const std::integral_constant<int, 16> kHalf;
                float *given = reinterpret_cast<float *>(buf) + lane;
                const float *got = reinterpret_cast<const float *>(staging + ((warp - 2) ^ 2) * kBlockBytes) + lane;
#pragma unroll 1
                for (int b = half; b < blocks; b += 2, turn ^= 512) {
                    uint32_t v[32];
                    tmem_ld_32x32(tbase + (uint32_t)(b * 32), v);
                    tmem_ld_wait();
                    // of the other warp's results' rows, what it needs (in turns, the tile before among them: it may still read what was given last, and has read
                    // what was given before that once it is at the barrier of the last)
#pragma unroll
                    for (int i = 0; i < 16; ++i) given[turn + i * 32] = __uint_as_float(up ? v[i] : v[16 + i]);
                    if (p.outs == 3) store(up ? 2 : 1, b * 32, channel0, p.channels, kAll, [&](int i) { return __uint_as_float(v[i]); });
                    asm volatile("bar.sync %0, 64;" ::"r"(1 + half * 2 + (q & 1)) : "memory");
                    float g[16], u[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float own = __uint_as_float(up ? v[16 + i] : v[i]), other = got[turn + i * 32];
                        g[i] = up ? other : own;
                        u[i] = up ? own : other;
                    }
#define ONNXB_GATE(kind) _Pragma("unroll") for (int i = 0; i < 16; ++i) g[i] = activate(kind, g[i]) * u[i]
                    if (p.activation == ONNXB_SILU) { ONNXB_GATE(ONNXB_SILU); }
                    else if (p.activation == ONNXB_GELU) { ONNXB_GATE(ONNXB_GELU); }
                    else if (p.activation == ONNXB_GELU_TANH) { ONNXB_GATE(ONNXB_GELU_TANH); }
                    else { ONNXB_GATE(ONNXB_RELU); }
#undef ONNXB_GATE
                    store(0, b * 32 + (up ? 16 : 0), channel0, p.channels, kHalf, [&](int i) { return g[i]; });
                }
            } else if (!kGrad || at.x) {
                // Lanes are channels (columns of the result), columns rows.  The two warps of a quarter share blocks of 32 rows in turns.
                const int all = kGrad ? p.width : p.channels, channel0 = (at.tn * kCtas + rank) * kBM + q * 32, blocks = channel0 < all ? (at.rows + 31) / 32 : 0;
                const std::integral_constant<int, 32> kAll;
#pragma unroll 1
                for (int b = half; b < blocks; b += 2) {
                    if (kParts && p.x_parts > 1) {
                        store_part(at.part, b * 32, channel0, all);
                        continue;
                    }
                    uint32_t v[32];
                    tmem_ld_32x32(tbase + (uint32_t)(b * 32), v);
                    tmem_ld_wait();
                    store(0, b * 32, channel0, all, kAll, [&](int i) { return __uint_as_float(v[i]); });
                }
            } else {
                // Lanes are channels (rows of the gradient), columns its columns.  The two warps of a quarter share its blocks of 64 columns in turns.
                const int row0 = (at.tm * kCtas + rank) * kBM + q * 32, rows = min(32, p.channels - row0), n0 = at.tn * p.BN;
                const int blocks = rows > 0 ? (min(p.BN, p.width - n0) + 63) / 64 : 0;
#pragma unroll 1
                for (int b = half; b < blocks; b += 2) {
#pragma unroll 1
                    for (int c = 0; c < 64; c += 32) {
                        uint32_t v[32], h[16];
                        if (some) {
                            tmem_ld_32x32(tbase + (uint32_t)(b * 64 + c), v);
                            tmem_ld_wait();
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = 0u;
                        }
                        if (kParts && p.w_parts > 1) {
                            // a part of the reduction: 32 columns of 32 rows laid out, and stored as they are, four rows at a time
                            if (b * 64 + c >= p.width - n0) break;
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                *reinterpret_cast<uint4 *>(buf + lane * kRowBytes + ((i ^ (lane & 7)) << 4)) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                            __syncwarp();
                            const int piece = lane & 7, col = n0 + b * 64 + c + piece * 4;
                            float *out = p.w_planes + (((long long)at.part * p.w_count + at.z) * p.groups + at.g) * p.channels * p.w_pitch + row0 * p.w_pitch + col;
                            if (col < p.width)
#pragma unroll 4
                                for (int r = lane >> 3; r < rows; r += 4)
                                    *reinterpret_cast<uint4 *>(out + r * p.w_pitch) = *reinterpret_cast<const uint4 *>(buf + r * kRowBytes + ((piece ^ (r & 7)) << 4));
                            __syncwarp();
                            continue;
                        }
                        float lo[16], hi[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            lo[i] = __uint_as_float(v[2 * i]);
                            hi[i] = __uint_as_float(v[2 * i + 1]);
                        }
                        words_of(lo, hi, h);
                        // the lane's row of the block, 16-byte piece i at position i ^ (lane % 8)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *reinterpret_cast<uint4 *>(buf + lane * kRowBytes + (((c / 8 + i) ^ (lane & 7)) << 4)) =
                                make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
                    }
                    if (kParts && p.w_parts > 1) continue;
                    __syncwarp();
                    // Stored by rows, four at a time in pieces of 16 bytes, or one in pairs of elements
                    const int w = p.w_first + at.z, left = min(64, p.width - n0 - b * 64);
                    const long long ld = p.d_ld[w];
                    uint16_t *out = static_cast<uint16_t *>(p.D[w]) + at.g * p.d_stride[w] + row0 * ld + n0 + b * 64;
                    if (p.d_wide[w]) {
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
                        // (as words, of rows that begin between two one lane's second element with its neighbour's first: 86 gradients of 8166 x 633 529 us
                        // instead of 356)
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

// The parts' planes added up, in their order, and rounded: four columns a thread, 8 rows by 128 columns a block.  Of the gated block (kGated) those of both factors, and the
// activation.
struct SumJob {
    const float *planes;
    long long pitch, plane, factor;  // floats of a row, of a plane (of both factors), of one factor's
    int parts, rows, cols;
    uint16_t *out[3];                // (the gated block: H, and G and U or NULL)
    long long ld[3], stride;
    int group_rows;                  // rows of a group's result
    const int *offsets;              // of results by row (else NULL), of which those alone are written that are a group's
};
struct SumProblem {
    SumJob job[3];
    int groups, bf16, activation;
};
template <bool kGated>
__global__ void __launch_bounds__(256) grouped_sum_kernel(const __grid_constant__ SumProblem problem) {
    const SumJob &p = problem.job[blockIdx.z];
    const int j = (blockIdx.x * 32 + threadIdx.x % 32) * 4;
    pdl_launch_dependents();
    pdl_wait();
    // (the offsets are on their way while the planes are read, of rows of no group too)
    int first = 0, last = p.rows;
    if (p.offsets) {
        first = max(p.offsets[0], 0);
        last = 0;
        for (int i = threadIdx.x % 32; i <= problem.groups; i += 32) last = max(last, p.offsets[i]);
    }
    auto sum = [&](const float *from) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < p.parts; s += 4, from += 4 * p.plane) {
            float4 w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) w[u] = s + u < p.parts ? *reinterpret_cast<const float4 *>(from + u * p.plane) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int u = 0; u < 4; ++u) v = make_float4(v.x + w[u].x, v.y + w[u].y, v.z + w[u].z, v.w + w[u].w);
        }
        return v;
    };
    auto put = [&](uint16_t *to, const float4 &v) {
        const uint32_t lo = problem.bf16 ? pack<__nv_bfloat162>(v.x, v.y) : pack<__half2>(v.x, v.y), hi = problem.bf16 ? pack<__nv_bfloat162>(v.z, v.w) : pack<__half2>(v.z, v.w);
        if (j + 4 <= p.cols && reinterpret_cast<uintptr_t>(to) % 8 == 0) *reinterpret_cast<uint2 *>(to) = make_uint2(lo, hi);
        else {
            const uint16_t e[4] = {(uint16_t)lo, (uint16_t)(lo >> 16), (uint16_t)hi, (uint16_t)(hi >> 16)};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (j + k < p.cols) to[k] = e[k];
        }
    };
    bool known = !p.offsets;
    for (long long i = blockIdx.y * 8 + threadIdx.x / 32; i < p.rows; i += gridDim.y * 8) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f), u = v;
        const float *from = p.planes + i * p.pitch + j;
        if (j < p.cols) {
            v = sum(from);
            if (kGated) u = sum(from + p.factor);
        }
        if (!known) {
            last = min(__reduce_max_sync(0xffffffffu, last), p.rows);
            known = true;
        }
        if (i < first || i >= last || j >= p.cols) continue;
        if (kGated) {
            if (p.out[1]) {
                put(p.out[1] + i * p.ld[1] + j, v);
                put(p.out[2] + i * p.ld[2] + j, u);
            }
            const int kind = problem.activation;
            put(p.out[0] + i * p.ld[0] + j, make_float4(activate(kind, v.x) * u.x, activate(kind, v.y) * u.y, activate(kind, v.z) * u.z, activate(kind, v.w) * u.w));
        } else {
            const int g = p.offsets ? 0 : (int)i / p.group_rows;
            put(p.out[0] + g * p.stride + (i - (long long)g * p.group_rows) * p.ld[0] + j, v);
        }
    }
}

typedef void (*Kernel)(const Maps, const Params);
// (of reductions in parts kernels of their own: one for both took 99 us instead of 91 for the gradients of a gated block of 512 rows, 16 groups, 1024 -> 2816)
template <int kCtas>
Kernel kernel_for(int mode, bool parts) {
    if (parts)
        return mode == kGroupedPlain ? tc_grouped_kernel<kCtas, kGroupedPlain, true> : mode == kGroupedGated ? tc_grouped_kernel<kCtas, kGroupedGated, true>
                                                                                   : tc_grouped_kernel<kCtas, kGroupedGrad, true>;
    return mode == kGroupedPlain ? tc_grouped_kernel<kCtas, kGroupedPlain, false> : mode == kGroupedGated ? tc_grouped_kernel<kCtas, kGroupedGated, false>
                                                                                : tc_grouped_kernel<kCtas, kGroupedGrad, false>;
}

// The kernel's shared memory allowed for, once a device
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

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// CTAs of a tile, and the most rows of one of rows
struct Tile {
    int ctas, rows;
};
bool tile_allowed(Tile t) {
    return (t.ctas == 1 || t.ctas == 2) && t.rows >= 16 && t.rows % 16 == 0 && t.rows <= 128 * t.ctas;
}
// K blocks of a stage.  Two where a forward product's reduction is whole blocks and the ring still has four stages: tiles of up to 128 rows
// (gated block of 2 rows 64 -> 60 us; tiles of 256 by 128 rows, 16384 x 2816 x 4096, 370 -> 331, but with three stages tiles of 256 by 256 265 -> 287).
// Of gradients, whose ring has five or six blocks, one.  ONNXB_GROUPED_KS = 1 or 2 pins it for forward products, where the ring has three stages at least.
int blocks_per_stage(const GroupedProblem &d, int blocks_in_ring) {
    if (d.mode == kGroupedGrad || d.width % kTerms) return 1;
    if (const char *e = getenv("ONNXB_GROUPED_KS")) return blocks_in_ring >= 6 && e[0] == '2' ? 2 : 1;
    return blocks_in_ring >= 8 ? 2 : 1;
}
long long plane_pitch(int cols) { return (cols + 3ll) / 4 * 4; }
// Tiles, and parts of the reductions (of tiles of rows, of the weights' gradients): by the sizes alone, since the workspace depends on the parts, and whichever
// gradients are wanted, so that each is the same bit by bit with others and without.
struct Plan {
    Tile tile;
    int x, w;
};
// SM cycles a B200's 148 SMs take for a forward product, roughly: waves of tiles whose stages cost what the single threads take (measured: 300 to 350 cycles a block in
// stages of two, 400 to 440 of one), or what L2 or DRAM bring.  Groups have rows that differ: a tile more each than whole ones.  Parts cost a launch, and planes of fp32.
double forward_cost(const GroupedProblem &d, Tile t, int parts) {
    const int groups = std::min(d.rows, d.groups), per = (d.rows + groups - 1) / groups, b = t.rows / t.ctas, ks = d.width % kTerms == 0 && b <= 64 ? 2 : 1;
    const int factors = d.mode == kGroupedGated ? 2 : 1;
    const double across = (double)ceil_div(d.channels, kBM / factors * t.ctas), kb = (double)ceil_div(d.width, kTerms);
    const double tiles = (double)groups * (groups > 1 ? per / t.rows + 1 : ceil_div(per, t.rows)) * across, waves = tiles * parts * t.ctas / 148;
    const double each = ceil(kb / parts) * (ks == 2 ? 270 + 1.2 * b : 380 + 0.5 * b) + 1500 + 12 * factors * t.rows + (t.ctas - 1) * 1000;
    const double l2 = tiles * t.ctas * kb * (kABytes + b * kRowBytes) / 8900, dram = 2.0 * groups * d.channels * d.width * factors / 3400;
    const double cost = std::max({(waves > 4 ? waves + 0.5 : ceil(waves)) * each, l2, dram});
    return cost + 11000 + (parts > 1 ? 3000 + 2000 * factors + (8.0 * parts + 2) * d.rows * (double)d.channels * factors / 4500 : 0);
}
// The same of gradients: the tiles of rows first, then the weights', each taken by the pair that is free first
double backward_cost(const GroupedProblem &d, Tile t, int x_parts, int w_parts) {
    const int groups = std::min(d.rows, d.groups), per = (d.rows + groups - 1) / groups, units = 148 / t.ctas;
    const double across = (double)ceil_div(d.width, kBM * t.ctas), of_rows = groups * (groups > 1 ? per / t.rows + 1 : ceil_div(per, t.rows)) * across * x_parts;
    const double of_weights = d.groups * d.terms * ceil_div(d.channels, kBM * t.ctas) * across * w_parts;
    const double x = ceil((double)d.terms * ceil_div(d.channels, kTerms) / x_parts) * 450 + 4500, w = ceil((double)ceil_div(per, kTerms) / w_parts) * 550 + 4500;
    // pairs that end their last tile of rows early, and late; until a time they have so many of the weights'
    const double waves = floor(of_rows / units), late = of_rows - waves * units, begins = waves * x, begins_late = begins + (late > 0 ? x : 0);
    auto has = [&](double until) { return late * floor(std::max(0.0, until - begins_late) / w) + (units - late) * floor(std::max(0.0, until - begins) / w); };
    // (not before all pairs would be done if they were done together)
    double end = begins_late;
    for (double k = std::max(0.0, floor((late * begins_late + (units - late) * begins + of_weights * w) / units / w - begins_late / w)); has(end) < of_weights; ++k) {
        end = std::max(begins_late, begins + k * w);
        if (has(end) < of_weights) end = begins_late + k * w;
    }
    return end + 11000 + (x_parts > 1 || w_parts > 1 ? 4000 : 0) + (x_parts > 1 ? (8.0 * x_parts + 2) * d.rows * (double)d.width / 3000 : 0) +
           (w_parts > 1 ? (8.0 * w_parts + 2) * d.groups * d.terms * (double)d.channels * d.width / 3000 : 0);
}
// Forward products.  Twice the rows that groups have on average, since some have more (32 groups of 32 rows, 2048 x 1408: gated block in tiles of 32, 64 and 128 rows 66, 60 and
// 63 us), and pairs from 33 rows on (64 rows: 68 us in tiles of one CTA, 66 of two).  Where that would be fewer tiles than SMs, what costs least (512 rows of 4 groups, 8192 ->
// 1024: 27.1 us in 40 tiles of 64 rows, 35.0 in 16 of 256, 20.9 with four parts of each; gated block, 512 of 8, 7168 -> 256, 24.6 and 17.9; 13926 rows of one, 64 -> 72: in tiles of 256 rows 9.7, of 128 6.6).
Plan forward_plan(const GroupedProblem &d, bool any_tile, Plan plan, bool any_parts) {
    const int groups = std::min(d.rows, d.groups), per_group = (d.rows + groups - 1) / groups, all = (d.rows + 15) / 16 * 16, kb = (int)ceil_div(d.width, kTerms);
    if (any_tile) {
        plan.tile = Tile{per_group > 32 ? 2 : 1, 32};
        while (plan.tile.rows < 128 * plan.tile.ctas && plan.tile.rows < 2 * per_group) plan.tile.rows *= 2;
        plan.tile.rows = std::min(plan.tile.rows, all);
    }
    const bool gated = d.mode == kGroupedGated;
    if (groups * ceil_div(per_group, plan.tile.rows) * ceil_div(d.channels, (gated ? kBox : kBM) * plan.tile.ctas) * plan.tile.ctas >= 148) return plan;
    const Plan first = plan;
    double best = 0.93 * forward_cost(d, first.tile, first.x);
    for (int ctas = 1; ctas <= 2; ++ctas)
        for (int rows = 32; rows <= 128 * ctas; rows *= 2)
            for (int parts = 1; parts <= 16; parts *= 2) {
                if (parts > 1 && kb < 8 * parts) continue;
                const Plan other{any_tile ? Tile{ctas, std::min(rows, all)} : first.tile, any_parts ? parts : first.x, 1};
                const double cost = forward_cost(d, other.tile, other.x);
                if (cost < best) {
                    best = cost;
                    plan = other;
                }
            }
    return plan;
}
// Gradients: pairs, and as many rows as they take (32 groups of 4 to 128 rows, 2048 x 1408: a tenth to a fifth faster than one CTA, and no slower with more rows than groups
// have).  Parts where there are few tiles and much to add up: of the weights' gradients (4096 rows of one group, 512 x 512: 25.3 us in one, 19.1, 15.7 and 16.8 in 2, 4 and 8;
// but 4096 of 4, 128 x 2048, 19.9, 22.8 and 25.9 in 1, 2 and 4), and of dX (gated block of 64 rows of one, 8192 x 512: 67.3 us in one, 30.3, 24.9 and 23.8 in 4, 8 and 16; but 300 of 4,
// plain, 4096 x 1024, 26.9, 26.9 and 28.0 in 1, 2 and 4).
Plan backward_plan(const GroupedProblem &d, bool any_tile, Plan plan, bool any_parts) {
    const int groups = std::min(d.rows, d.groups), per_group = (d.rows + groups - 1) / groups;
    if (any_tile) plan.tile = Tile{2, std::min(256, (d.rows + 15) / 16 * 16)};
    const long long across = ceil_div(d.width, kBM * plan.tile.ctas);
    const double tiles = (double)across * (groups * ceil_div(per_group, plan.tile.rows) + groups * d.terms * ceil_div(d.channels, kBM * plan.tile.ctas));
    if (!any_parts || tiles * plan.tile.ctas > 16 * 148) return plan;
    // Twice or four times the parts of either, as long as twice gains 7 %
    const int of_rows = d.terms * (int)ceil_div(d.channels, kTerms), of_weights = (int)ceil_div(per_group, kTerms);
    double best = backward_cost(d, plan.tile, 1, 1);
    for (bool gains = true; gains;) {
        const Plan from = plan;
        gains = false;
        for (int more = 2; more <= 4; more *= 2)
            for (int which = 0; which < 2; ++which) {
                const int x = which ? from.x : from.x * more, w = which ? from.w * more : from.w;
                if (x > 16 || w > 16 || (which ? of_weights < 4 * w : of_rows < 4 * x)) continue;
                const double cost = backward_cost(d, plan.tile, x, w), margin = more == 2 ? 1.07 : 1.145;
                if (cost * margin >= best) continue;
                best = cost * margin;
                plan.x = x;
                plan.w = w;
                gains = true;
            }
        if (gains) best = backward_cost(d, plan.tile, plan.x, plan.w);
    }
    return plan;
}
Plan pick_plan(const GroupedProblem &d) {
    // "<CTAs>x<rows>" in ONNXB_GROUPED_TILE, and "<parts>" or "<of rows>,<of weights>" in ONNXB_GROUPED_PARTS, pin them for A/B measurements and tests
    const char *shape = getenv("ONNXB_GROUPED_TILE"), *parts = getenv("ONNXB_GROUPED_PARTS"), *comma = parts ? strchr(parts, ',') : nullptr;
    const Tile tile{shape && shape[0] ? shape[0] - '0' : 0, shape && shape[0] && shape[1] == 'x' ? atoi(shape + 2) : 0};
    auto count = [](const char *e) { return std::max(1, std::min(16, atoi(e))); };
    const Plan plan{tile, parts ? count(parts) : 1, parts && d.mode == kGroupedGrad ? count(comma ? comma + 1 : parts) : 1};
    // (the last sizes' plan is kept: a call asks twice, and it takes a microsecond)
    const std::array<int, 6> sizes{d.mode, d.rows, d.groups, d.channels, d.width, d.terms};
    static thread_local std::array<int, 6> last_sizes{-1};
    static thread_local Plan last;
    const bool pinned = shape || parts;
    if (!pinned && sizes == last_sizes) return last;
    const Plan found = d.mode == kGroupedGrad ? backward_plan(d, !tile_allowed(tile), plan, !parts) : forward_plan(d, !tile_allowed(tile), plan, !parts);
    if (!pinned) {
        last_sizes = sizes;
        last = found;
    }
    return found;
}
// Rows that begin at multiples of 16 bytes, as (terms, rows, 1, 1) in boxes of 64 by `box`; groups' weights as (terms, channels, 1, groups).  Where `blocks` is not 0
// (terms of a block, rows, blocks, 1) and (terms of a block, channels, blocks, groups), `blocks` of them a copy: of reductions that are whole blocks.
bool rows_map(CUtensorMap *m, const DenseOperand &o, long long rows, long long cols, int box, int blocks = 0) {
    const uint64_t pitch = (uint64_t)(rows > 1 ? o.ld * 2 : (o.ld * 2 + 15) / 16 * 16);
    const uint64_t dims[4] = {(uint64_t)(blocks ? kTerms : cols), (uint64_t)rows, (uint64_t)(blocks ? cols / kTerms : 1), 1};
    const uint64_t pitches[3] = {pitch, blocks ? (uint64_t)kRowBytes : pitch, pitch};
    const uint32_t boxes[4] = {kTerms, (uint32_t)box, (uint32_t)(blocks ? blocks : 1), 1};
    return tc_host::make_tmap_of(2, m, o.p, 4, dims, pitches, boxes, tc_host::kTmapSwizzle128);
}
bool weights_map(CUtensorMap *m, const GroupedWeights &w, long long groups, long long channels, long long width, int box, int blocks = 0) {
    const uint64_t pitch = (uint64_t)(channels > 1 ? w.ld * 2 : (width * 2 + 15) / 16 * 16);
    const uint64_t dims[4] = {(uint64_t)(blocks ? kTerms : width), (uint64_t)channels, (uint64_t)(blocks ? width / kTerms : 1), (uint64_t)groups};
    const uint64_t pitches[3] = {pitch, blocks ? (uint64_t)kRowBytes : pitch, groups > 1 ? (uint64_t)w.stride * 2 : pitch};
    const uint32_t boxes[4] = {kTerms, (uint32_t)box, (uint32_t)(blocks ? blocks : 1), 1};
    return tc_host::make_tmap_of(2, m, w.p, 4, dims, pitches, boxes, tc_host::kTmapSwizzle128);
}
bool by_16(const void *p, long long ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }

}  // namespace

size_t tc_grouped_workspace(const GroupedProblem &d, bool rows, int weights) {
    const Plan plan = pick_plan(d);
    const long long of_rows = rows && plan.x > 1 ? plan.x * (d.mode == kGroupedGated ? 2ll : 1ll) * d.rows * plane_pitch(d.mode == kGroupedGrad ? d.width : d.channels) : 0;
    const long long of_weights = plan.w > 1 ? (long long)plan.w * weights * d.groups * d.channels * plane_pitch(d.width) : 0;
    return (size_t)(of_rows + of_weights) * 4;
}

int launch_tc_grouped(const GroupedProblem &d, cudaStream_t stream) {
    using namespace tc_host;
    const bool gated = d.mode == kGroupedGated, grad = d.mode == kGroupedGrad;
    const Plan plan = pick_plan(d);
    const Tile tile = plan.tile;
    Params p{};
    p.rows = d.rows; p.groups = d.groups; p.offsets = d.offsets;
    p.channels = d.channels; p.width = d.width;
    p.most_rows = tile.rows;
    const int columns = (gated ? kBox : kBM) * tile.ctas;  // of a tile of rows
    p.tiles_n = (int)ceil_div(grad ? d.width : d.channels, columns);
    p.band = 8;
    // small copies of rows: no more than all the rows that there are
    p.b_box = d.rows <= 16 ? 16 : 32;
    p.terms = d.terms;
    p.with_x = grad && d.Y[0] ? 1 : 0;
    p.w_first = d.D[0].p ? 0 : 1;
    p.w_count = grad ? (d.D[0].p != nullptr) + (d.D[1].p != nullptr) : 0;
    p.BN = kBM * tile.ctas;
    p.w_tiles_m = (int)ceil_div(d.channels, kBM * tile.ctas);
    p.w_tiles_n = (int)ceil_div(d.width, p.BN);
    p.x_parts = grad && !p.with_x ? 1 : plan.x;
    p.w_parts = p.w_count ? plan.w : 1;
    const long long w_total = (long long)d.groups * p.w_count * p.w_tiles_m * p.w_tiles_n;
    // tiles of rows: at most one more for each group than whole ones
    const long long row_tiles = grad && !p.with_x ? 0 : d.rows / tile.rows + std::min(d.groups, d.rows), most = row_tiles * p.tiles_n * p.x_parts + w_total * p.w_parts;
    if (most > 0x7fffffffLL / 4 || (long long)p.band * std::max(p.tiles_n, p.w_tiles_n) > 0x7fffffffLL) return (int)cudaErrorInvalidValue;
    p.w_total = (int)w_total;
    // (B: the rows of a CTA's part of a tile, or of the gradients of weights its columns)
    const int b_rows = grad ? kBM : std::max(tile.rows / tile.ctas > 2 * p.b_box ? kBM : 0, 2 * p.b_box);
    const int table = ((2 * d.groups + 2) * 4 + 15) / 16 * 16, staging = d.mode != kGroupedPlain ? kStagingBytes : 0;
    const int ring = kSmemLimit - 1024 - kBarrierBytes - staging - table, block_bytes = kABytes + b_rows * kRowBytes;
    p.ks = blocks_per_stage(d, ring / block_bytes);
    p.b_block = b_rows * kRowBytes;
    p.b_at = (uint32_t)(p.ks * kABytes);
    p.stage_bytes = (uint32_t)(p.ks * block_bytes);
    p.num_stages = std::min(kMaxStages, ring / (int)p.stage_bytes);
    p.num_kb = (int)ceil_div(grad ? d.channels : d.width, kTerms * p.ks);
    const int bf16 = d.type == ONNXB_BFLOAT16;
    p.idesc_x = make_idesc_f16(kBM * tile.ctas, 0, bf16, grad, 0);
    p.idesc_w = make_idesc_f16(kBM * tile.ctas, p.BN, bf16, 1, 1);
    p.bf16 = bf16;
    p.activation = d.activation;
    p.outs = gated && d.Y[1] ? 3 : 1;
    for (int i = 0; i < 3; ++i) { p.Y[i] = d.Y[i]; p.y_ld[i] = d.y_ld[i]; p.y_pairs[i] = reinterpret_cast<uintptr_t>(d.Y[i]) % 4 == 0 && d.y_ld[i] % 2 == 0; }
    for (int i = 0; i < 2; ++i) {
        p.D[i] = const_cast<void *>(d.D[i].p); p.d_ld[i] = d.D[i].ld; p.d_stride[i] = d.D[i].stride;
        p.d_wide[i] = by_16(d.D[i].p, d.D[i].ld) && d.D[i].stride % 8 == 0;
    }
    p.err = device_status_ptr();
    if (!p.err) return (int)cudaErrorUnknown;
    const int cols = grad ? d.width : d.channels;
    p.x_pitch = plane_pitch(cols);
    p.w_pitch = plane_pitch(d.width);
    p.x_planes = static_cast<float *>(d.planes);
    p.w_planes = p.x_planes + (p.x_parts > 1 ? p.x_parts * (long long)d.rows * p.x_pitch : 0);

    Maps maps{};
    bool fine = true;
    const int terms = grad ? d.terms : 1, along = grad ? d.channels : d.width;
    if (!grad || p.with_x) {
        const int blocks = p.ks > 1 ? p.ks : 0, single = p.ks > 1 ? 1 : 0;
        for (int i = 0; i < terms; ++i)
            fine = fine && rows_map(&maps.R[i], d.A[i], d.rows, along, kBM, blocks) && rows_map(&maps.R_small[i], d.A[i], d.rows, along, p.b_box, single);
        for (int i = 0; i < (gated ? 2 : terms); ++i)
            fine = fine && (grad ? weights_map(&maps.W[i], d.W[i], d.groups, d.channels, d.width, kBox)
                                 : weights_map(&maps.W[i], d.W[i], d.groups, d.channels, d.width, gated ? kBox : kBM, gated ? single : blocks));
    }
    if (p.w_count) {
        for (int i = 0; i < terms; ++i) fine = fine && rows_map(&maps.D[i], d.A[i], d.rows, d.channels, kBox);
        fine = fine && rows_map(&maps.X, d.X, d.rows, d.width, kBox);
    }
    if (!fine) return (int)cudaErrorInvalidValue;

    const size_t smem = smem_with_tmem(1024 + (size_t)p.num_stages * p.stage_bytes + staging + kBarrierBytes + table, 512);
    const bool in_parts = p.x_parts > 1 || p.w_parts > 1;
    const Kernel kernel = tile.ctas == 2 ? kernel_for<2>(d.mode, in_parts) : kernel_for<1>(d.mode, in_parts);
    const cudaError_t attr_err = allow_shared_memory(kernel, ((tile.ctas - 1) * 2 + in_parts) * 3 + d.mode);
    if (attr_err != cudaSuccess) return (int)attr_err;
    const int grid = (int)most * tile.ctas;
    const cudaError_t e = tile.ctas == 2 ? launch_pdl_cluster(kernel, 2u, dim3(grid), dim3(kThreads), smem, stream, maps, p)
                                         : launch_pdl(kernel, dim3(grid), dim3(kThreads), smem, stream, maps, p);
    count_launch();
    if (e != cudaSuccess || !in_parts) return (int)e;
    SumProblem sum{};
    sum.groups = d.groups; sum.bf16 = bf16; sum.activation = d.activation;
    int jobs = 0, most_rows = 1;
    if (p.x_parts > 1) {
        const long long factor = d.rows * p.x_pitch;
        SumJob &job = sum.job[jobs++];
        job = SumJob{p.x_planes, p.x_pitch, gated ? 2 * factor : factor, factor, p.x_parts, d.rows, cols, {}, {}, 0, 1, d.offsets};
        for (int i = 0; i < p.outs; ++i) { job.out[i] = static_cast<uint16_t *>(p.Y[i]); job.ld[i] = p.y_ld[i]; }
        most_rows = d.rows;
    }
    for (int i = 0; p.w_parts > 1 && i < p.w_count; ++i) {
        const int w = p.w_first + i, rows = d.groups * d.channels;
        const long long result = rows * p.w_pitch;
        sum.job[jobs++] = SumJob{p.w_planes + i * result, p.w_pitch, p.w_count * result, 0, p.w_parts, rows, d.width, {static_cast<uint16_t *>(p.D[w])}, {p.d_ld[w]},
                                 p.d_stride[w], d.channels, nullptr};
        most_rows = std::max(most_rows, rows);
    }
    const dim3 sum_grid((unsigned)ceil_div(cols, 128), (unsigned)std::min(65535ll, ceil_div(most_rows, 8)), (unsigned)jobs);
    const cudaError_t sum_err = launch_pdl(gated ? grouped_sum_kernel<true> : grouped_sum_kernel<false>, sum_grid, dim3(256), 0, stream, sum);
    count_launch();
    return (int)sum_err;
}

}  // namespace onnxb
