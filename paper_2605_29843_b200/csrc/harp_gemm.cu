// Products of a layer on the tensor cores (tcgen05.mma, operands and accumulators fed by bulk tensor copies):
//
//   FORWARD        y[r][n]  = sum_k x[r][k] w_e[n][k]       (8 bits: times row_scale[r] channel_scale_e[n])
//   GRAD_ROWS      dx[r][k] = sum_n dy[r][n] w_e[n][k]
//   GRAD_WEIGHTS   dw_e[n][k] = sum_{r in e} dy[r][n] x[r][k]
//
// e: the group that row r belongs to.  In all three the dimension that is contiguous in the output lies along the lanes of
// tensor memory and the other one along its columns.  A warp then stores 32 neighbouring elements of an output row, and
// the number of columns of an instruction follows the rows that a group has (N = 16, 32, ... 256), so that a group of 40
// rows costs the products of 64 and no more.
//
// Two CTAs of a cluster work on one tile of 256 lanes x up to 256 columns (cta_group::2: either holds half of both
// operands, 32 KB a stage of 128 bytes along the contracted dimension).  Where that leaves SMs idle or memory waiting, a CTA
// works on 128 lanes x 32 or 64 columns, two CTAs an SM, and up to four of them divide the contracted dimension and add up their
// accumulators through distributed shared memory, in the order of their ranks.  Tiles are handed out round robin; two
// accumulators fit tensor memory, so a tile's epilogue runs under the next one's products.
//
// What bounds it (B200, 1965 MHz, 6538 GB/s and 1670 bf16 TFLOP/s measured).  Large products: the way from L2, which gives 9.9 TB/s to
// 4096 rows over 8 groups, 8192 -> 4096 (tensor pipe 73 %), and under load the power limit: 8192^3 in 8 bits 336 us (3.3 POP/s; 360 in a long
// run), in bf16 724 us (1.52 PFLOP/s, the library's product 677; 766 and 733 in a long run).  Few rows: the weight's bytes: 8 groups of 4 rows, 4096 ->
// 14336, 146 us (6.4 TB/s); 16 rows, 8192 -> 28672 in 8 bits, 42 us (5.6 TB/s); below some 60 MB the 4 to 5 us that a launch,
// the first copy's way and the last stores take: 4096 -> 14336 14 us, 4096 -> 4096 8 us.  Weight gradients of short groups: their stores, which
// leave an SM at 32 bytes a cycle (32 groups of 31 rows, 2048 x 4096, bf16 106 us, 5.2 TB/s).
//
// Every operand is brought by tiled copies with the 128-byte swizzle, K-major where the contracted dimension is contiguous and
// MN-major where it is not (w in GRAD_ROWS, both operands in GRAD_WEIGHTS: no transposed copy of anything is made).  Copies
// past the end of a matrix fill zeros.  Past the end of a group they bring the next group's rows: harmless columns where rows lie
// along the columns; in GRAD_WEIGHTS a warp overwrites them with zeros before the products, in both
// operands, because the other group's values may be infinite.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <mutex>
#include <type_traits>

#include <cuda.h>

#include "harp_gemm_ptx.cuh"
#include "harp_internal.h"
#include "harp_linear.h"

namespace harp_linear {
namespace {

using namespace harp_gemm_ptx;

constexpr int kThreads = 384;                // warps: 0 copies, 1 products, 2 tensor memory, 3 offsets, then both ragged ends, 4-11 epilogue (two a lane quarter)
constexpr int kHalf = 16384;                 // the lane operand's part of a stage in one CTA
// The tensor core cuts its fp32 sums off instead of rounding them: the sum of n products of one sign comes out too small by 1.4e-9 n of itself
// after 512 of them, 4 to 6e-9 n from some thousand on (mixed signs: by chance, 1e-6 at most of the sum of magnitudes).  Results in fp32 are therefore summed in
// runs of 512 products, which the epilogue adds up, rounding to nearest: 7 to 9e-7 too small, and 2^-24 at most for each run that is added.  bf16
// results round off 2^-8 at most in any case and take one run of up to 32768 products (2e-4, a twentieth of that), whose sum the stores read where it lies.
// Beyond that they take runs of 512 too (one run of 2^20: 6e-3), in kernels of their own: the registers that hold sums cost short sums too much (both gradients of 32
// groups of 31 rows, 2048 x 4096, 218 -> 315 us in a kernel that could do either).  Weight gradients of 65536 rows, 2048 x 4096, 786 us as one run, 865 now.
constexpr int kRun = 8;                      // blocks
constexpr int kLone = 32768;                 // products
constexpr int kTurnBytes = 8 * 2048;         // where the epilogue warps of a pair's CTA turn bf16 results round
constexpr int kSumCols = 32;                 // columns whose sums a split adds up at a time
// COLS: most columns of a tile (256 for a pair of CTAs, 32 or 64 for one).  DEEP: a single CTA has the SM for itself, and the shared memory;
// else it leaves room for another one
__host__ __device__ constexpr int stage_bytes(int cols) { return kHalf + (cols == 256 ? 128 : cols) * 128; }
__host__ __device__ constexpr int stages(int cols, bool deep) { return cols == 256 ? 6 : cols == 64 ? (deep ? 7 : 3) : deep ? 9 : 4; }
constexpr uint32_t kSpin = 1u << 22;         // limit of every wait
constexpr int kMostSmem = 232448 - 4096;     // dynamic shared memory, less what the kernels have besides

__device__ int32_t g_gemm_err;

struct Params {
    int32_t lanes, cols, depth;              // cols: of GRAD_WEIGHTS alone; depth: of the others
    int32_t n_rows, n_groups;
    const int32_t *offsets;
    int32_t tile_cols;                       // most columns of a tile
    int32_t split;                           // CTAs that divide the contracted dimension
    void *out;
    int64_t ld_out, group_out;               // group_out: elements between two groups' outputs (GRAD_WEIGHTS)
    const float *row_scale, *channel_scale;
    int32_t accumulate;
    int32_t above, most;                     // GRAD_WEIGHTS: groups of more rows than `above`, of `most` at most; the others are another launch's
    int32_t chunked_a, chunked_b;            // MN-major operands: both chunks of 64 by one copy
    int32_t pairs, eights;                   // bf16 results may be stored two, eight lanes at a time
    int32_t *err;
};

struct Tile {
    int e, lane0, col0, cols, row0, blocks, tail;    // cols: valid ones; row0: first row; tail: rows in the last block (GRAD_WEIGHTS);
                                                     // blocks: -1 where the tile is another launch's
};

__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }
__device__ __forceinline__ int round_up(int a, int b) { return div_up(a, b) * b; }

// columns of the tiles of a group of n rows: as even as the instruction's sizes let them be
template <int CG>
__device__ __forceinline__ int even_cols(int n, int most) {
    return n <= 0 ? most : round_up(div_up(n, div_up(n, most)), CG == 2 ? 32 : 16);
}

// Which tile is number t, for rising t.  Neighbouring numbers share operands: bands of eight lane tiles, column tiles along a band.  Every
// role walks over the tiles by itself, from the group and band of its last one on: finding them by division took longer than the rest of
// a short tile (bf16 weight gradients of 32 groups of 31 rows 118 -> 111 us).
template <int CG, int PRODUCT, int BLOCK>
struct Walk {
    const Params &P;
    const int *off, *first;
    int lane_tiles, e, start, rows, tile_cols, col_tiles, band, band_start;      // start: number of the group's first tile; band_start: from there on

    __device__ __forceinline__ Walk(const Params &P_, const int *off_, const int *first_) : P(P_), off(off_), first(first_) {
        lane_tiles = div_up(P.lanes, 128 * CG);
        start = 0;
        if (PRODUCT == GRAD_WEIGHTS) {
            tile_cols = P.tile_cols;
            col_tiles = div_up(P.cols, P.tile_cols);
        }
        enter(0);
    }
    __device__ __forceinline__ void enter(int group) {
        e = group;
        band = band_start = 0;
        rows = off[e + 1] - off[e];
        if (PRODUCT != GRAD_WEIGHTS) {
            start = first[e];
            tile_cols = even_cols<CG>(rows, P.tile_cols);
            col_tiles = div_up(rows, tile_cols);
        }
    }
    __device__ __forceinline__ Tile at(int t) {
        if (PRODUCT == GRAD_WEIGHTS) {
            int group = e;
            while (t - start >= lane_tiles * col_tiles) start += lane_tiles * col_tiles, ++group;
            if (group != e) enter(group);
        } else {
            int group = e;
            while (first[group + 1] <= t) ++group;
            if (group != e) enter(group);
        }
        while (t - start - band_start >= 8 * col_tiles) band_start += 8 * col_tiles, ++band;
        const int in_band = t - start - band_start, width = min(8, lane_tiles - band * 8);
        const int col = width == 8 ? in_band >> 3 : in_band / width;
        Tile T;
        T.e = e;
        T.lane0 = (band * 8 + in_band - col * width) * 128 * CG;
        T.col0 = col * tile_cols;
        if (PRODUCT == GRAD_WEIGHTS) {
            T.cols = min(tile_cols, P.cols - T.col0);
            T.row0 = off[e];
            T.blocks = div_up(rows, BLOCK);
            T.tail = rows - (T.blocks - 1) * BLOCK;
            if (rows <= P.above || rows > P.most) T.blocks = -1;
        } else {
            T.cols = min(tile_cols, rows - T.col0);
            T.row0 = off[e] + T.col0;
            T.blocks = div_up(P.depth, BLOCK);
            T.tail = BLOCK;
        }
        return T;
    }
};

struct Waiter {
    volatile int *dead;
    int32_t *err;
    // false when the wait gave up (here or elsewhere in the CTA)
    template <bool CLUSTER = false>
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity, int code) const {
        for (uint32_t it = 0; it < kSpin; ++it) {
            if (CLUSTER ? mbar_try_cluster(bar, parity) : mbar_try(bar, parity)) return true;
            if ((it & 63) == 63 && *dead) return false;
        }
        *dead = 1;
        atomicExch(err, code);
        return false;
    }
    // behind stores of another CTA
    __device__ __forceinline__ bool cluster(uint32_t bar, uint32_t parity, int code) const { return operator()<true>(bar, parity, code); }
};

__device__ __forceinline__ void store(float *p, float v) { *p = v; }
__device__ __forceinline__ void store(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float load(const float *p) { return *p; }
__device__ __forceinline__ float load(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

// stage and phase of the ring of stages
template <int STAGES>
struct Ring {
    int s = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++s == STAGES) {
            s = 0;
            phase ^= 1;
        }
    }
    __device__ __forceinline__ void skip(int n) {
        n += s;
        phase ^= (n / STAGES) & 1;
        s = n % STAGES;
    }
};

__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }
__device__ __forceinline__ uint32_t pack_bf16(uint32_t lo, uint32_t hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(__uint_as_float(hi)), "f"(__uint_as_float(lo)));
    return r;
}

// RUNS: sums of runs of blocks are added up in registers
template <bool I8, int COLS, bool DEEP, int PRODUCT, typename Out, bool RUNS>
__global__ void __launch_bounds__(kThreads, COLS == 256 || DEEP ? 1 : 2)
harp_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                 const __grid_constant__ CUtensorMap map_b_small, const Params P) {
    constexpr int BLOCK = I8 ? 128 : 64;                     // contracted elements a stage
    constexpr int CG = COLS == 256 ? 2 : 1;                  // CTAs a tile
    constexpr int STAGES = stages(COLS, DEEP), kStage = stage_bytes(COLS);
    constexpr bool A_MN = PRODUCT != FORWARD, B_MN = PRODUCT == GRAD_WEIGHTS;
    constexpr int RUN = RUNS ? kRun : 1 << 30;
    constexpr uint32_t COLUMNS = 2 * COLS, ACC = COLS;       // two accumulators

    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[4 * STAGES + 6];
    __shared__ __align__(16) float s_scale[8][32];           // rows' scales of a chunk of columns, by epilogue warp
    __shared__ uint32_t s_columns;
    __shared__ int s_dead;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();                    // 0 without a cluster
    const int size = CG == 2 ? 2 : P.split;                  // CTAs a cluster
    const int cluster = blockIdx.x / size, clusters = gridDim.x / size;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char *const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t sums = base + STAGES * kStage;            // the other ranks' accumulators (split > 1)
    int *const off = reinterpret_cast<int *>(base_ptr + STAGES * kStage + (CG == 2 ? kTurnBytes : P.split > 1 ? kSumCols * 512 : 0));
    int *const first = off + P.n_groups + 1;

    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int s) { return bar0 + 8u * s; };                        // a stage has arrived (of a pair: both halves, in the first CTA)
    auto empty = [&](int s) { return bar0 + 8u * (STAGES + s); };            // a stage has been multiplied
    auto done = [&](int a) { return bar0 + 8u * (2 * STAGES + a); };         // an accumulator is complete
    auto taken = [&](int a) { return bar0 + 8u * (2 * STAGES + 2 + a); };    // ... has been read
    const uint32_t sums_full = bar0 + 8u * (2 * STAGES + 4), sums_free = bar0 + 8u * (2 * STAGES + 5);
    // one of either a stage: with few blocks a tile the copies are several ragged blocks ahead
    auto ragged = [&](int s) { return bar0 + 8u * (2 * STAGES + 6 + s); };   // this CTA's half of a ragged last block has arrived
    auto cleared = [&](int s) { return bar0 + 8u * (3 * STAGES + 6 + s); };  // ... and the second CTA's is clean

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
            mbar_init(ragged(s), 1);
            mbar_init(cleared(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(done(a), 1);
            mbar_init(taken(a), 8 * CG);
        }
        mbar_init(sums_full, 1);
        mbar_init(sums_free, 8 * P.split);
        mbar_init_fence();
        s_dead = 0;
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        prefetch_map(&map_b_small);
    }
    if (warp == 2) alloc_columns<CG, COLUMNS>(smem_u32(&s_columns));
    // offsets made to rise and to stay within the batch, and the number of tiles before each group
    auto lay_out = [&] {
        int before = 0, tiles = 0;
        for (int e0 = 0; e0 <= P.n_groups; e0 += 32) {
            const int e = e0 + lane;
            int o = P.offsets == nullptr ? (e == 0 ? 0 : P.n_rows) : e <= P.n_groups ? P.offsets[e] : P.n_rows;
            o = min(max(o, 0), P.n_rows);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int v = __shfl_up_sync(~0u, o, d);
                if (lane >= d) o = max(o, v);
            }
            o = max(o, before);
            int prev = __shfl_up_sync(~0u, o, 1);
            if (lane == 0) prev = before;
            int n = 0;                                        // tiles of group e - 1
            if (e > 0 && e <= P.n_groups && PRODUCT != GRAD_WEIGHTS && o > prev)
                n = div_up(P.lanes, 128 * CG) * div_up(o - prev, even_cols<CG>(o - prev, P.tile_cols));
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int v = __shfl_up_sync(~0u, n, d);
                if (lane >= d) n += v;
            }
            if (e <= P.n_groups) {
                off[e] = o;
                first[e] = tiles + n;
            }
            before = __shfl_sync(~0u, o, 31);
            tiles += __shfl_sync(~0u, n, 31);
        }
    };
    if (warp == 3 && P.offsets == nullptr) lay_out();
    tc_fence_before();
    if (size > 1) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    wait_for_previous();
    launch_dependents();
    if (P.offsets) {
        if (warp == 3) lay_out();
        __syncthreads();
    }

    const uint32_t columns = s_columns;
    const Waiter wait{&s_dead, P.err};
    const int n_tiles = PRODUCT == GRAD_WEIGHTS ? P.n_groups * div_up(P.lanes, 128 * CG) * div_up(P.cols, P.tile_cols) : first[P.n_groups];
    using Tiles = Walk<CG, PRODUCT, BLOCK>;
    // this CTA's share of the blocks
    auto from = [&](const Tile &T) { return CG == 2 ? 0 : (int)((int64_t)T.blocks * (int)rank / P.split); };
    auto to = [&](const Tile &T) { return CG == 2 ? T.blocks : (int)((int64_t)T.blocks * ((int)rank + 1) / P.split); };
    auto width = [&](const Tile &T) { return round_up(T.cols, CG == 2 ? 32 : 16); };     // columns of the instruction
    auto is_ragged = [&](const Tile &T, int b) { return PRODUCT == GRAD_WEIGHTS && b == T.blocks - 1 && T.tail % 16 != 0; };

    if (warp == 0 && lane == 0) {
        Tiles tiles(P, off, first);
        Ring<STAGES> ring;
        bool alive = true;
        for (int t = cluster; alive && t < n_tiles; t += clusters) {
            const Tile T = tiles.at(t);
            const int half = width(T) / CG;                  // columns of this CTA
            const int lane0 = T.lane0 + (CG == 2 ? (int)rank * 128 : 0), col0 = CG == 2 ? (int)rank * half : 0;
            // rows along the columns: one copy of 128 of them, or copies of 32
            const bool one = B_MN || (CG == 2 && half > 32);
            const int boxes = B_MN ? div_up(half, 64) : one ? 1 : div_up(half, 32);
            const uint32_t bytes = kHalf + (B_MN ? (uint32_t)boxes * 8192u : one ? 16384u : (uint32_t)boxes * 4096u);
            const int b1 = to(T);
            for (int b = from(T); b < b1; ++b, ring.next()) {
                const int s = ring.s;
                if (!wait(empty(s), ring.phase ^ 1, 1)) { alive = false; break; }
                const uint32_t a = base + (uint32_t)s * kStage, bb = a + kHalf;
                uint32_t bar = full(s);
                if (is_ragged(T, b)) mbar_expect_tx(bar = ragged(s), bytes);
                else if (CG == 1) mbar_expect_tx(bar, bytes);
                else if (rank == 0) mbar_expect_tx(bar, 2 * bytes);
                else bar = map_rank(bar, 0);
                const int k = b * BLOCK;
                if (PRODUCT == FORWARD) load_3d<CG>(a, &map_a, k, lane0, T.e, bar);
                else if (PRODUCT == GRAD_ROWS && P.chunked_a) load_4d<CG>(a, &map_a, 0, k, lane0 / 64, T.e, bar);
                else if (PRODUCT == GRAD_ROWS) {
                    load_3d<CG>(a, &map_a, lane0, k, T.e, bar);
                    load_3d<CG>(a + 8192, &map_a, lane0 + 64, k, T.e, bar);
                } else if (P.chunked_a) load_3d<CG>(a, &map_a, 0, T.row0 + k, lane0 / 64, bar);
                else {
                    load_2d<CG>(a, &map_a, lane0, T.row0 + k, bar);
                    load_2d<CG>(a + 8192, &map_a, lane0 + 64, T.row0 + k, bar);
                }
                if (B_MN && P.chunked_b && half == 128) load_3d<CG>(bb, &map_b, 0, T.row0 + k, (T.col0 + col0) / 64, bar);
                else if (B_MN) {
                    for (int i = 0; i < boxes; ++i) load_2d<CG>(bb + i * 8192, &map_b_small, T.col0 + col0 + i * 64, T.row0 + k, bar);
                } else if (one) load_2d<CG>(bb, &map_b, k, T.row0 + col0, bar);
                else
                    for (int i = 0; i < boxes; ++i) load_2d<CG>(bb + i * 4096, &map_b_small, k, T.row0 + col0 + i * 32, bar);
            }
        }
    } else if (warp == 1 && lane == 0 && (CG == 1 || rank == 0)) {
        Tiles tiles(P, off, first);
        Ring<STAGES> ring;
        int n = 0;
        bool alive = true;
        for (int t = cluster; alive && t < n_tiles; t += clusters) {
            const Tile T = tiles.at(t);
            const int b1 = to(T);
            const uint32_t idesc = instr(I8, A_MN, B_MN, 128 * CG, width(T));
            for (int b = from(T); alive && b < b1; ++n) {
                const int acc = n & 1, start = b, stop = min(b1, b + RUN);
                if (!wait(taken(acc), ((n >> 1) & 1) ^ 1, 2)) { alive = false; break; }
                tc_fence_after();
                const uint32_t d = columns + acc * ACC;
                for (; b < stop; ++b, ring.next()) {
                    const int s = ring.s;
                    if (!wait(full(s), ring.phase, 3)) { alive = false; break; }
                    tc_fence_after();
                    const uint32_t a = base + (uint32_t)s * kStage;
                    const uint64_t da = A_MN ? operand(a, 8192, 1024) : operand(a, 16, 1024);
                    const uint64_t db = B_MN ? operand(a + kHalf, 8192, 1024) : operand(a + kHalf, 16, 1024);
                    constexpr uint64_t step_a = A_MN ? 128 : 2, step_b = B_MN ? 128 : 2;
                    if (PRODUCT == GRAD_WEIGHTS && b == T.blocks - 1) {
                        for (int k = 0; k < div_up(T.tail, 16); ++k) mma_ss<I8, CG>(d, da + step_a * k, db + step_b * k, idesc, b > start || k > 0);
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma_ss<I8, CG>(d, da + step_a * k, db + step_b * k, idesc, b > start || k > 0);
                    }
                    commit<CG>(empty(s));
                }
                if (alive) commit<CG>(done(acc));
            }
        }
    } else if ((warp == 2 || warp == 3) && PRODUCT == GRAD_WEIGHTS) {
        // The other groups' rows of a ragged last block.  One takes some 2800 cycles (stores, the fence to the asynchronous side, the
        // release to the other CTA), a short tile's stores 2500: two warps take one for even stages, one for odd ones (not blocks in turn:
        // a warp that waits for a stage's phase after the next one finds the one before that, and goes on at once).
        Tiles tiles(P, off, first);
        Ring<STAGES> ring;
        uint32_t phases = 0;                                 // a bit a stage: its next ragged block's phase
        for (int t = cluster; t < n_tiles; t += clusters) {
            const Tile T = tiles.at(t);
            if (T.blocks <= 0) continue;
            ring.skip(T.blocks - 1);
            if (is_ragged(T, T.blocks - 1)) {
                if ((ring.s ^ warp) & 1) {
                    ring.next();
                    continue;
                }
                const uint32_t phase = phases >> ring.s & 1;
                phases ^= 1u << ring.s;
                if (!wait(ragged(ring.s), phase, 4)) break;
                const int chunks = 2 + div_up(width(T) / CG, 64);    // of 64 lanes or columns, 64 rows of 128 bytes each
                unsigned char *const stage = base_ptr + ring.s * kStage + (lane & 7) * 16;
                for (int c = 0; c < chunks; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {                    // four rows at a time
                        const int r = (T.tail & ~15) + i * 4 + (lane >> 3);
                        if (r >= T.tail) *reinterpret_cast<uint4 *>(stage + c * 8192 + r * 128) = make_uint4(0, 0, 0, 0);
                    }
                fence_async_smem();
                __syncwarp();
                if (CG == 2 && rank == 1) {
                    if (lane == 0) mbar_arrive_cluster(map_rank(cleared(ring.s), 0));
                } else {
                    if (CG == 2 && !wait.cluster(cleared(ring.s), phase, 8)) break;
                    if (lane == 0) mbar_arrive(full(ring.s));
                }
            }
            ring.next();
        }
    } else if (warp >= 4) {
        const int q = warp & 3, part = (warp - 4) >> 2;      // lanes 32 q .. 32 q + 31; chunks of 32 columns alternate between the two warps
        Tiles tiles(P, off, first);
        int n = 0;
        uint32_t sums_phase = 0;
        bool alive = true;
        for (int t = cluster; t < n_tiles; t += clusters) {
            const Tile T = tiles.at(t);
            const int l = T.lane0 + (CG == 2 ? (int)rank * 128 : 0) + q * 32 + lane;
            const bool inside = l < P.lanes;
            Out *const out = static_cast<Out *>(P.out) +
                (PRODUCT == GRAD_WEIGHTS ? T.e * P.group_out + (int64_t)T.col0 * P.ld_out : (int64_t)T.row0 * P.ld_out) + l;
            const float by_lane = I8 && inside ? P.channel_scale[(int64_t)T.e * P.lanes + l] : 1.0f;
            if (PRODUCT == GRAD_WEIGHTS && T.blocks < 0) continue;
            if (T.blocks == 0) {                             // a group without rows
                if (inside && !P.accumulate)
                    for (int c = part; c < T.cols; c += 2) store(out + (int64_t)c * P.ld_out, 0.0f);
                continue;
            }
            const int blocks = to(T) - from(T);
            const bool any = blocks > 0;                     // ranks of a split may have none
            // 8 bits: the rows' scales of this warp's next chunk, one a lane
            auto row_scale_of = [&](int c) { return I8 && c < T.cols ? P.row_scale[T.row0 + c] : 0.0f; };
            float by_row = row_scale_of(part * 32 + lane);
            const int w = width(T);
            const bool whole = CG == 2 || P.split == 1;
            // the accumulator that is to be read next; and what it takes to hand it back
            auto accumulator = [&] { return columns + (n & 1) * ACC + ((uint32_t)q << 21); };
            auto arrived = [&] {
                if (!wait(done(n & 1), (n >> 1) & 1, 5)) return false;
                tc_fence_after();
                return true;
            };
            auto hand_back = [&] {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_at(CG == 2 ? map_rank(taken(n & 1), 0) : taken(n & 1));
                ++n;
            };
            constexpr int CHUNKS = COLS / 64 ? COLS / 64 : 1;        // of 32 columns, of this warp
            // this warp's columns: chunks of 32, or of 16 out of 32 where sums are divided among ranks
            float held[RUNS ? (COLS == 256 ? 128 : 32) : 1];
            if (RUNS) {
#pragma unroll
                for (int i = 0; i < (int)(sizeof held / sizeof held[0]); ++i) held[i] = 0.0f;
                for (int r = 0; r < blocks; r += RUN) {
                    if (!arrived()) { alive = false; break; }
#pragma unroll
                    for (int i = 0; i < (int)(sizeof held / sizeof held[0]) / 16; ++i) {
                        const int c0 = whole ? (i & ~1) * 32 + part * 32 + (i & 1) * 16 : i * 32 + part * 16;
                        if (c0 < w) {
                            uint32_t v[16];
                            tmem_ld16(accumulator() + c0, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) held[i * 16 + j] += __uint_as_float(v[j]);
                        }
                    }
                    hand_back();
                }
                if (!alive) break;
            } else if (any && !arrived()) break;
            const uint32_t d = accumulator();
            if (CG == 2 && sizeof(Out) == 2 && !RUNS && P.eights) {
                // Results as mma.sync's fragments, pairs of columns packed, turned round in shared memory: eight lanes of a column are 16 bytes there.
                // A third of the instructions that storing lane by lane takes (8 bits, 16384 x 4096 x 14336 655 -> 619 us in
                // short bursts; 690 in a long run, at the power limit).
                unsigned char *const turn = base_ptr + STAGES * kStage + (warp - 4) * 2048;      // 32 columns of 64 bytes
                const uint32_t turn_s = smem_u32(turn);
                auto place = [](int c, int eight) { return c * 64 + ((eight ^ (c >> 1 & 3)) << 4); };
                float by_lanes[4];                           // 8 bits: scales of lanes lane / 4 + 8 h
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const int ch = T.lane0 + (int)rank * 128 + q * 32 + h * 8 + (lane >> 2);
                    by_lanes[h] = I8 && ch < P.lanes ? P.channel_scale[(int64_t)T.e * P.lanes + ch] : 0.0f;
                }
                const bool eight_inside = T.lane0 + (int)rank * 128 + q * 32 + (lane & 3) * 8 < P.lanes;
                Out *const to = out - lane + (lane & 3) * 8 + (int64_t)(lane >> 2) * P.ld_out;
#pragma unroll 1
                for (int c0 = part * 32; c0 < w; c0 += 64) {
                    uint32_t v[2][16];
                    load_fragments(d + c0, v[0]);
                    load_fragments(d + (16u << 16) + c0, v[1]);
                    __syncwarp();                            // what was turned round before has been read
                    if (I8) s_scale[warp - 4][lane] = by_row;
                    if (I8) __syncwarp();
                    if (I8) by_row = row_scale_of(c0 + 64 + lane);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 4; j += 2) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {        // lanes 16 k .. 16 k + 15
                            uint32_t tiles[4];
#pragma unroll
                            for (int m = 0; m < 4; ++m) {    // eight columns, eight lanes
                                const int jj = j + m / 2, h = m & 1;
                                uint32_t lo = v[k][4 * jj + 2 * h], hi = v[k][4 * jj + 2 * h + 1];
                                if (I8) {
                                    const float2 r = *reinterpret_cast<const float2 *>(&s_scale[warp - 4][8 * jj + 2 * (lane & 3)]);
                                    lo = __float_as_uint((float)(int32_t)lo * by_lanes[2 * k + h] * r.x);
                                    hi = __float_as_uint((float)(int32_t)hi * by_lanes[2 * k + h] * r.y);
                                }
                                tiles[m] = pack_bf16(lo, hi);
                            }
                            const int c = 8 * (j + (lane >> 4)) + (lane & 7);
                            store_transposed(turn_s + place(c, 2 * k + (lane >> 3 & 1)), tiles[0], tiles[1], tiles[2], tiles[3]);
                        }
                    }
                    __syncwarp();
                    Out *p = to + (int64_t)c0 * P.ld_out;
#pragma unroll
                    for (int i = 0; i < 4; ++i, p += 8 * P.ld_out) {
                        const int c = i * 8 + (lane >> 2);
                        const uint4 eight = *reinterpret_cast<const uint4 *>(turn + place(c, lane & 3));
                        if (eight_inside && c0 + c < T.cols) *reinterpret_cast<uint4 *>(p) = eight;
                    }
                }
            } else if (whole) {
                const bool pairs = sizeof(Out) == 2 && P.pairs;
                // (unrolled only where registers are indexed: four copies of the body missed the instruction cache: bf16 weight gradients of 32 groups
                // of 31 rows, 2048 x 4096, 145 us, 118 without)
#pragma unroll (RUNS ? CHUNKS : 1)
                for (int i = 0; i < CHUNKS; ++i) {
                    const int c0 = (2 * i + part) * 32;
                    if (c0 >= w) break;
                    uint32_t v[32];
                    if (RUNS) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(held[(i * 32 + j) % (sizeof held / sizeof held[0])]);
                    } else tmem_ld32(d + c0, v);
                    if (I8) {
                        __syncwarp();
                        s_scale[warp - 4][lane] = by_row;
                        __syncwarp();
                    }
                    if (I8) by_row = row_scale_of(c0 + 64 + lane);
                    if (!RUNS) tmem_wait_ld();
                    if (I8) {
                        const float4 *const scale = reinterpret_cast<const float4 *>(s_scale[warp - 4]);
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 r = scale[j / 4];
                            v[j] = __float_as_uint((float)(int32_t)v[j] * by_lane * r.x);
                            v[j + 1] = __float_as_uint((float)(int32_t)v[j + 1] * by_lane * r.y);
                            v[j + 2] = __float_as_uint((float)(int32_t)v[j + 2] * by_lane * r.z);
                            v[j + 3] = __float_as_uint((float)(int32_t)v[j + 3] * by_lane * r.w);
                        }
                    }
                    // A whole chunk goes without a test a column: with one, 18 instructions a store kept 64 x 128 rows, 2048 x 1024
                    // (fp32 weight gradients) at 259 us, 117 now.
                    const int left = T.cols - c0;
                    if (pairs) {
                        // neighbouring lanes trade halves of two columns: either then stores both lanes' elements of one
                        const int odd = lane & 1;
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const uint32_t got = __shfl_xor_sync(~0u, odd ? v[j] : v[j + 1], 1);
                            v[j] = pack_bf16(odd ? got : v[j], odd ? v[j + 1] : got);
                        }
                        if (inside) {
                            Out *p = out - odd + (int64_t)(c0 + odd) * P.ld_out;
                            const int64_t step = 2 * P.ld_out;
                            if (left >= 32) {
#pragma unroll
                                for (int j = 0; j < 32; j += 2, p += step) *reinterpret_cast<uint32_t *>(p) = v[j];
                            } else {
#pragma unroll
                                for (int j = 0; j < 32; j += 2, p += step)
                                    if (j + odd < left) *reinterpret_cast<uint32_t *>(p) = v[j];
                            }
                        }
                    } else if (inside) {
                        Out *p = out + (int64_t)c0 * P.ld_out;
                        if (PRODUCT == GRAD_WEIGHTS && P.accumulate) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j < left) v[j] = __float_as_uint(__uint_as_float(v[j]) + load(p + (int64_t)j * P.ld_out));
                        }
                        if (left >= 32) {
#pragma unroll
                            for (int j = 0; j < 32; ++j, p += P.ld_out) store(p, __uint_as_float(v[j]));
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j, p += P.ld_out)
                                if (j < left) store(p, __uint_as_float(v[j]));
                        }
                    }
                }
            } else {
                // 32 columns at a time, dealt out to the ranks in runs of 4 to 16; sums[source][four columns of the run][lane][4]
#pragma unroll
                for (int i = 0; i < COLS / kSumCols; ++i) {
                    const int h = i * kSumCols;
                    if (h >= w) break;
                    const int run = min(w - h, kSumCols) / P.split, shift = 31 - __clz(run);       // powers of two, as 16, 32 and the split are
                    if (threadIdx.x == 128) mbar_expect_tx(sums_full, (uint32_t)(P.split * run * 512));
                    if (!wait(sums_free, sums_phase ^ 1, 6)) { alive = false; break; }
                    const int c0 = h + part * 16;
                    if (c0 < w) {
                        uint32_t v[16];
                        if (RUNS) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(held[(i * 16 + j) % (sizeof held / sizeof held[0])]);
                        } else if (any) {
                            tmem_ld16(d + c0, v);
                            tmem_wait_ld();
                        }
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const int to_rank = (part * 16 + j) >> shift, c = (part * 16 + j) & (run - 1);
                            const uint32_t place = sums + (uint32_t)(((((int)rank * run + c) >> 2) * 128 + q * 32 + lane) * 16);
                            send16(map_rank(place, to_rank), any ? v[j] : 0u, any ? v[j + 1] : 0u, any ? v[j + 2] : 0u, any ? v[j + 3] : 0u,
                                   map_rank(sums_full, to_rank));
                        }
                    }
                    if (!wait.cluster(sums_full, sums_phase, 7)) { alive = false; break; }
                    const uint4 *const mine = reinterpret_cast<const uint4 *>(base_ptr + STAGES * kStage) + q * 32 + lane;
                    float x[2][4];                           // this warp's columns: every other four of at most sixteen
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const int c = (2 * g + part) * 4;
                        if (c < run) {
                            uint4 sum = make_uint4(0, 0, 0, 0);
                            for (int r = 0; r < P.split; ++r) {
                                const uint4 s = mine[((r * run + c) >> 2) * 128];
                                if (I8) sum.x += s.x, sum.y += s.y, sum.z += s.z, sum.w += s.w;
                                else sum.x = add(sum.x, s.x), sum.y = add(sum.y, s.y), sum.z = add(sum.z, s.z), sum.w = add(sum.w, s.w);
                            }
                            x[g][0] = I8 ? (float)(int32_t)sum.x : __uint_as_float(sum.x);
                            x[g][1] = I8 ? (float)(int32_t)sum.y : __uint_as_float(sum.y);
                            x[g][2] = I8 ? (float)(int32_t)sum.z : __uint_as_float(sum.z);
                            x[g][3] = I8 ? (float)(int32_t)sum.w : __uint_as_float(sum.w);
                        }
                    }
                    __syncwarp();
                    if (lane < P.split) mbar_arrive_at(map_rank(sums_free, lane));
#pragma unroll
                    for (int g = 0; g < 2; ++g)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int c = (2 * g + part) * 4 + j, col = h + (int)rank * run + c;
                            if (inside && c < run && col < T.cols)
                                store(out + (int64_t)col * P.ld_out, I8 ? x[g][j] * by_lane * P.row_scale[T.row0 + col] : x[g][j]);
                        }
                    sums_phase ^= 1;
                }
                if (!alive) break;
            }
            if (!RUNS && any) hand_back();
        }
    }
    __syncwarp();
    // (the thread whose wait gave up reads what it has written itself)
    for (int r = 0; *wait.dead && r < size; ++r) store_at(map_rank(smem_u32(&s_dead), r), 1);
    __syncwarp();
    tc_fence_before();
    if (size > 1) cluster_sync();                            // the others' barriers and memory stay until all are done
    else __syncthreads();
    if (*wait.dead) {
        // A wait gave up, as all CTAs of the cluster know by now.  Copies, products and sums that were on their way count at barriers of either CTA that
        // nobody need have armed, so no barrier tells when they have landed; they take microseconds.  All stay 10 ms longer with the memory that they go to.
        const long long start = clock64();
        for (int i = 0; threadIdx.x == 0 && i < 1 << 16 && clock64() - start < 20000000; ++i) __nanosleep(1000);
        __syncwarp();
        if (size > 1) cluster_sync();
        else __syncthreads();
    }
    if (warp == 2) {
        tc_fence_after();
        free_columns<CG, COLUMNS>(columns);
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool encode(CUtensorMap *map, bool i8, const void *ptr, int rank, const int64_t *extent, const int64_t *pitch, const int *box) {
    cuuint64_t dims[4], strides[3];
    cuuint32_t b[4], ones[4] = {1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) {
        dims[i] = (cuuint64_t)extent[i];
        b[i] = (cuuint32_t)box[i];
        if (i + 1 < rank) strides[i] = (cuuint64_t)pitch[i];
    }
    return reinterpret_cast<EncodeTiledFn>(harp_tensor_map_encoder(nullptr))(
               map, i8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void *>(ptr), dims,
               strides, b, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int smem_bytes(int cols, bool deep, int split, int n_groups) {
    return 1024 + stages(cols, deep) * stage_bytes(cols) + (cols == 256 ? kTurnBytes : split > 1 ? kSumCols * 512 : 0) + 8 * (n_groups + 1);
}

template <bool I8, int COLS, bool DEEP, int PRODUCT, typename Out, bool RUNS>
harp_status_t launch(const CUtensorMap (&maps)[3], const Params &P, int clusters, cudaStream_t s) {
    const auto kernel = harp_gemm_kernel<I8, COLS, DEEP, PRODUCT, Out, RUNS>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) != cudaSuccess) {
        cudaGetLastError();
        return HARP_ERR_CUDA;
    }
    const int size = COLS == 256 ? 2 : P.split;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(clusters * size));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem_bytes(COLS, DEEP, P.split, P.n_groups);
    cfg.stream = s;
    cudaLaunchAttribute la[2];
    la[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    la[0].val.programmaticStreamSerializationAllowed = 1;
    la[1].id = cudaLaunchAttributeClusterDimension;
    la[1].val.clusterDim.x = (unsigned)size;
    la[1].val.clusterDim.y = la[1].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = 2;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, maps[0], maps[1], maps[2], P);
    g_harp_launches.fetch_add(1, std::memory_order_relaxed);
    if (err != cudaSuccess) {
        cudaGetLastError();
        return HARP_ERR_CUDA;
    }
    return HARP_OK;
}

template <bool I8, int COLS, bool DEEP, int PRODUCT>
harp_status_t launch(harp_dtype_t out, bool runs, const CUtensorMap (&maps)[3], const Params &P, int clusters, cudaStream_t s) {
    if (out == HARP_F32) return launch<I8, COLS, DEEP, PRODUCT, float, !I8>(maps, P, clusters, s);
    if constexpr (!I8)
        if (runs) return launch<I8, COLS, DEEP, PRODUCT, __nv_bfloat16, true>(maps, P, clusters, s);
    return launch<I8, COLS, DEEP, PRODUCT, __nv_bfloat16, false>(maps, P, clusters, s);
}

// How a call is cut: by pairs of CTAs on 256 lanes x 256 columns, or by single ones on 128 x 32 or 128 x 64 in clusters of `split`.
struct Shape {
    int cols, split, slots;              // slots: clusters (pairs) that run at once
    int64_t tiles;                       // at most
    bool deep;                           // the longer ring
};
struct Cut {
    int32_t cols = 0, split = 1, deep = 0;
};
thread_local Cut asked, taken;           // by harp_linear_set_cut; by the last call

int64_t lanes_of(const Call &c) { return c.product == FORWARD ? c.d_out : c.d_in; }
int64_t most_tiles(const Call &c, int cols) {
    const int64_t across = cols == 256 ? (lanes_of(c) + 255) / 256 : (lanes_of(c) + 127) / 128;
    return across * ((c.n_rows + cols - 1) / cols + c.n_groups - 1);
}

// The cut with the least estimated time: the weight's bytes at the rate of memory, stretched by a last round of tiles that leaves SMs
// idle, or rounds of tiles times their blocks of 128 contracted bytes.  Constants from 8-bit products of 1 to 2048 rows, widths 2048 to 28672,
// and 8 to 64 groups of 1 to 128 rows, each cut every way (us a call):
//                                pairs   32 cols, split 1, 2, 4   64 cols, split 1, 2, 4
//    16 rows, 14336 -> 4096       40.3    35.4   22.1   17.3       41.0   25.9   19.0
//    64 rows, 4096 -> 14336       15.5    16.8   19.4   20.5       18.9   19.1   18.4
//    64 rows, 8192 -> 28672       52.1    53.3   56.1   54.3       43.5   46.9   50.7
//   128 rows, 14336 -> 4096       36.1    36.3   25.0   26.3       43.8   28.9   21.7
//   256 rows, 14336 -> 4096       37.1    38.6   44.1   47.0       44.3   30.9   32.5
//   256 rows, 4096 -> 14336       17.4    45.4   56.1   84.1       30.1   35.8   44.1
//   8 x 16 rows, 4096 -> 14336   173.9   159.2  147.7  148.4      162.8  154.4  152.6     (bf16)
//   64 x 64 rows, 2048 -> 2048    55.1    61.7   72.6  116.7       54.7   62.6  100.8
Shape choose(const Call &c, const Device &dev) {
    const int64_t pair_tiles = (lanes_of(c) + 255) / 256, tiles = (lanes_of(c) + 127) / 128;
    if (c.product == GRAD_WEIGHTS) return {256, 1, dev.pairs, c.n_groups * pair_tiles * ((c.d_out + 255) / 256), false};
    if (asked.cols) {
        const int slots = asked.cols == 256 ? dev.pairs : dev.clusters[asked.split / 2];
        return {asked.cols, asked.split, slots, most_tiles(c, asked.cols), asked.deep != 0};
    }
    const Shape pairs = {256, 1, dev.pairs, most_tiles(c, 256), false};
    // rows of a group, and a quarter more where there are several: they are not even, but many fit a tile that the mean fits
    const int64_t met = std::min<int64_t>(c.n_groups, c.n_rows), even = (c.n_rows + met - 1) / met, rows = met > 1 ? even + even / 4 : even;
    const double blocks = (double)(((c.product == FORWARD ? c.d_in : c.d_out) * (c.i8 ? 1 : 2) + 127) / 128), memory = (double)(met * tiles) * blocks * 16384 / 6.3e6;     // us
    auto cols_of = [&](int most) { return (double)((rows + most - 1) / most); };
    Shape best = pairs;
    double least;
    {
        const double n = (double)(met * pair_tiles) * cols_of(256), rounds = std::ceil(n / dev.pairs);
        const double width = std::min<double>(256, (double)rows / cols_of(256));
        const double stretch = rounds > 1 ? rounds * dev.pairs / n : 1;
        least = std::max(memory * stretch, rounds * (blocks * (0.29 + 0.00037 * width) + 0.5)) + 4.5;
    }
    for (int cols = 32; cols <= 64; cols *= 2)
        for (int i = 0; i < 3; ++i) {
            const double n = (double)(met * tiles) * cols_of(cols), rounds = std::ceil(n / dev.clusters[i]);
            const double stretch = rounds > 1 ? 0.75 + 0.25 * rounds * dev.clusters[i] / n : 1;
            const double join = i ? (cols == 32 ? 2.5 : 6) : 0.5;        // adding up a tile's sums
            const double block = n * (1 << i) > dev.sms ? (cols == 32 ? 0.37 : 0.42) : (cols == 32 ? 0.285 : 0.36);
            const double t = std::max(memory * stretch + join, rounds * (blocks / (1 << i) * block + join)) + 3.5;
            if (t < least) {
                least = t;
                best = {cols, 1 << i, dev.clusters[i], most_tiles(c, cols), false};
            }
        }
    // All tiles at once and one CTA an SM at most: a longer ring (1 row, 4096 -> 14336 14.9 -> 14.0 us, 64 rows 17.7 -> 15.3 us; clusters on
    // 32 columns are better off with the next kernel's CTAs beside them, 1 row 4096 -> 4096 8.0 against 8.5 us).
    best.deep = best.cols < 256 && best.tiles * best.split <= dev.sms && best.tiles <= best.slots / 2 && (best.split == 1 || best.cols == 64);
    return best;
}

bool describe(int dev, Device &d) {
    void *err = nullptr;
    if (!harp_tensor_map_encoder(nullptr) || cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaGetSymbolAddress(&err, g_gemm_err) != cudaSuccess)
        return false;
    auto resident = [&](auto kernel, int cols, int size) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(d.sms / size * size));
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = (size_t)smem_bytes(cols, false, cols == 256 ? 1 : size, kMaxGroups);
        cudaLaunchAttribute la;
        la.id = cudaLaunchAttributeClusterDimension;
        la.val.clusterDim.x = (unsigned)size;
        la.val.clusterDim.y = la.val.clusterDim.z = 1;
        cfg.attrs = &la;
        cfg.numAttrs = 1;
        int n = 0;
        const bool ok = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem) == cudaSuccess &&
                        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess;
        return ok ? n : 0;
    };
    d.pairs = resident(harp_gemm_kernel<false, 256, false, FORWARD, __nv_bfloat16, false>, 256, 2);
    // (the query counts one CTA an SM wherever tensor memory is used; two of these fit, and run)
    for (int i = 0; i < 3; ++i) d.clusters[i] = 2 * resident(harp_gemm_kernel<false, 32, false, FORWARD, __nv_bfloat16, false>, 32, 1 << i);
    d.err = static_cast<int32_t *>(err);
    return d.pairs > 0 && d.clusters[0] > 0 && d.clusters[1] > 0 && d.clusters[2] > 0;
}

}  // namespace

const Device *device() {
    constexpr int kMost = 64;
    static Device table[kMost];
    static std::atomic<bool> known[kMost];
    static std::mutex mu;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMost) {
        cudaGetLastError();
        return nullptr;
    }
    if (known[dev].load(std::memory_order_acquire)) return &table[dev];
    std::lock_guard<std::mutex> lock(mu);
    if (known[dev].load(std::memory_order_relaxed)) return &table[dev];
    Device d;
    if (!describe(dev, d)) {             // asked again at the next call
        cudaGetLastError();
        return nullptr;
    }
    table[dev] = d;
    known[dev].store(true, std::memory_order_release);
    return &table[dev];
}

harp_status_t gemm(const Call &c, const Device &dev, cudaStream_t stream) {
    const int es = c.i8 ? 1 : 2;
    Params P = {};
    P.n_rows = (int32_t)c.n_rows;
    P.n_groups = c.n_groups;
    P.offsets = c.offsets;
    P.row_scale = c.row_scale;
    P.channel_scale = c.channel_scale;
    P.out = c.out;
    P.ld_out = c.ld_out;
    P.group_out = c.d_out * c.ld_out;
    P.accumulate = c.accumulate;
    P.err = dev.err;
    P.lanes = (int32_t)(c.product == FORWARD ? c.d_out : c.d_in);
    P.cols = (int32_t)c.d_out;
    P.depth = (int32_t)(c.product == FORWARD ? c.d_in : c.d_out);
    P.pairs = reinterpret_cast<uintptr_t>(c.out) % 4 == 0 && c.ld_out % 2 == 0 && P.lanes % 2 == 0 && !c.accumulate;
    P.eights = P.pairs && reinterpret_cast<uintptr_t>(c.out) % 16 == 0 && c.ld_out % 8 == 0 && P.lanes % 8 == 0;
    const Shape shape = choose(c, dev);
    taken = {shape.cols, shape.split, shape.deep};
    if (shape.tiles > INT32_MAX / 16) return HARP_ERR_TOO_LARGE;
    P.tile_cols = shape.cols;
    P.split = shape.split;
    const int clusters = (int)std::min<int64_t>(shape.tiles, shape.slots);

    // A matrix whose width is a multiple of 64 is also a stack of chunks 64 wide: one copy then brings two of them, which an MN-major
    // operand keeps one behind the other (weight gradients of 8192 rows, 8192 x 8192, two copies a stage instead of four: 897 -> 815 us)
    CUtensorMap maps[3];
    const int elems = 128 / es;
    bool ok;
    P.chunked_a = c.product != FORWARD && c.d_in % 64 == 0;
    P.chunked_b = c.product == GRAD_WEIGHTS && c.d_out % 64 == 0;
    if (c.product == GRAD_WEIGHTS) {
        const int64_t pa[2] = {c.ld_rows * es, 128}, pb[2] = {c.ld_other * es, 128};
        const int64_t ea[2] = {c.d_in, c.n_rows}, ea_chunks[3] = {64, c.n_rows, c.d_in / 64};
        const int64_t eb[2] = {c.d_out, c.n_rows}, eb_chunks[3] = {64, c.n_rows, c.d_out / 64};
        const int box[3] = {64, 64, 2};
        ok = P.chunked_a ? encode(&maps[0], false, c.rows, 3, ea_chunks, pa, box) : encode(&maps[0], false, c.rows, 2, ea, pa, box);
        ok = ok && encode(&maps[2], false, c.other, 2, eb, pb, box);
        if (P.chunked_b) ok = ok && encode(&maps[1], false, c.other, 3, eb_chunks, pb, box);
        else maps[1] = maps[2];
    } else {
        const int64_t group = c.ld_other * es * c.d_out;
        if (P.chunked_a) {
            const int64_t e[4] = {64, c.d_out, c.d_in / 64, c.n_groups}, p[3] = {c.ld_other * es, 128, group};
            const int box[4] = {64, 64, 2, 1};
            ok = encode(&maps[0], false, c.other, 4, e, p, box);
        } else {
            const int64_t e[3] = {c.d_in, c.d_out, c.n_groups}, p[2] = {c.ld_other * es, group};
            const int box[3] = {elems, c.product == FORWARD ? 128 : 64, 1};
            ok = encode(&maps[0], c.i8, c.other, 3, e, p, box);
        }
        const int64_t e[2] = {c.d_rows, c.n_rows}, p[1] = {c.ld_rows * es};
        const int box[2] = {elems, 128}, box_small[2] = {elems, 32};
        ok = ok && encode(&maps[1], c.i8, c.rows, 2, e, p, box) && encode(&maps[2], c.i8, c.rows, 2, e, p, box_small);
    }
    if (!ok) return HARP_ERR_UNSUPPORTED;
    auto by_cols = [&](auto i8, auto product) {
        constexpr bool I8 = decltype(i8)::value;
        constexpr int PRODUCT = decltype(product)::value;
        const bool runs = P.depth > kLone;
        if (shape.cols == 256) return launch<I8, 256, false, PRODUCT>(c.out_dtype, runs, maps, P, clusters, stream);
        if (shape.cols == 64)
            return shape.deep ? launch<I8, 64, true, PRODUCT>(c.out_dtype, runs, maps, P, clusters, stream) : launch<I8, 64, false, PRODUCT>(c.out_dtype, runs, maps, P, clusters, stream);
        return shape.deep ? launch<I8, 32, true, PRODUCT>(c.out_dtype, runs, maps, P, clusters, stream) : launch<I8, 32, false, PRODUCT>(c.out_dtype, runs, maps, P, clusters, stream);
    };
    if (c.product == GRAD_WEIGHTS) {
        // only the GPU knows how long the groups are: where one may be too long for a single run, a launch for either kind
        P.above = -1;
        P.most = INT32_MAX;
        const bool two = c.out_dtype == HARP_BF16 && P.n_rows > kLone;
        if (two) P.most = kLone;
        const harp_status_t st = launch<false, 256, false, GRAD_WEIGHTS>(c.out_dtype, false, maps, P, clusters, stream);
        if (!two || st != HARP_OK) return st;
        P.above = kLone;
        P.most = INT32_MAX;
        return launch<false, 256, false, GRAD_WEIGHTS>(c.out_dtype, true, maps, P, clusters, stream);
    }
    if (c.product == GRAD_ROWS) return by_cols(std::false_type(), std::integral_constant<int, GRAD_ROWS>());
    return c.i8 ? by_cols(std::true_type(), std::integral_constant<int, FORWARD>()) : by_cols(std::false_type(), std::integral_constant<int, FORWARD>());
}

}  // namespace harp_linear

extern "C" harp_status_t harp_linear_set_cut(int32_t cols, int32_t split, int32_t deep) {
    const bool pairs = cols == 256 && split == 1 && deep == 0;
    const bool single = (cols == 32 || cols == 64) && (split == 1 || split == 2 || split == 4) &&
                        (deep == 0 || (deep == 1 && (split == 1 || cols == 64)));
    if (cols != 0 && !pairs && !single) return HARP_ERR_BAD_DIM;
    harp_linear::asked = {cols, split, deep};
    return HARP_OK;
}
extern "C" void harp_linear_last_cut(int32_t cut[3]) {
    cut[0] = harp_linear::taken.cols;
    cut[1] = harp_linear::taken.split;
    cut[2] = harp_linear::taken.deep;
}
