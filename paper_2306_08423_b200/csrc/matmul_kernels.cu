// Matrix products of the layer operators on the tensor cores, with their epilogues.
//
//   out[m][n] = epilogue( sum over k of a[m][k] b[n][k] ),   16-bit operands, 32-bit sums.
//
// Two kernels:
//
// pair_product_kernel   a persistent pair of blocks (two SMs) per 256 x 256 tile.  Per step of 64
//   reduction indices each block loads its 128 rows of a and its half of b's 256 rows with tiled
//   copies into a ring of stages; one thread of the pair's first block issues the products of both
//   (each SM multiplies its 128 rows of a with all 256 rows of b and reads half of b from its
//   neighbour, which halves the shared-memory traffic of b).  Accumulators: 128 lanes x 256 columns
//   of tensor memory, twice, so that the epilogue of a tile runs beside the products of the next.
//   Eight epilogue warps take 32 lanes x 128 columns each, through two 4 KB buffers of their own:
//   tiled copies bring residuals (activations to differentiate) in and results out, so every global
//   access is a full line whatever the lane layout, and ragged edges are clipped by the copy engine.
//
// split_product_kernel  for products with too few tiles to fill the device (few rows, or a small
//   weight gradient over many tokens): the same tile and products, once, whose reduction is split
//   over the 1, 2 or 4 pairs of a cluster.  Every block leaves its 32-bit partial rows in its shared
//   memory, and each sums a share of them over all pairs (in rank order: the result does not depend
//   on timing) and finishes it with plain row-wise loads and stores of any alignment.
//
// few_rows_kernel  for at most 64 rows of a (tokens): the other way round - 256 rows of the weight are
//   the tensor core's rows and the tokens its 16 to 64 columns, so that a step costs what the tokens
//   are worth (the tile above takes 0.27 us a step whatever part of it is real) and shared memory
//   holds little but the weight's stream.  The reduction is split like the split kernel's.
//
// Measured on several chips (bf16, of the 1669 TFLOP/s of a library product measured alone; the clock falls
// under the power limit): persistent, 8192 x 6144 -> 12288 with residual 800 to 972 us (76 to 92 %), 8192 x 1024 ->
// 4096 57 us, with gelu and its argument kept 67 to 81 us (the epilogue of 16 steps' tile is longer than the steps);
// gated block of 8192 tokens, 2048 x 8192, 590 to 700 us; split, 512 x 4096 -> 1024 14.5 us; few rows, 1 x 4096 -> 1024 5
// us, 7 tokens through a gated block of 2048 x 8192 28 us (100 MB of weights).  Small ones are bound by the fill of
// the ring, the exchange and the last rows, large ones by the tensor pipe, short reductions by the epilogue.
//
// Operands whose rows run over the reduction index and operands whose rows run over the output
// index are both read as they lie in memory (the tensor core takes either order), so no weight
// or activation is ever transposed.
#include <type_traits>

#include <cuda.h>

#include "activations.cuh"
#include "operators.h"
#include "tensor_core.cuh"

namespace distsim {

namespace {

constexpr int kStepBytes = 128;                  // reduction indices per step: 64 of 16 bits
constexpr int kOperandBytes = 128 * kStepBytes;  // one operand's 128 rows of a step
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kPairStages = 5;
constexpr int kSplitStages = 6;
constexpr int kEpiBytes = 4096;                  // one buffer of an epilogue warp: 32 rows of 128 bytes
constexpr int kPairThreads = 128 + 8 * 32;
constexpr int kSplitThreads = 64 + 8 * 32;
constexpr int kRowsAhead = 4;                    // rows of a partial tile that a warp sums at a time
constexpr int kPartialPitch = 260;               // floats per row of a partial tile (no bank conflicts)

// The tensor core cuts off what its 32-bit sums cannot hold, always towards zero: a sum of k terms
// shrinks by 9e-10 k of itself (measured: 4.7e-7 after 512 terms, 5e-5 after 32768).  Outputs of 16
// bits do not show it.  For 32-bit ones (gradients) the reduction goes in pieces of 1024 terms, and
// the epilogue's warps add each piece to a running sum, to nearest, that waits in the other half of
// tensor memory: 1e-6 at any length, for about 0.6 us a piece in which the products wait (a
// 4096 x 1024 gradient over 8192 tokens: 54 us in one piece).
constexpr int kPieceSteps = 16;

struct alignas(64) ProductParams {
    CUtensorMap a[2], b[2];
    CUtensorMap out[3], in[2];
    int32_t m, n;
    int32_t steps[2];                            // 64-wide reduction steps of the two operand pairs
    int32_t tiles_m, tiles_n, groups;
    int32_t a_mn, b_mn;
    uint32_t idesc;
    int32_t act;
    int32_t has_in, has_out1;
    const void *bias[2];
    int32_t *status;
    int32_t polls;                               // of a wait, before it gives up
    // split kernel only: pairs that share a tile, plain pointers
    int32_t split;
    int32_t few;                                 // few-rows kernel: columns the tokens take, 16 to 64
    const void *in_p[2];
    void *out_p[3];
    int64_t in_ld[2], out_ld[3];
    float *sums[2];                              // kEpiGatedBack: see Product::sums
    int64_t sums_ld;
};

__device__ __forceinline__ void give_up(int32_t *status) { *reinterpret_cast<volatile int32_t *>(status) = DISTSIM_E_TIMEOUT; }

// By a producer behind its last load (of `loads` so far): until every stage has been consumed, so that
// nothing arrives at the block's barriers or memory once it has left.  A producer that gave up, or does so
// here, waits as long as copies could take: some of them report to the other block's barriers.
template <int STAGES>
__device__ __forceinline__ bool consumed(const uint64_t (&empty)[STAGES], int loads, bool ok, const ProductParams &p)
{
    for (int i = max(0, loads - STAGES); i < loads && ok; ++i) ok = mbar_wait(smem_addr(&empty[i % STAGES]), (i / STAGES) & 1, p.polls);
    if (!ok) {
        give_up(p.status);
        for (int i = max(0, loads - STAGES); i < loads; ++i) mbar_wait(smem_addr(&empty[i % STAGES]), (i / STAGES) & 1, kDrainPolls);
    }
    return ok;
}
// By the thread that issues products, behind the last one: until all of them are done.
__device__ __forceinline__ bool products_done(uint64_t &drain, uint16_t own, bool ok, const ProductParams &p)
{
    tensor_commit(smem_addr(&drain), own);
    if (ok) ok = mbar_wait(smem_addr(&drain), 0, p.polls);
    if (!ok) {
        give_up(p.status);
        mbar_wait(smem_addr(&drain), 0, kDrainPolls);
    }
    return ok;
}

// Tile index -> (group, tile row, tile column): bands of 8 tile rows, rows fastest, so that the
// tiles in flight at a time share both operands in L2.
__device__ __forceinline__ void tile_coords(const ProductParams &p, int tile, int &group, int &tm, int &tn)
{
    constexpr int kBand = 8;
    const int per_group = p.tiles_m * p.tiles_n;
    group = tile / per_group;
    tile -= group * per_group;
    const int band = tile / (kBand * p.tiles_n);
    const int first = band * kBand;
    const int rows = min(kBand, p.tiles_m - first);
    tile -= band * kBand * p.tiles_n;
    tn = tile / rows;
    tm = first + tile - tn * rows;
}

// ------------------------------------------------------------------------------ pair kernel

// Position of 16-byte chunk c of row r in a buffer of 128-byte rows with the copies' 128-byte swizzle.
__device__ __forceinline__ uint32_t swizzled(uint32_t buf, int r, int c) { return buf + r * 128 + ((c ^ (r & 7)) << 4); }

__device__ __forceinline__ uint4 shared_load(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void shared_store(uint32_t a, uint4 v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" :: "r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

template <class T>
__device__ __forceinline__ void unpack8(const uint4 &w, Pair (&f)[4])
{
    f[0] = unpack<T>(w.x);
    f[1] = unpack<T>(w.y);
    f[2] = unpack<T>(w.z);
    f[3] = unpack<T>(w.w);
}
template <class T>
__device__ __forceinline__ uint4 pack8(const Pair *f) { return make_uint4(pack<T>(f[0]), pack<T>(f[1]), pack<T>(f[2]), pack<T>(f[3])); }

// 32 values of a lane's row to 16-byte chunks c0 .. c0 + 3 of its buffer row.
template <class T>
__device__ __forceinline__ void put32(uint32_t buf, int lane, int c0, const Pair (&v)[16])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) shared_store(swizzled(buf, lane, c0 + c), pack8<T>(v + 4 * c));
}
// 32 accumulator columns of the warp's lanes.
__device__ __forceinline__ void take32(Pair (&v)[16], uint32_t tmem)
{
    float f[32];
    tmem_load32(f, tmem);
    tmem_wait(f);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = make_pair2(f[2 * i], f[2 * i + 1]);
}

struct PairShared {
    uint64_t full[kPairStages], empty[kPairStages];
    uint64_t acc_full[2], acc_empty[2], drain;
    uint64_t in_full[8][2];
    uint32_t tmem;
};

constexpr int kBiasBytes = 128 * 2;               // staged bias of an epilogue warp's 128 columns
constexpr int kPairSmem = kPairStages * kStageBytes + 16 * kEpiBytes + 8 * kBiasBytes + (int)sizeof(PairShared);
static_assert(kPairSmem <= 232448, "pair kernel: shared memory");

// Adds a piece's 128 columns of the warp's lanes to the running sum (starts it with the first).
__device__ __forceinline__ void keep_piece(uint32_t acc, uint32_t running, bool first)
{
    for (int c = 0; c < 4; ++c) {
        float v[32];
        tmem_load32(v, acc + c * 32);
        tmem_wait(v);
        if (!first) {
            float w[32];
            tmem_load32(w, running + c * 32);
            tmem_wait(w);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += w[i];
        }
        tmem_store32(running + c * 32, v);
    }
}
// 32 columns of the last piece with the running sum added.
__device__ __forceinline__ void last_piece(float (&v)[32], uint32_t acc, uint32_t running, bool only)
{
    tmem_load32(v, acc);
    tmem_wait(v);
    if (!only) {
        float w[32];
        tmem_load32(w, running);
        tmem_wait(w);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] += w[i];
    }
}

// Eight columns' sums over the warp's rows, a lane's row in v: the lane has that of column lane / 4.
__device__ __forceinline__ float over_rows8(const Pair (&v)[4], bool live, int lane)
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 h = halves(v[i]);
        f[2 * i] = live ? h.x : 0.f;
        f[2 * i + 1] = live ? h.y : 0.f;
    }
#pragma unroll
    for (int n = 4, o = 16; n > 0; n /= 2, o /= 2) {         // a lane keeps half of its columns and gives the others away
        const bool upper = lane & o;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float keep = upper ? f[i + n] : f[i], give = upper ? f[i] : f[i + n];
            f[i] = keep + __shfl_xor_sync(~0u, give, o);
        }
    }
    f[0] += __shfl_xor_sync(~0u, f[0], 2);
    return f[0] + __shfl_xor_sync(~0u, f[0], 1);
}

// One epilogue warp's state.
struct EpiWarp {
    uint32_t buf[2];                             // its two buffers
    uint32_t bar[2];                             // completion of loads into them
    uint32_t phase[2];
    uint32_t bias;                               // staged bias of the warp's columns
    int lane;
};

// Starts the load of a 32-row box into buffer i (issued by one lane).
__device__ __forceinline__ void epi_fetch(const EpiWarp &w, int i, const CUtensorMap *map, int x, int y)
{
    if (w.lane == 0) {
        mbar_expect(w.bar[i], kEpiBytes);
        tile_load(w.buf[i], map, x, y, w.bar[i]);
    }
}
__device__ __forceinline__ bool epi_wait(EpiWarp &w, int i, int polls)
{
    const bool ok = mbar_wait(w.bar[i], w.phase[i], polls);
    w.phase[i] ^= 1;
    return __all_sync(~0u, ok);
}
// Hands buffer i to the copy engine.
__device__ __forceinline__ void epi_store(const EpiWarp &w, int i, const CUtensorMap *map, int x, int y)
{
    async_proxy_fence();
    __syncwarp();
    if (w.lane == 0) tile_store(map, w.buf[i], x, y);
}
// Waits until the copy engine has read every buffer handed to it.
__device__ __forceinline__ void epi_reclaim(const EpiWarp &w)
{
    if (w.lane == 0) tile_stores_read();
    __syncwarp();
}

__device__ __forceinline__ void stage_bias(uint32_t dst, const void *bias, int64_t col, int64_t n, int count, int lane)
{
    for (int i = lane; i < count; i += 32) {
        const uint16_t v = bias && col + i < n ? reinterpret_cast<const uint16_t *>(bias)[col + i] : (uint16_t)0;
        asm volatile("st.shared.u16 [%0], %1;" :: "r"(dst + i * 2), "h"(v) : "memory");
    }
}
// Adds 32 staged values, the same for every lane.
template <class T>
__device__ __forceinline__ void add_bias(Pair (&v)[16], uint32_t src)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        Pair b[4];
        unpack8<T>(shared_load(src + q * 16), b);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * q + i] = add2(v[4 * q + i], b[i]);
    }
}

template <int EPI, int ACT, class T, bool WIDE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
pair_product_kernel(const __grid_constant__ ProductParams p)
{
    extern __shared__ __align__(1024) uint8_t raw[];
    const uint32_t base = smem_addr(raw);
    const uint32_t epi_base = base + kPairStages * kStageBytes, bias_base = epi_base + 16 * kEpiBytes;
    PairShared &sh = *reinterpret_cast<PairShared *>(raw + kPairStages * kStageBytes + 16 * kEpiBytes + 8 * kBiasBytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int tiles = p.tiles_m * p.tiles_n * p.groups;
    const int steps = p.steps[0] + p.steps[1];
    const int pieces = WIDE ? (steps + kPieceSteps - 1) / kPieceSteps : 1;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairStages; ++i) { mbar_init(smem_addr(&sh.full[i]), 1); mbar_init(smem_addr(&sh.empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_addr(&sh.acc_full[i]), 1); mbar_init(smem_addr(&sh.acc_empty[i]), 16); }
        mbar_init(smem_addr(&sh.drain), 1);
        for (int i = 0; i < 8; ++i) { mbar_init(smem_addr(&sh.in_full[i][0]), 1); mbar_init(smem_addr(&sh.in_full[i][1]), 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1 && one_lane()) {
        prefetch_map(&p.a[0]);
        prefetch_map(&p.b[EPI == kEpiGated ? rank : 0]);
        prefetch_map(&p.out[0]);
    }
    if (warp == 2) tmem_alloc(smem_addr(&sh.tmem), 512);
    tensor_fence_before();
    __syncthreads();
    cluster_sync();
    tensor_fence_after();
    const uint32_t tmem = sh.tmem;
    grid_let_next();
    grid_wait();

    if (warp == 0 && one_lane()) {
        // ---- loads of both operands ----
        int it = 0;
        bool ok = true;
        for (int tile = pair; tile < tiles && ok; tile += pairs) {
            int g, tm, tn;
            tile_coords(p, tile, g, tm, tn);
            const int row_a = tm * 256 + (int)rank * 128;
            for (int s = 0; s < steps; ++s, ++it) {
                const int stage = it % kPairStages;
                if (it >= kPairStages && !mbar_wait(smem_addr(&sh.empty[stage]), (it / kPairStages - 1) & 1, p.polls)) { ok = false; break; }
                const int seg = s >= p.steps[0];
                const int k = (s - (seg ? p.steps[0] : 0)) * 64;
                const CUtensorMap *ma = &p.a[p.groups == 2 ? g : seg];
                const CUtensorMap *mb = &p.b[EPI == kEpiGated ? (int)rank : seg];
                const int row_b = EPI == kEpiGated ? tn * 128 : tn * 256 + (int)rank * 128;
                const uint32_t sa = base + stage * kStageBytes, sb = sa + kOperandBytes;
                const uint32_t bar = cluster_addr(smem_addr(&sh.full[stage]), 0);
                if (rank == 0) mbar_expect(smem_addr(&sh.full[stage]), 2 * kStageBytes);
                if (p.a_mn) {
                    tile_load_pair(sa, ma, row_a, k, bar);
                    tile_load_pair(sa + kOperandBytes / 2, ma, row_a + 64, k, bar);
                } else {
                    tile_load_pair(sa, ma, k, row_a, bar);
                }
                if (p.b_mn) {
                    tile_load_pair(sb, mb, row_b, k, bar);
                    tile_load_pair(sb + kOperandBytes / 2, mb, row_b + 64, k, bar);
                } else {
                    tile_load_pair(sb, mb, k, row_b, bar);
                }
            }
        }
        consumed(sh.empty, it, ok, p);
    } else if (warp == 1 && rank == 0 && one_lane()) {
        // ---- products of both blocks ----
        const uint32_t a_block = p.a_mn ? kOperandBytes / 2 : 16, b_block = p.b_mn ? kOperandBytes / 2 : 16;
        const uint64_t a_next = p.a_mn ? 2048 >> 4 : 32 >> 4, b_next = p.b_mn ? 2048 >> 4 : 32 >> 4;
        int it = 0, n_acc = 0;
        bool ok = true;
        for (int tile = pair; tile < tiles && ok; tile += pairs)
            for (int piece = 0; piece < pieces && ok; ++piece, ++n_acc) {
                // one accumulator with pieces (the other half holds the running sum), else two in turn
                const int acc = pieces > 1 ? 0 : n_acc & 1, use = pieces > 1 ? n_acc : n_acc >> 1;
                if (use > 0 && !mbar_wait(smem_addr(&sh.acc_empty[acc]), (use - 1) & 1, p.polls)) { ok = false; break; }
                tensor_fence_after();
                const uint32_t d = tmem + acc * 256;
                const int first = WIDE ? piece * kPieceSteps : 0, last = WIDE ? min(steps, first + kPieceSteps) : steps;
                for (int s = first; s < last; ++s, ++it) {
                    const int stage = it % kPairStages;
                    if (!mbar_wait(smem_addr(&sh.full[stage]), (it / kPairStages) & 1, p.polls)) { ok = false; break; }
                    tensor_fence_after();
                    const uint32_t sa = base + stage * kStageBytes;
                    uint64_t da = tile_descriptor(sa, a_block), db = tile_descriptor(sa + kOperandBytes, b_block);
#pragma unroll
                    for (int k = 0; k < 4; ++k, da += a_next, db += b_next) tensor_mma(d, da, db, p.idesc, s > first || k > 0);
                    tensor_commit(smem_addr(&sh.empty[stage]), 3);
                }
                if (ok) tensor_commit(smem_addr(&sh.acc_full[acc]), 3);
            }
        products_done(sh.drain, 1, ok, p);
    } else if (warp >= 4) {
        // ---- epilogue ----
        const int ew = warp - 4, quad = ew & 3, half = ew >> 2;
        EpiWarp w;
        w.lane = lane;
        w.bias = bias_base + ew * kBiasBytes;
        for (int i = 0; i < 2; ++i) {
            w.buf[i] = epi_base + (ew * 2 + i) * kEpiBytes;
            w.bar[i] = smem_addr(&sh.in_full[ew][i]);
            w.phase[i] = 0;
        }
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t empty0 = cluster_addr(smem_addr(&sh.acc_empty[0]), 0), empty1 = cluster_addr(smem_addr(&sh.acc_empty[1]), 0);
        int n_acc = 0;
        bool ok = true;
        for (int tile = pair; tile < tiles && ok; tile += pairs, ++n_acc) {
            int g, tm, tn;
            tile_coords(p, tile, g, tm, tn);
            const int acc = pieces > 1 ? 0 : n_acc & 1;
            const int row = tm * 256 + (int)rank * 128 + quad * 32;
            const uint32_t d = tmem + acc * 256 + lanes;
            const int col = EPI == kEpiGated ? tn * 128 + half * 64 : tn * 256 + half * 128;
            const bool rows_live = row < p.m;
            const int chunks = EPI == kEpiGated ? (col < p.n ? 1 : 0) : max(0, min(2, (p.n - col + 63) / 64));
            const CUtensorMap *out0 = &p.out[EPI == kEpiLinear ? g : 0];

            epi_reclaim(w);
            if (rows_live) {
                if (EPI == kEpiLinear && p.has_in) {
                    if (WIDE) {
                        if (chunks > 0) { epi_fetch(w, 0, &p.in[g], col, row); epi_fetch(w, 1, &p.in[g], col + 32, row); }
                    } else {
                        for (int c = 0; c < chunks; ++c) epi_fetch(w, c, &p.in[g], col + 64 * c, row);
                    }
                }
                if (EPI == kEpiGatedBack && chunks > 0) { epi_fetch(w, 0, &p.in[0], col, row); epi_fetch(w, 1, &p.in[1], col, row); }
            }
            if (EPI == kEpiLinear && p.bias[0]) stage_bias(w.bias, p.bias[0], col, p.n, 128, lane);
            if (EPI == kEpiGated && p.bias[0]) {
                stage_bias(w.bias, p.bias[0], col, p.n, 64, lane);
                stage_bias(w.bias + 128, p.bias[1], col, p.n, 64, lane);
            }
            __syncwarp();
            const uint32_t running = tmem + 256 + lanes + half * 128;
            for (int piece = 0; WIDE && piece < pieces - 1 && ok; ++piece, ++n_acc) {
                if (!(ok = __all_sync(~0u, mbar_wait(smem_addr(&sh.acc_full[0]), n_acc & 1, p.polls)))) break;
                tensor_fence_after();
                keep_piece(d + half * 128, running, piece == 0);
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(empty0);
            }
            if (!ok) break;
            ok = __all_sync(~0u, mbar_wait(smem_addr(&sh.acc_full[acc]), (pieces > 1 ? n_acc : n_acc >> 1) & 1, p.polls));
            if (!ok) break;
            tensor_fence_after();

            if (rows_live) {
                if (EPI == kEpiLinear) {
                    for (int c = 0; c < chunks && ok; ++c) {
                        if (WIDE) {
                            if (c > 0) {
                                epi_reclaim(w);
                                if (p.has_in) { epi_fetch(w, 0, &p.in[g], col + 64, row); epi_fetch(w, 1, &p.in[g], col + 96, row); }
                            }
                            for (int h = 0; h < 2; ++h) {
                                if (p.has_in && !(ok = epi_wait(w, h, p.polls))) break;
                                float v[32];
                                last_piece(v, d + half * 128 + c * 64 + h * 32, running + c * 64 + h * 32, pieces == 1);
#pragma unroll
                                for (int q = 0; q < 8; ++q) {
                                    const uint32_t at = swizzled(w.buf[h], lane, q);
                                    float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
                                    if (p.has_in) { const uint4 x = shared_load(at); r = *reinterpret_cast<const float4 *>(&x); }
                                    const float4 o = make_float4(v[4 * q] + r.x, v[4 * q + 1] + r.y, v[4 * q + 2] + r.z, v[4 * q + 3] + r.w);
                                    shared_store(at, *reinterpret_cast<const uint4 *>(&o));
                                }
                                if (col + c * 64 + h * 32 < p.n) epi_store(w, h, out0, col + c * 64 + h * 32, row);
                                else __syncwarp();
                            }
                        } else {
                            // with a residual both buffers hold it from the tile's start and the results
                            // replace it; the pre-activation then follows from the accumulators once more
                            const int at = p.has_in ? c : 0;
                            const bool both_out = p.has_out1 && !p.has_in;
                            if (p.has_in && !(ok = epi_wait(w, c, p.polls))) break;
                            if (c > 0 && !p.has_in) epi_reclaim(w);
                            for (int h = 0; h < 2; ++h) {
                                Pair v[16];
                                take32(v, d + half * 128 + c * 64 + h * 32);
                                if (p.bias[0]) add_bias<T>(v, w.bias + c * 128 + h * 64);
                                if (both_out) put32<T>(w.buf[1], lane, h * 4, v);
                                if (ACT != DISTSIM_ACT_NONE) {
#pragma unroll
                                    for (int i = 0; i < 16; ++i) v[i] = activation<ACT>(v[i]);
                                }
                                if (p.has_in) {
#pragma unroll
                                    for (int q = 0; q < 4; ++q) {
                                        Pair r[4];
                                        unpack8<T>(shared_load(swizzled(w.buf[c], lane, h * 4 + q)), r);
#pragma unroll
                                        for (int i = 0; i < 4; ++i) v[4 * q + i] = add2(v[4 * q + i], r[i]);
                                    }
                                }
                                put32<T>(w.buf[at], lane, h * 4, v);
                            }
                            epi_store(w, at, out0, col + 64 * c, row);
                            if (both_out) epi_store(w, 1, &p.out[1], col + 64 * c, row);
                        }
                    }
                    if (!WIDE && p.has_out1 && p.has_in && ok) {
                        epi_reclaim(w);
                        for (int c = 0; c < chunks; ++c) {
                            for (int h = 0; h < 2; ++h) {
                                Pair v[16];
                                take32(v, d + half * 128 + c * 64 + h * 32);
                                if (p.bias[0]) add_bias<T>(v, w.bias + c * 128 + h * 64);
                                put32<T>(w.buf[c], lane, h * 4, v);
                            }
                            epi_store(w, c, &p.out[1], col + 64 * c, row);
                        }
                    }
                } else if (EPI == kEpiGated) {
                    if (chunks > 0) {
                        for (int h = 0; h < 2; ++h) {
                            Pair gv[16], uv[16];
                            take32(gv, d + half * 64 + h * 32);
                            take32(uv, d + 128 + half * 64 + h * 32);
                            if (p.bias[0]) { add_bias<T>(gv, w.bias + h * 64); add_bias<T>(uv, w.bias + 128 + h * 64); }
                            if (p.has_out1) put32<T>(w.buf[1], lane, h * 4, gv);
#pragma unroll
                            for (int i = 0; i < 16; ++i) gv[i] = mul2(activation<ACT>(gv[i]), uv[i]);
                            put32<T>(w.buf[0], lane, h * 4, gv);
                        }
                        epi_store(w, 0, &p.out[0], col, row);
                        if (p.has_out1) {
                            epi_store(w, 1, &p.out[1], col, row);
                            epi_reclaim(w);
                            for (int h = 0; h < 2; ++h) {
                                Pair uv[16];
                                take32(uv, d + 128 + half * 64 + h * 32);
                                if (p.bias[0]) add_bias<T>(uv, w.bias + 128 + h * 64);
                                put32<T>(w.buf[0], lane, h * 4, uv);
                            }
                            epi_store(w, 0, &p.out[2], col, row);
                        }
                    }
                } else {
                    for (int c = 0; c < chunks && ok; ++c) {
                        if (c > 0) {
                            epi_reclaim(w);
                            epi_fetch(w, 0, &p.in[0], col + 64, row);
                            epi_fetch(w, 1, &p.in[1], col + 64, row);
                        }
                        ok = epi_wait(w, 0, p.polls);
                        ok = epi_wait(w, 1, p.polls) && ok;
                        if (!ok) break;
                        for (int h = 0; h < 2; ++h) {
                            Pair v[16];
                            take32(v, d + half * 128 + c * 64 + h * 32);
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const uint32_t ag = swizzled(w.buf[0], lane, h * 4 + q), au = swizzled(w.buf[1], lane, h * 4 + q);
                                Pair gq[4], uq[4];
                                unpack8<T>(shared_load(ag), gq);
                                unpack8<T>(shared_load(au), uq);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    Pair value, slope;
                                    activation_both<ACT>(gq[i], value, slope);
                                    const Pair dh = v[4 * q + i];
                                    gq[i] = mul2(mul2(dh, uq[i]), slope);
                                    uq[i] = mul2(dh, value);
                                }
                                shared_store(ag, pack8<T>(gq));
                                shared_store(au, pack8<T>(uq));
                                if (p.sums[0]) {
                                    const bool live = row + lane < p.m;
                                    const float sg = over_rows8(gq, live, lane), su = over_rows8(uq, live, lane);
                                    const int at = col + c * 64 + h * 32 + q * 8 + lane / 4;
                                    if (lane % 4 == 0 && at < p.n) {
                                        const int64_t to = (int64_t)(row / 32) * p.sums_ld + at;
                                        p.sums[0][to] = sg;
                                        p.sums[1][to] = su;
                                    }
                                }
                            }
                        }
                        epi_store(w, 0, &p.out[0], col + 64 * c, row);
                        epi_store(w, 1, &p.out[1], col + 64 * c, row);
                    }
                }
            }
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acc ? empty1 : empty0);
        }
        if (!ok && lane == 0) {
            give_up(p.status);
            for (int i = 0; i < 2; ++i) mbar_wait(w.bar[i], w.phase[i], kDrainPolls);   // loads of this tile, if any
        }
        if (lane == 0) tile_stores_read();                   // the buffers go with the block
        __syncwarp();
    }

    __syncwarp();
    tensor_fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 2) tmem_free(tmem, 512);
}

// ------------------------------------------------------------------------------ split kernel

struct SplitShared {
    uint64_t full[kSplitStages], empty[kSplitStages];
    uint64_t acc_full, acc_empty, drain;
    uint32_t tmem;
    int32_t failed;
};
constexpr int kSplitSmem = kSplitStages * kStageBytes + (int)sizeof(SplitShared);
static_assert(128 * kPartialPitch * 4 <= kSplitStages * kStageBytes, "a partial tile fits the ring");

// COUNT values at p, of which the first `valid` exist; one access where the address allows.
template <class TO, int COUNT>
__device__ __forceinline__ void row_load(const TO *p, int valid, float (&v)[COUNT])
{
    constexpr int kBytes = (int)sizeof(TO) * COUNT, kParts = kBytes > 16 ? kBytes / 16 : 1;
    using Vec = typename std::conditional<kBytes >= 16, uint4, uint2>::type;
    if (valid >= COUNT && (reinterpret_cast<uintptr_t>(p) & (sizeof(Vec) - 1)) == 0) {
        Vec w[kParts];
#pragma unroll
        for (int i = 0; i < kParts; ++i) w[i] = reinterpret_cast<const Vec *>(p)[i];
        const TO *e = reinterpret_cast<const TO *>(w);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = to_float(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = i < valid ? to_float(p[i]) : 0.f;
    }
}
template <class TO, int COUNT>
__device__ __forceinline__ void row_store(TO *p, int valid, const float (&v)[COUNT])
{
    constexpr int kBytes = (int)sizeof(TO) * COUNT, kParts = kBytes > 16 ? kBytes / 16 : 1;
    using Vec = typename std::conditional<kBytes >= 16, uint4, uint2>::type;
    if (valid >= COUNT && (reinterpret_cast<uintptr_t>(p) & (sizeof(Vec) - 1)) == 0) {
        Vec w[kParts];
        TO *e = reinterpret_cast<TO *>(w);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) e[i] = from_float<TO>(v[i]);
#pragma unroll
        for (int i = 0; i < kParts; ++i) reinterpret_cast<Vec *>(p)[i] = w[i];
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (i < valid) p[i] = from_float<TO>(v[i]);
    }
}

// Four neighbouring values of an epilogue, the activation chosen at run time:
// v = act(v) + add;  v = act(v) u;  g, u = d u act'(g), d act(g).
__device__ __forceinline__ void activate4(int act, float (&v)[4], const float (&add)[4])
{
    with_activation(act, [&](auto a) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const float2 f = halves(activation<decltype(a)::value>(make_pair2(v[i], v[i + 1])));
            v[i] = f.x + add[i];
            v[i + 1] = f.y + add[i + 1];
        }
    });
}
__device__ __forceinline__ void gate4(int act, float (&v)[4], const float (&u)[4])
{
    with_activation(act, [&](auto a) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const float2 f = halves(mul2(activation<decltype(a)::value>(make_pair2(v[i], v[i + 1])), make_pair2(u[i], u[i + 1])));
            v[i] = f.x;
            v[i + 1] = f.y;
        }
    });
}
__device__ __forceinline__ void gate_back4(int act, const float (&d)[4], float (&g)[4], float (&u)[4])
{
    with_activation(act, [&](auto a) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            Pair value, slope;
            activation_both<decltype(a)::value>(make_pair2(g[i], g[i + 1]), value, slope);
            const Pair dh = make_pair2(d[i], d[i + 1]);
            const float2 dg = halves(mul2(mul2(dh, make_pair2(u[i], u[i + 1])), slope)), du = halves(mul2(dh, value));
            g[i] = dg.x;
            g[i + 1] = dg.y;
            u[i] = du.x;
            u[i + 1] = du.y;
        }
    });
}

template <int EPI, class T, bool WIDE>
__global__ void __launch_bounds__(kSplitThreads, 1)
split_product_kernel(const __grid_constant__ ProductParams p)
{
    using TO = typename std::conditional<WIDE, float, T>::type;
    extern __shared__ __align__(1024) uint8_t ring[];
    const uint32_t base = smem_addr(ring);
    SplitShared &sh = *reinterpret_cast<SplitShared *>(ring + kSplitStages * kStageBytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t crank = cluster_rank(), half = crank & 1, leader = crank & ~1u;
    const int split = p.split, share = (int)crank >> 1;
    int g, tm, tn;
    tile_coords(p, (int)blockIdx.x / (2 * split), g, tm, tn);
    const int total = p.steps[0] + p.steps[1];
    const int s0 = (int)((int64_t)total * share / split), s1 = (int)((int64_t)total * (share + 1) / split);
    const int pieces = WIDE ? (s1 - s0 + kPieceSteps - 1) / kPieceSteps : 1;
    constexpr uint32_t kColumns = WIDE ? 512 : 256;
    const int valid_rows = min(128, p.m - tm * 256 - (int)half * 128);     // of this block; none or fewer: nothing of a is loaded

    if (threadIdx.x == 0) {
        for (int i = 0; i < kSplitStages; ++i) { mbar_init(smem_addr(&sh.full[i]), 1); mbar_init(smem_addr(&sh.empty[i]), 1); }
        mbar_init(smem_addr(&sh.acc_full), 1);
        mbar_init(smem_addr(&sh.acc_empty), 16);
        mbar_init(smem_addr(&sh.drain), 1);
        sh.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0 && one_lane()) {
        prefetch_map(&p.a[0]);
        prefetch_map(&p.b[EPI == kEpiGated ? half : 0]);
    }
    if (warp == 1) tmem_alloc(smem_addr(&sh.tmem), kColumns);
    tensor_fence_before();
    __syncthreads();
    cluster_sync();
    tensor_fence_after();
    const uint32_t tmem = sh.tmem;
    grid_let_next();
    grid_wait();

    if (warp == 0 && one_lane()) {
        const int row_a = tm * 256 + (int)half * 128;
        const uint32_t both_bytes = (p.m - tm * 256 > 128 ? 2 : 1) * kOperandBytes + 2 * kOperandBytes;
        bool ok = true;
        int it = 0;
        for (int s = s0; s < s1; ++s, ++it) {
            const int stage = it % kSplitStages;
            if (it >= kSplitStages && !mbar_wait(smem_addr(&sh.empty[stage]), (it / kSplitStages - 1) & 1, p.polls)) { ok = false; break; }
            const int seg = s >= p.steps[0];
            const int k = (s - (seg ? p.steps[0] : 0)) * 64;
            const CUtensorMap *ma = &p.a[p.groups == 2 ? g : seg];
            const CUtensorMap *mb = &p.b[EPI == kEpiGated ? (int)half : seg];
            const int row_b = EPI == kEpiGated ? tn * 128 : tn * 256 + (int)half * 128;
            const uint32_t sa = base + stage * kStageBytes, sb = sa + kOperandBytes;
            const uint32_t bar = cluster_addr(smem_addr(&sh.full[stage]), leader);
            if (half == 0) mbar_expect(smem_addr(&sh.full[stage]), both_bytes);
            if (valid_rows > 0) {
                if (p.a_mn) {
                    tile_load_pair(sa, ma, row_a, k, bar);
                    tile_load_pair(sa + kOperandBytes / 2, ma, row_a + 64, k, bar);
                } else {
                    tile_load_pair(sa, ma, k, row_a, bar);
                }
            }
            if (p.b_mn) {
                tile_load_pair(sb, mb, row_b, k, bar);
                tile_load_pair(sb + kOperandBytes / 2, mb, row_b + 64, k, bar);
            } else {
                tile_load_pair(sb, mb, k, row_b, bar);
            }
        }
        if (!consumed(sh.empty, it, ok, p)) sh.failed = 1;
    } else if (warp == 1 && half == 0 && one_lane()) {
        const uint32_t a_block = p.a_mn ? kOperandBytes / 2 : 16, b_block = p.b_mn ? kOperandBytes / 2 : 16;
        const uint64_t a_next = p.a_mn ? 2048 >> 4 : 32 >> 4, b_next = p.b_mn ? 2048 >> 4 : 32 >> 4;
        const uint16_t pair_mask = (uint16_t)(3u << leader);
        bool ok = true;
        int it = 0;
        for (int piece = 0; piece < pieces && ok; ++piece) {
            if (piece > 0 && !mbar_wait(smem_addr(&sh.acc_empty), (piece - 1) & 1, p.polls)) { ok = false; break; }
            tensor_fence_after();
            const int first = s0 + (WIDE ? piece * kPieceSteps : 0), last = WIDE ? min(s1, first + kPieceSteps) : s1;
            for (int s = first; s < last; ++s, ++it) {
                const int stage = it % kSplitStages;
                if (!mbar_wait(smem_addr(&sh.full[stage]), (it / kSplitStages) & 1, p.polls)) { ok = false; break; }
                tensor_fence_after();
                const uint32_t sa = base + stage * kStageBytes;
                uint64_t da = tile_descriptor(sa, a_block), db = tile_descriptor(sa + kOperandBytes, b_block);
#pragma unroll
                for (int k = 0; k < 4; ++k, da += a_next, db += b_next) tensor_mma(tmem, da, db, p.idesc, s > first || k > 0);
                tensor_commit(smem_addr(&sh.empty[stage]), pair_mask);
            }
            if (ok) tensor_commit(smem_addr(&sh.acc_full), pair_mask);
        }
        if (!products_done(sh.drain, (uint16_t)(1u << crank), ok, p)) sh.failed = 1;
    }
    __syncwarp();

    // ---- partial rows to shared memory (the ring is free once the products are done) ----
    float *part = reinterpret_cast<float *>(ring);
    if (warp >= 2) {
        const int quad = warp & 3, side = (warp - 2) >> 2, row = quad * 32 + lane;
        const uint32_t acc = tmem + ((uint32_t)(quad * 32) << 16) + side * 128, running = acc + 256;
        bool ok = true;
        for (int piece = 0; piece < pieces && ok; ++piece) {
            ok = __all_sync(~0u, mbar_wait(smem_addr(&sh.acc_full), piece & 1, p.polls));
            tensor_fence_after();
            if (!ok || piece == pieces - 1) break;
            keep_piece(acc, running, piece == 0);
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(cluster_addr(smem_addr(&sh.acc_empty), leader));
        }
        if (!ok) {
            if (lane == 0) { give_up(p.status); sh.failed = 1; }
        } else if (quad * 32 < valid_rows) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float v[32];
                last_piece(v, acc + c * 32, running + c * 32, pieces == 1);
                float4 *dst = reinterpret_cast<float4 *>(part + row * kPartialPitch + side * 128 + c * 32);
#pragma unroll
                for (int q = 0; q < 8; ++q) dst[q] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            }
        }
        tensor_fence_before();
    }
    __syncthreads();
    if (split > 1) cluster_sync();

    // ---- sum over the pairs and finish a share of the rows ----
    if (warp >= 2 && !sh.failed && valid_rows > 0) {
        // a lane has four columns of each half of the tile: of gate and up projection with kEpiGated
        const int col0 = (EPI == kEpiGated ? tn * 128 : tn * 256) + lane * 4, col1 = col0 + 128;
        const int valid0 = p.n - col0, valid1 = p.n - col1;
        float bias0[4], bias1[4];
        const T *b0 = reinterpret_cast<const T *>(p.bias[0]), *b1 = EPI == kEpiGated ? reinterpret_cast<const T *>(p.bias[1]) : b0 + 128;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bias0[i] = p.bias[0] && i < valid0 ? to_float(b0[col0 + i]) : 0.f;
            bias1[i] = p.bias[0] && i < (EPI == kEpiGated ? valid0 : valid1) ? to_float(b1[col0 + i]) : 0.f;
        }
        const TO *in0 = reinterpret_cast<const TO *>(p.in_p[EPI == kEpiLinear ? g : 0]);
        const TO *in1 = reinterpret_cast<const TO *>(p.in_p[1]);
        TO *out0 = reinterpret_cast<TO *>(p.out_p[EPI == kEpiLinear && g ? 1 : 0]);
        TO *out1 = reinterpret_cast<TO *>(p.out_p[1]), *out2 = reinterpret_cast<TO *>(p.out_p[2]);
        const int64_t in_ld = p.in_ld[EPI == kEpiLinear ? g : 0], out_ld = p.out_ld[EPI == kEpiLinear && g ? 1 : 0];
        const int r0 = valid_rows * share / split, r1 = valid_rows * (share + 1) / split;
        const uint32_t own = smem_addr(part) + lane * 16;
        float sum_g[2][4] = {}, sum_u[2][4] = {};             // kEpiGatedBack: over the warp's rows
        // four rows at a time: their loads are under way together
        for (int first = r0 + warp - 2; first < r1 && valid0 > 0; first += 8 * kRowsAhead) {
            float lo[kRowsAhead][4], hi[kRowsAhead][4];
#pragma unroll
            for (int q = 0; q < kRowsAhead; ++q) {
                const uint32_t at = own + min(first + 8 * q, r1 - 1) * (kPartialPitch * 4);
                const uint4 u = shared_load(at), w = shared_load(at + 512);
                *reinterpret_cast<uint4 *>(lo[q]) = u;
                *reinterpret_cast<uint4 *>(hi[q]) = w;
            }
            for (int b = 1; b < split; ++b) {                 // the others', from the next pair on: no block is everyone's first
                const uint32_t src = cluster_addr(own, 2 * ((share + b) & (split - 1)) + half);
#pragma unroll
                for (int q = 0; q < kRowsAhead; ++q) {
                    const uint32_t at = src + min(first + 8 * q, r1 - 1) * (kPartialPitch * 4);
                    const float4 u = load_cluster4(at), w = load_cluster4(at + 512);
                    lo[q][0] += u.x; lo[q][1] += u.y; lo[q][2] += u.z; lo[q][3] += u.w;
                    hi[q][0] += w.x; hi[q][1] += w.y; hi[q][2] += w.z; hi[q][3] += w.w;
                }
            }
#pragma unroll
            for (int q = 0; q < kRowsAhead; ++q) {
                const int r = first + 8 * q;
                if (r >= r1) break;
                const int64_t row = (int64_t)tm * 256 + half * 128 + r;
#pragma unroll
                for (int i = 0; i < 4; ++i) { lo[q][i] += bias0[i]; hi[q][i] += bias1[i]; }
                if (EPI == kEpiGated) {
                    if (p.has_out1) {
                        row_store<TO, 4>(out1 + row * p.out_ld[1] + col0, valid0, lo[q]);
                        row_store<TO, 4>(out2 + row * p.out_ld[2] + col0, valid0, hi[q]);
                    }
                    gate4(p.act, lo[q], hi[q]);
                    row_store<TO, 4>(out0 + row * out_ld + col0, valid0, lo[q]);
                } else if (EPI == kEpiLinear) {
                    float r0v[4] = {0.f, 0.f, 0.f, 0.f}, r1v[4] = {0.f, 0.f, 0.f, 0.f};
                    if (p.has_in) {
                        row_load<TO, 4>(in0 + row * in_ld + col0, valid0, r0v);
                        row_load<TO, 4>(in0 + row * in_ld + col1, valid1, r1v);
                    }
                    if (p.has_out1) {
                        row_store<TO, 4>(out1 + row * p.out_ld[1] + col0, valid0, lo[q]);
                        row_store<TO, 4>(out1 + row * p.out_ld[1] + col1, valid1, hi[q]);
                    }
                    activate4(p.act, lo[q], r0v);
                    activate4(p.act, hi[q], r1v);
                    row_store<TO, 4>(out0 + row * out_ld + col0, valid0, lo[q]);
                    row_store<TO, 4>(out0 + row * out_ld + col1, valid1, hi[q]);
                } else {
#pragma unroll
                    for (int side = 0; side < 2; ++side) {
                        const int col = side ? col1 : col0, valid = side ? valid1 : valid0;
                        float (&v)[4] = side ? hi[q] : lo[q];
                        float gv[4], uv[4];
                        row_load<TO, 4>(in0 + row * in_ld + col, valid, gv);
                        row_load<TO, 4>(in1 + row * p.in_ld[1] + col, valid, uv);
                        gate_back4(p.act, v, gv, uv);
                        row_store<TO, 4>(out0 + row * out_ld + col, valid, gv);
                        row_store<TO, 4>(out1 + row * p.out_ld[1] + col, valid, uv);
#pragma unroll
                        for (int i = 0; i < 4; ++i) { sum_g[side][i] += gv[i]; sum_u[side][i] += uv[i]; }
                    }
                }
            }
        }
        if (EPI == kEpiGatedBack && p.sums[0]) {
            const int64_t to = (((int64_t)tm * 2 + half) * split + share) * 8 + warp - 2;
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                const int col = side ? col1 : col0, valid = side ? valid1 : valid0;
                row_store<float, 4>(p.sums[0] + to * p.sums_ld + col, valid, sum_g[side]);
                row_store<float, 4>(p.sums[1] + to * p.sums_ld + col, valid, sum_u[side]);
            }
        }
    }
    __syncthreads();
    cluster_sync();                                           // the others may still read this block's partial rows
    if (warp == 1) tmem_free(tmem, kColumns);
}

// ------------------------------------------------------------------------------ few-rows kernel

constexpr int kFewRows = 64;
constexpr int kFewStages = 5;                    // two blocks to an SM
constexpr int kFewStageBytes = kOperandBytes + kFewRows / 2 * kStepBytes;
constexpr int kFewThreads = 64 + 4 * 32;
constexpr int kFewPitch = 132;
struct FewShared {
    uint64_t full[kFewStages], empty[kFewStages];
    uint64_t acc_full, drain;
    uint32_t tmem;
    int32_t failed;
};
constexpr int kFewSmem = kFewStages * kFewStageBytes + (int)sizeof(FewShared);
static_assert(kFewRows * kFewPitch * 4 <= kFewStages * kFewStageBytes, "the partial sums fit the ring");

template <int EPI, class T>
__global__ void __launch_bounds__(kFewThreads, 2)
few_rows_kernel(const __grid_constant__ ProductParams p)
{
    extern __shared__ __align__(1024) uint8_t ring[];
    const uint32_t base = smem_addr(ring);
    FewShared &sh = *reinterpret_cast<FewShared *>(ring + kFewStages * kFewStageBytes);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t crank = cluster_rank(), half = crank & 1, leader = crank & ~1u;
    const int split = p.split, share = (int)crank >> 1, tn = (int)blockIdx.x / (2 * split);
    const int total = p.steps[0] + p.steps[1];
    const int s0 = (int)((int64_t)total * share / split), s1 = (int)((int64_t)total * (share + 1) / split);
    // of this block: 128 rows of the weight (of the gate's or the up projection's with kEpiGated)
    const int row_w = EPI == kEpiGated ? tn * 128 : tn * 256 + (int)half * 128;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kFewStages; ++i) { mbar_init(smem_addr(&sh.full[i]), 1); mbar_init(smem_addr(&sh.empty[i]), 1); }
        mbar_init(smem_addr(&sh.acc_full), 1);
        mbar_init(smem_addr(&sh.drain), 1);
        sh.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0 && one_lane()) {
        prefetch_map(&p.a[0]);
        prefetch_map(&p.b[EPI == kEpiGated ? half : 0]);
    }
    if (warp == 1) tmem_alloc(smem_addr(&sh.tmem), 64);
    tensor_fence_before();
    __syncthreads();
    cluster_sync();
    tensor_fence_after();
    const uint32_t tmem = sh.tmem;
    grid_let_next();
    grid_wait();

    if (warp == 0 && one_lane()) {
        const uint32_t token_bytes = p.few / 2 * kStepBytes;
        bool ok = true;
        int it = 0;
        for (int s = s0; s < s1; ++s, ++it) {
            const int stage = it % kFewStages;
            if (it >= kFewStages && !mbar_wait(smem_addr(&sh.empty[stage]), (it / kFewStages - 1) & 1, p.polls)) { ok = false; break; }
            const int seg = s >= p.steps[0];
            const int k = (s - (seg ? p.steps[0] : 0)) * 64;
            const CUtensorMap *mw = &p.b[EPI == kEpiGated ? (int)half : seg];
            const uint32_t sw = base + stage * kFewStageBytes;
            const uint32_t bar = cluster_addr(smem_addr(&sh.full[stage]), leader);
            if (half == 0) mbar_expect(smem_addr(&sh.full[stage]), 2 * (kOperandBytes + token_bytes));
            if (p.b_mn) {
                tile_load_pair(sw, mw, row_w, k, bar);
                tile_load_pair(sw + kOperandBytes / 2, mw, row_w + 64, k, bar);
            } else {
                tile_load_pair(sw, mw, k, row_w, bar);
            }
            tile_load_pair(sw + kOperandBytes, &p.a[seg], k, (int)half * p.few / 2, bar);
        }
        if (!consumed(sh.empty, it, ok, p)) sh.failed = 1;
    } else if (warp == 1 && half == 0 && one_lane()) {
        const uint32_t w_block = p.b_mn ? kOperandBytes / 2 : 16;
        const uint64_t w_next = p.b_mn ? 2048 >> 4 : 32 >> 4;
        const uint16_t pair_mask = (uint16_t)(3u << leader);
        bool ok = true;
        int it = 0;
        for (int s = s0; s < s1; ++s, ++it) {
            const int stage = it % kFewStages;
            if (!mbar_wait(smem_addr(&sh.full[stage]), (it / kFewStages) & 1, p.polls)) { ok = false; break; }
            tensor_fence_after();
            const uint32_t sw = base + stage * kFewStageBytes;
            uint64_t dw = tile_descriptor(sw, w_block), dt = tile_descriptor(sw + kOperandBytes, 16);
#pragma unroll
            for (int k = 0; k < 4; ++k, dw += w_next, dt += 32 >> 4) tensor_mma(tmem, dw, dt, p.idesc, it > 0 || k > 0);
            tensor_commit(smem_addr(&sh.empty[stage]), pair_mask);
        }
        if (ok) tensor_commit(smem_addr(&sh.acc_full), pair_mask);
        if (!products_done(sh.drain, (uint16_t)(1u << crank), ok, p)) sh.failed = 1;
    }
    __syncwarp();

    // ---- partial sums to shared memory, by tokens ----
    float *part = reinterpret_cast<float *>(ring);
    if (warp >= 2) {
        const int quad = warp & 3;
        const bool ok = __all_sync(~0u, mbar_wait(smem_addr(&sh.acc_full), 0, p.polls));
        tensor_fence_after();
        if (!ok) {
            if (lane == 0) { give_up(p.status); sh.failed = 1; }
        } else {
            for (int t0 = 0; t0 < p.m; t0 += 32) {
                float v[32];
                tmem_load32(v, tmem + ((uint32_t)(quad * 32) << 16) + t0);
                tmem_wait(v);
#pragma unroll
                for (int t = 0; t < 32; ++t)
                    if (t0 + t < p.m) part[(t0 + t) * kFewPitch + quad * 32 + lane] = v[t];
            }
        }
        tensor_fence_before();
    }
    __syncthreads();
    cluster_sync();

    // ---- sum over the pairs and finish a share of the tokens ----
    if (warp >= 2 && !sh.failed) {
        const int parts = EPI == kEpiGated ? 2 * split : split, part_of = EPI == kEpiGated ? (int)crank : share;
        const int r0 = p.m * part_of / parts, r1 = p.m * (part_of + 1) / parts;
        const int col = (EPI == kEpiGated ? tn * 128 : row_w) + lane * 4, valid = p.n - col;
        const uint32_t own = smem_addr(part) + lane * 16;
        float bias0[4], bias1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bias0[i] = p.bias[0] && i < valid ? to_float(reinterpret_cast<const T *>(p.bias[0])[col + i]) : 0.f;
            bias1[i] = EPI == kEpiGated && p.bias[0] && i < valid ? to_float(reinterpret_cast<const T *>(p.bias[1])[col + i]) : 0.f;
        }
        T *out0 = reinterpret_cast<T *>(p.out_p[0]), *out1 = reinterpret_cast<T *>(p.out_p[1]), *out2 = reinterpret_cast<T *>(p.out_p[2]);
        const T *in0 = reinterpret_cast<const T *>(p.in_p[0]), *in1 = reinterpret_cast<const T *>(p.in_p[1]);
        float sum_g[4] = {}, sum_u[4] = {};                   // kEpiGatedBack: over the warp's tokens
        for (int64_t r = r0 + warp - 2; r < r1 && valid > 0; r += 4) {
            const uint32_t at = own + (uint32_t)r * (kFewPitch * 4);
            float lo[4] = {0.f, 0.f, 0.f, 0.f}, hi[4] = {0.f, 0.f, 0.f, 0.f};
            for (int b = 0; b < split; ++b) {
                const uint32_t rank = 2 * ((share + b) & (split - 1));
                const float4 u = load_cluster4(cluster_addr(at, EPI == kEpiGated ? rank : rank + half));
                lo[0] += u.x; lo[1] += u.y; lo[2] += u.z; lo[3] += u.w;
                if (EPI == kEpiGated) {
                    const float4 w = load_cluster4(cluster_addr(at, rank + 1));
                    hi[0] += w.x; hi[1] += w.y; hi[2] += w.z; hi[3] += w.w;
                }
            }
            if (EPI == kEpiGated) {
#pragma unroll
                for (int i = 0; i < 4; ++i) { lo[i] += bias0[i]; hi[i] += bias1[i]; }
                if (p.has_out1) {
                    row_store<T, 4>(out1 + r * p.out_ld[1] + col, valid, lo);
                    row_store<T, 4>(out2 + r * p.out_ld[2] + col, valid, hi);
                }
                gate4(p.act, lo, hi);
                row_store<T, 4>(out0 + r * p.out_ld[0] + col, valid, lo);
            } else if (EPI == kEpiLinear) {
                float res[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i) lo[i] += bias0[i];
                if (p.has_in) row_load<T, 4>(in0 + r * p.in_ld[0] + col, valid, res);
                if (p.has_out1) row_store<T, 4>(out1 + r * p.out_ld[1] + col, valid, lo);
                activate4(p.act, lo, res);
                row_store<T, 4>(out0 + r * p.out_ld[0] + col, valid, lo);
            } else {
                float gv[4], uv[4];
                row_load<T, 4>(in0 + r * p.in_ld[0] + col, valid, gv);
                row_load<T, 4>(in1 + r * p.in_ld[1] + col, valid, uv);
                gate_back4(p.act, lo, gv, uv);
                row_store<T, 4>(out0 + r * p.out_ld[0] + col, valid, gv);
                row_store<T, 4>(out1 + r * p.out_ld[1] + col, valid, uv);
#pragma unroll
                for (int i = 0; i < 4; ++i) { sum_g[i] += gv[i]; sum_u[i] += uv[i]; }
            }
        }
        if (EPI == kEpiGatedBack && p.sums[0]) {
            const int64_t to = (part_of * 4 + warp - 2) * p.sums_ld + col;
            row_store<float, 4>(p.sums[0] + to, valid, sum_g);
            row_store<float, 4>(p.sums[1] + to, valid, sum_u);
        }
    }
    __syncthreads();
    cluster_sync();                                           // the others may still read this block's partial sums
    if (warp == 1) tmem_free(tmem, 64);
}

// ------------------------------------------------------------------------------ host side

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_function()
{
    static EncodeTiled fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}

// Map of a rows x cols matrix, boxes of box_rows x 128 bytes, 128-byte swizzle.
bool encode(CUtensorMap *map, CUtensorMapDataType type, int elem, const Matrix &x, int64_t rows, int64_t cols, int box_rows)
{
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)x.ld * elem};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / elem), (cuuint32_t)box_rows}, ones[2] = {1, 1};
    return encode_function()(map, type, 2, const_cast<void *>(x.p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int EPI, int ACT, class T, bool WIDE>
cudaError_t launch_pair(OperatorLaunch &l, const ProductParams &p)
{
    const auto kernel = pair_product_kernel<EPI, ACT, T, WIDE>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), kPairSmem);
    if (e != cudaSuccess) return e;
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n * p.groups;
    const int64_t pairs = tiles < l.sm_count / 2 ? tiles : l.sm_count / 2;
    return launch_kernel(l, kEarly, kernel, (unsigned)(2 * pairs), 1, kPairThreads, kPairSmem, 0, p);
}

template <int EPI, class T, bool WIDE>
cudaError_t launch(OperatorLaunch &l, const ProductParams &p, const ProductPlan &plan)
{
    cudaError_t e;
    if (plan.few) {
        if constexpr (!WIDE) {
            const auto kernel = few_rows_kernel<EPI, T>;
            if ((e = ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), kFewSmem)) != cudaSuccess) return e;
            return launch_kernel(l, kEarly, kernel, (unsigned)(2 * p.tiles_n * plan.split), 1, kFewThreads, kFewSmem, 2 * plan.split, p);
        }
    }
    if (plan.pair) {
        if (WIDE) return launch_pair<EPI, DISTSIM_ACT_NONE, T, WIDE>(l, p);
        switch (p.act) {
        case DISTSIM_ACT_RELU: return launch_pair<EPI, WIDE ? 0 : DISTSIM_ACT_RELU, T, WIDE>(l, p);
        case DISTSIM_ACT_GELU: return launch_pair<EPI, WIDE ? 0 : DISTSIM_ACT_GELU, T, WIDE>(l, p);
        case DISTSIM_ACT_GELU_TANH: return launch_pair<EPI, WIDE ? 0 : DISTSIM_ACT_GELU_TANH, T, WIDE>(l, p);
        case DISTSIM_ACT_SILU: return launch_pair<EPI, WIDE ? 0 : DISTSIM_ACT_SILU, T, WIDE>(l, p);
        default: return launch_pair<EPI, DISTSIM_ACT_NONE, T, WIDE>(l, p);
        }
    }
    const auto kernel = split_product_kernel<EPI, T, WIDE>;
    if ((e = ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), kSplitSmem)) != cudaSuccess) return e;
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n * p.groups;
    if (tiles * plan.split > 0x3fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel(l, kEarly, kernel, (unsigned)(2 * tiles * plan.split), 1, kSplitThreads, kSplitSmem, 2 * plan.split, p);
}

template <class T>
cudaError_t dispatch(OperatorLaunch &l, const Product &q, const ProductParams &p, const ProductPlan &plan)
{
    switch (q.epilogue) {
    case kEpiLinear: return q.wide ? launch<kEpiLinear, T, true>(l, p, plan) : launch<kEpiLinear, T, false>(l, p, plan);
    case kEpiGated: return launch<kEpiGated, T, false>(l, p, plan);
    default: return launch<kEpiGatedBack, T, false>(l, p, plan);
    }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

int split_capacity(int split, int sm_count)
{
    const auto kernel = split_product_kernel<kEpiLinear, __nv_bfloat16, false>;       // the others take the same room
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3((unsigned)(2 * split * sm_count));
    cfg.blockDim = dim3(kSplitThreads);
    cfg.dynamicSmemBytes = kSplitSmem;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)(2 * split);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (ensure_dynamic_smem(reinterpret_cast<const void *>(kernel), kSplitSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = sm_count / (2 * split) > 1 ? sm_count / (2 * split) * 3 / 4 : 1;
    }
    return n;
}

bool few_rows(const Product &p) { return p.m <= kFewRows && !p.a_mn && !p.wide && p.groups == 1; }

ProductPlan choose_plan(const Product &p, const OperatorLaunch &l, int64_t unaligned_in, int64_t unaligned_out)
{
    ProductPlan plan;
    const int64_t steps = ceil_div(p.k[0], 64) + ceil_div(p.k[1], 64);
    const int64_t tiles = ceil_div(p.m, 256) * ceil_div(p.n, p.epilogue == kEpiGated ? 128 : 256) * p.groups;
    const double rows = p.m < 128 ? p.m / 128.0 : 1.0;
    const int64_t waves = ceil_div(tiles, l.sm_count / 2);
    plan.pair = true;
    double best = 4.7 + 1.1 * rows + 0.265 * (double)(waves * steps) + (waves > 1 ? 3.0 : 0.0);
    if (unaligned_in + unaligned_out > 0) best += 2.0 + (double)(unaligned_in + unaligned_out) / 2.3e6;
    const double direct = (double)unaligned_out / 3.8e6 + (double)unaligned_in / 0.6e6;
    for (int s = 1; s <= 4 && s <= steps; s *= 2) {
        const double wave = (s == 1 ? 4.2 : s == 2 ? 4.7 : 5.2) + 4.3 * rows + 0.265 * (double)ceil_div(steps, s);
        const double t = wave * (double)ceil_div(tiles, l.split_capacity[s / 2]) + direct;
        if (t < best) { best = t; plan.pair = false; plan.split = s; }
    }
    if (few_rows(p)) {
        // bound by the weight's stream: as many pairs as run at a time (two blocks to an SM).  Split 1 / 2 / 4
        // in us: 1 x 4096 x 1024 13.4 / 8.6 / 6.1; 7 x 2048 x 8192 11.8 / 9.3 / 8.9; 16 x 6144 x 12288 31.7 / 28.1 / 31.2
        plan.few = true;
        plan.pair = false;
        plan.split = 1;
        const int64_t columns = ceil_div(p.n, p.epilogue == kEpiGated ? 128 : 256);
        for (int s = 2; s <= 4 && s <= steps && columns * s <= l.sm_count; s *= 2) plan.split = s;
    }
    return plan;
}

int64_t product_sum_rows(const Product &p, const ProductPlan &plan)
{
    if (plan.few) return 4 * plan.split;
    return plan.pair ? ceil_div(p.m, 32) : ceil_div(p.m, 128) * plan.split * 8;
}

cudaError_t launch_product(OperatorLaunch &l, const Product &q, const ProductPlan &plan)
{
    if (!encode_function()) return cudaErrorNotSupported;
    ProductParams p{};
    const CUtensorMapDataType ty = q.in_type == DISTSIM_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const bool gated = q.epilogue == kEpiGated;
    const int tile_n = gated ? 128 : 256;
    p.m = (int32_t)q.m;
    p.n = (int32_t)q.n;
    p.tiles_m = (int32_t)ceil_div(q.m, 256);
    p.tiles_n = (int32_t)ceil_div(q.n, tile_n);
    p.groups = q.groups;
    p.a_mn = q.a_mn;
    p.b_mn = q.b_mn;
    p.act = q.act;
    p.split = plan.split;
    p.few = plan.few ? (int32_t)ceil_div(q.m, 16) * 16 : 0;
    p.status = l.status;
    p.polls = l.polls;
    p.sums_ld = q.sums_ld;
    bool ok = true;
    for (int i = 0; i < 2; ++i) {
        p.steps[i] = (int32_t)ceil_div(q.k[i], 64);
        p.bias[i] = q.bias[i];
        const int64_t k = q.k[q.groups == 2 || gated ? 0 : i];
        if (q.a[i].p && k > 0)
            ok = ok && (q.a_mn ? encode(&p.a[i], ty, 2, q.a[i], k, q.m, 64) : encode(&p.a[i], ty, 2, q.a[i], q.m, k, plan.few ? p.few / 2 : 128));
        if (q.b[i].p && k > 0)
            ok = ok && (q.b_mn ? encode(&p.b[i], ty, 2, q.b[i], k, q.n, 64)
                               : encode(&p.b[i], ty, 2, q.b[i], q.n, k, 128));
    }
    const int eo = q.wide ? 4 : 2;
    const CUtensorMapDataType to = q.wide ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : ty;
    for (int i = 0; i < 3; ++i) {
        p.out_p[i] = const_cast<void *>(q.out[i].p);
        p.out_ld[i] = q.out[i].ld;
        if (plan.pair && q.out[i].p) ok = ok && encode(&p.out[i], to, eo, q.out[i], q.m, q.n, 32);
    }
    for (int i = 0; i < 2; ++i) {
        p.in_p[i] = q.in[i].p;
        p.in_ld[i] = q.in[i].ld;
        p.sums[i] = q.sums[i];
        if (plan.pair && q.in[i].p) ok = ok && encode(&p.in[i], to, eo, q.in[i], q.m, q.n, 32);
    }
    if (!ok) return cudaErrorInvalidValue;
    p.has_in = q.in[0].p != nullptr;
    p.has_out1 = q.out[1].p != nullptr && q.groups == 1;
    // kind::f16 instruction: 32-bit accumulators, operand type, operand order, N / 8, M / 16
    const uint32_t fmt = q.in_type == DISTSIM_F16 ? 0 : 1;
    const uint32_t rows_mn = plan.few ? q.b_mn : q.a_mn, cols_mn = plan.few ? q.a_mn : q.b_mn, cols = plan.few ? (uint32_t)p.few : 256u;
    p.idesc = 1u << 4 | fmt << 7 | fmt << 10 | rows_mn << 15 | cols_mn << 16 | cols / 8 << 17 | 256u / 16 << 24;
    return q.in_type == DISTSIM_F16 ? dispatch<__half>(l, q, p, plan) : dispatch<__nv_bfloat16>(l, q, p, plan);
}

}  // namespace distsim
