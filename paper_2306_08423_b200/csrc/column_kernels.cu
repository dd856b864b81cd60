// Passes around the matrix products: a gradient times an activation's derivative with its column
// sums (the bias gradient), and copies into rows that the tiled copies can read.  Memory-bound:
// each value is read and written once, 16 bytes a thread.
//
// column_pass_kernel: a block takes 256 columns (a warp's row of 32 lanes x 8 columns, 512 bytes
// of a row) and a run of rows, warp w the rows w, w + 8, ..; sums stay in registers, are joined in
// shared memory and left as the block's partial.  The last block of a column range to finish adds
// the partials in block order, so sums do not depend on timing.
// As many blocks as run at a time take equal runs.  Measured (f16, bound by memory from about 30 MB on, by
// latency below): sums of 8192 x 4096 15.6 us (4.3 TB/s), 8192 x 1024 7.2 us; with a gelu's derivative 8192 x
// 4096 35 us (3.8 TB/s); 8192 x 4097, every row elsewhere behind a boundary, 24 us.
//
// move_kernel: two weights of 10560 x 3014 (f16) 44 us (5.8 TB/s read and written, of 6.46 of a copy).
#include "operators.h"
#include "pairs.cuh"
#include "tensor_core.cuh"

namespace distsim {

namespace {

constexpr int kColsPerBlock = 256;
constexpr int kBlocksPerSm = 3;
constexpr int kMinRows = 32;                     // rows a block takes at least

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Runs of rows that a column range is cut into: as many blocks as run at a time.  Several (which are
// counted) only where the ranges are half as many at most: fewer than kColumnCounters.
int64_t row_runs(int64_t rows, int64_t ranges, int sm_count)
{
    int64_t runs = (int64_t)sm_count * kBlocksPerSm / ranges;
    if (runs > ceil_div(rows, kMinRows)) runs = ceil_div(rows, kMinRows);
    return runs < 1 ? 1 : runs;
}

template <class T>
struct PassParams {
    struct {
        const T *x;
        const float *partials;                   // instead of x
        int64_t ld, cols, rows;
        void *sums;
        int first;                               // column range
    } part[kPassParts];
    int n;
    const T *z;
    T *out;
    int64_t ld_z, ld_out;
    bool vec_out, wide;                          // sums are 32-bit
    float *partial;
    int32_t *counters;
};

// EXACT: columns in whole aligned eights.
template <class T, int ACT, bool EXACT>
__global__ void __launch_bounds__(256, kBlocksPerSm)
column_pass_kernel(const __grid_constant__ PassParams<T> p)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int k = 0;
    while (k + 1 < p.n && (int)blockIdx.x >= p.part[k + 1].first) ++k;
    const T *const x = p.part[k].x, *const z = p.z;
    T *const out = p.out;
    const int64_t ld_x = p.part[k].ld, ld_z = p.ld_z, ld_out = p.ld_out, cols = p.part[k].cols, rows = p.part[k].rows;
    const int64_t start = (int64_t)((int)blockIdx.x - p.part[k].first) * kColsPerBlock, col = start + lane * 8;
    const int valid = (int)min(cols - col, (int64_t)8);
    const int64_t r0 = rows * blockIdx.y / gridDim.y, r1 = rows * (blockIdx.y + 1) / gridDim.y;
    const T *const x_end = x + (rows - 1) * ld_x + cols, *const z_end = z + (rows - 1) * ld_z + cols;
    Oct sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum.v[i] = both(0.f);
    constexpr int kRowsAhead = (ACT == DISTSIM_ACT_NONE ? 4 : 2) / (EXACT ? 1 : 2);      // rows a warp loads at a time
    grid_let_next();
    grid_wait();
    if (ACT == DISTSIM_ACT_NONE && p.part[k].partials) {
        if (valid > 0)
#pragma unroll 4
            for (int64_t r = r0 + warp; r < r1; r += 8) {
                const float4 *from = reinterpret_cast<const float4 *>(p.part[k].partials + r * ld_x + col);
                const float4 a = from[0], b = from[1];
                const Pair v[4] = {make_pair2(a.x, a.y), make_pair2(a.z, a.w), make_pair2(b.x, b.y), make_pair2(b.z, b.w)};
#pragma unroll
                for (int i = 0; i < 4; ++i) sum.v[i] = add2(sum.v[i], v[i]);
            }
    } else if (valid > 0)
        // some rows at a time: their loads are under way together
        for (int64_t r = r0 + warp; r < r1; r += 8 * kRowsAhead) {
            Request<EXACT> a[kRowsAhead], b[kRowsAhead];
#pragma unroll
            for (int q = 0; q < kRowsAhead; ++q) {
                const int64_t at = r + 8 * q;
                if (at >= r1) continue;
                request8(a[q], x + at * ld_x + col, x, x_end);
                if (ACT != DISTSIM_ACT_NONE) request8(b[q], z + at * ld_z + col, z, z_end);
            }
#pragma unroll
            for (int q = 0; q < kRowsAhead; ++q) {
                const int64_t at = r + 8 * q;
                if (at >= r1) continue;
                Oct v = receive8(a[q], x + at * ld_x + col, valid);
                if (ACT != DISTSIM_ACT_NONE) {
                    const Oct w = receive8(b[q], z + at * ld_z + col, valid);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        Pair value, slope;
                        activation_both<ACT>(w.v[i], value, slope);
                        v.v[i] = mul2(v.v[i], slope);
                    }
                }
                if (out) write8<T, EXACT>(out + at * ld_out + col, valid, p.vec_out, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum.v[i] = add2(sum.v[i], v.v[i]);
            }
        }
    if (!p.part[k].sums) return;
    __shared__ __align__(16) float joined[8][kColsPerBlock];
    __shared__ bool last;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = halves(sum.v[i]);
        joined[warp][lane * 8 + 2 * i] = f.x;
        joined[warp][lane * 8 + 2 * i + 1] = f.y;
    }
    __syncthreads();
    const int64_t c = start + threadIdx.x;
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += joined[w][threadIdx.x];
    if (gridDim.y > 1) {
        // a run's partials: all ranges, 256 a range
        const int64_t run = (int64_t)gridDim.x * kColsPerBlock;
        float *const partial = p.partial + (int64_t)blockIdx.x * kColsPerBlock;
        partial[blockIdx.y * run + threadIdx.x] = s;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            last = atomicAdd(p.counters + blockIdx.x, 1) == (int)gridDim.y - 1;
            if (last) p.counters[blockIdx.x] = 0;
        }
        __syncthreads();
        if (!last) return;
        __threadfence();
        // warp w adds the partials w, w + 8, .. of eight columns a lane, as two wide loads, eight under way
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f), u = t;
        const int runs = (int)gridDim.y;
#pragma unroll 4
        for (int b = warp; b < runs; b += 8) {
            const float4 *from = reinterpret_cast<const float4 *>(partial + b * run) + lane;
            const float4 f = __ldcg(from), g = __ldcg(from + 32);
            t.x += f.x; t.y += f.y; t.z += f.z; t.w += f.w;
            u.x += g.x; u.y += g.y; u.z += g.z; u.w += g.w;
        }
        *reinterpret_cast<float4 *>(&joined[warp][lane * 4]) = t;
        *reinterpret_cast<float4 *>(&joined[warp][128 + lane * 4]) = u;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += joined[w][threadIdx.x];
    }
    if (c < cols) {
        if (p.wide) static_cast<float *>(p.part[k].sums)[c] = s;
        else static_cast<T *>(p.part[k].sums)[c] = from_float<T>(s);
    }
}

struct Moves {
    Move m[kMostMoves];
    int32_t pieces[kMostMoves];                  // 16-byte pieces of dst that a row can touch
    uint32_t first[kMostMoves];                  // block
    int n;
};
constexpr int kRowsAThread = 4;

// A thread writes a 16-byte piece of dst in each of four rows; its values come from the two pieces of
// src that hold them, shifted into place.  The ends of rows go value by value, and so do pieces whose
// sources reach beyond src's first or last value.  A thread's loads are under way together.
__global__ void __launch_bounds__(256, 4)
move_kernel(const __grid_constant__ Moves all)
{
    int k = 0;
    while (k + 1 < all.n && blockIdx.x >= all.first[k + 1]) ++k;
    const Move &m = all.m[k];
    const uint32_t pieces = (uint32_t)all.pieces[k];
    const uint64_t place = (uint64_t)(blockIdx.x - all.first[k]) * 256 + threadIdx.x;
    const int64_t group = place >> 32 ? (int64_t)(place / pieces) : (int64_t)((uint32_t)place / pieces), r = group * kRowsAThread;
    const int64_t column = (int64_t)(place - (uint64_t)group * pieces) * 8;
    const int rows = (int)min(m.rows - r, (int64_t)kRowsAThread);
    const uintptr_t begin = reinterpret_cast<uintptr_t>(m.src), end = reinterpret_cast<uintptr_t>(m.src + (m.rows - 1) * m.ld_src + m.cols);
    uint16_t *const dst = m.dst + r * m.ld_dst + column;
    const uint16_t *const src = m.src + r * m.ld_src + column;
    const int left = (int)min(m.cols - column, (int64_t)64);
    uint4 v[kRowsAThread], w[kRowsAThread];
    uint32_t wide = 0;
    grid_let_next();
    grid_wait();
    if (m.src)
#pragma unroll
        for (int q = 0; q < kRowsAThread; ++q) {
            // the piece of dst starts `back` values before the column
            const int back = (int)((reinterpret_cast<uintptr_t>(dst + q * m.ld_dst) & 15) / 2);
            const uintptr_t from = reinterpret_cast<uintptr_t>(src + q * m.ld_src - back), a = from & ~(uintptr_t)15;
            const bool second = from & 15;
            v[q] = w[q] = make_uint4(0, 0, 0, 0);
            if (q < rows && a >= begin && a + (second ? 32 : 16) <= end) {
                wide |= 1u << q;
                v[q] = *reinterpret_cast<const uint4 *>(a);
                if (second) w[q] = *(reinterpret_cast<const uint4 *>(a) + 1);
            }
        }
#pragma unroll
    for (int q = 0; q < kRowsAThread; ++q) {
        if (q >= rows) break;
        const int back = (int)((reinterpret_cast<uintptr_t>(dst + q * m.ld_dst) & 15) / 2);
        const int lo = column < back ? back : 0, hi = min(left + back, 8);             // values of the piece that exist
        uint16_t *to = dst + q * m.ld_dst - back;
        const uint16_t *from = src + q * m.ld_src - back;
        if (m.src && !(wide >> q & 1)) {
            for (int i = lo; i < hi; ++i) to[i] = from[i];
            continue;
        }
        uint32_t c[8] = {v[q].x, v[q].y, v[q].z, v[q].w, w[q].x, w[q].y, w[q].z, w[q].w};
        if (m.src) shift_words(c, (uint32_t)reinterpret_cast<uintptr_t>(from) & 15);
        else c[0] = c[1] = c[2] = c[3] = 0;
        if (lo == 0 && hi == 8) {
            *reinterpret_cast<uint4 *>(to) = make_uint4(c[0], c[1], c[2], c[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= lo && i < hi) to[i] = (uint16_t)(c[i / 2] >> (16 * (i & 1)));
        }
    }
}

template <class T, int ACT>
cudaError_t column_pass(OperatorLaunch &l, const ColumnPass &c)
{
    PassParams<T> p{};
    int64_t ranges = 0;
    bool exact = (!c.z.p || aligned_rows(c.z, 2)) && (!c.out.p || aligned_rows(c.out, 2));
    int64_t rows = 0;
    for (const ColumnPass::Part &q : c.part) {
        if (!q.x.p) continue;
        auto &to = p.part[p.n++];
        if (q.partials) to.partials = (const float *)q.x.p;
        else to.x = (const T *)q.x.p;
        to.ld = q.x.ld;
        to.cols = q.cols;
        to.rows = q.partials ? q.partials : c.rows;
        rows = to.rows > rows ? to.rows : rows;
        to.sums = q.sums;
        to.first = (int)ranges;
        ranges += ceil_div(q.cols, kColsPerBlock);
        exact = exact && (q.partials || (q.cols % 8 == 0 && aligned_rows(q.x, 2)));
    }
    if (p.n == 0) return cudaSuccess;
    p.z = (const T *)c.z.p;
    p.ld_z = c.z.ld;
    p.out = (T *)const_cast<void *>(c.out.p);
    p.ld_out = c.out.ld;
    p.vec_out = aligned_rows(c.out, 2);
    p.wide = c.sums_type == DISTSIM_F32;
    p.partial = c.partial;
    p.counters = c.counters;
    return launch_kernel(l, kEarly, exact ? column_pass_kernel<T, ACT, true> : column_pass_kernel<T, ACT, false>, (unsigned)ranges,
                         (unsigned)row_runs(rows, ranges, l.sm_count), 256, 0, 0, p);
}

template <class T>
cudaError_t column_pass_of(OperatorLaunch &l, const ColumnPass &c)
{
    switch (c.z.p ? c.act : DISTSIM_ACT_NONE) {
    case DISTSIM_ACT_RELU: return column_pass<T, DISTSIM_ACT_RELU>(l, c);
    case DISTSIM_ACT_GELU: return column_pass<T, DISTSIM_ACT_GELU>(l, c);
    case DISTSIM_ACT_GELU_TANH: return column_pass<T, DISTSIM_ACT_GELU_TANH>(l, c);
    case DISTSIM_ACT_SILU: return column_pass<T, DISTSIM_ACT_SILU>(l, c);
    default: return column_pass<T, DISTSIM_ACT_NONE>(l, c);
    }
}

}  // namespace

int64_t column_pass_partials(int64_t cols, int sm_count)
{
    // `ranges` ranges are cut into at most ceil(kBlocksPerSm SMs / ranges) runs
    return ((int64_t)sm_count * kBlocksPerSm + ceil_div(cols, kColsPerBlock) + kPassParts) * kColsPerBlock;
}

cudaError_t launch_column_pass(OperatorLaunch &l, const ColumnPass &c)
{
    return c.type == DISTSIM_F16 ? column_pass_of<__half>(l, c) : column_pass_of<__nv_bfloat16>(l, c);
}

cudaError_t launch_moves(OperatorLaunch &l, const Move *moves, int n)
{
    Moves all{};
    uint64_t blocks = 0;
    for (int i = 0; i < n; ++i) {
        const Move &m = moves[i];
        if (m.rows < 1 || m.cols < 1) continue;
        const bool aligned = (reinterpret_cast<uintptr_t>(m.dst) & 15) == 0 && (m.ld_dst % 8 == 0 || m.rows == 1);
        all.m[all.n] = m;
        all.pieces[all.n] = (int32_t)((m.cols + (aligned ? 7 : 14)) / 8);
        all.first[all.n++] = (uint32_t)blocks;
        blocks += (uint64_t)ceil_div(ceil_div(m.rows, kRowsAThread) * (int64_t)all.pieces[all.n - 1], 256);
    }
    if (blocks == 0) return cudaSuccess;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_kernel(l, kEarly, move_kernel, (unsigned)blocks, 1, 256, 0, 0, all);
}

}  // namespace distsim
