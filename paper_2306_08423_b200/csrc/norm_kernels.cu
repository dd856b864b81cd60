// The residual connection around a block: norms after and before it, gate, residual scale, dropout.
//
//   t = norm(x) w1 + b1;  h = alpha r + gate dropout(t);  y = norm(h) w2 + b2
//
// A team of one or a few warps holds a row in registers, up to 32 columns a thread (16 backward),
// so every value is read and written once whatever the number of norms, and barriers are few; many
// teams share an SM.  Rows come into shared memory by bulk copies: forward as soon as a tensor's part
// of a row is in registers, the next row's is on its way; backward a row ahead, all tensors behind one
// barrier.  Arithmetic goes in pairs of floats where both halves take the same steps; dropout's mask is
// computed from its counter where it is needed.  Instructions fill 55 to 62 % of the issue slots (DRAM: 31 to
// 42 %), in the forward pass a third of them the generator's; the rest is waiting for a row's exchanges,
// which few warps an SM (12 backward) do not cover.  Backward, a thread also keeps four sums of its columns
// in registers, so rows of more than 4096 columns (2048 in 32 bits and backward) are held by the 2, 4 or 8
// blocks of a cluster, which send each other their parts of a row's sums (asynchronous stores that complete
// on the receiver's barrier; a cluster-wide barrier would wait for the row's global stores instead), and a
// row's last sums go in one exchange with the next row's statistics.  Statistics are joined as (mean,
// sum of squared distances from the mean) - the pairwise update of Chan, Golub and LeVeque - which
// takes one exchange and does not cancel; a warp that a row fills partly takes its own in two passes.
//
// Measured (bf16, of the copy bandwidth of 6.46 TB/s), with both norms, gate and dropout of 0.1.  Forward,
// root-mean-square / layer norms: 32768 x 2048 138 / 149 us (60 / 56 %; 98 / 109 us without dropout), 8192 x 12288
// 249 / 271 us.  Backward with all gradients, layer norms: 8192 x 12288 471 us (40 %), 32768 x 2048 336 us.  Rows
// that do not fill whole warps' pieces, forward (root-mean-square) / backward (layer) of 32768: 2056 columns
// 195 / 522 us, 2047: 260 / 704 us (element-wise accesses: 584 / 1133 us).  512 x 768 (f32) forward with the norm
// behind only 5 us, of which most is a launch's and a row's latency.
//
// Backward: with m = mask / (1 - p), hat(v) = (v - mean) / sd,
//   a = dy w2,   dH = dh + (a - mean(a) - hat(h) mean(a hat(h))) / sd_h,   dr = alpha dH,
//   q = m dH,    b = gate q w1,   dx = (b - mean(b) - hat(x) mean(b hat(x))) / sd_x,
// and every parameter's gradient follows from four column sums:
//   S0 = sum q, S1 = sum q hat(x) (q x without the first norm), S2 = sum dy hat(h), S3 = sum dy:
//   dgate = w1 S1 + b1 S0,  dw1 = gate S1,  db1 = gate S0,  dw2 = S2,  db2 = S3.
// A thread owns its columns' sums (no atomics, fixed order), a block joins its teams' and leaves one
// partial; a second kernel adds the blocks' partials in order.
#include <type_traits>

#include "operators.h"
#include "pairs.cuh"
#include "tensor_core.cuh"

namespace distsim {

namespace {

constexpr int kMaxEntries = 32;                  // warps that share a row, over a cluster
constexpr int kForwardThreads = 128, kBackwardThreads = 192;          // of a block, at most

struct NormParams {
    int64_t tokens;
    int32_t cols, team_threads, teams;           // threads of a block that share a row (or its part); rows of a block
    int32_t cluster;                             // blocks that share a row
    int32_t share, width;                        // a block's columns of a row; columns that its team can hold
    int32_t rms;
    float alpha, eps;
    uint32_t threshold;
    float keep_scale;
    uint64_t seed, offset;
    const void *x, *residual, *h_in, *dy, *dh;
    void *h, *y, *dx, *dresidual;
    const void *gate, *w1, *b1, *w2, *b2;
    int64_t ld_x, ld_residual, ld_h, ld_y, ld_dy, ld_dh, ld_dx, ld_dresidual;
    uint32_t ref_start, ref_pitch, ref_shift;    // addresses of the rows that phases follow (low words); log2 of a value's bytes
    float *partial;
    int32_t *status;
    int32_t polls;                               // of a wait, before it gives up
    bool sum_q, sum_qx, sum_y;                   // which column sums are wanted: S0; S1; S2 and S3
    int32_t slot[4];                             // place of S0..S3 among the kept sums (-1: not kept)
    int32_t n_sums;
    bool all_in_phase, all_aligned;              // all rows lie like the reference's; all are whole eights on 16-byte boundaries
};

// How rows lie.  kWhole: every thread's eights exist and start on 16-byte boundaries.  kAligned: so
// do those that exist, in whole eights.  kPhased: a row may start and end anywhere, in all tensors as
// far from a boundary.  kAny: no assumption.
enum Layout { kWhole, kAligned, kPhased, kAny };

// What the warps of a team share.
struct Scratch {
    float4 entry[2][2][kMaxEntries];             // a warp's numbers in an exchange, four and four
    uint64_t arrived[2];                         // all entries of an exchange are here (cluster)
    uint64_t row[4];                             // a tensor's part of a row is here
};

template <int NV>
struct Team {
    int id, thread, threads, cluster;
    uint32_t rank;
    Scratch *scratch;
    int32_t *status, polls;
    int exchanges = 0;
    // A wait of this thread gave up.  It goes through the remaining rows without waiting, starting copies or
    // sending, and in the end waits once for copies started before; the others' waits then give up, too.
    bool dead = false;
    int lack = 0;                                // columns that this warp could hold and the row does not have
    int phase;                                   // values that the team's pieces start before its columns
    float cols, inv_n;                           // columns of a row, and 1 / that
    float weight = 0.f;                          // columns of the warp whose entry the lane joins

    // row_arrivals: of the barrier of a row's copies
    __device__ __forceinline__ Team(const NormParams &p, Scratch *all, int row_arrivals)
    {
        threads = p.team_threads;
        id = threadIdx.x / p.team_threads;
        thread = threadIdx.x - id * p.team_threads;
        cluster = p.cluster;
        rank = p.cluster > 1 ? cluster_rank() : 0;
        scratch = all + id;
        status = p.status;
        polls = p.polls;
        cols = (float)p.cols;
        inv_n = 1.f / cols;
        phase = (int)(((p.ref_start + (uint32_t)((blockIdx.x / p.cluster) * p.teams + id) * p.ref_pitch) & 15) >> p.ref_shift);
        if (thread == 0) {
            for (int i = 0; i < 2; ++i) mbar_init(smem_addr(&scratch->arrived[i]), 1);
            for (int i = 0; i < 4; ++i) mbar_init(smem_addr(&scratch->row[i]), row_arrivals);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
        if (cluster > 1) cluster_sync();
        for (int i = 0, e = threadIdx.x & 31; i < 2; ++i) {
            const int warps = threads >> 5, of = e / warps, w = e - of * warps, columns = min(p.share, p.cols - of * p.share);
            int n = 0;
            for (int j = 0; j < NV; ++j) {
                const int at = (w + j * warps) * 256 - phase;        // the warp's first column of piece j
                n += max(0, min(at + 256, columns) - max(at, 0));
            }
            if (i == 0) weight = (float)n;
            else lack = 256 * NV - n;
            e = (int)rank * warps + (thread >> 5);
        }
        grid_let_next();
        grid_wait();
    }
    // After the last exchange, by every thread of the block.
    __device__ __forceinline__ void close() const
    {
        if (dead)                                // copies that were started before: of either phase that may be under way
            for (int i = 0; i < 8; ++i) mbar_wait(smem_addr(&scratch->row[i >> 1]), (uint32_t)i & 1, kDrainPolls);
        __syncthreads();
        if (cluster > 1) cluster_sync();
    }
    __device__ __forceinline__ void sync() const
    {
        if (threads == 32) __syncwarp();
        else asm volatile("bar.sync %0, %1;" :: "r"(1 + id), "r"(threads) : "memory");
    }
    __device__ __forceinline__ void wait(uint64_t *bar, int phase)
    {
        if (!dead && !mbar_wait(smem_addr(bar), (uint32_t)phase & 1, polls)) {
            dead = true;
            *reinterpret_cast<volatile int32_t *>(status) = DISTSIM_E_TIMEOUT;
            mbar_wait(smem_addr(bar), (uint32_t)phase & 1, kDrainPolls);     // what was sent stays in flight no longer
        }
    }
    template <int N>
    static __device__ __forceinline__ float4 shuffle(float4 v, int o)
    {
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
        r.x = __shfl_xor_sync(~0u, v.x, o);
        if (N > 1) r.y = __shfl_xor_sync(~0u, v.y, o);
        if (N > 2) r.z = __shfl_xor_sync(~0u, v.z, o);
        if (N > 3) r.w = __shfl_xor_sync(~0u, v.w, o);
        return r;
    }
    template <int N>
    static __device__ __forceinline__ float4 add(float4 a, float4 b)
    {
        a.x += b.x;
        if (N > 1) a.y += b.y;
        if (N > 2) a.z += b.z;
        if (N > 3) a.w += b.w;
        return a;
    }
    // One (N 2) or two (N 4) rows' moments (mean, sum of squares about it) over equal counts.
    template <int N>
    static __device__ __forceinline__ float4 join(float4 a, float4 b, float half)
    {
        const float d = b.x - a.x;
        a.y = fmaf(d * d, half, a.y + b.y);
        a.x = 0.5f * (a.x + b.x);
        if (N > 2) {
            const float e = b.z - a.z;
            a.w = fmaf(e * e, half, a.w + b.w);
            a.z = 0.5f * (a.z + b.z);
        }
        return a;
    }
    // What all warps hold goes to all of them.  Entries alternate between two buffers, so that one
    // barrier an exchange is enough; whatever a thread read before it has been read by all after.
    template <int FOURS>
    __device__ __forceinline__ const float4 (*share(const float4 (&v)[FOURS]))[kMaxEntries]
    {
        const int turn = exchanges & 1, warps = threads >> 5, lane = thread & 31;
        float4 (*entry)[kMaxEntries] = scratch->entry[turn];
        if (cluster == 1) {
            if (lane == 0)
#pragma unroll
                for (int k = 0; k < FOURS; ++k) entry[k][thread >> 5] = v[k];
            sync();
        } else {
            const uint32_t bar = smem_addr(&scratch->arrived[turn]);
            if (thread == 0 && !dead) mbar_expect(bar, (uint32_t)(warps * cluster * 16 * FOURS));
            __syncwarp();
            if (lane < cluster && !dead)
#pragma unroll
                for (int k = 0; k < FOURS; ++k)
                    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                                 :: "r"(cluster_addr(smem_addr(entry[k] + rank * warps + (thread >> 5)), (uint32_t)lane)), "f"(v[k].x), "f"(v[k].y),
                                    "f"(v[k].z), "f"(v[k].w), "r"(cluster_addr(bar, (uint32_t)lane)) : "memory");
            wait(&scratch->arrived[turn], exchanges >> 1);
            __syncwarp();
        }
        ++exchanges;
        return entry;
    }
    // v / columns of a row, as division rounds it: the mean of a row of equal values is their value.
    __device__ __forceinline__ float divided(float v) const
    {
        const float q = v * inv_n;
        return fmaf(fmaf(-q, cols, v), inv_n, q);
    }
    // Joins the warps' entries (sums, or moments); every warp does so for itself.
    template <int N, bool MOMENTS>
    __device__ __forceinline__ float4 join_entries(const float4 *entry) const
    {
        const int lane = threadIdx.x & 31, count = (threads >> 5) * cluster;
        const float4 own = lane < count ? entry[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
        const float n = lane < count ? weight : 0.f;
        float4 v = own;
        if (MOMENTS) { v.x *= n; v.z *= n; }
#pragma unroll
        for (int o = kMaxEntries / 2; o > 0; o >>= 1) v = add<N>(v, shuffle<N>(v, o));
        if (MOMENTS) {
            v.x = divided(v.x);
            if (N > 2) v.z = divided(v.z);
            const float d = own.x - v.x, e = own.z - v.z;
            float4 q = make_float4(d * d * n, e * e * n, 0.f, 0.f);
#pragma unroll
            for (int o = kMaxEntries / 2; o > 0; o >>= 1) q = add<N / 2>(q, shuffle<N / 2>(q, o));
            v.y += q.x;
            v.w += q.y;
        }
        return v;
    }
    // Over the warp: sums, or moments of 8 NV values a thread (a partly filled warp has its own already).
    template <int N, bool MOMENTS>
    __device__ __forceinline__ float4 over_warp(float4 v) const
    {
        if (MOMENTS && lack) return v;
        float half = 4.f * NV;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1, half *= 2.f) v = MOMENTS ? join<N>(v, shuffle<N>(v, o), half) : add<N>(v, shuffle<N>(v, o));
        return v;
    }
    __device__ __forceinline__ bool one_warp() const { return threads == 32 && cluster == 1; }
    template <int N, bool MOMENTS>
    __device__ __forceinline__ float4 over_row(float4 v)
    {
        const float4 all[1] = {over_warp<N, MOMENTS>(v)};
        return one_warp() ? all[0] : join_entries<N, MOMENTS>(share<1>(all)[0]);
    }
    // Sums of the first N numbers over the row.
    template <int N>
    __device__ __forceinline__ float4 sum(float4 v) { return over_row<N, false>(v); }
    // Moments over the row from every thread's, of 8 NV values each.  N: 2 (one row) or 4.
    template <int N>
    __device__ __forceinline__ float4 moments(float4 v) { return over_row<N, true>(v); }
    // Two sums of a row and the moments (sums of squares with SQUARES) of two others, in one exchange.
    template <bool SQUARES>
    __device__ __forceinline__ void sum_and_moments(float4 &s, float4 &m)
    {
        const float4 all[2] = {over_warp<2, false>(s), SQUARES ? over_warp<2, false>(m) : over_warp<4, true>(m)};
        if (one_warp()) {
            s = all[0];
            m = all[1];
            return;
        }
        const float4 (*entry)[kMaxEntries] = share<2>(all);
        s = join_entries<2, false>(entry[0]);
        m = SQUARES ? join_entries<2, false>(entry[1]) : join_entries<4, true>(entry[1]);
    }
    static __device__ __forceinline__ float own_sum(const Oct (&f)[NV])
    {
        Pair s[4] = {f[0].v[0], f[0].v[1], f[0].v[2], f[0].v[3]};
#pragma unroll
        for (int j = 1; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = add2(s[i], f[j].v[i]);
        return total(add2(add2(s[0], s[1]), add2(s[2], s[3])));
    }
    // Squares about `mean`.
    static __device__ __forceinline__ float own_squares(const Oct (&f)[NV], float mean)
    {
        Pair s[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};
        const Pair m = both(-mean);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Pair d = add2(f[j].v[i], m);
                s[i] = fma2(d, d, s[i]);
            }
        return total(add2(add2(s[0], s[1]), add2(s[2], s[3])));
    }
    // Values of the thread's first piece that lie before the row's (share's) first.
    template <Layout L>
    __device__ __forceinline__ int lead() const { return L >= kPhased && thread == 0 ? phase : 0; }
    // Puts `other` in place of the values that do not exist: the row ends `valid` columns behind the
    // thread's first one and starts `lead` behind it.
    template <Layout L>
    __device__ __forceinline__ void trim(Oct (&f)[NV], int valid, float other) const
    {
        if (L == kWhole || !lack) return;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (valid - j * threads * 8 < 8) cut8(f[j], valid - j * threads * 8, other);
        if (L >= kPhased && thread == 0) cut_front8(f[0], phase, other);
    }
    // The same, of values read: aligned rows bring zeros.
    template <Layout L>
    __device__ __forceinline__ void trim_read(Oct (&f)[NV], int valid) const
    {
        if (L >= kPhased) trim<L>(f, valid, 0.f);
    }
    // Moments of the thread's values (zero beyond the row); in a warp that the row fills partly, of the
    // warp's: the sum first, then squares about its mean.  valid: as in trim.
    template <Layout L>
    __device__ __forceinline__ void own_moments(const Oct (&f)[NV], int valid, float &mean, float &m2) const
    {
        if (L == kWhole || !lack) {
            mean = own_sum(f) * (0.125f / NV);
            m2 = own_squares(f, mean);
            return;
        }
        const int n = 256 * NV - lack;
        mean = n ? over_warp<1, false>(make_float4(own_sum(f), 0.f, 0.f, 0.f)).x / (float)n : 0.f;
        Oct d[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[j].v[i] = add2(f[j].v[i], both(-mean));
        trim<L>(d, valid, 0.f);
        m2 = over_warp<1, false>(make_float4(own_squares(d, 0.f), 0.f, 0.f, 0.f)).x;
    }
    // Mean and reciprocal deviation of a row's values, zero beyond the row.
    template <Layout L>
    __device__ __forceinline__ void statistics(const NormParams &p, const Oct (&f)[NV], int valid, float &mean, float &rstd)
    {
        if (p.rms) {
            mean = 0.f;
            rstd = rsqrtf(sum<1>(make_float4(own_squares(f, 0.f), 0.f, 0.f, 0.f)).x * inv_n + p.eps);
        } else {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            own_moments<L>(f, valid, v.x, v.y);
            v = moments<2>(v);
            mean = v.x;
            rstd = rsqrtf(v.y * inv_n + p.eps);
        }
    }
};

template <class T>
__device__ __forceinline__ Oct read_shared8(uint32_t from)
{
    Eight<T> e;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * 8 / 16); ++i)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(e.w[i].x), "=r"(e.w[i].y), "=r"(e.w[i].z), "=r"(e.w[i].w)
                     : "r"(from + 16 * i) : "memory");
    return widen(e);
}

// ---- rows of any alignment ---------------------------------------------------------------------
// A row (or a block's share of one) that does not start or end on a 16-byte boundary is copied from
// the boundary before to the boundary behind; what is read beyond its ends lies between the tensor's
// first and last element, except in the first and last row, which are read element by element.  A
// team's rows lie so far apart that all start as far behind a boundary (the phase), in every tensor
// whose rows lie like the reference's; its threads' pieces start that much before its columns, so that
// they are whole 16-byte pieces of memory.  Other tensors' pieces are shifted in registers and written
// value by value.

// Eight values from a shared address.
template <class T>
__device__ __forceinline__ Oct read_shifted8(uint32_t from)
{
    constexpr int kWords = (int)sizeof(T) * 2;
    const uint32_t off = from & 15;
    uint32_t c[kWords + 4];
#pragma unroll
    for (int i = 0; i < kWords / 4 + 1; ++i)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(c[4 * i]), "=r"(c[4 * i + 1]), "=r"(c[4 * i + 2]), "=r"(c[4 * i + 3])
                     : "r"(from - off + 16 * i) : "memory");
    shift_words(c, off);
    Eight<T> e;
    uint32_t *w = reinterpret_cast<uint32_t *>(e.w);
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = c[i];
    return widen(e);
}

__device__ __forceinline__ void put_shared(uint32_t at, __nv_bfloat16 v) { asm volatile("st.shared.u16 [%0], %1;" :: "r"(at), "h"(__bfloat16_as_ushort(v)) : "memory"); }
__device__ __forceinline__ void put_shared(uint32_t at, __half v) { asm volatile("st.shared.u16 [%0], %1;" :: "r"(at), "h"(__half_as_ushort(v)) : "memory"); }
__device__ __forceinline__ void put_shared(uint32_t at, float v) { asm volatile("st.shared.f32 [%0], %1;" :: "r"(at), "f"(v) : "memory"); }

// Eight values to p on, those from `lead` up to `left`.
template <class T, Layout L>
__device__ __forceinline__ void write_columns(T *p, int lead, int left, const Oct &o)
{
    if (L >= kPhased && (lead > 0 || left < 8 || (L == kAny && (reinterpret_cast<uintptr_t>(p) & 15)))) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = halves(o.v[i / 2]);
            if (i >= lead && i < left) p[i] = from_float<T>(i & 1 ? f.y : f.x);
        }
    } else if (L != kAligned || left > 0) {
        write8<T, true>(p, 8, true, o);
    }
}

// A tensor's rows on their way into shared memory.  `columns`: of the team's share that exist.
template <class T, int NV, Layout L>
struct Rows {
    const T *p;                                  // the tensor at the team's first column; null: not there
    int64_t ld, tokens;
    int columns;
    uint32_t start, pitch;                       // low words of the first row's address and of the rows' distance
    bool first_edge, last_edge;                  // whether the first (last) rows would be read beyond the tensor's ends
    bool in_phase;                               // rows lie like the reference's
    int ends;                                    // rows from which 16 bytes further is out of the tensor

    __device__ __forceinline__ void set(const NormParams &q, const void *tensor, int64_t ld_, int first)
    {
        p = tensor ? (const T *)tensor + first : nullptr;
        ld = ld_;
        tokens = q.tokens;
        columns = L == kWhole ? q.width : min(q.share, q.cols - first);
        start = (uint32_t)reinterpret_cast<uintptr_t>(p);
        pitch = (uint32_t)(ld * sizeof(T));
        in_phase = ((start ^ q.ref_start) & 15) == 0 && ((pitch ^ q.ref_pitch) & 15) == 0;
        ends = ld * (int64_t)sizeof(T) >= 16 ? 1 : 16;
        first_edge = ends > 1 || (start & 15);
        last_edge = ends > 1 || ((start + (uint32_t)(tokens - 1) * pitch + columns * sizeof(T)) & 15);
    }
    // Bytes of shared memory that hold a row wherever it starts; sixteen lie before.
    static __host__ __device__ __forceinline__ uint32_t room(int width) { return (uint32_t)(width * (int)sizeof(T) + (L >= kPhased ? 32 : 0)); }
    // How far behind a 16-byte boundary row r starts.
    __device__ __forceinline__ uint32_t offset(int64_t r) const { return (start + (uint32_t)r * pitch) & 15; }
    // By one thread: brings row r to `at` (its first value to the same place behind a 16-byte boundary,
    // from kPhased on) and arrives at `bar`.
    __device__ __forceinline__ void bring(uint32_t at, int64_t r, uint32_t bar) const
    {
        uint32_t n = (uint32_t)(columns * (int)sizeof(T));
        const T *const row = p + r * ld;
        const char *from = reinterpret_cast<const char *>(row);
        if (L >= kPhased) {
            const uint32_t off = offset(r), row_end = off + n;
            uint32_t begin = 0, end = (row_end + 15) & ~15u;
            if ((r < ends && first_edge) || (r >= tokens - ends && last_edge)) {
                // whole pieces within the row, the rest value by value
                begin = min((off + 15) & ~15u, end);
                end = max(row_end & ~15u, begin);
                for (uint32_t b = off; b < min(begin, row_end); b += (uint32_t)sizeof(T)) put_shared(at + b, row[(b - off) / (uint32_t)sizeof(T)]);
                for (uint32_t b = max(end, off); b < row_end; b += (uint32_t)sizeof(T)) put_shared(at + b, row[(b - off) / (uint32_t)sizeof(T)]);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            from += (int64_t)begin - (int64_t)off;
            at += begin;
            n = end - begin;
        }
        mbar_expect(bar, n);
        if (n) copy(at, from, n, bar);
    }
    // By every thread of the team, for `parts` tensors' parts: zeros where copies of aligned rows do not
    // reach.
    __device__ __forceinline__ static void clear(const NormParams &q, const Team<NV> &t, uint32_t at, int parts, int first)
    {
        if (L != kAligned) return;
        const int from = min(q.share, q.cols - first) * (int)sizeof(T) / 16, to = q.width * (int)sizeof(T) / 16;
        for (int k = 0; k < parts; ++k)
            for (int i = from + t.thread; i < to; i += t.threads)
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" :: "r"(at + (uint32_t)(k * to + i) * 16), "r"(0) : "memory");
    }
    __device__ __forceinline__ static void copy(uint32_t to, const void *from, uint32_t n, uint32_t bar)
    {
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     :: "r"(to), "l"(from), "r"(n), "r"(bar) : "memory");
    }
    // Piece j of row r, which was copied to `at`; beyond the row zeros, from kPhased on anything.
    __device__ __forceinline__ Oct read(const Team<NV> &t, uint32_t at, int64_t r, int j) const
    {
        at += (uint32_t)((t.thread + j * t.threads) * 8 * (int)sizeof(T));
        if (L != kAny || in_phase) return read_shared8<T>(at);
        return read_shifted8<T>(at + offset(r) - (uint32_t)(t.phase * (int)sizeof(T)));
    }
};

// One tensor's part of a row, refilled for the next row once it has been read.
template <class T, int NV, Layout L>
struct Ahead {
    Rows<T, NV, L> rows;
    uint32_t at;                                 // shared address
    uint64_t *bar;
    int seen = 0;

    __device__ __forceinline__ Ahead(const NormParams &q, const Team<NV> &t, const void *tensor, int64_t ld, int first, uint32_t smem, int slot)
    {
        rows.set(q, tensor, ld, first);
        at = smem + (uint32_t)slot * rows.room(q.width) + (L >= kPhased ? 16 : 0);
        bar = &t.scratch->row[slot];
    }
    // By every thread, once all have read the present row: starts copying row r, if there is one.
    __device__ __forceinline__ void start(const Team<NV> &t, int64_t r) const
    {
        if (!rows.p || t.thread != 0 || r >= rows.tokens || t.dead) return;
        rows.bring(at, r, smem_addr(bar));
    }
    __device__ __forceinline__ void wait(Team<NV> &t)
    {
        if (rows.p) t.wait(bar, seen++);
    }
    __device__ __forceinline__ Oct read(const Team<NV> &t, int64_t r, int j) const { return rows.read(t, at, r, j); }
};

// Several tensors' parts of a row and of the next one, each row's behind one barrier.
template <class T, int NV, Layout L, int TENSORS>
struct RowsAhead {
    Rows<T, NV, L> rows[TENSORS], mine;          // `mine`: the one that this thread copies
    uint32_t at, room;                           // shared address of the two rows; bytes of a tensor's place
    int seen = 0;

    __device__ __forceinline__ RowsAhead(const NormParams &q, uint32_t smem) : at(smem + (L >= kPhased ? 16 : 0)), room(Rows<T, NV, L>::room(q.width)) {}
    __device__ __forceinline__ void set(const NormParams &q, const Team<NV> &t, int k, const void *tensor, int64_t ld, int first)
    {
        rows[k].set(q, tensor, ld, first);
        if (t.thread == k) mine = rows[k];
    }
    // By every thread, once all have read the row whose place it takes: starts copying row r, if
    // there is one, into buffer `turn`, a thread a tensor.  Each arrives, be its tensor there or not.
    __device__ __forceinline__ void start(const Team<NV> &t, int64_t r, int turn) const
    {
        if (t.thread >= TENSORS || r >= rows[0].tokens || t.dead) return;
        const uint32_t bar = smem_addr(&t.scratch->row[turn]);
        if (mine.p) mine.bring(at + (turn * TENSORS + t.thread) * room, r, bar);
        else mbar_expect(bar, 0);
    }
    // Rows are waited for in order, in buffers 0, 1, 0, ..
    __device__ __forceinline__ void wait(Team<NV> &t)
    {
        t.wait(&t.scratch->row[seen & 1], seen >> 1);
        ++seen;
    }
    // Piece j of tensor k of row r, which is in buffer `turn`.
    __device__ __forceinline__ Oct read(const Team<NV> &t, int k, int64_t r, int j, int turn) const
    {
        return rows[k].read(t, at + (turn * TENSORS + k) * room, r, j);
    }
};

// A parameter's columns of a block, kept in shared memory for all its rows (zeros beyond the row):
// read for every row from L2 they would take more of its bandwidth than the rows themselves.
template <class T, int NV, Layout L>
struct Parameter {
    bool there;
    uint32_t at;

    // By every thread of the block; what a team holds from `first` on goes to `smem`, which moves on.
    // Without an alignment every team has its own, in its phase.
    __device__ __forceinline__ Parameter(const NormParams &q, const Team<NV> &t, const void *vector, int first, uint8_t *&smem)
        : there(vector != nullptr), at(smem_addr(smem))
    {
        if (!there) return;
        const T *p = (const T *)vector + first;
        const int columns = min(q.share, q.cols - first);
        if (L < kPhased) {
            for (int i = threadIdx.x; i < q.width * (int)sizeof(T) / 16; i += blockDim.x)
                reinterpret_cast<uint4 *>(smem)[i] = i < columns * (int)sizeof(T) / 16 ? reinterpret_cast<const uint4 *>(p)[i] : make_uint4(0, 0, 0, 0);
            smem += q.width * sizeof(T);
        } else {
            const uint32_t own = (uint32_t)(t.id * q.width * (int)sizeof(T));
            at += own;
            for (int i = t.thread; i < q.width; i += t.threads)
                reinterpret_cast<T *>(smem + own)[i] = i >= t.phase && i < columns + t.phase ? p[i - t.phase] : from_float<T>(0.f);
            smem += q.width * q.teams * sizeof(T);
        }
    }
    __device__ __forceinline__ Oct read(const Team<NV> &t, int j) const { return read_shared8<T>(at + (uint32_t)((t.thread + j * t.threads) * 8 * (int)sizeof(T))); }
};

// SplitMix64's finaliser (Steele, Lea, Flood 2014).
__device__ __forceinline__ uint64_t finalise(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
// State of the generator at a column's draw, which an even column and the next share.
__device__ __forceinline__ uint64_t draw_state(const NormParams &p, int64_t row, int col)
{
    const uint64_t draw = p.offset + (uint64_t)row * (uint64_t)((p.cols + 1) >> 1) + (uint64_t)(col >> 1);
    return p.seed + (draw + 1) * 0x9E3779B97F4A7C15ull;
}
// Zeros what dropout does not keep of eight values (and of `also`).  `odd`: the first is the second of
// its draw.
template <bool ALSO>
__device__ __forceinline__ void drop8(const NormParams &p, uint64_t state, bool odd, Oct &v, Oct &also)
{
    uint32_t draw[8];
    if (!odd) {
#pragma unroll
        for (int i = 0; i < 4; ++i, state += 0x9E3779B97F4A7C15ull) {
            const uint64_t z = finalise(state);
            draw[2 * i] = (uint32_t)z;
            draw[2 * i + 1] = (uint32_t)(z >> 32);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 5; ++i, state += 0x9E3779B97F4A7C15ull) {
            const uint64_t z = finalise(state);
            if (i > 0) draw[2 * i - 1] = (uint32_t)z;
            if (i < 4) draw[2 * i] = (uint32_t)(z >> 32);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool first = draw[2 * i] >= p.threshold, second = draw[2 * i + 1] >= p.threshold;
        const float2 f = halves(v.v[i]);
        v.v[i] = make_pair2(first ? f.x : 0.f, second ? f.y : 0.f);
        if (ALSO) {
            const float2 g = halves(also.v[i]);
            also.v[i] = make_pair2(first ? g.x : 0.f, second ? g.y : 0.f);
        }
    }
}

__device__ __forceinline__ void scale8(Oct &v, float f)
{
    const Pair s = both(f);
#pragma unroll
    for (int i = 0; i < 4; ++i) v.v[i] = mul2(v.v[i], s);
}
__device__ __forceinline__ Oct times8(const Oct &a, const Oct &b)
{
    Oct r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = mul2(a.v[i], b.v[i]);
    return r;
}
// (v - mean) * scale, in this order: a row of equal values becomes zeros, not what rounding mean * scale leaves.
__device__ __forceinline__ void centre8(Oct &v, float mean, float scale)
{
    const Pair s = both(scale), m = both(-mean);
#pragma unroll
    for (int i = 0; i < 4; ++i) v.v[i] = mul2(add2(v.v[i], m), s);
}
// v * weight + bias
template <class P, class TEAM>
__device__ __forceinline__ void affine8(Oct &v, const TEAM &team, const P &weight, const P &bias, int j)
{
    const Oct w = weight.read(team, j);
    if (bias.there) {
        const Oct b = bias.read(team, j);
#pragma unroll
        for (int i = 0; i < 4; ++i) v.v[i] = fma2(v.v[i], w.v[i], b.v[i]);
    } else {
        v = times8(v, w);
    }
}
__device__ __forceinline__ void add_to(Oct &sums, const Oct &v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) sums.v[i] = add2(sums.v[i], v.v[i]);
}

template <class T, int NV, Layout L>
__global__ void __launch_bounds__(kForwardThreads, L == kWhole || NV < 4 ? 5 : 4)
residual_norm_forward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ Scratch scratch[4];
    Team<NV> team(p, scratch, 1);
    const int step = p.team_threads * 8, first = (int)team.rank * p.share, phase = L >= kPhased ? team.phase : 0, c = first - phase + team.thread * 8;
    const int valid = min(p.share, p.cols - first) + phase - team.thread * 8;            // columns from the thread's first on
    const int lead = team.template lead<L>();
    const int64_t stride = (int64_t)(gridDim.x / p.cluster) * p.teams;
    int64_t row = (int64_t)(blockIdx.x / p.cluster) * p.teams + team.id;
    uint8_t *free = dynamic;
    const Parameter<T, NV, L> w1(p, team, p.w1, first, free), b1(p, team, p.b1, first, free), gate(p, team, p.gate, first, free), w2(p, team, p.w2, first, free),
        b2(p, team, p.b2, first, free);
    const uint32_t smem = smem_addr(free) + (uint32_t)team.id * 2 * Rows<T, NV, L>::room(p.width);
    Rows<T, NV, L>::clear(p, team, smem, 2, first);
    __syncthreads();
    Ahead<T, NV, L> x(p, team, p.x, p.ld_x, first, smem, 0), res(p, team, p.residual, p.ld_residual, first, smem, 1);
    x.start(team, row);
    res.start(team, row);
    for (; row < p.tokens; row += stride) {
        Oct v[NV];
        float mean, rstd;
        x.wait(team);
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = x.read(team, row, j);
        team.template trim_read<L>(v, valid);
        if (p.w1) {
            team.template statistics<L>(p, v, valid, mean, rstd);
            x.start(team, row + stride);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                centre8(v[j], mean, rstd);
                affine8(v[j], team, w1, b1, j);
            }
        }
        if (p.threshold) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                scale8(v[j], p.keep_scale);
                drop8<false>(p, draw_state(p, row, c + j * step), L >= kPhased && (c & 1), v[j], v[j]);
            }
        }
        if (p.gate) {
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = times8(v[j], gate.read(team, j));
        }
        if (res.rows.p) {
            const Pair alpha = both(p.alpha);
            res.wait(team);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const Oct r = res.read(team, row, j);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j].v[i] = fma2(alpha, r.v[i], v[j].v[i]);
            }
        }
        team.template trim<L>(v, valid, 0.f);                                        // the next statistics see the row only
        if (p.h) {
            T *h = (T *)p.h + row * p.ld_h + c;
#pragma unroll
            for (int j = 0; j < NV; ++j) write_columns<T, L>(h + j * step, j == 0 ? lead : 0, valid - j * step, v[j]);
        }
        if (p.w2) team.template statistics<L>(p, v, valid, mean, rstd);
        else team.sync();
        if (!p.w1) x.start(team, row + stride);
        res.start(team, row + stride);
        if (p.w2) {
            T *y = (T *)p.y + row * p.ld_y + c;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                centre8(v[j], mean, rstd);
                affine8(v[j], team, w2, b2, j);
                write_columns<T, L>(y + j * step, j == 0 ? lead : 0, valid - j * step, v[j]);
            }
        }
    }
    team.close();
}

// A thread holds the four sums of its columns in registers.  Shared memory: the parameters and the
// teams' rows; in the end, with several teams, their sums.
template <class T, int NV, Layout L>
__global__ void __launch_bounds__(kBackwardThreads, 2)
residual_norm_backward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ Scratch scratch[4];
    Team<NV> team(p, scratch, 4);
    const int step = p.team_threads * 8, width = step * NV;
    Oct sum_q[NV], sum_qx[NV], sum_yh[NV], sum_y[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum_q[j].v[i] = sum_qx[j].v[i] = sum_yh[j].v[i] = sum_y[j].v[i] = both(0.f);
    const int first = (int)team.rank * p.share, phase = L >= kPhased ? team.phase : 0, c = first - phase + team.thread * 8;
    const int valid = min(p.share, p.cols - first) + phase - team.thread * 8;            // columns from the thread's first on
    const int lead = team.template lead<L>();
    const float inv_n = team.inv_n;
    const bool need_x = p.w1 || p.sum_qx;
    const int64_t stride = (int64_t)(gridDim.x / p.cluster) * p.teams;
    int64_t row = (int64_t)(blockIdx.x / p.cluster) * p.teams + team.id;
    uint8_t *free = dynamic;
    const Parameter<T, NV, L> w1(p, team, p.w1, first, free), gate(p, team, p.gate, first, free), w2(p, team, p.w2, first, free);
    enum { X, H, DY, DH };
    RowsAhead<T, NV, L, 4> in(p, smem_addr(free) + (uint32_t)team.id * 8 * Rows<T, NV, L>::room(p.width));
    Rows<T, NV, L>::clear(p, team, in.at, 8, first);
    __syncthreads();
    in.set(p, team, X, need_x ? p.x : nullptr, p.ld_x, first);
    in.set(p, team, H, p.w2 ? p.h_in : nullptr, p.ld_h, first);
    in.set(p, team, DY, p.w2 ? p.dy : nullptr, p.ld_dy, first);
    in.set(p, team, DH, p.dh, p.ld_dh, first);
    const bool joined = p.w1 && p.dx;            // the last sums of a row are taken over it
    // A turn works on a row (not in the first one) up to its last sums, then on the statistics of the
    // next: one exchange takes both.
    float mean[2] = {0.f, 0.f}, rstd[2] = {1.f, 1.f};                    // of h and x
    int turn = 1;
    in.start(team, row, 0);
    for (row -= stride; row < p.tokens; row += stride, turn ^= 1) {
        const bool present = row >= 0;
        const int64_t next = row + stride;
        Oct dh[NV], hat[NV];
        const float mean_x = mean[1], rstd_x = rstd[1];
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (present) {
            in.start(team, next, turn ^ 1);
            if (p.w2) {
                Pair s0 = both(0.f), s1 = both(0.f);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    hat[j] = in.read(team, H, row, j, turn);
                    dh[j] = in.read(team, DY, row, j, turn);
                }
                team.template trim_read<L>(hat, valid);
                team.template trim_read<L>(dh, valid);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    centre8(hat[j], mean[0], rstd[0]);
                    const Oct w = w2.read(team, j), f = dh[j];                       // zero beyond the row
                    const Oct t = times8(f, hat[j]);
                    dh[j] = times8(f, w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s0 = add2(s0, dh[j].v[i]);
                        s1 = fma2(t.v[i], w.v[i], s1);
                    }
                    if (p.sum_y) {
                        add_to(sum_y[j], f);
                        add_to(sum_yh[j], t);
                    }
                }
                const float4 a = team.template sum<2>(make_float4(total(s0), total(s1), 0.f, 0.f));
                const Pair a0 = both(p.rms ? 0.f : -a.x * inv_n), a1 = both(-a.y * inv_n), r = both(rstd[0]);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    Oct f;
                    if (in.rows[DH].p) f = in.read(team, DH, row, j, turn);
                    else f.v[0] = f.v[1] = f.v[2] = f.v[3] = both(0.f);
#pragma unroll
                    for (int i = 0; i < 4; ++i) dh[j].v[i] = fma2(r, fma2(hat[j].v[i], a1, add2(dh[j].v[i], a0)), f.v[i]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < NV; ++j) dh[j] = in.read(team, DH, row, j, turn);
            }
            if (p.dresidual) {
                T *dr = (T *)p.dresidual + row * p.ld_dresidual + c;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    Oct t = dh[j];
                    scale8(t, p.alpha);
                    write_columns<T, L>(dr + j * step, j == 0 ? lead : 0, valid - j * step, t);
                }
            }
            if (need_x) {
#pragma unroll
                for (int j = 0; j < NV; ++j) hat[j] = in.read(team, X, row, j, turn);
                team.template trim_read<L>(hat, valid);
                if (p.w1)
#pragma unroll
                    for (int j = 0; j < NV; ++j) centre8(hat[j], mean_x, rstd_x);
            }
            if (p.threshold) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    scale8(dh[j], p.keep_scale);
                    // without a norm x is a factor of dropout's input: what was dropped counts nowhere, be it infinite
                    if (need_x && !p.w1) drop8<true>(p, draw_state(p, row, c + j * step), L >= kPhased && (c & 1), dh[j], hat[j]);
                    else drop8<false>(p, draw_state(p, row, c + j * step), L >= kPhased && (c & 1), dh[j], dh[j]);
                }
            }
            team.template trim<L>(dh, valid, 0.f);
            if (p.sum_q) {
#pragma unroll
                for (int j = 0; j < NV; ++j) add_to(sum_q[j], dh[j]);
            }
            if (p.sum_qx) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum_qx[j].v[i] = fma2(dh[j].v[i], hat[j].v[i], sum_qx[j].v[i]);
            }
            if (p.dx && p.gate) {
#pragma unroll
                for (int j = 0; j < NV; ++j) dh[j] = times8(dh[j], gate.read(team, j));
            }
            if (joined) {
                Pair s0 = both(0.f), s1 = both(0.f);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    dh[j] = times8(dh[j], w1.read(team, j));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s0 = add2(s0, dh[j].v[i]);
                        s1 = fma2(dh[j].v[i], hat[j].v[i], s1);
                    }
                }
                s.x = total(s0);
                s.y = total(s1);
            }
        }
        const bool more = next < p.tokens;
        float4 m = make_float4(0.f, 0.f, 0.f, 0.f);
        if (more) in.wait(team);
        if (more && (p.w1 || p.w2)) {
            const int at = turn ^ 1;
            const bool both_rows = p.w1 && p.w2;
            Oct f[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (L < kPhased) f[j] = in.read(team, p.w2 ? H : X, next, j, at);
                else f[j] = p.w2 ? in.read(team, H, next, j, at) : in.read(team, X, next, j, at);        // `rows` stays in registers
            }
            team.template trim_read<L>(f, valid);
            if (p.rms) {
                m.x = Team<NV>::own_squares(f, 0.f);
            } else {
                team.template own_moments<L>(f, valid, m.x, m.y);
            }
            if (both_rows) {
#pragma unroll
                for (int j = 0; j < NV; ++j) f[j] = in.read(team, X, next, j, at);
                team.template trim_read<L>(f, valid);
                if (p.rms) {
                    m.y = Team<NV>::own_squares(f, 0.f);
                } else {
                    team.template own_moments<L>(f, valid, m.z, m.w);
                }
            }
            if (p.rms) {
                team.template sum_and_moments<true>(s, m);
                rstd[0] = rsqrtf(m.x * inv_n + p.eps);
                rstd[1] = both_rows ? rsqrtf(m.y * inv_n + p.eps) : rstd[0];
            } else {
                team.template sum_and_moments<false>(s, m);
                mean[0] = m.x;
                rstd[0] = rsqrtf(m.y * inv_n + p.eps);
                mean[1] = both_rows ? m.z : m.x;
                rstd[1] = both_rows ? rsqrtf(m.w * inv_n + p.eps) : rstd[0];
            }
        } else if (joined) {
            s = team.template sum<2>(s);
        } else {
            team.sync();
        }
        if (present && p.dx) {
            if (joined) {
                const Pair b0 = both(p.rms ? 0.f : -s.x * inv_n * rstd_x), b1 = both(-s.y * inv_n * rstd_x), r = both(rstd_x);
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) dh[j].v[i] = fma2(r, dh[j].v[i], fma2(hat[j].v[i], b1, b0));
            }
            T *dx = (T *)p.dx + row * p.ld_dx + c;
#pragma unroll
            for (int j = 0; j < NV; ++j) write_columns<T, L>(dx + j * step, j == 0 ? lead : 0, valid - j * step, dh[j]);
        }
    }
    team.close();
    if (!p.n_sums) return;
    float *out = p.partial + (size_t)blockIdx.x * p.n_sums * width;
    float *mine = (p.teams > 1 ? reinterpret_cast<float *>(dynamic) + (size_t)team.id * p.n_sums * width : out) + team.thread * 8 - phase;
    const Oct (*const all[4])[NV] = {&sum_q, &sum_qx, &sum_yh, &sum_y};
#pragma unroll
    for (int s = 0; s < 4; ++s)
        if (p.slot[s] >= 0)
#pragma unroll
            for (int j = 0; j < NV; ++j) write_columns<float, L == kPhased ? kAny : L>(mine + p.slot[s] * width + j * step, j == 0 ? lead : 0, valid - j * step, (*all[s])[j]);
    if (p.teams == 1) return;
    __syncthreads();
    for (int i = threadIdx.x; i < p.n_sums * width; i += blockDim.x) {
        float v = 0.f;
        for (int q = 0; q < p.teams; ++q) v += reinterpret_cast<const float *>(dynamic)[(size_t)q * p.n_sums * width + i];
        out[i] = v;
    }
}

// Adds the blocks' partials and writes the parameters' gradients: 32 columns a block, 8 rows of
// threads that take every eighth partial.
template <class T, class G>
__global__ void __launch_bounds__(256)
residual_norm_parameters_kernel(const __grid_constant__ NormParams p, int blocks, G *dgate, G *dw1, G *db1, G *dw2, G *db2)
{
    __shared__ float joined[4][8][33];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    grid_let_next();
    grid_wait();
    const int width = p.width, rank = c / p.share, at = c - rank * p.share;       // the column's block of a cluster
    for (int s = 0; s < 4; ++s) {
        float v = 0.f;
        if (p.slot[s] >= 0 && c < p.cols)
            for (int b = part * p.cluster + rank; b < blocks; b += 8 * p.cluster) v += __ldcg(p.partial + ((size_t)b * p.n_sums + p.slot[s]) * width + at);
        joined[s][part][lane] = v;
    }
    __syncthreads();
    if (part != 0 || c >= p.cols) return;
    float total[4];
    for (int s = 0; s < 4; ++s) {
        total[s] = 0.f;
        for (int q = 0; q < 8; ++q) total[s] += joined[s][q][lane];
    }
    const float gate = p.gate ? to_float(((const T *)p.gate)[c]) : 1.f;
    const float w1 = p.w1 ? to_float(((const T *)p.w1)[c]) : 1.f, b1 = p.b1 ? to_float(((const T *)p.b1)[c]) : 0.f;
    if (dgate) dgate[c] = from_float<G>(w1 * total[1] + (p.b1 ? b1 * total[0] : 0.f));
    if (dw1) dw1[c] = from_float<G>(gate * total[1]);
    if (db1) db1[c] = from_float<G>(gate * total[0]);
    if (dw2) dw2[c] = from_float<G>(total[2]);
    if (db2) db2[c] = from_float<G>(total[3]);
}

bool aligned_vector(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

constexpr int kMostSmem = 216 * 1024;            // dynamic shared memory of a block

// Who holds a row: a team of whole warps, 8 nv columns a thread.  An aligned row that 1, 2, 4 or 8
// blocks' shares of at most `widest` columns cut into whole warps' pieces by one of the nv on offer
// takes the fewest blocks and the largest such nv (fewest warps, of at most `most_warps`).  Otherwise
// the fewest blocks that hold a row in shares of at most `loose` columns, and the nv that leaves the fewest threads idle.  Short rows: several
// teams to a block of `threads` threads, as far as `smem` bytes go for `column_bytes` of shared memory a
// column.
void team_shape(NormParams &p, int &nv, const int (&offer)[6], Layout &layout, int widest, int loose, int most_warps, int threads, int column_bytes, int smem)
{
    const auto share_of = [&](int cluster) { return ((p.cols + cluster - 1) / cluster + 7) & ~7; };
    int warps = 0, before = 0;                   // columns that a piece starts before a row
    nv = 0;
    p.cluster = 1;
    if (layout == kWhole) {
        while (share_of(p.cluster) > widest) p.cluster *= 2;
        for (int i = 0; i < 6 && !nv; ++i) {
            warps = offer[i] ? share_of(p.cluster) / (256 * offer[i]) : 0;
            if (offer[i] && p.cols % (256 * offer[i] * p.cluster) == 0 && warps <= most_warps && warps * p.cluster <= kMaxEntries) nv = offer[i];
        }
    }
    if (!nv) {
        if (layout == kWhole) layout = kAligned;
        const bool phases = layout >= kPhased && ((p.ref_start | p.ref_pitch) & 15);
        for (before = phases ? 7 : 0; !nv; before = 0) {
            for (p.cluster = 1; p.cluster <= 8 && !nv; p.cluster *= nv ? 1 : 2)
                for (const int v : offer) {
                    const int n = v ? (share_of(p.cluster) + before + 256 * v - 1) / (256 * v) : 99;
                    if (share_of(p.cluster) + before <= loose && n <= most_warps && n * p.cluster <= kMaxEntries && (!nv || n * v < warps * nv)) {
                        nv = v;
                        warps = n;
                    }
                }
            if (nv) break;
            layout = kAny;                       // no room for phases
        }
        if (!before) p.ref_start = p.ref_pitch = 0;
    }
    const int share = share_of(p.cluster);
    p.share = share;
    p.team_threads = warps * 32;
    p.width = p.team_threads * 8 * nv;
    p.teams = 1;
    while (p.cluster == 1 && p.teams * 2 * p.team_threads <= threads && p.teams * 2 * p.width * column_bytes <= smem) p.teams *= 2;
}

NormParams base_params(const ResidualNorm &r)
{
    NormParams p{};
    const int e = r.type == DISTSIM_F32 ? 4 : 2;
    p.tokens = r.tokens;
    p.cols = (int32_t)r.cols;
    p.rms = r.rms;
    p.alpha = r.alpha;
    p.eps = r.eps;
    p.threshold = r.threshold;
    p.keep_scale = r.keep_scale;
    p.seed = r.seed;
    p.offset = r.offset;
    p.x = r.x.p; p.ld_x = r.x.ld;
    p.residual = r.residual.p; p.ld_residual = r.residual.ld;
    p.h_in = r.h.p; p.h = const_cast<void *>(r.h.p); p.ld_h = r.h.ld;
    p.y = const_cast<void *>(r.y.p); p.ld_y = r.y.ld;
    p.dy = r.dy.p; p.ld_dy = r.dy.ld;
    p.dh = r.dh.p; p.ld_dh = r.dh.ld;
    p.dx = const_cast<void *>(r.dx.p); p.ld_dx = r.dx.ld;
    p.dresidual = const_cast<void *>(r.dresidual.p); p.ld_dresidual = r.dresidual.ld;
    p.gate = r.gate;
    p.w1 = r.post_weight;
    p.b1 = r.post_bias;
    p.w2 = r.weight;
    p.b2 = r.bias;
    for (int &s : p.slot) s = -1;
    // Phases follow the rows that lie alike in most tensors; those that are written count more.
    p.ref_shift = e == 4 ? 2 : 1;
    const struct { const Matrix &m; int votes; } all[] = {{r.x, 2}, {r.residual, 2}, {r.dy, 2}, {r.dh, 2}, {r.h, 3}, {r.y, 7}, {r.dx, 7}, {r.dresidual, 7}};
    int most = 0;
    const auto start = [](const Matrix &m) { return (uint32_t)reinterpret_cast<uintptr_t>(m.p) & 15; };
    const auto pitch = [e](const Matrix &m) { return (uint32_t)(m.ld * e) & 15; };
    for (const auto &a : all) {
        int votes = 0;
        for (const auto &b : all)
            if (a.m.p && b.m.p && start(a.m) == start(b.m) && pitch(a.m) == pitch(b.m)) votes += b.votes;
        if (votes > most) {
            most = votes;
            p.ref_start = start(a.m);
            p.ref_pitch = pitch(a.m);
        }
    }
    p.all_in_phase = true;
    p.all_aligned = r.cols % 8 == 0;
    for (const void *v : {r.gate, r.post_weight, r.post_bias, r.weight, r.bias}) p.all_aligned = p.all_aligned && (!v || aligned_vector(v));
    for (const auto &a : all) {
        if (!a.m.p) continue;
        p.all_in_phase = p.all_in_phase && start(a.m) == p.ref_start && pitch(a.m) == p.ref_pitch;
        p.all_aligned = p.all_aligned && aligned_rows(a.m, e);
    }
    return p;
}

Layout layout_of(const NormParams &p) { return p.all_aligned ? kWhole : p.all_in_phase ? kPhased : kAny; }

// Blocks of a launch: enough for every row, at most what the device holds at a time.
template <class K>
cudaError_t launch_rows(OperatorLaunch &l, K kernel, const NormParams &p, int bytes, int64_t most, int64_t &blocks)
{
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e != cudaSuccess) return e;
    const int threads = p.teams * p.team_threads;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)bytes;
    cfg.stream = l.stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.cluster > 1 ? 1 : 0;
    int64_t rows = (p.tokens + p.teams - 1) / p.teams, room = 0;
    if (p.cluster > 1) {
        int clusters = 0;
        cfg.gridDim = dim3((unsigned)(l.sm_count * p.cluster));
        if ((e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg)) != cudaSuccess) return e;
        room = clusters;
    } else {
        int per_sm = 0;
        if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, bytes)) != cudaSuccess) return e;
        room = (int64_t)l.sm_count * per_sm;
    }
    if (room < 1) room = 1;
    if (room > most / p.cluster) room = most / p.cluster;
    if (rows > room) {
        // a team's rows are a multiple of eight apart, so that they have one phase
        rows = p.ref_pitch == 0 ? room : room >= 8 ? room & ~(int64_t)7 : rows < 8 ? rows : 8;
    }
    blocks = rows * p.cluster;
    return launch_kernel(l, kInOrder, kernel, (unsigned)blocks, 1, threads, bytes, p.cluster > 1 ? p.cluster : 0, p);
}

constexpr int kPartialBlocks = 8;                // an SM, of the backward kernel
// A block's columns: rows of whole pieces take blocks of 2048 at most; others, which leave threads
// idle, the fewest blocks (2056 columns, 16 bits: 1 block 480 us, 2 of 1028 546 us), in 32 bits only as many
// columns as leave shared memory for two blocks an SM.
constexpr int kWidestBackward = 2048, kMostBackwardWarps = kBackwardThreads / 32;       // columns, warps of a block
template <int SIZE>
constexpr int kLooseBackward = SIZE == 4 ? 2048 : 3072;
constexpr int kForwardPieces[6] = {4, 3, 2, 1, 0, 0}, kBackwardPieces[6] = {2, 1, 0, 0, 0, 0};

template <class T>
cudaError_t backward(OperatorLaunch &l, NormParams &p, const ResidualNorm &r)
{
    const int column_bytes = 8 * (int)sizeof(T);                      // two rows of four tensors, in the end four sums
    const int parameters = !!p.w1 + !!p.gate + !!p.w2;
    const int64_t most = (int64_t)l.sm_count * kPartialBlocks;
    int nv;
    int64_t blocks = 0;
    cudaError_t e;
    Layout layout = layout_of(p);
    team_shape(p, nv, kBackwardPieces, layout, kWidestBackward, kLooseBackward<sizeof(T)>, kMostBackwardWarps, 128, column_bytes + (layout >= kPhased ? 3 * (int)sizeof(T) : 0), 48 * 1024);
    const int bytes = (p.teams * column_bytes + (layout >= kPhased ? p.teams : 1) * parameters * (int)sizeof(T)) * p.width + (layout >= kPhased ? p.teams * 8 * 32 : 0);
#define BACKWARD(nv, layout) launch_rows(l, residual_norm_backward_kernel<T, nv, layout>, p, bytes, most, blocks)
    if (layout == kWhole) e = nv == 2 ? BACKWARD(2, kWhole) : BACKWARD(1, kWhole);
    else if (layout == kAligned) e = nv == 2 ? BACKWARD(2, kAligned) : BACKWARD(1, kAligned);
    else if (layout == kPhased) e = nv == 2 ? BACKWARD(2, kPhased) : BACKWARD(1, kPhased);
    else e = nv == 2 ? BACKWARD(2, kAny) : BACKWARD(1, kAny);
#undef BACKWARD
    if (e != cudaSuccess || !p.n_sums) return e;
    const unsigned grid = (unsigned)((p.cols + 31) / 32);
    if (r.grad_type == DISTSIM_F32)
        return launch_kernel(l, kEarly, residual_norm_parameters_kernel<T, float>, grid, 1, 256, 0, 0, p, (int)blocks, (float *)r.dgate, (float *)r.dpost_weight,
                             (float *)r.dpost_bias, (float *)r.dweight, (float *)r.dbias);
    return launch_kernel(l, kEarly, residual_norm_parameters_kernel<T, T>, grid, 1, 256, 0, 0, p, (int)blocks, (T *)r.dgate, (T *)r.dpost_weight,
                         (T *)r.dpost_bias, (T *)r.dweight, (T *)r.dbias);
}
template <class T>
cudaError_t forward(OperatorLaunch &l, NormParams &p)
{
    const int column_bytes = 2 * (int)sizeof(T);                      // a row of two tensors
    const int widest = sizeof(T) == 4 ? 2048 : 4096;                  // with five parameters 56 KB of shared memory
    const int parameters = !!p.w1 + !!p.b1 + !!p.gate + !!p.w2 + !!p.b2;
    int nv;
    int64_t blocks = 0;
    const int64_t most = INT64_C(1) << 30;
    Layout layout = layout_of(p);
    team_shape(p, nv, kForwardPieces, layout, widest, widest, 4, 128, column_bytes + (layout >= kPhased ? 5 * (int)sizeof(T) : 0), 16 * 1024);
    const int bytes = (p.teams * column_bytes + (layout >= kPhased ? p.teams : 1) * parameters * (int)sizeof(T)) * p.width + (layout >= kPhased ? p.teams * 2 * 32 : 0);
#define FORWARD(nv, layout) launch_rows(l, residual_norm_forward_kernel<T, nv, layout>, p, bytes, most, blocks)
    if (layout == kWhole) return nv == 4 ? FORWARD(4, kWhole) : nv == 3 ? FORWARD(3, kWhole) : nv == 2 ? FORWARD(2, kWhole) : FORWARD(1, kWhole);
    if (layout == kAligned) return nv == 4 ? FORWARD(4, kAligned) : nv == 3 ? FORWARD(3, kAligned) : nv == 2 ? FORWARD(2, kAligned) : FORWARD(1, kAligned);
    if (layout == kPhased) return nv == 4 ? FORWARD(4, kPhased) : nv == 3 ? FORWARD(3, kPhased) : nv == 2 ? FORWARD(2, kPhased) : FORWARD(1, kPhased);
    return nv == 4 ? FORWARD(4, kAny) : nv == 3 ? FORWARD(3, kAny) : nv == 2 ? FORWARD(2, kAny) : FORWARD(1, kAny);
#undef FORWARD
}

}  // namespace

cudaError_t launch_residual_norm_forward(OperatorLaunch &l, const ResidualNorm &r)
{
    NormParams p = base_params(r);
    p.status = l.status;
    p.polls = l.polls;
    switch (r.type) {
    case DISTSIM_F32: return forward<float>(l, p);
    case DISTSIM_F16: return forward<__half>(l, p);
    default: return forward<__nv_bfloat16>(l, p);
    }
}

int64_t residual_norm_partials(int64_t cols, int sm_count)
{
    // four sums of a share a block, in the widest shape
    int width = 0;
    for (const int shape : {0, 1, 2, 3}) {
        NormParams p{};
        p.cols = (int32_t)cols;
        p.ref_pitch = shape & 1 ? 2 : 0;
        int nv;
        Layout layout = kAny;                    // without phases no wider than these are kAligned and kWhole
        team_shape(p, nv, kBackwardPieces, layout, kWidestBackward, shape & 2 ? kLooseBackward<4> : kLooseBackward<2>, kMostBackwardWarps, 128, 16, 0);
        if (p.width > width) width = p.width;
    }
    return (int64_t)sm_count * kPartialBlocks * 4 * width;
}

cudaError_t launch_residual_norm_backward(OperatorLaunch &l, const ResidualNorm &r)
{
    NormParams p = base_params(r);
    p.partial = r.partial;
    p.status = l.status;
    p.polls = l.polls;
    p.sum_q = r.dpost_bias || (r.dgate && r.post_weight && r.post_bias);
    p.sum_qx = r.dpost_weight || r.dgate;
    p.sum_y = r.dweight || r.dbias;
    if (p.sum_q) p.slot[0] = p.n_sums++;
    if (p.sum_qx) p.slot[1] = p.n_sums++;
    if (p.sum_y) { p.slot[2] = p.n_sums++; p.slot[3] = p.n_sums++; }
    switch (r.type) {
    case DISTSIM_F32: return backward<float>(l, p, r);
    case DISTSIM_F16: return backward<__half>(l, p, r);
    default: return backward<__nv_bfloat16>(l, p, r);
    }
}

}  // namespace distsim
