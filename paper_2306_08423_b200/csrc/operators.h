// Internal declarations of the layer operators (not part of the C ABI): the matrix products with
// their epilogues (matmul_kernels.cu), the passes around them (column_kernels.cu) and the residual
// connection with its norms (norm_kernels.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace distsim {

// Polls of an operator kernel's wait, of a microsecond each: it gives up after some seconds at most; the
// longest wait of a healthy launch (an accumulator's whole product) takes microseconds.
constexpr int32_t kOperatorPolls = 1 << 22;

// A matrix of `rows` rows, `ld` elements apart, whose columns are contiguous.
struct Matrix {
    const void *p = nullptr;
    int64_t ld = 0;
};

// What a tile's accumulators become (z, g, u, d: 32-bit sums; every output is rounded once).
enum Epilogue : int {
    kEpiLinear = 0,    // z = sum + bias0;  out0 = act(z) + in0;  out1 = z
    kEpiGated = 1,     // g, u = sums + bias0, bias1;  out0 = act(g) u;  out1 = g;  out2 = u
    kEpiGatedBack = 2  // d = sum, g = in0, u = in1;  out0 = d u act'(g);  out1 = d act(g)
};

// out[m][n] = sum over k of a[m][k] b[n][k].  An operand is given by the rows of its matrix: with
// *_mn false a row holds one m (n) and runs over k, with *_mn true a row holds one k and runs over m (n).
struct Product {
    int64_t m = 0, n = 0;
    int64_t k[2] = {0, 0};        // k[1] > 0: a second pair of operands, added to the first's sum
    Matrix a[2], b[2];            // kEpiGated: b[0], b[1] are the gate's and the up projection's weights
    bool a_mn = false, b_mn = false;
    int groups = 1;               // 2: two products of the same shape with a[g] and the same b[0];
                                  // their outputs are out[g], their inputs in[g]
    int epilogue = kEpiLinear;
    int act = 0;
    const void *bias[2] = {nullptr, nullptr};
    Matrix in[2];
    Matrix out[3];
    int in_type = 0;              // DISTSIM_BF16 or DISTSIM_F16: operands, bias, in and out
    bool wide = false;            // out and in are 32-bit floats (kEpiLinear without bias and activation)
    // kEpiGatedBack: column sums of out0 and out1 before they are rounded (both or none), as partials:
    // product_sum_rows() rows of n values, sums_ld (a multiple of 4) apart, which add up to them.
    float *sums[2] = {nullptr, nullptr};
    int64_t sums_ld = 0;
};

struct OperatorLaunch {
    cudaStream_t stream = nullptr;
    int sm_count = 0;
    const int *split_capacity = nullptr;         // of the device, for splits of 1, 2, 4
    int32_t *status = nullptr;    // host-mapped word that a kernel whose wait gave up writes
    int32_t polls = kOperatorPolls;
    int64_t launches = 0;
};

// Launches a kernel.  cluster 0: none, or the kernel's own.  kEarly: its blocks may start before the
// kernel in front has ended (see grid_wait()).  Not for kernels whose blocks fill the device and keep
// their rows: blocks of the kernel in front that are still there push some of theirs into a second
// wave (norms backward, 768 columns: 438 -> 687 us).
enum Start { kInOrder, kEarly };
template <class... Params, class... Args>
cudaError_t launch_kernel(OperatorLaunch &l, Start start, void (*kernel)(Params...), unsigned grid_x, unsigned grid_y, int threads, int smem,
                          int cluster, Args &&...args)
{
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    cfg.stream = l.stream;
    cfg.gridDim = dim3(grid_x, grid_y);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = start == kEarly;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    ++l.launches;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Args &&>(args)...);
}

// How a product is run: the estimate (in microseconds, fitted to products of 1 to 8192 rows) says
// which is faster.  A pair's step of 256 x 256 x 64 takes 0.265 us; a persistent kernel overlaps its
// tiles' epilogues with the next products, a split one shortens the longest reduction but finishes
// its rows after it.  Measured, persistent / split 1 / 2 / 4 in us (forward with bias, bf16): 100 x 4096 -> 1024
// 23.3 / 25.7 / 17.4 / 13.4;  512 x 4096 -> 1024 23.7 / 26.8 / 17.9 / 14.5;  512 x 1024 -> 4096 10.7 / 13.8 / 12.7 / 32.0;
// 1024 x 1024 -> 1024 10.5 / 13.4 / 11.3 / 20.9 (clusters of 8 blocks: fewer than 16 fit);  8192 x 1024 -> 4096 59 /
// 104 / 190 / 387;  gradient 768 x 768 over 8192, persistent / split 2 / 4: 41.4 / 27.1 / 19.8.
struct ProductPlan {
    bool pair = false;            // persistent pairs of blocks, else a cluster a tile
    bool few = false;             // tokens as the tensor core's columns (few_rows())
    int split = 1;                // pairs of a cluster that share the tile's reduction
};
// Whether the few-rows kernel serves: at most 64 tokens and no weight gradient.
bool few_rows(const Product &p);
// unaligned_in, unaligned_out: bytes of in and out that the persistent kernel can only reach through
// copies (2.3 MB a us); the others write them value by value (3.8 MB a us) and read them so (0.6 MB a
// us).  Measured, persistent / split 1 in us: 6969 x 56 x 925 14.6 / 20.8, with a residual 21.4 / 35.3;
// 8192 x 1024 x 4097 79.6 / 119, with a residual 109 / 243; 1537 x 2304 x 771 19.7 / 15.5 (split 2).
ProductPlan choose_plan(const Product &p, const OperatorLaunch &l, int64_t unaligned_in, int64_t unaligned_out);
// Clusters of `split` pairs of the split kernel that the current device holds at a time.
int split_capacity(int split, int sm_count);

// 16-byte aligned rows, as the tiled copies need them.
inline bool aligned_rows(const Matrix &x, int elem_bytes)
{
    return (reinterpret_cast<uintptr_t>(x.p) & 15) == 0 && (x.ld * elem_bytes) % 16 == 0;
}
// Operands have aligned rows; for plan.pair so have in and out, and the 16-byte piece that holds the last
// column of an out row is written whole.  m, n >= 1, k[0] >= 1.
int64_t product_sum_rows(const Product &p, const ProductPlan &plan);
cudaError_t launch_product(OperatorLaunch &l, const Product &p, const ProductPlan &plan);

// Column-wise passes over [rows][cols] matrices of 16-bit types (column_kernels.cu).
constexpr int kPassParts = 3;
struct ColumnPass {
    int64_t rows = 0;
    int type = 0;                 // DISTSIM_BF16 or DISTSIM_F16
    struct Part {
        int64_t cols = 0;
        Matrix x;                 // in; null: no such part
        void *sums = nullptr;     // [cols] column sums (of the unrounded product), nullable with `out` only
        int64_t partials = 0;     // > 0: x is that many rows of 32-bit partial sums instead, whole eights in aligned rows
    } part[kPassParts];           // all in one launch; with z or out one part
    Matrix z;                     // in, nullable: x is multiplied by act'(z)
    int act = 0;
    Matrix out;                   // the product, nullable
    int sums_type = 0;
    float *partial = nullptr;     // scratch of column_pass_partials() floats (with sums)
    int32_t *counters = nullptr;  // kColumnCounters zeroed words, left zero (with sums)
};
constexpr int kColumnCounters = 4096;
// For launches of any parts of `cols` columns together.
int64_t column_pass_partials(int64_t cols, int sm_count);
cudaError_t launch_column_pass(OperatorLaunch &l, const ColumnPass &c);

// Copies [rows][cols] matrices of 2-byte units between rows of any distance (column_kernels.cu), all
// in one launch; without src it fills dst with zeros.
struct Move {
    uint16_t *dst;
    const uint16_t *src;
    int64_t ld_dst, ld_src, rows, cols;
};
constexpr int kMostMoves = 11;
cudaError_t launch_moves(OperatorLaunch &l, const Move *moves, int n);

// The residual connection (norm_kernels.cu).
struct ResidualNorm {
    int64_t tokens = 0, cols = 0;
    int type = 0, grad_type = 0;
    bool rms = false;
    float alpha = 1.f, eps = 0.f;
    uint32_t threshold = 0;       // of dropout: kept where bits >= threshold; 0: no dropout
    float keep_scale = 1.f;
    uint64_t seed = 0, offset = 0;
    Matrix x, residual, h, y, dy, dh, dx, dresidual;
    const void *gate = nullptr, *post_weight = nullptr, *post_bias = nullptr, *weight = nullptr, *bias = nullptr;
    void *dgate = nullptr, *dpost_weight = nullptr, *dpost_bias = nullptr, *dweight = nullptr, *dbias = nullptr;
    float *partial = nullptr;     // backward: scratch of residual_norm_partials() floats
};
cudaError_t launch_residual_norm_forward(OperatorLaunch &l, const ResidualNorm &r);
int64_t residual_norm_partials(int64_t cols, int sm_count);
cudaError_t launch_residual_norm_backward(OperatorLaunch &l, const ResidualNorm &r);

}  // namespace distsim
