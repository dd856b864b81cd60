// Host side of the layer operators: checks of arguments, scratch, and which kernels run in which
// order.  No arithmetic happens here.
#include <cstdio>
#include <initializer_list>
#include <new>

#include "../../include/distsim_testing.h"
#include "engine.h"
#include "operators.h"

namespace distsim {

// The operators' part of a context: scratch that grows, the word kernels report to, and the order
// of calls on different streams.
struct OperatorState {
    void *scratch = nullptr;
    size_t capacity = 0;
    int32_t *counters = nullptr;                 // zeroed words, left zero by every kernel
    int32_t *status = nullptr;                   // host memory that the device writes
    int32_t *d_status = nullptr;
    cudaEvent_t done = nullptr;                  // behind the last call's kernels
    unsigned long long last = 0;                 // that call's stream, by its id: a later stream may get its handle
    bool used = false;
    bool captured = false;                       // a captured call uses the scratch: graphs hold its address
    struct Retired { void *block; Retired *next; };
    Retired *retired = nullptr;                  // earlier blocks that graphs may still hold
    int sm_count = 0;
    int split_capacity[3] = {};                  // of the context's device, see operators.h
    int32_t forced_plan = 0, polls = kOperatorPolls;         // testing hooks, see distsim_testing.h
    bool ready = false;

    ~OperatorState()
    {
        if (scratch) cudaFree(scratch);
        while (Retired *r = retired) {
            cudaFree(r->block);
            retired = r->next;
            delete r;
        }
        if (counters) cudaFree(counters);
        if (status) cudaFreeHost(status);
        if (done) cudaEventDestroy(done);
    }
};
OperatorState *new_operator_state() { return new (std::nothrow) OperatorState; }
void delete_operator_state(OperatorState *s) { delete s; }

}  // namespace distsim

using namespace distsim;

namespace {

struct StandIn;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t padded_ld(int64_t cols, int elem) { return ceil_div(cols * elem, 16) * 16 / elem; }

// One call: its context, its launches, and its scratch, laid out first and then reserved.
struct Call {
    distsim_ctx *ctx;
    OperatorAccess a{};
    OperatorLaunch l{};
    cudaStream_t stream;
    bool capturing = false;
    unsigned long long stream_id = 0;            // where scratch is used, outside a capture
    size_t need = 0;

    explicit Call(distsim_ctx *c, void *s) : ctx(c), stream(static_cast<cudaStream_t>(s)) {}

    int fail(int code, const char *text)
    {
        try {
            return a.fail(ctx, code, text);
        } catch (const std::bad_alloc &) {           // the text's copy; no exception leaves a C entry
            return code;
        }
    }
    int cuda(cudaError_t e, const char *what)
    {
        char text[256];
        snprintf(text, sizeof text, "%s: %s", what, cudaGetErrorString(e));
        return fail(DISTSIM_E_CUDA, text);
    }

    int begin()
    {
        a = operator_access(ctx);
        if (!a.state) return fail(DISTSIM_E_CUDA, "out of host memory");
        cudaError_t e = cudaSetDevice(a.device);
        if (e != cudaSuccess) return cuda(e, "cudaSetDevice");
        OperatorState &s = *a.state;
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        if ((e = cudaStreamIsCapturing(stream, &cap)) != cudaSuccess) return cuda(e, "stream");
        capturing = cap != cudaStreamCaptureStatusNone;
        if (!s.ready) {
            if (capturing) return fail(DISTSIM_E_STATE, "the first operator call of a context cannot be captured");
            if ((!s.counters && (e = cudaMalloc(&s.counters, kColumnCounters * sizeof(int32_t))) != cudaSuccess) ||
                (e = cudaMemset(s.counters, 0, kColumnCounters * sizeof(int32_t))) != cudaSuccess ||
                (e = cudaStreamSynchronize(nullptr)) != cudaSuccess ||
                (!s.status && (e = cudaHostAlloc(&s.status, 64, cudaHostAllocMapped)) != cudaSuccess) ||
                (e = cudaHostGetDevicePointer((void **)&s.d_status, s.status, 0)) != cudaSuccess ||
                (!s.done && (e = cudaEventCreateWithFlags(&s.done, cudaEventDisableTiming)) != cudaSuccess) ||
                (e = cudaDeviceGetAttribute(&s.sm_count, cudaDevAttrMultiProcessorCount, a.device)) != cudaSuccess)
                return cuda(e, "operator set-up");
            for (int i = 0; i < 3; ++i) s.split_capacity[i] = split_capacity(1 << i, s.sm_count);
            *s.status = 0;
            s.ready = true;
        }
        const int rc = take_status();
        if (rc != DISTSIM_OK) return rc;
        l.stream = stream;
        l.sm_count = s.sm_count;
        l.split_capacity = s.split_capacity;
        l.status = s.d_status;
        l.polls = s.polls;
        return DISTSIM_OK;
    }
    int take_status()
    {
        volatile int32_t *st = a.state->status;
        const int32_t code = *st;
        if (code == 0) return DISTSIM_OK;
        *st = 0;
        return fail(DISTSIM_E_TIMEOUT, "a bounded wait of an earlier operator call gave up: that call's outputs are undefined");
    }

    // How to run a product that reads `in` besides its operands and writes `out`.
    ProductPlan plan(const Product &p, std::initializer_list<const StandIn *> in, std::initializer_list<const StandIn *> out) const;
    ProductPlan plan_of(const Product &p, int64_t unaligned_in, int64_t unaligned_out) const
    {
        const int32_t f = a.state->forced_plan;
        if (f == 0) return choose_plan(p, l, unaligned_in, unaligned_out);
        ProductPlan q;
        q.pair = f == -1;
        q.few = f <= -2 && few_rows(p);
        const int64_t steps = (p.k[0] + 63) / 64 + (p.k[1] + 63) / 64;
        for (q.split = f == -1 ? 1 : f < 0 ? 1 << (-2 - f) : f; q.split > steps; q.split /= 2) {}
        return q;
    }

    // Room for `bytes` of scratch: an offset, to be turned into a pointer after reserve().
    size_t room(size_t bytes)
    {
        const size_t at = need;
        need = (need + bytes + 255) & ~(size_t)255;
        return at;
    }
    template <class T = void>
    T *at(size_t offset) { return reinterpret_cast<T *>(static_cast<char *>(a.state->scratch) + offset); }

    // Scratch of the laid-out size, and this call behind the last one that used it.
    int reserve()
    {
        OperatorState &s = *a.state;
        cudaError_t e;
        if (need == 0) return DISTSIM_OK;
        if (need > s.capacity) {
            if (capturing) return fail(DISTSIM_E_STATE, "operator scratch cannot grow while a call is captured: make one call of this size before");
            if (s.scratch && s.captured) {
                auto *r = new (std::nothrow) OperatorState::Retired{s.scratch, s.retired};
                if (!r) return fail(DISTSIM_E_CUDA, "out of host memory");
                s.retired = r;
            } else if (s.scratch && (e = cudaFree(s.scratch)) != cudaSuccess) {          // waits for the kernels that still use it
                return cuda(e, "operator scratch");
            }
            s.scratch = nullptr;
            s.capacity = 0;
            s.captured = false;
            if ((e = cudaMalloc(&s.scratch, need)) != cudaSuccess) { s.scratch = nullptr; return cuda(e, "operator scratch"); }
            s.capacity = need;
        }
        if (capturing) {
            s.captured = true;
            return DISTSIM_OK;
        }
        if ((e = cudaStreamGetId(stream, &stream_id)) != cudaSuccess) return cuda(e, "stream");
        if (s.used && s.last != stream_id && (e = cudaStreamWaitEvent(stream, s.done, 0)) != cudaSuccess) return cuda(e, "stream order");
        return DISTSIM_OK;
    }
    int end(cudaError_t e)
    {
        *a.launches += l.launches;
        cudaError_t order = cudaSuccess;
        if (need > 0 && !capturing) {                        // after a failure too: what was launched before it uses the scratch
            OperatorState &s = *a.state;
            order = cudaEventRecord(s.done, stream);
            if (order == cudaSuccess) {
                s.last = stream_id;
                s.used = true;
            }
        }
        if (e != cudaSuccess) return cuda(e, "operator launch");
        return order == cudaSuccess ? DISTSIM_OK : cuda(order, "stream order");
    }
};

Matrix mat(const void *p, int64_t ld) { return Matrix{p, ld}; }

bool overlong(int64_t rows, int64_t cols) { return rows > 0x7fffffff || cols > 0x7fffffff; }

// A matrix that a tiled copy must read or write: itself, or a stand-in in scratch whose rows are
// whole 16-byte pieces.
struct StandIn {
    Matrix own;                                  // as the caller has it
    int64_t rows, cols;
    int elem;
    bool moved = false;
    size_t offset = 0;
    Matrix use{};

    // written: by tiled copies.  They write rows up to a 16-byte boundary (zeros behind the last column), so
    // the caller's rows have to end on one: what follows a column range is not the operator's.
    bool apart(bool written) const { return own.p && (!aligned_rows(own, elem) || (written && cols * elem % 16 != 0)); }
    void plan(Call &c, bool needed, bool written = false)
    {
        moved = needed && apart(written);
        if (moved) offset = c.room((size_t)rows * padded_ld(cols, elem) * elem);
    }
    void place(Call &c) { use = moved ? Matrix{c.at(offset), padded_ld(cols, elem)} : own; }
};
int64_t unaligned(std::initializer_list<const StandIn *> all, bool written)
{
    int64_t bytes = 0;
    for (const StandIn *s : all)
        if (s->apart(written)) bytes += s->rows * s->cols * s->elem;
    return bytes;
}
ProductPlan Call::plan(const Product &p, std::initializer_list<const StandIn *> in, std::initializer_list<const StandIn *> out) const
{
    return plan_of(p, unaligned(in, false), unaligned(out, true));
}
Move move_of(const Matrix &dst, const Matrix &src, int64_t rows, int64_t cols, int elem)
{
    const int64_t units = elem / 2;
    return Move{(uint16_t *)const_cast<void *>(dst.p), (const uint16_t *)src.p, dst.ld * units, src.ld * units, rows, cols * units};
}
// Fills the stand-ins that are read; gives back what was written to stand-ins.
cudaError_t fetch(Call &c, std::initializer_list<const StandIn *> all)
{
    Move moves[kMostMoves];
    int n = 0;
    for (const StandIn *s : all)
        if (s->moved) moves[n++] = move_of(s->use, s->own, s->rows, s->cols, s->elem);
    return launch_moves(c.l, moves, n);
}
cudaError_t give_back(Call &c, std::initializer_list<const StandIn *> all)
{
    Move moves[kMostMoves];
    int n = 0;
    for (const StandIn *s : all)
        if (s->moved) moves[n++] = move_of(s->own, s->use, s->rows, s->cols, s->elem);
    return launch_moves(c.l, moves, n);
}
StandIn stand_in(const void *p, int64_t ld, int64_t rows, int64_t cols, int elem) { return StandIn{Matrix{p, ld}, rows, cols, elem}; }

// Runs steps in order until one fails.
#define TRY(expr)                              \
    do {                                       \
        if (e == cudaSuccess) e = (expr);      \
    } while (0)

bool bad_rows(const void *p, int64_t ld, int64_t cols) { return p && ld < cols; }

ColumnPass column_pass(Call &c, int type, int64_t rows, int sums_type, float *partial)
{
    ColumnPass q;
    q.rows = rows;
    q.type = type;
    q.sums_type = sums_type;
    q.partial = partial;
    q.counters = c.a.state->counters;
    return q;
}

cudaError_t zero_vector(Call &c, void *p, int64_t n, int type)
{
    return p ? cudaMemsetAsync(p, 0, (size_t)n * (type == DISTSIM_F32 ? 4 : 2), c.stream) : cudaSuccess;
}

int check_linear(Call &c, const distsim_linear *o)
{
    if (o->tokens < 0 || o->d_in < 1 || o->d_out < 1 || o->reserved != 0) return c.fail(DISTSIM_E_ARG, "linear: sizes");
    if (overlong(o->tokens, o->d_in) || overlong(0, o->d_out)) return c.fail(DISTSIM_E_UNSUPPORTED, "linear: a size above 2^31 - 1");
    if (o->dtype != DISTSIM_BF16 && o->dtype != DISTSIM_F16) return c.fail(DISTSIM_E_UNSUPPORTED, "linear: dtype must be bf16 or f16");
    if (o->activation < DISTSIM_ACT_NONE || o->activation > DISTSIM_ACT_SILU) return c.fail(DISTSIM_E_ARG, "linear: unknown activation");
    if (bad_rows(o->x, o->ld_x, o->d_in) || bad_rows(o->weight, o->ld_weight, o->d_in) || bad_rows(o->residual, o->ld_residual, o->d_out) ||
        bad_rows(o->y, o->ld_y, o->d_out) || bad_rows(o->preact, o->ld_preact, o->d_out) || bad_rows(o->dy, o->ld_dy, o->d_out) ||
        bad_rows(o->dx, o->ld_dx, o->d_in) || bad_rows(o->dweight, o->ld_dweight, o->d_in) ||
        bad_rows(o->dweight_in, o->ld_dweight_in, o->d_in))
        return c.fail(DISTSIM_E_ARG, "linear: rows closer together than they are long");
    return DISTSIM_OK;
}

}  // namespace

extern "C" {

int distsim_operator_status(distsim_ctx *ctx, void *stream)
{
    if (!ctx) return DISTSIM_E_ARG;
    Call c(ctx, stream);
    c.a = operator_access(ctx);
    if (!c.a.state) return c.fail(DISTSIM_E_CUDA, "out of host memory");
    cudaError_t e = cudaSetDevice(c.a.device);
    if (e == cudaSuccess) e = cudaStreamSynchronize(c.stream);
    if (e != cudaSuccess) return c.cuda(e, "stream");
    return c.a.state->ready ? c.take_status() : DISTSIM_OK;
}

int distsim_testing_set_product_plan(distsim_ctx *ctx, int32_t plan)
{
    if (!ctx || ((plan < -4 || plan > 2) && plan != 4)) return DISTSIM_E_ARG;
    Call c(ctx, nullptr);
    const int rc = c.begin();
    if (rc == DISTSIM_OK) c.a.state->forced_plan = plan;
    return rc;
}

int distsim_testing_set_operator_status(distsim_ctx *ctx, int32_t code)
{
    if (!ctx) return DISTSIM_E_ARG;
    Call c(ctx, nullptr);
    const int rc = c.begin();
    if (rc == DISTSIM_OK) *reinterpret_cast<volatile int32_t *>(c.a.state->status) = code;
    return rc;
}

int distsim_testing_set_operator_wait_polls(distsim_ctx *ctx, int32_t polls)
{
    if (!ctx || polls < 0 || polls > kOperatorPolls) return DISTSIM_E_ARG;
    Call c(ctx, nullptr);
    const int rc = c.begin();
    if (rc == DISTSIM_OK) c.a.state->polls = polls;
    return rc;
}

int distsim_linear_forward(distsim_ctx *ctx, void *stream, const distsim_linear *o)
{
    if (!ctx || !o) return DISTSIM_E_ARG;
    Call c(ctx, stream);
    int rc = c.begin();
    if (rc != DISTSIM_OK || (rc = check_linear(c, o)) != DISTSIM_OK) return rc;
    const int64_t t = o->tokens, d = o->d_in, f = o->d_out;
    if (t > 0 && (!o->x || !o->weight || !o->y)) return c.fail(DISTSIM_E_ARG, "linear forward: x, weight and y are needed");
    if (t == 0) return DISTSIM_OK;

    Product p;
    p.m = t;
    p.n = f;
    p.k[0] = d;
    p.act = o->activation;
    p.in_type = o->dtype;
    p.bias[0] = o->bias;
    StandIn x = stand_in(o->x, o->ld_x, t, d, 2), w = stand_in(o->weight, o->ld_weight, f, d, 2);
    StandIn r = stand_in(o->residual, o->ld_residual, t, f, 2), y = stand_in(o->y, o->ld_y, t, f, 2), z = stand_in(o->preact, o->ld_preact, t, f, 2);
    const ProductPlan plan = c.plan(p, {&r}, {&y, &z});
    for (StandIn *s : {&x, &w}) s->plan(c, true);
    r.plan(c, plan.pair);
    for (StandIn *s : {&y, &z}) s->plan(c, plan.pair, true);
    if ((rc = c.reserve()) != DISTSIM_OK) return rc;
    for (StandIn *s : {&x, &w, &r, &y, &z}) s->place(c);
    p.a[0] = x.use;
    p.b[0] = w.use;
    p.in[0] = r.use;
    p.out[0] = y.use;
    p.out[1] = z.use;
    cudaError_t e = cudaSuccess;
    TRY(fetch(c, {&x, &w, &r}));
    TRY(launch_product(c.l, p, plan));
    TRY(give_back(c, {&y, &z}));
    return c.end(e);
}

int distsim_linear_backward(distsim_ctx *ctx, void *stream, const distsim_linear *o)
{
    if (!ctx || !o) return DISTSIM_E_ARG;
    Call c(ctx, stream);
    int rc = c.begin();
    if (rc != DISTSIM_OK || (rc = check_linear(c, o)) != DISTSIM_OK) return rc;
    const int64_t t = o->tokens, d = o->d_in, f = o->d_out;
    const bool act = o->activation != DISTSIM_ACT_NONE;
    if (o->grad_dtype != o->dtype && o->grad_dtype != DISTSIM_F32) return c.fail(DISTSIM_E_UNSUPPORTED, "linear: grad_dtype must be dtype or f32");
    if (t > 0 && (!o->dy || (act && !o->preact) || (o->dx && !o->weight) || (o->dweight && !o->x)))
        return c.fail(DISTSIM_E_ARG, "linear backward: dy, preact (with an activation), weight (for dx) and x (for dweight) are needed");
    const int ge = o->grad_dtype == DISTSIM_F32 ? 4 : 2;
    cudaError_t e = cudaSuccess;
    if (t == 0) {
        if ((rc = c.reserve()) != DISTSIM_OK) return rc;
        if (o->dweight && o->dweight != o->dweight_in) {
            const Move whole = move_of(mat(o->dweight, o->ld_dweight), mat(o->dweight_in, o->ld_dweight_in), f, d, ge);
            TRY(launch_moves(c.l, &whole, 1));
        }
        TRY(zero_vector(c, o->dbias, f, o->grad_dtype));
        return c.end(e);
    }

    Product px, pw;
    px.m = t; px.n = d; px.k[0] = f; px.b_mn = true; px.in_type = o->dtype;
    pw.m = f; pw.n = d; pw.k[0] = t; pw.a_mn = pw.b_mn = true; pw.in_type = o->dtype; pw.wide = ge == 4;
    StandIn x = stand_in(o->x, o->ld_x, t, d, 2), w = stand_in(o->weight, o->ld_weight, f, d, 2), dy = stand_in(o->dy, o->ld_dy, t, f, 2);
    StandIn dx = stand_in(o->dx, o->ld_dx, t, d, 2), dw = stand_in(o->dweight, o->ld_dweight, f, d, ge), dwi = stand_in(o->dweight_in, o->ld_dweight_in, f, d, ge);
    const ProductPlan plan_x = c.plan(px, {}, {&dx}), plan_w = c.plan(pw, {&dwi}, {&dw});
    x.plan(c, o->dweight);
    w.plan(c, o->dx);
    dy.plan(c, !act && (o->dx || o->dweight));
    dx.plan(c, plan_x.pair, true);
    dw.plan(c, plan_w.pair, true);
    dwi.plan(c, plan_w.pair && o->dweight);
    const size_t dz_at = act ? c.room((size_t)t * padded_ld(f, 2) * 2) : 0;
    const size_t part_at = o->dbias ? c.room((size_t)column_pass_partials(f, c.l.sm_count) * 4) : 0;
    if ((rc = c.reserve()) != DISTSIM_OK) return rc;
    for (StandIn *s : {&x, &w, &dy, &dx, &dw, &dwi}) s->place(c);

    Matrix dz = dy.use;
    ColumnPass pass = column_pass(c, o->dtype, t, o->grad_dtype, o->dbias ? c.at<float>(part_at) : nullptr);
    TRY(fetch(c, {&x, &w, &dy, &dwi}));
    if (act) {
        dz = mat(c.at(dz_at), padded_ld(f, 2));
        if (o->dx || o->dweight) pass.out = dz;
        pass.z = mat(o->preact, o->ld_preact);
        pass.act = o->activation;
        pass.part[0] = {f, dy.own, o->dbias};
        TRY(launch_column_pass(c.l, pass));
    } else if (o->dbias) {
        pass.part[0] = {f, dy.use, o->dbias};
        TRY(launch_column_pass(c.l, pass));
    }
    if (o->dx) {
        px.a[0] = dz;
        px.b[0] = w.use;
        px.out[0] = dx.use;
        TRY(launch_product(c.l, px, plan_x));
    }
    if (o->dweight) {
        pw.a[0] = dz;
        pw.b[0] = x.use;
        pw.in[0] = dwi.use;
        pw.out[0] = dw.use;
        TRY(launch_product(c.l, pw, plan_w));
    }
    TRY(give_back(c, {&dx, &dw}));
    return c.end(e);
}

namespace {
int check_ffn(Call &c, const distsim_gated_ffn *o)
{
    if (o->tokens < 0 || o->d_in < 1 || o->d_hidden < 1 || o->reserved != 0) return c.fail(DISTSIM_E_ARG, "gated ffn: sizes");
    if (overlong(o->tokens, o->d_in) || overlong(0, o->d_hidden)) return c.fail(DISTSIM_E_UNSUPPORTED, "gated ffn: a size above 2^31 - 1");
    if (o->dtype != DISTSIM_BF16 && o->dtype != DISTSIM_F16) return c.fail(DISTSIM_E_UNSUPPORTED, "gated ffn: dtype must be bf16 or f16");
    if (o->activation < DISTSIM_ACT_NONE || o->activation > DISTSIM_ACT_SILU) return c.fail(DISTSIM_E_ARG, "gated ffn: unknown activation");
    if (!o->b_gate != !o->b_up) return c.fail(DISTSIM_E_ARG, "gated ffn: b_gate and b_up come together");
    const int64_t d = o->d_in, f = o->d_hidden;
    if (bad_rows(o->x, o->ld_x, d) || bad_rows(o->w_gate, o->ld_w_gate, d) || bad_rows(o->w_up, o->ld_w_up, d) ||
        bad_rows(o->w_down, o->ld_w_down, f) || bad_rows(o->residual, o->ld_residual, d) || bad_rows(o->y, o->ld_y, d) ||
        bad_rows(o->hidden, o->ld_hidden, f) || bad_rows(o->gate, o->ld_gate, f) || bad_rows(o->up, o->ld_up, f) ||
        bad_rows(o->dy, o->ld_dy, d) || bad_rows(o->dx, o->ld_dx, d) || bad_rows(o->dw_gate, o->ld_dw_gate, d) ||
        bad_rows(o->dw_up, o->ld_dw_up, d) || bad_rows(o->dw_down, o->ld_dw_down, f) || bad_rows(o->dw_gate_in, o->ld_dw_gate_in, d) ||
        bad_rows(o->dw_up_in, o->ld_dw_up_in, d) || bad_rows(o->dw_down_in, o->ld_dw_down_in, f))
        return c.fail(DISTSIM_E_ARG, "gated ffn: rows closer together than they are long");
    return DISTSIM_OK;
}
}  // namespace

int distsim_gated_ffn_forward(distsim_ctx *ctx, void *stream, const distsim_gated_ffn *o)
{
    if (!ctx || !o) return DISTSIM_E_ARG;
    Call c(ctx, stream);
    int rc = c.begin();
    if (rc != DISTSIM_OK || (rc = check_ffn(c, o)) != DISTSIM_OK) return rc;
    const int64_t t = o->tokens, d = o->d_in, f = o->d_hidden;
    if (t == 0) return DISTSIM_OK;
    if (!o->gate != !o->up) return c.fail(DISTSIM_E_ARG, "gated ffn forward: gate and up are kept together");
    if (!o->x || !o->w_gate || !o->w_up || !o->w_down || !o->y) return c.fail(DISTSIM_E_ARG, "gated ffn forward: x, the weights and y are needed");

    Product ph, py;
    ph.m = t; ph.n = f; ph.k[0] = d; ph.epilogue = kEpiGated; ph.act = o->activation; ph.in_type = o->dtype;
    ph.bias[0] = o->b_gate; ph.bias[1] = o->b_up;
    py.m = t; py.n = d; py.k[0] = f; py.in_type = o->dtype; py.bias[0] = o->b_down;
    StandIn x = stand_in(o->x, o->ld_x, t, d, 2), wg = stand_in(o->w_gate, o->ld_w_gate, f, d, 2), wu = stand_in(o->w_up, o->ld_w_up, f, d, 2);
    StandIn wd = stand_in(o->w_down, o->ld_w_down, d, f, 2), r = stand_in(o->residual, o->ld_residual, t, d, 2), y = stand_in(o->y, o->ld_y, t, d, 2);
    StandIn g = stand_in(o->gate, o->ld_gate, t, f, 2), u = stand_in(o->up, o->ld_up, t, f, 2);
    StandIn h = stand_in(o->hidden, o->ld_hidden, t, f, 2);
    const ProductPlan plan_h = c.plan(ph, {}, {&g, &u}), plan_y = c.plan(py, {&r}, {&y});
    for (StandIn *s : {&x, &wg, &wu, &wd}) s->plan(c, true);
    h.plan(c, true, plan_h.pair);
    r.plan(c, plan_y.pair);
    y.plan(c, plan_y.pair, true);
    for (StandIn *s : {&g, &u}) s->plan(c, plan_h.pair, true);
    const size_t h_at = o->hidden ? 0 : c.room((size_t)t * padded_ld(f, 2) * 2);
    if ((rc = c.reserve()) != DISTSIM_OK) return rc;
    for (StandIn *s : {&x, &wg, &wu, &wd, &h, &r, &y, &g, &u}) s->place(c);
    if (!o->hidden) h.use = mat(c.at(h_at), padded_ld(f, 2));
    ph.a[0] = x.use;
    ph.b[0] = wg.use;
    ph.b[1] = wu.use;
    ph.out[0] = h.use;
    ph.out[1] = g.use;
    ph.out[2] = u.use;
    py.a[0] = h.use;
    py.b[0] = wd.use;
    py.in[0] = r.use;
    py.out[0] = y.use;
    cudaError_t e = cudaSuccess;
    TRY(fetch(c, {&x, &wg, &wu, &wd, &r}));
    TRY(launch_product(c.l, ph, plan_h));
    TRY(launch_product(c.l, py, plan_y));
    TRY(give_back(c, {&y, &g, &u, &h}));
    return c.end(e);
}

int distsim_gated_ffn_backward(distsim_ctx *ctx, void *stream, const distsim_gated_ffn *o)
{
    if (!ctx || !o) return DISTSIM_E_ARG;
    Call c(ctx, stream);
    int rc = c.begin();
    if (rc != DISTSIM_OK || (rc = check_ffn(c, o)) != DISTSIM_OK) return rc;
    const int64_t t = o->tokens, d = o->d_in, f = o->d_hidden;
    if (o->grad_dtype != o->dtype && o->grad_dtype != DISTSIM_F32) return c.fail(DISTSIM_E_UNSUPPORTED, "gated ffn: grad_dtype must be dtype or f32");
    const int ge = o->grad_dtype == DISTSIM_F32 ? 4 : 2;
    const bool inner = o->dx || o->dw_gate || o->dw_up || o->db_gate || o->db_up;     // what needs dg and du
    cudaError_t e = cudaSuccess;
    if (t == 0) {
        if ((rc = c.reserve()) != DISTSIM_OK) return rc;
        Move whole[3];
        int n = 0;
        const auto take = [&](const Matrix &dw, const Matrix &in, int64_t rows, int64_t cols) {
            if (dw.p && dw.p != in.p) whole[n++] = move_of(dw, in, rows, cols, ge);
        };
        take(mat(o->dw_gate, o->ld_dw_gate), mat(o->dw_gate_in, o->ld_dw_gate_in), f, d);
        take(mat(o->dw_up, o->ld_dw_up), mat(o->dw_up_in, o->ld_dw_up_in), f, d);
        take(mat(o->dw_down, o->ld_dw_down), mat(o->dw_down_in, o->ld_dw_down_in), d, f);
        TRY(launch_moves(c.l, whole, n));
        TRY(zero_vector(c, o->db_gate, f, o->grad_dtype));
        TRY(zero_vector(c, o->db_up, f, o->grad_dtype));
        TRY(zero_vector(c, o->db_down, d, o->grad_dtype));
        return c.end(e);
    }
    if (!o->dy || (inner && (!o->w_down || !o->gate || !o->up)) || (o->dx && (!o->w_gate || !o->w_up)) ||
        ((o->dw_gate || o->dw_up) && !o->x) || (o->dw_down && !o->hidden))
        return c.fail(DISTSIM_E_ARG, "gated ffn backward: a tensor that a wanted gradient needs is missing");

    Product pi, px, pw, pd;
    pi.m = t; pi.n = f; pi.k[0] = d; pi.b_mn = true; pi.epilogue = kEpiGatedBack; pi.act = o->activation; pi.in_type = o->dtype;
    px.m = t; px.n = d; px.k[0] = px.k[1] = f; px.b_mn = true; px.in_type = o->dtype;
    pw.m = f; pw.n = d; pw.k[0] = t; pw.a_mn = pw.b_mn = true; pw.in_type = o->dtype; pw.wide = ge == 4;
    const bool two = o->dw_gate && o->dw_up;
    pw.groups = two && !o->dw_gate_in == !o->dw_up_in ? 2 : 1;            // in one launch, unless one alone is added to
    pd.m = d; pd.n = f; pd.k[0] = t; pd.a_mn = pd.b_mn = true; pd.in_type = o->dtype; pd.wide = ge == 4;
    StandIn x = stand_in(o->x, o->ld_x, t, d, 2), dy = stand_in(o->dy, o->ld_dy, t, d, 2), h = stand_in(o->hidden, o->ld_hidden, t, f, 2);
    StandIn g = stand_in(o->gate, o->ld_gate, t, f, 2), u = stand_in(o->up, o->ld_up, t, f, 2);
    StandIn wg = stand_in(o->w_gate, o->ld_w_gate, f, d, 2), wu = stand_in(o->w_up, o->ld_w_up, f, d, 2), wd = stand_in(o->w_down, o->ld_w_down, d, f, 2);
    StandIn dx = stand_in(o->dx, o->ld_dx, t, d, 2), dwg = stand_in(o->dw_gate, o->ld_dw_gate, f, d, ge), dwu = stand_in(o->dw_up, o->ld_dw_up, f, d, ge);
    StandIn dwd = stand_in(o->dw_down, o->ld_dw_down, d, f, ge), dwgi = stand_in(o->dw_gate ? o->dw_gate_in : nullptr, o->ld_dw_gate_in, f, d, ge);
    StandIn dwui = stand_in(o->dw_up ? o->dw_up_in : nullptr, o->ld_dw_up_in, f, d, ge), dwdi = stand_in(o->dw_down ? o->dw_down_in : nullptr, o->ld_dw_down_in, d, f, ge);
    const ProductPlan plan_i = c.plan(pi, {&g, &u}, {}), plan_x = c.plan(px, {}, {&dx}), plan_w = c.plan(pw, {&dwgi, &dwui}, {&dwg, &dwu}),
                      plan_d = c.plan(pd, {&dwdi}, {&dwd});
    x.plan(c, o->dw_gate || o->dw_up);
    dy.plan(c, inner || o->dw_down);
    h.plan(c, o->dw_down);
    wd.plan(c, inner);
    for (StandIn *s : {&g, &u}) s->plan(c, inner && plan_i.pair);
    for (StandIn *s : {&wg, &wu}) s->plan(c, o->dx);
    dx.plan(c, plan_x.pair, true);
    for (StandIn *s : {&dwg, &dwu}) s->plan(c, plan_w.pair, true);
    dwd.plan(c, plan_d.pair, true);
    for (StandIn *s : {&dwgi, &dwui}) s->plan(c, plan_w.pair);
    dwdi.plan(c, plan_d.pair);
    const int64_t ld_i = padded_ld(f, 2);
    const size_t dg_at = inner ? c.room((size_t)t * ld_i * 2) : 0, du_at = inner ? c.room((size_t)t * ld_i * 2) : 0;
    // db_gate and db_up: from the first product's epilogue, which has dg and du before they are rounded
    const bool inner_sums = o->db_gate || o->db_up;
    const int64_t sum_rows = inner_sums ? product_sum_rows(pi, plan_i) : 0, ld_sums = ceil_div(f, 8) * 8;
    const size_t sums_at = c.room((size_t)(2 * sum_rows * ld_sums) * 4);
    const size_t part_at = inner_sums || o->db_down
        ? c.room((size_t)column_pass_partials(2 * f + d, c.l.sm_count) * 4) : 0;
    if ((rc = c.reserve()) != DISTSIM_OK) return rc;
    for (StandIn *s : {&x, &dy, &h, &g, &u, &wg, &wu, &wd, &dx, &dwg, &dwu, &dwd, &dwgi, &dwui, &dwdi}) s->place(c);
    const Matrix dg = inner ? mat(c.at(dg_at), ld_i) : Matrix{}, du = inner ? mat(c.at(du_at), ld_i) : Matrix{};
    float *partial = inner_sums || o->db_down ? c.at<float>(part_at) : nullptr;
    Matrix sums[2];

    TRY(fetch(c, {&dy, &wd, &g, &u, &wg, &wu, &x, &h, &dwgi, &dwui, &dwdi}));
    if (inner) {
        pi.a[0] = dy.use;
        pi.b[0] = wd.use;
        pi.in[0] = g.use;
        pi.in[1] = u.use;
        pi.out[0] = dg;
        pi.out[1] = du;
        for (int i = 0; i < 2 && inner_sums; ++i) {
            pi.sums[i] = c.at<float>(sums_at) + i * sum_rows * ld_sums;
            sums[i] = mat(pi.sums[i], ld_sums);
        }
        pi.sums_ld = ld_sums;
        TRY(launch_product(c.l, pi, plan_i));
    }
    if (o->dx) {
        px.a[0] = dg;
        px.a[1] = du;
        px.b[0] = wg.use;
        px.b[1] = wu.use;
        px.out[0] = dx.use;
        TRY(launch_product(c.l, px, plan_x));
    }
    if (o->dw_gate || o->dw_up) {
        const Matrix a[2] = {dg, du}, in[2] = {dwgi.use, dwui.use}, out[2] = {dwg.use, dwu.use};
        pw.b[0] = x.use;
        for (int first = o->dw_gate ? 0 : 1; first < (o->dw_up ? 2 : 1); first += pw.groups) {
            for (int i = 0; i < pw.groups; ++i) {
                pw.a[i] = a[first + i];
                pw.in[i] = in[first + i];
                pw.out[i] = out[first + i];
            }
            TRY(launch_product(c.l, pw, plan_w));
        }
    }
    if (o->dw_down) {
        pd.a[0] = dy.use;
        pd.b[0] = h.use;
        pd.in[0] = dwdi.use;
        pd.out[0] = dwd.use;
        TRY(launch_product(c.l, pd, plan_d));
    }
    TRY(give_back(c, {&dx, &dwg, &dwu, &dwd}));
    ColumnPass pass = column_pass(c, o->dtype, t, o->grad_dtype, partial);
    if (o->db_gate) pass.part[0] = {f, sums[0], o->db_gate, sum_rows};
    if (o->db_up) pass.part[1] = {f, sums[1], o->db_up, sum_rows};
    if (o->db_down) pass.part[2] = {d, dy.use, o->db_down};
    TRY(launch_column_pass(c.l, pass));
    return c.end(e);
}

namespace {
// Common checks of both directions, and what both hand to the kernels.
int check_norm(Call &c, const distsim_residual_norm *o, ResidualNorm &r)
{
    if (o->tokens < 0 || o->cols < 1 || o->reserved != 0 || (o->kind != 0 && o->kind != 1)) return c.fail(DISTSIM_E_ARG, "residual norm: sizes or kind");
    if (o->cols > DISTSIM_MAX_COLS) return c.fail(DISTSIM_E_UNSUPPORTED, "residual norm: more than DISTSIM_MAX_COLS columns");
    if (o->dtype < DISTSIM_BF16 || o->dtype > DISTSIM_F32) return c.fail(DISTSIM_E_UNSUPPORTED, "residual norm: unknown dtype");
    if (!(o->p >= 0.0 && o->p < 1.0) || !(o->eps >= 0.0)) return c.fail(DISTSIM_E_ARG, "residual norm: need 0 <= p < 1 and eps >= 0");
    if ((o->post_bias && !o->post_weight) || (o->bias && !o->weight)) return c.fail(DISTSIM_E_ARG, "residual norm: a bias without its weight");
    const int64_t n = o->cols;
    if (bad_rows(o->x, o->ld_x, n) || bad_rows(o->residual, o->ld_residual, n) || bad_rows(o->h, o->ld_h, n) || bad_rows(o->y, o->ld_y, n) ||
        bad_rows(o->dy, o->ld_dy, n) || bad_rows(o->dh, o->ld_dh, n) || bad_rows(o->dx, o->ld_dx, n) || bad_rows(o->dresidual, o->ld_dresidual, n))
        return c.fail(DISTSIM_E_ARG, "residual norm: rows closer together than they are long");
    const double q = o->p * 4294967296.0;
    uint64_t threshold = (uint64_t)q;
    const double rest = q - (double)threshold;
    if (rest > 0.5 || (rest == 0.5 && (threshold & 1))) ++threshold;                   // to nearest, halves to even
    if (threshold > 0xffffffffull) return c.fail(DISTSIM_E_ARG, "residual norm: p rounds to 1");
    r.tokens = o->tokens;
    r.cols = n;
    r.type = o->dtype;
    r.grad_type = o->grad_dtype;
    r.rms = o->kind == 1;
    r.alpha = (float)o->alpha;
    r.eps = (float)o->eps;
    r.threshold = (uint32_t)threshold;
    r.keep_scale = (float)(1.0 / (1.0 - (double)threshold / 4294967296.0));
    r.seed = o->seed;
    r.offset = o->offset;
    r.x = mat(o->x, o->ld_x);
    r.h = mat(o->h, o->ld_h);
    r.gate = o->gate;
    r.post_weight = o->post_weight;
    r.post_bias = o->post_bias;
    r.weight = o->weight;
    r.bias = o->bias;
    return DISTSIM_OK;
}
}  // namespace

int distsim_residual_norm_forward(distsim_ctx *ctx, void *stream, const distsim_residual_norm *o)
{
    if (!ctx || !o) return DISTSIM_E_ARG;
    Call c(ctx, stream);
    ResidualNorm r;
    int rc = c.begin();
    if (rc != DISTSIM_OK || (rc = check_norm(c, o, r)) != DISTSIM_OK) return rc;
    if (o->tokens == 0) return DISTSIM_OK;                            // empty tensors may have no address
    if (!o->weight != !o->y) return c.fail(DISTSIM_E_ARG, "residual norm forward: y comes with weight");
    if (!o->h && !o->y) return c.fail(DISTSIM_E_ARG, "residual norm forward: neither h nor y is wanted");
    if (!o->x) return c.fail(DISTSIM_E_ARG, "residual norm forward: x is needed");
    r.residual = mat(o->residual, o->ld_residual);
    r.y = mat(o->y, o->ld_y);
    if ((rc = c.reserve()) != DISTSIM_OK) return rc;
    return c.end(launch_residual_norm_forward(c.l, r));
}

int distsim_residual_norm_backward(distsim_ctx *ctx, void *stream, const distsim_residual_norm *o)
{
    if (!ctx || !o) return DISTSIM_E_ARG;
    Call c(ctx, stream);
    ResidualNorm r;
    int rc = c.begin();
    if (rc != DISTSIM_OK || (rc = check_norm(c, o, r)) != DISTSIM_OK) return rc;
    if (o->grad_dtype != o->dtype && o->grad_dtype != DISTSIM_F32) return c.fail(DISTSIM_E_UNSUPPORTED, "residual norm: grad_dtype must be dtype or f32");
    if (((o->dpost_weight || o->dpost_bias) && !o->post_weight) || (o->dgate && !o->gate) || ((o->dweight || o->dbias) && !o->weight))
        return c.fail(DISTSIM_E_ARG, "residual norm backward: a gradient of a parameter that is not given");
    cudaError_t e = cudaSuccess;
    if (o->tokens == 0) {
        if ((rc = c.reserve()) != DISTSIM_OK) return rc;
        for (void *v : {o->dgate, o->dpost_weight, o->dpost_bias, o->dweight, o->dbias}) TRY(zero_vector(c, v, o->cols, o->grad_dtype));
        return c.end(e);
    }
    if ((o->weight && (!o->h || !o->dy)) || (!o->weight && !o->dh) || ((o->post_weight || o->dgate) && !o->x))
        return c.fail(DISTSIM_E_ARG, "residual norm backward: h and dy (with weight), dh (without) and x (with post_weight or dgate) are needed");
    r.dy = mat(o->weight ? o->dy : nullptr, o->ld_dy);
    r.dh = mat(o->dh, o->ld_dh);
    r.dx = mat(o->dx, o->ld_dx);
    r.dresidual = mat(o->dresidual, o->ld_dresidual);
    r.dgate = o->dgate;
    r.dpost_weight = o->dpost_weight;
    r.dpost_bias = o->dpost_bias;
    r.dweight = o->dweight;
    r.dbias = o->dbias;
    const size_t part_at = c.room((size_t)residual_norm_partials(o->cols, c.l.sm_count) * 4);
    if ((rc = c.reserve()) != DISTSIM_OK) return rc;
    r.partial = c.at<float>(part_at);
    return c.end(launch_residual_norm_backward(c.l, r));
}

}  // extern "C"
