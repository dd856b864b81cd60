"""Paths of the operators' kernels that the shapes of test_operators do not reach.  Plain implementations in
64 bits and tolerances as there, unless a test derives its own."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from .test_operators import U32, act64, close, ctx, ffn_case, linear_case, plan, randn, room  # noqa: E402, F401


@pytest.mark.gpu
@pytest.mark.parametrize("plan", [0, -1, 1, -2], indirect=True)
@pytest.mark.parametrize("shape", [(300, 72, 257, 143), (520, 131, 325, 3), (40, 65, 263, 1)])
def test_rows_with_gaps_that_an_odd_width_leaves(ctx, plan, shape):
    # rows that start on 16-byte boundaries and end off one: what lies between them is not the operator's
    from paper_2306_08423_b200 import engine as E
    t, d, f, gap = shape
    rng = np.random.default_rng(t)
    dt = torch.bfloat16
    gap_d = -d % 8 + 8

    def rows(n, cols, dtype=dt):
        align = 16 // torch.empty((), dtype=dtype).element_size()
        pad = gap if cols == f else gap_d
        assert (cols + pad) % align == 0
        return room(n, cols, dtype, pad, 0)
    x, w, b, dy = linear_case(rng, t, d, f, 0, 0, dt)
    (y, y_ok), (z, z_ok) = rows(t, f), rows(t, f)
    E.distsim_linear_forward(ctx, x, w, y, bias=b, preact=z)
    want = x.double() @ w.double().T + b.double()
    for name, v in (("y", y), ("z", z)):
        close(name, v, want, (d + 2) * U32 * (x.double().abs() @ w.double().abs().T + b.double().abs()))
    for ok in (y_ok, z_ok):
        ok()
    for grad in (dt, torch.float32):
        (dx, dx_ok), (dw, dw_ok) = rows(t, d), rows(f, d, grad)
        E.distsim_linear_backward(ctx, dy, x, w, dx=dx, dweight=dw)
        close("dx", dx, dy.double() @ w.double(), (f + 2) * U32 * dy.double().abs() @ w.double().abs())
        close("dw", dw, dy.double().T @ x.double(), (t + 2) * U32 * dy.double().abs().T @ x.double().abs())
        dx_ok()
        dw_ok()
    o = ffn_case(rng, t, d, f, 0, 0, dt)
    out = {n: rows(t, f) for n in ("hidden", "gate", "up")}
    out["y"] = rows(t, d)
    E.distsim_gated_ffn_forward(ctx, **o, **{n: q[0] for n, q in out.items()}, activation="none")
    h = out["hidden"][0].double()
    close("y", out["y"][0], h @ o["w_down"].double().T, (f + 3) * U32 * (h.abs() @ o["w_down"].double().abs().T))
    grads = dict(dx=rows(t, d), dw_gate=rows(f, d), dw_up=rows(f, d), dw_down=rows(d, f))
    dy = randn(rng, t, d, dtype=dt)
    E.distsim_gated_ffn_backward(ctx, dy, **o, hidden=out["hidden"][0], gate=out["gate"][0], up=out["up"][0],
                                 **{n: q[0] for n, q in grads.items()}, activation="none")
    close("dw_down", grads["dw_down"][0], dy.double().T @ h, (t + 2) * U32 * dy.double().abs().T @ h.abs())
    for _, ok in (*out.values(), *grads.values()):
        ok()


@pytest.mark.gpu
def test_replay_after_a_larger_call():
    # a graph's scratch stays when a later call needs more; on a context of its own, whose scratch is that small
    from paper_2306_08423_b200 import engine as E
    c = E.Context(0)
    try:
        rng = np.random.default_rng(6)
        t, d, f = 700, 136, 264
        x, w, _, dy = linear_case(rng, t, d, f, 1, 1, torch.bfloat16)
        z = randn(rng, t, f, dtype=torch.bfloat16)

        def outputs():
            return [torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((t, d), (f, d), (f,))]

        def run(o):
            E.distsim_linear_backward(c, dy, x, w, dx=o[0], dweight=o[1], dbias=o[2], preact=z, activation="gelu")
        eager, replayed = outputs(), outputs()
        run(eager)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(replayed)
        large = linear_case(rng, 9000, 640, 1032, 1, 1, torch.bfloat16)
        out = [torch.empty(9000, 640, dtype=torch.bfloat16, device="cuda"), torch.empty(1032, 640, dtype=torch.bfloat16, device="cuda")]
        E.distsim_linear_backward(c, large[3], large[0], large[1], dx=out[0], dweight=out[1], preact=large[3], activation="gelu")
        other = torch.full((1 << 26,), float("nan"), device="cuda")      # takes what has been freed
        for _ in range(2):
            for v in replayed:
                v.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, replayed))
        assert bool(torch.isnan(other).all())
        # a call that a capture cannot hold is refused before anything is captured
        wider = linear_case(rng, 30000, 640, 1032, 1, 1, torch.bfloat16)
        graph = torch.cuda.CUDAGraph()
        out = torch.empty(30000, 640, dtype=torch.bfloat16, device="cuda")
        with torch.cuda.graph(graph):
            with pytest.raises(E.DistsimError, match="captured") as e:
                E.distsim_linear_backward(c, wider[3], wider[0], wider[1], dx=out, preact=wider[3], activation="gelu")
            replayed[2].zero_()
        assert e.value.code == E.E_STATE
        E.distsim_linear_backward(c, wider[3], wider[0], wider[1], dx=out, preact=wider[3], activation="gelu")
        assert bool(torch.isfinite(out).all())
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_bias_gradients_of_more_than_a_million_columns(ctx, grad):
    from paper_2306_08423_b200 import engine as E
    t, d, f, dt = 5, 16, 2 ** 20 + 300, torch.bfloat16
    rng = np.random.default_rng(8)
    x, w, dy = randn(rng, t, d, dtype=dt), randn(rng, f, d, dtype=dt), randn(rng, t, f, dtype=dt)
    db, dx = torch.full((f,), 7.0, dtype=grad, device="cuda"), torch.empty_like(x)
    E.distsim_linear_backward(ctx, dy, x, w, dx=dx, dbias=db)
    close("db", db, dy.double().sum(0), (t + 2) * U32 * dy.double().abs().sum(0))
    close("dx", dx, dy.double() @ w.double(), (f + 2) * U32 * dy.double().abs() @ w.double().abs())
    # no activation: du = dh g, dg = dh u, rounded to 2^-8 at the most
    g, u, dy, wd = randn(rng, t, f, dtype=dt), dy, x, randn(rng, d, f, dtype=dt)
    grads = [torch.full((n,), 7.0, dtype=grad, device="cuda") for n in (f, f, d)]
    E.distsim_gated_ffn_backward(ctx, dy, x, w, w, wd, None, g, u, db_gate=grads[0], db_up=grads[1], db_down=grads[2], activation="none")
    dh = dy.double() @ wd.double()
    dh_off = (d + 2) * U32 * dy.double().abs() @ wd.double().abs()
    for name, got, other in (("db_gate", grads[0], u.double()), ("db_up", grads[1], g.double())):
        close(name, got, (dh * other).sum(0), ((2.0 ** -8 + (t + 2) * U32) * (dh * other).abs() + 2 * dh_off * other.abs()).sum(0))
    close("db_down", grads[2], dy.double().sum(0), (t + 2) * U32 * dy.double().abs().sum(0))


@pytest.mark.gpu
@pytest.mark.parametrize("plan", [-1, 1, -2], indirect=True)
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_negative_tails_of_activations(ctx, plan, act):
    """Values and slopes far below zero are products of small numbers, to a relative error: exponentials of arguments
    up to 2^7 in powers of two, rounded twice (2^7 2^-23 ln 2), and ten further roundings of 2^-23."""
    from paper_2306_08423_b200 import engine as E
    e = 2.0 ** 7 * U32 * math.log(2) + 10 * U32
    lowest = {"gelu": -12.0, "gelu_tanh": -9.0, "silu": -60.0}[act]
    z = torch.linspace(lowest, -1.5, 8 * 40, device="cuda").bfloat16().view(40, 8)
    eye = torch.eye(8, device="cuda").bfloat16()
    y, dx = torch.empty_like(z), torch.empty_like(z)
    E.distsim_linear_forward(ctx, z, eye, y, activation=act)
    want, slope = act64(z.double(), act)
    if act == "gelu":                                # 1 + erf cancels in 64 bits as well
        want = 0.5 * z.double() * torch.special.erfc(-z.double() / math.sqrt(2))
        slope = want / z.double() + z.double() * torch.exp(-z.double().square() / 2) / math.sqrt(2 * math.pi)
    elif act == "gelu_tanh":
        k = math.sqrt(8 / math.pi)
        s = torch.sigmoid(k * (z.double() + 0.044715 * z.double() ** 3))
        want = z.double() * s
        slope = s + want * (1 - s) * k * (1 + 0.134145 * z.double().square())
    bad = (y.double() - want).abs() > (2.0 ** -8 + e) * want.abs()
    assert not bad.any(), (z[bad], y[bad], want[bad])
    # the slope's two terms have opposite signs; by the preceding value, dz = slope (dy = 1), rounded on its way to dx
    E.distsim_linear_backward(ctx, torch.ones_like(z), z, eye, dx=dx, preact=z, activation=act)
    terms = (want / z.double()).abs() * (1 + 2 * z.double().abs() * (1 + z.double().square()))
    bad = (dx.double() - slope).abs() > (2.0 ** -8 + e) * slope.abs() + e * terms
    assert not bad.any(), (z[bad], dx[bad], slope[bad])
    if act == "gelu":                                # at the ends: z, 0, and no number for none
        z[0, :3] = torch.tensor([math.inf, -math.inf, math.nan], device="cuda").bfloat16()
        E.distsim_linear_forward(ctx, z.T.contiguous(), torch.eye(40, device="cuda").bfloat16()[:1], y.view(-1)[:8].view(8, 1), activation=act)
        ends = y.view(-1)[:3]
        assert ends[0] == math.inf and ends[1] == 0 and torch.isnan(ends[2])


@pytest.mark.gpu
@pytest.mark.parametrize("plan", [-1, 1, -2], indirect=True)
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_slopes_of_arguments_whose_square_is_infinite(ctx, plan, act):
    # they are 1 and 0, and the values z and 0
    from paper_2306_08423_b200 import engine as E
    z = torch.tensor([3e38, 1e20, 2e19, 1e4, 200.0, -3e38, -1e20, -200.0], device="cuda").bfloat16().expand(16, 8).contiguous()
    eye = torch.eye(8, device="cuda").bfloat16()
    dx, dg = torch.empty_like(z), torch.empty_like(z)
    E.distsim_linear_backward(ctx, torch.ones_like(z), z, eye, dx=dx, preact=z, activation=act)
    up = (z > 0).to(z.dtype)
    assert torch.equal(dx, up)
    # the gated block's: dx = dg + du, dh = 1, u = 1
    du = torch.where(z > 0, z, torch.zeros_like(z))
    E.distsim_gated_ffn_backward(ctx, torch.ones_like(z), z, eye, eye, eye, None, z, torch.ones_like(z), dx=dg, activation=act)
    assert torch.equal(dg, (up.float() + du.float()).bfloat16())


@pytest.mark.gpu
@pytest.mark.parametrize("plan", [0, -1, 1, 2, 4, -2, -3, -4], indirect=True)
@pytest.mark.parametrize("shape", [(1, 64, 64, 0, 0), (7, 100, 130, 0, 0), (64, 136, 263, 1, 0), (129, 72, 520, 3, 1), (385, 64, 1030, 0, 0), (2100, 64, 96, 0, 0)])
@pytest.mark.parametrize("act", ["silu", "none"])
def test_gated_bias_gradients_are_summed_before_rounding(ctx, plan, shape, act):
    """As the linear one's: what dg and du lose to bf16 on their way into the products does not reach db_gate and db_up.
    Off by dh's sum (k 2^-23 of its magnitudes), the activation's 2^-19 and the column sum's own 2^-23 a term."""
    from paper_2306_08423_b200 import engine as E
    t, d, f, pad, shift = shape
    rng = np.random.default_rng(t + f)
    dt = torch.bfloat16
    o = ffn_case(rng, *shape, dt)
    dy, g, u = randn(rng, t, d, dtype=dt), *(randn(rng, t, f, dtype=dt, pad=pad, shift=shift) for _ in range(2))
    db = {n: torch.full((k,), 7.0, device="cuda") for n, k in (("db_gate", f), ("db_up", f), ("db_down", d))}
    dx = torch.empty(t, d, dtype=dt, device="cuda")
    E.distsim_gated_ffn_backward(ctx, dy, **o, hidden=None, gate=g, up=u, dx=dx, activation=act, **db)
    dh = dy.double() @ o["w_down"].double()
    dh_off = (d + 2) * U32 * dy.double().abs() @ o["w_down"].double().abs()
    val, slope = act64(g.double(), act)
    approx = 2.0 ** -19 * g.double().abs().clamp_min(1) if act != "none" else 0
    dg, du = dh * u.double() * slope, dh * val
    for name, q, off in (("db_gate", dg, u.double().abs() * (dh_off * slope.abs() + (dh.abs() + dh_off) * approx)),
                         ("db_up", du, dh_off * val.abs() + (dh.abs() + dh_off) * approx)):
        close(name, db[name], q.sum(0), off.sum(0) + (t + 4) * U32 * q.abs().sum(0))
    close("db_down", db["db_down"], dy.double().sum(0), (t + 2) * U32 * dy.double().abs().sum(0))
    again = {n: torch.empty_like(v) for n, v in db.items()}
    E.distsim_gated_ffn_backward(ctx, dy, **o, hidden=None, gate=g, up=u, activation=act, **again)
    assert all(torch.equal(v, db[n]) for n, v in again.items())
