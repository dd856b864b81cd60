"""Paths of the operators' kernels that the shapes of test_operators do not reach.  Plain implementations in
64 bits and tolerances as there, unless a test derives its own."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from .test_operators import U32, act64, close, ctx, ffn_case, linear_case, norm_case, plan, randn, room, unit  # noqa: E402, F401


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
"""Paths of the operators' kernels that the shapes of test_operators do not reach.  Plain implementations in
64 bits and tolerances as there, unless a test derives its own."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from .test_operators import U32, act64, close, ctx, ffn_case, linear_case, norm_case, plan, randn, room, unit  # noqa: E402, F401


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


# ---------------------------------------------------------------- several pieces, many tiles, subsets

def near(name, got, want, bound):
    """The 2-norm of the difference, over that of the result."""
    off = float((got.double() - want).norm() / want.norm())
    assert off <= bound, (name, off, bound)


FEW_PLANS = pytest.mark.parametrize("plan", [0, -1, 1, 2, 4], indirect=True)


# 32-bit gradients are summed in pieces of 1024 terms.  The tensor core shrinks a sum of k terms by 9e-10 k of itself, so
# every piece, and with them the sum, by at most 9.2e-7; the pieces' additions (at most eight, to nearest) add 2^-24 times
# 0.6 each: 3e-7 at the most.
PIECES = 1.25e-6


@pytest.mark.gpu
@FEW_PLANS
@pytest.mark.parametrize("tokens", [1024, 1025, 2049, 8193])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_gradients_in_pieces(ctx, plan, tokens, accumulate):
    from paper_2306_08423_b200 import engine as E
    rng = np.random.default_rng(tokens)
    d, f, dt = 136, 264, torch.bfloat16
    x, _, _, dy = linear_case(rng, tokens, d, f, 0, 0, dt)
    w = randn(rng, f, d, dtype=dt)
    old = randn(rng, f, d, dtype=torch.float32, scale=tokens ** 0.5) if accumulate else None
    dw, dw_ok = room(f, d, torch.float32, 1, 3)
    db = torch.empty(f, device="cuda")
    E.distsim_linear_backward(ctx, dy, x, w, dweight=dw, dbias=db, dweight_in=old)
    want = dy.double().T @ x.double() + (old.double() if accumulate else 0)
    near("dw", dw, want, PIECES)
    # no element is off by more than the bound on a sum of all its magnitudes
    close("dw", dw, want, PIECES * (dy.double().abs().T @ x.double().abs()) + (2.0 ** -23 * old.double().abs() if accumulate else 0))
    close("db", db, dy.double().sum(0), (tokens + 2) * U32 * dy.double().abs().sum(0))
    dw_ok()


@pytest.mark.gpu
@FEW_PLANS
@pytest.mark.parametrize("tokens", [1025, 4097])
def test_gated_weight_gradients_in_pieces(ctx, plan, tokens):
    # both weights' gradients in one launch; dg and du are rounded on their way into it, which the bounds allow for
    from paper_2306_08423_b200 import engine as E
    rng = np.random.default_rng(tokens)
    d, f, dt = 72, 136, torch.float16
    o = ffn_case(rng, tokens, d, f, 0, 0, dt)
    dy, g, u, h = (randn(rng, tokens, n, dtype=dt) for n in (d, f, f, f))
    out = {n: room(a, b, torch.float32) for n, a, b in (("dw_gate", f, d), ("dw_up", f, d), ("dw_down", d, f))}
    E.distsim_gated_ffn_backward(ctx, dy, **o, hidden=h, gate=g, up=u, **{n: q[0] for n, q in out.items()}, activation="silu")
    dh = dy.double() @ o["w_down"].double()
    val, slope = act64(g.double(), "silu")
    dg, du, x = dh * u.double() * slope, dh * val, o["x"].double()
    near("dw_down", out["dw_down"][0], dy.double().T @ h.double(), PIECES)
    # independent roundings of the terms to 2^-11: as much of the sum's norm at the most
    near("dw_gate", out["dw_gate"][0], dg.T @ x, 2.0 ** -11)
    near("dw_up", out["dw_up"][0], du.T @ x, 2.0 ** -11)
    for name, q in (("dw_gate", dg), ("dw_up", du)):
        close(name, out[name][0], q.T @ x, (2.0 ** -11 + 2.0 ** -17) * (q.abs().T @ x.abs()) + 2.0 ** -24 * x.abs().sum(0))
    for _, ok in out.values():
        ok()


# 16 x 13 tiles of 256 x 256 (16 x 25 of the gated block's 128 columns): each of the 74 pairs takes two to six in turn
MANY = (3845, 200, 3081)
TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
LAYOUTS = pytest.mark.parametrize("pad,shift", [(7, 0), (15, 8)])       # rows of 3088 and 208, of 3096 and 216
PERSISTENT = pytest.mark.parametrize("plan", [-1], indirect=True)


@pytest.mark.gpu
@PERSISTENT
@TYPES
@LAYOUTS
def test_many_tiles_linear_forward(ctx, plan, dtype, pad, shift):
    from paper_2306_08423_b200 import engine as E
    t, d, f = MANY
    rng = np.random.default_rng(1)
    x, w = randn(rng, t, d, dtype=dtype), randn(rng, f, d, dtype=dtype, scale=d ** -0.5)
    b, r = randn(rng, f, dtype=dtype), randn(rng, t, f, dtype=dtype, pad=pad, shift=shift)
    zz = x.double() @ w.double().T
    off = (d + 2) * U32 * (x.double().abs() @ w.double().abs().T + 4)
    for act, bias, residual, save in (("gelu", True, True, True), ("none", False, False, False), ("silu", True, False, True), ("none", True, True, False)):
        y, y_ok = room(t, f, dtype, pad, shift)
        z, z_ok = room(t, f, dtype, pad, shift)
        E.distsim_linear_forward(ctx, x, w, y, bias=b if bias else None, residual=r if residual else None, preact=z if save else None, activation=act)
        v = zz + (b.double() if bias else 0)
        close((act, "y"), y, act64(v, act)[0] + (r.double() if residual else 0), 1.2 * off + 2.0 ** -20 * v.abs().clamp_min(1))
        y_ok()
        if save:
            close((act, "z"), z, v, off)
            z_ok()


@pytest.mark.gpu
@PERSISTENT
@TYPES
@LAYOUTS
def test_many_tiles_gated(ctx, plan, dtype, pad, shift):
    from paper_2306_08423_b200 import engine as E
    t, d, f = MANY
    rng = np.random.default_rng(2)
    o = ffn_case(rng, t, d, f, 0, 0, dtype)
    o["w_down"] = randn(rng, d, f, dtype=dtype, scale=f ** -0.5, pad=7)
    v = {k: q.double() for k, q in o.items()}
    bg, bu, bd = (randn(rng, n, dtype=dtype, scale=0.2) for n in (f, f, d))
    y, y_ok = room(t, d, dtype)
    kept = {n: room(t, f, dtype, pad, shift) for n in ("hidden", "gate", "up")}
    E.distsim_gated_ffn_forward(ctx, **o, y=y, b_gate=bg, b_up=bu, b_down=bd, **{n: q[0] for n, q in kept.items()}, activation="silu")
    gg, uu = v["x"] @ v["w_gate"].T + bg.double(), v["x"] @ v["w_up"].T + bu.double()
    g_off = (d + 2) * U32 * (v["x"].abs() @ v["w_gate"].abs().T + 1)
    u_off = (d + 2) * U32 * (v["x"].abs() @ v["w_up"].abs().T + 1)
    a = act64(gg, "silu")[0]
    h_off = uu.abs() * (1.2 * g_off + 2.0 ** -20 * gg.abs().clamp_min(1)) + (a.abs() + g_off) * u_off + U32 * (a * uu).abs()
    close("gate", kept["gate"][0], gg, g_off)
    close("up", kept["up"][0], uu, u_off)
    close("hidden", kept["hidden"][0], a * uu, h_off)
    hh = kept["hidden"][0].double()                                    # as it enters the second product
    close("y", y, hh @ v["w_down"].T + bd.double(), (f + 3) * U32 * (hh.abs() @ v["w_down"].abs().T + 1))
    y_ok()
    for _, ok in kept.values():
        ok()
    # backward; dg and du show in dx
    g, u = (randn(rng, t, f, dtype=dtype, pad=pad, shift=shift) for _ in range(2))
    dy = randn(rng, t, d, dtype=dtype)
    dx, dx_ok = room(t, d, dtype)
    E.distsim_gated_ffn_backward(ctx, dy, **o, hidden=None, gate=g, up=u, dx=dx, activation="silu")
    dh = dy.double() @ v["w_down"]
    dh_off = (d + 2) * U32 * dy.double().abs() @ v["w_down"].abs()
    val, slope = act64(g.double(), "silu")
    approx = 2.0 ** -19 * g.double().abs().clamp_min(1)

    def rounded(q, off):
        return off + unit(dtype) * (q.abs() + off) + 2.0 ** -25
    dg, du = dh * u.double() * slope, dh * val
    dg_off = rounded(dg, u.double().abs() * (dh_off * slope.abs() + (dh.abs() + dh_off) * approx))
    du_off = rounded(du, dh_off * val.abs() + (dh.abs() + dh_off) * approx)
    want = dg @ v["w_gate"] + du @ v["w_up"]
    close("dx", dx, want, (2 * f + 3) * U32 * (dg.abs() @ v["w_gate"].abs() + du.abs() @ v["w_up"].abs()) + dg_off @ v["w_gate"].abs() + du_off @ v["w_up"].abs())
    # independent roundings: of dx and of every term, 2^-8 or 2^-11 of the norm at the most each
    near("dx", dx, want, 2 * unit(dtype))
    dx_ok()


@pytest.mark.gpu
@PERSISTENT
@pytest.mark.parametrize("tokens", [200, 1100, 2200])
@pytest.mark.parametrize("accumulate", [False, True])
def test_many_tiles_of_weight_gradients(ctx, plan, tokens, accumulate):
    # tiles in turn, in one piece and in several, with the running sum in between
    from paper_2306_08423_b200 import engine as E
    d, f, dt = 3081, 3845, torch.bfloat16
    rng = np.random.default_rng(3)
    x, dy, w = randn(rng, tokens, d, dtype=dt, pad=7), randn(rng, tokens, f, dtype=dt, pad=3), randn(rng, f, d, dtype=dt)
    old = randn(rng, f, d, dtype=torch.float32, scale=tokens ** 0.5, pad=3) if accumulate else None
    dw, dw_ok = room(f, d, torch.float32, 3, 4)
    E.distsim_linear_backward(ctx, dy, x, w, dweight=dw, dweight_in=old)
    want = dy.double().T @ x.double() + (old.double() if accumulate else 0)
    near("dw", dw, want, PIECES)
    close("dw", dw, want, PIECES * (dy.double().abs().T @ x.double().abs()) + (2.0 ** -23 * old.double().abs() if accumulate else 0))
    dw_ok()


@pytest.mark.gpu
@pytest.mark.parametrize("plan", [0, -1, 2, -3], indirect=True)
@pytest.mark.parametrize("shape", [(7, 100, 130, 0, 0), (300, 136, 264, 8, 0), (129, 256, 257, 3, 1)])
@pytest.mark.parametrize("act", ["relu", "none", "silu"])
def test_gated_gradients_one_by_one(ctx, plan, shape, act):
    # any subset of the gradients gives the same bits as all of them together
    from paper_2306_08423_b200 import engine as E
    t, d, f, pad, shift = shape
    rng = np.random.default_rng(t)
    dt = torch.bfloat16
    o = ffn_case(rng, *shape, dt)
    dy, g, u, h = (randn(rng, t, n, dtype=dt, pad=pad, shift=shift) for n in (d, f, f, f))
    sizes = dict(dx=(t, d), dw_gate=(f, d), dw_up=(f, d), dw_down=(d, f), db_gate=(f,), db_up=(f,), db_down=(d,))

    def run(names):
        out = {n: torch.full(sizes[n], 7.0, dtype=dt, device="cuda") for n in names}
        need = set(names) - {"dw_down", "db_down"}
        E.distsim_gated_ffn_backward(ctx, dy, o["x"], o["w_gate"], o["w_up"], o["w_down"], h if "dw_down" in names else None,
                                     g if need else None, u if need else None, activation=act, **out)
        return out
    whole = run(sizes)
    for names in [(n,) for n in sizes] + [("dw_gate", "db_up"), ("dw_up", "dx"), ("db_gate", "db_down"), ("dw_gate", "dw_up")]:
        for n, v in run(names).items():
            assert torch.equal(v, whole[n]), (names, n)
    dh = dy.double() @ o["w_down"].double()
    dh_off = (d + 2) * U32 * dy.double().abs() @ o["w_down"].double().abs()
    val, slope = act64(g.double(), act)
    approx = 2.0 ** -19 * g.double().abs().clamp_min(1)
    x = o["x"].double()
    for name, q, off in (("dw_gate", dh * u.double() * slope, u.double().abs() * (dh_off * slope.abs() + (dh.abs() + dh_off) * approx)),
                         ("dw_up", dh * val, dh_off * val.abs() + (dh.abs() + dh_off) * approx)):
        off = off + unit(dt) * (q.abs() + off)
        close((act, name), whole[name], q.T @ x, (t + 2) * U32 * q.abs().T @ x.abs() + off.T @ x.abs())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(9, 256, 0, 0), (40, 768, 0, 0), (33, 1000, 1, 3), (3, 5000, 0, 0), (2, 12288, 0, 0), (300, 100, 0, 1)])
@pytest.mark.parametrize("parts", [(1, 1, 1, 1, 1, 0.1), (0, 1, 1, 1, 1, 0.25), (1, 0, 1, 1, 1, 0.0)])
def test_norm_gradients_one_by_one(ctx, dtype, shape, parts):
    """Any subset of the gradients, no dx among them, gives what all of them together give: the same bits where rows
    are aligned.  Others are cut into pieces by where most of a call's tensors start, so sums may go in another order:
    their norm moves by the 64 roundings of 2^-24 that a norm's values may be off by, and values of 16 bits that fall
    to the other side by 2^-7 of themselves, at most one in 2^6 (64 2^-24 against a spacing of 2^-8 is one in 2^10)."""
    from paper_2306_08423_b200 import engine as E
    t, n, pad, shift = shape
    post, pre = parts[:2]
    rng = np.random.default_rng(n)
    x, _, o, bias = norm_case(rng, shape, parts, dtype)
    h, dy, dh = (randn(rng, t, n, dtype=dtype, pad=pad, shift=shift) for _ in range(3))
    names = ["dx", "dresidual", "dgate"] + (["dpost_weight", "dpost_bias"] if post else []) + (["dweight", "dbias"] if pre else [])

    def run(wanted):
        out = {k: torch.full((t, n) if k in ("dx", "dresidual") else (n,), 7.0, dtype=dtype, device="cuda") for k in wanted}
        need_x = post or "dgate" in wanted
        E.distsim_residual_norm_backward(ctx, x if need_x else None, h if pre else None, dy=dy if pre else None, dh=dh, kind="layer", alpha=0.75,
                                         p=parts[5], seed=5, offset=9, **out, **o)
        return out
    whole = run(names)
    for wanted in [(k,) for k in names] + [tuple(names[1:]), ("dx", "dgate"), tuple(k for k in names if k not in ("dresidual", "dgate"))]:
        for k, v in run(wanted).items():
            if pad == shift == 0:
                assert torch.equal(v, whole[k]), (wanted, k)
            else:
                near((wanted, k), v, whole[k].double(), 64 * 2.0 ** -24 + (2.0 ** -10 if dtype != torch.float32 else 0))


@pytest.mark.gpu
@pytest.mark.parametrize("plan", [0, -1, 1, 2], indirect=True)
@pytest.mark.parametrize("shape", [(7, 100, 130, 0, 0), (300, 136, 264, 8, 0), (1300, 72, 257, 3, 1)])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_gated_weight_gradients_added_to_earlier_ones(ctx, plan, shape, grad):
    from paper_2306_08423_b200 import engine as E
    t, d, f, pad, shift = shape
    rng = np.random.default_rng(t)
    dt = torch.bfloat16
    o = ffn_case(rng, *shape, dt)
    dy, g, u, h = (randn(rng, t, n, dtype=dt, pad=pad, shift=shift) for n in (d, f, f, f))
    sizes = dict(dw_gate=(f, d), dw_up=(f, d), dw_down=(d, f))

    def run(earlier, in_place=()):
        out = {}
        for n, (a, b) in sizes.items():
            v, ok = room(a, b, grad, pad, shift)
            if n in in_place:
                v.copy_(earlier[n])
                earlier = {**earlier, n: v}
            out[n] = v, ok
        E.distsim_gated_ffn_backward(ctx, dy, **o, hidden=h, gate=g, up=u, **{n: q[0] for n, q in out.items()}, activation="silu",
                                     **{n + "_in": v for n, v in earlier.items()})
        for _, ok in out.values():
            ok()
        return {n: q[0] for n, q in out.items()}
    old = {n: randn(rng, a, b, dtype=grad, scale=t ** 0.5, pad=pad, shift=shift) for n, (a, b) in sizes.items()}
    plain = run({})
    whole = run(old)
    dh = dy.double() @ o["w_down"].double()
    dh_off = (d + 2) * U32 * dy.double().abs() @ o["w_down"].double().abs()
    val, slope = act64(g.double(), "silu")
    approx, x = 2.0 ** -19 * g.double().abs().clamp_min(1), o["x"].double()
    for name, q, off in (("dw_gate", dh * u.double() * slope, u.double().abs() * (dh_off * slope.abs() + (dh.abs() + dh_off) * approx)),
                         ("dw_up", dh * val, dh_off * val.abs() + (dh.abs() + dh_off) * approx)):
        off = off + unit(dt) * (q.abs() + off)
        close(name, whole[name], q.T @ x + old[name].double(), (t + 2) * U32 * (q.abs().T @ x.abs() + old[name].double().abs()) + off.T @ x.abs())
    close("dw_down", whole["dw_down"], dy.double().T @ h.double() + old["dw_down"].double(),
          (t + 2) * U32 * (dy.double().abs().T @ h.double().abs() + old["dw_down"].double().abs()))
    # in place, and with some of them only
    for names, in_place in ((sizes, sizes), (("dw_gate",), ()), (("dw_up", "dw_down"), ("dw_up",)), (("dw_gate", "dw_up"), ())):
        for n, v in run({k: old[k] for k in names}, in_place).items():
            if plan == 0 and n not in names:         # the choice of kernel goes by what a call reads
                continue
            assert torch.equal(v, (whole if n in names else plain)[n]) or plan == 0, (names, n)
    none = torch.empty(0, d, dtype=dt, device="cuda"), torch.empty(0, f, dtype=dt, device="cuda")
    out = {n: torch.full(s, 7.0, dtype=grad, device="cuda") for n, s in sizes.items()}
    E.distsim_gated_ffn_backward(ctx, none[0], none[0], o["w_gate"], o["w_up"], o["w_down"], none[1], none[1], none[1], **out,
                                 dw_gate_in=old["dw_gate"], dw_down_in=out["dw_down"])
    assert torch.equal(out["dw_gate"], old["dw_gate"]) and not out["dw_up"].any() and bool((out["dw_down"] == 7.0).all())


# ---------------------------------------------------------------- rows of equal values

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cols,shift", [(1, 0), (2, 1), (3, 0), (100, 0), (256, 0), (768, 0), (1000, 0), (2047, 0), (2048, 0), (4104, 0), (5000, 1), (12288, 0),
                                        (16384, 0), (16381, 0)])
def test_layer_norm_of_equal_values_is_its_bias(ctx, dtype, cols, shift):
    # values of 8 digits: their sums are exact in the 24 of 32 bits (at most 2^14 of them), so their distance from the mean is zero, and so is all that follows
    from paper_2306_08423_b200 import engine as E
    rng = np.random.default_rng(cols)
    value = torch.tensor([3.0, -0.6875, 100.0, 1.0, 0.01, -29.0, 0.0], device="cuda").bfloat16().to(dtype)
    x = randn(rng, 7, cols, dtype=dtype, shift=shift)
    x.copy_(value[:, None].expand(7, cols))
    w, b, w2, b2 = (randn(rng, cols, dtype=dtype) for _ in range(4))
    h, y = (torch.full((7, cols), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    E.distsim_residual_norm_forward(ctx, x, h=h, y=y, post_weight=w, post_bias=b, weight=w2, bias=b2)
    assert torch.equal(h, b.expand(7, cols))
    E.distsim_residual_norm_forward(ctx, x, y=y, weight=w2, bias=b2)
    assert torch.equal(y, b2.expand(7, cols))
    dy, dx, dw, dw2 = randn(rng, 7, cols, dtype=dtype), torch.empty_like(h), torch.ones_like(w), torch.ones_like(w)
    E.distsim_residual_norm_backward(ctx, x, x, dy=dy, dx=dx, dweight=dw2, dpost_weight=dw, weight=w2, post_weight=w)
    assert not dw.any() and not dw2.any()
    if cols == 1:
        assert not dx.any()


# ---------------------------------------------------------------- waits that give up

@pytest.fixture
def impatient():
    """A context of its own, and what makes the operators' waits give up at once while it runs."""
    from paper_2306_08423_b200 import engine as E
    c = E.Context(0)

    def gives_up(call):
        E.distsim_testing_set_operator_wait_polls(c, 0)
        call()
        with pytest.raises(E.DistsimError) as e:
            E.distsim_operator_status(c)
        assert e.value.code == E.E_TIMEOUT
        E.distsim_testing_set_operator_wait_polls(c, 1 << 22)
        E.distsim_operator_status(c)                 # reported once
    yield c, gives_up
    E.distsim_testing_set_product_plan(c, 0)
    E.distsim_operator_status(c)
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("plan_of", [-1, 1, 4, -2, -4])
@pytest.mark.parametrize("d", [64, 648])             # fewer steps than a ring has stages, and more
def test_products_that_give_up(impatient, plan_of, d):
    """Every wait of the product kernels gives up at once: the kernels end, say so, and leave nothing behind that the next
    call would meet."""
    from paper_2306_08423_b200 import engine as E
    c, gives_up = impatient
    E.distsim_testing_set_product_plan(c, plan_of)
    t, f = 60, 520
    rng = np.random.default_rng(d)
    dt = torch.bfloat16
    x, w, b, r = linear_case(rng, t, d, f, 0, 0, dt)
    y, z = torch.empty(t, f, dtype=dt, device="cuda"), torch.empty(t, f, dtype=dt, device="cuda")
    o = ffn_case(rng, t, d, f, 0, 0, dt)
    g, u = torch.empty_like(y), torch.empty_like(y)
    yd, dx, dw = torch.empty(t, d, dtype=dt, device="cuda"), torch.empty(t, d, dtype=dt, device="cuda"), torch.empty(f, d, device="cuda")
    many = randn(rng, 1100, d, dtype=dt), randn(rng, 1100, f, dtype=dt)
    calls = [(lambda: E.distsim_linear_forward(c, x, w, y, bias=b, residual=r, preact=z, activation="gelu"), (y, z)),
             (lambda: E.distsim_gated_ffn_forward(c, **o, y=yd, hidden=y, gate=g, up=u), (yd, y, g, u)),
             (lambda: E.distsim_gated_ffn_backward(c, yd, **o, hidden=None, gate=r, up=z, dx=dx), (dx,))]
    if plan_of > -2:                                 # in pieces
        calls.append((lambda: E.distsim_linear_backward(c, many[1], many[0], w, dweight=dw, dweight_in=dw), (dw,)))
    for call, out in calls:
        for v in out:
            v.fill_(1.0)
        call()
        first = [v.clone() for v in out]
        gives_up(call)
        for v in out:
            v.fill_(1.0)
        call()
        E.distsim_operator_status(c)
        assert all(torch.equal(a, v) for a, v in zip(first, out))


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(9, 256, 0, 0), (700, 768, 0, 0), (33, 1000, 1, 3), (5, 2047, 0, 1), (7, 5000, 0, 0), (40, 12288, 0, 0), (3, 16381, 0, 1)])
@pytest.mark.parametrize("parts", [(1, 1, 1, 1, 1, 0.1), (0, 0, 0, 1, 0, 0.0)])
def test_norms_that_give_up(impatient, shape, parts):
    from paper_2306_08423_b200 import engine as E
    c, gives_up = impatient
    t, n, pad, shift = shape
    post, pre = parts[:2]
    dt = torch.bfloat16
    rng = np.random.default_rng(n)
    x, r, o, bias = norm_case(rng, shape, parts, dt)
    h, dy, dh = (randn(rng, t, n, dtype=dt, pad=pad, shift=shift) for _ in range(3))
    out = [torch.empty(t, n, dtype=dt, device="cuda") for _ in range(4)]
    names = [k for k, v in (("dgate", parts[2]), ("dpost_weight", post), ("dpost_bias", post), ("dweight", pre), ("dbias", pre)) if v]
    grads = {k: torch.empty(n, dtype=dt, device="cuda") for k in names}
    kw = dict(kind="layer", alpha=0.75, p=parts[5], seed=5, offset=9)
    calls = [(lambda: E.distsim_residual_norm_forward(c, x, residual=r, h=out[0], y=out[1] if pre else None, bias=bias, **o, **kw), out[:1 + pre]),
             (lambda: E.distsim_residual_norm_backward(c, x, h if pre else None, dy=dy if pre else None, dh=dh, dx=out[2], dresidual=out[3],
                                                       **grads, **o, **kw), out[2:] + list(grads.values()))]
    for call, got in calls:
        call()
        first = [v.clone() for v in got]
        gives_up(call)
        for v in got:
            v.fill_(7.0)
        call()
        E.distsim_operator_status(c)
        assert all(torch.equal(a, v) for a, v in zip(first, got))


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [False, True])
def test_a_layer_refuses_its_own_buffers(ctx, gated):
    # they would be overwritten while the pass reads them, or before the backward pass does
    from paper_2306_08423_b200.layers import FeedForward
    one, two = (FeedForward(ctx, 40, 64, 128, gated=gated, seed=k) for k in range(2))
    y, h = (torch.randn(40, 64, device="cuda").bfloat16() for _ in range(2))
    out = one.forward(y, h)
    with pytest.raises(ValueError, match="own buffers"):
        one.forward(out[0], h)
    with pytest.raises(ValueError, match="own buffers"):
        one.forward(y, out[1])
    two.forward(*out)
    grads = two.backward(y, h)
    with pytest.raises(ValueError, match="own buffers"):
        two.backward(grads[0], h)
    with pytest.raises(ValueError, match="own buffers"):
        two.backward(y, grads[1])
    one.backward(*grads)
