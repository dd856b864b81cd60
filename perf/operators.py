"""Cases that measure the operators of a transformer layer: the product with bias, activation and
residual, the gated feed-forward block, and the residual connection with its norms and dropout,
forward and backward.

Where ``own`` is false ``run`` computes an operator from elementary torch operations in 32 bits;
where it is true it calls the framework.  The sizes are those of the framework's workloads
(hidden 768, 1024, 2048 and 12288; sequences of 512, 1024 and 2048 tokens; the widths of a
model-parallel shard), single tokens, and ragged ones.
"""
import functools
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
GAMMA = 0x9E3779B97F4A7C15


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one token through the up projection of the 64-device workload's layer: latency
        dict(name="linear_fwd_one_token", op="linear_fwd", tokens=1, d_in=1024, d_out=4096, type="bf16",
             act="gelu", bias=True, residual=False, save=False, pad=0),
        # the same projection for a micro-batch of 8 sequences of 1024, as training calls it
        dict(name="linear_fwd_1024", op="linear_fwd", tokens=8192, d_in=1024, d_out=4096, type="bf16",
             act="gelu", bias=True, residual=False, save=True, pad=0),
        # the down projection of the 12288-wide layer split over 8 devices, 4 sequences of 2048: the largest
        dict(name="linear_fwd_12288", op="linear_fwd", tokens=8192, d_in=6144, d_out=12288, type="bf16",
             act="none", bias=True, residual=True, save=False, pad=0),
        # backward of the second case
        dict(name="linear_bwd_1024", op="linear_bwd", tokens=8192, d_in=1024, d_out=4096, type="bf16",
             act="gelu", bias=True, pad=0),
        # a short, ragged batch and a width that no 16-byte row stride fits
        dict(name="linear_bwd_ragged", op="linear_bwd", tokens=1537, d_in=768, d_out=2311, type="f16",
             act="relu", bias=True, pad=8),
        # a few tokens through the expert of the MoE-like workload: bound by its weights
        dict(name="ffn_fwd_few_tokens", op="ffn_fwd", tokens=7, d_in=2048, d_hidden=8192, type="bf16",
             act="silu", bias=False, residual=True, save=False, pad=0),
        # a training step's forward of that expert, 8 sequences of 1024
        dict(name="ffn_fwd_2048", op="ffn_fwd", tokens=8192, d_in=2048, d_hidden=8192, type="bf16",
             act="silu", bias=False, residual=True, save=True, pad=0),
        # and its backward on half of that
        dict(name="ffn_bwd_2048", op="ffn_bwd", tokens=4096, d_in=2048, d_hidden=8192, type="bf16",
             act="silu", bias=False, pad=0),
        # the smallest workload's width, ragged tokens and hidden width, biases everywhere
        dict(name="ffn_bwd_ragged", op="ffn_bwd", tokens=517, d_in=768, d_hidden=2049, type="f16",
             act="gelu_tanh", bias=True, pad=0),
        # one sequence of the smallest workload in 32 bits: residual and the norm before the next block
        dict(name="norm_fwd_768", op="norm_fwd", tokens=512, d_in=768, type="f32", kind="layer", post=False,
             pre=True, gate=False, residual=True, alpha=1.0, p=0.0, pad=0),
        # norms after and before a block with gate, residual scale and dropout
        dict(name="norm_fwd_2048", op="norm_fwd", tokens=32768, d_in=2048, type="bf16", kind="rms", post=True,
             pre=True, gate=True, residual=True, alpha=0.75, p=0.1, pad=0),
        # backward at the widest layer, with every parameter's gradient
        dict(name="norm_bwd_12288", op="norm_bwd", tokens=8192, d_in=12288, type="bf16", kind="layer", post=True,
             pre=True, gate=True, residual=True, alpha=1.0, p=0.1, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    most = max(w["bytes"] + w["flops"] / 50 for w in map(work, listed()))
    while True:
        op = rng.choice(("linear_fwd", "linear_bwd", "ffn_fwd", "ffn_bwd", "norm_fwd", "norm_bwd"))
        case = dict(op=op, tokens=_log(rng, 1, 32768), d_in=_width(rng, 48, 12288),
                    type=rng.choice(("bf16", "bf16", "f16")), pad=rng.choice((0, 0, 8, 3)))
        if op.startswith("linear"):
            case.update(d_out=_width(rng, 48, 16384), act=rng.choice(ACTIVATIONS), bias=rng.random() < 0.7)
        elif op.startswith("ffn"):
            case.update(d_hidden=_width(rng, 48, 16384), act=rng.choice(("silu", "gelu", "gelu_tanh")),
                        bias=rng.random() < 0.3)
        else:
            post = rng.random() < 0.5
            case.update(type=rng.choice(("bf16", "f16", "f32")), kind=rng.choice(("layer", "rms")), post=post,
                        pre=not post or rng.random() < 0.7, gate=rng.random() < 0.5, residual=rng.random() < 0.8,
                        alpha=rng.choice((1.0, 0.75)), p=rng.choice((0.0, 0.1, 0.25)))
        if op in ("linear_fwd", "ffn_fwd"):
            case.update(residual=rng.random() < 0.5, save=rng.random() < 0.5)
        w = work(case)
        if w["bytes"] + w["flops"] / 50 <= most:
            return case


def work(case):
    c, t, d = case, case["tokens"], case["d_in"]
    e = TYPES[c["type"]].itemsize
    if c["op"] == "linear_fwd":
        f = c["d_out"]
        n = t * d + f * d + f * c["bias"] + t * f * (1 + c["residual"] + c["save"])
        return {"bytes": e * n, "flops": 2 * t * d * f}
    if c["op"] == "linear_bwd":
        f = c["d_out"]
        n = t * f * (1 + (c["act"] != "none")) + 2 * t * d + 2 * f * d + f * c["bias"]
        return {"bytes": e * n, "flops": 4 * t * d * f}
    if c["op"] == "ffn_fwd":
        f = c["d_hidden"]
        n = t * d * (2 + c["residual"]) + 3 * f * d + (2 * f + d) * c["bias"] + 3 * t * f * c["save"]
        return {"bytes": e * n, "flops": 6 * t * d * f}
    if c["op"] == "ffn_bwd":
        f = c["d_hidden"]
        n = 3 * t * d + 3 * t * f + 6 * f * d + (2 * f + d) * c["bias"]
        return {"bytes": e * n, "flops": 12 * t * d * f}
    vectors = d * (c["gate"] + 2 * c["post"] + 2 * c["pre"])
    if c["op"] == "norm_fwd":
        n = t * d * (2 + c["residual"] + c["pre"]) + vectors
        return {"bytes": e * n, "flops": 20 * t * d}
    reads_x = c["post"] or c["gate"]
    n = t * d * (1 + 2 * c["pre"] + reads_x + 1 + c["residual"]) + 2 * vectors
    return {"bytes": e * n, "flops": 40 * t * d}


# ---------------------------------------------------------------- inputs

def _normal(gen, rows, cols, dtype, scale=1.0, pad=0):
    """Normal values, rows of which lie `pad` elements further apart than they are long."""
    v = torch.randn(rows, cols + pad, generator=gen, device="cuda", dtype=torch.float32)
    return v.mul_(scale).to(dtype)[:, :cols]


def _vector(gen, n, dtype, mean=0.0, scale=0.1):
    return (torch.randn(n, generator=gen, device="cuda") * scale + mean).to(dtype)


def prepare(case, seed):
    c, t, d = case, case["tokens"], case["d_in"]
    ty = TYPES[c["type"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    empty = functools.partial(torch.empty, device="cuda", dtype=ty)
    s = dict(case=dict(c), x=_normal(gen, t, d, ty, pad=c["pad"]))
    if c["op"].startswith("linear"):
        f = c["d_out"]
        s["weight"] = _normal(gen, f, d, ty, d ** -0.5)
        s["bias"] = _vector(gen, f, ty) if c["bias"] else None
        if c["op"] == "linear_fwd":
            s["residual"] = _normal(gen, t, f, ty, pad=c["pad"]) if c["residual"] else None
            s.update(y=empty(t, f), preact=empty(t, f) if c["save"] else None)
        else:
            s["dy"] = _normal(gen, t, f, ty, 0.5, pad=c["pad"])
            s["preact"] = _normal(gen, t, f, ty) if c["act"] != "none" else None
            s.update(dx=empty(t, d), dweight=empty(f, d), dbias=empty(f) if c["bias"] else None)
    elif c["op"].startswith("ffn"):
        f = c["d_hidden"]
        for name in ("w_gate", "w_up"):
            s[name] = _normal(gen, f, d, ty, d ** -0.5)
        s["w_down"] = _normal(gen, d, f, ty, f ** -0.5)
        for name, n in (("b_gate", f), ("b_up", f), ("b_down", d)):
            s[name] = _vector(gen, n, ty) if c["bias"] else None
        if c["op"] == "ffn_fwd":
            s["residual"] = _normal(gen, t, d, ty, pad=c["pad"]) if c["residual"] else None
            s["y"] = empty(t, d)
            for name in ("hidden", "gate", "up"):
                s[name] = empty(t, f) if c["save"] else None
        else:
            s["dy"] = _normal(gen, t, d, ty, 0.5, pad=c["pad"])
            s["gate"], s["up"] = _normal(gen, t, f, ty), _normal(gen, t, f, ty)
            s["hidden"] = (_act(s["gate"].float(), c["act"]) * s["up"].float()).to(ty)
            s["dx"] = empty(t, d)
            for name in ("w_gate", "w_up", "w_down"):
                s["d" + name] = torch.empty_like(s[name])
            for name in ("b_gate", "b_up", "b_down"):
                s["d" + name] = torch.empty_like(s[name]) if c["bias"] else None
    else:
        s["residual"] = _normal(gen, t, d, ty, pad=c["pad"]) if c["residual"] else None
        s["gate"] = _vector(gen, d, ty, 0.5) if c["gate"] else None
        for name, used in (("post", c["post"]), ("pre", c["pre"])):
            s[name + "_weight"] = _vector(gen, d, ty, 1.0) if used else None
            s[name + "_bias"] = _vector(gen, d, ty) if used else None
        s["seed"] = int(torch.randint(0, 2 ** 62, (1,), generator=gen, device="cuda"))
        s["offset"] = int(torch.randint(0, 2 ** 40, (1,), generator=gen, device="cuda"))
        s["h"] = empty(t, d)
        if c["op"] == "norm_fwd":
            s["y"] = empty(t, d) if c["pre"] else None
        else:
            s["h"] = _normal(gen, t, d, ty) if c["pre"] else None
            s["dh"] = _normal(gen, t, d, ty, 0.5)
            s["dy"] = _normal(gen, t, d, ty, 0.5, pad=c["pad"]) if c["pre"] else None
            s["dx"] = empty(t, d)
            s["dresidual"] = empty(t, d) if c["residual"] else None
            for name in ("gate", "post_weight", "post_bias", "pre_weight", "pre_bias"):
                s["d" + name] = torch.empty_like(s[name]) if s[name] is not None else None
    return s


# ---------------------------------------------------------------- plain forms, in 32 bits

def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        th = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        sg = torch.sigmoid(z)
        return sg * (1 + z * (1 - sg))
    return torch.ones_like(z)


def _signed(v):
    return v - (1 << 64) if v >> 63 else v


def _shift(v, n):
    """Logical right shift of int64."""
    return (v >> n) & ((1 << (64 - n)) - 1)


def _kept(rows, cols, p, seed, offset):
    """What dropout keeps: draw number row * ceil(cols / 2) + col / 2 (+ offset) of SplitMix64 started
    at `seed` decides two neighbouring columns, the even one by its low 32 bits."""
    half = (cols + 1) // 2
    z = torch.arange(1, rows * half + 1, device="cuda", dtype=torch.int64)
    z = (z + _signed(offset)) * _signed(GAMMA) + _signed(seed)
    z = (z ^ _shift(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ _shift(z, 27)) * _signed(0x94D049BB133111EB)
    z = z ^ _shift(z, 31)
    bits = torch.stack((z & 0xFFFFFFFF, _shift(z, 32)), 1).reshape(rows, 2 * half)[:, :cols]
    return bits >= _threshold(p)


def _threshold(p):
    return int(round(p * 2.0 ** 32))


def _statistics(v, kind, eps=1e-5):
    mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    centred = v - mean
    rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + eps)
    return centred * rstd, rstd


def _norm_back(dout, v, weight, kind):
    """Gradients of norm(v) * weight + bias by v, weight and bias."""
    hat, rstd = _statistics(v, kind)
    dhat = dout * weight
    inner = dhat - hat * (dhat * hat).mean(1, keepdim=True)
    if kind == "layer":
        inner = inner - dhat.mean(1, keepdim=True)
    return inner * rstd, (dout * hat).sum(0), dout.sum(0)


def _plain(s, wide):
    """The operators' formulas; every floating input passes `wide` first."""
    c = s["case"]
    v = {k: wide(x) if isinstance(x, torch.Tensor) and x.is_floating_point() else x for k, x in s.items()}
    if c["op"] == "linear_fwd":
        z = v["x"] @ v["weight"].T
        if v["bias"] is not None:
            z = z + v["bias"]
        y = _act(z, c["act"])
        y = y if v["residual"] is None else y + v["residual"]
        return [y, z if c["save"] else None]
    if c["op"] == "linear_bwd":
        dz = v["dy"] if c["act"] == "none" else v["dy"] * _act_grad(v["preact"], c["act"])
        return [dz @ v["weight"], dz.T @ v["x"], dz.sum(0) if c["bias"] else None]
    if c["op"] == "ffn_fwd":
        g, u = v["x"] @ v["w_gate"].T, v["x"] @ v["w_up"].T
        if c["bias"]:
            g, u = g + v["b_gate"], u + v["b_up"]
        h = _act(g, c["act"]) * u
        y = h @ v["w_down"].T
        y = y + v["b_down"] if c["bias"] else y
        y = y if v["residual"] is None else y + v["residual"]
        return [y, h, g, u] if c["save"] else [y, None, None, None]
    if c["op"] == "ffn_bwd":
        dh = v["dy"] @ v["w_down"]
        dg, du = dh * v["up"] * _act_grad(v["gate"], c["act"]), dh * _act(v["gate"], c["act"])
        grads = [dg @ v["w_gate"] + du @ v["w_up"], dg.T @ v["x"], du.T @ v["x"], v["dy"].T @ v["hidden"]]
        return grads + ([dg.sum(0), du.sum(0), v["dy"].sum(0)] if c["bias"] else [None] * 3)
    rows, cols = c["tokens"], c["d_in"]
    kept = _kept(rows, cols, c["p"], s["seed"], s["offset"]) if c["p"] else None
    scale = 1.0 / (1.0 - _threshold(c["p"]) / 2.0 ** 32)
    t = v["x"]
    if c["post"]:
        t = _statistics(t, c["kind"])[0] * v["post_weight"] + v["post_bias"]
    t = t if kept is None else torch.where(kept, t * scale, 0.0)
    if c["op"] == "norm_fwd":
        h = t * v["gate"] if c["gate"] else t
        h = h + c["alpha"] * v["residual"] if c["residual"] else h
        y = _statistics(h, c["kind"])[0] * v["pre_weight"] + v["pre_bias"] if c["pre"] else None
        return [h, y]
    dh, dpre = v["dh"], [None, None]
    if c["pre"]:
        back, *dpre = _norm_back(v["dy"], v["h"], v["pre_weight"], c["kind"])
        dh = dh + back
    dgate = (dh * t).sum(0) if c["gate"] else None
    dt = dh * v["gate"] if c["gate"] else dh
    dt = dt if kept is None else torch.where(kept, dt * scale, 0.0)
    dpost = [None, None]
    if c["post"]:
        dt, *dpost = _norm_back(dt, v["x"], v["post_weight"], c["kind"])
    return [dt, dh * c["alpha"] if c["residual"] else None, dgate, *dpost, *dpre]


# ---------------------------------------------------------------- one pass

@functools.cache
def _context():
    from paper_2306_08423_b200 import engine
    return engine, engine.Context(0)


def _framework(s):
    engine, ctx = _context()
    c = s["case"]
    if c["op"] == "linear_fwd":
        engine.distsim_linear_forward(ctx, s["x"], s["weight"], s["y"], bias=s["bias"], residual=s["residual"],
                                      preact=s["preact"], activation=c["act"])
        return [s["y"], s["preact"]]
    if c["op"] == "linear_bwd":
        engine.distsim_linear_backward(ctx, s["dy"], s["x"], s["weight"], dx=s["dx"], dweight=s["dweight"],
                                       dbias=s["dbias"], preact=s["preact"], activation=c["act"])
        return [s["dx"], s["dweight"], s["dbias"]]
    if c["op"] == "ffn_fwd":
        engine.distsim_gated_ffn_forward(ctx, s["x"], s["w_gate"], s["w_up"], s["w_down"], s["y"],
                                         b_gate=s["b_gate"], b_up=s["b_up"], b_down=s["b_down"],
                                         residual=s["residual"], hidden=s["hidden"], gate=s["gate"], up=s["up"],
                                         activation=c["act"])
        return [s["y"], s["hidden"], s["gate"], s["up"]]
    if c["op"] == "ffn_bwd":
        engine.distsim_gated_ffn_backward(ctx, s["dy"], s["x"], s["w_gate"], s["w_up"], s["w_down"], s["hidden"],
                                          s["gate"], s["up"], dx=s["dx"], dw_gate=s["dw_gate"], dw_up=s["dw_up"],
                                          dw_down=s["dw_down"], db_gate=s["db_gate"], db_up=s["db_up"],
                                          db_down=s["db_down"], activation=c["act"])
        return [s[k] for k in ("dx", "dw_gate", "dw_up", "dw_down", "db_gate", "db_up", "db_down")]
    shared = dict(post_weight=s["post_weight"], post_bias=s["post_bias"], gate=s["gate"], weight=s["pre_weight"],
                  kind=c["kind"], alpha=c["alpha"], p=c["p"], seed=s["seed"], offset=s["offset"])
    if c["op"] == "norm_fwd":
        engine.distsim_residual_norm_forward(ctx, s["x"], residual=s["residual"], bias=s["pre_bias"], h=s["h"],
                                             y=s["y"], **shared)
        return [s["h"], s["y"]]
    engine.distsim_residual_norm_backward(ctx, s["x"], s["h"], dy=s["dy"], dh=s["dh"], dx=s["dx"],
                                          dresidual=s["dresidual"], dgate=s["dgate"],
                                          dpost_weight=s["dpost_weight"], dpost_bias=s["dpost_bias"],
                                          dweight=s["dpre_weight"], dbias=s["dpre_bias"], **shared)
    return [s[k] for k in ("dx", "dresidual", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")]


def run(state):
    if own:
        return _framework(state)
    ty = TYPES[state["case"]["type"]]
    return [None if v is None else v.to(ty) for v in _plain(state, torch.Tensor.float)]


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _exact_act(z, act):
    """act(z) and its derivative, from the distribution functions."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), torch.where(z > 0, 1.0, 0.0).to(z)
    if act == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z.square() / 2) / (2 * math.pi) ** 0.5
    # silu, and the tanh form of gelu: z times the logistic function of some inner(z)
    if act == "silu":
        inner, slope = z, torch.ones_like(z)
    else:
        k = (8 / math.pi) ** 0.5
        inner, slope = k * z * (1 + 0.044715 * z.square()), k * (1 + 0.134145 * z.square())
    up, down = 1 / (1 + torch.exp(-inner)), 1 / (1 + torch.exp(inner))
    return z * up, up + z * up * down * slope


def _exact_norm(v, weight, bias, kind, dout=None):
    """The norm's value, or with `dout` its gradients, row statistics by torch.var in 64 bits."""
    n = v.shape[1]
    if kind == "layer":
        var, mean = torch.var_mean(v, 1, correction=0, keepdim=True)
    else:
        var, mean = v.square().sum(1, keepdim=True) / n, torch.zeros_like(v[:, :1])
    sd = (var + 1e-5).sqrt()
    hat = (v - mean) / sd
    if dout is None:
        return hat * weight + bias
    a = dout * weight
    first = a.sum(1, keepdim=True) / n if kind == "layer" else 0.0
    second = torch.einsum("ij,ij->i", a, hat)[:, None] / n
    return (a - first - hat * second) / sd, torch.einsum("ij,ij->j", dout, hat), dout.sum(0)


def _exact_keep(rows, cols, p, seed, offset):
    """Dropout's keep flags by numpy's wrapping unsigned arithmetic."""
    import numpy as np
    half = (cols + 1) // 2
    with np.errstate(over="ignore"):
        n = np.arange(rows * half, dtype=np.uint64) + np.uint64((offset + 1) % 2 ** 64)
        state = np.uint64(seed % 2 ** 64) + n * np.uint64(GAMMA)
        state = (state ^ (state >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        state = (state ^ (state >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        state ^= state >> np.uint64(31)
    words = state.astype("<u8").view("<u4").reshape(rows, 2 * half)[:, :cols]
    return torch.from_numpy(words >= np.uint32(round(p * 2 ** 32))).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    w = {k: x.double() if isinstance(x, torch.Tensor) and x.is_floating_point() else x for k, x in s.items()}

    def affine(x, weight, bias):
        out = torch.einsum("td,fd->tf", x, weight)
        return out if bias is None else out.add_(bias)

    if c["op"] == "linear_fwd":
        z = affine(w["x"], w["weight"], w["bias"])
        y = _exact_act(z, c["act"])[0]
        return [y + w["residual"] if c["residual"] else y, z if c["save"] else None]
    if c["op"] == "linear_bwd":
        dz = w["dy"] * _exact_act(w["preact"], c["act"])[1] if c["act"] != "none" else w["dy"]
        return [torch.einsum("tf,fd->td", dz, w["weight"]), torch.einsum("tf,td->fd", dz, w["x"]),
                torch.einsum("tf->f", dz) if c["bias"] else None]
    if c["op"] == "ffn_fwd":
        g, u = affine(w["x"], w["w_gate"], w["b_gate"]), affine(w["x"], w["w_up"], w["b_up"])
        h = _exact_act(g, c["act"])[0] * u
        y = affine(h, w["w_down"], w["b_down"])
        y = y + w["residual"] if c["residual"] else y
        return [y, h, g, u] if c["save"] else [y, None, None, None]
    if c["op"] == "ffn_bwd":
        value, slope = _exact_act(w["gate"], c["act"])
        dh = torch.einsum("td,df->tf", w["dy"], w["w_down"])
        dg, du = dh * w["up"] * slope, dh * value
        out = [torch.einsum("tf,fd->td", dg, w["w_gate"]) + torch.einsum("tf,fd->td", du, w["w_up"]),
               torch.einsum("tf,td->fd", dg, w["x"]), torch.einsum("tf,td->fd", du, w["x"]),
               torch.einsum("td,tf->df", w["dy"], w["hidden"])]
        return out + ([torch.einsum("tf->f", q) for q in (dg, du, w["dy"])] if c["bias"] else [None] * 3)
    factor = torch.ones((), dtype=torch.float64, device="cuda")
    if c["p"]:
        keep = _exact_keep(c["tokens"], c["d_in"], c["p"], s["seed"], s["offset"])
        factor = keep.double() / (1 - round(c["p"] * 2 ** 32) / 2 ** 32)
    block = _exact_norm(w["x"], w["post_weight"], w["post_bias"], c["kind"]) if c["post"] else w["x"]
    gate = w["gate"] if c["gate"] else 1.0
    if c["op"] == "norm_fwd":
        h = block * factor * gate
        if c["residual"]:
            h = h + c["alpha"] * w["residual"]
        return [h, _exact_norm(h, w["pre_weight"], w["pre_bias"], c["kind"]) if c["pre"] else None]
    total, dpre = w["dh"], (None, None)
    if c["pre"]:
        back, *dpre = _exact_norm(w["h"], w["pre_weight"], None, c["kind"], w["dy"])
        total = total + back
    dgate = torch.einsum("ij,ij->j", total, block * factor) if c["gate"] else None
    dx, dpost = total * gate * factor, (None, None)
    if c["post"]:
        dx, *dpost = _exact_norm(w["x"], w["post_weight"], None, c["kind"], dx)
    return [dx, c["alpha"] * total if c["residual"] else None, dgate, *dpost, *dpre]
