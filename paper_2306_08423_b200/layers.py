"""The feed-forward half of a transformer layer from the layer operators, and its computation events.

DistSim's event profiler times every distinct computation event once on a device (paper Sec. 4.2);
its events are a layer's forward and backward at the shapes that a strategy presents, keyed by the
model-parallel degree and the micro-batch size (Sec. 4.1).  :class:`FeedForward` is such a layer's
shard on one device; :func:`measure_events` times it for every class of a search space, and
:func:`measured_table` lays the times out as an event table that the engine searches.

Attention is not among the operators: a table of whole layers adds its times through ``extra_ns``.
"""
from __future__ import annotations

from . import workloads as W


class FeedForward:
    """One device's shard of a feed-forward block and of the connection behind it, with its buffers.

    ``forward(y, h)`` takes the block's normalised input ``y`` and the residual stream ``h`` (both
    [tokens, hidden]) and returns the next block's pair:
        o = act(y W1^T + b1) W2^T          (or the gated block of W_gate, W_up, W_down)
        h' = h + dropout(o);  y' = layernorm(h') weight + bias
    ``backward(dy', dh')`` returns (dy, dh) and fills ``grads``.  What both return are the layer's own
    buffers, which its next pass overwrites: they are another layer's inputs, not its own.  With model-parallel degree mp the
    shard's hidden width is ``d_hidden / mp``; o is then a partial sum that the model-parallel
    all-reduce completes (an event of its own, not run here).
    """

    def __init__(self, ctx, tokens, hidden, d_hidden, gated=False, dtype=None, p=0.0, seed=0):
        import torch
        from . import engine
        self.engine, self.ctx = engine, ctx
        self.gated, self.p, self.seed, self.step = gated, p, seed, 0
        self.activation = "silu" if gated else "gelu"
        device, dtype = f"cuda:{ctx.device}", dtype or torch.bfloat16
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=gen, device=device) * cols ** -0.5).to(dtype)

        def room(*shape):
            return torch.empty(shape, device=device, dtype=dtype)
        if gated:
            self.params = dict(w_gate=weight(d_hidden, hidden), w_up=weight(d_hidden, hidden), w_down=weight(hidden, d_hidden))
        else:
            self.params = dict(w1=weight(d_hidden, hidden), b1=torch.zeros(d_hidden, device=device, dtype=dtype),
                               w2=weight(hidden, d_hidden))
        self.params.update(weight=torch.ones(hidden, device=device, dtype=dtype), bias=torch.zeros(hidden, device=device, dtype=dtype))
        self.grads = {k: torch.empty_like(v) for k, v in self.params.items()}
        self.inner = {k: room(tokens, d_hidden) for k in (("gate", "up", "hidden") if gated else ("preact", "act", "dact"))}
        self.outer = {k: room(tokens, hidden) for k in ("o", "h", "y", "do", "dh", "dy")}
        self.offset = 0
        self.draws = tokens * ((hidden + 1) // 2)

    def _not_own(self, **inputs):
        own = {v.data_ptr() for v in self.outer.values()}
        for name, v in inputs.items():
            if v.numel() and v.data_ptr() in own:
                raise ValueError(f"{name}: one of the layer's own buffers, which the pass overwrites; pass a copy")

    def forward(self, y, h, stream=None):
        self._not_own(y=y, h=h)
        e, p, i, o = self.engine, self.params, self.inner, self.outer
        self.offset = self.step * self.draws
        self.step += 1
        self.y = y
        if self.gated:
            e.distsim_gated_ffn_forward(self.ctx, y, p["w_gate"], p["w_up"], p["w_down"], o["o"], hidden=i["hidden"], gate=i["gate"],
                                        up=i["up"], activation=self.activation, stream=stream)
        else:
            e.distsim_linear_forward(self.ctx, y, p["w1"], i["act"], bias=p["b1"], preact=i["preact"], activation=self.activation,
                                     stream=stream)
            e.distsim_linear_forward(self.ctx, i["act"], p["w2"], o["o"], stream=stream)
        e.distsim_residual_norm_forward(self.ctx, o["o"], residual=h, h=o["h"], y=o["y"], weight=p["weight"], bias=p["bias"], p=self.p,
                                        seed=self.seed, offset=self.offset, stream=stream)
        return o["y"], o["h"]

    def backward(self, dy, dh, stream=None):
        self._not_own(dy=dy, dh=dh)
        e, p, g, i, o = self.engine, self.params, self.grads, self.inner, self.outer
        e.distsim_residual_norm_backward(self.ctx, None, o["h"], dy=dy, dh=dh, dx=o["do"], dresidual=o["dh"], dweight=g["weight"],
                                         dbias=g["bias"], weight=p["weight"], p=self.p, seed=self.seed, offset=self.offset, stream=stream)
        if self.gated:
            e.distsim_gated_ffn_backward(self.ctx, o["do"], self.y, p["w_gate"], p["w_up"], p["w_down"], i["hidden"], i["gate"], i["up"],
                                         dx=o["dy"], dw_gate=g["w_gate"], dw_up=g["w_up"], dw_down=g["w_down"],
                                         activation=self.activation, stream=stream)
        else:
            e.distsim_linear_backward(self.ctx, o["do"], i["act"], p["w2"], dx=i["dact"], dweight=g["w2"], stream=stream)
            e.distsim_linear_backward(self.ctx, i["dact"], self.y, p["w1"], dx=o["dy"], dweight=g["w1"], dbias=g["b1"],
                                      preact=i["preact"], activation=self.activation, stream=stream)
        return o["dy"], o["dh"]


def time_layer(ctx, tokens, hidden, d_hidden, gated=False, p=0.1, repeats=5):
    """(forward, backward) device time of a shard in ns: the median of ``repeats`` replays of each
    captured pass after three, with the L2 cache overwritten before it, by CUDA events."""
    import torch
    with torch.cuda.device(ctx.device):              # streams, captures and events are those of the current device
        return _time_layer(ctx, tokens, hidden, d_hidden, gated, p, repeats)


def _time_layer(ctx, tokens, hidden, d_hidden, gated, p, repeats):
    import torch
    layer = FeedForward(ctx, tokens, hidden, d_hidden, gated=gated, p=p)
    device = f"cuda:{ctx.device}"
    y, h, dy, dh = (torch.randn(tokens, hidden, device=device).to(torch.bfloat16) for _ in range(4))
    flush = torch.empty(64 << 20, dtype=torch.int32, device=device)
    passes = (lambda: layer.forward(y, h), lambda: layer.backward(dy, dh))
    for run in passes:                           # grows the context's scratch, which a capture cannot
        run()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in passes]
    for graph, run in zip(graphs, passes):
        with torch.cuda.graph(graph):
            run()
    times = []
    for k in range(3 + repeats):
        ev = [(torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)) for _ in graphs]
        for graph, (start, end) in zip(graphs, ev):
            flush.zero_()
            start.record()
            graph.replay()
            end.record()
        torch.cuda.synchronize()
        if k >= 3:
            times.append([start.elapsed_time(end) for start, end in ev])
    layer.engine.distsim_operator_status(ctx)
    return tuple(max(1, int(round(1e6 * sorted(t)[repeats // 2]))) for t in zip(*times))


def measure_events(ctx, classes, seq, hidden, d_hidden, gated=False, p=0.1, timer=time_layer):
    """{(mp, b): (forward ns, backward ns)} of a layer of ``d_hidden`` split over mp devices, b
    sequences a micro-batch, for every class; each distinct shape is timed once."""
    for mp, _ in classes:
        if d_hidden % mp:
            raise ValueError(f"d_hidden {d_hidden} is not divisible by the model-parallel degree {mp}")
    return {(mp, b): timer(ctx, b * seq, hidden, d_hidden // mp, gated, p) for mp, b in sorted(set(classes))}


def measured_table(ctx, *, space, n_layers, n_devices, gpus_per_node, global_batch, seq, hidden, d_hidden, expert_layers=(), p=0.1,
                   extra_ns=None, timer=time_layer, **cluster) -> "W.EventTable":
    """Event table of a model of feed-forward layers (gated ones at ``expert_layers``) timed on the
    context's device.  ``extra_ns(mp, b)`` gives (forward, backward) ns to add to every layer, for
    what the operators do not cover (attention); ``cluster`` are the table's link constants."""
    import numpy as np
    classes = W.event_classes(n_devices, global_batch, n_layers, space)
    expert = np.zeros(n_layers, dtype=np.uint8)
    expert[list(expert_layers)] = 1
    times = {kind: measure_events(ctx, classes, seq, hidden, d_hidden, bool(kind), p, timer) for kind in sorted(set(expert.tolist()))}
    fwd = np.zeros((len(classes), n_layers), dtype=np.int64)
    bwd = np.zeros((len(classes), n_layers), dtype=np.int64)
    for k, cls in enumerate(classes):
        add = extra_ns(*cls) if extra_ns else (0, 0)
        for layer, kind in enumerate(expert.tolist()):
            fwd[k, layer], bwd[k, layer] = (t + a for t, a in zip(times[kind][cls], add))
    matrices = np.where(expert == 1, 3, 2).astype(np.int64)
    return W.EventTable(n_layers=n_layers, n_devices=n_devices, gpus_per_node=gpus_per_node, global_batch=global_batch, seq=seq,
                        hidden=hidden, class_mp=[c[0] for c in classes], class_b=[c[1] for c in classes], fwd_ns=fwd, bwd_ns=bwd,
                        layer_is_expert=expert, grad_bytes=matrices * hidden * d_hidden * 2, **cluster)
