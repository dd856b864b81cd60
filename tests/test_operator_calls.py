"""The host side of an operator call - scratch, order between streams, captures, devices - on a CUDA
runtime without a device (fake_cuda_runtime.cpp): no GPU needed."""
import ctypes as C
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
E_ARG, E_STATE, E_CUDA = -1, -2, -6


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    """The library on the fake runtime."""
    return load(build(tmp_path_factory))


def build(tmp_path_factory):
    from paper_2306_08423_b200 import build as B
    B.build()
    so = str(tmp_path_factory.mktemp("fake") / "libdistsim_fake.so")
    objects = [os.path.join(B._OBJ, s.replace(".cu", ".o")) for s in B.SOURCES]
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-I/usr/local/cuda/include", "-o", so,
                    os.path.join(HERE, "fake_cuda_runtime.cpp"), *objects], check=True, capture_output=True, text=True)
    return so


def load(so):
    from paper_2306_08423_b200 import operators as O
    f = C.CDLL(so)
    f.path = so
    f.distsim_create.argtypes = [C.POINTER(C.c_void_p), C.c_int]
    f.distsim_destroy.argtypes = [C.c_void_p]
    f.distsim_last_error.argtypes = [C.c_void_p]
    f.distsim_last_error.restype = C.c_char_p
    f.distsim_operator_status.argtypes = [C.c_void_p, C.c_void_p]
    f.distsim_testing_set_product_plan.argtypes = [C.c_void_p, C.c_int32]
    for name, struct in (("linear", O._Linear), ("gated_ffn", O._GatedFfn), ("residual_norm", O._ResidualNorm)):
        for way in ("forward", "backward"):
            getattr(f, f"distsim_{name}_{way}").argtypes = [C.c_void_p, C.c_void_p, C.POINTER(struct)]
    f.fake_log.restype = C.c_char_p
    f.fake_stream.argtypes = [C.c_void_p, C.c_ulonglong, C.c_int]
    return f


class Context:
    def __init__(self, lib, device=0):
        self.lib, self.h = lib, C.c_void_p()
        assert lib.distsim_create(C.byref(self.h), device) == 0

    def close(self):
        self.lib.distsim_destroy(self.h)

    def backward(self, tokens, stream, d_in=64, d_out=128, rc=0):
        """A linear backward pass, which needs scratch that grows with the tokens."""
        from paper_2306_08423_b200 import operators as O
        o = O._Linear(tokens=tokens, d_in=d_in, d_out=d_out, activation=O.ACTIVATIONS["gelu"])
        for k, name in enumerate(("x", "weight", "preact", "dy", "dx", "dweight", "dbias")):
            setattr(o, name, (0x7000 + k) << 32)
            if name != "dbias":
                setattr(o, "ld_" + name, d_out if name in ("preact", "dy") else d_in)
        assert self.lib.distsim_linear_backward(self.h, stream, C.byref(o)) == rc, self.error()

    def error(self):
        return self.lib.distsim_last_error(self.h).decode()


@pytest.fixture
def ctx(lib):
    c = Context(lib)
    for handle in (0x10, 0x20, 0x30):
        lib.fake_stream(handle, handle, 0)
    log(lib)
    yield c
    c.close()
    log(lib)


def log(lib):
    return lib.fake_log().decode().splitlines()


def of(events, word):
    """The events of a kind; of allocations and frees their blocks."""
    found = [e for e in events if e.startswith(word)]
    return [re.search(r"block=(\S+)", e)[1] for e in found] if word in ("malloc", "free") else found


# ---------------------------------------------------------------- scratch and captures

def test_scratch_of_a_captured_call_stays(lib):
    ctx = Context(lib)
    before = lib.fake_blocks()
    log(lib)
    ctx.backward(100, 0x10)
    small = of(log(lib), "malloc")[-1]
    lib.fake_stream(0x20, 2, 1)
    ctx.backward(100, 0x20)                          # the graph holds addresses of this block
    lib.fake_stream(0x20, 2, 0)
    ctx.backward(10000, 0x10)
    events = log(lib)
    large = of(events, "malloc")
    assert len(large) == 1 and small not in of(events, "free")
    ctx.backward(20000, 0x10)                        # no graph holds that one
    events = log(lib)
    assert of(events, "free") == large and len(of(events, "malloc")) == 1
    ctx.close()
    assert small in of(log(lib), "free")
    assert lib.fake_blocks() < before                # nothing stays behind


def test_scratch_does_not_grow_in_a_capture(lib, ctx):
    lib.fake_stream(0x20, 2, 1)
    ctx.backward(100, 0x20, rc=E_STATE)              # a context's first call sets its state up
    assert "captured" in ctx.error() and not log(lib)
    lib.fake_stream(0x20, 2, 0)
    ctx.backward(100, 0x10)
    lib.fake_stream(0x20, 2, 1)
    log(lib)
    ctx.backward(10000, 0x20, rc=E_STATE)
    assert "captured" in ctx.error() and not log(lib)
    ctx.backward(90, 0x20)                           # the block that was there still serves
    events = log(lib)
    assert of(events, "launch") and not of(events, "malloc")
    lib.fake_stream(0x20, 2, 0)


# ---------------------------------------------------------------- devices

def test_products_on_two_devices(lib):
    # a kernel's limit on shared memory belongs to the device: every kind of product runs on both
    contexts = [Context(lib, d) for d in (0, 1)]
    for plan in (-1, 1, 2, 4, -2):
        for c in contexts:
            assert lib.distsim_testing_set_product_plan(c.h, plan) == 0
            log(lib)
            c.backward(40, 0x10)
            assert len(of(log(lib), "launch")) == 3
    for c in contexts:
        c.close()


def test_choice_of_kernel_goes_by_the_contexts_device(lib):
    # dx has 4 x 4 tiles with a reduction of 4096: split where the device holds clusters enough
    kinds = []
    for held in (70, 1):
        lib.fake_clusters(held)
        c = Context(lib, len(kinds))
        log(lib)
        c.backward(1000, 0x10, d_in=1024, d_out=4096)
        kinds.append(of(log(lib), "launch")[1])          # behind the column pass
        c.close()
    lib.fake_clusters(10)
    assert "split_product" in kinds[0] and "pair_product" in kinds[1], kinds


def test_a_layer_is_timed_on_the_contexts_device(monkeypatch):
    # streams, captures and events are those of PyTorch's current device: the timing takes the context's for it
    import torch
    from paper_2306_08423_b200 import layers
    now = [0]

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, now[0] = now[0], self.device

        def __exit__(self, *_):
            now[0] = self.before

    class Built(Exception):
        pass

    def build(ctx, *a, **k):
        raise Built(now[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(layers, "FeedForward", build)

    class Second:
        device = 1
    with pytest.raises(Built) as e:
        layers.time_layer(Second, 8, 64, 128)
    assert e.value.args == (1,) and now == [0]


def test_status_waits_for_the_contexts_device(lib, ctx, monkeypatch):
    # without a stream: PyTorch's current one of the context's device, as the operators themselves take it
    from paper_2306_08423_b200 import operators as O
    monkeypatch.setattr(O, "_lib", lib)
    monkeypatch.setattr(O, "_raw_stream", {0: 0x10, 1: 0x20}.__getitem__)

    class Second:
        device, _h = 1, ctx.h

        @staticmethod
        def _check(rc):
            assert rc == 0
    O.distsim_operator_status(Second)
    assert of(log(lib), "synchronize") == ["synchronize device=0 stream=0x20"]


# ---------------------------------------------------------------- order between streams

def test_calls_on_several_streams_wait_for_each_other(lib, ctx):
    ctx.backward(100, 0x10)
    log(lib)
    for stream, waits in ((0x10, 0), (0x20, 1), (0x20, 0), (0x10, 1)):
        ctx.backward(100, stream)
        events = log(lib)
        assert len(of(events, "wait")) == waits, events
        assert not waits or events[0] == f"wait stream={stream:#x}"
        assert events[-1] == f"record stream={stream:#x}"


def test_a_stream_with_an_earlier_ones_handle_waits(lib, ctx):
    # a stream is destroyed with work pending, and the next one gets its handle; the per-thread handle is another
    # stream in every thread
    ctx.backward(100, 0x10)
    log(lib)
    lib.fake_stream(0x10, 77, 0)
    ctx.backward(100, 0x10)
    assert log(lib)[0] == "wait stream=0x10"
    ctx.backward(100, 0x10)
    assert not of(log(lib), "wait")


def test_a_call_that_fails_half_way_is_waited_for(lib, ctx):
    ctx.backward(100, 0x10)
    log(lib)
    lib.fake_fail_launch(2)
    ctx.backward(100, 0x20, rc=E_CUDA)
    assert "operator launch" in ctx.error()
    events = log(lib)
    assert len(of(events, "launch")) == 2 and events[-1] == "record stream=0x20"
    ctx.backward(100, 0x10)
    assert log(lib)[0] == "wait stream=0x10"


# ---------------------------------------------------------------- host memory

def test_no_exception_leaves_a_call(lib):
    # in a process of its own, which an exception through a C entry would end
    code = f"""
import sys
sys.path.insert(0, {os.path.dirname(HERE)!r})
from tests.test_operator_calls import Context, load
lib = load({lib.path!r})
ctx = Context(lib)
for plan in (1, -2, -1):                             # kernels whose shared memory has not been asked for yet
    assert lib.distsim_testing_set_product_plan(ctx.h, plan) == 0
    lib.fake_fail_allocations(0)
    ctx.backward(40, 0x10)
    lib.fake_fail_allocations(-1)
ctx.backward(-1, 0x10, rc=-1)
assert ctx.error() == "linear: sizes"
ctx.close()
"""
    subprocess.run([sys.executable, "-c", code], check=True)
