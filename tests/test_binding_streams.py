"""What the binding allocates for a call on a named stream, without a GPU: every workspace and result is taken from that stream's
memory (a workspace of the current stream's would go back to it when the call returns, while the kernels still write there), and
results are kept until the caller's stream is done with them.  The library and the allocator are stand-ins that record."""
import contextlib
import types

import pytest
import torch

from paper_2512_24545_amd import binding as mb


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


CALLER, SIDE = Stream(1), Stream(2)


class Tensor:
    """Sizes of a contiguous device tensor."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, shape, dtype, made_on=None):
        self.shape, self.dtype, self.made_on, self.used_on = tuple(shape), dtype, made_on, []

    def data_ptr(self):
        return 4096

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        strides = [1]
        for s in self.shape[:0:-1]:
            strides.insert(0, strides[0] * s)
        return tuple(strides) if i is None else strides[i]

    def is_contiguous(self):
        return True

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def split(self, sizes):
        return [Tensor((n,), self.dtype, self.made_on) for n in sizes]

    def record_stream(self, stream):
        self.used_on.append(stream)


class Library:
    """The real one for host arithmetic; device calls record the stream that they were given (their last argument)."""
    HOST = ("mdbf_workspace_bytes", "mdbf_packed_bytes", "mdbf_msvid_block", "mdbf_msvid_workspace_bytes", "mdbf_kv_attention_workspace_bytes",
            "mdbf_kv_page_bytes")

    def __init__(self, real, log):
        self.real, self.log = real, log

    def __getattr__(self, name):
        if name in self.HOST:
            return getattr(self.real, name)

        def call(*args):
            self.log.append((name, args[-1]))
            return 0
        return call


@pytest.fixture
def world(monkeypatch):
    """(tensors made so far, device calls so far)"""
    mb._torch()                                  # the tables of types are the real ones
    real, made, calls, current = mb.lib(), [], [], [CALLER]

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def empty(*shape, dtype=None, device=None):
        shape = shape[0] if isinstance(shape[0], tuple) else shape
        made.append(Tensor(shape, dtype, current[-1]))
        return made[-1]

    fake = types.SimpleNamespace(empty=empty, cuda=types.SimpleNamespace(stream=on, current_stream=lambda device=None: current[-1]),
                                 **{n: getattr(torch, n) for n in ("float16", "bfloat16", "float32", "int8", "uint8", "int32", "int64")},
                                 _C=types.SimpleNamespace(_cuda_getDevice=lambda: 0, _cuda_getCurrentRawStream=lambda d: current[-1].cuda_stream))
    monkeypatch.setattr(mb, "_torch_module", fake)
    monkeypatch.setattr(mb, "_lib", Library(real, calls))
    return made, calls


def ints(*shape):
    return Tensor(shape, torch.int32)


def layer():
    f = lambda *shape: Tensor(shape, torch.float16)
    return mb.DeviceLayer(256, 256, 128, 16, f(1), f(1), f(256, 16), f(128, 16), f(128, 16), f(256, 16))


def cache():
    return mb.KVCache(40, 2, 128, 64, "bf16", buffer=Tensor((40 * 2 * 64 * 136,), torch.uint8))


def heads(T, H):
    return Tensor((T, H, 128), torch.bfloat16)


CALLS = {
    "mdbf_pack": (lambda s: mb.mdbf_pack(Tensor((64, 64), torch.int8), stream=s), 1),
    "mdbf_unpack": (lambda s: mb.mdbf_unpack(Tensor((512,), torch.uint8), 64, 64, stream=s), 1),
    "mdbf_pad_envelope": (lambda s: mb.mdbf_pad_envelope(Tensor((64, 4), torch.float16), 8, stream=s), 1),
    "mdbf_forward": (lambda s: mb.mdbf_forward(layer(), Tensor((8, 256), torch.float16), stream=s), 1),
    "mdbf_msvid": (lambda s: mb.mdbf_msvid(Tensor((256, 256), torch.float32), 16, Tensor((256, mb.mdbf_msvid_block(16)), torch.float32), stream=s), 4),
    "mdbf_kv_slots": (lambda s: mb.mdbf_kv_slots(ints(3), ints(3), ints(3, 9), ints(20), ints(1), 64, 3, stream=s), 2),
    "mdbf_kv_read": (lambda s: mb.mdbf_kv_read(cache(), Tensor((5,), torch.int64), stream=s), 2),
    "mdbf_qk_norm_rope": (lambda s: mb.mdbf_qk_norm_rope(heads(5, 4), heads(5, 2), None, None, stream=s), 2),
    "mdbf_kv_attention": (lambda s: mb.mdbf_kv_attention(cache(), heads(2, 4), ints(2, 40), ints(3), ints(2), 1, 2000, stream=s), 1),
}
WORKSPACES = {"mdbf_forward": 1, "mdbf_msvid": 1, "mdbf_kv_attention": 1}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_a_named_stream(world, name):
    made, calls = world
    call, results = CALLS[name]
    call(SIDE)
    assert calls == [(name, SIDE.cuda_stream)]
    assert len(made) == results + WORKSPACES.get(name, 0)
    assert all(t.made_on is SIDE for t in made)
    kept = [t for t in made if t.used_on]
    assert len(kept) == results and all(t.used_on == [CALLER] for t in kept)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_the_current_stream(world, name):
    made, calls = world
    call, results = CALLS[name]
    call(None)
    assert calls == [(name, CALLER.cuda_stream)]
    assert len(made) == results + WORKSPACES.get(name, 0)
    assert all(t.made_on is CALLER and not t.used_on for t in made)
