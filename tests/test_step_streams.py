"""What the binding allocates for the operators around the projections on a named stream, and what it refuses before any call, without a GPU: with the
stand-ins that record of test_binding_streams."""
import pytest
import torch

import test_binding_streams as tb
from paper_2512_24545_amd import binding as mb

world = tb.world
HOST = ("mdbf_adapter_tiles", "mdbf_adapters_workspace_bytes", "mdbf_sample_workspace_bytes")


@pytest.fixture(autouse=True)
def stand_ins(world, monkeypatch):
    monkeypatch.setattr(tb.Library, "HOST", tb.Library.HOST + HOST)
    monkeypatch.setattr(tb.Tensor, "get_device", lambda self: getattr(self, "index", 0), raising=False)
    monkeypatch.setattr(tb.Tensor, "as_strided", lambda self, shape, strides: tb.Tensor(shape, self.dtype, self.made_on), raising=False)
    monkeypatch.setattr(tb.Tensor, "split_with_sizes", tb.Tensor.split, raising=False)
    monkeypatch.setattr(tb.Tensor, "new_empty", lambda self, shape, dtype: mb._torch_module.empty(tuple(shape), dtype=dtype), raising=False)
    mb._torch_module.empty_like = lambda like, dtype=None: mb._torch_module.empty(tuple(like.shape), dtype=dtype)
    mb._torch_module.float8_e4m3fn = torch.float8_e4m3fn


def T16(*shape):
    return tb.Tensor(shape, torch.bfloat16)


def f32(*shape):
    return tb.Tensor(shape, torch.float32)


def rows(T=5, requests=3, adapters=4):
    return mb.AdapterRows(T, requests, adapters, rows=tb.ints(T), tiles=tb.ints(6, 4))


def pool():
    return mb.Adapters(T16(4, 8, 64), T16(4, 32, 8), f32(4))


CALLS = {
    "mdbf_add_norm": (lambda s: mb.mdbf_add_norm(T16(3, 64), T16(3, 64), f32(64), y_dtype="e4m3", stream=s), 3, 0),
    "mdbf_adapter_rows": (lambda s: mb.mdbf_adapter_rows(tb.ints(4), tb.ints(3), 4, 5, stream=s), 1, 0),
    "mdbf_adapters": (lambda s: mb.mdbf_adapters(rows(), [pool()], [T16(5, 64)], [T16(5, 32)], stream=s), 0, 1),
    "mdbf_sample": (lambda s: mb.mdbf_sample(f32(3, 100), f32(3), stream=s), 2, 1),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_a_named_stream(world, name):
    made, calls = world
    call, results, workspaces = CALLS[name]
    call(tb.SIDE)
    assert calls == [(name, tb.SIDE.cuda_stream)] and len(made) == results + workspaces
    assert all(t.made_on is tb.SIDE for t in made)
    kept = [t for t in made if t.used_on]
    assert len(kept) == results and all(t.used_on == [tb.CALLER] for t in kept)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_the_current_stream(world, name):
    made, calls = world
    call, results, workspaces = CALLS[name]
    call(None)
    assert calls == [(name, tb.CALLER.cuda_stream)] and len(made) == results + workspaces
    assert all(t.made_on is tb.CALLER and not t.used_on for t in made)


def _elsewhere(t):
    t.index = 1
    return t


REFUSED = {
    "norm: another device": lambda: mb.mdbf_add_norm(_elsewhere(T16(3, 64))),
    "norm: a weight of another device": lambda: mb.mdbf_add_norm(T16(3, 64), weight=_elsewhere(f32(64))),
    "norm: residual of another shape": lambda: mb.mdbf_add_norm(T16(3, 64), T16(4, 64)),
    "norm: residual_out without residual": lambda: mb.mdbf_add_norm(T16(3, 64), residual_out=T16(3, 64)),
    "norm: residual_out of another type": lambda: mb.mdbf_add_norm(T16(3, 64), T16(3, 64), residual_out=f32(3, 64)),
    "norm: scales without 8 bits": lambda: mb.mdbf_add_norm(T16(3, 64), scales=f32(3, 1)),
    "norm: scales of another shape": lambda: mb.mdbf_add_norm(T16(3, 64), y_dtype="e4m3", scale_group=32, scales=tb.Tensor((3, 3), torch.uint8)),
    "norm: a 16-bit weight": lambda: mb.mdbf_add_norm(T16(3, 64), weight=T16(64)),
    "norm: out of another type than asked for": lambda: mb.mdbf_add_norm(T16(3, 64), y_dtype="f32", out=T16(3, 64)),
    "rows: cu too short": lambda: mb.mdbf_adapter_rows(tb.ints(3), tb.ints(3), 4, 5),
    "rows: 64-bit adapters": lambda: mb.mdbf_adapter_rows(tb.ints(4), tb.Tensor((3,), torch.int64), 4, 5),
    "rows: tables of other sizes": lambda: mb.mdbf_adapter_rows(tb.ints(4), tb.ints(3), 4, 5, out=mb.AdapterRows(6, 3, 4)),
    "rows: tables made by other means": lambda: mb.mdbf_adapter_rows(tb.ints(4), tb.ints(3), 4, 5, out=rows()),
    "adapters: rows of other adapters": lambda: mb.mdbf_adapters(rows(adapters=5), [pool()], [T16(5, 64)], [T16(5, 32)]),
    "adapters: X too narrow": lambda: mb.mdbf_adapters(rows(), [pool()], [T16(5, 63)], [T16(5, 32)]),
    "adapters: X too short": lambda: mb.mdbf_adapters(rows(), [pool()], [T16(4, 64)], [T16(5, 32)]),
    "adapters: Y too wide": lambda: mb.mdbf_adapters(rows(), [pool()], [T16(5, 64)], [T16(5, 33)]),
    "adapters: X of another type": lambda: mb.mdbf_adapters(rows(), [pool()], [tb.Tensor((5, 64), torch.float16)], [T16(5, 32)]),
    "adapters: fewer Ys": lambda: mb.mdbf_adapters(rows(), [pool()], [T16(5, 64)], []),
    "adapters: none": lambda: mb.mdbf_adapters(rows(), [], [], []),
    "adapters: another device": lambda: mb.mdbf_adapters(rows(), [pool()], [T16(5, 64)], [_elsewhere(T16(5, 32))]),
    "adapters: factors that do not go together": lambda: mb.Adapters(T16(4, 8, 64), T16(4, 32, 9)),
    "adapters: a 16-bit scale": lambda: mb.Adapters(T16(4, 8, 64), T16(4, 32, 8), T16(4)),
    "sample: u of another length": lambda: mb.mdbf_sample(f32(3, 100), f32(4)),
    "sample: top_k of another type": lambda: mb.mdbf_sample(f32(3, 100), f32(3), top_k=tb.Tensor((3,), torch.int64)),
    "sample: a 64-bit temperature": lambda: mb.mdbf_sample(f32(3, 100), f32(3), temperature=tb.Tensor((3,), torch.float64)),
    "sample: tokens of another type": lambda: mb.mdbf_sample(f32(3, 100), f32(3), tokens=tb.Tensor((3,), torch.int64)),
    "sample: another device": lambda: mb.mdbf_sample(_elsewhere(f32(3, 100)), f32(3)),
}


@pytest.mark.parametrize("name", sorted(REFUSED))
def test_refused(world, name):
    with pytest.raises((AssertionError, mb.MdbfError)):
        REFUSED[name]()
    assert not world[1]


class Moved(tb.Tensor):
    """A tensor whose memory can be swapped, as set_ and data do."""
    at = 4096

    def data_ptr(self):
        return self.at


def test_adapters_that_get_other_memory(world, monkeypatch):
    """A call reads where its adapters lie then, and checks them again if that changed; they are not replaced behind its back."""
    A, B, scale = Moved((4, 8, 64), torch.bfloat16), Moved((4, 32, 8), torch.bfloat16), Moved((4,), torch.float32)
    p, sent = mb.Adapters(A, B, scale), []
    record = mb._lib
    monkeypatch.setattr(type(record), "mdbf_adapters", lambda self, count, arr, *rest: sent.append(mb.struct.unpack("4i7q", arr)[4:7]) or 0, raising=False)
    call = lambda: mb.mdbf_adapters(rows(), [p], [T16(5, 64)], [T16(5, 32)])             # noqa: E731
    call()
    A.at, B.at, scale.at = 1 << 20, 2 << 20, 3 << 20
    call()
    assert sent == [(4096, 4096, 4096), (1 << 20, 2 << 20, 3 << 20)]
    for t, attribute, other in ((A, "shape", (3, 8, 64)), (B, "shape", (4, 31, 8)), (B, "dtype", torch.float16), (scale, "dtype", torch.bfloat16)):
        kept = getattr(t, attribute)
        setattr(t, attribute, other)
        t.at += 16
        with pytest.raises(AssertionError):
            call()
        setattr(t, attribute, kept)
        call()
    for name in ("A", "B", "scale"):
        with pytest.raises(AttributeError):
            setattr(p, name, B)
    assert (p.A, p.B, p.scale) == (A, B, scale) and len(sent) == 6


@pytest.mark.parametrize("given", ["rows", "tiles"])
def test_half_of_the_tables(world, given):
    """Rows without tiles, or tiles without rows, are no tables, and are not dropped either."""
    with pytest.raises(AssertionError):
        mb.AdapterRows(5, 3, 4, **{given: tb.ints(5) if given == "rows" else tb.ints(6, 4)})
    assert not world[0]


@pytest.mark.parametrize("name,table", [("rows", (4,)), ("rows", (5, 2)), ("places", (2,)), ("tiles", (6, 3))])
def test_tables_whose_parts_were_replaced(world, name, table):
    """The parts of an AdapterRows that is handed to a call have the sizes that the kernel writes."""
    out = mb.AdapterRows(5, 3, 4)
    mb.mdbf_adapter_rows(tb.ints(4), tb.ints(3), 4, 5, out=out)
    setattr(out, name, tb.ints(*table))
    with pytest.raises(AssertionError):
        mb.mdbf_adapter_rows(tb.ints(4), tb.ints(3), 4, 5, out=out)
    assert len(world[1]) == 1
