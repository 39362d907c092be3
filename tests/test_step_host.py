"""The operators around the projections, without a GPU: the 64-bit oracle pinned by hand, and every refusal of the entry points (all of them before
any HIP call)."""
import ctypes as C

import numpy as np
import pytest

from oracle import step_oracle as so
from paper_2512_24545_amd import binding as mb

A = 4096          # an aligned address that no refused call touches
HUGE = 1 << 50


# ---- oracle ----------------------------------------------------------------------------------------
def test_norm_oracle_by_hand():
    y, h = so.add_norm(np.array([[1.0, 2.0]]), np.array([[2.0, 2.0]]), np.array([1.0, 10.0]), 3.5)
    assert h.tolist() == [[3.0, 4.0]] and np.allclose(y, [[3 / 4, 40 / 4]])     # mean 12.5, and 3.5: 16
    y, _ = so.add_norm(np.array([[1.0, -1.0, 1.0, 1.0]]), None, None, 0.0)
    assert y.tolist() == [[1.0, -1.0, 1.0, 1.0]]


def test_e4m3_by_hand():
    grid = sorted({(1 + m / 8) * 2.0 ** e for m in range(8) for e in range(-6, 9)} - {480.0} | {m / 8 * 2.0 ** -6 for m in range(8)})
    assert len(grid) == 127 and grid[-1] == 448.0
    v = np.concatenate((grid, [-g for g in grid]))
    assert np.array_equal(so.e4m3(v), v)
    mid = [(a + b) / 2 for a, b in zip(grid, grid[1:])]
    assert all(so.e4m3(m * (1 - 1e-9)) == a and so.e4m3(m * (1 + 1e-9)) == b for m, a, b in zip(mid, grid, grid[1:]))
    assert so.e4m3(np.array([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10])).tolist() == [16.0, 20.0, 0.0, 2.0 ** -8] and so.e4m3(460.0) == 448.0


def test_block_scales_by_hand():
    y = np.zeros((1, 32 * 7 + 5))
    for b, top in enumerate((448.0, 448.1, 1.75, 1.76, 1e-300, np.nan, -896.0, 0.0)):
        y[0, min(32 * b + 3, y.shape[1] - 1)] = top
    assert so.block_scales(y).tolist() == [[127, 128, 119, 120, 1, 255, 128, 1]]


def test_tables_oracle_by_hand():
    rows, tiles, places = so.adapter_tables([0, 2, 2, 70, 73], [1, 0, 1, -1], 2, 75, 3)
    assert rows.tolist() == [0, 1] + list(range(2, 70)) + [-1] * 5
    assert tiles.tolist() == [[1, 0, 64, 0], [1, 64, 6, 0], [-1, 0, 0, 0]] and places.tolist() == [0, 0, 2, 70]
    rows, tiles, places = so.adapter_tables([0, 1, 2, 3], [1, 0, 1], 2, 3, 2)
    assert rows.tolist() == [1, 0, 2] and tiles.tolist() == [[0, 0, 1, 0], [1, 1, 2, 0]] and places.tolist() == [1, 0, 2]


def test_adapters_oracle_by_hand():
    out = so.adapters(np.array([[1.0, 2.0], [1.0, 1.0], [5.0, 5.0]]), [1, 0, -1], np.array([[[1.0, 1.0]], [[1.0, 0.0]]]), np.array([[[2.0], [3.0]], [[4.0], [5.0]]]), [1.0, 0.5])
    assert out.tolist() == [[2.0, 2.5], [4.0, 6.0], [0.0, 0.0]]


def test_sampling_oracle_by_hand():
    z = np.log([0.1, 0.4, 0.2, 0.3])                     # in order: tokens 1, 3, 2, 0
    assert [so.sample(z, u)[0] for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91)] == [1, 1, 3, 3, 2, 2, 0]
    assert [so.sample(z, u, top_k=2)[0] for u in (0.5, 0.58, 0.99)] == [1, 3, 3]
    assert [so.sample(z, u, top_p=0.65)[0] for u in (0.5, 0.99)] == [1, 3] and np.isclose(so.sample(z, 0.0, top_p=0.65)[1], 4 / 7)
    assert [so.sample(z, 0.99, min_p=m)[0] for m in (0.2, 0.3, 0.6, 0.8)] == [0, 2, 3, 1]
    assert so.sample(z, 0.99, temperature=0.0) == (1, 1.0) and so.sample(np.full(3, -np.inf), 0.5) == (-1, 0.0)
    assert so.sample([1.0, 1.0, 1.0, 1.0], 0.5)[0] == 2 and so.sample([np.nan, -np.inf, 0.0], 0.99)[0] == 2
    assert np.isclose(so.sample(z, 0.0, temperature=0.5)[1], 0.16 / 0.30)


# ---- refusals --------------------------------------------------------------------------------------
def norm(**kw):
    d = dict(n=100, x_dtype=1, h_dtype=1, y_dtype=1, scale_group=0, eps=1e-6)
    d.update(kw)
    return mb.NormDesc(*[d[n] for n in ("n", "x_dtype", "h_dtype", "y_dtype", "scale_group", "eps")])


def test_add_norm_arguments():
    L = mb.lib()
    good = [norm(), A, 100, A, 100, A, 3, A, 100, A, 100, None, 0, None]
    for kw, status in ((dict(n=0), -1), (dict(n=-4), -1), (dict(n=65537), -1), (dict(x_dtype=3), -3), (dict(x_dtype=-1), -3), (dict(h_dtype=3), -3), (dict(y_dtype=4), -3),
                       (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(h_dtype=0), -5), (dict(scale_group=32), -1), (dict(y_dtype=3), -1)):
        args = list(good)
        args[0] = norm(**kw)
        assert L.mdbf_add_norm(*args) == status, kw
    for at, bad, status in ((0, None, -1), (1, None, -1), (1, A + 8, -2), (2, 99, -1), (3, A + 2, -2), (3, None, -1), (4, 99, -1), (5, A + 4, -2), (6, 0, -1), (6, -1, -1),
                            (7, A + 8, -2), (8, 99, -1), (9, None, -1), (9, A + 1, -2), (10, 99, -1), (11, A, -1)):
        args = list(good)
        args[at] = bad
        assert L.mdbf_add_norm(*args) == status, (at, bad)
    wide = [norm(n=65537), A, 70000, A, 70000, A, 3, A, 70000, A, 70000, None, 0, None]
    assert L.mdbf_add_norm(*wide) == -5
    eight = [norm(y_dtype=3, scale_group=32), A, 100, None, 0, None, 3, None, 0, A, 100, A, 4, None]
    for at, bad, status in ((0, norm(y_dtype=3, scale_group=16), -5), (11, None, -1), (11, A + 4, -2), (12, 3, -1), (7, A, -1)):
        args = list(eight)
        args[at] = bad
        assert L.mdbf_add_norm(*args) == status, (at, bad)
    assert L.mdbf_add_norm(norm(y_dtype=3), A, 100, None, 0, None, 3, None, 0, A, 100, A, 0, None) == -1


def test_adapter_tables_arguments():
    L = mb.lib()
    assert L.mdbf_adapter_tiles(64, 64, 32) == 33 and L.mdbf_adapter_tiles(63, 64, 100) == 63 and L.mdbf_adapter_tiles(1, 1, 1) == 1
    assert L.mdbf_adapter_tiles(6400, 3, 100) == 103 and L.mdbf_adapter_tiles(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1) == 2 ** 25 - 1 + 2 ** 31 - 1
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0)):
        assert L.mdbf_adapter_tiles(*bad) == -1
    good = [64, 64, 32, A, A, A, A, 33, A, None]
    for at, bad, status in ((0, 0, -1), (1, 0, -1), (2, 0, -1), (2, 8193, -1), (7, 32, -1), (7, -1, -1)) + tuple((i, None, -1) for i in (3, 4, 5, 6, 8)) + \
            tuple((i, A + 2, -2) for i in (3, 4, 5, 8)) + ((6, A + 4, -2),):
        args = list(good)
        args[at] = bad
        assert L.mdbf_adapter_rows(*args) == status, (at, bad)
    assert L.mdbf_adapter_rows(64, 64, 8193, A, A, A, A, 65, A, None) == -5


def adapter(**kw):
    d = dict(n=100, m=50, r=8, y_dtype=1, A_dev=A, B_dev=A, scale_dev=A, X_dev=A, ldx=100, Y_dev=A, ldy=50)
    d.update(kw)
    return mb.AdapterDesc(*[d[n] for n in ("n", "m", "r", "y_dtype", "A_dev", "B_dev", "scale_dev", "X_dev", "ldx", "Y_dev", "ldy")])


def test_adapters_arguments():
    L, out = mb.lib(), C.c_size_t(0)

    def call(*list_, count=None, dtype=1, adapters=4, T=10, rows=A, tiles=A, room=3, ws=A, size=HUGE):
        arr = (mb.AdapterDesc * max(len(list_), 1))(*list_) if list_ else None
        return L.mdbf_adapters(len(list_) if count is None else count, arr, dtype, adapters, T, rows, tiles, room, ws, size, None)

    for kw, status in ((dict(n=0), -1), (dict(m=0), -1), (dict(r=0), -1), (dict(r=257), -5), (dict(n=(1 << 23) + 1, ldx=1 << 24), -5), (dict(m=(1 << 23) + 1, ldy=1 << 24), -5), (dict(y_dtype=3), -3), (dict(A_dev=None), -1), (dict(B_dev=None), -1),
                       (dict(X_dev=None), -1), (dict(Y_dev=None), -1), (dict(ldx=99), -1), (dict(ldy=49), -1), (dict(A_dev=A + 8), -2), (dict(B_dev=A + 2), -2),
                       (dict(X_dev=A + 4), -2), (dict(Y_dev=A + 8), -2), (dict(scale_dev=A + 2), -2)):
        assert call(adapter(**kw)) == status, kw
        assert call(adapter(Y_dev=2 * A), adapter(**kw)) == status, kw
    for kw, status in ((dict(count=0), -1), (dict(dtype=2), -3), (dict(dtype=3), -3), (dict(adapters=0), -1), (dict(T=0), -1), (dict(rows=None), -1), (dict(tiles=None), -1),
                       (dict(room=0), -1), (dict(ws=None), -1), (dict(rows=A + 2), -2), (dict(tiles=A + 8), -2), (dict(ws=A + 8), -2), (dict(size=0), -4)):
        assert call(adapter(), **kw) == status, kw
    assert call() == -1 and call(*[adapter(Y_dev=A * (i + 1)) for i in range(9)]) == -1
    assert call(adapter(), adapter()) == -1                          # two projections of one Y
    arr = (mb.AdapterDesc * 1)(adapter())
    assert L.mdbf_adapters_workspace_bytes(1, arr, 1, 4, 10, 3, None) == -1 and L.mdbf_adapters_workspace_bytes(1, arr, 2, 4, 10, 3, C.byref(out)) == -3
    assert L.mdbf_adapters_workspace_bytes(1, arr, 1, 4, 10, 3, C.byref(out)) == 0 and out.value > 0
    assert call(adapter(), size=out.value - 1) == -4


def test_sample_arguments():
    L, out = mb.lib(), C.c_size_t(0)
    none = mb.SampleDesc(None, None, None, None)
    good = [none, A, 100, 2, 3, 100, A, A, A, A, HUGE, None]
    for at, bad, status in ((0, None, -1), (1, None, -1), (1, A + 8, -2), (2, 99, -1), (3, 3, -3), (3, -1, -3), (4, 0, -1), (5, 0, -1), (6, None, -1), (6, A + 2, -2),
                            (7, None, -1), (7, A + 2, -2), (8, A + 1, -2), (9, None, -1), (9, A + 8, -2), (10, 0, -4), (0, mb.SampleDesc(A + 2, None, None, None), -2),
                            (0, mb.SampleDesc(None, A + 2, None, None), -2), (0, mb.SampleDesc(None, None, A + 1, None), -2), (0, mb.SampleDesc(None, None, None, A + 2), -2)):
        args = list(good)
        args[at] = bad
        assert L.mdbf_sample(*args) == status, (at, bad)
    assert L.mdbf_sample(none, A, 1 << 21, 2, 3, (1 << 20) + 1, A, A, A, A, HUGE, None) == -5
    assert L.mdbf_sample_workspace_bytes(1, 10, None) == -1 and L.mdbf_sample_workspace_bytes(0, 10, C.byref(out)) == -1
    assert L.mdbf_sample_workspace_bytes(1, 0, C.byref(out)) == -1 and L.mdbf_sample_workspace_bytes(1, (1 << 20) + 1, C.byref(out)) == -5
    last = 0
    for T, vocab in ((1, 1), (1, 32000), (2, 32000), (2, 40000), (2, 128256), (600, 128256), (600, 262144), (70000, 262144), (70000, 1 << 20)):
        assert L.mdbf_sample_workspace_bytes(T, vocab, C.byref(out)) == 0 and out.value >= last
        last = out.value


def test_new_types_are_refused_where_they_were():
    """8-bit results are mdbf_add_norm's alone."""
    L = mb.lib()
    d = mb.Desc(16, 16, 16, 1, 3, 0, 2, 0)
    out = C.c_size_t(0)
    assert L.mdbf_workspace_bytes(C.byref(d), 1, C.byref(out)) == -3
    rope = mb.RopeDesc(4, 2, 128, 0, 0, 1, 3, 0, 1e-6)
    assert L.mdbf_qk_norm_rope(rope, A, 512, A, 256, None, None, None, None, 1, A, 512, A, 256, None, None, 0, None, 0, None, None) == -3


def test_more_tiles_than_a_launch_has():
    """2^24 tiles would be 2^32 threads, which a launch does not have."""
    L, out = mb.lib(), C.c_size_t(0)
    arr = (mb.AdapterDesc * 1)(adapter())
    for room, status in ((1 << 24, -5), (1 << 31, -5), ((1 << 24) - 1, -4)):
        assert L.mdbf_adapters(1, arr, 1, 4, 10, A, A, room, A, 0, None) == status
        assert L.mdbf_adapters_workspace_bytes(1, arr, 1, 4, 10, room, C.byref(out)) == (0 if status == -4 else status)
