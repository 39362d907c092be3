"""mdbf_adapter_rows and mdbf_adapters against the definitions.  Bounds of the products: sums of n and r terms in fp32 are off by at most their count times a step
of the sum of magnitudes; the inner values are carried to 2^-16 of themselves (bf16, 16-bit results), 2^-23 (fp32 results) or 2^-22 of their
row's largest (fp16); results are rounded once to their type."""
import numpy as np
import pytest

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2512_24545_amd import binding as mb
    mb.lib()
    return torch, mb


def _dt(torch, name):
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[name]


def _ints(torch, v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda:0")


def _step(rng, requests, adapters, fresh):
    f = rng.integers(0, fresh + 1, requests) if fresh > 1 else np.ones(requests, dtype=int)
    cu = np.concatenate(([0], np.cumsum(f)))
    return cu, rng.integers(-1, adapters + 1, requests)          # both -1 and `adapters` are none


@pytest.mark.parametrize("requests,adapters,fresh", [(1, 1, 1), (1, 3, 1000), (64, 32, 1), (300, 5, 1), (1500, 400, 1), (37, 9, 40), (500, 100, 300), (1024, 8000, 3),
                                                     (1025, 8192, 9), (3000, 7, 12), (4, 2, 9000), (5000, 5000, 1)])
def test_rows_and_tiles(gpu, requests, adapters, fresh):
    torch, mb = gpu
    rng = np.random.default_rng(requests + adapters)
    cu, of = _step(rng, requests, adapters, fresh)
    T = max(int(cu[-1]) + int(rng.integers(0, 3)) * 7, 1)        # rows behind the last request too
    got = mb.mdbf_adapter_rows(_ints(torch, cu), _ints(torch, of), adapters, T)
    rows, tiles, places = so.adapter_tables(cu.tolist(), of.tolist(), adapters, T, got.tiles.shape[0])
    assert np.array_equal(got.places.cpu().numpy(), places)
    assert np.array_equal(got.rows.cpu().numpy(), rows)
    assert np.array_equal(got.tiles.cpu().numpy(), tiles)
    again = mb.mdbf_adapter_rows(_ints(torch, cu), _ints(torch, of), adapters, T, out=got)
    assert again is got and np.array_equal(got.rows.cpu().numpy(), rows)


def test_rows_of_steps_without_adapters_or_tokens(gpu):
    torch, mb = gpu
    for cu, of in (([0, 0, 0], [0, 1]), ([0, 5, 9], [-1, 7]), ([0, 0, 64, 64, 128], [0, 1, 1, 1])):
        T = max(cu[-1], 1)
        got = mb.mdbf_adapter_rows(_ints(torch, cu), _ints(torch, of), 2, T)
        rows, tiles, places = so.adapter_tables(cu, of, 2, T, got.tiles.shape[0])
        assert np.array_equal(got.rows.cpu().numpy(), rows) and np.array_equal(got.tiles.cpu().numpy(), tiles)


def test_bad_row_bounds_write_nothing_outside(gpu):
    """cu that falls or leaves the step: the tables are of no use then, but what lies around them stays."""
    torch, mb = gpu
    T, n = 200, 6
    for cu in ([0, 500, 1000, -5, 7, 90000, 3], [0, 150, 20, 199, 0, 200, 200], [2 ** 31 - 1] * 7, [-2 ** 31, 0, 1, 2, 3, 2 ** 31 - 1, 0]):
        for long in (False, True):
            TT = 20000 if long else T
            room = mb.lib().mdbf_adapter_tiles(TT, n, 4)
            store = torch.full((4 * room + TT + n + 192,), 77, dtype=torch.int32, device="cuda:0")
            out = mb.AdapterRows(TT, n, 4)
            out.tiles = store[64:64 + 4 * room].view(room, 4)
            out.rows = store[128 + 4 * room:128 + 4 * room + TT]
            out.places = store[-n:]
            mb.mdbf_adapter_rows(_ints(torch, cu), _ints(torch, [0, 1, 2, 3, 0, 1]), 4, TT, out=out)
            torch.cuda.synchronize()
            assert (store[:64] == 77).all() and (store[64 + 4 * room:128 + 4 * room] == 77).all() and (store[128 + 4 * room + TT:-n] == 77).all()


def _bound(x, of, A, B, scale, y_before, want, x_dtype, y_dtype):
    n, r = A.shape[2], A.shape[1]
    out = np.zeros_like(want)
    carried = {"f16": 2.0 ** -22, "bf16": 2.0 ** -23 if y_dtype == "f32" else 2.0 ** -16}[x_dtype]
    for t, a in enumerate(of):
        if 0 <= a < A.shape[0]:
            inner, size = A[a] @ x[t], np.abs(A[a]) @ np.abs(x[t])
            off = (n + 8) * 2.0 ** -24 * size + carried * (np.abs(inner) if x_dtype == "bf16" else np.abs(inner).max())
            out[t] = abs(scale[a]) * (np.abs(B[a]) @ (off + (r + 8) * 2 * 2.0 ** -24 * np.abs(inner)))
            out[t] += 4 * 2.0 ** -24 * np.abs(y_before[t])
    return out * (1 + 2.0 ** -7) + HALF[y_dtype] * np.abs(want) + TINY[y_dtype]


def _check(gpu, requests, adapters, fresh, shapes, x_dtype, y_dtypes, seed=0, pad=0, scaled=True, same_x=True, x_scale=1.0):
    torch, mb = gpu
    rng = np.random.default_rng(seed)
    cu, of = _step(rng, requests, adapters, fresh)
    T = max(int(cu[-1]), 1) + 3
    of_row = np.full(T, -1)
    for r in range(requests):
        of_row[cu[r]:cu[r + 1]] = of[r]
    rows = mb.mdbf_adapter_rows(_ints(torch, cu), _ints(torch, of), adapters, T)
    dt = _dt(torch, x_dtype)
    # (at most fp16's largest: of deviates of 30000 one in thirty would be an infinity there, whose products are no numbers to compare)
    make = lambda shape, d, s=1.0: torch.from_numpy(np.clip(rng.standard_normal(shape) * s, -65504, 65504).astype(np.float32)).to("cuda:0").to(d)   # noqa: E731
    pools, Xs, Ys, wide = [], [], [], []
    for i, (n, m, r) in enumerate(shapes):
        scale = torch.from_numpy(rng.random(adapters).astype(np.float32)).to("cuda:0") if scaled else None
        pools.append(mb.Adapters(make((adapters, r, n), dt, n ** -0.5), make((adapters, m, r), dt, 0.5 * r ** -0.5), scale))
        Xs.append(Xs[0] if i and same_x and n == shapes[0][0] else make((T, n + pad), dt, x_scale)[:, :n])
        wide.append(make((T, m + pad), _dt(torch, y_dtypes[i])))
        Ys.append(wide[-1][:, :m])
    before = [w.clone() for w in wide]
    assert mb.mdbf_adapters(rows, pools, Xs, Ys) is Ys
    for i, (n, m, r) in enumerate(shapes):
        x, A, B = (v.double().cpu().numpy() for v in (Xs[i], pools[i].A, pools[i].B))
        scale = pools[i].scale.double().cpu().numpy() if scaled else np.ones(adapters)
        y0 = before[i][:, :m].double().cpu().numpy()
        want = y0 + so.adapters(x, of_row, A, B, scale)
        err = np.abs(Ys[i].double().cpu().numpy() - want)
        assert (err <= _bound(x, of_row, A, B, scale, y0, want, x_dtype, y_dtypes[i])).all(), (i, float(err.max()))
        none = torch.from_numpy((of_row < 0) | (of_row >= adapters)).to("cuda:0")
        assert torch.equal(Ys[i][none], before[i][:, :m][none]) and torch.equal(wide[i][:, m:], before[i][:, m:])
    first = [w.clone() for w in wide]
    for w, b in zip(wide, before):
        w.copy_(b)
    mb.mdbf_adapters(rows, pools, Xs, Ys)
    assert all(torch.equal(a, b) for a, b in zip(first, wide))


@pytest.mark.parametrize("r", [1, 2, 5, 8, 9, 16, 17, 24, 31, 32, 40, 64, 100, 128, 200, 256])
@pytest.mark.parametrize("x_dtype,y_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "f16")])
def test_ranks_and_types(gpu, r, x_dtype, y_dtype):
    _check(gpu, 9, 3, 30, [(264, 136, r)], x_dtype, [y_dtype], seed=r)


@pytest.mark.parametrize("n,m", [(1, 1), (7, 3), (31, 17), (32, 64), (33, 65), (127, 513), (128, 512), (129, 1000), (1601, 530), (4096, 255)])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_shapes_and_strides(gpu, n, m, pad):
    _check(gpu, 11, 4, 21, [(n, m, 8)], "bf16", ["bf16"], seed=n, pad=pad)
    _check(gpu, 11, 4, 21, [(n, m, 5)], "f16", ["f32"], seed=m, pad=pad, scaled=False)


@pytest.mark.parametrize("requests,adapters,fresh", [(1, 1, 1), (5, 9, 1), (64, 32, 1), (200, 2, 1), (3, 2, 64), (4, 1, 65), (6, 2, 500), (40, 40, 70)])
def test_steps(gpu, requests, adapters, fresh):
    _check(gpu, requests, adapters, fresh, [(520, 392, 16)], "bf16", ["bf16"], seed=requests)


def test_several_projections_in_one_call(gpu):
    shapes = [(256, 128, 16), (256, 128, 5), (256, 640, 40), (200, 64, 16), (256, 32, 1), (96, 72, 130), (256, 8, 16), (256, 264, 64)]
    _check(gpu, 20, 6, 9, shapes, "bf16", ["bf16", "f32", "bf16", "f16", "bf16", "f32", "f32", "bf16"], seed=1)
    _check(gpu, 20, 6, 9, shapes[:3], "f16", ["f16", "f16", "f16"], seed=2, same_x=False)
    _check(gpu, 3, 2, 1, [(96, 96, 256)] * 8, "f16", ["f32"] * 8, seed=3)


def test_fp16_inner_values_beyond_its_range(gpu):
    """Rows whose inner values are past 65504, or far below the smallest fp16 number."""
    _check(gpu, 6, 2, 8, [(2048, 64, 16)], "f16", ["f32"], seed=4, x_scale=30000.0)
    _check(gpu, 6, 2, 8, [(2048, 64, 16)], "f16", ["f32"], seed=5, x_scale=1e-6)


def test_rows_do_not_reach_each_other(gpu):
    """A NaN or an infinity in a row of X, or in an adapter, stays with the rows that read it."""
    torch, mb = gpu
    rng = np.random.default_rng(6)
    T, n, m, r = 70, 100, 90, 8
    cu, of = np.arange(T + 1), np.where(np.arange(T) % 2, 1, 0)
    for dt in (torch.float16, torch.bfloat16):
        make = lambda shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to("cuda:0").to(dt)   # noqa: E731
        A, B, X, Y = make((3, r, n)), make((3, m, r)), make((T, n)), make((T, m))
        A[2], B[2] = float("nan"), float("inf")                   # not in use
        rows = mb.mdbf_adapter_rows(_ints(torch, cu), _ints(torch, of), 3, T)
        clean = Y.clone()
        mb.mdbf_adapters(rows, [mb.Adapters(A, B)], [X], [clean])
        X2, got = X.clone(), Y.clone()
        X2[5, 3], X2[8] = float("inf"), float("nan")
        mb.mdbf_adapters(rows, [mb.Adapters(A, B)], [X2], [got])
        keep = [t for t in range(T) if t not in (5, 8)]
        assert torch.equal(got[keep], clean[keep]) and not torch.isfinite(got[[5, 8]]).any()


def test_tables_made_by_other_means(gpu):
    """Entries that name no row, no adapter or no place are left out."""
    torch, mb = gpu
    rng = np.random.default_rng(7)
    T, n, m, r = 20, 64, 48, 4
    A, B = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to("cuda:0").bfloat16() for s in ((2, r, n), (2, m, r)))
    X, Y = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to("cuda:0").bfloat16() for s in ((T, n), (T, m)))
    rows = _ints(torch, [3, 1, -1, 99, 7] + [-1] * 15)
    tiles = _ints(torch, [[0, 0, 5, 0], [2, 0, 3, 0], [-1, 0, 3, 0], [1, 30, 2, 0], [1, -4, 9, 0], [0, 0, -3, 0]])
    t = mb.AdapterRows(T, 3, 2, rows=rows, tiles=tiles)
    got = Y.clone()
    mb.mdbf_adapters(t, [mb.Adapters(A, B)], [X], [got])
    of = np.full(T, -1)
    of[[1, 3, 7]] = 0
    changed = (got != Y).any(1).cpu().numpy()
    assert np.array_equal(changed, of == 0)
    want = Y.double().cpu().numpy() + so.adapters(X.double().cpu().numpy(), of, A.double().cpu().numpy(), B.double().cpu().numpy(), None)
    bound = _bound(X.double().cpu().numpy(), of, A.double().cpu().numpy(), B.double().cpu().numpy(), np.ones(2), Y.double().cpu().numpy(), want, "bf16", "bf16")
    assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()


def test_pools_beyond_two_to_the_31_elements(gpu):
    """Adapters far apart: offsets pass 32 bits."""
    torch, mb = gpu
    n, m, r, count = 4096, 16, 64, 8200
    A = torch.zeros((count, r, n), dtype=torch.bfloat16, device="cuda:0")
    B = torch.zeros((count, m, r), dtype=torch.bfloat16, device="cuda:0")
    rng = np.random.default_rng(8)
    used = [0, 8191, 5]
    for a in used:
        A[a] = torch.from_numpy(rng.standard_normal((r, n)).astype(np.float32)).to("cuda:0") * n ** -0.5
        B[a] = torch.from_numpy(rng.standard_normal((m, r)).astype(np.float32)).to("cuda:0")
    X = torch.from_numpy(rng.standard_normal((6, n)).astype(np.float32)).to("cuda:0").bfloat16()
    Y = torch.zeros((6, m), dtype=torch.float32, device="cuda:0")
    of = np.array([8191, 0, 5, 8191, -1, 5])
    rows = _ints(torch, [1, 2, 5, 0, 3, -1])
    tiles = _ints(torch, [[0, 0, 1, 0], [5, 1, 2, 0], [8191, 3, 2, 0]])
    mb.mdbf_adapters(mb.AdapterRows(6, 6, count, rows=rows, tiles=tiles), [mb.Adapters(A, B)], [X], [Y])
    small = {a: i for i, a in enumerate(used)}
    A64, B64 = A[used].double().cpu().numpy(), B[used].double().cpu().numpy()
    of_small = np.array([small.get(a, -1) for a in of])
    x = X.double().cpu().numpy()
    want = so.adapters(x, of_small, A64, B64, None)
    assert (np.abs(Y.double().cpu().numpy() - want) <= _bound(x, of_small, A64, B64, np.ones(3), np.zeros_like(want), want, "bf16", "f32")).all()


def test_wide_projections(gpu):
    """More channels and columns than any chunk, split and row of tiles."""
    _check(gpu, 4, 2, 3, [(70001, 70003, 4)], "bf16", ["f32"], seed=9)
    _check(gpu, 70, 1, 1, [(40000, 16, 33), (40000, 30000, 16)], "f16", ["f16", "f16"], seed=10)


def test_a_step_of_one_row_and_many_adapters(gpu):
    _check(gpu, 1, 500, 1, [(256, 256, 16), (256, 8, 64)], "bf16", ["bf16", "bf16"], seed=11)


@pytest.mark.parametrize("requests,adapters,fresh,first", [(1, 1, 2, 2), (5, 3, 4, 1), (64, 32, 1, 64), (37, 9, 40, 1000), (1024, 100, 3, 77), (1500, 400, 1, 5),
                                                           (500, 100, 300, 9000), (3, 2, 9000, 12345)])
def test_a_step_whose_first_rows_are_no_requests(gpu, requests, adapters, fresh, first):
    """cu begins behind 0, as that of a part of a step's requests does: in one launch and in two."""
    torch, mb = gpu
    rng = np.random.default_rng(requests + first)
    for behind in (0, 7):
        cu, of = _step(rng, requests, adapters, fresh)
        cu = cu + first
        T = int(cu[-1]) + behind
        got = mb.mdbf_adapter_rows(_ints(torch, cu), _ints(torch, of), adapters, T)
        rows, tiles, places = so.adapter_tables(cu.tolist(), of.tolist(), adapters, T, got.tiles.shape[0])
        assert np.array_equal(got.rows.cpu().numpy(), rows)
        assert np.array_equal(got.tiles.cpu().numpy(), tiles) and np.array_equal(got.places.cpu().numpy(), places)


def test_a_workspace_of_a_larger_step(gpu):
    """A program's one workspace, of its largest step, serves every smaller one, though few rows are cut into more parts."""
    torch, mb = gpu
    rng = np.random.default_rng(15)
    n, m, r = 4096, 72, 16
    up = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to("cuda:0").bfloat16()   # noqa: E731
    pool = mb.Adapters(up(2, r, n) * n ** -0.5, up(2, m, r))
    steps = {}
    for T in (600, 200, 66, 9, 1):
        rows = mb.mdbf_adapter_rows(_ints(torch, [0, T]), _ints(torch, [1]), 2, T)
        X, Y = up(T, n), torch.zeros((T, m), dtype=torch.float32, device="cuda:0")
        steps[T] = rows, X, Y, mb.mdbf_adapters_workspace(rows, [pool], [X], [Y])
    sizes = {T: s[3].numel() for T, s in steps.items()}
    assert sizes[200] > sizes[600] // 3                              # (per row: more)
    for most in (600, 200, 66):
        for T in (t for t in steps if t <= most):
            rows, X, Y, _ = steps[T]
            store = torch.full((sizes[most] + 64,), 77, dtype=torch.uint8, device="cuda:0")
            x, a, b = (v.double().cpu().numpy() for v in (X, pool.A, pool.B))
            of = np.full(T, 1)
            want = so.adapters(x, of, a, b, None)
            for workspace in (store[:sizes[most]], store[:T * 16 * 4]):    # and the least that there is: one part
                Y.zero_()
                mb.mdbf_adapters(rows, [pool], [X], [Y], workspace=workspace)
                assert (np.abs(Y.double().cpu().numpy() - want) <= _bound(x, of, a, b, np.ones(2), np.zeros_like(want), want, "bf16", "f32")).all()
            assert (store[sizes[most]:] == 77).all()
            with pytest.raises(mb.MdbfError, match="EWORKSPACE"):
                mb.mdbf_adapters(rows, [pool], [X], [Y], workspace=store[:T * 16 * 4 - 16])


@pytest.mark.parametrize("x_dtype,y_dtype", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("r,below", [(8, 18), (16, 18), (40, 18), (16, 24)])
def test_ranks_far_below_a_rows_largest(gpu, r, below, x_dtype, y_dtype):
    """Columns of B that read only ranks 2^-below of the row's largest inner value.  Inner values are carried to 2^-23 of themselves or (fp16) 2^-38 of the row's
    largest; with the sums' own n steps that leaves results to half a step of their type and some 2^-15."""
    torch, mb = gpu
    rng = np.random.default_rng(r)
    T, n, m = 40, 64, 70
    dt = _dt(torch, x_dtype)
    up = lambda a: torch.from_numpy(a.astype(np.float32)).to("cuda:0").to(dt)                 # noqa: E731
    a = rng.standard_normal((1, r, n))
    a[0, 0] *= 2.0 ** 12
    a[0, 1:] *= 2.0 ** (12 - below)
    b = rng.standard_normal((1, m, r)) * 64
    b[0, :-1, 0] = 0                                                # (the last column reads the largest one)
    A, B, X = up(a), up(b), up(rng.standard_normal((T, n)))
    Y = torch.zeros((T, m), dtype=_dt(torch, y_dtype), device="cuda:0")
    rows = mb.mdbf_adapter_rows(_ints(torch, [0, T]), _ints(torch, [0]), 1, T)
    mb.mdbf_adapters(rows, [mb.Adapters(A, B)], [X], [Y])
    x, a, b = (v.double().cpu().numpy() for v in (X, A[0], B[0]))
    inner, size = x @ a.T, np.abs(x) @ np.abs(a).T
    off = (n + 8) * 2.0 ** -24 * size + 2.0 ** -23 * np.abs(inner) + (2.0 ** -38 * np.abs(inner).max(1, keepdims=True) if x_dtype == "f16" else 0)
    want = inner @ b.T
    bound = (off + 2 * (r + 8) * 2.0 ** -24 * np.abs(inner)) @ np.abs(b).T * (1 + 2.0 ** -7) + HALF[y_dtype] * np.abs(want) + TINY[y_dtype]
    got = Y.double().cpu().numpy()
    assert np.isfinite(got[:, :-1]).all() and (np.abs(got - want) <= bound)[:, :-1].all()
    if y_dtype != "f16":                                            # (the last column is beyond fp16)
        assert (np.abs(got - want) <= bound)[:, -1].all()


@pytest.mark.parametrize("x_dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [1e-37, 1e-30, 1e30])
def test_scales_near_the_ends_of_fp32(gpu, x_dtype, scale):
    """Small inner values with large columns of B, and the other way round: the products stay numbers of full precision."""
    torch, mb = gpu
    rng = np.random.default_rng(16)
    T, n, m, r = 9, 40, 24, 8
    dt = _dt(torch, x_dtype)
    up = lambda a: torch.from_numpy(a.astype(np.float32)).to("cuda:0").to(dt)                 # noqa: E731
    small, large = 2.0 ** -12, 2.0 ** 12
    a, b, x = (small, large, small) if scale < 1 else (large, small, 64.0)
    A, B, X = (up(rng.standard_normal(shape) * f) for shape, f in (((1, r, n), a), ((1, m, r), b), ((T, n), x)))
    Y = torch.zeros((T, m), dtype=torch.float32, device="cuda:0")
    rows = mb.mdbf_adapter_rows(_ints(torch, [0, T]), _ints(torch, [0]), 1, T)
    scales = torch.full((1,), scale, device="cuda:0")
    mb.mdbf_adapters(rows, [mb.Adapters(A, B, scales)], [X], [Y])
    x, a, b, s = (v.double().cpu().numpy() for v in (X, A, B, scales))
    want = so.adapters(x, [0] * T, a, b, s)
    bound = _bound(x, [0] * T, a, b, s, np.zeros_like(want), want, x_dtype, "f32")
    assert np.abs(want).max() < 2.0 ** 127 and (np.abs(Y.double().cpu().numpy() - want) <= bound).all()


def test_an_infinite_inner_value_beside_large_ones(gpu):
    """fp16: an infinity leaves the other inner values of its row within fp16's range, so that the sum is that infinity and no NaN."""
    torch, mb = gpu
    T, n, m, r = 20, 64, 40, 16
    A = torch.full((1, r, n), 60000.0, dtype=torch.float16, device="cuda:0")
    A[0, 3, 5] = float("inf")
    B = -torch.ones((1, m, r), dtype=torch.float16, device="cuda:0")
    B[0, :, 3] = 1.0
    X = torch.ones((T, n), dtype=torch.float16, device="cuda:0")
    X[::2] = -1.0
    Y = torch.zeros((T, m), dtype=torch.float32, device="cuda:0")
    rows = mb.mdbf_adapter_rows(_ints(torch, [0, T]), _ints(torch, [0]), 1, T)
    mb.mdbf_adapters(rows, [mb.Adapters(A, B)], [X], [Y])
    assert (Y[1::2] == float("inf")).all() and (Y[::2] == float("-inf")).all()


@pytest.mark.parametrize("x_dtype,y_dtype", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("r", [2, 8, 16, 24, 64])
def test_inner_values_that_cancel(gpu, r, x_dtype, y_dtype):
    """Whole numbers of 23 bits whose differences are small ones: every sum is exact in 32 bits, and so are the results."""
    torch, mb = gpu
    rng = np.random.default_rng(r)
    T, n, m = 50, 96, 33
    dt = _dt(torch, x_dtype)
    top = 2048 if x_dtype == "f16" else 256                          # whole numbers that the type holds
    x = rng.integers(1, 100, (T, n))
    x[:, n - 1] = rng.integers(1, 12, T)                             # what is left of a pair of ranks
    a = rng.integers(1, top, (1, r, n)) * (2048 // top)
    a[0, :, n - 1] = 0
    a[0, 1::2] = a[0, ::2][:, :n]
    a[0, 1::2, n - 1] = 1
    a[0, ::2, 0] = a[0, 1::2, 0]
    inner = x @ a[0].T
    assert inner.max() < 2 ** 23 and inner.max() > 2 ** 20
    sign = rng.integers(0, 2, (m, r // 2)) * 2 - 1
    b = np.zeros((1, m, r))
    b[0, :, ::2], b[0, :, 1::2] = sign, -sign
    up = lambda v: torch.from_numpy(v.astype(np.float32)).to("cuda:0").to(dt)                 # noqa: E731
    A, B, X = up(a), up(b), up(x)
    assert np.array_equal(A.double().cpu().numpy(), a) and np.array_equal(X.double().cpu().numpy(), x)
    Y = torch.zeros((T, m), dtype=_dt(torch, y_dtype), device="cuda:0")
    rows = mb.mdbf_adapter_rows(_ints(torch, [0, T]), _ints(torch, [0]), 1, T)
    mb.mdbf_adapters(rows, [mb.Adapters(A, B)], [X], [Y])
    want = inner @ b[0].T
    assert np.abs(want).max() <= 12 * r // 2 and np.array_equal(Y.double().cpu().numpy(), torch.from_numpy(want).to(_dt(torch, y_dtype)).double().numpy())
