"""mdbf_add_norm against 64 bits.  Bounds: h is one fp32 addition; 1 / sqrt of the mean is rounded once (the mean is fp64) and y is two more products,
so y is off by at most 4 steps of 2^-24 before its own rounding of half a step of its type (subnormals: half of the smallest)."""
import numpy as np
import pytest

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # half a step, relative
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}    # half of the smallest number
F32 = 4 * 2.0 ** -24


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2512_24545_amd import binding as mb
    mb.lib()
    return torch, mb


def _rows(torch, rng, T, n, dtype, pad, scale=1.0):
    dt = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    wide = torch.full((T, n + pad), float("nan"), dtype=dt, device="cuda:0")
    wide[:, :n] = torch.from_numpy((rng.standard_normal((T, n)) * scale).astype(np.float32)).to("cuda:0").to(dt)
    return wide[:, :n]


def _close(got, want, dtype, more=F32):
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= (HALF[dtype] + more) * np.abs(want) + TINY[dtype]).all(), float((err / np.abs(want)).max())


WIDTHS = [1, 5, 8, 31, 64, 300, 512, 513, 1601, 2048, 2056, 4096, 5000, 11008, 16384, 16385, 40001, 65536]


@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("x,h,y", [("bf16", "bf16", "bf16"), ("f16", "f32", "f16"), ("f32", None, "bf16"), ("bf16", "f32", "f32"), ("f16", "f16", "f32"), ("f32", "f32", "f16")])
def test_widths_and_types(gpu, n, x, h, y):
    torch, mb = gpu
    rng = np.random.default_rng(n)
    T, pad = 5, n % 3
    X = _rows(torch, rng, T, n, x, pad)
    H = None if h is None else _rows(torch, rng, T, n, h, 2 * pad, 3.0)
    W = torch.from_numpy((1 + 0.2 * rng.standard_normal(n)).astype(np.float32)).to("cuda:0")
    Y, Hout, S = mb.mdbf_add_norm(X, H, W, 1e-5, y_dtype=y)
    want, sums = so.add_norm(X.double().cpu().numpy(), None if H is None else H.double().cpu().numpy(), W.double().cpu().numpy(), float(np.float32(1e-5)))
    _close(Y, want, y)
    assert S is None and (h is None) == (Hout is None)
    if h is not None:
        # one addition in fp32, then one rounding to the stream's type
        _close(Hout, sums, h, 2.0 ** -24)
        assert torch.equal(Hout, (X.float() + H.float()).to(H.dtype))


@pytest.mark.parametrize("T", [1, 2, 3, 4, 7, 1000])
def test_row_counts_and_short_rows(gpu, T):
    torch, mb = gpu
    rng = np.random.default_rng(T)
    for n in (24, 512, 4096):
        X = _rows(torch, rng, T, n, "bf16", 8)
        Y, _, _ = mb.mdbf_add_norm(X, eps=0.0)
        _close(Y, so.add_norm(X.double().cpu().numpy(), None, None, 0.0)[0], "bf16")


@pytest.mark.parametrize("n", [1, 30, 32, 33, 500, 4096, 5001, 20000, 65536])
@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_eight_bits(gpu, n, group, x):
    torch, mb = gpu
    rng = np.random.default_rng(n + group)
    T = 6
    X, H = _rows(torch, rng, T, n, x, 1), _rows(torch, rng, T, n, "f32", 3)
    if n > 40:
        H[2, 40] = 900.0                                           # one far beyond the others
        H[3], X[3] = 0.0, 0.0                                      # a row of zeros
        H[4, :32], X[4, :32] = 0.0, 0.0                            # a block of zeros
    Y, Hout, S = mb.mdbf_add_norm(X, H, y_dtype="e4m3", scale_group=group)
    assert Y.dtype == torch.float8_e4m3fn and Y.shape == (T, n)
    y, _ = so.add_norm(X.double().cpu().numpy(), H.double().cpu().numpy(), None, float(np.float32(1e-6)))
    if group:
        bytes_ = S.cpu().numpy().astype(np.int64)
        assert S.dtype == torch.uint8 and np.array_equal(bytes_, so.block_scales(y))
        scale = np.repeat(2.0 ** (bytes_ - 127.0), 32, axis=1)[:, :n]
    else:
        top = np.abs(y).max(1, keepdims=True)
        scale = S.double().cpu().numpy()
        assert S.shape == (T, 1) and (np.abs(scale - np.where(top > 0, top / 448, 1)) <= 6 * 2.0 ** -24 * np.maximum(scale, 1e-30)).all()
    q = Y.float().double().cpu().numpy()
    # half a step of four significant bits, the fp32 steps in front of it (y, the scale and the quotient), and half of the smallest number
    assert (np.abs(q * scale - y) <= (2.0 ** -4 + 8 * 2.0 ** -24) * np.abs(y) + 2.0 ** -10 * scale).all()
    # and the very number but where y / scale lies on a border to those steps
    near = so.e4m3(y / scale)
    assert np.mean(near != q) <= 1e-3 + (1 if n * T < 1000 else 0)


def test_values_that_are_not_finite(gpu):
    torch, mb = gpu
    rng = np.random.default_rng(1)
    X = _rows(torch, rng, 5, 200, "bf16", 0)
    X[1, 70], X[2, 3], X[3, 199] = float("nan"), float("inf"), float("-inf")
    clean = [0, 4]
    Y, _, _ = mb.mdbf_add_norm(X)
    assert torch.isnan(Y[1]).all() and torch.isnan(Y[2, 3]) and torch.isnan(Y[3, 199]) and torch.isfinite(Y[clean]).all()
    for group in (0, 32):
        Y, _, S = mb.mdbf_add_norm(X, y_dtype="e4m3", scale_group=group)
        bad = torch.isnan(Y.float())
        if group:
            assert (S[1] == 255).all() and S[2, 0] == 255 and (S[2, 1:] != 255).all() and S[3, 6] == 255 and (S[clean] != 255).all()
            assert bad[1].all() and bad[2, :32].all() and not bad[2, 32:].any() and bad[3, 192:].all() and not bad[3, :192].any()
        else:
            assert torch.isnan(S[1:4]).all() and bad[1:4].all()
        assert not bad[clean].any()


def test_extremes_of_magnitude(gpu):
    torch, mb = gpu
    X = torch.full((4, 512), 1e-30, device="cuda:0")
    X[1], X[2], X[3] = 3e38, 1e-44, 1e19
    Y, _, _ = mb.mdbf_add_norm(X, eps=0.0)
    # squares do not leave fp64.  (A row of equal values x has 1 / x, off by half a step, times x, rounded once more: 1 to two halves of a step of
    # 2^-23, within F32.  1 / 1e-44 of the third row is beyond fp32.)
    want = so.add_norm(X.double().cpu().numpy(), None, None, 0.0)[0]
    assert (np.abs(Y.double().cpu().numpy() - want)[[0, 1, 3]] <= F32).all()
    _, _, S = mb.mdbf_add_norm(X * 0, y_dtype="e4m3", scale_group=32)
    assert (S == 1).all()


def test_in_place_and_outputs_given(gpu):
    torch, mb = gpu
    rng = np.random.default_rng(2)
    for n in (100, 4096, 11008):
        X, H = _rows(torch, rng, 9, n, "bf16", 8), _rows(torch, rng, 9, n, "bf16", 0)
        Y, Hout, _ = mb.mdbf_add_norm(X, H)
        x2, h2 = X.clone(), H.clone()
        y2, hout2, _ = mb.mdbf_add_norm(x2, h2, residual_out=h2, out=x2)
        assert y2.data_ptr() == x2.data_ptr() and torch.equal(x2, Y) and torch.equal(h2, Hout)
        around = torch.full((9, n + 16), 7.0, dtype=torch.bfloat16, device="cuda:0")
        mb.mdbf_add_norm(X, H, out=around[:, :n])
        assert torch.equal(around[:, :n], Y) and (around[:, n:] == 7).all()
        q = torch.full((9, n + 5), 3, dtype=torch.uint8, device="cuda:0")
        s = torch.full((9, -(-n // 32) + 3), 9, dtype=torch.uint8, device="cuda:0")
        mb.mdbf_add_norm(X, H, out=q.view(torch.float8_e4m3fn)[:, :n], scales=s[:, :-(-n // 32)], scale_group=32)
        Y8, _, S8 = mb.mdbf_add_norm(X, H, y_dtype="e4m3", scale_group=32)
        assert torch.equal(q[:, :n], Y8.view(torch.uint8)) and (q[:, n:] == 3).all()
        assert torch.equal(s[:, :-(-n // 32)], S8) and (s[:, -(-n // 32):] == 9).all()


def test_rows_beyond_two_to_the_31_elements(gpu):
    """Offsets of rows far apart pass 32 bits."""
    torch, mb = gpu
    store = torch.empty((2 ** 31 + 5000) * 2, dtype=torch.uint8, device="cuda:0").view(torch.bfloat16)
    X = torch.as_strided(store, (3, 1024), (2 ** 30, 1))
    rng = np.random.default_rng(3)
    X.copy_(torch.from_numpy(rng.standard_normal((3, 1024)).astype(np.float32)).to("cuda:0").to(torch.bfloat16))
    Y, _, _ = mb.mdbf_add_norm(X)
    _close(Y, so.add_norm(X.double().cpu().numpy(), None, None, float(np.float32(1e-6)))[0], "bf16")


def test_views_of_every_kind(gpu):
    """One row or one channel of something larger, rows that are not side by side: results are the same, and rows of their own."""
    torch, mb = gpu
    rng = np.random.default_rng(4)
    store = _rows(torch, rng, 12, 600, "f32", 0)
    for x in (store[3:4, 100:228], store[::3, :128], store[:, 4:5], store[5:6, 8:9], store[2:3], store[:, :0 + 1]):
        if x.data_ptr() % 16:
            x = torch.nn.functional.pad(x, (0, 7))[:, :x.shape[1]]
        y, h, _ = mb.mdbf_add_norm(x, x)
        want, sums = so.add_norm(x.double().cpu().numpy(), x.double().cpu().numpy(), None, float(np.float32(1e-6)))
        _close(y, want, "f32")
        assert torch.equal(h, x + x) and y.shape == h.shape == x.shape
    with pytest.raises(AssertionError):
        mb.mdbf_add_norm(store.T)
    with pytest.raises(mb.MdbfError):
        mb.mdbf_add_norm(store[:1].expand(12, 600))


def test_scales_that_round_to_a_coarse_number(gpu):
    """Rows whose largest over 448 has few bits: what passes 448 scales is 448, as the nearest such number, and no NaN."""
    torch, mb = gpu
    step = 2.0 ** -149
    tops = [100, 223, 225, 300, 448, 500, 600, 671, 673, 900, 1100, 5000, 100000]
    n = 96
    rng = np.random.default_rng(5)
    y = np.array([[t * step * (-1) ** i * (1 - i / n) for i in range(n)] for t in tops])
    # (a row of ones and its mean: y is the weight, a row of weights per call)
    for t, row in zip(tops, y):
        w = torch.from_numpy(row.astype(np.float32)).to("cuda:0")
        q, _, s = mb.mdbf_add_norm(torch.ones((3, n), device="cuda:0"), weight=w, eps=0.0, y_dtype="e4m3")
        scale = np.float32(t * step) / np.float32(448)
        scale = np.float32(1) if scale == 0 else scale
        assert (s.cpu().numpy() == scale).all()
        want = so.e4m3(w.double().cpu().numpy() / float(scale))
        assert np.array_equal(q.float().cpu().numpy(), np.broadcast_to(want, (3, n))), t


def test_more_rows_than_a_launch_has(gpu):
    """A launch ends at 2^32 threads: 2^26 rows of a wave each."""
    torch, mb = gpu
    T = 2 ** 26 + 5
    X = torch.randn(T, device="cuda:0").bfloat16().view(T, 1)
    X[X == 0] = 1
    Y, _, _ = mb.mdbf_add_norm(X, eps=0.0)
    assert torch.equal(Y, X.sign())


def test_more_rows_of_a_workgroup_each_than_a_launch_has(gpu):
    """2^23 rows of four waves: around the border between launches, and at the end."""
    torch, mb = gpu
    T, n = 2 ** 23 + 3, 520
    X = torch.empty((T, n), dtype=torch.bfloat16, device="cuda:0").normal_()
    Y, _, S = mb.mdbf_add_norm(X, y_dtype="e4m3")
    for rows in (slice(0, 5), slice(2 ** 23 - 3, T)):
        again, _, scales = mb.mdbf_add_norm(X[rows], y_dtype="e4m3")
        assert torch.equal(Y[rows].view(torch.uint8), again.view(torch.uint8)) and torch.equal(S[rows], scales)
    assert (S > 0).all() and (S < 1).all()
