"""Attention over the 4-bit cache in every form that a call can take, each by name (mdbf_kv_attention_kernel): few query rows and prompts, whole,
n-th row tiles and shares, with and without priorities, for every head size.  The data are small: the bounds max_fresh and
max_length and rows behind the last request's (T) steer the choice.  Against the 64-bit oracle.

Tolerances: those of test_gpu_kv.py, and for prompts, whose queries are rounded to e = 1.07 * 2^-14 (bf16) or 2^-18 (fp16) of the largest of each 32
channels, an error of a score of dz = scale * sum over blocks (e * largest |q| * sum |k|) at most, which changes a weight by a
factor of exp(2 dz) at most.  Numerators below fp32's normal range may be zero: 2^-126 of the largest value per token."""
import numpy as np
import pytest

from oracle import kv_oracle as kvo
from test_gpu_kv import Step, attention_tolerance, gpu, ints, rows  # noqa: F401  (gpu: the fixture)

pytestmark = pytest.mark.gpu

FRESH = {3: [150, 40, 60], 16: [17, 1, 9, 0, 5, 17, 2, 3, 11, 17, 1, 1, 0, 16, 8, 4]}
LENGTHS = {3: [330, 33, 90], 16: [17 + 300, 1, 40, 70, 2, 17, 130, 3 + 64, 11 + 53, 200, 0, 64, 0, 16, 95, 129]}

# head size, name, q heads, kv heads, requests, T, max_fresh, max_length, window, page size
PATHS = [
    (64, "few rows", 4, 2, 16, 114, 1, 500, 0, 16),
    (64, "few rows, shares", 4, 2, 16, 114, 17, 2000, 0, 32),
    (64, "few rows, shares", 16, 16, 16, 114, 17, 2000, 0, 64),
    (64, "prompts", 4, 2, 3, 500, 150, 500, 0, 16),
    (64, "prompts", 4, 2, 16, 114, 17, 2000, 130, 64),
    (64, "prompts, n-th row tiles", 4, 2, 16, 114, 150, 1000, 0, 32),
    (64, "prompts, n-th row tiles", 4, 2, 16, 114, 150, 500, 130, 128),
    (64, "prompts, shares", 4, 2, 16, 114, 150, 200000, 0, 16),
    (64, "prompts, shares", 7, 1, 3, 252, 200, 200000, 0, 64),
    (128, "few rows", 4, 2, 16, 114, 17, 1000, 0, 64),
    (128, "few rows", 4, 2, 16, 114, 17, 2000, 130, 16),
    (128, "few rows, shares", 4, 2, 16, 114, 17, 3000, 0, 32),
    (128, "few rows, shares", 16, 16, 16, 114, 17, 3000, 0, 128),
    (128, "prompts", 6, 2, 3, 1000, 150, 500, 0, 32),
    (128, "prompts", 4, 2, 3, 500, 150, 1000, 130, 64),
    (128, "prompts, n-th row tiles", 4, 2, 3, 1500, 1000, 500, 0, 16),
    (128, "prompts, n-th row tiles", 4, 2, 3, 500, 400, 2000, 130, 32),
    (128, "prompts, products first", 16, 16, 16, 1500, 150, 5000, 0, 64),
    (128, "prompts, n-th row tiles, products first", 64, 4, 3, 1000, 1000, 8000, 0, 16),
    (128, "prompts, shares", 6, 2, 3, 1500, 200, 3000, 0, 16),
    (128, "prompts, shares, products first", 4, 2, 16, 114, 150, 200000, 0, 256),
    (128, "prompts, shares, products first", 7, 1, 3, 252, 200, 200000, 0, 32),
    (256, "few rows", 4, 2, 16, 114, 17, 1000, 0, 16),
    (256, "few rows, shares", 4, 2, 16, 114, 17, 2000, 0, 64),
    (256, "few rows, shares", 16, 16, 16, 114, 17, 2000, 0, 32),
    (256, "prompts", 4, 2, 16, 1500, 17, 1000, 0, 64),
    (256, "prompts", 4, 2, 16, 1000, 17, 2000, 130, 16),
    (256, "prompts, n-th row tiles", 6, 2, 3, 1500, 1000, 500, 0, 32),
    (256, "prompts, n-th row tiles", 4, 2, 3, 1500, 1000, 2000, 130, 256),
    (256, "prompts, shares", 4, 2, 16, 114, 150, 200000, 0, 16),
    (256, "prompts, shares", 7, 1, 3, 252, 200, 200000, 0, 64),
]
every_path = pytest.mark.parametrize("path", PATHS, ids=lambda p: "%d, %s, %d on %d, %d" % (p[:5]))
both_types = pytest.mark.parametrize("dt", ["f16", "bf16"])


class Path:
    def __init__(self, gpu, path, dt, seed=0, q_pad=0, table_pad=0):
        d, self.name, Hq, Hkv, n, self.T, self.max_fresh, self.max_length, self.window, P = path
        self.torch, self.mb = gpu
        self.s = s = Step(gpu, LENGTHS[n], FRESH[n], Hq, Hkv, d, P, dt, seed=seed + d, table_pad=table_pad)
        s.q, s.q64 = rows(self.torch, np.random.default_rng(seed + d + 1).standard_normal((self.T, Hq, d)), dt, q_pad)
        self.real = int(s.cu[-1])

    def run(self, scale=None, causal=True, out=None, **kw):
        s = self.s
        bounds = (self.max_fresh, self.max_length, causal, self.window if causal else 0)
        assert self.mb.mdbf_kv_attention_kernel(s.cache, s.Hq, len(s.lengths), self.T, *bounds) == self.name
        return s.run(causal, bounds[3], scale, self.max_fresh, self.max_length, out, **kw)

    def check(self, scale=None, causal=True, out=None, **kw):
        s = self.s
        d, G, sc = s.d, s.Hq // s.Hkv, s.d ** -0.5 if scale is None else scale
        if out is None:
            out = self.torch.full(s.q.shape, 5.0, dtype=s.q.dtype, device="cuda:0")
        got = self.run(scale, causal, out, **kw).double().cpu().numpy()
        assert (got[self.real:] == 5.0).all()
        e = 1.07 * (2.0 ** -14 if s.dt == "bf16" else 2.0 ** -18) if self.name.startswith("prompts") else 0.0
        for r, (n, f) in enumerate(zip(s.lengths, s.fresh)):
            at, pos = slice(s.cu[r], s.cu[r] + f), n - f + np.arange(f)
            for h in range(s.Hq if f else 0):
                q, k, v = s.q64[at, h], s.k[r][:, h // G], s.v[r][:, h // G]
                ref, mag, den = kvo.attention(q, k, v, pos, causal, self.window if causal else 0, sc)
                tol = attention_tolerance(s.dt, ref, mag, den, q, k, v, abs(sc)) + n * 2.0 ** -126 * np.abs(v).max(initial=0)
                if e and n:
                    dz = abs(sc) * e * np.abs(q).reshape(f, -1, 32).max(2) @ np.abs(k).reshape(n, -1, 32).sum(2).max(0)
                    tol = tol + (np.exp(2 * dz) - 1)[:, None] * mag
                err = np.abs(got[at, h] - ref)
                assert (err <= tol).all(), (r, h, np.nanmax(err - tol), np.nanmax(err / tol))
        return got


@both_types
@every_path
def test_results(gpu, path, dt):
    Path(gpu, path, dt).check()


@both_types
@every_path
def test_rows_that_lie_apart(gpu, path, dt):
    """Strides that no wide access fits: the same bits."""
    p = Path(gpu, path, dt)
    want = p.check()
    for pad in (1, 4):
        p = Path(gpu, path, dt, q_pad=pad, table_pad=3)
        s = p.s
        wide = p.torch.full((p.T, s.Hq * s.d + pad + 2), 5.0, dtype=s.q.dtype, device="cuda:0")
        out = wide[:, :s.Hq * s.d].unflatten(1, (s.Hq, s.d))
        p.run(out=out)
        assert np.array_equal(out.double().cpu().numpy(), want) and (wide[:, s.Hq * s.d:] == 5.0).all()


@both_types
@every_path
def test_scales(gpu, path, dt):
    """Negative ones, and scores of some hundred, where the softmax is all but one-hot."""
    p = Path(gpu, path, dt, seed=1)
    p.check(scale=-0.3)
    p.check(scale=3.0)


@pytest.mark.parametrize("path", [p for p in PATHS if not p[8]], ids=lambda p: "%d, %s, %d on %d, %d" % (p[:5]))
def test_rows_that_see_everything(gpu, path):
    p = Path(gpu, path, "bf16", seed=2)
    s = p.s
    name = p.mb.mdbf_kv_attention_kernel(s.cache, s.Hq, len(s.lengths), p.T, p.max_fresh, p.max_length, False)
    assert name.startswith(p.name.split(",")[0])
    p.name = name
    p.check(causal=False)


@both_types
@every_path
def test_what_a_row_does_not_see_does_not_change_its_bits(gpu, path, dt):
    """Later tokens with large keys and values, earlier ones than the window has, and other rows' queries."""
    p = Path(gpu, path, dt, seed=6)
    s = p.s
    clean = p.run().double().cpu().numpy()
    rng = np.random.default_rng(6)
    changed = []
    for r, (n, f) in enumerate(zip(s.lengths, s.fresh)):
        for tok in sorted({n - 1, n - 1 - f // 3, n - 1 - f // 2, 1 if p.window else n - 1} & set(range(n))):
            changed.append((r, tok))
            for part in range(4):
                to = s.views[part][s.table_host[r, tok // s.P], :, tok % s.P]
                to[:] = rng.integers(0, 256, to.shape) if part < 2 else rng.integers(128, 132, to.shape)
    s.upload()
    big = {(t, h) for t in range(0, p.real, 5) for h in range(t % 3, s.Hq, 3)}
    for t, h in big:
        s.q[t, h] *= 16
    got = p.run().double().cpu().numpy()
    same = 0
    for r, (n, f) in enumerate(zip(s.lengths, s.fresh)):
        for i in range(f):
            pos = n - f + i
            if any(b == r and tok <= pos and (not p.window or tok > pos - p.window) for b, tok in changed):
                continue
            for h in range(s.Hq):
                if (s.cu[r] + i, h) not in big:
                    same += 1
                    assert np.array_equal(got[s.cu[r] + i, h], clean[s.cu[r] + i, h]), (r, i, h)
    assert same > p.real * s.Hq // 10


@both_types
@every_path
def test_queries_that_are_not_finite(gpu, path, dt):
    p = Path(gpu, path, dt, seed=3)
    s = p.s
    clean = p.run().double().cpu().numpy()
    seen = np.concatenate([n - f + np.arange(f) >= 0 for n, f in zip(s.lengths, s.fresh)])
    bad = {(t, h) for t in range(0, p.real, 7) for h in range(t % 3, s.Hq, 3)}
    for i, (t, h) in enumerate(sorted(bad)):
        s.q[t, h, (5 * i) % s.d] = [float("nan"), float("inf"), -float("inf")][i % 3]
    got = p.run().double().cpu().numpy()
    for t in range(p.real):
        for h in range(s.Hq):
            if (t, h) in bad and seen[t]:
                assert np.isnan(got[t, h]).all(), (t, h)
            else:
                assert np.array_equal(got[t, h], clean[t, h]), (t, h)


@both_types
@every_path
def test_blocks_that_are_not_finite(gpu, path, dt):
    """NaN in a key reaches the rows that see it, in a value its block of their channels; no other bit changes."""
    p = Path(gpu, path, dt, seed=4)
    s = p.s
    clean = p.run().double().cpu().numpy()
    G = s.Hq // s.Hkv
    keys, values = [], []               # (request, token, kv head, block)
    for r, n in enumerate(s.lengths):
        for i, tok in enumerate(sorted({0, n // 3, n - 2, n - 1} & set(range(n)))):
            (keys if i % 2 else values).append((r, tok, (r + i) % s.Hkv, (r + 2 * i) % (s.d // 32)))
    for part, where in ((2, keys), (3, values)):
        for r, tok, head, block in where:
            s.views[part][s.table_host[r, tok // s.P], head, tok % s.P, block] = 255
    s.upload()
    got = p.run().double().cpu().numpy()
    for r, (n, f) in enumerate(zip(s.lengths, s.fresh)):
        for i in range(f):
            pos = n - f + i
            sees = lambda tok: tok <= pos and (not p.window or tok > pos - p.window)
            for h in range(s.Hq):
                want = np.zeros(s.d, bool)
                for b, tok, head, block in keys:
                    if b == r and head == h // G and sees(tok):
                        want[:] = True
                for b, tok, head, block in values:
                    if b == r and head == h // G and sees(tok):
                        want[32 * block:32 * block + 32] = True
                t = s.cu[r] + i
                assert np.array_equal(np.isnan(got[t, h]), want), (r, i, h)
                assert np.array_equal(got[t, h][~want], clean[t, h][~want]), (r, i, h)


@every_path
def test_the_same_bits_again_from_a_graph_and_on_another_stream(gpu, path):
    """Whatever the workspace holds; on a named stream also without one."""
    torch, mb = gpu
    p = Path(gpu, path, "bf16", seed=5)
    s = p.s
    bounds = (p.max_fresh, p.max_length, True, p.window)
    ws = mb.mdbf_kv_attention_workspace(s.cache, s.Hq, len(s.lengths), p.T, *bounds)
    assert (ws is None) == (min(p.max_length, p.window or p.max_length) <= 1024)
    want = p.run(workspace=ws)[:p.real]
    for byte in (0, 255, 127):
        if ws is not None:
            ws.fill_(byte)
        assert torch.equal(p.run(workspace=ws)[:p.real], want)
    table, cu, lengths = s.table, ints(torch, s.cu), ints(torch, s.lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = mb.mdbf_kv_attention(s.cache, s.q, table, cu, lengths, p.max_fresh, p.max_length, window=p.window, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out[:p.real], want)
    g, out = torch.cuda.CUDAGraph(), torch.zeros_like(s.q)
    with torch.cuda.graph(g):
        mb.mdbf_kv_attention(s.cache, s.q, table, cu, lengths, p.max_fresh, p.max_length, window=p.window, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:p.real], want)
