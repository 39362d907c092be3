"""Attention over the 4-bit cache at the ends of the ranges of types and formats, in every form that a call can take.  Against the 64-bit
oracle; tolerances follow from the arithmetic at each test."""
import numpy as np
import pytest

from oracle import kv_oracle as kvo
from test_gpu_kv import U, attention_tolerance, gpu, rows  # noqa: F401  (gpu: the fixture)
from test_gpu_kv_paths import Path, both_types, every_path

pytestmark = pytest.mark.gpu


@both_types
@every_path
@pytest.mark.parametrize("gap", [12.0, 16.0, 17.0, 17.5, 19.0])
def test_a_long_tail_behind_tokens_of_high_score_and_no_value(gpu, path, dt, gap):
    """Every 50th token has a score `gap` above the others' and values of zero (an attention sink): the result is the tail's, whose
    numerators are e^-gap of the reference's.  Each is rounded by u of itself and in fp16 by 2^-32 of the reference's at most, the
    result by u; scores are off by dz = 2^-20 + (prompts) 1.07 * 2^-14 or 2^-18 of gap, each weight by 2 dz."""
    p = Path(gpu, path, dt, seed=7)
    s = p.s
    rng = np.random.default_rng(7)
    for r, n in enumerate(s.lengths):
        pos = np.arange(n)
        sink = pos % 50 == 0
        kc, vc = np.zeros((n, s.Hkv, s.d // 2), np.uint8), rng.integers(0, 8, (n, s.Hkv, s.d // 2, 2), dtype=np.uint8)
        kc[sink, :, 0] = 4                                # 2.0 in channel 0
        vc = vc[..., 0] | vc[..., 1] << 4
        vc[sink] = 0
        ksc, vsc = np.full((n, s.Hkv, s.d // 32), 127, np.uint8), np.full((n, s.Hkv, s.d // 32), 137, np.uint8)
        for view, x in zip(s.views, (kc, vc, ksc, vsc)):
            view[s.table_host[r, pos // s.P], :, pos % s.P] = x
        s.k[r], s.v[r] = kvo.values(kvo.unpack(kc), ksc), kvo.values(kvo.unpack(vc), vsc)
    s.upload()
    s.q.zero_()
    s.q[:, :, 0] = 1.0
    got = p.run(scale=gap / 2).double().cpu().numpy()
    q = np.zeros((1, s.d))
    q[0, 0] = 1
    dz = gap * (2.0 ** -20 + (0 if not p.name.startswith("prompts") else 1.07 * 2.0 ** (-14 if dt == "bf16" else -18)))
    u = U[dt] / 2
    for r, (n, f) in enumerate(zip(s.lengths, s.fresh)):
        for h in range(s.Hq if f else 0):
            k, v = s.k[r][:, h // (s.Hq // s.Hkv)], s.v[r][:, h // (s.Hq // s.Hkv)]
            pos = n - f + np.arange(f)
            ref, mag, den = kvo.attention(np.repeat(q, f, 0), k, v, pos, True, p.window, gap / 2)
            tol = (2.02 * u + 2.02 * dz) * mag + 2.0 ** -25
            if dt == "f16":
                seen = np.maximum(np.minimum(pos + 1, p.window or n), 0)
                tol += (seen * 2.0 ** -32 * np.abs(v).max(initial=0) / den)[:, None]
            err = np.abs(got[s.cu[r]:s.cu[r] + f, h] - ref)
            assert (err <= tol).all(), (r, h, (err / tol).max())


BEYOND = {"f16": [141, 160, 200, 254, 255], "bf16": [253, 254, 255]}      # scale bytes of numbers that the type does not have


@both_types
@every_path
def test_scale_bytes_beyond_the_type_are_nan(gpu, path, dt):
    """In a key for the rows that see it, in a value for its block of their channels; no other bit changes, with all codes at their
    largest."""
    p = Path(gpu, path, dt, seed=8)
    s = p.s
    clean = p.run().double().cpu().numpy()
    keys, values, i = [], [], 0         # (request, token, kv head, block)
    for r, (n, f) in enumerate(zip(s.lengths, s.fresh)):
        for tok in sorted({0, n // 2, n - 1 - f // 2, n - 2, n - 1} & set(range(n))):
            (keys if i % 3 == 0 else values).append((r, tok, (r + i) % s.Hkv, (r + 2 * i) % (s.d // 32)))
            i += 1
    for part, where in ((2, keys), (3, values)):
        for i, (r, tok, head, block) in enumerate(where):
            page, at = s.table_host[r, tok // s.P], tok % s.P
            s.views[part][page, head, at, block] = BEYOND[dt][i % len(BEYOND[dt])]
            s.views[part - 2][page, head, at, 16 * block:16 * block + 16] = 0xF7 if i % 2 else 0x77
    s.upload()
    got = p.run().double().cpu().numpy()
    for r, (n, f) in enumerate(zip(s.lengths, s.fresh)):
        for i in range(f):
            pos = n - f + i
            sees = lambda tok: tok <= pos and (not p.window or tok > pos - p.window)
            for h in range(s.Hq):
                head, want = h // (s.Hq // s.Hkv), np.zeros(s.d, bool)
                for b, tok, kv_head, block in keys:
                    if b == r and kv_head == head and sees(tok):
                        want[:] = True
                for b, tok, kv_head, block in values:
                    if b == r and kv_head == head and sees(tok):
                        want[32 * block:32 * block + 32] = True
                t = s.cu[r] + i
                assert np.array_equal(np.isnan(got[t, h]), want), (r, i, h)
                assert np.array_equal(got[t, h][~want], clean[t, h][~want]), (r, i, h)


@pytest.mark.parametrize("dt,largest", [("f16", 140), ("bf16", 252)])
@pytest.mark.parametrize("y_dt", ["f16", "bf16", "f32"])
def test_every_scale_byte_read_back(gpu, dt, largest, y_dt):
    torch, mb = gpu
    cache = mb.KVCache(16, 1, 64, 16, dt)
    views = kvo.page_views(cache.buffer.cpu().numpy(), 16, 1, 16, 64)
    rng = np.random.default_rng(9)
    codes, scales = rng.integers(0, 256, (2, 256, 32)).astype(np.uint8), np.arange(256, dtype=np.uint8)
    slot = rng.permutation(256)
    for part in (0, 1):
        views[part][slot // 16, 0, slot % 16] = codes[part]
        views[part + 2][slot // 16, 0, slot % 16] = scales[:, None]
    pool = np.concatenate([x.reshape(16, 1, -1) for x in views], 2).reshape(-1)
    cache = mb.KVCache(16, 1, 64, 16, dt, buffer=torch.from_numpy(pool).cuda())
    ttype = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[y_dt]
    out = [torch.empty((256, 1, 64), dtype=ttype, device="cuda:0") for _ in range(2)]
    for y, c in zip(mb.mdbf_kv_read(cache, torch.from_numpy(slot).cuda(), out=out), codes):
        y = y.double().cpu().numpy()[:, 0]
        assert np.isnan(y[largest + 1:]).all()
        known = slice({"f16": 104, "bf16": 2}[dt], largest + 1)
        with np.errstate(over="ignore"):
            want = kvo.values(kvo.unpack(c), np.repeat(scales[:, None], 2, 1))[known]
            if y_dt == "f16" and dt == "bf16":
                want = want.astype(np.float16).astype(np.float64)
        assert np.array_equal(y[known], want)


@both_types
@every_path
@pytest.mark.parametrize("times,exact", [(1, True), (32, True), (1000, True), (1, False), (32, False)])
def test_queries_with_channels_far_beyond_the_others(gpu, path, dt, times, exact):
    """One channel of 32 that many times the others, where all keys are zero: what is left of the scores must be that of the other
    channels.  Exact queries: the tolerance of few rows in every form; else with the rounding that prompts have (test_gpu_kv_paths.py)."""
    torch, _ = gpu
    p = Path(gpu, path, dt, seed=10)
    s = p.s
    q = np.random.default_rng(10).standard_normal((p.T, s.Hq, s.d))
    q[:, :, 3::32] *= times
    s.q, s.q64 = rows(torch, q, dt)
    s.views[0][..., 1::16] &= 0x0F                       # channels 3, 35, ...: the odd half of bytes 1, 17, ...
    for r in range(len(s.lengths)):
        s.k[r][..., 3::32] = 0
    s.upload()
    out = torch.full(s.q.shape, 5.0, dtype=s.q.dtype, device="cuda:0")
    got = p.run(out=out, exact_queries=exact).double().cpu().numpy()
    assert (got[p.real:] == 5.0).all()
    e = 0.0 if exact or not p.name.startswith("prompts") else 1.07 * 2.0 ** (-14 if dt == "bf16" else -18)
    for r, (n, f) in enumerate(zip(s.lengths, s.fresh)):
        at, pos = slice(s.cu[r], s.cu[r] + f), n - f + np.arange(f)
        for h in range(s.Hq if f else 0):
            x, k, v = s.q64[at, h], s.k[r][:, h // (s.Hq // s.Hkv)], s.v[r][:, h // (s.Hq // s.Hkv)]
            ref, mag, den = kvo.attention(x, k, v, pos, True, p.window, s.d ** -0.5)
            tol = attention_tolerance(dt, ref, mag, den, x, k, v, s.d ** -0.5) + n * 2.0 ** -126 * np.abs(v).max(initial=0)
            if e and n:
                dz = s.d ** -0.5 * e * np.abs(x).reshape(f, -1, 32).max(2) @ np.abs(k).reshape(n, -1, 32).sum(2).max(0)
                tol = tol + (np.exp(2 * dz) - 1)[:, None] * mag
            err = np.abs(got[at, h] - ref)
            assert (err <= tol).all(), (r, h, (err / tol).max())


@both_types
@every_path
def test_exact_queries_that_are_not_finite_and_lie_apart(gpu, path, dt):
    """NaN in the rows with such queries, the other rows' bits as they were; the same bits from strides that no wide access fits."""
    p = Path(gpu, path, dt, seed=11)
    s = p.s
    clean = p.run(scale=-0.2, exact_queries=True).double().cpu().numpy()
    seen = np.concatenate([n - f + np.arange(f) >= 0 for n, f in zip(s.lengths, s.fresh)])
    q = p.torch.zeros((p.T, s.Hq * s.d + 3), dtype=s.q.dtype, device="cuda:0")[:, :s.Hq * s.d].unflatten(1, (s.Hq, s.d))
    q.copy_(s.q)
    bad = {(t, h) for t in range(0, p.real, 7) for h in range(t % 3, s.Hq, 3)}
    for i, (t, h) in enumerate(sorted(bad)):
        q[t, h, (5 * i) % s.d] = [float("nan"), float("inf"), -float("inf")][i % 3]
    got = p.run(scale=-0.2, exact_queries=True, q=q).double().cpu().numpy()
    for t in range(p.real):
        for h in range(s.Hq):
            if (t, h) in bad and seen[t]:
                assert np.isnan(got[t, h]).all(), (t, h)
            else:
                assert np.array_equal(got[t, h], clean[t, h]), (t, h)
