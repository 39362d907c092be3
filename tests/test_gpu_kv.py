"""Attention block over the 4-bit paged cache on the GPU, through the binding, against the 64-bit oracle.

Tolerances follow from the arithmetic.  Slots, codes, scales and what they stand for are exact.  Norm and rotation: fp32
(at most some 30 roundings of 2^-24 of the head's largest magnitude: 4e-6 of it) and one rounding to the output's type.
Attention: numerators rounded once to the cache's type (u = 2^-8 or 2^-11 of each at most; in fp16 at least 2^-25), the result once
more, scores and exponentials in fp32 (an error of z of 2^-20 of the sum of the score's magnitudes, 2^-21 of each numerator)."""
import numpy as np
import pytest

from oracle import kv_oracle as kvo

pytestmark = pytest.mark.gpu

U = {"f16": 2.0 ** -10, "bf16": 2.0 ** -7, "f32": 2.0 ** -23}     # spacing of the types at 1 (torch.finfo's eps); a rounding errs by half of it


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2512_24545_amd import binding as mb
    mb.lib()
    return torch, mb


def tdt(torch, name):
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[name]


def typed(torch, x, name):
    """A numpy array as a device tensor of the type, and the 64-bit values it then holds."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(tdt(torch, name)).to("cuda:0")
    return t, t.double().cpu().numpy()


def rows(torch, x, name, pad=0):
    """The same as rows of heads, `pad` elements more between rows."""
    T, H, d = x.shape
    wide = torch.zeros((T, H * d + pad), dtype=tdt(torch, name), device="cuda:0")
    t, x64 = typed(torch, x, name)
    view = wide[:, :H * d].unflatten(1, (H, d))
    view.copy_(t)
    return view, x64


def ints(torch, v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda:0")


# ---- block tables and slot maps --------------------------------------------------------------------
def check_slots(gpu, cached, fresh, P, width, free_extra, tokens_extra, taken=3, seed=0, want_status=0, table_pad=0):
    torch, mb = gpu
    rng = np.random.default_rng(seed)
    n = len(cached)
    held = [max(0, -(-c // P)) for c in cached]
    total = sum(held)
    need = sum(max(0, -(-(c + f) // P) - -(-c // P)) for c, f in zip(cached, fresh) if c >= 0 and f >= 0)
    perm = rng.permutation(total + taken + need + free_extra + 50)
    table = np.full((n, width + table_pad), -7, np.int64)
    at = 0
    for r in range(n):
        m = min(held[r], width)
        table[r, :m] = perm[at:at + m]
        at += m
    free = perm[total:total + taken + need + free_extra]
    tokens = max(1, sum(f for f in fresh if f > 0) + tokens_extra)
    want = kvo.slots([int(c) for c in cached], [int(f) for f in fresh], table[:, :width], free, taken, P, tokens)
    assert want["status"] == want_status
    dev = ints(torch, table)
    got = mb.mdbf_kv_slots(ints(torch, cached), ints(torch, fresh), dev[:, :width], ints(torch, free), ints(torch, [taken]), P, tokens)
    for name in ("lengths", "cu", "slots", "positions"):
        assert np.array_equal(getattr(got, name).cpu().numpy(), want[name]), name
    assert got.status.item() == want["status"] and got.taken.item() == want["taken"]
    assert np.array_equal(dev[:, :width].cpu().numpy(), want["table"])
    assert (dev[:, width:] == -7).all()


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1023, 1024, 1025, 2500])
def test_slots_of_a_decode_step(gpu, n):
    rng = np.random.default_rng(n)
    check_slots(gpu, rng.integers(0, 200, n), np.ones(n, int), 16, 14, 0, 0, table_pad=n % 3)


@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("n,most", [(1, 1), (1, 5000), (1, 9000), (7, 3000), (300, 40), (1100, 30)])
def test_slots_of_prompts(gpu, P, n, most):
    rng = np.random.default_rng(P + n)
    fresh = rng.integers(0, most + 1, n)
    fresh[0] = most
    cached = rng.integers(0, 3 * P, n) * rng.integers(0, 2, n)
    check_slots(gpu, cached, fresh, P, -(-(3 * P + most) // P) + 1, 2, 5 * (n % 2), seed=n)


@pytest.mark.parametrize("cached,fresh", [([0], [0]), ([16], [0]), ([0, 0, 0], [0, 1, 0]), ([15, 16, 17], [1, 1, 1]), ([0, 32], [16, 16])])
def test_slots_at_page_borders(gpu, cached, fresh):
    check_slots(gpu, cached, fresh, 16, 4, 0, 2)


@pytest.mark.parametrize("cached,fresh,width,free_extra,tokens_extra,status", [
    ([5, -1, 3], [1, 1, 1], 4, 9, 0, 1), ([5, 1, 3], [1, -2, 1], 4, 9, 9, 1), ([60, 3], [5, 1], 4, 9, 0, 2), ([60, 3], [4, 1], 4, 0, -1, 4),
    ([60, 31], [4, 2], 4, -1, 0, 8), ([60, -31], [5, 90], 4, -30, -60, 13 - 8 + 2)])
def test_slots_refuse_a_step_as_a_whole(gpu, cached, fresh, width, free_extra, tokens_extra, status):
    if status == 7:      # a bad length, a narrow table and too few tokens at once
        cached, fresh, free_extra, tokens_extra, status = [60, -31], [5, 90], 9, -91, 7
    check_slots(gpu, cached, fresh, 16, width, free_extra, tokens_extra, want_status=status)


def test_slots_refuse_long_steps_and_lengths_beyond_32_bits(gpu):
    check_slots(gpu, [100, 3], [9000, 9000], 16, 2000, -1, 0, want_status=8)
    check_slots(gpu, [2 ** 31 - 5, 3], [9, 1], 256, 4, 4, 0, want_status=1)


def test_slots_go_on_in_place(gpu):
    """A decode loop: lengths and taken of one step are the next one's inputs; the map stays that of a request's own pages."""
    torch, mb = gpu
    rng = np.random.default_rng(1)
    n, P, width = 5, 16, 8
    cached, taken, table, free = ints(torch, [0] * n), ints(torch, [0]), ints(torch, np.full((n, width), -1)), ints(torch, rng.permutation(60))
    o = mb.KVSlots(n, 40)
    o.taken = taken
    seen = {}
    for step in range(30):
        fresh = rng.integers(0, 9, n)
        mb.mdbf_kv_slots(cached, ints(torch, fresh), table, free, taken, P, 40, out=o)
        cached.copy_(o.lengths)
        if o.status.item():
            break
        cu, slots, pos = (getattr(o, x).cpu().numpy() for x in ("cu", "slots", "positions"))
        for r in range(n):
            for t in range(cu[r], cu[r + 1]):
                assert slots[t] not in seen
                seen[slots[t]] = (r, pos[t])
    tb, ln = table.cpu().numpy(), cached.cpu().numpy()
    assert len(seen) == ln.sum() > 100
    for slot, (r, p) in seen.items():
        assert tb[r, p // P] * P + p % P == slot


# ---- tokens in and out ------------------------------------------------------------------------------
def awkward(rng, shape):
    """Normal values of many sizes, with zeros, blocks of zeros and ties among them."""
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-3, 3, shape[:-1] + (1,)))
    x[rng.random(shape) < 0.05] = 0
    flat = x.reshape(-1, 32)
    flat[rng.random(len(flat)) < 0.1] = 0
    ties = rng.random(len(flat)) < 0.2
    flat[ties] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, -0.25, -2.5, -6], (int(ties.sum()), 32))
    return x


@pytest.mark.parametrize("x_dt,kv_dt", [("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "f16"), ("f16", "bf16")])
@pytest.mark.parametrize("T,H,d,P,pad", [(1, 1, 64, 16, 0), (5, 3, 64, 32, 3), (17, 2, 128, 16, 8), (33, 8, 128, 256, 0), (9, 5, 256, 64, 1), (70, 1, 256, 128, 24)])
def test_append_and_read(gpu, x_dt, kv_dt, T, H, d, P, pad):
    torch, mb = gpu
    rng = np.random.default_rng(T + H + d)
    pages = T // P + 3
    pool = torch.full((pages * H * P * (d + d // 16) + 5,), 0xA5, dtype=torch.uint8, device="cuda:0")
    cache = mb.KVCache(pages, H, d, P, kv_dt, buffer=pool)
    k, k64 = rows(torch, awkward(rng, (T, H, d)), x_dt, pad)
    v, v64 = rows(torch, awkward(rng, (T, H, d)), x_dt, pad * 2)
    slots = rng.permutation(pages * P)[:T].astype(np.int64)
    skipped = rng.random(T) < 0.2
    given = np.where(skipped, rng.choice([-1, pages * P, 2 ** 40, -2 ** 40], T), slots)
    mb.mdbf_kv_append(cache, k, v, torch.from_numpy(given).cuda())
    views = kvo.page_views(pool[:-5].cpu().numpy(), pages, H, P, d)
    want = [np.full_like(x, 0xA5) for x in views]
    for part, x64 in enumerate((k64, v64)):
        codes, scales = kvo.quantise(x64, kv_dt)
        for t in np.flatnonzero(~skipped):
            want[part][slots[t] // P, :, slots[t] % P] = codes[t, :, 0::2] | (codes[t, :, 1::2] << 4)
            want[part + 2][slots[t] // P, :, slots[t] % P] = scales[t]
    for part in (0, 1):
        same = kvo.values(kvo.unpack(want[part]), want[part + 2]) == kvo.values(kvo.unpack(views[part]), views[part + 2])
        assert same.all()                   # (a zero's sign is its own matter)
        assert np.array_equal(views[part + 2], want[part + 2])
    assert (pool[-5:] == 0xA5).all()
    for y_dt in ("f16", "bf16", "f32"):
        outs = [rows(torch, np.full((T, H, d), 7.0), y_dt, pad)[0] for _ in range(2)]
        got = mb.mdbf_kv_read(cache, torch.from_numpy(given).cuda(), out=outs)
        for part, y in enumerate(got):
            exact = kvo.values(kvo.unpack(want[part]), want[part + 2])
            for t in range(T):
                ref = exact[slots[t] // P, :, slots[t] % P] if not skipped[t] else np.zeros((H, d))
                if y_dt == "f16" and kv_dt == "bf16":
                    ref = ref.astype(np.float16).astype(np.float64)
                assert np.array_equal(y[t].double().cpu().numpy(), ref)


@pytest.mark.parametrize("x_dt,kv_dt", [("f32", "bf16"), ("f32", "f16"), ("f16", "f16"), ("bf16", "bf16")])
def test_append_at_the_ends_of_the_range(gpu, x_dt, kv_dt):
    torch, mb = gpu
    big = {"f16": 65504.0, "bf16": 3.38e38, "f32": 3.4e38}[x_dt]
    small = {"f16": 2.0 ** -24, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}[x_dt]
    x = np.zeros((8, 1, 64))
    x[0, 0, 0], x[1, 0, :] = big, big
    x[2, 0, 0], x[2, 0, 1] = small, -3 * small
    x[3, 0, 0], x[3, 0, 40] = np.nan, 1.0
    x[4, 0, 33], x[4, 0, 2] = np.inf, 5.0
    x[5, 0, 33] = -np.inf
    x[6, 0, 0], x[6, 0, 1] = 1.75 * 2.0 ** 15 if x_dt == "f16" else 1.75 * 2.0 ** 100, 1.0
    k, k64 = rows(torch, x, x_dt)
    cache = mb.KVCache(1, 1, 64, 16, kv_dt)
    slots = torch.arange(8, device="cuda:0")
    mb.mdbf_kv_append(cache, k, k, slots)
    got = mb.mdbf_kv_read(cache, slots, out=[torch.empty((8, 1, 64), device="cuda:0") for _ in range(2)])
    ref = kvo.values(*kvo.quantise(k64, kv_dt))
    for y in got:
        assert np.array_equal(y.double().cpu().numpy(), ref, equal_nan=True)
    sixteen = mb.mdbf_kv_read(cache, slots)
    for y in sixteen:
        assert np.array_equal(y.double().cpu().numpy(), ref, equal_nan=True)    # every stored value is a number of the type


def test_offsets_beyond_32_bits(gpu):
    """Append, read and attention in a pool of more than 4 GiB, on its last pages."""
    torch, mb = gpu
    H, d, P = 8, 128, 64
    pages = (1 << 32) // (H * P * 136) + 9
    cache = mb.KVCache(pages, H, d, P, "bf16", buffer=torch.empty(pages * H * P * 136, dtype=torch.uint8, device="cuda:0"))
    rng = np.random.default_rng(5)
    T = 100
    k, k64 = rows(torch, rng.standard_normal((T, H, d)), "bf16")
    v, v64 = rows(torch, rng.standard_normal((T, H, d)), "bf16")
    pos = np.arange(T)
    table = np.array([[pages - 1, pages - 2]])
    slots = torch.from_numpy(table[0, pos // P] * P + pos % P).cuda()
    mb.mdbf_kv_append(cache, k, v, slots)
    kq, vq = (kvo.values(*kvo.quantise(x, "bf16")) for x in (k64, v64))
    got = mb.mdbf_kv_read(cache, slots)
    assert np.array_equal(got[0].double().cpu().numpy(), kq) and np.array_equal(got[1].double().cpu().numpy(), vq)
    q, q64 = rows(torch, rng.standard_normal((1, H, d)), "bf16")
    out = mb.mdbf_kv_attention(cache, q, ints(torch, table), ints(torch, [0, 1]), ints(torch, [T]), 1, T).double().cpu().numpy()
    for h in range(H):
        ref, mag, den = kvo.attention(q64[:, h], kq[:, h], vq[:, h], [T - 1], True, 0, d ** -0.5)
        assert (np.abs(out[:, h] - ref) <= attention_tolerance("bf16", ref, mag, den, q64[:, h], kq[:, h], vq[:, h], d ** -0.5)).all()


# ---- norm and rotation ------------------------------------------------------------------------------
def rope_table(rows_, rot, base=1e4):
    a = np.arange(rows_)[:, None] * base ** (-np.arange(rot // 2) * 2.0 / rot)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def rope_tolerance(y_dt, ref):
    return U[y_dt] / 2 * np.abs(ref) + 4e-6 * np.abs(ref).max(-1, keepdims=True) + (2.0 ** -25 if y_dt == "f16" else 1e-38)


@pytest.mark.parametrize("x_dt,y_dt", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f16"), ("f16", "bf16")])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,inter,pad,norm", [
    (1, 1, 1, 64, 64, False, 0, "qk"), (7, 4, 2, 64, 32, True, 1, "qk"), (3, 5, 1, 128, 128, False, 0, "qk"), (64, 32, 8, 128, 96, False, 8, "q"),
    (5, 3, 3, 128, 16, True, 0, "k"), (9, 2, 1, 256, 256, False, 3, ""), (6, 7, 1, 256, 48, False, 0, "qk"), (4, 2, 2, 128, 0, False, 0, "qk"),
    (5000, 2, 1, 64, 64, True, 0, "qk")])
def test_norm_and_rotation(gpu, x_dt, y_dt, T, Hq, Hkv, d, rot, inter, pad, norm):
    torch, mb = gpu
    rng = np.random.default_rng(T + d + rot)
    q, q64 = rows(torch, rng.standard_normal((T, Hq, d)) * 3, x_dt, pad)
    k, k64 = rows(torch, rng.standard_normal((T, Hkv, d)) / 3, x_dt, 2 * pad)
    qw = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32) if "q" in norm else None
    kw = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32) if "k" in norm else None
    table = rope_table(50, rot) if rot else None
    pos = rng.integers(0, 50, T)
    if T > 4:
        pos[2] = -1
    up = lambda x: None if x is None else torch.from_numpy(x).cuda()
    qo, _ = rows(torch, np.full((T, Hq, d), 9.0), y_dt, pad)
    ko, _ = rows(torch, np.full((T, Hkv, d), 9.0), y_dt, pad + 1)
    got = mb.mdbf_qk_norm_rope(q, k, up(table), ints(torch, pos), up(qw), up(kw), 1e-5, inter, q_out=qo, k_out=ko)
    for y, x64, w in ((got[0], q64, qw), (got[1], k64, kw)):
        ref = kvo.norm_rope(x64, w, table, pos if rot else None, 1e-5, inter)
        assert (np.abs(y.double().cpu().numpy() - ref) <= rope_tolerance(y_dt, ref)).all()
    new = mb.mdbf_qk_norm_rope(q, k, up(table), ints(torch, pos), up(qw), up(kw), 1e-5, inter, y_dtype=y_dt)
    assert torch.equal(new[0], got[0]) and torch.equal(new[1], got[1])


def test_norm_and_rotation_in_place(gpu):
    torch, mb = gpu
    rng = np.random.default_rng(2)
    qkv = torch.from_numpy(rng.standard_normal((37, (6 + 2 + 2) * 128))).cuda().bfloat16()
    heads = qkv.unflatten(1, (10, 128))
    q, k = heads[:, :6], heads[:, 6:8]
    table, pos = torch.from_numpy(rope_table(64, 128)).cuda(), ints(torch, rng.integers(0, 64, 37))
    w = torch.from_numpy((1 + 0.1 * rng.standard_normal(128)).astype(np.float32)).cuda()
    want = mb.mdbf_qk_norm_rope(q, k, table, pos, w, w)
    before = qkv.clone()
    mb.mdbf_qk_norm_rope(q, k, table, pos, w, w, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, 8 * 128:], before[:, 8 * 128:])


def test_positions_beyond_the_table_and_values_that_are_not_finite(gpu):
    torch, mb = gpu
    rng = np.random.default_rng(3)
    q, q64 = rows(torch, rng.standard_normal((4, 2, 128)), "f32")
    k, _ = rows(torch, rng.standard_normal((4, 1, 128)), "f32")
    q[1, 1, 5], q[2, 0, 7] = float("nan"), float("inf")
    table = rope_table(10, 64)
    w = torch.ones(128, device="cuda:0")
    got, _ = mb.mdbf_qk_norm_rope(q, k, torch.from_numpy(table).cuda(), ints(torch, [3, 3, 3, 10]), w, w)
    got = got.cpu().numpy()
    assert np.isnan(got[3, :, :64]).all() and np.isfinite(got[3, :, 64:]).all()
    assert np.isnan(got[1, 1]).all() and np.isfinite(got[1, 0]).all() and np.isnan(got[2, 0, 7]) and np.isfinite(got[2, 1]).all()
    ref = kvo.norm_rope(q64[:1], np.ones(128), table, [3], 1e-6, False)
    assert (np.abs(got[:1] - ref) <= rope_tolerance("f32", ref)).all()


@pytest.mark.parametrize("x_dt,y_dt,kv_dt", [("bf16", "bf16", "bf16"), ("f32", "f16", "f16"), ("f32", "f32", "bf16"), ("f16", "f16", "bf16")])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,inter", [(1, 2, 1, 64, 64, False), (19, 7, 1, 128, 128, False), (300, 4, 4, 128, 64, True), (40, 3, 2, 256, 16, False)])
def test_one_launch_writes_the_same_bytes_as_two(gpu, x_dt, y_dt, kv_dt, T, Hq, Hkv, d, rot, inter):
    torch, mb = gpu
    rng = np.random.default_rng(T)
    qkv, _ = rows(torch, rng.standard_normal((T, Hq + 2 * Hkv, d)), x_dt)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    table, pos = torch.from_numpy(rope_table(500, rot)).cuda(), rng.integers(0, 500, T)
    P, pages = 16, T // 16 + 2
    slots = rng.permutation(pages * P)[:T]
    if T > 3:
        pos[1], slots[1], slots[3] = -1, -1, -1          # padding; a token that is not cached
    slots = torch.from_numpy(slots).cuda()
    w = torch.from_numpy((1 + 0.2 * rng.standard_normal(d)).astype(np.float32)).cuda()
    one, two = (mb.KVCache(pages, Hkv, d, P, kv_dt) for _ in range(2))
    q1, none = mb.mdbf_qk_norm_rope(q, k, table, ints(torch, pos), w, w, 1e-6, inter, y_dtype=y_dt, cache=one, v=v, slots=slots)
    q2, k2 = mb.mdbf_qk_norm_rope(q, k, table, ints(torch, pos), w, w, 1e-6, inter, y_dtype=y_dt)
    if x_dt == y_dt:
        mb.mdbf_kv_append(two, k2, v, slots)
    else:       # the values are of x_dtype, the keys of y_dtype: one call each, the other half to be overwritten
        mb.mdbf_kv_append(two, k2, k2, slots)
        keep = mb.KVCache(pages, Hkv, d, P, kv_dt)
        mb.mdbf_kv_append(keep, v, v, slots)
        a, b = two.buffer.view(pages, Hkv, -1), keep.buffer.view(pages, Hkv, -1)
        a[:, :, P * d // 2:P * d], a[:, :, P * d + P * d // 32:] = b[:, :, P * d // 2:P * d], b[:, :, P * d + P * d // 32:]
    assert none is None and torch.equal(q1, q2) and torch.equal(one.buffer, two.buffer)
    k_out = torch.empty_like(k2)
    q3, k3 = mb.mdbf_qk_norm_rope(q, k, table, ints(torch, pos), w, w, 1e-6, inter, y_dtype=y_dt, cache=one, v=v, slots=slots, k_out=k_out)
    assert torch.equal(k3, k2) and torch.equal(one.buffer, two.buffer)


# ---- attention --------------------------------------------------------------------------------------
def attention_tolerance(dt, ref, mag, den, q, k, v, scale):
    u = U[dt] / 2
    size = (np.abs(q) @ np.abs(k).T).max() * scale if len(k) else 0.0      # of a score's terms
    vmax = np.nanmax(np.abs(v)) if len(v) else 0.0
    tiny = len(k) * 2.0 ** -25 * vmax / den[:, None] if dt == "f16" else 0.0
    floor = 2.0 ** -25 if dt == "f16" else 1e-38
    return (u + 2.0 ** -20 * size + 2.0 ** -20) * mag * 1.01 + u * np.abs(ref) * 1.01 + tiny + floor


class Step:
    """A pool with the keys and values of some requests in scattered pages; every byte that no request holds is garbage
    (scale bytes that mean NaN among it)."""

    def __init__(self, gpu, lengths, fresh, Hq, Hkv, d, P, dt, seed=0, q_pad=0, table_pad=0, v_scale=1.0):
        torch, mb = self.torch, self.mb = gpu
        rng = np.random.default_rng(seed)
        self.lengths, self.fresh, self.Hq, self.Hkv, self.d, self.P, self.dt = lengths, fresh, Hq, Hkv, d, P, dt
        held = [-(-n // P) for n in lengths]
        pages = sum(held) + 3
        perm = rng.permutation(pages)
        self.width = max(held + [1]) + 1
        table = np.full((len(lengths), self.width + table_pad), -1)
        pool = rng.integers(0, 256, pages * Hkv * P * (d + d // 16), dtype=np.uint8)
        views = kvo.page_views(pool, pages, Hkv, P, d)
        for s in views[2:]:
            s[rng.random(s.shape) < 0.5] = 255
        self.k, self.v, at = [], [], 0
        lo = 104 if dt == "f16" else 100
        for r, n in enumerate(lengths):
            table[r, :held[r]] = perm[at:at + held[r]]
            at += held[r]
            kc, vc = (rng.integers(0, 256, (n, Hkv, d // 2), dtype=np.uint8) for _ in range(2))
            ksc, vsc = (rng.integers(123, 127, (n, Hkv, d // 32)).astype(np.uint8) for _ in range(2))
            pos = np.arange(n)
            for view, x in zip(views, (kc, vc, ksc, vsc)):
                view[table[r, pos // P], :, pos % P] = x
            self.k.append(kvo.values(kvo.unpack(kc), ksc))
            self.v.append(kvo.values(kvo.unpack(vc), vsc))
        self.pool_host, self.pages, self.views, self.table_host = pool, pages, views, table
        self.q, self.q64 = rows(torch, rng.standard_normal((max(1, sum(fresh)) + 2, Hq, d)), dt, q_pad)
        self.cu = np.concatenate([[0], np.cumsum(fresh)])
        self.upload()

    def upload(self):
        torch, mb = self.torch, self.mb
        self.cache = mb.KVCache(self.pages, self.Hkv, self.d, self.P, self.dt, buffer=torch.from_numpy(self.pool_host).cuda())
        self.table = ints(self.torch, self.table_host)[:, :self.width]

    def run(self, causal=True, window=0, scale=None, max_fresh=None, max_length=None, out=None, q=None, **kw):
        return self.mb.mdbf_kv_attention(self.cache, self.q if q is None else q, self.table, ints(self.torch, self.cu), ints(self.torch, self.lengths),
                                         max_fresh or max(self.fresh + [1]), max_length or max(self.lengths + [1]), scale, causal, window, out=out, **kw)

    def check(self, causal=True, window=0, scale=None, **kw):
        sc = self.d ** -0.5 if scale is None else scale
        out = self.torch.full(self.q.shape, 5.0, dtype=self.q.dtype, device="cuda:0")
        got = self.run(causal, window, scale, out=out, **kw).double().cpu().numpy()
        G = self.Hq // self.Hkv
        for r, (n, f) in enumerate(zip(self.lengths, self.fresh)):
            at, pos = slice(self.cu[r], self.cu[r] + f), n - f + np.arange(f)
            for h in range(self.Hq):
                q, k, v = self.q64[at, h], self.k[r][:, h // G], self.v[r][:, h // G]
                ref, mag, den = kvo.attention(q, k, v, pos, causal, window, sc)
                if not f:
                    continue
                err, tol = np.abs(got[at, h] - ref), attention_tolerance(self.dt, ref, mag, den, q, k, v, sc)
                assert (err <= tol).all(), (r, h, np.nanmax(err - tol), np.nanmax(err / tol))
        assert (got[self.cu[-1]:] == 5.0).all()       # rows behind the last request's stay
        return got


LENGTHS = [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d,P", [(1, 1, 64, 16), (6, 2, 64, 32), (4, 4, 128, 16), (8, 2, 128, 64), (16, 1, 128, 256), (20, 1, 128, 32),
                                        (34, 2, 64, 16), (2, 1, 256, 16), (9, 3, 256, 128)])
def test_single_tokens(gpu, dt, Hq, Hkv, d, P):
    Step(gpu, LENGTHS, [1] * len(LENGTHS), Hq, Hkv, d, P, dt, seed=Hq + d).check()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d,P", [(2, 2, 64, 16), (4, 1, 128, 32), (3, 1, 128, 16), (14, 2, 64, 64), (2, 1, 256, 32)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 17), (True, 64), (True, 1000)])
def test_prompts(gpu, dt, Hq, Hkv, d, P, causal, window):
    lengths = [1, 2, 16, 33, 64, 100, 200, 257, 40, 130]
    fresh = [1, 2, 16, 33, 50, 1, 130, 257, 3, 65]
    Step(gpu, lengths, fresh, Hq, Hkv, d, P, dt, seed=d + window).check(causal, window)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("fresh", [[5], [300]])
def test_requests_without_tokens_and_tokens_that_see_nothing(gpu, dt, fresh):
    """Lengths of zero, no new tokens, more new tokens than the request is long: rows that see nothing are zeros."""
    for causal in (True, False):
        for window in ((0, 3) if causal else (0,)):
            s = Step(gpu, [0, 40, 3, 0, 64], [2, 0] + fresh + [0, 1], 4, 2, 128, 16, dt)
            got = s.check(causal, window)
            assert not got[:2].any()
            if causal:
                assert not got[2:2 + fresh[0] - 3].any()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("n,Hq,Hkv,d,P", [(1, 4, 2, 128, 64), (3, 8, 1, 64, 256), (2, 1, 1, 256, 16)])
@pytest.mark.parametrize("fresh", [1, 3])
@pytest.mark.parametrize("window", [0, 1500])
def test_long_caches(gpu, dt, n, Hq, Hkv, d, P, fresh, window):
    lengths = [7001, 2048, 33][:n]
    Step(gpu, lengths, [fresh] * n, Hq, Hkv, d, P, dt, seed=n).check(window=window)


@pytest.mark.parametrize("fresh", [1, 2, 150])
def test_strides(gpu, fresh):
    for q_pad in (1, 4, 8):
        s = Step(gpu, [200, 170], [fresh, 1], 4, 2, 128, 16, "bf16", q_pad=q_pad, table_pad=3)
        want = s.check()
        wide = s.torch.full((s.q.shape[0], 4 * 128 + q_pad + 1), 5.0, dtype=s.q.dtype, device="cuda:0")
        out = wide[:, :4 * 128].unflatten(1, (4, 128))
        s.run(out=out)
        assert np.array_equal(out.double().cpu().numpy(), want) and (wide[:, 4 * 128:] == 5.0).all()


@pytest.mark.parametrize("fresh", [[1, 1, 1], [3, 40, 1], [70, 200, 150]])
def test_sizes_are_hints(gpu, fresh):
    """A request with more new tokens or a longer cache than the call was told is served as well."""
    s = Step(gpu, [90, 2600, 150], fresh, 6, 2, 64, 16, "bf16")
    s.check()
    s.check(max_fresh=1, max_length=1)
    s.check(max_fresh=1)
    s.check(max_length=40)
    s.check(max_fresh=1000, max_length=100000)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("fresh,lengths", [([1, 1], [100, 3000]), ([70, 130], [100, 200])])
def test_large_scores(gpu, dt, fresh, lengths):
    """Scores of some hundred: the softmax is all but one-hot, and nothing overflows."""
    Step(gpu, lengths, fresh, 4, 2, 128, 16, dt).check(scale=3.0)


@pytest.mark.parametrize("fresh", [1, 70])
def test_negative_scale(gpu, fresh):
    Step(gpu, [100, 333], [fresh, 1], 4, 2, 64, 16, "bf16").check(scale=-0.3)


def not_finite_case(gpu, dt, fresh, lengths, seed, window=0):
    """Blocks of keys and values that are NaN reach the rows that see them, and no other."""
    s = Step(gpu, lengths, fresh, 4, 2, 128, 16, dt, seed=seed)
    clean = s.run(window=window).double().cpu().numpy()
    rng = np.random.default_rng(seed)
    for r, n in enumerate(lengths):
        f = fresh[r]
        for part, tok, head, block in ((2, n - 1, 0, 1), (3, max(0, n - 2), 1, 2), (3, n - 1, 1, 0), (3, n // 2, 0, 3)):
            before = s.views[part][s.table_host[r, tok // 16], head, tok % 16, block]
            s.views[part][s.table_host[r, tok // 16], head, tok % 16, block] = 255
            s.upload()
            got = s.run(window=window).double().cpu().numpy()
            pos = n - f + np.arange(f)
            hit = (pos >= tok) & ((tok > pos - window) if window else True)
            for t in range(len(clean)):
                row = t - s.cu[r]
                for h in range(4):
                    want = np.zeros(128, bool)
                    if 0 <= row < f and hit[row] and h // 2 == head:
                        want[slice(None) if part == 2 else slice(32 * block, 32 * block + 32)] = True
                    if t < s.cu[-1]:
                        assert np.array_equal(np.isnan(got[t, h]), want), (r, part, t, h)
                        assert np.array_equal(got[t, h][~want], clean[t, h][~want])
            s.views[part][s.table_host[r, tok // 16], head, tok % 16, block] = before


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("fresh,lengths,window", [([1, 1], [50, 33], 0), ([4, 1], [5, 129], 0), ([40, 9], [60, 9], 0), ([3, 20], [70, 40], 6),
                                                  ([140], [150], 0), ([140], [150], 20), ([1], [2500], 0)])
def test_blocks_that_are_not_finite(gpu, dt, fresh, lengths, window):
    not_finite_case(gpu, dt, fresh, lengths, sum(lengths), window)


@pytest.mark.parametrize("fresh", [1, 100])
def test_queries_that_are_not_finite(gpu, fresh):
    s = Step(gpu, [120, 130], [fresh, 1], 4, 2, 128, 16, "bf16")
    clean = s.run().double().cpu().numpy()
    s.q[0, 1, 5], s.q[fresh, 2, 9] = float("nan"), float("inf")
    got = s.run().double().cpu().numpy()
    for t in range(fresh + 1):
        for h in range(4):
            if (t, h) in ((0, 1), (fresh, 2)):
                assert np.isnan(got[t, h]).all()
            else:
                assert np.array_equal(got[t, h], clean[t, h])


@pytest.mark.parametrize("fresh", [1, 80])
def test_pages_outside_the_pool_read_as_nan(gpu, fresh):
    s = Step(gpu, [100, 90, 95], [fresh] * 3, 4, 2, 128, 16, "f16")
    clean = s.run().double().cpu().numpy()
    s.table_host[1, 0] = s.pages
    s.table_host[2, 0] = -1
    s.upload()
    got = s.run().double().cpu().numpy()
    n = s.cu[-1]
    assert np.array_equal(got[:fresh], clean[:fresh]) and np.isnan(got[fresh:n]).all()


def test_lengths_that_buffers_do_not_hold_are_cut(gpu):
    """Lengths beyond the table's row, new tokens beyond T and negative counts: reads and writes stay inside."""
    torch, mb = gpu
    s = Step(gpu, [96, 96], [1, 1], 2, 1, 64, 16, "bf16")
    s.width = 6
    s.upload()
    want = s.run()
    out = torch.full(s.q.shape, 5.0, dtype=s.q.dtype, device="cuda:0")
    mb.mdbf_kv_attention(s.cache, s.q, s.table, ints(torch, [0, 1, 2]), ints(torch, [2 ** 31 - 1, 97]), 1, 96, out=out)
    assert torch.equal(out[:2], want[:2]) and (out[2:] == 5).all()
    out.fill_(5.0)
    mb.mdbf_kv_attention(s.cache, s.q, s.table, ints(torch, [-3, -9, 2 ** 31 - 1]), ints(torch, [-5, 96]), 1, 96, out=out)
    assert out.isfinite().all()
    mb.mdbf_kv_attention(s.cache, s.q, s.table, ints(torch, [2 ** 31 - 1, -2 ** 31, 7]), ints(torch, [96, 96]), 1, 96, out=out)
    torch.cuda.synchronize()


@pytest.mark.parametrize("fresh,lengths", [(1, [5000, 700]), (90, [100, 200])])
def test_same_bits_again_on_another_stream_and_in_a_graph(gpu, fresh, lengths):
    torch, mb = gpu
    s = Step(gpu, lengths, [fresh, 1], 8, 2, 128, 64, "bf16")
    ws = mb.mdbf_kv_attention_workspace(s.cache, 8, 2, s.q.shape[0], fresh, max(lengths))
    table, cu, ln = s.table, ints(torch, s.cu), ints(torch, s.lengths)
    call = lambda out, stream=None: mb.mdbf_kv_attention(s.cache, s.q, table, cu, ln, fresh, max(lengths), out=out, workspace=ws, stream=stream)
    outs = [torch.zeros_like(s.q) for _ in range(4)]
    call(outs[0])
    call(outs[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(outs[2], side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(outs[3])
    for _ in range(3):
        outs[3].zero_()
        if ws is not None:
            ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[3], outs[0])
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_a_step_in_a_graph(gpu):
    """Slots, norm and rotation with the append, attention: captured once, replayed over a growing cache, each replay against
    the same calls made eagerly."""
    torch, mb = gpu
    rng = np.random.default_rng(9)
    n, Hq, Hkv, d, P, width, steps = 3, 4, 2, 128, 16, 6, 40
    table = torch.from_numpy(rope_table(200, d)).cuda()
    w = torch.ones(d, device="cuda:0")
    qkv = [torch.from_numpy(rng.standard_normal((n, Hq + 2 * Hkv, d))).cuda().bfloat16() for _ in range(steps)]

    class Loop:
        def __init__(self):
            self.x = torch.zeros_like(qkv[0])
            self.cached, self.fresh, self.taken = ints(torch, [0, 5, 0]), ints(torch, [1, 1, 1]), ints(torch, [1])
            self.table, self.free = ints(torch, np.full((n, width), -1)), ints(torch, np.arange(20)[::-1].copy())
            self.table[1, 0] = 19
            self.cache, self.o = mb.KVCache(20, Hkv, d, P), mb.KVSlots(n, n)
            self.o.taken = self.taken
            self.out = torch.zeros((n, Hq, d), dtype=torch.bfloat16, device="cuda:0")
            self.ws = mb.mdbf_kv_attention_workspace(self.cache, Hq, n, n, 1, width * P)

        def step(self):
            o = mb.mdbf_kv_slots(self.cached, self.fresh, self.table, self.free, self.taken, P, n, out=self.o)
            q, _ = mb.mdbf_qk_norm_rope(self.x[:, :Hq], self.x[:, Hq:Hq + Hkv], table, o.positions, w, w, cache=self.cache, v=self.x[:, Hq + Hkv:], slots=o.slots)
            mb.mdbf_kv_attention(self.cache, q, self.table, o.cu, o.lengths, 1, width * P, out=self.out, workspace=self.ws)
            self.cached.copy_(o.lengths)

    eager, graphed = Loop(), Loop()
    warm = Loop()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graphed.step()
    for x in qkv:
        eager.x.copy_(x)
        graphed.x.copy_(x)
        eager.step()
        g.replay()
        torch.cuda.synchronize()
        assert eager.o.status.item() == 0
        assert torch.equal(eager.out, graphed.out) and torch.equal(eager.table, graphed.table) and torch.equal(eager.cache.buffer, graphed.cache.buffer)
        assert eager.out.isfinite().all() and eager.out.abs().amax().item() > 0
    assert eager.cached.tolist() == [steps, steps + 5, steps]
