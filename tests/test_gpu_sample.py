"""mdbf_sample against the definition in 64 bits: tokens equal, shares to the rounding of their type.  A token could differ only where the
drawn number falls on an edge between two tokens to 1e-9 of the mass, which has a chance of 1e-4 over all rows here; rows are made from seeds."""
import numpy as np
import pytest

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -24        # a share is a quotient of 64-bit sums, rounded once to fp32


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2512_24545_amd import binding as mb
    mb.lib()
    return torch, mb


def _logits(rng, T, V, spread=2.0, likely=20):
    z = rng.standard_normal((T, V)) * spread
    for row in z:
        row[rng.integers(0, V, likely)] += 9 * rng.random(likely)
    return z


def _check(gpu, z, u, dtype="f32", pad=0, **settings):
    torch, mb = gpu
    T, V = z.shape
    dt = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    wide = torch.full((T, V + pad), float("inf"), dtype=dt, device="cuda:0")
    wide[:, :V] = torch.from_numpy(np.ascontiguousarray(z)).to(dt).to("cuda:0")
    held = wide[:, :V]
    on = {k: torch.from_numpy(np.array(np.broadcast_to(v, T))).to("cuda:0", torch.int32 if k == "top_k" else torch.float32)
          for k, v in settings.items()}
    ut = torch.from_numpy(np.ascontiguousarray(u, dtype=np.float32)).to("cuda:0")
    tokens, probs = mb.mdbf_sample(held, ut, **on)
    again = mb.mdbf_sample(held, ut, **on)
    assert torch.equal(tokens, again[0]) and torch.equal(probs, again[1])
    z64, u64 = held.double().cpu().numpy(), ut.double().cpu().numpy()
    host = {k: v.double().cpu().numpy() for k, v in on.items()}
    for t in range(T):
        token, share = so.sample(z64[t], u64[t], **{k: v[t] for k, v in host.items()})
        assert (int(tokens[t]), True) == (token, True), (t, int(tokens[t]), token, settings)
        assert abs(float(probs[t]) - share) <= TINY * share + 1e-9 * share, (t, float(probs[t]), share)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 8191, 8192, 8193, 32000, 70001])
def test_plain_draws(gpu, V, dtype):
    rng = np.random.default_rng(V)
    _check(gpu, _logits(rng, 9, V), rng.random(9), dtype, pad=V % 3)


@pytest.mark.parametrize("settings", [dict(top_k=1), dict(top_k=50), dict(top_k=5000), dict(top_p=0.9), dict(top_p=0.3), dict(top_p=0.999),
                                      dict(min_p=0.02), dict(min_p=1.0), dict(top_k=40, top_p=0.8), dict(top_k=200, min_p=0.1),
                                      dict(top_p=0.95, min_p=0.01), dict(top_k=30, top_p=0.9, min_p=0.05, temperature=0.7),
                                      dict(temperature=1.5, top_p=0.98), dict(temperature=0.05), dict(temperature=30.0, top_k=1000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bounds(gpu, settings, dtype):
    rng = np.random.default_rng(3)
    for V in (777, 20000):
        _check(gpu, _logits(rng, 16, V), rng.random(16), dtype, **settings)


def test_each_row_has_its_own_settings(gpu):
    rng = np.random.default_rng(4)
    T = 200
    _check(gpu, _logits(rng, T, 9000), rng.random(T), "bf16", temperature=rng.choice([0.0, 0.3, 1.0, 2.0], T), top_k=rng.choice([0, 1, 20, 4000], T),
           top_p=rng.choice([0.1, 0.9, 1.0], T), min_p=rng.choice([0.0, 0.05], T))


def test_more_rows_than_parts_are_cut_small_for(gpu):
    rng = np.random.default_rng(5)
    _check(gpu, _logits(rng, 300, 33000), rng.random(300), "f16", top_p=0.9)


@pytest.mark.parametrize("V", [64, 9001, 40000])
def test_equal_logits_go_by_index(gpu, V):
    """All tokens alike: more equal ones than the list holds, and every bound falls among them."""
    u = np.array([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24])
    z = np.full((5, V), 1.25)
    _check(gpu, z, u)
    _check(gpu, z, u, top_p=0.5)
    _check(gpu, z, u, top_k=V // 2, top_p=0.5)
    _check(gpu, z, u, min_p=1.0)
    z[:, V // 3:V // 2] = 2.25
    _check(gpu, z, u, top_k=V // 4)
    z[:, ::2] = -0.0
    z[:, 1::2] = 0.0
    _check(gpu, z, u)


def test_flat_rows_that_overflow_the_list(gpu):
    """Tokens in one bucket, but of different weights."""
    rng = np.random.default_rng(6)
    _check(gpu, rng.random((6, 50000)), rng.random(6), temperature=100.0)
    _check(gpu, rng.random((6, 50000)), rng.random(6), temperature=100.0, top_k=30000, top_p=0.7, min_p=0.99)


def test_bf16_ties_everywhere(gpu):
    rng = np.random.default_rng(7)
    z = np.round(rng.standard_normal((20, 30000)) * 2) / 2
    for settings in (dict(), dict(top_p=0.9), dict(top_k=777), dict(min_p=0.3), dict(top_k=500, top_p=0.5, min_p=0.01)):
        _check(gpu, z, rng.random(20), "bf16", **settings)


def test_masks_infinities_and_nan(gpu):
    rng = np.random.default_rng(8)
    V = 20000
    z = _logits(rng, 12, V)
    z[0] = -np.inf
    z[1] = np.nan
    z[2] = -np.inf
    z[2, 12345] = -3.0
    z[3, rng.integers(0, V, V // 2)] = np.nan
    z[4, [5, 17000]] = np.inf
    z[5] = np.inf
    z[6, 1:] = -np.inf
    z[7] = -3.4e38
    z[8, 8192:] = -np.inf                        # whole parts masked
    z[9, :16384] = -np.inf
    z[10] *= 1e30
    z[11] *= 1e-30
    u = rng.random(12)
    for settings in (dict(), dict(top_p=0.9), dict(top_k=3), dict(min_p=0.5, temperature=0.5), dict(temperature=0.0)):
        _check(gpu, z, u, **settings)
    _check(gpu, z[:10], u[:10], "f16", top_p=0.8)


def test_settings_at_their_ends(gpu):
    rng = np.random.default_rng(9)
    z = _logits(rng, 8, 5000)
    u = np.array([0.0, 1.0, -1.0, 2.0, np.nan, 0.5, 2.0 ** -24, 1 - 2.0 ** -24])
    inf, nan = np.inf, np.nan
    for settings in (dict(), dict(top_p=np.array([0, -1, nan, 1, 2, 1e-9, 1 - 2.0 ** -24, 0.5])), dict(min_p=np.array([0, -1, nan, 1, 2, 1e-30, 1e-45, 1.0])),
                     dict(top_k=np.array([0, -5, 1, 4999, 5000, 5001, 2 ** 31 - 1, 2])),
                     dict(temperature=np.array([0, -1, nan, inf, 1e-45, 1e-30, 3e38, 1.0]))):
        _check(gpu, z, u, **settings)


def test_more_rows_than_a_grid_has(gpu):
    """65535 rows are a grid's second dimension."""
    rng = np.random.default_rng(10)
    T, V = 65600, 24
    torch, mb = gpu
    z = torch.from_numpy(rng.standard_normal((T, V)).astype(np.float32)).to("cuda:0")
    u = torch.from_numpy(rng.random(T).astype(np.float32)).to("cuda:0")
    on = dict(temperature=torch.from_numpy((0.5 + rng.random(T)).astype(np.float32)).to("cuda:0"), top_k=torch.randint(0, 9, (T,), device="cuda:0", dtype=torch.int32))
    tokens, probs = mb.mdbf_sample(z, u, **on)
    for t in list(range(0, T, 997)) + list(range(65530, 65540)) + [T - 1]:
        token, share = so.sample(z[t].double().cpu().numpy(), float(u[t]), float(on["temperature"][t]), int(on["top_k"][t]))
        assert int(tokens[t]) == token and abs(float(probs[t]) - share) <= (TINY + 1e-9) * share


def test_many_light_tokens_behind_a_heavy_one(gpu):
    """More tokens of one bucket than the list holds, each of a weight of 1e-5."""
    rng = np.random.default_rng(11)
    z = np.full((6, 50000), np.log(1e-5)) + 1e-3 * rng.random((6, 50000))
    z[:, 31415] = 0.0
    for settings in (dict(), dict(top_p=0.9), dict(top_k=30000)):
        _check(gpu, z, 0.1 + 0.85 * rng.random(6), **settings)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_the_largest_vocabulary(gpu, dtype):
    """2^20 tokens, 128 parts: one near the end alone, thousands alike, and everything."""
    rng = np.random.default_rng(12)
    z = _logits(rng, 4, 1 << 20)
    z[1, :] = -np.inf
    z[1, (1 << 20) - 1] = -5.0
    z[2, ::300] = 12.0
    for settings in (dict(), dict(top_p=0.95, min_p=1e-4), dict(top_k=100000)):
        _check(gpu, z, rng.random(4), dtype, **settings)


def test_logits_at_every_scale(gpu):
    """Offsets and spreads from far below to far above 1: weights go by differences, over a temperature of that scale."""
    rng = np.random.default_rng(13)
    for scale in (1e-6, 1e-3, 1e3, 1e6):
        for offset in (0.0, 1.0, -300.0):
            z = (_logits(rng, 3, 6000) + offset) * scale
            _check(gpu, z, rng.random(3), temperature=scale)
            _check(gpu, z, rng.random(3), temperature=scale, top_p=0.9, top_k=1000)


@pytest.mark.parametrize("V", [9000, 128256, 1 << 20])
@pytest.mark.parametrize("logit", [-9.0, -18.0, -21.0])
def test_thousands_of_equal_light_tokens(gpu, V, logit):
    """One token of weight 1, the others alike and light: rounding of a weight is the same for all of them and adds up.  Sums held to 1e-11 of
    themselves move a place among the light ones by up to 1e-11 (1 / weight + V), 0.013 tokens; u and top_p are numbers whose place is no
    nearer than a tenth of a token to an edge, in 64 significant bits."""
    torch, mb = gpu
    rng = np.random.default_rng(V)
    heavy, w = V // 3, np.exp(np.longdouble(logit))
    z = torch.full((1, V), logit, device="cuda:0")
    z[0, heavy] = 0.0

    def numbers(kept, count):
        """fp32 numbers at which kept weights of 1 + (kept - 1) w are cut among the light ones, and the place of each cut."""
        total = 1 + (kept - 1) * w
        u = ((1 + (kept - 1) * w * rng.random(50 * count)) / total).astype(np.float32)
        place = (u.astype(np.longdouble) * total - 1) / w
        part = place - np.floor(place)
        good = (part > 0.1) & (part < 0.9) & (place > 0) & (u <= 1 - 2.0 ** -24)
        return u[good][:count], np.floor(place[good][:count]).astype(np.int64)

    def check(kept, **on):
        u, place = numbers(kept, 24)
        if len(u) == 0:                                             # (light ones that weigh less together than a step of u)
            return
        tokens, probs = mb.mdbf_sample(z.expand(len(u), V).contiguous(), torch.from_numpy(u).to("cuda:0"),
                                       **{k: torch.full((len(u),), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda:0") for k, v in on.items()})
        assert np.array_equal(tokens.cpu().numpy(), np.where(place < heavy, place, place + 1)), (on, kept)
        share = float(w / (1 + (kept - 1) * w))
        assert (np.abs(probs.double().cpu().numpy() - share) <= (TINY + 1e-11) * share).all()

    check(V)
    check(V // 2, top_k=V // 2)
    p, place = numbers(V, 3)
    for p, place in zip(p, place):
        check(int(place) + 2, top_p=float(p))                      # the one that the bound falls into is kept
    p, place = numbers(V // 2, 3)
    for p, place in zip(p, place):
        check(int(place) + 2, top_p=float(p), top_k=V // 2)


@pytest.mark.parametrize("temperature", [0.0888, 0.0815])
def test_logits_of_millions_of_temperatures(gpu, temperature):
    """Logits that differ by a last bit, ten million temperatures from zero: 500000 tokens in front of the few that are looked at and 540000 behind
    them, all summed by buckets.  u are the numbers whose place is 3e-5 to 1.5e-4 tokens from an edge, on either side; sums held to 1e-11
    of themselves move a place by 1e-11 V = 1.1e-5."""
    torch, mb = gpu
    rng = np.random.default_rng(14)
    T32, V, few = np.float32(temperature), 1 << 20, 6000
    level = np.float32(2.0 ** 20) - np.float32(2.0 ** -4) * np.arange(1, 8, dtype=np.float32)    # the next numbers below 2^20
    counts = [1, 0, 0, 0, 500000, few, V - few - 500001]
    z = np.repeat(level, counts)
    order = rng.permutation(V)
    row = np.empty(V, dtype=np.float32)
    row[order] = z
    w = np.exp((level.astype(np.longdouble) - level[0]) / np.longdouble(T32))
    before = 1 + counts[4] * w[4]
    total = before + few * w[5] + counts[6] * w[6]
    u = np.unique(rng.uniform(float(before / total), float((before + few * w[5]) / total), 400000).astype(np.float32))
    place = (u.astype(np.longdouble) * total - before) / w[5]
    part = place - np.floor(place)
    edge = np.minimum(part, 1 - part)
    pick = (edge > 3e-5) & (edge < 1.5e-4) & (place > 0) & (place < few)
    u, place = u[pick], np.floor(place[pick]).astype(np.int64)
    assert len(u) >= 4
    held = torch.from_numpy(row).to("cuda:0").expand(len(u), V).contiguous()
    tokens, _ = mb.mdbf_sample(held, torch.from_numpy(u).to("cuda:0"), torch.full((len(u),), float(T32), device="cuda:0"))
    want = np.sort(np.flatnonzero(row == level[5]))[place]
    assert np.array_equal(tokens.cpu().numpy(), want)


@pytest.mark.parametrize("V", [10, 40, 300, 5000, 20000])
def test_different_logits_of_equal_weight(gpu, V):
    """An infinite temperature: every sum is a whole number, and so are the places of bounds and draws, on edges too."""
    rng = np.random.default_rng(V + 1)
    z = rng.standard_normal((8, V))
    u = np.array([0.0, 0.5, 0.25, 0.75, 0.125, 1 - 2.0 ** -24, 0.875, 0.375])
    for settings in (dict(), dict(top_p=0.5), dict(top_p=0.25, top_k=V // 2), dict(top_p=0.75, min_p=1.0)):
        _check(gpu, z, u, temperature=np.inf, **settings)


@pytest.mark.parametrize("temperature", [np.inf, 1e6, 3e4])
@pytest.mark.parametrize("V", [300, 3000, 8000])
def test_thousands_of_different_logits_of_nearly_one_weight(gpu, V, temperature):
    """All of them in one bin of a bucket, or in a few: the bounds and the draw are found among their digits.  (A place is 1e-9 V tokens from where the
    64-bit sums have it, so 1e-5 of the draws could differ.)"""
    rng = np.random.default_rng(V)
    z = rng.standard_normal((6, V))
    z[3] = np.abs(z[3])
    z[4, ::7] = -np.inf
    z[5, :V // 2] = z[5, 0]
    for settings in (dict(), dict(top_k=V // 3), dict(top_k=5), dict(top_p=0.37), dict(top_p=0.9, top_k=V // 2), dict(min_p=1 - 1e-6), dict(min_p=1.0), dict(top_p=0.5, min_p=0.99999)):
        _check(gpu, z, rng.random(6), temperature=temperature, **settings)
        _check(gpu, z, rng.random(6), "bf16", temperature=temperature, **settings)
