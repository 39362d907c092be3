"""Attention block over the 4-bit cache, without a GPU: the 64-bit oracle pinned by hand and by brute force, and every
refusal of the entry points (all of them before any HIP call)."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv_oracle as kvo
from paper_2512_24545_amd import binding as mb

A = 4096          # an aligned address that no refused call touches
HUGE = 1 << 50


def test_levels_and_ties_by_hand():
    x = np.zeros(32)
    x[:15] = [6, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -0.5, -2.5, -6.9, 7, -0.1]
    codes, scales = kvo.quantise(x, "bf16")
    assert scales.tolist() == [127]
    want = [6, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, -0.5, -2, -6, 6, 0]
    assert kvo.values(codes, scales)[:15].tolist() == want


def test_scales_by_hand():
    for top, e in ((7.0, 0), (7.01, 1), (3.5, -1), (3.51, 0), (1.0, -2), (0.0, -125), (1e-45, -125), (3e38, 125)):
        x = np.zeros(32)
        x[3] = top
        assert kvo.quantise(x, "bf16")[1][0] == e + 127, top
    x = np.zeros(32)
    for top, e in ((65504.0, 13), (2.0 ** -24, -23), (7.0, 0)):
        x[5] = -top
        assert kvo.quantise(x, "f16")[1][0] == e + 127, top
    x[5] = 3e38                       # far beyond the range: saturated
    assert kvo.values(*kvo.quantise(x, "f16"))[5] == 6 * 2.0 ** 13
    for bad in (np.nan, np.inf, -np.inf):
        x[7] = bad
        codes, scales = kvo.quantise(x, "f16")
        assert scales[0] == 255 and np.isnan(kvo.values(codes, scales)).all()


def test_quantisation_is_the_nearest_number():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 64)) * np.exp(rng.standard_normal((50, 1)))
    codes, scales = kvo.quantise(x, "bf16")
    got = kvo.values(codes, scales).reshape(-1, 32)
    for block, y, s in zip(x.reshape(-1, 32), got, scales.reshape(-1)):
        unit = 2.0 ** (int(s) - 127)
        grid = np.concatenate([kvo.LEVELS, -kvo.LEVELS]) * unit
        assert np.array_equal(np.abs(block - y), np.abs(block[:, None] - grid).min(1))
        assert 3.5 * unit < np.abs(block).max() <= 7 * unit


def test_attention_oracle_by_hand():
    k = np.array([[0.0], [np.log(3.0)], [50.0]])
    v = np.array([[1.0, 5.0], [2.0, 7.0], [9.0, 9.0]])
    out, mag, den = kvo.attention(np.array([[1.0], [1.0], [1.0]]), k, v, [1, -1, 2], True, 0, 1.0)
    assert np.allclose(out[0], [1.75, 6.5]) and np.allclose(den[0], 4 / 3) and not out[1].any() and np.allclose(out[2], 9)
    out, _, _ = kvo.attention(np.array([[1.0]]), k, v, [1], True, 1, 1.0)
    assert np.allclose(out, [[2.0, 7.0]])
    out, _, _ = kvo.attention(np.array([[0.0]]), k, v, [0], False, 0, 1.0)
    assert np.allclose(out, v.mean(0))


def test_rotation_oracle_by_hand():
    rope = np.array([[1.0, 0.0, 0.0, 1.0], [0.6, 0.8, 0.8, 0.6]])     # two pairs
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    assert np.allclose(kvo.norm_rope(x, None, rope, [1], 0, False)[0, 0], [0.6 - 2.4, 1.6 - 2.4, 1.8 + 0.8, 3.2 + 1.2, 5])
    assert np.allclose(kvo.norm_rope(x, None, rope, [1], 0, True)[0, 0], [0.6 - 1.6, 1.2 + 0.8, 2.4 - 2.4, 3.2 + 1.8, 5])
    assert np.allclose(kvo.norm_rope(x, np.full(5, 2.0), None, None, 0, False)[0, 0], 2 * x[0, 0] / np.sqrt(11.0))


def test_slots_oracle_by_hand():
    got = kvo.slots([0, 15, 16, 5], [1, 2, 0, 12], [[-1, -1], [7, -1], [8, -1], [9, -1]], [3, 4, 5, 6], 1, 16, 16)
    assert got["status"] == 0 and got["taken"] == 4
    assert got["table"].tolist() == [[4, -1], [7, 5], [8, -1], [9, 6]]
    assert got["slots"][:3].tolist() == [64, 127, 80] and got["slots"][3:15].tolist() == list(range(149, 160)) + [96]
    assert got["slots"][15] == -1 and got["cu"].tolist() == [0, 1, 3, 3, 15]


# ---- refusals ------------------------------------------------------------------------------------
def kv(**kw):
    d = dict(pages=10, kv_heads=2, head_dim=128, page_size=16, dtype=1)
    d.update(kw)
    return mb.KvDesc(*[d[n] for n in ("pages", "kv_heads", "head_dim", "page_size", "dtype")])


BAD_KV = [(dict(pages=0), -1), (dict(kv_heads=0), -1), (dict(head_dim=0), -1), (dict(page_size=-16), -1), (dict(dtype=2), -3),
          (dict(dtype=9), -3), (dict(head_dim=96), -5), (dict(page_size=8), -5), (dict(page_size=48), -5), (dict(page_size=512), -5),
          (dict(kv_heads=70000), -5)]


@pytest.mark.parametrize("kw,status", BAD_KV)
def test_cache_descriptions(kw, status):
    out = C.c_size_t(0)
    L = mb.lib()
    assert L.mdbf_kv_page_bytes(kv(**kw), C.byref(out)) == status
    assert L.mdbf_kv_append(kv(**kw), A, HUGE, A, 256, A, 256, 1, A, 1, None) == status
    assert L.mdbf_kv_read(kv(**kw), A, HUGE, A, 1, A, 256, A, 256, 1, None) == status
    assert L.mdbf_kv_page_bytes(None, C.byref(out)) == -1 and L.mdbf_kv_page_bytes(kv(), None) == -1


def test_page_bytes():
    out = C.c_size_t(0)
    for heads in (1, 3, 8):
        for d in (64, 128, 256):
            for P in (16, 32, 64, 128, 256):
                assert mb.lib().mdbf_kv_page_bytes(kv(kv_heads=heads, head_dim=d, page_size=P), C.byref(out)) == 0
                assert out.value == heads * P * 2 * (d // 2 + d // 32) and out.value % 64 == 0


def test_append_and_read_arguments():
    L = mb.lib()
    size = 10 * 2 * 16 * 136
    good = [kv(), A, size, A, 256, A, 256, 1, A, 1, None]
    for at, bad, status in ((0, None, -1), (1, None, -1), (1, A + 8, -2), (2, size - 1, -4), (3, None, -1), (3, A + 2, -2), (4, 255, -1),
                            (5, None, -1), (5, A + 4, -2), (6, 0, -1), (7, 3, -3), (7, -1, -3), (8, None, -1), (8, A + 4, -2),
                            (9, 0, -1), (9, -5, -1)):
        args = list(good)
        args[at] = bad
        assert L.mdbf_kv_append(*args) == status, (at, bad)
    good = [kv(), A, size, A, 1, A, 256, A, 256, 1, None]
    for at, bad, status in ((1, None, -1), (2, 0, -4), (3, None, -1), (3, A + 4, -2), (4, 0, -1), (5, None, -1), (6, 255, -1), (7, A + 1, -2),
                            (8, 1, -1), (9, 7, -3)):
        args = list(good)
        args[at] = bad
        assert L.mdbf_kv_read(*args) == status, (at, bad)


def test_slots_arguments():
    good = [4, 16, A, A, A, 8, 8, A, 5, A, 7, A, A, A, A, A, A, None]
    for at, bad, status in [(0, 0, -1), (1, 24, -5), (1, 8, -5), (1, 512, -5), (5, 7, -1), (6, 0, -1), (7, None, -1), (7, A + 2, -2),
                            (8, -1, -1), (10, 0, -1)] + [(i, None, -1) for i in (2, 3, 4, 9, 11, 12, 13, 14, 15, 16)] + \
            [(i, A + 2, -2) for i in (2, 3, 4, 9, 11, 12, 14, 15, 16)] + [(13, A + 4, -2)]:
        args = list(good)
        args[at] = bad
        assert mb.lib().mdbf_kv_slots(*args) == status, (at, bad)


def rope(**kw):
    d = dict(q_heads=4, kv_heads=2, head_dim=128, rot_dim=128, rope_rows=100, x_dtype=1, y_dtype=1, flags=0, eps=1e-6)
    d.update(kw)
    return mb.RopeDesc(*[d[n] for n in ("q_heads", "kv_heads", "head_dim", "rot_dim", "rope_rows", "x_dtype", "y_dtype", "flags", "eps")])


def test_norm_rope_arguments():
    L = mb.lib()
    size = 10 * 2 * 16 * 136
    good = [rope(), A, 512, A, 256, A, A, A, A, 3, A, 512, A, 256, kv(), A, size, A, 256, A, None]
    for kw, status in ((dict(q_heads=0), -1), (dict(kv_heads=-1), -1), (dict(head_dim=0), -1), (dict(head_dim=80, rot_dim=16), -5),
                       (dict(rot_dim=130), -1), (dict(rot_dim=24), -5), (dict(rot_dim=-16), -1), (dict(rope_rows=0), -1), (dict(x_dtype=3), -3),
                       (dict(y_dtype=-1), -3), (dict(flags=2), -5), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(q_heads=70000), -5)):
        args = list(good)
        args[0] = rope(**kw)
        assert L.mdbf_qk_norm_rope(*args) == status, kw
    for at, bad, status in ((0, None, -1), (1, None, -1), (1, A + 8, -2), (2, 511, -1), (3, None, -1), (4, 255, -1), (5, A + 4, -2), (6, A + 4, -2),
                            (7, None, -1), (8, None, -1), (8, A + 2, -2), (9, 0, -1), (10, None, -1), (10, A + 2, -2), (11, 511, -1), (12, A + 2, -2),
                            (13, 255, -1), (14, kv(kv_heads=1), -1), (14, kv(head_dim=64), -1), (14, kv(dtype=2), -3), (15, None, -1),
                            (15, A + 8, -2), (16, size - 1, -4), (17, None, -1), (17, A + 2, -2), (18, 255, -1), (19, None, -1), (19, A + 4, -2)):
        args = list(good)
        args[at] = bad
        assert L.mdbf_qk_norm_rope(*args) == status, (at, bad)
    nowhere = good[:12] + [None, 0, None, None, 0, None, 0, None, None]     # neither k_out nor a cache
    assert L.mdbf_qk_norm_rope(*nowhere) == -1


def attn(**kw):
    d = dict(q_heads=4, flags=1, window=0, max_fresh=1, max_length=100, scale=0.1)
    d.update(kw)
    return mb.AttnDesc(*[d[n] for n in ("q_heads", "flags", "window", "max_fresh", "max_length", "scale")])


def test_attention_arguments():
    L = mb.lib()
    size, out = 10 * 2 * 16 * 136, C.c_size_t(0)
    good = [kv(), attn(), A, size, A, 9, 9, A, A, 2, A, 512, 3, A, 512, A, HUGE, None]
    bad_attn = ((dict(q_heads=0), -1), (dict(q_heads=5), -1), (dict(flags=4), -5), (dict(window=-1), -1), (dict(window=5, flags=0), -1),
                (dict(max_fresh=0), -1), (dict(max_length=0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(scale=0.0), -1),
                (dict(q_heads=140000), -5))
    for kw, status in bad_attn:
        args = list(good)
        args[1] = attn(**kw)
        assert L.mdbf_kv_attention(*args) == status, kw
        assert L.mdbf_kv_attention_workspace_bytes(kv(), attn(**kw), 2, 3, C.byref(out)) == status, kw
    for kw, status in BAD_KV:
        args = list(good)
        args[0] = kv(**kw)
        assert L.mdbf_kv_attention(*args) == status, kw
        assert L.mdbf_kv_attention_workspace_bytes(kv(**kw), attn(), 2, 3, C.byref(out)) == status, kw
    for at, bad, status in ((1, None, -1), (2, None, -1), (2, A + 8, -2), (3, size - 1, -4), (4, None, -1), (4, A + 2, -2), (5, 8, -1), (6, 0, -1),
                            (7, None, -1), (7, A + 2, -2), (8, None, -1), (8, A + 2, -2), (9, 0, -1), (10, None, -1), (10, A + 2, -2), (11, 511, -1),
                            (12, 0, -1), (13, None, -1), (13, A + 2, -2), (14, 511, -1), (15, A + 4, -2)):
        args = list(good)
        args[at] = bad
        assert L.mdbf_kv_attention(*args) == status, (at, bad)
    assert L.mdbf_kv_attention_workspace_bytes(kv(), attn(), 2, 3, None) == -1
    assert L.mdbf_kv_attention_workspace_bytes(kv(), attn(), 0, 3, C.byref(out)) == -1
    assert L.mdbf_kv_attention_workspace_bytes(kv(), attn(), 2, 0, C.byref(out)) == -1


def test_attention_workspace_is_bounded_and_enough():
    """Long single-token calls of few requests are split; the call refuses a workspace one byte short, on the host."""
    L, out = mb.lib(), C.c_size_t(0)
    for n, T, fresh, length in ((1, 1, 1, 1), (1, 1, 1, 200000), (64, 64, 1, 8192), (3, 300, 200, 50000), (1, 2048, 2048, 16384), (4096, 4096, 1, 2 ** 31 - 1)):
        a = attn(max_fresh=fresh, max_length=length)
        assert L.mdbf_kv_attention_workspace_bytes(kv(), a, n, T, C.byref(out)) == 0
        assert out.value <= 1 << 31
        if out.value:
            size = 10 * 2 * 16 * 136
            args = [kv(), a, A, size, A, 9, 9, A, A, n, A, 512, T, A, 512, A, out.value - 1, None]
            assert L.mdbf_kv_attention(*args) == -4
            args[15], args[16] = None, HUGE
            assert L.mdbf_kv_attention(*args) == -1
