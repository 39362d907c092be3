"""Which kernel a call of mdbf_kv_attention takes, without a GPU: every form that there is has a call in test_gpu_kv_paths.py, and what
a call refuses has no name."""
import ctypes as C

import pytest

import test_gpu_kv_paths as paths
from paper_2512_24545_amd import binding as mb

NAMES = {"few rows", "few rows, shares", "prompts", "prompts, n-th row tiles", "prompts, shares"}
FIRST = {"prompts, products first", "prompts, n-th row tiles, products first", "prompts, shares, products first"}


def kernel(d, Hq, Hkv, n, T, fresh, length, window=0, flags=1, dtype=1):
    kv, attn = mb.KvDesc(100, Hkv, d, 64, dtype), mb.AttnDesc(Hq, flags, window, fresh, length, 1.0)
    return mb.lib().mdbf_kv_attention_kernel(C.byref(kv), C.byref(attn), n, T).decode()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_every_form_is_run(d):
    taken = {kernel(d, Hq, Hkv, n, T, fresh, length, window) for dd, _, Hq, Hkv, n, T, fresh, length, window, _ in paths.PATHS if dd == d}
    assert taken == {name for dd, name, *_ in paths.PATHS if dd == d} == (NAMES | FIRST if d == 128 else NAMES)


def test_the_type_and_the_queries_form_do_not_matter():
    for d, name, Hq, Hkv, n, T, fresh, length, window, _ in paths.PATHS:
        assert kernel(d, Hq, Hkv, n, T, fresh, length, window, dtype=0) == kernel(d, Hq, Hkv, n, T, fresh, length, window, flags=3) == kernel(d, Hq, Hkv, n, T, fresh, length, window) == name


def test_what_is_refused_has_no_name():
    assert kernel(96, 4, 2, 1, 1, 1, 1) == kernel(128, 5, 2, 1, 1, 1, 1) == kernel(128, 4, 2, 0, 1, 1, 1) == kernel(128, 4, 2, 1, 1, 0, 1) == ""
    assert kernel(128, 4, 2, 1, 1, 1, 1, flags=4) == kernel(128, 4, 2, 1, 1, 1, 1, dtype=2) == kernel(128, 4, 2, 1, 1, 1, 1, window=-1) == ""
    assert mb.lib().mdbf_kv_attention_kernel(None, None, 1, 1) == b""
