"""Attention over the 4-bit cache at the ends of the ranges of types and formats, in every form that a call can take.  Against the 64-bit
oracle; tolerances follow from the arithmetic at each test."""
import numpy as np
import pytest

from oracle import kv_oracle as kvo
from test_gpu_kv import U, gpu  # noqa: F401  (gpu: the fixture)
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
