"""Attention over the 4-bit cache where the work is cut into shares: parts of row tiles left by several workgroups and joined, for
few rows and for prompts, requests of very unequal lengths, more requests than a wave has lanes.  Against the 64-bit oracle, with
the tolerances of test_gpu_kv.py (which hold although the prompts' kernel also rounds queries, to 2^-14 (bf16) or 2^-18 (fp16) of
the largest of 32 channels: some 1e-4 of a score)."""
import numpy as np
import pytest

from test_gpu_kv import Step, gpu, ints, not_finite_case  # noqa: F401  (gpu: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d,P", [(4, 1, 128, 64), (7, 1, 64, 16), (2, 1, 256, 32), (4, 4, 128, 32), (3, 3, 64, 128)])
@pytest.mark.parametrize("lengths,fresh", [([4000], [60]), ([2500, 70, 1300], [90, 33, 150]), ([3000, 1100], [17, 200])])
@pytest.mark.parametrize("window", [0, 1200])
def test_prompts_behind_long_caches(gpu, dt, Hq, Hkv, d, P, lengths, fresh, window):
    Step(gpu, lengths, fresh, Hq, Hkv, d, P, dt, seed=d + len(lengths)).check(window=window)


@pytest.mark.parametrize("d,P", [(64, 16), (128, 64), (256, 256)])
def test_prompts_that_see_everything(gpu, d, P):
    Step(gpu, [3000, 1500], [130, 40], 2, 1, d, P, "bf16").check(causal=False)


@pytest.mark.parametrize("n", [63, 64, 65, 256, 257, 300])
@pytest.mark.parametrize("fresh", [1, 0, 3])
def test_many_requests(gpu, n, fresh):
    """Prefix sums over the requests: by a wave for itself, by the workgroup, over several rounds; requests without tokens among
    them."""
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in rng.integers(0, 120, n)]
    lengths[n // 2] = 1500
    new = [int(x) for x in rng.integers(0, 2, n)] if fresh == 0 else [fresh] * n
    s = Step(gpu, lengths, new, 2, 1, 64, 16, "bf16", seed=n)
    s.check()
    s.check(max_length=10)       # not cut


@pytest.mark.parametrize("n", [70, 300])
def test_many_prompts(gpu, n):
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in rng.integers(1, 60, n)]
    fresh = [int(rng.integers(0, x + 1)) for x in lengths]
    lengths[3], fresh[3] = 2000, 60
    lengths[n - 1], fresh[n - 1] = 1100, 1
    Step(gpu, lengths, fresh, 4, 1, 64, 16, "f16", seed=n).check()


@pytest.mark.parametrize("lengths,fresh", [([4000], [300]), ([2000, 80, 5000], [270, 80, 300])])
@pytest.mark.parametrize("window", [0, 700])
def test_more_row_tiles_than_a_wave_has_lanes(gpu, lengths, fresh, window):
    """32 query heads share one of 64 channels: 300 tokens are 75 tiles of 128 rows or 600 of 16."""
    Step(gpu, lengths, fresh, 32, 1, 64, 32, "f16", seed=len(fresh)).check(window=window)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,d", [(7, 1, 64), (6, 2, 128), (4, 1, 256)])
@pytest.mark.parametrize("window", [0, 100])
def test_one_long_prompt_among_short_ones(gpu, dt, Hq, Hkv, d, window):
    """Row tiles without shares, far fewer than the longest prompt would have in every request; requests without any."""
    fresh = [3, 0, 500, 20, 130, 0, 60, 129, 1]
    s = Step(gpu, [n + extra for n, extra in zip(fresh, [200, 0, 90, 7, 0, 300, 64, 1, 400])], fresh, Hq, Hkv, d, 32, dt, seed=d)
    s.check(window=window)
    s.check(window=window, causal=True, max_fresh=713)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lengths,fresh,heads,window", [([5000], [70], 4, 0), ([6000, 4500], [33, 66], 4, 4400)])
def test_prompts_that_see_much(gpu, dt, lengths, fresh, heads, window):
    Step(gpu, lengths, fresh, heads, heads // 4, 128, 64, dt, seed=heads).check(window=window)


@pytest.mark.parametrize("Hkv", [1, 5])
def test_a_very_long_prompt_among_short_ones(gpu, Hkv):
    """More row tiles in a request than a wave has lanes."""
    fresh = [30, 5, 700, 1, 1]
    Step(gpu, [n + 40 for n in fresh], fresh, 16 * Hkv, Hkv, 64, 16, "bf16").check()


@pytest.mark.parametrize("heads", [(16, 1), (17, 1), (24, 8)])
def test_very_unequal_lengths(gpu, heads):
    """Shares that begin and end inside the cost of a row tile, row tiles in one share, in two and in many."""
    Hq, Hkv = heads
    Step(gpu, [6000, 1, 64, 65, 640, 0, 2, 127, 128, 1025, 3, 4500], [1] * 5 + [0] + [1] * 6, Hq, Hkv, 64, 64, "bf16").check()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("fresh,lengths,window", [([40], [3000], 0), ([70, 1], [1500, 1400], 1100)])
def test_blocks_that_are_not_finite_in_parts(gpu, dt, fresh, lengths, window):
    not_finite_case(gpu, dt, fresh, lengths, sum(lengths), window)


@pytest.mark.parametrize("fresh,lengths", [(200, [6000, 3000]), (60, [4000, 1100]), (16, [3000, 64])])
def test_same_bits_again_and_whatever_the_workspace_holds(gpu, fresh, lengths):
    torch, mb = gpu
    s = Step(gpu, lengths, [fresh, 1], 8, 2, 128, 64, "bf16")
    ws = mb.mdbf_kv_attention_workspace(s.cache, 8, 2, s.q.shape[0], fresh, max(lengths))
    assert ws is not None
    want = None
    for byte in (0, 255, 127):
        ws.fill_(byte)
        out = s.run(max_fresh=fresh, max_length=max(lengths), workspace=ws)
        want = out if want is None else want
        assert torch.equal(out[:fresh + 1], want[:fresh + 1])
    g, out = torch.cuda.CUDAGraph(), torch.zeros_like(s.q)
    table, cu, ln = s.table, ints(torch, s.cu), ints(torch, s.lengths)
    with torch.cuda.graph(g):
        mb.mdbf_kv_attention(s.cache, s.q, table, cu, ln, fresh, max(lengths), out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:fresh + 1], want[:fresh + 1])


def test_a_workspace_for_the_largest_call_serves_smaller_ones(gpu):
    torch, mb = gpu
    s = Step(gpu, [2000, 1500], [40, 1], 8, 2, 128, 64, "bf16")
    size = lambda fresh, length, **kw: (lambda w: 0 if w is None else w.numel())(mb.mdbf_kv_attention_workspace(s.cache, 8, 2, 100, fresh, length, **kw))
    largest = size(2048, 100000)
    for fresh in (1, 4, 5, 40, 700, 2048):
        for length in (1, 1024, 1025, 5000, 100000):
            assert size(fresh, length) <= largest and size(fresh, length) <= size(2048, length)
            for window in (1, 500, 2000):
                assert size(fresh, length, window=window) <= size(fresh, length)
    s.check(workspace=torch.empty(largest, dtype=torch.uint8, device="cuda:0"))


@pytest.mark.parametrize("requests,cached,fresh,kv_heads", [(3, 100, 1, 8), (2, 0, 40, 32), (1, 1500, 20, 4)])
def test_the_attention_block_of_a_layer(gpu, requests, cached, fresh, kv_heads):
    """The whole block as workloads.py runs it, eagerly and from a graph, against the oracles of its parts."""
    torch, mb = gpu
    from oracle import kv_oracle as kvo
    from paper_2512_24545_amd.workloads import AttentionBlock
    g = torch.Generator(device="cuda:0")
    g.manual_seed(cached + fresh)
    b = AttentionBlock(torch, g, requests, cached, fresh, kv_heads)
    Y = b.step().clone()
    torch.cuda.synchronize()
    assert b.places.status.item() == 0
    # the attention's inputs: what the projections gave, normed and turned; its result against the cache's contents
    table, d, group = b.table.cpu().numpy(), 128, 32 // kv_heads
    for r in range(requests):
        pos = np.arange(cached + fresh)
        slots = torch.from_numpy(table[r, pos // 64].astype(np.int64) * 64 + pos % 64).cuda()
        k, v = (x.double().cpu().numpy() for x in mb.mdbf_kv_read(b.cache, slots))
        rows = slice(r * fresh, (r + 1) * fresh)
        q_in, k_in, v_in = (x[rows].double().cpu().numpy() for x in b.heads)
        norm, rope = [w.cpu().numpy() for w in b.norm], b.rope.cpu().numpy()
        q_ref = kvo.norm_rope(q_in, norm[0], rope, pos[cached:], 1e-6, False)
        q = b.turned[rows].double().cpu().numpy()
        assert np.abs(q - q_ref).max() <= 2.0 ** -11 * np.abs(q_ref).max() + 4e-6 * np.abs(q_ref).max()
        assert np.array_equal(v[cached:], kvo.values(*kvo.quantise(v_in, "f16")))
        k_ref = kvo.norm_rope(k_in, norm[1], rope, pos[cached:], 1e-6, False)
        assert np.abs(k[cached:] - k_ref).max() <= np.abs(k_ref).max() / 4        # 4 bits: at most half a step of the largest numbers
        out = b.out[rows].double().cpu().numpy()
        for h in (0, 13, 31):
            ref, mag, den = kvo.attention(q[:, h], k[:, h // group], v[:, h // group], pos[cached:], True, 0, d ** -0.5)
            from test_gpu_kv import attention_tolerance
            assert (np.abs(out[:, h] - ref) <= attention_tolerance("f16", ref, mag, den, q[:, h], k[:, h // group], v[:, h // group], d ** -0.5)).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for _ in range(3):
        b.Y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.Y, Y)
