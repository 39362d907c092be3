"""The operators around the projections as they are used: together, from graphs, on other streams, with the workspaces of other calls."""
import numpy as np
import pytest

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu
H16, F32 = 2.0 ** -11, 2.0 ** -24


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2512_24545_amd import binding as mb
    mb.lib()
    return torch, mb


def _np(t):
    return t.double().cpu().numpy()


def _adapted(y0, x, of, pool):
    """(y0 + what the adapters add, its bound): sums of n and r terms in fp32, inner values to 2^-22 of a row's largest, one rounding to fp16."""
    A, B, scale = _np(pool.A), _np(pool.B), _np(pool.scale)
    want, off = y0 + so.adapters(x, of, A, B, scale), np.zeros_like(y0)
    for t, a in enumerate(of):
        if a >= 0:
            inner, size = A[a] @ x[t], np.abs(A[a]) @ np.abs(x[t])
            off[t] = scale[a] * (np.abs(B[a]) @ (A.shape[2] * F32 * size + 2.0 ** -22 * np.abs(inner).max() + 2 * A.shape[1] * F32 * np.abs(inner)))
    return want, off * 1.01 + (H16 + 4 * F32) * np.abs(want) + 2.0 ** -25


@pytest.mark.parametrize("requests,cached,fresh,kv_heads,rank", [(11, 70, 1, 8, 16), (3, 20, 9, 32, 5)])
def test_a_serving_step(gpu, requests, cached, fresh, kv_heads, rank):
    """A step of the workload, every operator's result against its definition on the inputs that it had, and the same from a graph."""
    torch, mb = gpu
    from paper_2512_24545_amd.workloads import AttentionBlock, ServingStep
    g = torch.Generator(device="cuda:0")
    g.manual_seed(1)
    s = ServingStep(torch, g, requests, cached, fresh, kv_heads, adapters=4, rank=rank)
    before = {}

    class Watched(ServingStep):
        def projected(self):
            before["qkv"] = [y.clone() for y in self.qkv]
            super().projected()

    s.__class__ = Watched
    tokens, probs = s.step()
    torch.cuda.synchronize()
    assert tokens is s.tokens and s.places.status.item() == 0
    eps = float(np.float32(1e-6))
    x, h = so.add_norm(_np(s.update), _np(s.stream), _np(s.weights[0]), eps)
    assert (np.abs(_np(s.X) - x) <= (H16 + 4 * F32) * np.abs(x) + 2.0 ** -25).all() and (np.abs(_np(s.between) - h) <= F32 * np.abs(h)).all()
    of = np.repeat(s.adapter.cpu().numpy(), fresh)
    for y0, y, pool in zip(before["qkv"], s.qkv, s.pools):
        want, off = _adapted(_np(y0), _np(s.X), of, pool)
        assert (np.abs(_np(y) - want) <= off).all()
    y0 = mb.mdbf_forward(s.o, s.out.flatten(1), y_dtype="f16")
    want, off = _adapted(_np(y0), _np(s.out.flatten(1)), of, s.pool_o)
    assert (np.abs(_np(s.Y) - want) <= off).all()
    x, h = so.add_norm(_np(s.Y), _np(s.between), _np(s.weights[1]), eps)
    assert (np.abs(_np(s.normed) - x) <= (H16 + 4 * F32) * np.abs(x) + 2.0 ** -25).all() and (np.abs(_np(s.behind) - h) <= F32 * np.abs(h)).all()
    assert torch.equal(s.logits, mb.mdbf_forward(s.head, s.normed[s.last], y_dtype="f32"))
    z, u = _np(s.logits), _np(s.u)
    for t in range(requests):
        token, share = so.sample(z[t], u[t], _np(s.temperature)[t], 50, _np(s.top_p)[t])
        assert int(tokens[t]) == token and abs(float(probs[t]) - share) <= (F32 + 1e-9) * share
    # from a graph, with other inputs between the replays
    s.__class__ = ServingStep
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for seed in range(4):
        torch.manual_seed(seed)
        s.update.copy_(torch.randn_like(s.update, dtype=torch.float32))
        s.u.copy_(torch.rand_like(s.u))
        s.adapter.copy_(torch.randint_like(s.adapter, -1, 4))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (s.X, s.Y, s.behind, s.logits, s.tokens, s.probs, s.rows.rows, s.rows.tiles)]
        s.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (s.X, s.Y, s.behind, s.logits, s.tokens, s.probs, s.rows.rows, s.rows.tiles)))
    assert issubclass(ServingStep, AttentionBlock)


def _sampling(torch, seed, T, V, dtype):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return torch.randn((T, V), generator=g, device="cuda:0").mul(3).to(dtype), torch.rand((T,), generator=g, device="cuda:0")


def test_one_workspace_for_calls_of_several_sizes_and_graphs(gpu):
    """Nothing is carried from one call to the next in a workspace, whatever lies there."""
    torch, mb = gpu
    sizes = [(40, 30000, torch.float32, dict()), (3, 100, torch.bfloat16, dict()), (40, 9000, torch.float16, dict(top_p=0.7)), (1, 30000, torch.float32, dict(top_k=9))]
    ws = mb.mdbf_sample_workspace(40, 30000)
    cases = []
    for i, (T, V, dtype, kw) in enumerate(sizes):
        z, u = _sampling(torch, i, T, V, dtype)
        on = {k: torch.full((T,), v, device="cuda:0", dtype=torch.int32 if k == "top_k" else torch.float32) for k, v in kw.items()}
        cases.append((z, u, on, mb.mdbf_sample(z, u, **on)))
    ws.fill_(255)
    graphs = []
    for z, u, on, _ in cases:
        out = (torch.zeros(len(u), dtype=torch.int32, device="cuda:0"), torch.zeros(len(u), device="cuda:0"))
        mb.mdbf_sample(z, u, **on, tokens=out[0], probs=out[1], workspace=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mb.mdbf_sample(z, u, **on, tokens=out[0], probs=out[1], workspace=ws)
        graphs.append((graph, out))
    for order in ((0, 1, 2, 3), (3, 2, 1, 0), (2, 2, 0, 1)):
        for i in order:
            for t in graphs[i][1]:
                t.fill_(-7)
            graphs[i][0].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(graphs[i][1], cases[i][3]))
        ws.random_(0, 256)


def test_adapters_from_graphs_that_share_a_workspace(gpu):
    torch, mb = gpu
    g = torch.Generator(device="cuda:0")
    g.manual_seed(3)
    N, n, r = 6, 512, 16
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")       # noqa: E731
    steps = []
    for T, m, requests in ((64, 300, 64), (200, 64, 3), (1, 1000, 1)):
        normal = lambda *shape: torch.randn(shape, generator=g, device="cuda:0").bfloat16()     # noqa: E731
        pool = mb.Adapters(normal(N, r, n), normal(N, m, r))
        cu = ints([T * i // requests for i in range(requests + 1)])
        rows = mb.mdbf_adapter_rows(cu, torch.randint(-1, N, (requests,), generator=g, device="cuda:0", dtype=torch.int32), N, T)
        X, Y = normal(T, n), normal(T, m)
        steps.append((rows, pool, X, Y))
    need = [mb.mdbf_adapters_workspace(rows, [pool], [X], [Y]).numel() for rows, pool, X, Y in steps]
    ws = torch.full((max(need),), 255, dtype=torch.uint8, device="cuda:0")
    graphs, want = [], []
    for rows, pool, X, Y in steps:
        y = Y.clone()
        mb.mdbf_adapters(rows, [pool], [X], [y])
        want.append(y)
        out = Y.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out.copy_(Y)
            mb.mdbf_adapters(rows, [pool], [X], [out], workspace=ws)
        graphs.append((graph, out))
    for order in ((0, 1, 2), (2, 0, 1), (1, 1, 0)):
        for i in order:
            graphs[i][0].replay()
            torch.cuda.synchronize()
            assert torch.equal(graphs[i][1], want[i])


def test_calls_on_named_streams_beside_each_other(gpu):
    """Two steps' calls on streams of their own, inputs made on a third, results read on the caller's."""
    torch, mb = gpu
    streams = [torch.cuda.Stream() for _ in range(2)]
    made = []
    for i in range(2):
        z, u = _sampling(torch, 10 + i, 20, 20000, torch.float32)
        x = torch.randn((300, 4096), device="cuda:0").half()
        made.append((z, u, x, mb.mdbf_sample(z, u), mb.mdbf_add_norm(x, y_dtype="e4m3", scale_group=32)))
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for (z, u, x, _, _), s in zip(made, streams):
            s.wait_stream(torch.cuda.current_stream())
            got.append((mb.mdbf_sample(z, u, stream=s), mb.mdbf_add_norm(x, y_dtype="e4m3", scale_group=32, stream=s)))
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        for (_, _, _, tokens, norm), (tokens2, norm2) in zip(made, got):
            assert torch.equal(tokens[0], tokens2[0]) and torch.equal(tokens[1], tokens2[1])
            assert torch.equal(norm[0].view(torch.uint8), norm2[0].view(torch.uint8)) and torch.equal(norm[2], norm2[2])


def test_eight_bits_and_a_product_in_them(gpu):
    """Rows in 8 bits, as a program hands them to a product in 8 bits of its own: the values that they stand for."""
    torch, mb = gpu
    torch.manual_seed(0)
    x, w = torch.randn((50, 640), device="cuda:0").bfloat16(), torch.randn((640, 30), device="cuda:0")
    y, _, _ = mb.mdbf_add_norm(x, y_dtype="f32")
    for group in (0, 32):
        q, _, s = mb.mdbf_add_norm(x, y_dtype="e4m3", scale_group=group)
        scale = s if group == 0 else torch.exp2(s.float() - 127).repeat_interleave(32, 1)
        got, want = (q.float() * scale) @ w, y @ w
        # each of 640 terms is off by at most 2^-4 of itself (and by half of the smallest number, 2^-10 of its scale), fp32 sums by 640 steps
        bound = (y.abs() * 2.0 ** -4 + 2.0 ** -10 * scale) @ w.abs() * (1 + 2.0 ** -10) + 2 * 640 * 2.0 ** -24 * (y.abs() @ w.abs())
        assert ((got - want).abs() <= bound).all()
