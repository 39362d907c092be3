"""Run one of the named synthetic workloads on cuda:0 and print its time per pass.

    python3 -m paper_2512_24545_amd.workloads stack   --budget 1.5 --tokens 8 --passes 300 --warmup 100
    python3 -m paper_2512_24545_amd.workloads prefill --tokens 2048 --x-dtype f16 --passes 200 --warmup 300
    python3 -m paper_2512_24545_amd.workloads attention --requests 16 --cached 4000 --fresh 1 --kv-heads 8
    python3 -m paper_2512_24545_amd.workloads step      --requests 16 --cached 4000 --fresh 1 --kv-heads 8 --adapters 8 --adapter-rank 16

`stack`: the 32-layer decoder stack (224 independent products per pass: q, k, v, o, gate, up, down per
layer, LLaMA-7B shapes at the given bit budget), `--tokens` activations per matrix, issued as one plan
through mdbf_forward_batch.  `prefill`: one 4096 x 4096, k = 2656, l = 16 layer with `--tokens` tokens
through mdbf_forward.  `attention`: the attention block of one decoder layer as a serving step runs it, `--fresh` new
tokens for each of `--requests` requests behind `--cached` ones: q, k, v projections as one plan, places in the cache
(mdbf_kv_slots), norm and rotation with keys and values into the 4-bit cache (mdbf_qk_norm_rope), attention over it
(mdbf_kv_attention), output projection.  `step`: the same between what stands around it, for requests that have low-rank adapters: the residual's
addition and norm in front and behind (mdbf_add_norm), the adapters beside the four projections (mdbf_adapter_rows, mdbf_adapters), and for the
last token of each request a compressed head and the choice of the next one (mdbf_sample).  Layers are drawn on the device (random packed sign words, envelopes
|N(0,1)| * 0.02 + 1e-3 in fp16, activations N(0,1)).  With few passes and no warm-up this is the program to
put under a profiler; bench.py remains the benchmark.
"""
import argparse
import json
import sys

from . import binding as mb
from . import synth


def _device_layer(torch, g, m, n, k, l):
    def words(nbytes):
        w = torch.randint(-2 ** 31, 2 ** 31 - 1, (nbytes // 4,), dtype=torch.int32, generator=g, device="cuda:0")
        return w.view(torch.uint8)

    def env(rows):
        return (torch.randn((rows, l), generator=g, device="cuda:0").abs() * 0.02 + 1e-3).half()

    return mb.DeviceLayer(m, n, k, l, words(mb.mdbf_packed_bytes(m, k)), words(mb.mdbf_packed_bytes(k, n)),
                          env(m), env(k), env(k), env(n))


def _time(torch, fn, warmup, passes):
    for _ in range(warmup):
        fn()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(passes):
        fn()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) / passes


def run_stack(torch, args):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(5)
    T = args.tokens
    specs = [synth.stack_matrix_spec(args.budget, 0, mat) for mat in range(7)]
    layers, Xs, Ys, nbytes = [], [], [], 0
    for _ in range(32):
        for sp in specs:
            m, n, k, l = sp["m"], sp["n"], sp["k"], sp["l"]
            layers.append(_device_layer(torch, g, m, n, k, l))
            Xs.append(torch.randn((T, n), generator=g, device="cuda:0").half())
            Ys.append(torch.zeros((T, m), dtype=torch.float16, device="cuda:0"))
            nbytes += (m + n) * k // 8 + 2 * l * (m + n + 2 * k) + T * 2 * (m + n)
    plan = mb.BatchPlan(layers, Xs, Ys)
    ms = _time(torch, plan.run, args.warmup, args.passes)
    return {"workload": "stack", "budget_bpw": args.budget, "matrices": len(layers), "tokens": T,
            "ms_per_pass": ms, "algorithmic_MB": nbytes / 1e6, "GB/s": nbytes / ms / 1e6,
            "pct_hbm_peak": nbytes / ms / 1e6 / 80.0}


def run_prefill(torch, args):
    m, n, k, l, T = 4096, 4096, 2656, 16, args.tokens
    g = torch.Generator(device="cuda:0")
    g.manual_seed(4)
    dl = _device_layer(torch, g, m, n, k, l)
    xdt = {"f16": torch.float16, "bf16": torch.bfloat16}[args.x_dtype]
    X = torch.randn((T, n), generator=g, device="cuda:0").to(xdt)
    Y = torch.empty((T, m), dtype=torch.float32, device="cuda:0")
    d = dl.desc(args.x_dtype, "f32")
    ws = torch.empty(mb.mdbf_workspace_bytes(d, T), dtype=torch.uint8, device="cuda:0")
    ms = _time(torch, lambda: mb.mdbf_forward(dl, X, y_dtype="f32", Y=Y, workspace=ws), args.warmup, args.passes)
    return {"workload": "prefill", "tokens": T, "x_dtype": args.x_dtype, "ms_per_call": ms,
            "tokens_per_s": T / ms * 1e3, "dense_equivalent_TFLOPs": 2.0 * m * n * T / ms / 1e9,
            "issued_TFLOPs": 2.0 * (m + n) * k * (T + l) / ms / 1e9}


class AttentionBlock:
    """The attention block of one decoder layer with compressed projections (4096 wide, 32 heads of 128) and its 4-bit cache;
    step() is what a serving program issues per step, and may be captured into a graph."""
    WIDTH, HEADS, HEAD_DIM = 4096, 32, 128

    def __init__(self, torch, g, requests, cached, fresh, kv_heads, budget="1.5", page_size=64, rope_rows=None):
        d, T = self.HEAD_DIM, requests * fresh
        n = self.WIDTH

        def layer(m):
            l = synth.stack_matrix_spec(budget, 0, 0)["l"]
            k = mb.mdbf_rank_for_budget(m, n, l, float(budget), 16, 32)
            return _device_layer(torch, g, m, n, k, l)

        self.q, self.k, self.v, self.o = layer(n), layer(kv_heads * d), layer(kv_heads * d), layer(n)
        half = lambda *shape: torch.zeros(shape, dtype=torch.float16, device="cuda:0")
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")
        self.X = torch.randn((T, n), generator=g, device="cuda:0").half()
        self.qkv = [half(T, n), half(T, kv_heads * d), half(T, kv_heads * d)]
        self.plan = mb.BatchPlan([self.q, self.k, self.v], [self.X] * 3, self.qkv)
        self.heads = [y.unflatten(1, (-1, d)) for y in self.qkv]
        self.turned, self.out, self.Y = half(T, self.HEADS, d), half(T, self.HEADS, d), half(T, n)
        self.workspace = torch.empty(mb.mdbf_workspace_bytes(self.o.desc("f16", "f16"), T), dtype=torch.uint8, device="cuda:0")
        # norm weights, and cosines and sines of every position that the cache can hold
        self.norm = [1 + 0.1 * torch.randn((d,), generator=g, device="cuda:0") for _ in range(2)]
        self.longest = cached + fresh
        angle = torch.arange(rope_rows or self.longest, device="cuda:0").double()[:, None] * \
            10000.0 ** (-torch.arange(0, d, 2, device="cuda:0").double() / d)
        self.rope = torch.cat([angle.cos(), angle.sin()], 1).float()
        # the requests' pages hold their cached tokens; what the new ones need is taken from the free list
        held, width = -(-cached // page_size), -(-self.longest // page_size)
        pages = requests * width
        perm = torch.randperm(pages, generator=g, device="cuda:0").int()
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda:0")
        self.table[:, :held] = perm[:requests * held].view(requests, held)
        self.free = perm[requests * held:].clone()
        self.cached, self.fresh, self.taken = ints([cached] * requests), ints([fresh] * requests), ints([0])
        self.cache = mb.KVCache(pages, kv_heads, d, page_size, "f16")
        for at in range(0, requests * held * page_size, 65536):
            slots = torch.arange(at, min(at + 65536, requests * held * page_size), device="cuda:0")
            slots = perm[slots // page_size].long() * page_size + slots % page_size
            k, v = (torch.randn((len(slots), kv_heads, d), generator=g, device="cuda:0").half() for _ in range(2))
            mb.mdbf_kv_append(self.cache, k, v, slots)
        self.places = mb.KVSlots(requests, T)
        self.most = fresh
        self.attention_workspace = mb.mdbf_kv_attention_workspace(self.cache, self.HEADS, requests, T, fresh, self.longest)

    def step(self):
        p = mb.mdbf_kv_slots(self.cached, self.fresh, self.table, self.free, self.taken, self.cache.page_size, self.X.shape[0], out=self.places)
        self.plan.run()
        self.projected()
        q, k, v = self.heads
        mb.mdbf_qk_norm_rope(q, k, self.rope, p.positions, q_weight=self.norm[0], k_weight=self.norm[1], q_out=self.turned,
                             cache=self.cache, v=v, slots=p.slots)
        mb.mdbf_kv_attention(self.cache, self.turned, self.table, p.cu, p.lengths, self.most, self.longest, out=self.out,
                             workspace=self.attention_workspace)
        return mb.mdbf_forward(self.o, self.out.flatten(1), y_dtype="f16", Y=self.Y, workspace=self.workspace)

    def projected(self):
        """What a program adds to q, k and v behind the projections."""


class ServingStep(AttentionBlock):
    """The attention block between residual additions with norm, low-rank adapters beside its projections, and a head with the choice of each
    request's next token behind it.  One request in nine has no adapter, one in eight takes the likeliest token."""
    VOCAB = 32000

    def __init__(self, torch, g, requests, cached, fresh, kv_heads, budget="1.5", adapters=8, rank=16, **kw):
        super().__init__(torch, g, requests, cached, fresh, kv_heads, budget, **kw)
        n, T, d = self.WIDTH, requests * fresh, kv_heads * self.HEAD_DIM
        normal = lambda scale, *shape: torch.randn(shape, generator=g, device="cuda:0") * scale
        self.stream, self.update = normal(2.0, T, n), normal(1.0, T, n).half()     # the residual stream, and what the layer in front adds to it
        self.weights = [1 + normal(0.1, n) for _ in range(2)]
        pool = lambda m: mb.Adapters(normal(n ** -0.5, adapters, rank, n).half(), normal(0.1 * rank ** -0.5, adapters, m, rank).half(), 0.5 + normal(0.1, adapters).abs())
        self.pools, self.pool_o = [pool(n), pool(d), pool(d)], pool(n)
        of = torch.randint(0, adapters, (requests,), generator=g, device="cuda:0", dtype=torch.int32)
        self.adapter = torch.where(torch.arange(requests, device="cuda:0") % 9 == 8, -1, of)
        self.rows = mb.AdapterRows(T, requests, adapters)
        flat = self.out.flatten(1)
        self.adapter_workspaces = [mb.mdbf_adapters_workspace(self.rows, self.pools, [self.X] * 3, self.qkv),
                                   mb.mdbf_adapters_workspace(self.rows, [self.pool_o], [flat], [self.Y])]
        self.between, self.behind = torch.zeros_like(self.stream), torch.zeros_like(self.stream)
        self.normed = torch.zeros((T, n), dtype=torch.float16, device="cuda:0")
        l = synth.stack_matrix_spec(budget, 0, 0)["l"]
        self.head = _device_layer(torch, g, self.VOCAB, n, mb.mdbf_rank_for_budget(self.VOCAB, n, l, float(budget), 16, 32), l)
        self.last = torch.arange(fresh - 1, T, fresh, device="cuda:0")
        self.logits = torch.zeros((requests, self.VOCAB), dtype=torch.float32, device="cuda:0")
        self.head_workspace = torch.empty(mb.mdbf_workspace_bytes(self.head.desc("f16", "f32"), requests), dtype=torch.uint8, device="cuda:0")
        row = torch.arange(requests, device="cuda:0")
        self.u = torch.rand((requests,), generator=g, device="cuda:0")
        self.temperature = (0.6 + 0.1 * (row % 5)) * (row % 8 != 7)
        self.top_k, self.top_p = torch.full_like(self.adapter, 50), torch.full_like(self.u, 0.9)
        self.tokens, self.probs = torch.zeros_like(self.adapter), torch.zeros_like(self.u)
        self.sample_workspace = mb.mdbf_sample_workspace(requests, self.VOCAB)

    def projected(self):
        mb.mdbf_adapter_rows(self.places.cu, self.adapter, self.rows.adapters, self.rows.tokens, out=self.rows)
        mb.mdbf_adapters(self.rows, self.pools, [self.X] * 3, self.qkv, workspace=self.adapter_workspaces[0])

    def step(self):
        mb.mdbf_add_norm(self.update, self.stream, self.weights[0], out=self.X, residual_out=self.between)
        super().step()
        mb.mdbf_adapters(self.rows, [self.pool_o], [self.out.flatten(1)], [self.Y], workspace=self.adapter_workspaces[1])
        mb.mdbf_add_norm(self.Y, self.between, self.weights[1], out=self.normed, residual_out=self.behind)
        mb.mdbf_forward(self.head, self.normed[self.last], y_dtype="f32", Y=self.logits, workspace=self.head_workspace)
        return mb.mdbf_sample(self.logits, self.u, self.temperature, self.top_k, self.top_p, tokens=self.tokens, probs=self.probs, workspace=self.sample_workspace)


def _run_block(torch, args, block):
    block.step()
    torch.cuda.synchronize()
    assert block.places.status.item() == 0 and bool(block.Y.isfinite().all())
    ms = _time(torch, block.step, args.warmup, args.passes)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.step()
    graph_ms = _time(torch, graph.replay, args.warmup, args.passes)
    return {"workload": args.workload, "requests": args.requests, "cached": args.cached, "fresh": args.fresh, "kv_heads": args.kv_heads,
            "budget_bpw": args.budget, "cache_MB": block.cache.buffer.numel() / 1e6, "ms_per_step": ms, "ms_per_step_from_a_graph": graph_ms}


def run_attention(torch, args):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(6)
    return _run_block(torch, args, AttentionBlock(torch, g, args.requests, args.cached, args.fresh, args.kv_heads, args.budget))


def run_step(torch, args):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(7)
    block = ServingStep(torch, g, args.requests, args.cached, args.fresh, args.kv_heads, args.budget, args.adapters, args.adapter_rank)
    return dict(_run_block(torch, args, block), adapters=args.adapters, adapter_rank=args.adapter_rank, vocab=block.VOCAB)


def main(argv=None):
    ap = argparse.ArgumentParser(prog="python3 -m paper_2512_24545_amd.workloads")
    ap.add_argument("workload", choices=["stack", "prefill", "attention", "step"])
    ap.add_argument("--budget", default="1.5", choices=["1.0", "1.5", "2.0"])
    ap.add_argument("--tokens", type=int, default=None)
    ap.add_argument("--x-dtype", default="f16", choices=["f16", "bf16"])
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--cached", type=int, default=4000)
    ap.add_argument("--fresh", type=int, default=1)
    ap.add_argument("--kv-heads", type=int, default=32, choices=[1, 2, 4, 8, 16, 32])
    ap.add_argument("--adapters", type=int, default=8)
    ap.add_argument("--adapter-rank", type=int, default=16)
    ap.add_argument("--passes", type=int, default=300)
    ap.add_argument("--warmup", type=int, default=100)
    args = ap.parse_args(argv)
    import torch
    if not torch.cuda.is_available():
        sys.exit("this program needs a GPU")
    mb.lib()
    if args.tokens is None:
        args.tokens = 8 if args.workload == "stack" else 2048
    out = {"stack": run_stack, "prefill": run_prefill, "attention": run_attention, "step": run_step}[args.workload](torch, args)
    print(json.dumps(out), flush=True)


if __name__ == "__main__":
    main()
