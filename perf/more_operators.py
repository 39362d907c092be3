"""What a serving step needs around its compressed projections besides attention, as measurable cases.

Operators of `paper_2512_24545_amd.binding`, called as a serving program calls them: the residual's addition with the
root-mean-square norm in front of the projections, in 16 or 32 bits or in 8 bits with scales (`norm`); the tables that put a
step's tokens in the order of their requests' low-rank adapters (`rows`), made once a step; the adapters' products, added to
what the shared projections have written (`adapters`); and the choice of the next tokens from the logits (`sample`).
With `own` false the same passes run as elementary torch operations in 32 bits, in 64 where a border decides: a scale of 8-bit
numbers, the mass of a token.

Sizes: 4096 and 11008 channels are the projections of the benchmark's workloads, 1601 one of its inner ranks; vocabularies,
adapter ranks and batches are generic.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"f16": 2, "bf16": 2, "f32": 4, "e4m3": 1}
EPS = 1e-6
TILE = 64          # rows of a tile of the adapters' tables


def _norm(name, T, n, x, h, y, group=0, pad=0):
    return dict(name=name, what="norm", T=T, n=n, x=x, h=h, y=y, group=group, pad=pad)


def _rows(name, requests, adapters, fresh):
    return dict(name=name, what="rows", requests=requests, adapters=adapters, fresh=fresh)


def _adapters(name, requests, adapters, fresh, r, n, m, count, x, y):
    return dict(name=name, what="adapters", requests=requests, adapters=adapters, fresh=fresh, r=r, n=n, m=m, count=count, x=x, y=y)


def _sample(name, T, V, x, top_k, top_p, min_p, masked=0.0):
    return dict(name=name, what="sample", T=T, V=V, x=x, top_k=top_k, top_p=top_p, min_p=min_p, masked=masked)


def listed():
    return [
        # a decode batch between two sublayers
        _norm("norm_decode", 64, 4096, "bf16", "bf16", "bf16"),
        # prompts in front of a product in 8 bits with a scale byte per 32 channels
        _norm("norm_prompts", 8192, 4096, "bf16", "bf16", "e4m3", group=32),
        # an odd width, a stream in 32 bits, rows with padding between them
        _norm("norm_odd", 777, 1601, "f16", "f32", "f16", pad=3),
        # a decode step of requests with adapters of their own or none
        _rows("rows_decode", 64, 32, 1),
        # many prompts
        _rows("rows_prompts", 500, 100, 1000),
        # a decode step's q, k and v: many adapters, few requests each
        _adapters("adapters_decode", 64, 32, 1, 16, 4096, 4096, 3, "bf16", "bf16"),
        # a large decode step's two projections into the MLP: few adapters of a high rank
        _adapters("adapters_shared", 256, 4, 1, 64, 4096, 11008, 2, "f16", "f16"),
        # odd everything, the projection's output in 32 bits
        _adapters("adapters_odd", 37, 9, 40, 5, 1601, 530, 1, "f16", "f32"),
        # prompts' q, k and v
        _adapters("adapters_prompts", 8, 5, 1500, 16, 4096, 4096, 3, "bf16", "bf16"),
        # one conversation, a wide vocabulary, the nucleus
        _sample("sample_one", 1, 128256, "f32", 0, 0.95, 0.0),
        # a batch of requests, each with its own settings, one of them greedy
        _sample("sample_batch", 64, 32000, "bf16", 50, 0.9, 0.02),
        # a large batch over a wide vocabulary, parts of it masked by grammars
        _sample("sample_wide", 200, 128256, "bf16", 0, 0.9, 0.0, masked=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["norm", "norm", "norm", "rows", "adapters", "adapters", "adapters", "sample", "sample", "sample"])
    if what == "norm":
        n = rng.choice([4096, 11008, _log_int(rng, 16, 16384), 8 * _log_int(rng, 2, 2000)])
        T, x, y = _log_int(rng, 1, 20_000_000 // n), rng.choice(["f16", "bf16", "bf16", "f32"]), rng.choice(["f16", "bf16", "f32", "e4m3", "e4m3"])
        return dict(what=what, T=T, n=n, x=x, h=rng.choice([x, "f32", "none"]), y=y, group=rng.choice([0, 32]) if y == "e4m3" else 0,
                    pad=rng.choice([0, 0, 1, 8, 40]))
    if what == "rows":
        return dict(what=what, requests=_log_int(rng, 1, 1500), adapters=_log_int(rng, 1, 500), fresh=rng.choice([1, 1, _log_int(rng, 2, 300)]))
    if what == "adapters":
        r, count = rng.choice([4, 8, 16, 16, 32, 64, 128, _log_int(rng, 1, 100)]), rng.choice([1, 1, 2, 3])
        n, m = (rng.choice([4096, 4096, 11008, 1024, _log_int(rng, 16, 8000), 8 * _log_int(rng, 2, 1000)]) for _ in range(2))
        adapters = _log_int(rng, 1, min(200, 100_000_000 // (count * r * (n + m))))
        most = 25_000_000 // (count * (n + m))
        fresh = rng.choice([1, 1, _log_int(rng, 2, max(2, min(1500, most)))])
        x = rng.choice(["f16", "bf16"])
        return dict(what=what, requests=max(1, min(_log_int(rng, 1, 300), 2 * most // (fresh + 1))), adapters=adapters, fresh=fresh, r=r, n=n, m=m, count=count,
                    x=x, y=rng.choice([x, x, "f32"]))
    V = rng.choice([32000, 128256, _log_int(rng, 50, 260000)])
    return dict(what=what, T=_log_int(rng, 1, min(1000, 25_000_000 // V)), V=V, x=rng.choice(["f16", "bf16", "f32", "f32"]),
                top_k=rng.choice([0, 0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 1.0, 0.5, 0.9, 0.99]), min_p=rng.choice([0.0, 0.0, 0.01, 0.1]),
                masked=rng.choice([0.0, 0.0, 0.3, 0.99]))


# ---------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, scale=1.0, pad=0):
    """Normal deviates of `shape` (rows, ...), rows `pad` elements apart."""
    x = torch.randn((shape[0], math.prod(shape[1:]) + pad), generator=g, device=DEV)
    x = (x * scale).to(DTYPES[dtype])
    return x[:, :x.shape[1] - pad].unflatten(1, shape[1:]) if len(shape) > 2 else x[:, :x.shape[1] - pad]


def _fresh(case):
    """New tokens of each request: one each in a decode step, prompts from the longest down to one, in no order."""
    B, most = case["requests"], case["fresh"]
    return [most if i == 0 or most == 1 else 1 + int((most - 1) * ((i * 0.6180339887) % 1.0)) for i in range(B)]


def _requests(g, case):
    """cu (first rows of the requests) and the adapter of each request; one in nine has none."""
    fresh = torch.tensor(_fresh(case), dtype=torch.int64, device=DEV)
    cu = torch.cat((fresh.new_zeros(1), torch.cumsum(fresh, 0))).to(torch.int32)
    adapter = torch.randint(0, case["adapters"], (case["requests"],), generator=g, device=DEV, dtype=torch.int32)
    none = torch.rand(case["requests"], generator=g, device=DEV) < 1 / 9
    return cu, torch.where(none, -1, adapter)


def _most_tiles(case):
    return sum(_fresh(case)) // TILE + min(case["adapters"], case["requests"])


def prepare(case, seed):
    g = _generator(seed)
    what = case["what"]
    s = dict(case=case)
    if what == "norm":
        T, n, pad = case["T"], case["n"], case["pad"]
        s["x"] = _normal(g, (T, n), case["x"], 1.0, pad)
        # the residual stream has a few channels far beyond the others
        large = 1 + 20 * (torch.rand(n, generator=g, device=DEV) < 0.01)
        if case["h"] != "none":
            s["h"] = (_normal(g, (T, n), "f32", 2.0, pad) * large).to(DTYPES[case["h"]])
            if pad:
                s["h"] = torch.cat((s["h"], s["h"][:, :pad]), 1)[:, :n]
        s["w"] = 1 + 0.1 * torch.randn(n, generator=g, device=DEV)
    elif what in ("rows", "adapters"):
        s["cu"], s["adapter"] = _requests(g, case)
        s["T"] = sum(_fresh(case))
        if what == "adapters":
            n, m, r, N = case["n"], case["m"], case["r"], case["adapters"]
            s["rows"], s["tiles"] = _tables(s)         # made once a step, for all layers
            s["x"] = _normal(g, (s["T"], n), case["x"])
            s["A"] = [_normal(g, (N, r, n), case["x"], n ** -0.5) for _ in range(case["count"])]
            s["B"] = [_normal(g, (N, m, r), case["x"], 0.1 * r ** -0.5) for _ in range(case["count"])]
            s["y"] = [_normal(g, (s["T"], m), case["y"]) for _ in range(case["count"])]
            s["scale"] = 0.5 + torch.rand(N, generator=g, device=DEV)
    else:
        T, V = case["T"], case["V"]
        # most tokens in a broad normal, some tens of likely ones above it, and more or less certain rows
        z = torch.randn((T, V), generator=g, device=DEV) * 2.2
        likely = torch.randint(0, V, (T, min(V, 40)), generator=g, device=DEV)
        z.scatter_add_(1, likely, 9 * torch.rand(likely.shape, generator=g, device=DEV))
        z *= 0.5 + torch.rand((T, 1), generator=g, device=DEV)
        if case["masked"]:
            z.masked_fill_((torch.rand((T, V), generator=g, device=DEV) < case["masked"]), float("-inf"))
        s["logits"] = z.to(DTYPES[case["x"]])
        row = torch.arange(T, device=DEV)
        s["u"] = torch.rand(T, generator=g, device=DEV)
        s["temperature"] = (0.5 + torch.rand(T, generator=g, device=DEV)) * (row % 64 != 63)      # one in 64 is greedy
        s["top_k"] = torch.full((T,), case["top_k"], dtype=torch.int32, device=DEV) * (row % 4 != 3) if case["top_k"] else None
        s["top_p"] = torch.where(row % 5 == 4, 1.0, case["top_p"]) if case["top_p"] < 1 else None
        s["min_p"] = torch.full((T,), case["min_p"], device=DEV) * (row % 3 != 2) if case["min_p"] else None
    return s


# ---------------------------------------------------------------- plain forms
def _plain_norm(s):
    """h = x + residual; y = h / sqrt(mean(h^2) + eps) * weight.  The mean in 64 bits: what is rounded to 8 bits afterwards
    goes by borders.  8-bit numbers are e4m3, of y over a scale: the row's largest over 448, or the least power of two that leaves
    the largest of 32 channels at most 448."""
    case, n = s["case"], s["case"]["n"]
    h = s["x"].float()
    if "h" in s:
        h = h + s["h"].float()
    r = ((h.double().square().sum(1, keepdim=True) / n + EPS).rsqrt()).float()
    y = h * r * s["w"]
    new_h = h.to(DTYPES[case["h"]]) if "h" in s else None
    if case["y"] != "e4m3":
        return y.to(DTYPES[case["y"]]), new_h, None
    if case["group"] == 0:
        scale = y.abs().amax(1, keepdim=True) / 448
        scale = torch.where(scale == 0, 1.0, scale)
        return (y / scale).to(torch.float8_e4m3fn), new_h, scale
    blocks = torch.nn.functional.pad(y, (0, -n % 32)).unflatten(1, (-1, 32))
    m, e = torch.frexp(blocks.abs().amax(2))                       # m in [0.5, 1); 448 = 0.875 * 2^9
    byte = torch.where(m == 0, 1, torch.where(m > 0.875, e + 1, e) - 9 + 127).clamp(1, 254)
    codes = torch.ldexp(blocks, (127 - byte)[..., None]).flatten(1)[:, :n]
    return codes.to(torch.float8_e4m3fn), new_h, byte.to(torch.uint8)


def _tables(s):
    """Rows by adapter, each adapter's in their order, -1 behind the last; tiles (adapter, first place, rows, 0) of up to TILE
    of them, no tile with rows of two adapters, (-1, 0, 0, 0) behind the last."""
    case, T = s["case"], s["T"]
    of = torch.repeat_interleave(s["adapter"].long(), torch.diff(s["cu"].long()), output_size=T)
    N = case["adapters"]
    key = torch.where(of < 0, N, of)
    order = torch.sort(key, stable=True).indices
    at = torch.arange(T, device=DEV)
    counts = torch.zeros(N + 1, dtype=torch.int64, device=DEV).scatter_add_(0, key, torch.ones_like(key))
    rows = torch.where(at < T - counts[N], order, -1).to(torch.int32)
    counts = counts[:N]
    first, of_tile = torch.cumsum(counts, 0) - counts, (counts + TILE - 1) // TILE
    ends = torch.cumsum(of_tile, 0)
    t = torch.arange(_most_tiles(case), device=DEV)
    a = torch.searchsorted(ends, t, right=True)
    there = a < N
    a = a.clamp(max=N - 1)
    done = (t - (ends - of_tile)[a]) * TILE
    tiles = torch.stack((a, first[a] + done, torch.minimum(counts[a] - done, torch.full_like(done, TILE)), torch.zeros_like(a)), 1)
    none = torch.tensor([-1, 0, 0, 0], device=DEV)
    return rows, torch.where(there[:, None], tiles, none).to(torch.int32)


def _plain_adapters(s):
    """y += scale[a] B[a] (A[a] x), a the adapter of the row's request: all adapters' inner values, those of others left out."""
    case = s["case"]
    N, r, m = case["adapters"], case["r"], case["m"]
    of = torch.repeat_interleave(s["adapter"].long(), torch.diff(s["cu"].long()), output_size=s["T"])
    mine = (of[:, None] == torch.arange(N, device=DEV))[:, :, None]
    x, factor = s["x"].float(), torch.where(of < 0, 0, s["scale"][of.clamp(min=0)])[:, None]
    for A, B, y in zip(s["A"], s["B"], s["y"]):
        inner = (x @ A.float().view(N * r, -1).T).view(-1, N, r)
        inner = torch.where(mine, inner, 0).view(-1, N * r)
        new = y.float() + factor * (inner @ B.float().transpose(1, 2).reshape(N * r, m))
        y.copy_(torch.where(of[:, None] < 0, y, new.to(y.dtype)))
    return s["y"]


def _plain_sample(s):
    """Tokens from the largest logit down, equal ones by index; weights exp((logit - largest) / temperature).  Kept are the first
    top_k; of those the least number whose weights add up to top_p of theirs; of those the ones with min_p of the largest weight.
    The token at the given number times the weight of all that are kept; a temperature of 0 takes the first."""
    z = s["logits"].double()
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    T, V = z.shape
    t = s["temperature"].double()[:, None]
    w = torch.exp((z - z[:, :1]) / torch.where(t > 0, t, 1.0))
    w = torch.where(z == float("-inf"), 0.0, w)
    rank = torch.arange(V, device=DEV)[None]
    keep = (rank == 0) | (t > 0)
    if s["top_k"] is not None:
        keep &= (rank < s["top_k"][:, None]) | (s["top_k"][:, None] <= 0)
    total = torch.cumsum(torch.where(keep, w, 0.0), 1)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        before = torch.cat((torch.zeros_like(t), total[:, :-1]), 1)
        keep &= (before < p * total[:, -1:]) | (p >= 1) | (rank == 0)
    if s["min_p"] is not None:
        keep &= (w >= s["min_p"].double()[:, None]) | (rank == 0)
    w = torch.where(keep, w, 0.0)
    total = torch.cumsum(w, 1)
    at = (total <= s["u"].double()[:, None] * total[:, -1:]).sum(1, keepdim=True).clamp(max=V - 1)
    token = order.gather(1, at).squeeze(1).to(torch.int32)
    prob = (w.gather(1, at) / total[:, -1:]).squeeze(1).float()
    none = z[:, 0] == float("-inf")
    return torch.where(none, -1, token), torch.where(none, 0.0, prob)


def run(s):
    case = s["case"]
    what = case["what"]
    if own:
        from paper_2512_24545_amd import binding as mb
        if what == "norm":
            return mb.mdbf_add_norm(s["x"], s.get("h"), s["w"], EPS, y_dtype=case["y"], scale_group=case["group"])
        if what == "rows":
            t = mb.mdbf_adapter_rows(s["cu"], s["adapter"], case["adapters"], s["T"])
            return t.rows, t.tiles
        if what == "adapters":
            t = mb.AdapterRows(s["T"], case["requests"], case["adapters"], rows=s["rows"], tiles=s["tiles"])
            mb.mdbf_adapters(t, [mb.Adapters(A, B, s["scale"]) for A, B in zip(s["A"], s["B"])], [s["x"]] * case["count"], s["y"])
            return s["y"]
        return mb.mdbf_sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    if what == "norm":
        return _plain_norm(s)
    if what == "rows":
        return _tables(s)
    if what == "adapters":
        return _plain_adapters(s)
    return _plain_sample(s)


def work(case):
    what = case["what"]
    if what == "norm":
        T, n = case["T"], case["n"]
        a_channel = BYTES[case["x"]] + BYTES[case["y"]] + 2 * BYTES.get(case["h"], 0)
        scales = 0 if case["y"] != "e4m3" else T * -(-n // 32) if case["group"] else 4 * T
        return {"bytes": T * n * a_channel + 4 * n + scales, "flops": 6 * T * n}
    T = sum(_fresh(case)) if what != "sample" else case["T"]
    if what == "rows":
        return {"bytes": 8 * case["requests"] + 4 * T + 16 * _most_tiles(case), "flops": 0}
    if what == "adapters":
        # of the requests eight in nine have an adapter; as many of the adapters are in use as that many throws hit
        N, n, m, r, e = case["adapters"], case["n"], case["m"], case["r"], BYTES[case["x"]]
        used, T = N * (1 - (1 - 1 / N) ** (case["requests"] * 8 / 9)), T * 8 / 9
        return {"bytes": T * n * e + case["count"] * (used * r * (n + m) * e + 2 * T * m * BYTES[case["y"]]),
                "flops": 2 * T * r * (n + m) * case["count"]}
    return {"bytes": T * case["V"] * BYTES[case["x"]] + 28 * T, "flops": 10 * T * case["V"]}


# ---------------------------------------------------------------- the definitions in 64 bits
def _e4m3(v):
    """The nearest e4m3 numbers, ties to even; what rounds beyond 448 stays there."""
    m, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), e.clamp(min=-5) - 4)
    return (torch.round(v / step) * step).clamp(-448, 448)


def _exact_norm(s):
    case, n = s["case"], s["case"]["n"]
    h = s["x"].double() + s["h"].double() if "h" in s else s["x"].double()
    y = h * s["w"].double() / torch.linalg.vector_norm(torch.cat((h / math.sqrt(n), torch.full_like(h[:, :1], math.sqrt(EPS))), 1), dim=1, keepdim=True)
    new_h = h if "h" in s else None
    if case["y"] != "e4m3":
        return y, new_h, None
    if case["group"] == 0:
        scale = y.abs().max(1, keepdim=True).values / 448
        return _e4m3(y / scale.where(scale > 0, torch.ones_like(scale))), new_h, scale
    out = torch.empty_like(y)
    for first in range(0, n, 32):
        part = y[:, first:first + 32]
        scale = torch.exp2(torch.ceil(torch.log2(part.abs().max(1, keepdim=True).values / 448)).clamp(-126, 127))
        out[:, first:first + 32] = _e4m3(part / scale)
    return out, new_h, None


def _exact_adapters(s):
    """Request by request."""
    out = [y.double() for y in s["y"]]
    cu = s["cu"].tolist()
    for r, a in enumerate(s["adapter"].tolist()):
        if a >= 0:
            x = s["x"][cu[r]:cu[r + 1]].double()
            for A, B, y in zip(s["A"], s["B"], out):
                y[cu[r]:cu[r + 1]] += (x @ A[a].double().T) @ B[a].double().T * s["scale"][a].double()
    return out


def _exact_sample(s):
    """Row by row over the different values and how often each occurs."""
    T = s["logits"].shape[0]
    tokens, probs = [], []
    setting = {k: (s[k].double().tolist() if s[k] is not None else [v] * T) for k, v in (("temperature", 1.0), ("top_k", 0), ("top_p", 1.0), ("min_p", 0.0), ("u", 0))}
    for i in range(T):
        row = s["logits"][i].double()
        t, k, p, least, u = (setting[n][i] for n in ("temperature", "top_k", "top_p", "min_p", "u"))
        values, times = torch.unique(row[row > float("-inf")], return_counts=True)
        if not len(values):
            tokens.append(-1), probs.append(0.0)
            continue
        values, times = values.flip(0), times.flip(0).double()
        if t <= 0:
            k, t, u = 1, 1.0, 0.0
        weight = torch.exp((values - values[0]) / t)
        before = torch.cumsum(times, 0) - times
        kept = (k - before).clamp(min=0).minimum(times) if k > 0 else times

        def below(kept):
            mass = torch.cumsum(kept * weight, 0)
            return mass - kept * weight, mass[-1]

        if p < 1:
            base, total = below(kept)
            kept = torch.ceil((p * total - base) / weight).clamp(min=0).minimum(kept)
            kept[0] = kept[0].clamp(min=1)
        kept = torch.where(weight >= least, kept, torch.zeros_like(kept))
        base, total = below(kept)
        j = int((base + kept * weight <= u * total).sum())
        equal = torch.nonzero(row == values[j]).flatten()
        tokens.append(int(equal[min(int((u * total - base[j]) / weight[j]), len(equal) - 1)]))
        probs.append(float(weight[j] / total))
    return torch.tensor(tokens, device=DEV, dtype=torch.int32), torch.tensor(probs, device=DEV, dtype=torch.float64)


def exact(case, seed):
    what = case["what"]
    if what == "rows":
        return None                    # whole numbers: the plain form is the definition
    if what == "sample" and case["T"] > 500:
        return None
    s = prepare(case, seed)
    if what == "norm":
        return _exact_norm(s)
    if what == "adapters":
        return _exact_adapters(s)
    return _exact_sample(s)
