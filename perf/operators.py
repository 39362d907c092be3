"""The operators of an attention block over a 4-bit paged cache, as measurable cases.

Four operators of `paper_2512_24545_amd.binding`, called as a serving program calls them between the projections of a
compressed decoder layer: block tables and slot maps from request lengths (`slots`), norm and rotation of queries and
keys (`rope`), keys and values into the cache and back (`append`), attention over the cache for single tokens and for
prompts (`attention`).  With `own` false the same passes run as elementary torch operations in 32 bits.

The cache is a pool of pages.  A page holds, for each kv head in turn, its tokens' key codes, value codes, key scales and
value scales: codes are 4-bit floating point numbers (e2m1, the even channel in the low half of a byte), one scale
byte b per 32 channels stands for 2^(b - 127), and 255 for a block that was not finite.

Sizes: 32 heads of 128 channels are the benchmark's attention layers (4096 x 4096); fewer kv heads, other head sizes and
odd counts are generic.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
SCALE_RANGE = {"f16": (104, 140), "bf16": (2, 252), "f32": (2, 252)}   # what the values' type can hold exactly
EPS = 1e-6


def _slots(name, B, P, cached, fresh):
    return dict(name=name, what="slots", B=B, P=P, cached=cached, fresh=fresh)


def _rope(name, T, Hq, Hkv, d, rot, x, y, inter=False, pad=0):
    return dict(name=name, what="rope", T=T, Hq=Hq, Hkv=Hkv, d=d, rot=rot, x=x, y=y, inter=inter, pad=pad)


def _append(name, T, Hkv, d, P, x, pad=0):
    return dict(name=name, what="append", T=T, Hkv=Hkv, d=d, P=P, x=x, pad=pad)


def _attention(name, B, Hq, Hkv, d, P, x, cached, fresh, window=0):
    return dict(name=name, what="attention", B=B, Hq=Hq, Hkv=Hkv, d=d, P=P, x=x, cached=cached, fresh=fresh, window=window)


def listed():
    return [
        # a decode step of 64 requests: one new token each, small pages; latency counts
        _slots("slots_decode", 64, 16, 8191, 1),
        # prompts of 500 requests join at once
        _slots("slots_prompts", 500, 64, 3000, 1000),
        # the queries and keys of a decode step, four queries to a key
        _rope("rope_decode", 64, 32, 8, 128, 128, "bf16", "bf16"),
        # a batch of prompts with as many keys as queries
        _rope("rope_prompts", 8192, 32, 32, 128, 128, "bf16", "bf16"),
        # odd counts, small heads, neighbouring pairs, half of the channels rotated, out of a joint qkv matrix in fp32
        _rope("rope_odd", 777, 14, 2, 64, 32, "f32", "f16", inter=True, pad=131),
        # the keys and values of a decode step, and a look at what was stored
        _append("append_decode", 64, 8, 128, 16, "bf16"),
        # those of a batch of prompts
        _append("append_prompts", 8192, 32, 128, 64, "f16"),
        # a few short conversations, a key per query, small pages
        _attention("attn_decode_short", 4, 32, 32, 128, 16, "f16", 700, 1),
        # a full decode batch of mixed lengths
        _attention("attn_decode_batch", 64, 32, 8, 128, 64, "bf16", 8191, 1),
        # one request over a very long cache
        _attention("attn_decode_long", 1, 32, 8, 128, 256, "bf16", 199999, 1),
        # prompts of odd lengths behind cached prefixes, small heads, a sliding window
        _attention("attn_prompts_odd", 5, 14, 2, 64, 32, "f16", 1501, 997, window=1111),
        # a piece of a long prompt
        _attention("attn_prompt_long", 1, 32, 8, 128, 64, "bf16", 14336, 2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["slots", "rope", "append", "decode", "decode", "decode", "prompt", "prompt", "prompt"])
    Hq, Hkv = rng.choice([(32, 32), (32, 8), (32, 8), (14, 2), (28, 4), (8, 1), (12, 12), (48, 3)])
    d, P = rng.choice([64, 128, 128, 256]), rng.choice([16, 32, 64, 128, 256])
    if what == "slots":
        return dict(what="slots", B=_log_int(rng, 1, 1500), P=P, cached=_log_int(rng, 1, 8000), fresh=rng.choice([1, 1, _log_int(rng, 2, 400)]))
    if what in ("rope", "append"):
        T, x = _log_int(rng, 1, 300000 // (Hkv + Hq)), rng.choice(["f16", "bf16", "bf16", "f32"])
        pad = rng.choice([0, 0, 1, 8, 40])
        if what == "append":
            return dict(what="append", T=T, Hkv=Hkv, d=d, P=P, x=x, pad=pad)
        return dict(what="rope", T=T, Hq=Hq, Hkv=Hkv, d=d, rot=rng.choice([d, d, d // 2, 16]), x=x, y=rng.choice([x, "bf16", "f16"]),
                    inter=rng.random() < 0.3, pad=pad)
    x, window = rng.choice(["f16", "bf16"]), rng.choice([0, 0, 0, _log_int(rng, 8, 4096)])
    if what == "decode":
        fresh, longest = rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 16, 100000)
        B = max(1, min(_log_int(rng, 1, 128), 300_000_000 // (longest * Hkv * d)))
    else:
        fresh, longest = _log_int(rng, 17, 1500), _log_int(rng, 1, 8000)
        B = max(1, min(rng.choice([1, 1, 2, 3, 7]), 16_000_000_000 // ((longest + fresh) * fresh * Hq * d)))
    return dict(what="attention", B=B, Hq=Hq, Hkv=Hkv, d=d, P=P, x=x, cached=longest, fresh=fresh, window=window)


# ---------------------------------------------------------------- inputs
def _spread(longest, least, count):
    """`count` lengths from the longest down, spread in no order over least .. longest."""
    return [longest if i == 0 else least + int((longest - least) * ((i * 0.6180339887) % 1.0)) for i in range(count)]


def _lengths(case):
    """(cached, fresh) of each request: a decode step has as many new tokens everywhere, prompts have their own."""
    B = case["B"]
    fresh = [case["fresh"]] * B if case["fresh"] <= 8 else _spread(case["fresh"], 1, B)
    return _spread(case["cached"], 0, B), fresh


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _token_bytes(d):
    """Bytes of one token of one kv head: codes and scales of its key and its value."""
    return d + d // 16


def _tables(g, B, pages_of, width, spare):
    """Block tables of requests that hold pages_of[r] pages each, -1 behind them, and the pages that are free, in no order."""
    total = sum(pages_of)
    perm = torch.randperm(total + spare, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    idx = torch.arange(width, device=DEV)
    of = torch.tensor(pages_of, device=DEV)
    first = torch.cumsum(of, 0) - of
    held = idx[None] < of[:, None]
    table[held] = perm[(first[:, None] + idx[None])[held]]
    return table, perm[total:].contiguous()


def _rows(g, T, H, d, dtype, pad):
    """T x H x d, rows `pad` elements apart: as they lie in a wider matrix."""
    wide = torch.randn((T, H * d + pad), generator=g, device=DEV).to(DTYPES[dtype])
    return wide[:, :H * d].unflatten(1, (H, d))


def _pool(g, pages, Hkv, P, d, dtype):
    """Pages of normally distributed keys and values, the scale of each head's channels its own."""
    pool = torch.empty((pages, Hkv, P * _token_bytes(d)), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 27) // (Hkv * P * d * 2))
    for p0 in range(0, pages, step):
        n = min(step, pages - p0)
        size = torch.exp(0.5 * torch.randn((1, Hkv, 1, 1, d), generator=g, device=DEV))
        x = torch.randn((n, Hkv, 2, P, d), generator=g, device=DEV) * size
        codes, scales = _quantise(x, dtype)
        both = codes[..., 0::2] | (codes[..., 1::2] << 4)
        pool[p0:p0 + n, :, :P * d] = both.reshape(n, Hkv, P * d)
        pool[p0:p0 + n, :, P * d:] = scales.reshape(n, Hkv, P * d // 16)
    return pool.view(-1)


def prepare(case, seed):
    g, what = _generator(seed), case["what"]
    s = dict(case=case)
    if what == "slots":
        cached, fresh = _lengths(case)
        P = case["P"]
        before = [-(-c // P) for c in cached]
        new = sum(-(-(c + f) // P) for c, f in zip(cached, fresh)) - sum(before)
        s["table"], s["free"] = _tables(g, case["B"], before, max(-(-(c + f) // P) for c, f in zip(cached, fresh)) + 3, new + 9)
        s.update(cached=_ints(cached), fresh=_ints(fresh), taken=_ints([4]), tokens=sum(fresh) + 5)
    elif what == "rope":
        T, d, rot = case["T"], case["d"], case["rot"]
        qkv = _rows(g, T, case["Hq"] + case["Hkv"], d, case["x"], case["pad"])
        rows = 4096
        angle = torch.arange(rows, device=DEV).double()[:, None] * 10000.0 ** (-torch.arange(rot // 2, device=DEV).double() * 2 / rot)
        s.update(q=qkv[:, :case["Hq"]], k=qkv[:, case["Hq"]:], rope=torch.cat([angle.cos(), angle.sin()], 1).float(),
                 positions=torch.randint(0, rows, (T,), generator=g, device=DEV, dtype=torch.int32),
                 qw=1 + 0.2 * torch.randn((d,), generator=g, device=DEV), kw=1 + 0.2 * torch.randn((d,), generator=g, device=DEV))
        s.update(q_out=torch.empty((T, case["Hq"], d), dtype=DTYPES[case["y"]], device=DEV),
                 k_out=torch.empty((T, case["Hkv"], d), dtype=DTYPES[case["y"]], device=DEV))
    elif what == "append":
        T, Hkv, d, P = case["T"], case["Hkv"], case["d"], case["P"]
        pages = T // P + 5
        s.update(k=_rows(g, T, Hkv, d, case["x"], case["pad"]), v=_rows(g, T, Hkv, d, case["x"], case["pad"]),
                 slots=torch.randperm(pages * P, generator=g, device=DEV)[:T].sort().values,
                 pool=torch.zeros(pages * P * Hkv * _token_bytes(d), dtype=torch.uint8, device=DEV))
        value = DTYPES["f16" if case["x"] == "f16" else "bf16"]
        s["back"] = tuple(torch.empty((T, Hkv, d), dtype=value, device=DEV) for _ in range(2))
        if own:
            from paper_2512_24545_amd import binding as mb
            s["cache"] = mb.KVCache(pages, Hkv, d, P, "f16" if case["x"] == "f16" else "bf16", buffer=s["pool"])
    else:
        B, Hq, Hkv, d, P = (case[n] for n in ("B", "Hq", "Hkv", "d", "P"))
        cached, fresh = _lengths(case)
        lengths = [c + f for c, f in zip(cached, fresh)]
        of = [-(-n // P) for n in lengths]
        s["table"], _ = _tables(g, B, of, max(of) + 1, 2)
        s["pool"] = _pool(g, sum(of) + 2, Hkv, P, d, case["x"])
        cu = [0]
        for f in fresh:
            cu.append(cu[-1] + f)
        s.update(cu=_ints(cu), lengths=_ints(lengths), q=_rows(g, cu[-1], Hq, d, case["x"], 0), longest=max(lengths), most=max(fresh),
                 out=torch.empty((cu[-1], Hq, d), dtype=DTYPES[case["x"]], device=DEV))
        if own:
            from paper_2512_24545_amd import binding as mb
            s["cache"] = mb.KVCache(sum(of) + 2, Hkv, d, P, case["x"], buffer=s["pool"])
            s["workspace"] = mb.mdbf_kv_attention_workspace(s["cache"], Hq, B, cu[-1], max(fresh), max(lengths), window=case["window"])
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    what = state["case"]["what"]
    if own:
        return {"slots": _own_slots, "rope": _own_rope, "append": _own_append, "attention": _own_attention}[what](state)
    return {"slots": _plain_slots, "rope": _plain_rope, "append": _plain_append, "attention": _plain_attention}[what](state)


def _own_slots(s):
    from paper_2512_24545_amd import binding as mb
    r = mb.mdbf_kv_slots(s["cached"], s["fresh"], s["table"], s["free"], s["taken"], s["case"]["P"], s["tokens"])
    return dict(lengths=r.lengths, cu=r.cu, slots=r.slots, positions=r.positions, taken=r.taken, status=r.status, table=s["table"])


def _own_rope(s):
    from paper_2512_24545_amd import binding as mb
    return mb.mdbf_qk_norm_rope(s["q"], s["k"], s["rope"], s["positions"], q_weight=s["qw"], k_weight=s["kw"], eps=EPS,
                                interleaved=s["case"]["inter"], q_out=s["q_out"], k_out=s["k_out"])


def _own_append(s):
    from paper_2512_24545_amd import binding as mb
    mb.mdbf_kv_append(s["cache"], s["k"], s["v"], s["slots"])
    return mb.mdbf_kv_read(s["cache"], s["slots"], out=s["back"])


def _own_attention(s):
    from paper_2512_24545_amd import binding as mb
    return mb.mdbf_kv_attention(s["cache"], s["q"], s["table"], s["cu"], s["lengths"], s["most"], s["longest"], causal=True,
                                window=s["case"]["window"], out=s["out"], workspace=s["workspace"])


# ---------------------------------------------------------------- the plain forms
def _plain_slots(s):
    P, tokens, table = s["case"]["P"], s["tokens"], s["table"]
    cached, fresh, taken = s["cached"].long(), s["fresh"].long(), s["taken"].long()
    before, after = (cached + P - 1) // P, (cached + fresh + P - 1) // P
    need = after - before
    base = taken + torch.cumsum(need, 0) - need
    cu = torch.cat([torch.zeros_like(taken), torch.cumsum(fresh, 0)])
    idx = torch.arange(table.shape[1], device=DEV)[None]
    new = (idx >= before[:, None]) & (idx < after[:, None])
    page = s["free"][(base[:, None] + idx - before[:, None]).clamp(0, s["free"].shape[0] - 1)]
    table = torch.where(new, page, table)
    t = torch.arange(tokens, device=DEV)
    r = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=cached.shape[0] - 1)
    pos = cached[r] + t - cu[r]
    real = t < cu[-1]
    at = table[r, (pos // P).clamp(max=table.shape[1] - 1)].long() * P + pos % P
    wrong = (cached < 0).any() | (fresh < 0).any()
    status = 1 * wrong + 2 * (after > table.shape[1]).any() + 4 * (cu[-1] > tokens) + 8 * (taken[0] + need.sum() > s["free"].shape[0])
    return dict(lengths=(cached + fresh).int(), cu=cu.int(), slots=torch.where(real, at, -1), positions=torch.where(real, pos, -1).int(),
                taken=(taken + need.sum()).int(), status=status.int().view(1), table=table)


def _turned(x, weight, table, positions, rot, inter):
    x = x.float()
    x = x * torch.rsqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight
    row = table[positions.long()][:, None]
    c, s = row[..., :rot // 2], row[..., rot // 2:]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * c - b * s, b * c + a * s
    turned = torch.stack([ra, rb], -1).flatten(-2) if inter else torch.cat([ra, rb], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_rope(s):
    case = s["case"]
    return tuple(_turned(s[n], s[n + "w"], s["rope"], s["positions"], case["rot"], case["inter"]).to(DTYPES[case["y"]]) for n in ("q", "k"))


def _quantise(x, dtype):
    """4-bit codes (uint8, one per entry) and scale bytes (one per 32) of x in fp32: the block's largest magnitude comes to lie in
    (3.5, 7] in units of its scale where the type's range allows it; a code is the nearest number, ties to the even one."""
    blocks = x.unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    bits = top.contiguous().view(torch.int32)
    lo, hi = SCALE_RANGE[dtype]
    scale = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x600000)).clamp(lo, hi)
    a = blocks.abs() * ((254 - scale) << 23).view(torch.float32)[..., None]
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)) | ((blocks < 0).to(torch.uint8) << 3)
    scale = torch.where(torch.isfinite(top), scale, 255)
    return code.flatten(-2).to(torch.uint8), scale.to(torch.uint8)


_LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values(codes, scales):
    """What codes (one per entry) and scale bytes (one per 32) stand for, in fp32."""
    level = torch.tensor(_LEVELS + [-v for v in _LEVELS], device=codes.device)
    size = torch.where(scales == 255, float("nan"), (scales.int() << 23).view(torch.float32))
    return (level[codes.int()].unflatten(-1, (-1, 32)) * size[..., None]).flatten(-2)


def _plain_append(s):
    x = s["case"]["x"]
    value = DTYPES["f16" if x == "f16" else "bf16"]
    return tuple(_values(*_quantise(s[n].float(), x)).to(value) for n in ("k", "v"))


def _unpacked(pages, P, d):
    """Keys and values (... x P x d, fp32) of pages given as bytes (... x P * token bytes)."""
    both = pages[..., :P * d].unflatten(-1, (2, P, d // 2))
    codes = torch.stack([both & 15, both >> 4], -1).flatten(-2)
    x = _values(codes, pages[..., P * d:].unflatten(-1, (2, P, d // 32)))
    return x[..., 0, :, :], x[..., 1, :, :]


def _plain_attention(s):
    case = s["case"]
    B, Hq, Hkv, d, P = (case[n] for n in ("B", "Hq", "Hkv", "d", "P"))
    G, L, most, cu, lengths = Hq // Hkv, s["longest"], s["most"], s["cu"].long(), s["lengths"].long()
    pool = s["pool"].view(-1, Hkv, P * _token_bytes(d))
    k, v = _unpacked(pool[s["table"][:, :-(-L // P)].clamp(min=0).long()], P, d)      # B x pages x Hkv x P x d
    k, v = (x.transpose(1, 2).flatten(2, 3)[:, :, :L].contiguous() for x in (k, v))
    j, i = torch.arange(L, device=DEV), torch.arange(most, device=DEV)
    fresh = cu[1:] - cu[:-1]
    pos = (lengths - fresh)[:, None] + i                                              # B x most
    sees = (j <= pos[..., None]) & (j < lengths[:, None, None])
    if case["window"]:
        sees &= j > pos[..., None] - case["window"]
    q = s["q"][(cu[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)].float() * d ** -0.5  # B x most x Hq x d
    q = q.unflatten(2, (Hkv, G)).permute(0, 2, 3, 1, 4).flatten(2, 3).contiguous()
    z = torch.matmul(q, k.transpose(2, 3).contiguous()).unflatten(2, (G, most))
    z = torch.where(sees[:, None, None], z, float("-inf"))
    p = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-3e38))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-38)
    v = torch.where((j < lengths[:, None])[:, None, :, None], v, 0.0)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (G, most))                       # B x Hkv x G x most x d
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)
    t = torch.arange(s["q"].shape[0], device=DEV)
    r = torch.searchsorted(cu, t, right=True) - 1
    return o[r, t - cu[r]].to(DTYPES[case["x"]])


# ---------------------------------------------------------------- what a pass cannot do without
def _pairs(case):
    """(cached tokens that some new token sees, pairs of a new token and one it sees), over all requests."""
    seen = pairs = 0
    for c, f in zip(*_lengths(case)):
        w = case["window"] or c + f
        seen += c + f - max(0, c + 1 - w)
        pairs += sum(min(c + i + 1, w) for i in range(f))
    return seen, pairs


def work(case):
    what = case["what"]
    if what == "slots":
        cached, fresh = _lengths(case)
        new = sum(-(-(c + f) // case["P"]) - -(-c // case["P"]) for c, f in zip(cached, fresh))
        return dict(bytes=16 * case["B"] + 12 * sum(fresh) + 8 * new, flops=0)
    if what == "rope":
        n = case["T"] * (case["Hq"] + case["Hkv"]) * case["d"]
        return dict(bytes=n * (BYTES[case["x"]] + BYTES[case["y"]]) + case["T"] * 4 * (case["rot"] + 1), flops=8 * n)
    if what == "append":   # read, stored, read again and written out
        n = case["T"] * case["Hkv"] * case["d"]
        return dict(bytes=2 * n * (BYTES[case["x"]] + 2) + 2 * case["T"] * case["Hkv"] * _token_bytes(case["d"]) + 16 * case["T"], flops=0)
    seen, pairs = _pairs(case)
    tokens = sum(_lengths(case)[1])
    return dict(bytes=seen * case["Hkv"] * _token_bytes(case["d"]) + 4 * tokens * case["Hq"] * case["d"],
                flops=4 * pairs * case["Hq"] * case["d"])


# ---------------------------------------------------------------- the same in 64 bits
_E2M1 = [s * m for s in (1.0, -1.0) for m in (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)]


def _exact_append(x, dtype):
    lo, hi = SCALE_RANGE[dtype]
    x = x.double().unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))           # m in [0.5, 1)
    e = torch.where(m > 0.875, e - 2, e - 3).clamp(lo - 127, hi - 127)
    unit = torch.ldexp(torch.ones_like(m), e)
    # the nearest number, ties to the even one: a grid of halves up to 2, of ones up to 4, of twos above
    a = (x / unit).abs()
    near = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2)).clamp(max=6)
    return (torch.sign(x) * near * unit).flatten(-2)


def _exact_rope(s):
    case, out = s["case"], []
    rot, h = case["rot"], case["rot"] // 2
    angle = s["rope"].double()[s["positions"].long()]
    turn = torch.complex(angle[:, :h], angle[:, h:])[:, None]
    for name in ("q", "k"):
        x = s[name].double()
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * s[name + "w"].double()
        first, second = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["inter"] else (x[..., :h], x[..., h:rot])
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        y = x.clone()
        if case["inter"]:
            y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
        else:
            y[..., :h], y[..., h:rot] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_attention(s):
    """Request by request and kv head by kv head, from the bytes of the pages."""
    case = s["case"]
    Hkv, d, P = case["Hkv"], case["d"], case["P"]
    G, half = case["Hq"] // Hkv, P * d // 2
    pool, level = s["pool"].view(-1, Hkv, P * _token_bytes(d)), torch.tensor(_E2M1, dtype=torch.float64, device=DEV)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)

    def read(codes, scales, n):
        codes, scales = codes.reshape(-1, d // 2), scales.reshape(-1, d // 32)
        x = torch.empty((codes.shape[0], d), dtype=torch.float64, device=DEV)
        x[:, 0::2], x[:, 1::2] = level[(codes & 15).long()], level[(codes >> 4).long()]
        return (x * torch.exp2(scales.double() - 127).repeat_interleave(32, 1))[:n]

    first = 0
    for r, (c, f) in enumerate(zip(*_lengths(case))):
        n = c + f
        pages = pool[s["table"][r, :-(-n // P)].long()]
        at = c + torch.arange(f, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)[None]
        hidden = (j > at) | (j <= at - case["window"]) if case["window"] else j > at
        for h in range(Hkv):
            page = pages[:, h]
            k = read(page[:, :half], page[:, P * d:P * d + P * d // 32], n)
            v = read(page[:, half:P * d], page[:, P * d + P * d // 32:], n)
            kt = k.T.contiguous()
            for g in range(G):
                x = s["q"][first:first + f, h * G + g].double()
                z = (x @ kt / math.sqrt(d)).masked_fill(hidden, float("-inf"))
                out[first:first + f, h * G + g] = torch.softmax(z, 1) @ v
        first += f
    return out


def exact(case, seed):
    what = case["what"]
    if what == "slots":
        return None                    # whole numbers: the plain form is the definition
    if what == "attention" and case["B"] * case["Hq"] > 20000:
        return None
    s = prepare(case, seed)
    if what == "rope":
        return _exact_rope(s)
    if what == "append":
        return tuple(_exact_append(s[n], case["x"]) for n in ("k", "v"))
    return _exact_attention(s)
