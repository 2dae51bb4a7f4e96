"""The attention of a drafter's layer, as a speculative-decoding program has this library do it.

Before a draft step there is the drafter's own layer: norms of queries and keys for each head with the position
rotation, keys and values written into a paged cache (as bf16, or as e4m3 with a power-of-two scale for each token and
head), and the attention of the new tokens -- one for each request, or the nodes of a tree level -- over what is cached.
A drafter is trained as well: the norms and the rotation have their backward pass.

Layouts.  q [n, q_heads, D], k and v [n, kv_heads, D]: views of one projection's output rows.  The cache: k and v
[pages, kv_heads, page, D], scale exponents [pages, kv_heads, page] (the scale is 2^(byte - 127)).  Token t of a
request is at page_table[request, t // page], place t % page; a slot is page number * page + place.  The rotation's
table is [positions, rotary dims]: cosines in its first half, sines in the second.  A row's tail mask says which of the
last 64 cached tokens it sees: bit j is token length - 64 + j.
"""
import torch

own = False      # set by whoever measures: run() then makes the calls of this library

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZES = {"bf16": 2, "f32": 4, "e4m3": 1}
EPS = 1e-6
E4M3_MAX = 448.0

# Drawn cases cost at most what the largest listed ones do.
MAX_NORM_VALUES = 8192 * 40 * 128
MAX_WRITE_VALUES = 8192 * 48 * 128
MAX_READ_VALUES = 65537 * 8 * 128
MAX_CACHED_VALUES = 48 * 16384 * 8 * 128 // 2
MAX_SCORES = 131072 * 32 * 32


def listed():
    return [
        # a prompt's queries and keys on an 8B model's layer, no cache: training, or a prefill that keeps its own
        {"name": "norm prompt", "op": "norm", "dtype": "bf16", "n": 4096, "hq": 32, "hk": 8, "D": 128, "rot": 128, "interleaved": False},
        # an fp32 toy model: odd head counts, a head size that is no power of two, part of it rotated, neighbours paired
        {"name": "norm toy fp32", "op": "norm", "dtype": "f32", "n": 333, "hq": 6, "hk": 2, "D": 96, "rot": 64, "interleaved": True},
        # the same layer's gradients over a training batch
        {"name": "norm gradients", "op": "grad", "dtype": "bf16", "n": 8192, "hq": 32, "hk": 8, "D": 128, "rot": 128, "interleaved": False},
        # gradients of a toy model in fp32
        {"name": "norm gradients toy fp32", "op": "grad", "dtype": "f32", "n": 777, "hq": 8, "hk": 8, "D": 64, "rot": 32, "interleaved": False},
        # one token of one request goes into the cache: nothing but latency
        {"name": "write one token", "op": "write", "dtype": "bf16", "cache": "e4m3", "n": 1, "hq": 32, "hk": 8, "D": 128, "rot": 128,
         "interleaved": False, "page": 64},
        # a long prompt goes into the cache and is read back
        {"name": "write prompt", "op": "write", "dtype": "bf16", "cache": "e4m3", "n": 8192, "hq": 32, "hk": 8, "D": 128, "rot": 128,
         "interleaved": False, "page": 64},
        # cached rows of many requests read back, for a prefill that attends in 16 bits
        {"name": "read back", "op": "read", "out": "bf16", "cache": "e4m3", "n": 65537, "hk": 8, "D": 128, "page": 64},
        # one token of an fp32 toy model with a short prompt: the smallest attention
        {"name": "attend toy fp32", "op": "attend", "dtype": "f32", "cache": "bf16", "hq": 4, "hk": 2, "D": 64, "page": 16, "requests": 1,
         "rows": 1, "length": 300},
        # chain drafting for one request, 8B layer: the most frequent call
        {"name": "attend chain", "op": "attend", "dtype": "bf16", "cache": "bf16", "hq": 32, "hk": 8, "D": 128, "page": 64, "requests": 1,
         "rows": 1, "length": 2500},
        # a tree level of up to eight nodes for each of four requests; a node sees its ancestors only
        {"name": "attend tree", "op": "attend", "dtype": "bf16", "cache": "bf16", "hq": 32, "hk": 8, "D": 128, "page": 64, "requests": 4,
         "rows": 8, "length": 4133},
        # a serving batch of ragged requests, one of them empty
        {"name": "attend batch", "op": "attend", "dtype": "bf16", "cache": "e4m3", "hq": 32, "hk": 8, "D": 128, "page": 32, "requests": 48,
         "rows": 1, "length": 16384},
        # one request with a very long context
        {"name": "attend long", "op": "attend", "dtype": "bf16", "cache": "bf16", "hq": 32, "hk": 8, "D": 128, "page": 64, "requests": 1,
         "rows": 1, "length": 131001},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choices(["norm", "grad", "write", "read", "attend"], [2, 2, 3, 1, 6])[0]
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    cache = rng.choice(["bf16", "e4m3"])
    while True:
        hk = rng.choice([1, 2, 4, 8, 8, 8, 16])
        hq = hk * rng.choice([1, 2, 3, 4, 4, 7, 8])
        D = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
        if hq <= 64:
            break
    page = rng.choice([16, 32, 64, 64, 128, 256])
    if op == "attend":
        while True:
            requests, rows = _log_uniform(rng, 1, 64), rng.choice([1, 1, 1, 2, 5, 8, 16])
            length = _log_uniform(rng, 1, 131072)
            if requests * length * hk * D <= MAX_CACHED_VALUES and requests * rows * hq * length <= MAX_SCORES:
                break
        return {"op": op, "dtype": dtype, "cache": cache, "hq": hq, "hk": hk, "D": D, "page": page, "requests": requests, "rows": rows,
                "length": length}
    if op == "read":
        return {"op": op, "out": rng.choice(["bf16", "bf16", "f32"]) if cache == "bf16" else "bf16", "cache": cache,
                "n": _log_uniform(rng, 1, min(65537, MAX_READ_VALUES // (2 * hk * D))), "hk": hk, "D": D, "page": page}
    rot = rng.choice([D, D, D // 2 // 8 * 8])
    values = MAX_WRITE_VALUES // (hq + 2 * hk) if op == "write" else MAX_NORM_VALUES // (hq + hk)
    case = {"op": op, "dtype": dtype, "n": _log_uniform(rng, 1, min(8192, values * 2 // SIZES[dtype] // D)), "hq": hq, "hk": hk, "D": D,
            "rot": rot, "interleaved": rng.random() < 0.25}
    return {**case, "cache": cache, "page": page} if op == "write" else case


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """The cached tokens of each request: from the longest down to a sixteenth of it, evenly over the logarithm; of four and more requests the last is empty."""
    B, length = case["requests"], case["length"]
    lengths = [max(1, round(length * 16 ** (-i / max(1, B - 1)))) for i in range(B)]
    if B >= 4:
        lengths[-1] = 0
    return lengths


def _rows(case):
    """The new tokens of each request: most have all there may be, every third fewer."""
    R = case["rows"]
    return [R if i % 3 != 2 else max(1, R - 1 - i % R) for i in range(case["requests"])]


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _projection(g, case, kv):
    """q, k (and v): views of a projection's rows."""
    n, hq, hk, D = case["n"], case["hq"], case["hk"], case["D"]
    rows = _randn(g, n, (hq + kv * hk) * D, dtype=DTYPES[case["dtype"]])
    parts = [rows[:, :hq * D].view(n, hq, D)]
    return parts + [rows[:, (hq + i * hk) * D:(hq + (i + 1) * hk) * D].view(n, hk, D) for i in range(kv)]


def _table(positions, rot):
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * (
        500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot))
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def _cache(g, case, pages):
    shape = (pages, case["hk"], case["page"], case["D"])
    state = {}
    for name in ("k", "v"):
        if case["cache"] == "e4m3":
            state[name] = _randn(g, *shape).mul_(120.0).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
            state[name + "_scale"] = torch.randint(119, 123, shape[:3], generator=g, device="cuda", dtype=torch.uint8)
        else:
            state[name] = _randn(g, *shape, dtype=torch.bfloat16)
            state[name + "_scale"] = None
    if own:
        import paper_2506_22694_amd as vt
        state["handle"] = vt.KVCache.of(state["k"], state["v"], state["k_scale"], state["v_scale"])
    return state


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, D = case["op"], case["D"]
    state = {"op": op, "case": dict(case)}
    if op in ("norm", "grad", "write"):
        n = case["n"]
        dtype = DTYPES[case["dtype"]]
        state["table"] = _table(max(8192, n), case["rot"])
        # a prompt's positions from somewhere on, as far as the table goes
        first = torch.randint(0, max(8192, n) - n + 1, (1,), generator=g, device="cuda")
        state["positions"] = first + torch.arange(n, device="cuda")
        state["wq"], state["wk"] = (_randn(g, D).mul_(0.1).add_(1.0).to(dtype) for _ in range(2))
        if op == "write":
            state["q"], state["k_new"], state["v_new"] = _projection(g, case, 2)
            pages = -(-n // case["page"]) + 3
            state.update(_cache(g, case, pages))
            state["slots"] = (torch.randperm(pages, generator=g, device="cuda")[:, None] * case["page"] +
                              torch.arange(case["page"], device="cuda")).flatten()[:n].contiguous()
        else:
            state["q"], state["k"] = _projection(g, case, 1)
        if op == "grad":
            state["gq"], state["gk"] = _randn(g, n, case["hq"], D, dtype=dtype), _randn(g, n, case["hk"], D, dtype=dtype)
        return state
    if op == "read":
        pages = -(-case["n"] // case["page"]) + 3
        state.update(_cache(g, case, pages))
        # the requests' rows lie in pages anywhere, each page's in order
        state["slots"] = (torch.randperm(pages, generator=g, device="cuda")[:, None] * case["page"] +
                          torch.arange(case["page"], device="cuda")).flatten()[:case["n"]].contiguous()
        return state
    lengths, rows, page = _lengths(case), _rows(case), case["page"]
    order = torch.randperm(len(lengths), generator=g, device="cuda").tolist()
    lengths, rows = [lengths[i] for i in order], [rows[i] for i in order]
    used = [-(-x // page) for x in lengths]
    state.update(_cache(g, case, sum(used) + 3))
    ids = torch.randperm(sum(used) + 3, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lengths), max(used)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, u in enumerate(used):
        table[i, :u] = ids[at:at + u]
        at += u
    n = sum(rows)
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    state.update(page_table=table, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                 max_length=case["length"], max_rows=case["rows"], row_start=None, tail_mask=None,
                 q=_randn(g, n, case["hq"], D).mul_(1.5).to(DTYPES[case["dtype"]]))
    if case["rows"] > 1:
        # the prompt's tokens are seen by all; of the last 32, the tree's, a node sees some, its own among them
        seen = torch.randint(0, 1 << 32, (n,), generator=g, device="cuda")
        state["tail_mask"] = (seen << 32) | ((1 << 32) - 1)
        state["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    if own:
        import paper_2506_22694_amd as vt
        state["ws"] = vt.AttentionWorkspace(n, case["hq"], case["hk"], D, len(lengths), case["rows"], case["length"], state["q"].device)
    return state


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _run_own(state)
    op = state["op"]
    if op == "norm":
        dtype = state["q"].dtype
        return _norm_rotate(state, state["q"], state["wq"]).to(dtype), _norm_rotate(state, state["k"], state["wk"]).to(dtype)
    if op == "grad":
        dq, dwq = _gradients(state, state["gq"], state["q"], state["wq"])
        dk, dwk = _gradients(state, state["gk"], state["k"], state["wk"])
        return dq, dk, dwq, dwk
    if op == "write":
        q = _norm_rotate(state, state["q"], state["wq"]).to(state["q"].dtype)
        _write(state, "k", _norm_rotate(state, state["k_new"], state["wk"]))
        _write(state, "v", state["v_new"].float())
        return q, _read(state, "k").to(torch.bfloat16), _read(state, "v").to(torch.bfloat16)
    if op == "read":
        return _read(state, "k").to(DTYPES[state["case"]["out"]]), _read(state, "v").to(DTYPES[state["case"]["out"]])
    return _attend(state)


def _run_own(state):
    import paper_2506_22694_amd as vt
    op, case = state["op"], state["case"]
    if op == "norm":
        return vt.qk_norm_rope(state["q"], state["k"], state["positions"], state["table"], state["wq"], state["wk"], eps=EPS,
                               interleaved=case["interleaved"])
    if op == "grad":
        return vt.qk_norm_rope_backward(state["gq"], state["gk"], state["q"], state["k"], state["positions"], state["table"],
                                        state["wq"], state["wk"], eps=EPS, interleaved=case["interleaved"])
    if op == "write":
        q = vt.qkv_to_cache(state["q"], state["k_new"], state["v_new"], state["handle"], state["slots"], state["positions"],
                            state["table"], state["wq"], state["wk"], eps=EPS, interleaved=case["interleaved"])
        return (q, *vt.kv_cache_read(state["handle"], state["slots"]))
    if op == "read":
        return vt.kv_cache_read(state["handle"], state["slots"], dtype=DTYPES[case["out"]])
    return vt.paged_attention(state["q"], state["handle"], state["page_table"], state["lengths"], row_start=state["row_start"],
                              max_rows=state["max_rows"], tail_mask=state["tail_mask"], max_length=state["max_length"],
                              ws=state["ws"], return_lse=True)


def _split(case, x):
    """The first and second values of the rotated pairs, and what is not rotated."""
    rot = case["rot"]
    if case["interleaved"]:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _joined(case, a, b, rest):
    pairs = torch.stack([a, b], dim=-1).flatten(-2) if case["interleaved"] else torch.cat([a, b], dim=-1)
    return torch.cat([pairs, rest], dim=-1)


def _angles(state):
    cos, sin = state["table"][state["positions"]][:, None, :].chunk(2, dim=-1)
    return cos, sin


def _norm_rotate(state, x, w):
    case, x = state["case"], x.float()
    z = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w.float()
    cos, sin = _angles(state)
    a, b, rest = _split(case, z)
    return _joined(case, a * cos - b * sin, b * cos + a * sin, rest)


def _gradients(state, g, x, w):
    case, dtype = state["case"], x.dtype
    g, x = g.float(), x.float()
    r = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS)
    y = x * r
    cos, sin = _angles(state)
    a, b, rest = _split(case, g)
    gz = _joined(case, a * cos + b * sin, b * cos - a * sin, rest)
    gy = gz * w.float()
    dx = r * (gy - y * (gy * y).mean(dim=-1, keepdim=True))
    return dx.to(dtype), (gz * y).sum(dim=(0, 1))


def _place(state):
    page = state["case"]["page"]
    return state["slots"] // page, state["slots"] % page


def _write(state, name, x):
    pages, places = _place(state)
    if state["case"]["cache"] == "bf16":
        state[name][pages, :, places] = x.to(torch.bfloat16)
        return
    half, exponent = torch.frexp(x.abs().amax(dim=-1))      # amax = half * 2^exponent, half in [0.5, 1); 448 = 0.875 * 2^9
    scale = (exponent - 9 + (half > E4M3_MAX / 512)).clamp(min=-126)
    codes = torch.ldexp(x, -scale[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    state[name].view(torch.uint8)[pages, :, places] = codes.view(torch.uint8)
    state[name + "_scale"][pages, :, places] = (scale + 127).to(torch.uint8)


def _scaled(codes, scale):
    """The values that codes of 8 bits stand for."""
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), scale[..., None].int() - 127)


def _read(state, name):
    pages, places = _place(state)
    if state["case"]["cache"] == "bf16":
        return state[name][pages, :, places].float()
    return _scaled(state[name].view(torch.uint8)[pages, :, places], state[name + "_scale"][pages, :, places])


def _cached(state, name):
    """Every request's cached rows [requests, heads, tokens, D]."""
    case, pages = state["case"], state["page_table"].clamp(min=0).long()
    if case["cache"] == "bf16":
        rows = state[name][pages].float()
    else:
        rows = _scaled(state[name].view(torch.uint8)[pages], state[name + "_scale"][pages])
    return rows.transpose(1, 2).reshape(pages.shape[0], case["hk"], -1, case["D"])


def _attend(state):
    case, q, lengths = state["case"], state["q"], state["lengths"].long()
    n, hq, D = q.shape
    hk, R, B = case["hk"], state["max_rows"], lengths.numel()
    starts = state["row_start"].long() if state["row_start"] is not None else torch.arange(n + 1, device=q.device)
    rows = (starts[:-1, None] + torch.arange(R, device=q.device)).clamp(max=n - 1)
    K, V = _cached(state, "k"), _cached(state, "v")
    token = torch.arange(K.shape[2], device=q.device)
    sees = (token < lengths[:, None])[:, None, :].expand(B, R, -1)
    if state["tail_mask"] is not None:
        bit = token - (lengths[:, None] - 64)
        tail = (state["tail_mask"][rows][:, :, None] >> bit.clamp(0, 63)[:, None, :]) & 1
        sees = sees & ((bit < 0)[:, None, :] | (tail != 0))
    x = q[rows].float().view(B, R, hk, hq // hk, D).transpose(1, 2).reshape(B, hk, -1, D)
    scores = (x @ K.transpose(-1, -2)).mul_(D ** -0.5).view(B, hk, R, hq // hk, -1)
    scores.masked_fill_(~sees[:, None, :, None, :], float("-inf"))
    top = scores.amax(dim=-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == float("-inf"), 0.0, top))
    total = p.sum(dim=-1, keepdim=True)
    out = (p.view(B, hk, -1, p.shape[-1]) @ V).view(B, hk, R, hq // hk, D) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).squeeze(-1)
    request = torch.searchsorted(starts[1:], torch.arange(n, device=q.device), right=True)
    at = torch.arange(n, device=q.device) - starts[request]
    return out[request, :, at].reshape(n, hq, D).to(q.dtype), lse[request, :, at].reshape(n, hq)


# ---------------------------------------------------------------------------------------------- work and exactness
def work(case):
    op, D, hk = case["op"], case["D"], case["hk"]
    if op == "read":
        return {"bytes": case["n"] * (8 + 2 * hk * (D * (SIZES[case["cache"]] + SIZES[case["out"]]) + (case["cache"] == "e4m3"))), "flops": 0}
    cached = 2 * hk * (D * SIZES[case.get("cache", "bf16")] + (case.get("cache") == "e4m3"))      # a token's, of both
    if op == "attend":
        lengths, rows = _lengths(case), _rows(case)
        return {"bytes": sum(lengths) * cached + sum(rows) * case["hq"] * (2 * D * SIZES[case["dtype"]] + 4),
                "flops": 4 * sum(a * b for a, b in zip(lengths, rows)) * case["hq"] * D}
    n, hq, size = case["n"], case["hq"], SIZES[case["dtype"]]
    if op == "norm":
        return {"bytes": n * (2 * (hq + hk) * D * size + case["rot"] * 4 + 8), "flops": 10 * n * (hq + hk) * D}
    if op == "grad":
        return {"bytes": n * (3 * (hq + hk) * D * size + case["rot"] * 4 + 8), "flops": 20 * n * (hq + hk) * D}
    # written, and read back in 16 bits
    return {"bytes": n * ((2 * hq + 2 * hk) * D * size + 2 * cached + 2 * hk * D * 2 + case["rot"] * 4 + 16),
            "flops": 10 * n * (hq + 2 * hk) * D}


def _exact_norm_rotate(case, s, x, w):
    """From the definition, in 64 bits: a unit root mean square, then each pair as a complex number turned by its angle."""
    rot = case["rot"]
    x = x / (x.pow(2).sum(-1, keepdim=True) / case["D"] + EPS).sqrt() * w
    angle = s["table"].double()[s["positions"]]
    turn = torch.complex(angle[:, :rot // 2], angle[:, rot // 2:])[:, None, :]
    pairs = x[..., :rot].unflatten(-1, (rot // 2, 2) if case["interleaved"] else (2, rot // 2))
    pairs = pairs if case["interleaved"] else pairs.transpose(-1, -2)
    turned = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
    turned = turned if case["interleaved"] else turned.transpose(-1, -2)
    return torch.cat([turned.flatten(-2), x[..., rot:]], dim=-1)


def _exact_held(case, x):
    """What the cache holds of rows x."""
    if case["cache"] == "bf16":
        return x.bfloat16().double()
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top / E4M3_MAX)).clamp(min=-126))
    return (x / scale).float().to(torch.float8_e4m3fn).double() * scale


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op in ("norm", "write"):
        q = _exact_norm_rotate(case, s, s["q"].double(), s["wq"].double())
        if op == "norm":
            return q, _exact_norm_rotate(case, s, s["k"].double(), s["wk"].double())
        return (q, _exact_held(case, _exact_norm_rotate(case, s, s["k_new"].double(), s["wk"].double())),
                _exact_held(case, s["v_new"].double()))
    if op == "grad":
        leaves = [s[name].double().requires_grad_() for name in ("q", "k", "wq", "wk")]
        torch.autograd.backward([_exact_norm_rotate(case, s, leaves[0], leaves[2]), _exact_norm_rotate(case, s, leaves[1], leaves[3])],
                                [s["gq"].double(), s["gk"].double()])
        return tuple(x.grad for x in leaves)

    def held(name, pages):      # [pages, heads, page, D]
        codes = s[name][pages].double() if case["cache"] == "bf16" else s[name].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double()
        return codes if s[name + "_scale"] is None else codes * torch.exp2(s[name + "_scale"][pages].double() - 127)[..., None]

    if op == "read":
        place = s["slots"] % case["page"]
        return tuple(torch.cat([held(name, p)[torch.arange(p.numel(), device=p.device), :, at] for p, at in
                                zip((s["slots"] // case["page"]).split(1024), place.split(1024))]) for name in ("k", "v"))
    q, out, lse, row = s["q"].double(), [], [], 0
    counts = s["row_start"].diff().tolist() if s["row_start"] is not None else [1] * case["requests"]
    for b, (length, count) in enumerate(zip(s["lengths"].tolist(), counts)):
        pages = s["page_table"][b, :-(-length // case["page"])].long()
        k, v = (held(name, pages).transpose(0, 1).flatten(1, 2)[:, :length] for name in ("k", "v"))
        for i in range(row, row + count):
            z = torch.matmul(k, q[i].view(case["hk"], -1, case["D"]).transpose(1, 2)).transpose(1, 2) / case["D"] ** 0.5
            if s["tail_mask"] is not None:
                bits = int(s["tail_mask"][i])
                for t in range(max(0, length - 64), length):
                    if not bits >> (t - (length - 64)) & 1:
                        z[..., t] = float("-inf")
            lse.append(torch.logsumexp(z, -1).flatten())
            weight = torch.exp(z - torch.where(lse[-1].isinf(), 0.0, lse[-1]).view(case["hk"], -1, 1))
            out.append(torch.matmul(weight, v).reshape(case["hq"], case["D"]))
        row += count
    return torch.stack(out), torch.stack(lse)
