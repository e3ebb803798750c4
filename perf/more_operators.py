"""The operators around the cache and the weights of a low-bit decode step, as cases that can be timed and compared.

pack    rows to 4-bit floats with a scale per 16 columns and one per row, and the values read back
product rows, packed on the way, times packed weights: single tokens to whole prompts
rotary  norms of the query and key heads and the rotation by their positions (one to three axes)
sample  tokens from logits by temperature, top-k, top-p, min-p and given random numbers

`own` selects who computes: elementary torch operations, or this package's kernels.
"""
import math

import torch

own = False


# ----------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the activations of a verification pass of 16 fp32 rows before a product
        {"name": "pack_step", "op": "pack", "rows": 16, "k": 4096, "dtype": "fp32"},
        # the MLP activations of an odd prompt of the 13B shape
        {"name": "pack_prompt", "op": "pack", "rows": 1531, "k": 13824, "dtype": "bf16"},
        # the 7B gate and up weights as they are loaded
        {"name": "pack_weight", "op": "pack", "rows": 22016, "k": 4096, "dtype": "bf16"},
        # one token through the 7B attention output projection: latency counts
        {"name": "product_single", "op": "product", "rows": 1, "n": 4096, "k": 4096, "dtype": "bf16"},
        # the verification rows of 16 requests through the 7B gate and up projections, the engine's fp32 rows
        {"name": "product_verify", "op": "product", "rows": 96, "n": 22016, "k": 4096, "dtype": "fp32"},
        # a 640-row prompt (576 visual rows and 64 ids) through the 7B down projection
        {"name": "product_prompt", "op": "product", "rows": 640, "n": 4096, "k": 11008, "dtype": "bf16"},
        # the rows of several ragged prompts through the 13B gate and up projections
        {"name": "product_prompts", "op": "product", "rows": 5003, "n": 27648, "k": 5120, "dtype": "bf16"},
        # a verification pass of 16 requests, 7B heads, fp32 rows, one axis and no norm
        {"name": "rotary_step", "op": "rotary", "rows": 96, "heads": 32, "kv_heads": 32, "dim": 128, "turn": 128,
         "axes": 1, "norm": False, "dtype": "fp32"},
        # image and text prompts with grouped heads, norms and three axes (time, height, width)
        {"name": "rotary_prompts", "op": "rotary", "rows": 16381, "heads": 32, "kv_heads": 8, "dim": 128, "turn": 128,
         "axes": 3, "norm": True, "dtype": "bf16"},
        # one request's next token, 7B vocabulary
        {"name": "sample_single", "op": "sample", "rows": 1, "vocab": 32000, "mixed": False, "dtype": "fp32"},
        # a batch whose requests have their own settings, the encoder-decoder's vocabulary
        {"name": "sample_mixed", "op": "sample", "rows": 16, "vocab": 32128, "mixed": True, "dtype": "fp32"},
        # a large batch over a large, odd vocabulary
        {"name": "sample_large", "op": "sample", "rows": 256, "vocab": 150001, "mixed": True, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(map(_cost, listed()))
    while True:
        op = rng.choice(("pack", "product", "rotary", "sample"))
        dtype = rng.choice(("bf16", "fp32"))
        if op == "pack":
            c = {"op": op, "rows": _log(rng, 1, 32000), "k": _log(rng, 16, 14336), "dtype": dtype}
            if c["rows"] * c["k"] > 1 << 27:
                continue
        elif op == "product":
            c = {"op": op, "rows": _log(rng, 1, 8192), "n": _log(rng, 64, 40000), "k": _log(rng, 128, 14336),
                 "dtype": dtype}
            if c["n"] * c["k"] > 1 << 27 or c["rows"] * c["n"] > 1 << 27:
                continue
        elif op == "rotary":
            kv, dim = rng.choice((1, 4, 8, 32, 40)), rng.choice((64, 80, 96, 128, 256))
            c = {"op": op, "rows": _log(rng, 1, 16384), "heads": kv * rng.choice((1, 2, 4, 8)), "kv_heads": kv,
                 "dim": dim, "turn": rng.choice((dim, dim, dim // 2)), "axes": rng.randint(1, 3),
                 "norm": rng.random() < 0.5, "dtype": dtype}
            if c["heads"] > 64 or c["rows"] * (c["heads"] + kv) * dim > 1 << 27:
                continue
        else:
            c = {"op": op, "rows": _log(rng, 1, 512), "vocab": _log(rng, 1000, 160000), "mixed": rng.random() < 0.7,
                 "dtype": dtype}
        if _cost(c) <= most:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _size(case):
    return 4 if case["dtype"] == "fp32" else 2


def work(case):
    m, size = case["rows"], _size(case)
    if case["op"] == "pack":  # rows in, packed out and in, fp32 values out
        k = case["k"]
        return {"bytes": m * k * (size + 4.0) + 2 * (0.5625 * m * k + 4 * m), "flops": 0}
    if case["op"] == "product":
        n, k = case["n"], case["k"]
        return {"bytes": 0.5625 * n * k + 4 * n + m * (n + k) * size, "flops": 2.0 * m * n * k}
    if case["op"] == "rotary":
        return {"bytes": 2.0 * m * (case["heads"] + case["kv_heads"]) * case["dim"] * size + 4 * m * case["axes"],
                "flops": 0}
    return {"bytes": m * (case["vocab"] * size + (28.0 if case["mixed"] else 12.0)), "flops": 0}


# ----------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _rows(case, g):
    """Activations: normal values, rows of unequal size, some channels much larger."""
    x = torch.randn(case["rows"], case["k"], device="cuda", generator=g)
    x *= torch.exp(0.3 * torch.randn(case["rows"], 1, device="cuda", generator=g))
    x *= torch.exp(torch.randn(1, case["k"], device="cuda", generator=g))
    return x.to(_dtype(case))


def prepare(case, seed):
    return {"pack": _prepare_pack, "product": _prepare_product, "rotary": _prepare_rotary,
            "sample": _prepare_sample}[case["op"]](case, _generator(seed)) | {"case": case}


def _prepare_pack(case, g):
    return {"x": _rows(case, g)}


def _weight(case, g):
    return (0.02 * torch.randn(case["n"], case["k"], device="cuda", generator=g)).to(torch.bfloat16)


def _prepare_product(case, g):
    st, w = {"x": _rows(case, g)}, _weight(case, g)
    if own:
        import paper_2510_22641_gb300 as lib
        return st | {"w": lib.F4Weight(w)}
    return st | dict(zip(("codes", "scales", "row"), _pack(w)))


def _sections(case):
    """Pairs that turn with each axis: a quarter by time and the rest shared, where there are three."""
    pairs, axes = case["turn"] // 2, case["axes"]
    first = pairs // (4 if axes == 3 else axes)
    return [first] if axes == 1 else [first, pairs - first] if axes == 2 else \
        [first, (pairs - first) // 2, pairs - first - (pairs - first) // 2]


def _prepare_rotary(case, g):
    m, d, t = case["rows"], case["dim"], _dtype(case)
    # q, k and v of a row lie next to each other, as a fused projection leaves them
    heads = case["heads"] + 2 * case["kv_heads"]
    qkv = torch.randn(m, heads, d, device="cuda", generator=g)
    qkv *= torch.exp(0.5 * torch.randn(m, heads, 1, device="cuda", generator=g))
    qkv = qkv.to(t)
    st = {"q": qkv[:, :case["heads"]], "k": qkv[:, case["heads"]:case["heads"] + case["kv_heads"]]}
    # requests at positions of their own, up to 131072
    start = torch.randint(0, 131072 - 64, (-(-m // 64), 1, case["axes"]), device="cuda", generator=g)
    step = torch.randint(0, 64, (len(start), 64, case["axes"]), device="cuda", generator=g)
    step[:, :, 0] = torch.arange(64, device="cuda")
    st["pos"] = (start + step).view(-1, case["axes"])[:m].to(torch.int32).contiguous()
    st["q_gain"] = st["k_gain"] = None
    if case["norm"]:
        st["q_gain"], st["k_gain"] = (
            (1 + 0.1 * torch.randn(d, device="cuda", generator=g)).to(torch.bfloat16) for _ in range(2))
    if own:
        import paper_2510_22641_gb300 as lib
        st["rotary"] = lib.Rotary(d, rotary_dim=case["turn"], theta=10000.0, sections=_sections(case), eps=1e-5)
    return st


def _prepare_sample(case, g):
    m, v = case["rows"], case["vocab"]
    # a decoder's logits: most words unlikely, a few far ahead, some rows surer than others
    z = 2.5 * torch.randn(m, v, device="cuda", generator=g)
    for ahead in (4.0, 8.0):
        at = torch.randint(0, v, (m, 20), device="cuda", generator=g)
        z.scatter_add_(1, at, ahead * torch.rand(m, 20, device="cuda", generator=g))
    z *= 0.6 + 0.8 * torch.rand(m, 1, device="cuda", generator=g)
    st = {"logits": z.to(_dtype(case)), "u": torch.rand(m, device="cuda", generator=g)}
    if not case["mixed"]:
        return st | {"temperature": 0.8, "top_k": 0, "top_p": 0.95, "min_p": 0.0}
    pick = lambda values: values[torch.randint(0, len(values), (m,), device="cuda", generator=g)]  # noqa: E731
    floats = lambda *values: pick(torch.tensor(values, device="cuda"))  # noqa: E731
    return st | {"temperature": floats(0.0, 0.6, 0.8, 1.0, 1.3), "top_p": floats(1.0, 0.95, 0.9, 0.5),
                 "top_k": pick(torch.tensor((0, 0, 1, 50, 200), dtype=torch.int32, device="cuda")),
                 "min_p": floats(0.0, 0.0, 0.02, 0.1)}


# ----------------------------------------------------------------------------------------- one pass

def run(state):
    op, s = state["case"]["op"], state
    if own:
        import paper_2510_22641_gb300 as lib
        if op == "pack":
            return lib.F4Rows(s["x"]).dequantize()
        if op == "product":
            return s["w"].matmul(s["x"])
        if op == "rotary":
            q, k = s["rotary"].rotate(s["q"], s["k"], s["pos"], s["q_gain"], s["k_gain"])
            return {"q": q, "k": k}
        token, prob = lib.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                                 top_p=s["top_p"], min_p=s["min_p"], with_prob=True)
        return {"token": token, "prob": prob}
    return {"pack": _run_pack, "product": _run_product, "rotary": _run_rotary, "sample": _run_sample}[op](state)


def _pack(x):
    """Codes (twice the 4-bit float, int8) [rows][groups][16], scales [rows][groups] and row scales [rows]."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -k % 16))
    amax = x.abs().amax(1)
    finite = torch.isfinite(amax)
    part, e = torch.frexp(torch.where(finite, amax, torch.zeros_like(amax)))
    # the smallest 2^e with amax <= 2688 * 2^e, 2688 = 0.65625 * 2^12
    e = (e - 12 + (part > 0.65625)).clamp(min=-100)
    y = torch.ldexp(x, -e[:, None]).view(rows, -1, 16)
    y = torch.where(finite[:, None, None], y, torch.zeros_like(y))
    # quotients in 64 bits, rounded to 32: a division by a number is a product with its reciprocal in 32
    s = (y.abs().amax(2).double() / 6).float()
    unit = torch.exp2((torch.frexp(s)[1] - 1).clamp(min=-6) - 3.0)  # 8 steps from a power of two to the next
    s = torch.round(s / unit) * unit
    q = torch.where(s[:, :, None] > 0, (y.double() / s.double()[:, :, None]).float(), torch.zeros_like(y)).abs()
    unit = torch.where(q < 2, 0.5, torch.where(q < 4, 1.0, 2.0))
    q = (torch.round(q / unit) * unit).clamp(max=6)
    code = torch.copysign(2 * q, y).to(torch.int8)
    row = torch.ldexp(torch.ones_like(amax), e)
    return code, s, torch.where(finite, row, torch.full_like(row, math.nan))


def _values(code, s, row, k):
    v = code.float() * (0.5 * s)[:, :, None] * row[:, None, None]
    return v.view(len(row), -1)[:, :k]


def _run_pack(st):
    return _values(*_pack(st["x"]), st["x"].shape[1])


def _run_product(st):
    k = st["x"].shape[1]
    return (_values(*_pack(st["x"]), k) @ _values(st["codes"], st["scales"], st["row"], k).T).to(st["x"].dtype)


def _run_rotary(st):
    c = st["case"]
    half = c["turn"] // 2
    i = torch.arange(half, device="cuda", dtype=torch.float64)
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_sections(c), device="cuda"))
    angle = st["pos"].double()[:, axis] * torch.exp(i * (-math.log(10000.0) / half))
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    out = {}
    for name in "qk":
        x, gain = st[name].float(), st[name + "_gain"]
        if gain is not None:
            x = x / torch.sqrt((x * x).mean(2, keepdim=True) + 1e-5) * gain.float()
        a, b, rest = x[:, :, :half], x[:, :, half:2 * half], x[:, :, 2 * half:]
        out[name] = torch.cat([a * cos - b * sin, b * cos + a * sin, rest], 2).to(st[name].dtype)
    return out


def _column(v, like):
    return (v if torch.is_tensor(v) else torch.tensor([v], device=like.device)).double()[:, None]


def _run_sample(st):
    z = st["logits"].double()
    m, v = z.shape
    t, k, p, least, u = (_column(st[n], z) for n in ("temperature", "top_k", "top_p", "min_p", "u"))
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp((z - z[:, :1]) / torch.where(t > 0, t, torch.ones_like(t)))
    rank = torch.arange(v, device=z.device)
    w = torch.where((t > 0) | (rank == 0), w, torch.zeros_like(w))
    kept = torch.where((rank < k) | (k < 1), w, torch.zeros_like(w))
    ahead = torch.cumsum(kept, 1) - kept
    keep = ((ahead < p * kept.sum(1, keepdim=True)) | (p >= 1)) & (w >= least)
    kept = torch.where(keep | (rank == 0), kept, torch.zeros_like(w))
    kept = torch.zeros_like(w).scatter(1, order, kept)
    run_mass = torch.cumsum(kept, 1)
    total = run_mass[:, -1:]
    token = (run_mass <= u * total).sum(1, keepdim=True).clamp(max=v - 1)
    return {"token": token[:, 0].int(), "prob": (kept.gather(1, token) / total)[:, 0].float()}


# ----------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    global own
    was, own = own, False
    try:
        g = _generator(seed)
        if case["op"] == "pack":
            return _exact_values(_rows(case, g))
        if case["op"] == "product":
            x, w = _exact_values(_rows(case, g)), _exact_values(_weight(case, g))
            return torch.cat([torch.mm(part, w.t()) for part in x.split(1024)])
        return (_exact_rotary if case["op"] == "rotary" else _exact_sample)(prepare(case, seed))
    finally:
        own = was


def _exact_values(x):
    """What rows stand for once packed, by tables of all values that a scale and a code can have."""
    minifloat = lambda e, man: man * 2.0 ** (e - 9) if e == 0 else (8 + man) * 2.0 ** (e - 10)  # noqa: E731
    sizes = torch.tensor([minifloat(i >> 3, i & 7) for i in range(127)], dtype=torch.float64, device="cuda")
    floats = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")

    def nearest(v, table):
        """Index of the nearest value, of two as near the even index."""
        border = (table[1:] + table[:-1]) / 2
        low, high = torch.searchsorted(border, v), torch.searchsorted(border, v, right=True)
        return torch.where(low % 2 == 0, low, high)

    out = []
    for part in x.split(2048):
        v = part.double()
        a = v.abs().amax(1, keepdim=True)
        row = torch.exp2(torch.ceil(torch.log2(a / 2688)).clamp(min=-100))
        row = torch.where(a > 2688 * row, 2 * row, torch.where((a <= 1344 * row) & (row > 2.0 ** -100), row / 2, row))
        y = torch.zeros(len(v), -(-v.shape[1] // 16) * 16, dtype=torch.float64, device="cuda")
        y[:, :v.shape[1]] = v / row
        y = y.view(len(v), -1, 16)
        s = sizes[nearest((y.abs().amax(2) / 6).float().double(), sizes)][:, :, None]
        c = floats[nearest((y.abs() / s.clamp(min=2.0 ** -9)).float().double(), floats)]
        y = (torch.sign(y) * c * s).flatten(1)[:, :v.shape[1]] * row
        out.append(torch.where(torch.isfinite(a), y, torch.full_like(y, math.nan)))
    return torch.cat(out)


def _exact_rotary(st):
    """The rotation as a product of complex numbers."""
    c, out, half = st["case"], {}, st["case"]["turn"] // 2
    freq = torch.tensor([10000.0 ** (-2 * i / c["turn"]) for i in range(half)], dtype=torch.float64, device="cuda")
    axis = sum(([a] * n for a, n in enumerate(_sections(c))), [])
    angle = torch.stack([st["pos"][:, a] for a in axis], 1).double() * freq
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    for name in "qk":
        x = st[name].double()
        if st[name + "_gain"] is not None:
            x = x * st[name + "_gain"].double() * (x.square().sum(2, keepdim=True) / c["dim"] + 1e-5).rsqrt()
        z = torch.complex(x[:, :, :half], x[:, :, half:2 * half]) * turn
        x[:, :, :half], x[:, :, half:2 * half] = z.real, z.imag
        out[name] = x
    return out


def _exact_sample(st):
    """Row by row: the tokens of each rule found in the row's sorted values."""
    tokens, probs = [], []
    for r, row in enumerate(st["logits"].double()):
        t, k, p, least, u = (float(x[r if len(x) > 1 else 0]) for x in
                             (_column(st[n], row)[:, 0] for n in ("temperature", "top_k", "top_p", "min_p", "u")))
        ranked = torch.argsort(row, descending=True, stable=True)
        if t <= 0:
            ranked, t = ranked[:1], 1.0
        if k >= 1:
            ranked = ranked[:int(k)]
        w = torch.exp(row[ranked] / t - row[ranked[0]] / t)
        if p < 1:
            # as many as there are running masses below the limit, and the one that reaches it
            n = int(torch.searchsorted(torch.cumsum(w, 0), p * w.sum())) + 1
            ranked, w = ranked[:n], w[:n]
        ranked = ranked[:max(1, int((w >= least).sum()))]
        ranked = torch.sort(ranked)[0]
        w = torch.exp(row[ranked] / t - row[ranked].max() / t)
        mass = torch.cumsum(w, 0)
        at = min(int(torch.searchsorted(mass, u * mass[-1], right=True)), len(ranked) - 1)
        tokens.append(ranked[at])
        probs.append(w[at] / mass[-1])
    return {"token": torch.stack(tokens).int(), "prob": torch.stack(probs)}
