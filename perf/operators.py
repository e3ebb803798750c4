"""The operators of the low-bit decode step, as cases that can be timed and compared.

plan    block tables and slot maps of a paged cache, from the requests' lengths
append  new K/V rows quantised into the 8-bit cache (one scale per block of tokens and head), and read back
attn    attention of 1..16 query rows per request over the 8-bit cache
w4      products of 1..16 activation rows with 4-bit weights and group scales

`own` selects who computes: elementary torch operations, or this package's kernels.
"""
import math
import random

import torch

own = False

TINY_SCALE = 2.0 ** -100  # smallest block scale the cache stores


# ----------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one verification step of 16 ragged requests (576 + 16..64 prompt rows, up to 384 new tokens)
        {"name": "plan_verify", "op": "plan", "batch": 16, "length": 1024, "rows": 7, "block": 32, "ragged": 1},
        # admission of 64 prompts of up to 16k tokens, some seats being released meanwhile
        {"name": "plan_admit", "op": "plan", "batch": 64, "length": 0, "rows": 16384, "block": 64, "ragged": 2},
        # the new K/V rows of a verification pass, 13B-shaped heads, the engine's fp32 rows
        {"name": "append_verify", "op": "append", "batch": 16, "length": 1024, "rows": 7, "kv_heads": 40, "dim": 128,
         "block": 32, "dtype": "fp32", "ragged": 3},
        # a 640-row prompt (576 visual rows and 64 ids) of the 7B shape
        {"name": "append_prompt", "op": "append", "batch": 1, "length": 0, "rows": 640, "kv_heads": 32, "dim": 128,
         "block": 64, "dtype": "bf16", "ragged": 4},
        # ragged prompts of 8 requests with grouped heads and an odd length
        {"name": "append_ragged", "op": "append", "batch": 8, "length": 0, "rows": 8189, "kv_heads": 8, "dim": 128,
         "block": 16, "dtype": "bf16", "ragged": 5},
        # a single request's single token after a 7B prompt: latency counts
        {"name": "attn_single", "op": "attn", "batch": 1, "length": 640, "rows": 1, "heads": 32, "kv_heads": 32,
         "dim": 128, "block": 64, "dtype": "bf16", "ragged": 6},
        # the verification rows of 16 ragged 13B-shaped requests, fp32 rows
        {"name": "attn_verify", "op": "attn", "batch": 16, "length": 1024, "rows": 7, "heads": 40, "kv_heads": 40,
         "dim": 128, "block": 32, "dtype": "fp32", "ragged": 7},
        # 64 ragged requests with grouped heads, two rows each
        {"name": "attn_grouped", "op": "attn", "batch": 64, "length": 8191, "rows": 2, "heads": 32, "kv_heads": 8,
         "dim": 128, "block": 16, "dtype": "bf16", "ragged": 8},
        # two very long contexts: the work has to be split along the keys
        {"name": "attn_long", "op": "attn", "batch": 2, "length": 131072, "rows": 6, "heads": 32, "kv_heads": 8,
         "dim": 128, "block": 64, "dtype": "bf16", "ragged": 9},
        # the 7B attention output projection for one token
        {"name": "w4_single", "op": "w4", "rows": 1, "n": 4096, "k": 4096, "group": 128, "dtype": "bf16"},
        # the 7B gate and up projections for a verification pass of 6 fp32 rows
        {"name": "w4_verify", "op": "w4", "rows": 6, "n": 22016, "k": 4096, "group": 128, "dtype": "fp32"},
        # the 7B vocabulary head for 16 rows, finer groups
        {"name": "w4_head", "op": "w4", "rows": 16, "n": 32000, "k": 4096, "group": 64, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(max(w["bytes"], w["flops"] / 50) for w in map(work, listed()))
    while True:
        op = rng.choice(("plan", "append", "attn", "w4"))
        ragged = rng.randrange(1 << 20)
        dtype = rng.choice(("bf16", "fp32"))
        if op == "plan":
            prompt = rng.random() < 0.5
            c = {"op": op, "batch": _log(rng, 1, 256), "length": 0 if prompt else _log(rng, 1, 16384),
                 "rows": _log(rng, 16, 16384) if prompt else rng.randint(1, 16),
                 "block": rng.choice((16, 32, 64, 128)), "ragged": ragged}
            if c["batch"] * max(c["rows"], c["length"]) > 1 << 20:
                continue
        elif op == "append":
            prompt = rng.random() < 0.5
            c = {"op": op, "batch": _log(rng, 1, 64), "length": 0 if prompt else _log(rng, 1, 4096),
                 "rows": _log(rng, 16, 8192) if prompt else rng.randint(1, 16),
                 "kv_heads": rng.choice((1, 4, 8, 32, 40)), "dim": rng.choice((64, 128)),
                 "block": rng.choice((16, 32, 64, 128)), "dtype": dtype, "ragged": ragged}
            if c["batch"] * (c["rows"] + c["length"]) * c["kv_heads"] * c["dim"] > 1 << 27:
                continue
        elif op == "attn":
            kv = rng.choice((1, 4, 8, 32, 40))
            c = {"op": op, "batch": _log(rng, 1, 64), "length": _log(rng, 1, 131072), "rows": rng.randint(1, 16),
                 "heads": kv * rng.choice((1, 2, 4, 8)), "kv_heads": kv, "dim": rng.choice((64, 128)),
                 "block": rng.choice((16, 32, 64, 128)), "dtype": dtype, "ragged": ragged}
            if c["heads"] > 64 or c["batch"] * (c["length"] + c["rows"]) * kv * c["dim"] > 1 << 28:
                continue
        else:
            c = {"op": op, "rows": rng.randint(1, 16), "n": _log(rng, 64, 40000), "k": _log(rng, 128, 14336),
                 "group": rng.choice((32, 64, 128)), "dtype": dtype}
            if c["n"] * c["k"] > 1 << 27:
                continue
        if 3072 in c.values():
            continue
        w = work(c)
        if max(w["bytes"], w["flops"] / 50) <= most:
            return c


def _lengths(case):
    """(cached tokens, new rows) of each request: the first has the full length, the others are ragged."""
    rng = random.Random(case["ragged"])
    length, add = [case["length"]], [case["rows"]]
    for _ in range(case["batch"] - 1):
        length.append(int(case["length"] * rng.random() ** 0.5))
        add.append(rng.randint(1, case["rows"]))
    return length, add


def _released(case):
    """Seats of a plan that are given back: every seventh, where there are several requests."""
    return [b % 7 == 3 for b in range(case["batch"])]


def _up(a, b):
    return -(-a // b)


def work(case):
    if case["op"] == "w4":
        m, n, k, size = case["rows"], case["n"], case["k"], 4 if case["dtype"] == "fp32" else 2
        return {"bytes": n * k / 2 + 2 * n * _up(k, case["group"]) + m * (n + k) * size, "flops": 2.0 * m * n * k}
    length, add = _lengths(case)
    bs = case["block"]
    if case["op"] == "plan":
        gone = _released(case)
        rows = sum(a for a, g in zip(add, gone) if not g)
        new = sum(_up(l + a, bs) - _up(l, bs) for l, a, g in zip(length, add, gone) if not g)
        back = sum(_up(l + a, bs) for l, a, g in zip(length, add, gone) if g)
        return {"bytes": 4.0 * (rows + 2 * new + 2 * back + 5 * case["batch"]), "flops": 0}
    hkv, d, size = case["kv_heads"], case["dim"], 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "append":
        seen = sum(l % bs + a for l, a in zip(length, add))
        return {"bytes": 2.0 * hkv * d * (sum(add) * (size + 1) + seen * (1 + size)), "flops": 0}
    ctx = sum(l + a for l, a in zip(length, add))
    pairs = sum(a * l + a * (a + 1) // 2 for l, a in zip(length, add))
    blocks = sum(_up(l + a, bs) for l, a in zip(length, add))
    return {"bytes": 2.0 * hkv * d * ctx + 8.0 * hkv * blocks + 2.0 * sum(add) * case["heads"] * d * size,
            "flops": 4.0 * pairs * case["heads"] * d}


# ----------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _rows_of(case, counts, g):
    """K or V rows as a decoder makes them: normal values, tokens of unequal size, some channels larger."""
    n, h, d = sum(counts), case["kv_heads"], case["dim"]
    x = torch.randn(n, h, d, device="cuda", generator=g)
    x *= torch.exp(0.3 * torch.randn(n, h, 1, device="cuda", generator=g))
    x *= torch.exp(0.5 * torch.randn(1, h, d, device="cuda", generator=g))
    return x.to(_dtype(case))


def _paged(case, g):
    """Lengths, new rows, and a paged cache of them: block ids in a random order."""
    length, add = _lengths(case)
    bs, batch = case["block"], case["batch"]
    wide = max(_up(l + a, bs) for l, a in zip(length, add))
    total = sum(_up(l + a, bs) for l, a in zip(length, add))
    n_blocks = total + 8
    order = torch.randperm(n_blocks, device="cuda", generator=g).to(torch.int32)
    return {"case": case, "length": length, "add": add, "wide": wide, "n_blocks": n_blocks, "order": order,
            "batch": batch, "bs": bs}


def _slots(table, starts, counts, bs):
    """Slots of `counts[b]` tokens of each request from position starts[b] on (plain, for the inputs)."""
    n = torch.tensor(counts, device="cuda")
    first = torch.cumsum(n, 0) - n
    req = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), n)
    pos = torch.arange(int(n.sum()), device="cuda") - first[req] + torch.tensor(starts, device="cuda")[req]
    return table[req, pos // bs].long() * bs + pos % bs


def _table_of(p):
    """The table that handing out blocks in order gives: the free stack is popped from its end."""
    held = torch.tensor([_up(l + a, p["bs"]) for l, a in zip(p["length"], p["add"])], device="cuda")
    j = torch.arange(p["wide"], device="cuda")[None]
    index = (torch.cumsum(held, 0) - held)[:, None] + j
    ids = p["order"].flip(0)[index.clamp(max=p["n_blocks"] - 1)]
    return torch.where(j < held[:, None], ids, -torch.ones_like(ids))


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "w4":
        return _prepare_w4(case, g)
    if case["op"] == "plan":
        return _prepare_plan(case, g)
    p = _paged(case, g)
    hist = [_rows_of(case, p["length"], g), _rows_of(case, p["length"], g)]
    new = [_rows_of(case, p["add"], g), _rows_of(case, p["add"], g)]
    st = {"case": case, "k": new[0], "v": new[1]}
    table = _table_of(p)
    after = [l + a for l, a in zip(p["length"], p["add"])]
    if case["op"] == "append":
        first = [l // p["bs"] * p["bs"] for l in p["length"]]
        st["read"] = _slots(table, first, [n - f for n, f in zip(after, first)], p["bs"]).to(torch.int32)
    else:
        st["q"] = torch.randn(sum(p["add"]), case["heads"], case["dim"], device="cuda", generator=g).to(_dtype(case))
        st["q"] *= 1.5
    if own:
        import paper_2510_22641_gb300 as lib
        heads = case.get("heads", case["kv_heads"])
        cache = lib.KV8Cache(1, heads, case["kv_heads"], case["dim"], p["bs"], p["n_blocks"], p["batch"], p["wide"])
        cache.pool.copy_(p["order"])
        zero = torch.zeros(p["batch"], dtype=torch.int32, device="cuda")
        # one plan hands out the blocks of history and new rows, so that both sides have the same table
        cache.plan(cache.new_step(p["batch"], sum(after)), zero, _ints(after))
        if sum(p["length"]):
            past = cache.new_step(p["batch"], sum(p["length"]))
            cache.plan(past, zero, _ints(p["length"]))
            cache.append(0, hist[0], hist[1], past)
        step = cache.new_step(p["batch"], sum(p["add"]))
        cache.plan(step, _ints(p["length"]), _ints(p["add"]))
        if case["op"] == "attn":
            cache.append(0, st["k"], st["v"], step)
        return st | {"cache": cache, "step": step}
    shape = (p["n_blocks"], p["bs"], case["kv_heads"], case["dim"])
    st["codes"] = [torch.zeros(shape, dtype=torch.int8, device="cuda") for _ in range(2)]
    st["scales"] = [torch.zeros(shape[0], shape[2], device="cuda") for _ in range(2)]
    st["add"] = _ints(p["add"]).long()
    st["slots"] = _slots(table, p["length"], p["add"], p["bs"])
    past = _slots(table, [0] * p["batch"], p["length"], p["bs"])
    for i in range(2):
        if sum(p["length"]):
            _append(st["codes"][i], st["scales"][i], hist[i], past, _ints(p["length"]))
        if case["op"] == "attn":
            _append(st["codes"][i], st["scales"][i], new[i], st["slots"], _ints(p["add"]))
    if case["op"] == "attn":
        st["table"] = table.long()
        st["len"] = _ints(p["length"]).long()
        st["wide"], st["most"] = p["wide"], max(p["add"])
    return st


def _prepare_plan(case, g):
    p = _paged(case, g)
    batch, bs = p["batch"], p["bs"]
    # before the step each request holds the blocks of its cached tokens, and the rest are free;
    # a seat that is given back holds those of its whole finished request
    gone = _released(case)
    held = [_up(l + a if x else l, bs) for l, a, x in zip(p["length"], p["add"], gone)]
    length = _ints([-1 if x else l for l, x in zip(p["length"], gone)])
    mask = torch.arange(p["wide"], device="cuda")[None] < _ints(held)[:, None]
    table = torch.full((batch, p["wide"]), -1, dtype=torch.int32, device="cuda")
    n = sum(held)
    table[mask] = p["order"][p["n_blocks"] - n:]
    st = {"case": case, "length": length, "add": _ints(p["add"]), "rows": sum(p["add"]), "table": table,
          "pool": p["order"].clone(), "state": _ints([p["n_blocks"] - n] + held)}
    if own:
        import paper_2510_22641_gb300 as lib
        st["cache"] = lib.KV8Cache(1, 1, 1, 64, bs, p["n_blocks"], batch, p["wide"])
        st["cache"].table.copy_(table)
        st["cache"].pool.copy_(p["order"])
        st["step"] = st["cache"].new_step(batch, st["rows"])
        st["after"] = torch.zeros_like(st["state"])
    return st


def _quantize4(w, group):
    """4-bit codes and bf16 group scales of w [n][k], k padded to whole groups with zeros."""
    n, k = w.shape
    w = torch.nn.functional.pad(w.float(), (0, -k % group)).view(n, -1, group)
    s = (w.abs().amax(2) / 7).to(torch.bfloat16).float()
    inv = torch.where(s > 0, 1 / s, torch.zeros_like(s))
    return torch.round(w * inv[:, :, None]).clamp(-8, 7).to(torch.int8).view(n, -1), s


def _prepare_w4(case, g):
    w = (0.02 * torch.randn(case["n"], case["k"], device="cuda", generator=g)).to(torch.bfloat16)
    x = torch.randn(case["rows"], case["k"], device="cuda", generator=g)
    x *= torch.exp(torch.randn(1, case["k"], device="cuda", generator=g))  # some channels are much larger
    st = {"case": case, "x": x.to(_dtype(case))}
    if own:
        import paper_2510_22641_gb300 as lib
        return st | {"w": lib.W4Weight(w, group=case["group"])}
    codes, scales = _quantize4(w, case["group"])
    return st | {"codes": codes, "scales": scales}


# ----------------------------------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    if own:
        if op == "plan":
            c, s = state["cache"], state["step"]
            c.plan(s, state["length"], state["add"], state=state["state"], state_out=state["after"])
            return {"table": c.table, "state": state["after"], "row_start": s.row_start, "slot": s.slot}
        if op == "append":
            c = state["cache"]
            c.append(0, state["k"], state["v"], state["step"])
            k, v = c.read(0, state["read"], state["k"].dtype)
            return {"k": k, "v": v}
        if op == "attn":
            return state["cache"].attention(0, state["q"], state["step"])
        return state["w"].matmul(state["x"])
    return {"plan": _run_plan, "append": _run_append, "attn": _run_attn, "w4": _run_w4}[op](state)


def _run_plan(st):
    bs, table, pool = st["case"]["block"], st["table"], st["pool"]
    wide, n_blocks = table.shape[1], pool.shape[0]
    free, held = st["state"][0].long(), st["state"][1:].long()
    live = st["length"] >= 0
    length = st["length"].clamp(min=0).long()
    add = torch.where(live, st["add"].long(), 0)
    need = (length + add + bs - 1) // bs
    new = torch.where(live, (need - held).clamp(min=0), 0)
    back = torch.where(live, 0, held)
    first = lambda n: torch.cumsum(n, 0) - n  # noqa: E731
    j = torch.arange(wide, device=table.device)[None]
    # released blocks go on top of the free stack
    top = torch.where(j < back[:, None], free + first(back)[:, None] + j, n_blocks)
    stack = torch.cat([pool, pool[:1]]).scatter(0, top.flatten(), table.flatten())
    total = free + back.sum()
    pop = total - 1 - (first(new)[:, None] + j - held[:, None])
    mine = (j >= held[:, None]) & (j < (held + new)[:, None])
    ids = torch.where(pop >= 0, stack[pop.clamp(0, n_blocks)], -1)
    table = torch.where(mine, ids, table)
    got = (total - first(new)).clamp(min=0).minimum(new)
    held = torch.where(live, held + got, 0)
    start = torch.cumsum(add, 0)
    r = torch.arange(st["rows"], device=table.device)
    b = torch.searchsorted(start, r, right=True).clamp(max=len(add) - 1)
    pos = length[b] + r - (start - add)[b]
    block = table[b, (pos // bs).clamp(max=wide - 1)].long()
    slot = torch.where((r < start[-1]) & (block >= 0), block * bs + pos % bs, -1)
    state = torch.cat([(total - new.sum()).clamp(min=0)[None], held])
    rows = torch.cat([torch.zeros_like(start[:1]), start])
    return {"table": table.int(), "state": state.int(), "row_start": rows.int(), "slot": slot.int()}


def _append(codes, scales, x, slots, counts):
    """Quantises the rows x, counts[b] of request b, into the cache, in place."""
    n_blocks, bs, h, d = codes.shape
    x, block = x.float(), slots // bs
    amax = torch.zeros_like(scales).index_reduce_(0, block, x.abs().amax(2), "amax")
    touched = torch.zeros(n_blocks, dtype=torch.bool, device=x.device).index_fill_(0, block, True)
    opened = torch.zeros(n_blocks, device=x.device).index_add_(0, block, (slots % bs == 0).float()) > 0
    old = torch.where(opened[:, None], torch.zeros_like(scales), scales)
    new = torch.where(touched[:, None], torch.maximum(old, (amax / 127).clamp(min=TINY_SCALE)), scales)
    # only a request's first new row can fall into a block that holds earlier tokens
    head = block[(torch.cumsum(counts, 0) - counts).clamp(max=len(block) - 1)]
    ratio = old[head] / new[head]
    codes[head] = torch.round(codes[head].float() * ratio[:, None, :, None]).to(torch.int8)
    scales.copy_(new)
    q = torch.round(x * (1 / new)[block][:, :, None]).clamp(-127, 127)
    codes.view(n_blocks * bs, h, d)[slots] = q.to(torch.int8)


def _run_append(st):
    out = {}
    for i, name in enumerate("kv"):
        codes, scales = st["codes"][i], st["scales"][i]
        _append(codes, scales, st[name], st["slots"], st["add"])
        read = st["read"].long()
        vals = codes.view(-1, *codes.shape[2:])[read].float() * scales[read // codes.shape[1]][:, :, None]
        out[name] = vals.to(st[name].dtype)
    return out


def _run_attn(st):
    c = st["case"]
    hkv, d = c["kv_heads"], c["dim"]
    group = c["heads"] // hkv
    batch, most, keys = c["batch"], st["most"], st["wide"] * c["block"]
    table = st["table"].clamp(min=0)
    k, v = ((codes[table].float() * scales[table][:, :, None, :, None]).view(batch, keys, hkv, d)
            for codes, scales in zip(st["codes"], st["scales"]))
    first = torch.cumsum(st["add"], 0) - st["add"]
    i = torch.arange(most, device=k.device)
    row = (first[:, None] + i).clamp(max=len(st["q"]) - 1)
    q = st["q"].float()[row].view(batch, most, hkv, group, d)
    s = torch.einsum("brhgd,bkhd->bhrgk", q, k) / math.sqrt(d)
    seen = torch.arange(keys, device=k.device) <= (st["len"][:, None] + i)[:, :, None]
    s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    s = torch.exp(s - s.amax(4, keepdim=True))
    s /= s.sum(4, keepdim=True)
    o = torch.einsum("bhrgk,bkhd->brhgd", s, v).reshape(batch, most, c["heads"], d)
    return o[i < st["add"][:, None]].to(st["q"].dtype)


def _run_w4(st):
    n, k = st["codes"].shape
    w = (st["codes"].float().view(n, -1, st["case"]["group"]) * st["scales"][:, :, None]).view(n, k)
    x = st["x"].float()
    return (x @ w[:, :x.shape[1]].T).to(st["x"].dtype)


# ----------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    if case["op"] == "plan":
        return None
    st = prepare(case, seed)
    if case["op"] == "w4":
        g = case["group"]
        w = st["codes"].double() * torch.repeat_interleave(st["scales"].double(), g, dim=1)
        return torch.mm(st["x"].double(), w[:, :case["k"]].t())
    length, add = _lengths(case)
    if case["op"] == "append":
        del st
        few = sum(_up(a, case["block"]) for a in add) < 20000  # it goes block by block
        return _exact_append(case, seed) if few else None
    group, start, out = case["heads"] // case["kv_heads"], 0, []
    for b in range(case["batch"]):
        n = length[b] + add[b]
        ids = st["table"][b, :_up(n, case["block"])]
        kv = [(c[ids].double() * s[ids].double()[:, None, :, None]).flatten(0, 1)[:n].transpose(0, 1)
              for c, s in zip(st["codes"], st["scales"])]
        q = st["q"][start:start + add[b]].double().transpose(0, 1)  # [heads][rows][d]
        for_kv = q.reshape(case["kv_heads"], group * add[b], case["dim"])
        s = torch.bmm(for_kv, kv[0].transpose(1, 2)) * case["dim"] ** -0.5
        future = torch.arange(n, device="cuda")[None] > length[b] + torch.arange(add[b], device="cuda")[:, None]
        s = s.view(case["kv_heads"], group, add[b], n).masked_fill(future, -math.inf)
        o = torch.bmm(torch.softmax(s, 3).view(case["kv_heads"], group * add[b], n), kv[1])
        out.append(o.view(case["heads"], add[b], case["dim"]).transpose(0, 1))
        start += add[b]
    return torch.cat(out)


def _exact_append(case, seed):
    g = _generator(seed)
    p = _paged(case, g)
    hist = [_rows_of(case, p["length"], g), _rows_of(case, p["length"], g)]
    new = [_rows_of(case, p["add"], g), _rows_of(case, p["add"], g)]
    bs, out = case["block"], {"k": [], "v": []}
    for name, old_rows, new_rows in zip("kv", hist, new):
        a = b = 0
        for l, n in zip(p["length"], p["add"]):
            past, now = old_rows[a + l - l % bs:a + l].double(), new_rows[b:b + n].double()
            a, b, at = a + l, b + n, 0
            # block by block: the first may continue `past`, the others hold new rows only
            while at < n:
                part = now[at:at + bs - (len(past) if at == 0 else 0)]
                at += len(part)
                size = (part.abs().amax((0, 2)) / 127).clamp(min=TINY_SCALE)
                rows = []
                if len(past) and at == len(part):
                    before = (past.abs().amax((0, 2)) / 127).clamp(min=TINY_SCALE)
                    q = torch.round(past / before[None, :, None])
                    size = torch.maximum(size, before)
                    rows = [torch.round(q * (before / size)[None, :, None]) * size[None, :, None]]
                rows.append(torch.round(part / size[None, :, None]) * size[None, :, None])
                out[name] += rows
    return {n: torch.cat(v) for n, v in out.items()}
