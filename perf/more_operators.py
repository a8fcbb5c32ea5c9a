"""What the performance of integer attention over a cache of blocks is measured on: block tables and slots made from
request lengths (iodf_attn_plan), rotary positions with the cache in 8 bits (iodf_attn_append), and the attention that reads it
(iodf_attn_forward), from one token of one request to long prompts. Everything is integer arithmetic with one right answer.

A block holds 128 tokens. Requests hold `held` tokens and get `add` more in the call ("pattern"):
  "decode"   a token each, behind contexts of any length up to ctx
  "images"   ctx tokens each, nothing before them
  "chunks"   any number of new tokens (none, one, many; `rows` together with 2 % of padding behind the last request), behind contexts up to ctx

A case of the plan ("op": "plan"): n requests, pattern, rows (room for new tokens), ctx; every 16th request of a decode step ends.
A case of the append ("op": "append"): the same, and heads, kv (heads of keys and values), dim (of a head), x ("int8" / "int32"),
  rot (dimensions that are rotated), layout ("half" / "interleaved"), stretch (positions are divided by it).
A case of the attention ("op": "attn"): the same sizes, causal, window (0: none), y ("int8" / "int32").
"""
import math
import random

import torch

own = False

BLOCK = 128
MOST_PAIRS = 32 * 16384 * 16384        # heads x rows x keys of the largest listed case
MOST_TOKENS = 1 << 19                  # held by all requests together ...
MOST_BYTES = 1 << 30                   # ... and the bytes of their keys and values
MOST_ELEMS = 16384 * 48 * 128          # queries, keys and values of the largest listed step


def _plan(name, n, rows, ctx, pattern):
    return {"name": name, "op": "plan", "n": n, "rows": rows, "ctx": ctx, "pattern": pattern}


def _append(name, n, rows, ctx, pattern, heads, kv, dim, x, rot, layout, stretch):
    return {"name": name, "op": "append", "n": n, "rows": rows, "ctx": ctx, "pattern": pattern, "heads": heads, "kv": kv, "dim": dim,
            "x": x, "rot": rot, "layout": layout, "stretch": stretch}


def _attn(name, n, rows, ctx, pattern, heads, kv, dim, causal, window, y):
    return {"name": name, "op": "attn", "n": n, "rows": rows, "ctx": ctx, "pattern": pattern, "heads": heads, "kv": kv, "dim": dim,
            "causal": causal, "window": window, "y": y}


def listed():
    return [
        # the next token of one request: latency
        _plan("plan one request", 1, 1, 1000, "decode"),
        # a step of a full server, requests that end among them
        _plan("plan 1024 requests", 1024, 1024, 8192, "decode"),
        # prompts of any length and their continuations
        _plan("plan chunks", 128, 65536, 32768, "chunks"),
        # one token at the widths of a network of 4096 channels
        _append("append one token", 1, 1, 1000, "decode", 32, 8, 128, "int32", 128, "half", 1),
        # chunks of prompts, part of each head rotated, 8-bit projections
        _append("append chunks", 37, 20011, 8192, "chunks", 16, 4, 64, "int8", 32, "interleaved", 1),
        # one long prompt, positions stretched
        _append("append long prompt", 1, 16384, 16384, "images", 32, 8, 128, "int32", 128, "half", 4),
        # the next token of one request
        _attn("attn one token", 1, 1, 1000, "decode", 32, 8, 128, True, 0, "int8"),
        # a step of 64 requests with contexts of any length
        _attn("attn 64 requests", 64, 64, 8192, "decode", 32, 8, 128, True, 0, "int8"),
        # the next token of one request with a very long context
        _attn("attn long context", 1, 1, 131072, "decode", 32, 8, 128, True, 0, "int8"),
        # 128 images of 16 x 16 pixels, every pixel sees its image
        _attn("attn 16x16 images", 128, 128 * 256, 256, "images", 4, 4, 64, False, 0, "int8"),
        # chunks of prompts behind earlier ones, a sliding window, an odd number of heads for each cache head
        _attn("attn chunks window", 24, 6007, 4096, "chunks", 12, 4, 64, True, 1000, "int32"),
        # one long prompt: bound by arithmetic
        _attn("attn long prompt", 1, 16384, 16384, "images", 32, 8, 128, True, 0, "int8"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["plan", "append", "append", "attn", "attn", "attn"])
    pattern = rng.choice(["decode", "images", "chunks", "chunks"])
    dim = rng.choice([32, 64, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 5, 8])
    if pattern == "decode":
        n = _log_int(rng, 1, 1024 if op == "plan" else 256)
        ctx = _log_int(rng, 2, min(131072, MOST_TOKENS // n, MOST_BYTES // (2 * n * kv * dim)))
        rows = n
    elif pattern == "images":
        n = _log_int(rng, 1, 128)
        ctx = _log_int(rng, 1, min(16384, 65536 // n, MOST_ELEMS // (n * (heads + 2 * kv) * dim), int(math.sqrt(MOST_PAIRS / (n * heads)))))
        rows = n * ctx
    else:
        n = _log_int(rng, 1, 128)
        ctx = _log_int(rng, 64, 8192)
        rows = _log_int(rng, 2 * n, max(2 * n, min(n * ctx // 2, 20000)))
        if op == "attn":                # the longest chunk against the longest context, for every request
            while n * heads * min(rows, ctx) * ctx > MOST_PAIRS:
                rows, ctx = max(2 * n, rows // 2), max(64, ctx // 2)
    if op == "plan":
        c = _plan("", n, rows, ctx, pattern)
    elif op == "append":
        c = _append("", n, rows, ctx, pattern, heads, kv, dim, rng.choice(["int8", "int32"]), rng.choice([0, 16, dim, dim]),
                    rng.choice(["half", "interleaved"]), rng.choice([1, 1, 2, 8]))
    else:
        causal = pattern != "images" or rng.random() < 0.5
        c = _attn("", n, rows, ctx, pattern, heads, kv, dim, causal, rng.choice([0, 0, _log_int(rng, 1, 4096)]) if causal else 0,
                  rng.choice(["int8", "int8", "int32"]))
    del c["name"]
    return c


# ---- requests -----------------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens that each request holds before the call, and how many it gets (-1: it ends)."""
    rng = random.Random("%s %s %d %d %d" % (case["op"], case["pattern"], case["n"], case["rows"], case["ctx"]))
    n, ctx = case["n"], case["ctx"]
    if case["pattern"] == "decode":
        held = [ctx - 1] + [_log_int(rng, 1, ctx - 1) for _ in range(n - 1)]
        return held, [-1 if case["op"] == "plan" and q % 16 == 15 else 1 for q in range(n)]
    if case["pattern"] == "images":
        return [0] * n, [ctx] * n
    left = case["rows"] - case["rows"] // 50
    cuts = sorted(rng.randrange(left + 1) for _ in range(n - 1))
    for i in range(2, len(cuts), 7):
        cuts[i] = cuts[i - 1]                                  # a request without new tokens
    for i in range(4, len(cuts), 9):
        cuts[i] = min(left, cuts[i - 1] + 1)                   # one with a single one
    cuts = [0] + sorted(cuts) + [left]
    add = [min(ctx, b - a) for a, b in zip(cuts, cuts[1:])]
    return [0 if q % 3 == 0 else rng.randrange(ctx - a + 1) for q, a in enumerate(add)], add


def _blocks(tokens):
    return -(-tokens // BLOCK)


_TORCH = {"int8": torch.int8, "int32": torch.int32}


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(gen, shape, sigma, limit, dtype):
    """Rounded normal values; large arrays a part at a time."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        part = flat[at:at + (1 << 28)]
        part.copy_(torch.empty(part.shape, dtype=torch.float32, device="cuda").normal_(0.0, sigma, generator=gen).round_().clamp_(-limit, limit))
    return out


def _requests(case, gen):
    """Block table (any free blocks in any order), rows and slots as they are after the step's plan."""
    held, add = _lengths(case)
    add = [max(0, a) for a in add]
    total = [h + a for h, a in zip(held, add)]
    width = max(1, max(_blocks(t) for t in total))
    counts = torch.tensor([_blocks(t) for t in total], device="cuda")
    blocks = int(sum(_blocks(t) for t in total)) + 3
    order = torch.randperm(blocks, generator=gen, device="cuda")
    column = torch.arange(width, device="cuda")[None]
    at = (torch.cumsum(counts, 0) - counts)[:, None] + column
    table = torch.where(column < counts[:, None], order[at.clamp(max=blocks - 1)], torch.zeros_like(at)).to(torch.int32)
    start = [0]
    for a in add:
        start.append(start[-1] + a)
    rows = max(case["rows"], start[-1], 1)
    row_start = torch.tensor(start, device="cuda")
    r = torch.arange(rows, device="cuda")
    q = torch.searchsorted(row_start[1:].contiguous(), r, right=True).clamp(max=len(add) - 1)
    pos = torch.tensor(held, device="cuda")[q] + r - row_start[q]
    live = r < start[-1]
    pos = torch.where(live, pos, torch.zeros_like(pos))
    slot = torch.where(live, table[q, pos // BLOCK].long() * BLOCK + pos % BLOCK, torch.full_like(pos, -1))
    return {"case": case, "blocks": blocks, "width": width, "table": table, "held": _ints(total), "row_start": row_start.to(torch.int32),
            "rows": rows, "used": start[-1], "most_add": max(add), "position": pos.to(torch.int32), "slot": slot.to(torch.int32)}


# ---- inputs -------------------------------------------------------------------------------------------------
def _plan_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    held, add = _lengths(case)
    n, have = len(held), [_blocks(h) for h in held]
    width = max(1, max(_blocks(h + max(0, a)) for h, a in zip(held, add)))
    need = sum(_blocks(h + a) - _blocks(h) for h, a in zip(held, add) if a > 0)
    blocks = sum(have) + need + 16
    order = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    counts = torch.tensor(have, device="cuda")
    column = torch.arange(width, device="cuda")[None]
    at = (torch.cumsum(counts, 0) - counts)[:, None] + column
    table = torch.where(column < counts[:, None], order[at.clamp(max=blocks - 1).long()], torch.full_like(at, -1).to(torch.int32))
    # the free blocks lie in a ring, from a place in its middle on
    free = order[sum(have):]
    head = random.Random(seed).randrange(blocks)
    ring = torch.full((blocks,), -1, dtype=torch.int32, device="cuda")
    ring[(head + torch.arange(len(free), device="cuda")) % blocks] = free
    rows = max(case["rows"], 1)
    return {"case": case, "held": _ints(held), "add": _ints(add), "table": table, "ring": ring, "state": _ints([head, len(free)]), "rows": rows,
            "held_out": torch.zeros(n, dtype=torch.int32, device="cuda"), "row_start": torch.zeros(n + 1, dtype=torch.int32, device="cuda"),
            "slot": torch.zeros(rows, dtype=torch.int32, device="cuda"), "position": torch.zeros(rows, dtype=torch.int32, device="cuda"),
            "state_out": torch.zeros(2, dtype=torch.int32, device="cuda")}


def _rotary(positions, rot, stretch):
    """cos and sin in units of 2^-14 of every position and pair, from angles in 64 bits."""
    if rot == 0:
        return None
    freq = torch.pow(torch.tensor(10000.0, dtype=torch.float64), -torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    angle = (torch.arange(positions, dtype=torch.float64) / stretch)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], dim=-1).mul_(16384).round_().to(torch.int16)


def _cache(case, blocks, gen):
    kv, dim = case["kv"], case["dim"]
    exps = [torch.randint(3, 7, (blocks, kv), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8) for _ in range(2)]
    return {"k": _normal(gen, (blocks, kv, BLOCK, dim), 28.0, 127, torch.int8), "v": _normal(gen, (blocks, kv, dim, BLOCK), 28.0, 127, torch.int8),
            "k_exp": exps[0], "v_exp": exps[1]}


HEADROOM = (2, 4)              # of keys and values, in eighths


def _append_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = _requests(case, gen)
    heads, kv, dim, rows = case["heads"], case["kv"], case["dim"], st["rows"]
    sigma, limit = (32.0, 127) if case["x"] == "int8" else (2500.0, 30000)
    # the projection's output holds queries, keys and values side by side
    x = _normal(gen, (rows, (heads + 2 * kv) * dim), sigma, limit, _TORCH[case["x"]])
    st["q"], st["k"], st["v"] = x[:, :heads * dim], x[:, heads * dim:(heads + kv) * dim], x[:, (heads + kv) * dim:]
    st["cache"] = _cache(case, st["blocks"], gen)
    st["q8"] = torch.zeros((rows, heads, dim), dtype=torch.int8, device="cuda")
    st["q_exp"] = torch.zeros((rows, heads), dtype=torch.uint8, device="cuda")
    host = _rotary(max(case["ctx"], case["rows"]), case["rot"], case["stretch"])
    st["rotary_host"], st["rotary"] = host, None if host is None else host.cuda()
    return st


def _score(case):
    """Multiplier and shift with which scores of inputs like these spread over about two octaves."""
    sigma = 36.0 * 28.0 * math.sqrt(case["dim"]) * 2.0 ** 9.5
    gain = 2.0 * 2.0 ** 36 / sigma                 # weights of one octave are 2^13 of t, and t = s W / 2^23
    s = max(0, math.ceil(math.log2(2.0 ** 30 / gain)))
    return min((1 << 31) - 1, max(1 << 30, int(gain * 2.0 ** s))), s


def _attn_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = _requests(case, gen)
    heads, dim, rows = case["heads"], case["dim"], st["rows"]
    st["cache"] = _cache(case, st["blocks"], gen)
    st["q8"] = _normal(gen, (rows, heads, dim), 36.0, 127, torch.int8)
    st["q_exp"] = torch.randint(3, 8, (rows, heads), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
    st["score"] = _score(case)
    st["m0"] = torch.randint(1 << 30, 1 << 31, (heads * dim,), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    st["s"] = torch.full((heads * dim,), 11 if case["y"] == "int8" else 2, dtype=torch.int32, device="cuda")
    st["clamp"] = (-128, 127) if case["y"] == "int8" else None
    st["y"] = torch.full((rows, heads * dim), 3, dtype=_TORCH[case["y"]], device="cuda")
    return st


def _inputs(case, seed):
    return {"plan": _plan_inputs, "append": _append_inputs, "attn": _attn_inputs}[case["op"]](case, seed)


def _handle(st):
    import paper_2206_08869_b200 as G
    case = st["case"]
    heads, kv, dim = case.get("heads", 1), case.get("kv", 1), case.get("dim", 32)
    desc = {"heads": heads, "kv_heads": kv, "head_dim": dim, "x_dtype": _TORCH[case.get("x", "int32")], "headroom": HEADROOM,
            "score": st.get("score", (1 << 30, 20)), "causal": case.get("causal", True), "window": case.get("window", 0),
            "out": {"m0": st["m0"].cpu().numpy() if "m0" in st else [1 << 30] * (heads * dim),
                    "s": st["s"].cpu().numpy() if "s" in st else [0] * (heads * dim), "clamp": st.get("clamp"),
                    "dtype": _TORCH[case.get("y", "int32")]}}
    if st.get("rotary_host") is not None:
        desc["rotary"] = {"dim": case["rot"], "layout": case["layout"], "table": st["rotary_host"].numpy()}
    return G.iodf_attn_create(desc)


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        st["handle"] = _handle(st)
    return st


# ---- plain forms --------------------------------------------------------------------------------------------
def _plain_plan(st):
    held, add, ring, table = st["held"].long(), st["add"].long(), st["ring"], st["table"]
    rows, size, width = st["rows"], ring.numel(), table.shape[1]
    head, count = st["state"][0].long(), st["state"][1].long()
    ends, grow = add == -1, add.clamp(min=0)
    have, want = (held + BLOCK - 1) // BLOCK, (held + grow + BLOCK - 1) // BLOCK
    end = torch.cumsum(grow, 0)
    start = torch.cat([torch.zeros_like(end[:1]), end])
    fits = ~ends & (want <= width) & (end <= rows)
    need = torch.where(fits, want - have, torch.zeros_like(want))
    upto = torch.cumsum(need, 0)
    granted = fits & ((need == 0) | (upto <= count))
    taken = torch.where(granted, need, torch.zeros_like(need)).sum()
    back = torch.where(ends, have, torch.zeros_like(have))
    column = torch.arange(width, device="cuda")[None]
    # blocks of requests that end go behind the free ones; entries of all others to a place that is cut off
    give = torch.where(ends[:, None] & (column < have[:, None]), (head + count + (torch.cumsum(back, 0) - back)[:, None] + column) % size,
                       torch.full_like(column, size))
    fresh = ring[(head + (upto - need)[:, None] + column - have[:, None]) % size]
    new = granted[:, None] & (column >= have[:, None]) & (column < want[:, None])
    ring.copy_(torch.cat([ring, ring[:1]]).scatter(0, give.flatten(), table.flatten())[:size])
    table.copy_(torch.where(new, fresh, table))
    r = torch.arange(rows, device="cuda")
    q = torch.searchsorted(end, r, right=True).clamp(max=held.numel() - 1)
    live = r < end[-1]
    pos = torch.where(live, held[q] + r - start[q], torch.zeros_like(r))
    slot = table[q, (pos // BLOCK).clamp(max=width - 1)].long() * BLOCK + pos % BLOCK
    slot = torch.where(live & granted[q], slot, torch.full_like(slot, -1))
    held_out = torch.where(ends, torch.zeros_like(held), torch.where(granted, held + grow, held))
    state = torch.stack([(head + taken) % size, count - taken + back.sum()])
    return [table, held_out.to(torch.int32), start.clamp(max=rows).to(torch.int32), slot.to(torch.int32), pos.to(torch.int32), state.to(torch.int32), ring]


def _rounded(x, e):
    """floor(x / 2^e + 1/2)"""
    return (x + ((1 << e.long()) >> 1)) >> e.long()


def _exponent(amax, headroom):
    """The smallest e with amax (8 + headroom) <= 1016 * 2^e."""
    return (amax[..., None] * (8 + headroom) > 1016 << torch.arange(12, device=amax.device)).sum(dim=-1)


def _rotated(x, st):
    """x [rows, heads, dim] in 16 bits, its first `rot` dimensions rotated."""
    x, rot = x.long().clamp(-32768, 32767), st["case"]["rot"]
    if rot == 0:
        return x
    cs = st["rotary"][st["position"].long()].long()[:, None]
    c, s = cs[..., 0], cs[..., 1]
    part = x[..., :rot]
    if st["case"]["layout"] == "half":
        a, b = part[..., :rot // 2], part[..., rot // 2:]
    else:
        a, b = part[..., 0::2], part[..., 1::2]
    a, b = (a * c - b * s + 8192) >> 14, (a * s + b * c + 8192) >> 14
    part = torch.cat([a, b], dim=-1) if st["case"]["layout"] == "half" else torch.stack([a, b], dim=-1).flatten(-2)
    return torch.cat([part, x[..., rot:]], dim=-1)


def _plain_append(st):
    case, cache, used = st["case"], st["cache"], st["used"]
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    q = _rotated(st["q"].unflatten(1, (heads, dim)), st)
    e = _exponent(q.abs().amax(dim=-1), 0)
    st["q8"].copy_(_rounded(q, e[..., None]).clamp(-127, 127))
    st["q_exp"].copy_(e)
    slot = st["slot"][:used].long()
    block, off = slot // BLOCK, slot % BLOCK
    first = torch.arange(used, device="cuda") - off            # the row that holds the block's first token, if this call has it
    here = (first >= 0) & (slot[first.clamp(min=0)] == slot - off)
    for name, x, headroom in (("k", _rotated(st["k"].unflatten(1, (kv, dim)), st), HEADROOM[0]),
                              ("v", st["v"].unflatten(1, (kv, dim)).long().clamp(-32768, 32767), HEADROOM[1])):
        x, exps = x[:used], cache[name + "_exp"]
        e = torch.where(here[:, None], _exponent(x.abs().amax(dim=-1), headroom)[first.clamp(min=0)], exps[block].long())
        exps[block] = e.to(torch.uint8)
        x = _rounded(x, e[..., None]).clamp(-127, 127).to(torch.int8)
        if name == "k":
            cache["k"].transpose(1, 2)[block, off] = x
        else:
            cache["v"].permute(0, 3, 1, 2)[block, off] = x
    return [st["q8"], st["q_exp"], cache["k"], cache["v"], cache["k_exp"], cache["v_exp"]]


def _segments():
    """Mantissas (in 2^-23) of the weights' 64 segments of an octave; within one they rise by 2^-13 a step."""
    c = torch.arange(64, dtype=torch.float64, device="cuda")
    return (torch.pow(2.0, 23 + (2 * c + 1) / 128).round() - 65536).clamp(min=2.0 ** 23)


def _weight(n):
    """Weight of a distance n <= 0 from the maximum, in 2^-13 octaves: 2^(15 + n / 8192), rounded to a whole number."""
    n = n.clamp(min=-(1 << 18))
    g = n & 8191
    return torch.ldexp(_segments()[g >> 7] + 1024 * (g & 127), (n >> 13) - 8).round()


def _out(A, L, V, st, channel):
    """Sums of weighted values and of weights, to the output's units: A 2^(V + 8) / L through a reciprocal of 32 bits."""
    a = 32 - torch.frexp(L.clamp(min=1).double())[1].long()
    left = lambda x, n: torch.where(n >= 0, x << n.clamp(min=0), x >> (-n).clamp(min=0))     # noqa: E731
    rho = ((1 << 63) - 1) // left(L.clamp(min=1), a)
    o = (left(A, (a - 8)[..., None]) * rho[..., None] + (1 << (46 - V))[..., None]) >> (47 - V)[..., None]
    o = torch.where((L > 0)[..., None], o, torch.zeros_like(o))
    m, s = st["m0"].long()[channel], st["s"].long()[channel]
    y = (o * m + (1 << (30 + s))) >> (31 + s)
    return y.clamp(*st["clamp"]) if st["clamp"] else y


def _plain_attn(st):
    case, cache, table, y = st["case"], st["cache"], st["table"].long(), st["y"]
    heads, kv, dim, n, width = case["heads"], case["kv"], case["dim"], case["n"], st["width"]
    group, most, keys = heads // kv, st["most_add"], width * BLOCK
    start, held = st["row_start"].long(), st["held"].long()
    m0, shift = st["score"]
    key = torch.arange(keys, device="cuda")
    channels = torch.arange(heads * dim, device="cuda").view(kv, 1, group, dim)
    # scores of as many rows, heads and requests at a time as fit
    step_q = max(1, min(most, (1 << 27) // (keys * group)))
    step_h = max(1, min(kv, (1 << 27) // (keys * group * step_q), (1 << 28) // (keys * dim)))
    step_n = max(1, min(n, (1 << 27) // (keys * group * step_q * step_h), (1 << 28) // (keys * dim * step_h)))
    for n0 in range(0, n, step_n):
        tab, s0, s1, lens = table[n0:n0 + step_n], start[:n][n0:n0 + step_n], start[1:][n0:n0 + step_n], held[n0:n0 + step_n]
        for h0 in range(0, kv, step_h):
            hs = slice(h0, h0 + step_h)
            k = cache["k"][tab, hs].permute(0, 2, 1, 3, 4).flatten(2, 3).float()                  # [requests, heads, keys, dim]
            v = cache["v"][tab, hs].permute(0, 2, 1, 4, 3).flatten(2, 3).double()
            ek, ev = (cache[x][tab, hs].long().clamp(max=12).transpose(1, 2)[:, :, None, None] for x in ("k_exp", "v_exp"))
            for q0 in range(0, most, step_q):
                i = q0 + torch.arange(min(step_q, most - q0), device="cuda")
                row = (s0[:, None] + i).clamp(max=st["rows"] - 1)
                live = s0[:, None] + i < s1[:, None]
                pos = lens[:, None] - (s1 - s0)[:, None] + i
                see = live[..., None] & (key < lens[:, None, None])
                if case["causal"]:
                    see = see & (key <= pos[..., None])
                if case["window"]:
                    see = see & (key > pos[..., None] - case["window"])
                see = see[:, None, :, None].unflatten(-1, (width, BLOCK))                         # [requests, 1, rows, 1, blocks, 128]
                q = st["q8"][row].unflatten(2, (kv, group))[:, :, hs].transpose(1, 2)             # [requests, heads, rows, group, dim]
                eq = st["q_exp"][row].unflatten(2, (kv, group))[:, :, hs].transpose(1, 2).long().clamp(max=12)
                s = torch.matmul(q.flatten(2, 3).float(), k.transpose(2, 3)).view(q.shape[:4] + (width, BLOCK))
                W = ((m0 << (eq[..., None] + ek)) >> shift).clamp(max=(1 << 31) - 1)
                t = torch.where(see, (s.long() * W[..., None]) >> 23, torch.full_like(s, -1 << 40, dtype=torch.int64))
                T = t.amax(dim=(-2, -1))
                V = torch.where(see.any(dim=-1), ev, torch.zeros_like(ev)).amax(dim=-1).expand_as(T)
                d = (V[..., None] - ev).clamp(min=0)
                p = torch.where(see, _weight(t - T[..., None, None] - 8192 * d[..., None]), torch.zeros_like(t, dtype=torch.float64))
                L = (p.sum(dim=-1).long() << d).sum(dim=-1)
                A = torch.matmul(p.view(q.shape[:2] + (-1, keys)), v).long().view(q.shape)
                out = _out(A, L, V, st, channels[hs]).to(y.dtype).transpose(1, 2)                 # [requests, rows, heads, group, dim]
                at = torch.where(live, row, torch.full_like(row, st["rows"]))                     # rows of no request: to a place that is cut off
                part = y.unflatten(1, (kv, group, dim))[:, hs]
                whole = torch.cat([part, part[:1]])
                whole[at.flatten()] = out.flatten(0, 1)
                part.copy_(whole[:-1])
    return y


def run(st):
    op = st["case"]["op"]
    if own:
        import paper_2206_08869_b200 as G
        h = st["handle"]
        if op == "plan":
            G.iodf_attn_plan(h, st["held"], st["add"], st["table"], st["ring"], st["state"], st["rows"], held_out=st["held_out"],
                             row_start=st["row_start"], slot=st["slot"], position=st["position"], state_out=st["state_out"])
            return [st["table"], st["held_out"], st["row_start"], st["slot"], st["position"], st["state_out"], st["ring"]]
        if op == "append":
            G.iodf_attn_append(h, st["q"], st["k"], st["v"], st["slot"], st["position"], st["cache"], q8=st["q8"], q_exp=st["q_exp"])
            c = st["cache"]
            return [st["q8"], st["q_exp"], c["k"], c["v"], c["k_exp"], c["v_exp"]]
        return G.iodf_attn_forward(h, st["q8"], st["q_exp"], st["row_start"], st["held"], st["table"], st["cache"], y=st["y"])
    return {"plan": _plain_plan, "append": _plain_append, "attn": _plain_attn}[op](st)


# ---- work ---------------------------------------------------------------------------------------------------
def _visible(case):
    """Pairs of rows and keys of one head, and the keys of a request that some row sees, summed over the requests."""
    pairs = keys = 0
    for h, a in zip(*_lengths(case)):
        total, w = h + a, case["window"]
        if not a:
            continue
        if not case["causal"]:
            pairs, keys = pairs + a * total, keys + total
            continue
        w = w or total
        full = max(0, min(a, total - max(h, w)))               # rows behind a whole window
        part = a - full                                        # the ones before them see h + 1, h + 2, ... keys
        pairs += full * w + part * h + part * (part + 1) // 2
        keys += min(total, a + w - 1)
    return pairs, keys


def work(case):
    held, add = _lengths(case)
    new = sum(max(0, a) for a in add)
    if case["op"] == "plan":
        n = len(held)
        fresh = sum(_blocks(h + a) - _blocks(h) for h, a in zip(held, add) if a > 0)
        gone = sum(_blocks(h) for h, a in zip(held, add) if a < 0)
        used = sum(_blocks(h + a) - h // BLOCK for h, a in zip(held, add) if a > 0)
        return {"bytes": 4 * (4 * n + 5 + 2 * max(case["rows"], 1) + 2 * fresh + 2 * gone + used), "flops": 0}
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    if case["op"] == "append":
        size = 1 if case["x"] == "int8" else 4
        rows = max(case["rows"], new)
        return {"bytes": rows * heads * (dim * (size + 1) + 1) + new * 2 * kv * dim * (size + 1) + rows * 8 + new * 2 * case["rot"], "flops": 6 * new * (heads + kv) * case["rot"]}
    pairs, keys = _visible(case)
    size = 1 if case["y"] == "int8" else 4
    return {"bytes": keys * kv * 2 * dim + new * heads * (dim * (1 + size) + 1), "flops": 4 * pairs * heads * dim}


# ---- the definition in 64 bits --------------------------------------------------------------------------------
def _exact_plan(st):
    held, add, table, ring = (st[k].tolist() for k in ("held", "add", "table", "ring"))
    head, count = st["state"].tolist()
    size, rows, width = len(ring), st["rows"], st["table"].shape[1]
    slot, position, start, held_out = [-1] * rows, [0] * rows, [0], []
    taken = asked = given = 0
    pushed = []
    for q, (h, a) in enumerate(zip(held, add)):
        at, grow = start[-1], max(0, a)
        start.append(at + grow)
        have, want = _blocks(h), _blocks(h + grow)
        ok = a != -1 and want <= width and at + grow <= rows
        if ok:
            asked += want - have
            ok = want == have or asked <= count
        if ok:
            for c in range(have, want):
                table[q][c] = ring[(head + taken) % size]
                taken += 1
        if a == -1:
            pushed += table[q][:have]
            given += have
        held_out.append(0 if a == -1 else h + grow if ok else h)
        for i in range(min(grow, max(0, rows - at))):
            p = h + i
            position[at + i] = p
            slot[at + i] = table[q][p // BLOCK] * BLOCK + p % BLOCK if ok else -1
    for i, b in enumerate(pushed):
        ring[(head + count + i) % size] = b
    state = [(head + taken) % size, count - taken + given]
    return [_ints(table), _ints(held_out), _ints([min(rows, s) for s in start]), _ints(slot), _ints(position), _ints(state), _ints(ring)]


def _exact_exponent(amax, headroom):
    """From the quotient instead of from thresholds: the number of doublings of 1016 that amax (8 + headroom) is beyond."""
    over = (amax * (8 + headroom) + 1015) // 1016              # amax (8 + headroom) <= 1016 2^e exactly if this is <= 2^e
    m, e = torch.frexp(over.double())
    return torch.where(over <= 1, torch.zeros_like(over), e.long() - (m == 0.5).long())


def _exact_append(st):
    case, cache = st["case"], {k: v.clone() for k, v in st["cache"].items()}
    rot, used = case["rot"], st["used"]

    def turned(x, heads):
        x = x.unflatten(1, (heads, case["dim"])).double().clamp(-32768, 32767).clone()
        if rot:
            cs = st["rotary"].double()[st["position"].long()]
            i = torch.arange(rot // 2, device="cuda")
            lo, hi = (i, i + rot // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
            a, b, c, s = x[..., lo], x[..., hi], cs[:, None, :, 0], cs[:, None, :, 1]
            x[..., lo], x[..., hi] = torch.floor((a * c - b * s) / 16384 + 0.5), torch.floor((a * s + b * c) / 16384 + 0.5)
        return x

    q = turned(st["q"], case["heads"])
    e = _exact_exponent(q.abs().amax(dim=-1).long(), 0)
    q8 = torch.floor(q / torch.pow(2.0, e.double())[..., None] + 0.5).clamp(-127, 127)
    slots, start = st["slot"].tolist(), st["row_start"].tolist()
    k, v = turned(st["k"], case["kv"]), st["v"].unflatten(1, (case["kv"], case["dim"])).double().clamp(-32768, 32767)
    for a, b in zip(start, start[1:]):
        r = a
        while r < b:                                           # a block's part of the request at a time
            block, off = divmod(slots[r], BLOCK)
            m = min(b - r, BLOCK - off)
            for name, x, headroom in (("k", k, HEADROOM[0]), ("v", v, HEADROOM[1])):
                exps = cache[name + "_exp"]
                if off == 0:
                    exps[block] = _exact_exponent(x[r].abs().amax(dim=-1).long(), headroom).to(torch.uint8)
                part = torch.floor(x[r:r + m] / torch.pow(2.0, exps[block].double())[None, :, None] + 0.5).clamp(-127, 127).to(torch.int8)
                if name == "k":
                    cache["k"][block, :, off:off + m] = part.transpose(0, 1)
                else:
                    cache["v"][block, :, :, off:off + m] = part.permute(1, 2, 0)
            r += m
    assert r <= used or not used
    return [q8.to(torch.int8), e.to(torch.uint8), cache["k"], cache["v"], cache["k_exp"], cache["v_exp"]]


def _exact_segments():
    """The same mantissas by whole numbers alone: x = 2^(23 + (2 c + 1) / 128) rounded has (2 x - 1)^128 <= 2^(128 * 24 + 2 c + 1) < (2 x + 1)^128."""
    out = []
    for c in range(64):
        x = 1 << 23
        for bit in range(22, -1, -1):
            if (2 * (x + (1 << bit)) - 1) ** 128 <= 1 << (128 * 24 + 2 * c + 1):
                x += 1 << bit
        out.append(max(1 << 23, x - 65536))
    return torch.tensor(out, device="cuda")


def _exact_weight(n, segments):
    """2^15 2^(n / 8192) by the segments, with the rounding done in whole numbers (to nearest, ties to even)."""
    n = n.clamp(min=-(1 << 18))
    octave, g = torch.div(n, 8192, rounding_mode="floor"), torch.remainder(n, 8192)
    mantissa = segments[torch.div(g, 128, rounding_mode="floor")] + 1024 * torch.remainder(g, 128)
    drop = (8 - octave).clamp(max=40)
    whole, rest, half = mantissa >> drop, mantissa & ((1 << drop) - 1), 1 << (drop - 1)
    return whole + ((rest > half) | ((rest == half) & (whole % 2 == 1))).long()


def _exact_scaled(x, n):
    """floor(x 2^n)"""
    up, down = 1 << n.clamp(min=0), 1 << (-n).clamp(min=0)
    return torch.div(x * up, down, rounding_mode="floor")


def _exact_out(A, L, V, st, channel):
    bits = torch.zeros_like(L)                                 # length of L in bits
    for b in range(48):
        bits += (L >= 1 << b).long()
    L = L[..., None]
    a = 32 - bits[..., None]
    rho = torch.div((1 << 63) - 1, _exact_scaled(L, a).clamp(min=1), rounding_mode="floor")
    cut = 1 << (47 - V[..., None])
    o = torch.div(_exact_scaled(A, a - 8) * rho + torch.div(cut, 2, rounding_mode="floor"), cut, rounding_mode="floor").masked_fill(L == 0, 0)
    m, s = st["m0"].long()[channel], st["s"].long()[channel]
    y = torch.div(o * m + (1 << (30 + s)), 1 << (31 + s), rounding_mode="floor")
    return y if st["clamp"] is None else y.clamp(*st["clamp"])


def _exact_attn(st):
    segments = _exact_segments()
    case, cache, y = st["case"], st["cache"], st["y"].clone().long()
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    group = heads // kv
    start, held, table = st["row_start"].tolist(), st["held"].tolist(), st["table"].tolist()
    m0, shift = st["score"]
    for q in range(case["n"]):
        r0, r1, length = start[q], start[q + 1], held[q]
        if r0 == r1:
            continue
        nb = _blocks(length)
        ids = torch.tensor(table[q][:nb], device="cuda")
        for h in range(kv):
            k = cache["k"][ids, h].reshape(nb * BLOCK, dim)[:length].double()
            v = cache["v"][ids, h].permute(0, 2, 1).reshape(nb * BLOCK, dim)[:length].double()
            ek, ev = (cache[x][ids, h].long().clamp(max=12).repeat_interleave(BLOCK)[:length] for x in ("k_exp", "v_exp"))
            channel = torch.arange(heads * dim, device="cuda").view(heads, dim)[h * group:(h + 1) * group]
            step = max(1, (1 << 26) // (length * group))
            for a in range(r0, r1, step):
                b = min(r1, a + step)
                pos = length - (r1 - r0) + torch.arange(a - r0, b - r0, device="cuda")[:, None, None]
                key = torch.arange(length, device="cuda")
                see = torch.ones_like(pos * key, dtype=torch.bool)
                if case["causal"]:
                    see &= key <= pos
                if case["window"]:
                    see &= pos - key < case["window"]
                s = torch.einsum("rgd,kd->rgk", st["q8"][a:b, h * group:(h + 1) * group].double(), k).long()
                e = st["q_exp"][a:b, h * group:(h + 1) * group].long().clamp(max=12)[..., None] + ek
                W = torch.div(m0 * (1 << e), 1 << shift, rounding_mode="floor").clamp(max=(1 << 31) - 1)
                t = torch.div(s * W, 1 << 23, rounding_mode="floor").masked_fill_(~see, -1 << 40)
                T = t.amax(dim=-1, keepdim=True)
                V = ev.masked_fill(~see, 0).amax(dim=-1, keepdim=True)
                p = _exact_weight(t - T - 8192 * (V - ev), segments).masked_fill_(~see, 0)
                L = (p * (1 << (V - ev).clamp(min=0))).sum(dim=-1)
                A = torch.einsum("rgk,kd->rgd", p.double(), v).long()
                y[a:b].unflatten(1, (heads, dim))[:, h * group:(h + 1) * group] = _exact_out(A, L, V[..., 0].expand_as(L), st, channel)
    return y.to(_TORCH[case["y"]])


def exact(case, seed):
    st = _inputs(case, seed)
    return {"plan": _exact_plan, "append": _exact_append, "attn": _exact_attn}[case["op"]](st)
