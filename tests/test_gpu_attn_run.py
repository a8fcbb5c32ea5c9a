"""Plan, append and attention as they are used: together with projections and norms, cut into steps, captured, on other streams."""
import numpy as np
import pytest

from oracle import attention as A
from oracle import layers as OL
from tests import attn_cases as C

pytestmark = pytest.mark.gpu


def _modules():
    import torch
    import paper_2206_08869_b200 as G
    return torch, G


class _Server:
    """A cache with its free blocks and requests, and the three calls of a step."""

    def __init__(self, torch, G, desc, requests, blocks, width, seed=0):
        self.torch, self.G, self.attn = torch, G, G.iodf_attn_create(desc)
        self.desc, self.cache = desc, G.iodf_attn_cache(self.attn, blocks)
        for t in self.cache.values():
            t.random_(0, 100)                               # what the cache holds before does not matter
        rng = np.random.default_rng(seed)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")        # noqa: E731
        self.table, self.ring, self.state = ints([[-1] * width] * requests), ints(rng.permutation(blocks)), ints([rng.integers(blocks), blocks])
        self.held = ints([0] * requests)

    def step(self, x, add, rows=None, y=None):
        G, d = self.G, self.desc
        nq, nk = d["heads"] * d["head_dim"], d["kv_heads"] * d["head_dim"]
        rows = x.shape[0] if rows is None else rows
        add = self.torch.tensor(add, dtype=self.torch.int32, device="cuda") if isinstance(add, list) else add
        held, start, slot, position, state = G.iodf_attn_plan(self.attn, self.held, add, self.table, self.ring, self.state, rows)
        q8, q_exp = G.iodf_attn_append(self.attn, x[:, :nq], x[:, nq:nq + nk], x[:, nq + nk:], slot, position, self.cache)
        y = G.iodf_attn_forward(self.attn, q8, q_exp, start, held, self.table, self.cache, y=y)
        self.held, self.state = held, state
        return y, start


@pytest.mark.parametrize("dim,heads,kv,window", [(64, 4, 2, 0), (128, 8, 1, 0), (32, 3, 3, 150)])
def test_any_cut_of_the_tokens_gives_the_same(dim, heads, kv, window):
    """What an encoder computes in one pass a decoder gets token by token, bit for bit: prompts, chunks and single tokens, alone and beside
    other requests, go through different kernels, splits and blocks."""
    torch, G = _modules()
    d = C.description(torch, heads, kv, dim, "int32", 32, window=window)
    total = 700
    gen = torch.Generator(device="cuda").manual_seed(dim)
    x = torch.randn((3, total, (heads + 2 * kv) * dim), generator=gen, device="cuda").mul_(2500).round_().to(torch.int32)
    whole, _ = _Server(torch, G, d, 1, 9, 6).step(x[0], [total])
    assert whole.abs().float().mean() > 5
    for cuts in ([300, 400], [1] * 40 + [87, 1, 128, 256, 1] + [1] * 60 + [127]):
        s = _Server(torch, G, d, 1, 9, 6, seed=3)
        parts, at = [], 0
        for m in cuts:
            parts.append(s.step(x[0, at:at + m], [m])[0])
            at += m
        assert at == total and torch.equal(torch.cat(parts), whole)
        G.iodf_attn_check(s.attn)
    # beside two others that run at another pace
    s, at = _Server(torch, G, d, 3, 40, 6, seed=4), [0, 0, 0]
    parts = []
    for m in [(5, 100, 0), (1, 1, 200), (250, 3, 1), (1, 0, 1), (443, 130, 90)]:
        rows = torch.cat([x[q, at[q]:at[q] + m[q]] for q in (1, 0, 2)])
        y, start = s.step(rows, [m[1], m[0], m[2]])
        parts.append(y[m[1]:m[1] + m[0]])
        at = [a + b for a, b in zip(at, m)]
    assert torch.equal(torch.cat(parts), whole)
    G.iodf_attn_check(s.attn)


def test_blocks_come_back_and_serve_others():
    torch, G = _modules()
    d = C.description(torch, 2, 1, 32)
    x = torch.randint(-3000, 3000, (400, 4 * 32), device="cuda", dtype=torch.int32)
    fresh, _ = _Server(torch, G, d, 1, 4, 4).step(x, [400])
    s = _Server(torch, G, d, 2, 5, 4)
    s.step(x[:300], [300, 0])
    s.step(x[:150], [0, 150])                               # all five blocks are taken
    with pytest.raises(G.IodfError):
        s.step(x[:200], [200, 0])
        G.iodf_attn_check(s.attn)
    s.step(x[:0], [-1, -1], rows=0)
    assert s.held.tolist() == [0, 0] and s.state[1].item() == 5
    y, _ = s.step(x, [0, 400])
    assert torch.equal(y, fresh)
    G.iodf_attn_check(s.attn)


def _layer(rng, k, n, y):
    return {"k": 1, "c_in": k, "c_out": n, "w": rng.integers(-60, 61, (n, k)).astype(np.int8), "bias": rng.integers(-4000, 4000, n).astype(np.int32),
            "m0": rng.integers(1 << 30, 1 << 31, n).astype(np.int32), "s": np.full(n, 2 if y == "int32" else 8, np.int32), "relu": False,
            "clamp": None if y == "int32" else (-128, 127)}


def test_a_block_of_norm_projection_attention_projection_and_residual():
    """One block of a network over tokens: n = N(r); q, k, v = W n; a = attention; r += scale * U a, against the plain definitions of all."""
    torch, G = _modules()
    rng = np.random.default_rng(8)
    width, heads, kv, dim, rows = 96, 4, 2, 32, 333
    d = C.description(torch, heads, kv, dim, "int32", 32, "interleaved", seed=2)
    qkv, out = _layer(rng, width, (heads + 2 * kv) * dim, "int32"), _layer(rng, heads * dim, width, "int8")
    pre = {"norm": "rms", "mult": np.full(width, 1 << 30, np.int32), "shift": 12, "bias": np.zeros(width, np.int32), "clamp": (-128, 127), "dtype": torch.int8}
    post = {"norm": None, "mult": np.full(width, 7 << 28, np.int32), "shift": 1}
    first = G.iodf_norm_create({"c": width, "res_dtype": torch.int32, "eps": 96, "pre": pre})
    last = G.iodf_norm_create({"c": width, "res_dtype": torch.int32, "block_dtype": torch.int8, "eps": 96, "post": post, "res_range": (-2 ** 23, 2 ** 23 - 1)})
    up = G.iodf_proj_create(qkv, rows, x_dtype=torch.int8, y_dtype=torch.int32)
    down = G.iodf_proj_create(out, rows, x_dtype=torch.int8, y_dtype=torch.int8)
    r_host = rng.normal(0, 900, (rows, width)).astype(np.int32)
    s = _Server(torch, G, d, 2, 9, 4)

    def block(r, add):
        _, n = G.iodf_norm_forward(first, r)
        a, _ = s.step(G.iodf_proj_forward(up, n), add)
        r, _ = G.iodf_norm_forward(last, r, G.iodf_proj_forward(down, a), r_out=r)
        return n, r
    add = [200, 133]
    n, r = block(torch.from_numpy(r_host).cuda(), add)
    n = n.cpu().numpy()
    x = OL.projection(qkv, n)
    table, ring = np.zeros((2, 4), np.int64), np.arange(9)
    held, start, slot, position, state, refused = A.plan([0, 0], add, table, ring, [0, 9], rows)
    cache = {"k": np.zeros((9, kv, 128, dim), np.int8), "v": np.zeros((9, kv, dim, 128), np.int8), "k_exp": np.zeros((9, kv), np.uint8), "v_exp": np.zeros((9, kv), np.uint8)}
    nq, nk = heads * dim, kv * dim
    q8, e = A.append(d, x[:, :nq], x[:, nq:nq + nk], x[:, nq + nk:], slot, position, cache)
    a = A.forward(d, q8, e, start, held, table, cache, np.zeros((rows, nq), np.int64))
    b = np.clip(OL.projection(out, a), -128, 127)
    want = OL.norm_step({"eps": 96, "post": dict(post, mult=post["mult"].astype(np.int64)), "res_range": (-2 ** 23, 2 ** 23 - 1)}, r_host, b)[0]
    np.testing.assert_array_equal(r.cpu().numpy(), want)
    # and the same rows with the requests' tokens one step after the other
    s = _Server(torch, G, d, 2, 9, 4, seed=1)
    got = []
    for lo in range(0, 133, 19):
        rows_now = np.concatenate([np.arange(lo, min(200, lo + 19)), 200 + np.arange(lo, min(133, lo + 19))])
        got.append((rows_now, block(torch.from_numpy(r_host[rows_now]).cuda(), [min(200, lo + 19) - lo, min(133, lo + 19) - lo])[1].cpu().numpy()))
    for rows_now, r_now in got:
        np.testing.assert_array_equal(r_now, want[rows_now])
    G.iodf_attn_check(s.attn)


def test_captured_and_replayed_with_other_requests():
    """One graph of a step with room for padding serves other lengths, tables and tokens."""
    torch, G = _modules()
    d = C.description(torch, 4, 2, 64, "int32", 64)
    rows, n, blocks, width = 50, 6, 40, 5
    s = _Server(torch, G, d, n, blocks, width)
    x = torch.zeros((rows, 8 * 64), dtype=torch.int32, device="cuda")
    add = torch.zeros(n, dtype=torch.int32, device="cuda")
    held, state = s.held.clone(), s.state.clone()
    y = torch.full((rows, 4 * 64), 9, dtype=torch.int8, device="cuda")

    def step():
        h, start, slot, position, st = G.iodf_attn_plan(s.attn, held, add, s.table, s.ring, state, rows)
        q8, e = G.iodf_attn_append(s.attn, x[:, :256], x[:, 256:384], x[:, 384:], slot, position, s.cache)
        G.iodf_attn_forward(s.attn, q8, e, start, h, s.table, s.cache, y=y)
        held.copy_(h)
        state.copy_(st)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()                                              # nothing to do: all rows are padding
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
    torch.cuda.synchronize()
    plain = _Server(torch, G, d, n, blocks, width, seed=7)
    gen = torch.Generator().manual_seed(1)
    for turn in range(12):
        m = [[1] * n, [20, 0, 3, 1, 0, 9], [0, 0, 0, 0, 0, 0], [7, 7, 7, 7, 7, 7]][turn % 4]
        tokens = (torch.randn((sum(m), 8 * 64), generator=gen) * 2500).round().to(torch.int32).cuda()
        x.fill_(-7)
        x[:sum(m)] = tokens
        add.copy_(torch.tensor(m, dtype=torch.int32))
        y.fill_(9)
        graph.replay()
        want, _ = plain.step(tokens, m)
        assert torch.equal(y[:sum(m)], want) and bool((y[sum(m):] == 9).all())
    G.iodf_attn_check(s.attn)


def test_streams_of_their_own():
    """A call on another stream than the current one, outputs made by it, and two handles' calls at once on one cache."""
    torch, G = _modules()
    d = C.description(torch, 8, 2, 64, "int32")
    x = torch.randint(-3000, 3000, (500, 12 * 64), device="cuda", dtype=torch.int32)
    want, _ = _Server(torch, G, d, 1, 6, 4).step(x, [500])
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")            # noqa: E731
    a, b = G.iodf_attn_create(d), G.iodf_attn_create(d)
    cache = G.iodf_attn_cache(a, 6)
    held, add, table, ring, state = ints([0]), ints([500]), ints([[-1] * 4]), ints([5, 2, 0, 1, 4, 3]), ints([4, 6])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    torch.empty(1 << 26, device="cuda").fill_(1.0)          # the current stream is busy
    h, start, slot, position, _ = G.iodf_attn_plan(a, held, add, table, ring, state, 500, stream=st)
    q8, e = G.iodf_attn_append(a, x[:, :512], x[:, 512:640], x[:, 640:], slot, position, cache, stream=st)
    y = G.iodf_attn_forward(a, q8, e, start, h, table, cache, stream=st)
    G.iodf_attn_check(a, st)
    assert torch.equal(y, want)
    outs, one = [], ints([0, 1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    for i in range(24):                                     # readers of one cache, some of single rows (another kernel)
        k = streams[i % 4]
        if i % 3:
            outs.append((G.iodf_attn_forward((a, b)[i % 2], q8, e, start, h, table, cache, stream=k), want))
        else:
            outs.append((G.iodf_attn_forward(a, q8[499:], e[499:], one, h, table, cache, stream=k), want[499:]))
    torch.cuda.synchronize()
    for got, right in outs:
        assert torch.equal(got, right)
    G.iodf_attn_check(a)
    G.iodf_attn_check(b)


def test_a_cache_beyond_32_bits():
    """Blocks whose keys and values lie more than 2^32 bytes behind the cache's beginning."""
    torch, G = _modules()
    d = C.description(torch, 8, 8, 128, "int32", 128, positions=600)
    blocks = (1 << 32) // (8 * 128 * 128) + 6               # keys of 4.3 GB, and values
    x = torch.randint(-3000, 3000, (600, 24 * 128), device="cuda", dtype=torch.int32)
    want, _ = _Server(torch, G, d, 1, 6, 5).step(x, [600])
    attn = G.iodf_attn_create(d)
    cache = {k: torch.empty(s, dtype=t, device="cuda") for k, s, t in (("k", (blocks, 8, 128, 128), torch.int8), ("v", (blocks, 8, 128, 128), torch.int8),
                                                                      ("k_exp", (blocks, 8), torch.uint8), ("v_exp", (blocks, 8), torch.uint8))}
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")            # noqa: E731
    ring = torch.arange(blocks - 1, -1, -1, device="cuda").to(torch.int32)
    h, start, slot, position, _ = G.iodf_attn_plan(attn, ints([0]), ints([600]), ints([[0] * 5]).requires_grad_(False), ring, ints([0, blocks]), 600)
    table = (slot[::128] // 128)[None].contiguous()
    q8, e = G.iodf_attn_append(attn, x[:, :1024], x[:, 1024:2048], x[:, 2048:], slot, position, cache)
    assert torch.equal(G.iodf_attn_forward(attn, q8, e, start, h, table, cache), want)
    assert torch.equal(G.iodf_attn_forward(attn, q8[599:], e[599:], ints([0, 1]), h, table, cache), want[599:])
    G.iodf_attn_check(attn)


def test_what_a_call_refuses():
    torch, G = _modules()
    d = C.description(torch, 4, 2, 32, "int32")
    attn = G.iodf_attn_create(d)
    cache = G.iodf_attn_cache(attn, 4)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")            # noqa: E731
    held, add, table, ring, state = ints([0, 3]), ints([1, 1]), ints([[0, 0], [1, 0]]), ints([0, 1, 2, 3]), ints([2, 2])

    def status(f, *args, **kw):
        with pytest.raises(G.IodfError) as e:
            f(*args, **kw)
        return e.value.status
    plan, append, forward = G.iodf_attn_plan, G.iodf_attn_append, G.iodf_attn_forward
    assert status(plan, attn, held, add, table, ring, state, 2, held_out=held) == -1          # outputs on inputs
    assert status(plan, attn, held, add, table, ring, state, 2, state_out=state) == -1
    assert status(plan, attn, held, add, table, ring, state, 2, slot=ring[:2], position=ring[2:]) == -1
    assert status(plan, attn, held, add, ints([[0] * 1025] * 2), ring, state, 2) == -6
    x = torch.zeros((2, 8 * 32), dtype=torch.int32, device="cuda")
    q8, e = torch.zeros((2, 4, 32), dtype=torch.int8, device="cuda"), torch.zeros((2, 4), dtype=torch.uint8, device="cuda")
    slot, position, start = ints([0, 131]), ints([0, 3]), ints([0, 1, 2])
    assert status(append, attn, x[:, :128], x[:, 128:192], x[:, 192:], slot, position, cache, q8=x.view(torch.int8).view(-1)[:256].view(2, 4, 32)) == -1
    whole = torch.zeros(4 * 2 * 128 * 32 + 16, dtype=torch.int8, device="cuda")
    shifted = dict(cache, k=whole[8:8 + 32768].view(4, 2, 128, 32))
    assert status(append, attn, x[:, :128], x[:, 128:192], x[:, 192:], slot, position, shifted) == -1
    assert status(append, attn, x[:, :128], x[:, 128:192], x[:, 192:], slot, position, dict(cache, v=cache["k"].view(4, 2, 32, 128))) == -1
    assert status(forward, attn, q8, e, start, held, table, cache, y=q8.view(2, 128)) == -1
    assert status(forward, attn, q8, e, start, held, table, cache, y=cache["v"].view(-1)[:256].view(2, 128)) == -1
    for call in (lambda: plan(attn, held.cpu(), add, table, ring, state, 2), lambda: plan(attn, held, add[:1], table, ring, state, 2),
                 lambda: plan(attn, held, add, table[:1], ring, state, 2), lambda: plan(attn, held.long(), add, table, ring, state, 2),
                 lambda: plan(attn, held, add, table, ring, state, -1), lambda: plan(attn, held, add, table.t().contiguous().t(), ring, state, 2),
                 lambda: append(attn, x[:, :127], x[:, 128:192], x[:, 192:], slot, position, cache),
                 lambda: append(attn, x[:, :128].char(), x[:, 128:192], x[:, 192:], slot, position, cache),
                 lambda: append(attn, x[:, :128], x[:, 128:192], x[:, 192:], slot[:1], position, cache),
                 lambda: append(attn, x[:, :128], x[:, 128:192], x[:, 192:], slot, position, dict(cache, k=cache["k"].transpose(2, 3))),
                 lambda: forward(attn, q8[:, :3], e, start, held, table, cache), lambda: forward(attn, q8, e, start[:2], held, table, cache),
                 lambda: forward(attn, q8, e, start, held, table, cache, y=torch.zeros((2, 128), dtype=torch.int32, device="cuda")),
                 lambda: forward(attn, q8, e, start, held, table, dict(cache, k_exp=cache["k_exp"][:2]))):
        with pytest.raises(ValueError):
            call()
    assert bool((cache["k"] == 0).all()) and held.tolist() == [0, 3] and ring.tolist() == [0, 1, 2, 3]
    G.iodf_attn_check(attn)


def test_bad_slots_positions_and_rows_are_counted():
    """They are neither written nor followed; what else the call has to do is done."""
    torch, G = _modules()
    d = C.description(torch, 2, 1, 32, "int32", 32, positions=10)
    attn = G.iodf_attn_create(d)
    cache = G.iodf_attn_cache(attn, 2)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")            # noqa: E731
    x = torch.randint(-3000, 3000, (5, 4 * 32), device="cuda", dtype=torch.int32)
    G.iodf_attn_append(attn, x[:, :64], x[:, 64:96], x[:, 96:], ints([0, 256, -5, 2 ** 31 - 1, 128]), ints([0, 1, 2, 3, 10]), cache)
    with pytest.raises(G.IodfError) as e:
        G.iodf_attn_check(attn)
    assert e.value.status == -9 and "(4 " in str(e.value)
    assert bool((cache["k"][:, :, 1:] == 0).all()) and bool((cache["k"][:, :, 0] != 0).any())
    q8, qe = torch.zeros((5, 2, 32), dtype=torch.int8, device="cuda"), torch.zeros((5, 2), dtype=torch.uint8, device="cuda")
    y = torch.full((5, 64), 3, dtype=torch.int8, device="cuda")
    G.iodf_attn_forward(attn, q8, qe, ints([4, 2]), ints([1]), ints([[0]]), cache, y=y)       # bounds that decrease: no rows
    assert bool((y == 3).all())
    G.iodf_attn_forward(attn, q8, qe, ints([-7, 2, 99]), ints([1, 1]), ints([[0], [1]]), cache, y=y)
    torch.cuda.synchronize()
    G.iodf_attn_forward(attn, q8[:1], qe[:1], ints([0, 1]), ints([-4]), ints([[0]]), cache, y=y[:1])
    assert bool((y[0] == 0).all())
    with pytest.raises(G.IodfError):
        G.iodf_attn_check(attn)


def test_more_free_blocks_than_the_ring_has_places_are_counted():
    torch, G = _modules()
    attn = G.iodf_attn_create(C.description(torch, 2, 1, 32, "int32"))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")            # noqa: E731
    for count, add, bad in ((2, [-1, 1], 0), (3, [-1, 1], 1), (3, [-1, 200], 1)):
        out = G.iodf_attn_plan(attn, ints([300, 0]), ints(add), ints([[0, 1, 2], [7, 7, 7]]), ints([3, 4, 5, 6, 7]), ints([0, count]), 200)
        assert out[4].tolist()[1] <= 5
        if bad:
            with pytest.raises(G.IodfError) as e:
                G.iodf_attn_check(attn)
            assert e.value.status == -9
        else:
            G.iodf_attn_check(attn)
