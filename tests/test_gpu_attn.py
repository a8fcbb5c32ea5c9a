"""Integer attention over a cache of blocks against the plain 64-bit definition, bit for bit."""
import numpy as np
import pytest

from oracle import attention as A
from tests import attn_cases as C

pytestmark = pytest.mark.gpu


def _modules():
    import torch
    import paper_2206_08869_b200 as G
    return torch, G


# ---- plan ---------------------------------------------------------------------------------------------------
def _plan_both(held, add, width, free, rows, head, blocks, seed=0, pad=0):
    torch, G = _modules()
    rng = np.random.default_rng(seed)
    order = rng.permutation(blocks)
    table, at = np.full((max(1, len(held)), width + pad), -9, np.int32), free
    for q, h in enumerate(held):
        n = min(A.blocks_of(max(0, int(h))), width)
        table[q, :n] = order[np.arange(at, at + n) % blocks]
        at += n
    table = table[:len(held)]
    ring = np.full(blocks, -3, np.int32)
    ring[(head + np.arange(free)) % blocks] = order[:free]
    held, add, state = np.array(held, np.int32), np.array(add, np.int32), np.array([head, free], np.int32)
    attn = G.iodf_attn_create(C.description(torch))
    g = [C.on_gpu(torch, x) for x in (held, add, table, ring, state)]
    if len(held):
        g[2] = g[2][:, :width] if width > 1 or pad else g[2]
    got = G.iodf_attn_plan(attn, g[0], g[1], g[2], g[3], g[4], rows)
    want_table, want_ring = table[:, :width].copy(), ring.copy()
    want = A.plan(held, add, want_table, want_ring, state, rows)
    for a, b, name in zip(got, want, ("held_out", "row_start", "slot", "position", "state_out")):
        np.testing.assert_array_equal(a.cpu().numpy(), b, err_msg=name)
    np.testing.assert_array_equal(g[2].cpu().numpy().reshape(want_table.shape), want_table)
    np.testing.assert_array_equal(g[3].cpu().numpy(), want_ring)
    for x, y in zip((g[0], g[1], g[4]), (held, add, state)):
        np.testing.assert_array_equal(x.cpu().numpy(), y)
    if want[5]:
        with pytest.raises(G.IodfError) as e:
            G.iodf_attn_check(attn)
        assert e.value.status == -9 and "(%d " % want[5] in str(e.value)
    G.iodf_attn_check(attn)


@pytest.mark.parametrize("held,add,width,free,rows,head,blocks", [
    ([0], [1], 1, 1, 1, 0, 4),                                   # a request's first token
    ([127], [1], 1, 0, 1, 0, 4),                                 # fits the block that it has
    ([128], [1], 2, 3, 1, 3, 4),                                 # the next block, from the ring's end
    ([128], [129], 3, 2, 129, 3, 5),                             # ... and over it
    ([5, 0, 300], [0, 0, 0], 3, 2, 4, 1, 9),                     # nothing new
    ([200, 5, 129], [-1, 3, -1], 2, 0, 3, 7, 9),                 # two end; nothing is free
    ([200, 5, 129], [-1, 130, 1], 2, 1, 140, 8, 12),             # what one gives back is for the next call
    ([0, 0, 0], [200, 300, 50], 4, 5, 600, 2, 8),                # the last one asks for one block too many
    ([0, 100, 0], [600, 3, 10], 8, 2, 700, 2, 12),               # the first is refused; one that needs no block is served, the last not
    ([0, 0], [300, 5], 2, 9, 400, 0, 12),                        # wider than the table: takes nothing
    ([0, 0, 0], [100, 60, 40], 2, 9, 150, 0, 12),                # the second's rows end behind the room
    ([-1, 3, 700], [5, -2, 1], 2, 9, 20, 0, 12),                 # not lengths
    ([10, 20], [1, 2], 1, 3, 3, 0, 5),
    ([], [], 1, 2, 3, 1, 4),                                     # no requests: all rows are padding
    ([7, 9], [-1, -1], 1, 0, 0, 3, 4),                           # no rows
])
@pytest.mark.parametrize("pad", [0, 3])
def test_plan(held, add, width, free, rows, head, blocks, pad):
    _plan_both(held, add, width, free, rows, head, blocks, pad=pad)


@pytest.mark.parametrize("n,rows,most", [(1, 5000, 5000), (37, 4001, 900), (511, 900, 300), (512, 4096, 9), (1025, 3000, 2000), (4000, 9000, 700)])
def test_plan_of_many(n, rows, most):
    rng = np.random.default_rng(n)
    held = rng.integers(0, most, n) * rng.integers(0, 2, n)
    add = np.minimum(rng.integers(0, max(2, 2 * rows // n), n) if n > 1 else [most], most)
    add[rng.random(n) < 0.2] = 0
    ends = (rng.random(n) < 0.1) & (n > 1)
    add[ends] = -1
    width = A.blocks_of(2 * most)
    need = int(sum(A.blocks_of(int(h + a)) - A.blocks_of(int(h)) for h, a in zip(held, add) if a > 0))
    used = int(sum(A.blocks_of(int(h)) for h in held))
    for free in (need + 5, need // 2):
        _plan_both(held, add, width, free, rows, (used + need) // 3, used + need + 9, seed=n)


# ---- append -------------------------------------------------------------------------------------------------
def _append_both(desc, rows, slot, position, blocks, seed, views="columns", limit=30000):
    torch, G = _modules()
    rng = np.random.default_rng(seed)
    heads, kv, dim = desc["heads"], desc["kv_heads"], desc["head_dim"]
    wide = (heads + 2 * kv) * dim + {"columns": 0, "odd": 3, "apart": 0}[views]
    int8 = desc["x_dtype"] is torch.int8
    x = np.clip(np.round(rng.normal(0, 32 if int8 else limit / 8, (rows, wide))), -128 if int8 else -2 ** 31, 127 if int8 else 2 ** 31 - 1)
    x = x.astype(np.int8 if int8 else np.int32)
    x[rng.random(rows) < 0.1] = 0                                # rows of zeros
    x[rng.random(rows) < 0.05, :] = -128 if int8 else -2 ** 31   # and of the lowest value
    at = {"columns": 0, "odd": 1, "apart": 0}[views]
    cut = [at, at + heads * dim, at + (heads + kv) * dim, at + (heads + 2 * kv) * dim]
    q, k, v = (x[:, a:b] for a, b in zip(cut, cut[1:]))
    cache = C.cache(desc, blocks, rng)
    gx, gc = C.on_gpu(torch, x), C.on_gpu(torch, cache)
    gq, gk, gv = (gx[:, a:b] for a, b in zip(cut, cut[1:]))
    if views == "apart":
        gq, gk, gv = (t.contiguous() for t in (gq, gk, gv))
    attn = G.iodf_attn_create(desc)
    q8, q_exp = G.iodf_attn_append(attn, gq, gk, gv, C.on_gpu(torch, slot.astype(np.int32)), C.on_gpu(torch, position.astype(np.int32)), gc)
    G.iodf_attn_check(attn)
    w8, we = A.append(desc, q, k, v, slot, position, cache)
    np.testing.assert_array_equal(q8.cpu().numpy(), w8)
    np.testing.assert_array_equal(q_exp.cpu().numpy(), we)
    for name in cache:
        np.testing.assert_array_equal(gc[name].cpu().numpy(), cache[name], err_msg=name)


def _slots(held, add, rng, extra=3, padding=0):
    total = [h + a for h, a in zip(held, add)]
    _, table, blocks = C.requests(total, add, rng, extra)
    slot = [int(table[q, t // 128]) * 128 + t % 128 for q in range(len(held)) for t in range(held[q], total[q])] + [-1] * padding
    position = [t for q in range(len(held)) for t in range(held[q], total[q])] + [0] * padding
    return np.array(slot), np.array(position), blocks


@pytest.mark.parametrize("x", ["int8", "int32"])
@pytest.mark.parametrize("dim,rot,layout", [(32, 0, "half"), (32, 32, "half"), (32, 16, "interleaved"), (64, 64, "interleaved"), (64, 16, "half"),
                                            (128, 128, "half"), (128, 128, "interleaved"), (128, 48, "half"), (128, 112, "interleaved")])
def test_append_layouts(dim, rot, layout, x):
    torch, _ = _modules()
    rng = np.random.default_rng(dim + rot)
    slot, position, blocks = _slots([0, 130, 60, 128], [3, 1, 70, 140], rng, padding=3)
    _append_both(C.description(torch, 6, 2, dim, x, rot, layout), len(slot), slot, position, blocks, dim + rot)


@pytest.mark.parametrize("held,add", [([0], [1]), ([127], [1]), ([128], [1]), ([127], [2]), ([0], [128]), ([3], [300]), ([0, 0, 0], [0, 0, 1]),
                                      ([5, 127, 250, 128], [1, 1, 1, 1]), ([0], [1111]), ([200, 0], [57, 33])])
@pytest.mark.parametrize("views", ["columns", "odd", "apart"])
def test_append_lengths_and_strides(held, add, views):
    torch, _ = _modules()
    rng = np.random.default_rng(sum(held) + len(add))
    slot, position, blocks = _slots(held, add, rng, padding=len(add) - 1)
    _append_both(C.description(torch, 3, 1, 64, "int32", 32, "half"), len(slot), slot, position, blocks, 5, views)


@pytest.mark.parametrize("heads,kv,rows,headroom", [(1, 1, 40, (0, 0)), (8, 8, 33, (8, 8)), (5, 1, 2100, (0, 8)), (40, 8, 9, (3, 0)), (8, 4, 4000, (2, 4))])
def test_append_heads(heads, kv, rows, headroom):
    torch, _ = _modules()
    rng = np.random.default_rng(rows)
    slot, position, blocks = _slots([77], [rows], rng)
    _append_both(C.description(torch, heads, kv, 32, "int32", 32, "interleaved", positions=4300, headroom=headroom), rows, slot, position, blocks, rows)


# ---- forward ------------------------------------------------------------------------------------------------
def _forward_both(desc, held, add, seed, padding=0, exps=(3, 7), strided=False, mangle=None, q_exps=(3, 8)):
    torch, G = _modules()
    rng = np.random.default_rng(seed)
    row_start, table, blocks = C.requests(held, add, rng)
    cache = C.cache(desc, blocks, rng, exps)
    rows, N = int(row_start[-1]) + padding, desc["heads"] * desc["head_dim"]
    q8, q_exp = C.queries(desc, max(rows, 1), rng, q_exps)
    q8, q_exp = q8[:rows], q_exp[:rows]
    held = np.array(held, np.int32)
    if mangle:
        mangle(cache, q8, q_exp, held, table)
    attn = G.iodf_attn_create(desc)
    wide = torch.full((rows, N + 8), 3, dtype=desc["out"]["dtype"], device="cuda")
    y = wide[:, 5:5 + N] if strided else wide[:, :N].contiguous()
    gt = C.on_gpu(torch, np.pad(table, ((0, 0), (0, 3))))[:, :table.shape[1]] if strided else C.on_gpu(torch, table)
    G.iodf_attn_forward(attn, C.on_gpu(torch, q8), C.on_gpu(torch, q_exp), C.on_gpu(torch, row_start), C.on_gpu(torch, held), gt,
                        C.on_gpu(torch, cache), y=y)
    want = A.forward(desc, q8, q_exp, row_start, held, table, cache, np.full((rows, N), 3, np.int64))
    np.testing.assert_array_equal(y.cpu().numpy(), want)
    if strided:
        assert (wide[:, :5] == 3).all() and (wide[:, 5 + N:] == 3).all()
    return attn


LENGTHS = [([1], [1]), ([127], [1]), ([128], [1]), ([129], [1]), ([1000], [1]), ([5], [5]), ([300], [129]), ([256], [256]),
           ([0, 7, 0, 130], [0, 3, 0, 1]), ([40, 300, 129, 2], [1, 1, 1, 1]), ([260, 1, 515], [100, 1, 17]), ([2500], [3])]


@pytest.mark.parametrize("held,add", LENGTHS)
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_forward_lengths(held, add, dim):
    torch, G = _modules()
    G.iodf_attn_check(_forward_both(C.description(torch, 4, 2, dim), held, add, dim + len(held), padding=2))


@pytest.mark.parametrize("held,add,heads,kv,dim,window", [([1500, 1300], [1500, 200], 2, 1, 32, 0), ([2300], [700], 4, 2, 128, 0), ([1100] * 5, [150] * 5, 8, 8, 64, 0),
                                                          ([3000], [260], 16, 2, 64, 1400), ([1025, 1024, 1152, 1153], [129, 128, 40, 300], 6, 2, 32, 0)])
def test_forward_of_many_blocks(held, add, heads, kv, dim, window):
    """Rows that see more than eight blocks, and more units than fit on the GPU at once."""
    torch, G = _modules()
    G.iodf_attn_check(_forward_both(C.description(torch, heads, kv, dim, window=window), held, add, len(held)))


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (8, 8), (8, 1), (10, 2), (17, 1), (40, 2), (64, 1), (129, 3)])
@pytest.mark.parametrize("held,add", [([200], [1]), ([300, 77], [1, 1]), ([140, 3], [40, 3])])
def test_forward_heads(heads, kv, held, add):
    torch, G = _modules()
    G.iodf_attn_check(_forward_both(C.description(torch, heads, kv, 32, y="int32"), held, add, heads))


@pytest.mark.parametrize("causal,window", [(True, 1), (True, 2), (True, 100), (True, 128), (True, 129), (True, 400), (False, 0), (False, 50), (True, 1 << 30)])
@pytest.mark.parametrize("held,add", [([700], [1]), ([300, 513], [300, 140]), ([4], [4]), ([260, 400], [2, 1])])
def test_forward_masks(causal, window, held, add):
    torch, G = _modules()
    G.iodf_attn_check(_forward_both(C.description(torch, 4, 2, 64, causal=causal, window=window), held, add, window % 1000 + len(held), padding=1))


@pytest.mark.parametrize("causal", [True, False])
def test_forward_rows_that_see_nothing(causal):
    """More rows than tokens: those before the first token see nothing if causal; without any token no row sees any."""
    torch, G = _modules()
    d = C.description(torch, 2, 1, 32, causal=causal)
    G.iodf_attn_check(_forward_both(d, [3, 0, 130], [10, 5, 200], 1))
    d["window"] = 1
    G.iodf_attn_check(_forward_both(d, [3, 0, 130], [10, 5, 200], 1))


@pytest.mark.parametrize("y", ["int8", "uint8", "int32"])
@pytest.mark.parametrize("held,add", [([333, 9], [1, 1]), ([333, 9], [150, 9])])
def test_forward_types_and_strides(y, held, add):
    torch, G = _modules()
    d = C.description(torch, 6, 2, 64, y=y)
    if y == "int8":
        d["out"]["clamp"] = (-20, 90)
    G.iodf_attn_check(_forward_both(d, held, add, 3, padding=3, strided=True))


@pytest.mark.parametrize("held,add", [([700, 260], [1, 1]), ([700, 260], [130, 260])])
@pytest.mark.parametrize("exps,q_exps,octaves", [((0, 13), (0, 13), 2.0), ((0, 1), (0, 1), 2000.0), ((12, 13), (12, 13), 2.0), ((3, 256), (0, 256), 2.0),
                                                 ((3, 7), (3, 8), 1e-4), ((3, 7), (3, 8), 300.0)])
def test_forward_scales(held, add, exps, q_exps, octaves):
    """Exponents at both ends and beyond, scores from flat to a single peak, a multiplier that saturates."""
    torch, G = _modules()
    G.iodf_attn_check(_forward_both(C.description(torch, 4, 2, 128, y="int32", octaves=octaves), held, add, 11, exps=exps, q_exps=q_exps))


@pytest.mark.parametrize("held,add", [([300, 1000], [1, 1]), ([300, 500], [129, 140])])
@pytest.mark.parametrize("what", ["zeros", "alike", "extremes", "lone"])
def test_forward_values(held, add, what):
    torch, G = _modules()

    def mangle(cache, q8, q_exp, held, table):
        if what == "zeros":                       # all scores alike, all values 0
            cache["v"][:] = 0
            q8[:] = 0
        elif what == "alike":                     # all scores at the range's end
            cache["k"][:] = q8[:] = 127
        elif what == "extremes":                  # sums as large as they get
            cache["k"][:] = np.where(np.arange(128)[:, None] % 2, 127, -127)
            cache["v"][:] = 127
            q8[:] = np.where(np.arange(q8.shape[0])[:, None, None] % 2, 127, -127)
        else:                                     # one key far above the rest
            q8[:] = 100
            cache["k"][:] = -50
            cache["k"][table[0, 0], :, 17] = 120
    G.iodf_attn_check(_forward_both(C.description(torch, 4, 2, 128, y="int32"), held, add, 2, mangle=mangle))


@pytest.mark.parametrize("add", [[1, 1, 1], [9, 130, 5]])
def test_forward_counts_what_it_cannot_read(add):
    """Blocks outside the cache are seen by nobody, contexts beyond the table are cut to it; both are counted."""
    torch, G = _modules()

    def mangle(cache, q8, q_exp, held, table):
        table[0, 1], table[1, 0], table[1, 2] = -1, len(cache["k"]), 2 ** 31 - 1
        held[2] = table.shape[1] * 128 + 5
        table[2] = table[2] % len(cache["k"])
    attn = _forward_both(C.description(torch, 2, 1, 64), [300, 400, 500], add, 4, mangle=mangle)
    with pytest.raises(G.IodfError) as e:
        G.iodf_attn_check(attn)
    assert e.value.status == -9
    G.iodf_attn_check(attn)
