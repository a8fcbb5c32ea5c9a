"""Requests, caches and handles that the tests of integer attention share."""
import numpy as np

from oracle import attention as A


def rotary_table(positions, rot, stretch=1):
    freq = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    angle = np.arange(positions)[:, None] / stretch * freq
    return np.round(np.stack([np.cos(angle), np.sin(angle)], -1) * 16384).astype(np.int16)


def description(torch, heads=4, kv=2, dim=64, x="int32", rot=0, layout="half", positions=4096, headroom=(2, 4), octaves=2.0, causal=True,
                window=0, y="int8", seed=0):
    """A handle's description, with scores of random inputs spread over about `octaves` octaves."""
    rng = np.random.default_rng(seed)
    gain = octaves * 2.0 ** 36 / (36 * 28 * dim ** 0.5 * 2 ** 9.5)
    s = max(0, int(np.ceil(np.log2(2.0 ** 30 / gain))))
    d = {"heads": heads, "kv_heads": kv, "head_dim": dim, "x_dtype": getattr(torch, x), "headroom": headroom,
         "score": (min(2 ** 31 - 1, max(2 ** 30, int(gain * 2.0 ** s))), s), "causal": causal, "window": window,
         "out": {"m0": rng.integers(1 << 30, 1 << 31, heads * dim).astype(np.int32), "s": np.full(heads * dim, {"int32": 2}.get(y, 11), np.int32),
                 "clamp": {"int8": (-128, 127), "uint8": (0, 255), "int32": None}[y], "dtype": getattr(torch, y)}}
    if rot:
        d["rotary"] = {"dim": rot, "layout": layout, "table": rotary_table(positions, rot)}
    return d


def cache(desc, blocks, rng, exps=(3, 7)):
    kv, dim = desc["kv_heads"], desc["head_dim"]
    ints = lambda shape: np.clip(np.round(rng.normal(0, 28, shape)), -127, 127).astype(np.int8)     # noqa: E731
    return {"k": ints((blocks, kv, 128, dim)), "v": ints((blocks, kv, dim, 128)),
            "k_exp": rng.integers(*exps, (blocks, kv)).astype(np.uint8), "v_exp": rng.integers(*exps, (blocks, kv)).astype(np.uint8)}


def requests(held, rows_of, rng, extra=2):
    """(row_start, table, blocks) of requests that hold `held` tokens, rows_of new ones among them: any blocks in any order."""
    counts = [A.blocks_of(h) for h in held]
    blocks = sum(counts) + extra
    order, width = rng.permutation(blocks), max(1, max(counts, default=1))
    table = np.full((len(held), width), -7, np.int32)
    at = 0
    for q, n in enumerate(counts):
        table[q, :n] = order[at:at + n]
        at += n
    return np.concatenate([[0], np.cumsum(rows_of)]).astype(np.int32), table, blocks


def queries(desc, rows, rng, exps=(3, 8)):
    q8 = np.clip(np.round(rng.normal(0, 36, (rows, desc["heads"], desc["head_dim"]))), -127, 127).astype(np.int8)
    return q8, rng.integers(*exps, (rows, desc["heads"])).astype(np.uint8)


def on_gpu(torch, x):
    return {k: on_gpu(torch, v) for k, v in x.items()} if isinstance(x, dict) else torch.from_numpy(np.ascontiguousarray(x)).cuda()
