"""How far integer attention is from softmax attention of the same integers, in blocks whose values have unlike exponents: on the plain
definition, CPU only."""
import numpy as np
import pytest
import torch

from oracle import attention as A
from tests import attn_cases as C

DIM, BLOCKS = 64, 8


def _both(exps, seed, lonely=False):
    """Outputs of one row in 2^-7, the same by floating point, and the bound on their difference. lonely: the last block is seen and has no weight."""
    d = C.description(torch, 1, 1, DIM, y="int32", causal=False)
    d["out"].update(m0=np.full(DIM, 1 << 30, np.int32), s=np.zeros(DIM, np.int32))                 # y = o / 2
    rng = np.random.default_rng(seed)
    start, table, blocks = C.requests([128 * BLOCKS], [1], rng)
    cache = C.cache(d, blocks, rng)
    q8, e = C.queries(d, 1, rng)
    ids, (m0, s) = table[0], d["score"]
    cache["v_exp"][ids, 0] = exps
    if lonely:
        cache["k"][ids[-1], 0], cache["k_exp"][ids[-1], 0] = -q8[0, 0], 12
    y = A.forward(d, q8, e, start, [128 * BLOCKS], table, cache, np.zeros((1, DIM), np.int64))[0]
    W = (m0 << (int(e[0, 0]) + cache["k_exp"][ids, 0].astype(np.int64))) >> s
    t = ((cache["k"][ids, 0].astype(np.int64) @ q8[0, 0].astype(np.int64) * W[:, None]) >> 23).reshape(-1)
    w = 2.0 ** ((t - t.max()) / 8192)
    u = (cache["v"][ids, 0].transpose(0, 2, 1).astype(float) * 2.0 ** np.asarray(exps)[:, None, None]).reshape(-1, DIM)
    want = w @ u / w.sum()
    # A weight is off by 0.47 % of itself (the chord), and by half a step of 2^(V - v_exp - 15) of the largest one. The quotient of two sums
    # with weights w + r is off by sum r (u - out) / sum (w + r). An output's roundings: o half a unit of 2^-8, the quotient's floors 2^(V - 15)
    # and |o| 2^-31 <= 2^-4 of it, y half a unit of 2^-7.
    r = 0.0047 * w + np.repeat(2.0 ** (max(exps) - np.asarray(exps) - 16.0), 128)
    least = w.sum() - r.sum()
    bound = np.abs(u - want).T @ r / least * 128 + 0.5 * (0.5 + 2.0 ** (max(exps) - 15) + 2.0 ** -4) + 0.5 if least > 0 else np.inf
    return y, want * 128, bound


@pytest.mark.parametrize("exps", [[3] * 8, [0] * 8, [12] * 8, [3, 4, 5, 6, 3, 4, 5, 6], [3] * 7 + [6], [3] * 7 + [9], [9] + [3] * 7, [0] * 7 + [8], [4] * 7 + [0]])
@pytest.mark.parametrize("lonely", [False, True])
def test_the_error_is_within_the_exponents_bound(exps, lonely):
    for seed in range(4):
        y, want, bound = _both(exps, seed, lonely)
        assert (np.abs(y - want) <= bound).all()
