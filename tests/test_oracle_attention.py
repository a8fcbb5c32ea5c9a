"""The plain definition of integer attention against what it stands for, and the kernels' constants against the definition. CPU only."""
import os
import re

import numpy as np
import pytest
import torch

from oracle import attention as A
from tests import attn_cases as C

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2206_08869_b200", "csrc")


def test_weights_are_powers_of_two():
    n = -np.arange(0, 1 << 18, 7, dtype=np.int64)
    p, true = A.weight(n), 2.0 ** (15 + n / 8192)
    assert p[0] == 32768 and A.weight(np.array([-8192, -(1 << 17), -(1 << 20)])).tolist() == [16384, 0, 0]
    # a segment's line rises by 1024 a step where 2^(n / 2^13) rises by 709.8 times itself: 64 steps from the middle of the third segment, at
    # 1.027, that is 64 (1024 / 1.027 - 709.8) / 2^23 = 0.0022 of the value, less in the later ones; the first begins at 1 itself and is off
    # by 127 steps of it at its end, (1.0155 - 1.0108) / 1.0108 = 0.00465; and half a rounding
    assert (np.abs(p - true) <= 0.5 + true * 0.0047).all()
    assert (np.abs(p - true) <= 0.5 + true * 0.0023)[(n & 8191) >= 256].all()


def test_the_kernels_table_is_the_definitions():
    with open(os.path.join(CSRC, "attn_device.cuh")) as f:
        text = f.read()
    body = re.search(r"kSegments\[kWeightSegments\] = \{(.*?)\}", text, re.S).group(1)
    assert [int(v) for v in body.replace("\n", " ").split(",")] == (A.SEGMENTS - (1 << 23)).tolist()


def test_the_kernels_weights_are_the_definitions():
    """The kernels add 2^10 n to the bits of a float and round it by adding 2^23 + 128: for every n the definition's weight."""
    n = -np.arange(0, (1 << 18) + 1, dtype=np.int64)
    c = (n >> 7) & 63
    bits = (((127 + 15) << 23) + (A.SEGMENTS[c] - (1 << 23)) - c * (128 << 10) + (n << 10)).astype(np.int32)
    x = (bits.view(np.float32) + np.float32(8388608 + 128)).view(np.int32).astype(np.int64) - 0x4B000080
    assert np.array_equal(x, A.weight(n))
    hi, lo = (x + 128) >> 8, ((x + 128) & 255) - 128                 # as the MMAs take them
    assert np.array_equal(256 * hi + lo, x) and hi.max() == 128 and hi.min() == 0 and lo.min() >= -128 and lo.max() <= 127


def test_exponents_are_the_smallest():
    for headroom in (0, 3, 8):
        for amax in list(range(0, 3000)) + [32767, 32768, 65535, 65536]:
            e = A.exponent(amax, headroom)
            assert amax * (8 + headroom) <= 1016 << e and (e == 0 or amax * (8 + headroom) > 1016 << (e - 1)) and e <= 11


def _steps(desc, x, cuts, rng_seed=0):
    """Outputs of a request whose tokens come in the given numbers."""
    heads, kv, dim = desc["heads"], desc["kv_heads"], desc["head_dim"]
    total = sum(cuts)
    rng = np.random.default_rng(rng_seed)
    blocks = A.blocks_of(total) + 1
    table, ring = np.zeros((1, blocks), np.int64), rng.permutation(blocks)
    cache = {"k": rng.integers(-127, 128, (blocks, kv, 128, dim)).astype(np.int8), "v": rng.integers(-127, 128, (blocks, kv, dim, 128)).astype(np.int8),
             "k_exp": np.full((blocks, kv), 200, np.uint8), "v_exp": np.full((blocks, kv), 200, np.uint8)}
    held, state, out, at = np.zeros(1, np.int64), np.array([0, blocks]), [], 0
    for m in cuts:
        held, start, slot, position, state, refused = A.plan(held, [m], table, ring, state, m)
        assert not refused
        part = x[at:at + m]
        q, k, v = (part[:, a:b] for a, b in ((0, heads * dim), (heads * dim, (heads + kv) * dim), ((heads + kv) * dim, (heads + 2 * kv) * dim)))
        q8, e = A.append(desc, q, k, v, slot, position, cache)
        out.append(A.forward(desc, q8, e, start, held, table, cache, np.zeros((m, heads * dim), np.int64)))
        at += m
    return np.concatenate(out)


@pytest.mark.parametrize("window", [0, 70])
def test_any_cut_of_the_tokens_gives_the_same(window):
    d = C.description(torch, 2, 1, 32, "int32", 32, window=window)
    x = np.random.default_rng(1).normal(0, 2500, (290, 4 * 32)).astype(np.int64)
    whole = _steps(d, x, [290])
    for cuts in ([1] * 290, [127, 1, 1, 128, 33], [200, 90]):
        assert np.array_equal(_steps(d, x, cuts), whole)


def test_it_is_attention():
    """Against softmax attention of the same keys, values and scores in floating point: weights are off by 0.5 % at most, one in a hundred of the
    largest values' unit at most after the sum's rounding."""
    d = C.description(torch, 2, 2, 64, y="int32", causal=False, seed=3)
    d["out"].update(m0=np.full(128, 1 << 30, np.int32), s=np.zeros(128, np.int32))                 # y = o / 2
    rng = np.random.default_rng(5)
    start, table, blocks = C.requests([300], [7], rng)
    cache = C.cache(d, blocks, rng)
    q8, e = C.queries(d, 7, rng)
    y = A.forward(d, q8, e, start, [300], table, cache, np.zeros((7, 128), np.int64))
    ids = table[0][:3]
    for h in range(2):
        k = (cache["k"][ids, h].astype(float) * 2.0 ** cache["k_exp"][ids, h][:, None, None]).reshape(-1, 64)[:300]
        v = (cache["v"][ids, h].transpose(0, 2, 1).astype(float) * 2.0 ** cache["v_exp"][ids, h][:, None, None]).reshape(-1, 64)[:300]
        s = (q8[:, h] * 2.0 ** e[:, h][:, None]) @ k.T * (d["score"][0] / 2.0 ** d["score"][1]) / 2.0 ** 36
        p = 2.0 ** (s - s.max(1, keepdims=True))
        want = (p / p.sum(1, keepdims=True)) @ v * 128
        assert (np.abs(y[:, h * 64:(h + 1) * 64] - want) <= 0.01 * np.abs(v).max() * 128).all()


def test_a_wait_is_never_two_phases_late():
    """Who reads S of which block in the kernel for many rows, as it assigns them: a barrier's wait is for one of two parities, so between two
    uses that one reader waits for there must be no use of the same barrier by another one that it does not meet in between."""
    with open(os.path.join(CSRC, "attn_tile.cu")) as f:
        text = f.read()
    lead = int(re.search(r"constexpr int kLead = (\d+);", text).group(1))
    assert "return j < kLead ? 4 + (j & 1) : j & 3;" in text
    assert "int slot = leading ? 4 + half : w + 2 * half, j1 = leading ? half : kLead + slot;" in text
    place = lambda j: 4 + (j & 1) if j < lead else j & 3              # noqa: E731
    for n in (1, 2, lead, lead + 1, lead + 7, 40):
        seen = {}
        for w in (0, 1):
            for half in (0, 1):
                j, leading, slot = (half, True, 4 + half) if w else (lead + 2 * half, False, 2 * half)
                while True:
                    if leading and j >= min(n, lead):
                        leading, slot = False, w + 2 * half
                        j = lead + slot
                    if j >= n:
                        break
                    assert place(j) == slot
                    seen.setdefault(j, []).append((w, half))
                    j += 2 if leading else 4
        assert sorted(seen) == list(range(n)) and all(len(v) == 1 for v in seen.values())
        readers = {}
        for j, v in seen.items():
            readers.setdefault(place(j), set()).add(v[0])
        assert all(len(v) == 1 for v in readers.values())              # one reader for each barrier until the groups meet
