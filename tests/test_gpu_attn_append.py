"""Appends of as many tokens as give each warp four rows, and of just too few, against the plain 64-bit definition, bit for bit."""
import numpy as np
import pytest

from oracle import attention as A
from tests import attn_cases as C
from tests import test_gpu_attn as T

pytestmark = pytest.mark.gpu


def _description(torch, dim, x, rot=32, layout="half"):
    """32 parts of 128 elements of a row's keys."""
    kv = 32 * 128 // dim
    return C.description(torch, kv, kv, dim, x, rot, layout)


def _least(torch):
    """Rows of such a call from which on a warp takes four: two CTAs of 32 rows and one part for each SM."""
    return torch.cuda.get_device_properties(0).multi_processor_count * 2 * 32 // 32


def _filled(held, add, rows):
    """The requests again and again, and a last one with what is left."""
    h, a = [], []
    while sum(a) + sum(add) < rows:
        h, a = h + held, a + add
    return h + [3], a + [rows - sum(a)]


@pytest.mark.parametrize("dim,x", [(32, "int8"), (64, "int32"), (128, "int8"), (128, "int32")])
@pytest.mark.parametrize("held,add", [([0, 101], [101, 3]), ([0, 133], [5, 7]), ([0, 2], [2, 1]), ([0, 259], [131, 2]), ([256, 161], [33, 30]),
                                      ([0, 3, 128, 7], [3, 4, 7, 1])])
def test_requests_that_begin_where_others_end(held, add, dim, x):
    """A request's tokens start a block, and the next one's lie as far from the start of theirs, which is in the cache with its exponents."""
    torch, _ = T._modules()
    rows = _least(torch) + 8
    held, add = _filled(held, add, rows)
    slot, position, blocks = T._slots(held, add, np.random.default_rng(rows + dim), padding=3)
    T._append_both(_description(torch, dim, x), len(slot), slot, position, blocks, dim)


@pytest.mark.parametrize("held,more", [(0, -1), (1, -1), (0, 0), (1, 0), (2, 1), (3, 0), (126, 1), (131, 0)])
def test_one_request_around_the_least_number_of_rows(held, more):
    torch, _ = T._modules()
    rows = _least(torch) + more
    slot, position, blocks = T._slots([held], [rows], np.random.default_rng(held))
    T._append_both(_description(torch, 128, "int32"), rows, slot, position, blocks, held)


@pytest.mark.parametrize("dim,layout,seed,views,x", [(32, "interleaved", 0, "columns", "int8"), (64, "half", 1, "odd", "int32"), (128, "interleaved", 2, "apart", "int8"),
                                                     (32, "half", 3, "odd", "int8"), (64, "interleaved", 4, "columns", "int32"), (128, "half", 5, "columns", "int32")])
def test_requests_of_any_lengths(dim, layout, seed, views, x):
    torch, _ = T._modules()
    rng = np.random.default_rng(seed)
    rows = _least(torch) + 40
    add = [int(v) for v in rng.integers(0, 9, 20)] + [int(v) for v in rng.integers(0, 60, 6)]
    held = [int(v) for v in rng.integers(0, 300, len(add))]
    held, add = _filled(held, add, max(rows, sum(add) + 1))
    slot, position, blocks = T._slots(held, add, rng, padding=5)
    T._append_both(_description(torch, dim, x, 32, layout), len(slot), slot, position, blocks, seed, views)


@pytest.mark.parametrize("dim,rot,layout", [(32, 32, "half"), (64, 64, "interleaved"), (64, 16, "half"), (128, 128, "half"), (128, 48, "interleaved")])
@pytest.mark.parametrize("x", ["int8", "int32"])
def test_factors_that_are_no_rotation(x, dim, rot, layout):
    """Cosines and sines of 1 at once double the largest element: 2^16, whose exponent is 11 with all the headroom there is."""
    torch, G = T._modules()
    d = C.description(torch, 2, 2, dim, x, rot, layout, headroom=(8, 8))
    d["rotary"]["table"] = np.stack([np.full((4, rot // 2, 2), 16384), np.full((4, rot // 2, 2), -16384)]).reshape(8, rot // 2, 2).astype(np.int16)
    low, high = (-128, 127) if x == "int8" else (-2 ** 31, 2 ** 31 - 1)
    rng = np.random.default_rng(dim)
    rows = 96
    slot, position, blocks = T._slots([0] * rows, [1] * rows, rng)
    position = rng.integers(0, 8, rows)
    values = np.where(rng.integers(0, 2, (rows, 1, 1)) == 0, np.int64(low), rng.choice([low, high, 0, 1], (rows, 6, dim))).reshape(rows, 6 * dim)
    values = values.astype(np.int8 if x == "int8" else np.int32)
    cache = C.cache(d, blocks, rng)
    gx, gc = C.on_gpu(torch, values), C.on_gpu(torch, cache)
    attn = G.iodf_attn_create(d)
    cut = [0, 2 * dim, 4 * dim, 6 * dim]
    q8, e = G.iodf_attn_append(attn, *(gx[:, a:b] for a, b in zip(cut, cut[1:])), C.on_gpu(torch, slot.astype(np.int32)),
                               C.on_gpu(torch, position.astype(np.int32)), gc)
    G.iodf_attn_check(attn)
    w8, we = A.append(d, *(values[:, a:b] for a, b in zip(cut, cut[1:])), slot, position, cache)
    assert cache["k_exp"][slot // 128].max() == (11 if x == "int32" else 3) and we.max() == (10 if x == "int32" else 2)
    np.testing.assert_array_equal(q8.cpu().numpy(), w8)
    np.testing.assert_array_equal(e.cpu().numpy(), we)
    for name in cache:
        np.testing.assert_array_equal(gc[name].cpu().numpy(), cache[name], err_msg=name)
