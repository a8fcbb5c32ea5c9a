"""Attention through both kernels and the shapes of the one for few rows. Rows behind the last sequence count for the choice of a kernel, which the
host makes from the call's sizes: with many of them the kernel for many rows gets what the other one has in test_gpu_attn.py."""
import numpy as np
import pytest

from tests import attn_cases as C
from tests import test_gpu_attn as T

pytestmark = pytest.mark.gpu


@pytest.fixture
def many(monkeypatch):
    plain = T._forward_both

    def padded(desc, held, add, seed, **kw):
        return plain(desc, held, add, seed, **{**kw, "padding": 16000 // desc["heads"]})
    monkeypatch.setattr(T, "_forward_both", padded)


@pytest.mark.parametrize("held,add", T.LENGTHS + [([500] * 70, [17] * 70), ([129, 0, 900], [129, 0, 128])])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_lengths(many, held, add, dim):
    T.test_forward_lengths(held, add, dim)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (8, 8), (8, 1), (10, 2), (17, 1), (40, 2), (129, 3), (128, 1)])
@pytest.mark.parametrize("held,add", [([200], [1]), ([300, 77], [1, 1]), ([140, 3], [40, 3])])
def test_heads(many, heads, kv, held, add):
    T.test_forward_heads(heads, kv, held, add)


@pytest.mark.parametrize("causal,window", [(True, 1), (True, 2), (True, 100), (True, 128), (True, 129), (True, 400), (False, 0), (False, 50), (True, 1 << 30)])
@pytest.mark.parametrize("held,add", [([700], [1]), ([300, 513], [300, 140]), ([4], [4]), ([260, 400], [2, 1])])
def test_masks(many, causal, window, held, add):
    T.test_forward_masks(causal, window, held, add)


@pytest.mark.parametrize("causal", [True, False])
def test_rows_that_see_nothing(many, causal):
    T.test_forward_rows_that_see_nothing(causal)


@pytest.mark.parametrize("y", ["int8", "uint8", "int32"])
@pytest.mark.parametrize("held,add", [([333, 9], [1, 1]), ([333, 9], [150, 9])])
def test_types_and_strides(many, y, held, add):
    T.test_forward_types_and_strides(y, held, add)


@pytest.mark.parametrize("held,add", [([700, 260], [1, 1]), ([700, 260], [130, 260])])
@pytest.mark.parametrize("exps,q_exps,octaves", [((0, 13), (0, 13), 2.0), ((0, 1), (0, 1), 2000.0), ((12, 13), (12, 13), 2.0), ((3, 256), (0, 256), 2.0)])
def test_scales(many, held, add, exps, q_exps, octaves):
    T.test_forward_scales(held, add, exps, q_exps, octaves)


@pytest.mark.parametrize("held,add", [([300, 1000], [1, 1]), ([300, 500], [129, 140])])
@pytest.mark.parametrize("what", ["zeros", "alike", "extremes", "lone"])
def test_values(many, held, add, what):
    T.test_forward_values(held, add, what)


@pytest.mark.parametrize("add", [[1, 1, 1], [9, 130, 5]])
def test_counts_what_it_cannot_read(many, add):
    T.test_forward_counts_what_it_cannot_read(add)


@pytest.mark.parametrize("clamp,y", [((-100, 127), "int8"), ((5, 6), "uint8"), ((-128, 127), "int8")])
@pytest.mark.parametrize("held,add", [([400, 20], [300, 20]), ([400, 20], [3, 1])])
def test_clips(held, add, clamp, y):
    torch, G = T._modules()
    for padding in (0, 4000):
        d = C.description(torch, 4, 2, 64, y=y)
        d["out"]["clamp"] = clamp
        G.iodf_attn_check(T._forward_both(d, held, add, 3, padding=padding))


@pytest.mark.parametrize("blocks", [9, 10, 11, 13, 15, 16, 17, 40])
def test_a_cluster_for_one_request(blocks):
    torch, G = T._modules()
    G.iodf_attn_check(T._forward_both(C.description(torch, 4, 1, 128), [blocks * 128 - 5], [1], blocks))


@pytest.mark.parametrize("heads,kv", [(7, 7), (8, 8), (22, 11), (12, 12), (15, 15), (16, 16), (120, 60)])
def test_heads_that_share_the_clusters(heads, kv):
    torch, G = T._modules()
    G.iodf_attn_check(T._forward_both(C.description(torch, heads, kv, 64), [2100], [1], heads))


@pytest.mark.parametrize("heads,kv,add,dim", [(4, 4, 1, 64), (8, 2, 1, 128), (8, 2, 2, 32), (8, 1, 1, 64), (32, 2, 1, 32), (5, 1, 3, 128), (24, 2, 2, 64)])
@pytest.mark.parametrize("n", [3, 30, 90])
def test_requests_of_many_lengths(heads, kv, add, dim, n):
    """Teams of every size share the clusters: contexts of up to 21 blocks, among them empty ones, and one of many."""
    torch, G = T._modules()
    rng = np.random.default_rng(n)
    held = np.minimum(rng.geometric(0.0015, n), 2600)
    held[rng.integers(n, size=n // 10)] = 0
    held[n // 2] = 2650 if n > 3 else 9000
    G.iodf_attn_check(T._forward_both(C.description(torch, heads, kv, dim), held.tolist(), np.minimum(held, add).tolist(), n + heads))


@pytest.mark.parametrize("tokens,heads,dim,window", [(131072, 2, 32, 0), (131071, 8, 32, 0), (50000, 16, 128, 0), (60000, 16, 64, 45000), (39000, 12, 32, 38000)])
def test_contexts_whose_scores_are_computed_again(tokens, heads, dim, window):
    torch, G = T._modules()
    G.iodf_attn_check(T._forward_both(C.description(torch, heads, 1, dim, window=window), [tokens, 200], [1, 1], 1))


def test_more_requests_than_the_kernel_for_few_rows_takes():
    torch, G = T._modules()
    rng = np.random.default_rng(0)
    held = rng.integers(0, 200, 9000)
    G.iodf_attn_check(T._forward_both(C.description(torch, 1, 1, 32), held.tolist(), np.minimum(held, rng.integers(0, 2, 9000)).tolist(), 1))


@pytest.mark.parametrize("held,add,dim,window", [([131072], [5], 32, 0), ([131071, 1000], [2, 700], 64, 0), ([40000], [130], 128, 0), ([131072], [3], 128, 90000)])
def test_long_contexts(many, held, add, dim, window):
    torch, G = T._modules()
    G.iodf_attn_check(T._forward_both(C.description(torch, 2, 1, dim, window=window), held, add, 5))


@pytest.mark.parametrize("padding", [0, 4000])
def test_rows_before_the_first_request(padding):
    """Rows that no request has, before, between (a request of none) and behind them, stay as they are."""
    torch, G = T._modules()
    d = C.description(torch, 4, 2, 64)
    rng = np.random.default_rng(9)
    held, add = np.array([200, 0, 77], np.int32), [5, 0, 70]
    start, table, blocks = C.requests(held, add, rng)
    start += 3
    rows = int(start[-1]) + 2 + padding
    cache = C.cache(d, blocks, rng)
    q8, e = C.queries(d, rows, rng)
    y = torch.full((rows, 256), 3, dtype=torch.int8, device="cuda")
    attn, g = G.iodf_attn_create(d), lambda x: C.on_gpu(torch, x)
    G.iodf_attn_forward(attn, g(q8), g(e), g(start), g(held), g(table), g(cache), y=y)
    from oracle import attention as A
    want = A.forward(d, q8, e, start, held, table, cache, np.full((rows, 256), 3, np.int64))
    np.testing.assert_array_equal(y.cpu().numpy(), want)
    assert (want[:3] == 3).all() and (want[start[-1]:] == 3).all()
    G.iodf_attn_check(attn)
