"""Attention of few rows whose units go to teams of nine or ten CTAs, which do not divide a head's dimensions evenly, with more blocks for each CTA
than have their scores in tensor memory."""
import numpy as np
import pytest

from oracle import attention as A
from tests import attn_cases as C

pytestmark = pytest.mark.gpu


# 8 units: the largest clusters of which eight run at once; 12: smaller ones. 26 blocks' scores stay in tensor memory.
@pytest.mark.parametrize("heads,kv,blocks", [(32, 8, 261), (8, 8, 270), (64, 8, 281), (128, 8, 300), (48, 12, 237), (12, 12, 244), (33, 11, 262)])
def test_teams_that_do_not_divide_a_head(heads, kv, blocks):
    import torch
    import paper_2206_08869_b200 as G
    rng = np.random.default_rng(blocks)
    d = C.description(torch, heads, kv, 128, y="int32")
    held = np.array([blocks * 128 - 3], np.int32)
    start, table, total = C.requests(held, [1], rng)
    cache = C.cache(d, total, rng)
    q8, e = C.queries(d, 1, rng)
    want = A.forward(d, q8, e, start, held, table, cache, np.zeros((1, heads * 128), np.int64))
    attn, g = G.iodf_attn_create(d), lambda x: C.on_gpu(torch, x)
    args, gc = [g(x) for x in (q8, e, start, held, table)], g(cache)
    out = [G.iodf_attn_forward(attn, *args, gc) for _ in range(50)]
    G.iodf_attn_check(attn)
    for y in out:
        np.testing.assert_array_equal(y.cpu().numpy(), want)
