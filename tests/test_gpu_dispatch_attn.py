"""Which kernel, and how many CTAs of it, an attention of a given size is. Outputs are the same bits either way, so the comparisons with the definition
tell nothing of it; these are the sizes with which they reach each kernel."""
import numpy as np
import pytest

from tests import attn_cases as C
from tests import test_gpu_attn as T
from test_gpu_dispatch import _launches

pytestmark = pytest.mark.gpu


def _calls(calls, tmp_path):
    """Kernel and CTAs of each call (description, held, add, rows behind the last request)."""
    import torch
    import paper_2206_08869_b200 as G
    rng, ready = np.random.default_rng(0), []
    for d, held, add, padding in calls:
        start, table, blocks = C.requests(held, add, rng)
        rows = int(start[-1]) + padding
        attn = G.iodf_attn_create(d)
        g = lambda x: C.on_gpu(torch, x)                                          # noqa: E731
        q8, e = C.queries(d, rows, rng)
        y = torch.zeros((rows, d["heads"] * d["head_dim"]), dtype=d["out"]["dtype"], device="cuda")
        ready.append((attn, (g(q8), g(e), g(start), g(np.array(held, np.int32)), g(table), G.iodf_attn_cache(attn, blocks)), y))

    def run():
        for attn, args, y in ready:
            G.iodf_attn_forward(attn, *args, y=y)
    got = [(name, ctas) for name, ctas, _ in _launches(run, tmp_path)]
    for attn, _, _ in ready:
        G.iodf_attn_check(attn)
    assert len(got) == len(calls)
    return got


def test_padding_makes_it_the_kernel_for_many_rows(tmp_path):
    """The sizes of test_gpu_attn_shapes.py, whose fixture adds the padding."""
    import torch
    calls = [(C.description(torch, 4, 2, dim), h, a, 4000) for h, a in T.LENGTHS + [([500] * 70, [17] * 70), ([129, 0, 900], [129, 0, 128])] for dim in (32, 64, 128)]
    calls += [(C.description(torch, heads, kv, 32), h, a, 16000 // heads) for heads, kv in [(1, 1), (3, 1), (8, 8), (8, 1), (10, 2), (17, 1), (40, 2), (129, 3), (128, 1)]
              for h, a in [([200], [1]), ([300, 77], [1, 1]), ([140, 3], [40, 3])]]
    calls += [(C.description(torch, 2, 1, dim, window=w), h, a, 8000) for h, a, dim, w in [([131072], [5], 32, 0), ([131071, 1000], [2, 700], 64, 0), ([40000], [130], 128, 0),
                                                                                          ([131072], [3], 128, 90000)]]
    assert {name for name, _ in _calls(calls, tmp_path)} == {"tile_kernel"}


def test_few_rows_have_a_kernel_of_their_own(tmp_path):
    import torch
    calls = [(C.description(torch, 4, 2, dim), h, a, 2) for h, a in T.LENGTHS if sum(a) <= 5 for dim in (32, 64, 128)]
    calls += [(C.description(torch, heads, 1, dim, window=w), [t, 200], [1, 1], 0) for t, heads, dim, w in
              [(131072, 2, 32, 0), (131071, 8, 32, 0), (50000, 16, 128, 0), (60000, 16, 64, 45000), (39000, 12, 32, 38000)]]
    assert {name for name, _ in _calls(calls, tmp_path)} == {"split_kernel"}


def test_teams_that_do_not_divide_a_head(tmp_path):
    """The units of test_gpu_attn_teams.py: a cluster each, of a number of CTAs that does not divide 128."""
    import torch
    units = [8, 8, 12, 11]
    calls = [(C.description(torch, heads, kv, 128), [blocks * 128 - 3], [1], 0) for heads, kv, blocks in [(32, 8, 261), (128, 8, 300), (12, 12, 244), (33, 11, 262)]]
    for n, (name, ctas) in zip(units, _calls(calls, tmp_path)):
        assert name == "split_kernel" and ctas % n == 0 and 128 % (ctas // n) and ctas // n > 8


def test_appends_of_four_rows_to_a_warp(tmp_path):
    """The sizes of test_gpu_attn_append.py: CTAs of 32 rows from its least number of them on, of 8 below."""
    import torch
    import paper_2206_08869_b200 as G
    from tests import test_gpu_attn_append as P
    d = P._description(torch, 128, "int8")
    attn, least, calls = G.iodf_attn_create(d), P._least(torch), []
    cache = G.iodf_attn_cache(attn, 4)
    for rows in (least - 1, least, least + 8):
        x = torch.zeros((rows, 3 * 32 * 128), dtype=torch.int8, device="cuda")
        none, at = torch.full((rows,), -1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
        calls.append((x[:, :4096], x[:, 4096:8192], x[:, 8192:], none, at, cache))
    got = _launches(lambda: [G.iodf_attn_append(attn, *c) for c in calls], tmp_path)
    G.iodf_attn_check(attn)
    got = [ctas for name, ctas, _ in got if name == "append_kernel"]
    assert got == [-(-(least - 1) // 8) * 32, -(-least // 32) * 32, -(-(least + 8) // 32) * 32]
