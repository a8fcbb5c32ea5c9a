"""Sizes of caches and rings at their limits: told from wrong arguments, on the host."""
import ctypes as C

import pytest

from tests import attn_cases

pytestmark = pytest.mark.gpu
EINVAL, EUNSUPPORTED = -1, -6


@pytest.mark.parametrize("kv", [1, 2, 3, 8])
def test_blocks_of_a_cache(kv):
    import torch
    import paper_2206_08869_b200 as G
    from paper_2206_08869_b200 import binding as B
    attn, L = G.iodf_attn_create(attn_cases.description(torch, kv, kv, 32)), G.load_library()
    most = ((1 << 24) - 1) // kv
    at = torch.zeros(64, dtype=torch.uint8, device="cuda").data_ptr()
    stream = torch.cuda.current_stream().cuda_stream

    def calls(**kw):                                        # of no rows: nothing is launched
        c = B.AttnCacheDesc(**{**dict(k=at, v=at + 16, k_exp=at + 32, v_exp=at + 48, blocks=1), **kw})
        return (L.iodf_attn_append(attn.handle, 0, None, 1, None, 1, None, 1, None, None, C.byref(c), None, None, stream),
                L.iodf_attn_forward(attn.handle, 0, None, None, None, None, 0, None, 1, 1, C.byref(c), None, 1, stream))
    assert calls() == calls(blocks=most) == (0, 0)
    for blocks in (most + 1, 1 << 24, (1 << 32) - 1):
        assert calls(blocks=blocks) == (EUNSUPPORTED, EUNSUPPORTED)
    for bad in (dict(blocks=0), dict(k=None), dict(v_exp=None), dict(k=at + 8), dict(v=at + 8), dict(k=at + 8, blocks=most + 1)):
        assert calls(**bad) == (EINVAL, EINVAL)


def test_places_of_a_ring():
    import torch
    import paper_2206_08869_b200 as G
    attn = G.iodf_attn_create(attn_cases.description(torch, 1, 1, 32))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")            # noqa: E731
    ring = torch.full((1 << 24,), 5, dtype=torch.int32, device="cuda")
    most = (1 << 24) - 1
    got = G.iodf_attn_plan(attn, ints([0]), ints([1]), ints([[-1]]), ring[:most], ints([most - 1, 1]), 1)
    assert got[2].tolist() == [5 * 128] and got[4].tolist() == [0, 0]
    with pytest.raises(G.IodfError) as e:
        G.iodf_attn_plan(attn, ints([0]), ints([1]), ints([[-1]]), ring, ints([0, 1]), 1)
    assert e.value.status == EUNSUPPORTED
    G.iodf_attn_check(attn)
