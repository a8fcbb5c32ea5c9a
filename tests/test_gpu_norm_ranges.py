"""Norms of rows whose squares all lie with one thread: the widest values that a thread's sum may meet, at every width and layout."""
import numpy as np
import pytest
import torch

from oracle import layers as P
from test_gpu_norm import make_desc, place

pytestmark = pytest.mark.gpu

LO, HI = -2 ** 23, 2 ** 23 - 1


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


def _rows(rng, C):
    """Rows at one end of the range but for up to 16 channels at the other: neighbours, a thread's share at a stride, the last, the first."""
    rows = []
    for base, other in ((HI, LO), (LO, HI)):
        for stride in (1, 8, 16, 32, 64, 128, 256, 512):
            for start in (0, max(0, C - 1 - 15 * stride)):
                v = np.full(C, base, np.int64)
                v[start:start + 16 * stride:stride] = other
                rows.append(v)
                if C > 128:                          # sixteen in vectors of eight, as an aligned row's thread has them
                    v = np.full(C, base, np.int64)
                    v[start:start + 8] = other
                    v[start + C // 2:start + C // 2 + 8] = other
                    rows.append(v)
        rows += [np.full(C, base, np.int64), np.where(np.arange(C) == C - 1, other, base)]
    return np.array(rows).astype(np.int32)


@pytest.mark.parametrize("C", [1, 8, 33, 64, 128, 173, 256, 512, 600, 1024, 2048, 4096, 8191, 8192])
@pytest.mark.parametrize("pre", ["centred", "rms"])
def test_wide_values_in_one_thread(G, C, pre):
    rng = np.random.default_rng(C)
    r = _rows(rng, C)
    for eps in (1, C):
        d = make_desc(rng, C, torch.int32, None, None, pre, eps=eps)
        h = G.iodf_norm_create(d)
        want = P.norm_step(d, r)[1]
        for skip in (0, 1):                          # aligned, and one element per access
            _, n = G.iodf_norm_forward(h, place(r, C, skip))
            np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), want)


@pytest.mark.parametrize("C", [6, 32, 48, 128, 256])
def test_wide_values_in_one_thread_of_planes(G, C):
    rng = np.random.default_rng(C)
    r = _rows(rng, C)
    b = np.ascontiguousarray(r[::-1])
    px = 7
    r, b = r[:len(r) // px * px], b[:len(r) // px * px]
    planes = torch.from_numpy(np.ascontiguousarray(r.reshape(-1, px, C).transpose(0, 2, 1))).cuda()
    d = make_desc(rng, C, torch.int32, torch.int32, "centred", "centred")
    o, n = G.iodf_norm_forward(G.iodf_norm_create(d), planes, torch.from_numpy(b).cuda())
    wo, wn = P.norm_step(d, r, b)
    np.testing.assert_array_equal(o.cpu().numpy().astype(np.int64).transpose(0, 2, 1).reshape(-1, C), wo)
    np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), wn)
