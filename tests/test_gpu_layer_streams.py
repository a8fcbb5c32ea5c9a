"""Single integer layers on another stream than the current one: their outputs, and what is read right after they are made."""
import numpy as np
import pytest
import torch

from oracle import layers as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


def _busy():
    """Some 50 ms of work on the current stream."""
    torch.cuda._sleep(100_000_000)


def _layer(rng, K, N):
    return {"k": 1, "c_in": K, "c_out": N, "w": rng.integers(-127, 128, (N, K)).astype(np.int8),
            "bias": rng.integers(-3000, 3000, N).astype(np.int32), "m0": rng.integers(2 ** 30, 2 ** 31, N).astype(np.int32),
            "s": np.full(N, 8, np.int32), "relu": False, "clamp": (-128, 127)}


def _norm_desc(rng, C, block=torch.int8):
    mult = lambda: rng.integers(2 ** 29, 2 ** 31, C).astype(np.int32)
    d = {"c": C, "res_dtype": torch.int16, "eps": C, "block_dtype": block, "res_range": (-32768, 32767),
         "pre": {"norm": "rms", "mult": mult(), "shift": 13, "bias": np.zeros(C, np.int32), "clamp": (-128, 127), "dtype": torch.int8}}
    if block:
        d["post"] = {"norm": "rms", "mult": mult(), "shift": 15}
    return d


@pytest.mark.parametrize("given", ["stream", "handle"])
def test_outputs_made_by_a_projection_on_a_side_stream(G, given):
    """The zero fill of a y that the call makes comes before the kernel, however late the current stream is."""
    rng = np.random.default_rng(1)
    rows, K, N = 300, 64, 48
    layer = _layer(rng, K, N)
    h = G.iodf_proj_create(layer, rows, 1, 1, y_dtype=torch.int8)
    xh = rng.integers(-128, 128, (rows, K)).astype(np.int8)
    x = torch.from_numpy(xh).cuda()
    st, wh = torch.tensor([5, 290], dtype=torch.int32, device="cuda"), torch.tensor([-1], dtype=torch.int32, device="cuda")
    want = P.projection(layer, xh, [None], [5, 290], [-1], np.zeros((rows, N)))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    junk = torch.full((rows, N), 77, dtype=torch.int8, device="cuda")      # what y's memory held
    del junk
    _busy()
    y = G.iodf_proj_forward(h, x, st, wh, stream=side if given == "stream" else side.cuda_stream)
    side.synchronize()
    with torch.cuda.stream(side):
        early = y.cpu().numpy()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(early, want)
    np.testing.assert_array_equal(y.cpu().numpy(), want)


def test_outputs_made_by_a_norm_on_a_side_stream(G):
    """Their memory is not what work of the current stream still writes."""
    rng = np.random.default_rng(2)
    rows, C = 65536, 192                             # from 10 MB on a tensor has an allocation of its own, which the next of its size takes
    h = G.iodf_norm_create(_norm_desc(rng, C))
    r = torch.from_numpy(rng.integers(-900, 900, (rows, C)).astype(np.int16)).cuda()
    b = torch.from_numpy(rng.integers(-60, 60, (rows, C)).astype(np.int8)).cuda()
    want = [t.cpu() for t in G.iodf_norm_forward(h, r, b, r_out=torch.empty_like(r), n=torch.empty_like(b))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    late = [torch.empty_like(r), torch.empty_like(b)]
    _busy()
    for t in late:
        t.fill_(33)                                  # waits behind the work of the current stream
    del t, late
    o, n = G.iodf_norm_forward(h, r, b, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(o.cpu(), want[0]) and torch.equal(n.cpu(), want[1])


def test_handles_used_at_once_on_a_stream_that_waits_for_nobody(G):
    rng = np.random.default_rng(3)
    rows, C = 3, 8192
    r, b = rng.integers(-900, 900, (rows, C)).astype(np.int16), rng.integers(-60, 60, (rows, C)).astype(np.int8)
    rt, bt = torch.from_numpy(r).cuda(), torch.from_numpy(b).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(6):
        d = _norm_desc(rng, C)
        o, n = G.iodf_norm_forward(G.iodf_norm_create(d), rt, bt, stream=side)
        side.synchronize()
        wo, wn = P.norm_step(d, r, b)
        np.testing.assert_array_equal(o.cpu().numpy().astype(np.int64), wo)
        np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), wn)
