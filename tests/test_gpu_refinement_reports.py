"""What a codec says of a refinement that went wrong, and codecs that share the layers of their refinements."""
import numpy as np
import pytest
import torch

from test_gpu_refinement import _set, _setup

pytestmark = pytest.mark.gpu

ETIMEOUT, EDATA = -5, -9


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


def _status(G, f, *a, **k):
    with pytest.raises(G.IodfError) as e:
        f(*a, **k)
    return e.value.status


def test_a_wait_that_runs_out_in_a_refinement_is_reported_by_the_codec(G):
    m, codec, blocks, x = _setup(G, 0xD0DE, batch=3)
    xh = torch.from_numpy(x).pin_memory()
    assert _status(G, G.iodf_codec_selftest_timeout, codec, 0) == -1       # no refinement yet
    _set(G, codec, blocks, torch.tensor([0, 2, -1], dtype=torch.int32, device="cuda"))
    assert _status(G, G.iodf_codec_selftest_timeout, codec, 2) == -1       # no prior head
    assert _status(G, G.iodf_codec_selftest_timeout, codec, 0, tries=101) == -1
    buf, n = G.iodf_compress_host(m, codec, xh)
    want = buf[:n].clone()
    G.iodf_codec_check(codec)
    for level in blocks:
        G.iodf_codec_selftest_timeout(codec, level)
        for _ in range(2):                           # no bytes until somebody has looked
            assert _status(G, G.iodf_compress_host, m, codec, xh) == ETIMEOUT
        assert _status(G, G.iodf_codec_check, codec) == ETIMEOUT
        G.iodf_codec_check(codec)
        buf, n = G.iodf_compress_host(m, codec, xh)
        assert torch.equal(buf[:n], want)
        out = G.iodf_decompress_host(m, codec, buf, n, 3)
        G.iodf_codec_selftest_timeout(codec, level)
        assert _status(G, G.iodf_codec_check, codec) == ETIMEOUT
        np.testing.assert_array_equal(out.numpy(), x)
    for b in blocks.values():
        G.iodf_proj_check(b.up)
        G.iodf_proj_check(b.down)


def test_an_adapter_slot_that_is_not_there_is_reported_by_the_codec(G):
    m, codec, blocks, x = _setup(G, 0xD0DF, batch=4)
    xh = torch.from_numpy(x).pin_memory()
    who = torch.tensor([0, -1, 2, -1], dtype=torch.int32, device="cuda")
    _set(G, codec, blocks, who)
    buf, n = G.iodf_compress_host(m, codec, xh)
    want = buf[:n].clone()
    G.iodf_codec_check(codec)
    who.copy_(torch.tensor([0, 3, 2, -2], dtype=torch.int32))
    buf, n = G.iodf_compress_host(m, codec, xh)      # as none
    assert torch.equal(buf[:n], want)
    assert _status(G, G.iodf_codec_check, codec) == EDATA
    G.iodf_codec_check(codec)
    out = G.iodf_decompress_host(m, codec, buf, n, 4)
    assert _status(G, G.iodf_codec_check, codec) == EDATA
    np.testing.assert_array_equal(out.numpy(), x)
    z, prior = G.iodf_forward(m, torch.from_numpy(x).cuda())
    G.iodf_refine_prior(codec, 1, prior)
    assert _status(G, G.iodf_codec_check, codec) == EDATA


def test_codecs_in_flight_share_the_layers_of_their_refinements(G):
    """Each with batches and customers of its own on a stream of its own, the owner of the projections beside them."""
    import iodf_synth as S
    n, B = 3, 64
    m, codec, blocks, x = _setup(G, 0xD0E0, batch=B)
    codecs = [codec] + [G.iodf_codec_create(m, S.logistic_codec()) for _ in range(n - 1)]
    rng = np.random.default_rng(7)
    b = blocks[1]
    c, px, off = b.c, b.px, int(m.layout.prior_off[1])
    lanes = []
    for c_ in codecs:
        who = rng.integers(-1, 3, B)
        _set(G, c_, blocks, torch.from_numpy(who.astype(np.int32)).cuda())
        z, prior = G.iodf_forward(m, torch.from_numpy(x).cuda())
        want = prior.clone()
        mu = prior[:, 0, off:off + c * px].reshape(B, c, px).cpu().numpy()
        want[:, 0, off:off + c * px] = torch.from_numpy(b.plain(mu, who.tolist()).reshape(B, -1).astype(np.int32)).cuda()
        lanes.append((c_, torch.cuda.Stream(), [prior.clone() for _ in range(12)], want))
    own_x = torch.from_numpy(rng.integers(0, 256, (B * px, b.down.c_in + 15)).astype(np.uint8)).cuda()
    own_x = own_x[:, :b.down.c_in // 16 * 16 + 16].contiguous()[:, :b.down.c_in]
    starts, slots = torch.tensor([0, B * px // 2, B * px], dtype=torch.int32, device="cuda"), torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    own_want = G.iodf_proj_forward(b.down, own_x, starts, slots)
    own = [torch.zeros_like(own_want) for _ in range(12)]
    mine = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(12):
        for c_, stream, priors, _ in lanes:
            G.iodf_refine_prior(c_, 1, priors[i], stream=stream)
        G.iodf_proj_forward(b.down, own_x, starts, slots, y=own[i], stream=mine)
    torch.cuda.synchronize()
    for c_, _, priors, want in lanes:
        G.iodf_codec_check(c_)
        for p in priors:
            assert torch.equal(p, want)
    assert all(torch.equal(y, own_want) for y in own)


def test_a_refinement_captured_and_replayed(G):
    """What the graph reads, the means and the images' customers, changes between replays."""
    m, codec, blocks, x = _setup(G, 0xD0E1, batch=6)
    who = torch.tensor([0, 1, 2, -1, 1, 0], dtype=torch.int32, device="cuda")
    _set(G, codec, blocks, who)
    z, prior = G.iodf_forward(m, torch.from_numpy(x).cuda())
    buf = prior.clone()
    G.iodf_refine_prior(codec, 0, buf)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for level in blocks:
            G.iodf_refine_prior(codec, level, buf)
    for i, slots in enumerate(([2, 2, 0, 1, -1, 1], [-1] * 6, [0, 1, 2, 0, 1, 2])):
        who.copy_(torch.tensor(slots, dtype=torch.int32))
        buf.copy_(prior.roll(i, 0))
        want = buf.cpu().numpy()
        for level, b in blocks.items():
            off = int(m.layout.prior_off[level])
            part = want[:, 0, off:off + b.c * b.px]
            part[:] = b.plain(part.reshape(6, b.c, b.px), slots).reshape(6, -1)
        graph.replay()
        np.testing.assert_array_equal(buf.cpu().numpy(), want)
        G.iodf_codec_check(codec)
    del graph
