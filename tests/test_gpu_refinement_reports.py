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
