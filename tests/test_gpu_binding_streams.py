"""Outputs that the binding makes, and what it reads back itself, for calls on another stream than the current one."""
import numpy as np
import pytest
import torch

import iodf_synth as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


@pytest.fixture(scope="module")
def coded(G):
    model = S.make_model(0x57E0, 3, 32, 32, [True, True, False], 2, 24, prune=(0.4, 0.7))
    x = torch.from_numpy(S.smooth_field_images(0x57E1, 64, 32, 32, 2.0)).cuda()
    m = G.iodf_create(model, 64)
    codec = G.iodf_codec_create(m, S.logistic_codec())
    z, prior = G.iodf_forward(m, x)
    words, counts = G.iodf_rans_encode(codec, z, prior)
    packed, total = G.iodf_rans_pack(codec, words, counts)
    G.iodf_rans_unpack(codec, packed, total, 64)     # a kernel's first launch may wait for the device
    torch.zeros_like(packed)
    torch.cuda.synchronize()
    return m, codec, x, z, prior, words, counts, packed, total


def _busy(cycles=100_000_000):
    torch.cuda._sleep(cycles)


def _late(*like):
    """Tensors of these shapes that the current stream fills late, freed at once: the next of their size get their memory."""
    made = [torch.empty_like(t) for t in like]
    _busy()
    for t in made:
        t.fill_(33)


def test_the_size_of_a_byte_stream_is_read_on_the_calls_stream(G, coded):
    m, codec, x, z, prior, words, counts, packed, total = coded
    side = torch.cuda.Stream()
    out = torch.zeros_like(packed)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        _busy()
    p, n = G.iodf_rans_pack(codec, words, counts, packed=out, stream=side)
    assert n == total and torch.equal(p[:n], packed[:n])


def test_an_unpacked_container_is_not_erased_by_its_own_fill(G, coded):
    m, codec, x, z, prior, words, counts, packed, total = coded
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _busy()
    w, c = G.iodf_rans_unpack(codec, packed, total, 64, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(c, counts) and int(c.sum()) > 0
    z2 = torch.zeros_like(z)
    for q in range(codec.n_blocks):
        G.iodf_rans_decode_block(codec, q, w, c, prior, z2)
    G.iodf_codec_check(codec)
    assert torch.equal(z2, z)


def test_outputs_on_a_side_stream_are_not_what_the_current_stream_still_writes(G):
    """From 10 MB on a tensor has an allocation of its own, which the next of its size takes."""
    model = S.make_model(0x57E2, 3, 64, 64, [True, False], 1, 16)
    m = G.iodf_create(model, 1024)
    x = torch.from_numpy(S.smooth_field_images(0x57E3, 4, 64, 64, 2.0)).cuda().repeat(256, 1, 1, 1)
    z, prior = G.iodf_forward(m, x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _late(z, prior)
    z2, p2 = G.iodf_forward(m, x, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(z2, z) and torch.equal(p2, prior)
    _late(x)
    x2 = G.iodf_inverse(m, z, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(x2, x)


def test_outputs_on_a_side_stream_stay_until_the_current_stream_has_read_them(G):
    model = S.make_model(0x57E2, 3, 64, 64, [True, False], 1, 16)
    m = G.iodf_create(model, 1024)
    x = torch.from_numpy(S.smooth_field_images(0x57E3, 4, 64, 64, 2.0)).cuda().repeat(256, 1, 1, 1)
    other = 255 - x
    want = G.iodf_forward(m, x)[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    z, prior = G.iodf_forward(m, x, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    _busy()
    got = z.clone()                                  # late
    del z, prior
    z2, p2 = G.iodf_forward(m, other, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
