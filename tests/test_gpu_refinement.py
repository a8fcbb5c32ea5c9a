"""A codec that refines its prior parameters: the compressor and decompressor for host buffers, and the steps by hand."""
import numpy as np
import pytest
import torch

import iodf_synth as S
from oracle import layers as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


def _layer(rng, K, N, relu, clamp):
    return {"k": 1, "c_in": K, "c_out": N, "w": np.clip(np.round(rng.normal(0, 32, (N, K))), -127, 127).astype(np.int8),
            "bias": rng.integers(-2000, 2000, N).astype(np.int32), "m0": rng.integers(2 ** 30, 2 ** 31, N).astype(np.int32),
            "s": np.full(N, 7, np.int32), "relu": relu, "clamp": clamp}


def _adapter(rng, K, N, R):
    return {"rank": R, "down": np.clip(np.round(rng.normal(0, 32, (R, K))), -127, 127).astype(np.int8),
            "m0": rng.integers(2 ** 30, 2 ** 31, R).astype(np.int32), "s": np.full(R, 6, np.int32),
            "up": np.clip(np.round(rng.normal(0, 16, (N, R))), -127, 127).astype(np.int8)}


class Block:
    def __init__(self, G, rng, c, px, max_batch, customers, hidden, wide):
        """wide: the block's output as int32 instead of int8."""
        rows, self.c, self.px = max_batch * px, c, px
        bt = torch.int32 if wide else torch.int8
        self.layers = [_layer(rng, c, hidden, True, (0, 255)), _layer(rng, hidden, c, False, None if wide else (-128, 127))]
        self.adapters = [[_adapter(rng, l["c_in"], l["c_out"], R) for _ in range(customers)] for l, R in zip(self.layers, (5, 18))]
        self.up = G.iodf_proj_create(self.layers[0], rows, customers, 18, x_dtype=torch.int8, y_dtype=torch.uint8)
        self.down = G.iodf_proj_create(self.layers[1], rows, customers, 18, x_dtype=torch.uint8, y_dtype=bt)
        for p, ads in ((self.up, self.adapters[0]), (self.down, self.adapters[1])):
            for i, ad in enumerate(ads):
                G.iodf_proj_set_adapter(p, i, ad)
        unit = 2 ** 22 / np.sqrt(c)
        one = lambda: rng.integers(2 ** 30, 2 ** 31, c).astype(np.int32)
        self.d_first = {"c": c, "res_dtype": torch.int32, "eps": c, "pre": {
            "norm": "rms", "mult": one(), "shift": int(np.log2(unit / 40)), "bias": np.zeros(c, np.int32), "clamp": (-128, 127), "dtype": torch.int8}}
        self.d_last = {"c": c, "res_dtype": torch.int32, "eps": c, "block_dtype": bt, "res_range": (-4096, 4095),
                       "post": {"norm": "centred", "mult": one(), "shift": int(np.log2(unit / 3))}}
        self.first, self.last = G.iodf_norm_create(self.d_first), G.iodf_norm_create(self.d_last)
        self.gate_host = (rng.random(c) < 0.7).astype(np.uint8)
        self.gate = torch.from_numpy(self.gate_host).cuda()

    def plain(self, mu, who):
        B = mu.shape[0]
        start = [i * self.px for i in range(B + 1)]
        r = mu.transpose(0, 2, 1).reshape(-1, self.c)
        _, n = P.norm_step(self.d_first, r)
        u = P.projection(self.layers[0], n.astype(np.int8), self.adapters[0], start, who)
        b = P.projection(self.layers[1], u.astype(np.uint8), self.adapters[1], start, who)
        out, _ = P.norm_step(self.d_last, r, b.astype(np.int32), self.gate_host)
        return out.reshape(B, self.px, self.c).transpose(0, 2, 1)


def _setup(G, seed, side=32, batch=7, customers=3):
    rng = np.random.default_rng(seed)
    model = S.make_model(seed, 3, side, side, [True, True, False], 2, 24, prune=(0.4, 0.7))
    m = G.iodf_create(model, batch)
    codec = G.iodf_codec_create(m, S.logistic_codec())
    blocks = {}
    for li in range(2):
        c, px = m.layout.level_c[li] // 2, m.layout.level_h[li] * m.layout.level_w[li]
        blocks[li] = Block(G, rng, c, px, batch, customers, 40 + 31 * li, wide=li == 1)
    x = S.smooth_field_images(seed + 1, batch, side, side, 2.0)
    return m, codec, blocks, x


def _set(G, codec, blocks, who):
    for li, b in blocks.items():
        G.iodf_codec_set_refinement(codec, li, b.first, b.up, b.down, b.last, b.gate, who)


def test_compressor_and_decompressor(G):
    m, codec, blocks, x = _setup(G, 0xC0DE)
    who = torch.tensor([0, 2, 1, -1, 1, 0, 2], dtype=torch.int32, device="cuda")
    xh = torch.from_numpy(x).pin_memory()
    plain_buf, plain_n = G.iodf_compress_host(m, codec, xh)
    plain_bytes = plain_buf[:plain_n].clone()
    _set(G, codec, blocks, who)
    for B in (7, 3, 1):
        buf, n = G.iodf_compress_host(m, codec, xh[:B])
        # the steps by hand give the same stream ...
        z, prior = G.iodf_forward(m, torch.from_numpy(x[:B]).cuda())
        want = prior.cpu().numpy().copy()
        for li, b in blocks.items():
            off = int(m.layout.prior_off[li])
            want[:, 0, off:off + b.c * b.px] = b.plain(want[:, 0, off:off + b.c * b.px].reshape(B, b.c, b.px), who.tolist()[:B]).reshape(B, -1)
            G.iodf_refine_prior(codec, li, prior)
        np.testing.assert_array_equal(prior.cpu().numpy(), want)
        words, counts = G.iodf_rans_encode(codec, z, prior)
        packed, total = G.iodf_rans_pack(codec, words, counts)
        assert total == n and torch.equal(packed[:n].cpu(), buf[:n])
        # ... and it decodes
        out = G.iodf_decompress_host(m, codec, buf, n, B)
        torch.cuda.synchronize()
        G.iodf_codec_check(codec)
        G.iodf_check(m)
        np.testing.assert_array_equal(out.numpy(), x[:B])
    for b in blocks.values():
        G.iodf_proj_check(b.up)
        G.iodf_proj_check(b.down)
    # another customer's adapters are not this one's
    who.fill_(1)
    out = G.iodf_decompress_host(m, codec, buf, n, 1)
    torch.cuda.synchronize()
    try:
        G.iodf_codec_check(codec)
    except G.IodfError:
        pass
    assert not np.array_equal(out.numpy(), x[:1])
    # and without the refinement the codec is what it was
    for li in blocks:
        G.iodf_codec_set_refinement(codec, li)
    buf, n = G.iodf_compress_host(m, codec, xh)
    assert n == plain_n and torch.equal(buf[:n], plain_bytes)
    z, prior = G.iodf_forward(m, torch.from_numpy(x).cuda())
    before = prior.clone()
    G.iodf_refine_prior(codec, 0, prior)
    assert torch.equal(prior, before)


def test_without_adapters_and_gate(G):
    m, codec, blocks, x = _setup(G, 0xC0DF, batch=4)
    b = blocks[0]
    G.iodf_codec_set_refinement(codec, 0, b.first, b.up, b.down, b.last)
    buf, n = G.iodf_compress_host(m, codec, torch.from_numpy(x).pin_memory())
    out = G.iodf_decompress_host(m, codec, buf, n, 4)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(out.numpy(), x)
    b.gate_host[:] = 1
    z, prior = G.iodf_forward(m, torch.from_numpy(x).cuda())
    want = b.plain(prior[:, 0, :b.c * b.px].reshape(4, b.c, b.px).cpu().numpy(), [-1] * 4)
    G.iodf_refine_prior(codec, 0, prior)
    np.testing.assert_array_equal(prior[:, 0, :b.c * b.px].reshape(4, b.c, b.px).cpu().numpy(), want)


def test_refusals(G):
    m, codec, blocks, x = _setup(G, 0xC0E0)
    b0, b1 = blocks[0], blocks[1]
    rows = 7 * b0.px

    def refused(level, *parts, **kw):
        with pytest.raises(G.IodfError) as e:
            G.iodf_codec_set_refinement(codec, level, *parts, **kw)
        assert e.value.status == -1

    good = (b0.first, b0.up, b0.down, b0.last)
    refused(2, *good)                                    # no prior head
    refused(-1, *good)
    refused(8, *good)
    refused(1, *good)                                    # another level's channels
    refused(0, b0.last, b0.up, b0.down, b0.last)         # a norm with a block in front
    refused(0, b0.first, b0.up, b0.down, b0.first)       # and one without behind
    refused(0, b0.first, b0.up, b0.up, b0.last)
    few = G.iodf_proj_create(b0.layers[0], rows - 1, x_dtype=torch.int8, y_dtype=torch.uint8)
    refused(0, b0.first, few, b0.down, b0.last)
    unsigned = G.iodf_proj_create(b0.layers[0], rows, x_dtype=torch.uint8, y_dtype=torch.uint8)
    refused(0, b0.first, unsigned, b0.down, b0.last)
    wide = G.iodf_proj_create(dict(b0.layers[1], clamp=None), rows, x_dtype=torch.uint8, y_dtype=torch.int32)
    refused(0, b0.first, b0.up, wide, b0.last)
    short = dict(b0.d_first, res_dtype=torch.int16)
    refused(0, G.iodf_norm_create(short), b0.up, b0.down, b0.last)
    with pytest.raises(ValueError):
        G.iodf_codec_set_refinement(codec, 0, b0.first, b0.up)
    with pytest.raises(ValueError):
        G.iodf_codec_set_refinement(codec, 0, *good, gate=b0.gate[:-1])
    with pytest.raises(ValueError):
        G.iodf_codec_set_refinement(codec, 0, *good, image_adapter=torch.zeros(6, dtype=torch.int32, device="cuda"))
    prior = torch.zeros((8, 2, m.d_fact), dtype=torch.int32, device="cuda")
    with pytest.raises(G.IodfError):
        G.iodf_refine_prior(codec, 0, prior)             # more images than the codec holds
    with pytest.raises(G.IodfError):
        G.iodf_refine_prior(codec, 2, prior[:2])


def test_a_model_whose_prior_buffer_has_another_size_is_refused(G):
    m, codec, blocks, x = _setup(G, 0xC0E1, batch=2)
    other = G.iodf_create(S.make_model(5, 3, 32, 32, [False, True, False], 2, 24), 2)
    assert other.d == m.d and other.d_fact != m.d_fact
    _set(G, codec, {0: blocks[0]}, None)
    xh = torch.from_numpy(x).pin_memory()
    with pytest.raises(G.IodfError) as e:
        G.iodf_compress_host(other, codec, xh)
    assert e.value.status == -1
    buf, n = G.iodf_compress_host(m, codec, xh)
    with pytest.raises(G.IodfError) as e:
        G.iodf_decompress_host(other, codec, buf, n, 2)
    assert e.value.status == -1
