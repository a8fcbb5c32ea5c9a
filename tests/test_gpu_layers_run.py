"""The single integer layers together, as a codec uses them: a residual block with adapters of each image's
customer refines the prior parameters between the flow and the entropy coder, on both sides of the codec."""
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


class Refinement:
    """mu += scale * norm(down(relu(up(norm(mu)))), per level, with an adapter per image in both projections."""

    def __init__(self, G, rng, c, px, batch, customers, hidden=72):
        self.G, self.c, self.px = G, c, px
        rows = batch * px
        cp = (c + 15) // 16 * 16
        self.layers = [_layer(rng, c, hidden, True, (0, 255)), _layer(rng, hidden, c, False, (-128, 127))]
        self.adapters = [[_adapter(rng, l["c_in"], l["c_out"], R) for _ in range(customers)] for l, R in zip(self.layers, (6, 17))]
        types = [(torch.int8, torch.uint8), (torch.uint8, torch.int8)]
        self.proj = []
        for l, ads, (xt, yt) in zip(self.layers, self.adapters, types):
            p = G.iodf_proj_create(l, rows, customers, 32, x_dtype=xt, y_dtype=yt)
            for i, ad in enumerate(ads):
                G.iodf_proj_set_adapter(p, i, ad)
            self.proj.append(p)
        unit = 2 ** 22 / np.sqrt(c)
        one = lambda: rng.integers(2 ** 30, 2 ** 31, c).astype(np.int32)
        self.first = {"c": c, "res_dtype": torch.int32, "eps": c, "pre": {
            "norm": "rms", "mult": one(), "shift": int(np.log2(unit / 40)), "bias": np.zeros(c, np.int32), "clamp": (-128, 127), "dtype": torch.int8}}
        self.last = {"c": c, "res_dtype": torch.int32, "eps": c, "block_dtype": torch.int8, "res_range": (-4096, 4095),
                     "post": {"norm": "rms", "mult": one(), "shift": int(np.log2(unit / 3))}}
        self.gate = (rng.random(c) < 0.7).astype(np.uint8)
        self.norms = [G.iodf_norm_create(self.first), G.iodf_norm_create(self.last)]
        self.gate_dev = torch.from_numpy(self.gate).cuda()
        self.n = torch.zeros((rows, cp), dtype=torch.int8, device="cuda")[:, :c]
        self.u = torch.zeros((rows, (hidden + 15) // 16 * 16), dtype=torch.uint8, device="cuda")[:, :hidden]
        self.b = torch.zeros((rows, c), dtype=torch.int8, device="cuda")
        self.start = torch.arange(batch + 1, dtype=torch.int32, device="cuda") * px

    def __call__(self, mu, customer):
        """mu: [batch, c, px] planes inside the prior buffer, refined in place."""
        G = self.G
        G.iodf_norm_forward(self.norms[0], mu, n=self.n)
        G.iodf_proj_forward(self.proj[0], self.n, self.start, customer, y=self.u)
        G.iodf_proj_forward(self.proj[1], self.u, self.start, customer, y=self.b)
        G.iodf_norm_forward(self.norms[1], mu, self.b, self.gate_dev, r_out=mu)

    def plain(self, mu, customer):
        B = mu.shape[0]
        start = [i * self.px for i in range(B + 1)]
        r = mu.transpose(0, 2, 1).reshape(-1, self.c)
        _, n = P.norm_step(self.first, r)
        u = P.projection(self.layers[0], n.astype(np.int8), self.adapters[0], start, customer)
        b = P.projection(self.layers[1], u.astype(np.uint8), self.adapters[1], start, customer)
        out, _ = P.norm_step(self.last, r, b.astype(np.int8), self.gate)
        return out.reshape(B, self.px, self.c).transpose(0, 2, 1)


def _levels(lay):
    for li in range(int(lay.n_levels) - 1):
        yield li, lay.level_c[li] // 2, lay.level_h[li] * lay.level_w[li], int(lay.prior_off[li])


def test_refined_prior_on_both_sides_of_the_codec(G):
    rng = np.random.default_rng(0x1DF)
    batch, customers = 9, 4
    model = S.make_model(0x1DF0, 3, 32, 32, [True, True, False], 2, 24, prune=(0.4, 0.7))
    x = S.smooth_field_images(0x1DF1, batch, 32, 32, 2.0)
    m = G.iodf_create(model, batch)
    codec = G.iodf_codec_create(m, S.logistic_codec())
    refine = {li: Refinement(G, rng, c, px, batch, customers) for li, c, px, _ in _levels(m.layout)}
    customer = torch.tensor([0, 1, 2, 3, -1, 0, 0, 2, 1], dtype=torch.int32, device="cuda")
    who = customer.cpu().tolist()

    def planes(prior, li, c, px, off):
        return prior[:, 0, off:off + c * px].unflatten(1, (c, px))

    xt = torch.from_numpy(x).cuda()
    z, prior = G.iodf_forward(m, xt)
    plain_prior = prior.cpu().numpy().copy()
    for li, c, px, off in _levels(m.layout):
        refine[li](planes(prior, li, c, px, off), customer)
        plain_prior[:, 0, off:off + c * px] = refine[li].plain(
            plain_prior[:, 0, off:off + c * px].reshape(batch, c, px), who).reshape(batch, -1)
    np.testing.assert_array_equal(prior.cpu().numpy(), plain_prior)
    words, counts = G.iodf_rans_encode(codec, z, prior)

    # the decoder meets the levels from the deepest on and refines each level's prior before it decodes its block
    blocks = {codec.layout.block_level[q]: q for q in range(codec.n_blocks)}
    z2, prior2 = torch.full_like(z, -777), torch.full_like(prior, -777)
    x2 = torch.empty_like(xt)
    G.iodf_rans_decode_block(codec, blocks[-1], words, counts, prior2, z2)
    shapes = {li: (c, px, off) for li, c, px, off in _levels(m.layout)}
    for li in range(int(m.layout.n_levels) - 1, -1, -1):
        if li in shapes:
            G.iodf_inverse_level(m, li, G.IODF_LEVEL_PRIOR, z2, prior=prior2)
            refine[li](planes(prior2, li, *shapes[li]), customer)
            G.iodf_rans_decode_block(codec, blocks[li], words, counts, prior2, z2)
        G.iodf_inverse_level(m, li, G.IODF_LEVEL_COUPLINGS, z2, x_u8=x2)
    G.iodf_codec_check(codec)
    G.iodf_check(m)
    for r in refine.values():
        for p in r.proj:
            G.iodf_proj_check(p)
    np.testing.assert_array_equal(prior2.cpu().numpy(), plain_prior)
    assert torch.equal(z2, z)
    np.testing.assert_array_equal(x2.cpu().numpy(), x)


def test_a_chain_of_blocks_over_tokens(G):
    """norm, projection up with adapters, projection down, gate, scale, residual sum and the next norm, twice,
    for a prompt and then row by row: a row's values do not depend on what it is computed with."""
    rng = np.random.default_rng(33)
    C, H, rows = 144, 400, 37
    up, down = _layer(rng, C, H, True, (0, 255)), _layer(rng, H, C, False, (-128, 127))
    ads = [_adapter(rng, C, H, 16) for _ in range(3)]
    pu = G.iodf_proj_create(up, rows, 3, 16, x_dtype=torch.int8, y_dtype=torch.uint8)
    pd = G.iodf_proj_create(down, rows, x_dtype=torch.uint8, y_dtype=torch.int8)
    for i, ad in enumerate(ads):
        G.iodf_proj_set_adapter(pu, i, ad)
    unit = 2 ** 22 / np.sqrt(C)
    mult = lambda: rng.integers(2 ** 30, 2 ** 31, C).astype(np.int32)
    pre = {"norm": "rms", "mult": mult(), "shift": int(np.log2(unit / 40)), "bias": np.zeros(C, np.int32), "clamp": (-128, 127), "dtype": torch.int8}
    d0 = {"c": C, "res_dtype": torch.int16, "eps": C, "pre": pre}
    d1 = {"c": C, "res_dtype": torch.int16, "eps": C, "block_dtype": torch.int8, "res_range": (-32768, 32767),
          "post": {"norm": "rms", "mult": mult(), "shift": int(np.log2(unit * 128 / 50))}, "pre": pre}
    n0, n1 = G.iodf_norm_create(d0), G.iodf_norm_create(d1)
    r = rng.integers(-900, 900, (rows, C)).astype(np.int16)
    gate = rng.integers(0, 256, (rows, C)).astype(np.uint8)
    starts, which = [0, 5, 6, 30, rows], [0, 1, 2, -1]
    slot = P.slots_of_rows(rows, starts, which)

    def chain(r, gate, start, who):
        r, gate = r.clone(), gate.contiguous()
        st = torch.tensor(start, dtype=torch.int32, device="cuda")
        wh = torch.tensor(who, dtype=torch.int32, device="cuda")
        _, n = G.iodf_norm_forward(n0, r)
        for _ in range(2):
            b = G.iodf_proj_forward(pd, G.iodf_proj_forward(pu, n, st, wh))
            _, n = G.iodf_norm_forward(n1, r, b, gate, r_out=r)
        return r, n

    rt, gt = torch.from_numpy(r).cuda(), torch.from_numpy(gate).cuda()
    ro, no = chain(rt, gt, starts, which)
    pr = r
    _, pn = P.norm_step(d0, pr)
    for _ in range(2):
        b = P.projection(down, P.projection(up, pn.astype(np.int8), ads, starts, which).astype(np.uint8))
        pr, pn = P.norm_step(d1, pr, b.astype(np.int8), gate)
    np.testing.assert_array_equal(ro.cpu().numpy().astype(np.int64), pr)
    np.testing.assert_array_equal(no.cpu().numpy().astype(np.int64), pn)
    for row in (0, 5, 17, 36):
        r1, n1_ = chain(rt[row:row + 1], gt[row:row + 1], [0, 1], [int(slot[row])])
        assert torch.equal(r1[0], ro[row]) and torch.equal(n1_[0], no[row])
