"""Norms before and after a block with its gate and residual scale on the GPU, bit for bit against the plain definition."""
import numpy as np
import pytest
import torch

from oracle import layers as P

pytestmark = pytest.mark.gpu

NP = {torch.int8: np.int8, torch.uint8: np.uint8, torch.int16: np.int16, torch.int32: np.int32}


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


def make_desc(rng, C, res, block, post, pre, n_dtype=torch.int8, eps=None, res_range=None, shifts=None):
    unit = 2 ** 22 / np.sqrt(C)
    sh = shifts or (int(np.clip(np.log2(unit), 1, 31)), int(np.clip(np.log2(unit / 64), 1, 31)))
    mult = lambda: rng.choice([-1, 1], C) * rng.integers(2 ** 29, 2 ** 31, C)
    d = {"c": C, "res_dtype": res, "eps": eps or C, "block_dtype": block,
         "res_range": res_range or ((-32768, 32767) if res == torch.int16 else (-2 ** 23, 2 ** 23 - 1))}
    if block:
        d["post"] = {"norm": post, "mult": mult().astype(np.int32), "shift": sh[0] if post else 3}
    if pre:
        d["pre"] = {"norm": pre, "mult": mult().astype(np.int32), "shift": sh[1], "bias": rng.integers(-40, 40, C).astype(np.int32),
                    "clamp": (-128, 127) if n_dtype == torch.int8 else (0, 255), "dtype": n_dtype}
    return d


def values(rng, rows, C, dtype, sigma):
    i = np.iinfo(NP[dtype])
    v = np.clip(np.round(rng.normal(0, sigma, (rows, C))), i.min, i.max).astype(NP[dtype])
    if rows > 2:
        v[1] = 0                              # nothing but zeros
        v[2] = i.max                          # beyond 24 bits for int32
    return v


def place(v, ld=None, skip=0):
    """The rows of v on the device with row stride ld, `skip` elements into a buffer."""
    rows, C = v.shape
    ld = ld or C
    buf = torch.zeros(skip + rows * ld, dtype=torch.from_numpy(v).dtype, device="cuda")
    t = buf[skip:].view(rows, ld)[:, :C]
    t.copy_(torch.from_numpy(v))
    return t


def check(G, rng, rows, C, res, block, post, pre, gated="", n_dtype=torch.int8, pad=(0, 0, 0, 0, 0), skip=0, in_place=False, **kw):
    d = make_desc(rng, C, res, block, post, pre, n_dtype, **kw)
    h = G.iodf_norm_create(d)
    r = values(rng, rows, C, res, 700)
    b = values(rng, rows, C, block, 30 if block == torch.int8 else 20000) if block else None
    gate = None
    if gated:
        gate = rng.integers(0, 256, (rows, C) if gated == "row" else C).astype(np.uint8)
    rt = place(r, C + pad[0], skip)
    bt = place(b, C + pad[1], skip) if block else None
    gt = None
    if gated:
        gt = place(gate, C + pad[2], skip) if gated == "row" else torch.from_numpy(gate).cuda()
    ot = None
    if block:
        ot = rt if in_place else place(np.full((rows, C), 99, NP[res]), C + pad[3], skip)
    nt = place(np.full((rows, C), 55, NP[n_dtype]), C + pad[4], skip) if pre else None
    o, n = G.iodf_norm_forward(h, rt, bt, gt, r_out=ot, n=nt)
    wo, wn = P.norm_step(d, r, b, gate)
    if block:
        np.testing.assert_array_equal(o.cpu().numpy().astype(np.int64), wo)
    if pre:
        np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), wn)


@pytest.mark.parametrize("res", [torch.int16, torch.int32])
@pytest.mark.parametrize("block", [torch.int8, torch.int32])
@pytest.mark.parametrize("rows,C", [(1, 1), (3, 2), (5, 7), (4, 8), (9, 31), (33, 64), (6, 65), (17, 128), (5, 173), (8, 256),
                                    (3, 257), (4, 512), (3, 1000), (3, 1024), (2, 2050), (3, 4096), (3, 8191), (3, 8192)])
def test_every_width(G, rows, C, res, block):
    rng = np.random.default_rng(C + rows)
    check(G, rng, rows, C, res, block, "rms", "rms", "row")
    check(G, rng, rows, C, res, block, "centred", "centred", "channel", n_dtype=torch.uint8)


@pytest.mark.parametrize("post", [None, "rms", "centred"])
@pytest.mark.parametrize("pre", [None, "rms", "centred"])
@pytest.mark.parametrize("gated", ["", "row", "channel"])
def test_every_combination(G, post, pre, gated):
    rng = np.random.default_rng(5)
    for res, block, C in ((torch.int16, torch.int8, 96), (torch.int32, torch.int32, 300), (torch.int32, torch.int8, 41)):
        check(G, rng, 21, C, res, block, post, pre, gated)


@pytest.mark.parametrize("pre", ["rms", "centred"])
@pytest.mark.parametrize("res", [torch.int16, torch.int32])
@pytest.mark.parametrize("C", [5, 64, 173, 640, 3000, 5000])
def test_norm_alone(G, res, pre, C):
    check(G, np.random.default_rng(C), 13, C, res, None, None, pre)


@pytest.mark.parametrize("pad,skip", [((0, 0, 0, 0, 0), 1), ((1, 0, 3, 0, 5), 0), ((8, 16, 16, 8, 16), 16), ((3, 1, 1, 7, 1), 3),
                                      ((8, 0, 0, 8, 0), 8)])
@pytest.mark.parametrize("C", [64, 173, 256, 1032])
def test_strides_and_alignment(G, C, pad, skip):
    rng = np.random.default_rng(C + skip)
    for res, block in ((torch.int16, torch.int8), (torch.int32, torch.int32), (torch.int16, torch.int32)):
        check(G, rng, 19, C, res, block, "rms", "rms", "row", pad=pad, skip=skip)


@pytest.mark.parametrize("C", [24, 256, 777])
def test_in_place(G, C):
    check(G, np.random.default_rng(C), 50, C, torch.int16, torch.int8, "rms", "centred", "row", in_place=True)
    check(G, np.random.default_rng(C), 50, C, torch.int32, torch.int32, None, "rms", in_place=True)


def test_many_rows(G):
    check(G, np.random.default_rng(1), 4001, 24, torch.int32, torch.int8, "rms", "rms", "row")
    check(G, np.random.default_rng(2), 2500, 130, torch.int16, torch.int32, "rms", "rms", "channel")


@pytest.mark.parametrize("eps", [1, 2, 3, 7, 1 << 31, (1 << 60) - 1, 1 << 60])
def test_small_and_large_sums_of_squares(G, eps):
    """Every position of the leading bit of D, perfect squares and their neighbours, and the widest rows."""
    rng = np.random.default_rng(eps % 1000)
    for C in (1, 2, 8192):
        d = make_desc(rng, C, torch.int32, None, None, "rms", eps=eps, shifts=(1, 15))
        h = G.iodf_norm_create(d)
        r = np.array([[v if c == 0 else (v if C > 2 and c % 3 == 0 else 0) for c in range(C)]
                      for v in [0, 1, 2, 3, 4, 15, 16, 17, 255, -256, 1000, -4096, 2 ** 15, 2 ** 20 + 1, -2 ** 23, 2 ** 23 - 1, 2 ** 31 - 1,
                                -2 ** 31]], dtype=np.int64).astype(np.int32)
        _, n = G.iodf_norm_forward(h, torch.from_numpy(r).cuda())
        np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), P.norm_step(d, r)[1])


def test_clips_of_the_residual_stream(G):
    rng = np.random.default_rng(3)
    for res, rg in ((torch.int16, (-100, 50)), (torch.int32, (0, 63)), (torch.int32, (7, 7))):
        check(G, rng, 40, 33, res, torch.int8, None, "rms", res_range=rg)
    # gates of 255 and the widest block values under the largest multiplier
    d = make_desc(rng, 16, torch.int32, torch.int32, None, None)
    d["post"]["mult"][:] = rng.choice([-2 ** 31 + 1, 2 ** 31 - 1], 16)
    d["post"]["shift"] = 1
    b = rng.choice([-2 ** 31, 2 ** 31 - 1, 2 ** 23, -2 ** 23], (9, 16)).astype(np.int32)
    r = rng.choice([-2 ** 31, 2 ** 31 - 1], (9, 16)).astype(np.int32)
    gate = np.full((9, 16), 255, np.uint8)
    o, _ = G.iodf_norm_forward(G.iodf_norm_create(d), torch.from_numpy(r).cuda(), torch.from_numpy(b).cuda(), torch.from_numpy(gate).cuda())
    np.testing.assert_array_equal(o.cpu().numpy().astype(np.int64), P.norm_step(d, r, b, gate)[0])


@pytest.mark.parametrize("C,px,images", [(1, 1, 1), (6, 1024, 2), (3, 17, 5), (24, 64, 3), (48, 100, 2), (96, 16, 9), (256, 33, 2)])
@pytest.mark.parametrize("post,pre", [(None, "rms"), ("rms", "centred"), ("centred", None)])
def test_planes(G, C, px, images, post, pre):
    """The residual stream as planes inside larger buffers, as the prior parameters of a level lie in theirs."""
    rng = np.random.default_rng(C * px)
    rows = images * px
    for block, res in ((torch.int8, torch.int32), (torch.int32, torch.int32), (torch.int32, torch.int16)):
        d = make_desc(rng, C, res, block, post, pre)
        h = G.iodf_norm_create(d)
        r, b = values(rng, rows, C, res, 500), values(rng, rows, C, block, 25)
        gate = rng.integers(0, 256, (rows, C)).astype(np.uint8)
        planes = lambda v: torch.from_numpy(np.ascontiguousarray(v.reshape(images, px, C).transpose(0, 2, 1)))
        buf = torch.full((images, 3, C * px + 5), 31, dtype=res, device="cuda")
        rt = buf[:, 1, 2:2 + C * px].unflatten(1, (C, px))
        rt.copy_(planes(r))
        o, n = G.iodf_norm_forward(h, rt, torch.from_numpy(b).cuda(), torch.from_numpy(gate).cuda(), r_out=rt)
        wo, wn = P.norm_step(d, r, b, gate)
        np.testing.assert_array_equal(rt.cpu().numpy().astype(np.int64), planes(wo).numpy())
        if pre:
            np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), wn)
        rest = buf.clone()
        rest[:, 1, 2:2 + C * px] = 31
        assert (rest == 31).all()                                     # nothing beside the planes
    if pre:                                                            # without a block, into rows with a stride
        d = make_desc(rng, C, torch.int32, None, None, pre)
        n = torch.full((rows, C + 11), 7, dtype=torch.int8, device="cuda")
        G.iodf_norm_forward(G.iodf_norm_create(d), planes(r.astype(np.int32)).cuda(), n=n[:, :C])
        np.testing.assert_array_equal(n[:, :C].cpu().numpy().astype(np.int64), P.norm_step(d, r)[1])
        assert (n[:, C:] == 7).all()


def test_planes_in_and_rows_out(G):
    rng = np.random.default_rng(20)
    images, px, C = 3, 40, 12
    d = make_desc(rng, C, torch.int32, torch.int8, "rms", "rms")
    r, b = values(rng, images * px, C, torch.int32, 500), values(rng, images * px, C, torch.int8, 25)
    h = G.iodf_norm_create(d)
    rt = torch.from_numpy(r).cuda().view(images, px, C)
    planes = rt.transpose(1, 2).contiguous()
    wo, wn = P.norm_step(d, r, b)
    import ctypes
    from paper_2206_08869_b200 import binding as B
    out, n = torch.empty((images * px, C), dtype=torch.int32, device="cuda"), torch.empty((images * px, C), dtype=torch.int8, device="cuda")
    bt = torch.from_numpy(b).cuda()
    rv, ov = B.View(px, C * px, px, 1), B.View(images * px, 0, 1, C)
    rc = G.load_library().iodf_norm_forward(h.handle, images * px, planes.data_ptr(), ctypes.byref(rv), bt.data_ptr(), C, None, 0,
                                            out.data_ptr(), ctypes.byref(ov), n.data_ptr(), C, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    np.testing.assert_array_equal(out.cpu().numpy().astype(np.int64), wo)
    np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), wn)
    back = torch.empty_like(planes)                                    # and rows in, planes out
    rc = G.load_library().iodf_norm_forward(h.handle, images * px, rt.data_ptr(), ctypes.byref(ov), bt.data_ptr(), C, None, 0,
                                            back.data_ptr(), ctypes.byref(rv), n.data_ptr(), C, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    np.testing.assert_array_equal(back.transpose(1, 2).reshape(-1, C).cpu().numpy().astype(np.int64), wo)
    np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), wn)


def test_captured_on_another_stream_and_twice_at_once(G):
    rng = np.random.default_rng(8)
    C, rows = 200, 900
    d = make_desc(rng, C, torch.int16, torch.int8, "rms", "rms")
    h = G.iodf_norm_create(d)
    r, b = values(rng, rows, C, torch.int16, 500), values(rng, rows, C, torch.int8, 25)
    rt, bt = torch.from_numpy(r).cuda(), torch.from_numpy(b).cuda()
    wo, wn = P.norm_step(d, r, b)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [G.iodf_norm_forward(h, rt, bt, r_out=torch.empty_like(rt), n=torch.empty_like(bt), stream=s) for s in streams for _ in range(4)]
    torch.cuda.synchronize()
    for o, n in outs:
        np.testing.assert_array_equal(o.cpu().numpy(), wo)
        np.testing.assert_array_equal(n.cpu().numpy(), wn)
    o, n = torch.empty_like(rt), torch.empty_like(bt)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        G.iodf_norm_forward(h, rt, bt, r_out=o, n=n)
    r2 = values(rng, rows, C, torch.int16, 100)
    rt.copy_(torch.from_numpy(r2))
    g.replay()
    wo, wn = P.norm_step(d, r2, b)
    np.testing.assert_array_equal(o.cpu().numpy(), wo)
    np.testing.assert_array_equal(n.cpu().numpy(), wn)


def test_refusals(G):
    rng = np.random.default_rng(0)
    h = G.iodf_norm_create(make_desc(rng, 12, torch.int16, torch.int8, "rms", "rms"))
    alone = G.iodf_norm_create(make_desc(rng, 12, torch.int16, None, None, "rms"))
    r, b = torch.zeros((5, 12), dtype=torch.int16, device="cuda"), torch.zeros((5, 12), dtype=torch.int8, device="cuda")
    for f in (lambda: G.iodf_norm_forward(h, r), lambda: G.iodf_norm_forward(alone, r, b), lambda: G.iodf_norm_forward(h, r.int(), b),
              lambda: G.iodf_norm_forward(h, r, b[:4]), lambda: G.iodf_norm_forward(h, r[:, :11], b), lambda: G.iodf_norm_forward(h, r, b.int()),
              lambda: G.iodf_norm_forward(h, r.cpu(), b), lambda: G.iodf_norm_forward(h, r, b, gate=b),
              lambda: G.iodf_norm_forward(h, r, b, gate=torch.zeros(11, dtype=torch.uint8, device="cuda")),
              lambda: G.iodf_norm_forward(h, r, b, n=torch.zeros((5, 12), dtype=torch.uint8, device="cuda")),
              lambda: G.iodf_norm_forward(h, r, b, r_out=torch.zeros((12, 5), dtype=torch.int16, device="cuda"))):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(G.IodfError) as e:                              # a gate without a block
        G.iodf_norm_forward(alone, r, gate=torch.zeros(12, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -1
    wide = G.iodf_norm_create(make_desc(rng, 257, torch.int32, None, None, "rms"))
    with pytest.raises(G.IodfError) as e:                              # more planes than the kernel takes
        G.iodf_norm_forward(wide, torch.zeros((2, 257, 4), dtype=torch.int32, device="cuda"))
    assert e.value.status == -1
    o, n = G.iodf_norm_forward(h, r[:0], b[:0])
    assert o.shape == (0, 12) and n.shape == (0, 12)


@pytest.mark.parametrize("C", [3, 40, 300, 2500])
def test_rows_of_images_with_gaps(G, C):
    """Channels side by side, images that do not follow each other: a view that only the C interface can name."""
    import ctypes
    from paper_2206_08869_b200 import binding as B
    rng = np.random.default_rng(C)
    images, px, pad = 3, 7, 5
    rows = images * px
    d = make_desc(rng, C, torch.int32, torch.int8, "rms", "centred")
    r, b = values(rng, rows, C, torch.int32, 500), values(rng, rows, C, torch.int8, 25)
    h = G.iodf_norm_create(d)
    step = C + 3
    buf = torch.full((images, px * step + pad), 17, dtype=torch.int32, device="cuda")
    view = buf[:, :px * step].unflatten(1, (px, step))[:, :, :C]
    view.copy_(torch.from_numpy(r).view(images, px, C))
    out, n = torch.full_like(buf, 17), torch.empty((rows, C), dtype=torch.int8, device="cuda")
    bt = torch.from_numpy(b).cuda()
    v = B.View(px, px * step + pad, 1, step)
    stream = torch.cuda.current_stream().cuda_stream
    f = lambda ov: G.load_library().iodf_norm_forward(h.handle, rows, buf.data_ptr(), v, bt.data_ptr(), C, None, 0, out.data_ptr(), ov,
                                                      n.data_ptr(), C, stream)
    assert f(v) == 0
    wo, wn = P.norm_step(d, r, b)
    got = out[:, :px * step].unflatten(1, (px, step))
    np.testing.assert_array_equal(got[:, :, :C].reshape(rows, C).cpu().numpy().astype(np.int64), wo)
    np.testing.assert_array_equal(n.cpu().numpy().astype(np.int64), wn)
    assert (got[:, :, C:] == 17).all() and (out[:, px * step:] == 17).all()
    # places that rows or images share are refused
    assert f(B.View(px, px * step + pad, 1, C - 1)) == -1
    assert f(B.View(px, step, 1, step)) == -1
    assert f(B.View(px, 0, 1, step)) == -1


def test_a_plane_layout_with_channels_outermost(G):
    rng = np.random.default_rng(2)
    images, C, px = 4, 10, 33
    d = make_desc(rng, C, torch.int32, torch.int8, "rms", None)
    r, b = values(rng, images * px, C, torch.int32, 500), values(rng, images * px, C, torch.int8, 25)
    t = torch.from_numpy(r).cuda().view(images, px, C).permute(2, 0, 1).contiguous().permute(1, 0, 2)     # [images, C, px], C outermost
    out = torch.empty_like(t.permute(1, 0, 2).contiguous()).permute(1, 0, 2)
    o, _ = G.iodf_norm_forward(G.iodf_norm_create(d), t, torch.from_numpy(b).cuda(), r_out=out)
    np.testing.assert_array_equal(o.permute(0, 2, 1).reshape(-1, C).cpu().numpy().astype(np.int64), P.norm_step(d, r, b)[0])
    with pytest.raises(G.IodfError):
        G.iodf_norm_forward(G.iodf_norm_create(d), t, torch.from_numpy(b).cuda(), r_out=out[:1].expand(images, C, px))


@pytest.mark.parametrize("rows,C", [(9000, 256), (700, 4096), (5000, 128), (3000, 512), (2000, 1024), (1200, 2048), (400, 8192), (6000, 64),
                                    (9000, 160), (1500, 136), (5000, 97), (4000, 225)])
def test_many_rows_of_every_form(G, rows, C):
    rng = np.random.default_rng(rows)
    check(G, rng, rows, C, torch.int16, torch.int32, "rms", "rms", "row")
    check(G, rng, rows // 3, C, torch.int32, torch.int8, "centred", "rms", "channel", n_dtype=torch.uint8)
