"""Single integer layers at the ends of what their calls allow: offsets beyond 32 bits, the last adapter slot, handles without adapters."""
import numpy as np
import pytest
import torch

from oracle import layers as P
from test_gpu_norm import make_desc
from test_gpu_proj import make_adapter, make_layer, make_x, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


@pytest.mark.parametrize("K,N,y_dtype", [(64, 48, torch.int8), (64, 48, torch.int32), (1300, 140, torch.int8)])
def test_a_projections_rows_beyond_four_gigabytes(G, K, N, y_dtype):
    rng = np.random.default_rng(K)
    rows, ld = 70001, 65536
    h = G.iodf_proj_create(make_layer(rng, K, N, y_dtype), rows, 2, 16, y_dtype=y_dtype)
    for i in range(2):
        G.iodf_proj_set_adapter(h, i, make_adapter(rng, K, N, 16))
    x = torch.randint(-128, 128, (rows, (K + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :K]
    st = torch.tensor([1, 100, 69000, rows - 1], dtype=torch.int32, device="cuda")
    wh = torch.tensor([0, -1, 1], dtype=torch.int32, device="cuda")
    want = G.iodf_proj_forward(h, x, st, wh)
    far_x = torch.empty((rows, ld), dtype=torch.int8, device="cuda")[:, :K]
    far_x.copy_(x)
    far_y = torch.zeros((rows, ld), dtype=y_dtype, device="cuda")
    G.iodf_proj_forward(h, far_x, st, wh, y=far_y[:, 100:100 + N])
    G.iodf_proj_check(h)
    assert torch.equal(far_y[:, 100:100 + N], want)
    assert not far_y[-1].any() and not far_y[:, :100].any() and not far_y[:, 100 + N:].any()


@pytest.mark.parametrize("C,odd", [(64, 0), (173, 1)])
def test_a_norms_rows_beyond_four_gigabytes(G, C, odd):
    rng = np.random.default_rng(C)
    rows, ld = 70001, 65536
    h = G.iodf_norm_create(make_desc(rng, C, torch.int16, torch.int8, "rms", "centred"))
    r = torch.randint(-900, 900, (rows, C), dtype=torch.int16, device="cuda")
    b = torch.randint(-90, 90, (rows, C), dtype=torch.int8, device="cuda")
    gate = torch.randint(0, 256, (rows, C), dtype=torch.int32, device="cuda").to(torch.uint8)
    want = G.iodf_norm_forward(h, r, b, gate)
    far = lambda t: torch.empty((rows, ld), dtype=t.dtype, device="cuda")[:, odd:odd + C].copy_(t)
    o, n = G.iodf_norm_forward(h, far(r), far(b), far(gate), r_out=far(r), n=far(b))
    assert torch.equal(o, want[0]) and torch.equal(n, want[1])


def test_a_norms_planes_beyond_four_gigabytes(G):
    rng = np.random.default_rng(2)
    images, C, px, ld = 300, 12, 64, 1 << 24
    h = G.iodf_norm_create(make_desc(rng, C, torch.int16, torch.int8, "rms", "rms"))
    r = torch.randint(-900, 900, (images, C, px), dtype=torch.int16, device="cuda")
    b = torch.randint(-90, 90, (images * px, C), dtype=torch.int8, device="cuda")
    want = G.iodf_norm_forward(h, r, b)
    far = torch.empty(images * ld, dtype=torch.int16, device="cuda")
    t = far.as_strided((images, C, px), (ld, 1 << 20, 1), 5)
    t.copy_(r)
    o, n = G.iodf_norm_forward(h, t, b, r_out=t)
    assert torch.equal(o, want[0]) and torch.equal(n, want[1])


@pytest.mark.parametrize("rows,K", [(1, 64), (40, 64), (900, 64), (3000, 1300)])
def test_the_last_slot_of_many(G, rows, K):
    rng = np.random.default_rng(rows)
    N, slots = 32, 65536 if K == 64 else 2000
    layer, ad = make_layer(rng, K, N, torch.int8), make_adapter(rng, K, N, 5)
    h = G.iodf_proj_create(layer, rows, slots, 5, y_dtype=torch.int8)
    G.iodf_proj_set_adapter(h, slots - 1, ad)
    xh, x = make_x(rng, rows, K, torch.int8)
    cut = rows // 2
    st = torch.tensor([0, cut, rows], dtype=torch.int32, device="cuda")
    for a in (slots - 1, 0, slots - 2):
        y = G.iodf_proj_forward(h, x, st, torch.tensor([-1, a], dtype=torch.int32, device="cuda"))
        G.iodf_proj_check(h)
        ads = {-1: None, a: ad if a == slots - 1 else None}
        np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh, ads, [0, cut, rows], [-1, a]))
    G.iodf_proj_forward(h, x, st, torch.tensor([0, slots], dtype=torch.int32, device="cuda"))
    with pytest.raises(G.IodfError) as e:
        G.iodf_proj_check(h)
    assert e.value.status == -9


@pytest.mark.parametrize("rows,K,N", [(1, 64, 40), (33, 300, 130), (900, 96, 72), (9000, 96, 72), (3000, 1300, 300)])
def test_requests_of_a_handle_without_adapters(G, rows, K, N):
    """Which rows are computed is then all that they say; any slot but -1 is bad."""
    rng = np.random.default_rng(rows)
    starts = [0, 0, rows // 3, rows - rows // 9]
    run(G, rng, rows, K, N, [], starts, [-1, -1, -1])
    layer = make_layer(rng, K, N, torch.int8)
    h = G.iodf_proj_create(layer, rows, y_dtype=torch.int8)
    xh, x = make_x(rng, rows, K, torch.int8)
    y = G.iodf_proj_forward(h, x, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    with pytest.raises(G.IodfError) as e:
        G.iodf_proj_check(h)
    assert e.value.status == -9
    np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh))


def test_a_layer_at_the_most_channels(G):
    rng = np.random.default_rng(5)
    run(G, rng, 3, 32768, 130, [16], [0, 3], [0])
    run(G, rng, 300, 32768, 130, [16], [0, 290], [0])
    run(G, rng, 3, 40, 32768, [16], [0, 3], [0])
    run(G, rng, 700, 40, 32768, [16, 9], [0, 300, 700], [1, 0])
