"""Projections whose x and y lie in one buffer."""
import numpy as np
import pytest
import torch

from oracle import layers as P
from test_gpu_proj import make_layer, make_x

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


def _refused(G, *a, **k):
    with pytest.raises(G.IodfError) as e:
        G.iodf_proj_forward(*a, **k)
    assert e.value.status == -1


@pytest.mark.parametrize("y_dtype", [torch.int8, torch.int32])
@pytest.mark.parametrize("rows", [1, 40, 700])
def test_columns_of_one_matrix(G, rows, y_dtype):
    rng = np.random.default_rng(rows)
    K, N = 64, 48
    layer = make_layer(rng, K, N, y_dtype)
    h = G.iodf_proj_create(layer, rows, y_dtype=y_dtype)
    size = y_dtype.itemsize
    for x_at, y_at in ((0, 64), (256, 64), (64 + 48 * size, 64), (0, 64 + 16)):
        buf = torch.full((rows, 512), 9, dtype=torch.int8, device="cuda")
        x_at = (x_at + 15) // 16 * 16
        xh, x = make_x(rng, rows, K, torch.int8)
        buf[:, x_at:x_at + K] = x
        xs, ys = buf[:, x_at:x_at + K], buf.view(y_dtype)[:, y_at // size:y_at // size + N]
        G.iodf_proj_forward(h, xs, y=ys)
        np.testing.assert_array_equal(ys.cpu().numpy().astype(np.int64), P.projection(layer, xh))
        np.testing.assert_array_equal(xs.cpu().numpy(), xh)
    for x_at, y_at in ((0, 0), (0, 48), (64, 64 - 48 * size + 16 if size == 1 else 16), (0, 60 // size * size)):
        buf = torch.full((rows, 512), 9, dtype=torch.int8, device="cuda")
        _refused(G, h, buf[:, x_at:x_at + K], y=buf.view(y_dtype)[:, y_at // size:y_at // size + N])
        assert (buf == 9).all()


def test_the_same_rows_and_rows_at_another_stride(G):
    rng = np.random.default_rng(3)
    rows, K = 200, 64
    h = G.iodf_proj_create(make_layer(rng, K, K, torch.int8), rows, y_dtype=torch.int8)
    flat = torch.full((rows * 128 + 64,), 5, dtype=torch.int8, device="cuda")
    x = flat[:rows * K].view(rows, K)
    _refused(G, h, x, y=x)
    _refused(G, h, x, y=flat[:rows * 128].view(rows, 128)[:, 64:])
    _refused(G, h, x, y=flat[rows * K - 1:2 * rows * K - 1].view(rows, K))          # the last row's last channel
    _refused(G, h, flat[64:64 + rows * K].view(rows, K), y=flat[1:1 + rows * K].view(rows, K))
    assert (flat == 5).all()
    G.iodf_proj_forward(h, x, y=flat[rows * K:2 * rows * K].view(rows, K))          # side by side
    G.iodf_proj_forward(h, flat[rows * K:2 * rows * K].view(rows, K), y=x)
