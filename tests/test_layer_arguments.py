"""What the binding of the single integer layers refuses before the library is called: tensors that stand for a GPU's, no device needed."""
import numpy as np
import pytest
import torch

import paper_2206_08869_b200 as G
from paper_2206_08869_b200 import binding as B


class Called(Exception):
    pass


@pytest.fixture(autouse=True)
def library(monkeypatch):
    """Every entry point raises: whoever gets there has not been refused."""
    class Library:
        def __getattr__(self, name):
            def f(*a):
                raise Called(name)
            return f
    monkeypatch.setattr(B, "load_library", lambda path=None: Library())
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(B, "_layer_stream", lambda stream, device: 0)


class Tensor:
    """Shape, type, strides and place of a tensor; no memory behind them."""
    def __init__(self, shape, dtype, device=0, strides=None):
        self.shape, self.dtype, self.device, self.place = torch.Size(shape), dtype, "cuda:%d" % device, device
        self.strides = strides or tuple(int(np.prod(shape[i + 1:], dtype=object)) for i in range(len(shape)))

    def get_device(self):
        return self.place

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape, dtype=object))

    def is_contiguous(self):
        return self.strides == Tensor(self.shape, None).strides

    def data_ptr(self):
        return 1 << 40


def _codec():
    model = B.Model(None, type("Layout", (), {"d": 300, "d_fact": 200})(), (3, 10, 10), 4)
    model.device = 1
    return B.Codec(None, type("Layout", (), {"n_blocks": 1, "n_streams": 1, "words_per_stream": 1})(), model)


def test_refine_prior_takes_the_codecs_prior_buffer_only():
    codec = _codec()
    good = lambda **k: Tensor(**{**dict(shape=(4, 2, 200), dtype=torch.int32, device=1), **k})
    with pytest.raises(Called):
        G.iodf_refine_prior(codec, 0, good())
    for bad in (good(device=0), good(device=-1), good(dtype=torch.int16), good(dtype=torch.float32), good(dtype=torch.int64), good(shape=(4, 200)),
                good(shape=(4, 2, 100)), good(shape=(4, 2, 400)), good(shape=(4, 1, 200)), good(shape=(800,)), good(shape=(4, 2, 10, 20)),
                good(strides=(800, 200, 1)), good(strides=(400, 1, 2)), good(strides=(0, 200, 1)), torch.zeros((4, 2, 200), dtype=torch.int32)):
        with pytest.raises(ValueError):
            G.iodf_refine_prior(codec, 0, bad)


def _projection(c_in=64, c_out=48, max_rows=100):
    return B.Projection(None, 0, c_in, c_out, max_rows, torch.int8, torch.int8)


def test_the_rows_of_requests_need_their_adapters_and_the_adapters_their_rows():
    p, x, y = _projection(), Tensor((9, 64), torch.int8), Tensor((9, 48), torch.int8)
    start, which = Tensor((4,), torch.int32), Tensor((3,), torch.int32)
    with pytest.raises(Called):
        G.iodf_proj_forward(p, x, start, which, y=y)
    with pytest.raises(Called):
        G.iodf_proj_forward(p, x, y=y)
    for k in (dict(seg_start=start), dict(seg_adapter=which)):
        with pytest.raises(ValueError):
            G.iodf_proj_forward(p, x, y=y, **k)


def test_no_requests_left_own_no_rows(monkeypatch):
    p, x, y = _projection(), Tensor((9, 64), torch.int8), Tensor((9, 48), torch.int8)
    none = Tensor((1,), torch.int32), Tensor((0,), torch.int32)
    assert G.iodf_proj_forward(p, x, *none, y=y) is y
    made = []
    monkeypatch.setattr(B, "_made", lambda make, shape, dtype, device, stream: made.append(make) or Tensor(shape, dtype))
    G.iodf_proj_forward(p, x, *none)
    assert made == [torch.zeros]
    with pytest.raises(ValueError):
        G.iodf_proj_forward(p, x, *none, y=Tensor((8, 48), torch.int8))
    with pytest.raises(ValueError):
        G.iodf_proj_forward(p, x, Tensor((0,), torch.int32), none[1], y=y)
