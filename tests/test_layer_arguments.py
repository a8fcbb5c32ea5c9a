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


WRAP = 2 ** 32


def _layer(K=8, N=4, **kw):
    return {"k": 1, "c_in": K, "c_out": N, "w": np.ones((N, K), np.int8), "bias": np.zeros(N, np.int32), "m0": np.full(N, 1 << 30, np.int32),
            "s": np.zeros(N, np.int32), "relu": False, "clamp": (-128, 127), **kw}


def _desc(**kw):
    one = np.full(4, 1 << 30, np.int32)
    d = {"c": 4, "res_dtype": torch.int16, "block_dtype": torch.int8, "eps": 1, "res_range": (-32768, 32767),
         "post": {"norm": "rms", "mult": one, "shift": 8},
         "pre": {"norm": "rms", "mult": one, "shift": 8, "bias": np.zeros(4, np.int32), "clamp": (-128, 127), "dtype": torch.int8}}
    return {k: dict(v, **kw[k]) if isinstance(kw.get(k), dict) else kw.get(k, v) for k, v in d.items()}


def _wrapped(n, value=5 + WRAP):
    a = np.ones(n, np.int64)
    a[-1] = value
    return a


def test_numbers_that_the_librarys_types_do_not_hold():
    codec, p = _codec(), _projection()
    norm = B.Norm(None, 0, 12, torch.int16, None, torch.int8)
    ad = {"rank": 2, "down": np.ones((2, 64), np.int8), "m0": np.full(2, 1 << 30), "s": np.zeros(2, int), "up": np.ones((48, 2), np.int8)}
    fine = [lambda: G.iodf_proj_create(_layer(), 4), lambda: G.iodf_proj_create(_layer(w=np.ones((4, 8), np.int64), clamp=(-2 ** 31, 2 ** 31 - 1)), 4),
            lambda: G.iodf_norm_create(_desc()), lambda: G.iodf_proj_set_adapter(p, 0, ad), lambda: G.iodf_proj_set_adapter(p, 0, None),
            lambda: G.iodf_norm_create(_desc(eps=2 ** 64 - 1)),
            lambda: G.iodf_norm_forward(norm, Tensor((2 ** 31 - 1, 12), torch.int16), n=Tensor((2 ** 31 - 1, 12), torch.int8)),
            lambda: G.iodf_proj_forward(p, Tensor((2 ** 31 - 1, 64), torch.int8), y=Tensor((2 ** 31 - 1, 48), torch.int8))]
    for f in fine:
        with pytest.raises(Called):
            f()
    bad = [lambda: G.iodf_proj_create(_layer(), 4 + WRAP), lambda: G.iodf_proj_create(_layer(), -1), lambda: G.iodf_proj_create(_layer(), 4, WRAP, 1),
           lambda: G.iodf_proj_create(_layer(), 4, 1, 1 + WRAP), lambda: G.iodf_proj_create(_layer(), 4, device=WRAP),
           lambda: G.iodf_proj_create(_layer(clamp=(-128 - WRAP, 127)), 4), lambda: G.iodf_proj_create(_layer(clamp=(0, 127 + WRAP)), 4),
           lambda: G.iodf_proj_create(_layer(w=np.full((4, 8), 129)), 4), lambda: G.iodf_proj_create(_layer(bias=_wrapped(4)), 4),
           lambda: G.iodf_proj_create(_layer(m0=_wrapped(4, (1 << 30) + WRAP)), 4), lambda: G.iodf_proj_create(_layer(s=[0, 0, 0, 0.5]), 4),
           lambda: G.iodf_proj_create(_layer(bias=np.zeros(5, np.int32)), 4), lambda: G.iodf_proj_create(_layer(w=np.ones((4, 9), np.int8)), 4),
           lambda: G.iodf_proj_create(_layer(c_in=8 + WRAP), 4),
           lambda: G.iodf_proj_set_adapter(p, WRAP, ad), lambda: G.iodf_proj_set_adapter(p, -1, ad),
           lambda: G.iodf_proj_set_adapter(p, 0, dict(ad, up=np.full((48, 2), 200))), lambda: G.iodf_proj_set_adapter(p, 0, dict(ad, m0=_wrapped(2))),
           lambda: G.iodf_proj_set_adapter(p, 0, dict(ad, m0=np.full(3, 1 << 30), s=np.zeros(1, int))),
           lambda: G.iodf_norm_create(_desc(eps=1 + 2 ** 64)), lambda: G.iodf_norm_create(_desc(eps=-1)), lambda: G.iodf_norm_create(_desc(c=4 + WRAP)),
           lambda: G.iodf_norm_create(_desc(res_range=(-WRAP, 5))), lambda: G.iodf_norm_create(_desc(post={"shift": 8 + WRAP})),
           lambda: G.iodf_norm_create(_desc(pre={"clamp": (-128, 127 + WRAP)})), lambda: G.iodf_norm_create(_desc(post={"mult": _wrapped(4)})),
           lambda: G.iodf_norm_create(_desc(pre={"bias": _wrapped(4)})), lambda: G.iodf_norm_create(_desc(), device=WRAP),
           lambda: G.iodf_norm_forward(norm, Tensor((WRAP + 5, 12), torch.int16), n=Tensor((WRAP + 5, 12), torch.int8)),
           lambda: G.iodf_proj_forward(p, Tensor((WRAP + 5, 64), torch.int8), y=Tensor((WRAP + 5, 48), torch.int8)),
           lambda: G.iodf_proj_forward(p, Tensor((5, 64), torch.int8), Tensor((WRAP + 2,), torch.int32), Tensor((WRAP + 1,), torch.int32),
                                       y=Tensor((5, 48), torch.int8)),
           lambda: G.iodf_codec_set_refinement(codec, WRAP), lambda: G.iodf_codec_selftest_timeout(codec, 0, 3 + WRAP),
           lambda: G.iodf_refine_prior(codec, WRAP, Tensor((4, 2, 200), torch.int32, 1)),
           lambda: G.iodf_refine_prior(codec, 0, Tensor((WRAP + 4, 2, 200), torch.int32, 1))]
    for i, f in enumerate(bad):
        try:
            with pytest.raises(ValueError):
                f()
        except Called:
            pytest.fail("case %d was not refused" % i)
