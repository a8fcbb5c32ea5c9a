"""What the single integer layers refuse, on the host and before any device is asked for."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2206_08869_b200 as G
from paper_2206_08869_b200 import binding as B

EINVAL, ECUDA, EVERSION, EUNSUPPORTED, EOVERFLOW = -1, -3, -4, -6, -7


def _layer(K=8, N=4, **kw):
    d = {"k": 1, "c_in": K, "c_out": N, "w": np.ones((N, K), np.int8), "bias": np.zeros(N, np.int32),
         "m0": np.full(N, 1 << 30, np.int32), "s": np.zeros(N, np.int32), "relu": False, "clamp": (-128, 127)}
    d.update(kw)
    return d


def _proj(layer, y=torch.int8, x=torch.int8, rows=4, adapters=0, rank=0):
    try:
        G.iodf_proj_create(layer, rows, adapters, rank, x_dtype=x, y_dtype=y)
    except G.IodfError as e:
        return e.status
    return 0


def _valid():
    return 0 if torch.cuda.is_available() else ECUDA


@pytest.mark.parametrize("case,want", [
    (dict(), None),
    (dict(layer=dict(k=3, w=np.ones((4, 72), np.int8))), EUNSUPPORTED),
    (dict(layer=dict(k=2)), EINVAL),
    (dict(layer=dict(m0=np.full(4, (1 << 30) - 1, np.int32))), EINVAL),
    (dict(layer=dict(s=np.full(4, 32, np.int32))), EINVAL),
    (dict(layer=dict(s=np.full(4, -1, np.int32))), EINVAL),
    (dict(layer=dict(clamp=(5, 4))), EINVAL),
    (dict(layer=dict(clamp=None)), EINVAL),                         # int8 out needs a clip inside its range
    (dict(layer=dict(clamp=(-129, 127))), EINVAL),
    (dict(layer=dict(clamp=(0, 255))), EINVAL),
    (dict(layer=dict(clamp=(0, 255)), y=torch.uint8), None),
    (dict(layer=dict(clamp=(-4, 255), relu=True), y=torch.uint8), None),
    (dict(layer=dict(clamp=(-4, 255)), y=torch.uint8), EINVAL),
    (dict(layer=dict(clamp=None), y=torch.int32), None),
    (dict(layer=dict(bias=np.full(4, 2 ** 31 - 1, np.int32))), EOVERFLOW),
    (dict(layer=dict(bias=np.full(4, 2 ** 31 - 1 - 8 * 128, np.int32))), None),
    (dict(layer=dict(bias=np.full(4, 2 ** 31 - 1 - 8 * 128, np.int32)), x=torch.uint8), EOVERFLOW),
    (dict(rows=0), EINVAL),
    (dict(adapters=1, rank=0), EINVAL),
    (dict(adapters=1, rank=129), EINVAL),
    (dict(adapters=65537, rank=1), EINVAL),
])
def test_projection_descriptors(case, want):
    case = dict(case)
    assert _proj(_layer(**case.pop("layer", {})), **case) == (_valid() if want is None else want)


def test_projection_blobs_and_versions():
    L = G.load_library()
    w, par = np.ones(32, np.int8), np.zeros(12, np.int32)
    par[4:8] = 1 << 30
    out = C.c_void_p()

    def create(version=B.IODF_ABI_VERSION, woff=0, roff=0, nw=32, nr=12, c_in=8, xt=1, yt=4):
        d = B.ProjDesc(version, B.LayerDesc(1, c_in, 4, 0, 0, 0, 0, woff, roff), xt, yt, 4, 0, 0)
        return L.iodf_proj_create(C.byref(d), w.ctypes.data, nw, par.ctypes.data, nr, 0, C.byref(out))

    assert create(version=2) == EVERSION
    assert create(woff=1) == EINVAL and create(nw=31) == EINVAL
    assert create(roff=1) == EINVAL and create(nr=11) == EINVAL
    assert create(woff=2 ** 64 - 1) == EINVAL
    assert create(c_in=0) == EINVAL and create(c_in=32769) == EUNSUPPORTED
    assert create(xt=3) == EINVAL and create(yt=3) == EINVAL
    assert L.iodf_proj_create(None, w.ctypes.data, 32, par.ctypes.data, 12, 0, C.byref(out)) == EINVAL
    assert L.iodf_proj_forward(None, None, 16, 0, None, None, 0, None, 8, None) == EINVAL
    assert L.iodf_proj_set_adapter(None, 0, 0, None, None, None, None) == EINVAL
    assert L.iodf_proj_check(None, None, None) == EINVAL
    L.iodf_proj_destroy(None)


def _desc(**kw):
    one = np.full(4, 1 << 30, np.int32)
    d = {"c": 4, "res_dtype": torch.int16, "block_dtype": torch.int8, "eps": 1, "res_range": (-32768, 32767),
         "post": {"norm": "rms", "mult": one, "shift": 8},
         "pre": {"norm": "rms", "mult": one, "shift": 8, "bias": np.zeros(4, np.int32), "clamp": (-128, 127), "dtype": torch.int8}}
    for k, v in kw.items():
        if isinstance(v, dict):
            d[k] = dict(d[k], **v)
        else:
            d[k] = v
    return d


@pytest.mark.parametrize("kw,want", [
    (dict(), None),
    (dict(eps=0), EINVAL),
    (dict(eps=2 ** 60), None),
    (dict(eps=2 ** 60 + 1), EINVAL),
    (dict(post={"shift": 0}), EINVAL),
    (dict(post={"shift": 32}), EINVAL),
    (dict(post={"mult": np.array([1, 2, -2 ** 31, 4], np.int64).astype(np.int32)}), EINVAL),
    (dict(post={"mult": np.array([0, -2 ** 31 + 1, 2 ** 31 - 1, 4], np.int64).astype(np.int32)}), None),
    (dict(pre={"shift": 0}), EINVAL),
    (dict(pre={"bias": np.full(4, 1 << 30, np.int32)}), EINVAL),
    (dict(pre={"clamp": (-129, 0)}), EINVAL),
    (dict(pre={"clamp": (1, 0)}), EINVAL),
    (dict(pre={"clamp": (0, 255)}), EINVAL),
    (dict(pre={"clamp": (0, 255), "dtype": torch.uint8}), None),
    (dict(pre={"clamp": (-1, 255), "dtype": torch.uint8}), EINVAL),
    (dict(res_range=(-32769, 0)), EINVAL),
    (dict(res_range=(0, 32768)), EINVAL),
    (dict(res_range=(3, 2)), EINVAL),
    (dict(res_dtype=torch.int32, res_range=(-2 ** 23, 2 ** 23 - 1)), None),
    (dict(res_dtype=torch.int32, res_range=(0, 2 ** 23)), EINVAL),
    (dict(block_dtype=None, post=None), None),
    (dict(block_dtype=None), EINVAL),                               # a norm of no block
    (dict(block_dtype=None, post=None, pre=None), EINVAL),          # nothing to do
    (dict(pre=None), None),
    (dict(post=None), EINVAL),                                      # a block without its scale
])
def test_norm_descriptors(kw, want):
    try:
        G.iodf_norm_create(_desc(**kw))
        got = 0
    except G.IodfError as e:
        got = e.status
    assert got == (_valid() if want is None else want)


def test_norm_versions_sizes_and_null_pointers():
    L = G.load_library()
    out = C.c_void_p()
    one = np.full(9000, 1 << 30, np.int32)

    def create(version=B.IODF_ABI_VERSION, channels=4, res=4, block=1, post=1, pre=0, mult=one.ctypes.data):
        d = B.NormDesc(version, channels, res, block, post, pre, 0, 1, 1, 0, 0, 0, 0, 1, mult, None, None)
        return L.iodf_norm_create(C.byref(d), 0, C.byref(out))

    assert create(version=1) == EVERSION
    assert create(channels=0) == EINVAL and create(channels=8193) == EUNSUPPORTED
    assert create(res=1) == EINVAL and create(block=2) == EINVAL and create(post=3) == EINVAL
    assert create(mult=None) == EINVAL and create(pre=1) == EINVAL
    assert L.iodf_norm_create(None, 0, C.byref(out)) == EINVAL
    assert L.iodf_norm_forward(None, 0, None, None, None, 0, None, 0, None, None, None, 0, None) == EINVAL
    L.iodf_norm_destroy(None)


def test_wrong_element_types_are_named():
    with pytest.raises(ValueError):
        G.iodf_proj_create(_layer(), 4, x_dtype=torch.int32)
    with pytest.raises(ValueError):
        G.iodf_proj_create(_layer(), 4, y_dtype=torch.float32)
    with pytest.raises(ValueError):
        G.iodf_norm_create(_desc(res_dtype=torch.int8))
    with pytest.raises(ValueError):
        G.iodf_proj_create(_layer(gate=np.ones(4, np.uint8)), 4)
