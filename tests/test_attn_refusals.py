"""What integer attention refuses, on the host and before any device is asked for."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2206_08869_b200 as G
from paper_2206_08869_b200 import binding as B
from tests import attn_cases

EINVAL, ECUDA, EVERSION, EUNSUPPORTED = -1, -3, -4, -6


def _create(**kw):
    d = attn_cases.description(torch, heads=4, kv=2, dim=32, rot=16, positions=8)
    d["out"].update(kw.pop("out", {}))
    if "rotary" in kw and isinstance(kw["rotary"], dict):
        d["rotary"] = {**d["rotary"], **kw.pop("rotary")}
    d.update(kw)
    n = d["heads"] * d["head_dim"]
    if len(d["out"]["m0"]) == 128 and n != 128:
        d["out"].update(m0=np.full(n, 1 << 30, np.int32), s=np.zeros(n, np.int32))
    try:
        G.iodf_attn_create(d)
    except G.IodfError as e:
        return e.status
    return 0


def _valid():
    return 0 if torch.cuda.is_available() else ECUDA


def _out(n, m0=1 << 30, s=0):
    return {"m0": np.full(n, m0, np.int32), "s": np.full(n, s, np.int32)}


@pytest.mark.parametrize("case,want", [
    (dict(), None),
    (dict(rotary=None), None),
    (dict(heads=0), EINVAL),
    (dict(kv_heads=0), EINVAL),
    (dict(kv_heads=3), EINVAL),                                     # no whole number of heads for each
    (dict(heads=258), EUNSUPPORTED),                                # 129 for each
    (dict(heads=2048, kv_heads=2048), EUNSUPPORTED),
    (dict(head_dim=48), EUNSUPPORTED),
    (dict(head_dim=256), EUNSUPPORTED),
    (dict(x_dtype=torch.int32), None),
    (dict(headroom=(8, 8)), None),
    (dict(headroom=(9, 0)), EINVAL),
    (dict(headroom=(0, 9)), EINVAL),
    (dict(score=((1 << 30) - 1, 4)), EINVAL),
    (dict(score=(1 << 30, -1)), EINVAL),
    (dict(score=(1 << 30, 62)), None),
    (dict(score=(1 << 30, 63)), EINVAL),
    (dict(window=1 << 30), None),
    (dict(window=(1 << 30) + 1), EINVAL),
    (dict(out=dict(clamp=None)), EINVAL),                           # 8-bit outputs need a clip inside their range
    (dict(out=dict(clamp=(-129, 127))), EINVAL),
    (dict(out=dict(clamp=(5, 4))), EINVAL),
    (dict(out=dict(clamp=(0, 255), dtype=torch.uint8)), None),
    (dict(out=dict(clamp=(-1, 255), dtype=torch.uint8)), EINVAL),
    (dict(out=dict(clamp=None, dtype=torch.int32)), None),
    (dict(out=_out(128, m0=(1 << 30) - 1)), EINVAL),
    (dict(out=_out(128, s=32)), EINVAL),
    (dict(out=_out(128, s=-1)), EINVAL),
    (dict(rotary=dict(dim=8, table=np.zeros((8, 4, 2), np.int16))), EUNSUPPORTED),
    (dict(rotary=dict(dim=48, table=np.zeros((8, 24, 2), np.int16))), EINVAL),        # more than the head has
    (dict(rotary=dict(dim=16, table=np.full((8, 8, 2), 16385, np.int16))), EINVAL),
    (dict(rotary=dict(dim=16, table=np.full((8, 8, 2), -16384, np.int16), layout="interleaved")), None),
    (dict(rotary=dict(dim=16, table=np.zeros((0, 8, 2), np.int16))), EINVAL),
])
def test_descriptors(case, want):
    assert _create(**case) == (_valid() if want is None else want)


def test_python_arguments():
    for bad in (dict(x_dtype=torch.uint8), dict(x_dtype=torch.int16), dict(out=dict(dtype=torch.int16)), dict(window=-1), dict(heads=-1),
                dict(score=(1 << 31, 0)), dict(out=dict(m0=np.full(3, 1 << 30))), dict(rotary=dict(table=np.zeros((8, 7, 2), np.int16))),
                dict(rotary=dict(table=np.full((8, 8, 2), 40000)))):
        with pytest.raises(ValueError):
            _create(**bad)
    with pytest.raises(KeyError):
        _create(rotary=dict(layout="other"))


def test_versions_and_null_handles():
    L = G.load_library()
    out, d = C.c_void_p(), B.AttnDesc()
    assert L.iodf_attn_create(None, 0, C.byref(out)) == EINVAL
    assert L.iodf_attn_create(C.byref(d), 0, None) == EINVAL
    assert L.iodf_attn_create(C.byref(d), 0, C.byref(out)) == EVERSION and not out.value
    L.iodf_attn_destroy(None)
    cache = B.AttnCacheDesc()
    assert L.iodf_attn_plan(None, 0, None, None, None, 1, 1, None, 1, None, 0, None, None, None, None, None, None) == EINVAL
    assert L.iodf_attn_append(None, 0, None, 1, None, 1, None, 1, None, None, C.byref(cache), None, None, None) == EINVAL
    assert L.iodf_attn_forward(None, 0, None, None, None, None, 0, None, 1, 1, C.byref(cache), None, 1, None) == EINVAL
    assert L.iodf_attn_check(None, None, None) == EINVAL
