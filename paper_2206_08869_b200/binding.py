"""ctypes binding of include/iodf.h. Argument marshalling only: model dicts (numpy arrays) become
the C descriptor structs, torch tensors become device pointers, the current torch stream becomes
the cudaStream_t. The function names are those of the C ABI."""
import ctypes as C
import os

import numpy as np

from . import build as _build

IODF_ABI_VERSION = 3
IODF_PLAN_LATENCY, IODF_PLAN_THROUGHPUT = 0, 1
IODF_MAX_LEVELS = 8

DECLARED_SYMBOLS = ["iodf_create", "iodf_destroy", "iodf_get_layout", "iodf_forward", "iodf_inverse",
                    "iodf_inverse_level", "iodf_forward_patches", "iodf_inverse_patches",
                    "iodf_codec_create", "iodf_codec_destroy", "iodf_codec_get_layout", "iodf_rans_encode",
                    "iodf_rans_decode_block", "iodf_codec_check", "iodf_rans_packed_capacity", "iodf_rans_pack",
                    "iodf_rans_unpack", "iodf_compress_host", "iodf_decompress_host",
                    "iodf_forward_host", "iodf_inverse_host", "iodf_forward_timed", "iodf_inverse_timed", "iodf_forward_static",
                    "iodf_static_scratch_bytes_per_image", "iodf_check", "iodf_launches_per_call",
                    "iodf_selftest_timeout", "iodf_int8_mma_peak", "iodf_level_kernel_name",
                    "iodf_level_images_per_cta",
                    "iodf_proj_create", "iodf_proj_destroy", "iodf_proj_set_adapter", "iodf_proj_forward",
                    "iodf_proj_check", "iodf_norm_create", "iodf_norm_destroy", "iodf_norm_forward",
                    "iodf_codec_set_refinement", "iodf_refine_prior", "iodf_codec_selftest_timeout",
                    "iodf_strerror", "iodf_last_cuda_error"]


class LayerDesc(C.Structure):
    _fields_ = [("k", C.c_uint32), ("c_in", C.c_uint32), ("c_out", C.c_uint32), ("relu", C.c_uint32),
                ("has_clamp", C.c_uint32), ("clamp_lo", C.c_int32), ("clamp_hi", C.c_int32),
                ("weight_off", C.c_uint64), ("requant_off", C.c_uint64)]


class ResBlockDesc(C.Structure):
    _fields_ = [("short_m0", C.c_int32), ("short_s", C.c_int32), ("clamp_lo", C.c_int32), ("clamp_hi", C.c_int32),
                ("n_idx", C.c_uint32), ("idx", C.POINTER(C.c_int32))]


class CouplingDesc(C.Structure):
    _fields_ = [("perm", C.POINTER(C.c_int32)), ("in_m0", C.c_int32), ("in_s", C.c_int32),
                ("n_layers", C.c_uint32), ("layers", C.POINTER(LayerDesc)),
                ("n_blocks", C.c_uint32), ("blocks", C.POINTER(ResBlockDesc))]


class LevelDesc(C.Structure):
    _fields_ = [("n_couplings", C.c_uint32), ("couplings", C.POINTER(CouplingDesc)), ("split", C.c_uint32),
                ("has_prior", C.c_uint32), ("prior_in_m0", C.c_int32), ("prior_in_s", C.c_int32),
                ("prior_layer", LayerDesc), ("ls_lo", C.c_int32), ("ls_hi", C.c_int32)]


class ModelDesc(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("in_c", C.c_uint32), ("in_h", C.c_uint32), ("in_w", C.c_uint32),
                ("n_levels", C.c_uint32), ("max_batch", C.c_uint32), ("levels", C.POINTER(LevelDesc)),
                ("plan", C.c_uint32)]


class Layout(C.Structure):
    _fields_ = [("d", C.c_uint64), ("d_fact", C.c_uint64), ("n_levels", C.c_uint32),
                ("level_c", C.c_uint32 * IODF_MAX_LEVELS), ("level_h", C.c_uint32 * IODF_MAX_LEVELS),
                ("level_w", C.c_uint32 * IODF_MAX_LEVELS), ("z_off", C.c_uint64 * IODF_MAX_LEVELS),
                ("prior_off", C.c_uint64 * IODF_MAX_LEVELS), ("z_final_off", C.c_uint64),
                ("macs_per_image", C.c_uint64)]


class CodecDesc(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("sigmoid_table", C.c_void_p), ("umax", C.c_uint32),
                ("inv_scale", C.c_void_p), ("n_scales", C.c_uint32), ("final_ls", C.c_int32),
                ("elems_per_stream", C.c_uint32)]


class CodecLayout(C.Structure):
    _fields_ = [("n_blocks", C.c_uint32), ("n_streams", C.c_uint32), ("words_per_stream", C.c_uint32),
                ("block_level", C.c_int32 * (IODF_MAX_LEVELS + 1)), ("block_z_off", C.c_uint64 * (IODF_MAX_LEVELS + 1)),
                ("block_elems", C.c_uint64 * (IODF_MAX_LEVELS + 1)),
                ("block_first_stream", C.c_uint32 * (IODF_MAX_LEVELS + 1)),
                ("block_streams", C.c_uint32 * (IODF_MAX_LEVELS + 1))]


class ProjDesc(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("layer", LayerDesc), ("x_type", C.c_uint32), ("y_type", C.c_uint32),
                ("max_rows", C.c_uint32), ("max_adapters", C.c_uint32), ("max_rank", C.c_uint32)]


class NormDesc(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("channels", C.c_uint32), ("res_type", C.c_uint32),
                ("block_type", C.c_uint32), ("post_norm", C.c_uint32), ("pre_norm", C.c_uint32),
                ("n_type", C.c_uint32), ("shift", C.c_int32), ("n_shift", C.c_int32), ("res_lo", C.c_int32),
                ("res_hi", C.c_int32), ("n_lo", C.c_int32), ("n_hi", C.c_int32), ("eps", C.c_uint64),
                ("mult", C.c_void_p), ("n_mult", C.c_void_p), ("n_bias", C.c_void_p)]


class View(C.Structure):
    _fields_ = [("pixels", C.c_uint64), ("image_stride", C.c_uint64), ("channel_stride", C.c_uint64),
                ("pixel_stride", C.c_uint64)]


class RefinementDesc(C.Structure):
    _fields_ = [("first", C.c_void_p), ("up", C.c_void_p), ("down", C.c_void_p), ("last", C.c_void_p),
                ("gate", C.c_void_p), ("image_adapter", C.c_void_p)]


class IodfError(RuntimeError):
    def __init__(self, status, what):
        super().__init__("%s failed: %s (status %d)" % (what, iodf_strerror(status), status))
        self.status = status


_lib = None


def load_library(path=None):
    """Load libiodf_b200.so (building it with nvcc if it is missing or stale). Raises if that is
    impossible: there is no fallback implementation."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    lib_path = path or _build.build()
    if not os.path.exists(lib_path):
        raise RuntimeError("libiodf_b200.so is missing: run paper_2206_08869_b200.build.build()")
    L = C.CDLL(lib_path)
    vp = C.c_void_p
    L.iodf_create.restype = C.c_int
    L.iodf_create.argtypes = [C.POINTER(ModelDesc), vp, C.c_size_t, vp, C.c_size_t, C.c_int, C.POINTER(vp)]
    L.iodf_destroy.restype = None
    L.iodf_destroy.argtypes = [vp]
    L.iodf_get_layout.restype = C.c_int
    L.iodf_get_layout.argtypes = [vp, C.POINTER(Layout)]
    L.iodf_forward.restype = C.c_int
    L.iodf_forward.argtypes = [vp, vp, C.c_int, vp, vp, vp]
    L.iodf_inverse.restype = C.c_int
    L.iodf_inverse.argtypes = [vp, vp, C.c_int, vp, vp, vp, vp]
    L.iodf_inverse_level.restype = C.c_int
    L.iodf_inverse_level.argtypes = [vp, C.c_int, C.c_int, vp, C.c_int, vp, vp, vp, vp]
    L.iodf_forward_patches.restype = C.c_int
    L.iodf_forward_patches.argtypes = [vp, vp, C.c_int, C.c_int, vp, vp, vp]
    L.iodf_inverse_patches.restype = C.c_int
    L.iodf_inverse_patches.argtypes = [vp, vp, C.c_int, C.c_int, vp, vp, vp, vp]
    L.iodf_codec_create.restype = C.c_int
    L.iodf_codec_create.argtypes = [vp, C.POINTER(CodecDesc), C.POINTER(vp)]
    L.iodf_codec_destroy.restype = None
    L.iodf_codec_destroy.argtypes = [vp]
    L.iodf_codec_get_layout.restype = C.c_int
    L.iodf_codec_get_layout.argtypes = [vp, C.POINTER(CodecLayout)]
    L.iodf_rans_encode.restype = C.c_int
    L.iodf_rans_encode.argtypes = [vp, vp, vp, C.c_int, vp, vp, vp]
    L.iodf_rans_decode_block.restype = C.c_int
    L.iodf_rans_decode_block.argtypes = [vp, C.c_int, vp, vp, vp, C.c_int, vp, vp]
    L.iodf_codec_check.restype = C.c_int
    L.iodf_codec_check.argtypes = [vp, vp, C.POINTER(C.c_uint32)]
    L.iodf_rans_packed_capacity.restype = C.c_size_t
    L.iodf_rans_packed_capacity.argtypes = [vp, C.c_int]
    L.iodf_rans_pack.restype = C.c_int
    L.iodf_rans_pack.argtypes = [vp, vp, vp, C.c_int, vp, vp]
    L.iodf_rans_unpack.restype = C.c_int
    L.iodf_rans_unpack.argtypes = [vp, vp, C.c_size_t, C.c_int, vp, vp, vp]
    L.iodf_compress_host.restype = C.c_int
    L.iodf_compress_host.argtypes = [vp, vp, vp, C.c_int, vp, C.c_size_t, C.POINTER(C.c_size_t), vp]
    L.iodf_decompress_host.restype = C.c_int
    L.iodf_decompress_host.argtypes = [vp, vp, vp, C.c_size_t, C.c_int, vp, vp]
    L.iodf_forward_host.restype = C.c_int
    L.iodf_forward_host.argtypes = [vp, vp, C.c_int, vp, vp, vp]
    L.iodf_inverse_host.restype = C.c_int
    L.iodf_inverse_host.argtypes = [vp, vp, C.c_int, vp, vp]
    L.iodf_forward_timed.restype = C.c_int
    L.iodf_forward_timed.argtypes = [vp, vp, C.c_int, vp, vp, vp, C.POINTER(C.c_float)]
    L.iodf_inverse_timed.restype = C.c_int
    L.iodf_inverse_timed.argtypes = [vp, vp, C.c_int, vp, vp, vp, vp, C.POINTER(C.c_float)]
    L.iodf_forward_static.restype = C.c_int
    L.iodf_forward_static.argtypes = [vp, vp, C.c_int, vp, vp, vp]
    L.iodf_static_scratch_bytes_per_image.restype = C.c_size_t
    L.iodf_static_scratch_bytes_per_image.argtypes = [vp]
    L.iodf_check.restype = C.c_int
    L.iodf_check.argtypes = [vp, vp]
    L.iodf_selftest_timeout.restype = C.c_int
    L.iodf_selftest_timeout.argtypes = [vp, C.c_uint32, vp]
    L.iodf_int8_mma_peak.restype = C.c_int
    L.iodf_int8_mma_peak.argtypes = [vp, C.c_uint32, vp, C.POINTER(C.c_ulonglong)]
    L.iodf_level_kernel_name.restype = C.c_char_p
    L.iodf_level_kernel_name.argtypes = [vp, C.c_int]
    L.iodf_level_images_per_cta.restype = C.c_int
    L.iodf_level_images_per_cta.argtypes = [vp, C.c_int]
    L.iodf_launches_per_call.restype = C.c_int
    L.iodf_launches_per_call.argtypes = [vp, C.c_int]
    L.iodf_proj_create.restype = C.c_int
    L.iodf_proj_create.argtypes = [C.POINTER(ProjDesc), vp, C.c_size_t, vp, C.c_size_t, C.c_int, C.POINTER(vp)]
    L.iodf_proj_destroy.restype = None
    L.iodf_proj_destroy.argtypes = [vp]
    L.iodf_proj_set_adapter.restype = C.c_int
    L.iodf_proj_set_adapter.argtypes = [vp, C.c_uint32, C.c_uint32, vp, vp, vp, vp]
    L.iodf_proj_forward.restype = C.c_int
    L.iodf_proj_forward.argtypes = [vp, vp, C.c_size_t, C.c_int, vp, vp, C.c_int, vp, C.c_size_t, vp]
    L.iodf_proj_check.restype = C.c_int
    L.iodf_proj_check.argtypes = [vp, vp, C.POINTER(C.c_uint32)]
    L.iodf_norm_create.restype = C.c_int
    L.iodf_norm_create.argtypes = [C.POINTER(NormDesc), C.c_int, C.POINTER(vp)]
    L.iodf_norm_destroy.restype = None
    L.iodf_norm_destroy.argtypes = [vp]
    L.iodf_norm_forward.restype = C.c_int
    L.iodf_norm_forward.argtypes = [vp, C.c_int, vp, C.POINTER(View), vp, C.c_size_t, vp, C.c_size_t, vp,
                                    C.POINTER(View), vp, C.c_size_t, vp]
    L.iodf_codec_set_refinement.restype = C.c_int
    L.iodf_codec_set_refinement.argtypes = [vp, C.c_int, C.POINTER(RefinementDesc)]
    L.iodf_refine_prior.restype = C.c_int
    L.iodf_refine_prior.argtypes = [vp, C.c_int, vp, C.c_int, vp]
    L.iodf_codec_selftest_timeout.restype = C.c_int
    L.iodf_codec_selftest_timeout.argtypes = [vp, C.c_int, C.c_uint32, vp]
    L.iodf_strerror.restype = C.c_char_p
    L.iodf_strerror.argtypes = [C.c_int]
    L.iodf_last_cuda_error.restype = C.c_int
    L.iodf_last_cuda_error.argtypes = [vp]
    if path is None:
        _lib = L
    return L


def iodf_strerror(status):
    return load_library().iodf_strerror(int(status)).decode()


class _Marshalled:
    """C descriptor structs for a model dict, with every referenced array kept alive."""

    def __init__(self, model, max_batch, plan=0):
        self.keep = []
        wts, par = [], []
        self.woff = self.poff = 0

        def layer(ly):
            w = np.ascontiguousarray(ly["w"], dtype=np.int8)
            cl = ly["clamp"]
            if ly.get("gate") is not None:
                raise ValueError("gated (masked-dense) layers must be compacted before deployment")
            d = LayerDesc(ly["k"], ly["c_in"], ly["c_out"], int(ly["relu"]), int(cl is not None),
                          cl[0] if cl else 0, cl[1] if cl else 0, self.woff, self.poff)
            wts.append(w.reshape(-1))
            self.woff += w.size
            for a in (ly["bias"], ly["m0"], ly["s"]):
                par.append(np.asarray(a, dtype=np.int32).reshape(-1))
                self.poff += ly["c_out"]
            return d

        levels = (LevelDesc * len(model["levels"]))()
        for li, lv in enumerate(model["levels"]):
            cps = (CouplingDesc * max(1, len(lv["couplings"])))()
            for ki, cp in enumerate(lv["couplings"]):
                perm = np.ascontiguousarray(cp["perm"], dtype=np.int32)
                lays = (LayerDesc * len(cp["layers"]))(*[layer(ly) for ly in cp["layers"]])
                self.keep += [perm, lays]
                rblocks = cp.get("blocks") or []
                rbs = (ResBlockDesc * max(1, len(rblocks)))()
                for bi, rb in enumerate(rblocks):
                    idx = np.ascontiguousarray(rb["idx"], dtype=np.int32)
                    self.keep.append(idx)
                    rbs[bi] = ResBlockDesc(rb["short_m0"], rb["short_s"], rb["clamp"][0], rb["clamp"][1], len(idx),
                                           idx.ctypes.data_as(C.POINTER(C.c_int32)))
                self.keep.append(rbs)
                cps[ki] = CouplingDesc(perm.ctypes.data_as(C.POINTER(C.c_int32)), cp["in_m0"], cp["in_s"],
                                       len(cp["layers"]), lays, len(rblocks), rbs)
            self.keep.append(cps)
            levels[li].n_couplings = len(lv["couplings"])
            levels[li].couplings = cps
            levels[li].split = int(lv["split"])
            levels[li].has_prior = int(lv["prior"] is not None)
            if lv["prior"] is not None:
                hd = lv["prior"]
                levels[li].prior_in_m0, levels[li].prior_in_s = hd["in_m0"], hd["in_s"]
                levels[li].prior_layer = layer(hd["layer"])
                levels[li].ls_lo, levels[li].ls_hi = hd["ls_lo"], hd["ls_hi"]
        self.levels = levels
        self.desc = ModelDesc(IODF_ABI_VERSION, model["in_c"], model["in_h"], model["in_w"], len(model["levels"]),
                              int(max_batch), levels, int(plan))
        self.wts = np.concatenate(wts) if wts else np.zeros(1, np.int8)
        self.par = np.concatenate(par) if par else np.zeros(1, np.int32)


class Model:
    """Handle of an iodf_model; destroyed when garbage collected."""

    def __init__(self, handle, layout, in_shape, max_batch, device=0):
        self.handle, self.layout, self.in_shape, self.max_batch, self.device = handle, layout, in_shape, max_batch, device
        self.d, self.d_fact = int(layout.d), int(layout.d_fact)

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.iodf_destroy(h)


def iodf_create(model, max_batch, device=0, marshalled=None, plan=IODF_PLAN_LATENCY):
    """plan: IODF_PLAN_LATENCY (the shortest step) or IODF_PLAN_THROUGHPUT (fewer CTAs per launch, for
    several batches in flight on streams and handles of their own); see include/iodf.h."""
    L = load_library()
    m = marshalled or _Marshalled(model, max_batch, plan)
    out = C.c_void_p()
    rc = L.iodf_create(C.byref(m.desc), m.wts.ctypes.data, m.wts.size, m.par.ctypes.data, m.par.size, int(device),
                       C.byref(out))
    if rc != 0:
        raise IodfError(rc, "iodf_create")
    lay = Layout()
    L.iodf_get_layout(out, C.byref(lay))
    return Model(out, lay, (model["in_c"], model["in_h"], model["in_w"]), int(max_batch), int(device))


def iodf_destroy(model):
    h, model.handle = model.handle, None
    if h:
        load_library().iodf_destroy(h)


def iodf_get_layout(model):
    return model.layout


def _stream(stream):
    if stream is None:
        import torch
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    return C.c_void_p(int(getattr(stream, "cuda_stream", stream)))    # a torch stream or a raw handle


def _ptr(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def _on_stream(stream, device):
    """The torch stream of a call's `stream` argument as the current one; None leaves the current one."""
    import contextlib
    import torch
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)) & ~1, device)   # 1: the legacy default stream, 0 to torch
    return torch.cuda.stream(stream)


def _made(make, shape, dtype, device, stream):
    """An output of a call on `stream` that the caller did not bring, in that stream's order: its memory is nobody's that the
    current stream still works on, and a fill of it comes before the call's kernels. Nor is it the next call's before the
    current stream has done with it."""
    with _on_stream(stream, device):
        t = make(shape, dtype=dtype, device=device)
    if stream is not None:
        import torch
        t.record_stream(torch.cuda.current_stream(device))
    return t


def iodf_forward(model, x_u8, z=None, prior=None, stream=None, want_prior=True):
    """x_u8: cuda uint8 [B,C,H,W]. Returns (z int32 [B,d], prior int32 [B,2,d_fact] | None)."""
    import torch
    B = x_u8.shape[0]
    assert x_u8.is_cuda and x_u8.dtype == torch.uint8 and x_u8.is_contiguous()
    if z is None:
        z = _made(torch.empty, (B, model.d), torch.int32, x_u8.device, stream)
    if prior is None and want_prior and model.d_fact:
        prior = _made(torch.empty, (B, 2, model.d_fact), torch.int32, x_u8.device, stream)
    rc = load_library().iodf_forward(model.handle, _ptr(x_u8), B, _ptr(z), _ptr(prior), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_forward")
    return z, prior


def iodf_inverse(model, z, x_u8=None, prior=None, out_of_range=None, stream=None):
    """z: cuda int32 [B,d]. Returns x_u8 uint8 [B,C,H,W]."""
    import torch
    B = z.shape[0]
    assert z.is_cuda and z.dtype == torch.int32 and z.is_contiguous()
    if x_u8 is None:
        x_u8 = _made(torch.empty, (B,) + tuple(model.in_shape), torch.uint8, z.device, stream)
    rc = load_library().iodf_inverse(model.handle, _ptr(z), B, _ptr(x_u8), _ptr(prior), _ptr(out_of_range),
                                     _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_inverse")
    return x_u8


IODF_LEVEL_PRIOR = 1
IODF_LEVEL_COUPLINGS = 2


def iodf_inverse_level(model, level, phase, z, x_u8=None, prior=None, out_of_range=None, stream=None):
    """One step of the level-stepped decode (see include/iodf.h). z: cuda int32 [B,d] (full size)."""
    rc = load_library().iodf_inverse_level(model.handle, level, phase, _ptr(z), z.shape[0], _ptr(x_u8), _ptr(prior),
                                           _ptr(out_of_range), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_inverse_level")


def iodf_forward_patches(model, image_u8, z=None, prior=None, stream=None):
    """image_u8: cuda uint8 [C,H,W], H and W multiples of the model's input size. Returns (z, prior)
    of the batch of patches in row-major patch order."""
    import torch
    _, H, W = image_u8.shape
    B = (H // model.in_shape[1]) * (W // model.in_shape[2])
    if z is None:
        z = _made(torch.empty, (B, model.d), torch.int32, image_u8.device, stream)
    if prior is None and model.d_fact:
        prior = _made(torch.empty, (B, 2, model.d_fact), torch.int32, image_u8.device, stream)
    rc = load_library().iodf_forward_patches(model.handle, _ptr(image_u8), H, W, _ptr(z), _ptr(prior), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_forward_patches")
    return z, prior


def iodf_inverse_patches(model, z, H, W, image_u8=None, prior=None, out_of_range=None, stream=None):
    """z: cuda int32 [B,d] of the patch batch. Returns the image uint8 [C,H,W]."""
    import torch
    if image_u8 is None:
        image_u8 = _made(torch.empty, (model.in_shape[0], H, W), torch.uint8, z.device, stream)
    rc = load_library().iodf_inverse_patches(model.handle, _ptr(z), H, W, _ptr(image_u8), _ptr(prior),
                                             _ptr(out_of_range), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_inverse_patches")
    return image_u8


class Codec:
    """Handle of an iodf_codec; destroyed when garbage collected."""

    def __init__(self, handle, layout, model):
        self.handle, self.layout, self.model = handle, layout, model
        self.n_blocks, self.n_streams = int(layout.n_blocks), int(layout.n_streams)
        self.words_per_stream = int(layout.words_per_stream)

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.iodf_codec_destroy(h)


def iodf_codec_create(model, codec):
    """codec: dict with the tables G (uint16), R (uint32), umax, final_ls, elems_per_stream."""
    L = load_library()
    G = np.ascontiguousarray(codec["G"], dtype=np.uint16)
    R = np.ascontiguousarray(codec["R"], dtype=np.uint32)
    desc = CodecDesc(IODF_ABI_VERSION, G.ctypes.data, int(codec["umax"]), R.ctypes.data, len(R),
                     int(codec["final_ls"]), int(codec["elems_per_stream"]))
    out = C.c_void_p()
    rc = L.iodf_codec_create(model.handle, C.byref(desc), C.byref(out))
    if rc != 0:
        raise IodfError(rc, "iodf_codec_create")
    lay = CodecLayout()
    L.iodf_codec_get_layout(out, C.byref(lay))
    return Codec(out, lay, model)


def iodf_rans_encode(codec, z, prior, words=None, counts=None, stream=None):
    """z cuda int32 [B,d], prior cuda int32 [B,2,d_fact] -> (words uint16 [B,S,cap], counts uint32-as-int32 [B,S])."""
    import torch
    B = z.shape[0]
    if words is None:
        words = _made(torch.empty, (B, codec.n_streams, codec.words_per_stream), torch.int16, z.device, stream)
    if counts is None:
        counts = _made(torch.empty, (B, codec.n_streams), torch.int32, z.device, stream)
    rc = load_library().iodf_rans_encode(codec.handle, _ptr(z), _ptr(prior), B, _ptr(words), _ptr(counts), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_rans_encode")
    return words, counts


def iodf_rans_decode_block(codec, block, words, counts, prior, z, stream=None):
    rc = load_library().iodf_rans_decode_block(codec.handle, int(block), _ptr(words), _ptr(counts), _ptr(prior),
                                               z.shape[0], _ptr(z), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_rans_decode_block")


def iodf_rans_packed_capacity(codec, B):
    return int(load_library().iodf_rans_packed_capacity(codec.handle, int(B)))


def iodf_rans_pack(codec, words, counts, packed=None, stream=None):
    """Container -> compact byte stream. Returns (packed cuda uint8 tensor of full capacity, total bytes);
    reading the total synchronises."""
    import torch
    B = counts.shape[0]
    if packed is None:
        packed = _made(torch.empty, iodf_rans_packed_capacity(codec, B), torch.uint8, counts.device, stream)
    rc = load_library().iodf_rans_pack(codec.handle, _ptr(words), _ptr(counts), B, _ptr(packed), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_rans_pack")
    with _on_stream(stream, packed.device):
        payload = int(packed[4 * B:4 * B + 4].cpu().numpy().view(np.uint32)[0])
    return packed, 4 * (B + 1) + payload


def iodf_rans_unpack(codec, packed, nbytes, B, words=None, counts=None, stream=None):
    import torch
    if words is None:
        words = _made(torch.zeros, (B, codec.n_streams, codec.words_per_stream), torch.int16, packed.device, stream)
    if counts is None:
        counts = _made(torch.zeros, (B, codec.n_streams), torch.int32, packed.device, stream)
    rc = load_library().iodf_rans_unpack(codec.handle, _ptr(packed), int(nbytes), int(B), _ptr(words), _ptr(counts),
                                         _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_rans_unpack")
    return words, counts


def iodf_compress_host(model, codec, x_u8_host, out_host=None, stream=None):
    """Host uint8 images [B,C,H,W] -> (host uint8 buffer, number of valid bytes). Synchronises."""
    import torch
    B = x_u8_host.shape[0]
    if out_host is None:
        out_host = torch.empty(iodf_rans_packed_capacity(codec, B), dtype=torch.uint8).pin_memory()
    n = C.c_size_t(0)
    rc = load_library().iodf_compress_host(model.handle, codec.handle, _ptr(x_u8_host), B, _ptr(out_host),
                                           out_host.numel(), C.byref(n), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_compress_host")
    return out_host, int(n.value)


def iodf_decompress_host(model, codec, in_host, nbytes, B, x_u8_host=None, stream=None):
    """Compact byte stream (host) -> host uint8 images; valid after the stream is synchronised."""
    import torch
    if x_u8_host is None:
        x_u8_host = torch.empty((B,) + tuple(model.in_shape), dtype=torch.uint8).pin_memory()
    rc = load_library().iodf_decompress_host(model.handle, codec.handle, _ptr(in_host), int(nbytes), int(B),
                                             _ptr(x_u8_host), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_decompress_host")
    return x_u8_host


def iodf_codec_check(codec, stream=None):
    n = C.c_uint32(0)
    rc = load_library().iodf_codec_check(codec.handle, _stream(stream), C.byref(n))
    if rc != 0:
        raise IodfError(rc, "iodf_codec_check (%d streams)" % n.value)


def iodf_forward_host(model, x_u8, z, prior=None, stream=None):
    """Host (ideally pinned) torch tensors in and out; results valid after the stream is synchronised."""
    rc = load_library().iodf_forward_host(model.handle, _ptr(x_u8), x_u8.shape[0], _ptr(z), _ptr(prior),
                                          _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_forward_host")


def iodf_inverse_host(model, z, x_u8, stream=None):
    rc = load_library().iodf_inverse_host(model.handle, _ptr(z), z.shape[0], _ptr(x_u8), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_inverse_host")


def iodf_forward_timed(model, x_u8, z, prior=None, stream=None):
    """Encode with per-level event timing; returns the list of per-level kernel times in ms."""
    n = int(model.layout.n_levels)
    ms = (C.c_float * n)()
    rc = load_library().iodf_forward_timed(model.handle, _ptr(x_u8), x_u8.shape[0], _ptr(z), _ptr(prior),
                                           _stream(stream), ms)
    if rc != 0:
        raise IodfError(rc, "iodf_forward_timed")
    return list(ms)


def iodf_inverse_timed(model, z, x_u8, prior=None, out_of_range=None, stream=None):
    n = int(model.layout.n_levels)
    ms = (C.c_float * n)()
    rc = load_library().iodf_inverse_timed(model.handle, _ptr(z), z.shape[0], _ptr(x_u8), _ptr(prior),
                                           _ptr(out_of_range), _stream(stream), ms)
    if rc != 0:
        raise IodfError(rc, "iodf_inverse_timed")
    return list(ms)


IODF_STATIC_SCRATCH_BYTES = 8 * 1024 * 1024


def iodf_static_scratch_bytes_per_image(model):
    return int(load_library().iodf_static_scratch_bytes_per_image(model.handle))


def iodf_forward_static(model, x_u8, z, prior=None, stream=None):
    """Encode using the library's fixed scratch array instead of the model's allocated workspace.
    The caller passes every buffer (this wrapper allocates nothing either)."""
    rc = load_library().iodf_forward_static(model.handle, _ptr(x_u8), x_u8.shape[0], _ptr(z), _ptr(prior),
                                            _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_forward_static")


def iodf_check(model, stream=None):
    rc = load_library().iodf_check(model.handle, _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_check")


def iodf_selftest_timeout(model, tries=3, stream=None):
    rc = load_library().iodf_selftest_timeout(model.handle, int(tries), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_selftest_timeout")


def iodf_int8_mma_peak(model, mma_groups, stream=None):
    """Enqueue the MMA-only kernel; returns the int8 OPs of the launch."""
    ops = C.c_ulonglong(0)
    rc = load_library().iodf_int8_mma_peak(model.handle, int(mma_groups), _stream(stream), C.byref(ops))
    if rc != 0:
        raise IodfError(rc, "iodf_int8_mma_peak")
    return int(ops.value)


def iodf_level_kernel_name(model, level):
    return load_library().iodf_level_kernel_name(model.handle, int(level)).decode()


def iodf_launches_per_call(model, inverse=False):
    return load_library().iodf_launches_per_call(model.handle, int(inverse))


def iodf_level_images_per_cta(model, level):
    n = load_library().iodf_level_images_per_cta(model.handle, int(level))
    if n < 0:
        raise IodfError(n, "iodf_level_images_per_cta")
    return n


# ---- single integer layers ---------------------------------------------------------------------------------
IODF_I8, IODF_U8, IODF_I16, IODF_I32 = 1, 2, 3, 4
IODF_NORM_RMS, IODF_NORM_CENTRED = 1, 2
_MOST = 2 ** 31 - 1                    # rows and requests of a call


def _fits(value, ctype, what):
    """The value as the library's integer type takes it; ctypes would cut it off."""
    value = int(value)
    if ctype(value).value != value:
        raise ValueError("%s = %d is out of range" % (what, value))
    return value


def _record(cls, *values):
    """A descriptor of the library, every integer in its range."""
    return cls(*[_fits(v, t, name) if t in (C.c_uint32, C.c_int32, C.c_uint64) else v for (name, t), v in zip(cls._fields_, values)])


def _integers(a, dtype, what):
    """The array's values in another integer type, contiguous; a value that the type does not have is refused."""
    a = np.asarray(a)
    out = np.ascontiguousarray(a, dtype=dtype)
    if a.dtype != out.dtype and not np.array_equal(a, out):
        raise ValueError("%s holds values that are not %s" % (what, out.dtype))
    return out


def _type_code(dtype, allowed):
    import torch
    codes = {torch.int8: IODF_I8, torch.uint8: IODF_U8, torch.int16: IODF_I16, torch.int32: IODF_I32}
    if dtype not in codes or codes[dtype] not in allowed:
        raise ValueError("element type %s is not one of the operator's" % (dtype,))
    return codes[dtype]


def _on(t, handle, dtype, what):
    if t.get_device() != handle.device or t.dtype is not dtype:    # -1: not on a GPU
        raise ValueError("%s must be a %s tensor on cuda:%d" % (what, dtype, handle.device))
    return t


def _rows_of(t, handle, dtype, rows, channels, what):
    """Row stride of a [rows, channels] tensor whose channels lie side by side."""
    if t.get_device() != handle.device or t.dtype is not dtype:
        _on(t, handle, dtype, what)
    strides = t.stride()
    if t.shape != (rows, channels) or (strides[1] != 1 and channels > 1):
        raise ValueError("%s must be [%d, %d] with channels side by side" % (what, rows, channels))
    return strides[0] if rows > 1 else max(channels, strides[0])


def _layer_stream(stream, device):
    if stream is None:
        import torch
        return torch._C._cuda_getCurrentRawStream(device)
    return int(getattr(stream, "cuda_stream", stream))


def _addr(t):
    return None if t is None else t.data_ptr()


class Projection:
    """Handle of an iodf_proj; destroyed when garbage collected."""

    def __init__(self, handle, device, c_in, c_out, max_rows, x_dtype, y_dtype):
        self.handle, self.device, self.c_in, self.c_out, self.max_rows = handle, device, c_in, c_out, max_rows
        self.x_dtype, self.y_dtype = x_dtype, y_dtype
        import torch
        self.int32 = torch.int32

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.iodf_proj_destroy(h)


def iodf_proj_create(layer, max_rows, max_adapters=0, max_rank=0, x_dtype=None, y_dtype=None, device=0):
    """layer: a layer dict with k = 1 (w, bias, m0, s, relu, clamp), as in a model's couplings. x_dtype int8
    (default) or uint8; y_dtype int32 (default), int8 or uint8. Adapters are put into their slots by
    iodf_proj_set_adapter."""
    import torch
    L = load_library()
    x_dtype, y_dtype = x_dtype or torch.int8, y_dtype or torch.int32
    if layer.get("gate") is not None:
        raise ValueError("gated (masked-dense) layers must be compacted before deployment")
    w = _integers(layer["w"], np.int8, "w").reshape(-1)
    par = [_integers(layer[k], np.int32, k).reshape(-1) for k in ("bias", "m0", "s")]
    if any(a.size != layer["c_out"] for a in par) or w.size > layer["k"] ** 2 * layer["c_in"] * layer["c_out"]:
        raise ValueError("w, bias, m0 and s do not match the layer's k, c_in and c_out")
    par = np.concatenate(par)
    cl = layer["clamp"]
    lay = _record(LayerDesc, layer["k"], layer["c_in"], layer["c_out"], int(layer["relu"]), int(cl is not None),
                  cl[0] if cl else 0, cl[1] if cl else 0, 0, 0)
    desc = _record(ProjDesc, IODF_ABI_VERSION, lay, _type_code(x_dtype, (IODF_I8, IODF_U8)),
                   _type_code(y_dtype, (IODF_I8, IODF_U8, IODF_I32)), max_rows, max_adapters, max_rank)
    out = C.c_void_p()
    rc = L.iodf_proj_create(C.byref(desc), w.ctypes.data, w.size, par.ctypes.data, par.size, _fits(device, C.c_int, "device"), C.byref(out))
    if rc != 0:
        raise IodfError(rc, "iodf_proj_create")
    return Projection(out, int(device), int(layer["c_in"]), int(layer["c_out"]), int(max_rows), x_dtype, y_dtype)


def iodf_proj_set_adapter(proj, slot, adapter, stream=None):
    """adapter: dict rank, down int8 [rank, c_in], m0 and s int32 [rank], up int8 [c_out, rank]; None empties the slot."""
    rank = int(adapter["rank"]) if adapter else 0
    down = rq = up = None
    if rank:
        down, up = _integers(adapter["down"], np.int8, "down"), _integers(adapter["up"], np.int8, "up")
        rq = [_integers(adapter[k], np.int32, k).reshape(-1) for k in ("m0", "s")]
        if down.shape != (rank, proj.c_in) or up.shape != (proj.c_out, rank) or any(a.size != rank for a in rq):
            raise ValueError("adapter arrays do not match its rank and the layer's channels")
        rq = np.concatenate(rq)
    ptr = [None if a is None else a.ctypes.data for a in (down, rq, up)]
    rc = load_library().iodf_proj_set_adapter(proj.handle, _fits(slot, C.c_uint32, "slot"), _fits(rank, C.c_uint32, "rank"), ptr[0], ptr[1], ptr[2],
                                              _layer_stream(stream, proj.device))
    if rc != 0:
        raise IodfError(rc, "iodf_proj_set_adapter")


def iodf_proj_forward(proj, x, seg_start=None, seg_adapter=None, y=None, stream=None):
    """x: cuda [rows, c_in] of the handle's type, row stride a multiple of 16 bytes. seg_start int32 [n + 1] and
    seg_adapter int32 [n] on the device: the rows and the slot of each request. Returns y [rows, c_out]; rows in no
    request keep what y held (zero where y is made here), with n = 0 all of them. Without requests (both None) every row is
    computed without an adapter. On another stream than the current one, what the call reads has to be
    ready on that stream; a y made here belongs to it."""
    rows = x.shape[0]
    ldx = _rows_of(x, proj, proj.x_dtype, rows, proj.c_in, "x")
    if rows == 1:
        ldx = (ldx + 15) // 16 * 16          # a single row has no stride of its own
    n_seg, start, which = 0, None, None
    if (seg_start is None) != (seg_adapter is None):
        raise ValueError("seg_start and seg_adapter are given together or not at all")
    if seg_start is not None:
        n_seg = seg_adapter.numel()
        _on(seg_start, proj, proj.int32, "seg_start")
        _on(seg_adapter, proj, proj.int32, "seg_adapter")
        if seg_start.numel() != n_seg + 1 or not seg_start.is_contiguous() or not seg_adapter.is_contiguous():
            raise ValueError("seg_start must hold %d contiguous values, one more than seg_adapter" % (n_seg + 1))
        start, which = seg_start.data_ptr(), seg_adapter.data_ptr()
    if y is None:
        import torch
        y = _made(torch.empty if seg_start is None else torch.zeros, (rows, proj.c_out), proj.y_dtype, x.device, stream)
    ldy = _rows_of(y, proj, proj.y_dtype, rows, proj.c_out, "y")
    if rows > _MOST or n_seg > _MOST:
        raise ValueError("%d rows of %d requests are out of range" % (rows, n_seg))
    if start is not None and not n_seg:
        return y                             # no request owns a row; to the library n_seg = 0 is a call without requests
    rc = (_lib or load_library()).iodf_proj_forward(proj.handle, x.data_ptr(), ldx, rows, start, which, n_seg, y.data_ptr(), ldy,
                                                    _layer_stream(stream, proj.device))
    if rc != 0:
        raise IodfError(rc, "iodf_proj_forward")
    return y


def iodf_proj_check(proj, stream=None):
    n = C.c_uint32(0)
    rc = load_library().iodf_proj_check(proj.handle, _layer_stream(stream, proj.device), C.byref(n))
    if rc != 0:
        raise IodfError(rc, "iodf_proj_check (%d requests)" % n.value)


class Norm:
    """Handle of an iodf_norm; destroyed when garbage collected."""

    def __init__(self, handle, device, channels, res_dtype, block_dtype, n_dtype):
        self.handle, self.device, self.channels = handle, device, channels
        self.res_dtype, self.block_dtype, self.n_dtype = res_dtype, block_dtype, n_dtype
        import torch
        self.uint8, self.views = torch.uint8, {}

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.iodf_norm_destroy(h)


_NORMS = {None: 0, "rms": IODF_NORM_RMS, "centred": IODF_NORM_CENTRED}


def iodf_norm_create(desc, device=0):
    """desc: dict with c, res_dtype (int16 | int32) and, as far as used, eps, block_dtype (int8 | int32 | None),
    res_range (lo, hi), post {norm: None | "rms" | "centred", mult int32 [c], shift} and
    pre {norm, mult int32 [c], shift, bias int32 [c], clamp (lo, hi), dtype int8 | uint8}."""
    L = load_library()
    c, post, pre = int(desc["c"]), desc.get("post"), desc.get("pre")
    tabs = {}
    for name, part, key in (("mult", post, "mult"), ("n_mult", pre, "mult"), ("n_bias", pre, "bias")):
        if part is not None:
            tabs[name] = _integers(part[key], np.int32, name).reshape(-1)
            if tabs[name].size != c:
                raise ValueError("%s must hold one value per channel" % name)
    ptr = {k: tabs[k].ctypes.data if k in tabs else None for k in ("mult", "n_mult", "n_bias")}
    block, (lo, hi) = desc.get("block_dtype"), desc.get("res_range", (0, 0))
    n_dtype = pre["dtype"] if pre else None
    d = _record(NormDesc, IODF_ABI_VERSION, c, _type_code(desc["res_dtype"], (IODF_I16, IODF_I32)),
                _type_code(block, (IODF_I8, IODF_I32)) if block else 0,
                _NORMS[post["norm"]] if post else 0, _NORMS[pre["norm"]] if pre else 0,
                _type_code(n_dtype, (IODF_I8, IODF_U8)) if pre else 0,
                post["shift"] if post else 0, pre["shift"] if pre else 0, lo, hi,
                pre["clamp"][0] if pre else 0, pre["clamp"][1] if pre else 0, desc.get("eps", 0),
                ptr["mult"], ptr["n_mult"], ptr["n_bias"])
    out = C.c_void_p()
    rc = L.iodf_norm_create(C.byref(d), _fits(device, C.c_int, "device"), C.byref(out))
    if rc != 0:
        raise IodfError(rc, "iodf_norm_create")
    return Norm(out, int(device), c, desc["res_dtype"], block, n_dtype)


def _view(t, norm, what):
    """rows and strides of a residual stream: [rows, c] or planes [images, c, pixels]."""
    shape, strides, channels = t.shape, t.stride(), norm.channels
    known = norm.views.get((shape, strides))          # by shape: the descriptor costs as much to make as the rest of the call's checks
    if known is not None:
        return known
    if len(shape) == 2 and shape[1] == channels and (channels == 1 or strides[1] == 1):
        made = shape[0], View(max(1, shape[0]), 0, 1, strides[0])
    elif len(shape) == 3 and shape[1] == channels and (shape[2] == 1 or strides[2] == 1):
        made = shape[0] * shape[2], View(max(1, shape[2]), strides[0], strides[1], 1)
    else:
        raise ValueError("%s must be [rows, %d] or [images, %d, pixels] with the last axis contiguous" % (what, channels, channels))
    if len(norm.views) >= 64:
        norm.views.clear()
    norm.views[(shape, strides)] = made
    return made


def iodf_norm_forward(norm, r, b=None, gate=None, r_out=None, n=None, stream=None):
    """r: the residual stream, cuda [rows, c] or planes [images, c, pixels] (any outer strides); b [rows, c] the
    block's output; gate uint8 [rows, c] or [c]. Returns (r_out, n), None where the handle has no such part.
    r_out may be r; else no output may overlap another operand. Outputs made here belong to the call's stream."""
    c = norm.channels
    _on(r, norm, norm.res_dtype, "r")
    rows, rv = _view(r, norm, "r")
    if (b is not None) != (norm.block_dtype is not None):
        raise ValueError("b is given exactly if the handle has a block")
    ldb = ldg = ldn = 0
    ov = None
    if b is not None:
        ldb = _rows_of(b, norm, norm.block_dtype, rows, c, "b")
        if r_out is r:
            ov = rv
        else:
            if r_out is None:
                import torch
                r_out = _made(torch.empty, r.shape, r.dtype, r.device, stream)
            if _on(r_out, norm, norm.res_dtype, "r_out").shape != r.shape:
                raise ValueError("r_out must have the shape of r")
            ov = _view(r_out, norm, "r_out")[1]
    if gate is not None:
        if gate.dim() == 1:
            if _on(gate, norm, norm.uint8, "gate").shape[0] != c or (c > 1 and gate.stride(0) != 1):
                raise ValueError("gate must be [%d] or [%d, %d]" % (c, rows, c))
        else:
            ldg = _rows_of(gate, norm, norm.uint8, rows, c, "gate")
    if norm.n_dtype is not None:
        if n is None:
            import torch
            n = _made(torch.empty, (rows, c), norm.n_dtype, r.device, stream)
        ldn = _rows_of(n, norm, norm.n_dtype, rows, c, "n")
    if rows > _MOST:
        raise ValueError("%d rows are out of range" % rows)
    rc = (_lib or load_library()).iodf_norm_forward(norm.handle, rows, r.data_ptr(), rv, _addr(b), ldb, _addr(gate), ldg,
                                                    _addr(r_out), ov, _addr(n), ldn, _layer_stream(stream, norm.device))
    if rc != 0:
        raise IodfError(rc, "iodf_norm_forward")
    return r_out, n


def iodf_codec_set_refinement(codec, level, first=None, up=None, down=None, last=None, gate=None, image_adapter=None):
    """Give a level of the codec a refinement of its prior's means (see include/iodf.h), or take it away (no handles):
    first, last: norms; up, down: projections; gate uint8 [c] and image_adapter int32 [max_batch] on the device."""
    desc = None
    if first is not None:
        for h in (first, up, down, last):
            if h is None:
                raise ValueError("a refinement has two norms and two projections")
        import torch
        c = first.channels
        if gate is not None and (_on(gate, first, torch.uint8, "gate").numel() != c or not gate.is_contiguous()):
            raise ValueError("gate must hold %d contiguous values" % c)
        if image_adapter is not None and (_on(image_adapter, first, torch.int32, "image_adapter").numel() < codec.model.max_batch
                                          or not image_adapter.is_contiguous()):
            raise ValueError("image_adapter must hold %d contiguous values" % codec.model.max_batch)
        desc = RefinementDesc(first.handle, up.handle, down.handle, last.handle, _addr(gate), _addr(image_adapter))
    rc = load_library().iodf_codec_set_refinement(codec.handle, _fits(level, C.c_int, "level"), C.byref(desc) if desc is not None else None)
    if rc != 0:
        raise IodfError(rc, "iodf_codec_set_refinement")
    if not hasattr(codec, "refinements"):
        codec.refinements = {}
    codec.refinements[int(level)] = (first, up, down, last, gate, image_adapter)     # kept alive


def iodf_refine_prior(codec, level, prior, stream=None):
    """Apply a level's refinement to prior int32 [B, 2, d_fact] in place."""
    import torch
    _on(prior, codec.model, torch.int32, "prior")
    if prior.dim() != 3 or prior.shape[1:] != (2, codec.model.d_fact) or not prior.is_contiguous():
        raise ValueError("prior must be a contiguous [B, 2, %d]" % codec.model.d_fact)
    rc = load_library().iodf_refine_prior(codec.handle, _fits(level, C.c_int, "level"), prior.data_ptr(), _fits(prior.shape[0], C.c_int, "B"),
                                          _layer_stream(stream, prior.get_device()))
    if rc != 0:
        raise IodfError(rc, "iodf_refine_prior")


def iodf_codec_selftest_timeout(codec, level, tries=3, stream=None):
    """Make a bounded wait of a level's refinement run out (see include/iodf.h); iodf_codec_check reports it."""
    rc = load_library().iodf_codec_selftest_timeout(codec.handle, _fits(level, C.c_int, "level"), _fits(tries, C.c_uint32, "tries"), _stream(stream))
    if rc != 0:
        raise IodfError(rc, "iodf_codec_selftest_timeout")
