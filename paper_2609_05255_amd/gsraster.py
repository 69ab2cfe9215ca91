"""Python binding of libgsraster.so (the C ABI of include/gsraster.h).

Argument marshalling only: torch tensors provide device memory and the stream,
every step of the rasterizer runs in the HIP library. The library must have
been built (``python -m paper_2609_05255_amd.build``); importing this module
raises if it is missing, there is no fallback.

Function names follow the C ABI: gs_preprocess, gs_bin_sort, gs_render_fwd,
gs_render_bwd, gs_workspace_size. ``Frame`` owns the buffers of one camera's
forward + backward pass for a scene of n Gaussians.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgsraster.so")

GS_OK, GS_ERR_INVALID_ARG, GS_ERR_CAPACITY, GS_ERR_DEVICE, GS_ERR_UNSUPPORTED = range(5)
GS_PAIRS_ON_DEVICE = (1 << 64) - 1   # gs_bin_sort reads the pair count on the device
GS_APP_SH3, GS_APP_LATENT_MLP, GS_APP_NEURAL, GS_APP_NEURAL_FOLDED, GS_APP_NASG, GS_APP_NASGABOR = range(6)
LOBE_ROWS = {GS_APP_NASG: 8, GS_APP_NASGABOR: 9}
NEURAL_FEATURES = 8
NEURAL_WEIGHTS = 816


def neural_weight_count(arch=None) -> int:
    """Weights of the neural decoder with arch = (hidden layers, width, raw16); None: the paper's (2, 16, 0)."""
    layers, width = (2, 16) if arch is None else (int(arch[0]), int(arch[1]))
    return 32 * width + (layers - 1) * width * width + 3 * width
KERNEL_NAMES = ["preprocess", "pair_count", "depth_sort", "entry_offsets", "block_entries", "block_sort", "tile_lists",
                "blend_fwd", "bwd_prep", "blend_bwd", "preprocess_bwd", "mlp_reduce", "adam", "neural_fold",
                "layer_norm_fwd", "layer_norm_bwd", "linear_fwd", "linear_bwd", "grad_norm", "sort_rows", "embedding_fwd",
                "embedding_bwd", "route_fwd", "route_bwd", "dispatch_fwd", "dispatch_bwd", "combine_fwd", "combine_bwd",
                "experts_fwd", "experts_bwd"]
TYPE_IDS = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}   # GS_F32, GS_F16, GS_BF16
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "tanh": 4, "sigmoid": 5}   # GS_ACT_*
ADAM_MAX_TENSORS = 8
ADAM_MAX_ROWS = 128
SPLAT_BYTES = 64
MLP_WEIGHTS = 1664


class GsError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("gsraster status %d: %s" % (status, msg))
        self.status = status


# gs_splat's fields as 4-byte word offsets into its 64-byte record (the four
# int16 of the rectangle fill words 12 and 13)
SPLAT_WORDS = dict(mean_x=0, mean_y=1, conic_a=2, conic_b=3, conic_c=4, opacity=5, color=6, power_min=9,
                   ext_x=10, ext_y=11, rect=12, depth=14)


class Camera(C.Structure):
    _fields_ = [("viewmat", C.c_float * 12), ("campos", C.c_float * 3), ("fx", C.c_float), ("fy", C.c_float),
                ("cx", C.c_float), ("cy", C.c_float), ("width", C.c_int32), ("height", C.c_int32),
                ("near_plane", C.c_float), ("bg", C.c_float * 3)]


class Gaussians(C.Structure):
    _fields_ = [("n", C.c_int64), ("means", C.c_void_p), ("log_scales", C.c_void_p), ("quats", C.c_void_p),
                ("opacity_logits", C.c_void_p)]


class Appearance(C.Structure):
    _fields_ = [("kind", C.c_int32), ("sh_degree", C.c_int32), ("sh", C.c_void_p), ("latent", C.c_void_p),
                ("mlp_w", C.c_void_p), ("base_color", C.c_void_p), ("features", C.c_void_p),
                ("preact", C.c_void_p), ("lobes", C.c_void_p), ("sh_y0_folded", C.c_int32),
                ("neural_layers", C.c_int32), ("neural_width", C.c_int32), ("neural_raw16", C.c_int32)]


class Preprocessed(C.Structure):
    _fields_ = [("splats", C.c_void_p), ("tiles_touched", C.c_void_p), ("depth_key", C.c_void_p),
                ("num_pairs", C.c_void_p), ("color_jac", C.c_void_p)]


class Grads(C.Structure):
    _fields_ = [("dmeans", C.c_void_p), ("dlog_scales", C.c_void_p), ("dquats", C.c_void_p),
                ("dopacity_logits", C.c_void_p), ("dsh", C.c_void_p), ("dlatent", C.c_void_p),
                ("dmlp_w", C.c_void_p), ("dmean2d", C.c_void_p), ("dbase_color", C.c_void_p),
                ("dfeatures", C.c_void_p), ("dlobes", C.c_void_p)]


class AdamTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("exp_avg", C.c_void_p), ("exp_avg_sq", C.c_void_p),
                ("param_half", C.c_void_p), ("n", C.c_int64), ("rows", C.c_int32), ("beta2", C.c_float),
                ("lr", C.POINTER(C.c_float))]


class Linear(C.Structure):
    _fields_ = [("type", C.c_int32), ("act", C.c_int32), ("rows", C.c_int64), ("n_in", C.c_int64),
                ("n_out", C.c_int64), ("x", C.c_void_p), ("w", C.c_void_p), ("bias", C.c_void_p), ("ldx", C.c_int64),
                ("ldw", C.c_int64)]


class GradTensor(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("type", C.c_int32)]


class Experts(C.Structure):
    _fields_ = [("layer", Linear), ("experts", C.c_int64), ("w_stride", C.c_int64), ("offsets", C.c_void_p)]


class RowOrderArrays(C.Structure):
    _fields_ = [("count", C.c_int64), ("groups", C.c_int64), ("order", C.c_void_p), ("sorted", C.c_void_p),
                ("place", C.c_void_p), ("offsets", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libgsraster.so is not built (python -m paper_2609_05255_amd.build)")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_size_t
        P = C.POINTER
        L.gs_preprocess.argtypes = [P(Camera), P(Gaussians), P(Appearance), P(Preprocessed), P(u64), vp, sz, vp]
        L.gs_preprocess_noalloc.argtypes = [P(Camera), P(Gaussians), P(Appearance), P(Preprocessed), P(u64), vp]
        L.gs_bin_sort.argtypes = [P(Camera), P(Preprocessed), i64, u64, u64, vp, vp, vp, vp, sz, vp]
        L.gs_render_fwd.argtypes = [P(Camera), P(Preprocessed), i64, vp, vp, vp, vp, vp, vp]
        L.gs_render_work.argtypes = [P(Camera), P(Preprocessed), i64, vp, vp, vp, vp]
        L.gs_render_bwd.argtypes = [P(Camera), P(Gaussians), P(Appearance), P(Preprocessed), vp, vp, vp, vp, vp,
                                    P(Grads), vp, sz, vp]
        L.gs_workspace_size.argtypes = [i64, i32, i32, u64, i32, P(sz)]
        L.gs_mlp_eval.argtypes = [vp, i64, vp, vp, vp]
        L.gs_neural_fold.argtypes = [vp, vp, i64, vp, vp]
        L.gs_adam_step.argtypes = [P(AdamTensor), i32, C.c_float, C.c_float, i64, vp]
        L.gs_adam_step_scaled.argtypes = [P(AdamTensor), i32, C.c_float, C.c_float, i64, vp, vp]
        L.gs_layer_norm_fwd.argtypes = [i32, i64, i64, vp, i64, vp, vp, C.c_float, vp, i64, vp, vp, vp]
        L.gs_layer_norm_bwd.argtypes = [i32, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz,
                                        vp]
        L.gs_layer_norm_workspace_size.argtypes = [i32, i64, i64, P(sz)]
        L.gs_linear_fwd.argtypes = [P(Linear), vp, i64, vp, i64, vp, i64, vp, sz, vp]
        L.gs_linear_bwd.argtypes = [P(Linear), vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, vp, sz, vp]
        L.gs_linear_workspace_size.argtypes = [i32, i32, i64, i64, i64, i32, P(sz)]
        L.gs_grad_norm.argtypes = [P(GradTensor), i32, C.c_float, vp, vp, sz, vp]
        L.gs_grad_clip.argtypes = [P(GradTensor), i32, C.c_float, vp, vp, sz, vp]
        L.gs_grad_workspace_size.argtypes = [P(GradTensor), i32, P(sz)]
        O = P(RowOrderArrays)
        L.gs_sort_rows.argtypes = [vp, O, vp, sz, vp]
        L.gs_sort_rows_workspace_size.argtypes = [i64, i64, P(sz)]
        L.gs_embedding_fwd.argtypes = [i32, i64, i64, i64, vp, i64, vp, C.c_float, vp, i64, vp]
        L.gs_embedding_bwd.argtypes = [i32, i64, vp, i64, O, C.c_float, vp, i64, i32, vp, sz, vp]
        L.gs_embedding_workspace_size.argtypes = [i32, i64, i64, P(sz)]
        L.gs_route_fwd.argtypes = [i32, i64, i64, i32, vp, i64, i32, vp, vp, vp]
        L.gs_route_bwd.argtypes = [i32, i64, i64, i32, vp, vp, i64, vp, vp, i32, vp, i64, vp]
        L.gs_dispatch_fwd.argtypes = [i32, i64, i64, vp, i64, O, vp, i64, vp]
        L.gs_dispatch_bwd.argtypes = [i32, i64, i64, vp, i64, O, vp, i64, vp, i64, vp]
        L.gs_combine_fwd.argtypes = [i32, i64, i64, vp, i64, O, vp, vp, i64, vp, i64, vp]
        L.gs_combine_bwd.argtypes = [i32, i64, i64, vp, i64, vp, i64, O, vp, vp, i64, vp, vp]
        L.gs_experts_fwd.argtypes = [P(Experts), vp, i64, vp, i64, vp, sz, vp]
        L.gs_experts_bwd.argtypes = [P(Experts), vp, i64, vp, i64, vp, i64, vp, i64, i64, i32, vp, vp, sz, vp]
        L.gs_experts_workspace_size.argtypes = [i32, i32, i64, i64, i64, i64, i32, P(sz)]
        L.gs_render_bwd_adam.argtypes = [P(Camera), P(Gaussians), P(Appearance), P(Preprocessed), vp, vp, vp, vp,
                                         vp, P(Grads), P(AdamTensor), C.c_float, C.c_float, i64, vp, sz, vp]
        L.gs_timer_create.argtypes = [P(vp)]
        L.gs_timer_destroy.argtypes = [vp]
        L.gs_timer_attach.argtypes = [vp]
        L.gs_timer_reset.argtypes = [vp]
        L.gs_timer_read.argtypes = [vp, P(C.c_double), P(i64), i32]
        for f in ("gs_preprocess", "gs_preprocess_noalloc", "gs_bin_sort", "gs_render_fwd", "gs_render_work",
                  "gs_render_bwd", "gs_render_bwd_adam", "gs_workspace_size", "gs_mlp_eval", "gs_neural_fold",
                  "gs_adam_step", "gs_adam_step_scaled", "gs_layer_norm_fwd", "gs_layer_norm_bwd",
                  "gs_layer_norm_workspace_size", "gs_linear_fwd", "gs_linear_bwd", "gs_linear_workspace_size",
                  "gs_grad_norm", "gs_grad_clip", "gs_grad_workspace_size", "gs_sort_rows", "gs_sort_rows_workspace_size",
                  "gs_embedding_fwd", "gs_embedding_bwd", "gs_embedding_workspace_size", "gs_route_fwd", "gs_route_bwd",
                  "gs_dispatch_fwd", "gs_dispatch_bwd", "gs_combine_fwd", "gs_combine_bwd", "gs_experts_fwd",
                  "gs_experts_bwd", "gs_experts_workspace_size", "gs_timer_create", "gs_timer_destroy", "gs_timer_attach", "gs_timer_reset",
                  "gs_timer_read"):
            getattr(L, f).restype = C.c_int
        L.gs_last_error.restype = C.c_char_p
        L.gs_version.restype = C.c_char_p
        L.gs_kernel_name.restype = C.c_char_p
        L.gs_kernel_name.argtypes = [i32]
        _lib = L
    return _lib


def _check(status: int):
    if status != GS_OK:
        raise GsError(status, lib().gs_last_error().decode())


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return C.c_void_p(t.data_ptr())


# The current stream's handle without an object around it, where this torch has the call (0.1 us instead of 2.7)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:
            return C.c_void_p(_raw_stream(torch.cuda.current_device()))
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, torch.cuda.Stream):
        return C.c_void_p(stream.cuda_stream)
    return C.c_void_p(stream)


def camera_struct(cam) -> Camera:
    c = Camera()
    vm = [float(v) for v in list(cam.viewmat.reshape(-1))]
    for k in range(12):
        c.viewmat[k] = vm[k]
    for k in range(3):
        c.campos[k] = float(cam.campos[k])
        c.bg[k] = float(cam.bg[k])
    c.fx, c.fy, c.cx, c.cy = float(cam.fx), float(cam.fy), float(cam.cx), float(cam.cy)
    c.width, c.height = int(cam.width), int(cam.height)
    c.near_plane = float(cam.near)
    return c


class SceneTensors:
    """Scene parameters resident on the GPU (planar, contiguous)."""

    def __init__(self, scene, device="cuda"):
        f32 = lambda a: torch.from_numpy(a).to(device=device, dtype=torch.float32).contiguous()
        h16 = lambda a: torch.from_numpy(a.view("int16")).to(device=device).contiguous()
        self.n = int(scene.n)
        self.means = f32(scene.means)
        self.log_scales = f32(scene.log_scales)
        self.quats = f32(scene.quats)
        self.opacity_logits = f32(scene.opacity_logits)
        self.sh = f32(scene.sh) if getattr(scene, "sh", None) is not None else None
        self.latent = h16(scene.latent) if getattr(scene, "latent", None) is not None else None
        self.mlp_w = h16(scene.mlp_w) if getattr(scene, "mlp_w", None) is not None else None
        self.base_color = f32(scene.base_color) if getattr(scene, "base_color", None) is not None else None
        self.features = h16(scene.features) if getattr(scene, "features", None) is not None else None
        self.neural_w = h16(scene.neural_w) if getattr(scene, "neural_w", None) is not None else None
        self.preact = None   # [n][16] binary16 pre-activations of the folded form (fold_neural)
        self.sh_y0_folded = bool(getattr(scene, "sh_y0_folded", False))
        self.neural_arch = getattr(scene, "neural_arch", None)
        self.lobes = f32(scene.lobes) if getattr(scene, "lobes", None) is not None else None
        self.lobes_gabor = f32(scene.lobes_gabor) if getattr(scene, "lobes_gabor", None) is not None else None

    def fold_neural(self, stream=None):
        """Computes the folded form's per-Gaussian pre-activations (gs_neural_fold)."""
        if self.preact is None:
            self.preact = torch.empty((self.n, 16), dtype=torch.int16, device=self.features.device)
        gs_neural_fold(self.features, self.neural_w, self.n, self.preact, stream)
        return self.preact

    def gaussians(self) -> Gaussians:
        return Gaussians(self.n, _ptr(self.means), _ptr(self.log_scales), _ptr(self.quats),
                         _ptr(self.opacity_logits))

    def appearance(self, kind: int, sh_degree: int = 3) -> Appearance:
        if kind == GS_APP_NEURAL:
            layers, width, raw16 = self.neural_arch if self.neural_arch is not None else (0, 0, 0)
            return Appearance(kind, sh_degree, None, None, _ptr(self.neural_w), _ptr(self.base_color),
                              _ptr(self.features), None, None, 0, layers, width, raw16)
        if kind == GS_APP_NEURAL_FOLDED:
            if self.preact is None:
                raise RuntimeError("fold_neural() first: the folded form reads its pre-activations")
            return Appearance(kind, sh_degree, None, None, _ptr(self.neural_w), _ptr(self.base_color), None,
                              _ptr(self.preact), None)
        if kind in LOBE_ROWS:
            lobes = self.lobes_gabor if kind == GS_APP_NASGABOR else self.lobes
            return Appearance(kind, sh_degree, None, None, None, _ptr(self.base_color), None, None, _ptr(lobes))
        return Appearance(kind, sh_degree, _ptr(self.sh), _ptr(self.latent), _ptr(self.mlp_w), None, None, None,
                          None, int(self.sh_y0_folded))


def gs_workspace_size(n: int, width: int, height: int, capacity: int, kind: int) -> int:
    out = C.c_size_t(0)
    _check(lib().gs_workspace_size(n, width, height, capacity, kind, C.byref(out)))
    return out.value


def gs_preprocess(cam: Camera, g: Gaussians, app: Appearance, pre: Preprocessed, workspace, ws_bytes: int,
                  stream=None, sync_pairs: bool = True):
    p = C.c_uint64(0)
    _check(lib().gs_preprocess(C.byref(cam), C.byref(g), C.byref(app), C.byref(pre),
                               C.byref(p) if sync_pairs else None, _ptr(workspace), ws_bytes, _stream(stream)))
    return p.value if sync_pairs else None


def gs_preprocess_noalloc(cam: Camera, g: Gaussians, app: Appearance, pre: Preprocessed, stream=None,
                          sync_pairs: bool = True):
    """gs_preprocess without a workspace (the library's static per-GPU scratch)."""
    p = C.c_uint64(0)
    _check(lib().gs_preprocess_noalloc(C.byref(cam), C.byref(g), C.byref(app), C.byref(pre),
                                       C.byref(p) if sync_pairs else None, _stream(stream)))
    return p.value if sync_pairs else None


def gs_bin_sort(cam: Camera, pre: Preprocessed, n: int, num_pairs: int, capacity: int, values, tile_ids,
                tile_ranges, workspace, ws_bytes: int, stream=None):
    _check(lib().gs_bin_sort(C.byref(cam), C.byref(pre), n, num_pairs, capacity, _ptr(values), _ptr(tile_ids),
                             _ptr(tile_ranges), _ptr(workspace), ws_bytes, _stream(stream)))


def gs_render_fwd(cam: Camera, pre: Preprocessed, n: int, values, tile_ranges, image, final_T, n_contrib,
                  stream=None):
    _check(lib().gs_render_fwd(C.byref(cam), C.byref(pre), n, _ptr(values), _ptr(tile_ranges), _ptr(image),
                               _ptr(final_T), _ptr(n_contrib), _stream(stream)))


def gs_render_work(cam: Camera, pre: Preprocessed, n: int, values, tile_ranges, counts, stream=None):
    """counts: int64 device tensor [5] (blended, listed, evaluated backward, evaluated forward,
    visited forward)."""
    _check(lib().gs_render_work(C.byref(cam), C.byref(pre), n, _ptr(values), _ptr(tile_ranges), _ptr(counts),
                                _stream(stream)))


def gs_render_bwd(cam: Camera, g: Gaussians, app: Appearance, pre: Preprocessed, values, tile_ranges, final_T,
                  n_contrib, dL_dimage, grads: Grads, workspace, ws_bytes: int, stream=None):
    _check(lib().gs_render_bwd(C.byref(cam), C.byref(g), C.byref(app), C.byref(pre), _ptr(values),
                               _ptr(tile_ranges), _ptr(final_T), _ptr(n_contrib), _ptr(dL_dimage), C.byref(grads),
                               _ptr(workspace), ws_bytes, _stream(stream)))


def gs_mlp_eval(x, rows: int, mlp_w, colors, stream=None):
    _check(lib().gs_mlp_eval(_ptr(x), rows, _ptr(mlp_w), _ptr(colors), _stream(stream)))


def gs_neural_fold(features, neural_w, n: int, preact, stream=None):
    _check(lib().gs_neural_fold(_ptr(features), _ptr(neural_w), n, _ptr(preact), _stream(stream)))


def _adam_tensors(tensors):
    arr = (AdamTensor * max(1, len(tensors)))()
    keep = []
    for k, t in enumerate(tensors):
        lr = None
        if t["lr"] is not None:
            if len(t["lr"]) < int(t["rows"]):
                raise ValueError("lr needs one entry per row")
            lr = (C.c_float * len(t["lr"]))(*[float(x) for x in t["lr"]])
            keep.append(lr)
        arr[k] = AdamTensor(_ptr(t["param"]), _ptr(t.get("grad")), _ptr(t["exp_avg"]), _ptr(t["exp_avg_sq"]),
                            _ptr(t.get("param_half")), int(t["n"]), int(t["rows"]), float(t["beta2"]),
                            C.cast(lr, C.POINTER(C.c_float)) if lr is not None else None)
    return arr, keep


def gs_adam_step(tensors, beta1: float, eps: float, step: int, stream=None, grad_scale=None):
    """tensors: list of dicts with param, grad, exp_avg, exp_avg_sq (device fp32 [rows][n]), optional
    param_half (device int16/uint16 [rows][n]), rows, n, beta2 and lr (a sequence of `rows` floats).
    grad_scale: optional device fp32 value (gs_grad_norm's coefficient) that multiplies every gradient."""
    arr, keep = _adam_tensors(tensors)
    if grad_scale is None:
        _check(lib().gs_adam_step(arr, len(tensors), float(beta1), float(eps), int(step), _stream(stream)))
    else:
        if grad_scale.dtype != torch.float32 or grad_scale.numel() < 1 or not grad_scale.is_cuda:
            raise ValueError("grad_scale: a float32 value on the GPU expected")
        _check(lib().gs_adam_step_scaled(arr, len(tensors), float(beta1), float(eps), int(step), _ptr(grad_scale),
                                         _stream(stream)))


GS_RENDER_ADAM_TENSORS = 5


def gs_render_bwd_adam(cam: Camera, g: Gaussians, app: Appearance, pre: Preprocessed, values, tile_ranges, final_T,
                       n_contrib, dL_dimage, grads: Grads, tensors, beta1: float, eps: float, step: int, workspace,
                       ws_bytes: int, stream=None):
    """tensors: the GS_RENDER_ADAM_TENSORS per-Gaussian tensors (dicts as for gs_adam_step, grad unused) in
    the order means, log_scales, quats, opacity_logits, sh."""
    if len(tensors) != GS_RENDER_ADAM_TENSORS:
        raise ValueError("gs_render_bwd_adam takes %d tensors" % GS_RENDER_ADAM_TENSORS)
    arr, keep = _adam_tensors(tensors)
    _check(lib().gs_render_bwd_adam(C.byref(cam), C.byref(g), C.byref(app), C.byref(pre), _ptr(values),
                                    _ptr(tile_ranges), _ptr(final_T), _ptr(n_contrib), _ptr(dL_dimage),
                                    C.byref(grads), arr, float(beta1), float(eps), int(step), _ptr(workspace),
                                    ws_bytes, _stream(stream)))


# ---- row operators: layer norm, linear, gradient clipping ----------------------


def _type_id(t) -> int:
    k = TYPE_IDS.get(t.dtype)
    if k is None:
        raise ValueError("element type %s: float32, float16 or bfloat16 expected" % t.dtype)
    return k


def _matrix(name, t, rows, cols, dtype):
    """Address and row stride of a [rows][cols] matrix on the GPU, its columns next to each other."""
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols or t.dtype != dtype:
        raise ValueError("%s: %s of %s, a [%d][%d] matrix of %s expected" % (name, tuple(t.shape), t.dtype, rows, cols,
                                                                            dtype))
    if not t.is_cuda:
        raise ValueError("%s is not on the GPU" % name)
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError("%s: columns %d elements apart, neighbours expected" % (name, step))
    return t.data_ptr(), (ld if rows > 1 else cols)


def _vector(name, t, n):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s: a contiguous float32 array of %d values on the GPU expected" % (name, n))
    return t.data_ptr()


def _space(workspace):
    if workspace is None:
        return None, 0
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous tensor on the GPU expected")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _shape(name, t):
    if t.dim() != 2:
        raise ValueError("%s: a matrix expected, not %s" % (name, tuple(t.shape)))
    return t.shape


def gs_layer_norm_workspace_size(x) -> int:
    """Workspace bytes of gs_layer_norm_bwd for x's shape and type."""
    rows, dim = _shape("x", x)
    out = C.c_size_t(0)
    _check(lib().gs_layer_norm_workspace_size(_type_id(x), rows, dim, C.byref(out)))
    return out.value


def gs_layer_norm_fwd(x, w, b, eps: float, y, mean=None, rstd=None, stream=None):
    """Layer norm of each row of x into y (matrices of one type); w and b: float32 [dim] or None; mean and rstd:
    float32 [rows], kept for the backward."""
    rows, dim = _shape("x", x)
    px, ldx = _matrix("x", x, rows, dim, x.dtype)
    py, ldy = _matrix("y", y, rows, dim, x.dtype)
    _check(lib().gs_layer_norm_fwd(_type_id(x), rows, dim, px, ldx, _vector("w", w, dim), _vector("b", b, dim), eps, py,
                                   ldy, _vector("mean", mean, rows), _vector("rstd", rstd, rows), _stream(stream)))


def gs_layer_norm_bwd(dy, x, w, mean, rstd, dx, dw, db, workspace, add=None, stream=None):
    """Backward of gs_layer_norm_fwd: dx (plus `add`, a gradient of x's shape), and float32 dw, db (or None)."""
    rows, dim = _shape("x", x)
    t = x.dtype
    px, ldx = _matrix("x", x, rows, dim, t)
    pdy, lddy = _matrix("dy", dy, rows, dim, t)
    pdx, lddx = _matrix("dx", dx, rows, dim, t)
    padd, ldadd = (None, 0) if add is None else _matrix("add", add, rows, dim, t)
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_layer_norm_bwd(_type_id(x), rows, dim, pdy, lddy, px, ldx, _vector("w", w, dim),
                                   _vector("mean", mean, rows), _vector("rstd", rstd, rows), padd, ldadd, pdx, lddx,
                                   _vector("dw", dw, dim), _vector("db", db, dim), ws, ws_bytes, _stream(stream)))


def _activation(act) -> int:
    k = ACTIVATIONS.get(act)
    if k is None:
        raise ValueError("activation %r: one of %s expected" % (act, ", ".join(ACTIVATIONS)))
    return k


def gs_linear_workspace_size(x, w, act: str = "none", dw_type=torch.float32) -> int:
    """Workspace bytes of gs_linear_fwd and gs_linear_bwd for these shapes; dw_type: the weight gradient's type
    (float32: enough for one of x's type too; None: for the forward alone)."""
    rows, n_in = _shape("x", x)
    n_out = _shape("w", w)[0]
    out = C.c_size_t(0)
    _check(lib().gs_linear_workspace_size(_type_id(x), _activation(act), rows, n_in, n_out,
                                          -1 if dw_type is None else TYPE_IDS[dw_type], C.byref(out)))
    return out.value


def _layer(x, w, bias, act):
    rows, n_in = _shape("x", x)
    n_out = _shape("w", w)[0]
    px, ldx = _matrix("x", x, rows, n_in, x.dtype)
    pw, ldw = _matrix("w", w, n_out, n_in, x.dtype)
    return Linear(_type_id(x), _activation(act), rows, n_in, n_out, px, pw, _vector("bias", bias, n_out), ldx, ldw)


def gs_linear_fwd(x, w, bias, y, workspace=None, act: str = "none", residual=None, z=None, stream=None):
    """y = act(x w^T + bias) + residual; w: [out][in] of x's type, bias: float32 [out] or None; z, if given, receives
    x w^T + bias for the backward."""
    p = _layer(x, w, bias, act)
    rows, n_out, t = p.rows, p.n_out, x.dtype
    py, ldy = _matrix("y", y, rows, n_out, t)
    pr, ldr = (None, 0) if residual is None else _matrix("residual", residual, rows, n_out, t)
    pz, ldz = (None, 0) if z is None else _matrix("z", z, rows, n_out, t)
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_linear_fwd(C.byref(p), pr, ldr, py, ldy, pz, ldz, ws, ws_bytes, _stream(stream)))


def gs_linear_bwd(dy, x, w, z, dx, dw, db, workspace, act: str = "none", stream=None):
    """Backward of gs_linear_fwd: dx of x's type, dw float32 or of x's type, db float32 (each may be None); z as the
    forward wrote it (None without an activation)."""
    p = _layer(x, w, None, act)
    rows, n_in, n_out, t = p.rows, p.n_in, p.n_out, x.dtype
    pdy, lddy = _matrix("dy", dy, rows, n_out, t)
    pz, ldz = (None, 0) if z is None else _matrix("z", z, rows, n_out, t)
    pdx, lddx = (None, 0) if dx is None else _matrix("dx", dx, rows, n_in, t)
    pdw, lddw, dw_type = None, 0, 0
    if dw is not None:
        pdw, lddw = _matrix("dw", dw, n_out, n_in, torch.float32 if dw.dtype == torch.float32 else t)
        dw_type = TYPE_IDS[dw.dtype]
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_linear_bwd(C.byref(p), pdy, lddy, pz, ldz, pdx, lddx, pdw, lddw, dw_type, _vector("db", db, n_out),
                               ws, ws_bytes, _stream(stream)))


class GradSet:
    """The gradients of one global norm, as gs_grad_norm and gs_grad_clip take them: contiguous tensors of any element
    type, clipped in place or, where `out` has a float32 tensor for them, into that. Keeps the tensors alive; the
    values may change between calls, the storage may not."""

    def __init__(self, grads, out=None):
        self.grads = list(grads)
        self.out = [None] * len(self.grads) if out is None else list(out)
        if len(self.out) != len(self.grads):
            raise ValueError("out needs an entry for each gradient")
        self.array = (GradTensor * max(1, len(self.grads)))()
        for k, (g, o) in enumerate(zip(self.grads, self.out)):
            if not g.is_contiguous() or not g.is_cuda:
                raise ValueError("gradient %d: a contiguous tensor on the GPU expected" % k)
            if o is not None:
                _vector("out %d" % k, o, g.numel())
            self.array[k] = GradTensor(g.data_ptr(), None if o is None else o.data_ptr(), g.numel(), _type_id(g))


def gs_grad_workspace_size(grads: GradSet) -> int:
    out = C.c_size_t(0)
    _check(lib().gs_grad_workspace_size(grads.array, len(grads.grads), C.byref(out)))
    return out.value


def gs_grad_norm(grads: GradSet, max_norm: float, result, workspace, stream=None):
    """result (float32 [2] on the GPU) = the global norm and the coefficient min(1, max_norm / (norm + 1e-6))."""
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_grad_norm(grads.array, len(grads.grads), max_norm, _vector("result", result, 2), ws, ws_bytes,
                              _stream(stream)))


def gs_grad_clip(grads: GradSet, max_norm: float, result, workspace, stream=None):
    """gs_grad_norm, and every gradient times the coefficient, in place or into the set's `out`."""
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_grad_clip(grads.array, len(grads.grads), max_norm, _vector("result", result, 2), ws, ws_bytes,
                              _stream(stream)))


# ---- codebooks and mixtures: rows by key, lookup, routing, rows to experts and back ----


def _array(name, t, shape, dtype):
    """Address of a contiguous array of this shape and type on the GPU."""
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or not t.is_cuda:
        raise ValueError("%s: %s of %s, a contiguous %s of %s on the GPU expected" % (name, tuple(t.shape), t.dtype,
                                                                                      tuple(shape), dtype))
    return t.data_ptr()


def _one_device(*tensors):
    """The launches go to the current device: all tensors (None: left out) have to be there."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device and t.is_cuda:
            raise ValueError("a tensor on %s while the current device is %d" % (t.device, device))


def _order_array(name):
    def get(self):
        return self._tensors[name]

    def put(self, t):
        n = self.groups + 1 if name == "offsets" else self.count
        address = None if t is None else _array(name, t, (n,), torch.int32)
        devices = {o.device for o in (*self._tensors.values(), t) if o is not None}
        if len(devices) > 1:
            raise ValueError("%s: the arrays of an order are on one device" % name)
        self._tensors[name] = t
        setattr(self._arrays, name, address)

    return property(get, put)


class RowOrder:
    """The order of `count` positions by their group (gs_row_order): int32 tensors order, sorted, place and offsets,
    which gs_sort_rows fills. sorted is what gs_embedding_bwd needs, place what rows on their way back from experts do;
    either may be left out. A tensor may be put in the place of one of them; its storage may not change after that."""

    order, sorted = _order_array("order"), _order_array("sorted")
    place, offsets = _order_array("place"), _order_array("offsets")
    count, groups = property(lambda self: self._arrays.count), property(lambda self: self._arrays.groups)

    def __init__(self, count: int, groups: int, device="cuda", sorted: bool = True, place: bool = True):
        self._tensors, self._arrays = dict.fromkeys(("order", "sorted", "place", "offsets")), RowOrderArrays()
        self._arrays.count, self._arrays.groups = int(count), int(groups)
        ints = lambda n: torch.empty(n, dtype=torch.int32, device=device)  # noqa: E731
        self.order, self.offsets = ints(self.count), ints(self.groups + 1)
        if sorted:
            self.sorted = ints(self.count)
        if place:
            self.place = ints(self.count)


def gs_sort_rows_workspace_size(order: RowOrder) -> int:
    out = C.c_size_t(0)
    _check(lib().gs_sort_rows_workspace_size(order.count, order.groups, C.byref(out)))
    return out.value


def gs_sort_rows(group_of, order: RowOrder, workspace=None, stream=None):
    """Fills `order` from the groups of its positions (a contiguous int32 tensor of order.count values, of any shape);
    values outside [0, order.groups) are no group."""
    if group_of.numel() != order.count:
        raise ValueError("group_of: %d values, %d expected" % (group_of.numel(), order.count))
    _one_device(group_of, order.offsets, workspace)
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_sort_rows(_array("group_of", group_of, group_of.shape, torch.int32), C.byref(order._arrays), ws,
                              ws_bytes, _stream(stream)))


def gs_embedding_fwd(table, index, scale: float, y, stream=None):
    """y[i] = scale * table[index[i]] (matrices of one type, index int32 [rows]); zero where the index is none of the
    table's."""
    entries, dim = _shape("table", table)
    rows = index.numel()
    _one_device(table, index, y)
    pt, ldt = _matrix("table", table, entries, dim, table.dtype)
    py, ldy = _matrix("y", y, rows, dim, table.dtype)
    _check(lib().gs_embedding_fwd(_type_id(table), rows, dim, entries, pt, ldt,
                                  _array("index", index, (rows,), torch.int32), scale, py, ldy, _stream(stream)))


def gs_embedding_workspace_size(dy) -> int:
    """Workspace bytes of gs_embedding_bwd for dy's shape and type."""
    rows, dim = _shape("dy", dy)
    out = C.c_size_t(0)
    _check(lib().gs_embedding_workspace_size(_type_id(dy), rows, dim, C.byref(out)))
    return out.value


def gs_embedding_bwd(dy, order: RowOrder, scale: float, dtable, workspace, stream=None):
    """dtable[v] = scale times the sum of dy's rows with index v, dtable float32 or of dy's type; order: the rows sorted
    by index, with `sorted`."""
    rows, dim = _shape("dy", dy)
    if rows != order.count:
        raise ValueError("dy: %d rows, %d sorted" % (rows, order.count))
    _one_device(dy, order.offsets, dtable, workspace)
    pdy, lddy = _matrix("dy", dy, rows, dim, dy.dtype)
    out_type = torch.float32 if dtable.dtype == torch.float32 else dy.dtype
    pdt, lddt = _matrix("dtable", dtable, order.groups, dim, out_type)
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_embedding_bwd(_type_id(dy), dim, pdy, lddy, C.byref(order._arrays), scale, pdt, lddt,
                                  TYPE_IDS[out_type], ws, ws_bytes, _stream(stream)))


def gs_route_fwd(logits, expert, weight, normalise: bool = True, stream=None):
    """The experts (int32 [rows][k]) of each row's k largest logits and their weights (float32 [rows][k]): the softmax
    over the chosen ones (normalise) or over all."""
    rows, experts = _shape("logits", logits)
    k = _shape("expert", expert)[1]
    _one_device(logits, expert, weight)
    pl, ldl = _matrix("logits", logits, rows, experts, logits.dtype)
    _check(lib().gs_route_fwd(_type_id(logits), rows, experts, k, pl, ldl, int(normalise),
                              _array("expert", expert, (rows, k), torch.int32),
                              _array("weight", weight, (rows, k), torch.float32), _stream(stream)))


def gs_route_bwd(dweight, logits, expert, weight, dlogits, normalise: bool = True, stream=None):
    """The logits' gradient from that of the weights; logits, expert and weight as gs_route_fwd took and wrote them."""
    rows, experts = _shape("dlogits", dlogits)
    k = _shape("expert", expert)[1]
    t = dlogits.dtype
    _one_device(dweight, logits, expert, weight, dlogits)
    pl, ldl = (None, 0) if logits is None else _matrix("logits", logits, rows, experts, t)
    pd, ldd = _matrix("dlogits", dlogits, rows, experts, t)
    _check(lib().gs_route_bwd(_type_id(dlogits), rows, experts, k,
                              _array("dweight", dweight, (rows, k), torch.float32), pl, ldl,
                              _array("expert", expert, (rows, k), torch.int32),
                              _array("weight", weight, (rows, k), torch.float32), int(normalise), pd, ldd,
                              _stream(stream)))


def _choices(name, t, rows, order: RowOrder):
    """Address of a float32 [rows][choices] array."""
    if rows == 0:
        return None
    return _array(name, t, (rows, order.count // rows), torch.float32)


def gs_dispatch_fwd(x, order: RowOrder, xs, stream=None):
    """xs[p] = x[order[p] // k]: x [rows][dim] copied to where its k choices are sorted; xs [order.count][dim], rows
    behind the last place in use stay as they are."""
    rows, dim = _shape("x", x)
    _one_device(x, order.offsets, xs)
    px, ldx = _matrix("x", x, rows, dim, x.dtype)
    pxs, ldxs = _matrix("xs", xs, order.count, dim, x.dtype)
    _check(lib().gs_dispatch_fwd(_type_id(x), rows, dim, px, ldx, C.byref(order._arrays), pxs, ldxs, _stream(stream)))


def gs_dispatch_bwd(dxs, order: RowOrder, dx, add=None, stream=None):
    """dx[i] = the sum of dxs over the places of row i's choices, plus `add`, a gradient of dx's shape."""
    rows, dim = _shape("dx", dx)
    t = dx.dtype
    _one_device(dxs, order.offsets, dx, add)
    ps, lds = _matrix("dxs", dxs, order.count, dim, t)
    pa, lda = (None, 0) if add is None else _matrix("add", add, rows, dim, t)
    pd, ldd = _matrix("dx", dx, rows, dim, t)
    _check(lib().gs_dispatch_bwd(_type_id(dx), rows, dim, ps, lds, C.byref(order._arrays), pa, lda, pd, ldd,
                                 _stream(stream)))


def gs_combine_fwd(ys, order: RowOrder, weight, y, residual=None, stream=None):
    """y[i] = the sum over row i's choices of weight (float32 [rows][k]) times their rows of ys, plus the residual."""
    rows, dim = _shape("y", y)
    t = y.dtype
    _one_device(ys, order.offsets, weight, y, residual)
    ps, lds = _matrix("ys", ys, order.count, dim, t)
    pr, ldr = (None, 0) if residual is None else _matrix("residual", residual, rows, dim, t)
    py, ldy = _matrix("y", y, rows, dim, t)
    _check(lib().gs_combine_fwd(_type_id(y), rows, dim, ps, lds, C.byref(order._arrays),
                                _choices("weight", weight, rows, order), pr, ldr, py, ldy, _stream(stream)))


def gs_combine_bwd(dy, ys, order: RowOrder, weight, dys, dweight, stream=None):
    """Backward of gs_combine_fwd: dys of ys's shape (rows behind the last place in use stay as they are) and dweight
    (float32 [rows][k])."""
    rows, dim = _shape("dy", dy)
    t = dy.dtype
    _one_device(dy, ys, order.offsets, weight, dys, dweight)
    pdy, lddy = _matrix("dy", dy, rows, dim, t)
    ps, lds = _matrix("ys", ys, order.count, dim, t)
    pd, ldd = _matrix("dys", dys, order.count, dim, t)
    _check(lib().gs_combine_bwd(_type_id(dy), rows, dim, pdy, lddy, ps, lds, C.byref(order._arrays),
                                _choices("weight", weight, rows, order), pd, ldd,
                                _choices("dweight", dweight, rows, order), _stream(stream)))


def _stack(name, t, shape, dtype):
    """Address, row stride and stride between the matrices of an [experts][rows][cols] tensor on the GPU."""
    if t.shape != shape or t.dtype != dtype or not t.is_cuda:
        raise ValueError("%s: %s of %s, %s of %s on the GPU expected" % (name, tuple(t.shape), t.dtype, tuple(shape),
                                                                        dtype))
    _, rows, cols = shape
    stride, ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError("%s: columns %d elements apart, neighbours expected" % (name, step))
    return t.data_ptr(), (ld if rows > 1 else cols), stride


def _experts(x, offsets, w, bias, act):
    rows, n_in = _shape("x", x)
    if w.dim() != 3:
        raise ValueError("w: [experts][out][in] expected, not %s" % (tuple(w.shape),))
    experts, n_out, _ = w.shape
    px, ldx = _matrix("x", x, rows, n_in, x.dtype)
    pw, ldw, stride = _stack("w", w, (experts, n_out, n_in), x.dtype)
    pb = None if bias is None else _array("bias", bias, (experts, n_out), torch.float32)
    po = _array("offsets", offsets, (experts + 1,), torch.int32)
    return Experts(Linear(_type_id(x), _activation(act), rows, n_in, n_out, px, pw, pb, ldx, ldw), experts, stride, po)


def gs_experts_workspace_size(x, w, act: str = "none", dw_type=torch.float32) -> int:
    """Workspace bytes of gs_experts_fwd and gs_experts_bwd for these shapes; dw_type: the weight gradient's type
    (float32: enough for one of x's type too; None: for the forward alone)."""
    rows, n_in = _shape("x", x)
    out = C.c_size_t(0)
    _check(lib().gs_experts_workspace_size(_type_id(x), _activation(act), rows, w.shape[0], n_in, w.shape[1],
                                           -1 if dw_type is None else TYPE_IDS[dw_type], C.byref(out)))
    return out.value


def gs_experts_fwd(x, offsets, w, bias, y, workspace=None, act: str = "none", z=None, stream=None):
    """y = act(x w[e]^T + bias[e]) for the rows offsets[e] .. offsets[e + 1] - 1 of every expert e; x: [rows][in] sorted
    by expert, offsets: int32 [experts + 1] (RowOrder.offsets), w: [experts][out][in] of x's type, bias: float32
    [experts][out] or None; z, if given, receives what the activation takes, for the backward. Rows that are no expert's
    stay as they are."""
    _one_device(x, offsets, w, bias, y, workspace, z)
    p = _experts(x, offsets, w, bias, act)
    rows, n_out, t = p.layer.rows, p.layer.n_out, x.dtype
    py, ldy = _matrix("y", y, rows, n_out, t)
    pz, ldz = (None, 0) if z is None else _matrix("z", z, rows, n_out, t)
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_experts_fwd(C.byref(p), py, ldy, pz, ldz, ws, ws_bytes, _stream(stream)))


def gs_experts_bwd(dy, x, offsets, w, z, dx, dw, db, workspace, act: str = "none", stream=None):
    """Backward of gs_experts_fwd: dx of x's type, dw [experts][out][in] float32 or of x's type, db float32
    [experts][out] (each may be None); z as the forward wrote it (None without an activation)."""
    _one_device(dy, x, offsets, w, z, dx, dw, db, workspace)
    p = _experts(x, offsets, w, None, act)
    rows, n_in, n_out, t = p.layer.rows, p.layer.n_in, p.layer.n_out, x.dtype
    pdy, lddy = _matrix("dy", dy, rows, n_out, t)
    pz, ldz = (None, 0) if z is None else _matrix("z", z, rows, n_out, t)
    pdx, lddx = (None, 0) if dx is None else _matrix("dx", dx, rows, n_in, t)
    pdw, lddw, stride, dw_type = None, 0, 0, 0
    if dw is not None:
        pdw, lddw, stride = _stack("dw", dw, w.shape, torch.float32 if dw.dtype == torch.float32 else t)
        dw_type = TYPE_IDS[dw.dtype]
    pdb = None if db is None else _array("db", db, (p.experts, n_out), torch.float32)
    ws, ws_bytes = _space(workspace)
    _check(lib().gs_experts_bwd(C.byref(p), pdy, lddy, pz, ldz, pdx, lddx, pdw, lddw, stride, dw_type, pdb, ws, ws_bytes,
                                _stream(stream)))


class Timer:
    """A caller-owned kernel-timing context (gs_timer_*): while attached to the
    calling thread, every kernel the library launches from it is timed."""

    def __init__(self):
        h = C.c_void_p()
        _check(lib().gs_timer_create(C.byref(h)))
        self.handle = h

    def attach(self):
        _check(lib().gs_timer_attach(self.handle))

    @staticmethod
    def detach():
        _check(lib().gs_timer_attach(None))

    def reset(self):
        _check(lib().gs_timer_reset(self.handle))

    def read(self) -> dict:
        k = len(KERNEL_NAMES)
        ms = (C.c_double * k)()
        cnt = (C.c_int64 * k)()
        _check(lib().gs_timer_read(self.handle, ms, cnt, k))
        return {KERNEL_NAMES[i]: (ms[i], cnt[i]) for i in range(k)}

    def close(self):
        if self.handle:
            _check(lib().gs_timer_destroy(self.handle))
            self.handle = None


_timer = None


def timing_enable(on: bool = True):
    """Attaches (on) or detaches (off) this module's timer to the calling thread."""
    global _timer
    if on:
        if _timer is None:
            _timer = Timer()
        _timer.attach()
    else:
        Timer.detach()


def timing_reset():
    _timer.reset()


def timing_read() -> dict:
    return _timer.read()


class Frame:
    """Device buffers for rendering one image of a scene and its backward pass."""

    def __init__(self, n: int, width: int, height: int, kind: int, capacity: int, device="cuda",
                 want_tile_ids: bool = False, want_dmean2d: bool = False, neural_arch=None):
        self.n, self.width, self.height, self.kind, self.capacity = n, width, height, kind, capacity
        d = device
        nn = max(n, 1)
        self.tiles_x, self.tiles_y = (width + 15) // 16, (height + 15) // 16
        self.splats = torch.empty(nn * SPLAT_BYTES // 4, dtype=torch.float32, device=d)
        self.tiles_touched = torch.empty(nn, dtype=torch.int32, device=d)
        self.depth_key = torch.empty(nn, dtype=torch.int32, device=d)
        self.num_pairs = torch.zeros(1, dtype=torch.int64, device=d)
        self.values = torch.empty(max(capacity, 1), dtype=torch.int32, device=d)
        self.tile_ids = torch.empty(max(capacity, 1), dtype=torch.int32, device=d) if want_tile_ids else None
        self.ranges = torch.empty(self.tiles_x * self.tiles_y * 2, dtype=torch.int32, device=d)
        self.image = torch.empty(3, height, width, dtype=torch.float32, device=d)
        self.final_T = torch.empty(height, width, dtype=torch.float32, device=d)
        self.n_contrib = torch.empty(height, width, dtype=torch.int32, device=d)
        self.ws_bytes = gs_workspace_size(n, width, height, capacity, kind)
        self.workspace = torch.empty(max(self.ws_bytes, 256) // 4 + 64, dtype=torch.float32, device=d)
        self.dmeans = torch.empty(3, nn, device=d)
        self.dlog_scales = torch.empty(3, nn, device=d)
        self.dquats = torch.empty(4, nn, device=d)
        self.dopacity_logits = torch.empty(nn, device=d)
        self.dsh = torch.empty(48, nn, device=d) if kind == GS_APP_SH3 else None
        self.dlatent = torch.empty(14, nn, device=d) if kind == GS_APP_LATENT_MLP else None
        self.dmlp_w = (torch.empty(MLP_WEIGHTS, device=d) if kind == GS_APP_LATENT_MLP else
                       torch.empty(neural_weight_count(neural_arch), device=d) if kind == GS_APP_NEURAL else None)
        self.dmean2d = torch.empty(2, nn, device=d) if want_dmean2d else None
        self.dbase_color = torch.empty(3, nn, device=d) if kind in (GS_APP_NEURAL, *LOBE_ROWS) else None
        raw16 = neural_arch is not None and bool(neural_arch[2])
        self.dfeatures = torch.empty(16 if raw16 else NEURAL_FEATURES, nn, device=d) if kind == GS_APP_NEURAL else None
        self.dlobes = torch.empty(LOBE_ROWS[kind], nn, device=d) if kind in LOBE_ROWS else None
        # SH3: the colour's view-direction Jacobian, for the backward (gs_preprocessed.color_jac)
        self.color_jac = torch.empty(10 * nn, dtype=torch.float32, device=d) if kind == GS_APP_SH3 else None
        self.pre = Preprocessed(_ptr(self.splats), _ptr(self.tiles_touched), _ptr(self.depth_key),
                                _ptr(self.num_pairs), _ptr(self.color_jac))
        self.grads = Grads(_ptr(self.dmeans), _ptr(self.dlog_scales), _ptr(self.dquats),
                           _ptr(self.dopacity_logits), _ptr(self.dsh), _ptr(self.dlatent), _ptr(self.dmlp_w),
                           _ptr(self.dmean2d), _ptr(self.dbase_color), _ptr(self.dfeatures), _ptr(self.dlobes))
        self.last_pairs = 0

    def forward(self, cam: Camera, scene: SceneTensors, sh_degree: int = 3, stream=None,
                sync_pairs: bool = True):
        """Preprocess, bin-sort and blend one image. sync_pairs=True reads the
        pair count back to the host (and returns it) and fails with GS_ERR_CAPACITY
        before sorting if it exceeds the capacity; sync_pairs=False keeps the count
        on the device (no synchronisation): check pairs_overflowed() afterwards."""
        g, app = scene.gaussians(), scene.appearance(self.kind, sh_degree)
        P = gs_preprocess(cam, g, app, self.pre, self.workspace, self.ws_bytes, stream, sync_pairs=sync_pairs)
        gs_bin_sort(cam, self.pre, self.n, P if sync_pairs else GS_PAIRS_ON_DEVICE, self.capacity, self.values,
                    self.tile_ids, self.ranges, self.workspace, self.ws_bytes, stream)
        gs_render_fwd(cam, self.pre, self.n, self.values, self.ranges, self.image, self.final_T, self.n_contrib,
                      stream)
        self.last_pairs = P
        return P

    def pairs_overflowed(self) -> bool:
        """After a device-mode forward: did the pair count exceed the capacity (synchronises)?"""
        return int(self.num_pairs.item()) > self.capacity

    def backward(self, cam: Camera, scene: SceneTensors, dL_dimage, sh_degree: int = 3, stream=None):
        g, app = scene.gaussians(), scene.appearance(self.kind, sh_degree)
        gs_render_bwd(cam, g, app, self.pre, self.values, self.ranges, self.final_T, self.n_contrib, dL_dimage,
                      self.grads, self.workspace, self.ws_bytes, stream)

    def splat_fields(self) -> dict:
        """Host copy of the splat records, split into fields."""
        raw = self.splats.view(-1, 16).cpu()
        f = raw.numpy()
        w = SPLAT_WORDS
        rect = raw.view(torch.int32).numpy()[:, w["rect"]:w["rect"] + 2]
        r01, r23 = rect[:, 0].astype("int64") & 0xFFFFFFFF, rect[:, 1].astype("int64") & 0xFFFFFFFF
        import numpy as np
        rects = np.stack([r01 & 0xFFFF, r01 >> 16, r23 & 0xFFFF, r23 >> 16]).astype(np.int32)
        return dict(mean2d=f[:, w["mean_x"]:w["mean_y"] + 1].T.copy(), conic=f[:, w["conic_a"]:w["conic_c"] + 1].T.copy(),
                    opacity=f[:, w["opacity"]].copy(), color=f[:, w["color"]:w["color"] + 3].T.copy(),
                    power_min=f[:, w["power_min"]].copy(), ext=f[:, w["ext_x"]:w["ext_y"] + 1].T.copy(),
                    depth=f[:, w["depth"]].copy(), rect=rects)
