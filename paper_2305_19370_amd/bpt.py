"""ctypes binding of libbpt (argument marshalling only).

Every step of the layer runs inside libbpt's HIP kernels. This module only
mirrors the C structs of ``include/libbpt.h``, allocates the caller-owned
buffers with torch (device memory plumbing) and passes raw pointers plus the
current HIP stream. If the library is not built, loading fails loudly; there
is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Dict, List, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbpt.so")

BPT_F32, BPT_BF16 = 0, 1
BPT_GELU, BPT_RELU = 0, 1
STATUS = {0: "BPT_OK", 1: "BPT_ERR_INVALID_ARG", 2: "BPT_ERR_UNSUPPORTED", 3: "BPT_ERR_WORKSPACE",
          4: "BPT_ERR_HIP"}

c_i64, c_i32, c_f32, c_sz, c_vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p
c_f64 = ctypes.c_double


class Config(ctypes.Structure):
    _fields_ = [("B", c_i64), ("S", c_i64), ("D", c_i64), ("H", c_i64), ("F", c_i64), ("Bq", c_i64),
                ("Bkv", c_i64), ("causal", c_i32), ("dtype", c_i32), ("out_dtype", c_i32),
                ("group_blocks", c_i32), ("ln_eps", c_f32), ("activation", c_i32), ("dropout", c_f32),
                ("dropout_seed", ctypes.c_uint64)]


PARAM_FIELDS = ("ln1_g", "ln1_b", "Wq", "Wk", "Wv", "Wo", "ln2_g", "ln2_b", "W1", "b1", "W2", "b2")
GRAD_FIELDS = ("dln1_g", "dln1_b", "dWq", "dWk", "dWv", "dWo", "dln2_g", "dln2_b", "dW1", "db1", "dW2", "db2")
SAVED_FIELDS = ("qkv", "o", "lse", "h", "mu1", "rstd1", "mu2", "rstd2", "total")


class Params(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in PARAM_FIELDS]


class Grads(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in GRAD_FIELDS]


class SavedLayout(ctypes.Structure):
    _fields_ = [(n, c_sz) for n in SAVED_FIELDS]


class XentConfig(ctypes.Structure):
    _fields_ = [("T", c_i64), ("D", c_i64), ("V", c_i64), ("ldw", c_i64), ("block_rows", c_i64),
                ("dtype", c_i32), ("reserved", c_i32)]


class EmbedConfig(ctypes.Structure):
    _fields_ = [("B", c_i64), ("S", c_i64), ("D", c_i64), ("V", c_i64), ("dtype", c_i32), ("grad_dtype", c_i32)]


class LnConfig(ctypes.Structure):
    _fields_ = [("rows", c_i64), ("D", c_i64), ("eps", c_f32), ("in_dtype", c_i32), ("out_dtype", c_i32),
                ("reserved", c_i32)]


class AdamWConfig(ctypes.Structure):
    _fields_ = [("lr", c_f32), ("beta1", c_f32), ("beta2", c_f32), ("eps", c_f32), ("weight_decay", c_f32),
                ("lowp_dtype", c_i32), ("step", c_i64)]


class RopeConfig(ctypes.Structure):
    _fields_ = [("rows", c_i64), ("S", c_i64), ("H", c_i64), ("dh", c_i64), ("rot", c_i64), ("ldx", c_i64), ("ldy", c_i64),
                ("pos0", c_i64), ("orig_len", c_i64), ("theta", c_f64), ("factor", c_f64), ("beta_fast", c_f64),
                ("beta_slow", c_f64), ("mscale", c_f64), ("interleaved", c_i32), ("scaling", c_i32), ("dtype", c_i32),
                ("reserved", c_i32)]


class LayerOptions(ctypes.Structure):
    _fields_ = [("rot", c_i64), ("pos0", c_i64), ("orig_len", c_i64), ("theta", c_f64), ("factor", c_f64), ("beta_fast", c_f64),
                ("beta_slow", c_f64), ("mscale", c_f64), ("interleaved", c_i32), ("scaling", c_i32), ("window", c_i64),
                ("sinks", c_i64)]


class AttnStrides(ctypes.Structure):
    _fields_ = [("sb", c_i64), ("st", c_i64), ("sh", c_i64)]


class AttnConfig(ctypes.Structure):
    _fields_ = [("B", c_i64), ("Sq", c_i64), ("Skv", c_i64), ("Hq", c_i64), ("Hkv", c_i64), ("dh", c_i64), ("q", AttnStrides),
                ("k", AttnStrides), ("v", AttnStrides), ("o", AttnStrides), ("window", c_i64), ("sinks", c_i64), ("scale", c_f32),
                ("causal", c_i32), ("dtype", c_i32), ("reserved", c_i32)]


class AdamWTensor(ctypes.Structure):
    _fields_ = [("n", c_i64), ("p", c_vp), ("g", c_vp), ("m", c_vp), ("v", c_vp), ("exps", c_vp), ("p_lowp", c_vp),
                ("weight_decay", c_f64)]


class AdamWMultiConfig(ctypes.Structure):
    _fields_ = [("lr", c_f64), ("beta1", c_f64), ("beta2", c_f64), ("eps", c_f64), ("step", c_i64), ("seed", ctypes.c_uint64),
                ("state_bits", c_i32), ("grad_dtype", c_i32), ("lowp_dtype", c_i32), ("reserved", c_i32)]


EXPORTS = ("bpt_validate", "bpt_group_rows", "bpt_saved_bytes", "bpt_saved_layout_of", "bpt_workspace_bytes",
           "bpt_layer_fwd", "bpt_layer_bwd", "bpt_status_string", "bpt_last_error", "bpt_describe",
           "bpt_profile_enable", "bpt_profile_report", "bpt_xent_validate", "bpt_xent_workspace_bytes",
           "bpt_xent_fwd", "bpt_xent_bwd", "bpt_embed_fwd", "bpt_embed_bwd", "bpt_ln_workspace_bytes",
           "bpt_ln_fwd", "bpt_ln_bwd", "bpt_adamw_step", "bpt_bwd_qkv_grad_offset",
           "bpt_layer_fwd_noalloc", "bpt_rope_validate", "bpt_rope_fwd", "bpt_rope_bwd", "bpt_attn_validate",
           "bpt_attn_workspace_bytes", "bpt_attn_fwd", "bpt_attn_bwd", "bpt_adamw_multi", "bpt_layer_options_validate",
           "bpt_layer_fwd_options", "bpt_layer_bwd_options")

_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libbpt.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                           "(python -m paper_2305_19370_amd.build)")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    lib.bpt_validate.argtypes = [P(Config)]
    lib.bpt_validate.restype = c_i32
    lib.bpt_group_rows.argtypes = [P(Config)]
    lib.bpt_group_rows.restype = c_i64
    lib.bpt_saved_bytes.argtypes = [P(Config)]
    lib.bpt_saved_bytes.restype = c_sz
    lib.bpt_saved_layout_of.argtypes = [P(Config), P(SavedLayout)]
    lib.bpt_saved_layout_of.restype = c_i32
    lib.bpt_workspace_bytes.argtypes = [P(Config), c_i32]
    lib.bpt_workspace_bytes.restype = c_sz
    lib.bpt_layer_fwd.argtypes = [P(Config), c_vp, P(Params), c_vp, c_vp, c_vp, c_sz, c_vp]
    lib.bpt_layer_fwd.restype = c_i32
    lib.bpt_layer_fwd_noalloc.argtypes = [P(Config), c_vp, P(Params), c_vp, c_vp, c_vp]
    lib.bpt_layer_fwd_noalloc.restype = c_i32
    lib.bpt_layer_bwd.argtypes = [P(Config), c_vp, P(Params), c_vp, c_vp, c_vp, P(Grads), c_vp, c_sz, c_vp]
    lib.bpt_layer_bwd.restype = c_i32
    lib.bpt_bwd_qkv_grad_offset.argtypes = [P(Config), P(c_sz)]
    lib.bpt_bwd_qkv_grad_offset.restype = c_i32
    lib.bpt_status_string.argtypes = [c_i32]
    lib.bpt_status_string.restype = ctypes.c_char_p
    lib.bpt_last_error.argtypes = []
    lib.bpt_last_error.restype = ctypes.c_char_p
    lib.bpt_describe.argtypes = [P(Config), ctypes.c_char_p, c_sz]
    lib.bpt_describe.restype = c_sz
    lib.bpt_profile_enable.argtypes = [c_i32]
    lib.bpt_profile_enable.restype = c_i32
    lib.bpt_profile_report.argtypes = [ctypes.c_char_p, c_sz]
    lib.bpt_profile_report.restype = c_sz
    lib.bpt_xent_validate.argtypes = [P(XentConfig)]
    lib.bpt_xent_validate.restype = c_i32
    lib.bpt_xent_workspace_bytes.argtypes = [P(XentConfig), c_i32]
    lib.bpt_xent_workspace_bytes.restype = c_sz
    lib.bpt_xent_fwd.argtypes = [P(XentConfig), c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
    lib.bpt_xent_fwd.restype = c_i32
    lib.bpt_xent_bwd.argtypes = [P(XentConfig), c_vp, c_vp, c_vp, c_vp, c_f32, c_vp, c_vp, c_vp, c_sz, c_vp]
    lib.bpt_xent_bwd.restype = c_i32
    lib.bpt_embed_fwd.argtypes = [P(EmbedConfig), c_vp, c_vp, c_vp, c_vp, c_vp]
    lib.bpt_embed_fwd.restype = c_i32
    lib.bpt_embed_bwd.argtypes = [P(EmbedConfig), c_vp, c_vp, c_vp, c_vp, c_vp]
    lib.bpt_embed_bwd.restype = c_i32
    lib.bpt_ln_workspace_bytes.argtypes = [P(LnConfig)]
    lib.bpt_ln_workspace_bytes.restype = c_sz
    lib.bpt_ln_fwd.argtypes = [P(LnConfig), c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]
    lib.bpt_ln_fwd.restype = c_i32
    lib.bpt_ln_bwd.argtypes = [P(LnConfig), c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp]
    lib.bpt_ln_bwd.restype = c_i32
    lib.bpt_adamw_step.argtypes = [P(AdamWConfig), c_i64, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]
    lib.bpt_adamw_step.restype = c_i32
    lib.bpt_rope_validate.argtypes = [P(RopeConfig)]
    lib.bpt_rope_validate.restype = c_i32
    for fn in (lib.bpt_rope_fwd, lib.bpt_rope_bwd):
        fn.argtypes = [P(RopeConfig), c_vp, c_vp, c_vp, c_vp]
        fn.restype = c_i32
    lib.bpt_attn_validate.argtypes = [P(AttnConfig)]
    lib.bpt_attn_validate.restype = c_i32
    lib.bpt_attn_workspace_bytes.argtypes = [P(AttnConfig), c_i32]
    lib.bpt_attn_workspace_bytes.restype = c_sz
    lib.bpt_attn_fwd.argtypes = [P(AttnConfig)] + [c_vp] * 8 + [c_sz, c_vp]
    lib.bpt_attn_fwd.restype = c_i32
    lib.bpt_attn_bwd.argtypes = [P(AttnConfig)] + [c_vp] * 12 + [c_sz, c_vp]
    lib.bpt_attn_bwd.restype = c_i32
    lib.bpt_layer_options_validate.argtypes = [P(Config), P(LayerOptions)]
    lib.bpt_layer_options_validate.restype = c_i32
    lib.bpt_layer_fwd_options.argtypes = [P(Config), P(LayerOptions), c_vp, P(Params), c_vp, c_vp, c_vp, c_sz, c_vp]
    lib.bpt_layer_fwd_options.restype = c_i32
    lib.bpt_layer_bwd_options.argtypes = [P(Config), P(LayerOptions), c_vp, P(Params), c_vp, c_vp, c_vp, P(Grads), c_vp, c_sz, c_vp]
    lib.bpt_layer_bwd_options.restype = c_i32
    lib.bpt_adamw_multi.argtypes = [P(AdamWMultiConfig), P(AdamWTensor), c_i64, c_vp]
    lib.bpt_adamw_multi.restype = c_i32
    _lib = lib
    return lib


class BptError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


def _check(status: int) -> None:
    if status != 0:
        raise BptError(status, load().bpt_last_error().decode())


def make_config(B: int, S: int, D: int, H: int, F: int, Bq: int, Bkv: int, causal: bool = True,
                dtype: str = "bf16", out_dtype: Optional[str] = None, group_blocks: int = 0,
                ln_eps: float = 1e-5, activation: str = "gelu", dropout: float = 0.0,
                dropout_seed: int = 0) -> Config:
    dt = {"f32": BPT_F32, "bf16": BPT_BF16}
    act = {"gelu": BPT_GELU, "relu": BPT_RELU}
    return Config(B, S, D, H, F, Bq, Bkv, int(bool(causal)), dt[dtype], dt[out_dtype or dtype],
                  group_blocks, ln_eps, act[activation], dropout, dropout_seed & (2 ** 64 - 1))


def validate(cfg: Config) -> int:
    return load().bpt_validate(ctypes.byref(cfg))


def saved_bytes(cfg: Config) -> int:
    return load().bpt_saved_bytes(ctypes.byref(cfg))


def workspace_bytes(cfg: Config, backward: bool) -> int:
    return load().bpt_workspace_bytes(ctypes.byref(cfg), int(backward))


def group_rows(cfg: Config) -> int:
    return load().bpt_group_rows(ctypes.byref(cfg))


def saved_layout(cfg: Config) -> Dict[str, int]:
    out = SavedLayout()
    _check(load().bpt_saved_layout_of(ctypes.byref(cfg), ctypes.byref(out)))
    return {n: getattr(out, n) for n in SAVED_FIELDS}


def bwd_qkv_grad_offset(cfg: Config) -> int:
    off = c_sz()
    _check(load().bpt_bwd_qkv_grad_offset(ctypes.byref(cfg), ctypes.byref(off)))
    return off.value


def describe(cfg: Config) -> str:
    buf = ctypes.create_string_buffer(1024)
    load().bpt_describe(ctypes.byref(cfg), buf, 1024)
    return buf.value.decode()


def profile_enable(on: bool) -> None:
    _check(load().bpt_profile_enable(int(on)))


def profile_report() -> Dict[str, Dict[str, float]]:
    """Per call-site launch timings recorded since profile_enable(True); call after a
    device synchronisation."""
    import json
    lib = load()
    n = lib.bpt_profile_report(None, 0)
    buf = ctypes.create_string_buffer(n + 1)
    lib.bpt_profile_report(buf, n + 1)
    return json.loads(buf.value.decode())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _int32(t: Optional[torch.Tensor], n: int, name: str) -> Optional[int]:
    """The address of n contiguous int32 on the GPU, or None."""
    if t is None:
        return None
    if t.dtype != torch.int32 or t.numel() != n or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name} must be {n} contiguous int32 on the GPU")
    return t.data_ptr()


def _stream_on(dev: int, same: bool) -> int:
    """The current stream of the current GPU, where a call's kernels run. dev: the device of one of its tensors; same: whether the
    others are there too."""
    if dev < 0:
        raise ValueError("the tensors must be on the GPU")
    if not same or dev != torch._C._cuda_getDevice():
        raise ValueError(f"the tensors must be on the current device, cuda:{torch._C._cuda_getDevice()}")
    return torch._C._cuda_getCurrentRawStream(dev)


def _check_layout(t: torch.Tensor, layout: Tuple[torch.dtype, Tuple[int, ...], Tuple[int, ...]], name: str) -> None:
    """Raises unless a tensor has this type, shape and strides (those of dimensions of one element count for nothing)."""
    dtype, shape, strides = layout
    if t.dtype != dtype or t.shape != shape or any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), strides)):
        raise ValueError(f"{name} must be {shape} of {dtype} with strides {strides}, as the configuration has it; not "
                         f"{tuple(t.shape)} of {t.dtype} with strides {t.stride()}")


def _stream() -> int:
    """The current device's current stream (read without torch's stream object, 2.4 us less a call)."""
    if torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def params_struct(params: Dict[str, Optional[torch.Tensor]]) -> Params:
    return Params(*[_ptr(params.get(n)) for n in PARAM_FIELDS])


def make_layer_options(rot: int = 0, layout: str = "half", theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       orig_len: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0, mscale: float = 1.0, pos0: int = 0,
                       window: int = 0, sinks: int = 0) -> LayerOptions:
    """Rotary positions of Q and K (rot > 0) and a window of the attention (window > 0) for a layer."""
    return LayerOptions(rot, pos0, orig_len, theta, factor, beta_fast, beta_slow, mscale, {"half": 0, "interleaved": 1}[layout],
                        ROPE_SCALING[scaling], window, sinks)


def layer_options_validate(cfg: Config, options: LayerOptions) -> int:
    return load().bpt_layer_options_validate(ctypes.byref(cfg), ctypes.byref(options))


def layer_fwd(cfg: Config, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]], Y: torch.Tensor,
              saved: torch.Tensor, workspace: torch.Tensor, options: Optional[LayerOptions] = None) -> None:
    p = params_struct(params)
    if options is not None:
        _check(load().bpt_layer_fwd_options(ctypes.byref(cfg), ctypes.byref(options), X.data_ptr(), ctypes.byref(p), Y.data_ptr(),
                                            saved.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                            _stream()))
        return
    _check(load().bpt_layer_fwd(ctypes.byref(cfg), X.data_ptr(), ctypes.byref(p), Y.data_ptr(),
                                saved.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                _stream()))


NOALLOC_SCRATCH_BYTES = 64 << 20


def layer_fwd_noalloc(cfg: Config, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]], Y: torch.Tensor,
                      saved: torch.Tensor) -> None:
    """bpt_layer_fwd_noalloc: the forward with the library's static scratch as workspace."""
    p = params_struct(params)
    _check(load().bpt_layer_fwd_noalloc(ctypes.byref(cfg), X.data_ptr(), ctypes.byref(p), Y.data_ptr(),
                                        saved.data_ptr(), _stream()))


def layer_bwd(cfg: Config, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]], saved: torch.Tensor,
              dY: torch.Tensor, dX: torch.Tensor, grads: Dict[str, Optional[torch.Tensor]],
              workspace: torch.Tensor, options: Optional[LayerOptions] = None) -> None:
    p = params_struct(params)
    g = Grads(*[_ptr(grads.get(n)) for n in GRAD_FIELDS])
    if options is not None:
        _check(load().bpt_layer_bwd_options(ctypes.byref(cfg), ctypes.byref(options), X.data_ptr(), ctypes.byref(p),
                                            saved.data_ptr(), dY.data_ptr(), dX.data_ptr(), ctypes.byref(g), workspace.data_ptr(),
                                            workspace.numel() * workspace.element_size(), _stream()))
        return
    _check(load().bpt_layer_bwd(ctypes.byref(cfg), X.data_ptr(), ctypes.byref(p), saved.data_ptr(),
                                dY.data_ptr(), dX.data_ptr(), ctypes.byref(g), workspace.data_ptr(),
                                workspace.numel() * workspace.element_size(), _stream()))


_TORCH_DT = {BPT_F32: torch.float32, BPT_BF16: torch.bfloat16}


class Layer:
    """One BPT layer: owns nothing but the buffers it allocates through torch."""

    def __init__(self, cfg: Config, device: str = "cuda", options: Optional[LayerOptions] = None):
        _check(validate(cfg) if options is None else layer_options_validate(cfg, options))
        self.cfg, self.device, self.options = cfg, device, options
        self.out_dtype = _TORCH_DT[cfg.out_dtype]

    def _bytes(self, n: int) -> torch.Tensor:
        return torch.empty(max(n, 256), dtype=torch.uint8, device=self.device)

    def forward(self, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]],
                workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        Y = torch.empty(X.shape, dtype=self.out_dtype, device=self.device)
        saved = self._bytes(saved_bytes(self.cfg))
        ws = workspace if workspace is not None else self._bytes(workspace_bytes(self.cfg, False))
        layer_fwd(self.cfg, X, params, Y, saved, ws, self.options)
        return Y, saved

    def backward(self, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]], saved: torch.Tensor,
                 dY: torch.Tensor, want: Optional[Tuple[str, ...]] = None,
                 workspace: Optional[torch.Tensor] = None,
                 qkv_grads: bool = False) -> Tuple[torch.Tensor, Dict[str, torch.Tensor]]:
        """dX and the parameter gradients; with qkv_grads, also "dQ", "dK", "dV" [B, S, D], the gradients of
        Q = U Wq, K, V (copies of what the backward leaves in its workspace, bpt_bwd_qkv_grad_offset; not with a window)."""
        if qkv_grads and self.options is not None and self.options.window:
            raise ValueError("qkv_grads is for a layer without a window")
        D, F = self.cfg.D, self.cfg.F
        shapes = {"dln1_g": (D,), "dln1_b": (D,), "dWq": (D, D), "dWk": (D, D), "dWv": (D, D), "dWo": (D, D),
                  "dln2_g": (D,), "dln2_b": (D,), "dW1": (D, F), "db1": (F,), "dW2": (F, D), "db2": (D,)}
        src = {"dln1_g": "ln1_g", "dln1_b": "ln1_b", "dln2_g": "ln2_g", "dln2_b": "ln2_b", "db1": "b1", "db2": "b2"}
        grads = {}
        for n, shp in shapes.items():
            if want is not None and n not in want:
                continue
            if n in src and params.get(src[n]) is None:
                continue
            grads[n] = torch.empty(shp, dtype=torch.float32, device=self.device)
        dX = torch.empty(X.shape, dtype=self.out_dtype, device=self.device)
        ws = workspace if workspace is not None else self._bytes(workspace_bytes(self.cfg, True))
        layer_bwd(self.cfg, X, params, saved, dY, dX, grads, ws, self.options)
        if qkv_grads:
            c = self.cfg
            E = _TORCH_DT[c.dtype]
            Sp = (c.S + 63) // 64 * 64
            off, n = bwd_qkv_grad_offset(c), 3 * c.D * c.B * Sp
            m = ws[off:off + n * (2 if E == torch.bfloat16 else 4)].view(E).view(3, c.D, c.B, Sp)[..., :c.S]
            for i, name in enumerate(("dQ", "dK", "dV")):
                grads[name] = m[i].permute(1, 2, 0).contiguous()
        return dX, grads

    def saved_views(self, saved: torch.Tensor) -> Dict[str, torch.Tensor]:
        """Typed views of the saved activations (see bpt_saved_layout in include/libbpt.h)."""
        c = self.cfg
        lay = saved_layout(c)
        E = _TORCH_DT[c.dtype]
        T, D, Sp = c.B * c.S, c.D, (c.S + 63) // 64 * 64

        def view(name, n, dt, shape):
            off = lay[name]
            nbytes = n * (2 if dt == torch.bfloat16 else 4)
            return saved[off:off + nbytes].view(dt).view(*shape)

        return {
            "qkv": view("qkv", T * 3 * D, E, (T, 3 * D)),
            "o": view("o", T * D, E, (T, D)),
            "lse": view("lse", c.B * c.H * Sp, torch.float32, (c.B, c.H, Sp)),
            "h": view("h", T * D, torch.float32, (T, D)),
            "mu1": view("mu1", T, torch.float32, (T,)),
            "rstd1": view("rstd1", T, torch.float32, (T,)),
            "mu2": view("mu2", T, torch.float32, (T,)),
            "rstd2": view("rstd2", T, torch.float32, (T,)),
        }


# ---------------------------------------------------------------- cross-entropy of an LM head
def make_xent_config(T: int, D: int, V: int, ldw: Optional[int] = None, block_rows: int = 0,
                     dtype: str = "bf16") -> XentConfig:
    dt = {"f32": BPT_F32, "bf16": BPT_BF16}
    return XentConfig(T, D, V, ldw if ldw is not None else (V + 63) // 64 * 64, block_rows, dt[dtype], 0)


def xent_validate(cfg: XentConfig) -> int:
    return load().bpt_xent_validate(ctypes.byref(cfg))


def xent_workspace_bytes(cfg: XentConfig, backward: bool) -> int:
    return load().bpt_xent_workspace_bytes(ctypes.byref(cfg), int(backward))


def xent_fwd(cfg: XentConfig, h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, loss: torch.Tensor,
             lse: torch.Tensor, workspace: torch.Tensor) -> None:
    _check(load().bpt_xent_fwd(ctypes.byref(cfg), h.data_ptr(), W.data_ptr(), targets.data_ptr(),
                               loss.data_ptr(), lse.data_ptr(), workspace.data_ptr(),
                               workspace.numel() * workspace.element_size(), _stream()))


def xent_bwd(cfg: XentConfig, h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
             dloss: float, dh: torch.Tensor, dW: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(load().bpt_xent_bwd(ctypes.byref(cfg), h.data_ptr(), W.data_ptr(), targets.data_ptr(),
                               lse.data_ptr(), float(dloss), dh.data_ptr(), _ptr(dW), workspace.data_ptr(),
                               workspace.numel() * workspace.element_size(), _stream()))


class LMHeadLoss:
    """Cross-entropy of an LM head through libbpt; allocates its buffers with torch."""

    def __init__(self, cfg: XentConfig, device: str = "cuda"):
        _check(xent_validate(cfg))
        self.cfg, self.device = cfg, device

    def _bytes(self, n: int) -> torch.Tensor:
        return torch.empty(max(n, 256), dtype=torch.uint8, device=self.device)

    def forward(self, h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        loss = torch.empty(1, dtype=torch.float32, device=self.device)
        lse = torch.empty(self.cfg.T, dtype=torch.float32, device=self.device)
        xent_fwd(self.cfg, h, W, targets, loss, lse, self._bytes(xent_workspace_bytes(self.cfg, False)))
        return loss, lse

    def backward(self, h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                 dloss: float = 1.0, want_dW: bool = True) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        dh = torch.empty(h.shape, dtype=h.dtype, device=self.device)
        dW = torch.empty((self.cfg.D, self.cfg.ldw), dtype=torch.float32, device=self.device) if want_dW else None
        xent_bwd(self.cfg, h, W, targets, lse, dloss, dh, dW, self._bytes(xent_workspace_bytes(self.cfg, True)))
        return dh, dW


# ---------------------------------------------------------------- GPT training step pieces
_DT = {"f32": BPT_F32, "bf16": BPT_BF16}


def make_embed_config(B: int, S: int, D: int, V: int, dtype: str = "bf16", grad_dtype: Optional[str] = None):
    return EmbedConfig(B, S, D, V, _DT[dtype], _DT[grad_dtype or dtype])


def embed_fwd(cfg: EmbedConfig, tokens: torch.Tensor, Wte: torch.Tensor, Wpe: Optional[torch.Tensor],
              X: torch.Tensor) -> None:
    _check(load().bpt_embed_fwd(ctypes.byref(cfg), tokens.data_ptr(), Wte.data_ptr(), _ptr(Wpe), X.data_ptr(),
                                _stream()))


def embed_bwd(cfg: EmbedConfig, tokens: torch.Tensor, dX: torch.Tensor, dWte: Optional[torch.Tensor],
              dWpe: Optional[torch.Tensor]) -> None:
    _check(load().bpt_embed_bwd(ctypes.byref(cfg), tokens.data_ptr(), dX.data_ptr(), _ptr(dWte), _ptr(dWpe),
                                _stream()))


def make_ln_config(rows: int, D: int, eps: float = 1e-5, in_dtype: str = "bf16",
                   out_dtype: Optional[str] = None) -> LnConfig:
    return LnConfig(rows, D, eps, _DT[in_dtype], _DT[out_dtype or in_dtype], 0)


def ln_workspace_bytes(cfg: LnConfig) -> int:
    return load().bpt_ln_workspace_bytes(ctypes.byref(cfg))


def ln_fwd(cfg: LnConfig, X: torch.Tensor, g: Optional[torch.Tensor], b: Optional[torch.Tensor], Y: torch.Tensor,
           mean: torch.Tensor, rstd: torch.Tensor) -> None:
    _check(load().bpt_ln_fwd(ctypes.byref(cfg), X.data_ptr(), _ptr(g), _ptr(b), Y.data_ptr(), mean.data_ptr(),
                             rstd.data_ptr(), _stream()))


def ln_bwd(cfg: LnConfig, X: torch.Tensor, g: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
           dY: torch.Tensor, dX: torch.Tensor, dg: Optional[torch.Tensor], db: Optional[torch.Tensor],
           workspace: torch.Tensor) -> None:
    _check(load().bpt_ln_bwd(ctypes.byref(cfg), X.data_ptr(), _ptr(g), mean.data_ptr(), rstd.data_ptr(),
                             dY.data_ptr(), dX.data_ptr(), _ptr(dg), _ptr(db), workspace.data_ptr(),
                             workspace.numel() * workspace.element_size(), _stream()))


def adamw_step(p: torch.Tensor, g: torch.Tensor, m: torch.Tensor, v: torch.Tensor, step: int, lr: float,
               beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, weight_decay: float = 0.1,
               p_lowp: Optional[torch.Tensor] = None) -> None:
    """One AdamW update of the fp32 tensor p (in place, with its moments m, v); p_lowp,
    if given, receives p rounded to its dtype."""
    lowp = BPT_BF16 if p_lowp is not None and p_lowp.dtype == torch.bfloat16 else BPT_F32
    cfg = AdamWConfig(lr, beta1, beta2, eps, weight_decay, lowp, step)
    _check(load().bpt_adamw_step(ctypes.byref(cfg), p.numel(), p.data_ptr(), g.data_ptr(), m.data_ptr(),
                                 v.data_ptr(), _ptr(p_lowp), _stream()))


# ---------------------------------------------------------------- rotary positions
ROPE_SCALING = {"none": 0, "linear": 1, "base": 2, "by_parts": 3}


def make_rope_config(rows: int, S: int, H: int, dh: int, rot: Optional[int] = None, ldx: Optional[int] = None,
                     ldy: Optional[int] = None, layout: str = "half", theta: float = 10000.0, scaling: str = "none",
                     factor: float = 1.0, orig_len: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0,
                     mscale: float = 1.0, pos0: int = 0, dtype: str = "bf16") -> RopeConfig:
    """Rotary positions of H heads of width dh on `rows` tokens; see include/libbpt.h."""
    w = H * dh
    return RopeConfig(rows, S, H, dh, dh if rot is None else rot, w if ldx is None else ldx, w if ldy is None else ldy, pos0,
                      orig_len, theta, factor, beta_fast, beta_slow, mscale, {"half": 0, "interleaved": 1}[layout],
                      ROPE_SCALING[scaling], _DT[dtype], 0)


def rope_validate(cfg: RopeConfig) -> int:
    return load().bpt_rope_validate(ctypes.byref(cfg))


@functools.lru_cache(maxsize=1024)
def _rope_layout(cfg: bytes):
    """(type, shape, strides) of the rows at ldx and of those at ldy, as a tensor [rows, H, dh]."""
    c = RopeConfig.from_buffer_copy(cfg)
    return tuple((_TORCH_DT.get(c.dtype), (c.rows, c.H, c.dh), (ld, c.dh, 1)) for ld in (c.ldx, c.ldy))


def _check_rows(t: torch.Tensor, layout, name: str) -> None:
    """Raises unless a tensor holds a configuration's rows: its last dimensions are one row's heads (and what follows them there)
    and its first ones count the rows, or it is a buffer of them, flat or contiguous and just as long."""
    dtype, (rows, H, dh), (ld, _, _) = layout
    if t.dtype == dtype:
        if t.numel() == rows * ld and t.is_contiguous():
            return
        dims = [(n, st) for n, st in zip(t.shape, t.stride()) if n != 1]
        if len(dims) == 1 and dims[0][1] == 1 and dims[0][0] >= (rows - 1) * ld + H * dh:
            return
        inner, outer = 1, 1
        while dims and inner < H * dh and dims[-1][1] == inner:
            inner *= dims.pop()[0]
        while dims and dims[-1][1] == outer * ld:
            outer *= dims.pop()[0]
        if not dims and inner >= H * dh and outer == rows:
            return
    raise ValueError(f"{name} must hold {rows} rows of {H} x {dh} {dtype}, {ld} elements apart, as the configuration has it; not "
                     f"{tuple(t.shape)} of {t.dtype} with strides {t.stride()}")


def rope_fwd(cfg: RopeConfig, X: torch.Tensor, Y: torch.Tensor, positions: Optional[torch.Tensor] = None) -> None:
    at_x, at_y = _rope_layout(bytes(cfg))
    if (X.dtype, X.shape, X.stride()) != at_x:
        _check_rows(X, at_x, "X")
    if (Y.dtype, Y.shape, Y.stride()) != at_y:
        _check_rows(Y, at_y, "Y")
    dev, pos = X.get_device(), None
    same = Y.get_device() == dev
    if positions is not None:
        pos, same = _int32(positions, at_x[1][0], "positions"), same and positions.get_device() == dev
    _check(load().bpt_rope_fwd(cfg, pos, X.data_ptr(), Y.data_ptr(), _stream_on(dev, same)))


def rope_bwd(cfg: RopeConfig, dY: torch.Tensor, dX: torch.Tensor, positions: Optional[torch.Tensor] = None) -> None:
    at_x, at_y = _rope_layout(bytes(cfg))
    if (dY.dtype, dY.shape, dY.stride()) != at_y:
        _check_rows(dY, at_y, "dY")
    if (dX.dtype, dX.shape, dX.stride()) != at_x:
        _check_rows(dX, at_x, "dX")
    dev, pos = dX.get_device(), None
    same = dY.get_device() == dev
    if positions is not None:
        pos, same = _int32(positions, at_x[1][0], "positions"), same and positions.get_device() == dev
    _check(load().bpt_rope_bwd(cfg, pos, dY.data_ptr(), dX.data_ptr(), _stream_on(dev, same)))


# ---------------------------------------------------------------- attention with a window and sinks
def _strides(t: torch.Tensor) -> AttnStrides:
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError("attention tensors are [B, S, heads, dh] with adjacent features")
    unit = 16 // t.element_size()
    # the stride of a dimension of one element says nothing and may be any number
    return AttnStrides(*(0 if n == 1 and (st % unit or not 0 <= st < most) else st
                         for n, st, most in zip(t.shape, t.stride(), (1 << 40, 1 << 22, 1 << 40))))


def attn_config_of(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, causal: bool = True, window: int = 0,
                   sinks: int = 0, scale: Optional[float] = None) -> AttnConfig:
    """The configuration of attention on tensors of these shapes and strides: q, o [B, Sq, Hq, dh],
    k, v [B, Skv, Hkv, dh] (dq, dk, dv laid out like q, k, v; do like o)."""
    B, Sq, Hq, dh = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != dh or o.shape != q.shape:
        raise ValueError(f"shapes do not fit: q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}, o {tuple(o.shape)}")
    if not q.dtype == k.dtype == v.dtype == o.dtype or q.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("q, k, v and o must share a type, float32 or bfloat16")
    return AttnConfig(B, Sq, k.shape[1], Hq, k.shape[2], dh, _strides(q), _strides(k), _strides(v), _strides(o), window, sinks,
                      dh ** -0.5 if scale is None else scale, int(bool(causal)), BPT_BF16 if q.dtype == torch.bfloat16 else BPT_F32,
                      0)


def attn_validate(cfg: AttnConfig) -> int:
    return load().bpt_attn_validate(ctypes.byref(cfg))


def attn_workspace_bytes(cfg: AttnConfig, backward: bool) -> int:
    return load().bpt_attn_workspace_bytes(ctypes.byref(cfg), int(backward))


@functools.lru_cache(maxsize=1024)
def _attn_layout(cfg: bytes):
    """(type, shape, strides) that a configuration gives q, k, v and o; sequences; rows of the log-sum-exp."""
    c = AttnConfig.from_buffer_copy(cfg)
    dt, qs, ks = _TORCH_DT.get(c.dtype), (c.B, c.Sq, c.Hq, c.dh), (c.B, c.Skv, c.Hkv, c.dh)
    return (*((dt, shape, (s.sb, s.st, s.sh, 1)) for shape, s in ((qs, c.q), (ks, c.k), (ks, c.v), (qs, c.o))),
            c.B, c.B * c.Hq * c.Sq)


def _check_lse(lse: torch.Tensor, n: int) -> None:
    if lse.dtype != torch.float32 or lse.numel() != n or not lse.is_contiguous():
        raise ValueError(f"lse must be [B, Hq, Sq] contiguous float32, {n} elements; not {tuple(lse.shape)} of {lse.dtype}")


def attn_fwd(cfg: AttnConfig, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
             workspace: Optional[torch.Tensor] = None, q_lens: Optional[torch.Tensor] = None,
             kv_lens: Optional[torch.Tensor] = None) -> None:
    """Every tensor has the shape, strides and type that cfg gives it."""
    at_q, at_k, at_v, at_o, B, rows = _attn_layout(bytes(cfg))
    if (q.dtype, q.shape, q.stride()) != at_q:
        _check_layout(q, at_q, "q")
    if (k.dtype, k.shape, k.stride()) != at_k:
        _check_layout(k, at_k, "k")
    if (v.dtype, v.shape, v.stride()) != at_v:
        _check_layout(v, at_v, "v")
    if (o.dtype, o.shape, o.stride()) != at_o:
        _check_layout(o, at_o, "o")
    _check_lse(lse, rows)
    dev, nb = q.get_device(), 0
    same = dev == k.get_device() == v.get_device() == o.get_device() == lse.get_device()
    ql = kl = None
    if q_lens is not None:
        ql, same = _int32(q_lens, B, "q_lens"), same and q_lens.get_device() == dev
    if kv_lens is not None:
        kl, same = _int32(kv_lens, B, "kv_lens"), same and kv_lens.get_device() == dev
    if workspace is not None:
        nb, same = workspace.numel() * workspace.element_size(), same and workspace.get_device() == dev
    _check(load().bpt_attn_fwd(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), ql, kl, o.data_ptr(), lse.data_ptr(),
                               workspace.data_ptr() if nb else None, nb, _stream_on(dev, same)))


def attn_bwd(cfg: AttnConfig, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
             do: torch.Tensor, dq: Optional[torch.Tensor], dk: Optional[torch.Tensor], dv: Optional[torch.Tensor],
             workspace: torch.Tensor, q_lens: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None) -> None:
    """Every tensor has the shape, strides and type that cfg gives it: dq, dk and dv those of q, k and v, do those of o."""
    at_q, at_k, at_v, at_o, B, rows = _attn_layout(bytes(cfg))
    if (q.dtype, q.shape, q.stride()) != at_q:
        _check_layout(q, at_q, "q")
    if (k.dtype, k.shape, k.stride()) != at_k:
        _check_layout(k, at_k, "k")
    if (v.dtype, v.shape, v.stride()) != at_v:
        _check_layout(v, at_v, "v")
    if (o.dtype, o.shape, o.stride()) != at_o:
        _check_layout(o, at_o, "o")
    if (do.dtype, do.shape, do.stride()) != at_o:
        _check_layout(do, at_o, "do")
    _check_lse(lse, rows)
    dev = q.get_device()
    same = dev == k.get_device() == v.get_device() == o.get_device() == do.get_device() == lse.get_device() == workspace.get_device()
    if dq is not None:
        if (dq.dtype, dq.shape, dq.stride()) != at_q:
            _check_layout(dq, at_q, "dq")
        same = same and dq.get_device() == dev
    if dk is not None:
        if (dk.dtype, dk.shape, dk.stride()) != at_k:
            _check_layout(dk, at_k, "dk")
        same = same and dk.get_device() == dev
    if dv is not None:
        if (dv.dtype, dv.shape, dv.stride()) != at_v:
            _check_layout(dv, at_v, "dv")
        same = same and dv.get_device() == dev
    ql = kl = None
    if q_lens is not None:
        ql, same = _int32(q_lens, B, "q_lens"), same and q_lens.get_device() == dev
    if kv_lens is not None:
        kl, same = _int32(kv_lens, B, "kv_lens"), same and kv_lens.get_device() == dev
    _check(load().bpt_attn_bwd(cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), ql, kl, o.data_ptr(), lse.data_ptr(), do.data_ptr(),
                               _ptr(dq), _ptr(dk), _ptr(dv), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                               _stream_on(dev, same)))


def _span(t: torch.Tensor) -> int:
    """Elements from a tensor's first to behind its last."""
    return 1 + sum((n - 1) * st for n, st in zip(t.shape, t.stride()))


def _apart(t: torch.Tensor) -> bool:
    """Whether no two elements of a tensor share a place, features are adjacent and rows of heads start at whole 16 bytes."""
    dims = sorted((st, n) for st, n in zip(t.stride(), t.shape) if n > 1)
    end, unit = 1, 16 // t.element_size()
    for st, n in dims:
        if st < end:
            return False
        end += st * (n - 1)
    return t.data_ptr() % 16 == 0 and t.stride(-1) == 1 and all(st % unit == 0 for st, n in dims if st > 1)


def _side_by_side(tensors: Tuple[torch.Tensor, ...]) -> Optional[List[torch.Tensor]]:
    """For parts of the rows of one tensor (Q, K and V as columns of one projection): new tensors that are such parts of
    a new one. None for others."""
    first = tensors[0]
    st, (B, S) = first.stride(), first.shape[:2]
    at = sorted((t.storage_offset(), t.storage_offset() + (t.shape[2] - 1) * st[2] + t.shape[3]) for t in tensors)
    low, high = at[0][0], at[-1][1]
    if (any(t.stride() != st or t.shape[:2] != (B, S) or t.dtype != first.dtype
            or t.untyped_storage().data_ptr() != first.untyped_storage().data_ptr() or not _apart(t) for t in tensors)
            or any(a[1] > b[0] for a, b in zip(at, at[1:])) or (S > 1 and high - low > st[1])
            or (B > 1 and (S - 1) * st[1] + high - low > st[0])):
        return None
    n = (B - 1) * st[0] + (S - 1) * st[1] + high - low
    if n > 2 * sum(t.numel() for t in tensors):      # mostly something else
        return None
    buf = torch.empty(n, dtype=first.dtype, device=first.device)
    return [buf.as_strided(t.shape, st, t.storage_offset() - low) for t in tensors]


class WindowAttention:
    """Attention with a window and sinks through libbpt; allocates its buffers with torch."""

    def __init__(self, causal: bool = True, window: int = 0, sinks: int = 0, scale: Optional[float] = None):
        self.kw = dict(causal=causal, window=window, sinks=sinks, scale=scale)

    @staticmethod
    def _bytes(n: int, device) -> torch.Tensor:
        return torch.empty(max(n, 256), dtype=torch.uint8, device=device)

    def forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_lens: Optional[torch.Tensor] = None,
                kv_lens: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """O [B, Sq, Hq, dh] and the log-sum-exp [B, Hq, Sq]."""
        if not (q.is_cuda and q.device == k.device == v.device):
            raise ValueError("q, k and v must be on one GPU")
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
        cfg = attn_config_of(q, k, v, o, **self.kw)
        attn_fwd(cfg, q, k, v, o, lse, self._bytes(attn_workspace_bytes(cfg, False), q.device), q_lens, kv_lens)
        return o, lse

    def backward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor, do: torch.Tensor,
                 q_lens: Optional[torch.Tensor] = None,
                 kv_lens: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """dQ, dK, dV; q, k, v as they were, o, lse from forward. Gradients of columns of one projection are columns of one
        tensor, those of a tensor without gaps are laid out like it, others are contiguous (and their input is copied)."""
        if any(t.dim() != 4 for t in (q, k, v, o)):
            raise ValueError("attention tensors are [B, S, heads, dh]")
        if do.shape != o.shape or do.dtype != o.dtype:
            raise ValueError(f"do must be {tuple(o.shape)} of {o.dtype}, not {tuple(do.shape)} of {do.dtype}")
        if do.stride() != o.stride():                # they share their strides
            o, do = o.contiguous(), do.contiguous()
        grads = _side_by_side((q, k, v))
        if grads is None:
            q, k, v = (t if _apart(t) and _span(t) == t.numel() else t.contiguous() for t in (q, k, v))
            grads = [torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device) for t in (q, k, v)]
        cfg = attn_config_of(q, k, v, o, **self.kw)
        attn_bwd(cfg, q, k, v, o, lse, do, *grads, self._bytes(attn_workspace_bytes(cfg, True), q.device), q_lens, kv_lens)
        return tuple(grads)


# ---------------------------------------------------------------- AdamW over many tensors
class AdamWTensors:
    """A list of tensors that adamw_multi updates together: dicts of p, g, m and v (32-bit moments, fp32) or
    r and exps (8-bit moments: e4m3 bytes and two exponent bytes per block of 256 elements, all zero at the
    start), p_lowp (None: no copy) and weight_decay. Keeps the tensors alive."""

    def __init__(self, tensors, bits: int = 32):
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        self.tensors, self.bits = list(tensors), bits
        second = "r" if bits == 8 else "v"
        state = torch.uint8 if bits == 8 else torch.float32
        gts = {t["g"].dtype for t in self.tensors}
        lows = {t["p_lowp"].dtype for t in self.tensors if t.get("p_lowp") is not None}
        if len(gts) > 1 or len(lows) > 1 or not (gts | lows) <= {torch.float32, torch.bfloat16}:
            raise ValueError("gradients share one type, low-precision copies too: float32 or bfloat16")
        for t in self.tensors:
            n = t["p"].numel()
            need = {"p": (torch.float32, n), "g": (t["g"].dtype, n), "m": (state, n), second: (state, n)}
            if bits == 8:
                need["exps"] = (torch.uint8, 2 * ((n + 255) // 256))
            if t.get("p_lowp") is not None:
                need["p_lowp"] = (t["p_lowp"].dtype, n)
            for name, (dt, size) in need.items():
                if t[name].dtype != dt or t[name].numel() != size or not t[name].is_contiguous():
                    raise ValueError(f"{name} must be contiguous, of type {dt} and of {size} elements")
        self.device = self.tensors[0]["p"].device if self.tensors else None
        if any(x.device != self.device for t in self.tensors for x in t.values() if isinstance(x, torch.Tensor)):
            raise ValueError("the tensors of a list must be on one device")
        self.grad_dtype = BPT_BF16 if gts == {torch.bfloat16} else BPT_F32
        self.lowp_dtype = BPT_BF16 if lows == {torch.bfloat16} else BPT_F32
        self.array = (AdamWTensor * max(len(self.tensors), 1))(*[
            AdamWTensor(t["p"].numel(), t["p"].data_ptr(), t["g"].data_ptr(), t["m"].data_ptr(), t[second].data_ptr(),
                        _ptr(t.get("exps")) if bits == 8 else None, _ptr(t.get("p_lowp")), float(t.get("weight_decay", 0.0)))
            for t in self.tensors])


def adamw_multi(tensors: AdamWTensors, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8,
                seed: int = 0) -> None:
    """One AdamW update of every tensor of the list, in place."""
    if tensors.device is not None and tensors.device.type != "cuda":
        raise ValueError("the tensors must be on the GPU")
    stream = _stream_on(tensors.device.index, True) if tensors.tensors else _stream()
    cfg = AdamWMultiConfig(lr, beta1, beta2, eps, step, seed & (2 ** 64 - 1), tensors.bits, tensors.grad_dtype, tensors.lowp_dtype, 0)
    _check(load().bpt_adamw_multi(ctypes.byref(cfg), tensors.array, len(tensors.tensors), stream))
