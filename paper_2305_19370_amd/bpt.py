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


class RecurStrides(ctypes.Structure):
    _fields_ = [("sb", c_i64), ("st", c_i64)]


class RecurConfig(ctypes.Structure):
    _fields_ = [("B", c_i64), ("S", c_i64), ("D", c_i64), ("x", RecurStrides), ("r", RecurStrides), ("i", RecurStrides),
                ("y", RecurStrides), ("c", c_f32), ("dtype", c_i32), ("reserved", c_i64)]


class RecurMixer(ctypes.Structure):
    _fields_ = [("c", c_f32), ("lam", c_vp), ("h0", c_vp), ("hT", c_vp)]


class DistillConfig(ctypes.Structure):
    _fields_ = [("T", c_i64), ("D", c_i64), ("V", c_i64), ("K", c_i64), ("ldw", c_i64), ("block_rows", c_i64), ("keep_bytes", c_i64),
                ("tau", c_f32), ("soft", c_f32), ("hard", c_f32), ("dtype", c_i32), ("grad_dtype", c_i32), ("reserved", c_i32)]


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
           "bpt_layer_fwd_options", "bpt_layer_bwd_options", "bpt_recur_validate", "bpt_recur_saved_bytes",
           "bpt_recur_workspace_bytes", "bpt_recur_fwd", "bpt_recur_bwd", "bpt_distill_validate", "bpt_distill_saved_bytes",
           "bpt_distill_workspace_bytes", "bpt_distill_fwd", "bpt_distill_bwd", "bpt_layer_recurrent_validate",
           "bpt_layer_recurrent_saved_bytes", "bpt_layer_recurrent_workspace_bytes", "bpt_layer_fwd_recurrent",
           "bpt_layer_bwd_recurrent")

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
    lib.bpt_recur_validate.argtypes = [P(RecurConfig)]
    lib.bpt_recur_validate.restype = c_i32
    lib.bpt_recur_saved_bytes.argtypes = [P(RecurConfig)]
    lib.bpt_recur_saved_bytes.restype = c_sz
    lib.bpt_recur_workspace_bytes.argtypes = [P(RecurConfig), c_i32]
    lib.bpt_recur_workspace_bytes.restype = c_sz
    lib.bpt_recur_fwd.argtypes = [P(RecurConfig)] + [c_vp] * 10 + [c_sz, c_vp]
    lib.bpt_recur_fwd.restype = c_i32
    lib.bpt_recur_bwd.argtypes = [P(RecurConfig)] + [c_vp] * 15 + [c_sz, c_vp]
    lib.bpt_recur_bwd.restype = c_i32
    lib.bpt_layer_recurrent_validate.argtypes = [P(Config), P(RecurMixer)]
    lib.bpt_layer_recurrent_validate.restype = c_i32
    lib.bpt_layer_recurrent_saved_bytes.argtypes = [P(Config)]
    lib.bpt_layer_recurrent_saved_bytes.restype = c_sz
    lib.bpt_layer_recurrent_workspace_bytes.argtypes = [P(Config), c_i32]
    lib.bpt_layer_recurrent_workspace_bytes.restype = c_sz
    lib.bpt_layer_fwd_recurrent.argtypes = [P(Config), P(RecurMixer), c_vp, P(Params), c_vp, c_vp, c_vp, c_sz, c_vp]
    lib.bpt_layer_fwd_recurrent.restype = c_i32
    lib.bpt_layer_bwd_recurrent.argtypes = [P(Config), P(RecurMixer), c_vp, P(Params), c_vp, c_vp, c_vp, c_vp, P(Grads), c_vp, c_vp,
                                            c_vp, c_sz, c_vp]
    lib.bpt_layer_bwd_recurrent.restype = c_i32
    lib.bpt_distill_validate.argtypes = [P(DistillConfig)]
    lib.bpt_distill_validate.restype = c_i32
    lib.bpt_distill_saved_bytes.argtypes = [P(DistillConfig)]
    lib.bpt_distill_saved_bytes.restype = c_sz
    lib.bpt_distill_workspace_bytes.argtypes = [P(DistillConfig), c_i32]
    lib.bpt_distill_workspace_bytes.restype = c_sz
    lib.bpt_distill_fwd.argtypes = [P(DistillConfig)] + [c_vp] * 10 + [c_sz, c_vp]
    lib.bpt_distill_fwd.restype = c_i32
    lib.bpt_distill_bwd.argtypes = [P(DistillConfig)] + [c_vp] * 3 + [c_f32] + [c_vp] * 3 + [c_sz, c_vp]
    lib.bpt_distill_bwd.restype = c_i32
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

    def _grads(self, params: Dict[str, Optional[torch.Tensor]], want: Optional[Tuple[str, ...]]) -> Dict[str, torch.Tensor]:
        """Buffers of the parameter gradients: those wanted (None: all) of the parameters that are there."""
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
        return grads

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
        grads = self._grads(params, want)
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


# ---------------------------------------------------------------- gated linear recurrence
def recur_config_of(x: torch.Tensor, r: torch.Tensor, i: torch.Tensor, y: torch.Tensor, c: float = 8.0) -> RecurConfig:
    """The configuration of a recurrence over [B, S, D] tensors of any strides with adjacent channels; see include/libbpt.h."""
    if x.dim() != 3 or r.shape != x.shape or i.shape != x.shape or y.shape != x.shape:
        raise ValueError("x, r, i and y are [B, S, D], all the same")
    if x.dtype not in (torch.float32, torch.bfloat16) or not (x.dtype == r.dtype == i.dtype == y.dtype):
        raise ValueError("x, r, i and y must share a type, float32 or bfloat16")
    B, S, D = x.shape
    unit = 16 // x.element_size()

    def strides(t: torch.Tensor) -> RecurStrides:
        sb, st, sd = t.stride()
        if sd != 1 and D > 1:
            raise ValueError("channels must be adjacent")
        # the stride of a dimension of one element counts for nothing
        return RecurStrides(sb if B > 1 else 0, st if S > 1 else (D + unit - 1) // unit * unit)

    return RecurConfig(B, S, D, strides(x), strides(r), strides(i), strides(y), c, BPT_BF16 if x.dtype == torch.bfloat16 else BPT_F32, 0)


def recur_validate(cfg: RecurConfig) -> int:
    return load().bpt_recur_validate(ctypes.byref(cfg))


def recur_saved_bytes(cfg: RecurConfig) -> int:
    return load().bpt_recur_saved_bytes(ctypes.byref(cfg))


def recur_workspace_bytes(cfg: RecurConfig, backward: bool) -> int:
    return load().bpt_recur_workspace_bytes(ctypes.byref(cfg), int(backward))


@functools.lru_cache(maxsize=1024)
def _recur_layout(cfg: bytes):
    """(type, shape, strides) that a configuration gives x, r, i and y."""
    c = RecurConfig.from_buffer_copy(cfg)
    return tuple((_TORCH_DT.get(c.dtype), (c.B, c.S, c.D), (s.sb, s.st, 1)) for s in (c.x, c.r, c.i, c.y))


def _f32(t: Optional[torch.Tensor], shape: Tuple[int, ...], name: str) -> Optional[int]:
    """The address of contiguous float32 of a shape, or None."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be {list(shape)} contiguous float32, not {list(t.shape)} of {t.dtype}")
    return t.data_ptr()


def _nbytes(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _saved_ptr(t: Optional[torch.Tensor], need: int) -> Optional[int]:
    if t is not None and (not t.is_contiguous() or _nbytes(t) < need):
        raise ValueError(f"saved must be {need} contiguous bytes, not {_nbytes(t)}")
    return t.data_ptr() if need and t is not None else None


def recur_fwd(cfg: RecurConfig, x: torch.Tensor, r: torch.Tensor, i: torch.Tensor, lam: torch.Tensor, y: torch.Tensor,
              h0: Optional[torch.Tensor] = None, hT: Optional[torch.Tensor] = None, saved: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None, lens: Optional[torch.Tensor] = None) -> None:
    """Every tensor has the shape, strides and type that cfg gives it. hT may be h0."""
    for t, at, name in zip((x, r, i, y), _recur_layout(bytes(cfg)), "xriy"):
        if (t.dtype, t.shape, t.stride()) != at:
            _check_layout(t, at, name)
    B, D = cfg.B, cfg.D
    lp, h0p, hTp = _f32(lam, (D,), "lam"), _f32(h0, (B, D), "h0"), _f32(hT, (B, D), "hT")
    sp = None if saved is None else _saved_ptr(saved, recur_saved_bytes(cfg))
    dev, nb = x.get_device(), _nbytes(workspace)
    same = all(t is None or t.get_device() == dev for t in (r, i, lam, y, h0, hT, saved, workspace, lens))
    stream = _stream_on(dev, same)
    _check(load().bpt_recur_fwd(cfg, x.data_ptr(), r.data_ptr(), i.data_ptr(), lp, _int32(lens, B, "lens"), h0p, y.data_ptr(), hTp,
                                sp, workspace.data_ptr() if nb else None, nb, stream))


def recur_bwd(cfg: RecurConfig, x: torch.Tensor, r: torch.Tensor, i: torch.Tensor, lam: torch.Tensor, saved: Optional[torch.Tensor],
              dy: torch.Tensor, dx: torch.Tensor, dr: torch.Tensor, di: torch.Tensor, workspace: torch.Tensor,
              dlam: Optional[torch.Tensor] = None, h0: Optional[torch.Tensor] = None, dhT: Optional[torch.Tensor] = None,
              dh0: Optional[torch.Tensor] = None, lens: Optional[torch.Tensor] = None) -> None:
    """Every tensor has the shape, strides and type that cfg gives it: dx, dr and di those of x, r and i, dy those of y. dh0 may
    be dhT."""
    at = _recur_layout(bytes(cfg))
    for t, lay, name in zip((x, r, i, dy, dx, dr, di), at + at[:3], ("x", "r", "i", "dy", "dx", "dr", "di")):
        if (t.dtype, t.shape, t.stride()) != lay:
            _check_layout(t, lay, name)
    B, D = cfg.B, cfg.D
    lp, dlp = _f32(lam, (D,), "lam"), _f32(dlam, (D,), "dlam")
    h0p, dhTp, dh0p = _f32(h0, (B, D), "h0"), _f32(dhT, (B, D), "dhT"), _f32(dh0, (B, D), "dh0")
    sp, dev = _saved_ptr(saved, recur_saved_bytes(cfg)), x.get_device()
    same = all(t is None or t.get_device() == dev for t in (r, i, lam, saved, dy, dx, dr, di, workspace, dlam, h0, dhT, dh0, lens))
    stream = _stream_on(dev, same)
    _check(load().bpt_recur_bwd(cfg, x.data_ptr(), r.data_ptr(), i.data_ptr(), lp, _int32(lens, B, "lens"), h0p,
                                sp, dy.data_ptr(), dhTp, dx.data_ptr(), dr.data_ptr(),
                                di.data_ptr(), dlp, dh0p, workspace.data_ptr(), _nbytes(workspace), stream))


@functools.lru_cache(maxsize=1024)
def _recur_plan(dtype: torch.dtype, shape: Tuple[int, ...], sx, sr, si, c: float):
    """Configuration of a forward into a dense y, its bytes of saved and workspace, and the shape of the states."""
    meta = lambda st: torch.empty_strided(shape, st, dtype=dtype, device="meta")  # noqa: E731
    cfg = recur_config_of(meta(sx), meta(sr), meta(si), torch.empty(shape, dtype=dtype, device="meta"), c)
    _check(recur_validate(cfg))
    return cfg, recur_saved_bytes(cfg), recur_workspace_bytes(cfg, False), (cfg.B, cfg.D)


@functools.lru_cache(maxsize=1024)
def _recur_back_plan(dtype: torch.dtype, shape: Tuple[int, ...], strides, sdy, offsets: Optional[Tuple[int, ...]], c: float):
    """For x, r and i of these strides (offsets: of parts of one tensor from the first of them, or None) at whole 16 bytes: the configuration of
    a backward, its bytes of saved and workspace, the shape of the states; elements of the tensor whose parts the gradients
    are (0: each its own) with their strides and offsets, and which of x, r and i are copied. Formed once: 25 us of a call."""
    size = max(1 + sum((n - 1) * st for n, st in zip(shape, sts)) for sts in strides) + (max(offsets) if offsets else 0)
    base = torch.empty(size, dtype=dtype, device="meta")
    views = [base.as_strided(shape, st, offsets[k] if offsets else 0) for k, st in enumerate(strides)]
    four = tuple(t.unsqueeze(2) for t in views)
    parts = _side_by_side(four) if offsets else None
    if parts is not None:
        n, copied = parts[0].untyped_storage().nbytes() // parts[0].element_size(), (False,) * 3
        at = tuple((t.stride(), g.storage_offset()) for t, g in zip(views, parts))
    else:
        n, copied = 0, tuple(not (_apart(f) and _span(t) == t.numel()) for t, f in zip(views, four))
        views, at = [torch.empty(shape, dtype=dtype, device="meta") if no else t for t, no in zip(views, copied)], ()
    cfg = recur_config_of(*views, torch.empty_strided(shape, sdy, dtype=dtype, device="meta"), c)
    _check(recur_validate(cfg))
    return cfg, recur_saved_bytes(cfg), recur_workspace_bytes(cfg, True), (cfg.B, cfg.D), n, at, copied


class GatedRecurrence:
    """A gated linear recurrence through libbpt; allocates its buffers with torch. For one new token of each sequence, call
    forward with S = 1 and the states as h0."""

    def __init__(self, c: float = 8.0):
        self.c = c

    @staticmethod
    def _bytes(n: int, device) -> torch.Tensor:
        return torch.empty(max(n, 256), dtype=torch.uint8, device=device)

    def forward(self, x: torch.Tensor, r: torch.Tensor, i: torch.Tensor, lam: torch.Tensor, h0: Optional[torch.Tensor] = None,
                lens: Optional[torch.Tensor] = None,
                save: bool = False) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
        """y [B, S, D], the last states [B, D] (float32), and with `save` what backward takes. Inputs off 16 bytes are copied."""
        if not x.dtype == r.dtype == i.dtype or not x.shape == r.shape == i.shape:
            raise ValueError("x, r and i must share a type and a shape")
        xp, rp, ip = x.data_ptr(), r.data_ptr(), i.data_ptr()
        if (xp | rp | ip) & 15:
            x, r, i = (t.clone(memory_format=torch.contiguous_format) if t.data_ptr() % 16 else t for t in (x, r, i))
            xp, rp, ip = x.data_ptr(), r.data_ptr(), i.data_ptr()
        cfg, ns, nb, states = _recur_plan(x.dtype, x.shape, x.stride(), r.stride(), i.stride(), self.c)
        at = x.get_device()
        same = at == r.get_device() == i.get_device() == lam.get_device()
        ap, hp, lp = _f32(lam, states[1:], "lam"), None, None
        if h0 is not None:
            hp, same = _f32(h0, states, "h0"), same and h0.get_device() == at
        if lens is not None:
            lp, same = _int32(lens, cfg.B, "lens"), same and lens.get_device() == at
        stream = _stream_on(at, same)
        # a new token is a call of some 8 us: tensors like others are made in half the time
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        hT = lam.new_empty(states) if h0 is None else torch.empty_like(h0)
        saved = self._bytes(ns, x.device) if save else None
        ws = self._bytes(nb, x.device) if nb else None
        _check(load().bpt_recur_fwd(cfg, xp, rp, ip, ap, lp, hp, y.data_ptr(),
                                    hT.data_ptr(), saved.data_ptr() if save and ns else None, ws.data_ptr() if nb else None, nb, stream))
        return y, hT, saved

    def backward(self, x: torch.Tensor, r: torch.Tensor, i: torch.Tensor, lam: torch.Tensor, saved: torch.Tensor, dy: torch.Tensor,
                 dhT: Optional[torch.Tensor] = None, h0: Optional[torch.Tensor] = None,
                 lens: Optional[torch.Tensor] = None) -> Dict[str, torch.Tensor]:
        """dx, dr, di, dlam and dh0; x, r, i, lam, h0 and lens as they were, saved from forward. Gradients of columns of one
        projection are columns of one tensor, those of a tensor without gaps are laid out like it, others are contiguous (and
        their input is copied)."""
        if dy.dim() != 3 or dy.shape != x.shape or dy.dtype != x.dtype:
            raise ValueError(f"dy must be {tuple(x.shape)} of {x.dtype}, not {tuple(dy.shape)} of {dy.dtype}")
        if not x.dtype == r.dtype == i.dtype or not x.shape == r.shape == i.shape:
            raise ValueError("x, r and i must share a type and a shape")
        # a broadcast one too: its rows share memory, as those of the y that it is laid out like may not
        if (not dy.is_contiguous() or dy.data_ptr() % 16) and not _apart(dy):
            dy = dy.clone(memory_format=torch.contiguous_format)
        x, r, i = (t.clone(memory_format=torch.contiguous_format) if t.data_ptr() % 16 else t for t in (x, r, i))
        offsets = None
        if not (x.is_contiguous() and r.is_contiguous() and i.is_contiguous()) or x.shape[0] * x.shape[1] == 1:
            where = x.untyped_storage().data_ptr()
            if where == r.untyped_storage().data_ptr() == i.untyped_storage().data_ptr():
                low = min(x.storage_offset(), r.storage_offset(), i.storage_offset())
                offsets = (x.storage_offset() - low, r.storage_offset() - low, i.storage_offset() - low)
        cfg, ns, nb, states, n, at, copied = _recur_back_plan(x.dtype, x.shape, (x.stride(), r.stride(), i.stride()), dy.stride(), offsets, self.c)
        x, r, i = (t.contiguous() if no else t for t, no in zip((x, r, i), copied)) if any(copied) else (x, r, i)
        sp, lp = _saved_ptr(saved, ns), _f32(lam, states[1:], "lam")
        h0p, dhTp, dev = _f32(h0, states, "h0"), _f32(dhT, states, "dhT"), x.get_device()
        same = all(t is None or t.get_device() == dev for t in (r, i, lam, saved, dy, dhT, h0, lens))
        np, stream = _int32(lens, cfg.B, "lens"), _stream_on(dev, same)
        if n:
            buf = x.new_empty(n)
            grads = [buf.as_strided(x.shape, st, first) for st, first in at]
        else:
            grads = [torch.empty_like(t) for t in (x, r, i)]      # without gaps: their strides too
        dlam, dh0, ws = torch.empty_like(lam), lam.new_empty(states), self._bytes(nb, x.device)
        _check(load().bpt_recur_bwd(cfg, x.data_ptr(), r.data_ptr(), i.data_ptr(), lp, np, h0p, sp, dy.data_ptr(), dhTp, grads[0].data_ptr(),
                                    grads[1].data_ptr(), grads[2].data_ptr(), dlam.data_ptr(), dh0.data_ptr(), ws.data_ptr(), nb, stream))
        return dict(zip(("dx", "dr", "di"), grads), dlam=dlam, dh0=dh0)


# ---------------------------------------------------------------- the layer with a recurrence
def recur_mixer(cfg: Config, lam: torch.Tensor, c: float = 8.0, h0: Optional[torch.Tensor] = None,
                hT: Optional[torch.Tensor] = None) -> RecurMixer:
    """The recurrence of a layer: lam [D], states before and after [B, D], float32 on the GPU. It holds addresses alone."""
    tensors = [t for t in (lam, h0, hT) if t is not None]
    _stream_on(lam.get_device(), all(t.get_device() == lam.get_device() for t in tensors))
    return RecurMixer(c, _f32(lam, (cfg.D,), "lam"), _f32(h0, (cfg.B, cfg.D), "h0"), _f32(hT, (cfg.B, cfg.D), "hT"))


def layer_recurrent_validate(cfg: Config, c: float = 8.0) -> int:
    return load().bpt_layer_recurrent_validate(ctypes.byref(cfg), RecurMixer(c, None, None, None))


def layer_recurrent_saved_bytes(cfg: Config) -> int:
    return load().bpt_layer_recurrent_saved_bytes(ctypes.byref(cfg))


def layer_recurrent_workspace_bytes(cfg: Config, backward: bool) -> int:
    return load().bpt_layer_recurrent_workspace_bytes(ctypes.byref(cfg), int(backward))


def _check_layer(cfg: Config, saved: torch.Tensor, others, **tensors: torch.Tensor) -> int:
    """Raises unless X, Y, dX (and dY) hold the tokens of a configuration, contiguous, and saved a recurrent layer's bytes. Their
    stream: others are on their device too."""
    for name, t in tensors.items():
        dt = _TORCH_DT.get(cfg.dtype if name in ("X", "dY") else cfg.out_dtype)
        if t.dtype != dt or t.numel() != cfg.B * cfg.S * cfg.D or not t.is_contiguous():
            raise ValueError(f"{name} must be {cfg.B} x {cfg.S} x {cfg.D} contiguous {dt}, not {tuple(t.shape)} of {t.dtype}")
    _saved_ptr(saved, layer_recurrent_saved_bytes(cfg))
    dev = tensors["X"].get_device()
    return _stream_on(dev, all(t is None or t.get_device() == dev for t in (saved, *others, *tensors.values())))


def layer_fwd_recurrent(cfg: Config, mixer: RecurMixer, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]], Y: torch.Tensor,
                        saved: torch.Tensor, workspace: torch.Tensor) -> None:
    stream = _check_layer(cfg, saved, (workspace, *params.values()), X=X, Y=Y)
    p = params_struct(params)
    _check(load().bpt_layer_fwd_recurrent(ctypes.byref(cfg), ctypes.byref(mixer), X.data_ptr(), ctypes.byref(p), Y.data_ptr(),
                                          saved.data_ptr(), workspace.data_ptr(), _nbytes(workspace), stream))


def layer_bwd_recurrent(cfg: Config, mixer: RecurMixer, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]], saved: torch.Tensor,
                        dY: torch.Tensor, dX: torch.Tensor, grads: Dict[str, Optional[torch.Tensor]], workspace: torch.Tensor,
                        dlam: Optional[torch.Tensor] = None, dhT: Optional[torch.Tensor] = None,
                        dh0: Optional[torch.Tensor] = None) -> None:
    stream = _check_layer(cfg, saved, (workspace, dlam, dhT, dh0, *params.values(), *grads.values()), X=X, dY=dY, dX=dX)
    p = params_struct(params)
    g = Grads(*[_ptr(grads.get(n)) for n in GRAD_FIELDS])
    _check(load().bpt_layer_bwd_recurrent(ctypes.byref(cfg), ctypes.byref(mixer), X.data_ptr(), ctypes.byref(p), saved.data_ptr(),
                                          dY.data_ptr(), _f32(dhT, (cfg.B, cfg.D), "dhT"), dX.data_ptr(), ctypes.byref(g),
                                          _f32(dlam, (cfg.D,), "dlam"), _f32(dh0, (cfg.B, cfg.D), "dh0"), workspace.data_ptr(),
                                          _nbytes(workspace), stream))


class RecurrentLayer(Layer):
    """A layer with the recurrence in place of attention; parameters as for Layer, and "lam" [D] (float32)."""

    def __init__(self, cfg: Config, device: str = "cuda", c: float = 8.0):
        super().__init__(cfg, device)
        _check(layer_recurrent_validate(cfg, c))
        self.c = c

    def forward(self, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]], h0: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """Y, the last states [B, D] and what backward takes."""
        Y = torch.empty(X.shape, dtype=self.out_dtype, device=self.device)
        hT = torch.empty((self.cfg.B, self.cfg.D), dtype=torch.float32, device=self.device)
        saved = self._bytes(layer_recurrent_saved_bytes(self.cfg))
        ws = workspace if workspace is not None else self._bytes(layer_recurrent_workspace_bytes(self.cfg, False))
        layer_fwd_recurrent(self.cfg, recur_mixer(self.cfg, params["lam"], self.c, h0, hT), X, params, Y, saved, ws)
        return Y, hT, saved

    def backward(self, X: torch.Tensor, params: Dict[str, Optional[torch.Tensor]], saved: torch.Tensor, dY: torch.Tensor,
                 h0: Optional[torch.Tensor] = None, dhT: Optional[torch.Tensor] = None, want: Optional[Tuple[str, ...]] = None,
                 workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Dict[str, torch.Tensor]]:
        """dX and the parameter gradients, with "dlam" and "dh0"; h0 as it was."""
        grads = self._grads(params, want)
        dX = torch.empty(X.shape, dtype=self.out_dtype, device=self.device)
        ws = workspace if workspace is not None else self._bytes(layer_recurrent_workspace_bytes(self.cfg, True))
        dlam = torch.empty(self.cfg.D, dtype=torch.float32, device=self.device)
        dh0 = torch.empty((self.cfg.B, self.cfg.D), dtype=torch.float32, device=self.device)
        layer_bwd_recurrent(self.cfg, recur_mixer(self.cfg, params["lam"], self.c, h0), X, params, saved, dY, dX, grads, ws, dlam, dhT, dh0)
        return dX, dict(grads, dlam=dlam, dh0=dh0)


# ---------------------------------------------------------------- distillation from a teacher's largest logits
DISTILL_MAX_K = 256                                  # pairs of a list


def make_distill_config(T: int, D: int, V: int, K: int, ldw: Optional[int] = None, block_rows: int = 0, tau: float = 1.0,
                        soft: float = 1.0, hard: float = 0.0, dtype: str = "bf16", grad_dtype: str = "f32", keep_bytes: int = 0) -> DistillConfig:
    """T tokens of width D, V logits, lists of K; see include/libbpt.h."""
    return DistillConfig(T, D, V, K, ldw if ldw is not None else (V + 63) // 64 * 64, block_rows, keep_bytes, tau, soft, hard, _DT[dtype],
                         _DT[grad_dtype], 0)


def distill_validate(cfg: DistillConfig) -> int:
    return load().bpt_distill_validate(ctypes.byref(cfg))


def distill_saved_bytes(cfg: DistillConfig) -> int:
    return load().bpt_distill_saved_bytes(ctypes.byref(cfg))


def distill_workspace_bytes(cfg: DistillConfig, backward: bool) -> int:
    return load().bpt_distill_workspace_bytes(ctypes.byref(cfg), int(backward))


@functools.lru_cache(maxsize=256)
def _distill_sizes(cfg: bytes) -> Tuple[int, int, int]:
    """Bytes of saved and of a forward's and a backward's workspace."""
    c = DistillConfig.from_buffer_copy(cfg)
    return distill_saved_bytes(c), distill_workspace_bytes(c, False), distill_workspace_bytes(c, True)


def _dense(t: Optional[torch.Tensor], dtype: torch.dtype, shape: Tuple[int, ...], name: str) -> Optional[int]:
    """The address of a contiguous tensor of a type and shape, or None."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be {list(shape)} contiguous {dtype}, not {list(t.shape)} of {t.dtype}")
    return t.data_ptr()


def distill_fwd(cfg: DistillConfig, h: torch.Tensor, W: torch.Tensor, values: torch.Tensor, index: torch.Tensor, loss: torch.Tensor,
                tokens: torch.Tensor, saved: torch.Tensor, workspace: torch.Tensor, targets: Optional[torch.Tensor] = None,
                weights: Optional[torch.Tensor] = None) -> None:
    T, D, K, dt = cfg.T, cfg.D, cfg.K, _TORCH_DT.get(cfg.dtype)
    ptrs = (_dense(h, dt, (T, D), "h"), _dense(W, dt, (D, cfg.ldw), "W"), _dense(values, torch.float32, (T, K), "values"),
            _dense(index, torch.int32, (T, K), "index"), _dense(targets, torch.int32, (T,), "targets"),
            _dense(weights, torch.float32, (T,), "weights"), _dense(loss, torch.float32, (3,), "loss"),
            _dense(tokens, torch.float32, (2, T), "tokens"))
    sp, dev = _saved_ptr(saved, _distill_sizes(bytes(cfg))[0]), h.get_device()
    same = all(t is None or t.get_device() == dev for t in (W, values, index, targets, weights, loss, tokens, saved, workspace))
    stream = _stream_on(dev, same)
    _check(load().bpt_distill_fwd(cfg, *ptrs, sp, workspace.data_ptr(), _nbytes(workspace), stream))


def distill_bwd(cfg: DistillConfig, h: torch.Tensor, W: torch.Tensor, saved: torch.Tensor, dloss: float, dh: torch.Tensor,
                dW: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    T, D, dt = cfg.T, cfg.D, _TORCH_DT.get(cfg.dtype)
    hp, Wp = _dense(h, dt, (T, D), "h"), _dense(W, dt, (D, cfg.ldw), "W")
    dhp, dWp = _dense(dh, dt, (T, D), "dh"), _dense(dW, _TORCH_DT.get(cfg.grad_dtype), (D, cfg.ldw), "dW")
    sp, dev = _saved_ptr(saved, _distill_sizes(bytes(cfg))[0]), h.get_device()
    same = all(t is None or t.get_device() == dev for t in (W, saved, dh, dW, workspace))
    stream = _stream_on(dev, same)
    _check(load().bpt_distill_bwd(cfg, hp, Wp, sp, float(dloss), dhp, dWp, workspace.data_ptr(), _nbytes(workspace), stream))


class DistillLoss:
    """Distillation loss of an LM head through libbpt; allocates its buffers with torch."""

    def __init__(self, cfg: DistillConfig):
        _check(distill_validate(cfg))
        self.cfg = cfg

    @staticmethod
    def _bytes(n: int, device) -> torch.Tensor:
        return torch.empty(max(n, 256), dtype=torch.uint8, device=device)

    def forward(self, h: torch.Tensor, W: torch.Tensor, values: torch.Tensor, index: torch.Tensor, targets: Optional[torch.Tensor] = None,
                weights: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """(loss, sum w kl, sum w ce) as three floats, kl and ce of each token [2, T], and what backward takes. For a loss without a
        backward, a configuration with keep_bytes = -1 stores no logits."""
        c, dev = self.cfg, h.device
        loss = torch.empty(3, dtype=torch.float32, device=dev)
        tokens = torch.empty((2, c.T), dtype=torch.float32, device=dev)
        ns, nb, _ = _distill_sizes(bytes(c))
        saved = self._bytes(ns, dev)
        distill_fwd(c, h, W, values, index, loss, tokens, saved, self._bytes(nb, dev), targets, weights)
        return loss, tokens, saved

    def backward(self, h: torch.Tensor, W: torch.Tensor, saved: torch.Tensor, dloss: float = 1.0,
                 want_dW: bool = True) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        c = self.cfg
        dh = torch.empty_like(h)
        dW = torch.empty_like(W, dtype=_TORCH_DT[c.grad_dtype]) if want_dW else None
        distill_bwd(c, h, W, saved, dloss, dh, dW, self._bytes(_distill_sizes(bytes(c))[2], h.device))
        return dh, dW
