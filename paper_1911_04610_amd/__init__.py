"""Python binding of libxpipe: XPipe's one-stage training step on MI355X.

The binding only marshals arguments to the C ABI declared in include/xpipe.h;
every step of the path runs in the library's HIP kernels.  PyTorch is used to
allocate device memory and to supply the HIP stream.  If the built library is
missing the import of any entry point raises: there is no CPU fallback.

Entry points (same names as the C ABI):
  xpipe_version_difference, xpipe_stage_query, Stage (xpipe_stage_create /
  _param_layout / _output_shape / xpipe_predict_weights / xpipe_stage_fwd /
  xpipe_stage_bwd / xpipe_adam_step / xpipe_rule_step / xpipe_stage_destroy /
  timing / recorded passes / xpipe_stage_run / xpipe_stage_set_clip), xpipe_schedule,
  xpipe_predict_flat, xpipe_adam_flat, xpipe_rule_flat (with clip= their _clipped forms);
  around a stage: xpipe_linear_fwd, xpipe_linear_bwd, xpipe_act_bwd,
  xpipe_embedding_fwd, xpipe_embedding_bwd, xpipe_grad_norm (over a TensorList),
  xpipe_clip_coef, xpipe_rmsnorm_fwd, xpipe_rmsnorm_bwd, xpipe_relbias_fwd,
  xpipe_relbias_bwd, xpipe_attention_fwd, xpipe_attention_bwd.
The last group checks devices, types and shapes (ValueError), runs on its
tensors' device (on `stream`, or that device's current stream) and allocates
the workspace that a call needs from torch on that stream, unless it is given one.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os
import struct
from typing import List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libxpipe.so")

OK, EINVAL, ESTATE, EHIP, EUNSUPPORTED = 0, 1, 2, 3, 4
F32, BF16 = 0, 1
FWD, BWD = 0, 1
KEEP_PRED = 2
PRED_EQ3, PRED_ADAMDIR, PRED_LITERAL, PRED_SMOOTHED = 0, 1, 2, 3
RULE_MOMENTUM_SGD, RULE_RMSPROP = 1, 2
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = 0, 1, 2, 3
ROUND_HALF_UP, ROUND_HALF_EVEN, ROUND_HALF_DOWN = 0, 1, 2
KINDS = {"linear": 0, "conv": 1, "bn": 2, "relu": 3, "add": 4, "maxpool2": 5, "avgpool3": 6,
         "gap": 7, "concat": 8, "softmax_ce": 9, "maxpool3s2": 10}
MAX_INPUTS = 4


class XPipeError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"xpipe status {status}: {msg}")
        self.status = status


class LayerDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("n_inputs", ctypes.c_int32),
                ("inputs", ctypes.c_int32 * MAX_INPUTS), ("cin", ctypes.c_int32),
                ("cout", ctypes.c_int32), ("k", ctypes.c_int32), ("has_bias", ctypes.c_int32),
                ("classes", ctypes.c_int32), ("stride", ctypes.c_int32), ("kw", ctypes.c_int32),
                ("pad", ctypes.c_int32)]


class HParams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("t", ctypes.c_int64), ("mode", ctypes.c_int32)]


class SchedEvent(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("time", "kind", "micro", "mini", "bellwether",
                                             "update_after", "version", "s_eq", "s_excl", "s_incl")]


class RunIO(ctypes.Structure):
    _fields_ = [("n_micro", ctypes.c_int32), ("x", ctypes.c_void_p), ("dy", ctypes.c_void_p),
                ("labels", ctypes.c_void_p), ("y", ctypes.c_void_p), ("loss", ctypes.c_void_p),
                ("dx", ctypes.c_void_p)]


class RuleParams(ctypes.Structure):
    _fields_ = [("rule", ctypes.c_int32), ("lr", ctypes.c_double), ("momentum", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("alpha", ctypes.c_double), ("eps", ctypes.c_double)]


class TensorDesc(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("n", ctypes.c_int64)]


class LinearFwdArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cin", ctypes.c_int32), ("cout", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("act", ctypes.c_int32),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64),
                ("bias", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64),
                ("preact", ctypes.c_void_p), ("ldz", ctypes.c_int64), ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64)]


class LinearBwdArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cin", ctypes.c_int32), ("cout", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("act", ctypes.c_int32),
                ("dz", ctypes.c_void_p), ("lddz", ctypes.c_int64), ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("preact", ctypes.c_void_p), ("ldz", ctypes.c_int64),
                ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64), ("dx", ctypes.c_void_p),
                ("lddx", ctypes.c_int64), ("grad_W", ctypes.c_void_p), ("grad_b", ctypes.c_void_p)]


class RmsnormFwdArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_double),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("sum", ctypes.c_void_p), ("lds", ctypes.c_int64),
                ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64)]


class RmsnormBwdArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_double),
                ("dy", ctypes.c_void_p), ("lddy", ctypes.c_int64), ("h", ctypes.c_void_p), ("ldh", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64),
                ("dx", ctypes.c_void_p), ("lddx", ctypes.c_int64), ("grad_weight", ctypes.c_void_p)]


class Heads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class AttentionInputs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "nq", "nk", "heads", "kv_heads", "head_dim", "dtype", "causal", "bias_range")] + \
               [("scale", ctypes.c_double), ("cap", ctypes.c_double), ("q", Heads), ("k", Heads), ("v", Heads)] + \
               [(n, ctypes.c_void_p) for n in ("q_len", "k_len", "prefix", "q_doc", "k_doc", "bias")]


class AttentionFwdArgs(ctypes.Structure):
    _fields_ = [("in_", AttentionInputs), ("o", Heads), ("stats", ctypes.c_void_p)]


class AttentionBwdArgs(ctypes.Structure):
    _fields_ = [("in_", AttentionInputs), ("dout", Heads), ("o", Heads), ("stats", ctypes.c_void_p),
                ("dq", Heads), ("dk", Heads), ("dv", Heads), ("grad_bias", ctypes.c_void_p)]


@dataclasses.dataclass
class Rule:
    """Update rule besides Adam (xpipe_rule_hparams)."""
    rule: int = RULE_MOMENTUM_SGD
    lr: float = 1e-2
    momentum: float = 0.9
    weight_decay: float = 0.0
    alpha: float = 0.99
    eps: float = 1e-8

    def c(self) -> RuleParams:
        return RuleParams(int(self.rule), self.lr, self.momentum, self.weight_decay, self.alpha, self.eps)


@dataclasses.dataclass
class Hyper:
    lr: float = 1e-3
    beta1: float = 0.9
    beta2: float = 0.999
    eps: float = 1e-8
    mode: int = PRED_EQ3

    def c(self, t: int) -> HParams:
        return HParams(self.lr, self.beta1, self.beta2, self.eps, int(t), int(self.mode))


_lib = None
_torch = None  # set with the library
_P = ctypes.c_void_p
_I32, _I64, _SZ = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t

_SIGS = {
    "xpipe_version_difference": [_I32, _I32, _I32, _I32, _I32, _I32, ctypes.POINTER(_I32)],
    "xpipe_stage_query": [_P, _I32, _I32, _I32, _I32, _I32, _I32, ctypes.POINTER(_I64),
                          ctypes.POINTER(_SZ)],
    "xpipe_stage_create": [_P, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _P, _P, _P, _P, _P,
                           _P, _P, _P, _SZ, ctypes.POINTER(_P)],
    "xpipe_stage_create_static": [_P, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _P, _P, _P, _P,
                                  _P, _P, _P, ctypes.POINTER(_P)],
    "xpipe_stage_num_param_tensors": [_P, ctypes.POINTER(_I32)],
    "xpipe_stage_param_layout": [_P, _I32, ctypes.POINTER(_I64), ctypes.POINTER(_I64)],
    "xpipe_stage_output_shape": [_P] + [ctypes.POINTER(_I32)] * 4,
    "xpipe_predict_weights": [_P, _I32, _I32, ctypes.POINTER(HParams)],
    "xpipe_stage_fwd": [_P, _P, _P, _P, _P],
    "xpipe_stage_bwd": [_P, _P, _P, _P, _P],
    "xpipe_adam_step": [_P, ctypes.POINTER(HParams), _I32, _I32, _I32],
    "xpipe_partition": [_P, _I32, _I32, ctypes.POINTER(_I32)],
    "xpipe_schedule": [_I32, _I32, _I32, _I32, _I32, _I32, _P, _I32, ctypes.POINTER(_I32)],
    "xpipe_stage_run": [_P, _P, _I32, ctypes.POINTER(RunIO), ctypes.POINTER(HParams), _P, _P, _P, _I32],
    "xpipe_rule_step": [_P, ctypes.POINTER(RuleParams), ctypes.POINTER(HParams), _P, _P, _I32, _I32,
                        _I32],
    "xpipe_rule_flat": [_P, _P, _P, _P, _P, _P, _I64, ctypes.POINTER(RuleParams),
                        ctypes.POINTER(HParams), _I32, _P, _I32, _P, _I32, _P],
    "xpipe_stage_destroy": [_P],
    "xpipe_predict_flat": [_P, _P, _P, _P, _P, _I64, _I32, ctypes.POINTER(HParams), _P],
    "xpipe_adam_flat": [_P, _P, _P, _P, _I64, ctypes.POINTER(HParams), _I32, _P, _I32, _P, _I32,
                        _P],
    "xpipe_adam_flat_clipped": [_P, _P, _P, _P, _I64, ctypes.POINTER(HParams), _I32, _P, _I32, _P, _I32,
                                _P, _P],
    "xpipe_rule_flat_clipped": [_P, _P, _P, _P, _P, _P, _I64, ctypes.POINTER(RuleParams),
                                ctypes.POINTER(HParams), _I32, _P, _I32, _P, _I32, _P, _P],
    "xpipe_stage_set_clip": [_P, ctypes.c_double, _P, _P, _SZ],
    "xpipe_grad_norm_query": [_P, _I32, ctypes.POINTER(_SZ)],
    "xpipe_grad_norm": [_P, _I32, _I32, ctypes.c_double, _P, _P, _P, _SZ, _P],
    "xpipe_clip_coef": [_P, _I64, ctypes.c_double, _P, _P],
    "xpipe_linear_fwd_query": [_P, ctypes.POINTER(_SZ)],  # _P: LinearFwdArgs / LinearBwdArgs
    "xpipe_linear_bwd_query": [_P, ctypes.POINTER(_SZ)],
    "xpipe_linear_fwd": [_P, _P, _SZ, _P],
    "xpipe_linear_bwd": [_P, _P, _SZ, _P],
    "xpipe_act_bwd": [_P, _P, _P, _I64, _I32, _I32, _P],
    "xpipe_embedding_fwd": [_P, _P, _I64, _I32, _I32, ctypes.c_double, _I32, _P, _P],
    "xpipe_embedding_bwd_query": [_I64, _I32, _I32, ctypes.POINTER(_SZ)],
    "xpipe_embedding_bwd": [_P, _P, _I64, _I32, _I32, ctypes.c_double, _I32, _P, _P, _SZ, _P],
    "xpipe_rmsnorm_fwd": [_P, _P],
    "xpipe_rmsnorm_bwd_query": [_P, ctypes.POINTER(_SZ)],
    "xpipe_rmsnorm_bwd": [_P, _P, _SZ, _P],
    "xpipe_relbias_fwd": [_P, _I32, _I32, _I32, _I32, _P, _P],
    "xpipe_relbias_bwd": [_P, _I32, _I32, _I32, _I32, _P, _P],
    "xpipe_attention_fwd_query": [_P, ctypes.POINTER(_SZ)],
    "xpipe_attention_bwd_query": [_P, ctypes.POINTER(_SZ)],
    "xpipe_attention_fwd": [_P, _P, _SZ, _P],
    "xpipe_attention_bwd": [_P, _P, _SZ, _P],
    "xpipe_probe_copy": [_P, _P, _I64, _P],
    "xpipe_probe_mfma": [_P, _I32, _I32, _P],
    "xpipe_probe_graph": [_P, _I32, _I32, _I32, _I32, ctypes.POINTER(ctypes.c_double), _P],
    "xpipe_probe_stream": [ctypes.POINTER(_P), _I32, ctypes.POINTER(_P), _I32, _I64, _P],
    "xpipe_stage_set_timing": [_P, _I32],
    "xpipe_stage_set_graphs": [_P, _I32],
    "xpipe_stage_set_fwd_stream": [_P, _P, ctypes.c_size_t, ctypes.POINTER(_P)],
    "xpipe_stage_timing_count": [_P, ctypes.POINTER(_I32)],
    "xpipe_stage_timing_entry": [_P, _I32, ctypes.POINTER(ctypes.c_char_p),
                                 ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_I64),
                                 ctypes.POINTER(ctypes.c_double)],
}


def lib() -> ctypes.CDLL:
    """The loaded libxpipe.so; raises if it has not been built."""
    global _lib, _torch
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_1911_04610_amd.build`")
        # The library and PyTorch must share one HIP runtime (the library
        # launches on torch's streams and into torch's allocations).  torch
        # ships its own copy of the runtime; loaded after the library, it would
        # come in as a second runtime with its own device contexts.  Importing
        # torch first makes the library bind to torch's copy.
        import torch
        L = ctypes.CDLL(LIB_PATH)
        for name, args in _SIGS.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        L.xpipe_last_error.argtypes = []
        L.xpipe_last_error.restype = ctypes.c_char_p
        _torch = torch
        _lib = L
    return _lib


def _check(status: int):
    if status != OK:
        raise XPipeError(status, lib().xpipe_last_error().decode())


def layer_descs(layers: Sequence[dict]):
    """Layer dicts (kind, inputs, cin, cout, k, bias, classes) -> LayerDesc array."""
    arr = (LayerDesc * len(layers))()
    for i, L in enumerate(layers):
        d = arr[i]
        d.kind = KINDS[L["kind"]]
        ins = list(L["inputs"])
        d.n_inputs = len(ins)
        for j in range(MAX_INPUTS):
            d.inputs[j] = ins[j] if j < len(ins) else 0
        d.cin = int(L.get("cin", 0))
        d.cout = int(L.get("cout", 0))
        d.k = int(L.get("k", 1))
        d.has_bias = int(bool(L.get("bias", False)))
        d.classes = int(L.get("classes", 0))
        d.stride = int(L.get("stride", 1))
        d.kw = int(L.get("kw", d.k))
        d.pad = {"same": 0, "valid": 1}[L.get("pad", "same")]
    return arr


def xpipe_version_difference(size: int, T: int, rank: int, direction: int,
                             rounding: int = ROUND_HALF_UP, ceil_half_rank: bool = False) -> int:
    out = _I32(0)
    _check(lib().xpipe_version_difference(size, T, rank, direction, rounding,
                                          int(ceil_half_rank), ctypes.byref(out)))
    return out.value


def xpipe_stage_query(layers, micro_batch: int, in_shape, dtype: int):
    H, W, C = _hwc(in_shape)
    d = layer_descs(layers)
    P = _I64(0)
    ws = _SZ(0)
    _check(lib().xpipe_stage_query(d, len(layers), micro_batch, H, W, C, dtype, ctypes.byref(P),
                                   ctypes.byref(ws)))
    return P.value, ws.value


def _hwc(in_shape):
    if len(in_shape) == 1:
        return 1, 1, int(in_shape[0])
    return int(in_shape[0]), int(in_shape[1]), int(in_shape[2])


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_ptr(stream) -> Optional[int]:
    import torch
    if stream is None and torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


class Stage:
    """One stage on the current GPU: parameters, moments, gradient accumulator,
    prediction caches and workspace are torch tensors owned by this object."""

    def __init__(self, layers: List[dict], micro_batch: int, T: int, in_shape, dtype: int = F32,
                 device="cuda", stream=None, static_workspace: bool = False):
        """static_workspace=True creates the stage with xpipe_stage_create_static
        (the library's static device workspace; no workspace tensor here)."""
        import torch
        self.layers = layers
        self.micro_batch, self.T, self.dtype = micro_batch, T, dtype
        self.in_shape = tuple(in_shape)
        self.device = torch.device(device)
        self.stream = stream
        self.P, ws = xpipe_stage_query(layers, micro_batch, in_shape, dtype)
        self.ws_bytes = ws
        self.fwd_workspace = self.fwd_stream = None
        self._clip = self._clip_ws = None
        f32 = dict(dtype=torch.float32, device=self.device)
        self.W = torch.zeros(self.P, **f32)
        self.m = torch.zeros(self.P, **f32)
        self.v = torch.zeros(self.P, **f32)
        self.grad = torch.zeros(self.P, **f32)
        self.w_pred_fwd = torch.zeros(self.P, **f32)
        self.w_pred_bwd = torch.zeros(self.P, **f32)
        self._h = _P()
        H, W, C = _hwc(in_shape)
        self._descs = layer_descs(layers)
        # what the stage runs on, whatever stream is current later
        self._run_stream = stream if stream is not None else torch.cuda.current_stream()
        if static_workspace:
            self.workspace = None
            _check(lib().xpipe_stage_create_static(self._descs, len(layers), micro_batch, T, H, W, C,
                                                   dtype, _stream_ptr(stream), _ptr(self.W),
                                                   _ptr(self.m), _ptr(self.v), _ptr(self.grad),
                                                   _ptr(self.w_pred_fwd), _ptr(self.w_pred_bwd),
                                                   ctypes.byref(self._h)))
        else:
            self.workspace = torch.empty(max(ws, 256) + 256, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            ws_ptr = (base + 255) // 256 * 256
            _check(lib().xpipe_stage_create(self._descs, len(layers), micro_batch, T, H, W, C, dtype,
                                            _stream_ptr(stream), _ptr(self.W), _ptr(self.m),
                                            _ptr(self.v), _ptr(self.grad), _ptr(self.w_pred_fwd),
                                            _ptr(self.w_pred_bwd), ws_ptr, ws, ctypes.byref(self._h)))
        n = _I32(0)
        _check(lib().xpipe_stage_num_param_tensors(self._h, ctypes.byref(n)))
        self.layout = []
        for i in range(n.value):
            off, cnt = _I64(0), _I64(0)
            _check(lib().xpipe_stage_param_layout(self._h, i, ctypes.byref(off), ctypes.byref(cnt)))
            self.layout.append((off.value, cnt.value))
        dims = [_I32(0) for _ in range(4)]
        _check(lib().xpipe_stage_output_shape(self._h, *[ctypes.byref(d) for d in dims]))
        self.out_shape = tuple(d.value for d in dims)

    # ---- parameter marshalling (host <-> flat device buffers)
    def set_flat(self, buf, tensors):
        """Copy per-tensor host arrays into a flat device buffer (padding stays 0)."""
        import numpy as np
        import torch
        host = np.zeros(self.P, np.float32)
        for (off, cnt), a in zip(self.layout, tensors):
            host[off:off + cnt] = np.asarray(a, np.float32).ravel()
        buf.copy_(torch.from_numpy(host).to(self.device))

    def get_tensors(self, buf):
        """Split a flat device buffer into per-tensor host arrays (fp64 copies)."""
        import numpy as np
        host = buf.detach().cpu().numpy().astype(np.float64)
        return [host[off:off + cnt] for off, cnt in self.layout]

    # ---- the ABI calls
    def xpipe_predict_weights(self, which: int, s: int, hp: Hyper, t: int):
        c = hp.c(t)
        _check(lib().xpipe_predict_weights(self._h, which, s, ctypes.byref(c)))

    def xpipe_stage_fwd(self, x, y, labels=None, loss=None):
        _check(lib().xpipe_stage_fwd(self._h, _ptr(x), _ptr(y), _ptr(labels), _ptr(loss)))

    def xpipe_stage_set_fwd_stream(self, enable: bool):
        """Forwards on a stream of the stage's own, with a workspace of their
        own (allocated here), beside the backwards on the stage's stream.
        Returns that stream as a torch.cuda.ExternalStream (None when
        disabled), for ordering the forwards' inputs and outputs."""
        import torch
        if not enable:
            _check(lib().xpipe_stage_set_fwd_stream(self._h, None, 0, None))
            self.fwd_workspace = self.fwd_stream = None
            return None
        buf = torch.empty(max(self.ws_bytes, 256) + 256, dtype=torch.uint8, device=self.device)
        ptr = (buf.data_ptr() + 255) // 256 * 256
        s = _P()
        _check(lib().xpipe_stage_set_fwd_stream(self._h, ptr, self.ws_bytes, ctypes.byref(s)))
        self.fwd_workspace = buf
        self.fwd_stream = torch.cuda.ExternalStream(s.value, device=self.device)
        return self.fwd_stream

    def xpipe_stage_bwd(self, x, dy=None, labels=None, dx=None):
        _check(lib().xpipe_stage_bwd(self._h, _ptr(x), _ptr(dy), _ptr(labels), _ptr(dx)))

    def xpipe_adam_step(self, hp: Hyper, t: int, s_fwd_next: int = 0, s_bwd_next: int = 0,
                        emit_pred: bool = False):
        c = hp.c(t)
        _check(lib().xpipe_adam_step(self._h, ctypes.byref(c), s_fwd_next, s_bwd_next,
                                     int(emit_pred)))

    def xpipe_rule_step(self, rule: Rule, hp: Hyper, t: int, buf, sq=None, s_fwd_next: int = 0,
                        s_bwd_next: int = 0, emit_pred: bool = False):
        """Update with momentum SGD or RMSProp; buf / sq are fp32 device tensors
        of n_params elements carried between calls (zero before the first)."""
        r, c = rule.c(), hp.c(t)
        _check(lib().xpipe_rule_step(self._h, ctypes.byref(r), ctypes.byref(c), _ptr(buf), _ptr(sq),
                                     s_fwd_next, s_bwd_next, int(emit_pred)))

    def xpipe_stage_run(self, events, x, y, hp: Hyper, t: int, dy=None, labels=None, loss=None,
                        dx=None, rule: Optional[Rule] = None, buf=None, sq=None, draft=False):
        """Run schedule events (from xpipe_schedule) on this stage.  x, y, dy,
        labels, dx: lists of device tensors indexed by micro-batch - 1; loss: a
        device fp32 tensor [n_micro] or None."""
        n = len(x)
        arr = lambda ts: None if ts is None else (ctypes.c_void_p * n)(*[_ptr(a) for a in ts])
        keep = [arr(x), arr(dy), arr(labels), arr(y), arr(dx)]
        io = RunIO(n, *(ctypes.cast(a, ctypes.c_void_p) if a is not None else None for a in keep[:3]),
                   ctypes.cast(keep[3], ctypes.c_void_p), _ptr(loss),
                   ctypes.cast(keep[4], ctypes.c_void_p) if keep[4] is not None else None)
        ev = (SchedEvent * len(events))(*events)
        c = hp.c(t)
        r = rule.c() if rule is not None else None
        _check(lib().xpipe_stage_run(self._h, ctypes.cast(ev, ctypes.c_void_p), len(events),
                                     ctypes.byref(io), ctypes.byref(c),
                                     ctypes.cast(ctypes.pointer(r), ctypes.c_void_p) if r is not None else None,
                                     _ptr(buf), _ptr(sq), int(draft)))

    def xpipe_stage_set_clip(self, max_norm: float, norm_coef):
        """Clip every later update by the global gradient norm.  norm_coef: fp32
        device tensor of two elements {norm, coefficient} (None: off).  With
        max_norm > 0 each update computes them over this stage's accumulator
        (workspace allocated here); with 0 the caller writes them before the
        update (xpipe_grad_norm over several buffers)."""
        ws, size = None, _SZ(0)
        if norm_coef is not None:
            _check_norm_coef(norm_coef, self.grad.get_device())
            # the stage's stream writes and reads it: given out again only behind the updates in flight
            norm_coef.record_stream(self._run_stream)
            if max_norm > 0:
                one = TensorDesc(_ptr(self.grad), self.P)
                _check(lib().xpipe_grad_norm_query(ctypes.byref(one), 1, ctypes.byref(size)))
                if self._clip_ws is None:  # kept from then on: updates in flight may use it
                    with _torch.cuda.stream(self._run_stream):
                        self._clip_ws = _torch.empty(max(size.value, 8), dtype=_torch.uint8, device=self.device)
                ws = self._clip_ws
        _check(lib().xpipe_stage_set_clip(self._h, max_norm, _ptr(norm_coef), _ptr(ws), size.value))
        self._clip = norm_coef  # kept while the stage uses it

    def set_timing(self, enable: bool):
        _check(lib().xpipe_stage_set_timing(self._h, int(enable)))

    def set_graphs(self, enable: bool):
        _check(lib().xpipe_stage_set_graphs(self._h, int(enable)))

    def timing(self):
        """{kernel name: (ms, launches, work)} over the launches since set_timing(True)."""
        n = _I32(0)
        _check(lib().xpipe_stage_timing_count(self._h, ctypes.byref(n)))
        out = {}
        for i in range(n.value):
            name, ms, cnt, work = ctypes.c_char_p(), ctypes.c_double(0), _I64(0), ctypes.c_double(0)
            _check(lib().xpipe_stage_timing_entry(self._h, i, ctypes.byref(name), ctypes.byref(ms),
                                                  ctypes.byref(cnt), ctypes.byref(work)))
            out[name.value.decode()] = (ms.value, cnt.value, work.value)
        return out

    def destroy(self):
        if self._h:
            lib().xpipe_stage_destroy(self._h)
            self._h = _P()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def xpipe_predict_flat(W, m, v, out, out_bf16, s: int, hp: Hyper, t: int, stream=None):
    c = hp.c(t)
    _check(lib().xpipe_predict_flat(_ptr(W), _ptr(m), _ptr(v), _ptr(out), _ptr(out_bf16),
                                    W.numel(), s, ctypes.byref(c), _stream_ptr(stream)))


def xpipe_partition(layers, stages: int) -> List[int]:
    """first layer index of each stage, and len(layers) (Sec. IV-B's partition)."""
    arr = layer_descs(layers)
    first = (_I32 * (stages + 1))()
    _check(lib().xpipe_partition(arr, len(layers), stages, first))
    return list(first)


def xpipe_schedule(size: int, T: int, rank: int, minibatches: int, rounding: int = 0,
                   ceil_half_rank: bool = False) -> List[SchedEvent]:
    """Events of GPU `rank` in the unit-time pipeline schedule (host only)."""
    n = _I32(0)
    _check(lib().xpipe_schedule(size, T, rank, minibatches, rounding, int(ceil_half_rank), None, 0,
                                ctypes.byref(n)))
    ev = (SchedEvent * max(n.value, 1))()
    _check(lib().xpipe_schedule(size, T, rank, minibatches, rounding, int(ceil_half_rank),
                                ctypes.cast(ev, ctypes.c_void_p), n.value, ctypes.byref(n)))
    return list(ev)[:n.value]


def xpipe_rule_flat(W, buf, sq, m, v, G, rule: Rule, hp: Hyper, t: int, zero_grad=True, pred_fwd=None,
                    s_fwd=0, pred_bwd=None, s_bwd=0, stream=None, clip=None):
    """clip: {norm, coefficient} of xpipe_grad_norm; the update reads G times the coefficient."""
    r, c = rule.c(), hp.c(t)
    if clip is not None:
        _check_norm_coef(clip, W.get_device())
        _check(lib().xpipe_rule_flat_clipped(_ptr(W), _ptr(buf), _ptr(sq), _ptr(m), _ptr(v), _ptr(G), W.numel(),
                                             ctypes.byref(r), ctypes.byref(c), int(zero_grad), _ptr(pred_fwd), s_fwd,
                                             _ptr(pred_bwd), s_bwd, _ptr(clip), _stream_ptr(stream)))
        return
    _check(lib().xpipe_rule_flat(_ptr(W), _ptr(buf), _ptr(sq), _ptr(m), _ptr(v), _ptr(G), W.numel(),
                                 ctypes.byref(r), ctypes.byref(c), int(zero_grad), _ptr(pred_fwd), s_fwd,
                                 _ptr(pred_bwd), s_bwd, _stream_ptr(stream)))


def xpipe_probe_copy(src, dst, stream=None):
    """dst[:] = src[:] (same byte size, multiple of 16) with the library's copy probe."""
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("src and dst must have the same byte size")
    _check(lib().xpipe_probe_copy(_ptr(src), _ptr(dst), nbytes, _stream_ptr(stream)))


def xpipe_probe_mfma(out, iters: int, stream=None):
    """One wave per element of the float32 tensor `out`, `iters` rounds of 8 MFMAs each."""
    _check(lib().xpipe_probe_mfma(_ptr(out), out.numel(), int(iters), _stream_ptr(stream)))


def xpipe_probe_graph(scratch, width: int, length: int, reps: int, spin: int, stream=None):
    """Recorded-graph fork/join probe: (us per diamond with `width` branches of
    `length` launches, us for the same launches as one chain).  scratch: a
    float32 device tensor of at least 2048 elements."""
    if scratch.numel() < 2048:
        raise ValueError("scratch needs at least 2048 floats")
    out = (ctypes.c_double * 2)()
    _check(lib().xpipe_probe_graph(_ptr(scratch), int(width), int(length), int(reps), int(spin),
                                   out, _stream_ptr(stream)))
    return out[0], out[1]


def xpipe_probe_stream(srcs, dsts, stream=None):
    """Bare stream: every float32 tensor in srcs read once, every one in dsts
    written once (all of one size, a multiple of 4 elements)."""
    n = dsts[0].numel()
    S = (_P * max(len(srcs), 1))(*[_ptr(t) for t in srcs])
    D = (_P * len(dsts))(*[_ptr(t) for t in dsts])
    _check(lib().xpipe_probe_stream(S, len(srcs), D, len(dsts), n, _stream_ptr(stream)))


def xpipe_adam_flat(W, m, v, G, hp: Hyper, t: int, zero_grad=True, pred_fwd=None, s_fwd=0,
                    pred_bwd=None, s_bwd=0, stream=None, clip=None):
    """clip: {norm, coefficient} of xpipe_grad_norm; the update reads G times the coefficient."""
    c = hp.c(t)
    if clip is not None:
        _check_norm_coef(clip, W.get_device())
        _check(lib().xpipe_adam_flat_clipped(_ptr(W), _ptr(m), _ptr(v), _ptr(G), W.numel(), ctypes.byref(c),
                                             int(zero_grad), _ptr(pred_fwd), s_fwd, _ptr(pred_bwd), s_bwd,
                                             _ptr(clip), _stream_ptr(stream)))
        return
    _check(lib().xpipe_adam_flat(_ptr(W), _ptr(m), _ptr(v), _ptr(G), W.numel(), ctypes.byref(c),
                                 int(zero_grad), _ptr(pred_fwd), s_fwd, _ptr(pred_bwd), s_bwd,
                                 _stream_ptr(stream)))


# ---------------------------------------------------------------- operators around a stage
# A small call's time is the host's: checks are `if`s, so that a message is only made
# where one fails, and a tensor is asked for each property once.
def _check_norm_coef(t, dev: int):
    lib()
    if t.dtype is not _torch.float32 or t.numel() != 2 or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError("{norm, coefficient}: two contiguous float32 elements on the gradients' device expected")


def _dtype_of(t) -> int:
    if t.dtype is _torch.bfloat16:
        return BF16
    if t.dtype is _torch.float32:
        return F32
    raise ValueError(f"bfloat16 or float32 expected, not {t.dtype}")


def _matrix(name, t, dtype, dev, rows, cols):
    """(pointer, row pitch in elements) of a [rows, cols] tensor of that type and device, its rows contiguous."""
    if t is None:
        return 0, 0
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name}: another type or device")
    if t.shape != (rows, cols):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, ({rows}, {cols}) expected")
    ld, inner = t.stride()
    if rows <= 1:
        ld = cols
    if ld < cols or (inner != 1 and cols > 1):
        raise ValueError(f"{name}: rows must be contiguous")
    return t.data_ptr(), ld


def _vector(name, t, dev, n):
    if t is None:
        return 0
    if t.dtype is not _torch.float32 or t.get_device() != dev or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous float32 elements on the same device expected")
    return t.data_ptr()


def _device_of(t):
    """(index of the tensor's GPU, whether it is the current one); raises for a CPU tensor."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError("tensors on the GPU expected")
    return dev, dev == _torch._C._cuda_getDevice()


def _raw_stream(dev, stream):
    """The HIP stream of a call on GPU dev (the current one): `stream`, or the device's current stream."""
    if stream is None:
        return _torch._C._cuda_getCurrentRawStream(dev)
    if stream.device.index != dev:
        raise ValueError("the stream is another device's")
    return stream.cuda_stream


def _workspace(need, given, t, stream):
    """(pointer, bytes, tensor to hold during the call) of a 256-byte aligned workspace."""
    if need == 0:
        return None, 0, None
    if given is not None:
        if given.get_device() != t.get_device() or not given.is_contiguous():
            raise ValueError("workspace: contiguous, on the same device expected")
        skip = -given.data_ptr() % 256
        return given.data_ptr() + skip, max(0, given.numel() * given.element_size() - skip), given
    if stream is None:
        ws = _torch.empty(need + 256, dtype=_torch.uint8, device=t.device)
    else:  # the allocator then gives it out again in that stream's order
        with _torch.cuda.stream(stream):
            ws = _torch.empty(need + 256, dtype=_torch.uint8, device=t.device)
    ptr = ws.data_ptr()
    return ptr + -ptr % 256, need, ws


# LinearFwdArgs and LinearBwdArgs as struct formats: packing is a quarter of a
# ctypes structure's time
_FWD_FORMAT, _BWD_FORMAT = struct.Struct("qiiiiPqPqPPqPqPq"), struct.Struct("qiiiiPqPqPqPqPqPqPP")
assert _FWD_FORMAT.size == ctypes.sizeof(LinearFwdArgs) and _BWD_FORMAT.size == ctypes.sizeof(LinearBwdArgs)


def xpipe_linear_fwd(x, W, bias, y, act: int = ACT_NONE, residual=None, preact=None, workspace=None, stream=None):
    """y = act(x W^T + bias) + residual; preact (optional) receives the
    pre-activation.  Matrices of one type (bfloat16 or float32), their rows
    contiguous; bias float32 or None.  residual may be y itself."""
    L = lib()
    dev, here = _device_of(x)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_linear_fwd(x, W, bias, y, act, residual, preact, workspace, stream)
    if x.dim() != 2 or W.dim() != 2:
        raise ValueError("x [rows, cin] and W [cout, cin] expected")
    (rows, cin), cout, dt = x.shape, W.shape[0], x.dtype
    a = _FWD_FORMAT.pack(rows, cin, cout, _dtype_of(x), act, *_matrix("x", x, dt, dev, rows, cin),
                         *_matrix("W", W, dt, dev, cout, cin), _vector("bias", bias, dev, cout),
                         *_matrix("residual", residual, dt, dev, rows, cout), *_matrix("preact", preact, dt, dev, rows, cout),
                         *_matrix("y", y, dt, dev, rows, cout))
    need = _SZ()
    _check(L.xpipe_linear_fwd_query(a, ctypes.byref(need)))
    ptr, size, keep = _workspace(need.value, workspace, x, stream)
    _check(L.xpipe_linear_fwd(a, ptr, size, _raw_stream(dev, stream)))


def xpipe_linear_bwd(dz, x, W, dx=None, grad_W=None, grad_b=None, act: int = ACT_NONE, preact=None, residual=None,
                     workspace=None, stream=None):
    """Gradients of a linear layer from dz, the gradient of its pre-activation:
    dx = (dz W) act'(preact) + residual, grad_W += dz^T x, grad_b += dz's row sum
    (float32), each optional.  act and preact are those of the layer whose output
    x is, so dx is that layer's dz; residual is a gradient that reaches x another
    way and may be dx itself."""
    L = lib()
    dev, here = _device_of(dz)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_linear_bwd(dz, x, W, dx, grad_W, grad_b, act, preact, residual, workspace, stream)
    given = x if x is not None else W
    if dz.dim() != 2 or given is None or given.dim() != 2:
        raise ValueError("dz [rows, cout], and x [rows, cin] or W [cout, cin] expected")
    (rows, cout), cin, dt = dz.shape, given.shape[1], dz.dtype
    a = _BWD_FORMAT.pack(rows, cin, cout, _dtype_of(dz), act, *_matrix("dz", dz, dt, dev, rows, cout),
                         *_matrix("x", x, dt, dev, rows, cin), *_matrix("W", W, dt, dev, cout, cin),
                         *_matrix("preact", preact, dt, dev, rows, cin), *_matrix("residual", residual, dt, dev, rows, cin),
                         *_matrix("dx", dx, dt, dev, rows, cin), _vector("grad_W", grad_W, dev, cout * cin),
                         _vector("grad_b", grad_b, dev, cout))
    need = _SZ()
    _check(L.xpipe_linear_bwd_query(a, ctypes.byref(need)))
    ptr, size, keep = _workspace(need.value, workspace, dz, stream)
    _check(L.xpipe_linear_bwd(a, ptr, size, _raw_stream(dev, stream)))


def xpipe_act_bwd(dy, z, dz, act: int, stream=None):
    """dz = dy act'(z): contiguous tensors of one type and shape (dz may be dy or z)."""
    L = lib()
    dev, here = _device_of(dy)
    for t in (dy, z, dz):
        if t.shape != dy.shape or t.dtype is not dy.dtype or t.get_device() != dev or not t.is_contiguous():
            raise ValueError("contiguous tensors of one type, shape and device expected")
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_act_bwd(dy, z, dz, act, stream)
    _check(L.xpipe_act_bwd(dy.data_ptr(), z.data_ptr(), dz.data_ptr(), dy.numel(), act, _dtype_of(dy),
                           _raw_stream(dev, stream)))


def _check_embedding(rows, name, tokens, table, dev):
    """(vocab, dim, number of tokens)"""
    if table.dim() != 2 or not table.is_contiguous():
        raise ValueError("table and grad: contiguous [vocab, dim] expected")
    (vocab, dim), n = table.shape, tokens.numel()
    if vocab >= 1 << 31 or dim >= 1 << 31:  # (ctypes would cut them to 32 bits)
        raise ValueError("table and grad: 2^31 rows or columns or more")
    if tokens.dtype is not _torch.int32 or not tokens.is_contiguous() or tokens.get_device() != dev:
        raise ValueError("tokens: contiguous int32 on the same device expected")
    if (rows.dim() < 1 or not rows.is_contiguous() or rows.get_device() != dev or rows.shape[-1] != dim or
            rows.numel() != n * dim):
        raise ValueError(f"{name}: contiguous [tokens, dim] on the same device expected")
    return vocab, dim, n


def xpipe_embedding_fwd(table, tokens, y, scale: float = 1.0, stream=None):
    """y[i] = scale * table[tokens[i]] (zeros where a token is outside the table).
    table [vocab, dim] and y [..., dim] of one type; tokens int32."""
    L = lib()
    dev, here = _device_of(table)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_embedding_fwd(table, tokens, y, scale, stream)
    vocab, dim, n = _check_embedding(y, "y", tokens, table, dev)
    if y.dtype is not table.dtype:
        raise ValueError("y: the table's type expected")
    _check(L.xpipe_embedding_fwd(table.data_ptr(), tokens.data_ptr(), n, vocab, dim, scale, _dtype_of(table), y.data_ptr(),
                                 _raw_stream(dev, stream)))


def xpipe_embedding_bwd(dy, tokens, grad, scale: float = 1.0, workspace=None, stream=None):
    """grad[tokens[i]] += scale * dy[i], for the tokens inside the table.
    grad: contiguous float32 [vocab, dim]; dy [..., dim]; tokens int32."""
    L = lib()
    dev, here = _device_of(grad)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_embedding_bwd(dy, tokens, grad, scale, workspace, stream)
    vocab, dim, n = _check_embedding(dy, "dy", tokens, grad, dev)
    if grad.dtype is not _torch.float32:
        raise ValueError("grad: float32 expected")
    need = _SZ()
    _check(L.xpipe_embedding_bwd_query(n, vocab, dim, ctypes.byref(need)))
    ptr, size, keep = _workspace(need.value, workspace, grad, stream)
    _check(L.xpipe_embedding_bwd(dy.data_ptr(), tokens.data_ptr(), n, vocab, dim, scale, _dtype_of(dy), grad.data_ptr(),
                                 ptr, size, _raw_stream(dev, stream)))


class TensorList:
    """Gradients that one norm is taken over: contiguous tensors of one type on
    one device, kept with their descriptors for repeated xpipe_grad_norm calls.
    A call looks at the tensors' addresses and sizes again: one whose storage was
    exchanged in between is read where it is now."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self._describe()

    def _describe(self):
        L = lib()
        if not self.tensors:
            raise ValueError("at least one tensor expected")
        first = self.tensors[0]
        self.dtype = _dtype_of(first)
        for t in self.tensors:
            if t.dtype is not first.dtype or t.get_device() != first.get_device() or not t.is_contiguous():
                raise ValueError("contiguous tensors of one type on one device expected")
        self.places = self._places()
        self.descs = (TensorDesc * len(self.tensors))(*self.places)
        need = _SZ()
        _check(L.xpipe_grad_norm_query(self.descs, len(self.tensors), ctypes.byref(need)))
        self.workspace_bytes = need.value

    def _places(self):
        return [(t.data_ptr(), t.numel()) for t in self.tensors]

    def refresh(self):
        if self._places() != self.places:
            self._describe()


def xpipe_grad_norm(tensors, max_norm: float, norm_coef=None, sumsq=None, workspace=None, stream=None):
    """Global L2 norm over `tensors` (a TensorList, or an iterable of tensors):
    norm_coef (float32, two elements) receives {norm, min(1, max_norm / (norm +
    1e-6))}, sumsq (float64, one element) the sum of squares; either may be None."""
    L = lib()
    if isinstance(tensors, TensorList):
        ts = tensors
        ts.refresh()
    else:
        ts = TensorList(tensors)
    t = ts.tensors[0]
    dev, here = _device_of(t)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_grad_norm(ts, max_norm, norm_coef, sumsq, workspace, stream)
    if norm_coef is not None:
        _check_norm_coef(norm_coef, dev)
    if sumsq is not None and (sumsq.dtype is not _torch.float64 or sumsq.numel() != 1 or sumsq.get_device() != dev):
        raise ValueError("sumsq: one float64 element on the gradients' device expected")
    ptr, size, keep = _workspace(ts.workspace_bytes, workspace, t, stream)
    _check(L.xpipe_grad_norm(ts.descs, len(ts.tensors), ts.dtype, max_norm, _ptr(sumsq), _ptr(norm_coef), ptr, size,
                             _raw_stream(dev, stream)))


def xpipe_clip_coef(sumsq, max_norm: float, norm_coef, stream=None):
    """{norm, coefficient} from float64 sums of squares (one per stage), added in an order that their number decides."""
    L = lib()
    dev, here = _device_of(sumsq)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_clip_coef(sumsq, max_norm, norm_coef, stream)
    if sumsq.dtype is not _torch.float64 or not sumsq.is_contiguous():
        raise ValueError("sumsq: contiguous float64 expected")
    _check_norm_coef(norm_coef, dev)
    _check(L.xpipe_clip_coef(sumsq.data_ptr(), sumsq.numel(), max_norm, norm_coef.data_ptr(), _raw_stream(dev, stream)))


_RMS_FWD_FORMAT, _RMS_BWD_FORMAT = struct.Struct("qiidPqPqPPqPq"), struct.Struct("qiidPqPqPPqPqP")
assert _RMS_FWD_FORMAT.size == ctypes.sizeof(RmsnormFwdArgs) and _RMS_BWD_FORMAT.size == ctypes.sizeof(RmsnormBwdArgs)


def xpipe_rmsnorm_fwd(x, weight, y, eps: float = 1e-6, residual=None, sum=None, stream=None):
    """h = x + residual; y = h / sqrt(mean(h^2) + eps) * weight; sum (optional)
    receives h.  Matrices [rows, dim] of one type, their rows contiguous; weight
    float32.  y and sum may each be x or residual itself."""
    L = lib()
    dev, here = _device_of(x)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_rmsnorm_fwd(x, weight, y, eps, residual, sum, stream)
    if x.dim() != 2:
        raise ValueError("x [rows, dim] expected")
    (rows, dim), dt = x.shape, x.dtype
    a = _RMS_FWD_FORMAT.pack(rows, dim, _dtype_of(x), eps, *_matrix("x", x, dt, dev, rows, dim),
                             *_matrix("residual", residual, dt, dev, rows, dim), _vector("weight", weight, dev, dim),
                             *_matrix("sum", sum, dt, dev, rows, dim), *_matrix("y", y, dt, dev, rows, dim))
    _check(L.xpipe_rmsnorm_fwd(a, _raw_stream(dev, stream)))


def xpipe_rmsnorm_bwd(dy, h, weight, dx=None, grad_weight=None, eps: float = 1e-6, residual=None, workspace=None, stream=None):
    """Gradients of the norm from dy and h (the forward's sum): dx, plus residual (a
    gradient that reaches h another way), and grad_weight (float32, added to), each
    optional.  dx may be dy, h or residual itself."""
    L = lib()
    dev, here = _device_of(dy)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_rmsnorm_bwd(dy, h, weight, dx, grad_weight, eps, residual, workspace, stream)
    if dy.dim() != 2:
        raise ValueError("dy [rows, dim] expected")
    (rows, dim), dt = dy.shape, dy.dtype
    a = _RMS_BWD_FORMAT.pack(rows, dim, _dtype_of(dy), eps, *_matrix("dy", dy, dt, dev, rows, dim), *_matrix("h", h, dt, dev, rows, dim),
                             _vector("weight", weight, dev, dim), *_matrix("residual", residual, dt, dev, rows, dim),
                             *_matrix("dx", dx, dt, dev, rows, dim), _vector("grad_weight", grad_weight, dev, dim))
    need = _SZ()
    _check(L.xpipe_rmsnorm_bwd_query(a, ctypes.byref(need)))
    ptr, size, keep = _workspace(need.value, workspace, dy, stream)
    _check(L.xpipe_rmsnorm_bwd(a, ptr, size, _raw_stream(dev, stream)))


def _relbias(table, name, values, dev):
    """(buckets, heads, max_distance) of a [buckets, heads] table and its [heads, 2 max_distance + 1] values."""
    for t in (table, values):
        if t.dtype is not _torch.float32 or t.dim() != 2 or not t.is_contiguous() or t.get_device() != dev:
            raise ValueError("contiguous float32 matrices on one device expected")
    (buckets, heads), (rows, width) = table.shape, values.shape
    if rows != heads or width % 2 != 1:
        raise ValueError(f"{name}: [heads, 2 max_distance + 1] expected")
    if max(buckets, heads, width) >= 1 << 31:  # (ctypes would cut them to 32 bits)
        raise ValueError("2^31 rows or columns or more")
    return buckets, heads, width // 2


def xpipe_relbias_fwd(table, bias, bidirectional: bool = True, stream=None):
    """bias[h, max_distance + d] = table[bucket(d), h] for the distances d (key position
    less query position) from -max_distance to max_distance, bias's width deciding
    max_distance.  table [buckets, heads] and bias float32."""
    L = lib()
    dev, here = _device_of(table)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_relbias_fwd(table, bias, bidirectional, stream)
    buckets, heads, far = _relbias(table, "bias", bias, dev)
    _check(L.xpipe_relbias_fwd(table.data_ptr(), buckets, heads, far, bool(bidirectional), bias.data_ptr(), _raw_stream(dev, stream)))


def xpipe_relbias_bwd(dbias, grad_table, bidirectional: bool = True, stream=None):
    """grad_table[b, h] += the sum of dbias[h] over the distances of bucket b."""
    L = lib()
    dev, here = _device_of(dbias)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_relbias_bwd(dbias, grad_table, bidirectional, stream)
    buckets, heads, far = _relbias(grad_table, "dbias", dbias, dev)
    _check(L.xpipe_relbias_bwd(dbias.data_ptr(), buckets, heads, far, bool(bidirectional), grad_table.data_ptr(), _raw_stream(dev, stream)))


_HEADS = "Pqqq"
_ATTN_IN = "9i4xdd" + 3 * _HEADS + "6P"
_ATTN_FWD_FORMAT = struct.Struct("@" + _ATTN_IN + _HEADS + "P")
_ATTN_BWD_FORMAT = struct.Struct("@" + _ATTN_IN + 2 * _HEADS + "P" + 3 * _HEADS + "P")
assert _ATTN_FWD_FORMAT.size == ctypes.sizeof(AttentionFwdArgs) and _ATTN_BWD_FORMAT.size == ctypes.sizeof(AttentionBwdArgs)


def _heads(name, t, dtype, dev, shape):
    """(pointer, strides of batch, token and head) of a [batch, tokens, heads, dim] tensor, dim contiguous."""
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name}: another type or device")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, {tuple(shape)} expected")
    b, n, h, d = t.stride()
    if d != 1 and shape[3] > 1:
        raise ValueError(f"{name}: contiguous in its last dimension expected")
    return t.data_ptr(), b, n, h


def _ints(name, t, dev, shape):
    if t is None:
        return 0
    if t.dtype is not _torch.int32 or t.get_device() != dev or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous int32 {tuple(shape)} on the same device expected")
    return t.data_ptr()


def _floats(name, t, dev, shape):
    if t is None:
        return 0
    if t.dtype is not _torch.float32 or t.get_device() != dev or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous float32 {tuple(shape)} on the same device expected")
    return t.data_ptr()


def _attention_inputs(q, k, v, dev, scale, causal, cap, bias, q_len, k_len, prefix, q_doc, k_doc):
    """xpipe_attention_inputs as _ATTN_IN's values."""
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q [batch, nq, heads, dim], k and v [batch, nk, kv_heads, dim] expected")
    (batch, nq, heads, dim), dt = q.shape, q.dtype
    nk, kv_heads = k.shape[1], k.shape[2]
    kv = (batch, nk, kv_heads, dim)
    reach = 0
    if bias is not None:
        if bias.dim() != 2 or bias.shape[1] % 2 != 1:
            raise ValueError("bias: [heads, 2 range + 1] expected")
        reach = bias.shape[1] // 2
    if max(batch, nq, nk, heads, kv_heads, dim, reach) >= 1 << 31:
        raise ValueError("a size of 2^31 or more")
    return (batch, nq, nk, heads, kv_heads, dim, _dtype_of(q), bool(causal), reach, dim ** -0.5 if scale is None and dim else scale or 0.0, cap,
            *_heads("q", q, dt, dev, q.shape), *_heads("k", k, dt, dev, kv), *_heads("v", v, dt, dev, kv),
            _ints("q_len", q_len, dev, (batch,)), _ints("k_len", k_len, dev, (batch,)), _ints("prefix", prefix, dev, (batch,)),
            _ints("q_doc", q_doc, dev, (batch, nq)), _ints("k_doc", k_doc, dev, (batch, nk)),
            0 if bias is None else _floats("bias", bias, dev, (heads, 2 * reach + 1)))


def xpipe_attention_fwd(q, k, v, o, scale: Optional[float] = None, causal: bool = False, cap: float = 0.0, bias=None, q_len=None,
                        k_len=None, prefix=None, q_doc=None, k_doc=None, stats=None, workspace=None, stream=None):
    """o = softmax(scores) v per head; scores = cap tanh(scale q.k / cap) + bias.
    q and o [batch, nq, heads, dim], k and v [batch, nk, kv_heads, dim] of one type, contiguous
    in dim; scale: dim^-0.5 unless given; cap 0: none; bias float32 [heads, 2 range + 1] by
    distance (key less query position; further ones as the furthest).  q_len, k_len,
    prefix: int32 [batch]; q_doc, k_doc: int32 documents of the tokens.  The queries are
    the last q_len of a sequence of k_len tokens.  stats (for the
    backward): float32 [batch, heads, nq, 2], the largest score times log2(e) and the
    sum of exp(score - largest)."""
    L = lib()
    dev, here = _device_of(q)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_attention_fwd(q, k, v, o, scale, causal, cap, bias, q_len, k_len, prefix, q_doc, k_doc, stats, workspace, stream)
    given = _attention_inputs(q, k, v, dev, scale, causal, cap, bias, q_len, k_len, prefix, q_doc, k_doc)
    batch, nq, heads, _ = q.shape
    a = _ATTN_FWD_FORMAT.pack(*given, *_heads("o", o, q.dtype, dev, q.shape),
                              _floats("stats", stats, dev, (batch, heads, nq, 2)))
    need = _SZ()
    _check(L.xpipe_attention_fwd_query(a, ctypes.byref(need)))
    ptr, size, keep = _workspace(need.value, workspace, q, stream)
    _check(L.xpipe_attention_fwd(a, ptr, size, _raw_stream(dev, stream)))


def xpipe_attention_bwd(dout, q, k, v, o, stats, dq, dk, dv, grad_bias=None, scale: Optional[float] = None, causal: bool = False,
                        cap: float = 0.0, bias=None, q_len=None, k_len=None, prefix=None, q_doc=None, k_doc=None, workspace=None,
                        stream=None):
    """Gradients of attention from dout: dq, dk, dv (written, types and shapes as q, k,
    v), and grad_bias (float32 like bias, added to).  The forward's other arguments
    as they were; o and stats are what it wrote."""
    L = lib()
    dev, here = _device_of(q)
    if not here:
        with _torch.cuda.device(dev):
            return xpipe_attention_bwd(dout, q, k, v, o, stats, dq, dk, dv, grad_bias, scale, causal, cap, bias, q_len, k_len, prefix, q_doc,
                                       k_doc, workspace, stream)
    given = _attention_inputs(q, k, v, dev, scale, causal, cap, bias, q_len, k_len, prefix, q_doc, k_doc)
    batch, nq, heads, _ = q.shape
    dt = q.dtype
    if stats is None:
        raise ValueError("stats: the forward's expected")
    if grad_bias is not None and bias is None:
        raise ValueError("grad_bias without bias")
    a = _ATTN_BWD_FORMAT.pack(*given, *_heads("dout", dout, dt, dev, q.shape), *_heads("o", o, dt, dev, q.shape),
                              _floats("stats", stats, dev, (batch, heads, nq, 2)), *_heads("dq", dq, dt, dev, q.shape),
                              *_heads("dk", dk, dt, dev, k.shape), *_heads("dv", dv, dt, dev, k.shape),
                              0 if grad_bias is None else _floats("grad_bias", grad_bias, dev, bias.shape))
    need = _SZ()
    _check(L.xpipe_attention_bwd_query(a, ctypes.byref(need)))
    ptr, size, keep = _workspace(need.value, workspace, q, stream)
    _check(L.xpipe_attention_bwd(a, ptr, size, _raw_stream(dev, stream)))
