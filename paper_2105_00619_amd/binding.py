"""ctypes binding of liboptorch_seq.so -- argument marshalling only.

Every step of the path runs inside the library's HIP kernels; torch is used here
to allocate the two device arenas and to supply the HIP stream.  There is no CPU
fallback: if the shared library is missing the import of the library fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liboptorch_seq.so")

OK, E_INVALID, E_BUDGET, E_HIP, E_ORDER = 0, -1, -2, -3, -4

SYMBOLS = (
    "optorch_seq_create", "optorch_seq_query", "optorch_seq_bind", "optorch_seq_set_params", "optorch_seq_update_params",
    "optorch_seq_get_params", "optorch_seq_step", "optorch_seq_schedule_info", "optorch_seq_last_error",
    "optorch_seq_destroy", "optorch_seq_predict", "optorch_seq_running_stats", "optorch_seq_profile_enable", "optorch_seq_profile_select", "optorch_seq_profile_read", "optorch_seq_profile_read_entries",
    "optorch_seq_step_encoded", "optorch_seq_predict_encoded", "optorch_seq_plan_info", "optorch_seq_step_static", "optorch_seq_debug_unit_output",
    "optorch_encoded_words", "optorch_encode", "optorch_decode", "optorch_decode_normalized", "optorch_encode_lossless",
    "optorch_decode_lossless", "optorch_dataflow_last_error",
    "optorch_linear_workspace", "optorch_linear_forward", "optorch_linear_backward",
    "optorch_layer_norm_workspace", "optorch_layer_norm_forward", "optorch_layer_norm_backward",
    "optorch_softmax_loss_workspace", "optorch_softmax_loss_forward", "optorch_softmax_loss_backward", "optorch_ortho_create", "optorch_ortho_query",
    "optorch_ortho_bind", "optorch_orthogonalize", "optorch_muon_update", "optorch_ortho_destroy", "optorch_matrix_last_error",
)

KERNEL_CLASSES = ("cast_in", "conv_fwd", "conv_dgrad", "conv_wgrad", "bn_stats", "bn_apply", "bn_bwd", "pool", "head",
                  "relu_bias_bwd", "optimizer", "conv1x1_fwd", "conv1x1_dgrad", "conv1x1_wgrad")


class optorch_unit_t(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("kind", "cin", "cout", "ksize", "stride", "pad", "has_bn", "has_relu", "has_bias", "reserved")]


class optorch_seq_config_t(C.Structure):
    _fields_ = [
        ("k_segments", C.c_int32), ("boundaries", C.POINTER(C.c_int32)), ("plan_mode", C.c_int32),
        ("precision", C.c_int32), ("batch", C.c_int32), ("height", C.c_int32), ("width", C.c_int32),
        ("channels", C.c_int32), ("num_classes", C.c_int32), ("activation_budget_bytes", C.c_uint64),
        ("momentum", C.c_float), ("bn_eps", C.c_float), ("bn_momentum", C.c_float),
        ("loss_scale_init", C.c_float), ("scale_growth", C.c_float), ("scale_backoff", C.c_float),
        ("growth_interval", C.c_int32), ("storage_mode", C.c_int32),
    ]


class optorch_linear_t(C.Structure):
    _fields_ = [
        ("precision", C.c_int32), ("activation", C.c_int32), ("rows", C.c_int64), ("in_features", C.c_int32),
        ("out_features", C.c_int32), ("x", C.c_void_p), ("ldx", C.c_int64), ("w", C.c_void_p), ("ldw", C.c_int64),
        ("bias", C.c_void_p), ("residual", C.c_void_p), ("ldr", C.c_int64), ("y", C.c_void_p), ("ldy", C.c_int64),
        ("z", C.c_void_p), ("ldz", C.c_int64), ("dy", C.c_void_p), ("lddy", C.c_int64), ("dx", C.c_void_p),
        ("lddx", C.c_int64), ("dw", C.c_void_p), ("lddw", C.c_int64), ("dbias", C.c_void_p), ("workspace", C.c_void_p),
        ("workspace_bytes", C.c_uint64), ("hip_stream", C.c_void_p),
    ]


class optorch_layer_norm_t(C.Structure):
    _fields_ = [
        ("precision", C.c_int32), ("cols", C.c_int32), ("rows", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64),
        ("weight", C.c_void_p), ("bias", C.c_void_p), ("eps", C.c_float), ("reserved", C.c_int32), ("y", C.c_void_p),
        ("ldy", C.c_int64), ("mean", C.c_void_p), ("rstd", C.c_void_p), ("dy", C.c_void_p), ("lddy", C.c_int64),
        ("residual", C.c_void_p), ("ldr", C.c_int64), ("dx", C.c_void_p), ("lddx", C.c_int64), ("dweight", C.c_void_p),
        ("dbias", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("hip_stream", C.c_void_p),
    ]


class optorch_softmax_loss_t(C.Structure):
    _fields_ = [
        ("precision", C.c_int32), ("teacher_precision", C.c_int32), ("rows", C.c_int64), ("in_features", C.c_int32),
        ("classes", C.c_int32), ("x", C.c_void_p), ("ldx", C.c_int64), ("w", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p),
        ("labels", C.c_void_p), ("indices", C.c_void_p), ("ldi", C.c_int64), ("teacher", C.c_void_p), ("ldt", C.c_int64),
        ("top", C.c_int32), ("temperature", C.c_float), ("label_smoothing", C.c_float), ("z_loss", C.c_float), ("loss", C.c_void_p),
        ("lse", C.c_void_p), ("dloss", C.c_void_p), ("dx", C.c_void_p), ("lddx", C.c_int64), ("dw", C.c_void_p), ("lddw", C.c_int64),
        ("dbias", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("hip_stream", C.c_void_p),
    ]


class optorch_matrix_t(C.Structure):
    _fields_ = [("offset", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32), ("ld", C.c_int64)]


class optorch_ortho_config_t(C.Structure):
    _fields_ = [("steps", C.c_int32), ("coefficients", C.POINTER(C.c_float)), ("eps", C.c_float), ("reserved", C.c_int32)]


class optorch_muon_t(C.Structure):
    _fields_ = [("g_precision", C.c_int32), ("g", C.c_void_p), ("w", C.c_void_p), ("v", C.c_void_p),
                ("w16_precision", C.c_int32), ("w16", C.c_void_p), ("lr", C.c_float), ("momentum", C.c_float),
                ("weight_decay", C.c_float), ("grad_scale", C.c_float), ("nesterov", C.c_int32), ("scale_mode", C.c_int32),
                ("skipped", C.c_void_p)]


_lib = None


def load_library() -> C.CDLL:
    """Loads the HIP library built in-tree; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("%s not found: build it with `python -m paper_2105_00619_amd.build` "
                          "(there is no CPU fallback)" % LIB_PATH)
    lib = C.CDLL(LIB_PATH)
    H = C.c_void_p
    lib.optorch_seq_create.argtypes = [C.POINTER(optorch_unit_t), C.c_int32, C.POINTER(optorch_seq_config_t), C.POINTER(H)]
    lib.optorch_seq_create.restype = C.c_int
    lib.optorch_seq_query.argtypes = [H, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64), C.POINTER(C.c_uint64),
                                      C.POINTER(C.c_uint64), C.POINTER(C.c_int32)]
    lib.optorch_seq_query.restype = C.c_int
    lib.optorch_seq_bind.argtypes = [H, C.c_void_p, C.c_uint64, C.c_void_p, C.c_uint64, C.c_void_p]
    lib.optorch_seq_bind.restype = C.c_int
    lib.optorch_seq_set_params.argtypes = [H, C.c_void_p, C.c_uint64, C.c_int32]
    lib.optorch_seq_set_params.restype = C.c_int
    lib.optorch_seq_update_params.argtypes = [H, C.c_void_p, C.c_uint64, C.c_int32]
    lib.optorch_seq_update_params.restype = C.c_int
    lib.optorch_seq_get_params.argtypes = [H, C.c_void_p, C.c_uint64, C.c_int32]
    lib.optorch_seq_get_params.restype = C.c_int
    lib.optorch_seq_step.argtypes = [H, C.c_void_p, C.c_void_p, C.c_float, C.POINTER(C.c_float), C.c_void_p,
                                     C.POINTER(C.c_uint64), C.POINTER(C.c_uint64), C.POINTER(C.c_float),
                                     C.POINTER(C.c_int32)]
    lib.optorch_seq_step.restype = C.c_int
    lib.optorch_seq_step_static.argtypes = lib.optorch_seq_step.argtypes
    lib.optorch_seq_step_static.restype = C.c_int
    lib.optorch_seq_debug_unit_output.argtypes = [H, C.c_void_p, C.c_int32, C.c_void_p, C.c_uint64, C.POINTER(C.c_uint64),
                                                  C.POINTER(C.c_int32)]
    lib.optorch_seq_debug_unit_output.restype = C.c_int
    lib.optorch_seq_step_encoded.argtypes = [H, C.c_void_p, C.c_int32, C.POINTER(C.c_float), C.POINTER(C.c_float), C.c_void_p,
                                             C.c_float, C.POINTER(C.c_float), C.c_void_p, C.POINTER(C.c_uint64),
                                             C.POINTER(C.c_uint64), C.POINTER(C.c_float), C.POINTER(C.c_int32)]
    lib.optorch_seq_step_encoded.restype = C.c_int
    lib.optorch_seq_predict_encoded.argtypes = [H, C.c_void_p, C.c_int32, C.POINTER(C.c_float), C.POINTER(C.c_float), C.c_void_p]
    lib.optorch_seq_predict_encoded.restype = C.c_int
    lib.optorch_encoded_words.argtypes = [C.c_int32, C.c_int32]
    lib.optorch_encoded_words.restype = C.c_int32
    lib.optorch_encode.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p]
    lib.optorch_encode.restype = C.c_int
    lib.optorch_decode.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p]
    lib.optorch_decode.restype = C.c_int
    lib.optorch_decode_normalized.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_int32, C.POINTER(C.c_float),
                                              C.POINTER(C.c_float), C.c_int32, C.c_void_p, C.c_void_p]
    lib.optorch_decode_normalized.restype = C.c_int
    lib.optorch_encode_lossless.argtypes = [C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.optorch_encode_lossless.restype = C.c_int
    lib.optorch_decode_lossless.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p]
    lib.optorch_decode_lossless.restype = C.c_int
    lib.optorch_dataflow_last_error.argtypes = []
    lib.optorch_dataflow_last_error.restype = C.c_char_p
    L = C.POINTER(optorch_linear_t)
    lib.optorch_linear_workspace.argtypes = [L, C.c_int32]
    lib.optorch_linear_workspace.restype = C.c_int64
    lib.optorch_linear_forward.argtypes = [L]
    lib.optorch_linear_forward.restype = C.c_int
    lib.optorch_linear_backward.argtypes = [L]
    lib.optorch_linear_backward.restype = C.c_int
    N = C.POINTER(optorch_layer_norm_t)
    lib.optorch_layer_norm_workspace.argtypes = [N]
    lib.optorch_layer_norm_workspace.restype = C.c_int64
    lib.optorch_layer_norm_forward.argtypes = [N]
    lib.optorch_layer_norm_forward.restype = C.c_int
    lib.optorch_layer_norm_backward.argtypes = [N]
    lib.optorch_layer_norm_backward.restype = C.c_int
    X = C.POINTER(optorch_softmax_loss_t)
    lib.optorch_softmax_loss_workspace.argtypes = [X, C.c_int32]
    lib.optorch_softmax_loss_workspace.restype = C.c_int64
    lib.optorch_softmax_loss_forward.argtypes = [X]
    lib.optorch_softmax_loss_forward.restype = C.c_int
    lib.optorch_softmax_loss_backward.argtypes = [X]
    lib.optorch_softmax_loss_backward.restype = C.c_int
    lib.optorch_ortho_create.argtypes = [C.POINTER(optorch_matrix_t), C.c_int32, C.POINTER(optorch_ortho_config_t), C.POINTER(H)]
    lib.optorch_ortho_create.restype = C.c_int
    lib.optorch_ortho_query.argtypes = [H, C.POINTER(C.c_uint64), C.POINTER(C.c_int64)]
    lib.optorch_ortho_query.restype = C.c_int
    lib.optorch_ortho_bind.argtypes = [H, C.c_void_p, C.c_uint64]
    lib.optorch_ortho_bind.restype = C.c_int
    lib.optorch_orthogonalize.argtypes = [H, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
    lib.optorch_orthogonalize.restype = C.c_int
    lib.optorch_muon_update.argtypes = [H, C.POINTER(optorch_muon_t), C.c_void_p]
    lib.optorch_muon_update.restype = C.c_int
    lib.optorch_ortho_destroy.argtypes = [H]
    lib.optorch_ortho_destroy.restype = None
    lib.optorch_matrix_last_error.argtypes = []
    lib.optorch_matrix_last_error.restype = C.c_char_p
    lib.optorch_seq_predict.argtypes = [H, C.c_void_p, C.c_void_p]
    lib.optorch_seq_predict.restype = C.c_int
    lib.optorch_seq_running_stats.argtypes = [H, C.c_void_p, C.c_uint64, C.POINTER(C.c_uint64), C.c_int32]
    lib.optorch_seq_running_stats.restype = C.c_int
    lib.optorch_seq_plan_info.argtypes = [H, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.optorch_seq_plan_info.restype = C.c_int
    lib.optorch_seq_schedule_info.argtypes = [H, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.optorch_seq_schedule_info.restype = C.c_int
    lib.optorch_seq_profile_enable.argtypes = [H, C.c_int32]
    lib.optorch_seq_profile_enable.restype = C.c_int
    lib.optorch_seq_profile_select.argtypes = [H, C.c_uint32]
    lib.optorch_seq_profile_select.restype = C.c_int
    lib.optorch_seq_profile_read.argtypes = [H, C.POINTER(C.c_int32), C.POINTER(C.c_uint64), C.POINTER(C.c_uint64),
                                             C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.optorch_seq_profile_read.restype = C.c_int
    lib.optorch_seq_profile_read_entries.argtypes = [H, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                                     C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_double),
                                                     C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.optorch_seq_profile_read_entries.restype = C.c_int
    lib.optorch_seq_last_error.argtypes = [H]
    lib.optorch_seq_last_error.restype = C.c_char_p
    lib.optorch_seq_destroy.argtypes = [H]
    lib.optorch_seq_destroy.restype = None
    _lib = lib
    return lib


class OptorchError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__("optorch_seq error %d: %s" % (code, message))
        self.code = code


class SeqPlan:
    """optorch_seq_create + optorch_seq_query: host-side plan, no device needed."""

    def __init__(self, units: Sequence, *, k_segments: int, precision: int, batch: int, height: int, width: int,
                 channels: int, num_classes: int, boundaries: Optional[Sequence[int]] = None, plan_mode: int = 0,
                 activation_budget_bytes: int = 0, momentum: float = 0.0, bn_eps: float = 0.0, bn_momentum: float = 0.0,
                 loss_scale_init: float = 0.0, scale_growth: float = 0.0, scale_backoff: float = 0.0,
                 growth_interval: int = 0, storage_mode: int = 0):
        self.lib = load_library()
        self.handle = C.c_void_p()
        arr = (optorch_unit_t * len(units))()
        for i, u in enumerate(units):
            arr[i] = optorch_unit_t(u.kind, u.cin, u.cout, u.ksize, u.stride, u.pad, u.has_bn, u.has_relu, u.has_bias, 0)
        cfg = optorch_seq_config_t()
        cfg.k_segments = k_segments
        barr = None
        if boundaries is not None:
            barr = (C.c_int32 * max(1, len(boundaries)))(*boundaries)
            cfg.boundaries = C.cast(barr, C.POINTER(C.c_int32))
        cfg.plan_mode, cfg.precision = plan_mode, precision
        cfg.batch, cfg.height, cfg.width, cfg.channels, cfg.num_classes = batch, height, width, channels, num_classes
        cfg.activation_budget_bytes = activation_budget_bytes
        cfg.momentum, cfg.bn_eps, cfg.bn_momentum = momentum, bn_eps, bn_momentum
        cfg.loss_scale_init, cfg.scale_growth, cfg.scale_backoff = loss_scale_init, scale_growth, scale_backoff
        cfg.growth_interval = growth_interval
        cfg.storage_mode = storage_mode
        rc = self.lib.optorch_seq_create(arr, len(units), C.byref(cfg), C.byref(self.handle))
        if rc != OK:
            msg = self.lib.optorch_seq_last_error(None).decode()
            self.handle = C.c_void_p()
            raise OptorchError(rc, msg)
        kk, sm = C.c_int32(), C.c_int32()
        self._check(self.lib.optorch_seq_plan_info(self.handle, C.byref(kk), C.byref(sm)))
        k_segments = kk.value  # the plan's choice when 0 was asked for
        self.k_segments, self.storage_mode = k_segments, sm.value
        self.batch, self.height, self.width, self.channels = batch, height, width, channels
        self.num_classes = num_classes
        pc, pb, ab, ps = C.c_uint64(), C.c_uint64(), C.c_uint64(), C.c_uint64()
        bo = (C.c_int32 * max(1, k_segments - 1))()
        self._check(self.lib.optorch_seq_query(self.handle, C.byref(pc), C.byref(pb), C.byref(ab), C.byref(ps), bo))
        self.param_count, self.param_arena_bytes = pc.value, pb.value
        self.act_arena_bytes, self.planned_peak_saved_bytes = ab.value, ps.value
        self.boundaries = [bo[i] for i in range(k_segments - 1)]
        nl, nr = C.c_int32(), C.c_int32()
        self._check(self.lib.optorch_seq_schedule_info(self.handle, C.byref(nl), C.byref(nr)))
        self.n_launches, self.n_replay_launches = nl.value, nr.value

    @classmethod
    def from_workload(cls, w, **override):
        kw = dict(k_segments=w.k_segments, precision=w.precision, batch=w.batch, height=w.height, width=w.width,
                  channels=w.channels, num_classes=w.classes, plan_mode=w.plan_mode,
                  activation_budget_bytes=w.budget_bytes, momentum=w.momentum, loss_scale_init=w.loss_scale_init)
        kw.update(override)
        return cls(w.units, **kw)

    def _check(self, rc: int):
        if rc != OK:
            raise OptorchError(rc, self.lib.optorch_seq_last_error(self.handle).decode())

    def close(self):
        if getattr(self, "handle", None) and self.handle.value:
            self.lib.optorch_seq_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class SeqTrainer(SeqPlan):
    """A bound plan: device arenas allocated through torch, steps run on torch's current stream."""

    GUARD_BYTE = 0xA5

    def __init__(self, units, *, device="cuda:0", guard_bytes: int = 0, **kw):
        """guard_bytes > 0: each arena is allocated with that many bytes of a fixed pattern in front of and behind the
        bytes lent to the library, and `guards_intact()` checks that no kernel wrote outside them."""
        import torch
        super().__init__(units, **kw)
        self.torch = torch
        self.device = torch.device(device)
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the training step only runs on the HIP path")
        self.guard_bytes = g = (int(guard_bytes) + 255) // 256 * 256
        self._arenas = []
        ptrs = []
        for nbytes in (self.param_arena_bytes, self.act_arena_bytes):
            buf = torch.empty(nbytes + 2 * g + 256, dtype=torch.uint8, device=self.device)
            start = (buf.data_ptr() + 255) // 256 * 256 - buf.data_ptr() + g  # offset of the lent bytes inside buf
            if g:
                buf[:start].fill_(self.GUARD_BYTE)
                buf[start + nbytes:].fill_(self.GUARD_BYTE)
            self._arenas.append((buf, start, nbytes))
            ptrs.append(buf.data_ptr() + start)
        self.param_arena, self.act_arena = self._arenas[0][0], self._arenas[1][0]
        self.stream = torch.cuda.current_stream(self.device)
        self._check(self.lib.optorch_seq_bind(self.handle, ptrs[0], self.param_arena_bytes, ptrs[1], self.act_arena_bytes,
                                              self.stream.cuda_stream))

    def guards_intact(self) -> bool:
        """True if every guard byte around both arenas still holds the pattern (needs guard_bytes > 0)."""
        assert self.guard_bytes > 0, "the trainer was created without guard bands"
        self.torch.cuda.synchronize(self.device)
        for buf, start, nbytes in self._arenas:
            if not bool((buf[:start] == self.GUARD_BYTE).all()) or not bool((buf[start + nbytes:] == self.GUARD_BYTE).all()):
                return False
        return True

    @classmethod
    def from_workload(cls, w, device="cuda:0", **override):
        kw = dict(k_segments=w.k_segments, precision=w.precision, batch=w.batch, height=w.height, width=w.width,
                  channels=w.channels, num_classes=w.classes, plan_mode=w.plan_mode,
                  activation_budget_bytes=w.budget_bytes, momentum=w.momentum, loss_scale_init=w.loss_scale_init)
        kw.update(override)
        return cls(w.units, device=device, **kw)

    def set_params(self, params):
        self._put_params(self.lib.optorch_seq_set_params, params)

    def update_params(self, params):
        """Weights that an update outside of `step` has made: momentum, running statistics and loss scale go on."""
        self._put_params(self.lib.optorch_seq_update_params, params)

    def _put_params(self, call, params):
        torch = self.torch
        if isinstance(params, np.ndarray):
            p = np.ascontiguousarray(params, dtype=np.float32)
            self._check(call(self.handle, p.ctypes.data, p.size, 0))
        else:
            p = params.to(device=self.device, dtype=torch.float32).contiguous()
            self._check(call(self.handle, p.data_ptr(), p.numel(), 1))

    def get_params(self) -> np.ndarray:
        out = np.empty(self.param_count, dtype=np.float32)
        self._check(self.lib.optorch_seq_get_params(self.handle, out.ctypes.data, out.size, 0))
        return out

    def step(self, x, y, lr: float, grads=None, static_arena: bool = False) -> dict:
        """x: cuda float32 NHWC tensor, y: cuda int32 tensor, grads: optional cuda float32 tensor (param_count).
        static_arena: run optorch_seq_step_static (the library's static activation arena; allocates nothing)."""
        torch = self.torch
        assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()
        assert tuple(x.shape) == (self.batch, self.height, self.width, self.channels)
        assert y.is_cuda and y.dtype == torch.int32 and y.numel() == self.batch
        if grads is not None:
            assert grads.is_cuda and grads.dtype == torch.float32 and grads.numel() == self.param_count
        loss, scale, skipped = C.c_float(), C.c_float(), C.c_int32()
        ps, pa = C.c_uint64(), C.c_uint64()
        fn = self.lib.optorch_seq_step_static if static_arena else self.lib.optorch_seq_step
        self._check(fn(self.handle, x.data_ptr(), y.data_ptr(), lr, C.byref(loss),
                                              grads.data_ptr() if grads is not None else None, C.byref(ps), C.byref(pa),
                                              C.byref(scale), C.byref(skipped)))
        return {"loss": loss.value, "peak_saved_bytes": ps.value, "peak_arena_bytes": pa.value,
                "loss_scale": scale.value, "skipped": bool(skipped.value)}

    def step_encoded(self, a, z: int, scale, shift, y, lr: float, grads=None) -> dict:
        """`step` on a batch in encoded form: a = `encode(pixels, z)` of the batch's 8-bit pixels; the decode layer maps
        every pixel to pixel * scale[c] + shift[c] (`channels` floats each)."""
        torch = self.torch
        words = encoded_words(z)
        groups = -(-self.batch // z)
        assert a.is_cuda and a.dtype == torch.int64 and a.is_contiguous()
        assert a.numel() == groups * self.height * self.width * self.channels * words
        assert y.is_cuda and y.dtype == torch.int32 and y.numel() == self.batch
        if grads is not None:
            assert grads.is_cuda and grads.dtype == torch.float32 and grads.numel() == self.param_count
        sc, sh = _float_array(scale, self.channels), _float_array(shift, self.channels)
        loss, lscale, skipped = C.c_float(), C.c_float(), C.c_int32()
        ps, pa = C.c_uint64(), C.c_uint64()
        self._check(self.lib.optorch_seq_step_encoded(self.handle, a.data_ptr(), z, sc, sh, y.data_ptr(), lr, C.byref(loss),
                                                      grads.data_ptr() if grads is not None else None, C.byref(ps),
                                                      C.byref(pa), C.byref(lscale), C.byref(skipped)))
        return {"loss": loss.value, "peak_saved_bytes": ps.value, "peak_arena_bytes": pa.value,
                "loss_scale": lscale.value, "skipped": bool(skipped.value)}

    def predict(self, x):
        """Inference-mode logits (running BatchNorm statistics): cuda float32 tensor batch x num_classes."""
        torch = self.torch
        assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()
        assert tuple(x.shape) == (self.batch, self.height, self.width, self.channels)
        out = torch.empty((self.batch, self.num_classes), dtype=torch.float32, device=self.device)
        self._check(self.lib.optorch_seq_predict(self.handle, x.data_ptr(), out.data_ptr()))
        return out

    def predict_encoded(self, a, z: int, scale, shift):
        """`predict` on a batch in encoded form (see `step_encoded`)."""
        torch = self.torch
        groups = -(-self.batch // z)
        assert a.is_cuda and a.dtype == torch.int64 and a.is_contiguous()
        assert a.numel() == groups * self.height * self.width * self.channels * encoded_words(z)
        out = torch.empty((self.batch, self.num_classes), dtype=torch.float32, device=self.device)
        self._check(self.lib.optorch_seq_predict_encoded(self.handle, a.data_ptr(), z, _float_array(scale, self.channels),
                                                         _float_array(shift, self.channels), out.data_ptr()))
        return out

    def unit_output(self, x, unit: int):
        """The output activation of body unit `unit` in a training-mode forward pass on x: cuda float32 NHWC tensor
        (optorch_seq_debug_unit_output)."""
        torch = self.torch
        assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()
        n, shape = C.c_uint64(), (C.c_int32 * 4)()
        self._check(self.lib.optorch_seq_debug_unit_output(self.handle, None, unit, None, 0, C.byref(n), shape))
        out = torch.empty(tuple(shape), dtype=torch.float32, device=self.device)
        self._check(self.lib.optorch_seq_debug_unit_output(self.handle, x.data_ptr(), unit, out.data_ptr(), n.value,
                                                           C.byref(n), shape))
        return out

    def running_stats(self) -> np.ndarray:
        """Per BatchNorm in parameter order: C running means, then C running variances."""
        n = C.c_uint64()
        self._check(self.lib.optorch_seq_running_stats(self.handle, None, 0, C.byref(n), 0))
        out = np.empty(n.value, dtype=np.float32)
        if n.value:
            self._check(self.lib.optorch_seq_running_stats(self.handle, out.ctypes.data, out.size, C.byref(n), 0))
        return out

    def profile_enable(self, enable: bool = True):
        self._check(self.lib.optorch_seq_profile_enable(self.handle, 1 if enable else 0))

    def profile_select(self, classes=None):
        """Restrict event timing to the named kernel classes (None: all)."""
        mask = 0xFFFFFFFF if classes is None else sum(1 << KERNEL_CLASSES.index(c) for c in classes)
        self._check(self.lib.optorch_seq_profile_select(self.handle, mask))

    def profile_read(self) -> dict:
        """Per kernel class: launches, schedule entries, GPU ms, algorithmic FLOPs and bytes, summed over the
        profiled steps; plus "steps"."""
        n = len(KERNEL_CLASSES)
        steps = C.c_int32()
        la, en = (C.c_uint64 * n)(), (C.c_uint64 * n)()
        ms, fl, by = (C.c_double * n)(), (C.c_double * n)(), (C.c_double * n)()
        self._check(self.lib.optorch_seq_profile_read(self.handle, C.byref(steps), la, en, ms, fl, by))
        out = {"steps": steps.value, "classes": {}}
        for i, name in enumerate(KERNEL_CLASSES):
            out["classes"][name] = {"launches": la[i], "entries": en[i], "gpu_ms": ms[i], "flops": fl[i], "bytes": by[i]}
        return out

    def profile_read_entries(self) -> list:
        """Per schedule entry, in launch order: kernel class, unit, phase, GPU ms, algorithmic FLOPs and bytes."""
        cap = 8192
        n = C.c_int32()
        kind, unit, phase = (C.c_int32 * cap)(), (C.c_int32 * cap)(), (C.c_int32 * cap)()
        ms, fl, by = (C.c_double * cap)(), (C.c_double * cap)(), (C.c_double * cap)()
        self._check(self.lib.optorch_seq_profile_read_entries(self.handle, cap, C.byref(n), kind, unit, phase, ms, fl, by))
        return [{"kind": KERNEL_CLASSES[kind[i]], "unit": unit[i], "phase": phase[i], "gpu_ms": ms[i], "flops": fl[i],
                 "bytes": by[i]} for i in range(min(n.value, cap))]


# ---- image data-flow (optorch_dataflow.h): tensors allocated through torch, kernels on torch's current stream ----------
# Encoded words are unsigned 64-bit; torch carries them as int64 tensors of the same bits.

def _float_array(values, n: int):
    v = [float(t) for t in values]
    if len(v) != n:
        raise ValueError("expected %d values, got %d" % (n, len(v)))
    return (C.c_float * n)(*v)


def _df_check(rc: int):
    if rc != OK:
        raise OptorchError(rc, (load_library().optorch_dataflow_last_error() or b"").decode())


def _stream(torch):
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def encoded_words(z: int, lossless: bool = False) -> int:
    """64-bit words per position for groups of z images; raises for z outside the form's range."""
    n = load_library().optorch_encoded_words(z, 1 if lossless else 0)
    if n == 0:
        raise OptorchError(E_INVALID, "images per group must be 1..%d, got %d" % (32 if lossless else 16, z))
    return n


def _batch_shape(x):
    batch = x.shape[0]
    n_pos = 1
    for d in x.shape[1:]:
        n_pos *= d
    return batch, n_pos


def encode(x, z: int, out=None):
    """Algorithm "Encode": x cuda uint8 [batch, ...] -> cuda int64 [ceil(batch / z), n_pos, words]."""
    import torch
    assert x.is_cuda and x.dtype == torch.uint8 and x.is_contiguous()
    batch, n_pos = _batch_shape(x)
    words = encoded_words(z)
    if out is None:
        out = torch.empty((-(-batch // z), n_pos, words), dtype=torch.int64, device=x.device)
    assert out.is_cuda and out.dtype == torch.int64 and out.is_contiguous() and out.numel() == -(-batch // z) * n_pos * words
    _df_check(load_library().optorch_encode(x.data_ptr(), batch, n_pos, z, out.data_ptr(), _stream(torch)))
    return out


def decode(a, batch: int, n_pos: int, z: int, out=None):
    """Algorithm "Decode": the inverse of `encode`; returns cuda uint8 [batch, n_pos]."""
    import torch
    words = encoded_words(z)
    assert a.is_cuda and a.dtype == torch.int64 and a.is_contiguous() and a.numel() == -(-batch // z) * n_pos * words
    if out is None:
        out = torch.empty((batch, n_pos), dtype=torch.uint8, device=a.device)
    assert out.is_cuda and out.dtype == torch.uint8 and out.is_contiguous() and out.numel() == batch * n_pos
    _df_check(load_library().optorch_decode(a.data_ptr(), batch, n_pos, z, out.data_ptr(), _stream(torch)))
    return out


def decode_normalized(a, batch: int, n_pos: int, z: int, channels: int, scale, shift, precision: int, out=None):
    """Decode fused with pixel * scale[c] + shift[c] and the cast: cuda [batch, n_pos] in fp32 / bf16 / fp16."""
    import torch
    words = encoded_words(z)
    assert a.is_cuda and a.dtype == torch.int64 and a.is_contiguous() and a.numel() == -(-batch // z) * n_pos * words
    dtype = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}[precision]
    if out is None:
        out = torch.empty((batch, n_pos), dtype=dtype, device=a.device)
    assert out.is_cuda and out.dtype == dtype and out.is_contiguous() and out.numel() == batch * n_pos
    _df_check(load_library().optorch_decode_normalized(a.data_ptr(), batch, n_pos, z, channels, _float_array(scale, channels),
                                                       _float_array(shift, channels), precision, out.data_ptr(),
                                                       _stream(torch)))
    return out


def encode_lossless(x, z: int):
    """Algorithm "Loss-less Forced Encoding": x cuda uint8 [batch, ...] -> (cuda int64 [G, n_pos, words], cuda int32 [G, n_pos])."""
    import torch
    assert x.is_cuda and x.dtype == torch.uint8 and x.is_contiguous()
    batch, n_pos = _batch_shape(x)
    words = encoded_words(z, True)
    groups = -(-batch // z)
    a = torch.empty((groups, n_pos, words), dtype=torch.int64, device=x.device)
    o = torch.empty((groups, n_pos), dtype=torch.int32, device=x.device)
    _df_check(load_library().optorch_encode_lossless(x.data_ptr(), batch, n_pos, z, a.data_ptr(), o.data_ptr(), _stream(torch)))
    return a, o


def decode_lossless(a, o, batch: int, n_pos: int, z: int):
    """The inverse of `encode_lossless`; returns cuda uint8 [batch, n_pos]."""
    import torch
    words = encoded_words(z, True)
    groups = -(-batch // z)
    assert a.is_cuda and a.dtype == torch.int64 and a.is_contiguous() and a.numel() == groups * n_pos * words
    assert o.is_cuda and o.dtype == torch.int32 and o.is_contiguous() and o.numel() == groups * n_pos
    out = torch.empty((batch, n_pos), dtype=torch.uint8, device=a.device)
    _df_check(load_library().optorch_decode_lossless(a.data_ptr(), o.data_ptr(), batch, n_pos, z, out.data_ptr(), _stream(torch)))
    return out


# ---- matrix operators (optorch_matrix.h): tensors and workspaces allocated through torch, kernels on torch's current stream ----

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
SCALE_MODES = {"none": 0, "aspect": 1, "rms": 2}
_PRECISION = {}  # torch dtype -> optorch_precision_t, filled on first use (torch is imported lazily)


def _precision(dtype) -> int:
    if not _PRECISION:
        import torch
        _PRECISION.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    try:
        return _PRECISION[dtype]
    except KeyError:
        raise TypeError("expected a float32, bfloat16 or float16 tensor, got %s" % dtype) from None


def _mat_fail(rc: int):
    raise OptorchError(rc, (load_library().optorch_matrix_last_error() or b"").decode())


def _int32(name, v):
    """v as an int that its C field holds (ctypes cuts off what does not fit)."""
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError("%s: %d is too large" % (name, v))
    return v


def _check_matrix(name, t, rows, cols, like):
    """A rows x cols matrix of like's type and device whose rows lie one behind the other (any distance)."""
    if t.shape != (rows, cols):
        raise ValueError("%s: expected a %d x %d matrix, got %s" % (name, rows, cols, tuple(t.shape)))
    if t is not like and (t.dtype != like.dtype or t.device != like.device):
        raise TypeError("%s: expected %s on %s, got %s on %s" % (name, like.dtype, like.device, t.dtype, t.device))
    if cols > 1 and t.stride(1) != 1:
        raise ValueError("%s: the elements of a row must lie next to each other" % name)


def _ld(t):
    """Distance of a matrix' rows.  (One row or none: torch's stride says nothing.)"""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _check_vector(name, t, n, like):
    import torch
    if t.dtype != torch.float32 or t.device != like.device:
        raise TypeError("%s: expected float32 on %s, got %s on %s" % (name, like.device, t.dtype, t.device))
    if t.numel() != n or not t.is_contiguous():
        raise ValueError("%s: expected %d contiguous values" % (name, n))


def _linear_args(x, activation, rows, cin, cout):
    if activation not in ACTIVATIONS:
        raise ValueError("activation must be one of %s" % ", ".join(sorted(ACTIVATIONS)))
    if not x.is_cuda:
        raise ValueError("the operands must be on the GPU")
    a = optorch_linear_t()
    a.precision, a.activation = _precision(x.dtype), ACTIVATIONS[activation]
    a.rows, a.in_features, a.out_features = rows, _int32("in_features", cin), _int32("out_features", cout)
    return a


def _matrix_call(torch, fn, a, device, workspace=None):
    """fn(a) on device's current stream; workspace(a): the bytes it needs."""
    if torch._C._cuda_getDevice() != device.index:  # (torch.cuda.current_device() asks whether there is one first: 0.5 us)
        with torch.cuda.device(device):
            return _matrix_call(torch, fn, a, device, workspace)
    if workspace is not None:
        n = workspace(a)
        if n < 0:
            _mat_fail(n)
        if n:
            ws = torch.empty(n, dtype=torch.uint8, device=device)  # (torch aligns allocations to 512 bytes)
            a.workspace, a.workspace_bytes = ws.data_ptr(), n
    a.hip_stream = torch._C._cuda_getCurrentRawStream(device.index)  # (current_stream() makes an object: 2.6 us of a call's 12)
    rc = fn(C.byref(a))
    if rc != OK:
        _mat_fail(rc)


def linear_forward(x, w, bias=None, *, residual=None, activation="none", save_pre=False, out=None):
    """y = activation(x w^T + bias) + residual: x [rows, in] and w [out, in] in fp32, bf16 or fp16, bias float32 [out],
    residual [rows, out].  save_pre: also returns z = x w^T + bias, which `linear_backward` reads.  out: where y goes; it may
    be the residual, and share no element with anything else.  Nothing is recorded for autograd: the gradients are
    `linear_backward`'s, whether or not the tensors require them."""
    import torch
    rows, cin = x.shape
    cout = w.shape[0]
    a = _linear_args(x, activation, rows, cin, cout)
    _check_matrix("x", x, rows, cin, x)
    _check_matrix("w", w, cout, cin, x)
    a.x, a.ldx, a.w, a.ldw = x.data_ptr(), _ld(x), w.data_ptr(), _ld(w)
    if bias is not None:
        _check_vector("bias", bias, cout, x)
        a.bias = bias.data_ptr()
    if residual is not None:
        _check_matrix("residual", residual, rows, cout, x)
        a.residual, a.ldr = residual.data_ptr(), _ld(residual)
    if out is None:
        out = torch.empty((rows, cout), dtype=x.dtype, device=x.device)
    else:
        _check_matrix("out", out, rows, cout, x)
    a.y, a.ldy = out.data_ptr(), _ld(out)
    z = None
    if save_pre:
        z = torch.empty((rows, cout), dtype=x.dtype, device=x.device)
        a.z, a.ldz = z.data_ptr(), cout
    lib = load_library()
    _matrix_call(torch, lib.optorch_linear_forward, a, x.device, lambda a: lib.optorch_linear_workspace(C.byref(a), 0))
    return (out, z) if save_pre else out


def linear_backward(dy, x, w, z=None, *, activation="none", need=("dx", "dw", "dbias"), dx=None, dw=None, dbias=None):
    """The gradients (dx, dw, dbias) of `linear_forward` from dy [rows, out] and what forward was given and saved; those not
    in `need` are not computed and come back as None.  dbias is float32, the others have x's type.  dx, dw, dbias: tensors to write
    them to (dw may be a view of a flat vector of gradients); they share no element with each other or with what is read."""
    import torch
    rows, cin = x.shape
    cout = w.shape[0]
    if not need or not set(need) <= {"dx", "dw", "dbias"}:
        raise ValueError("need must name some of dx, dw, dbias")
    a = _linear_args(x, activation, rows, cin, cout)
    _check_matrix("x", x, rows, cin, x)
    _check_matrix("w", w, cout, cin, x)
    _check_matrix("dy", dy, rows, cout, x)
    a.x, a.ldx, a.w, a.ldw, a.dy, a.lddy = x.data_ptr(), _ld(x), w.data_ptr(), _ld(w), dy.data_ptr(), _ld(dy)
    if activation != "none":
        if z is None:
            raise ValueError("z (linear_forward's save_pre) is needed for the slope of %s" % activation)
        _check_matrix("z", z, rows, cout, x)
        a.z, a.ldz = z.data_ptr(), _ld(z)
    for name, t in (("dx", dx), ("dw", dw), ("dbias", dbias)):
        if t is not None and name not in need:
            raise ValueError("%s: given, but not in need" % name)
    if "dx" in need:
        if dx is None:
            dx = torch.empty((rows, cin), dtype=x.dtype, device=x.device)
        _check_matrix("dx", dx, rows, cin, x)
        a.dx, a.lddx = dx.data_ptr(), _ld(dx)
    if "dw" in need:
        if dw is None:
            dw = torch.empty((cout, cin), dtype=x.dtype, device=x.device)
        _check_matrix("dw", dw, cout, cin, x)
        a.dw, a.lddw = dw.data_ptr(), _ld(dw)
    if "dbias" in need:
        if dbias is None:
            dbias = torch.empty(cout, dtype=torch.float32, device=x.device)
        _check_vector("dbias", dbias, cout, x)
        a.dbias = dbias.data_ptr()
    lib = load_library()
    _matrix_call(torch, lib.optorch_linear_backward, a, x.device, lambda a: lib.optorch_linear_workspace(C.byref(a), 1))
    return dx, dw, dbias


def _norm_args(x, weight):
    if not x.is_cuda:
        raise ValueError("the operands must be on the GPU")
    rows, cols = x.shape
    a = optorch_layer_norm_t()
    a.precision, a.cols, a.rows = _precision(x.dtype), _int32("cols", cols), rows
    _check_matrix("x", x, rows, cols, x)
    a.x, a.ldx = x.data_ptr(), _ld(x)
    if weight is not None:
        _check_vector("weight", weight, cols, x)
        a.weight = weight.data_ptr()
    return a, rows, cols


def layer_norm_forward(x, weight=None, bias=None, *, eps=1e-5, save_stats=False, out=None):
    """y = (x - mean) / sqrt(variance + eps) * weight + bias for every row of x [rows, cols] in fp32, bf16 or fp16; weight and
    bias float32 [cols], without them ones and zeros.  save_stats: returns (y, mean, rstd), which `layer_norm_backward` reads, float32
    [rows] each.  out: where y goes; it shares no element with anything else.  Nothing is recorded for autograd."""
    import torch
    a, rows, cols = _norm_args(x, weight)
    if bias is not None:
        _check_vector("bias", bias, cols, x)
        a.bias = bias.data_ptr()
    a.eps = eps
    if out is None:
        out = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
    else:
        _check_matrix("out", out, rows, cols, x)
    a.y, a.ldy = out.data_ptr(), _ld(out)
    if save_stats:
        mean, rstd = torch.empty((2, rows), dtype=torch.float32, device=x.device).unbind()
        a.mean, a.rstd = mean.data_ptr(), rstd.data_ptr()
    _matrix_call(torch, load_library().optorch_layer_norm_forward, a, x.device)
    return (out, mean, rstd) if save_stats else out


def layer_norm_backward(dy, x, mean, rstd, weight=None, *, residual=None, need=("dx", "dweight", "dbias"), dx=None, dweight=None, dbias=None):
    """The gradients (dx, dweight, dbias) of `layer_norm_forward` from dy [rows, cols], what it was given and the mean and rstd that
    it returned; those not in `need` are not computed and come back as None.  residual [rows, cols]: added to dx, the gradient that
    reaches x past the norm.  dweight and dbias are float32, dx has x's type.  dx, dweight, dbias: tensors to write them to; dx may be
    the residual, otherwise they share no element with each other or with what is read."""
    import torch
    a, rows, cols = _norm_args(x, weight)
    if not need or not set(need) <= {"dx", "dweight", "dbias"}:
        raise ValueError("need must name some of dx, dweight, dbias")
    for name, t in (("dx", dx), ("dweight", dweight), ("dbias", dbias)):
        if t is not None and name not in need:
            raise ValueError("%s: given, but not in need" % name)
    _check_matrix("dy", dy, rows, cols, x)
    _check_vector("mean", mean, rows, x)
    _check_vector("rstd", rstd, rows, x)
    a.dy, a.lddy, a.mean, a.rstd = dy.data_ptr(), _ld(dy), mean.data_ptr(), rstd.data_ptr()
    if residual is not None:
        if "dx" not in need:
            raise ValueError("residual: given, but dx is not in need")
        _check_matrix("residual", residual, rows, cols, x)
        a.residual, a.ldr = residual.data_ptr(), _ld(residual)
    if "dx" in need:
        if dx is None:
            dx = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        _check_matrix("dx", dx, rows, cols, x)
        a.dx, a.lddx = dx.data_ptr(), _ld(dx)
    if "dweight" in need:
        if dweight is None:
            dweight = torch.empty(cols, dtype=torch.float32, device=x.device)
        _check_vector("dweight", dweight, cols, x)
        a.dweight = dweight.data_ptr()
    if "dbias" in need:
        if dbias is None:
            dbias = torch.empty(cols, dtype=torch.float32, device=x.device)
        _check_vector("dbias", dbias, cols, x)
        a.dbias = dbias.data_ptr()
    lib = load_library()
    _matrix_call(torch, lib.optorch_layer_norm_backward, a, x.device, lambda a: lib.optorch_layer_norm_workspace(C.byref(a)))
    return dx, dweight, dbias


def _loss_args(x, w, bias):
    if not x.is_cuda:
        raise ValueError("the operands must be on the GPU")
    rows, cin = x.shape
    classes = w.shape[0]
    a = optorch_softmax_loss_t()
    a.precision, a.rows, a.in_features, a.classes = _precision(x.dtype), rows, _int32("in_features", cin), _int32("classes", classes)
    _check_matrix("x", x, rows, cin, x)
    _check_matrix("w", w, classes, cin, x)
    a.x, a.ldx, a.w, a.ldw = x.data_ptr(), _ld(x), w.data_ptr(), _ld(w)
    if bias is not None:
        _check_vector("bias", bias, classes, x)
        a.bias = bias.data_ptr()
    return a


def _labels(a, x, labels, label_smoothing, z_loss):
    import torch
    if labels.dtype != torch.int32 or labels.device != x.device:
        raise TypeError("labels: expected int32 on %s, got %s on %s" % (x.device, labels.dtype, labels.device))
    if labels.numel() != a.rows or not labels.is_contiguous():
        raise ValueError("labels: expected %d contiguous values" % a.rows)
    a.labels, a.label_smoothing, a.z_loss = labels.data_ptr(), label_smoothing, z_loss


def _teacher(a, x, indices, teacher, temperature):
    import torch
    if indices.dtype != torch.int32 or indices.device != x.device or teacher.device != x.device:
        raise TypeError("expected int32 indices and the teacher's logits on %s, got %s on %s and %s" % (x.device, indices.dtype, indices.device, teacher.device))
    if indices.dim() != 2 or indices.shape[0] != a.rows or indices.shape != teacher.shape:
        raise ValueError("indices and teacher: expected two matrices of %d rows and the same columns, got %s and %s" % (
            a.rows, tuple(indices.shape), tuple(teacher.shape)))
    if a.rows and indices.shape[1] > 1 and (indices.stride(1) != 1 or teacher.stride(1) != 1):
        raise ValueError("indices and teacher: the elements of a row must lie next to each other")
    a.teacher_precision, a.top, a.temperature = _precision(teacher.dtype), _int32("top", indices.shape[1]), temperature
    a.indices, a.ldi, a.teacher, a.ldt = indices.data_ptr(), _ld(indices), teacher.data_ptr(), _ld(teacher)


def _loss_forward(a, x):
    import torch
    loss, lse = torch.empty((2, a.rows), dtype=torch.float32, device=x.device).unbind()
    a.loss, a.lse = loss.data_ptr(), lse.data_ptr()
    lib = load_library()
    _matrix_call(torch, lib.optorch_softmax_loss_forward, a, x.device, lambda a: lib.optorch_softmax_loss_workspace(C.byref(a), 0))
    return loss, lse


def _loss_backward(a, dloss, x, lse, bias, need, dx, dw, dbias):
    import torch
    rows, cin, classes = a.rows, a.in_features, a.classes
    if need is None:
        need = ("dx", "dw") if bias is None else ("dx", "dw", "dbias")
    if not need or not set(need) <= {"dx", "dw", "dbias"}:
        raise ValueError("need must name some of dx, dw, dbias")
    for name, t in (("dx", dx), ("dw", dw), ("dbias", dbias)):
        if t is not None and name not in need:
            raise ValueError("%s: given, but not in need" % name)
    _check_vector("dloss", dloss, rows, x)
    _check_vector("lse", lse, rows, x)
    a.dloss, a.lse = dloss.data_ptr(), lse.data_ptr()
    if "dx" in need:
        if dx is None:
            dx = torch.empty((rows, cin), dtype=x.dtype, device=x.device)
        _check_matrix("dx", dx, rows, cin, x)
        a.dx, a.lddx = dx.data_ptr(), _ld(dx)
    if "dw" in need:
        if dw is None:
            dw = torch.empty((classes, cin), dtype=x.dtype, device=x.device)
        _check_matrix("dw", dw, classes, cin, x)
        a.dw, a.lddw = dw.data_ptr(), _ld(dw)
    if "dbias" in need:
        if dbias is None:
            dbias = torch.empty(classes, dtype=torch.float32, device=x.device)
        _check_vector("dbias", dbias, classes, x)
        a.dbias = dbias.data_ptr()
    lib = load_library()
    _matrix_call(torch, lib.optorch_softmax_loss_backward, a, x.device, lambda a: lib.optorch_softmax_loss_workspace(C.byref(a), 1))
    return dx, dw, dbias


def cross_entropy_forward(x, w, labels, bias=None, *, label_smoothing=0.0, z_loss=0.0):
    """(loss, lse), float32 [rows] each: with s = x w^T + bias, lse = log(sum(exp(s))) and loss = lse - (target . s) + z_loss lse^2 for
    every row, where target is 1 at the row's label, or 1 - label_smoothing there and label_smoothing / classes everywhere.  x [rows, in]
    and w [classes, in] in fp32, bf16 or fp16, labels int32 [rows], bias float32 [classes] (-infinity leaves a class out; with label_smoothing losses are then
    infinite).  A
    negative label leaves the row out: its loss is zero; a label not below `classes` makes it NaN.  The logits are never held.  Nothing
    is recorded for autograd: the gradients are `cross_entropy_backward`'s."""
    a = _loss_args(x, w, bias)
    _labels(a, x, labels, label_smoothing, z_loss)
    return _loss_forward(a, x)


def cross_entropy_backward(dloss, x, w, labels, lse, bias=None, *, label_smoothing=0.0, z_loss=0.0, need=None, dx=None, dw=None, dbias=None):
    """The gradients (dx, dw, dbias) of sum(dloss * loss) from dloss, float32 [rows], what `cross_entropy_forward` was given and the
    lse that it returned; those not in `need` (all, dbias with a bias) are not computed and come back as None.  dbias is float32, the
    others have x's type.  dx, dw, dbias: tensors to write them to; they share no element with each other or with what is read."""
    a = _loss_args(x, w, bias)
    _labels(a, x, labels, label_smoothing, z_loss)
    return _loss_backward(a, dloss, x, lse, bias, need, dx, dw, dbias)


def distillation_forward(x, w, indices, teacher, bias=None, *, temperature=1.0):
    """(loss, lse), float32 [rows] each: the divergence sum(q (log q - log p)) of p = softmax(s), s = (x w^T + bias) / temperature,
    from a teacher's distribution q = softmax(teacher / temperature) over the classes of a row's indices, and lse = log(sum(exp(s))).
    indices int32 and teacher (fp32, bf16 or fp16) [rows, top]; entries with a negative index or a logit of -infinity are unused, a row
    without any other is left out, with a loss of zero; entries of one class add up; an index not below `classes` makes the loss NaN.
    x, w, bias as in `cross_entropy_forward`.  (The gradients of a temperature's loss are smaller by its square: multiply dloss by it.)"""
    a = _loss_args(x, w, bias)
    _teacher(a, x, indices, teacher, temperature)
    return _loss_forward(a, x)


def distillation_backward(dloss, x, w, indices, teacher, lse, bias=None, *, temperature=1.0, need=None, dx=None, dw=None, dbias=None):
    """The gradients (dx, dw, dbias) of sum(dloss * loss) of `distillation_forward`; arguments and results as in `cross_entropy_backward`."""
    a = _loss_args(x, w, bias)
    _teacher(a, x, indices, teacher, temperature)
    return _loss_backward(a, dloss, x, lse, bias, need, dx, dw, dbias)


class OrthoPlan:
    """optorch_ortho_create + optorch_ortho_query: the host-side plan for a list of matrices, no device needed.

    matrices: (rows, cols) each, one behind the other in a flat vector, or (offset, rows, cols, ld) for other places.
    steps: 5 where none or fewer are asked for.  coefficients: (a, b, c) for every step, or one such triple per step."""

    def __init__(self, matrices, *, steps: int = 5, coefficients=None, eps: float = 1e-7):
        self.lib = load_library()
        self.handle = C.c_void_p()
        arr = (optorch_matrix_t * max(1, len(matrices)))()
        at = self.elements = 0
        for i, m in enumerate(matrices):
            if len(m) == 2:
                m = (at, m[0], m[1], m[1])
            arr[i] = optorch_matrix_t(int(m[0]), _int32("rows", m[1]), _int32("cols", m[2]), int(m[3]))
            at = m[0] + (m[1] - 1) * m[3] + m[2]
            self.elements += m[1] * m[2]
        steps = steps if steps > 0 else 5  # (what the library takes it for, and reads coefficients of)
        cfg = optorch_ortho_config_t()
        cfg.steps, cfg.eps = steps, eps
        if coefficients is not None:
            co = list(coefficients)
            co = [float(v) for c in co for v in c] if hasattr(co[0], "__len__") else [float(v) for v in co] * steps
            if len(co) != 3 * steps:
                raise ValueError("expected %d coefficients, got %d" % (3 * steps, len(co)))
            cfg.coefficients = C.cast((C.c_float * len(co))(*co), C.POINTER(C.c_float))
        rc = self.lib.optorch_ortho_create(arr, len(matrices), C.byref(cfg), C.byref(self.handle))
        if rc != OK:
            self.handle = C.c_void_p()
            _mat_fail(rc)
        wb, span = C.c_uint64(), C.c_int64()
        self._check(self.lib.optorch_ortho_query(self.handle, C.byref(wb), C.byref(span)))
        self.workspace_bytes, self.span = wb.value, span.value

    def _check(self, rc: int):
        if rc != OK:
            _mat_fail(rc)

    def close(self):
        if getattr(self, "handle", None) and self.handle.value:
            self.lib.optorch_ortho_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Orthogonalizer(OrthoPlan):
    """A bound plan: workspace allocated through torch, calls on torch's current stream.  Calls of one object share the
    workspace: on different streams they have to be ordered by the caller.  An object may be dropped while its calls are still under way on any
    stream, but a graph that has captured one needs it alive for as long as it is replayed."""

    def __init__(self, matrices, *, device="cuda:0", **kw):
        import torch
        super().__init__(matrices, **kw)
        self.torch = torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the matrix operators only run on the HIP path")
        index = torch.device(device).index
        self.index = torch.cuda.current_device() if index is None else index
        self.device = torch.device("cuda", self.index)
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)
            self.home = torch.cuda.current_stream(self.device).cuda_stream  # whose work the allocator waits for before it gives the memory away
            # (the memory may have been another stream's until now)
            torch.cuda.current_stream(self.device).synchronize()
            self._check(self.lib.optorch_ortho_bind(self.handle, self.workspace.data_ptr(), self.workspace_bytes))

    def _here(self, t):
        return t.is_cuda and t.device.index == self.index

    def _flat(self, name, t, dtypes=None):
        if not self._here(t):
            raise TypeError("%s: expected a tensor on %s" % (name, self.device))
        if not t.is_contiguous() or t.numel() < self.span:
            raise ValueError("%s: expected at least %d contiguous elements" % (name, self.span))
        p = _precision(t.dtype)
        if dtypes is not None and p not in dtypes:
            raise TypeError("%s: unexpected type %s" % (name, t.dtype))
        return p

    def _stream(self):
        s = self.torch.cuda.current_stream(self.device)
        if s.cuda_stream != self.home and not self.torch.cuda.is_current_stream_capturing():
            self.workspace.record_stream(s)  # or it goes back to its first stream alone, tables and all, while this one's kernels read it
        return s.cuda_stream

    def orthogonalize(self, g, out=None):
        """Newton-Schulz steps on every matrix of the flat tensor g, into out, whose other elements are left alone (by default a new tensor of
        g's type, zero between the matrices)."""
        if out is None:
            out = self.torch.empty_like(g) if g.numel() == self.elements else self.torch.zeros_like(g)
        gp, op = self._flat("g", g), self._flat("out", out)
        with self.torch.cuda.device(self.device):
            self._check(self.lib.optorch_orthogonalize(self.handle, gp, g.data_ptr(), op, out.data_ptr(), self._stream()))
        return out

    def muon_update(self, w, v, g, *, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale="aspect", grad_scale=1.0,
                    weights16=None, skipped=None):
        """One update of all matrices in place (optorch_muon_update): float32 weights w and momentum v, gradients g, all flat;
        weights16: a bf16 or fp16 copy of w that is refreshed; skipped: cuda int32 tensor of one element, set to 1 if the
        update was skipped because of a gradient that is not finite, else 0."""
        a = optorch_muon_t()
        a.g_precision = self._flat("g", g)
        self._flat("w", w, (0,))
        self._flat("v", v, (0,))
        a.g, a.w, a.v = g.data_ptr(), w.data_ptr(), v.data_ptr()
        if weights16 is not None:
            a.w16_precision, a.w16 = self._flat("weights16", weights16, (1, 2)), weights16.data_ptr()
        if scale not in SCALE_MODES:
            raise ValueError("scale must be one of %s" % ", ".join(sorted(SCALE_MODES)))
        a.lr, a.momentum, a.weight_decay, a.grad_scale = lr, momentum, weight_decay, grad_scale
        a.nesterov, a.scale_mode = int(nesterov), SCALE_MODES[scale]
        if skipped is not None:
            if skipped.dtype != self.torch.int32 or skipped.numel() != 1 or not self._here(skipped):
                raise TypeError("skipped: expected one int32 on %s" % self.device)
            a.skipped = skipped.data_ptr()
        with self.torch.cuda.device(self.device):
            self._check(self.lib.optorch_muon_update(self.handle, C.byref(a), self._stream()))
