"""ctypes binding of include/lqsgd.h, include/lqsgd_linear.h and include/lqsgd_block.h.  Argument marshalling only: every step of
the compressor, of the linear layer and of what stands around it runs in the HIP library.  torch is used for device memory and
the stream handle, nothing else."""
from __future__ import annotations

import ctypes as C
import os
import types
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# LQSGD_LIB points at another build of the same library (kernel experiments)
LIB_PATH = os.environ.get("LQSGD_LIB") or os.path.join(_HERE, "liblqsgd.so")

OK, EINVAL, ESHAPE, EUNSUPPORTED, ENOMEM, EHIP, ESTATE = 0, -1, -2, -3, -4, -5, -6
LAYER_MATRIX, LAYER_VECTOR = 0, 1
FLAG_NONE, FLAG_EAGER_RESIDUAL, FLAG_AGGREGATE_FIRST, FLAG_BF16_GRADIENTS, FLAG_NO_COOPERATIVE_LAUNCH = 0, 1, 2, 4, 8
PHASE_P, PHASE_Q = 0, 1
FACTOR_P_PRE, FACTOR_P_ORTH, FACTOR_P_BAR, FACTOR_Q_W, FACTOR_Q_BAR, FACTOR_VMEAN, FACTOR_P_MEAN = range(7)
(KERNEL_ADD_PROJECT, KERNEL_ORTH, KERNEL_EXCHANGE_P, KERNEL_BACK_PROJECT, KERNEL_REDUCE_Q,
 KERNEL_EXCHANGE_Q, KERNEL_RESIDUAL, KERNEL_REDUCE_P) = range(8)
KERNEL_COUNT = 8
MAX_RANK, MAX_WORKERS = 64, 64

# every symbol the header declares
SYMBOLS = [
    "lqsgd_create", "lqsgd_destroy", "lqsgd_synchronize", "lqsgd_last_error", "lqsgd_set_q",
    "lqsgd_get_state", "lqsgd_set_state", "lqsgd_compress", "lqsgd_decompress", "lqsgd_step", "lqsgd_step_update",
    "lqsgd_get_packet", "lqsgd_set_packet", "lqsgd_get_packet_raw", "lqsgd_packet_device", "lqsgd_get_factor",
    "lqsgd_set_factor", "lqsgd_wire_bytes", "lqsgd_plan_query", "lqsgd_plan_tiles",
    "lqsgd_timing_enable", "lqsgd_timing_read", "lqsgd_kernel_name", "lqsgd_launched_kernel", "lqsgd_step_static",
]
# ... and lqsgd_linear.h
LINEAR_SYMBOLS = [
    "lqsgd_linear_create", "lqsgd_linear_destroy", "lqsgd_linear_synchronize", "lqsgd_linear_last_error", "lqsgd_checkpoint_stride",
    "lqsgd_checkpoint_save", "lqsgd_checkpoint_load", "lqsgd_linear_forward", "lqsgd_linear_activation_backward",
    "lqsgd_linear_input_grad", "lqsgd_linear_weight_grad",
]
# ... and lqsgd_block.h
BLOCK_SYMBOLS = ["lqsgd_rows_save", "lqsgd_rows_load", "lqsgd_rms_norm", "lqsgd_rms_norm_backward", "lqsgd_int8_forward", "lqsgd_dropout"]
TYPE_F32, TYPE_BF16, TYPE_F16 = range(3)
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
CHECKPOINT_GROUP = 32
INT8_MAX_COLS = 131040


class LqsgdError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("lqsgd error %d: %s" % (code, msg))
        self.code = code


class Layer(C.Structure):
    _fields_ = [("rows", C.c_int32), ("cols", C.c_int32), ("flags", C.c_uint32)]


class Config(C.Structure):
    _fields_ = [("rank", C.c_int32), ("bits_p", C.c_int32), ("bits_q", C.c_int32),
                ("workers", C.c_int32), ("alpha", C.c_float), ("flags", C.c_uint32)]


class PlanInfo(C.Structure):
    _fields_ = [("device_bytes", C.c_int64), ("wire_bytes", C.c_int64), ("matrix_elements", C.c_int64),
                ("n_matrix", C.c_int32), ("n_vector", C.c_int32), ("rank_pad", C.c_int32),
                ("tiles", C.c_int32 * 3), ("reserved", C.c_int32),
                ("residual_stride", C.c_int64), ("warm_q_floats", C.c_int64)]


_lib = None


def lib():
    """The loaded library.  Raises if it has not been built: there is no
    fallback path."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("%s is missing: build it with `python -m paper_2506_17974_amd.build` "
                           "(there is no CPU or PyTorch fallback)" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    fp = C.POINTER(C.c_float)
    u8p = C.POINTER(C.c_uint8)
    L.lqsgd_create.argtypes = [C.POINTER(Config), C.POINTER(Layer), i32, vp, C.POINTER(vp)]
    L.lqsgd_destroy.argtypes = [vp]
    L.lqsgd_synchronize.argtypes = [vp]
    L.lqsgd_last_error.argtypes = [vp]
    L.lqsgd_last_error.restype = C.c_char_p
    L.lqsgd_set_q.argtypes = [vp, i32, fp]
    L.lqsgd_get_state.argtypes = [vp, i32, i32, fp, fp]
    L.lqsgd_set_state.argtypes = [vp, i32, i32, fp, fp]
    L.lqsgd_compress.argtypes = [vp, i32, C.POINTER(vp)]
    L.lqsgd_decompress.argtypes = [vp, i32]
    L.lqsgd_step.argtypes = [vp, C.POINTER(vp), C.POINTER(vp)]
    L.lqsgd_step_update.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), C.c_float]
    L.lqsgd_step_static.argtypes = [C.POINTER(Config), C.POINTER(Layer), i32, vp, C.POINTER(vp), vp, vp, C.POINTER(vp)]
    L.lqsgd_get_packet.argtypes = [vp, i32, i32, i32, u8p, u8p, fp]
    L.lqsgd_set_packet.argtypes = [vp, i32, i32, i32, u8p, u8p, C.c_float]
    L.lqsgd_get_packet_raw.argtypes = [vp, i32, i32, i32, u8p, C.POINTER(i64), u8p, C.POINTER(i64)]
    L.lqsgd_packet_device.argtypes = [vp, i32, i32, i32, C.POINTER(C.c_void_p), C.POINTER(i64), C.POINTER(C.c_void_p),
                                      C.POINTER(i64), C.POINTER(C.c_void_p)]
    L.lqsgd_get_factor.argtypes = [vp, i32, i32, i32, fp]
    L.lqsgd_set_factor.argtypes = [vp, i32, i32, fp]
    L.lqsgd_wire_bytes.argtypes = [vp]
    L.lqsgd_wire_bytes.restype = i64
    L.lqsgd_plan_query.argtypes = [C.POINTER(Config), C.POINTER(Layer), i32, C.POINTER(PlanInfo)]
    L.lqsgd_plan_tiles.argtypes = [C.POINTER(Config), C.POINTER(Layer), i32, i32, C.POINTER(i32), i64]
    L.lqsgd_plan_tiles.restype = i64
    L.lqsgd_timing_enable.argtypes = [vp, i32]
    L.lqsgd_timing_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(i64)]
    L.lqsgd_kernel_name.argtypes = [i32]
    L.lqsgd_kernel_name.restype = C.c_char_p
    L.lqsgd_launched_kernel.argtypes = [vp, i32]
    L.lqsgd_launched_kernel.restype = C.c_char_p
    L.lqsgd_linear_create.argtypes = [vp, C.POINTER(vp)]
    L.lqsgd_linear_destroy.argtypes = [vp]
    L.lqsgd_linear_synchronize.argtypes = [vp]
    L.lqsgd_linear_last_error.argtypes = [vp]
    L.lqsgd_linear_last_error.restype = C.c_char_p
    L.lqsgd_checkpoint_stride.argtypes = [i32]
    L.lqsgd_checkpoint_stride.restype = i64
    L.lqsgd_checkpoint_save.argtypes = [vp, i32, i64, i32, vp, i64, vp, vp]
    L.lqsgd_checkpoint_load.argtypes = [vp, i32, i64, i32, vp, vp, vp, i64]
    L.lqsgd_linear_forward.argtypes = [vp, i32, i32, i64, i32, i32, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp, vp, vp]
    L.lqsgd_linear_activation_backward.argtypes = [vp, i32, i32, i64, i32, vp, i64, vp, vp, vp, i64, vp, i32]
    L.lqsgd_linear_input_grad.argtypes = [vp, i32, i64, i32, i32, vp, i64, vp, i64, vp, i64]
    L.lqsgd_linear_weight_grad.argtypes = [vp, i32, i64, i32, i32, vp, i64, vp, vp, i32, vp, i64, i32]
    L.lqsgd_rows_save.argtypes = [vp, i32, i64, i32, vp, i64, vp, vp]
    L.lqsgd_rows_load.argtypes = [vp, i32, i64, i32, vp, vp, vp, i64]
    L.lqsgd_rms_norm.argtypes = [vp, i32, i64, i32, C.c_double, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp, vp, vp, vp]
    L.lqsgd_rms_norm_backward.argtypes = [vp, i32, i64, i32, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, i64, vp, i32]
    L.lqsgd_int8_forward.argtypes = [vp, i32, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, i64, vp, i64]
    L.lqsgd_dropout.argtypes = [vp, i32, i64, i32, C.c_double, C.c_uint64, C.c_uint64, vp, vp, i64, vp, i64, vp, i64, vp, vp]
    _lib = L
    return L


def _layers_array(layers: Sequence):
    arr = (Layer * len(layers))()
    for i, l in enumerate(layers):
        rows, cols = int(l[0]), int(l[1])
        flags = int(l[2]) if len(l) > 2 else LAYER_MATRIX
        arr[i] = Layer(rows, cols, flags)
    return arr


def layer_list(matrices, vectors=()):
    """[(rows, cols, flags)] with the matrices first, then the 1-D tensors."""
    return [(r, c, LAYER_MATRIX) for r, c in matrices] + [(n, 1, LAYER_VECTOR) for n in vectors]


def _f32p(a: np.ndarray):
    return a.ctypes.data_as(C.POINTER(C.c_float))


def _u8p(a: np.ndarray):
    return a.ctypes.data_as(C.POINTER(C.c_uint8))


def plan_query(layers, rank, bits_p, bits_q, workers, alpha=255.0, flags=0) -> PlanInfo:
    cfg = Config(rank, bits_p, bits_q, workers, alpha, flags)
    info = PlanInfo()
    rc = lib().lqsgd_plan_query(C.byref(cfg), _layers_array(layers), len(layers), C.byref(info))
    if rc:
        raise LqsgdError(rc, lib().lqsgd_last_error(None).decode())
    return info


def plan_tiles(layers, rank, bits_p, bits_q, workers, sweep, alpha=255.0) -> np.ndarray:
    cfg = Config(rank, bits_p, bits_q, workers, alpha, 0)
    arr = _layers_array(layers)
    n = lib().lqsgd_plan_tiles(C.byref(cfg), arr, len(layers), sweep, None, 0)
    if n < 0:
        raise LqsgdError(int(n), lib().lqsgd_last_error(None).decode())
    out = np.zeros((int(n), 6), np.int32)
    lib().lqsgd_plan_tiles(C.byref(cfg), arr, len(layers), sweep,
                           out.ctypes.data_as(C.POINTER(C.c_int32)), int(n))
    return out


class Compressor:
    """One lqsgd_ctx.  Gradients are torch CUDA tensors (or anything with
    .data_ptr()); the context's kernels run on torch's current stream at
    construction time."""

    def __init__(self, layers, rank, bits_p=8, bits_q=None, workers=1, alpha=255.0, flags=0, stream=None):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the LQ-SGD compressor has no CPU path")
        self.layers = [tuple(l) if len(l) > 2 else (l[0], l[1], LAYER_MATRIX) for l in layers]
        self.rank, self.workers = rank, workers
        self.bits_p = bits_p
        self.bits_q = bits_p if bits_q is None else bits_q
        self.alpha = alpha
        self._cfg = Config(rank, self.bits_p, self.bits_q, workers, alpha, flags)
        self._h = C.c_void_p()
        if stream is None:
            stream = torch.cuda.current_stream().cuda_stream
        self.stream_handle = int(stream)
        rc = lib().lqsgd_create(C.byref(self._cfg), _layers_array(self.layers), len(self.layers),
                                C.c_void_p(self.stream_handle), C.byref(self._h))
        if rc:
            self._h = C.c_void_p()
            raise LqsgdError(rc, lib().lqsgd_last_error(None).decode())
        self._keep = None

    # -- helpers ---------------------------------------------------------
    def _check(self, rc):
        if rc:
            raise LqsgdError(rc, lib().lqsgd_last_error(self._h).decode())

    def layer_rank(self, l):
        rows, cols, _ = self.layers[l]
        return min(self.rank, rows, cols)

    def _ptr_table(self, grads):
        """grads[w][l] tensors -> (c_void_p * (W*L))"""
        n = len(self.layers)
        tab = (C.c_void_p * (self.workers * n))()
        for w in range(self.workers):
            for l in range(n):
                tab[w * n + l] = grads[w][l].data_ptr()
        return tab

    def close(self):
        if self._h:
            lib().lqsgd_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- state -----------------------------------------------------------
    def set_q(self, layer, q: np.ndarray):
        q = np.ascontiguousarray(q, np.float32)
        rows, cols, _ = self.layers[layer]
        assert q.shape == (cols, self.layer_rank(layer)), q.shape
        self._check(lib().lqsgd_set_q(self._h, layer, _f32p(q)))

    def get_state(self, layer, worker, want_e=True, want_q=True):
        if not (0 <= layer < len(self.layers)):      # let the library report it
            self._check(lib().lqsgd_get_state(self._h, layer, worker, None, None))
        rows, cols, _ = self.layers[layer]
        e = np.empty((rows, cols), np.float32) if want_e else None
        q = np.empty((cols, self.layer_rank(layer)), np.float32) if want_q else None
        self._check(lib().lqsgd_get_state(self._h, layer, worker, _f32p(e) if want_e else None,
                                          _f32p(q) if want_q else None))
        return e, q

    def set_state(self, layer, worker, e: Optional[np.ndarray] = None, q: Optional[np.ndarray] = None):
        if e is not None:
            e = np.ascontiguousarray(e, np.float32)
        if q is not None:
            q = np.ascontiguousarray(q, np.float32)
        self._check(lib().lqsgd_set_state(self._h, layer, worker, _f32p(e) if e is not None else None,
                                          _f32p(q) if q is not None else None))

    # -- the compressor --------------------------------------------------
    def compress(self, phase, grads=None):
        tab = self._ptr_table(grads) if grads is not None else None
        self._keep = grads if grads is not None else self._keep
        self._check(lib().lqsgd_compress(self._h, phase, tab))

    def decompress(self, phase):
        self._check(lib().lqsgd_decompress(self._h, phase))

    def step(self, grads, ghat=None):
        tab = self._ptr_table(grads)
        gt = None
        if ghat is not None:
            gt = (C.c_void_p * len(self.layers))()
            for l, t in enumerate(ghat):
                gt[l] = t.data_ptr() if t is not None else None
        self._keep = (grads, ghat)
        self._check(lib().lqsgd_step(self._h, tab, gt))

    def step_update(self, grads, params, eta):
        """lqsgd_step_update: the iteration plus w <- w - eta G-hat on `params`
        (a list over layers of device tensors or None), in place."""
        tab = self._ptr_table(grads)
        pt = (C.c_void_p * len(self.layers))()
        for l, t in enumerate(params):
            pt[l] = t.data_ptr() if t is not None else None
        self._keep = (grads, params)
        self._check(lib().lqsgd_step_update(self._h, tab, pt, float(eta)))

    def step_raw(self, tab, gt=None):
        """lqsgd_step with a pointer table made earlier by pointer_table()."""
        self._check(lib().lqsgd_step(self._h, tab, gt))

    def pointer_table(self, grads):
        self._keep = grads
        return self._ptr_table(grads)

    def synchronize(self):
        self._check(lib().lqsgd_synchronize(self._h))

    # -- taps ------------------------------------------------------------
    def _factor_len(self, phase, layer):
        rows, cols, _ = self.layers[layer]
        return (cols if phase == PHASE_Q else rows) * self.layer_rank(layer)

    def get_packet(self, phase, layer, worker):
        n = self._factor_len(phase, layer)
        k = np.empty(n, np.uint8)
        s = np.empty(n, np.uint8)
        sc = C.c_float()
        self._check(lib().lqsgd_get_packet(self._h, phase, layer, worker, _u8p(k), _u8p(s), C.byref(sc)))
        shape = (n // self.layer_rank(layer), self.layer_rank(layer))
        return k.reshape(shape), s.reshape(shape), np.float32(sc.value)

    def set_packet(self, phase, layer, worker, k, s, scale):
        k = np.ascontiguousarray(k, np.uint8).ravel()
        s = np.ascontiguousarray(s, np.uint8).ravel()
        assert k.size == self._factor_len(phase, layer) == s.size
        self._check(lib().lqsgd_set_packet(self._h, phase, layer, worker, _u8p(k), _u8p(s), float(scale)))

    def packet_device(self, phase, layer, worker):
        """(mag_ptr, mag_len, sign_ptr, sign_len, scale_ptr): device addresses of one packet."""
        mp, sp, cp = C.c_void_p(), C.c_void_p(), C.c_void_p()
        ml, sl = C.c_int64(), C.c_int64()
        self._check(lib().lqsgd_packet_device(self._h, phase, layer, worker, C.byref(mp), C.byref(ml), C.byref(sp),
                                              C.byref(sl), C.byref(cp)))
        return mp.value, ml.value, sp.value, sl.value, cp.value

    def get_packet_raw(self, phase, layer, worker):
        ml, sl = C.c_int64(), C.c_int64()
        self._check(lib().lqsgd_get_packet_raw(self._h, phase, layer, worker, None, C.byref(ml), None, C.byref(sl)))
        mag = np.empty(ml.value, np.uint8)
        sgn = np.empty(sl.value, np.uint8)
        self._check(lib().lqsgd_get_packet_raw(self._h, phase, layer, worker, _u8p(mag), C.byref(ml),
                                               _u8p(sgn), C.byref(sl)))
        return mag, sgn

    def get_factor(self, which, layer, worker=0):
        rows, cols, flags = self.layers[layer]
        if which == FACTOR_VMEAN:
            out = np.empty(rows, np.float32)
        elif which in (FACTOR_Q_W, FACTOR_Q_BAR):
            out = np.empty((cols, self.layer_rank(layer)), np.float32)
        else:
            out = np.empty((rows, self.layer_rank(layer)), np.float32)
        self._check(lib().lqsgd_get_factor(self._h, which, layer, worker, _f32p(out)))
        return out

    def set_factor(self, which, layer, value):
        value = np.ascontiguousarray(value, np.float32)
        self._check(lib().lqsgd_set_factor(self._h, which, layer, _f32p(value)))

    def wire_bytes(self) -> int:
        return int(lib().lqsgd_wire_bytes(self._h))

    # -- timing ----------------------------------------------------------
    def timing_enable(self, on=True):
        self._check(lib().lqsgd_timing_enable(self._h, 1 if on else 0))

    def launched_kernel(self, k: int) -> str:
        """Device function last launched for timing slot k (template arguments included)."""
        return lib().lqsgd_launched_kernel(self._h, k).decode()

    def timing_read(self):
        ms = (C.c_double * KERNEL_COUNT)()
        n = (C.c_int64 * KERNEL_COUNT)()
        self._check(lib().lqsgd_timing_read(self._h, ms, n))
        return [float(x) for x in ms], [int(x) for x in n]


def step_static(layers, rank, bits_p, bits_q, workers, alpha, flags, grads, residual, warm_q, ghat=None, stream=None):
    """lqsgd_step_static: one iteration on caller-held state, no device allocation.
    grads[w][l]: device tensors; residual, warm_q: device tensors laid out as the header says
    (None when there is no matrix layer); ghat: list over layers of device tensors / None."""
    import torch
    cfg = Config(rank, bits_p, bits_q, workers, alpha, flags)
    n = len(layers)
    tab = (C.c_void_p * (workers * n))()
    for w in range(workers):
        for l in range(n):
            tab[w * n + l] = grads[w][l].data_ptr()
    gt = None
    if ghat is not None:
        gt = (C.c_void_p * n)()
        for l, t in enumerate(ghat):
            gt[l] = t.data_ptr() if t is not None else None
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    rc = lib().lqsgd_step_static(C.byref(cfg), _layers_array(layers), n, C.c_void_p(int(stream)), tab,
                                 C.c_void_p(residual.data_ptr() if residual is not None else None),
                                 C.c_void_p(warm_q.data_ptr() if warm_q is not None else None), gt)
    if rc:
        raise LqsgdError(rc, lib().lqsgd_last_error(None).decode())


def kernel_name(k: int) -> str:
    return lib().lqsgd_kernel_name(k).decode()


# -- the linear layer --------------------------------------------------------
class Checkpoint:
    """A samples x features tensor kept in 8 bits, as include/lqsgd_linear.h lays it out: `codes` (int8, samples x the features rounded
    up to groups of 32) and `exponents` (uint8, samples x groups).  Made of those two, or by empty() with both in one allocation."""
    __slots__ = ("features", "_codes", "_exponents", "_both", "_at")

    def __init__(self, codes, exponents, features):
        self.features, self._codes, self._exponents = int(features), codes, exponents
        self._both = self._at = None

    @classmethod
    def empty(cls, samples, features, device="cuda"):
        """One whose values are yet to be written."""
        import torch
        self = cls(None, None, features)
        groups = -(-self.features // CHECKPOINT_GROUP)
        n = samples * groups * CHECKPOINT_GROUP
        self._both = torch.empty(n + samples * groups, dtype=torch.uint8, device=device)
        at = self._both.data_ptr()
        self._at = (samples, self._both.get_device(), at, at + n, self.features)       # what LinearOps would find out about the two
        return self

    def _parts(self):
        samples, groups = self._at[0], -(-self._at[4] // CHECKPOINT_GROUP)
        n = samples * groups * CHECKPOINT_GROUP
        import torch
        self._codes = self._both[:n].view(torch.int8).view(samples, groups * CHECKPOINT_GROUP)
        self._exponents = self._both[n:].view(samples, groups)

    @property
    def codes(self):
        if self._codes is None:
            self._parts()
        return self._codes

    @property
    def exponents(self):
        if self._exponents is None:
            self._parts()
        return self._exponents

    @property
    def samples(self):
        return self._at[0] if self._at else self._codes.shape[0]

    @property
    def nbytes(self):
        return self.samples * -(-self.features // CHECKPOINT_GROUP) * (CHECKPOINT_GROUP + 1)


class RowCodes:
    """A samples x features tensor kept in 8 bits with a scale a row, as include/lqsgd_block.h lays it out: `codes` (int8, samples x the
    features rounded up to groups of 32) and `scales` (float32, samples).  Made of those two, or by empty() with both in one allocation."""
    __slots__ = ("features", "_codes", "_scales", "_both", "_at")

    def __init__(self, codes, scales, features):
        self.features, self._codes, self._scales = int(features), codes, scales
        self._both = self._at = None

    @classmethod
    def empty(cls, samples, features, device="cuda"):
        """One whose values are yet to be written."""
        import torch
        self = cls(None, None, features)
        n = samples * -(-self.features // CHECKPOINT_GROUP) * CHECKPOINT_GROUP
        self._both = torch.empty(n + 4 * samples, dtype=torch.uint8, device=device)
        at = self._both.data_ptr()
        self._at = (samples, self._both.get_device(), at, at + n, self.features)       # what LinearOps would find out about the two
        return self

    def _parts(self):
        import torch
        samples, stride = self._at[0], -(-self._at[4] // CHECKPOINT_GROUP) * CHECKPOINT_GROUP
        self._codes = self._both[:samples * stride].view(torch.int8).view(samples, stride)
        self._scales = self._both[samples * stride:].view(torch.float32)

    @property
    def codes(self):
        if self._codes is None:
            self._parts()
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            self._parts()
        return self._scales

    @property
    def samples(self):
        return self._at[0] if self._at else self._codes.shape[0]

    @property
    def nbytes(self):
        return self.samples * (-(-self.features // CHECKPOINT_GROUP) * CHECKPOINT_GROUP + 4)


_no_backward = None


def _without_autograd(out, *inputs):
    """`out`, a result that was just made from `inputs`.  Where autograd records and one of them has to have a gradient, `out` becomes
    part of the graph with a backward pass that raises: the gradient is not left out in silence."""
    global _no_backward
    import torch
    if not torch.is_grad_enabled() or not any(t is not None and t.requires_grad for t in inputs):
        return out
    if _no_backward is None:
        class NoBackward(torch.autograd.Function):
            @staticmethod
            def forward(ctx, out, *inputs):
                ctx.mark_dirty(out)
                return out

            @staticmethod
            def backward(ctx, *grads):
                raise LqsgdError(EINVAL, "autograd does not pass through the linear layer's calls: their gradients are made by "
                                         "activation_backward, input_grad, weight_grad, rms_norm_backward and dropout")
        _no_backward = NoBackward
    return _no_backward.apply(out, *inputs)


class LinearOps:
    """One lqsgd_linear context: the forward and backward passes of linear layers, and of the norms, 8-bit rows and dropout around them, on
    torch CUDA tensors (float32, bfloat16 or float16;
    two-dimensional, the elements of a row contiguous, rows at any stride).  Every call checks shapes, types and devices on the host
    and enqueues kernels on the stream that was current at construction; it raises where another stream is current, since the outputs
    that it allocates would belong to that one, and where another device is, since kernels would be launched there.
    Tensors made on other streams are the caller's to order, as with torch's own calls.
    So are the replays of a graph that the calls were captured into (on this stream: torch.cuda.graph(g, stream=...)): they use the context's
    workspace, and may run neither beside each other nor beside its other calls, nor after close() or the end of this object.  What is to run
    side by side takes a LinearOps each.

    The calls are a layer's passes, made by hand; autograd does not go through them.  A new tensor that a call returns, made from tensors that
    require a gradient while autograd records (the scales of RowCodes among them), raises where a backward() reaches it; a call that would make
    one from a tensor with a forward-mode tangent is refused.  Checkpoints and RowCodes that a call writes, and tensors given for the
    results, are plain memory: nothing is recorded for those."""

    def __init__(self):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the linear layer has no CPU path")
        import torch.autograd.forward_ad as dual
        self._torch, self._Tensor, self._empty = torch, torch.Tensor, torch.empty
        # inputs are asked for tangents within a level of forward-mode differentiation, or always where torch does not say that there is one
        self._dual = dual if hasattr(dual, "_current_level") else types.SimpleNamespace(_current_level=0, unpack_dual=dual.unpack_dual)
        self._types = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}
        self._f32, self._codes_type, self._exponents_type = torch.float32, torch.int8, torch.uint8
        self._h = C.c_void_p()
        self._index = torch.cuda.current_device()
        self.device = torch.device("cuda", self._index)
        # the current stream's handle, without the Stream object around it where torch has that
        self._stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        # kernels go to the current device: which that is has to be asked only where there are others
        self._current_device = torch.cuda.current_device if torch.cuda.device_count() > 1 else None
        self.stream_handle = int(self._stream(self._index))
        self._L = lib()
        rc = self._L.lqsgd_linear_create(C.c_void_p(self.stream_handle), C.byref(self._h))
        if rc:
            self._h = C.c_void_p()
            raise LqsgdError(rc, self._L.lqsgd_linear_last_error(None).decode())

    # -- helpers ---------------------------------------------------------
    def _check(self, rc):
        if rc:
            raise LqsgdError(rc, self._L.lqsgd_linear_last_error(self._h).decode())

    def _begin(self):
        """Whether the call may go on; True: after a look for tangents."""
        if not self._h:
            raise LqsgdError(ESTATE, "the context is closed")
        if self._current_device is not None and self._current_device() != self._index:
            raise LqsgdError(ESTATE, "the current device is not the one this context was made on, %s" % self.device)
        if self._stream(self._index) != self.stream_handle:
            raise LqsgdError(ESTATE, "the current stream is not the one this context was made on")
        return self._dual._current_level >= 0                 # inputs may have forward-mode tangents

    def _bad(self, what, t):
        raise LqsgdError(ESHAPE, "%s: %s" % (what, "%s %s on %s, strides %s" % (t.dtype, tuple(t.shape), t.device, t.stride())
                                             if isinstance(t, self._Tensor) else type(t).__name__))

    def _matrix(self, what, t, dtype=None, rows=None, cols=None):
        """(rows, cols, the distance between rows) of a two-dimensional tensor that the kernels take as it is."""
        if not isinstance(t, self._Tensor) or t.get_device() != self._index or t.dim() != 2:
            self._bad("%s has to be a two-dimensional tensor on %s" % (what, self.device), t)
        m, n = t.shape
        if t.dtype is not dtype if dtype is not None else t.dtype not in self._types:
            self._bad("%s has the wrong type" % what, t)
        if (rows is not None and m != rows) or (cols is not None and n != cols):
            self._bad("%s has the wrong shape, %s x %s wanted" % (what, rows, cols), t)
        ld, step = t.stride()
        if step != 1 and n > 1:
            self._bad("%s: the elements of a row have to be contiguous" % what, t)
        return m, n, ld if m > 1 else max(n, 1)

    def _vector(self, what, t, dtype, n):
        if not isinstance(t, self._Tensor) or t.get_device() != self._index or t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
            self._bad("%s has to be a contiguous vector of %d %s" % (what, n, dtype), t)
        return t.data_ptr()

    def _held(self, what, c, samples, features):
        if not isinstance(c, Checkpoint):
            raise LqsgdError(EINVAL, "%s has to be a Checkpoint" % what)
        if c.features != features:
            raise LqsgdError(ESHAPE, "%s has %d features, %d wanted" % (what, c.features, features))
        at = c._at
        if at is not None and at[0] == samples and at[1] == self._index and at[4] == features:
            return at[2], at[3]
        groups = -(-features // CHECKPOINT_GROUP)
        codes, exps = c.codes, c.exponents
        if codes.dtype is not self._codes_type or codes.shape != (samples, groups * CHECKPOINT_GROUP) or \
                codes.get_device() != self._index or not codes.is_contiguous():
            self._bad("%s: contiguous int8 codes of %d x %d wanted" % (what, samples, groups * CHECKPOINT_GROUP), codes)
        if exps.dtype is not self._exponents_type or exps.shape != (samples, groups) or exps.get_device() != self._index or \
                not exps.is_contiguous():
            self._bad("%s: contiguous uint8 exponents of %d x %d wanted" % (what, samples, groups), exps)
        return codes.data_ptr(), exps.data_ptr()

    def _rows(self, what, c, samples=None, features=None):
        if not isinstance(c, RowCodes):
            raise LqsgdError(EINVAL, "%s has to be RowCodes" % what)
        if features is not None and c.features != features:
            raise LqsgdError(ESHAPE, "%s has %d features, %d wanted" % (what, c.features, features))
        if samples is None:
            samples = c.samples
        at = c._at
        if at is not None and at[0] == samples and at[1] == self._index and at[4] == c.features:
            return at[2], at[3]
        stride = -(-c.features // CHECKPOINT_GROUP) * CHECKPOINT_GROUP
        codes, scales = c.codes, c.scales
        if codes.dtype is not self._codes_type or codes.shape != (samples, stride) or codes.get_device() != self._index or \
                not codes.is_contiguous():
            self._bad("%s: contiguous int8 codes of %d x %d wanted" % (what, samples, stride), codes)
        return codes.data_ptr(), self._vector("%s's scales" % what, scales, self._f32, samples)

    def _no_tangents(self, *inputs):
        """Forward-mode tangents would be left out of a new result in silence."""
        for t in inputs:
            if isinstance(t, self._Tensor) and self._dual.unpack_dual(t).tangent is not None:
                raise LqsgdError(EINVAL, "an input carries a forward-mode tangent, which the linear layer's calls do not pass on")

    def close(self):
        if self._h:
            self._L.lqsgd_linear_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def synchronize(self):
        self._check(self._L.lqsgd_linear_synchronize(self._h))

    # -- checkpoints -----------------------------------------------------
    def save(self, x, out=None):
        """x in 8 bits."""
        self._begin()
        m, n, ld = self._matrix("x", x)
        if out is None:
            out = Checkpoint.empty(m, n, self.device)
        codes, exps = self._held("out", out, m, n)
        self._check(self._L.lqsgd_checkpoint_save(self._h, self._types[x.dtype], m, n, x.data_ptr(), ld, codes, exps))
        return out

    def load(self, held, dtype=None, out=None):
        """The tensor that a checkpoint stands for, in `dtype` (default: out's, else bfloat16)."""
        self._begin()
        if not isinstance(held, Checkpoint):
            raise LqsgdError(EINVAL, "held has to be a Checkpoint")
        m, n = held.samples, held.features
        codes, exps = self._held("held", held, m, n)
        if out is None:
            dtype, ld = dtype or self._torch.bfloat16, n
            if dtype not in self._types:
                raise LqsgdError(EINVAL, "a checkpoint is not loaded as %s" % (dtype,))
            out = self._empty(m, n, dtype=dtype, device=self.device)
        else:
            ld = self._matrix("out", out, dtype, m, n)[2]
        self._check(self._L.lqsgd_checkpoint_load(self._h, self._types[out.dtype], m, n, codes, exps, out.data_ptr(), ld))
        return out

    # -- forward ---------------------------------------------------------
    def forward(self, x, w, bias=None, residual=None, act="none", out=None, save_z=None, save_y=None):
        """act(x w^T + bias) + residual.  save_z, save_y: Checkpoints of samples x rows that receive z and y as well."""
        if self._begin() and out is None:
            self._no_tangents(x, w, bias, residual)
        m, k, ldx = self._matrix("x", x)
        T = x.dtype
        n, _, ldw = self._matrix("w", w, T, None, k)
        if act not in ACTS:
            raise LqsgdError(EINVAL, "unknown activation %r" % (act,))
        b = self._vector("bias", bias, T, n) if bias is not None else None
        new = out is None
        r, ldr = (residual.data_ptr(), self._matrix("residual", residual, T, m, n)[2]) if residual is not None else (None, 0)
        if out is None:
            out, ldy = self._empty(m, n, dtype=T, device=self.device), n
        else:
            ldy = self._matrix("out", out, T, m, n)[2]
        zc, ze = self._held("save_z", save_z, m, n) if save_z is not None else (None, None)
        yc, ye = self._held("save_y", save_y, m, n) if save_y is not None else (None, None)
        self._check(self._L.lqsgd_linear_forward(self._h, self._types[T], ACTS[act], m, n, k, x.data_ptr(), ldx, w.data_ptr(), ldw,
                                                 b, r, ldr, out.data_ptr(), ldy, zc, ze, yc, ye))
        if new and (x.requires_grad or w.requires_grad or (b and bias.requires_grad) or (residual is not None and residual.requires_grad)):
            return _without_autograd(out, x, w, bias, residual)
        return out

    # -- backward --------------------------------------------------------
    def activation_backward(self, dy, z=None, act="none", dz=None, dbias=None, accumulate=False, want_dz=True, want_dbias=True):
        """(dz, dbias) of dy and the checkpoint z (not needed without an activation); what is not wanted is None.  dz may be dy."""
        if self._begin() and ((dz is None and want_dz) or (dbias is None and want_dbias)):
            self._no_tangents(dy)
        m, n, lddy = self._matrix("dy", dy)
        T = dy.dtype
        if act not in ACTS:
            raise LqsgdError(EINVAL, "unknown activation %r" % (act,))
        if z is None and act != "none":
            raise LqsgdError(EINVAL, "the activation's backward needs the checkpoint of z")
        zc, ze = self._held("z", z, m, n) if z is not None else (None, None)
        pz, lddz = None, 0
        new_dz, new_db = dz is None, dbias is None
        if dz is not None:
            pz, lddz = dz.data_ptr(), self._matrix("dz", dz, T, m, n)[2]
        elif want_dz:
            dz = self._empty(m, n, dtype=T, device=self.device)
            pz, lddz = dz.data_ptr(), n
        if dbias is None and want_dbias:
            if accumulate:
                raise LqsgdError(EINVAL, "accumulate needs the dbias to add to")
            dbias = self._empty(n, dtype=self._f32, device=self.device)
        db = self._vector("dbias", dbias, self._f32, n) if dbias is not None else None
        self._check(self._L.lqsgd_linear_activation_backward(self._h, self._types[T], ACTS[act], m, n, dy.data_ptr(), lddy, zc, ze, pz, lddz,
                                                             db, 1 if accumulate else 0))
        if dy.requires_grad:
            if new_dz and dz is not None:
                dz = _without_autograd(dz, dy)
            if new_db and dbias is not None:
                dbias = _without_autograd(dbias, dy)
        return dz, dbias

    def input_grad(self, dz, w, out=None):
        """dz w."""
        if self._begin() and out is None:
            self._no_tangents(dz, w)
        m, n, lddz = self._matrix("dz", dz)
        T = dz.dtype
        _, k, ldw = self._matrix("w", w, T, n, None)
        new = out is None
        if new:
            out, lddx = self._empty(m, k, dtype=T, device=self.device), k
        else:
            lddx = self._matrix("out", out, T, m, k)[2]
        self._check(self._L.lqsgd_linear_input_grad(self._h, self._types[T], m, n, k, dz.data_ptr(), lddz, w.data_ptr(), ldw, out.data_ptr(),
                                                    lddx))
        if new and (dz.requires_grad or w.requires_grad):
            return _without_autograd(out, dz, w)
        return out

    def weight_grad(self, dz, x, out=None, dtype=None, accumulate=False):
        """dz^T x^ of the checkpoint x, in float32 or bfloat16 (`dtype`; default: out's, else float32): a gradient for Compressor.step."""
        if self._begin() and out is None:
            self._no_tangents(dz)
        m, n, lddz = self._matrix("dz", dz)
        if not isinstance(x, Checkpoint):
            raise LqsgdError(EINVAL, "x has to be a Checkpoint")
        k = x.features
        xc, xe = self._held("x", x, m, k)
        new = out is None
        if new:
            if accumulate:
                raise LqsgdError(EINVAL, "accumulate needs the gradient to add to")
            dtype, lddw = dtype or self._f32, k
            if dtype not in self._types:
                raise LqsgdError(EINVAL, "a gradient is not written as %s" % (dtype,))
            out = self._empty(n, k, dtype=dtype, device=self.device)
        else:
            lddw = self._matrix("out", out, dtype, n, k)[2]
        self._check(self._L.lqsgd_linear_weight_grad(self._h, self._types[dz.dtype], m, n, k, dz.data_ptr(), lddz, xc, xe,
                                                     self._types[out.dtype], out.data_ptr(), lddw, 1 if accumulate else 0))
        if new and dz.requires_grad:
            return _without_autograd(out, dz)
        return out

    # -- around the layer --------------------------------------------------
    def quantize(self, x, out=None):
        """x as 8-bit rows with a scale each."""
        self._begin()
        m, n, ld = self._matrix("x", x)
        if out is None:
            out = RowCodes.empty(m, n, self.device)
        codes, scales = self._rows("out", out, m, n)
        self._check(self._L.lqsgd_rows_save(self._h, self._types[x.dtype], m, n, x.data_ptr(), ld, codes, scales))
        return out

    def dequantize(self, rows, dtype=None, out=None):
        """The tensor that 8-bit rows stand for, in `dtype` (default: out's, else bfloat16)."""
        if self._begin() and out is None:
            self._no_tangents(getattr(rows, "_scales", None))
        codes, scales = self._rows("rows", rows)
        m, n = rows.samples, rows.features
        new = out is None
        if new:
            dtype, ld = dtype or self._torch.bfloat16, n
            if dtype not in self._types:
                raise LqsgdError(EINVAL, "8-bit rows are not read back as %s" % (dtype,))
            out = self._empty(m, n, dtype=dtype, device=self.device)
        else:
            ld = self._matrix("out", out, dtype, m, n)[2]
        self._check(self._L.lqsgd_rows_load(self._h, self._types[out.dtype], m, n, codes, scales, out.data_ptr(), ld))
        if new and rows._scales is not None and rows._scales.requires_grad:       # of those of empty(): not unless somebody has had them
            return _without_autograd(out, rows._scales)
        return out

    def rms_norm(self, x, gain=None, residual=None, eps=1e-6, h=None, out=None, rstd=None, save_y=None, quantize_y=None, want_h=True,
                 want_y=True, want_rstd=False):
        """(y, h, rstd): h = x + residual (None without a residual, and where it is not wanted), y = h gain / sqrt(mean h^2 + eps), and
        rstd, which the backward pass needs.  save_y: a Checkpoint that receives y as well; quantize_y: RowCodes that do.  h may be x or the
        residual."""
        if self._begin() and ((h is None and want_h and residual is not None) or (out is None and want_y) or (rstd is None and want_rstd)):
            self._no_tangents(x, gain, residual)
        m, n, ldx = self._matrix("x", x)
        T = x.dtype
        g = self._vector("gain", gain, T, n) if gain is not None else None
        new_h, new_y, new_rstd = h is None, out is None, rstd is None
        r, ldr, ph, ldh, py, ldy = None, 0, None, 0, None, 0
        if residual is not None:
            r, ldr = residual.data_ptr(), self._matrix("residual", residual, T, m, n)[2]
            if new_h and want_h:
                h, ldh = self._empty(m, n, dtype=T, device=self.device), n
                ph = h.data_ptr()
        if not new_h:
            if residual is None:
                raise LqsgdError(EINVAL, "h is wanted without a residual: it is x")
            ph, ldh = h.data_ptr(), self._matrix("h", h, T, m, n)[2]
        if not new_y:
            py, ldy = out.data_ptr(), self._matrix("out", out, T, m, n)[2]
        elif want_y:
            out, ldy = self._empty(m, n, dtype=T, device=self.device), n
            py = out.data_ptr()
        if new_rstd and want_rstd:
            rstd = self._empty(m, dtype=self._f32, device=self.device)
        ps = self._vector("rstd", rstd, self._f32, m) if rstd is not None else None
        yc, ye = self._held("save_y", save_y, m, n) if save_y is not None else (None, None)
        qc, qs = self._rows("quantize_y", quantize_y, m, n) if quantize_y is not None else (None, None)
        self._check(self._L.lqsgd_rms_norm(self._h, self._types[T], m, n, eps, x.data_ptr(), ldx, r, ldr, g, ph, ldh, py, ldy, ps, yc, ye, qc, qs))
        if x.requires_grad or (g and gain.requires_grad) or (residual is not None and residual.requires_grad):
            out, h, rstd = (_without_autograd(t, x, gain, residual) if new and t is not None else t
                            for new, t in ((new_y, out), (new_h, h), (new_rstd, rstd)))
        return out, h, rstd

    def rms_norm_backward(self, dy, h, rstd, gain=None, dh=None, dx=None, dgain=None, accumulate=False, want_dx=True, want_dgain=True):
        """(dx, dgain) of dy and of dh, which came to h past the norm: dx is the gradient of rms_norm's x and of its residual alike.  h: the
        tensor that the norm was taken of (x without a residual), or a Checkpoint of it.  What is not wanted is None.  dx may be dy or dh."""
        if self._begin() and ((dx is None and want_dx) or (dgain is None and want_dgain)):
            self._no_tangents(dy, h, rstd, gain, dh)
        m, n, lddy = self._matrix("dy", dy)
        T = dy.dtype
        t = None if isinstance(h, Checkpoint) else h
        if t is None:
            ph, ldh = None, 0
            hc, he = self._held("h", h, m, n)
        else:
            ldh = self._matrix("h", h, T, m, n)[2]
            ph, hc, he = h.data_ptr(), None, None
        ps = self._vector("rstd", rstd, self._f32, m)
        g = self._vector("gain", gain, T, n) if gain is not None else None
        pdh, lddh = (dh.data_ptr(), self._matrix("dh", dh, T, m, n)[2]) if dh is not None else (None, 0)
        new_dx, new_dg = dx is None, dgain is None
        pdx, lddx = None, 0
        if not new_dx:
            pdx, lddx = dx.data_ptr(), self._matrix("dx", dx, T, m, n)[2]
        elif want_dx:
            dx, lddx = self._empty(m, n, dtype=T, device=self.device), n
            pdx = dx.data_ptr()
        if new_dg and want_dgain:
            if accumulate:
                raise LqsgdError(EINVAL, "accumulate needs the dgain to add to")
            dgain = self._empty(n, dtype=self._f32, device=self.device)
        pdg = self._vector("dgain", dgain, self._f32, n) if dgain is not None else None
        self._check(self._L.lqsgd_rms_norm_backward(self._h, self._types[T], m, n, dy.data_ptr(), lddy, ph, ldh, hc, he, ps, g, pdh, lddh,
                                                    pdx, lddx, pdg, 1 if accumulate else 0))
        if dy.requires_grad or rstd.requires_grad or (gain is not None and gain.requires_grad) or (dh is not None and dh.requires_grad) or \
                (t is not None and t.requires_grad):
            inputs = (dy, t, rstd, gain, dh)
            dx, dgain = (_without_autograd(o, *inputs) if new and o is not None else o for new, o in ((new_dx, dx), (new_dg, dgain)))
        return dx, dgain

    def int8_forward(self, x, w, bias=None, residual=None, act="none", dtype=None, out=None):
        """act(x w^T + bias) + residual of RowCodes x and w, in `dtype` (default: out's, the residual's or the bias', else bfloat16)."""
        if self._begin() and out is None:
            self._no_tangents(bias, residual, getattr(x, "_scales", None), getattr(w, "_scales", None))
        if act not in ACTS:
            raise LqsgdError(EINVAL, "unknown activation %r" % (act,))
        xc, xs = self._rows("x", x)
        m, k = x.samples, x.features
        wc, ws = self._rows("w", w, None, k)
        n = w.samples
        new = out is None
        T = dtype or next((t.dtype for t in (out, residual, bias) if isinstance(t, self._Tensor)), self._torch.bfloat16)
        if T not in self._types:
            raise LqsgdError(EINVAL, "a product is not written as %s" % (T,))
        b = self._vector("bias", bias, T, n) if bias is not None else None
        r, ldr = (residual.data_ptr(), self._matrix("residual", residual, T, m, n)[2]) if residual is not None else (None, 0)
        if new:
            out, ldy = self._empty(m, n, dtype=T, device=self.device), n
        else:
            ldy = self._matrix("out", out, T, m, n)[2]
        self._check(self._L.lqsgd_int8_forward(self._h, self._types[T], ACTS[act], m, n, k, xc, xs, wc, ws, b, r, ldr, out.data_ptr(), ldy))
        sx, sw = x._scales, w._scales
        if new and ((b and bias.requires_grad) or (residual is not None and residual.requires_grad) or (sx is not None and sx.requires_grad) or
                    (sw is not None and sw.requires_grad)):
            return _without_autograd(out, bias, residual, sx, sw)
        return out

    def dropout(self, x, p, seed, offset=0, residual=None, out=None, save_y=None, more_offset=None):
        """x with a share p of its values dropped and the others divided by 1 - p (p to a multiple of 2^-16), plus residual.  Which, is
        decided by seed, offset (64 bits each) and the place in the tensor: the gradient of x is dropout(dy, p, seed, offset).  out may be x or the
        residual; save_y: a Checkpoint that receives the result as well.  more_offset: an int64 tensor of one element on the device
        that is added to offset when the call runs: a graph that counts it up has another mask at each replay."""
        if self._begin() and out is None:
            self._no_tangents(x, residual)
        m, n, ldx = self._matrix("x", x)
        T = x.dtype
        if not 0 <= seed < 1 << 64 or not 0 <= offset < 1 << 64:
            raise LqsgdError(EINVAL, "seed and offset have 64 bits")
        more = None
        if more_offset is not None:
            if not isinstance(more_offset, self._Tensor) or more_offset.get_device() != self._index or more_offset.dtype is not self._torch.int64 or \
                    more_offset.numel() != 1:
                self._bad("more_offset has to be one int64 on %s" % self.device, more_offset)
            more = more_offset.data_ptr()
        new = out is None
        r, ldr = (residual.data_ptr(), self._matrix("residual", residual, T, m, n)[2]) if residual is not None else (None, 0)
        if new:
            out, ldy = self._empty(m, n, dtype=T, device=self.device), n
        else:
            ldy = self._matrix("out", out, T, m, n)[2]
        yc, ye = self._held("save_y", save_y, m, n) if save_y is not None else (None, None)
        self._check(self._L.lqsgd_dropout(self._h, self._types[T], m, n, p, seed, offset, more, x.data_ptr(), ldx, r, ldr, out.data_ptr(), ldy,
                                          yc, ye))
        if new and (x.requires_grad or (residual is not None and residual.requires_grad)):
            return _without_autograd(out, x, residual)
        return out
