"""ctypes binding of ``libnitro.so`` (declared in ``include/nitro.h``).

Argument marshalling only: every step of the block training step runs in the
library's CUDA kernels.  The module-level functions carry the C-ABI names and
return its status codes; ``Block`` wraps one handle for callers that hold
their activations and labels in torch CUDA tensors.  There is no CPU path:
loading fails loudly when the library has not been built.
"""
import ctypes
import os

import numpy as np

from . import build as _build

NITRO_OK, NITRO_ERR_ARG, NITRO_ERR_OVERFLOW, NITRO_ERR_TIMEOUT, NITRO_ERR_CUDA, \
    NITRO_ERR_UNSUPPORTED = range(6)
NITRO_CONV3X3, NITRO_LINEAR = 0, 1
NITRO_ROUND_FLOOR, NITRO_ROUND_TRUNC = 0, 1
STATUS_BIT_OVERFLOW, STATUS_BIT_BAD_LABEL, STATUS_BIT_TIMEOUT = 1, 2, 4
NITRO_CONTRACT_FWD, NITRO_CONTRACT_WGRAD, NITRO_CONTRACT_DGRAD = 0, 1, 2
NITRO_BF16, NITRO_I8, NITRO_F32, NITRO_I64 = range(4)
NITRO_ACT_NONE, NITRO_ACT_RELU, NITRO_ACT_SILU, NITRO_ACT_GELU = range(4)
(NITRO_T_W, NITRO_T_DW, NITRO_T_WLR, NITRO_T_DWLR, NITRO_T_ACT, NITRO_T_REGION,
 NITRO_T_ARGMAX, NITRO_T_DELTA, NITRO_T_GRAD_L, NITRO_T_SSE, NITRO_T_LR_IN, NITRO_T_LR_ARGMAX,
 NITRO_T_STEP) = range(13)

TENSOR_DTYPE = {
    NITRO_T_W: np.int32, NITRO_T_DW: np.int64, NITRO_T_WLR: np.int32, NITRO_T_DWLR: np.int64,
    NITRO_T_ACT: np.int8, NITRO_T_REGION: np.int8, NITRO_T_ARGMAX: np.int8,
    NITRO_T_DELTA: np.int32, NITRO_T_GRAD_L: np.int32, NITRO_T_SSE: np.int64,
    NITRO_T_LR_IN: np.int8, NITRO_T_LR_ARGMAX: np.uint8, NITRO_T_STEP: np.uint32,
}


class nitro_layer_desc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("cin", ctypes.c_int), ("cout", ctypes.c_int),
                ("h", ctypes.c_int), ("w", ctypes.c_int), ("pool2x2", ctypes.c_int)]


class nitro_clip_matrix(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld_in", ctypes.c_int64), ("ld_out", ctypes.c_int64),
                ("type", ctypes.c_int)]


class nitro_block_desc(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int), ("layers", ctypes.POINTER(nitro_layer_desc)),
                ("in_features", ctypes.c_int), ("num_classes", ctypes.c_int),
                ("alpha_inv", ctypes.c_int), ("gamma_inv_lr", ctypes.c_int64),
                ("eta_inv_fw", ctypes.c_int64), ("eta_inv_lr", ctypes.c_int64),
                ("sgd_round", ctypes.c_int), ("max_batch", ctypes.c_int),
                ("d_lr", ctypes.c_int), ("dropout_p16", ctypes.c_int)]


class NitroError(RuntimeError):
    def __init__(self, status, what=""):
        self.status = int(status)
        super().__init__("%s: %s (status %d)" % (what, status_str(status), int(status)))


_lib = None
_VP = ctypes.c_void_p


def lib():
    """The loaded ``libnitro.so``; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        raise RuntimeError("libnitro.so is missing (%s): build it with "
                           "paper_2407_11698_gb300.build.build() first" % _build.LIB)
    L = ctypes.CDLL(_build.LIB)
    L.nitro_init_block.argtypes = [ctypes.POINTER(nitro_block_desc), ctypes.c_uint64, _VP,
                                   ctypes.POINTER(_VP)]
    L.nitro_block_forward.argtypes = [_VP, _VP, ctypes.c_int, _VP, _VP]
    L.nitro_block_backward.argtypes = [_VP, _VP, _VP, ctypes.c_int, _VP, _VP]
    L.nitro_integersgd_step.argtypes = [_VP, _VP]
    L.nitro_block_backward_update.argtypes = [_VP, _VP, _VP, ctypes.c_int, _VP, _VP]
    L.nitro_block_tensor_bytes.argtypes = [_VP, ctypes.c_int, ctypes.c_int,
                                           ctypes.POINTER(ctypes.c_size_t)]
    L.nitro_block_get_tensor.argtypes = [_VP, ctypes.c_int, ctypes.c_int, _VP, ctypes.c_size_t]
    L.nitro_block_set_tensor.argtypes = [_VP, ctypes.c_int, ctypes.c_int, _VP, ctypes.c_size_t]
    L.nitro_block_status.argtypes = [_VP, ctypes.c_int]
    L.nitro_block_status_bits.argtypes = [_VP]
    L.nitro_block_status_bits.restype = ctypes.c_uint32
    L.nitro_destroy_block.argtypes = [_VP]
    L.nitro_destroy_block.restype = None
    L.nitro_status_str.argtypes = [ctypes.c_int]
    L.nitro_status_str.restype = ctypes.c_char_p
    L.nitro_kernel_launches.argtypes = []
    L.nitro_kernel_launches.restype = ctypes.c_uint64
    L.nitro_profile_enable.argtypes = [ctypes.c_int]
    L.nitro_profile_enable.restype = None
    L.nitro_profile_reset.argtypes = []
    L.nitro_profile_reset.restype = None
    L.nitro_profile_kernel_count.argtypes = []
    L.nitro_profile_kernel_count.restype = ctypes.c_int
    L.nitro_profile_kernel_name.argtypes = [ctypes.c_int]
    L.nitro_profile_kernel_name.restype = ctypes.c_char_p
    _PD = ctypes.POINTER(ctypes.c_double)
    L.nitro_profile_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_uint64), _PD, _PD, _PD]
    L.nitro_profile_read.restype = ctypes.c_int
    L.nitro_profile_record_count.argtypes = []
    L.nitro_profile_record_count.restype = ctypes.c_int
    L.nitro_profile_record.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_int), _PD, _PD, _PD]
    L.nitro_profile_record.restype = ctypes.c_int
    L.nitro_conv3x3_forward_noalloc.argtypes = [_VP, _VP] + [ctypes.c_int] * 7 + [_VP, _VP, _VP, _VP]
    L.nitro_conv3x3_forward_noalloc.restype = ctypes.c_int
    L.nitro_conv3x3_noalloc_status.argtypes = [ctypes.c_int]
    L.nitro_conv3x3_noalloc_status.restype = ctypes.c_int
    L.nitro_conv3x3_create.argtypes = [ctypes.c_int] * 5 + [ctypes.POINTER(_VP)]
    L.nitro_conv3x3_contract.argtypes = [_VP, ctypes.c_int, _VP, _VP, ctypes.c_int, _VP, _VP]
    L.nitro_conv3x3_status.argtypes = [_VP]
    L.nitro_conv3x3_destroy.argtypes = [_VP]
    L.nitro_conv3x3_destroy.restype = None
    L.nitro_gemm_create.argtypes = [ctypes.c_int] * 3 + [ctypes.POINTER(_VP)]
    L.nitro_gemm_run.argtypes = [_VP, _VP, _VP, ctypes.c_int, ctypes.c_int, ctypes.c_int, _VP, _VP]
    L.nitro_gemm_status.argtypes = [_VP]
    L.nitro_gemm_destroy.argtypes = [_VP]
    L.nitro_gemm_destroy.restype = None
    L.nitro_block_set_hyper.argtypes = [_VP, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64]
    L.nitro_block_set_hyper.restype = ctypes.c_int
    L.nitro_block_set_dropout.argtypes = [_VP, ctypes.c_int]
    L.nitro_block_set_dropout.restype = ctypes.c_int
    L.nitro_block_diag_timeout.argtypes = [_VP, ctypes.c_int, _VP]
    L.nitro_block_diag_timeout.restype = ctypes.c_int
    L.nitro_block_grad_device.argtypes = [_VP, ctypes.c_int, ctypes.c_int, ctypes.POINTER(_VP),
                                          ctypes.POINTER(ctypes.c_size_t)]
    L.nitro_block_grad_device.restype = ctypes.c_int
    L.nitro_prep_create.argtypes = [ctypes.POINTER(_VP)]
    L.nitro_prep_fit.argtypes = [_VP, _VP, ctypes.c_int64, _VP]
    L.nitro_prep_apply.argtypes = [_VP, _VP, ctypes.c_int64, _VP, _VP]
    L.nitro_prep_stats.argtypes = [_VP, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
    L.nitro_prep_destroy.argtypes = [_VP]
    L.nitro_prep_destroy.restype = None
    _I, _L, _F = ctypes.c_int, ctypes.c_int64, ctypes.c_float
    _PS = ctypes.POINTER(ctypes.c_size_t)
    L.nitro_xent_create.argtypes = [_I, _I, _I, ctypes.POINTER(_VP)]
    L.nitro_xent_forward.argtypes = [_VP, _VP, _I, _L, _VP, _L, _VP, _I, _F, _VP, _VP, _VP]
    L.nitro_xent_backward.argtypes = [_VP, _VP, _I, _L, _VP, _L, _VP, _I, _F, _VP, _VP, _VP, _L, _VP, _L, _VP]
    L.nitro_orth_create.argtypes = [_I, _I, _I, ctypes.POINTER(_VP)]
    L.nitro_orth_run.argtypes = [_VP, _VP, _I, _L, _L, _I, _I, ctypes.POINTER(_F), _VP, _L, _L, _VP]
    L.nitro_mx4_bytes.argtypes = [_I, _I, _PS, _PS]
    L.nitro_mx4_quantize.argtypes = [_VP, _I, _L, _I, _I, _VP, _VP, _VP]
    L.nitro_mx4_dequantize.argtypes = [_VP, _VP, _I, _I, _VP, _I, _L, _VP, _VP]
    L.nitro_mx4_create.argtypes = [_I, _I, _I, ctypes.POINTER(_VP)]
    L.nitro_mx4_linear.argtypes = [_VP, _VP, _I, _L, _I, _VP, _VP, _VP, _I, _L, _VP]
    L.nitro_gnorm_create.argtypes = [_I, _I, _I, _I, ctypes.POINTER(_VP)]
    L.nitro_gnorm_forward.argtypes = [_VP, _VP, _I, _L, _L, _I, _I, _VP, _VP, _F, _I, _VP, _I, _L, _L, _VP, _VP, _VP]
    L.nitro_gnorm_backward.argtypes = [_VP, _VP, _I, _L, _L, _I, _I, _VP, _VP, _VP, _VP, _I, _VP, _I, _L, _L, _VP, _L, _L, _VP,
                                       _VP, _VP]
    L.nitro_glu_create.argtypes = [_I, _I, _I, ctypes.POINTER(_VP)]
    L.nitro_glu_forward.argtypes = [_VP, _VP, _I, _L, _VP, _L, _I, _F, _I, _VP, _L, _VP, _VP]
    L.nitro_glu_backward.argtypes = [_VP, _VP, _I, _L, _VP, _L, _I, _F, _I, _VP, _VP, _L, _VP, _L, _VP, _L, _VP]
    L.nitro_clip_create.argtypes = [ctypes.POINTER(nitro_clip_matrix), _I, ctypes.POINTER(_VP)]
    L.nitro_clip_run.argtypes = [_VP, _F, _VP, _VP]
    for op in ("xent", "orth", "mx4", "gnorm", "glu", "clip"):
        getattr(L, "nitro_%s_status" % op).argtypes = [_VP, _I]
        getattr(L, "nitro_%s_status" % op).restype = _I
        getattr(L, "nitro_%s_create" % op).restype = _I
        getattr(L, "nitro_%s_destroy" % op).argtypes = [_VP]
        getattr(L, "nitro_%s_destroy" % op).restype = None
    for name in ("nitro_xent_forward", "nitro_xent_backward", "nitro_orth_run", "nitro_mx4_bytes",
                 "nitro_mx4_quantize", "nitro_mx4_dequantize", "nitro_mx4_linear",
                 "nitro_gnorm_forward", "nitro_gnorm_backward", "nitro_glu_forward", "nitro_glu_backward", "nitro_clip_run",
                 "nitro_conv3x3_create", "nitro_conv3x3_contract", "nitro_conv3x3_status",
                 "nitro_gemm_create", "nitro_gemm_run", "nitro_gemm_status",
                 "nitro_prep_create", "nitro_prep_fit", "nitro_prep_apply", "nitro_prep_stats"):
        getattr(L, name).restype = ctypes.c_int
    for name in ("nitro_init_block", "nitro_block_forward", "nitro_block_backward",
                 "nitro_block_backward_update", "nitro_integersgd_step", "nitro_block_tensor_bytes", "nitro_block_get_tensor",
                 "nitro_block_set_tensor", "nitro_block_status"):
        getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def status_str(s):
    try:
        return lib().nitro_status_str(int(s)).decode()
    except RuntimeError:
        return "status"


# ---------------------------------------------------------------- C-ABI names
def nitro_init_block(desc, seed, stream=None):
    """Returns (status, handle)."""
    h = _VP()
    st = lib().nitro_init_block(ctypes.byref(desc), int(seed) & (2**64 - 1), stream, ctypes.byref(h))
    return st, h


def nitro_block_forward(blk, a_in, batch, a_out, stream=None):
    return lib().nitro_block_forward(blk, a_in, int(batch), a_out, stream)


def nitro_block_backward(blk, a_in, labels, batch, loss_dev, stream=None):
    return lib().nitro_block_backward(blk, a_in, labels, int(batch), loss_dev, stream)


def nitro_integersgd_step(blk, stream=None):
    return lib().nitro_integersgd_step(blk, stream)


def nitro_block_backward_update(blk, a_in, labels, batch, loss_dev, stream=None):
    return lib().nitro_block_backward_update(blk, a_in, labels, int(batch), loss_dev, stream)


def nitro_block_tensor_bytes(blk, which, layer=0):
    n = ctypes.c_size_t()
    st = lib().nitro_block_tensor_bytes(blk, int(which), int(layer), ctypes.byref(n))
    return st, n.value


def nitro_block_get_tensor(blk, which, layer, host_ptr, nbytes):
    return lib().nitro_block_get_tensor(blk, int(which), int(layer), host_ptr, int(nbytes))


def nitro_block_set_tensor(blk, which, layer, host_ptr, nbytes):
    return lib().nitro_block_set_tensor(blk, int(which), int(layer), host_ptr, int(nbytes))


def nitro_block_status(blk, clear=False):
    return lib().nitro_block_status(blk, 1 if clear else 0)


def nitro_block_status_bits(blk):
    return lib().nitro_block_status_bits(blk)


def nitro_conv3x3_forward_noalloc(a_in, weights, batch, h, w, cin, cout, pool2x2, alpha_inv,
                                  a_out, region, argmax, stream=None):
    return lib().nitro_conv3x3_forward_noalloc(a_in, weights, int(batch), int(h), int(w), int(cin),
                                               int(cout), int(pool2x2), int(alpha_inv), a_out,
                                               region, argmax, stream)


def nitro_conv3x3_noalloc_status(clear=False):
    return lib().nitro_conv3x3_noalloc_status(1 if clear else 0)


def nitro_destroy_block(blk):
    lib().nitro_destroy_block(blk)


# ---------------------------------------------------------------- helpers
def make_block_desc(layers, in_features, num_classes=10, alpha_inv=10, gamma_inv_lr=512,
                    eta_inv_fw=0, eta_inv_lr=0, sgd_round=NITRO_ROUND_FLOOR, max_batch=1,
                    d_lr=0, dropout_p16=0):
    """Build a ``nitro_block_desc`` from layer tuples (kind, cin, cout, h, w, pool).
    Returns (desc, keepalive) - keep the second value alive while desc is used."""
    arr = (nitro_layer_desc * max(1, len(layers)))()
    for i, l in enumerate(layers):
        arr[i] = nitro_layer_desc(*[int(v) for v in l])
    d = nitro_block_desc(len(layers), arr if layers else None, int(in_features), int(num_classes),
                         int(alpha_inv), int(gamma_inv_lr), int(eta_inv_fw), int(eta_inv_lr),
                         int(sgd_round), int(max_batch), int(d_lr), int(dropout_p16))
    return d, arr


class _DeviceArray:
    """A 1-D device buffer described by __cuda_array_interface__ (so torch can
    view library-owned memory without copying it)."""

    def __init__(self, ptr, n, typestr):
        self.__cuda_array_interface__ = {"shape": (int(n),), "typestr": typestr,
                                         "data": (int(ptr or 0), False), "version": 3,
                                         "strides": None}


_raw_stream = None


def _current_stream():
    """Handle of torch's current stream on the current device.  Building the
    Stream object of torch.cuda.current_stream() takes 3 us, more than the rest of
    a call; the handle itself 0.2 us."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()           # initialises CUDA
        get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        dev = getattr(torch._C, "_cuda_getDevice", None)
        _raw_stream = (lambda: get(dev())) if get and dev else \
            (lambda: torch.cuda.current_stream().cuda_stream)
    return _raw_stream()


def _stream_ptr(stream):
    if stream is None:
        return _VP(_current_stream())
    return _VP(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _ptr(t):
    return None if t is None else _VP(t.data_ptr())


class Block:
    """One local-loss block handle.  Activations / labels / loss are torch CUDA
    tensors (int8 / int32 / int64); calls queue work on the given (or current)
    torch stream."""

    def __init__(self, layers, in_features, seed=0, max_batch=1, stream=None, **hyper):
        self.layers = [tuple(int(v) for v in l) for l in layers]
        self.desc, self._keep = make_block_desc(self.layers, in_features, max_batch=max_batch,
                                                **hyper)
        st, self.h = nitro_init_block(self.desc, seed, _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_init_block")
        self.in_features = int(in_features)
        self.num_classes = self.desc.num_classes
        if self.layers:
            k, cin, cout, h, w, pool = self.layers[-1]
            self.out_features = (h // 2) * (w // 2) * cout if pool else h * w * cout
        else:
            self.out_features = 0

    def forward(self, a_in, a_out=None, stream=None):
        st = nitro_block_forward(self.h, _ptr(a_in), a_in.shape[0], _ptr(a_out), _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_forward")
        return a_out

    def backward(self, a_in, labels, loss=None, stream=None):
        st = nitro_block_backward(self.h, _ptr(a_in), _ptr(labels), labels.shape[0], _ptr(loss),
                                  _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_backward")
        return loss

    def backward_update(self, a_in, labels, loss=None, stream=None):
        """backward() then sgd() in one call, the update fused into the
        tensor-core weight-gradient kernels (same results)."""
        st = nitro_block_backward_update(self.h, _ptr(a_in), _ptr(labels), labels.shape[0],
                                         _ptr(loss), _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_backward_update")
        return loss

    def sgd(self, stream=None):
        st = nitro_integersgd_step(self.h, _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_integersgd_step")

    def set_hyper(self, gamma_inv_lr, eta_inv_fw=0, eta_inv_lr=0):
        st = lib().nitro_block_set_hyper(self.h, int(gamma_inv_lr), int(eta_inv_fw),
                                         int(eta_inv_lr))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_set_hyper")

    def set_dropout(self, dropout_p16):
        st = lib().nitro_block_set_dropout(self.h, int(dropout_p16))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_set_dropout")

    def get(self, which, layer=0, check=True):
        """Host copy of a tensor as a flat numpy array (synchronises)."""
        st, n = nitro_block_tensor_bytes(self.h, which, layer)
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_tensor_bytes")
        dt = np.dtype(TENSOR_DTYPE[which])
        out = np.empty(n // dt.itemsize, dtype=dt)
        st = nitro_block_get_tensor(self.h, which, layer, out.ctypes.data_as(_VP), n)
        if check and st not in (NITRO_OK,):
            raise NitroError(st, "nitro_block_get_tensor")
        return out

    def set(self, which, layer, values):
        dt = np.dtype(TENSOR_DTYPE[which])
        arr = np.ascontiguousarray(values, dtype=dt)
        st = nitro_block_set_tensor(self.h, which, layer, arr.ctypes.data_as(_VP), arr.nbytes)
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_set_tensor")

    def status(self, clear=False):
        return nitro_block_status(self.h, clear)

    def grad_device(self, which, layer=0):
        """The block's int64 weight gradient (NITRO_T_DW / NITRO_T_DWLR) as a
        flat torch CUDA tensor that views the block's own memory (no copy)."""
        import torch
        p, n = _VP(), ctypes.c_size_t()
        st = lib().nitro_block_grad_device(self.h, int(which), int(layer), ctypes.byref(p),
                                           ctypes.byref(n))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_grad_device")
        return torch.as_tensor(_DeviceArray(p.value, n.value // 8, "<i8"), device="cuda")

    def diag_timeout(self, wait_us, stream=None):
        """Queue the bounded-wait failure check (nitro_block_diag_timeout)."""
        st = lib().nitro_block_diag_timeout(self.h, int(wait_us), _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_block_diag_timeout")

    def status_bits(self):
        return nitro_block_status_bits(self.h)

    def close(self):
        if getattr(self, "h", None):
            nitro_destroy_block(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Conv3x3:
    """One 3x3 conv layer's contractions (kernel-level entry points)."""

    def __init__(self, max_batch, h, w, cin, cout):
        self.h = _VP()
        st = lib().nitro_conv3x3_create(int(max_batch), int(h), int(w), int(cin), int(cout),
                                        ctypes.byref(self.h))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_conv3x3_create")

    def contract(self, mode, x, y, out, stream=None):
        st = lib().nitro_conv3x3_contract(self.h, int(mode), _ptr(x), _ptr(y), int(x.shape[0]),
                                          _ptr(out), _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_conv3x3_contract")
        return out

    def status(self):
        return lib().nitro_conv3x3_status(self.h)

    def close(self):
        if getattr(self, "h", None):
            lib().nitro_conv3x3_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class IntGemm:
    """C = A B^T with A int8 [M][K], B int32 [N][K], C int64 (kernel-level)."""

    def __init__(self, max_m, max_n, max_k):
        self.h = _VP()
        st = lib().nitro_gemm_create(int(max_m), int(max_n), int(max_k), ctypes.byref(self.h))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_gemm_create")

    def run(self, a, b, c, stream=None):
        m, k = a.shape
        n = b.shape[0]
        st = lib().nitro_gemm_run(self.h, _ptr(a), _ptr(b), int(m), int(n), int(k), _ptr(c),
                                  _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_gemm_run")
        return c

    def status(self):
        return lib().nitro_gemm_status(self.h)

    def close(self):
        if getattr(self, "h", None):
            lib().nitro_gemm_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class IntPrep:
    """Integer data pre-processing (App. A): fit mu / omega on a uint8 device
    tensor, then map uint8 tensors to int8 x_hat with them."""

    def __init__(self):
        self.h = _VP()
        st = lib().nitro_prep_create(ctypes.byref(self.h))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_prep_create")

    def fit(self, x, stream=None):
        st = lib().nitro_prep_fit(self.h, _ptr(x), int(x.numel()), _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_prep_fit")

    def apply(self, x, out, stream=None):
        if out.numel() != x.numel():
            raise ValueError("out must have as many elements as x")
        st = lib().nitro_prep_apply(self.h, _ptr(x), int(x.numel()), _ptr(out), _stream_ptr(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_prep_apply")
        return out

    def stats(self):
        mu, om = ctypes.c_int64(), ctypes.c_int64()
        st = lib().nitro_prep_stats(self.h, ctypes.byref(mu), ctypes.byref(om))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_prep_stats")
        return mu.value, om.value

    def close(self):
        if getattr(self, "h", None):
            lib().nitro_prep_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------- floating-point head
_codes = {}     # torch dtype -> NITRO_* type (int32 and uint8: codes of this module's own)
_INT32, _UINT8 = -1, -2


def _code(t):
    """The type of a torch tensor as a code; None if the library knows none."""
    c = _codes.get(t.dtype)
    if c is None and not _codes:
        import torch
        _codes.update({torch.bfloat16: NITRO_BF16, torch.int8: NITRO_I8, torch.float32: NITRO_F32,
                       torch.int64: NITRO_I64, torch.int32: _INT32, torch.uint8: _UINT8})
        c = _codes.get(t.dtype)
    return c


def _matrix(t, rows, cols, allowed, what):
    """(address, type, row stride) of a CUDA matrix [rows x cols] whose rows are contiguous."""
    code = _codes.get(t.dtype) if _codes else _code(t)
    if code not in allowed or not t.is_cuda or t.shape != (rows, cols):
        raise ValueError("%s must be a CUDA tensor [%d x %d] of a supported type, not %s %s on %s"
                         % (what, rows, cols, tuple(t.shape), t.dtype, t.device))
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("the rows of %s must be contiguous" % what)
    # the stride of a lone row is never used
    return t.data_ptr(), code, max(ld, cols) if rows <= 1 else ld


def _vector(t, n, code, what):
    if (_codes.get(t.dtype) if _codes else _code(t)) != code or not t.is_cuda or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor of %d values of its type, not %s %s on %s"
                         % (what, n, tuple(t.shape), t.dtype, t.device))
    return t.data_ptr()


def _stream_int(stream):
    """A stream's handle as a number, which ctypes takes for a pointer."""
    if stream is None:
        return _current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_X, _W, _ORTH = (NITRO_BF16, NITRO_I8), (NITRO_BF16,), (NITRO_BF16, NITRO_F32, NITRO_I64)
_MX4 = (NITRO_BF16, NITRO_F32)


class _Handle:
    """A C handle of the operator `_op`: its status, and its end."""
    _op = ""

    def _create(self, *shape):
        self.h = _VP()
        name = "nitro_%s_create" % self._op
        st = getattr(lib(), name)(*[int(v) for v in shape], ctypes.byref(self.h))
        if st != NITRO_OK:
            raise NitroError(st, name)

    def status(self, clear=False):
        return getattr(lib(), "nitro_%s_status" % self._op)(self.h, 1 if clear else 0)

    def close(self):
        if getattr(self, "h", None):
            getattr(lib(), "nitro_%s_destroy" % self._op)(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class SoftmaxXent(_Handle):
    """Softmax cross entropy of a linear head z = scale x W^T over many classes,
    without keeping z.  x: bf16 or int8 [rows x features]; W: bf16 [classes x
    features]; labels int32, -1 leaves a row out."""
    _op = "xent"

    def __init__(self, max_rows, features, classes):
        self.features, self.classes = int(features), int(classes)
        self._create(max_rows, features, classes)

    def _inputs(self, x, w, labels):
        n = x.shape[0]
        xp, xt, ldx = _matrix(x, n, self.features, _X, "x")
        wp, _, ldw = _matrix(w, self.classes, self.features, _W, "w")
        return n, (xp, xt, ldx, wp, ldw, _vector(labels, n, _INT32, "labels"), n)

    def forward(self, x, w, labels, loss, lse, scale=1.0, stream=None):
        """Writes the rows' losses and log-sums (fp32 [rows]); returns loss."""
        n, a = self._inputs(x, w, labels)
        st = lib().nitro_xent_forward(self.h, *a, scale, _vector(loss, n, NITRO_F32, "loss"),
                                      _vector(lse, n, NITRO_F32, "lse"), _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_xent_forward")
        return loss

    def backward(self, x, w, labels, lse, gout=None, dx=None, dw=None, scale=1.0, stream=None):
        """Writes dx [rows x features] and dw [classes x features] (bf16; either may be
        None) from the lse of a forward on the same inputs; gout: the gradient of each
        row's loss (fp32), None for ones."""
        n, a = self._inputs(x, w, labels)
        dxp = dwp = None
        lddx = lddw = self.features
        if dx is not None:
            dxp, _, lddx = _matrix(dx, n, self.features, _W, "dx")
        if dw is not None:
            dwp, _, lddw = _matrix(dw, self.classes, self.features, _W, "dw")
        st = lib().nitro_xent_backward(self.h, *a, scale, _vector(lse, n, NITRO_F32, "lse"),
                                       None if gout is None else _vector(gout, n, NITRO_F32, "gout"),
                                       dxp, lddx, dwp, lddw, _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_xent_backward")
        return dx, dw


class Orthogonalizer(_Handle):
    """Newton-Schulz orthogonalisation of up to max_count matrices [rows x cols]."""
    _op = "orth"

    def __init__(self, max_count, rows, cols):
        self.rows, self.cols = int(rows), int(cols)
        self._create(max_count, rows, cols)

    def run(self, m, out, steps=5, coef=None, stream=None):
        """m: [rows x cols] or [count x rows x cols] in bf16, fp32 or int64; out: bf16 of the
        same shape.  coef: (a, b, c) of the step, None for the default."""
        a, b = (m.unsqueeze(0), out.unsqueeze(0)) if m.dim() == 2 and out.dim() == 2 else (m, out)
        n = a.shape[0]
        if a.dim() != 3 or b.shape != a.shape or a.shape != (n, self.rows, self.cols):
            raise ValueError("m and out must be [count x %d x %d]" % (self.rows, self.cols))
        mt = ot = NITRO_BF16
        ldm = ldo = self.cols
        if n:
            _, mt, ldm = _matrix(a[0], self.rows, self.cols, _ORTH, "m")
            _, ot, ldo = _matrix(b[0], self.rows, self.cols, _W, "out")
        k = None if coef is None else (ctypes.c_float * 3)(*coef)
        st = lib().nitro_orth_run(self.h, a.data_ptr(), mt, ldm, a.stride(0), n, steps, k, b.data_ptr(), ldo,
                                  b.stride(0), _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_orth_run")
        return out


def mx4_bytes(rows, cols):
    """(bytes of codes, bytes of scales) of a 4-bit matrix [rows x cols]: nitro_mx4_bytes."""
    blocks = -(-cols // 32)
    return rows * blocks * 16, -(-rows // 128) * -(-blocks // 4) * 512


def _mx4_buffers(codes, scales, rows, cols):
    nq, ns = mx4_bytes(rows, cols)
    return _vector(codes, nq, _UINT8, "codes"), _vector(scales, ns, _UINT8, "scales")


def mx4_quantize(x, codes, scales, stream=None):
    """x (bf16 or fp32) [rows x cols] as 4-bit codes and block scales (uint8, mx4_bytes)."""
    rows, cols = x.shape
    xp, t, ld = _matrix(x, rows, cols, _MX4, "x")
    q, s = _mx4_buffers(codes, scales, rows, cols)
    st = lib().nitro_mx4_quantize(xp, t, ld, rows, cols, q, s, _stream_int(stream))
    if st != NITRO_OK:
        raise NitroError(st, "nitro_mx4_quantize")
    return codes, scales


def mx4_dequantize(codes, scales, out, scale_values=None, stream=None):
    """The values as out (bf16 or fp32) [rows x cols]; scale_values: fp32 [rows x blocks] or None."""
    rows, cols = out.shape
    op, t, ld = _matrix(out, rows, cols, _MX4, "out")
    q, s = _mx4_buffers(codes, scales, rows, cols)
    sv = None if scale_values is None else _vector(scale_values, rows * -(-cols // 32), NITRO_F32, "scale_values")
    st = lib().nitro_mx4_dequantize(q, s, rows, cols, op, t, ld, sv, _stream_int(stream))
    if st != NITRO_OK:
        raise NitroError(st, "nitro_mx4_dequantize")
    return out


class Mx4Linear(_Handle):
    """y = Q(x) W^T for x [rows x in] (quantised on the way) and 4-bit weights W [out x in]."""
    _op = "mx4"

    def __init__(self, max_rows, in_features, out_features):
        self.in_features, self.out_features = int(in_features), int(out_features)
        self._create(max_rows, in_features, out_features)

    def run(self, x, codes, scales, y, stream=None):
        n = x.shape[0]
        xp, xt, ldx = _matrix(x, n, self.in_features, _MX4, "x")
        yp, yt, ldy = _matrix(y, n, self.out_features, _MX4, "y")
        q, s = _mx4_buffers(codes, scales, self.out_features, self.in_features)
        st = lib().nitro_mx4_linear(self.h, xp, xt, ldx, n, q, s, yp, yt, ldy, _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_mx4_linear")
        return y


def _map(t, shape, allowed, what):
    """(address, type, pixel stride, sample stride) of a CUDA map [samples x pixels x channels] whose channels are
    contiguous."""
    code = _codes.get(t.dtype) if _codes else _code(t)
    if code not in allowed or not t.is_cuda or t.shape != shape:
        raise ValueError("%s must be a CUDA tensor %s of a supported type, not %s %s on %s"
                         % (what, list(shape), tuple(t.shape), t.dtype, t.device))
    n, p, c = shape
    if t.is_contiguous():
        return t.data_ptr(), code, c, p * c
    stride, ld, step = t.stride()
    if step != 1 and c > 1:
        raise ValueError("the channels of %s must be contiguous" % what)
    # the strides of a lone pixel or sample are never used
    if p <= 1:
        ld = c
    return t.data_ptr(), code, ld, stride if n > 1 else p * ld


_GN_X, _GN_Y = (NITRO_I8, NITRO_BF16, NITRO_F32), (NITRO_BF16, NITRO_F32)


class GroupNorm(_Handle):
    """Group norm with an activation (NITRO_ACT_*) on channels-last maps [samples x pixels x channels];
    gamma and beta: fp32 [channels], None for ones and zeros."""
    _op = "gnorm"

    def __init__(self, max_samples, max_pixels, channels, groups):
        self.channels, self.groups = int(channels), int(groups)
        self._create(max_samples, max_pixels, channels, groups)
        self._calls = lib().nitro_gnorm_forward, lib().nitro_gnorm_backward

    def forward(self, x, gamma, beta, y, mean=None, rstd=None, eps=1e-5, act=NITRO_ACT_NONE, stream=None):
        """Writes y (bf16 or fp32) and, if given, mean and rstd (fp32 [samples x groups]); x: int8, bf16 or fp32."""
        n, p = x.shape[:2]
        c, m = self.channels, n * self.groups
        shape = (n, p, c)
        xp, xt, ldx, sx = _map(x, shape, _GN_X, "x")
        yp, yt, ldy, sy = _map(y, shape, _GN_Y, "y")
        st = self._calls[0](self.h, xp, xt, ldx, sx, n, p, None if gamma is None else _vector(gamma, c, NITRO_F32, "gamma"),
                            None if beta is None else _vector(beta, c, NITRO_F32, "beta"), eps, act, yp, yt, ldy, sy,
                            None if mean is None else _vector(mean, m, NITRO_F32, "mean"),
                            None if rstd is None else _vector(rstd, m, NITRO_F32, "rstd"),
                            _current_stream() if stream is None else _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_gnorm_forward")
        return y

    def backward(self, x, gamma, beta, mean, rstd, dy, dx=None, dgamma=None, dbeta=None, act=NITRO_ACT_NONE, stream=None):
        """Writes dx (of dy's type), dgamma and dbeta (fp32 [channels]), each unless None, from mean and rstd of a
        forward on the same inputs."""
        n, p = x.shape[:2]
        c, m = self.channels, n * self.groups
        shape = (n, p, c)
        xp, xt, ldx, sx = _map(x, shape, _GN_X, "x")
        gp, gt, ldg, sg = _map(dy, shape, _GN_Y, "dy")
        dp, _, ldd, sd = (None, gt, ldg, sg) if dx is None else _map(dx, shape, (gt,), "dx")
        st = self._calls[1](self.h, xp, xt, ldx, sx, n, p, None if gamma is None else _vector(gamma, c, NITRO_F32, "gamma"),
                            None if beta is None else _vector(beta, c, NITRO_F32, "beta"),
                            None if mean is None else _vector(mean, m, NITRO_F32, "mean"),
                            None if rstd is None else _vector(rstd, m, NITRO_F32, "rstd"), act, gp, gt, ldg, sg, dp, ldd, sd,
                            None if dgamma is None else _vector(dgamma, c, NITRO_F32, "dgamma"),
                            None if dbeta is None else _vector(dbeta, c, NITRO_F32, "dbeta"),
                            _current_stream() if stream is None else _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_gnorm_backward")
        return dx, dgamma, dbeta


class GatedLinear(_Handle):
    """out = act(a) b of z = [a b] = scale x W^T, W bf16 [2 hidden x features], the gate's rows first; x: bf16 or
    int8 [rows x features]."""
    _op = "glu"

    def __init__(self, max_rows, features, hidden):
        self.features, self.hidden = int(features), int(hidden)
        self._create(max_rows, features, hidden)
        self._calls = lib().nitro_glu_forward, lib().nitro_glu_backward

    def forward(self, x, w, out, saved=None, act=NITRO_ACT_SILU, scale=1.0, stream=None):
        """Writes out (bf16 [rows x hidden]) and, for a backward, z to saved (fp32 [rows x 2 hidden], in an order of the
        library's own)."""
        n, f, hidden = x.shape[0], self.features, self.hidden
        xp, xt, ldx = _matrix(x, n, f, _X, "x")
        wp, _, ldw = _matrix(w, 2 * hidden, f, _W, "w")
        op, _, ldo = _matrix(out, n, hidden, _W, "out")
        st = self._calls[0](self.h, xp, xt, ldx, wp, ldw, n, scale, act, op, ldo,
                            None if saved is None else _vector(saved, 2 * n * hidden, NITRO_F32, "saved"),
                            _current_stream() if stream is None else _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_glu_forward")
        return out

    def backward(self, x, w, saved, dout, dx=None, dw=None, act=NITRO_ACT_SILU, scale=1.0, stream=None):
        """Writes dx [rows x features] and dw [2 hidden x features] (bf16; either may be None) from the
        gradient dout (bf16 [rows x hidden]) and the saved of a forward on the same inputs.  The gradient of z is
        rounded to bf16 on the way (up to 32 rows: kept as two bf16 halves)."""
        n, f, hidden = x.shape[0], self.features, self.hidden
        xp, xt, ldx = _matrix(x, n, f, _X, "x")
        wp, _, ldw = _matrix(w, 2 * hidden, f, _W, "w")
        gp, _, ldg = _matrix(dout, n, hidden, _W, "dout")
        dxp, _, lddx = (None, 0, f) if dx is None else _matrix(dx, n, f, _W, "dx")
        dwp, _, lddw = (None, 0, f) if dw is None else _matrix(dw, 2 * hidden, f, _W, "dw")
        st = self._calls[1](self.h, xp, xt, ldx, wp, ldw, n, scale, act, _vector(saved, 2 * n * hidden, NITRO_F32, "saved"), gp, ldg,
                            dxp, lddx, dwp, lddw, _current_stream() if stream is None else _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_glu_backward")
        return dx, dw


class GradClip(_Handle):
    """The norm over the values of all `grads` (bf16, fp32, or int64 where it is not scaled), and each scaled by
    min(1, max_norm / norm) into its tensor of `outs` (None: not written; grads themselves: in
    place).  Where a value is infinite or NaN, so is the norm, and the outs are the grads as they are.  Tensors are
    contiguous, or matrices with contiguous rows.  The handle keeps them and reads their values at every run."""
    _op = "clip"

    def __init__(self, grads, outs=None):
        grads = list(grads)
        outs = [None] * len(grads) if outs is None else list(outs)
        if len(outs) != len(grads):
            raise ValueError("as many outs as grads")
        self.tensors = grads, outs
        table = (nitro_clip_matrix * max(1, len(grads)))()
        for m, g, o in zip(table, grads, outs):
            code = _code(g)
            if code not in _ORTH or not g.is_cuda:
                raise ValueError("gradients must be CUDA tensors of a supported type, not %s on %s" % (g.dtype, g.device))
            if o is not None and (o.shape != g.shape or o.dtype != g.dtype or not o.is_cuda):
                raise ValueError("an out must be as its gradient, %s %s, not %s %s on %s"
                                 % (tuple(g.shape), g.dtype, tuple(o.shape), o.dtype, o.device))
            both = (g,) if o is None else (g, o)
            if all(t.is_contiguous() for t in both):
                m.rows, m.cols = 1, g.numel()
                m.ld_in = m.ld_out = m.cols
            elif g.dim() == 2:
                m.rows, m.cols = g.shape
                for t in both:
                    if t.stride(1) != 1 and m.cols > 1:
                        raise ValueError("the rows of a matrix must be contiguous")
                m.ld_in, m.ld_out = g.stride(0), both[-1].stride(0)
            else:
                raise ValueError("a gradient must be contiguous, or a matrix with contiguous rows")
            m.in_, m.type = g.data_ptr(), code
            m.out = None if o is None else o.data_ptr()
        self.h = _VP()
        st = lib().nitro_clip_create(table, len(grads), ctypes.byref(self.h))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_clip_create")

    def run(self, norm, max_norm=None, stream=None):
        """Writes the norm (fp32, one value) and with max_norm (above 0) the outs; returns norm."""
        limit = 0.0 if max_norm is None else ctypes.c_float(max_norm).value
        if max_norm is not None and not limit > 0:
            raise ValueError("max_norm must be above 0 (in fp32)")
        st = lib().nitro_clip_run(self.h, limit, _vector(norm, 1, NITRO_F32, "norm"),
                                  _stream_int(stream))
        if st != NITRO_OK:
            raise NitroError(st, "nitro_clip_run")
        return norm
