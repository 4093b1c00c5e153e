"""ctypes binding of ``libquasar.so`` (declared in ``include/quasar.h``).

Functions carry the C names and only marshal arguments: tensors become
device pointers, the clip list becomes a host float array, the stream
becomes its ``cudaStream_t`` handle.  Every step of the reconstruction runs
in the library's CUDA kernels; there is no Python or CPU fallback, and the
module raises at import-time use if the library cannot be loaded.
"""
from __future__ import annotations

import ctypes
import enum
import os
import threading

from . import build as _build

_lib = None
_lock = threading.Lock()


class QuasarStatus(enum.IntEnum):
    OK = 0
    ERR_INVALID_ARG = 1
    ERR_UNSUPPORTED = 2
    ERR_CUDA = 3
    ERR_TIMEOUT = 4


class QuasarError(RuntimeError):
    def __init__(self, status):
        self.status = QuasarStatus(status)
        super().__init__(quasar_status_string(status))


F32, BF16 = 0, 1

# Every function declared in include/quasar.h, with its ctypes prototype.
_P, _I, _I64, _F = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
PROTOTYPES = {
    "quasar_recon_int": (_I, [_P, _P, _I, _P, _F, _I, _I, _P, _I, _I64, _I64, _P, _I, _P, _P, _P,
                              _P, _P]),
    "quasar_recon_nvfp4": (_I, [_P, _P, _I, _P, _F, _P, _I, _I64, _I64, _P, _P, _I, _P, _P, _P,
                                _P, _P]),
    "quasar_recon_int_batch": (_I, [_P, _I, _I, _F, _I, _I, _P, _I, _I, _P]),
    "quasar_recon_int_batch_ex": (_I, [_P, _I, _I, _F, _I, _I, _P, _I, _I, _P, _P]),
    "quasar_adamw_recon_int_batch": (_I, [_P, _I, _I, _F, _F, _F, _F, _F, _I64, _I, _I, _P, _I,
                                          _I, _P, _P]),
    "quasar_recon_nvfp4_batch": (_I, [_P, _I, _I, _F, _P, _I, _I, _P]),
    "quasar_recon_nvfp4_batch_ex": (_I, [_P, _I, _I, _F, _P, _I, _I, _P, _P]),
    "quasar_recon_lut_batch": (_I, [_P, _I, _I, _F, _P, _I, _I, _P, _P]),
    "quasar_adamw_recon_nvfp4_batch": (_I, [_P, _I, _I, _F, _F, _F, _F, _F, _I64, _P, _I, _I, _P,
                                            _P]),
    "quasar_tensor_amax": (_I, [_P, _I64, _P, _P]),
    "quasar_linear": (_I, [_P, _I64, _P, _I64, _P, _I, _P, _I64, _I64, _I64, _I64, _P, _I, _I64,
                           _P, _I64, _P]),
    "quasar_linear_grad_input": (_I, [_P, _I64, _P, _I64, _P, _I64, _I, _P, _I64, _I64, _I64, _I64,
                                      _P, _I, _I64, _P]),
    "quasar_linear_grad_weight": (_I, [_P, _I64, _P, _I64, _I64, _I64, _I64, _P, _I, _I64, _P,
                                       _P]),
    "quasar_activation_grad": (_I, [_P, _I64, _P, _I64, _I, _I64, _I64, _P, _I64, _P]),
    "quasar_top_logits": (_I, [_P, _I, _I64, _I64, _I64, _I, _F, _P, _P, _P, _P]),
    "quasar_distill_top": (_I, [_P, _I, _I64, _I64, _I64, _P, _P, _I, _P, _P, _F, _P, _P, _P, _I64,
                                _P]),
    "quasar_distill_top_backward": (_I, [_P, _I, _I64, _I64, _I64, _P, _P, _I, _P, _P, _P, _F, _P,
                                         _I64, _P]),
    "quasar_embedding": (_I, [_P, _I, _I64, _P, _I, _I64, _I64, _I64, _F, _P, _I64, _P, _I, _I64,
                              _P]),
    "quasar_embedding_backward_workspace": (_I, [_I64, _I64, _P]),
    "quasar_embedding_backward": (_I, [_P, _I, _I64, _P, _I, _I64, _I64, _I64, _F, _P, _I, _I64,
                                       _I, _P, _I64, _P]),
    "quasar_layer_norm": (_I, [_P, _I, _I64, _P, _P, _I64, _I64, _I, _F, _P, _I, _I64, _P, _P]),
    "quasar_layer_norm_backward_workspace": (_I, [_I64, _I64, _P]),
    "quasar_layer_norm_backward": (_I, [_P, _I, _I64, _P, _I, _I64, _P, _P, _I64, _I64, _I, _P,
                                        _I64, _P, _I, _I64, _P, _P, _P, _I64, _P]),
    "quasar_attention": (_I, [_P, _I64, _P, _I64, _P, _I64, _I64, _I64, _I64, _I64, _I64, _P, _P,
                              _I64, _I, _F, _P, _I64, _P, _P]),
    "quasar_attention_backward_workspace": (_I, [_I64, _I64, _P]),
    "quasar_attention_backward": (_I, [_P, _I64, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P, _I64,
                                       _I64, _I64, _I64, _I64, _P, _P, _I64, _I, _F, _P, _I64, _P,
                                       _I64, _P, _I64, _P, _I64, _P]),
    "quasar_get_device_status": (_I, [_P]),
    "quasar_debug_force_timeout": (None, [_I64]),
    "quasar_debug_set_stats": (None, [_P]),
    "quasar_debug_set_hoist": (None, [_I]),
    "quasar_status_string": (ctypes.c_char_p, [_I]),
    "quasar_version": (_I, []),
}


def library_path() -> str:
    return os.environ.get("QUASAR_LIBRARY") or _build.LIB


def load(build_if_missing: bool = True):
    """Load libquasar.so (building it first if asked and needed).  The
    environment variable QUASAR_LIBRARY names another build of the same
    library to load instead (no build step then)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = _build.LIB
        if os.environ.get("QUASAR_LIBRARY"):
            path = os.environ["QUASAR_LIBRARY"]
        elif build_if_missing:
            path = _build.build()
        if not os.path.exists(path):
            raise OSError(f"libquasar.so not found at {path}; run paper_2608_13966_gb300.build")
        lib = ctypes.CDLL(path)
        for name, (res, args) in PROTOTYPES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
        return lib


def _ptr(x):
    """Device pointer of a tensor, an int, or None."""
    if x is None or isinstance(x, int):
        return x
    return x.data_ptr()


def _dtype_code(t, default=F32):
    if t is None:
        return default
    if isinstance(t, int):
        return default
    import torch
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _current_stream():
    """Handle of the current device's current stream."""
    global _current_stream
    import torch
    try:  # without building a Stream object for every call (2.7 us on the GPU's host)
        raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        torch.cuda.init()
        handle = lambda: raw(device())  # noqa: E731
        handle()
    except AttributeError:
        handle = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    _current_stream = handle
    return handle()


def _clip_array(clip):
    arr = (ctypes.c_float * len(clip))(*[float(c) for c in clip])
    return arr, len(clip)


def quasar_recon_int(w, g, v, beta2, bits, group_size, clip, rows, cols, r, codes, a, b,
                     cand_idx=None, stream=None, g_dtype=None, r_dtype=None) -> QuasarStatus:
    lib = load()
    carr, nclip = _clip_array(clip)
    gd = g_dtype if g_dtype is not None else _dtype_code(g)
    rd = r_dtype if r_dtype is not None else _dtype_code(r)
    st = lib.quasar_recon_int(_ptr(w), _ptr(g), gd, _ptr(v), beta2, bits, group_size, carr, nclip,
                              rows, cols, _ptr(r), rd, _ptr(codes), _ptr(a), _ptr(b),
                              _ptr(cand_idx), _stream(stream))
    return QuasarStatus(st)


class QuasarIntTensor(ctypes.Structure):
    """quasar_int_tensor: one tensor's buffers (device pointers) and shape."""
    _fields_ = [("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("r", ctypes.c_void_p), ("codes", ctypes.c_void_p), ("a", ctypes.c_void_p),
                ("b", ctypes.c_void_p), ("cand_idx", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64)]


def int_tensor_array(items):
    """A ctypes array of QuasarIntTensor from dicts with keys w, g, v, r,
    codes, a, b, cand_idx (tensors, pointers or None), rows, cols."""
    arr = (QuasarIntTensor * len(items))()
    for i, d in enumerate(items):
        arr[i] = QuasarIntTensor(_ptr(d["w"]), _ptr(d.get("g")), _ptr(d["v"]), _ptr(d["r"]),
                                 _ptr(d.get("codes")), _ptr(d["a"]), _ptr(d["b"]),
                                 _ptr(d.get("cand_idx")), int(d["rows"]), int(d["cols"]))
    return arr


def quasar_recon_int_batch(tensors, beta2, bits, group_size, clip, g_dtype=BF16, r_dtype=BF16,
                           stream=None) -> QuasarStatus:
    """tensors: a ctypes array from int_tensor_array (or a list of dicts)."""
    lib = load()
    if not isinstance(tensors, ctypes.Array):
        tensors = int_tensor_array(tensors)
    carr, nclip = _clip_array(clip)
    st = lib.quasar_recon_int_batch(ctypes.cast(tensors, ctypes.c_void_p), len(tensors), g_dtype,
                                    beta2, bits, group_size, carr, nclip, r_dtype, _stream(stream))
    return QuasarStatus(st)


# quasar_saliency / quasar_codes_layout
SALIENCY = {"ema": 0, "ema_squared": 1, "uniform": 2}
CODES_U8, CODES_PACKED = 0, 1


class QuasarOptions(ctypes.Structure):
    """quasar_options: variant of the reconstruction (saliency, codes layout,
    integer grid)."""
    _fields_ = [("saliency", ctypes.c_int), ("codes_layout", ctypes.c_int), ("grid", ctypes.c_int)]


def options(saliency="ema", packed_codes=False, symmetric=False):
    """A QuasarOptions; saliency is "ema", "ema_squared", "uniform" or a raw
    integer, packed_codes and symmetric booleans or raw integers (raw values
    pass through unchecked, for the library's own validation)."""
    raw = lambda x: isinstance(x, int) and not isinstance(x, bool)
    sal = SALIENCY[saliency] if isinstance(saliency, str) else int(saliency)
    lay = packed_codes if raw(packed_codes) else (CODES_PACKED if packed_codes else CODES_U8)
    grid = symmetric if raw(symmetric) else (1 if symmetric else 0)
    return QuasarOptions(sal, lay, grid)


def _opt_ptr(opt):
    return None if opt is None else ctypes.cast(ctypes.pointer(opt), ctypes.c_void_p)


def quasar_recon_int_batch_ex(tensors, beta2, bits, group_size, clip, options=None, g_dtype=BF16,
                              r_dtype=BF16, stream=None) -> QuasarStatus:
    """quasar_recon_int_batch with a QuasarOptions (None = defaults)."""
    lib = load()
    if not isinstance(tensors, ctypes.Array):
        tensors = int_tensor_array(tensors)
    carr, nclip = _clip_array(clip)
    st = lib.quasar_recon_int_batch_ex(ctypes.cast(tensors, ctypes.c_void_p), len(tensors), g_dtype,
                                       beta2, bits, group_size, carr, nclip, r_dtype,
                                       _opt_ptr(options), _stream(stream))
    return QuasarStatus(st)


class QuasarAdamwTensor(ctypes.Structure):
    """quasar_adamw_tensor: one tensor's buffers (device pointers) and shape."""
    _fields_ = [("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("r", ctypes.c_void_p), ("codes", ctypes.c_void_p),
                ("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("cand_idx", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


def adamw_tensor_array(items):
    """A ctypes array of QuasarAdamwTensor from dicts with keys w, g, m, v,
    r, codes, a, b, cand_idx (tensors, pointers or None), rows, cols."""
    arr = (QuasarAdamwTensor * len(items))()
    for i, d in enumerate(items):
        arr[i] = QuasarAdamwTensor(_ptr(d["w"]), _ptr(d.get("g")), _ptr(d.get("m")), _ptr(d["v"]),
                                   _ptr(d["r"]), _ptr(d.get("codes")), _ptr(d["a"]), _ptr(d["b"]),
                                   _ptr(d.get("cand_idx")), int(d["rows"]), int(d["cols"]))
    return arr


def quasar_adamw_recon_int_batch(tensors, lr, beta1, beta2, eps, weight_decay, step, bits,
                                 group_size, clip, g_dtype=BF16, r_dtype=BF16, options=None,
                                 stream=None) -> QuasarStatus:
    """tensors: a ctypes array from adamw_tensor_array (or a list of dicts)."""
    lib = load()
    if not isinstance(tensors, ctypes.Array):
        tensors = adamw_tensor_array(tensors)
    carr, nclip = _clip_array(clip)
    st = lib.quasar_adamw_recon_int_batch(ctypes.cast(tensors, ctypes.c_void_p), len(tensors),
                                          g_dtype, lr, beta1, beta2, eps, weight_decay, step,
                                          bits, group_size, carr, nclip, r_dtype,
                                          _opt_ptr(options), _stream(stream))
    return QuasarStatus(st)


class QuasarNvfp4Tensor(ctypes.Structure):
    """quasar_nvfp4_tensor: one tensor's buffers (device pointers) and shape."""
    _fields_ = [("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("tensor_amax", ctypes.c_void_p), ("r", ctypes.c_void_p),
                ("codes", ctypes.c_void_p), ("block_scale", ctypes.c_void_p),
                ("tensor_scale", ctypes.c_void_p), ("cand_idx", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


def nvfp4_tensor_array(items):
    """A ctypes array of QuasarNvfp4Tensor from dicts with keys w, g, v,
    tensor_amax, r, codes, block_scale, tensor_scale, cand_idx, rows, cols."""
    arr = (QuasarNvfp4Tensor * len(items))()
    for i, d in enumerate(items):
        arr[i] = QuasarNvfp4Tensor(_ptr(d["w"]), _ptr(d.get("g")), _ptr(d["v"]),
                                   _ptr(d.get("tensor_amax")), _ptr(d["r"]), _ptr(d.get("codes")),
                                   _ptr(d["block_scale"]), _ptr(d["tensor_scale"]),
                                   _ptr(d.get("cand_idx")), int(d["rows"]), int(d["cols"]))
    return arr


def quasar_recon_nvfp4_batch(tensors, beta2, clip, g_dtype=BF16, r_dtype=BF16,
                             stream=None) -> QuasarStatus:
    """tensors: a ctypes array from nvfp4_tensor_array (or a list of dicts)."""
    lib = load()
    if not isinstance(tensors, ctypes.Array):
        tensors = nvfp4_tensor_array(tensors)
    carr, nclip = _clip_array(clip)
    st = lib.quasar_recon_nvfp4_batch(ctypes.cast(tensors, ctypes.c_void_p), len(tensors), g_dtype,
                                      beta2, carr, nclip, r_dtype, _stream(stream))
    return QuasarStatus(st)


def quasar_recon_nvfp4_batch_ex(tensors, beta2, clip, options=None, g_dtype=BF16, r_dtype=BF16,
                                stream=None) -> QuasarStatus:
    """quasar_recon_nvfp4_batch with a QuasarOptions (None = defaults)."""
    lib = load()
    if not isinstance(tensors, ctypes.Array):
        tensors = nvfp4_tensor_array(tensors)
    carr, nclip = _clip_array(clip)
    st = lib.quasar_recon_nvfp4_batch_ex(ctypes.cast(tensors, ctypes.c_void_p), len(tensors),
                                         g_dtype, beta2, carr, nclip, r_dtype, _opt_ptr(options),
                                         _stream(stream))
    return QuasarStatus(st)


class QuasarAdamwNvfp4Tensor(ctypes.Structure):
    """quasar_adamw_nvfp4_tensor: one tensor's buffers (device pointers) and shape."""
    _fields_ = [("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("r", ctypes.c_void_p), ("codes", ctypes.c_void_p),
                ("block_scale", ctypes.c_void_p), ("tensor_scale", ctypes.c_void_p),
                ("cand_idx", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


def adamw_nvfp4_tensor_array(items):
    """A ctypes array of QuasarAdamwNvfp4Tensor from dicts with keys w, g, m,
    v, r, codes, block_scale, tensor_scale, cand_idx, rows, cols."""
    arr = (QuasarAdamwNvfp4Tensor * len(items))()
    for i, d in enumerate(items):
        arr[i] = QuasarAdamwNvfp4Tensor(
            _ptr(d["w"]), _ptr(d.get("g")), _ptr(d.get("m")), _ptr(d["v"]), _ptr(d["r"]),
            _ptr(d.get("codes")), _ptr(d["block_scale"]), _ptr(d["tensor_scale"]),
            _ptr(d.get("cand_idx")), int(d["rows"]), int(d["cols"]))
    return arr


def quasar_adamw_recon_nvfp4_batch(tensors, lr, beta1, beta2, eps, weight_decay, step, clip,
                                   g_dtype=BF16, r_dtype=BF16, options=None,
                                   stream=None) -> QuasarStatus:
    """tensors: a ctypes array from adamw_nvfp4_tensor_array (or a list of dicts)."""
    lib = load()
    if not isinstance(tensors, ctypes.Array):
        tensors = adamw_nvfp4_tensor_array(tensors)
    carr, nclip = _clip_array(clip)
    st = lib.quasar_adamw_recon_nvfp4_batch(ctypes.cast(tensors, ctypes.c_void_p), len(tensors),
                                            g_dtype, lr, beta1, beta2, eps, weight_decay, step,
                                            carr, nclip, r_dtype, _opt_ptr(options),
                                            _stream(stream))
    return QuasarStatus(st)


class QuasarLutTensor(ctypes.Structure):
    """quasar_lut_tensor: one tensor's buffers (device pointers) and shape."""
    _fields_ = [("w", ctypes.c_void_p), ("g", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("r", ctypes.c_void_p), ("codes", ctypes.c_void_p), ("book", ctypes.c_void_p),
                ("cand_idx", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


def lut_tensor_array(items):
    """A ctypes array of QuasarLutTensor from dicts with keys w, g, v, r,
    codes, book, cand_idx (tensors, pointers or None), rows, cols."""
    arr = (QuasarLutTensor * len(items))()
    for i, d in enumerate(items):
        arr[i] = QuasarLutTensor(_ptr(d["w"]), _ptr(d.get("g")), _ptr(d["v"]), _ptr(d["r"]),
                                 _ptr(d.get("codes")), _ptr(d["book"]), _ptr(d.get("cand_idx")),
                                 int(d["rows"]), int(d["cols"]))
    return arr


def quasar_recon_lut_batch(tensors, beta2, clip, options=None, g_dtype=BF16, r_dtype=BF16,
                           stream=None) -> QuasarStatus:
    """tensors: a ctypes array from lut_tensor_array (or a list of dicts)."""
    lib = load()
    if not isinstance(tensors, ctypes.Array):
        tensors = lut_tensor_array(tensors)
    carr, nclip = _clip_array(clip)
    st = lib.quasar_recon_lut_batch(ctypes.cast(tensors, ctypes.c_void_p), len(tensors), g_dtype,
                                    beta2, carr, nclip, r_dtype, _opt_ptr(options), _stream(stream))
    return QuasarStatus(st)


def quasar_recon_nvfp4(w, g, v, beta2, clip, rows, cols, tensor_amax, r, codes, block_scale,
                       tensor_scale, cand_idx=None, stream=None, g_dtype=None,
                       r_dtype=None) -> QuasarStatus:
    lib = load()
    carr, nclip = _clip_array(clip)
    gd = g_dtype if g_dtype is not None else _dtype_code(g)
    rd = r_dtype if r_dtype is not None else _dtype_code(r)
    st = lib.quasar_recon_nvfp4(_ptr(w), _ptr(g), gd, _ptr(v), beta2, carr, nclip, rows, cols,
                                _ptr(tensor_amax), _ptr(r), rd, _ptr(codes), _ptr(block_scale),
                                _ptr(tensor_scale), _ptr(cand_idx), _stream(stream))
    return QuasarStatus(st)


def quasar_tensor_amax(w, n, amax_out, stream=None) -> QuasarStatus:
    return QuasarStatus(load().quasar_tensor_amax(_ptr(w), n, _ptr(amax_out), _stream(stream)))


# quasar_activation
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


def _act_code(activation):
    """The enumerator of an activation's name (raw integers pass through
    unchecked, for the library's own validation)."""
    return ACTIVATIONS[activation] if isinstance(activation, str) else int(activation)


def _status(st):
    return QuasarStatus(st) if st else QuasarStatus.OK


def quasar_linear(x, ld_x, r, ld_r, bias, activation, residual, ld_residual, tokens, features,
                  inputs, y, y_dtype, ld_y, pre=None, ld_pre=0, stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_linear(
        _ptr(x), ld_x, _ptr(r), ld_r, _ptr(bias), _act_code(activation), _ptr(residual),
        ld_residual, tokens, features, inputs, _ptr(y), y_dtype, ld_y, _ptr(pre), ld_pre,
        _stream(stream)))


def quasar_linear_grad_input(dz, ld_dz, r, ld_r, pre_in, ld_pre_in, activation_in, residual,
                             ld_residual, tokens, features, inputs, dx, dx_dtype, ld_dx,
                             stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_linear_grad_input(
        _ptr(dz), ld_dz, _ptr(r), ld_r, _ptr(pre_in), ld_pre_in, _act_code(activation_in),
        _ptr(residual), ld_residual, tokens, features, inputs, _ptr(dx), dx_dtype, ld_dx,
        _stream(stream)))


def quasar_linear_grad_weight(dz, ld_dz, x, ld_x, tokens, features, inputs, dr, dr_dtype, ld_dr,
                              dbias=None, stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_linear_grad_weight(
        _ptr(dz), ld_dz, _ptr(x), ld_x, tokens, features, inputs, _ptr(dr), dr_dtype, ld_dr,
        _ptr(dbias), _stream(stream)))


def quasar_activation_grad(dy, ld_dy, pre, ld_pre, activation, rows, cols, dz, ld_dz,
                           stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_activation_grad(
        _ptr(dy), ld_dy, _ptr(pre), ld_pre, _act_code(activation), rows, cols, _ptr(dz), ld_dz,
        _stream(stream)))


def quasar_top_logits(logits, dtype, ld, rows, vocab, k, temperature, values, indices, lse=None,
                      stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_top_logits(
        _ptr(logits), dtype, ld, rows, vocab, k, temperature, _ptr(values), _ptr(indices),
        _ptr(lse), _stream(stream)))


def quasar_distill_top(logits, dtype, ld, rows, vocab, indices, values, k, teacher_lse, row_weight,
                       temperature, loss, stats=None, grad=None, ld_grad=0,
                       stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_distill_top(
        _ptr(logits), dtype, ld, rows, vocab, _ptr(indices), _ptr(values), k, _ptr(teacher_lse),
        _ptr(row_weight), temperature, _ptr(loss), _ptr(stats), _ptr(grad), ld_grad,
        _stream(stream)))


def quasar_distill_top_backward(logits, dtype, ld, rows, vocab, indices, values, k, teacher_lse,
                                stats, row_weight, temperature, grad, ld_grad,
                                stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_distill_top_backward(
        _ptr(logits), dtype, ld, rows, vocab, _ptr(indices), _ptr(values), k, _ptr(teacher_lse),
        _ptr(stats), _ptr(row_weight), temperature, _ptr(grad), ld_grad, _stream(stream)))


# quasar_index_type
I32, I64 = 0, 1


def _bytes_of(call, *sizes) -> int:
    """What a workspace call answers."""
    n = ctypes.c_int64()
    st = call(*sizes, ctypes.byref(n))
    if st:
        raise QuasarError(st)
    return n.value


def quasar_embedding(ids, ids_type, tokens, table, table_dtype, ld_table, vocab, width, scale,
                     residual, ld_residual, y, y_dtype, ld_y, stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_embedding(
        _ptr(ids), ids_type, tokens, _ptr(table), table_dtype, ld_table, vocab, width, scale,
        _ptr(residual), ld_residual, _ptr(y), y_dtype, ld_y, _stream(stream)))


def quasar_embedding_backward_workspace(tokens, width) -> int:
    return _bytes_of((_lib or load()).quasar_embedding_backward_workspace, tokens, width)


def quasar_embedding_backward(dy, dy_dtype, ld_dy, ids, ids_type, tokens, vocab, width, scale,
                              dtable, dtable_dtype, ld_dtable, accumulate, workspace,
                              workspace_bytes, stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_embedding_backward(
        _ptr(dy), dy_dtype, ld_dy, _ptr(ids), ids_type, tokens, vocab, width, scale, _ptr(dtable),
        dtable_dtype, ld_dtable, accumulate, _ptr(workspace), workspace_bytes, _stream(stream)))


def quasar_layer_norm(x, x_dtype, ld_x, weight, bias, rows, cols, center, eps, y, y_dtype, ld_y,
                      stats=None, stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_layer_norm(
        _ptr(x), x_dtype, ld_x, _ptr(weight), _ptr(bias), rows, cols, center, eps, _ptr(y), y_dtype,
        ld_y, _ptr(stats), _stream(stream)))


def quasar_layer_norm_backward_workspace(rows, cols) -> int:
    return _bytes_of((_lib or load()).quasar_layer_norm_backward_workspace, rows, cols)


def quasar_layer_norm_backward(dy, dy_dtype, ld_dy, x, x_dtype, ld_x, weight, stats, rows, cols,
                               center, residual, ld_residual, dx, dx_dtype, ld_dx, dweight, dbias,
                               workspace, workspace_bytes, stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_layer_norm_backward(
        _ptr(dy), dy_dtype, ld_dy, _ptr(x), x_dtype, ld_x, _ptr(weight), _ptr(stats), rows, cols,
        center, _ptr(residual), ld_residual, _ptr(dx), dx_dtype, ld_dx, _ptr(dweight), _ptr(dbias),
        _ptr(workspace), workspace_bytes, _stream(stream)))


def quasar_attention(q, ld_q, k, ld_k, v, ld_v, tokens, keys, heads, kv_heads, head_dim, starts,
                     key_starts, sequences, causal, scale, y, ld_y, lse=None,
                     stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_attention(
        _ptr(q), ld_q, _ptr(k), ld_k, _ptr(v), ld_v, tokens, keys, heads, kv_heads, head_dim,
        _ptr(starts), _ptr(key_starts), sequences, causal, scale, _ptr(y), ld_y, _ptr(lse),
        _stream(stream)))


def quasar_attention_backward_workspace(tokens, heads) -> int:
    return _bytes_of((_lib or load()).quasar_attention_backward_workspace, tokens, heads)


def quasar_attention_backward(dy, ld_dy, q, ld_q, k, ld_k, v, ld_v, y, ld_y, lse, tokens, keys, heads,
                              kv_heads, head_dim, starts, key_starts, sequences, causal, scale, dq,
                              ld_dq, dk, ld_dk, dv, ld_dv, workspace, workspace_bytes,
                              stream=None) -> QuasarStatus:
    return _status((_lib or load()).quasar_attention_backward(
        _ptr(dy), ld_dy, _ptr(q), ld_q, _ptr(k), ld_k, _ptr(v), ld_v, _ptr(y), ld_y, _ptr(lse),
        tokens, keys, heads, kv_heads, head_dim, _ptr(starts), _ptr(key_starts), sequences, causal,
        scale, _ptr(dq), ld_dq, _ptr(dk), ld_dk, _ptr(dv), ld_dv, _ptr(workspace), workspace_bytes,
        _stream(stream)))


def quasar_get_device_status(stream=None) -> QuasarStatus:
    return QuasarStatus(load().quasar_get_device_status(_stream(stream)))


def quasar_debug_force_timeout(nanoseconds: int) -> None:
    load().quasar_debug_force_timeout(int(nanoseconds))


def quasar_debug_set_stats(counters) -> None:
    load().quasar_debug_set_stats(_ptr(counters))


def quasar_debug_set_hoist(enable: bool) -> None:
    load().quasar_debug_set_hoist(1 if enable else 0)


def quasar_status_string(status) -> str:
    return load().quasar_status_string(int(status)).decode()


def quasar_version() -> int:
    return int(load().quasar_version())
