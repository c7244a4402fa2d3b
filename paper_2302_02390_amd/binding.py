"""Thin Python binding of the C ABI in ``include/qsdp.h`` (``libqsdp.so``).

Argument marshalling only: torch tensors supply device memory and the current stream; every
step of the computation runs in the HIP kernels. The functions have the names and argument
order of the C entry points. There is no fallback: if the library is not built, importing
the symbols raises.
"""
import ctypes as C
import functools
import os
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqsdp.so")

QSDP_OK, QSDP_EINVAL, QSDP_EALIGN, QSDP_ELAUNCH = 0, -1, -2, -3
QSDP_F32, QSDP_BF16, QSDP_F16 = 0, 1, 2
QSDP_FLAG_GRAD_SHIFT, QSDP_FLAG_NO_SHIFT, QSDP_FLAG_SYMMETRIC, QSDP_FLAG_KEEP_MASTER = 1, 2, 4, 8

# Signature of every export of include/qsdp.h: name -> (result, arguments). vp: pointer (device memory unless the
# header says host), the last vp of an entry point that launches work is the stream.
_u64, _u32, _i32, _f32, _vp = C.c_uint64, C.c_uint32, C.c_int, C.c_float, C.c_void_p
_SIGNATURES = {
    "qsdp_spec_version": (_u32, []),
    "qsdp_codes_bytes": (C.c_size_t, [_u64, _i32, _i32]),
    "qsdp_meta_bytes": (C.c_size_t, [_u64, _i32]),
    "qsdp_status_string": (C.c_char_p, [_i32]),
    "qsdp_quantize_grad": (_i32, [_vp, _u64, _i32, _i32, _u64, _u64, _vp, _vp, _vp]),
    "qsdp_quantize_grad_ex": (_i32, [_vp, _u64, _i32, _i32, _u64, _u64, _u32, _vp, _vp, _vp]),
    "qsdp_quantize_grad_g16": (_i32, [_vp, _i32, _u64, _i32, _i32, _u64, _u64, _u32, _vp, _vp, _vp]),
    "qsdp_quantize_weight": (_i32, [_vp, _u64, _i32, _i32, _f32, _u64, _vp, _vp, _vp, _vp]),
    "qsdp_quantize_weight_ex": (_i32, [_vp, _u64, _i32, _i32, _f32, _u64, _u32, _vp, _vp, _vp, _vp]),
    "qsdp_dequantize": (_i32, [_vp, _vp, _u64, _i32, _i32, _i32, _vp, _vp]),
    "qsdp_fused_step": (_i32, [_vp, _vp, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _vp, _vp, _vp, _vp]),
    "qsdp_fused_step_ex": (_i32,
        [_vp, _vp, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _u32, _vp, _vp, _vp, _vp]),
    "qsdp_fused_step_g16": (_i32,
        [_vp, _vp, _i32, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _u32, _vp, _vp, _vp, _vp]),
    "qsdp_fused_step_mp": (_i32,
        [_vp, _vp, _i32, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _u32, _vp, _vp, _vp, _i32, _vp, _vp]),
    "qsdp_fused_step_dseed": (_i32,
        [_vp, _vp, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _vp, _u64, _u32, _vp, _vp, _vp, _vp]),
    "qsdp_fused_step_opts": (_i32, [_vp, _vp, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _vp, _vp]),
    "qsdp_fused_adamw_step_opts": (_i32, [_vp, _vp, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _vp, _vp]),
    "qsdp_fused_step_codes": (_i32, [_vp, _vp, _vp, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _u32, _vp, _vp]),
    "qsdp_fused_adamw_step": (_i32,
        [_vp, _vp, _vp, _vp, _u64, _f32, _f32, _f32, _f32, _f32, _f32, _f32, _i32, _i32, _i32, _f32, _u64,
         _u64, _u32, _vp, _vp, _vp, _vp]),
    "qsdp_fused_adamw_step_mp": (_i32,
        [_vp, _vp, _i32, _vp, _vp, _u64, _f32, _f32, _f32, _f32, _f32, _f32, _f32, _i32, _i32, _i32, _f32, _u64,
         _u64, _u32, _vp, _vp, _vp, _i32, _vp, _vp]),
    "qsdp_fused_adamw_step_codes": (_i32,
        [_vp, _vp, _vp, _vp, _vp, _u64, _f32, _f32, _f32, _f32, _f32, _f32, _f32, _i32, _i32, _i32, _f32,
         _u64, _u64, _u32, _vp, _vp]),
    "qsdp_dequantize_add": (_i32, [_vp, _u64, _vp, _u64, _i32, _u64, _i32, _i32, _f32, _vp, _vp]),
    "qsdp_dequantize_gathered": (_i32, [_vp, _u64, _vp, _u64, _i32, _u64, _u64, _i32, _i32, _i32, _vp, _vp]),
    "qsdp_recv_step": (_i32,
        [_vp, _vp, _u64, _vp, _u64, _i32, _u64, _f32, _f32, _i32, _i32, _i32, _f32, _u64, _u32, _vp, _vp,
         _vp, _vp]),
    "qsdp_recv_adamw_step": (_i32,
        [_vp, _vp, _vp, _vp, _u64, _vp, _u64, _i32, _u64, _f32, _f32, _f32, _f32, _f32, _f32, _f32, _f32,
         _i32, _i32, _i32, _f32, _u64, _u32, _vp, _vp, _vp, _vp]),
    "qsdp_levels_uniform": (_i32, [_i32, _vp]),
    "qsdp_quantize_levels": (_i32, [_vp, _u64, _i32, _i32, _vp, _vp, _vp, _vp]),
    "qsdp_quantize_levels_stochastic": (_i32, [_vp, _u64, _i32, _i32, _vp, _u64, _u64, _vp, _vp, _vp]),
    "qsdp_dequantize_levels": (_i32, [_vp, _vp, _u64, _i32, _i32, _vp, _i32, _vp, _vp]),
    "qsdp_dequantize_levels_gathered": (_i32,
        [_vp, _u64, _vp, _u64, _i32, _u64, _u64, _i32, _i32, _vp, _i32, _vp, _vp]),
    "qsdp_fit_levels": (_i32, [_vp, _u64, _i32, _i32, _f32, _u64, _vp, _vp]),
    "qsdp_segments_build": (_u64, [_vp, _u32, _i32, _vp]),
    "qsdp_quantize_grad_segmented": (_i32, [_vp, _vp, _u32, _u64, _i32, _i32, _u64, _u64, _vp, _vp, _vp]),
    "qsdp_quantize_weight_segmented": (_i32, [_vp, _vp, _u32, _u64, _i32, _i32, _f32, _u64, _vp, _vp, _vp, _vp]),
    "qsdp_fused_step_segmented": (_i32,
        [_vp, _vp, _vp, _u32, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _vp, _vp, _vp, _vp]),
    "qsdp_fused_step_segmented_mp": (_i32,
        [_vp, _vp, _i32, _vp, _u32, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _u32, _vp, _vp, _vp, _i32,
         _vp, _vp]),
    "qsdp_dequantize_segmented": (_i32, [_vp, _vp, _vp, _u32, _u64, _i32, _i32, _i32, _vp, _vp]),
    "qsdp_fused_adamw_step_segmented": (_i32,
        [_vp, _vp, _vp, _vp, _vp, _u32, _u64, _f32, _f32, _f32, _f32, _f32, _f32, _f32, _i32, _i32, _i32,
         _f32, _u64, _u64, _u32, _vp, _vp, _vp, _vp]),
    "qsdp_fused_step_codes_segmented": (_i32,
        [_vp, _vp, _vp, _vp, _u32, _u64, _f32, _i32, _i32, _i32, _f32, _u64, _u64, _u32, _vp, _vp]),
    "qsdp_recv_step_segmented": (_i32,
        [_vp, _vp, _u32, _u64, _vp, _u64, _vp, _u64, _i32, _f32, _f32, _i32, _i32, _i32, _f32, _u64, _u32,
         _vp, _vp, _vp, _vp]),
    "qsdp_recv_adamw_step_segmented": (_i32,
        [_vp, _vp, _vp, _vp, _u32, _u64, _vp, _u64, _vp, _u64, _i32, _f32, _f32, _f32, _f32, _f32, _f32,
         _f32, _f32, _i32, _i32, _i32, _f32, _u64, _u32, _vp, _vp, _vp, _vp]),
    "qsdp_fit_levels_segmented": (_i32, [_vp, _vp, _u32, _i32, _i32, _f32, _u64, _vp, _vp]),
    "qsdp_quantize_levels_segmented": (_i32,
        [_vp, _vp, _u32, _u64, _i32, _i32, _vp, _i32, _u64, _u64, _vp, _vp, _vp]),
    "qsdp_dequantize_levels_segmented": (_i32, [_vp, _vp, _vp, _u32, _u64, _i32, _i32, _vp, _i32, _vp, _vp]),
    "qsdp_token_logprobs_bytes": (C.c_size_t, [_u64, _u64, _i32]),
    "qsdp_token_logprobs": (_i32,
        [_vp, _i32, _u64, _u64, _u64, _vp, _f32, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _u64, _vp]),
    "qsdp_token_logprobs_backward": (_i32,
        [_vp, _i32, _u64, _u64, _u64, _vp, _f32, _vp, _vp, _vp, _vp, _vp, _u64, _vp]),
    "qsdp_distill_loss": (_i32,
        [_vp, _i32, _u64, _u64, _u64, _vp, _vp, _i32, _vp, _f32, _f32, _vp, _vp, _vp, _vp, _u64, _vp]),
    "qsdp_distill_loss_backward": (_i32,
        [_vp, _i32, _u64, _u64, _u64, _vp, _vp, _i32, _vp, _f32, _f32, _vp, _vp, _vp, _u64, _vp]),
    "qsdp_tokens_bytes": (C.c_size_t, [_u64, _u64, _i32]),
    "qsdp_quantize_tokens": (_i32, [_vp, _i32, _u64, _u64, _u64, _i32, _vp, _vp, _vp, _vp]),
    "qsdp_matmul_codes": (_i32, [_vp, _vp, _vp, _u64, _vp, _vp, _u64, _u64, _i32, _vp, _i32, _vp, _u64, _vp]),
    "qsdp_linear_codes": (_i32,
        [_vp, _i32, _u64, _u64, _u64, _vp, _vp, _u64, _i32, _vp, _i32, _vp, _u64, _vp, _u64, _vp]),
    "qsdp_layer_norm": (_i32, [_vp, _i32, _u64, _u64, _u64, _vp, _vp, _i32, _f32, _vp, _i32, _u64, _vp, _vp]),
    "qsdp_layer_norm_backward_bytes": (C.c_size_t, [_u64, _u64]),
    "qsdp_layer_norm_backward": (_i32,
        [_vp, _i32, _u64, _u64, _u64, _vp, _i32, _vp, _vp, _i32, _u64, _vp, _u64, _vp, _vp, _i32, _vp, _u64, _vp]),
    "qsdp_quantize_blocks": (_i32, [_vp, _i32, _u64, _u64, _u64, _i32, _vp, _vp, _vp, _vp, _vp]),
    "qsdp_matmul_blocks_bytes": (C.c_size_t, [_u64, _u64, _u64]),
    "qsdp_matmul_blocks": (_i32,
        [_vp, _vp, _u64, _vp, _vp, _i32, _u64, _u64, _vp, _i32, _vp, _u64, _i32, _vp, _u64, _vp]),
    "qsdp_linear_blocks_bytes": (C.c_size_t, [_u64, _u64, _u64]),
    "qsdp_linear_blocks": (_i32,
        [_vp, _i32, _u64, _u64, _u64, _vp, _vp, _u64, _vp, _i32, _vp, _u64, _vp, _u64, _vp]),
    "qsdp_adamw_build": (_u64, [_vp, _u32]),
    "qsdp_adamw_tensors": (_i32,
        [_vp, _u32, _u64, _f32, _f32, _f32, _f32, _f32, _f32, _u64, _vp, _vp, _vp, _vp]),
}
EXPORTS = tuple(_SIGNATURES)
# Where the entry points take pointers, the stream left out.
_POINTERS = {name: tuple(i for i, kind in enumerate(kinds[:-1]) if kind is _vp)
             for name, (_, kinds) in _SIGNATURES.items()}

_lib = None
_lib_lock = threading.Lock()
# The functions of this file that lib() replaces by native ones of the same name, where these are built for the running
# torch. The native ones call them for the uncommon cases.
_IN_PYTHON = dict.fromkeys(("_is", "_is_rows", "_packed_ok", "_rows_ok", "_step_outputs", "_launch", "_devices_ok"))


class QsdpError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


def lib():
    """Load libqsdp.so (built by ``python -m paper_2302_02390_amd.build``)."""
    global _lib
    if _lib is None:
        with _lib_lock:
            if _lib is None:
                _lib = _load()
    return _lib


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2302_02390_amd.build`")
    L = C.CDLL(LIB_PATH)
    for name, (restype, argtypes) in _SIGNATURES.items():
        fn = getattr(L, name)
        fn.restype = restype
        fn.argtypes = argtypes
    own = globals()
    for name in _IN_PYTHON:
        _IN_PYTHON[name] = own[name]
    native = _native_marshalling()
    if native is not None:
        native.attach(own, *_IN_PYTHON.values())
        for name in _IN_PYTHON:
            own[name] = getattr(native, name[1:])
    return L


def _native_marshalling():
    """The module of csrc/qsdp_marshal.cpp, which takes about 3.5 us of host time off a call, or None if it is not built
    or was compiled against another torch: it reads tensors through torch's C++ headers, and the functions of this file
    do the same without."""
    try:
        from . import _marshal
    except ImportError:
        return None
    built_for = getattr(_marshal, "torch_version", None)
    return _marshal if built_for == f"{torch.__version__} {torch.version.git_version}" else None


def status_string(status):
    return lib().qsdp_status_string(int(status)).decode()


def spec_version():
    return int(lib().qsdp_spec_version())


def codes_bytes(n, bits, bucket):
    return int(lib().qsdp_codes_bytes(int(n), int(bits), int(bucket)))


def meta_bytes(n, bucket):
    return int(lib().qsdp_meta_bytes(int(n), int(bucket)))


def _stream_handle(device):
    return torch.cuda.current_stream(device).cuda_stream


def _check(status, what):
    if status != QSDP_OK:
        raise QsdpError(status, what)


# The handle alone, where torch offers it (a private name): a Stream object costs a small call as much as its kernel.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or _stream_handle


def _launch(t, name, *args):
    """Calls entry point `name` with the current stream of t's device as its last argument, t's device being the
    current one meanwhile; a tensor in the place of a pointer stands for its address. This is the general form; plain
    tensors on the current device go through csrc/qsdp_marshal.cpp."""
    args = list(args)
    for i in _POINTERS[name][:len(args)]:
        a = args[i]
        if a is not None:
            address = getattr(a, "data_ptr", None)
            if address is not None:
                args[i] = address()
    _call(t, name, *args)


def _call(t, name, *args):
    """_launch with addresses in the place of tensors."""
    device = t.get_device()
    stream = _raw_stream(device)
    if device == torch.cuda.current_device():
        status = getattr(_lib or lib(), name)(*args, stream)
    else:
        with torch.cuda.device(device):
            status = getattr(_lib or lib(), name)(*args, stream)
    if status != QSDP_OK:
        raise QsdpError(status, name)


def _is(t, dtype):
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"expected a contiguous {dtype} tensor on the GPU")


_DTYPES = {torch.float32: QSDP_F32, torch.bfloat16: QSDP_BF16, torch.float16: QSDP_F16}


def _out_dtype(out):
    """The decoders' output formats: float32, bfloat16 or float16 (IEEE binary16)."""
    dt = _DTYPES.get(out.dtype)
    if dt is None:
        raise TypeError("out must be float32, bfloat16 or float16")
    return dt


def _is_rows(t, dtype):
    """A 2-D tensor whose rows are contiguous (the rows themselves may be strided apart)."""
    if not (t.is_cuda and t.dtype == dtype and t.dim() == 2 and (t.shape[1] == 1 or t.stride(1) == 1)):
        raise TypeError(f"expected a {dtype} GPU tensor [rows, row length] with contiguous rows")


def _step_outputs(wcodes, wmeta, n_saturated):
    """The optional outputs of a step."""
    for t, dt in ((wcodes, torch.int32), (wmeta, torch.float32), (n_saturated, torch.int64)):
        if t is not None:
            _is(t, dt)


def _need(t, numel, what):
    if t.numel() < numel:
        raise ValueError(f"{what} holds {t.numel()} elements, {numel} are needed")


def _packed_ok(codes, meta, n, bits, bucket):
    """The packed buffers are large enough for n elements (the C ABI takes raw pointers and cannot
    check this itself). Invalid n / bits / bucket are left to the library to report."""
    if codes is None and meta is None:
        return
    cb, mb = codes_bytes(n, bits, bucket), meta_bytes(n, bucket)
    if cb and mb:
        if codes is not None:
            _need(codes, cb // 4, "codes")
        if meta is not None:
            _need(meta, mb // 4, "meta")


def _rows_ok(codes, meta, n, bits, bucket):
    """Every row (peer slot) of the 2-D buffers is large enough for n elements."""
    cb, mb = codes_bytes(n, bits, bucket), meta_bytes(n, bucket)
    if cb and mb:
        if codes.shape[1] < cb // 4:
            raise ValueError(f"code rows hold {codes.shape[1]} words, {cb // 4} are needed")
        if meta.shape[1] < mb // 4:
            raise ValueError(f"meta rows hold {meta.shape[1]} floats, {mb // 4} are needed")


def alloc_packed(n, bits, bucket, device):
    """Empty (codes uint32-as-int32[...], meta float32[nb, 2]) buffers of the right size."""
    cb, mb = codes_bytes(n, bits, bucket), meta_bytes(n, bucket)
    if cb == 0 or mb == 0:
        raise QsdpError(QSDP_EINVAL, "alloc_packed")
    codes = torch.empty(cb // 4, dtype=torch.int32, device=device)
    meta = torch.empty((mb // 8, 2), dtype=torch.float32, device=device)
    return codes, meta


def qsdp_quantize_grad(g, bits, bucket, seed, index_offset, codes, meta):
    _is(g, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    n = g.numel()
    _packed_ok(codes, meta, n, bits, bucket)
    _launch(g, "qsdp_quantize_grad", g, n, bits, bucket, seed, index_offset, codes, meta)


def qsdp_quantize_grad_ex(g, bits, bucket, seed, index_offset, flags, codes, meta):
    _is(g, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    n = g.numel()
    _packed_ok(codes, meta, n, bits, bucket)
    _launch(g, "qsdp_quantize_grad_ex", g, n, bits, bucket, seed, index_offset, flags, codes, meta)


def qsdp_quantize_weight_ex(x, bits, bucket, delta, seed, flags, codes, meta, n_saturated=None):
    _is(x, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    n = x.numel()
    _packed_ok(codes, meta, n, bits, bucket)
    if n_saturated is not None:
        _is(n_saturated, torch.int64)
    _launch(x, "qsdp_quantize_weight_ex", x, n, bits, bucket, delta, seed, flags, codes, meta, n_saturated)


def qsdp_fused_step_ex(x, g, lr, wbits, gbits, bucket, delta, seed, index_offset, flags, wcodes=None,
                       wmeta=None, n_saturated=None):
    _is(x, torch.float32); _is(g, torch.float32)
    n = x.numel()
    if g.numel() != n:
        raise ValueError("x and g differ in size")
    _step_outputs(wcodes, wmeta, n_saturated)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(x, "qsdp_fused_step_ex", x, g, n, lr, wbits, gbits, bucket, delta, seed, index_offset, flags, wcodes, wmeta,
            n_saturated)


def qsdp_quantize_weight(x, bits, bucket, delta, seed, codes, meta, n_saturated=None):
    _is(x, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    n = x.numel()
    _packed_ok(codes, meta, n, bits, bucket)
    if n_saturated is not None:
        _is(n_saturated, torch.int64)
    _launch(x, "qsdp_quantize_weight", x, n, bits, bucket, delta, seed, codes, meta, n_saturated)


def qsdp_dequantize(codes, meta, n, bits, bucket, out):
    _is(codes, torch.int32); _is(meta, torch.float32)
    dt = _out_dtype(out)
    _is(out, out.dtype)
    if out.numel() < n:
        raise ValueError("out is too small")
    _packed_ok(codes, meta, n, bits, bucket)
    _launch(out, "qsdp_dequantize", codes, meta, n, bits, bucket, dt, out)


def levels_uniform(bits, device):
    """The uniform starting table k/(2^bits-1) as a device tensor."""
    import numpy as np
    host = np.zeros(1 << bits, dtype=np.float32)
    _check(lib().qsdp_levels_uniform(bits, host.ctypes.data_as(C.c_void_p)), "qsdp_levels_uniform")
    return torch.from_numpy(host).to(device)


def qsdp_quantize_levels(v, bits, bucket, levels, codes, meta):
    _is(v, torch.float32); _is(levels, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    n = v.numel()
    if levels.numel() != (1 << bits):
        raise ValueError("levels must hold 2^bits entries")
    _packed_ok(codes, meta, n, bits, bucket)
    _launch(v, "qsdp_quantize_levels", v, n, bits, bucket, levels, codes, meta)


def qsdp_quantize_levels_stochastic(v, bits, bucket, levels, seed, index_offset, codes, meta):
    _is(v, torch.float32); _is(levels, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    n = v.numel()
    if levels.numel() != (1 << bits):
        raise ValueError("levels must hold 2^bits entries")
    _packed_ok(codes, meta, n, bits, bucket)
    _launch(v, "qsdp_quantize_levels_stochastic", v, n, bits, bucket, levels, seed, index_offset, codes, meta)


def qsdp_dequantize_levels(codes, meta, n, bits, bucket, levels, out):
    _is(codes, torch.int32); _is(meta, torch.float32); _is(levels, torch.float32)
    if levels.numel() != (1 << bits):
        raise ValueError("levels must hold 2^bits entries")
    dt = _out_dtype(out)
    _is(out, out.dtype)
    if out.numel() < n:
        raise ValueError("out is too small")
    _packed_ok(codes, meta, n, bits, bucket)
    _launch(out, "qsdp_dequantize_levels", codes, meta, n, bits, bucket, levels, dt, out)


def qsdp_fit_levels(v, bits, bucket, lr, levels, max_batches=0):
    _is(v, torch.float32); _is(levels, torch.float32)
    if levels.numel() != (1 << bits):
        raise ValueError("levels must hold 2^bits entries")
    _launch(v, "qsdp_fit_levels", v, v.numel(), bits, bucket, lr, max_batches, levels)


def qsdp_dequantize_add(codes, meta, npeers, n, bits, bucket, alpha, out):
    """codes int32[npeers, words], meta float32[npeers, nb*2] (row p = peer p's slice)."""
    _is(codes, torch.int32); _is(meta, torch.float32); _is(out, torch.float32)
    if codes.dim() != 2 or meta.dim() != 2 or codes.shape[0] != npeers or meta.shape[0] != npeers:
        raise ValueError("codes and meta must be [npeers, ...]")
    if out.numel() < n:
        raise ValueError("out is too small")
    _rows_ok(codes, meta, n, bits, bucket)
    _launch(out, "qsdp_dequantize_add", codes, codes.stride(0) * 4, meta, meta.stride(0) * 4, npeers, n, bits, bucket,
            alpha, out)


def qsdp_fused_step(x, g, lr, wbits, gbits, bucket, delta, seed, index_offset=0, wcodes=None,
                    wmeta=None, n_saturated=None):
    _is(x, torch.float32); _is(g, torch.float32)
    n = x.numel()
    if g.numel() != n:
        raise ValueError("x and g differ in size")
    _step_outputs(wcodes, wmeta, n_saturated)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(x, "qsdp_fused_step", x, g, n, lr, wbits, gbits, bucket, delta, seed, index_offset, wcodes, wmeta,
            n_saturated)


def qsdp_fused_adamw_step(x, g, m, v, lr, beta1, beta2, eps, weight_decay, bias1, bias2, wbits, gbits, bucket,
                          delta, seed, index_offset=0, flags=0, wcodes=None, wmeta=None, n_saturated=None):
    for t in (x, g, m, v):
        _is(t, torch.float32)
    if not (g.numel() == x.numel() == m.numel() == v.numel()):
        raise ValueError("x, g, m, v differ in size")
    _step_outputs(wcodes, wmeta, n_saturated)
    _packed_ok(wcodes, wmeta, x.numel(), wbits, bucket)
    _launch(x, "qsdp_fused_adamw_step", x, g, m, v, x.numel(), lr, beta1, beta2, eps, weight_decay, bias1, bias2, wbits,
            gbits, bucket, delta, seed, index_offset, flags, wcodes, wmeta, n_saturated)


def qsdp_fused_step_codes(wcodes, wmeta, g, lr, wbits, gbits, bucket, delta, seed, index_offset=0,
                          n_saturated=None, flags=0):
    _is(wcodes, torch.int32); _is(wmeta, torch.float32); _is(g, torch.float32)
    n = g.numel()
    if n_saturated is not None:
        _is(n_saturated, torch.int64)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(g, "qsdp_fused_step_codes", wcodes, wmeta, g, n, lr, wbits, gbits, bucket, delta, seed, index_offset, flags,
            n_saturated)


class Segments:
    """Host table built by qsdp_segments_build plus its device copy (an int64 tensor holding the
    {offset, n, first_bucket} triples)."""

    def __init__(self, sizes, bucket, device):
        import numpy as np
        sizes_np = np.ascontiguousarray(sizes, dtype=np.uint64)
        self.nseg = int(sizes_np.size)
        self.bucket = int(bucket)
        self.host = np.zeros((self.nseg, 3), dtype=np.uint64)
        self.total_buckets = int(lib().qsdp_segments_build(
            sizes_np.ctypes.data_as(C.c_void_p), self.nseg, self.bucket, self.host.ctypes.data_as(C.c_void_p)))
        if self.total_buckets == 0:
            raise QsdpError(QSDP_EINVAL, "qsdp_segments_build")
        self.n = int(sizes_np.sum())
        self.device = torch.from_numpy(self.host.view(np.int64).copy()).to(device)

    def check_packed(self, codes, meta, bits, rows=False):
        """codes / meta (or every row of them, for per-peer buffers) cover all buckets of the table."""
        words, floats = self.total_buckets * self.bucket * bits // 32, 2 * self.total_buckets
        for t, need, what in ((codes, words, "codes"), (meta, floats, "meta")):
            if t is None:
                continue
            have = t.shape[1] if rows else t.numel()
            if have < need:
                raise ValueError(f"{what} holds {have} elements{' per row' if rows else ''}, {need} are needed")

    def alloc_packed(self, bits):
        cb = self.total_buckets * self.bucket * bits // 8
        codes = torch.empty(cb // 4, dtype=torch.int32, device=self.device.device)
        meta = torch.empty((self.total_buckets, 2), dtype=torch.float32, device=self.device.device)
        return codes, meta


def qsdp_quantize_grad_segmented(g, segs, bits, seed, index_offset, codes, meta):
    _is(g, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    if g.numel() < segs.n:
        raise ValueError("g is smaller than the segments")
    segs.check_packed(codes, meta, bits)
    _launch(g, "qsdp_quantize_grad_segmented", g, segs.device, segs.nseg, segs.total_buckets, bits, segs.bucket, seed,
            index_offset, codes, meta)


def qsdp_quantize_weight_segmented(x, segs, bits, delta, seed, codes, meta, n_saturated=None):
    _is(x, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    if x.numel() < segs.n:
        raise ValueError("x is smaller than the segments")
    if n_saturated is not None:
        _is(n_saturated, torch.int64)
    segs.check_packed(codes, meta, bits)
    _launch(x, "qsdp_quantize_weight_segmented", x, segs.device, segs.nseg, segs.total_buckets, bits, segs.bucket,
            delta, seed, codes, meta, n_saturated)


def qsdp_fused_step_segmented(x, g, segs, lr, wbits, gbits, delta, seed, index_offset=0, wcodes=None,
                              wmeta=None, n_saturated=None):
    _is(x, torch.float32); _is(g, torch.float32)
    if x.numel() < segs.n or g.numel() < segs.n:
        raise ValueError("x or g is smaller than the segments")
    _step_outputs(wcodes, wmeta, n_saturated)
    segs.check_packed(wcodes, wmeta, wbits)
    _launch(x, "qsdp_fused_step_segmented", x, g, segs.device, segs.nseg, segs.total_buckets, lr, wbits, gbits,
            segs.bucket, delta, seed, index_offset, wcodes, wmeta, n_saturated)


def qsdp_dequantize_segmented(codes, meta, segs, bits, out):
    _is(codes, torch.int32); _is(meta, torch.float32)
    dt = _out_dtype(out)
    _is(out, out.dtype)
    if out.numel() < segs.n:
        raise ValueError("out is smaller than the segments")
    if codes.numel() * 32 < segs.total_buckets * segs.bucket * bits or meta.numel() < 2 * segs.total_buckets:
        raise ValueError("codes or meta is smaller than the segments")
    _launch(out, "qsdp_dequantize_segmented", codes, meta, segs.device, segs.nseg, segs.total_buckets, bits,
            segs.bucket, dt, out)


def qsdp_dequantize_gathered(codes, meta, npeers, n, shard, bits, bucket, out, levels=None):
    """codes int32[npeers, >= words of a shard], meta float32[npeers, >= 2 * buckets of a shard]
    (row p = peer p's slot; rows may be views into one receive buffer); out float32/bfloat16[n].
    levels: the table the slots were encoded with by qsdp_quantize_levels, or None for uniform codes."""
    _is_rows(codes, torch.int32); _is_rows(meta, torch.float32)
    dt = _out_dtype(out)
    _is(out, out.dtype)
    if codes.shape[0] != npeers or meta.shape[0] != npeers:
        raise ValueError("codes and meta must be [npeers, ...]")
    if out.numel() < n:
        raise ValueError("out is too small")
    _rows_ok(codes, meta, min(n, shard) if shard > 0 else n, bits, bucket)
    if levels is not None:
        _is(levels, torch.float32)
        if levels.numel() != (1 << bits):
            raise ValueError("levels must hold 2^bits entries")
        _launch(out, "qsdp_dequantize_levels_gathered", codes, codes.stride(0) * 4, meta, meta.stride(0) * 4, npeers, n,
                shard, bits, bucket, levels, dt, out)
        return
    _launch(out, "qsdp_dequantize_gathered", codes, codes.stride(0) * 4, meta, meta.stride(0) * 4, npeers, n, shard,
            bits, bucket, dt, out)


def qsdp_recv_step(x, gcodes, gmeta, npeers, alpha, lr, wbits, gbits, bucket, delta, seed, flags=0, wcodes=None,
                   wmeta=None, n_saturated=None):
    """gcodes int32[npeers, words], gmeta float32[npeers, nb*2] (row k = peer k's slice)."""
    _is(x, torch.float32); _is_rows(gcodes, torch.int32); _is_rows(gmeta, torch.float32)
    n = x.numel()
    if gcodes.shape[0] != npeers or gmeta.shape[0] != npeers:
        raise ValueError("gcodes and gmeta must be [npeers, ...]")
    _step_outputs(wcodes, wmeta, n_saturated)
    _rows_ok(gcodes, gmeta, n, gbits, bucket)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(x, "qsdp_recv_step", x, gcodes, gcodes.stride(0) * 4, gmeta, gmeta.stride(0) * 4, npeers, n, alpha, lr,
            wbits, gbits, bucket, delta, seed, flags, wcodes, wmeta, n_saturated)


def qsdp_recv_adamw_step(x, m, v, gcodes, gmeta, npeers, alpha, lr, beta1, beta2, eps, weight_decay, bias1, bias2,
                         wbits, gbits, bucket, delta, seed, flags=0, wcodes=None, wmeta=None, n_saturated=None):
    """As qsdp_recv_step with the AdamW update; m, v float32[n] moment estimates, updated in place."""
    for t in (x, m, v):
        _is(t, torch.float32)
    if not (x.numel() == m.numel() == v.numel()):
        raise ValueError("x, m, v differ in size")
    _is_rows(gcodes, torch.int32); _is_rows(gmeta, torch.float32)
    if gcodes.shape[0] != npeers or gmeta.shape[0] != npeers:
        raise ValueError("gcodes and gmeta must be [npeers, ...]")
    _step_outputs(wcodes, wmeta, n_saturated)
    _rows_ok(gcodes, gmeta, x.numel(), gbits, bucket)
    _packed_ok(wcodes, wmeta, x.numel(), wbits, bucket)
    _launch(x, "qsdp_recv_adamw_step", x, m, v, gcodes, gcodes.stride(0) * 4, gmeta, gmeta.stride(0) * 4, npeers,
            x.numel(), alpha, lr, beta1, beta2, eps, weight_decay, bias1, bias2, wbits, gbits, bucket, delta, seed,
            flags, wcodes, wmeta, n_saturated)


def qsdp_recv_step_segmented(x, segs, gcodes, gmeta, npeers, alpha, lr, wbits, gbits, delta, seed, flags=0,
                             wcodes=None, wmeta=None, n_saturated=None, adamw=None):
    """The receive-side step over the tensors of `segs` in one launch. adamw: None, or
    (m, v, beta1, beta2, eps, weight_decay, bias1, bias2) for the AdamW form."""
    _is(x, torch.float32); _is_rows(gcodes, torch.int32); _is_rows(gmeta, torch.float32)
    if x.numel() < segs.n:
        raise ValueError("x is smaller than the segments")
    if gcodes.shape[0] != npeers or gmeta.shape[0] != npeers:
        raise ValueError("gcodes and gmeta must be [npeers, ...]")
    _step_outputs(wcodes, wmeta, n_saturated)
    segs.check_packed(gcodes, gmeta, gbits, rows=True)
    segs.check_packed(wcodes, wmeta, wbits)
    if adamw is None:
        _launch(x, "qsdp_recv_step_segmented", x, segs.device, segs.nseg, segs.total_buckets, gcodes,
                gcodes.stride(0) * 4, gmeta, gmeta.stride(0) * 4, npeers, alpha, lr, wbits, gbits, segs.bucket, delta,
                seed, flags, wcodes, wmeta, n_saturated)
    else:
        m, v, b1, b2, eps, wd, c1, c2 = adamw
        _is(m, torch.float32); _is(v, torch.float32)
        if m.numel() < segs.n or v.numel() < segs.n:
            raise ValueError("m or v is smaller than the segments")
        _launch(x, "qsdp_recv_adamw_step_segmented", x, m, v, segs.device, segs.nseg, segs.total_buckets, gcodes,
                gcodes.stride(0) * 4, gmeta, gmeta.stride(0) * 4, npeers, alpha, lr, b1, b2, eps, wd, c1, c2, wbits,
                gbits, segs.bucket, delta, seed, flags, wcodes, wmeta, n_saturated)


def qsdp_fused_adamw_step_segmented(x, g, m, v, segs, lr, beta1, beta2, eps, weight_decay, bias1, bias2, wbits, gbits,
                                    delta, seed, index_offset=0, flags=0, wcodes=None, wmeta=None, n_saturated=None):
    for t in (x, g, m, v):
        _is(t, torch.float32)
        if t.numel() < segs.n:
            raise ValueError("a tensor is smaller than the segments")
    _step_outputs(wcodes, wmeta, n_saturated)
    segs.check_packed(wcodes, wmeta, wbits)
    _launch(x, "qsdp_fused_adamw_step_segmented", x, g, m, v, segs.device, segs.nseg, segs.total_buckets, lr, beta1,
            beta2, eps, weight_decay, bias1, bias2, wbits, gbits, segs.bucket, delta, seed, index_offset, flags, wcodes,
            wmeta, n_saturated)


def qsdp_fused_step_codes_segmented(wcodes, wmeta, g, segs, lr, wbits, gbits, delta, seed, index_offset=0, flags=0,
                                    n_saturated=None):
    _is(wcodes, torch.int32); _is(wmeta, torch.float32); _is(g, torch.float32)
    if g.numel() < segs.n:
        raise ValueError("g is smaller than the segments")
    if n_saturated is not None:
        _is(n_saturated, torch.int64)
    segs.check_packed(wcodes, wmeta, wbits)
    _launch(g, "qsdp_fused_step_codes_segmented", wcodes, wmeta, g, segs.device, segs.nseg, segs.total_buckets, lr,
            wbits, gbits, segs.bucket, delta, seed, index_offset, flags, n_saturated)


def qsdp_fit_levels_segmented(v, segs, bits, lr, levels, max_batches=0):
    """levels float32[nseg, 2^bits]: row t is the start table of tensor t and receives its fitted levels."""
    _is(v, torch.float32); _is(levels, torch.float32)
    if v.numel() < segs.n:
        raise ValueError("v is smaller than the segments")
    if levels.numel() != segs.nseg * (1 << bits):
        raise ValueError("levels must hold nseg * 2^bits entries")
    _launch(v, "qsdp_fit_levels_segmented", v, segs.device, segs.nseg, bits, segs.bucket, lr, max_batches, levels)


def qsdp_fused_step_dseed(x, g, lr, wbits, gbits, bucket, delta, seed, seed_dev, index_offset=0, flags=0, wcodes=None,
                          wmeta=None, n_saturated=None):
    """qsdp_fused_step_ex with the seed in force = seed + seed_dev[0] (an int64 GPU tensor read by the
    kernel), so that a step captured in a graph can be replayed with an advancing seed."""
    _is(x, torch.float32); _is(g, torch.float32); _is(seed_dev, torch.int64)
    n = x.numel()
    if g.numel() != n:
        raise ValueError("x and g differ in size")
    _step_outputs(wcodes, wmeta, n_saturated)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(x, "qsdp_fused_step_dseed", x, g, n, lr, wbits, gbits, bucket, delta, seed, seed_dev, index_offset, flags,
            wcodes, wmeta, n_saturated)


def qsdp_quantize_levels_segmented(v, segs, bits, levels, codes, meta, stochastic=False, seed=0, index_offset=0):
    """levels float32[nseg, 2^bits]: row t is the level table of tensor t."""
    _is(v, torch.float32); _is(levels, torch.float32); _is(codes, torch.int32); _is(meta, torch.float32)
    if v.numel() < segs.n:
        raise ValueError("v is smaller than the segments")
    if levels.numel() != segs.nseg * (1 << bits):
        raise ValueError("levels must hold nseg * 2^bits entries")
    segs.check_packed(codes, meta, bits)
    _launch(v, "qsdp_quantize_levels_segmented", v, segs.device, segs.nseg, segs.total_buckets, bits, segs.bucket,
            levels, int(bool(stochastic)), seed, index_offset, codes, meta)


def qsdp_dequantize_levels_segmented(codes, meta, segs, bits, levels, out):
    _is(codes, torch.int32); _is(meta, torch.float32); _is(levels, torch.float32)
    dt = _out_dtype(out)
    _is(out, out.dtype)
    if out.numel() < segs.n:
        raise ValueError("out is smaller than the segments")
    if levels.numel() != segs.nseg * (1 << bits):
        raise ValueError("levels must hold nseg * 2^bits entries")
    segs.check_packed(codes, meta, bits)
    _launch(out, "qsdp_dequantize_levels_segmented", codes, meta, segs.device, segs.nseg, segs.total_buckets, bits,
            segs.bucket, levels, dt, out)



_G16 = {torch.bfloat16: 1, torch.float16: 2}


def qsdp_quantize_grad_g16(g, bits, bucket, seed, index_offset, codes, meta, flags=0):
    """qsdp_quantize_grad_ex on a float16 or bfloat16 gradient (widened exactly to float32 inside the kernel)."""
    if g.dtype not in _G16:
        raise TypeError("g must be float16 or bfloat16")
    _is(g, g.dtype); _is(codes, torch.int32); _is(meta, torch.float32)
    n = g.numel()
    _packed_ok(codes, meta, n, bits, bucket)
    _launch(g, "qsdp_quantize_grad_g16", g, _G16[g.dtype], n, bits, bucket, seed, index_offset, flags, codes, meta)


def qsdp_fused_step_g16(x, g, lr, wbits, gbits, bucket, delta, seed, index_offset=0, flags=0, wcodes=None, wmeta=None,
                        n_saturated=None):
    """qsdp_fused_step_ex with a float16 or bfloat16 gradient (widened exactly to float32 inside the kernel)."""
    if g.dtype not in _G16:
        raise TypeError("g must be float16 or bfloat16")
    _is(x, torch.float32); _is(g, g.dtype)
    n = x.numel()
    if g.numel() != n:
        raise ValueError("x and g differ in size")
    _step_outputs(wcodes, wmeta, n_saturated)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(x, "qsdp_fused_step_g16", x, g, _G16[g.dtype], n, lr, wbits, gbits, bucket, delta, seed, index_offset,
            flags, wcodes, wmeta, n_saturated)


def qsdp_fused_adamw_step_codes(wcodes, wmeta, g, m, v, lr, beta1, beta2, eps, weight_decay, bias1, bias2, wbits, gbits,
                                bucket, delta, seed, index_offset=0, flags=0, n_saturated=None):
    """The AdamW step on weights held as packed codes + meta (updated in place); m, v float32, updated in place."""
    _is(wcodes, torch.int32); _is(wmeta, torch.float32); _is(g, torch.float32); _is(m, torch.float32)
    _is(v, torch.float32)
    n = g.numel()
    if m.numel() != n or v.numel() != n:
        raise ValueError("g, m and v differ in size")
    if n_saturated is not None:
        _is(n_saturated, torch.int64)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(g, "qsdp_fused_adamw_step_codes", wcodes, wmeta, g, m, v, n, lr, beta1, beta2, eps, weight_decay, bias1,
            bias2, wbits, gbits, bucket, delta, seed, index_offset, flags, n_saturated)


def qsdp_fused_step_mp(x, g, lr, wbits, gbits, bucket, delta, seed, index_offset=0, flags=0, wcodes=None, wmeta=None,
                       x16=None, n_saturated=None):
    """The fused step with a float32 / float16 / bfloat16 gradient and, optionally, the new quantized weights
    written once more as float16 / bfloat16 into x16."""
    gdt = _DTYPES.get(g.dtype)
    if gdt is None:
        raise TypeError("g must be float32, float16 or bfloat16")
    _is(x, torch.float32); _is(g, g.dtype)
    n = x.numel()
    if g.numel() != n:
        raise ValueError("x and g differ in size")
    xdt = QSDP_BF16
    if x16 is not None:
        if x16.dtype not in _G16:
            raise TypeError("x16 must be float16 or bfloat16")
        _is(x16, x16.dtype)
        _need(x16, n, "x16")
        xdt = _G16[x16.dtype]
    _step_outputs(wcodes, wmeta, n_saturated)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(x, "qsdp_fused_step_mp", x, g, gdt, n, lr, wbits, gbits, bucket, delta, seed, index_offset, flags, wcodes,
            wmeta, x16, xdt, n_saturated)


def qsdp_fused_step_segmented_mp(x, g, segs, lr, wbits, gbits, delta, seed, index_offset=0, flags=0, wcodes=None,
                                 wmeta=None, x16=None, n_saturated=None):
    """qsdp_fused_step_mp over the tensors of a segment table, one launch."""
    gdt = _DTYPES.get(g.dtype)
    if gdt is None:
        raise TypeError("g must be float32, float16 or bfloat16")
    _is(x, torch.float32); _is(g, g.dtype)
    _need(x, segs.n, "x"); _need(g, segs.n, "g")
    xdt = QSDP_BF16
    if x16 is not None:
        if x16.dtype not in _G16:
            raise TypeError("x16 must be float16 or bfloat16")
        _is(x16, x16.dtype)
        _need(x16, segs.n, "x16")
        xdt = _G16[x16.dtype]
    _step_outputs(wcodes, wmeta, n_saturated)
    segs.check_packed(wcodes, wmeta, wbits)
    _launch(x, "qsdp_fused_step_segmented_mp", x, g, gdt, segs.device, segs.nseg, segs.total_buckets, lr, wbits, gbits,
            segs.bucket, delta, seed, index_offset, flags, wcodes, wmeta, x16, xdt, n_saturated)


def qsdp_fused_adamw_step_mp(x, g, m, v, lr, beta1, beta2, eps, weight_decay, bias1, bias2, wbits, gbits, bucket, delta,
                             seed, index_offset=0, flags=0, wcodes=None, wmeta=None, x16=None, n_saturated=None):
    """qsdp_fused_adamw_step with a float32 / float16 / bfloat16 gradient and an optional float16 / bfloat16
    copy x16 of the new quantized weights."""
    gdt = _DTYPES.get(g.dtype)
    if gdt is None:
        raise TypeError("g must be float32, float16 or bfloat16")
    _is(x, torch.float32); _is(g, g.dtype); _is(m, torch.float32); _is(v, torch.float32)
    n = x.numel()
    if g.numel() != n or m.numel() != n or v.numel() != n:
        raise ValueError("x, g, m and v differ in size")
    xdt = QSDP_BF16
    if x16 is not None:
        if x16.dtype not in _G16:
            raise TypeError("x16 must be float16 or bfloat16")
        _is(x16, x16.dtype)
        _need(x16, n, "x16")
        xdt = _G16[x16.dtype]
    _step_outputs(wcodes, wmeta, n_saturated)
    _packed_ok(wcodes, wmeta, n, wbits, bucket)
    _launch(x, "qsdp_fused_adamw_step_mp", x, g, gdt, m, v, n, lr, beta1, beta2, eps, weight_decay, bias1, bias2, wbits,
            gbits, bucket, delta, seed, index_offset, flags, wcodes, wmeta, x16, xdt, n_saturated)


class StepOptions(C.Structure):
    """qsdp_step_options of include/qsdp.h, field for field."""
    _fields_ = [("size", C.c_uint32), ("flags", C.c_uint32), ("g_dtype", C.c_int), ("x16_dtype", C.c_int),
                ("x16", C.c_void_p), ("segments", C.c_void_p), ("nseg", C.c_uint32), ("reserved", C.c_uint32),
                ("total_buckets", C.c_uint64), ("seed_increment", C.c_void_p), ("wcodes", C.c_void_p),
                ("wmeta", C.c_void_p), ("n_saturated", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float), ("weight_decay", C.c_float),
                ("bias1", C.c_float), ("bias2", C.c_float)]


def _step_opts(entry, x, g, lr, wbits, gbits, bucket, delta, seed, index_offset, flags, segs, x16, seed_increment,
               wcodes, wmeta, n_saturated, adamw):
    gdt = _DTYPES.get(g.dtype)
    if gdt is None:
        raise TypeError("g must be float32, float16 or bfloat16")
    _is(x, torch.float32); _is(g, g.dtype)
    n = x.numel() if segs is None else segs.n
    if x.numel() < n or g.numel() < n or (segs is None and g.numel() != n):
        raise ValueError("x and g do not cover the elements of the call")
    o = StepOptions()
    o.size = C.sizeof(StepOptions)
    o.flags = flags
    o.g_dtype = gdt
    if x16 is not None:
        if x16.dtype not in _G16:
            raise TypeError("x16 must be float16 or bfloat16")
        _is(x16, x16.dtype)
        _need(x16, n, "x16")
        o.x16, o.x16_dtype = x16.data_ptr(), _G16[x16.dtype]
    for t, dt in ((wcodes, torch.int32), (wmeta, torch.float32), (n_saturated, torch.int64),
                  (seed_increment, torch.int64)):
        if t is not None:
            _is(t, dt)
    if segs is None:
        _packed_ok(wcodes, wmeta, n, wbits, bucket)
    else:
        if bucket != segs.bucket:
            raise ValueError("bucket differs from the segment table's")
        segs.check_packed(wcodes, wmeta, wbits)
        o.segments, o.nseg, o.total_buckets = segs.device.data_ptr(), segs.nseg, segs.total_buckets
    for name, t in (("wcodes", wcodes), ("wmeta", wmeta), ("n_saturated", n_saturated),
                    ("seed_increment", seed_increment)):
        if t is not None:
            setattr(o, name, t.data_ptr())
    if adamw is not None:
        m, v, o.beta1, o.beta2, o.eps, o.weight_decay, o.bias1, o.bias2 = adamw
        _is(m, torch.float32); _is(v, torch.float32)
        _need(m, n, "m"); _need(v, n, "v")
        o.m, o.v = m.data_ptr(), v.data_ptr()
    _call(x, entry, x.data_ptr(), g.data_ptr(), 0 if segs is not None else n, lr, wbits, gbits, bucket, delta, seed,
          index_offset, C.byref(o))


def qsdp_fused_step_opts(x, g, lr, wbits, gbits, bucket, delta, seed, index_offset=0, flags=0, segs=None, x16=None,
                         seed_increment=None, wcodes=None, wmeta=None, n_saturated=None):
    """The fused step with its optional parts in one options block (qsdp_step_options): gradient in float32 /
    float16 / bfloat16 (taken from g's dtype), a segment table, a 16-bit copy of the new weights, a device-resident
    seed increment, code output, the saturation counter."""
    _step_opts("qsdp_fused_step_opts", x, g, lr, wbits, gbits, bucket, delta, seed, index_offset, flags, segs, x16,
               seed_increment, wcodes, wmeta, n_saturated, None)


def qsdp_fused_adamw_step_opts(x, g, m, v, lr, beta1, beta2, eps, weight_decay, bias1, bias2, wbits, gbits, bucket,
                               delta, seed, index_offset=0, flags=0, segs=None, x16=None, seed_increment=None,
                               wcodes=None, wmeta=None, n_saturated=None):
    """The same with AdamW (moments m, v in float32, updated in place) between the two quantizers."""
    _step_opts("qsdp_fused_adamw_step_opts", x, g, lr, wbits, gbits, bucket, delta, seed, index_offset, flags, segs,
               x16, seed_increment, wcodes, wmeta, n_saturated, (m, v, beta1, beta2, eps, weight_decay, bias1, bias2))


# ---- operators on logits and on packed weights ------------------------------------------------------------------
def _matrix(t):
    """The format and the distance of the rows of a 2-D GPU tensor with contiguous rows in one of the three formats."""
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError("expected float32, bfloat16 or float16")
    _is_rows(t, t.dtype)
    return dt, t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _per_row(rows, dtype, *tensors):
    for t in tensors:
        if t is not None:
            _is(t, dtype)
            if t.numel() != rows:
                raise ValueError(f"{t.numel()} values for {rows} rows")


def _like_logits(logits, d_logits):
    if d_logits.dtype != logits.dtype or d_logits.shape != logits.shape:
        raise ValueError("the gradient has the logits' format and shape")
    return _matrix(d_logits)[1]


def _bytes_of(workspace):
    if workspace is None:
        return 0
    _is(workspace, torch.uint8)
    return workspace.numel()


def token_logprobs_bytes(rows, vocab, top):
    """Bytes of workspace with which qsdp_token_logprobs shares each of few rows among workgroups."""
    return int(lib().qsdp_token_logprobs_bytes(int(rows), int(vocab), int(top)))


def qsdp_token_logprobs(logits, tokens, temperature, logprob, entropy=None, stats=None, top_logprob=None, top_index=None,
                        workspace=None):
    """logits [rows, vocab] in float32, bfloat16 or float16; tokens int64[rows]; logprob, entropy float32[rows]; stats
    float32[rows, 2]; top_logprob float32 and top_index int32 [rows, top]; workspace uint8 or None."""
    dt, stride = _matrix(logits)
    rows, vocab = logits.shape
    _per_row(rows, torch.int64, tokens)
    _per_row(rows, torch.float32, logprob, entropy)
    _per_row(2 * rows, torch.float32, stats)
    top = 0
    if (top_logprob is None) != (top_index is None):
        raise ValueError("top_logprob and top_index come together")
    if top_index is not None:
        _is(top_logprob, torch.float32); _is(top_index, torch.int32)
        if top_index.dim() != 2 or top_index.shape[0] != rows or top_logprob.shape != top_index.shape:
            raise ValueError("top_logprob and top_index must be [rows, top]")
        top = top_index.shape[1]
    _launch(logits, "qsdp_token_logprobs", logits, dt, rows, vocab, stride, tokens, temperature, top, logprob, entropy,
            stats, top_logprob, top_index, workspace, _bytes_of(workspace))


def qsdp_token_logprobs_backward(logits, tokens, temperature, stats, entropy, d_logprob, d_entropy, d_logits):
    """d_logits: as logits, which it may be; d_logprob or d_entropy may be None."""
    dt, stride = _matrix(logits)
    rows, vocab = logits.shape
    _per_row(rows, torch.int64, tokens)
    _per_row(rows, torch.float32, entropy, d_logprob, d_entropy)
    _per_row(2 * rows, torch.float32, stats)
    _launch(logits, "qsdp_token_logprobs_backward", logits, dt, rows, vocab, stride, tokens, temperature, stats, entropy,
            d_logprob, d_entropy, d_logits, _like_logits(logits, d_logits))


def _teacher_list(rows, index, logit):
    if index is None and logit is None:
        return 0
    _is(index, torch.int32); _is(logit, torch.float32)
    if index.dim() != 2 or index.shape[0] != rows or index.shape != logit.shape:
        raise ValueError("teacher_index and teacher_logit must be [rows, top]")
    return index.shape[1]


def qsdp_distill_loss(logits, teacher_index, teacher_logit, labels, temperature, alpha, row_scale, loss, stats=None,
                      d_logits=None):
    """logits [rows, vocab]; teacher_index int32, teacher_logit float32 [rows, top] (None with alpha 0); labels int64[rows]
    (None with alpha 1); row_scale (or None), loss float32[rows]; stats float32[rows, 3]; d_logits: as logits, which it may
    be."""
    dt, stride = _matrix(logits)
    rows, vocab = logits.shape
    top = _teacher_list(rows, teacher_index, teacher_logit)
    _per_row(rows, torch.int64, labels)
    _per_row(rows, torch.float32, row_scale, loss)
    _per_row(3 * rows, torch.float32, stats)
    _launch(logits, "qsdp_distill_loss", logits, dt, rows, vocab, stride, teacher_index, teacher_logit, top, labels,
            temperature, alpha, row_scale, loss, stats, d_logits, 0 if d_logits is None else _like_logits(logits, d_logits))


def qsdp_distill_loss_backward(logits, teacher_index, teacher_logit, labels, temperature, alpha, stats, d_loss, d_logits):
    """The gradient alone, for d_loss float32[rows]; stats as qsdp_distill_loss gave them."""
    dt, stride = _matrix(logits)
    rows, vocab = logits.shape
    top = _teacher_list(rows, teacher_index, teacher_logit)
    _per_row(rows, torch.int64, labels)
    _per_row(rows, torch.float32, d_loss)
    _per_row(3 * rows, torch.float32, stats)
    _launch(logits, "qsdp_distill_loss_backward", logits, dt, rows, vocab, stride, teacher_index, teacher_logit, top, labels,
            temperature, alpha, stats, d_loss, d_logits, _like_logits(logits, d_logits))


def tokens_bytes(m, k, bucket):
    """Bytes of workspace that qsdp_linear_codes needs."""
    return int(lib().qsdp_tokens_bytes(int(m), int(k), int(bucket)))


def _channels_ok(wcodes, wmeta, n, k, bucket, bias):
    """The packed weights hold n channels of whole buckets. An invalid bucket is left to the library to report."""
    _is(wcodes, torch.int32); _is(wmeta, torch.float32)
    if bucket > 0:
        buckets = -(-k // bucket)
        _need(wcodes, -(-n * buckets * bucket // 4), "codes")
        _need(wmeta, 2 * n * buckets, "meta")
    if bias is not None:
        _is(bias, torch.float32)
        if bias.numel() != n:
            raise ValueError(f"{bias.numel()} bias values for {n} channels")


def qsdp_quantize_tokens(x, bucket, codes, scale, sums):
    """x [m, k]; codes int8[m, k rounded up to 128], scale float32[m], sums float32[m, buckets of a channel]."""
    dt, stride = _matrix(x)
    m, k = x.shape
    _is(codes, torch.int8); _is(sums, torch.float32)
    _per_row(m, torch.float32, scale)
    if bucket > 0:
        _need(codes, m * (-(-k // 128) * 128), "codes")
        _need(sums, m * -(-k // bucket), "sums")
    _launch(x, "qsdp_quantize_tokens", x, dt, m, k, stride, bucket, codes, scale, sums)


def qsdp_matmul_codes(codes, scale, sums, wcodes, wmeta, n, k, bucket, bias, y):
    """y [m, n] in any of the three formats, from qsdp_quantize_tokens' outputs and packed 8-bit weights [n, k]."""
    dt, stride = _matrix(y)
    m = y.shape[0]
    _is(codes, torch.int8); _is(sums, torch.float32)
    _per_row(m, torch.float32, scale)
    _channels_ok(wcodes, wmeta, n, k, bucket, bias)
    if bucket > 0:
        _need(codes, m * (-(-k // 128) * 128), "codes")
        _need(sums, m * -(-k // bucket), "sums")
    if y.shape[1] != n:
        raise ValueError(f"y has {y.shape[1]} columns for {n} channels")
    _launch(y, "qsdp_matmul_codes", codes, scale, sums, m, wcodes, wmeta, n, k, bucket, bias, dt, y, stride)


def qsdp_linear_codes(x, wcodes, wmeta, n, bucket, bias, y, workspace=None):
    """y [m, n] = x [m, k] W^T + bias with packed 8-bit weights W [n, k]. Without a workspace (uint8, tokens_bytes) one is
    taken from torch's allocator for the call."""
    dt, stride = _matrix(x)
    out, y_stride = _matrix(y)
    m, k = x.shape
    if y.shape[0] != m or y.shape[1] != n:
        raise ValueError(f"y is {tuple(y.shape)}, not {(m, n)}")
    _channels_ok(wcodes, wmeta, n, k, bucket, bias)
    if workspace is None:
        workspace = torch.empty(tokens_bytes(m, k, bucket), dtype=torch.uint8, device=x.device)
    _launch(x, "qsdp_linear_codes", x, dt, m, k, stride, wcodes, wmeta, n, bucket, bias, out, y, y_stride, workspace,
            _bytes_of(workspace))


# ---- operators of a training step in few bits ---------------------------------------------------------------------
def _parameters(n, like, *tensors):
    """The format that a norm's weight and bias share: float32 or that of `like`."""
    kinds = {t.dtype for t in tensors if t is not None}
    if len(kinds) > 1:
        raise TypeError("weight and bias differ in format")
    dtype = kinds.pop() if kinds else torch.float32
    if dtype not in (torch.float32, like.dtype):
        raise TypeError(f"weight and bias are float32 or {like.dtype}")
    _per_row(n, dtype, *tensors)
    return _DTYPES[dtype]


def _same_shape(x, *tensors):
    for t in tensors:
        if t is not None and t.shape != x.shape:
            raise ValueError(f"{tuple(t.shape)} for rows of {tuple(x.shape)}")


def _norm_formats(x, y):
    if x.dtype != torch.float32 and y.dtype != x.dtype:
        raise TypeError(f"rows in {x.dtype} have outputs in {x.dtype}")


def qsdp_layer_norm(x, weight, bias, eps, y, stats=None):
    """x [rows, n] in float32, bfloat16 or float16; weight, bias [n] (float32 or y's format) or None; y [rows, n] in x's format,
    or any where x is float32; stats float32[rows, 2]."""
    dt, stride = _matrix(x)
    out, y_stride = _matrix(y)
    _same_shape(x, y); _norm_formats(x, y)
    rows, n = x.shape
    wdt = _parameters(n, y, weight, bias)
    _per_row(2 * rows, torch.float32, stats)
    _launch(x, "qsdp_layer_norm", x, dt, rows, n, stride, weight, bias, wdt, eps, y, out, y_stride, stats)


def layer_norm_backward_bytes(rows, n):
    """Bytes of workspace that qsdp_layer_norm_backward needs for the gradients of weight and bias."""
    return int(lib().qsdp_layer_norm_backward_bytes(int(rows), int(n)))


def qsdp_layer_norm_backward(x, weight, stats, dy, dx, dw=None, db=None, accumulate=False, workspace=None):
    """stats as qsdp_layer_norm gave them; dy in y's format; dx (or None) in x's, which may be dy or x where they are alike; dw, db
    float32[n] or None. Without a workspace (uint8, layer_norm_backward_bytes) one is taken from torch's allocator."""
    dt, stride = _matrix(x)
    dy_dt, dy_stride = _matrix(dy)
    _same_shape(x, dy, dx); _norm_formats(x, dy)
    rows, n = x.shape
    dx_stride = 0
    if dx is not None:
        if dx.dtype != x.dtype:
            raise TypeError(f"the gradient of rows in {x.dtype} is {dx.dtype}")
        dx_stride = _matrix(dx)[1]
    wdt = _parameters(n, dy, weight)
    _per_row(2 * rows, torch.float32, stats)
    _per_row(n, torch.float32, dw, db)
    if workspace is None and (dw is not None or db is not None):
        workspace = torch.empty(layer_norm_backward_bytes(rows, n), dtype=torch.uint8, device=x.device)
    _launch(x, "qsdp_layer_norm_backward", x, dt, rows, n, stride, weight, wdt, stats, dy, dy_dt, dy_stride, dx, dx_stride, dw,
            db, int(accumulate), workspace, _bytes_of(workspace))


def _codes8(t, rows, cols, what):
    """e4m3 codes of a matrix, as float8_e4m3fn or uint8: whole blocks of 128 to a row."""
    if t.dtype not in (torch.float8_e4m3fn, torch.uint8):
        raise TypeError(f"{what}: expected float8_e4m3fn or uint8")
    _is(t, t.dtype)
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != -(-cols // 128) * 128:
        raise ValueError(f"{what} is {tuple(t.shape)}, not {(rows, -(-cols // 128) * 128)}")


def _scales8(t, blocks, rows, what):
    _is(t, torch.float32)
    if tuple(t.shape) != (blocks, rows):
        raise ValueError(f"{what} is {tuple(t.shape)}, not {(blocks, rows)}")


def alloc_blocks(rows, cols, square, device):
    """Empty (codes, scales, codes_t, scales_t) of a matrix and its transpose for qsdp_quantize_blocks."""
    r, c = -(-rows // 128), -(-cols // 128)
    codes = torch.empty((rows, 128 * c), dtype=torch.float8_e4m3fn, device=device)
    codes_t = torch.empty((cols, 128 * r), dtype=torch.float8_e4m3fn, device=device)
    return (codes, torch.empty((c, r if square else rows), dtype=torch.float32, device=device),
            codes_t, torch.empty((r, c if square else cols), dtype=torch.float32, device=device))


def qsdp_quantize_blocks(x, square, codes=None, scales=None, codes_t=None, scales_t=None):
    """x [rows, cols] to e4m3 codes (float8_e4m3fn or uint8) with a scale for 128 elements of a row, or for 128 x 128; the
    transposed matrix's as well, in blocks along the columns of x. Shapes as alloc_blocks gives them; either pair may be None."""
    dt, stride = _matrix(x)
    rows, cols = x.shape
    r, c = -(-rows // 128), -(-cols // 128)
    if (codes is None) != (scales is None) or (codes_t is None) != (scales_t is None):
        raise ValueError("codes and scales come together")
    if codes is not None:
        _codes8(codes, rows, cols, "codes")
        _scales8(scales, c, r if square else rows, "scales")
    if codes_t is not None:
        _codes8(codes_t, cols, rows, "codes_t")
        _scales8(scales_t, r, c if square else cols, "scales_t")
    _launch(x, "qsdp_quantize_blocks", x, dt, rows, cols, stride, int(square), codes, scales, codes_t, scales_t)


def _square(b, b_scales, n, k):
    """Whether b [n, k] is in square blocks, by the shape of its scales."""
    _codes8(b, n, k, "codes")
    _is(b_scales, torch.float32)
    blocks = -(-k // 128)
    if tuple(b_scales.shape) == (blocks, -(-n // 128)):
        return 1
    _scales8(b_scales, blocks, n, "scales")
    return 0


def matmul_blocks_bytes(m, n, k):
    """Bytes of workspace with which qsdp_matmul_blocks shares long sums of few tiles among workgroups."""
    return int(lib().qsdp_matmul_blocks_bytes(int(m), int(n), int(k)))


def _bias(bias, n):
    if bias is not None:
        _is(bias, torch.float32)
        if bias.numel() != n:
            raise ValueError(f"{bias.numel()} bias values for {n} columns")


def qsdp_matmul_blocks(a, a_scales, b, b_scales, k, bias, y, accumulate=False, workspace=None):
    """y [m, n] = A B^T (+ bias) (+ y) with A [m, k] in blocks of a row and B [n, k] in square blocks or blocks of a row, codes and
    scales as qsdp_quantize_blocks gives them; y in any of the three formats. workspace: uint8 of matmul_blocks_bytes, or None, which
    is not replaced by one: a call of few tiles and a long sum is then slower (21.8 us for 13.1 at 125 x 2048 x 8192 to bf16) and adds up
    in another order."""
    dt, stride = _matrix(y)
    m, n = y.shape
    _codes8(a, m, k, "codes")
    _scales8(a_scales, -(-k // 128), m, "scales")
    square = _square(b, b_scales, n, k)
    _bias(bias, n)
    _launch(y, "qsdp_matmul_blocks", a, a_scales, m, b, b_scales, square, n, k, bias, dt, y, stride, int(accumulate), workspace,
            _bytes_of(workspace))


def linear_blocks_bytes(m, n, k):
    """Bytes of workspace that qsdp_linear_blocks needs."""
    return int(lib().qsdp_linear_blocks_bytes(int(m), int(n), int(k)))


def qsdp_linear_blocks(x, w, w_scales, bias, y, workspace=None):
    """y [m, n] = x [m, k] W^T + bias, x rounded on the way, W [n, k] in square blocks. Without a workspace (uint8,
    linear_blocks_bytes) one is taken from torch's allocator for the call."""
    dt, stride = _matrix(x)
    out, y_stride = _matrix(y)
    m, k = x.shape
    n = y.shape[1]
    if y.shape[0] != m:
        raise ValueError(f"y is {tuple(y.shape)} for {m} rows")
    _codes8(w, n, k, "codes")
    _scales8(w_scales, -(-k // 128), -(-n // 128), "scales")
    _bias(bias, n)
    if workspace is None:
        workspace = torch.empty(linear_blocks_bytes(m, n, k), dtype=torch.uint8, device=x.device)
    _launch(x, "qsdp_linear_blocks", x, dt, m, k, stride, w, w_scales, n, bias, out, y, y_stride, workspace,
            _bytes_of(workspace))


class AdamWTensor(C.Structure):
    """qsdp_adamw_tensor."""
    _fields_ = [("x", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("scale", C.c_void_p),
                ("x16", C.c_void_p), ("n", _u64), ("first", _u64), ("lr_scale", _f32), ("weight_decay", _f32),
                ("g_dtype", C.c_int32), ("x16_dtype", C.c_int32), ("state_bits", C.c_int32), ("reserved", C.c_int32)]


def alloc_moments(x, bits):
    """(m, v, scale) of a new state for the tensor x: float32 zeros and None, or 8-bit codes and their blocks' scales."""
    n = x.numel()
    if bits == 32:
        return (*(torch.zeros(n, dtype=torch.float32, device=x.device) for _ in range(2)), None)
    if bits != 8:
        raise QsdpError(QSDP_EINVAL, "alloc_moments")
    return (torch.zeros(n, dtype=torch.int8, device=x.device), torch.zeros(n, dtype=torch.uint8, device=x.device),
            torch.zeros(2 * -(-n // 256), dtype=torch.float32, device=x.device))


class AdamWTensors:
    """The table of qsdp_adamw_tensors for lists of tensors, one entry of each per parameter: params float32, grads in any of
    the three formats, moments and scales as alloc_moments gives them (which says how many bits they have), copies bfloat16 or
    float16 or None. weight_decay and lr_scale: a number, or one per parameter. The table holds addresses, and this object the
    tensors: where a gradient becomes another tensor, a new table is needed, which takes the host some 2 us a tensor and a copy to the
    device that it waits for (380 us for 194 short tensors, whose step takes 5): keep the gradients (zero_grad(set_to_none=False)), or copy
    into those of the table. A step writes the parameters, moments, scales and
    copies of its table, none of which may share memory with another."""

    def __init__(self, params, grads, m, v, scales=None, copies=None, weight_decay=0.0, lr_scale=1.0):
        count = len(params)
        each = [list(a) if isinstance(a, (list, tuple)) else [a] * count for a in (scales, copies, weight_decay, lr_scale)]
        lists = [list(params), list(grads), list(m), list(v)] + each
        if count == 0 or any(len(a) != count for a in lists):
            raise ValueError("lists of one entry per parameter are needed")
        table = (AdamWTensor * count)()
        devices = set()
        for t, x, g, m_, v_, scale, copy, decay, rate in zip(table, *lists):
            _is(x, torch.float32)
            gdt = _DTYPES.get(g.dtype)
            if gdt is None:
                raise TypeError("gradients are float32, bfloat16 or float16")
            _is(g, g.dtype)
            n, eight = x.numel(), scale is not None
            _is(m_, torch.int8 if eight else torch.float32)
            _is(v_, torch.uint8 if eight else torch.float32)
            if any(o.numel() != n for o in (g, m_, v_)):
                raise ValueError("a parameter, its gradient and its moments differ in size")
            if eight:
                _is(scale, torch.float32)
                if scale.numel() != 2 * -(-n // 256):
                    raise ValueError(f"{scale.numel()} scales for {n} elements, {2 * -(-n // 256)} are needed")
            if copy is not None:
                if copy.dtype not in _G16:
                    raise TypeError("copies are float16 or bfloat16")
                _is(copy, copy.dtype)
                if copy.numel() != n:
                    raise ValueError("a parameter and its copy differ in size")
                t.x16, t.x16_dtype = copy.data_ptr(), _G16[copy.dtype]
            t.x, t.g, t.m, t.v, t.n = x.data_ptr(), g.data_ptr(), m_.data_ptr(), v_.data_ptr(), n
            t.scale = scale.data_ptr() if eight else None
            t.g_dtype, t.state_bits, t.weight_decay, t.lr_scale = gdt, 8 if eight else 32, decay, rate
            devices.update(o.device for o in (x, g, m_, v_, scale, copy) if o is not None)
        if len(devices) != 1:
            raise ValueError(f"tensors on {sorted(map(str, devices))}")
        self.pieces = int(lib().qsdp_adamw_build(table, count))
        if self.pieces == 0:
            raise QsdpError(QSDP_EINVAL, "qsdp_adamw_build")
        self.count, self.tensors = count, lists[:6]
        self.device = torch.frombuffer(bytearray(table), dtype=torch.uint8).to(devices.pop())


def qsdp_adamw_tensors(table, lr, beta1, beta2, eps, bias1, bias2, seed=0, seed_increment=None, schedule=None,
                       grad_scale=None):
    """One step of every tensor of an AdamWTensors. seed_increment int64[1], schedule float32[3] {lr, bias1, bias2}, grad_scale
    float32[1], all on the GPU, or None."""
    for t, dtype, count in ((seed_increment, torch.int64, 1), (schedule, torch.float32, 3), (grad_scale, torch.float32, 1)):
        if t is not None:
            _is(t, dtype)
            _need(t, count, "a device value")
    _launch(table.device, "qsdp_adamw_tensors", table.device, table.count, table.pieces, lr, beta1, beta2, eps, bias1, bias2,
            seed, seed_increment, schedule, grad_scale)


def _devices_ok(name, args, kwargs):
    """Every tensor argument of an entry point (and a segment table) must live on the same device: the
    kernel runs on the device of the first one and would fault on memory of another."""
    device = None
    for a in list(args) + list(kwargs.values()):
        for t in (a if isinstance(a, (tuple, list)) else (a,)):
            if isinstance(t, (Segments, AdamWTensors)):
                t = t.device
            if isinstance(t, torch.Tensor):
                if device is None:
                    device = t.device
                elif t.device != device:
                    raise ValueError(f"{name}: tensors on {device} and on {t.device}")


def _one_device(fn):
    name = fn.__name__

    @functools.wraps(fn)
    def checked(*args, **kwargs):
        _devices_ok(name, args, kwargs)
        return fn(*args, **kwargs)
    return checked


for _name, _fn in list(globals().items()):
    if _name.startswith("qsdp_") and callable(_fn):
        globals()[_name] = _one_device(_fn)
del _name, _fn
