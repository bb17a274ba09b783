"""The operators that stand beside the sparse product in a layer with compressed weights (include/spmm_layers.h): the
product with 4-bit weights, the root-mean-square norm that makes its operand, and the gated activation between two
products.

Argument marshalling only, as in binding.py: every step runs in the shared library.  Activations are torch device
tensors (features, tokens), as B and C of Plan.execute, with a stride of 1 along either; outputs that are not handed
in are allocated in the order of the input, those in 8 bits with one token a row of memory.  Calls run on torch's
current stream, or on `stream` (as under ``torch.cuda.stream(stream)``: allocations belong to that stream too).  They
give no gradient.
"""
import ctypes
import importlib.util
import os
from collections import namedtuple

import numpy as np

from . import binding
from .binding import SpmmError

LAYERS_EXT_PATH = os.path.join(binding.HERE, "lib", "_spmm_layers.so")
LAYER_EXPORTS = ("spmm_quant_create", "spmm_quant_destroy", "spmm_quant_describe", "spmm_quant_workspace", "spmm_quant_execute",
                 "spmm_norm_workspace", "spmm_norm", "spmm_gate_workspace", "spmm_gate")
ACTS = {"silu": 0, "gelu": 1, "relu": 2}

Normed = namedtuple("Normed", "out total scales")
Gated = namedtuple("Gated", "out scales")

_ext = None
_lib = None


def load():
    """Load the library and the native entries of these operators (raises if they have not been built)."""
    global _ext, _lib
    if _ext is not None:
        return _lib
    lib = binding.load()
    if not os.path.exists(LAYERS_EXT_PATH):
        raise RuntimeError("%s is missing: run `python -m paper_2506_15174_amd.build` (there is no fallback path)" % LAYERS_EXT_PATH)
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    lib.spmm_quant_create.restype = ctypes.c_int
    lib.spmm_quant_create.argtypes = [ctypes.POINTER(vp), i64, i64, i64, vp, vp, vp]
    lib.spmm_quant_destroy.restype = ctypes.c_int
    lib.spmm_quant_destroy.argtypes = [vp]
    lib.spmm_quant_describe.restype = ctypes.c_int
    lib.spmm_quant_describe.argtypes = [vp] + [ctypes.POINTER(i64)] * 4
    spec = importlib.util.spec_from_file_location("_spmm_layers", LAYERS_EXT_PATH)
    ext = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ext)
    ext.answer_types(Normed, Gated)
    _lib, _ext = lib, ext
    return lib


def _on(stream, call, *args):
    import torch
    with torch.cuda.stream(stream):
        return call(*args)


class QuantPlan:
    """Owner of one spmm_quant_t*: a matrix of 4-bit weights on the device that was current when it was made."""

    def __init__(self, handle, M, K, group):
        self._h = handle
        self._address, self._M, self._K, self._group = handle.value, M, K, group

    @property
    def handle(self):
        return self._h

    def describe(self):
        out = [ctypes.c_int64(0) for _ in range(4)]
        binding._check(load().spmm_quant_describe(self._h, *map(ctypes.byref, out)), "spmm_quant_describe")
        return dict(zip(("M", "K", "group", "device_bytes"), (x.value for x in out)))

    def execute(self, B, C=None, scales=None, dtype=None, stream=None):
        """C = W x B (spmm_quant_execute).

        B: (K, N), float32, float16, bfloat16, or int8 codes (one token a row of memory) with `scales`, float32 (N,).
        C: optional output (M, N), float32, float16 or bfloat16; else allocated in `dtype` (B's type; float32 for
        codes) and in B's order.  Returns C.
        """
        if stream is None:
            C = _ext.quant_execute(self._address, self._M, self._K, B, C, scales, dtype)
        else:
            C = _on(stream, _ext.quant_execute, self._address, self._M, self._K, B, C, scales, dtype)
        if type(C) is int:
            raise SpmmError(C, "spmm_quant_execute")
        return C

    def destroy(self):
        if self._h is not None:
            binding._check(load().spmm_quant_destroy(self._h), "spmm_quant_destroy")
            self._h, self._address = None, 0

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _host(array, dtype, shape, name):
    """A C-contiguous host array of the dtype: numpy arrays and torch tensors, the latter also from the device.  Only
    conversions that change no value are made."""
    if hasattr(array, "detach"):
        array = array.detach()
        if not array.dtype.is_floating_point:
            array = array.cpu().numpy()
        elif array.element_size() <= 4:
            array = array.float().cpu().numpy()
        else:
            array = array.cpu().numpy()
    array = np.asarray(array)
    if array.shape != shape:
        raise ValueError("%s has shape %s, not %s" % (name, tuple(array.shape), shape))
    if not np.can_cast(array.dtype, dtype, "safe"):
        raise ValueError("%s is of type %s, not %s" % (name, array.dtype, np.dtype(dtype)))
    return np.ascontiguousarray(array, dtype=dtype)


def quant_plan_create(M, K, codes, scales, zeros=None, group=128):
    """spmm_quant_create: a plan of M x K weights scale * (code - zero).

    codes: uint8 (M, ceil(K / 2)), two codes a byte, the even column's in the low half.  scales: float32, float16 or
    bfloat16 (M, ceil(K / group)).  zeros: uint8 of that shape, 0..15, or None: 8 everywhere.  group: 32, 64 or a
    multiple of 128.  Arrays are numpy's or torch's.
    """
    M, K, group = int(M), int(K), int(group)
    if max(abs(M), abs(K), abs(group)) >= 2 ** 63:   # (they would reach the library cut off, and the arrays no longer be those of its sizes)
        raise ValueError("M, K and group are 64-bit numbers")
    lib = load()
    groups = -(-K // group) if group > 0 else 0
    if M >= 0 and K >= 0:
        codes = _host(codes, np.uint8, (M, (K + 1) // 2), "codes")
        scales = _host(scales, np.float32, (M, groups), "scales")
        zeros = None if zeros is None else _host(zeros, np.uint8, (M, groups), "zeros")
    handle = ctypes.c_void_p()
    ptr = binding._ptr
    binding._check(lib.spmm_quant_create(ctypes.byref(handle), M, K, group, ptr(codes), ptr(scales), ptr(zeros)), "spmm_quant_create")
    return QuantPlan(handle, M, K, group)


def norm(x, weight, eps=1e-6, residual=None, total=None, out=None, scales=None, dtype=None, stream=None):
    """Root-mean-square norm of every token with the residual's addition (spmm_norm): t = x + residual in x's type,
    out = t / sqrt(mean t^2 + eps) * weight.

    x: (K, N), float32, float16 or bfloat16; residual, total: the same, in x's order; weight: (K,).  `total` receives
    t (it may be x or residual itself); it is allocated where there is a residual and no total.  dtype: out's, x's
    type if not given; torch.int8 makes codes with a scale a token.  Returns Normed(out, total, scales), None for what
    there is not.
    """
    if _ext is None:
        load()
    if stream is None:
        res = _ext.norm(x, weight, eps, residual, total, residual is not None, out, scales, dtype)
    else:
        res = _on(stream, _ext.norm, x, weight, eps, residual, total, residual is not None, out, scales, dtype)
    if type(res) is int:
        raise SpmmError(res, "spmm_norm")
    return res


def gate(a, b=None, act="silu", out=None, scales=None, dtype=None, stream=None):
    """Gated activation act(a) * b (spmm_gate); act: "silu", "gelu" (by tanh) or "relu"; without b: act(a).

    a, b: (F, N), float32, float16 or bfloat16, in one order.  dtype as in norm.  Returns Gated(out, scales).
    """
    if act not in ACTS:
        raise ValueError("act must be one of %s" % ", ".join(sorted(ACTS)))
    if _ext is None:
        load()
    if stream is None:
        res = _ext.gate(a, b, ACTS[act], out, scales, dtype)
    else:
        res = _on(stream, _ext.gate, a, b, ACTS[act], out, scales, dtype)
    if type(res) is int:
        raise SpmmError(res, "spmm_gate")
    return res
