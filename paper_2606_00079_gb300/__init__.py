"""Python binding of libbitsmoe, the GB300 BitsMoE quantized MoE-layer forward.

Argument marshalling only: every step of the forward runs in the library's
CUDA kernels.  The functions carry the C ABI's names (see include/bitsmoe.h);
PyTorch is used only for device memory and streams by the convenience wrapper
``moe_forward``.  There is no CPU fallback: if the compiled library is missing
every entry point raises ``BitsMoEUnavailable``.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, NamedTuple, Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbitsmoe.so")

OK = 0
ERR = {
    -1: "INVALID_ARG", -2: "SHAPE", -3: "UNSUPPORTED_BITS", -4: "WORKSPACE_TOO_SMALL",
    -5: "ALIGNMENT", -6: "CUDA", -7: "OOM", -8: "TIMEOUT", -9: "DEVICE_BOUNDS", -10: "BLOB",
    -11: "WORKSPACE_STATE",
}
ERR_CODE = {v: k for k, v in ERR.items()}

# Every C entry point declared in include/bitsmoe.h, with (restype, argtypes).
_P = ctypes.c_void_p
_I = ctypes.c_int
_SZ = ctypes.c_size_t
_addressof = ctypes.addressof


class _LayerHost(ctypes.Structure):
    _fields_ = [("D", ctypes.c_int32), ("E", ctypes.c_int32), ("I", ctypes.c_int32),
                ("n", ctypes.c_int32), ("group", ctypes.c_int32),
                ("basis", _P * 3), ("bits", _P), ("alpha", _P), ("codes", _P),
                ("scale", _P), ("zero", _P)]


class _Bytes(ctypes.Structure):
    _fields_ = [("total", ctypes.c_uint64), ("basis", ctypes.c_uint64),
                ("codes_padded", ctypes.c_uint64), ("meta", ctypes.c_uint64)]


class _Microscale(ctypes.Structure):
    _fields_ = [("format", ctypes.c_int32), ("rows", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("scale", ctypes.c_float), ("codes", _P), ("scales", _P)]


class _BlockNormArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("T", "D", "h_type", "y_type", "gate_type", "gain_type", "x_type",
                                               "post_norm", "gate_kind", "gate_sigmoid")]
                + [(n, ctypes.c_float) for n in ("post_eps", "pre_eps", "gain_offset", "residual_scale",
                                                 "branch_scale")]
                + [(n, _P) for n in ("h", "y", "gate", "post_gain", "pre_gain", "channel_scale", "h_out", "x")]
                + [(n, ctypes.c_int64) for n in ("h_ld", "y_ld", "gate_ld", "h_out_ld", "x_ld")])


class _Rowscale(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("ld", ctypes.c_int64), ("codes", _P),
                ("scales", _P)]


class _ExpertMatrices(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("type", "experts", "rows", "cols")]
                + [(n, ctypes.c_int64) for n in ("ld", "expert_ld", "scale_ld")] + [("data", _P), ("scales", _P)])


class _ExpertProductArgs(ctypes.Structure):
    _fields_ = [("w", _P), ("up", _P), ("x", _P),
                ("x_scales", _P), ("x_ld", ctypes.c_int64), ("x_rows", ctypes.c_int32), ("P", ctypes.c_int32),
                ("offsets", _P), ("index", _P), ("fan", ctypes.c_int32), ("y_type", ctypes.c_int32), ("y", _P),
                ("y_ld", ctypes.c_int64), ("status", _P)]


SIGNATURES = {
    "bitsmoe_pack": (_I, [ctypes.POINTER(_LayerHost), _I, ctypes.POINTER(_P)]),
    "bitsmoe_pack_to_host": (_I, [ctypes.POINTER(_LayerHost), ctypes.POINTER(_P), ctypes.POINTER(_SZ)]),
    "bitsmoe_blob_free": (None, [_P]),
    "bitsmoe_load_blob": (_I, [_P, _SZ, _I, ctypes.POINTER(_P)]),
    "bitsmoe_unpack_blob": (_I, [_P, _SZ, ctypes.POINTER(_LayerHost)]),
    "bitsmoe_unpack": (_I, [_P, ctypes.POINTER(_LayerHost)]),
    "bitsmoe_layer_dims": (_I, [_P, ctypes.POINTER(ctypes.c_int32)]),
    "bitsmoe_layer_bytes": (_I, [_P, ctypes.POINTER(_Bytes)]),
    "bitsmoe_expert_moved_bytes": (_I, [_P, _I, ctypes.POINTER(ctypes.c_uint64)]),
    "bitsmoe_profile_forward": (_I, [_P, _P, _I, _I, _P, _P, _P, _SZ, _P, ctypes.POINTER(ctypes.c_float)]),
    "bitsmoe_workspace_bytes": (_SZ, [_P, _I, _I]),
    "bitsmoe_forward_launches": (_I, [_P, _I, _I]),
    "bitsmoe_block_forward_launches": (_I, [_P, _I, _I]),
    "bitsmoe_forward_plan": (_I, [_P, _I, _I]),
    "bitsmoe_moe_forward": (_I, [_P, _P, _I, _I, _P, _P, _P, _SZ, _P]),
    "bitsmoe_moe_forward_host": (_I, [_P, _P, _I, _I, _P, _P, _P, _SZ, _P]),
    "bitsmoe_moe_forward_host_async": (_I, [_P, _P, _I, _I, _P, _P, _P, _SZ, _P]),
    "bitsmoe_moe_forward_noalloc": (_I, [_P, _P, _I, _I, _P, _P, _P]),
    "bitsmoe_noalloc_last_status": (_I, [_P]),
    "bitsmoe_rmsnorm_router": (_I, [_P, _P, ctypes.c_float, _I, _I, _I, _P, _P, _P]),
    "bitsmoe_moe_block_forward": (_I, [_P, _P, ctypes.c_float, _I, _I, _P, _P, _SZ, _P]),
    "bitsmoe_quantize_units": (_I, [_P, _P, ctypes.c_int64, _I, _I, _I, _P, _P, _P, _P, _P]),
    "bitsmoe_allocate_workspace_bytes": (_SZ, [ctypes.c_int64]),
    "bitsmoe_projection_budget": (_I, [ctypes.c_int64] * 5 + [ctypes.POINTER(ctypes.c_int64)]),
    "bitsmoe_allocate_bits": (_I, [_P, _P, _P, ctypes.c_float, ctypes.c_int64, _I, ctypes.POINTER(ctypes.c_float),
                                   ctypes.c_int64, _P, _P, _SZ, _P]),
    "bitsmoe_profile_allocate_bits": (_I, [_P, _P, _P, ctypes.c_float, ctypes.c_int64, _I,
                                           ctypes.POINTER(ctypes.c_float), ctypes.c_int64, _P, _P, _SZ, _P,
                                           ctypes.POINTER(ctypes.c_float)]),
    "bitsmoe_importance_workspace_bytes": (_SZ, [ctypes.c_int64, _I, _I, _I, _I]),
    "bitsmoe_importance": (_I, [_P, _P, ctypes.c_int64, _I, _I, _I, _I, _I, ctypes.POINTER(_P), ctypes.POINTER(_P),
                                ctypes.POINTER(_P), _P, _P, _SZ, _P]),
    "bitsmoe_decompose_workspace_bytes": (_SZ, [_I, _I, _I, _I]),
    "bitsmoe_shared_basis": (_I, [_I, _P, _I, _I, _I, _P, _P, _P, _P, _P, _SZ, _I, _P, _P, _P]),
    "bitsmoe_calibration_gram": (_I, [_P, _P, ctypes.c_int64, _I, _P, _P]),
    "bitsmoe_microscale_bytes": (_I, [_I, _I, _I, ctypes.POINTER(_SZ), ctypes.POINTER(_SZ)]),
    "bitsmoe_microscale_quantize": (_I, [_P, _I, ctypes.c_int64, ctypes.POINTER(_Microscale), _P]),
    "bitsmoe_microscale_dequantize": (_I, [ctypes.POINTER(_Microscale), _P, _I, ctypes.c_int64, _P]),
    "bitsmoe_microscale_align": (_I, [_P, ctypes.c_int64, _I, _I, _P, ctypes.c_int64, _P]),
    "bitsmoe_microscale_product": (_I, [ctypes.POINTER(_Microscale), ctypes.POINTER(_Microscale), _P, ctypes.c_int64,
                                        ctypes.POINTER(_Microscale), _I, _P, _I, ctypes.c_int64, _P, _P]),
    "bitsmoe_block_norm": (_I, [ctypes.POINTER(_BlockNormArgs), _P]),
    "bitsmoe_rowscale_quantize": (_I, [_P, _I, ctypes.c_int64, ctypes.POINTER(_Rowscale), _P]),
    "bitsmoe_rowscale_dequantize": (_I, [ctypes.POINTER(_Rowscale), _P, _I, ctypes.c_int64, _P]),
    "bitsmoe_block_norm_rowscale": (_I, [ctypes.POINTER(_BlockNormArgs), _P, _P]),
    "bitsmoe_route_workspace_bytes": (_SZ, [_I, _I, _I]),
    "bitsmoe_route": (_I, [_P, ctypes.c_int64, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "bitsmoe_expert_product": (_I, [ctypes.POINTER(_ExpertProductArgs), _P]),
    "bitsmoe_expert_combine": (_I, [_P, _I, ctypes.c_int64, _I, _P, _P, _I, _I, _I, _P, ctypes.c_int64, _P, _I,
                                    ctypes.c_int64, _P]),
    "bitsmoe_block_norm_outputs": (_I, [_P, _I, _I, ctypes.POINTER(_SZ), ctypes.POINTER(_SZ)]),
    "bitsmoe_last_device_status": (_I, [_P, _P]),
    "bitsmoe_free": (None, [_P]),
    "bitsmoe_strerror": (ctypes.c_char_p, [_I]),
    "bitsmoe_last_cuda_error": (_I, []),
    "bitsmoe_debug_wait_limit": (_I, [_I, ctypes.c_longlong]),
    "bitsmoe_debug_single_token_kernel": (_I, [_I]),
    "bitsmoe_debug_bounds": (_I, [_I]),
    "bitsmoe_debug_shift_expert_records": (_I, [_P, _I, ctypes.c_longlong]),
}


class BitsMoEUnavailable(RuntimeError):
    pass


class BitsMoEError(RuntimeError):
    def __init__(self, code: int, where: str = ""):
        self.code = code
        name = ERR.get(code, str(code))
        extra = ""
        if code == -6:
            extra = f" (cudaError {_lib().bitsmoe_last_cuda_error()})"
        super().__init__(f"{where}: BITSMOE_ERR_{name}{extra}")


_lib_handle = None


def _lib():
    global _lib_handle
    if _lib_handle is None:
        if not os.path.exists(LIB_PATH):
            raise BitsMoEUnavailable(
                f"{LIB_PATH} is not built; build it with __graft_entry__.build() "
                "(the BitsMoE forward has no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(lib, name)
            f.restype = res
            f.argtypes = args
        _lib_handle = lib
    return _lib_handle


def library_path() -> str:
    _lib()
    return LIB_PATH


def _check(rc: int, where: str):
    if rc != OK:
        raise BitsMoEError(rc, where)


def _ptr(a: np.ndarray) -> int:
    return a.ctypes.data


def _host_struct(layer: Dict):
    """ctypes view of a host layer dict (see synth.make_layer); returns (struct, keepalive)."""
    keep = {}
    for k, dt in (("bits", np.uint8), ("alpha", np.float32), ("codes", np.uint16),
                  ("scale", np.uint16), ("zero", np.uint16)):
        keep[k] = np.ascontiguousarray(layer[k], dtype=dt)
    bases = [np.ascontiguousarray(layer["basis"][h], dtype=np.uint16) for h in range(3)]
    s = _LayerHost(int(layer["D"]), int(layer["E"]), int(layer["I"]), int(layer["n"]), int(layer["group"]))
    s.basis = (_P * 3)(*[_ptr(b) for b in bases])
    for k in ("bits", "alpha", "codes", "scale", "zero"):
        setattr(s, k, _ptr(keep[k]))
    keep["bases"] = bases
    return s, keep


def _empty_host(dims) -> Dict:
    D, E, I, n, group = dims
    ng = I // group
    return dict(D=D, E=E, I=I, n=n, group=group,
                basis=np.zeros((3, D, n), np.uint16), bits=np.zeros((3, E, n), np.uint8),
                alpha=np.zeros((3, E, n), np.float32), codes=np.zeros((3, E, n, I), np.uint16),
                scale=np.zeros((3, E, n, ng), np.uint16), zero=np.zeros((3, E, n, ng), np.uint16))


def _out_struct(out: Dict):
    s = _LayerHost(out["D"], out["E"], out["I"], out["n"], out["group"])
    s.basis = (_P * 3)(*[_ptr(out["basis"][h]) for h in range(3)])
    for k in ("bits", "alpha", "codes", "scale", "zero"):
        setattr(s, k, _ptr(out[k]))
    return s


class Layer:
    """A packed, device-resident layer (owns the library handle)."""

    def __init__(self, handle: int):
        self.handle = handle
        dims = (ctypes.c_int32 * 5)()
        _check(_lib().bitsmoe_layer_dims(handle, dims), "bitsmoe_layer_dims")
        self.D, self.E, self.I, self.n, self.group = (int(v) for v in dims)

    def free(self):
        if self.handle:
            _lib().bitsmoe_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def bytes(self) -> Dict[str, int]:
        b = _Bytes()
        _check(_lib().bitsmoe_layer_bytes(self.handle, ctypes.byref(b)), "bitsmoe_layer_bytes")
        return dict(total=b.total, basis=b.basis, codes_padded=b.codes_padded, meta=b.meta)

    def expert_moved_bytes(self, e: int):
        """Algorithmic bytes of expert e per projection (gate, up, down)."""
        v = (ctypes.c_uint64 * 3)()
        _check(_lib().bitsmoe_expert_moved_bytes(self.handle, e, v), "bitsmoe_expert_moved_bytes")
        return [int(a) for a in v]


# --------------------------------------------------------------------------
# C-ABI entry points
# --------------------------------------------------------------------------
def bitsmoe_pack(layer: Dict, device: int = 0) -> Layer:
    s, keep = _host_struct(layer)
    h = _P()
    _check(_lib().bitsmoe_pack(ctypes.byref(s), device, ctypes.byref(h)), "bitsmoe_pack")
    return Layer(h.value)


def bitsmoe_pack_to_host(layer: Dict) -> np.ndarray:
    s, keep = _host_struct(layer)
    blob, nbytes = _P(), _SZ()
    _check(_lib().bitsmoe_pack_to_host(ctypes.byref(s), ctypes.byref(blob), ctypes.byref(nbytes)),
           "bitsmoe_pack_to_host")
    try:
        out = np.empty(nbytes.value, np.uint8)
        ctypes.memmove(_ptr(out), blob.value, nbytes.value)
    finally:
        _lib().bitsmoe_blob_free(blob)
    return out


def bitsmoe_load_blob(blob: np.ndarray, device: int = 0) -> Layer:
    blob = np.ascontiguousarray(blob, dtype=np.uint8)
    h = _P()
    _check(_lib().bitsmoe_load_blob(_ptr(blob), blob.nbytes, device, ctypes.byref(h)), "bitsmoe_load_blob")
    return Layer(h.value)


def bitsmoe_unpack_blob(blob: np.ndarray, dims) -> Dict:
    blob = np.ascontiguousarray(blob, dtype=np.uint8)
    out = _empty_host(dims)
    s = _out_struct(out)
    _check(_lib().bitsmoe_unpack_blob(_ptr(blob), blob.nbytes, ctypes.byref(s)), "bitsmoe_unpack_blob")
    return out


def bitsmoe_unpack(layer: Layer) -> Dict:
    out = _empty_host((layer.D, layer.E, layer.I, layer.n, layer.group))
    s = _out_struct(out)
    _check(_lib().bitsmoe_unpack(layer.handle, ctypes.byref(s)), "bitsmoe_unpack")
    return out


def bitsmoe_workspace_bytes(layer: Layer, T: int, top_k: int) -> int:
    return int(_lib().bitsmoe_workspace_bytes(layer.handle, T, top_k))


def bitsmoe_forward_launches(layer: Layer, T: int, top_k: int) -> int:
    """Kernels one forward call launches (1: the fused single-token kernel; 5: the chain)."""
    n = int(_lib().bitsmoe_forward_launches(layer.handle, T, top_k))
    if n < 0:
        raise BitsMoEError(n, "bitsmoe_forward_launches")
    return n


PLAN_FUSED, PLAN_DECODE_CHAIN, PLAN_TC_PROJECTIONS, PLAN_TC_GATE_UP, PLAN_TC_DOWN = 1, 2, 4, 8, 16
PLAN_CLUSTERED = 32


def bitsmoe_forward_plan(layer: Layer, T: int, top_k: int) -> int:
    """Bit set of how a T-token forward runs: PLAN_FUSED, PLAN_DECODE_CHAIN, PLAN_TC_PROJECTIONS,
    PLAN_TC_GATE_UP, PLAN_TC_DOWN, PLAN_CLUSTERED (with PLAN_FUSED: the clustered single-token kernel)."""
    n = int(_lib().bitsmoe_forward_plan(layer.handle, T, top_k))
    if n < 0:
        raise BitsMoEError(n, "bitsmoe_forward_plan")
    return n


def bitsmoe_block_forward_launches(layer: Layer, T: int, top_k: int) -> int:
    """Kernels one block forward launches (1: the fused kernel with its pre-norm; else norm/router + chain)."""
    n = int(_lib().bitsmoe_block_forward_launches(layer.handle, T, top_k))
    if n < 0:
        raise BitsMoEError(n, "bitsmoe_block_forward_launches")
    return n


def bitsmoe_moe_forward(x_ptr: int, logits_ptr: int, T: int, top_k: int, layer: Layer, y_ptr: int,
                        ws_ptr: int, ws_bytes: int, stream: int = 0) -> None:
    _check(_lib().bitsmoe_moe_forward(x_ptr, logits_ptr, T, top_k, layer.handle, y_ptr, ws_ptr,
                                      ws_bytes, stream), "bitsmoe_moe_forward")


def bitsmoe_moe_forward_host(x_bits: np.ndarray, logits: np.ndarray, top_k: int, layer: Layer,
                             ws_ptr: int, ws_bytes: int, stream: int = 0,
                             y_out: Optional[np.ndarray] = None) -> np.ndarray:
    """Forward from host arrays (x bf16 bits T x D, logits fp32 T x E) -> y fp32 T x D."""
    T = int(x_bits.shape[0])
    y = y_out if y_out is not None else np.empty((T, layer.D), np.float32)
    _check(_lib().bitsmoe_moe_forward_host(x_bits.ctypes.data, logits.ctypes.data, T, top_k, layer.handle,
                                           y.ctypes.data, ws_ptr, ws_bytes, stream), "bitsmoe_moe_forward_host")
    return y


NOALLOC_SCRATCH_BYTES = 8 << 20   # BITSMOE_NOALLOC_SCRATCH_BYTES


def bitsmoe_moe_forward_noalloc(x_ptr: int, logits_ptr: int, T: int, top_k: int, layer: Layer, y_ptr: int,
                                stream: int = 0) -> None:
    """The forward for callers that cannot allocate device memory: its scratch is
    the library's built-in array (NOALLOC_SCRATCH_BYTES per device, shared by all
    calls on that device, so overlapping calls race)."""
    _check(_lib().bitsmoe_moe_forward_noalloc(x_ptr, logits_ptr, T, top_k, layer.handle, y_ptr, stream),
           "bitsmoe_moe_forward_noalloc")


def bitsmoe_rmsnorm_router(h_ptr: int, w_router_ptr: int, eps: float, T: int, D: int, E: int,
                           x_out_ptr: int, logits_out_ptr: int, stream: int = 0) -> None:
    _check(_lib().bitsmoe_rmsnorm_router(h_ptr, w_router_ptr, eps, T, D, E, x_out_ptr, logits_out_ptr, stream),
           "bitsmoe_rmsnorm_router")


def bitsmoe_moe_block_forward(h_ptr: int, w_router_ptr: int, eps: float, T: int, top_k: int, layer: Layer,
                              ws_ptr: int, ws_bytes: int, stream: int = 0) -> None:
    _check(_lib().bitsmoe_moe_block_forward(h_ptr, w_router_ptr, eps, T, top_k, layer.handle, ws_ptr, ws_bytes,
                                            stream), "bitsmoe_moe_block_forward")


def bitsmoe_profile_forward(x_ptr: int, logits_ptr: int, T: int, top_k: int, layer: Layer, y_ptr: int,
                            ws_ptr: int, ws_bytes: int, stream: int = 0):
    """Forward with the five phases serialised and timed; returns their durations (ms)."""
    ms = (ctypes.c_float * 5)()
    _check(_lib().bitsmoe_profile_forward(x_ptr, logits_ptr, T, top_k, layer.handle, y_ptr, ws_ptr,
                                          ws_bytes, stream, ms), "bitsmoe_profile_forward")
    return [float(v) for v in ms]


def bitsmoe_quantize_units(p_ptr: int, bits_ptr: int, U: int, I: int, group: int, grid: int, codes_ptr: int,
                           scale_ptr: int, zero_ptr: int, status_ptr: int = 0, stream: int = 0) -> None:
    """Quantise U float units (device U x I fp32) into codes / fp16 scale / fp16 zero (device)."""
    _check(_lib().bitsmoe_quantize_units(p_ptr, bits_ptr, U, I, group, grid, codes_ptr, scale_ptr, zero_ptr,
                                         status_ptr, stream), "bitsmoe_quantize_units")


def bitsmoe_projection_budget(E: int, n: int, m: int, b_eq) -> int:
    """B_h = floor(E n b_eq - 16 n^2 / m) for b_eq given as a float, an int or a (num, den) pair."""
    from fractions import Fraction
    fr = Fraction(*b_eq) if isinstance(b_eq, tuple) else Fraction(str(b_eq))
    out = ctypes.c_int64()
    _check(_lib().bitsmoe_projection_budget(E, n, m, fr.numerator, fr.denominator, ctypes.byref(out)),
           "bitsmoe_projection_budget")
    return int(out.value)


def bitsmoe_allocate_workspace_bytes(U: int) -> int:
    return int(_lib().bitsmoe_allocate_workspace_bytes(U))


def bitsmoe_allocate_bits(p_ptr: int, alpha_ptr: int, beta_ptr: int, gamma: float, U: int, d: int, kappa,
                          budget: int, bits_ptr: int, ws_ptr: int, ws_bytes: int, stream: int = 0,
                          profile: bool = False):
    """Bit-width per unit (device, U bytes) for one projection type; with profile=True the call
    synchronises and returns the phase durations (ms: costs and hull, cut, fill)."""
    k = (ctypes.c_float * 3)(*[float(v) for v in kappa])
    if profile:
        ms = (ctypes.c_float * 3)()
        _check(_lib().bitsmoe_profile_allocate_bits(p_ptr, alpha_ptr, beta_ptr, gamma, U, d, k, budget, bits_ptr,
                                                    ws_ptr, ws_bytes, stream, ms), "bitsmoe_profile_allocate_bits")
        return [float(v) for v in ms]
    _check(_lib().bitsmoe_allocate_bits(p_ptr, alpha_ptr, beta_ptr, gamma, U, d, k, budget, bits_ptr, ws_ptr,
                                        ws_bytes, stream), "bitsmoe_allocate_bits")
    return None


def bitsmoe_last_device_status(ws_ptr: int, stream: int = 0) -> int:
    return int(_lib().bitsmoe_last_device_status(ws_ptr, stream))


def bitsmoe_block_norm_outputs(layer: Layer, T: int, top_k: int):
    """Byte offsets of a block forward's normalised x and router logits in its workspace."""
    xo, lo = _SZ(0), _SZ(0)
    _check(_lib().bitsmoe_block_norm_outputs(layer.handle, T, top_k, ctypes.byref(xo), ctypes.byref(lo)),
           "bitsmoe_block_norm_outputs")
    return int(xo.value), int(lo.value)


def bitsmoe_noalloc_last_status(stream: int = 0) -> int:
    """Device status of the no-allocation scratch on the current device (read and cleared)."""
    return int(_lib().bitsmoe_noalloc_last_status(stream))


def bitsmoe_strerror(code: int) -> str:
    return _lib().bitsmoe_strerror(code).decode()


# --------------------------------------------------------------------------
# torch convenience (device memory + streams only)
# --------------------------------------------------------------------------
class Workspace:
    """Device workspace sized for (T, top_k) on a layer, allocated (zero-filled) with torch."""

    def __init__(self, layer: Layer, T: int, top_k: int, device=None):
        import torch
        self.nbytes = bitsmoe_workspace_bytes(layer, T, top_k)
        if self.nbytes == 0:
            raise BitsMoEError(ERR_CODE["INVALID_ARG"], "bitsmoe_workspace_bytes")
        self.buf = torch.zeros(self.nbytes + 256, dtype=torch.uint8,
                               device=device if device is not None else f"cuda:{torch.cuda.current_device()}")
        base = self.buf.data_ptr()
        self.ptr = (base + 255) // 256 * 256


def moe_forward(layer: Layer, x_bits, logits, top_k: int, ws: Optional[Workspace] = None, y=None, stream=None):
    """y (fp32 T x D) = BitsMoE MoE-layer forward of x (int16/uint16 tensor of bf16 bits or a
    torch.bfloat16 tensor, T x D) with router logits (fp32 T x E), all on the device."""
    import torch
    T = int(x_bits.shape[0])
    if ws is None:
        ws = Workspace(layer, T, top_k, device=x_bits.device)
    if y is None:
        y = torch.empty((T, layer.D), dtype=torch.float32, device=x_bits.device)
    st = stream if stream is not None else torch.cuda.current_stream(x_bits.device)
    bitsmoe_moe_forward(x_bits.data_ptr(), logits.data_ptr(), T, top_k, layer, y.data_ptr(),
                        ws.ptr, ws.nbytes, st.cuda_stream)
    return y


def quantize_units(p, bits, group: int, grid: int = 256, stream=None):
    """Quantise the units in the rows of `p` (torch fp32 U x I on the device) with per-unit
    bit-widths `bits` (torch uint8, U) into the stored format; returns (codes uint16-as-int16
    U x I, scale, zero fp16 bit patterns U x I/group, status int32 tensor of one element)."""
    import torch
    U, I = int(p.shape[0]), int(p.shape[1])
    dev = p.device
    codes = torch.empty((U, I), dtype=torch.int16, device=dev)
    scale = torch.empty((U, I // group), dtype=torch.int16, device=dev)
    zero = torch.empty((U, I // group), dtype=torch.int16, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    st = stream if stream is not None else torch.cuda.current_stream(dev)
    bitsmoe_quantize_units(p.data_ptr(), bits.data_ptr(), U, I, group, grid, codes.data_ptr(), scale.data_ptr(),
                           zero.data_ptr(), status.data_ptr(), st.cuda_stream)
    return codes, scale, zero, status


def allocate_bits(p, alpha, beta, gamma: float, kappa, budget: int, stream=None):
    """Bit-widths (torch uint8, U) of the units in the rows of `p` (torch fp32 U x d on the
    device) with spectral energies `alpha` and importances `beta` (fp32, U) under `budget`."""
    import torch
    U, d = int(p.shape[0]), int(p.shape[1])
    dev = p.device
    bits = torch.empty(U, dtype=torch.uint8, device=dev)
    nb = bitsmoe_allocate_workspace_bytes(U)
    ws = torch.empty(nb + 256, dtype=torch.uint8, device=dev)
    st = stream if stream is not None else torch.cuda.current_stream(dev)
    bitsmoe_allocate_bits(p.data_ptr(), alpha.data_ptr(), beta.data_ptr(), gamma, U, d, kappa, budget,
                          bits.data_ptr(), (ws.data_ptr() + 255) // 256 * 256, nb, st.cuda_stream)
    ws.record_stream(st)   # the workspace is freed here but used by the kernels still queued on st
    return bits


def importance(x, logits, top_k: int, basis, alpha, factor, stream=None):
    """Importance beta (torch fp32, 3 x E x n) of every unit from calibration tokens: x (torch
    int16 bf16 bit patterns, T x D), logits (fp32, T x E), basis = (Phi_gate, Phi_up) fp32 D x n,
    alpha = (alpha_gate, alpha_up) fp32 E x n, factor = (P_gate, P_up, P_down) fp32 E x I x n,
    all on the device."""
    import torch
    T, D = int(x.shape[0]), int(x.shape[1])
    E = int(logits.shape[1])
    _, I, n = (int(v) for v in factor[0].shape)
    dev = x.device
    beta = torch.empty((3, E, n), dtype=torch.float32, device=dev)
    nb = int(_lib().bitsmoe_importance_workspace_bytes(T, E, I, n, top_k))
    ws = torch.empty(nb + 256, dtype=torch.uint8, device=dev)
    st = stream if stream is not None else torch.cuda.current_stream(dev)
    bp = (_P * 2)(*[b.data_ptr() for b in basis])
    ap = (_P * 2)(*[a.data_ptr() for a in alpha])
    fp = (_P * 3)(*[f.data_ptr() for f in factor])
    _check(_lib().bitsmoe_importance(x.data_ptr(), logits.data_ptr(), T, D, E, I, n, top_k, bp, ap, fp,
                                     beta.data_ptr(), (ws.data_ptr() + 255) // 256 * 256, nb, st.cuda_stream),
           "bitsmoe_importance")
    ws.record_stream(st)
    return beta


def shared_basis(W, side: str, max_sweeps: int = 30, stream=None):
    """Shared-basis decomposition of one projection type (torch fp32 on the device): side "in"
    takes W = E x d x D (gate/up, W_e = d x D), side "out" W = E x D x d (down, W_e = D x d).
    Returns (phi D x n, sigma n, alpha E x n, P E x n x d unit-major, sweeps, status) with
    n = min(D, E d); sweeps and status are device int tensors (one element each)."""
    import torch
    sd = {"in": 0, "out": 1}[side]
    E = int(W.shape[0])
    d, D = (int(W.shape[1]), int(W.shape[2])) if sd == 0 else (int(W.shape[2]), int(W.shape[1]))
    n = min(D, E * d)
    dev = W.device
    phi = torch.empty((D, n), dtype=torch.float32, device=dev)
    sigma = torch.empty((n,), dtype=torch.float32, device=dev)
    alpha = torch.empty((E, n), dtype=torch.float32, device=dev)
    P = torch.empty((E, n, d), dtype=torch.float32, device=dev)
    info = torch.zeros((2,), dtype=torch.int32, device=dev)   # sweeps, status
    nb = int(_lib().bitsmoe_decompose_workspace_bytes(sd, E, d, D))
    ws = torch.empty(nb + 256, dtype=torch.uint8, device=dev)
    st = stream if stream is not None else torch.cuda.current_stream(dev)
    _check(_lib().bitsmoe_shared_basis(sd, W.data_ptr(), E, d, D, phi.data_ptr(), sigma.data_ptr(), alpha.data_ptr(),
                                       P.data_ptr(), (ws.data_ptr() + 255) // 256 * 256, nb, max_sweeps,
                                       info.data_ptr(), info.data_ptr() + 4, st.cuda_stream),
           "bitsmoe_shared_basis")
    ws.record_stream(st)
    return phi, sigma, alpha, P, info[0:1], info[1:2]


def calibration_gram(x, g=None, stream=None):
    """H = sum_t g_t x_t x_t^T (torch fp32 D x D) from x (torch int16 bf16 bit patterns, T x D)
    and optional per-token weights g (fp32, T), on the device."""
    import torch
    T, D = int(x.shape[0]), int(x.shape[1])
    H = torch.empty((D, D), dtype=torch.float32, device=x.device)
    st = stream if stream is not None else torch.cuda.current_stream(x.device)
    _check(_lib().bitsmoe_calibration_gram(x.data_ptr(), g.data_ptr() if g is not None else None, T, D,
                                           H.data_ptr(), st.cuda_stream), "bitsmoe_calibration_gram")
    return H


# --------------------------------------------------------------------------
# microscaled 4-bit matrices and the norms between blocks (torch tensors)
# --------------------------------------------------------------------------
MICRO_FORMATS = {"e8m0": 0, "e4m3": 1}       # BITSMOE_MICRO_*: blocks of 32 and of 16 columns
_MICRO_BLOCK = {"e8m0": 32, "e4m3": 16}
BLOCK_NORM_MAX_D = 32768                     # BITSMOE_BLOCK_NORM_MAX_D
_GATE_NONE, _GATE_TOKEN, _GATE_ELEMENT = 0, 1, 2


_torch = None
_DENSE = {}          # torch dtype -> BITSMOE_F32 / BITSMOE_BF16
_E4M3 = 2            # BITSMOE_E4M3
_raw_stream = None   # device index -> the current stream's handle
_current = None      # the current device's index


_MAX_ROWS = 1 << 24   # the library's limit of rows; beyond 32 bits a size would be cut on its way there


def _load_torch():
    global _torch, _DENSE, _raw_stream, _current
    import torch
    _DENSE = {torch.float32: 0, torch.bfloat16: 1}
    # the handle without a Stream object around it, where torch has it (0.1 us instead of 2)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
        lambda i: torch.cuda.current_stream(i).cuda_stream)
    _current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _torch = torch
    return torch


def _refuse(where: str, why: str, code: str = "INVALID_ARG"):
    raise BitsMoEError(ERR_CODE[code], f"{where}: {why}")


def _dense_type(where: str, name: str, dtype) -> int:
    ty = _DENSE.get(dtype)
    if ty is None:
        _refuse(where, f"{name} must be float32 or bfloat16, got {dtype}")
    return ty


def _rows(where: str, name: str, x, rows=None, cols=None, device=None, dtype=None):
    """Checks of a 2-d device tensor whose rows are dense (the pitch between them is free); its pitch."""
    shape = x.shape
    if len(shape) != 2 or not x.is_cuda:
        _refuse(where, f"{name} must be a 2-d CUDA tensor")
    if device is not None and x.device != device:
        _refuse(where, f"{name} is on {x.device}, expected {device}")
    r, c = shape
    if r > _MAX_ROWS or c > _MAX_ROWS:
        _refuse(where, f"{name} has shape {tuple(shape)}", "SHAPE")
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        _refuse(where, f"{name} has shape {tuple(shape)}, expected {(rows, cols)}", "SHAPE")
    if dtype is not None and x.dtype != dtype:
        _refuse(where, f"{name} must be {dtype}, got {x.dtype}")
    ld, step = x.stride()
    if step != 1 and c > 1 and r > 0:
        _refuse(where, f"{name} must have dense rows (stride 1 along them)")
    if r <= 1:
        return c if c > 0 else 1
    if ld < c:
        _refuse(where, f"{name}'s rows overlap (stride {ld})")
    return ld


def _vector(where: str, name: str, v, n: int, device, dtype):
    shape = v.shape
    if len(shape) != 1 or shape[0] != n:
        _refuse(where, f"{name} has shape {tuple(shape)}, expected {(n,)}", "SHAPE")
    if v.device != device or (n > 1 and v.stride(0) != 1):
        _refuse(where, f"{name} must be a dense vector on {device}")
    if v.dtype != dtype:
        _refuse(where, f"{name} must be {dtype}, got {v.dtype}")
    return v.data_ptr()


def _elsewhere(where: str, device, stream):
    """Context for a call on another stream than the current one, or on a device that is not current: inside it
    both are, so that outputs belong to the stream that writes them."""
    if stream is not None and stream.device != device:
        _refuse(where, f"the stream is of {stream.device}, the tensors are on {device}")
    return _torch.cuda.stream(stream if stream is not None else _torch.cuda.current_stream(device))


class Microscale:
    """A microscaled 4-bit matrix on the device: `codes` (torch uint8, rows x 16 ceil(cols / 32)) and
    `scales` (uint8, the stored tile order), see bitsmoe_microscale in include/bitsmoe.h; `fmt` is
    "e8m0" (blocks of 32 columns) or "e4m3" (16), `scale` the tensor scale."""

    __slots__ = ("_codes", "_scales", "_buf", "_c", "device", "rows", "cols", "fmt")   # _c: what the library reads

    def __init__(self, codes, scales, rows: int, cols: int, fmt: str = "e8m0", scale: float = 1.0):
        torch = _torch or _load_torch()
        if fmt not in MICRO_FORMATS or rows < 0 or cols < 1:
            _refuse("Microscale", f"{rows} rows, {cols} columns, format {fmt!r}")
        if rows > _MAX_ROWS or cols > _MAX_ROWS:
            _refuse("Microscale", f"{rows} rows, {cols} columns", "SHAPE")
        nc, ns = _micro_sizes(fmt, rows, cols)
        u8 = torch.uint8
        if codes.dtype is not u8 or codes.numel() != nc or not codes.is_contiguous():
            _refuse("Microscale", f"codes must be {nc} contiguous bytes (uint8)", "SHAPE")
        if scales.dtype is not u8 or scales.numel() != ns or not scales.is_contiguous():
            _refuse("Microscale", f"scales must be {ns} contiguous bytes (uint8)", "SHAPE")
        self.device = dev = codes.device
        if scales.device != dev:
            _refuse("Microscale", "codes and scales are on different devices")
        self._codes, self._scales, self._buf = codes, scales, None
        self.rows, self.cols, self.fmt = rows, cols, fmt
        self._c = _Microscale(MICRO_FORMATS[fmt], rows, cols, scale, codes.data_ptr(), scales.data_ptr())

    @classmethod
    def empty(cls, rows: int, cols: int, fmt: str = "e8m0", scale: float = 1.0, device=None) -> "Microscale":
        torch = _torch or _load_torch()
        if fmt not in MICRO_FORMATS or rows < 0 or cols < 1:
            _refuse("Microscale.empty", f"{rows} rows, {cols} columns, format {fmt!r}")
        if rows > _MAX_ROWS or cols > _MAX_ROWS:
            _refuse("Microscale.empty", f"{rows} rows, {cols} columns", "SHAPE")
        nc, ns = _micro_sizes(fmt, rows, cols)
        self = cls.__new__(cls)   # one allocation for both; the tensors are made when asked for
        at = (nc + 255) // 256 * 256
        self._buf = buf = torch.empty(at + ns, dtype=torch.uint8,
                                      device=device if device is not None else torch.cuda.current_device())
        self._codes = self._scales = None
        base = buf.data_ptr()
        self.device = buf.device
        self.rows, self.cols, self.fmt = rows, cols, fmt
        self._c = _Microscale(MICRO_FORMATS[fmt], rows, cols, scale, base, base + at)
        return self

    @property
    def scale(self) -> float:
        return self._c.scale   # (as the library has it: fp32)

    @scale.setter
    def scale(self, value: float):
        self._c.scale = value

    @property
    def codes(self):
        if self._codes is None:
            self._codes = self._buf[:_micro_sizes(self.fmt, self.rows, self.cols)[0]]
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            n = _micro_sizes(self.fmt, self.rows, self.cols)[1]
            self._scales = self._buf[self._buf.numel() - n:]
        return self._scales

    @classmethod
    def from_rows(cls, codes, block_scales, cols: int, fmt: str = "e8m0", scale: float = 1.0) -> "Microscale":
        """From a checkpoint's arrays: codes uint8 rows x ceil(cols / 2) (even column in the lower half) and
        one scale byte per block, uint8 rows x ceil(cols / block)."""
        import torch
        import torch.nn.functional as F
        if fmt not in MICRO_FORMATS:
            _refuse("Microscale.from_rows", f"unknown format {fmt!r}")
        rows, nb = int(codes.shape[0]), -(-cols // _MICRO_BLOCK[fmt])
        if tuple(codes.shape) != (rows, (cols + 1) // 2) or tuple(block_scales.shape) != (rows, nb):
            _refuse("Microscale.from_rows", f"codes {tuple(codes.shape)}, scales {tuple(block_scales.shape)}", "SHAPE")
        if codes.dtype != torch.uint8 or block_scales.dtype != torch.uint8:
            _refuse("Microscale.from_rows", "codes and scales must be uint8")
        if cols % 2:
            codes = codes.clone()
            codes[:, -1] &= 15
        c = F.pad(codes, (0, 16 * (-(-cols // 32)) - codes.shape[1])).contiguous()
        s = F.pad(block_scales, (0, -nb % 4, 0, -rows % 128))
        s = s.view(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1)
        return cls(c.view(-1), s.contiguous(), rows, cols, fmt, scale)

    def block_scales(self):
        """The scale bytes by row and block (uint8, rows x blocks)."""
        nb = -(-self.cols // _MICRO_BLOCK[self.fmt])
        rt, ct = -(-self.rows // 128), -(-nb // 4)
        s = self.scales.view(rt, ct, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, ct * 4)
        return s[:self.rows, :nb]


def _micro_sizes(fmt: str, rows: int, cols: int):
    """The sizes that bitsmoe_microscale_bytes gives, of codes and scales."""
    tile = 4 * _MICRO_BLOCK[fmt]   # columns of a 512-byte scale tile
    return rows * ((cols + 31) // 32 * 16), (rows + 127) // 128 * ((cols + tile - 1) // tile * 512)


def microscale_bytes(fmt: str, rows: int, cols: int):
    """Bytes of a microscaled matrix's codes and scales."""
    if fmt not in MICRO_FORMATS:
        _refuse("microscale_bytes", f"unknown format {fmt!r}")
    nc, ns = _SZ(0), _SZ(0)
    _check(_lib().bitsmoe_microscale_bytes(MICRO_FORMATS[fmt], int(rows), int(cols), ctypes.byref(nc),
                                           ctypes.byref(ns)), "bitsmoe_microscale_bytes")
    return int(nc.value), int(ns.value)


def microscale_quantize(x, fmt: str = "e8m0", scale: float = 1.0, out: Optional[Microscale] = None,
                        stream=None) -> Microscale:
    """Quantise the rows of x (torch fp32 or bf16, 2-d, dense rows, on the device) into a Microscale with
    tensor scale `scale` (a power of two); `out` reuses an existing one of the same shape and format (a call that is
    refused leaves it as it was)."""
    torch = _torch or _load_torch()
    where = "microscale_quantize"
    dev = x.device
    ty = _dense_type(where, "x", x.dtype)
    ld = _rows(where, "x", x)
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return microscale_quantize(x, fmt, scale, out)
    rows, cols = x.shape
    if out is None:
        out = Microscale.empty(rows, cols, fmt, scale, dev)
    elif (out.rows, out.cols, out.fmt) != (rows, cols, fmt) or out.device != dev:
        _refuse(where, "out has another shape, format or device", "SHAPE")
    before, out.scale = out.scale, scale
    rc = _lib().bitsmoe_microscale_quantize(x.data_ptr(), ty, ld, out._c, _raw_stream(dev.index))
    if rc:
        out.scale = before   # its codes are the old ones
    _check(rc, "bitsmoe_microscale_quantize")
    return out


def microscale_dequantize(q: Microscale, dtype=None, out=None, stream=None):
    """The values of a Microscale as a torch tensor rows x cols (float32, or bfloat16)."""
    torch = _torch or _load_torch()
    where = "microscale_dequantize"
    dev = q.device
    if dev.type != "cuda":
        _refuse(where, "the matrix must be on a CUDA device")
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return microscale_dequantize(q, dtype, out)
    if out is None:
        out, ld = torch.empty((q.rows, q.cols), dtype=dtype if dtype is not None else torch.float32, device=dev), q.cols
    else:
        ld = _rows(where, "out", out, q.rows, q.cols, dev)
    _check(_lib().bitsmoe_microscale_dequantize(q._c, out.data_ptr(), _dense_type(where, "out", out.dtype), ld,
                                                _raw_stream(dev.index)), "bitsmoe_microscale_dequantize")
    return out


def microscale_product(w: Microscale, x, up: Optional[Microscale] = None, dtype=None, y=None, status=None,
                       stream=None):
    """y (T x w.rows, fp32 by default, or bf16) = x w^T for x a torch bf16 tensor (T x w.cols, dense rows) or a
    Microscale of w's format; with `up` (w's shape and format) SiLU(x w^T) * (x up^T).  `status`: an optional
    int32 tensor of one element that receives a device-side timeout (the results that it cost are NaN, with and
    without it).  Of large products, x's rows off 16-byte boundaries are copied to a temporary first."""
    torch = _torch or _load_torch()
    where = "microscale_product"
    dev = w.device
    if dev.type != "cuda" or x.device != dev or (up is not None and up.device != dev):
        _refuse(where, "the operands must be on one CUDA device")
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return microscale_product(w, x, up, dtype, y, status)
    if isinstance(x, Microscale):
        T, x_ptr, x_ld, xq = x.rows, None, 0, x._c
    else:
        x_ld = _rows(where, "x", x, None, w.cols, None, torch.bfloat16)
        T, x_ptr, xq = x.shape[0], x.data_ptr(), None
        # Many rows off 16-byte boundaries are brought onto them first (us with and without: 60 x 4999 by 7000 rows
        # 26 and 38, 500 55 and 228; 37 x 2041 by 1001 rows 9 and 8, and 6 more on the host).
        if T > 16 and (x_ptr % 16 or x_ld % 8) and T * w.rows * w.cols > 1 << 29:
            ld = (w.cols + 7) // 8 * 8
            rows = torch.empty((T, ld), dtype=torch.bfloat16, device=dev)
            _check(_lib().bitsmoe_microscale_align(x_ptr, x_ld, T, w.cols, rows.data_ptr(), ld, _raw_stream(dev.index)),
                   "bitsmoe_microscale_align")
            x_ptr, x_ld = rows.data_ptr(), ld
    st_ptr = None
    if status is not None:
        if status.dtype != torch.int32 or status.numel() != 1 or status.device != dev:
            _refuse(where, "status must be one int32 on the operands' device")
        st_ptr = status.data_ptr()
    if y is None:
        y, y_ld = torch.empty((T, w.rows), dtype=dtype if dtype is not None else torch.float32, device=dev), w.rows
    else:
        y_ld = _rows(where, "y", y, T, w.rows, dev)
    _check(_lib().bitsmoe_microscale_product(w._c, up._c if up is not None else None, x_ptr, x_ld, xq, T,
                                             y.data_ptr(), _dense_type(where, "y", y.dtype), y_ld, st_ptr,
                                             _raw_stream(dev.index)), "bitsmoe_microscale_product")
    return y


def block_norm(h, y=None, *, post_norm: bool = False, post_gain=None, post_eps: float = 1e-6, gate=None,
               gate_sigmoid: bool = False, channel_scale=None, branch_scale: float = 1.0,
               residual_scale: float = 1.0, pre_norm: bool = True, pre_gain=None, pre_eps: float = 1e-6,
               gain_offset: float = 0.0, h_out=None, x=None, x_dtype=None, stream=None):
    """What stands between a block's output y and the next block's input (see bitsmoe_block_norm):
    returns (h', x), h' = residual_scale h + branch_scale channel_scale gate norm(y) and x = norm(h').

    h (T x D, fp32 or bf16) is the residual stream; y None: h' is not formed (the result's first item is h
    times residual_scale only when h_out is given, else None); gate is a vector of T (one value per row) or
    T x D; the gains and channel_scale are vectors of D of one type.  h_out and x are allocated when not
    given (h_out may be h: in place); pre_norm False returns x None.  x_dtype torch.float8_e4m3fn, or x a Rowscale:
    x in 8 bits with a scale a row (see bitsmoe_block_norm_rowscale), returned as a Rowscale."""
    torch = _torch or _load_torch()
    where = "block_norm"
    dev = h.device
    h_type, h_ld = _dense_type(where, "h", h.dtype), _rows(where, "h", h)
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return block_norm(h, y, post_norm=post_norm, post_gain=post_gain, post_eps=post_eps, gate=gate,
                              gate_sigmoid=gate_sigmoid, channel_scale=channel_scale, branch_scale=branch_scale,
                              residual_scale=residual_scale, pre_norm=pre_norm, pre_gain=pre_gain, pre_eps=pre_eps,
                              gain_offset=gain_offset, h_out=h_out, x=x, x_dtype=x_dtype)
    T, D = h.shape
    y_type = y_ld = gate_type = gate_kind = gate_ld = gain_type = ho_ld = x_type = x_ld = 0
    y_ptr = gate_ptr = post_ptr = pre_ptr = chan_ptr = ho_ptr = x_ptr = None
    if y is not None:
        y_type, y_ld, y_ptr = _dense_type(where, "y", y.dtype), _rows(where, "y", y, T, D, dev), y.data_ptr()
    if gate is not None:
        gate_type, gate_ptr = _dense_type(where, "gate", gate.dtype), gate.data_ptr()
        if gate.dim() == 1:
            if gate.shape[0] != T or gate.device != dev:
                _refuse(where, f"gate has shape {tuple(gate.shape)} on {gate.device}, expected {(T,)} on {dev}", "SHAPE")
            gate_kind, gate_ld = _GATE_TOKEN, gate.stride(0)
            if gate_ld < 1:
                if T > 1:
                    _refuse(where, "gate's elements overlap")
                gate_ld = 1
        else:
            gate_kind, gate_ld = _GATE_ELEMENT, _rows(where, "gate", gate, T, D, dev)
    gt = None
    if post_gain is not None:
        gt = post_gain.dtype
        post_ptr = _vector(where, "post_gain", post_gain, D, dev, gt)
    if pre_gain is not None:
        gt = gt or pre_gain.dtype
        pre_ptr = _vector(where, "pre_gain", pre_gain, D, dev, gt)
    if channel_scale is not None:
        gt = gt or channel_scale.dtype
        chan_ptr = _vector(where, "channel_scale", channel_scale, D, dev, gt)
    if gt is not None:
        gain_type = _dense_type(where, "gains", gt)
    if h_out is not None:
        ho_ld, ho_ptr = _rows(where, "h_out", h_out, T, D, dev, h.dtype), h_out.data_ptr()
    elif y is not None:
        h_out, ho_ld = torch.empty((T, D), dtype=h.dtype, device=dev), D
        ho_ptr = h_out.data_ptr()
    if isinstance(x, Rowscale) or (x is None and x_dtype is torch.float8_e4m3fn):
        if not pre_norm:
            _refuse(where, "x in 8 bits is asked for but pre_norm is off")
        if x is None:
            x = Rowscale.empty((T, D), dev)
        xc = _rowscale_rows(where, "x", x, T, D, dev)
        x_type, x_ld, x_ptr = _E4M3, xc.ld, xc.codes
    elif x is not None:
        if not pre_norm:
            _refuse(where, "x is given but pre_norm is off")
        x_type, x_ld, x_ptr = _dense_type(where, "x", x.dtype), _rows(where, "x", x, T, D, dev), x.data_ptr()
    elif pre_norm:
        x = torch.empty((T, D), dtype=x_dtype if x_dtype is not None else torch.bfloat16, device=dev)
        x_type, x_ld, x_ptr = _dense_type(where, "x", x.dtype), D, x.data_ptr()
    args = _BlockNormArgs(T, D, h_type, y_type, gate_type, gain_type, x_type, 1 if post_norm else 0, gate_kind,
                          1 if gate_sigmoid else 0, post_eps, pre_eps, gain_offset, residual_scale, branch_scale,
                          h.data_ptr(), y_ptr, gate_ptr, post_ptr, pre_ptr, chan_ptr, ho_ptr, x_ptr,
                          h_ld, y_ld, gate_ld, ho_ld, x_ld)
    if x_type == _E4M3:
        _check(_lib().bitsmoe_block_norm_rowscale(args, xc.scales, _raw_stream(dev.index)),
               "bitsmoe_block_norm_rowscale")
    else:
        _check(_lib().bitsmoe_block_norm(args, _raw_stream(dev.index)), "bitsmoe_block_norm")
    return h_out, x


# --------------------------------------------------------------------------
# rows in 8 bits, routing and experts that are dense matrices (torch tensors)
# --------------------------------------------------------------------------
class Rowscale:
    """Rows in 8 bits on the device: `codes` (torch.float8_e4m3fn, rows x cols, or experts x rows x cols with dense
    rows) and `scales` (float32, one for each row); value = code * scale, see bitsmoe_rowscale in include/bitsmoe.h."""

    __slots__ = ("_codes", "_scales", "_c", "shape", "device")   # _c: what the library reads, formed when first needed

    def __init__(self, codes, scales):
        torch = _torch or _load_torch()
        if codes.dtype is not torch.float8_e4m3fn or codes.dim() not in (2, 3):
            _refuse("Rowscale", f"codes must be 2-d or 3-d float8_e4m3fn, got {codes.dim()}-d {codes.dtype}")
        if scales.dtype is not torch.float32 or scales.device != codes.device:
            _refuse("Rowscale", f"scales must be float32 on {codes.device}")
        if scales.shape != codes.shape[:-1]:
            _refuse("Rowscale", f"scales have shape {tuple(scales.shape)}, codes {tuple(codes.shape)}", "SHAPE")
        if scales.shape[-1] > 1 and scales.stride(-1) != 1:
            _refuse("Rowscale", "scales must be dense along the rows")
        self._codes, self._scales, self._c = codes, scales, None
        self.shape, self.device = codes.shape, codes.device

    @property
    def codes(self):
        return self._codes

    @property
    def scales(self):
        return self._scales

    @classmethod
    def empty(cls, shape, device=None) -> "Rowscale":
        """Uninitialised rows on a pitch of a multiple of 16 bytes."""
        torch = _torch or _load_torch()
        dims = len(shape)
        if dims not in (2, 3) or min(shape) < 0 or shape[-1] < 1:
            _refuse("Rowscale.empty", f"shape {tuple(shape)}")
        n, cols = (shape[0] if dims == 2 else shape[0] * shape[1]), shape[-1]
        if n > _MAX_ROWS or cols > _MAX_ROWS:
            _refuse("Rowscale.empty", f"shape {tuple(shape)}", "SHAPE")
        pitch = (cols + 15) & ~15
        dev = device if device is not None else torch.cuda.current_device()
        self = cls.__new__(cls)   # (an allocation each: parts of one cost the host more)
        if pitch == cols:
            codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device=dev)
        else:
            codes = torch.empty_strided(shape, (pitch, 1) if dims == 2 else (shape[1] * pitch, pitch, 1),
                                        dtype=torch.float8_e4m3fn, device=dev)
        self._codes = codes
        self._scales = scales = torch.empty(shape[:-1], dtype=torch.float32, device=dev)
        self.shape, self.device = shape if isinstance(shape, tuple) else tuple(shape), codes.device
        self._c = _Rowscale(n, cols, pitch, codes.data_ptr(), scales.data_ptr())
        return self


def _flat(where: str, name: str, x):
    """x as a matrix: its experts' rows one after the other."""
    if x.dim() == 2:
        return x
    if x.dim() != 3:
        _refuse(where, f"{name} must be 2-d or 3-d")
    try:
        return x.view(-1, x.shape[-1]) if x.shape[-1] else x.flatten(0, 1)
    except RuntimeError:
        _refuse(where, f"{name}'s matrices must lie one after the other")


def _rowscale_c(where: str, q: Rowscale):
    """The library's view of a Rowscale (experts' rows one after the other)."""
    if q._c is None:
        codes = _flat(where, "codes", q.codes)
        ld = _rows(where, "codes", codes)
        if not q.scales.is_contiguous():
            _refuse(where, "scales must be dense")
        q._c = _Rowscale(codes.shape[0], codes.shape[1], ld, codes.data_ptr(), q.scales.data_ptr())
    return q._c


def _rowscale_rows(where: str, name: str, q: Rowscale, rows, cols: int, device):
    """Checks of a 2-d Rowscale; the library's view of it."""
    if len(q.shape) != 2 or q.device != device or device.type != "cuda":
        _refuse(where, f"{name} must be 2-d on {device}, got {len(q.shape)}-d on {q.device}")
    c = q._c or _rowscale_c(where, q)
    if c.cols != cols or (rows is not None and c.rows != rows):
        _refuse(where, f"{name} has shape {tuple(q.shape)}, expected {(rows, cols)}", "SHAPE")
    return c


def rowscale_quantize(x, out: Optional[Rowscale] = None, stream=None) -> Rowscale:
    """Code the rows of x (torch fp32 or bf16, 2-d, or 3-d matrices one after the other, dense rows, on the device) as
    a Rowscale with power-of-two scales; `out` reuses an existing one of the same shape."""
    _torch or _load_torch()
    where = "rowscale_quantize"
    dev = x.device
    ty = _dense_type(where, "x", x.dtype)
    flat = x if x.dim() == 2 else _flat(where, "x", x)
    ld = _rows(where, "x", flat)
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return rowscale_quantize(x, out)
    if out is None:
        out = Rowscale.empty(x.shape, dev)
    elif out.shape != x.shape or out.device != dev:
        _refuse(where, "out has another shape or device", "SHAPE")
    rc = _lib().bitsmoe_rowscale_quantize(flat.data_ptr(), ty, ld, out._c or _rowscale_c(where, out), _raw_stream(dev.index))
    if rc:
        _check(rc, "bitsmoe_rowscale_quantize")
    return out


def rowscale_dequantize(q: Rowscale, dtype=None, out=None, stream=None):
    """The values of a Rowscale as a torch tensor of its shape (float32, or bfloat16)."""
    torch = _torch or _load_torch()
    where = "rowscale_dequantize"
    dev = q.device
    if dev.type != "cuda":
        _refuse(where, "the rows must be on a CUDA device")
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return rowscale_dequantize(q, dtype, out)
    c = q._c or _rowscale_c(where, q)
    if out is None:
        out, ld = torch.empty(q.codes.shape, dtype=dtype if dtype is not None else torch.float32, device=dev), c.cols
        ptr = out.data_ptr()
    elif out.shape != q.shape:
        _refuse(where, f"out has shape {tuple(out.shape)}, expected {tuple(q.shape)}", "SHAPE")
    else:
        flat = _flat(where, "out", out)
        ld, ptr = _rows(where, "out", flat, None, None, dev), flat.data_ptr()
    rc = _lib().bitsmoe_rowscale_dequantize(c, ptr, _dense_type(where, "out", out.dtype), ld, _raw_stream(dev.index))
    if rc:
        _check(rc, "bitsmoe_rowscale_dequantize")
    return out


class Routing(NamedTuple):
    """What `route` returns (see bitsmoe_route): the tokens' experts and weights (T x top_k), where each expert's pairs
    begin (experts + 1), the pairs t * top_k + j in the order of their experts, and each pair's place there."""
    experts: object
    weights: object
    offsets: object
    pairs: object
    places: object


_ROUTE_WS = {}   # (T, experts, top_k) -> bytes of the workspace


def route(logits, top_k: int, renormalize: bool = True, stream=None) -> Routing:
    """Routing of the rows of logits (torch fp32, T x experts, on the device): the top_k largest (ties to the lower
    expert), weighted by the softmax over them (renormalize) or over all; a logit of -inf or NaN is never selected, and
    a token that has fewer others gets expert -1, weight 0 and place -1 for the rest."""
    torch = _torch or _load_torch()
    where = "route"
    dev = logits.device
    ld = _rows(where, "logits", logits, dtype=torch.float32)
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return route(logits, top_k, renormalize)
    T, E = logits.shape
    if not 1 <= top_k <= min(E, 32):
        _refuse(where, f"top_k is {top_k} of {E} experts (32 at most)")
    nws = _ROUTE_WS.get((T, E, top_k))
    if nws is None:
        if len(_ROUTE_WS) > 4096:
            _ROUTE_WS.clear()
        nws = _ROUTE_WS[T, E, top_k] = int(_lib().bitsmoe_route_workspace_bytes(T, E, top_k))
    # (an allocation each: parts of one cost the host more)
    i32 = torch.int32
    experts = torch.empty((T, top_k), dtype=i32, device=dev)
    places = torch.empty((T, top_k), dtype=i32, device=dev)
    pairs = torch.empty(T * top_k, dtype=i32, device=dev)
    offsets = torch.empty(E + 1, dtype=i32, device=dev)
    weights = torch.empty((T, top_k), dtype=torch.float32, device=dev)
    ws = torch.empty(nws, dtype=torch.uint8, device=dev) if nws else None
    rc = _lib().bitsmoe_route(logits.data_ptr(), ld, T, E, top_k, 1 if renormalize else 0, experts.data_ptr(),
                              weights.data_ptr(), offsets.data_ptr(), pairs.data_ptr(), places.data_ptr(),
                              ws.data_ptr() if nws else None, nws, _raw_stream(dev.index))
    if rc:
        _check(rc, "bitsmoe_route")
    return Routing(experts, weights, offsets, pairs, places)


def _matrices(where: str, name: str, w, device=None):
    """The library's view of the experts' matrices: a 3-d bf16 tensor or a Rowscale of 3-d codes."""
    if isinstance(w, Rowscale):
        data, ty, scales = w.codes, _E4M3, w.scales   # (kept: matrices are used for long)
    else:
        data, ty, scales = w, 1, None
        if w.dtype is not _torch.bfloat16:
            _refuse(where, f"{name} must be bfloat16 or a Rowscale, got {w.dtype}")
    if data.dim() != 3 or not data.is_cuda:
        _refuse(where, f"{name} must be a 3-d CUDA tensor (experts x rows x cols)")
    if device is not None and data.device != device:
        _refuse(where, f"{name} is on {data.device}, expected {device}")
    E, R, C = data.shape
    if R > _MAX_ROWS or C > _MAX_ROWS or E > _MAX_ROWS:
        _refuse(where, f"{name} has shape {tuple(data.shape)}", "SHAPE")
    eld, ld, step = data.stride()
    if step != 1 and C > 1:
        _refuse(where, f"{name} must have dense rows (stride 1 along them)")
    if R <= 1:
        ld = C
    elif ld < C:
        _refuse(where, f"{name}'s rows overlap (stride {ld})")
    return _ExpertMatrices(ty, E, R, C, ld, eld, scales.stride(0) if scales is not None else 0, data.data_ptr(),
                           scales.data_ptr() if scales is not None else None)


def _ints(where: str, name: str, v, n, device):
    if v.dim() != 1 or (n is not None and v.shape[0] != n):
        _refuse(where, f"{name} has shape {tuple(v.shape)}, expected {(n,)}", "SHAPE")
    if v.dtype is not _torch.int32 or v.device != device or (v.shape[0] > 1 and v.stride(0) != 1):
        _refuse(where, f"{name} must be a dense int32 vector on {device}")
    return v.data_ptr()


def expert_product(w, x, offsets, index=None, fan: int = 1, up=None, dtype=None, y=None, status=None, stream=None):
    """Products grouped by expert, ragged: y[p] = W_e x[q] for offsets[e] <= p < offsets[e + 1], with q = p, or
    index[p] // fan (see bitsmoe_expert_product); with `up` SiLU(W_e x) * (U_e x).

    w, up: the experts' matrices (torch bf16, experts x rows x cols, or a Rowscale of such codes); x: rows x cols of the
    same kind; offsets, index: int32 vectors (`route`'s offsets and pairs, with fan = top_k).  y (P x w's rows, P the
    length of index, or x's rows; float32 unless `dtype` or y says bfloat16): rows that no expert has are not written.
    float32 results are summed to nearest, and of large products take up to twice the time of bfloat16 ones.
    `status`: an optional int32 tensor of one element that receives a device-side timeout.  Rows and matrices on 16-byte
    boundaries are read fastest; of large products bf16 rows of x off them (up to four for each of y) are copied to a
    temporary first."""
    torch = _torch or _load_torch()
    where = "expert_product"
    coded = isinstance(w, Rowscale)
    if isinstance(x, Rowscale) != coded or (up is not None and isinstance(up, Rowscale) != coded):
        _refuse(where, "w, up and x must be of one kind, bf16 or Rowscale")
    dev = w.device
    if dev.type != "cuda":
        _refuse(where, "w must be on a CUDA device")
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return expert_product(w, x, offsets, index, fan, up, dtype, y, status)
    wc = _matrices(where, "w", w, dev)
    uc = _matrices(where, "up", up, dev) if up is not None else None
    if coded:
        xc = _rowscale_rows(where, "x", x, None, wc.cols, dev)
        x_rows, x_ld, x_ptr, xs_ptr = xc.rows, xc.ld, xc.codes, xc.scales
    else:
        x_ld = _rows(where, "x", x, None, wc.cols, dev, torch.bfloat16)
        x_rows, x_ptr, xs_ptr = x.shape[0], x.data_ptr(), None
    off_ptr = _ints(where, "offsets", offsets, wc.experts + 1, dev)
    P, idx_ptr = x_rows, None
    if index is not None:
        idx_ptr = _ints(where, "index", index, None, dev)
        P = index.shape[0]
        if P > _MAX_ROWS:
            _refuse(where, f"index has {P} entries", "SHAPE")
    if not 1 <= fan <= _MAX_ROWS:
        _refuse(where, f"fan is {fan}")
    # Large products: rows of x off 16-byte boundaries are brought onto them first, unless x has many more than y (us with and
    # without; bf16 results of one matrix of 4096 x 4095 on boundaries: 1100 rows of y, as many of x 43 and 141, 4 times as many
    # 54 and 163, 64 times 247 and 165; gate and up of 16 experts of 1001 x 2041 off them: 4800 rows 265 and 422, 4 times 285
    # and 421, 64 times 716 and 423; 600 rows, so below the size, 144 and 166).
    if (not coded and 0 < x_rows <= 4 * P and (x_ptr % 16 or (x_ld % 8 and x_rows > 1))
            and P * wc.rows * wc.cols > 1 << 31):
        ld = (wc.cols + 7) & ~7
        rows = torch.empty((x_rows, ld), dtype=torch.bfloat16, device=dev)
        _check(_lib().bitsmoe_microscale_align(x_ptr, x_ld, x_rows, wc.cols, rows.data_ptr(), ld, _raw_stream(dev.index)),
               "bitsmoe_microscale_align")
        x_ptr, x_ld = rows.data_ptr(), ld
    st_ptr = None
    if status is not None:
        if status.dtype != torch.int32 or status.numel() != 1 or status.device != dev:
            _refuse(where, "status must be one int32 on the operands' device")
        st_ptr = status.data_ptr()
    if y is None:
        y, y_ld = torch.empty((P, wc.rows), dtype=dtype if dtype is not None else torch.float32, device=dev), max(wc.rows, 1)
    else:
        y_ld = _rows(where, "y", y, P, wc.rows, dev)
    args = _ExpertProductArgs(_addressof(wc), _addressof(uc) if uc is not None else None, x_ptr, xs_ptr, x_ld, x_rows, P,
                              off_ptr, idx_ptr, fan, _dense_type(where, "y", y.dtype), y.data_ptr(), y_ld, st_ptr)
    rc = _lib().bitsmoe_expert_product(args, _raw_stream(dev.index))
    if rc:
        _check(rc, "bitsmoe_expert_product")
    return y


def expert_combine(y, places, weights, base=None, dtype=None, out=None, stream=None):
    """The weighted sum that ends a layer of experts: out[t] = base[t] + sum_j weights[t][j] y[places[t][j]] (places as
    `route` gives them: a place outside y's rows adds nothing).  y: rows x D (fp32 or bf16); places int32 and weights
    fp32, T x top_k; base: T x D of out's type (it may be out itself); out: fp32 unless `dtype`, base or out says bf16."""
    torch = _torch or _load_torch()
    where = "expert_combine"
    dev = y.device
    y_ld = _rows(where, "y", y)
    if stream is not None or _current() != dev.index:
        with _elsewhere(where, dev, stream):
            return expert_combine(y, places, weights, base, dtype, out)
    P, D = y.shape
    if places.dim() != 2 or places.shape != weights.shape:
        _refuse(where, f"places have shape {tuple(places.shape)}, weights {tuple(weights.shape)}", "SHAPE")
    if places.dtype is not torch.int32 or weights.dtype is not torch.float32:
        _refuse(where, "places must be int32, weights float32")
    if places.device != dev or weights.device != dev or not places.is_contiguous() or not weights.is_contiguous():
        _refuse(where, f"places and weights must be dense on {dev}")
    T, k = places.shape
    if T > _MAX_ROWS:
        _refuse(where, f"{T} tokens", "SHAPE")
    if out is None:
        want = dtype if dtype is not None else base.dtype if base is not None else torch.float32
        out, out_ld = torch.empty((T, D), dtype=want, device=dev), D
    else:
        out_ld = _rows(where, "out", out, T, D, dev)
    base_ptr, base_ld = None, 0
    if base is not None:
        base_ld, base_ptr = _rows(where, "base", base, T, D, dev, out.dtype), base.data_ptr()
    rc = _lib().bitsmoe_expert_combine(y.data_ptr(), _dense_type(where, "y", y.dtype), y_ld, P, places.data_ptr(),
                                       weights.data_ptr(), T, k, D, base_ptr, base_ld, out.data_ptr(),
                                       _dense_type(where, "out", out.dtype), out_ld, _raw_stream(dev.index))
    if rc:
        _check(rc, "bitsmoe_expert_combine")
    return out


def bitsmoe_debug_single_token_kernel(which: int) -> None:
    """Testing hook: 1 keeps single-token forwards on the fused kernel without clusters, 2 takes the
    clustered one wherever it fits, 0 restores the automatic choice."""
    _check(_lib().bitsmoe_debug_single_token_kernel(which), "bitsmoe_debug_single_token_kernel")


def bitsmoe_debug_bounds(on: int) -> None:
    """Testing hook: debug bounds checks of the single-token kernels' staging records (and a
    zero-filled slack after the image of layers packed while it is on); 2: also an impossible
    count in the routing that the expert kernels of several tokens check."""
    _check(_lib().bitsmoe_debug_bounds(on), "bitsmoe_debug_bounds")


def bitsmoe_debug_shift_expert_records(layer, e: int, delta: int) -> None:
    """Testing hook: shift the code offsets of expert e's gate/up staging records by delta bytes."""
    _check(_lib().bitsmoe_debug_shift_expert_records(layer.handle, e, delta), "bitsmoe_debug_shift_expert_records")


def bitsmoe_debug_wait_limit(skip_arrival: int, spin_clocks: int) -> None:
    """Testing hook: bound the kernels' waits to spin_clocks SM clocks (0: default) and let block 0 skip
    an arrival (skip_arrival = 1), or the plan of its tiles in products grouped by expert (2)."""
    _check(_lib().bitsmoe_debug_wait_limit(skip_arrival, spin_clocks), "bitsmoe_debug_wait_limit")
