"""ctypes binding of ``liblgn.so`` (declared in ``include/lgn.h``).

Argument marshalling only: torch supplies device memory and the current CUDA
stream, every step of the path runs in the library's kernels.  There is no CPU
fallback: if the shared library is missing or cannot be loaded, importing this
module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, NamedTuple, Optional, Sequence, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblgn.so")      # the in-tree build, and nothing else

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} not found: build it with `python -m paper_2006_08173_b200.build` "
        "(nvcc, sm_100a); this package has no CPU fallback")
_lib = C.CDLL(LIB_PATH)

LGN_OK = 0
F32, BF16 = 0, 1
ROUND_NEAREST, ROUND_STOCHASTIC = 0, 1
MODE_PRUNE, MODE_QUANTIZE = 0, 1
SCALE_CENTRED, SCALE_FROM_MAX = 0, 1
E4M3, E5M2 = 0, 1
BLOCK_ROW, BLOCK_SQUARE = 0, 1


class StatsT(C.Structure):
    _fields_ = [("n", C.c_uint64), ("nnz", C.c_uint64), ("sum_ln", C.c_double),
                ("sum_ln2", C.c_double), ("mu", C.c_double), ("sigma", C.c_double)]


class FpFormatT(C.Structure):
    _fields_ = [("nbits", C.c_int32), ("exp_bits", C.c_int32), ("man_bits", C.c_int32),
                ("scale_exp", C.c_int32)]


class AllocLayerT(C.Structure):
    _fields_ = [("n", C.c_uint64), ("sigma", C.c_double), ("zero_frac", C.c_double), ("k", C.c_double),
                ("min_cos", C.c_double)]


class QuantileT(C.Structure):
    _fields_ = [("value", C.c_float), ("pad", C.c_uint32), ("nnz", C.c_uint64)]


class LayerT(C.Structure):
    _fields_ = [("g", C.c_void_p), ("out", C.c_void_p), ("n", C.c_uint64),
                ("dt", C.c_int32), ("mode", C.c_int32), ("S", C.c_double),
                ("nbits", C.c_int32), ("rounding", C.c_int32), ("seed", C.c_uint64),
                ("use_override", C.c_int32), ("scale_mode", C.c_int32),
                ("mu_override", C.c_double), ("sigma_override", C.c_double), ("right_mode", C.c_void_p),
                ("counters", C.c_int32), ("reserved", C.c_int32)]


class LayerResultT(C.Structure):
    _fields_ = [("stats", StatsT), ("tau", C.c_double), ("fmt", FpFormatT),
                ("status", C.c_int32), ("max_abs", C.c_float), ("n_right_mode", C.c_uint64),
                ("n_zero_out", C.c_uint64), ("n_snapped", C.c_uint64), ("n_saturated", C.c_uint64),
                ("n_underflow", C.c_uint64)]


class GradT(C.Structure):
    _fields_ = [("g", C.c_void_p), ("out", C.c_void_p), ("n", C.c_uint64), ("dt", C.c_int32), ("reserved", C.c_int32)]


class NormT(C.Structure):
    _fields_ = [("norm", C.c_float), ("coef", C.c_float), ("n_nonfinite", C.c_uint64), ("sum_sq", C.c_double)]


assert C.sizeof(GradT) == 32 and C.sizeof(NormT) == 24
assert C.sizeof(StatsT) == 48 and C.sizeof(LayerT) == 96 and C.sizeof(LayerResultT) == 120

_vp, _u64, _sz, _dbl, _i32 = C.c_void_p, C.c_uint64, C.c_size_t, C.c_double, C.c_int
_lib.lgn_status_string.argtypes = [_i32]
_lib.lgn_status_string.restype = C.c_char_p
_lib.lgn_workspace_bytes.argtypes = [C.POINTER(_u64), _i32]
_lib.lgn_workspace_bytes.restype = _sz
_lib.lgn_codes_bytes.argtypes = [_u64, _i32]
_lib.lgn_codes_bytes.restype = _sz
_lib.lgn_stats.argtypes = [_vp, _u64, _i32, _vp, _vp, _sz, _vp]
_lib.lgn_stats.restype = _i32
_lib.lgn_threshold.argtypes = [_dbl, _dbl, _dbl, _dbl, C.POINTER(_dbl)]
_lib.lgn_threshold.restype = _i32
_lib.lgn_snap_threshold.argtypes = [_dbl, _i32]
_lib.lgn_snap_threshold.restype = _dbl
_lib.lgn_fp_format.argtypes = [_dbl, _dbl, _i32, C.POINTER(FpFormatT)]
_lib.lgn_fp_format.restype = _i32
_lib.lgn_cosine_similarity.argtypes = [_dbl, _dbl, _dbl, _dbl, C.POINTER(_dbl)]
_lib.lgn_cosine_similarity.restype = _i32
_lib.lgn_allocate_sparsity.argtypes = [C.POINTER(AllocLayerT), _i32, _i32, _dbl, _dbl, C.POINTER(_dbl), C.POINTER(_dbl)]
_lib.lgn_allocate_sparsity.restype = _i32
_lib.lgn_quantile_workspace_bytes.argtypes = []
_lib.lgn_quantile_workspace_bytes.restype = _sz
_lib.lgn_quantile.argtypes = [_vp, _u64, _i32, _dbl, _vp, _vp, _sz, _vp]
_lib.lgn_quantile.restype = _i32
_lib.lgn_combine_stats.argtypes = [C.POINTER(StatsT), _i32, C.POINTER(StatsT)]
_lib.lgn_combine_stats.restype = _i32
_lib.lgn_scale_from_max.argtypes = [_dbl, _i32, C.POINTER(C.c_int32)]
_lib.lgn_scale_from_max.restype = _i32
_lib.lgn_prune.argtypes = [_vp, _vp, _u64, _i32, _dbl, _u64, _vp]
_lib.lgn_prune.restype = _i32
_lib.lgn_quantize.argtypes = [_vp, _vp, _u64, _i32, C.POINTER(FpFormatT), _i32, _u64, _vp]
_lib.lgn_quantize.restype = _i32
_lib.lgn_compress_layers.argtypes = [C.POINTER(LayerT), _i32, _vp, _vp, _sz, _vp]
_lib.lgn_compress_layers.restype = _i32
_lib.lgn_host_staging_bytes.argtypes = [C.POINTER(LayerT), _i32]
_lib.lgn_host_staging_bytes.restype = _sz
_lib.lgn_compress_layers_host.argtypes = [C.POINTER(LayerT), _i32, C.POINTER(LayerResultT), _vp, _sz, _vp]
_lib.lgn_compress_layers_host.restype = _i32
_lib.lgn_selftest_wait_expires.argtypes = [C.POINTER(LayerT), _i32, _vp, _vp, _sz, _vp]
_lib.lgn_selftest_wait_expires.restype = _i32
_lib.lgn_prefix_blocks.argtypes = [_u64]
_lib.lgn_prefix_blocks.restype = _u64
_lib.lgn_prefix_bound_words.argtypes = [_u64, _i32]
_lib.lgn_prefix_bound_words.restype = _u64
_lib.lgn_prefix_workspace_bytes.argtypes = [_u64]
_lib.lgn_prefix_workspace_bytes.restype = _sz
_lib.lgn_prefix_encode.argtypes = [_vp, _u64, _i32, C.c_double, _u64, _i32, _vp, _vp, _u64, _vp, _vp, _sz, _vp]
_lib.lgn_prefix_encode.restype = _i32
_lib.lgn_prefix_decode.argtypes = [_vp, _vp, _u64, _i32, C.c_double, _vp, _vp, _vp]
_lib.lgn_prefix_decode.restype = _i32
_lib.lgn_dequantize.argtypes = [_vp, _u64, C.POINTER(FpFormatT), _i32, _vp, _vp]
_lib.lgn_dequantize.restype = _i32
_lib.lgn_launches_per_call.argtypes = [_i32]
_lib.lgn_launches_per_call.restype = _i32
_lib.lgn_stats_static_scratch.argtypes = [_vp, _u64, _i32, _vp, _vp]
_lib.lgn_stats_static_scratch.restype = _i32
STATS_STATIC_MAX_ELEMS = 1 << 28
_lib.lgn_fp8_codes_bytes.argtypes = [_u64, _u64]
_lib.lgn_fp8_codes_bytes.restype = _sz
_lib.lgn_fp8_scales_bytes.argtypes = [_u64, _u64]
_lib.lgn_fp8_scales_bytes.restype = _sz
_lib.lgn_fp8_quantize.argtypes = [_vp, _u64, _u64, _u64, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp]
_lib.lgn_fp8_quantize.restype = _i32
_lib.lgn_fp8_matmul.argtypes = [_vp, _vp, _i32, _vp, _vp, _i32, _u64, _u64, _u64, _vp, _u64, _i32, _i32, _vp, _vp]
_lib.lgn_fp8_matmul.restype = _i32
_lib.lgn_selftest_matmul_wait_expires.argtypes = [_vp, _vp, _vp, _vp, _u64, _u64, _u64, _vp, _i32, _vp, _vp]
_lib.lgn_selftest_matmul_wait_expires.restype = _i32
_lib.lgn_embedding.argtypes = [_vp, _u64, _u64, _u64, _i32, _vp, _i32, _u64, _dbl, _vp, _u64, _i32, _vp, _vp]
_lib.lgn_embedding.restype = _i32
_lib.lgn_embedding_grad_workspace_bytes.argtypes = [_u64, _u64, _u64]
_lib.lgn_embedding_grad_workspace_bytes.restype = _sz
_lib.lgn_embedding_grad.argtypes = [_vp, _u64, _i32, _vp, _i32, _u64, _u64, _u64, _dbl, C.c_int64, _vp, _u64, _i32, _i32, _vp, _sz, _vp]
_lib.lgn_embedding_grad.restype = _i32
_lib.lgn_clip_workspace_bytes.argtypes = [_i32]
_lib.lgn_clip_workspace_bytes.restype = _sz
_lib.lgn_grad_norm.argtypes = [C.POINTER(GradT), _i32, _vp, _vp, _sz, _vp]
_lib.lgn_grad_norm.restype = _i32
_lib.lgn_clip_grad_norm.argtypes = [C.POINTER(GradT), _i32, _dbl, _vp, _vp, _sz, _vp]
_lib.lgn_clip_grad_norm.restype = _i32
_lib.lgn_clip_apply.argtypes = [C.POINTER(GradT), _i32, _dbl, _vp, _vp]
_lib.lgn_clip_apply.restype = _i32


_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
_uint8 = torch.uint8
_DT_CODE = {torch.float32: F32, torch.bfloat16: BF16}


class LgnError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {_lib.lgn_status_string(code).decode()} (status {code})")


def _check(code: int, where: str) -> None:
    if code != LGN_OK:
        raise LgnError(code, where)


def raw():
    """The loaded ctypes library (for tests of the ABI itself)."""
    return _lib


def dtype_code(t: torch.Tensor) -> int:
    code = _DT_CODE.get(t.dtype)
    if code is None:
        raise TypeError(f"gradient tensors are float32 or bfloat16, got {t.dtype}")
    return code


def _dev(t: torch.Tensor, what: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _word(t: torch.Tensor, size: int, what: str) -> int:
    """The address of a tensor that one value of ``size`` bytes is written to."""
    at = _dev(t, what)
    if t.numel() * t.element_size() < size:
        raise ValueError(f"{what} must hold {size} bytes")
    return at


def _stream(stream) -> int:
    if stream is None:          # the current stream of the current device, without a Stream object (3.5 us -> 0.2 us a call)
        return _raw_stream(_current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _empty(shape, dtype: torch.dtype, device, stream) -> torch.Tensor:
    """Uninitialised memory that belongs to the stream the call runs on: torch hands a freed block out again as soon
    as the stream it was allocated on allows, whatever other streams still do with it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        raise ValueError("outputs and workspaces have to be given when the stream is a raw handle")
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _elsewhere(device: int, stream, *others) -> bool:
    """Whether ``device``, that of a call's first tensor, is not the current one, so that the call has to be made under
    torch.cuda.device(device).  ``others``: the device numbers of its other tensors, None for those not given."""
    for d in others:
        if d is not None and d != device:
            raise ValueError(f"tensors on different devices: {device} and {d}")
    if stream is not None and isinstance(stream, torch.cuda.Stream) and stream.device_index != device:
        raise ValueError(f"a stream of device {stream.device_index} for tensors on device {device}")
    return device != _current_device()


# --------------------------------------------------------------------------- sizes
def lgn_workspace_bytes(n_per_layer: Sequence[int]) -> int:
    arr = (_u64 * max(1, len(n_per_layer)))(*n_per_layer)
    return int(_lib.lgn_workspace_bytes(arr, len(n_per_layer)))


def lgn_launches_per_call(num_layers: int) -> int:
    return int(_lib.lgn_launches_per_call(num_layers))


def lgn_codes_bytes(n: int, nbits: int) -> int:
    return int(_lib.lgn_codes_bytes(n, nbits))


def new_workspace(n_per_layer: Sequence[int], device) -> torch.Tensor:
    return torch.empty(max(16, lgn_workspace_bytes(n_per_layer)), dtype=torch.uint8, device=device)


# --------------------------------------------------------------------------- host closed forms
def lgn_threshold(mu: float, sigma: float, zero_frac: float, S: float) -> float:
    tau = _dbl()
    _check(_lib.lgn_threshold(mu, sigma, zero_frac, S, C.byref(tau)), "lgn_threshold")
    return tau.value


def lgn_snap_threshold(tau: float, dt: int) -> float:
    return float(_lib.lgn_snap_threshold(tau, dt))


def lgn_fp_format(mu: float, sigma: float, nbits: int) -> Dict[str, int]:
    f = FpFormatT()
    _check(_lib.lgn_fp_format(mu, sigma, nbits, C.byref(f)), "lgn_fp_format")
    return {"nbits": f.nbits, "exp_bits": f.exp_bits, "man_bits": f.man_bits, "scale_exp": f.scale_exp}


def lgn_cosine_similarity(mu: float, sigma: float, k: float, tau: float) -> float:
    c = _dbl()
    _check(_lib.lgn_cosine_similarity(mu, sigma, k, tau, C.byref(c)), "lgn_cosine_similarity")
    return c.value


def lgn_allocate_sparsity(layers: Sequence[Dict[str, float]], num_deep: int, S: float, s_max: float):
    """``layers``: dicts with n, sigma, zero_frac, k and (deep layers) min_cos, deepest first.
    Returns (per-layer sparsity list, element-weighted mean allocated)."""
    L = len(layers)
    arr = (AllocLayerT * max(1, L))(*[AllocLayerT(int(a["n"]), float(a["sigma"]), float(a["zero_frac"]),
                                                  float(a.get("k", 0.0)), float(a.get("min_cos", 0.0))) for a in layers])
    out = (_dbl * max(1, L))()
    mean = _dbl()
    _check(_lib.lgn_allocate_sparsity(arr, L, num_deep, S, s_max, out, C.byref(mean)), "lgn_allocate_sparsity")
    return [out[i] for i in range(L)], mean.value


def lgn_quantile_workspace_bytes() -> int:
    return int(_lib.lgn_quantile_workspace_bytes())


def lgn_quantile(g: torch.Tensor, q: float, ws: Optional[torch.Tensor] = None, stream=None) -> Dict[str, float]:
    """The order statistic of rank ceil(q nnz) of |g| over the nonzeros (synchronises to read it back)."""
    ws = ws if ws is not None else torch.empty(lgn_quantile_workspace_bytes(), dtype=torch.uint8, device=g.device)
    out = torch.empty(16, dtype=torch.uint8, device=g.device)
    _check(_lib.lgn_quantile(_dev(g, "g") if g.numel() else None, g.numel(), dtype_code(g), float(q), _dev(out, "out"),
                             _dev(ws, "ws"), ws.numel(), _stream(stream)), "lgn_quantile")
    r = QuantileT.from_buffer_copy(out.cpu().numpy().tobytes())
    return {"value": float(r.value), "nnz": int(r.nnz)}


def lgn_combine_stats(parts: Sequence[Dict[str, float]]) -> Dict[str, float]:
    """Statistics of the union of tensors from each one's n, nnz, sum_ln, sum_ln2."""
    arr = (StatsT * max(1, len(parts)))(*[StatsT(int(p["n"]), int(p["nnz"]), float(p["sum_ln"]), float(p["sum_ln2"]),
                                                 0.0, 0.0) for p in parts])
    out = StatsT()
    _check(_lib.lgn_combine_stats(arr, len(parts), C.byref(out)), "lgn_combine_stats")
    return {"n": out.n, "nnz": out.nnz, "sum_ln": out.sum_ln, "sum_ln2": out.sum_ln2, "mu": out.mu, "sigma": out.sigma}


def lgn_scale_from_max(max_abs: float, exp_bits: int) -> int:
    e = C.c_int32()
    _check(_lib.lgn_scale_from_max(float(max_abs), int(exp_bits), C.byref(e)), "lgn_scale_from_max")
    return e.value


def _fmt_struct(fmt: Dict[str, int]) -> FpFormatT:
    return FpFormatT(fmt["nbits"], fmt["exp_bits"], fmt["man_bits"], fmt["scale_exp"])


# --------------------------------------------------------------------------- device entry points
def lgn_stats_async(g: torch.Tensor, out_dev: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """Enqueue the statistics pass; ``out_dev`` (>= 48 bytes, uint8, CUDA) receives one lgn_stats_t."""
    _check(_lib.lgn_stats(_dev(g, "g"), g.numel(), dtype_code(g), _dev(out_dev, "out_dev"),
                          _dev(ws, "ws"), ws.numel() * ws.element_size(), _stream(stream)), "lgn_stats")


def lgn_stats_static_scratch_async(g: torch.Tensor, out_dev: torch.Tensor, stream=None) -> None:
    """lgn_stats without a workspace argument: the scratch is an array inside
    the library (at most STATS_STATIC_MAX_ELEMS elements; calls that may overlap
    on the GPU must not share a device).  Allocates nothing."""
    _check(_lib.lgn_stats_static_scratch(_dev(g, "g") if g.numel() else None, g.numel(), dtype_code(g),
                                         _dev(out_dev, "out_dev"), _stream(stream)), "lgn_stats_static_scratch")


def read_stats(out_dev: torch.Tensor) -> Dict[str, float]:
    raw_bytes = out_dev.cpu().numpy().tobytes()[:C.sizeof(StatsT)]
    st = StatsT.from_buffer_copy(raw_bytes)
    return {"n": st.n, "nnz": st.nnz, "sum_ln": st.sum_ln, "sum_ln2": st.sum_ln2,
            "mu": st.mu, "sigma": st.sigma}


def lgn_stats(g: torch.Tensor, ws: Optional[torch.Tensor] = None, stream=None) -> Dict[str, float]:
    """Statistics of one tensor, read back to the host (synchronises)."""
    ws = ws if ws is not None else new_workspace([g.numel()], g.device)
    out = torch.empty(64, dtype=torch.uint8, device=g.device)
    lgn_stats_async(g, out, ws, stream)
    return read_stats(out)


def lgn_prune(g: torch.Tensor, tau: float, seed: int, out: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    out = out if out is not None else torch.empty_like(g)
    _check(_lib.lgn_prune(_dev(g, "g"), _dev(out, "out"), g.numel(), dtype_code(g), float(tau),
                          int(seed), _stream(stream)), "lgn_prune")
    return out


def lgn_quantize(g: torch.Tensor, fmt: Dict[str, int], rounding: int, seed: int,
                 out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Packed codes as a uint8 tensor of lgn_codes_bytes(n, nbits) bytes."""
    if out is None:
        out = torch.empty(max(16, lgn_codes_bytes(g.numel(), fmt["nbits"])), dtype=torch.uint8, device=g.device)
    f = _fmt_struct(fmt)
    _check(_lib.lgn_quantize(_dev(g, "g"), _dev(out, "codes"), g.numel(), dtype_code(g), C.byref(f),
                             int(rounding), int(seed), _stream(stream)), "lgn_quantize")
    return out


def lgn_dequantize(codes: torch.Tensor, n: int, fmt: Dict[str, int], out: torch.Tensor, stream=None) -> torch.Tensor:
    """Decode ``n`` packed codes (uint8 CUDA tensor) into ``out`` (float32 or bfloat16, n elements)."""
    if out.numel() != n:
        raise ValueError("out must hold n elements")
    if codes.numel() * codes.element_size() < lgn_codes_bytes(n, fmt["nbits"]):
        raise ValueError("codes shorter than lgn_codes_bytes(n, nbits)")
    f = _fmt_struct(fmt)
    _check(_lib.lgn_dequantize(_dev(codes, "codes") if n else None, n, C.byref(f), dtype_code(out),
                               _dev(out, "out") if n else None, _stream(stream)), "lgn_dequantize")
    return out


def make_layer(g: torch.Tensor, out: torch.Tensor, mode: int, S: float = 0.0, nbits: int = 0,
               rounding: int = ROUND_NEAREST, seed: int = 0, mu_override: Optional[float] = None,
               sigma_override: Optional[float] = None, scale_mode: int = SCALE_CENTRED,
               right_mode: Optional[torch.Tensor] = None, counters: bool = False) -> LayerT:
    """``right_mode``: uint8/bool CUDA tensor of g.numel() bytes (bi-modal pruning), or None.
    ``counters``: have the apply pass fill n_zero_out .. n_underflow of the layer's result."""
    use = mu_override is not None and sigma_override is not None
    mask = None
    if right_mode is not None:
        if right_mode.element_size() != 1 or right_mode.numel() != g.numel():
            raise ValueError("right_mode must hold one byte per element of g")
        mask = _dev(right_mode, "right_mode") if g.numel() else None
    return LayerT(_dev(g, "g") if g.numel() else (g.data_ptr() or None),
                  _dev(out, "out") if out.numel() else (out.data_ptr() or None), g.numel(), dtype_code(g),
                  mode, float(S), int(nbits), int(rounding), int(seed), 1 if use else 0, int(scale_mode),
                  float(mu_override) if use else 0.0, float(sigma_override) if use else 0.0, mask,
                  1 if counters else 0, 0)


def lgn_compress_layers(layers: Sequence[LayerT], results_dev: torch.Tensor, ws: torch.Tensor,
                        stream=None) -> None:
    """Enqueue the grouped path.  ``results_dev``: uint8 CUDA tensor of at least
    120 bytes per layer; ``ws``: uint8 CUDA tensor of lgn_workspace_bytes(...)."""
    L = len(layers)
    arr = (LayerT * max(1, L))(*layers)
    if results_dev.numel() * results_dev.element_size() < L * C.sizeof(LayerResultT):
        raise ValueError("results_dev too small")
    _check(_lib.lgn_compress_layers(arr, L, _dev(results_dev, "results_dev"), _dev(ws, "ws"),
                                    ws.numel() * ws.element_size(), _stream(stream)), "lgn_compress_layers")


def lgn_selftest_wait_expires(layers: Sequence[LayerT], results_dev: torch.Tensor, ws: torch.Tensor,
                              stream=None) -> None:
    """lgn_compress_layers with one statistics tile of layer 0 withheld: layer 0
    must come back with status LGN_ERR_TIMEOUT after about a second."""
    L = len(layers)
    arr = (LayerT * max(1, L))(*layers)
    _check(_lib.lgn_selftest_wait_expires(arr, L, _dev(results_dev, "results_dev"), _dev(ws, "ws"),
                                          ws.numel() * ws.element_size(), _stream(stream)),
           "lgn_selftest_wait_expires")


def new_results(num_layers: int, device) -> torch.Tensor:
    return torch.zeros(max(1, num_layers) * C.sizeof(LayerResultT), dtype=torch.uint8, device=device)


def status_of(results_dev: torch.Tensor, k: int = 0) -> torch.Tensor:
    """Layer k's status as an int32 tensor of one element on the device (a view)."""
    at = (k * C.sizeof(LayerResultT) + LayerResultT.status.offset) // 4
    return results_dev.view(torch.int32)[at:at + 1]


def read_results(results_dev: torch.Tensor, num_layers: int) -> List[Dict]:
    """Host copy of the per-layer results (synchronises)."""
    buf = results_dev.cpu().numpy().tobytes()
    out = []
    for k in range(num_layers):
        r = LayerResultT.from_buffer_copy(buf[k * C.sizeof(LayerResultT):(k + 1) * C.sizeof(LayerResultT)])
        out.append({"n": r.stats.n, "nnz": r.stats.nnz, "sum_ln": r.stats.sum_ln, "sum_ln2": r.stats.sum_ln2,
                    "mu": r.stats.mu, "sigma": r.stats.sigma, "tau": r.tau,
                    "fmt": {"nbits": r.fmt.nbits, "exp_bits": r.fmt.exp_bits, "man_bits": r.fmt.man_bits,
                            "scale_exp": r.fmt.scale_exp},
                    "status": r.status, "max_abs": r.max_abs, "n_right_mode": r.n_right_mode,
                    "n_zero_out": r.n_zero_out, "n_snapped": r.n_snapped, "n_saturated": r.n_saturated,
                    "n_underflow": r.n_underflow})
    return out


# --------------------------------------------------------------------------- host-buffer form
def _result_dict(r: LayerResultT) -> Dict:
    return {"n": r.stats.n, "nnz": r.stats.nnz, "sum_ln": r.stats.sum_ln, "sum_ln2": r.stats.sum_ln2,
            "mu": r.stats.mu, "sigma": r.stats.sigma, "tau": r.tau,
            "fmt": {"nbits": r.fmt.nbits, "exp_bits": r.fmt.exp_bits, "man_bits": r.fmt.man_bits,
                    "scale_exp": r.fmt.scale_exp},
            "status": r.status, "max_abs": r.max_abs, "n_right_mode": r.n_right_mode,
            "n_zero_out": r.n_zero_out, "n_snapped": r.n_snapped, "n_saturated": r.n_saturated,
            "n_underflow": r.n_underflow}


def make_host_layer(g: torch.Tensor, out: torch.Tensor, mode: int, **kw) -> LayerT:
    """Descriptor whose g/out are HOST tensors (pinned memory recommended)."""
    if g.is_cuda or out.is_cuda or not g.is_contiguous() or not out.is_contiguous():
        raise ValueError("host layers take contiguous CPU tensors")
    lay = LayerT(g.data_ptr() or None, out.data_ptr() or None, g.numel(), dtype_code(g), mode,
                 float(kw.get("S", 0.0)), int(kw.get("nbits", 0)), int(kw.get("rounding", ROUND_NEAREST)),
                 int(kw.get("seed", 0)), 0, int(kw.get("scale_mode", SCALE_CENTRED)), 0.0, 0.0,
                 (kw["right_mode"].data_ptr() or None) if kw.get("right_mode") is not None else None,
                 1 if kw.get("counters") else 0, 0)
    return lay


def lgn_host_staging_bytes(layers: Sequence[LayerT]) -> int:
    arr = (LayerT * max(1, len(layers)))(*layers)
    return int(_lib.lgn_host_staging_bytes(arr, len(layers)))


def lgn_compress_layers_host(layers: Sequence[LayerT], dev_buf: torch.Tensor, stream=None) -> List[Dict]:
    """Host tensors in, host tensors out; copies and the kernel run inside the
    call, which returns when everything has landed."""
    L = len(layers)
    arr = (LayerT * max(1, L))(*layers)
    res = (LayerResultT * max(1, L))()
    _check(_lib.lgn_compress_layers_host(arr, L, res, _dev(dev_buf, "dev_buf"),
                                         dev_buf.numel() * dev_buf.element_size(), _stream(stream)),
           "lgn_compress_layers_host")
    return [_result_dict(res[k]) for k in range(L)]


# --------------------------------------------------------------------------- prefix code (appendix "Encoding")
PREFIX_BLOCK = 2048


def lgn_prefix_blocks(n: int) -> int:
    return int(_lib.lgn_prefix_blocks(n))


def lgn_prefix_bound_words(n: int, dtype_code_: int) -> int:
    return int(_lib.lgn_prefix_bound_words(n, dtype_code_))


def lgn_prefix_workspace_bytes(n: int) -> int:
    return int(_lib.lgn_prefix_workspace_bytes(n))


def lgn_prefix_encode(g: torch.Tensor, tau: float, seed: int, apply_prune: bool, stream_dev: torch.Tensor,
                      off_dev: torch.Tensor, ws: torch.Tensor, tau_from_dev: Optional[int] = None,
                      stream=None) -> None:
    """``stream_dev``: int32/uint32 CUDA tensor (capacity = its length in words);
    ``off_dev``: int64 CUDA tensor of lgn_prefix_blocks(n) + 1 entries;
    ``tau_from_dev``: device address of a layer result record, or None."""
    if off_dev.numel() < lgn_prefix_blocks(g.numel()) + 1 or off_dev.element_size() != 8:
        raise ValueError("off_dev too small")
    if stream_dev.element_size() != 4:
        raise ValueError("stream_dev must hold 32-bit words")
    _check(_lib.lgn_prefix_encode(_dev(g, "g") if g.numel() else None, g.numel(), dtype_code(g), float(tau), int(seed),
                                  1 if apply_prune else 0, tau_from_dev,
                                  _dev(stream_dev, "stream_dev") if stream_dev.numel() else None, stream_dev.numel(),
                                  _dev(off_dev, "off_dev"), _dev(ws, "ws"), ws.numel() * ws.element_size(),
                                  _stream(stream)), "lgn_prefix_encode")


def lgn_prefix_decode(stream_dev: torch.Tensor, off_dev: torch.Tensor, out: torch.Tensor, tau: float,
                      tau_from_dev: Optional[int] = None, stream=None) -> torch.Tensor:
    _check(_lib.lgn_prefix_decode(_dev(stream_dev, "stream_dev") if stream_dev.numel() else None,
                                  _dev(off_dev, "off_dev"), out.numel(), dtype_code(out), float(tau), tau_from_dev,
                                  _dev(out, "out") if out.numel() else None, _stream(stream)), "lgn_prefix_decode")
    return out


# --------------------------------------------------------------------------- 8-bit matrix product
class Fp8Operand:
    """A matrix of ``rows`` x ``k`` in 8-bit codes with one scale per block of 128 along k.

    codes   uint8, lgn_fp8_codes_bytes(rows, k), rows padded to a multiple of 16
    scales  uint8, lgn_fp8_scales_bytes(rows, k), in the order lgn.h describes"""
    __slots__ = ("rows", "k", "fmt", "_codes", "_scales", "_buffer", "_codes_ptr", "_scales_ptr", "_device")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, rows: int, k: int, fmt: int):
        need_codes, need_scales = _fp8_bytes(rows, k)
        for t, need, what in ((codes, need_codes, "codes"), (scales, need_scales, "scales")):
            if t.dtype != _uint8:
                raise TypeError(f"{what} are uint8")
            if _dev(t, what) and t.numel() < need:
                raise ValueError(f"{what} shorter than the extents need")
        self.rows, self.k, self.fmt, self._codes, self._scales, self._buffer = rows, k, fmt, codes, scales, None
        self._codes_ptr, self._scales_ptr = codes.data_ptr(), scales.data_ptr()
        self._device = codes.get_device()
        if scales.get_device() != self._device:
            raise ValueError("codes and scales on different devices")

    @classmethod
    def empty(cls, rows: int, k: int, fmt: int, device, stream=None) -> "Fp8Operand":
        """Uninitialised, codes and scales in one allocation; for use on ``stream`` (default: the current one)."""
        total = rows * ((k + 15) & -16) + ((rows + 127) >> 7) * ((k + 511) >> 9) * 512 + 16         # as in _fp8_bytes
        return cls._of_buffer(torch.empty(total, dtype=_uint8, device=device) if stream is None else _empty(total, _uint8, device, stream), rows, k, fmt)

    @classmethod
    def _of_buffer(cls, buffer: torch.Tensor, rows: int, k: int, fmt: int) -> "Fp8Operand":
        """The operand in an allocation that empty() made, or in a copy of it."""
        if not buffer.is_cuda:
            raise ValueError("operands are CUDA memory")
        o = cls.__new__(cls)
        o.rows, o.k, o.fmt, o._buffer = rows, k, fmt, buffer
        o._codes_ptr = at = buffer.data_ptr()
        o._scales_ptr = at + rows * ((k + 15) & -16)
        o._device = buffer.get_device()
        return o

    @property
    def codes(self) -> torch.Tensor:
        return self._codes if self._buffer is None else self._buffer[:max(16, _fp8_bytes(self.rows, self.k)[0])]

    @property
    def scales(self) -> torch.Tensor:
        if self._buffer is None:
            return self._scales
        codes, scales = _fp8_bytes(self.rows, self.k)
        return self._buffer[codes:codes + max(16, scales)]

    @property
    def device(self) -> torch.device:
        return (self._codes if self._buffer is None else self._buffer).device

    def _replace(self, **kw) -> "Fp8Operand":
        return Fp8Operand(*(kw.get(n, getattr(self, n)) for n in ("codes", "scales", "rows", "k", "fmt")))


def _matrix3(t: torch.Tensor, what: str) -> Tuple[int, int, int]:
    """Rows, columns and leading dimension of a CUDA matrix whose rows are contiguous."""
    shape = t.shape
    if len(shape) != 2 or not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA matrix")
    rows, cols = shape
    ld, step = t.stride()
    if rows == 0 or cols == 0:                             # strides without a meaning: an expanded scalar's are 0
        return rows, cols, cols or 1
    if cols > 1 and step != 1:
        raise ValueError(f"{what} must be a matrix with contiguous rows")
    if rows <= 1:
        return rows, cols, cols or 1
    if ld < cols:
        raise ValueError(f"{what} must have rows that do not overlap")
    return rows, cols, ld


def _matrix(t: torch.Tensor, what: str) -> int:
    """The leading dimension alone."""
    return _matrix3(t, what)[2]


def _fp8_bytes(rows: int, k: int) -> Tuple[int, int]:
    """lgn_fp8_codes_bytes and lgn_fp8_scales_bytes, without two calls into the library."""
    return rows * ((k + 15) & -16), ((rows + 127) >> 7) * ((k + 511) >> 9) * 512


def new_fp8_operand(rows: int, k: int, fmt: int, device) -> Fp8Operand:
    return Fp8Operand.empty(rows, k, fmt, device)


def lgn_fp8_quantize(x: torch.Tensor, fmt: int = E4M3, block: int = BLOCK_ROW, rowwise: bool = True,
                     transposed: bool = False, out: Optional[Fp8Operand] = None, out_t: Optional[Fp8Operand] = None,
                     stream=None) -> Tuple[Optional[Fp8Operand], Optional[Fp8Operand]]:
    """(operand, operand of the transpose) of a matrix, each only if asked for (else None).  ``out`` and
    ``out_t`` are operands of the same extents to write to (new_fp8_operand)."""
    rows, cols, ld = _matrix3(x, "x")
    if not (rowwise or transposed):
        raise ValueError("neither the operand nor its transpose is asked for")
    device = x.get_device()
    if _elsewhere(device, stream, out._device if out is not None else None, out_t._device if out_t is not None else None):
        with torch.cuda.device(device):
            return lgn_fp8_quantize(x, fmt, block, rowwise, transposed, out, out_t, stream)
    q = t = pq = sq = pt = st = None
    if rowwise:
        if out is None:
            q = Fp8Operand.empty(rows, cols, fmt, x.device, stream)
        else:
            q = out
            if (q.rows, q.k, q.fmt) != (rows, cols, fmt):
                raise ValueError("out: extents or format differ from the matrix")
        pq, sq = q._codes_ptr, q._scales_ptr
    if transposed:
        if out_t is None:
            t = Fp8Operand.empty(cols, rows, fmt, x.device, stream)
        else:
            t = out_t
            if (t.rows, t.k, t.fmt) != (cols, rows, fmt):
                raise ValueError("out_t: extents or format differ from the transpose")
        pt, st = t._codes_ptr, t._scales_ptr
    code = _lib.lgn_fp8_quantize(x.data_ptr() or None, rows, cols, ld, dtype_code(x), fmt, block, pq, sq, pt, st,
                                 _raw_stream(device) if stream is None else _stream(stream))
    if code != LGN_OK:
        _check(code, "lgn_fp8_quantize")
    return q, t


def lgn_fp8_matmul(a: Fp8Operand, b: Fp8Operand, out: Optional[torch.Tensor] = None,
                   out_dtype: torch.dtype = torch.bfloat16, accumulate: bool = False,
                   status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[i, j] = sum over c of a[i, c] b[j, c] (+ out[i, j] with ``accumulate``)."""
    m, k, n = a.rows, a.k, b.rows
    if k != b.k:
        raise ValueError("operands contract over different extents")
    device = a._device
    if _elsewhere(device, stream, b._device, out.get_device() if out is not None else None, status.get_device() if status is not None else None):
        with torch.cuda.device(device):
            return lgn_fp8_matmul(a, b, out, out_dtype, accumulate, status, stream)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty((m, n), dtype=out_dtype, device=a.device) if stream is None else _empty((m, n), out_dtype, a.device, stream)
        ldo = n or 1
    else:
        if tuple(out.shape) != (m, n):
            raise ValueError("out must be a.rows x b.rows")
        ldo = _matrix(out, "out")
    code = _lib.lgn_fp8_matmul(a._codes_ptr, a._scales_ptr, a.fmt, b._codes_ptr, b._scales_ptr, b.fmt,
                               m, n, k, out.data_ptr() or None, ldo, dtype_code(out), 1 if accumulate else 0,
                               _word(status, 4, "status") if status is not None else None,
                               _raw_stream(device) if stream is None else _stream(stream))
    if code != LGN_OK:
        _check(code, "lgn_fp8_matmul")
    return out


def lgn_selftest_matmul_wait_expires(a: Fp8Operand, b: Fp8Operand, out: torch.Tensor, status: torch.Tensor, stream=None) -> None:
    """A product whose first copies are withheld: ``status`` must become LGN_ERR_TIMEOUT after a few seconds."""
    if (a.fmt, b.fmt, a.k) != (E4M3, E4M3, b.k) or tuple(out.shape) != (a.rows, b.rows):
        raise ValueError("E4M3 operands and an out of a.rows x b.rows")
    if _elsewhere(a._device, stream, b._device, out.get_device(), status.get_device()):
        with torch.cuda.device(a._device):
            return lgn_selftest_matmul_wait_expires(a, b, out, status, stream)
    _check(_lib.lgn_selftest_matmul_wait_expires(a._codes_ptr, a._scales_ptr, b._codes_ptr, b._scales_ptr, a.rows, b.rows, a.k,
                                                 _dev(out, "out"), dtype_code(out), _word(status, 4, "status"), _stream(stream)),
           "lgn_selftest_matmul_wait_expires")


# --------------------------------------------------------------------------- embedding
def _ids(ids: torch.Tensor) -> int:
    if ids.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"ids are int32 or int64, got {ids.dtype}")
    return 32 if ids.dtype == torch.int32 else 64


def lgn_embedding(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                  out_dtype: Optional[torch.dtype] = None, n_outside: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """scale * table[ids], zeros for ids outside the table: ids.numel() x dim.  ``n_outside``: int64 CUDA tensor of
    one element to which the number of ids outside the table is added."""
    vocab, dim, ld = _matrix3(table, "table")
    n = ids.numel()
    device = table.get_device()
    if _elsewhere(device, stream, ids.get_device(), out.get_device() if out is not None else None,
                  n_outside.get_device() if n_outside is not None else None):
        with torch.cuda.device(device):
            return lgn_embedding(table, ids, scale, out, out_dtype, n_outside, stream)
    if out is None:
        out = _empty((n, dim), out_dtype or table.dtype, table.device, stream)
        ldo = dim or 1
    else:
        if tuple(out.shape) != (n, dim):
            raise ValueError("out must be ids.numel() x dim")
        ldo = _matrix(out, "out")
    if n_outside is not None and n_outside.dtype != torch.int64:
        raise TypeError("n_outside is int64")
    _check(_lib.lgn_embedding(table.data_ptr() or None, vocab, dim, ld, dtype_code(table), _dev(ids, "ids") or None, _ids(ids), n,
                              float(scale), out.data_ptr() or None, ldo, dtype_code(out),
                              _word(n_outside, 8, "n_outside") if n_outside is not None else None, _stream(stream)), "lgn_embedding")
    return out


def new_embedding_grad_workspace(tokens: int, vocab: int, dim: int, device) -> torch.Tensor:
    return torch.empty(max(16, int(_lib.lgn_embedding_grad_workspace_bytes(tokens, vocab, dim))), dtype=torch.uint8, device=device)


def lgn_embedding_grad(dout: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0, padding_idx: int = -1,
                       out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
                       accumulate: bool = False, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Gradient of the table (vocab x dim) from ``dout`` (ids.numel() x dim); with ``accumulate`` added to ``out``."""
    ld = _matrix(dout, "dout")
    n, dim = dout.shape
    if ids.numel() != n:
        raise ValueError("dout must have one row per id")
    device = dout.get_device()
    if _elsewhere(device, stream, ids.get_device(), out.get_device() if out is not None else None, ws.get_device() if ws is not None else None):
        with torch.cuda.device(device):
            return lgn_embedding_grad(dout, ids, vocab, scale, padding_idx, out, out_dtype, accumulate, ws, stream)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = _empty((vocab, dim), out_dtype, dout.device, stream)
    elif tuple(out.shape) != (vocab, dim):
        raise ValueError("out must be vocab x dim")
    if ws is None:
        ws = _empty(max(16, int(_lib.lgn_embedding_grad_workspace_bytes(n, vocab, dim))), _uint8, dout.device, stream)
    _check(_lib.lgn_embedding_grad(dout.data_ptr() or None, ld, dtype_code(dout), _dev(ids, "ids") or None, _ids(ids), n, vocab, dim,
                                   float(scale), int(padding_idx), out.data_ptr() or None, _matrix(out, "out"), dtype_code(out),
                                   1 if accumulate else 0, _dev(ws, "ws"), ws.numel() * ws.element_size(), _stream(stream)),
           "lgn_embedding_grad")
    return out


# --------------------------------------------------------------------------- gradient norm and clipping
class Grads(NamedTuple):
    """Descriptors of a list of tensors, kept from step to step as long as the tensors stay where they are."""
    array: C.Array
    count: int
    tensors: tuple           # keeps them alive
    device: Optional[int]    # None: no tensors
    disjoint: bool           # no tensor's out shares memory with another tensor or its out


def _disjoint(arr: C.Array, count: int) -> bool:
    spans = []                                             # first byte, end, written?
    for x in arr[:count]:
        if x.n:
            size = x.n * (2 if x.dt == BF16 else 4)
            spans.append((x.out, x.out + size, True))
            if x.g + size <= x.out or x.out + size <= x.g:  # not in place (or over itself, which the library refuses)
                spans.append((x.g, x.g + size, False))
    written = seen = 0                                     # ends so far
    for start, end, write in sorted(spans):
        if start < (seen if write else written):
            return False
        seen = max(seen, end)
        if write:
            written = max(written, end)
    return True


def make_grads(grads: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None) -> Grads:
    """``outs``: where the clipped gradients go, tensor by tensor; None: in place."""
    outs = grads if outs is None else outs
    if len(outs) != len(grads):
        raise ValueError("one out per gradient")
    arr = (GradT * max(1, len(grads)))()
    devices = set()
    for i, (g, o) in enumerate(zip(grads, outs)):
        if o.numel() != g.numel() or o.dtype != g.dtype:
            raise ValueError("out must have its gradient's size and type")
        arr[i] = GradT(_dev(g, "gradient") or None, _dev(o, "out") or None, g.numel(), dtype_code(g), 0)
        devices.add(g.get_device())
        devices.add(o.get_device())
    if len(devices) > 1:
        raise ValueError(f"tensors on different devices: {sorted(devices)}")
    return Grads(arr, len(grads), (tuple(grads), tuple(outs)), devices.pop() if devices else None, _disjoint(arr, len(grads)))


def new_norm_record(device) -> torch.Tensor:
    return torch.zeros(C.sizeof(NormT), dtype=torch.uint8, device=device)


def norm_of(record: torch.Tensor) -> torch.Tensor:
    """The record's norm as a float32 scalar on the device (a view)."""
    return record.view(torch.float32)[0]


def sum_sq_of(record: torch.Tensor) -> torch.Tensor:
    """The record's sum of squares as a float64 scalar on the device (a view): what sharded ranks all-reduce before
    lgn_clip_apply."""
    return record.view(torch.float64)[2]


def read_norm_record(record: torch.Tensor) -> Dict[str, float]:
    """Host copy of a record (synchronises)."""
    r = NormT.from_buffer_copy(record.cpu().numpy().tobytes())
    return {"norm": r.norm, "coef": r.coef, "n_nonfinite": r.n_nonfinite, "sum_sq": r.sum_sq}


def new_clip_workspace(device, count: int = 512) -> torch.Tensor:
    return torch.empty(int(_lib.lgn_clip_workspace_bytes(count)), dtype=torch.uint8, device=device)


def _record(record: torch.Tensor) -> int:
    if record.numel() * record.element_size() < C.sizeof(NormT):
        raise ValueError("record too small")
    return _dev(record, "record")


def lgn_grad_norm(grads: Grads, record: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """The record of the tensors' global norm; nothing is scaled."""
    device = record.get_device()
    if _elsewhere(device, stream, grads.device, ws.get_device()):
        with torch.cuda.device(device):
            return lgn_grad_norm(grads, record, ws, stream)
    _check(_lib.lgn_grad_norm(grads.array, grads.count, _record(record), _dev(ws, "ws"), ws.numel() * ws.element_size(),
                              _stream(stream)), "lgn_grad_norm")


def lgn_clip_grad_norm(grads: Grads, max_norm: float, record: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """The record, and every tensor scaled by min(1, max_norm / norm); no host round trip."""
    device = record.get_device()
    if _elsewhere(device, stream, grads.device, ws.get_device()):
        with torch.cuda.device(device):
            return lgn_clip_grad_norm(grads, max_norm, record, ws, stream)
    if not grads.disjoint:
        raise ValueError("a tensor would be written over another one")
    _check(_lib.lgn_clip_grad_norm(grads.array, grads.count, float(max_norm), _record(record), _dev(ws, "ws"),
                                   ws.numel() * ws.element_size(), _stream(stream)), "lgn_clip_grad_norm")


def lgn_clip_apply(grads: Grads, max_norm: float, record: torch.Tensor, stream=None) -> None:
    """Every tensor scaled by the norm that the record's sum of squares gives."""
    device = record.get_device()
    if _elsewhere(device, stream, grads.device):
        with torch.cuda.device(device):
            return lgn_clip_apply(grads, max_norm, record, stream)
    if not grads.disjoint:
        raise ValueError("a tensor would be written over another one")
    _check(_lib.lgn_clip_apply(grads.array, grads.count, float(max_norm), _record(record), _stream(stream)), "lgn_clip_apply")
