"""Python binding of libawsrc, the HIP (gfx950) implementation of the AWSRC
encoder/decoder hot path.

The functions carry the names of the C entry points declared in
include/awsrc.h and only marshal arguments: torch allocates the device
buffers and supplies the stream; every step of the codec runs in the
library's kernels.  Importing this module fails loudly if the library has
not been built (python paper_2608_23144_amd/build.py).
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Dict, List, Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libawsrc.so")

AWSRC_OK, AWSRC_EINVAL, AWSRC_ENOSPC, AWSRC_ECORRUPT, AWSRC_EDEVICE = 0, -1, -2, -3, -4
AWSRC_DTYPE_F32, AWSRC_DTYPE_BF16, AWSRC_DTYPE_F16 = 0, 1, 2
AWSRC_D_PER_COL, AWSRC_D_PER_ELEM = 0, 1
AWSRC_MODE_GLOBAL, AWSRC_MODE_PER_MODULE = 0, 1
AWSRC_SCALE_FP16, AWSRC_SCALE_POW2 = 0, 1

EXPORTED = ("awsrc_abi_version", "awsrc_last_error", "awsrc_backbone_rtn", "awsrc_sdq_encode",
            "awsrc_backbone_sdq_dequant", "awsrc_encode_tiles",
            "awsrc_encode_modules", "awsrc_encode_screen_lists", "awsrc_encode_tiles_noalloc", "awsrc_encode_noalloc_max_bytes",
            "awsrc_encode_scored", "awsrc_rank_prefix", "awsrc_decode_add", "awsrc_decode_prepare", "awsrc_decode_apply",
            "awsrc_reconstruct_bf16", "awsrc_reconstruct_bf16_prefixes", "awsrc_reconstruct_bf16_sdq",
            "awsrc_quantize_rows_i8", "awsrc_matmul_i8", "awsrc_linear_i8", "awsrc_kv_append", "awsrc_kv_read",
            "awsrc_kv_attention", "awsrc_quantize_blocks_f8", "awsrc_dequantize_blocks_f8", "awsrc_matmul_f8", "awsrc_linear_f8",
            "awsrc_kv_plan", "awsrc_verify_drafts", "awsrc_record_bytes", "awsrc_header_bytes", "awsrc_budget_bytes", "awsrc_prefix_K")


class AwsrcError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"awsrc status {status}: {msg}")
        self.status = status


class awsrc_params(ctypes.Structure):
    _fields_ = [("C", ctypes.c_int32), ("P", ctypes.c_int32), ("b", ctypes.c_int32), ("S", ctypes.c_int32),
                ("scale_fmt", ctypes.c_int32), ("idx_bits", ctypes.c_int32), ("gen_version", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("basis_key", ctypes.c_uint64), ("ridge_lambda", ctypes.c_double)]


class awsrc_decode_plan(ctypes.Structure):
    _fields_ = [("C", ctypes.c_int32), ("P", ctypes.c_int32), ("b", ctypes.c_int32), ("S", ctypes.c_int32),
                ("idx_bits", ctypes.c_int32), ("seed_bits", ctypes.c_int32), ("L_rec", ctypes.c_int32),
                ("n_modules", ctypes.c_int32), ("w0_dtype", ctypes.c_int32), ("scale_fmt", ctypes.c_int32),
                ("K", ctypes.c_int64), ("T_total", ctypes.c_uint64), ("h", ctypes.c_uint64),
                ("records", ctypes.c_void_p), ("workspace", ctypes.c_void_p)]


class awsrc_kv_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class awsrc_page_pool(ctypes.Structure):
    _fields_ = [("free_pages", ctypes.c_void_p), ("n_free", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
                ("page_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32)]


def make_params(C: int, P: int, b: int, S: int, basis_key: int = 0, ridge_lambda: float = 1e-6,
                idx_bits: int = 32, scale_fmt: int = AWSRC_SCALE_FP16, gen_version: int = 1) -> awsrc_params:
    return awsrc_params(C, P, b, S, scale_fmt, idx_bits, gen_version, 0, basis_key, ridge_lambda)


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2608_23144_amd/build.py`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
    pp = ctypes.POINTER(awsrc_params)
    P64 = ctypes.POINTER(ctypes.c_int64)
    sig = {
        "awsrc_abi_version": (i32, []),
        "awsrc_last_error": (ctypes.c_char_p, []),
        "awsrc_backbone_rtn": (i32, [vp, i32, i64, i64, i32, vp, vp, vp, vp, vp]),
        "awsrc_sdq_encode": (i32, [vp, i64, vp, vp, vp, vp]),
        "awsrc_backbone_sdq_dequant": (i32, [vp, vp, vp, vp, vp, i64, i64, i32, vp, vp]),
        "awsrc_encode_tiles": (i32, [pp, vp, i32, vp, i64, i64, vp, i32, vp, vp, vp, vp, vp, vp,
                                     ctypes.POINTER(sz), vp]),
        "awsrc_encode_modules": (i32, [pp, i32, ctypes.POINTER(vp), i32, ctypes.POINTER(vp), ctypes.POINTER(vp), i32,
                                       P64, P64, vp, vp, vp, vp, vp, vp, ctypes.POINTER(sz), vp]),
        "awsrc_encode_screen_lists": (i32, [pp, i32, P64, P64, i32, vp, vp, vp, ctypes.POINTER(i32), vp]),
        "awsrc_encode_tiles_noalloc": (i32, [pp, vp, i32, vp, i64, i64, vp, i32, vp, vp, vp, vp, vp, vp]),
        "awsrc_encode_noalloc_max_bytes": (u64, []),
        "awsrc_encode_scored": (i32, [vp, ctypes.POINTER(u64), vp]),
        "awsrc_rank_prefix": (i32, [pp, i32, P64, P64, i32, ctypes.c_double, vp, vp, vp, vp, vp, u64,
                                    ctypes.POINTER(u64), P64, P64, vp, ctypes.POINTER(sz), vp]),
        "awsrc_decode_add": (i32, [vp, u64, i32, ctypes.POINTER(vp), P64, P64, i32, vp,
                                   ctypes.POINTER(sz), vp]),
        "awsrc_decode_prepare": (i32, [vp, u64, i32, ctypes.POINTER(vp), P64, P64, i32,
                                       ctypes.POINTER(awsrc_decode_plan), vp, ctypes.POINTER(sz), vp]),
        "awsrc_decode_apply": (i32, [ctypes.POINTER(awsrc_decode_plan), vp]),
        "awsrc_reconstruct_bf16": (i32, [ctypes.POINTER(awsrc_decode_plan), i32, ctypes.POINTER(vp),
                                         ctypes.POINTER(vp), ctypes.POINTER(vp), vp]),
        "awsrc_reconstruct_bf16_prefixes": (i32, [ctypes.POINTER(awsrc_decode_plan), i32, P64, ctypes.POINTER(vp),
                                                  i32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                                  vp]),
        "awsrc_reconstruct_bf16_sdq": (i32, [ctypes.POINTER(awsrc_decode_plan), i32, P64, ctypes.POINTER(vp), i32,
                                             ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                             ctypes.POINTER(vp), ctypes.POINTER(vp), vp]),
        "awsrc_quantize_rows_i8": (i32, [vp, i32, i64, i64, i64, vp, i64, vp, vp]),
        "awsrc_matmul_i8": (i32, [vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64, vp, ctypes.POINTER(sz),
                                  vp]),
        "awsrc_linear_i8": (i32, [vp, i32, i64, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64, vp, ctypes.POINTER(sz),
                                  vp]),
        "awsrc_kv_append": (i32, [ctypes.POINTER(awsrc_kv_cache), vp, i64, vp, i64, vp, i64, i32, vp, i64, i32, vp, vp,
                                  i64, i32, i32, i32, i64, vp, vp, vp, i64, i64, vp]),
        "awsrc_kv_read": (i32, [ctypes.POINTER(awsrc_kv_cache), i32, i64, vp, vp, vp, i64, i64, vp, vp, i32, vp]),
        "awsrc_kv_attention": (i32, [ctypes.POINTER(awsrc_kv_cache), vp, i64, i32, i32, i32, i64, vp, vp, vp, i64, i64,
                                     i64, ctypes.c_float, i32, vp, i64, vp, ctypes.POINTER(sz), vp]),
        "awsrc_quantize_blocks_f8": (i32, [vp, i32, i64, i64, i64, i32, vp, i64, vp, vp]),
        "awsrc_dequantize_blocks_f8": (i32, [vp, i64, vp, i64, i64, i32, vp, i32, i64, vp]),
        "awsrc_matmul_f8": (i32, [vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64, vp, ctypes.POINTER(sz), vp]),
        "awsrc_linear_f8": (i32, [vp, i32, i64, vp, i64, vp, vp, i64, i64, i64, vp, i32, i64, vp, ctypes.POINTER(sz), vp]),
        "awsrc_kv_plan": (i32, [ctypes.POINTER(awsrc_page_pool), i32, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, vp,
                                ctypes.POINTER(sz), vp]),
        "awsrc_verify_drafts": (i32, [vp, i64, vp, i64, i32, i64, i32, i64, vp, vp, vp, vp, vp, vp, vp, vp,
                                      ctypes.POINTER(sz), vp]),
        "awsrc_record_bytes": (i64, [pp, i64]),
        "awsrc_header_bytes": (i64, [i32]),
        "awsrc_budget_bytes": (i64, [ctypes.c_double, i64]),
        "awsrc_prefix_K": (i64, [i64, i64, i64, i64]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    return lib


LIB = _load()


def _check(status: int) -> None:
    if status != AWSRC_OK:
        raise AwsrcError(status, LIB.awsrc_last_error().decode(errors="replace"))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return AWSRC_DTYPE_F32
    if t.dtype == torch.bfloat16:
        return AWSRC_DTYPE_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dev(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("tensors must be contiguous device tensors")


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


# ------------------------------------------------------------------ host-only helpers
def awsrc_abi_version() -> int:
    return LIB.awsrc_abi_version()


def awsrc_record_bytes(p: awsrc_params, T_total: int) -> int:
    return LIB.awsrc_record_bytes(ctypes.byref(p), T_total)


def awsrc_header_bytes(n_modules: int) -> int:
    return LIB.awsrc_header_bytes(n_modules)


def awsrc_budget_bytes(bpw: float, n_weights: int) -> int:
    return LIB.awsrc_budget_bytes(bpw, n_weights)


def awsrc_prefix_K(budget_bytes: int, h: int, L_rec: int, n_eligible: int) -> int:
    return LIB.awsrc_prefix_K(budget_bytes, h, L_rec, n_eligible)


# ------------------------------------------------------------------ device calls
def awsrc_backbone_rtn(W: torch.Tensor, group: int = 128, want_W0: bool = True, out=None, stream=None):
    """RTN-INT4 backbone; returns (codes u8, scale fp16-bits i16-view, zero u8, W0 fp32 or None)."""
    _dev(W)
    rows, cols = W.shape
    if out is None:
        dev = W.device
        out = (torch.empty(rows, cols // 2, dtype=torch.uint8, device=dev),
               torch.empty(rows, cols // group, dtype=torch.int16, device=dev),
               torch.empty(rows, cols // group, dtype=torch.uint8, device=dev),
               torch.empty(rows, cols, dtype=torch.float32, device=dev) if want_W0 else None)
    codes, scale, zero, W0 = out
    _check(LIB.awsrc_backbone_rtn(_ptr(W), _dtype_code(W), rows, cols, group, _ptr(codes), _ptr(scale),
                                  _ptr(zero), _ptr(W0), _stream(stream)))
    return codes, scale, zero, W0


def encode_workspace_bytes(p: awsrc_params, W: torch.Tensor, d_mode: int) -> int:
    rows, cols = W.shape
    n = ctypes.c_size_t(0)
    _check(LIB.awsrc_encode_tiles(ctypes.byref(p), None, _dtype_code(W), None, rows, cols, None, d_mode,
                                  None, None, None, None, None, None, ctypes.byref(n), None))
    return n.value


SDQ_BLOCK = 256


def awsrc_sdq_encode(scale_f16: torch.Tensor, stream=None):
    """SDQ of fp16 group scales (int16 bit patterns, any shape, row-major):
    returns (codes int8 [n], block mean fp32 [nb], block step fp32 [nb])."""
    _dev(scale_f16)
    n = scale_f16.numel()
    nb = (n + SDQ_BLOCK - 1) // SDQ_BLOCK
    dev = scale_f16.device
    codes = torch.empty(n, dtype=torch.int8, device=dev)
    mean = torch.empty(nb, dtype=torch.float32, device=dev)
    step = torch.empty(nb, dtype=torch.float32, device=dev)
    _check(LIB.awsrc_sdq_encode(_ptr(scale_f16), n, _ptr(codes), _ptr(mean), _ptr(step), _stream(stream)))
    return codes, mean, step


def awsrc_backbone_sdq_dequant(codes: torch.Tensor, zero: torch.Tensor, sdq, group: int = 128,
                               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """W0 [rows, cols] fp32 of the RTN-INT4-SDQ backbone (sdq = awsrc_sdq_encode's result)."""
    sc, mean, step = sdq
    _dev(codes, zero, sc, mean, step)
    rows, cols = codes.shape[0], codes.shape[1] * 2
    if out is None:
        out = torch.empty(rows, cols, dtype=torch.float32, device=codes.device)
    _check(LIB.awsrc_backbone_sdq_dequant(_ptr(codes), _ptr(zero), _ptr(sc), _ptr(mean), _ptr(step), rows, cols,
                                          group, _ptr(out), _stream(stream)))
    return out


def awsrc_encode_tiles(p: awsrc_params, W: torch.Tensor, W0: torch.Tensor, d: torch.Tensor,
                       want_alpha: bool = False, out: Optional[Dict[str, torch.Tensor]] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> Dict[str, torch.Tensor]:
    """Per-tile best seed, codes, fp16 scale bits, fp64 gain (and fp32 alpha*)."""
    _dev(W, W0, d)
    rows, cols = W.shape
    d_mode = AWSRC_D_PER_COL if d.dim() == 1 else AWSRC_D_PER_ELEM
    T = rows * cols // p.C
    dev = W.device
    if out is None:
        out = {"seed": torch.empty(T, dtype=torch.int16, device=dev),
               "codes": torch.empty(T, p.P, dtype=torch.int8, device=dev),
               "scale": torch.empty(T, dtype=torch.int16, device=dev),
               "gain": torch.empty(T, dtype=torch.float64, device=dev),
               "alpha": torch.empty(T, p.P, dtype=torch.float32, device=dev) if want_alpha else None}
    nbytes = encode_workspace_bytes(p, W, d_mode)
    if workspace is None or workspace.numel() < nbytes:
        workspace = _workspace(nbytes, dev)
    n = ctypes.c_size_t(workspace.numel())
    _check(LIB.awsrc_encode_tiles(ctypes.byref(p), _ptr(W), _dtype_code(W), _ptr(W0), rows, cols, _ptr(d),
                                  d_mode, _ptr(out["seed"]), _ptr(out["codes"]), _ptr(out["scale"]),
                                  _ptr(out["gain"]), _ptr(out.get("alpha")), _ptr(workspace),
                                  ctypes.byref(n), _stream(stream)))
    out["workspace"] = workspace
    return out


def _ptr_array(ts):
    return (ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts])


def encode_modules_workspace_bytes(p: awsrc_params, shapes: Sequence[Tuple[int, int]], w_dtype: int,
                                   d_mode: int) -> int:
    n = ctypes.c_size_t(0)
    rows = _i64arr([s[0] for s in shapes])
    cols = _i64arr([s[1] for s in shapes])
    _check(LIB.awsrc_encode_modules(ctypes.byref(p), len(shapes), None, w_dtype, None, None, d_mode, rows, cols,
                                    None, None, None, None, None, None, ctypes.byref(n), None))
    return n.value


def awsrc_encode_modules(p: awsrc_params, W_list: Sequence[torch.Tensor], W0_list: Sequence[torch.Tensor],
                         d_list: Sequence[torch.Tensor], want_alpha: bool = False,
                         out: Optional[Dict[str, torch.Tensor]] = None, workspace: Optional[torch.Tensor] = None,
                         stream=None) -> Dict[str, torch.Tensor]:
    """awsrc_encode_tiles over several modules in one call; outputs
    concatenated in module order."""
    _dev(*W_list, *W0_list, *d_list)
    shapes = [tuple(w.shape) for w in W_list]
    dts = {_dtype_code(w) for w in W_list}
    if len(dts) != 1:
        raise TypeError("all W must share one dtype")
    w_dtype = dts.pop()
    modes = {AWSRC_D_PER_COL if d.dim() == 1 else AWSRC_D_PER_ELEM for d in d_list}
    if len(modes) != 1:
        raise TypeError("all d must be per column or all per element")
    d_mode = modes.pop()
    T = sum(r * c // p.C for r, c in shapes)
    dev = W_list[0].device
    if out is None:
        out = {"seed": torch.empty(T, dtype=torch.int16, device=dev),
               "codes": torch.empty(T, p.P, dtype=torch.int8, device=dev),
               "scale": torch.empty(T, dtype=torch.int16, device=dev),
               "gain": torch.empty(T, dtype=torch.float64, device=dev),
               "alpha": torch.empty(T, p.P, dtype=torch.float32, device=dev) if want_alpha else None}
    nbytes = encode_modules_workspace_bytes(p, shapes, w_dtype, d_mode)
    if workspace is None or workspace.numel() < nbytes:
        workspace = _workspace(nbytes, dev)
    n = ctypes.c_size_t(workspace.numel())
    rows = _i64arr([s[0] for s in shapes])
    cols = _i64arr([s[1] for s in shapes])
    _check(LIB.awsrc_encode_modules(ctypes.byref(p), len(shapes), _ptr_array(W_list), w_dtype, _ptr_array(W0_list),
                                    _ptr_array(d_list), d_mode, rows, cols, _ptr(out["seed"]), _ptr(out["codes"]),
                                    _ptr(out["scale"]), _ptr(out["gain"]), _ptr(out.get("alpha")), _ptr(workspace),
                                    ctypes.byref(n), _stream(stream)))
    out["workspace"] = workspace
    return out


def awsrc_encode_screen_lists(p: awsrc_params, shapes: Sequence[Tuple[int, int]], d_mode: int,
                              workspace: torch.Tensor, stream=None):
    """The fp32 screen's kept lists of the last encode with this workspace:
    (gain f32 [T, nsplit, 2], seed word int32 [T, nsplit, 2]: seed in bits
    0-15, bit 16 set for a candidate whose rounding was on a knife edge)."""
    rows = _i64arr([s[0] for s in shapes])
    cols = _i64arr([s[1] for s in shapes])
    ns = ctypes.c_int32(0)
    _check(LIB.awsrc_encode_screen_lists(ctypes.byref(p), len(shapes), rows, cols, d_mode, _ptr(workspace), None,
                                         None, ctypes.byref(ns), _stream(stream)))
    T = sum(r * c // p.C for r, c in shapes)
    g = torch.empty(T, ns.value, 2, dtype=torch.float32, device=workspace.device)
    sd = torch.empty(T, ns.value, 2, dtype=torch.int32, device=workspace.device)
    _check(LIB.awsrc_encode_screen_lists(ctypes.byref(p), len(shapes), rows, cols, d_mode, _ptr(workspace), _ptr(g),
                                         _ptr(sd), ctypes.byref(ns), _stream(stream)))
    return g, sd


def awsrc_encode_noalloc_max_bytes() -> int:
    return int(LIB.awsrc_encode_noalloc_max_bytes())


def awsrc_encode_tiles_noalloc(p: awsrc_params, W: torch.Tensor, W0: torch.Tensor, d: torch.Tensor,
                               out: Dict[str, torch.Tensor], stream=None) -> Dict[str, torch.Tensor]:
    """awsrc_encode_tiles into caller-provided outputs (keys seed, codes,
    scale, gain, optional alpha), with the library's fixed scratch array
    instead of a workspace: allocates nothing."""
    _dev(W, W0, d, *[v for v in out.values() if isinstance(v, torch.Tensor)])
    rows, cols = W.shape
    d_mode = AWSRC_D_PER_COL if d.dim() == 1 else AWSRC_D_PER_ELEM
    _check(LIB.awsrc_encode_tiles_noalloc(ctypes.byref(p), _ptr(W), _dtype_code(W), _ptr(W0), rows, cols, _ptr(d),
                                          d_mode, _ptr(out["seed"]), _ptr(out["codes"]), _ptr(out["scale"]),
                                          _ptr(out["gain"]), _ptr(out.get("alpha")), _stream(stream)))
    return out


def awsrc_encode_scored(out: Dict[str, torch.Tensor], stream=None) -> int:
    """Candidates scored in full by the last awsrc_encode_tiles call that filled `out`."""
    v = ctypes.c_uint64(0)
    _check(LIB.awsrc_encode_scored(_ptr(out["workspace"]), ctypes.byref(v), _stream(stream)))
    return int(v.value)


def _i64arr(v: Sequence[int]):
    return (ctypes.c_int64 * len(v))(*[int(x) for x in v])


def awsrc_rank_prefix(p: awsrc_params, modules: Sequence[Tuple[int, int]], mode: int, bpw: float,
                      seed: torch.Tensor, codes: torch.Tensor, scale: torch.Tensor, gain: torch.Tensor,
                      stream_cap: Optional[int] = None, out: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None):
    """Rank and serialize; returns (stream bytes tensor [stream_len], K, n_eligible)."""
    _dev(seed, codes, scale, gain)
    rows = _i64arr([m[0] for m in modules])
    cols = _i64arr([m[1] for m in modules])
    n = ctypes.c_size_t(0)
    slen, K, ne = ctypes.c_uint64(0), ctypes.c_int64(0), ctypes.c_int64(0)
    _check(LIB.awsrc_rank_prefix(ctypes.byref(p), len(modules), rows, cols, mode, bpw, None, None, None, None,
                                 None, 0, ctypes.byref(slen), ctypes.byref(K), None, None, ctypes.byref(n), None))
    dev = gain.device
    if workspace is None or workspace.numel() < n.value:
        workspace = _workspace(n.value, dev)
    if out is None:
        if stream_cap is None:
            T = sum(r * c // p.C for r, c in modules)
            L = awsrc_record_bytes(p, T)
            N = sum(r * c for r, c in modules)
            if mode == AWSRC_MODE_GLOBAL:
                cap_rec = max(0, (awsrc_budget_bytes(bpw, N) - awsrc_header_bytes(len(modules))) // L)
            else:
                cap_rec = sum(awsrc_budget_bytes(bpw, r * c) // L for r, c in modules)
            stream_cap = awsrc_header_bytes(len(modules)) + min(cap_rec, T) * L
        out = torch.empty(int(stream_cap), dtype=torch.uint8, device=dev)
    cap = out.numel() if stream_cap is None else min(int(stream_cap), out.numel())
    n = ctypes.c_size_t(workspace.numel())
    _check(LIB.awsrc_rank_prefix(ctypes.byref(p), len(modules), rows, cols, mode, bpw, _ptr(seed), _ptr(codes),
                                 _ptr(scale), _ptr(gain), _ptr(out), cap, ctypes.byref(slen),
                                 ctypes.byref(K), ctypes.byref(ne), _ptr(workspace), ctypes.byref(n),
                                 _stream(stream)))
    return out[: slen.value], K.value, ne.value


def _decode_args(stream_bytes, W0_list, stream_len):
    _dev(stream_bytes, *W0_list)
    if stream_len is None:
        stream_len = stream_bytes.numel()
    dt = {_dtype_code(w) for w in W0_list}
    if len(dt) != 1:
        raise TypeError("all W0 must share one dtype")
    rows = _i64arr([w.shape[0] for w in W0_list])
    cols = _i64arr([w.shape[1] for w in W0_list])
    ptrs = (ctypes.c_void_p * len(W0_list))(*[w.data_ptr() for w in W0_list])
    return stream_len, rows, cols, ptrs, dt.pop()


def awsrc_decode_add(stream_bytes: torch.Tensor, W0_list: List[torch.Tensor], stream_len: Optional[int] = None,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """In-place W0 += B_s alpha_hat for every record of the stream (or of its prefix)."""
    stream_len, rows, cols, ptrs, dt = _decode_args(stream_bytes, W0_list, stream_len)
    n = ctypes.c_size_t(0)
    st = _stream(stream)
    _check(LIB.awsrc_decode_add(_ptr(stream_bytes), stream_len, len(W0_list), ptrs, rows, cols, dt,
                                None, ctypes.byref(n), st))
    if workspace is None or workspace.numel() < n.value:
        workspace = _workspace(n.value, stream_bytes.device)
    n = ctypes.c_size_t(workspace.numel())
    _check(LIB.awsrc_decode_add(_ptr(stream_bytes), stream_len, len(W0_list), ptrs, rows, cols, dt,
                                _ptr(workspace), ctypes.byref(n), st))


def awsrc_decode_prepare(stream_bytes: torch.Tensor, W0_list: List[torch.Tensor], stream_len: Optional[int] = None,
                         workspace: Optional[torch.Tensor] = None, stream=None):
    """Validate a stream and build its decode tables; returns (plan, workspace).
    Keep both (and the stream bytes) alive while the plan is applied.  A
    workspace passed in (e.g. the one a previous plan used, once that plan is
    no longer needed) is used directly when it is large enough, which saves
    the size query's header read."""
    stream_len, rows, cols, ptrs, dt = _decode_args(stream_bytes, W0_list, stream_len)
    st = _stream(stream)
    plan = awsrc_decode_plan()
    if workspace is not None:
        n = ctypes.c_size_t(workspace.numel())
        rc = LIB.awsrc_decode_prepare(_ptr(stream_bytes), stream_len, len(W0_list), ptrs, rows, cols, dt,
                                      ctypes.byref(plan), _ptr(workspace), ctypes.byref(n), st)
        if rc != AWSRC_ENOSPC:
            _check(rc)
            return plan, workspace
    n = ctypes.c_size_t(0)
    _check(LIB.awsrc_decode_prepare(_ptr(stream_bytes), stream_len, len(W0_list), ptrs, rows, cols, dt, None,
                                    None, ctypes.byref(n), st))
    workspace = _workspace(n.value, stream_bytes.device)
    n = ctypes.c_size_t(workspace.numel())
    _check(LIB.awsrc_decode_prepare(_ptr(stream_bytes), stream_len, len(W0_list), ptrs, rows, cols, dt,
                                    ctypes.byref(plan), _ptr(workspace), ctypes.byref(n), st))
    return plan, workspace


def awsrc_decode_apply(plan: awsrc_decode_plan, stream=None) -> None:
    """One asynchronous launch adding every record of a prepared stream onto W0."""
    _check(LIB.awsrc_decode_apply(ctypes.byref(plan), _stream(stream)))


def awsrc_reconstruct_bf16(plan: awsrc_decode_plan, backbones: Sequence[Tuple[torch.Tensor, torch.Tensor,
                                                                               torch.Tensor]],
                           group: int = 128, stream=None) -> None:
    """Dense bf16(W0 + R_hat) into the bf16 buffers the plan was prepared on;
    `backbones` holds each module's (codes, scale, zero) as awsrc_backbone_rtn
    returns them."""
    if len(backbones) != plan.n_modules:
        raise ValueError(f"{len(backbones)} backbones for a plan of {plan.n_modules} modules")
    for bb in backbones:
        _dev(*bb)
    arr = [(ctypes.c_void_p * len(backbones))(*[bb[k].data_ptr() for bb in backbones]) for k in range(3)]
    _check(LIB.awsrc_reconstruct_bf16(ctypes.byref(plan), group, arr[0], arr[1], arr[2], _stream(stream)))


def awsrc_reconstruct_bf16_prefixes(plan: awsrc_decode_plan, K_out: Sequence[int],
                                    outs: Sequence[Sequence[torch.Tensor]],
                                    backbones: Sequence[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]],
                                    group: int = 128, stream=None) -> None:
    """Dense bf16(W0 + R_hat of the first K_out[o] records) into outs[o] (one
    bf16 tensor per module) for every o, in one pass over the backbone."""
    n = plan.n_modules
    if len(backbones) != n or len(outs) != len(K_out) or any(len(o) != n for o in outs):
        raise ValueError("need one backbone and, per prefix, one target per module")
    for bb in backbones:
        _dev(*bb)
    for o in outs:
        _dev(*o)
        if any(t.dtype != torch.bfloat16 for t in o):
            raise TypeError("targets must be bf16")
    arr = [(ctypes.c_void_p * n)(*[bb[k].data_ptr() for bb in backbones]) for k in range(3)]
    optr = (ctypes.c_void_p * (n * len(outs)))(*[t.data_ptr() for o in outs for t in o])
    _check(LIB.awsrc_reconstruct_bf16_prefixes(ctypes.byref(plan), len(K_out), _i64arr(list(K_out)), optr, group,
                                               arr[0], arr[1], arr[2], _stream(stream)))


def awsrc_reconstruct_bf16_sdq(plan: awsrc_decode_plan,
                               backbones: Sequence[Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor,
                                                         torch.Tensor]],
                               K_out: Optional[Sequence[int]] = None,
                               outs: Optional[Sequence[Sequence[torch.Tensor]]] = None,
                               group: int = 128, stream=None) -> None:
    """Dense bf16 repaired weights on the RTN-INT4-SDQ backbone: `backbones`
    holds each module's (codes, zero, sdq_code, sdq_mean, sdq_step), the RTN
    codes and zero points with awsrc_sdq_encode's outputs for its scales.
    Without K_out / outs: into the bf16 buffers the plan was prepared on, every
    record; else outs[o] receives the first K_out[o] records' prefix."""
    n = plan.n_modules
    if len(backbones) != n:
        raise ValueError(f"{len(backbones)} backbones for a plan of {n} modules")
    for bb in backbones:
        _dev(*bb)
    if (K_out is None) != (outs is None):
        raise ValueError("K_out and outs go together")
    arr = [(ctypes.c_void_p * n)(*[bb[k].data_ptr() for bb in backbones]) for k in range(5)]
    if outs is None:
        n_out, kp, optr = 0, None, None
    else:
        if len(outs) != len(K_out) or any(len(o) != n for o in outs):
            raise ValueError("need, per prefix, one target per module")
        for o in outs:
            _dev(*o)
            if any(t.dtype != torch.bfloat16 for t in o):
                raise TypeError("targets must be bf16")
        n_out, kp = len(K_out), _i64arr(list(K_out))
        optr = (ctypes.c_void_p * (n * n_out))(*[t.data_ptr() for o in outs for t in o])
    _check(LIB.awsrc_reconstruct_bf16_sdq(ctypes.byref(plan), n_out, kp, optr, group, arr[0], arr[2], arr[3], arr[4],
                                          arr[1], _stream(stream)))


# ------------------------------------------------------------------ 8-bit serving
# These calls are made many times per token: what they check of their arguments
# is kept to cheap attribute reads, sizes that depend on shapes alone are remembered.
# They serve: none of them records a gradient, also for inputs that require one.
KVCache = Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]  # codes of keys and values, their scales

_ACT_CODE = {torch.float32: AWSRC_DTYPE_F32, torch.bfloat16: AWSRC_DTYPE_BF16, torch.float16: AWSRC_DTYPE_F16}
_WS_SIZES = 4096  # shapes whose workspace sizes are remembered


def _act_code(dtype: torch.dtype) -> int:
    code = _ACT_CODE.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}")
    return code


def _device_of(t: torch.Tensor) -> int:
    i = t.get_device()
    if i < 0:
        raise ValueError("tensors must be device tensors")
    return i


def _on_device(i: int, *ts: Optional[torch.Tensor]) -> None:
    for t in ts:
        if t is not None and t.get_device() != i:
            raise ValueError(f"tensors must be on one device: {t.device} and cuda:{i}")


def _empty(shape, like: torch.Tensor, dtype, stream):
    """A new tensor whose memory belongs to the stream that will use it."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _raw_stream(i: int, stream) -> int:
    if torch._C._cuda_getDevice() != i:
        raise ValueError(f"tensors on cuda:{i}, which is not the current device")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(i)
    if stream.device_index != i:
        raise ValueError(f"stream on {stream.device}, tensors on cuda:{i}")
    return stream.cuda_stream


def _rows_of(t: torch.Tensor, what: str):
    """(rows, cols, row stride) of a matrix whose rows are contiguous."""
    if t.dim() != 2:
        raise ValueError(f"{what} must be a matrix")
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{what} must be a matrix with contiguous rows")
    return rows, cols, (ld if rows > 1 or ld > cols else cols)


def _i8_rows(t: torch.Tensor, what: str, dtype: torch.dtype = torch.int8):
    """_rows_of for an operand of 8-bit codes: its rows are read in pieces of 16 bytes."""
    rows, cols, ld = _rows_of(t, what)
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, not {t.dtype}")
    if cols % 16 == 0:
        return rows, cols, ld if rows > 1 or ld % 16 == 0 else cols
    wide = -(-cols // 16) * 16
    if rows <= 1:
        ld = max(ld, wide) if ld % 16 == 0 else wide
    if rows and t.untyped_storage().nbytes() < t.storage_offset() + (rows - 1) * ld + wide:
        raise ValueError(f"{what}: the last row must be readable up to a multiple of 16 bytes")
    return rows, cols, ld


def _code_rows(t: torch.Tensor) -> int:
    """The row stride of codes that are written; rows on 16 bytes are filled up to a multiple of 16."""
    rows, cols, ld = _rows_of(t, "codes")
    wide = -(-cols // 16) * 16
    if rows and ld % 16 == 0 and t.data_ptr() % 16 == 0 and t.untyped_storage().nbytes() < t.storage_offset() + (rows - 1) * ld + wide:
        raise ValueError("codes: the last row must be writable up to a multiple of 16 bytes")
    return ld


def _heads_of(t: torch.Tensor, what: str, heads: Optional[int], dim: int, dtype: torch.dtype):
    """(rows, heads, row stride) of a [rows, heads, dim] tensor whose heads lie side by side."""
    if t.dim() != 3:
        raise ValueError(f"{what}: expected [rows, heads, {dim}]")
    n, h, d = t.shape
    if d != dim or (heads is not None and h != heads):
        raise ValueError(f"{what}: expected [rows, {heads if heads else 'heads'}, {dim}], got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{what}: expected {dtype}, got {t.dtype}")
    ld, sh, sd = t.stride()
    if sd != 1 or (sh != dim and h > 1):
        raise ValueError(f"{what}: the heads of a row must lie side by side")
    return n, h, ld if n > 1 else h * dim


def make_kv_cache(n_pages: int, kv_heads: int, head_dim: int, page_tokens: int = 64, device="cuda") -> KVCache:
    """An empty paged cache: codes k [n_pages, kv_heads, page_tokens, head_dim], v [n_pages, kv_heads, head_dim,
    page_tokens], scales [n_pages, kv_heads] (not initialised: a page's scale starts with its first token)."""
    k = torch.empty(n_pages, kv_heads, page_tokens, head_dim, dtype=torch.int8, device=device)
    v = torch.empty(n_pages, kv_heads, head_dim, page_tokens, dtype=torch.int8, device=device)
    return (k, v, torch.empty(n_pages, kv_heads, dtype=torch.float32, device=device),
            torch.empty(n_pages, kv_heads, dtype=torch.float32, device=device))


def _cache_of(cache: KVCache):
    """(the C description, kv_heads, head_dim, page_tokens, device index)"""
    k, v, ks, vs = cache
    n, h, p, d = k.shape
    if v.shape != (n, h, d, p) or ks.shape != (n, h) or vs.shape != (n, h):
        raise ValueError("cache: k [pages, heads, tokens, dim], v [pages, heads, dim, tokens], scales [pages, heads]")
    if k.dtype != torch.int8 or v.dtype != torch.int8 or ks.dtype != torch.float32 or vs.dtype != torch.float32:
        raise TypeError("cache: int8 codes and fp32 scales")
    if not (k.is_contiguous() and v.is_contiguous() and ks.is_contiguous() and vs.is_contiguous()):
        raise ValueError("cache tensors must be contiguous")
    dev = _device_of(k)
    _on_device(dev, v, ks, vs)
    return awsrc_kv_cache(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), n, h, d, p, 0), h, d, p, dev


def _batch_of(dev: int, cu, kv_len, page_table):
    """(sequences, table stride) of a batch's int32 device tensors."""
    if cu.dtype != torch.int32 or kv_len.dtype != torch.int32 or page_table.dtype != torch.int32:
        raise TypeError("cu, kv_len and page_table must be int32")
    _on_device(dev, cu, kv_len, page_table)
    if page_table.dim() != 2:
        raise ValueError("page_table [sequences, pages]")
    n, ld = page_table.shape
    if cu.shape != (n + 1,) or kv_len.shape != (n,):
        raise ValueError("cu [sequences + 1], kv_len [sequences], page_table [sequences, pages]")
    if not (cu.is_contiguous() and kv_len.is_contiguous() and page_table.is_contiguous()):
        raise ValueError("cu, kv_len and page_table must be contiguous")
    return n, ld


def awsrc_quantize_rows_i8(x: torch.Tensor, out=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """int8 codes [rows, cols] and fp32 scales [rows] of a matrix (activations per token, weights per output channel).
    The codes' rows lie a multiple of 16 bytes apart, as awsrc_matmul_i8 and awsrc_linear_i8 take them.  Codes given in
    `out` on such rows are filled with 0 up to the next multiple of 16; on others nothing past their columns is written."""
    rows, cols, ld = _rows_of(x, "x")
    dev = _device_of(x)
    if out is None:
        out = (_empty((rows, -(-cols // 16) * 16), x, torch.int8, stream)[:, :cols], _empty((rows,), x, torch.float32, stream))
    codes, scale = out
    _on_device(dev, codes, scale)
    if (codes.shape != x.shape or codes.dtype != torch.int8 or scale.shape != (rows,) or scale.dtype != torch.float32
            or not scale.is_contiguous()):
        raise ValueError("out: int8 codes of x's shape and fp32 scales [rows]")
    _check(LIB.awsrc_quantize_rows_i8(x.data_ptr(), _act_code(x.dtype), rows, cols, ld, codes.data_ptr(),
                                      _code_rows(codes), scale.data_ptr(), _raw_stream(dev, stream)))
    return codes, scale


def _check_product_args(dev: int, N: int, scale, bias):
    if scale.get_device() != dev or (bias is not None and bias.get_device() != dev):
        raise ValueError(f"scales and bias must be on cuda:{dev}")
    if scale.shape != (N,) or scale.dtype != torch.float32 or not scale.is_contiguous():
        raise ValueError("weight scales: fp32 [N]")
    if bias is not None and (bias.shape != (N,) or bias.dtype != torch.float32 or not bias.is_contiguous()):
        raise ValueError("bias: fp32 [N]")


def _out_rows(dev: int, out, M: int, N: int) -> int:
    _on_device(dev, out)
    if out.shape != (M, N):
        raise ValueError(f"out: expected {(M, N)}, got {tuple(out.shape)}")
    return _rows_of(out, "out")[2]


@functools.lru_cache(_WS_SIZES)
def matmul_i8_workspace_bytes(M: int, N: int, K: int) -> int:
    n = ctypes.c_size_t(0)
    ld = -(-K // 16) * 16
    _check(LIB.awsrc_matmul_i8(None, ld, None, None, ld, None, None, M, N, K, None, AWSRC_DTYPE_F32, N, None,
                               ctypes.byref(n), None))
    return n.value


@functools.lru_cache(_WS_SIZES)
def linear_i8_workspace_bytes(M: int, N: int, K: int) -> int:
    n = ctypes.c_size_t(0)
    ld = -(-K // 16) * 16
    _check(LIB.awsrc_linear_i8(None, AWSRC_DTYPE_F32, K, None, ld, None, None, M, N, K, None, AWSRC_DTYPE_F32, N, None,
                               ctypes.byref(n), None))
    return n.value


def _sized_workspace(workspace, need: int, like: torch.Tensor, stream):
    """(address, size, the tensor that holds it)"""
    if workspace is None:
        if need == 0:
            return None, 0, None
    else:  # a kernel writes to it: its own device's memory, as much as it says
        if workspace.device != like.device:
            raise ValueError(f"workspace on {workspace.device}, tensors on {like.device}")
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
    if workspace is None or workspace.nbytes < need:
        workspace = _empty((need,), like, torch.uint8, stream)
    return workspace.data_ptr(), workspace.nbytes, workspace


def awsrc_matmul_i8(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor,
                    bias: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """a [M, K] times b [N, K] transposed, int8 codes with fp32 scales per row: [M, N] in out_dtype (or out's)."""
    M, K, lda = _i8_rows(a, "a")
    N, Kb, ldb = _i8_rows(b, "b")
    if K != Kb:
        raise ValueError(f"a has {K} columns, b {Kb}")
    dev = _device_of(a)
    _on_device(dev, a_scale, b)
    if a_scale.shape != (M,) or a_scale.dtype != torch.float32 or not a_scale.is_contiguous():
        raise ValueError("a_scale: fp32 [M]")
    if out is None:
        out, ldo = _empty((M, N), a, out_dtype, stream), N
    else:
        ldo = _out_rows(dev, out, M, N)
    _check_product_args(dev, N, b_scale, bias)
    ws, n, keep = _sized_workspace(workspace, matmul_i8_workspace_bytes(M, N, K), a, stream)
    if M and N:
        _check(LIB.awsrc_matmul_i8(a.data_ptr(), lda, a_scale.data_ptr(), b.data_ptr(), ldb, b_scale.data_ptr(),
                                   None if bias is None else bias.data_ptr(), M, N, K, out.data_ptr(), _act_code(out.dtype),
                                   ldo, ws, ctypes.c_size_t(n), _raw_stream(dev, stream)))
    return out


def awsrc_linear_i8(x: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                    out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """A linear layer on int8 weights: x [M, K] quantized per row, times w [N, K] (codes and scales as
    awsrc_quantize_rows_i8 makes them from the weight matrix) transposed, plus bias; [M, N] in x's type by default.
    For inference: the result carries no gradient."""
    M, K, ldx = _rows_of(x, "x")
    N, Kw, ldw = _i8_rows(w, "w")
    if K != Kw:
        raise ValueError(f"x has {K} columns, w {Kw}")
    dev = _device_of(x)
    if out is None:
        out, ldo = _empty((M, N), x, x.dtype if out_dtype is None else out_dtype, stream), N
    else:
        ldo = _out_rows(dev, out, M, N)
    if w.get_device() != dev:
        raise ValueError(f"tensors must be on one device: {w.device} and cuda:{dev}")
    _check_product_args(dev, N, w_scale, bias)
    ws, n, keep = _sized_workspace(workspace, linear_i8_workspace_bytes(M, N, K), x, stream)
    if M and N:
        _check(LIB.awsrc_linear_i8(x.data_ptr(), _act_code(x.dtype), ldx, w.data_ptr(), ldw, w_scale.data_ptr(),
                                   None if bias is None else bias.data_ptr(), M, N, K, out.data_ptr(), _act_code(out.dtype),
                                   ldo, ws, ctypes.c_size_t(n), _raw_stream(dev, stream)))
    return out


def awsrc_kv_append(cache: KVCache, k: torch.Tensor, v: torch.Tensor, cu: torch.Tensor, kv_len: torch.Tensor,
                    page_table: torch.Tensor, max_new: int, cos: Optional[torch.Tensor] = None,
                    sin: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, interleaved: bool = False,
                    q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """Appends rows of k and v [rows, kv_heads, head_dim] (views of a fused projection's output will do) to the cache,
    keys rotated by the tables cos, sin [positions, rot / 2]; returns q [rows, q_heads, head_dim] rotated the same way.
    kv_len counts the appended tokens; max_new is at least the most rows that one sequence brings.  q_out does not
    overlap q.  For inference: no gradient is recorded."""
    c, heads, dim, _, dev = _cache_of(cache)
    n_seq, table_ld = _batch_of(dev, cu, kv_len, page_table)
    _on_device(dev, k, v, q, cos, sin, q_out)
    dtype = k.dtype
    rows, _, ldk = _heads_of(k, "k", heads, dim, dtype)
    rows_v, _, ldv = _heads_of(v, "v", heads, dim, dtype)
    if rows_v != rows:
        raise ValueError("k, v and q must have the same rows")
    rot = rope_len = 0
    cos_p = sin_p = q_p = qo_p = None
    if cos is not None:
        if sin is None or cos.dim() != 2 or cos.shape != sin.shape or cos.dtype != torch.float32 or sin.dtype != torch.float32:
            raise ValueError("cos, sin: fp32 [positions, rot / 2]")
        if not (cos.is_contiguous() and sin.is_contiguous()):
            raise ValueError("cos and sin must be contiguous")
        rope_len, rot = cos.shape
        rot, cos_p, sin_p = 2 * rot, cos.data_ptr(), sin.data_ptr()
    elif sin is not None:
        raise ValueError("cos and sin go together")
    ldq = ldqo = q_heads = 0
    if q is not None:
        rows_q, q_heads, ldq = _heads_of(q, "q", None, dim, dtype)
        if rows_q != rows:
            raise ValueError("k, v and q must have the same rows")
        if q_out is None:
            q_out, ldqo = _empty((rows, q_heads, dim), q, dtype, stream), q_heads * dim
        elif q_out.shape != q.shape:
            raise ValueError("q_out: q's shape")
        else:
            ldqo = _heads_of(q_out, "q_out", q_heads, dim, dtype)[2]
        q_p, qo_p = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    _check(LIB.awsrc_kv_append(c, k.data_ptr(), ldk, v.data_ptr(), ldv, q_p, ldq, q_heads, qo_p, ldqo, _act_code(dtype), cos_p,
                               sin_p, rope_len, rot, interleaved, n_seq, rows, cu.data_ptr(), kv_len.data_ptr(),
                               page_table.data_ptr(), table_ld, min(max_new, rows), _raw_stream(dev, stream)))
    return q_out


def awsrc_kv_read(cache: KVCache, cu: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor, rows: int, max_new: int,
                  dtype: torch.dtype = torch.bfloat16, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """What the cache holds for the last cu[s + 1] - cu[s] tokens of each sequence: dense keys and values
    [rows, kv_heads, head_dim], rows = cu[-1]."""
    c, heads, dim, _, dev = _cache_of(cache)
    n_seq, table_ld = _batch_of(dev, cu, kv_len, page_table)
    k = _empty((rows, heads, dim), cu, dtype, stream)
    v = _empty((rows, heads, dim), cu, dtype, stream)
    _check(LIB.awsrc_kv_read(c, n_seq, rows, cu.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(), table_ld,
                             min(max_new, rows), k.data_ptr(), v.data_ptr(), _act_code(dtype), _raw_stream(dev, stream)))
    return k, v


@functools.lru_cache(_WS_SIZES)
def kv_attention_workspace_bytes(n_seq: int, rows: int, max_new: int, max_kv: int, table_ld: int, q_heads: int, kv_heads: int,
                                 head_dim: int, page_tokens: int) -> int:
    c = awsrc_kv_cache(None, None, None, None, 1, kv_heads, head_dim, page_tokens, 0)
    n = ctypes.c_size_t(0)
    w = q_heads * head_dim
    _check(LIB.awsrc_kv_attention(c, None, w, q_heads, AWSRC_DTYPE_BF16, n_seq, rows, None, None, None, table_ld, max_new,
                                  max_kv, 1.0, 1, None, w, None, ctypes.byref(n), None))
    return n.value


def awsrc_kv_attention(cache: KVCache, q: torch.Tensor, cu: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor,
                       max_new: int, max_kv: int, scale: Optional[float] = None, causal: bool = True,
                       out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """Attention of q [rows, q_heads, head_dim] (rotated, bf16 or fp16) over the cache; scale defaults to
    head_dim ** -0.5.  max_new and max_kv bound the rows and the cached tokens of a sequence.  For inference: the result
    carries no gradient."""
    c, kv_heads, dim, page, dev = _cache_of(cache)
    n_seq, table_ld = _batch_of(dev, cu, kv_len, page_table)
    _on_device(dev, q, out)
    dtype = q.dtype
    rows, heads, ldq = _heads_of(q, "q", None, dim, dtype)
    if out is None:
        out, ldo = _empty((rows, heads, dim), q, dtype, stream), heads * dim
    elif out.shape != q.shape:
        raise ValueError("out: q's shape")
    else:
        ldo = _heads_of(out, "out", heads, dim, dtype)[2]
    max_new = min(max_new, rows)
    ws, n, keep = _sized_workspace(workspace, kv_attention_workspace_bytes(n_seq, rows, max_new, max_kv, table_ld, heads,
                                                                           kv_heads, dim, page), q, stream)
    if rows:
        _check(LIB.awsrc_kv_attention(c, q.data_ptr(), ldq, heads, _act_code(dtype), n_seq, rows, cu.data_ptr(), kv_len.data_ptr(),
                                      page_table.data_ptr(), table_ld, max_new, max_kv, dim ** -0.5 if scale is None else scale,
                                      causal, out.data_ptr(), ldo, ws, ctypes.c_size_t(n), _raw_stream(dev, stream)))
    return out


# ------------------------------------------------------------------ e4m3 codes
BLOCK_F8 = 128  # columns, and rows of a weight matrix, that share a scale
_F8 = torch.float8_e4m3fn


def _blocks_shape(rows: int, cols: int, block_rows: int):
    if block_rows not in (1, BLOCK_F8):
        raise ValueError("block_rows must be 1 or 128")
    nb = -(-cols // BLOCK_F8)
    return (nb, rows) if block_rows == 1 else (-(-rows // BLOCK_F8), nb)


def _check_scales(dev: int, scale: torch.Tensor, shape, what: str) -> None:
    if scale.get_device() != dev:
        raise ValueError(f"{what} must be on cuda:{dev}")
    if scale.shape != shape or scale.dtype != torch.float32 or not scale.is_contiguous():
        raise ValueError(f"{what}: contiguous fp32 {list(shape)}")


def awsrc_quantize_blocks_f8(x: torch.Tensor, block_rows: int = 1, out=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """e4m3 codes [rows, cols] (torch.float8_e4m3fn) and fp32 scales of a matrix: block_rows 1, a scale for each row and 128
    columns, [ceil(cols / 128), rows] (activations); 128, one for each block of 128 x 128, [ceil(rows / 128),
    ceil(cols / 128)] (weights).  The codes' rows lie a multiple of 16 bytes apart, as the products take them."""
    rows, cols, ld = _rows_of(x, "x")
    dev = _device_of(x)
    shape = _blocks_shape(rows, cols, block_rows)
    if out is None:
        out = (_empty((rows, -(-cols // 16) * 16), x, _F8, stream)[:, :cols], _empty(shape, x, torch.float32, stream))
    codes, scale = out
    _on_device(dev, codes)
    if codes.shape != x.shape or codes.dtype != _F8:
        raise ValueError(f"out: codes of x's shape in {_F8}")
    _check_scales(dev, scale, shape, "scales")
    _check(LIB.awsrc_quantize_blocks_f8(x.data_ptr(), _act_code(x.dtype), rows, cols, ld, block_rows, codes.data_ptr(),
                                        _rows_of(codes, "codes")[2], scale.data_ptr(), _raw_stream(dev, stream)))
    return codes, scale


def awsrc_dequantize_blocks_f8(codes: torch.Tensor, scale: torch.Tensor, block_rows: int = 1, dtype: torch.dtype = torch.bfloat16,
                               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The values that codes stand for as a dense matrix of `dtype` (or out's): code * scale, rounded once."""
    if codes.dtype != _F8:
        raise TypeError(f"codes must be {_F8}, not {codes.dtype}")
    rows, cols, ld = _rows_of(codes, "codes")
    dev = _device_of(codes)
    _check_scales(dev, scale, _blocks_shape(rows, cols, block_rows), "scales")
    if out is None:
        out, ldo = _empty((rows, cols), codes, dtype, stream), cols
    else:
        ldo = _out_rows(dev, out, rows, cols)
    _check(LIB.awsrc_dequantize_blocks_f8(codes.data_ptr(), ld, scale.data_ptr(), rows, cols, block_rows, out.data_ptr(),
                                          _act_code(out.dtype), ldo, _raw_stream(dev, stream)))
    return out


@functools.lru_cache(_WS_SIZES)
def matmul_f8_workspace_bytes(M: int, N: int, K: int) -> int:
    n = ctypes.c_size_t(0)
    ld = -(-K // 16) * 16
    _check(LIB.awsrc_matmul_f8(None, ld, None, None, ld, None, None, M, N, K, None, AWSRC_DTYPE_F32, N, None,
                               ctypes.byref(n), None))
    return n.value


@functools.lru_cache(_WS_SIZES)
def linear_f8_workspace_bytes(M: int, N: int, K: int) -> int:
    n = ctypes.c_size_t(0)
    ld = -(-K // 16) * 16
    _check(LIB.awsrc_linear_f8(None, AWSRC_DTYPE_F32, K, None, ld, None, None, M, N, K, None, AWSRC_DTYPE_F32, N, None,
                               ctypes.byref(n), None))
    return n.value


def _check_product_f8(dev: int, N: int, K: int, scale, bias):
    _check_scales(dev, scale, (-(-N // BLOCK_F8), -(-K // BLOCK_F8)), "weight scales")
    if bias is not None and (bias.get_device() != dev or bias.shape != (N,) or bias.dtype != torch.float32 or not bias.is_contiguous()):
        raise ValueError(f"bias: fp32 [N] on cuda:{dev}")


def awsrc_matmul_f8(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor,
                    bias: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """a [M, K] times b [N, K] transposed, e4m3 codes with fp32 scales as awsrc_quantize_blocks_f8 makes them (a with
    block_rows 1, b with 128): [M, N] in out_dtype (or out's), sums in fp32 for each type."""
    M, K, lda = _i8_rows(a, "a", _F8)
    N, Kb, ldb = _i8_rows(b, "b", _F8)
    if K != Kb:
        raise ValueError(f"a has {K} columns, b {Kb}")
    dev = _device_of(a)
    _on_device(dev, b)
    _check_scales(dev, a_scale, (-(-K // BLOCK_F8), M), "a_scale")
    if out is None:
        out, ldo = _empty((M, N), a, out_dtype, stream), N
    else:
        ldo = _out_rows(dev, out, M, N)
    _check_product_f8(dev, N, K, b_scale, bias)
    ws, n, keep = _sized_workspace(workspace, matmul_f8_workspace_bytes(M, N, K), a, stream)
    if M and N:
        _check(LIB.awsrc_matmul_f8(a.data_ptr(), lda, a_scale.data_ptr(), b.data_ptr(), ldb, b_scale.data_ptr(),
                                   None if bias is None else bias.data_ptr(), M, N, K, out.data_ptr(), _act_code(out.dtype),
                                   ldo, ws, ctypes.c_size_t(n), _raw_stream(dev, stream)))
    return out


def awsrc_linear_f8(x: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                    out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """A linear layer on e4m3 weights: x [M, K] quantized per row and 128 columns, times w [N, K] (codes and scales as
    awsrc_quantize_blocks_f8 makes them from the weight matrix with block_rows 128) transposed, plus bias; [M, N] in x's type
    by default.  For inference: the result carries no gradient."""
    M, K, ldx = _rows_of(x, "x")
    N, Kw, ldw = _i8_rows(w, "w", _F8)
    if K != Kw:
        raise ValueError(f"x has {K} columns, w {Kw}")
    dev = _device_of(x)
    if out is None:
        out, ldo = _empty((M, N), x, x.dtype if out_dtype is None else out_dtype, stream), N
    else:
        ldo = _out_rows(dev, out, M, N)
    _on_device(dev, w)
    _check_product_f8(dev, N, K, w_scale, bias)
    ws, n, keep = _sized_workspace(workspace, linear_f8_workspace_bytes(M, N, K), x, stream)
    if M and N:
        _check(LIB.awsrc_linear_f8(x.data_ptr(), _act_code(x.dtype), ldx, w.data_ptr(), ldw, w_scale.data_ptr(),
                                   None if bias is None else bias.data_ptr(), M, N, K, out.data_ptr(), _act_code(out.dtype),
                                   ldo, ws, ctypes.c_size_t(n), _raw_stream(dev, stream)))
    return out


# ------------------------------------------------------------------ steps with drafted tokens
PagePool = Tuple[torch.Tensor, torch.Tensor]  # free pages [n_pages], how many of them are free [1], int32


def make_page_pool(n_pages: int, device="cuda") -> PagePool:
    """The pool of a cache of which no page is held yet: (free pages, a stack; their number)."""
    return (torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device),
            torch.tensor([n_pages], dtype=torch.int32, device=device))


_I32 = torch.int32


def _ints(t: torch.Tensor, n: int, what: str, dev: int) -> int:
    """The address of n int32 values."""
    if t.dtype is not _I32 or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous int32 [{n}] on cuda:{dev}, got {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


@functools.lru_cache(_WS_SIZES)
def kv_plan_workspace_bytes(n_seq: int, rows: int) -> int:
    n = ctypes.c_size_t(0)
    _check(LIB.awsrc_kv_plan(awsrc_page_pool(None, None, 1, 16, 0), n_seq, None, None, None, None, 1, rows, None, None, None, None,
                             None, None, None, ctypes.byref(n), None))
    return n.value


def awsrc_kv_plan(pool: PagePool, kv_len: torch.Tensor, keep: torch.Tensor, new_len: torch.Tensor, page_table: torch.Tensor,
                  page_tokens: int, rows: int, kv_len_out: Optional[torch.Tensor] = None, n_free_out: Optional[torch.Tensor] = None,
                  out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                  workspace: Optional[torch.Tensor] = None,
                  stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Plans a step on the device: slot s of the batch holds kv_len[s] cached tokens, keeps the first keep[s] of them and
    appends new_len[s], of at most `rows` in all.  Pages are given back to the pool and taken from it; page_table, kv_len
    and the pool's count are brought up to date in place (or written to kv_len_out and n_free_out).  Returns cu [slots + 1],
    and for each of the `rows` its slot, its position (int32) and page * page_tokens + position % page_tokens (int64), -1
    past the last.  A slot for which there are no pages gets no rows (cu tells) and keeps its tokens."""
    free, n_free = pool
    dev = _device_of(kv_len)
    n = kv_len.numel()
    if page_table.dim() != 2 or page_table.shape[0] != n:
        raise ValueError("page_table [slots, pages]")
    ld = page_table.shape[1]
    n_pages = free.numel()
    c = awsrc_page_pool(_ints(free, n_pages, "free pages", dev), _ints(n_free, 1, "number of free pages", dev), n_pages, page_tokens, 0)
    kv_p = _ints(kv_len, n, "kv_len", dev)
    keep_p, new_p = _ints(keep, n, "keep", dev), _ints(new_len, n, "new_len", dev)
    table_p = _ints(page_table, n * ld, "page_table", dev)
    kv_out_p = kv_p if kv_len_out is None else _ints(kv_len_out, n, "kv_len_out", dev)
    free_out_p = c.n_free if n_free_out is None else _ints(n_free_out, 1, "n_free_out", dev)
    if out is None:
        cu, seq, slot = _empty(n + 1, kv_len, _I32, stream), _empty(rows, kv_len, _I32, stream), _empty(rows, kv_len, torch.int64, stream)
        pos = _empty(rows, kv_len, _I32, stream)
        cu_p, seq_p, pos_p = cu.data_ptr(), seq.data_ptr(), pos.data_ptr()
    else:
        cu, seq, pos, slot = out
        cu_p, seq_p, pos_p = _ints(cu, n + 1, "cu", dev), _ints(seq, rows, "row slots", dev), _ints(pos, rows, "row positions", dev)
        if slot.dtype != torch.int64 or slot.numel() != rows or not slot.is_contiguous() or slot.get_device() != dev:
            raise ValueError(f"row places: contiguous int64 [{rows}] on cuda:{dev}")
    ws, size, held = _sized_workspace(workspace, kv_plan_workspace_bytes(n, rows), kv_len, stream)
    _check(LIB.awsrc_kv_plan(c, n, kv_p, keep_p, new_p, table_p, ld, rows, kv_out_p, free_out_p, cu_p, seq_p, pos_p,
                             slot.data_ptr(), ws, ctypes.c_size_t(size), _raw_stream(dev, stream)))
    return cu, seq, pos, slot


@functools.lru_cache(_WS_SIZES)
def verify_drafts_workspace_bytes(n_seq: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    _check(LIB.awsrc_verify_drafts(None, vocab, None, 0, AWSRC_DTYPE_F32, vocab, n_seq, 0, None, None, None, None, None, None,
                                   None, None, ctypes.byref(n), None))
    return n.value


def awsrc_verify_drafts(p: torch.Tensor, tokens: torch.Tensor, u: torch.Tensor, cu: torch.Tensor, q: Optional[torch.Tensor] = None,
                        kv_len: Optional[torch.Tensor] = None, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
                        keep: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        stream=None) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Verifies a step's drafts: tokens [rows] packed by cu, each sequence's last certain token and then its drafts; p
    [rows, vocab] the target's probabilities of what follows each row, q those that the drafts were drawn from (None:
    drafts that were not drawn); u [rows] uniform random numbers in [0, 1).  Returns the tokens that follow (int32 [rows],
    from each sequence's first row on, then -1; rows of no sequence stay as they were), how many they are (int32
    [sequences]), and, given kv_len, how many cached tokens stay (awsrc_kv_plan's keep), else None."""
    rows, V, ldp = _rows_of(p, "p")
    dev = _device_of(p)
    dtype = p.dtype
    q_p = None
    ldq = 0
    if q is not None:
        if q.shape != p.shape or q.dtype != dtype or q.get_device() != dev:
            raise ValueError("q: p's shape, type and device")
        ldq, q_p = _rows_of(q, "q")[2], q.data_ptr()
    n = cu.numel() - 1
    if n < 0:
        raise ValueError("cu [sequences + 1]")
    if u.dtype != torch.float32 or u.numel() != rows or not u.is_contiguous() or u.get_device() != dev:
        raise ValueError(f"u: contiguous fp32 [{rows}] on cuda:{dev}")
    cu_p, tokens_p = _ints(cu, n + 1, "cu", dev), _ints(tokens, rows, "tokens", dev)
    if out is None:
        out = (_empty(rows, p, _I32, stream), _empty(n, p, _I32, stream))
        out_p, n_p = out[0].data_ptr(), out[1].data_ptr()
    else:
        out_p, n_p = _ints(out[0], rows, "tokens that follow", dev), _ints(out[1], n, "numbers of tokens", dev)
    kv_p = keep_p = None
    if kv_len is not None:
        kv_p = _ints(kv_len, n, "kv_len", dev)
        if keep is None:
            keep = _empty(n, p, _I32, stream)
            keep_p = keep.data_ptr()
        else:
            keep_p = _ints(keep, n, "keep", dev)
    elif keep is not None:
        raise ValueError("keep without kv_len")
    ws, size, held = _sized_workspace(workspace, verify_drafts_workspace_bytes(n, V), p, stream)
    _check(LIB.awsrc_verify_drafts(p.data_ptr(), ldp, q_p, ldq, _act_code(dtype), V, n, rows, cu_p, tokens_p, u.data_ptr(), kv_p,
                                   out_p, n_p, keep_p, ws, ctypes.c_size_t(size), _raw_stream(dev, stream)))
    return out[0], out[1], keep
