"""Python binding of libhilo.so: argument marshalling only.

Every function here has the name of its C entry point (include/hilo.h), takes torch tensors that
already live on the GPU, passes their device pointers and the current HIP stream to the library,
and raises HiloError on a non-zero status.  All arithmetic happens in the library's kernels; there
is no fallback of any kind -- without the built library every call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libhilo.so")

F32, BF16 = 0, 1
THRESHOLD, TOPK = 0, 1
PARTITION, OVERLAP, DROP = 0, 1, 2  # hilo_token_set
ROPE_ADJACENT, ROPE_ONE_SPECTRUM = 1, 2  # hilo_rope_flags
NORM_LAYER, NORM_RMS = 0, 1  # hilo_norm_kind
ACT_NONE, ACT_GELU, ACT_SILU = 0, 1, 2  # hilo_act
DTYPES = {"f32": F32, "bf16": BF16}
TORCH_DTYPES = {F32: torch.float32, BF16: torch.bfloat16}


class HiloError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed with status {status}: {status_str(status)}")


class hilo_shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("batch", "images", "grid_h", "grid_w", "text_len", "dim", "heads", "head_dim",
                 "mlp_dim", "dtype")]


class hilo_attn_w(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_qkv", "b_qkv", "w_o", "b_o")]


class hilo_mlp_w(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w1", "b1", "w2", "b2")]


class hilo_attn_w_fp8(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_qkv", "s_qkv", "b_qkv", "w_o", "s_o", "b_o")]


class hilo_mlp_w_fp8(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w1", "s1", "b1", "w2", "s2", "b2")]


class hilo_rotary(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("heads", "head_dim", "axes", "flags")] + [
        ("pairs", ctypes.c_int32 * 4), ("base", ctypes.c_double * 4)]


class hilo_norms(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("mod_stride", ctypes.c_int64), ("gate", ctypes.c_void_p), ("shift", ctypes.c_void_p),
                ("scale", ctypes.c_void_p), ("post_gain", ctypes.c_void_p * 2), ("pre_gain", ctypes.c_void_p * 2)]


class hilo_norm_grads(ctypes.Structure):
    _fields_ = [("mod_stride", ctypes.c_int64), ("gate", ctypes.c_void_p), ("shift", ctypes.c_void_p),
                ("scale", ctypes.c_void_p), ("post_gain", ctypes.c_void_p * 2), ("pre_gain", ctypes.c_void_p * 2)]


class hilo_linear_w_i8(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w", "s", "b")]


class hilo_linear_w(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w", "b", "w_gate", "b_gate")]


class hilo_linear_grads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w", "b", "w_gate", "b_gate")]


class hilo_linear_w_fp8(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w", "s", "b", "w_gate", "s_gate", "b_gate")]


_lib = None

_P = ctypes.c_void_p
_SIG = {
    "hilo_score": [ctypes.POINTER(hilo_shape), _P, _P, _P],
    "hilo_score_pixels": [ctypes.POINTER(hilo_shape), _P, _P, _P],
    "hilo_select": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.c_int32, ctypes.c_int32,
                    ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32),
                    _P, _P, _P, _P, _P, _P, _P],
    "hilo_select_tokens": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.c_int32, ctypes.c_int32,
                           ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32),
                           ctypes.c_int32, _P, _P, _P, _P, _P, _P, _P],
    "hilo_compress": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P, _P, _P, _P, _P, _P],
    "hilo_compress_norm": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                           ctypes.c_size_t, _P],
    "hilo_attention_normed": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.POINTER(hilo_attn_w), _P, _P,
                              ctypes.c_size_t, _P],
    "hilo_decompress_delta": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P, _P, _P, _P, _P, _P],
    "hilo_attention": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.POINTER(hilo_attn_w), _P, _P,
                       ctypes.c_size_t, _P],
    "hilo_mlp": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.POINTER(hilo_mlp_w), _P, _P,
                 ctypes.c_size_t, _P],
    "hilo_compress_norm_fp8": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                               ctypes.c_size_t, _P],
    "hilo_attention_fp8_normed": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.POINTER(hilo_attn_w_fp8), _P,
                                  _P, ctypes.c_size_t, _P],
    "hilo_attention_fp8": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.POINTER(hilo_attn_w_fp8), _P, _P,
                           ctypes.c_size_t, _P],
    "hilo_mlp_fp8": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.POINTER(hilo_mlp_w_fp8), _P, _P,
                     ctypes.c_size_t, _P],
    "hilo_quantize_rows": [ctypes.c_int32, _P, ctypes.c_int64, ctypes.c_int64, _P, _P, _P],
    "hilo_blocks": [ctypes.POINTER(hilo_shape), _P, _P, ctypes.POINTER(hilo_attn_w),
                    ctypes.POINTER(hilo_mlp_w), _P, ctypes.c_int32, _P, ctypes.c_size_t, _P],
    "hilo_decompress": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P, _P, _P, _P],
    "hilo_attention_core": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P, ctypes.c_size_t, _P],
    "hilo_attention_core_noalloc": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P],
    "hilo_attention_core_fp8": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P, ctypes.c_size_t, _P],
    "hilo_rope": [ctypes.c_int32, ctypes.POINTER(hilo_rotary), _P, ctypes.c_int64, _P, ctypes.c_int64, _P,
                  ctypes.c_int32, _P, ctypes.c_int64, _P],
    "hilo_token_positions": [ctypes.POINTER(hilo_shape), _P, _P, _P, _P, _P, _P, _P, _P],
    "hilo_norm_residual": [ctypes.c_int32, ctypes.POINTER(hilo_norms), _P, _P, _P, _P, _P, _P, ctypes.c_int64,
                           ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _P, _P],
    "hilo_norm_residual_backward": [ctypes.c_int32, ctypes.POINTER(hilo_norms), _P, _P, _P, _P, _P, _P, _P,
                                    ctypes.POINTER(hilo_norm_grads), ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                    ctypes.c_int32, _P, _P, ctypes.c_size_t, _P],
    "hilo_norm_residual_workspace_bytes": [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32],
    "hilo_quantize_rows_i8": [ctypes.c_int32, _P, ctypes.c_int64, ctypes.c_int64, _P, _P, _P, _P],
    "hilo_linear_i8": [ctypes.c_int32, ctypes.POINTER(hilo_linear_w_i8), _P, _P, _P, ctypes.c_int64, ctypes.c_int32,
                       ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _P, _P, ctypes.c_size_t, _P],
    "hilo_linear_i8_workspace_bytes": [ctypes.c_int64, ctypes.c_int32],
    "hilo_linear": [ctypes.c_int32, ctypes.POINTER(hilo_linear_w), _P, _P, _P, ctypes.c_int64, ctypes.c_int32,
                    ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _P, _P, ctypes.c_size_t, _P],
    "hilo_linear_workspace_bytes": [ctypes.c_int32, ctypes.c_int64] + [ctypes.c_int32] * 4,
    "hilo_linear_backward": [ctypes.c_int32, ctypes.POINTER(hilo_linear_w), _P, _P, _P, _P,
                             ctypes.POINTER(hilo_linear_grads), ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                             ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _P, _P, ctypes.c_size_t, _P],
    "hilo_linear_backward_workspace_bytes": [ctypes.c_int32, ctypes.c_int64] + [ctypes.c_int32] * 4,
    "hilo_quantize_blocks": [ctypes.c_int32, _P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, _P, _P, _P, _P],
    "hilo_linear_fp8": [ctypes.c_int32, ctypes.POINTER(hilo_linear_w_fp8), _P, _P, _P, _P, ctypes.c_int64,
                        ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _P, _P,
                        ctypes.c_size_t, _P],
    "hilo_linear_fp8_workspace_bytes": [ctypes.c_int64] + [ctypes.c_int32] * 3,
    "hilo_workspace_bytes": [ctypes.POINTER(hilo_shape)],
    "hilo_workspace_bytes_fp8": [ctypes.POINTER(hilo_shape)],
    "hilo_max_tokens": [ctypes.POINTER(hilo_shape)],
    "hilo_status_str": [ctypes.c_int32],
    "hilo_abi_version": [],
    "hilo_profile_enable": [ctypes.c_int32],
    "hilo_profile_read": [ctypes.c_int32, ctypes.POINTER(ctypes.c_double),
                          ctypes.POINTER(ctypes.c_int64)],
    "hilo_profile_kinds": [],
    "hilo_profile_name": [ctypes.c_int32],
}
_RES = {"hilo_workspace_bytes": ctypes.c_size_t, "hilo_workspace_bytes_fp8": ctypes.c_size_t, "hilo_max_tokens": ctypes.c_int64,
        "hilo_norm_residual_workspace_bytes": ctypes.c_size_t, "hilo_linear_i8_workspace_bytes": ctypes.c_size_t,
        "hilo_linear_workspace_bytes": ctypes.c_size_t, "hilo_linear_backward_workspace_bytes": ctypes.c_size_t,
        "hilo_linear_fp8_workspace_bytes": ctypes.c_size_t,
        "hilo_status_str": ctypes.c_char_p, "hilo_profile_name": ctypes.c_char_p}


def lib() -> ctypes.CDLL:
    """Load libhilo.so (built in-tree by paper_2606_13898_amd.build); raise if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2606_13898_amd.build`"
                              " (there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        for name, args in _SIG.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = _RES.get(name, ctypes.c_int32)
        _lib = L
    return _lib


def make_shape(s) -> hilo_shape:
    """hilo_shape from anything with the BlockShape attributes (dtype 'f32'/'bf16' or 0/1)."""
    dt = s.dtype if isinstance(s.dtype, int) else DTYPES[s.dtype]
    return hilo_shape(s.batch, s.images, s.grid_h, s.grid_w, s.text_len, s.dim, s.heads,
                      s.head_dim, s.mlp_dim, dt)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libhilo takes device tensors only")
    if not t.is_contiguous():
        raise ValueError("libhilo takes contiguous tensors only")
    return t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(fn: str, st: int):
    if st != 0:
        raise HiloError(fn, st)


def status_str(st: int) -> str:
    return lib().hilo_status_str(int(st)).decode()


def hilo_abi_version() -> int:
    return lib().hilo_abi_version()


def hilo_max_tokens(shape: hilo_shape) -> int:
    return lib().hilo_max_tokens(ctypes.byref(shape))


def hilo_workspace_bytes_fp8(shape: hilo_shape) -> int:
    return int(lib().hilo_workspace_bytes_fp8(ctypes.byref(shape)))


def hilo_workspace_bytes(shape: hilo_shape) -> int:
    return lib().hilo_workspace_bytes(ctypes.byref(shape))


def hilo_score(shape, x_img, energy, stream=None):
    _check("hilo_score", lib().hilo_score(ctypes.byref(shape), _ptr(x_img), _ptr(energy),
                                          _stream(stream)))


def hilo_score_pixels(shape, rgb, energy, stream=None):
    _check("hilo_score_pixels", lib().hilo_score_pixels(ctypes.byref(shape), _ptr(rgb), _ptr(energy),
                                                        _stream(stream)))


def hilo_select(shape, energy, force, dilate_r: int, mode: int, tau: Optional[Sequence[float]],
                keep: Optional[Sequence[int]], idx_map, fine_idx, pool_idx, counts, cu_seqlens,
                seg_off, stream=None):
    G = shape.batch * shape.images
    tau_arr = (ctypes.c_double * G)(*[float(t) for t in tau]) if tau is not None else None
    keep_arr = (ctypes.c_int32 * G)(*[int(k) for k in keep]) if keep is not None else None
    _check("hilo_select", lib().hilo_select(
        ctypes.byref(shape), _ptr(energy), _ptr(force), int(dilate_r), int(mode), tau_arr, keep_arr,
        _ptr(idx_map), _ptr(fine_idx), _ptr(pool_idx), _ptr(counts), _ptr(cu_seqlens),
        _ptr(seg_off), _stream(stream)))


def hilo_select_tokens(shape, energy, force, dilate_r: int, mode: int, tau: Optional[Sequence[float]],
                       keep: Optional[Sequence[int]], token_set: int, idx_map, fine_idx, pool_idx, counts,
                       cu_seqlens, seg_off, stream=None):
    G = shape.batch * shape.images
    tau_arr = (ctypes.c_double * G)(*[float(t) for t in tau]) if tau is not None else None
    keep_arr = (ctypes.c_int32 * G)(*[int(k) for k in keep]) if keep is not None else None
    _check("hilo_select_tokens", lib().hilo_select_tokens(
        ctypes.byref(shape), _ptr(energy), _ptr(force), int(dilate_r), int(mode), tau_arr, keep_arr,
        int(token_set), _ptr(idx_map), _ptr(fine_idx), _ptr(pool_idx), _ptr(counts), _ptr(cu_seqlens),
        _ptr(seg_off), _stream(stream)))


def hilo_decompress_delta(shape, z, x_img, idx_map, counts, cu_seqlens, seg_off, y_img, y_txt, stream=None):
    _check("hilo_decompress_delta", lib().hilo_decompress_delta(
        ctypes.byref(shape), _ptr(z), _ptr(x_img), _ptr(idx_map), _ptr(counts), _ptr(cu_seqlens),
        _ptr(seg_off), _ptr(y_img), _ptr(y_txt), _stream(stream)))


def hilo_compress(shape, x_img, x_txt, fine_idx, pool_idx, counts, cu_seqlens, seg_off, z,
                  stream=None):
    _check("hilo_compress", lib().hilo_compress(
        ctypes.byref(shape), _ptr(x_img), _ptr(x_txt), _ptr(fine_idx), _ptr(pool_idx),
        _ptr(counts), _ptr(cu_seqlens), _ptr(seg_off), _ptr(z), _stream(stream)))


def hilo_compress_norm(shape, x_img, x_txt, fine_idx, pool_idx, counts, cu_seqlens, seg_off, mod, z,
                       workspace, stream=None):
    _check("hilo_compress_norm", lib().hilo_compress_norm(
        ctypes.byref(shape), _ptr(x_img), _ptr(x_txt), _ptr(fine_idx), _ptr(pool_idx),
        _ptr(counts), _ptr(cu_seqlens), _ptr(seg_off), _ptr(mod), _ptr(z), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def attn_weights(ws: Sequence[dict]):
    arr = (hilo_attn_w * 2)()
    for k in range(2):
        arr[k] = hilo_attn_w(_ptr(ws[k]["w_qkv"]), _ptr(ws[k]["b_qkv"]), _ptr(ws[k]["w_o"]),
                             _ptr(ws[k]["b_o"]))
    return arr


def mlp_weights(ws: Sequence[dict]):
    arr = (hilo_mlp_w * 2)()
    for k in range(2):
        arr[k] = hilo_mlp_w(_ptr(ws[k]["w1"]), _ptr(ws[k]["b1"]), _ptr(ws[k]["w2"]),
                            _ptr(ws[k]["b2"]))
    return arr


def hilo_attention(shape, z, cu_seqlens, w, mod, workspace, stream=None):
    _check("hilo_attention", lib().hilo_attention(
        ctypes.byref(shape), _ptr(z), _ptr(cu_seqlens), w, _ptr(mod), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def hilo_attention_normed(shape, z, cu_seqlens, w, mod, workspace, stream=None):
    _check("hilo_attention_normed", lib().hilo_attention_normed(
        ctypes.byref(shape), _ptr(z), _ptr(cu_seqlens), w, _ptr(mod), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def hilo_mlp(shape, z, cu_seqlens, w, mod, workspace, stream=None):
    _check("hilo_mlp", lib().hilo_mlp(
        ctypes.byref(shape), _ptr(z), _ptr(cu_seqlens), w, _ptr(mod), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def hilo_quantize_rows(x, codes, scale, stream=None):
    """Per-row E4M3 codes (uint8 [rows][cols]) and float32 scales [rows] of x (float32 or bf16)."""
    dt = {torch.float32: F32, torch.bfloat16: BF16}.get(x.dtype, -1)
    rows, cols = (x.shape[0], x.shape[1]) if x.dim() == 2 else (-1, -1)
    _check("hilo_quantize_rows", lib().hilo_quantize_rows(
        dt, _ptr(x), rows, cols, _ptr(codes), _ptr(scale), _stream(stream)))


def quantize_fp8_weights(ws: Sequence[dict], stream=None):
    """Per stream, the FP8 codes and scales of the four projection weights (hilo_quantize_rows) next
    to the bf16 biases: the weight dicts hilo_attention_fp8 / hilo_mlp_fp8 take (keys w_qkv, s_qkv,
    b_qkv, w_o, s_o, b_o, w1, s1, b1, w2, s2, b2)."""
    out = []
    for w in ws:
        d = dict(w)
        for name, sname in (("w_qkv", "s_qkv"), ("w_o", "s_o"), ("w1", "s1"), ("w2", "s2")):
            src = w[name]
            codes = torch.empty(src.shape, dtype=torch.uint8, device=src.device)
            scale = torch.empty(src.shape[0], dtype=torch.float32, device=src.device)
            hilo_quantize_rows(src, codes, scale, stream)
            d[name], d[sname] = codes, scale
        out.append(d)
    return out


def attn_weights_fp8(ws: Sequence[dict]):
    arr = (hilo_attn_w_fp8 * 2)()
    for k in range(2):
        arr[k] = hilo_attn_w_fp8(_ptr(ws[k]["w_qkv"]), _ptr(ws[k]["s_qkv"]), _ptr(ws[k]["b_qkv"]),
                                 _ptr(ws[k]["w_o"]), _ptr(ws[k]["s_o"]), _ptr(ws[k]["b_o"]))
    return arr


def mlp_weights_fp8(ws: Sequence[dict]):
    arr = (hilo_mlp_w_fp8 * 2)()
    for k in range(2):
        arr[k] = hilo_mlp_w_fp8(_ptr(ws[k]["w1"]), _ptr(ws[k]["s1"]), _ptr(ws[k]["b1"]),
                                _ptr(ws[k]["w2"]), _ptr(ws[k]["s2"]), _ptr(ws[k]["b2"]))
    return arr


def hilo_attention_fp8(shape, z, cu_seqlens, w, mod, workspace, stream=None):
    _check("hilo_attention_fp8", lib().hilo_attention_fp8(
        ctypes.byref(shape), _ptr(z), _ptr(cu_seqlens), w, _ptr(mod), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def hilo_compress_norm_fp8(shape, x_img, x_txt, fine_idx, pool_idx, counts, cu_seqlens, seg_off, mod, z,
                           workspace, stream=None):
    _check("hilo_compress_norm_fp8", lib().hilo_compress_norm_fp8(
        ctypes.byref(shape), _ptr(x_img), _ptr(x_txt), _ptr(fine_idx), _ptr(pool_idx),
        _ptr(counts), _ptr(cu_seqlens), _ptr(seg_off), _ptr(mod), _ptr(z), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def hilo_attention_fp8_normed(shape, z, cu_seqlens, w, mod, workspace, stream=None):
    _check("hilo_attention_fp8_normed", lib().hilo_attention_fp8_normed(
        ctypes.byref(shape), _ptr(z), _ptr(cu_seqlens), w, _ptr(mod), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def hilo_mlp_fp8(shape, z, cu_seqlens, w, mod, workspace, stream=None):
    _check("hilo_mlp_fp8", lib().hilo_mlp_fp8(
        ctypes.byref(shape), _ptr(z), _ptr(cu_seqlens), w, _ptr(mod), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def stack_weights(blocks: Sequence[Sequence[dict]]):
    """Host arrays [n_blocks][2] of attention and MLP weight pointers for hilo_blocks."""
    n = len(blocks)
    aw = (hilo_attn_w * (2 * n))()
    mw = (hilo_mlp_w * (2 * n))()
    for l, ws in enumerate(blocks):
        for k in range(2):
            aw[2 * l + k] = hilo_attn_w(_ptr(ws[k]["w_qkv"]), _ptr(ws[k]["b_qkv"]), _ptr(ws[k]["w_o"]),
                                        _ptr(ws[k]["b_o"]))
            mw[2 * l + k] = hilo_mlp_w(_ptr(ws[k]["w1"]), _ptr(ws[k]["b1"]), _ptr(ws[k]["w2"]),
                                       _ptr(ws[k]["b2"]))
    return aw, mw


def hilo_blocks(shape, z, cu_seqlens, aw, mw, mod, n_blocks: int, workspace, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check("hilo_blocks", lib().hilo_blocks(
        ctypes.byref(shape), _ptr(z), _ptr(cu_seqlens), aw, mw, _ptr(mod), n_blocks, _ptr(workspace),
        ws_bytes, _stream(stream)))


def hilo_decompress(shape, z, idx_map, cu_seqlens, seg_off, y_img, y_txt, stream=None):
    _check("hilo_decompress", lib().hilo_decompress(
        ctypes.byref(shape), _ptr(z), _ptr(idx_map), _ptr(cu_seqlens), _ptr(seg_off),
        _ptr(y_img), _ptr(y_txt), _stream(stream)))


def hilo_attention_core(shape, qkv, cu_seqlens, out, workspace=None, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check("hilo_attention_core", lib().hilo_attention_core(
        ctypes.byref(shape), _ptr(qkv), _ptr(cu_seqlens), _ptr(out), _ptr(workspace), ws_bytes,
        _stream(stream)))


def hilo_attention_core_fp8(shape, qkv8, cu_seqlens, out, workspace, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("hilo_attention_core_fp8", lib().hilo_attention_core_fp8(
        ctypes.byref(shape), _ptr(qkv8), _ptr(cu_seqlens), _ptr(out), _ptr(workspace), ws_bytes,
        _stream(stream)))


def hilo_attention_core_noalloc(shape, qkv, cu_seqlens, out, stream=None):
    _check("hilo_attention_core_noalloc", lib().hilo_attention_core_noalloc(
        ctypes.byref(shape), _ptr(qkv), _ptr(cu_seqlens), _ptr(out), _stream(stream)))


# ---------------------------------------------------- rotary positions, sandwich norms, int8 products
#
# These calls check what the library cannot see: types, shapes, layouts and devices of the tensors, and sizes that its
# 32-bit arguments would cut to others.  They run on the current stream of the tensors' device, or on `stream`, which has
# to be one of that device.

_FLOATS = {torch.float32: F32, torch.bfloat16: BF16}


def _float_code(t: torch.Tensor) -> int:
    code = _FLOATS.get(t.dtype)
    if code is None:
        raise ValueError(f"float32 or bfloat16 expected, not {t.dtype}")
    return code


def _arg(t: Optional[torch.Tensor], dtype: torch.dtype, shape, dev: int, what: str) -> Optional[int]:
    """The pointer of a contiguous tensor of this type and shape on device `dev`, or None."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == dev and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what}: expected {dtype} {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{what}: on {t.device}, other tensors on device {dev}")
    raise ValueError(f"{what}: libhilo takes contiguous tensors only")


def _on_device(t: torch.Tensor) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError("libhilo takes device tensors only")
    return dev


# The current stream's handle without a Stream object around it (2.7 us of the 8 us that a small call took).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(fn, dev: int, stream, *args):
    """fn(*args, stream) with `dev` as the current device."""
    if dev != _current_device():
        with torch.cuda.device(dev):
            return _launch(fn, dev, stream, *args)
    st = getattr(lib(), fn)(*args, _raw_stream(dev) if stream is None else _stream(stream))
    if st != 0:
        raise HiloError(fn, st)


def _int32(*values: int):
    for v in values:
        if not -(1 << 31) <= v < 1 << 31:
            raise ValueError(f"{v} does not fit 32 bits")


def _packed(cu: torch.Tensor, dev: int):
    if cu.dtype is not torch.int32 or cu.dim() != 1 or cu.numel() < 2 or not cu.is_contiguous():
        raise ValueError("cu_seqlens: expected int32 [batch + 1]")
    if cu.get_device() != dev:
        raise ValueError(f"cu_seqlens: on {cu.device}, other tensors on device {dev}")
    return cu.numel() - 1, cu.data_ptr()


def rotary(heads: int, head_dim: int, pairs: Sequence[int], base=10000.0, flags: int = 0) -> hilo_rotary:
    """What hilo_rope turns: pairs of every axis, base one number or one per axis, flags ROPE_*."""
    axes = len(pairs)
    if not 1 <= axes <= 4:
        raise ValueError("1 to 4 axes")
    bases = [float(base)] * axes if isinstance(base, (int, float)) else [float(b) for b in base]
    if len(bases) != axes:
        raise ValueError("one base, or one per axis")
    _int32(heads, head_dim, flags, *pairs)
    return hilo_rotary(heads, head_dim, axes, flags, (ctypes.c_int32 * 4)(*pairs), (ctypes.c_double * 4)(*bases))


def hilo_rope(r: hilo_rotary, x: torch.Tensor, pos: torch.Tensor, out: torch.Tensor, cu: Optional[torch.Tensor] = None,
              backward: bool = False, stream=None):
    """out = the heads of x turned by their rows' positions (backward: by minus them).  x, out: [rows][heads *
    head_dim], any row stride (a view of the packed projection will do), out may be x; pos [rows][axes] float32; cu:
    the boundaries, whose last one bounds the rows."""
    dev, dtype = _on_device(x), _float_code(x)
    if x.dim() != 2 or x.shape[1] != r.heads * r.head_dim or out.shape != x.shape or out.dtype is not x.dtype:
        raise ValueError(f"x and out: expected [rows][{r.heads * r.head_dim}] of one type")
    rows = x.shape[0]
    if rows and (x.stride(1) != 1 or out.stride(1) != 1):
        raise ValueError("x and out: the last index is contiguous")
    if out.get_device() != dev:
        raise ValueError("x and out: on one device")
    ldx, ldo = (x.stride(0), out.stride(0)) if rows > 1 else (x.shape[1], x.shape[1])
    end = None
    if cu is not None:
        b, end = _packed(cu, dev)
        end += 4 * b
    _launch("hilo_rope", dev, stream, dtype, ctypes.byref(r), x.data_ptr(), ldx,
            _arg(pos, torch.float32, (rows, r.axes), dev, "pos"), rows, end, 1 if backward else 0, out.data_ptr(), ldo)


def hilo_token_positions(shape, fine_idx, pool_idx, counts, cu_seqlens, seg_off, text_pos, pos, stream=None):
    """pos [hilo_max_tokens(shape) rows or more][3] float32 of a compressed sequence's tokens from the int32 index lists of
    hilo_select, shaped as it leaves them: fine_idx [G][N], pool_idx [G][N / 4], counts [G][2], cu_seqlens [batch + 1],
    seg_off [G]; text_pos [text_len][3] float32 or None.  How many tokens there are only the device knows, so pos has to
    hold the most that any token set can have."""
    rows = hilo_max_tokens(shape)
    if rows < 0:
        raise HiloError("hilo_token_positions", 2)
    if pos is None:
        raise HiloError("hilo_token_positions", 1)
    dev, grids, patches, i32, f32 = _on_device(pos), shape.batch * shape.images, shape.grid_h * shape.grid_w, torch.int32, torch.float32
    if len(pos.shape) != 2 or pos.shape[0] < rows:
        raise ValueError(f"pos: expected [{rows} rows or more][3], not {tuple(pos.shape)}")
    _launch("hilo_token_positions", dev, stream, ctypes.byref(shape), _arg(fine_idx, i32, (grids, patches), dev, "fine_idx"),
            _arg(pool_idx, i32, (grids, patches // 4), dev, "pool_idx"), _arg(counts, i32, (grids, 2), dev, "counts"),
            _arg(cu_seqlens, i32, (shape.batch + 1,), dev, "cu_seqlens"), _arg(seg_off, i32, (grids,), dev, "seg_off"),
            _arg(text_pos, f32, (shape.text_len, 3), dev, "text_pos"), _arg(pos, f32, (pos.shape[0], 3), dev, "pos"))


def _vectors(h, vectors: dict, gains: dict):
    """Fills the pointers of a hilo_norms or hilo_norm_grads; keeps the tensors and what they are on it."""
    h.batch = h.dim = h.dev = None
    h.kept = [vectors]
    for name, v in vectors.items():
        if v is None:
            continue
        if v.dtype is not torch.float32 or v.dim() != 3 or v.shape[1] != 2 or (v.numel() and v.stride(2) != 1):
            raise ValueError(f"{name}: expected float32 [batch][2][dim]")
        stride = v.stride(1)
        if v.shape[0] > 1 and v.stride(0) != 2 * stride:
            raise ValueError(f"{name}: its (sample, stream) vectors have to be evenly spaced")
        if h.batch is not None and (tuple(v.shape), v.stride(1)) != ((h.batch, 2, h.dim), h.mod_stride):
            raise ValueError("gate, shift and scale: one shape and one spacing")
        h.batch, h.dim, h.mod_stride = v.shape[0], v.shape[2], stride
        _same_device(h, v, name)
        setattr(h, name, v.data_ptr())
    for name, pair in gains.items():
        if pair is None:
            continue
        for k in range(2):
            g = pair[k]
            if g is None:
                continue
            if g.dtype is not torch.float32 or g.dim() != 1 or not g.is_contiguous() or h.dim not in (None, g.numel()):
                raise ValueError(f"{name}: expected float32 [dim] for the image and the text stream")
            h.dim = g.numel()
            _same_device(h, g, name)
            h.kept.append(g)
            getattr(h, name)[k] = g.data_ptr()
    h.fits = (h.dim, h.batch, h.dev)
    return h


def _same_device(h, t, name):
    if h.dev is None:
        h.dev = _on_device(t)
    if t.get_device() != h.dev:
        raise ValueError(f"{name}: on {t.device}, other tensors on device {h.dev}")


def norms(kind: int = NORM_LAYER, eps: float = 1e-6, residual_scale: float = 1.0, *, gate=None, shift=None, scale=None,
          post_gain=None, pre_gain=None) -> hilo_norms:
    """The norms on both sides of a block: gate, shift, scale float32 [batch][2][dim] (views of one modulation tensor
    will do: mod[:, :, 2] of [batch][2][6][dim]), gains a pair of float32 [dim] (image, text stream).  Keeps the
    tensors alive; their values are read by each call."""
    _int32(kind)
    return _vectors(hilo_norms(kind, eps, residual_scale), {"gate": gate, "shift": shift, "scale": scale},
                    {"post_gain": post_gain, "pre_gain": pre_gain})


def norm_grads(*, gate=None, shift=None, scale=None, post_gain=None, pre_gain=None) -> hilo_norm_grads:
    """Where hilo_norm_residual_backward leaves the gradients of the vectors: shapes as in norms()."""
    return _vectors(hilo_norm_grads(), {"gate": gate, "shift": shift, "scale": scale},
                    {"post_gain": post_gain, "pre_gain": pre_gain})


def _norm_rows(fn: str, n, like: torch.Tensor, cu: torch.Tensor, text_len: int, others=None):
    if like.dim() != 2:
        raise ValueError("expected [rows][dim] tensors")
    dev, dim = _on_device(like), like.shape[1]
    batch, cu_ptr = _packed(cu, dev)
    if (dim | batch | text_len) >> 31:  # negative, or more than 31 bits
        raise HiloError(fn, 2)
    if n.fits != (dim, batch, dev):
        _fit(n, dim, batch, dev)
    if others is not None and others.fits != (dim, batch, dev):
        _fit(others, dim, batch, dev)
    return dev, dim, batch, cu_ptr


def _fit(h, dim: int, batch: int, dev: int):
    if h.dim not in (None, dim) or h.batch not in (None, batch) or h.dev not in (None, dev):
        raise ValueError(f"vectors for dim {h.dim}, batch {h.batch} on device {h.dev}; rows have dim {dim}, batch {batch} "
                         f"on device {dev}")


def hilo_norm_residual(n: hilo_norms, y, x, x_out, h, cu, text_len: int = 0, *, h_scale=None, stats=None, stream=None):
    """x_out = residual_scale x + gate norm(y), h = norm(x_out) (1 + scale) + shift; y and x_out, or h, may be None.
    h int8 with h_scale [rows]: codes and row scales.  stats [rows][4] float32: for the backward pass."""
    dev, dim, batch, cu_ptr = _norm_rows("hilo_norm_residual", n, x, cu, text_len)
    shape, rows, f32 = x.shape, x.shape[0], torch.float32
    like = y if y is not None else h
    if like is None:
        raise HiloError("hilo_norm_residual", 1)
    if h_scale is not None:
        hp = _arg(h, torch.int8, shape, dev, "h")
        dtype = F32 if y is None else _float_code(y)
    else:
        dtype = _float_code(like)
        hp = _arg(h, like.dtype, shape, dev, "h")
    _launch("hilo_norm_residual", dev, stream, dtype, ctypes.byref(n),
            None if y is None else _arg(y, y.dtype, shape, dev, "y"), _arg(x, f32, shape, dev, "x"),
            _arg(x_out, f32, shape, dev, "x_out"), hp, _arg(h_scale, f32, (rows,), dev, "h_scale"),
            _arg(stats, f32, (rows, 4), dev, "stats"), rows, dim, batch, text_len, cu_ptr)


def hilo_norm_residual_workspace_bytes(rows: int, batch: int, dim: int) -> int:
    return 0 if (batch | dim) >> 31 else lib().hilo_norm_residual_workspace_bytes(rows, batch, dim)


def hilo_norm_residual_backward(n: hilo_norms, dx_out, dh, y, x_out, stats, dx, dy, grads: Optional[hilo_norm_grads],
                                cu, text_len: int = 0, workspace=None, stream=None):
    """Gradients of hilo_norm_residual from dx_out (or None) and dh (or None): dx, dy, and those in grads."""
    dev, dim, batch, cu_ptr = _norm_rows("hilo_norm_residual_backward", n, dx, cu, text_len, grads)
    shape, rows, f32 = dx.shape, dx.shape[0], torch.float32
    like = dh if dh is not None else y
    if like is None:
        raise HiloError("hilo_norm_residual_backward", 1)
    dt, nbytes = like.dtype, 0
    if workspace is not None:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace: contiguous, on the tensors' device")
        nbytes = workspace.numel() * workspace.element_size()
    _launch("hilo_norm_residual_backward", dev, stream, _float_code(like), ctypes.byref(n),
            _arg(dx_out, f32, shape, dev, "dx_out"), _arg(dh, dt, shape, dev, "dh"), _arg(y, dt, shape, dev, "y"),
            _arg(x_out, f32, shape, dev, "x_out"), _arg(stats, f32, (rows, 4), dev, "stats"),
            _arg(dx, f32, shape, dev, "dx"), _arg(dy, dt, shape, dev, "dy"), None if grads is None else ctypes.byref(grads),
            rows, dim, batch, text_len, cu_ptr, None if workspace is None else workspace.data_ptr(), nbytes)


def hilo_quantize_rows_i8(x, codes, scale, cu=None, stream=None):
    """Per-row int8 codes [rows][cols] and float32 scales [rows] of x; cu: the boundaries, whose last one bounds the rows."""
    dev, dtype = _on_device(x), _float_code(x)
    if x.dim() != 2:
        raise ValueError("x: expected [rows][cols]")
    end = None
    if cu is not None:
        b, end = _packed(cu, dev)
        end += 4 * b
    rows, cols = x.shape
    _launch("hilo_quantize_rows_i8", dev, stream, dtype, _arg(x, x.dtype, x.shape, dev, "x"), rows, cols, end,
            _arg(codes, torch.int8, x.shape, dev, "codes"), _arg(scale, torch.float32, (rows,), dev, "scale"))


def quantize_i8_weights(w, b=None, stream=None) -> dict:
    """A projection's weights for linear_weights_i8: codes and scales of w [out][in], the bias kept."""
    codes = torch.empty(w.shape, dtype=torch.int8, device=w.device)
    scale = torch.empty(w.shape[0], dtype=torch.float32, device=w.device)
    hilo_quantize_rows_i8(w, codes, scale, stream=stream)
    return {"w": codes, "s": scale, "b": b}


def linear_weights_i8(ws: Sequence[dict]):
    """Weights of hilo_linear_i8: {"w": int8 [out][in], "s": float32 [out], "b": [out] or None} of the image and the text
    stream (one dict: of both).  Keeps the tensors alive."""
    ws = [dict(w) for w in ws]  # kept below, whatever the caller does with theirs
    if not 1 <= len(ws) <= 2:
        raise ValueError("weights of one or two streams")
    arr = (hilo_linear_w_i8 * 2)()
    arr.kept, arr.shape, arr.bias, arr.dev = ws, ws[0]["w"].shape, None, _on_device(ws[0]["w"])
    if len(arr.shape) != 2:
        raise ValueError("w: expected [out][in]")
    for k in range(2):
        w = ws[min(k, len(ws) - 1)]
        b = w.get("b")
        if b is not None:
            _float_code(b)
            if arr.bias not in (None, b.dtype):
                raise ValueError("b: of one type")
            arr.bias = b.dtype
        arr[k] = hilo_linear_w_i8(_arg(w["w"], torch.int8, arr.shape, arr.dev, "w"),
                                  _arg(w["s"], torch.float32, arr.shape[:1], arr.dev, "s"),
                                  None if b is None else _arg(b, b.dtype, arr.shape[:1], arr.dev, "b"))
    return arr


def hilo_linear_i8_workspace_bytes(rows: int, in_dim: int) -> int:
    return 0 if in_dim >> 31 else lib().hilo_linear_i8_workspace_bytes(rows, in_dim)


def hilo_linear_i8(w, x, out, cu, text_len: int = 0, *, x_scale=None, act: int = ACT_NONE, workspace=None, stream=None):
    """out [rows][out] = act(x w^T) of linear_weights_i8 w: x int8 codes with x_scale, or of out's type, quantised here."""
    dev, dtype = _on_device(out), _float_code(out)
    if dev != w.dev:
        raise ValueError(f"weights on device {w.dev}, out on device {dev}")
    if w.bias is not None and w.bias is not out.dtype:
        raise ValueError(f"b: {w.bias}, out: {out.dtype}")
    if workspace is None:
        raise HiloError("hilo_linear_i8", 1)
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous, on the tensors' device")
    if out.dim() != 2:
        raise ValueError("out: expected [rows][out]")
    rows = out.shape[0]
    n, k = w.shape
    batch, cu_ptr = _packed(cu, dev)
    if (n | k | batch | text_len) >> 31:
        raise HiloError("hilo_linear_i8", 2)
    if act >> 31:
        raise HiloError("hilo_linear_i8", 4)
    _launch("hilo_linear_i8", dev, stream, dtype, w,
            _arg(x, out.dtype if x_scale is None else torch.int8, (rows, k), dev, "x"),
            _arg(x_scale, torch.float32, (rows,), dev, "x_scale"), _arg(out, out.dtype, (rows, n), dev, "out"), rows, k, n,
            act, batch, text_len, cu_ptr, workspace.data_ptr(), workspace.numel() * workspace.element_size())


# ---------------------------------------------------------- products of a feed-forward, gradients, FP8 blocks

def _workspace(workspace, dev: int):
    """Pointer and bytes of a workspace, or of none."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous, on the tensors' device")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _gated_pointers(struct, ds: Sequence[dict], dtype):
    """Two of `struct` from dicts of tensors (one dict: for both streams): weights of one shape [out][in], biases [out] of one
    type; dtype the weights' type, or None: float32 or bfloat16, that of the biases too.  Any may be missing."""
    ds = [dict(d) for d in ds]  # kept below, whatever the caller does with theirs
    if not 1 <= len(ds) <= 2:
        raise ValueError("of one or two streams")
    arr = (struct * 2)()
    arr.kept, arr.shape, arr.dtype, arr.dev, arr.gated = ds, None, dtype, None, False
    biases = []
    for d in ds:
        for name in ("w", "w_gate"):
            w = d.get(name)
            if w is None:
                continue
            if arr.shape is None:
                arr.shape, arr.dev = w.shape, _on_device(w)
                if len(arr.shape) != 2:
                    raise ValueError("w: expected [out][in]")
                if dtype is None:
                    _float_code(w)
                    arr.dtype = w.dtype
            arr.gated = arr.gated or name == "w_gate"
        biases += [(name, d[name]) for name in ("b", "b_gate") if d.get(name) is not None]
    arr.bias = None
    for name, b in biases:
        _float_code(b)
        if arr.dev is None:
            arr.dev = _on_device(b)
        if arr.bias not in (None, b.dtype) or (dtype is None and arr.dtype not in (None, b.dtype)):
            raise ValueError(f"{name}: of one type")
        arr.bias = b.dtype
        arr.gated = arr.gated or name == "b_gate"
    arr.out = arr.shape[0] if arr.shape is not None else biases[0][1].numel() if biases else None
    for k in range(2):
        d = ds[min(k, len(ds) - 1)]
        for name in [f[0] for f in struct._fields_]:
            t = d.get(name)
            if t is None:
                continue
            if name[0] == "w":
                ptr = _arg(t, arr.dtype, arr.shape, arr.dev, name)
            elif name[0] == "s":
                ptr = _arg(t, torch.uint8, (-(-arr.shape[0] // 128), scale_stride(arr.shape[1])), arr.dev, name)
            else:
                ptr = _arg(t, arr.bias, (arr.out,), arr.dev, name)
            setattr(arr[k], name, ptr)
    return arr


def linear_weights(ws: Sequence[dict]):
    """Weights of hilo_linear: {"w": [out][in], "b": [out] or None, "w_gate", "b_gate": the gate's, or missing} of the image
    and the text stream (one dict: of both), all float32 or all bfloat16.  Keeps the tensors alive."""
    ws = list(ws)
    if any(d.get("w") is None for d in ws):
        raise ValueError("w: missing")
    return _gated_pointers(hilo_linear_w, ws, None)


def linear_grads(ds: Sequence[dict]):
    """Where hilo_linear_backward leaves the gradients: dicts as in linear_weights, any tensor None (one dict: sums over
    both streams)."""
    return _gated_pointers(hilo_linear_grads, ds, None)


def _product_rows(fn: str, w, rows_of: torch.Tensor, cols: int, cu: torch.Tensor, text_len: int, act: int):
    dev = _on_device(rows_of)
    if dev != w.dev:
        raise ValueError(f"weights on device {w.dev}, rows on device {dev}")
    if rows_of.dim() != 2 or rows_of.shape[1] != cols:
        raise ValueError(f"expected [rows][{cols}], not {tuple(rows_of.shape)}")
    n, k = w.shape
    batch, cu_ptr = _packed(cu, dev)
    if (n | k | batch | text_len) >> 31:
        raise HiloError(fn, 2)
    if act >> 31:
        raise HiloError(fn, 4)
    return dev, rows_of.shape[0], n, k, batch, cu_ptr


def hilo_linear_workspace_bytes(dtype: torch.dtype, rows: int, in_dim: int, out_dim: int, batch: int, gated: bool = False) -> int:
    return 0 if (in_dim | out_dim | batch) >> 31 else lib().hilo_linear_workspace_bytes(
        _FLOATS.get(dtype, -1), rows, in_dim, out_dim, batch, 1 if gated else 0)


def hilo_linear(w, x, out, cu, text_len: int = 0, *, act: int = ACT_NONE, pre=None, workspace=None, stream=None):
    """out [rows][out] = x w^T + b of linear_weights w, or act(x w_gate^T + b_gate) (x w^T + b); pre [rows][2][out]: g and u
    for the backward pass."""
    dev, rows, n, k, batch, cu_ptr = _product_rows("hilo_linear", w, out, w.shape[0], cu, text_len, act)
    dt = w.dtype
    ws, nbytes = _workspace(workspace, dev)
    _launch("hilo_linear", dev, stream, _FLOATS[dt], w, _arg(x, dt, (rows, k), dev, "x"), _arg(out, dt, (rows, n), dev, "out"),
            _arg(pre, dt, (rows, 2, n), dev, "pre"), rows, k, n, act, batch, text_len, cu_ptr, ws, nbytes)


def hilo_linear_backward_workspace_bytes(dtype: torch.dtype, rows: int, in_dim: int, out_dim: int, batch: int,
                                         gated: bool = False) -> int:
    return 0 if (in_dim | out_dim | batch) >> 31 else lib().hilo_linear_backward_workspace_bytes(
        _FLOATS.get(dtype, -1), rows, in_dim, out_dim, batch, 1 if gated else 0)


def hilo_linear_backward(w, x, pre, dout, dx, grads, cu, text_len: int = 0, *, act: int = ACT_NONE, workspace=None,
                         stream=None):
    """Gradients of hilo_linear from dout: dx (or None), and those in linear_grads grads (or None)."""
    dev, rows, n, k, batch, cu_ptr = _product_rows("hilo_linear_backward", w, dout, w.shape[0], cu, text_len, act)
    dt = w.dtype
    if grads is not None:
        if grads.dev not in (None, dev):
            raise ValueError(f"gradients on device {grads.dev}, rows on device {dev}")
        if grads.shape not in (None, w.shape) or grads.out not in (None, n):
            raise ValueError(f"gradients: expected the shapes of w {tuple(w.shape)}")
        if grads.dtype not in (None, dt) or grads.bias not in (None, dt):
            raise ValueError(f"gradients: expected {dt}")
    ws, nbytes = _workspace(workspace, dev)
    _launch("hilo_linear_backward", dev, stream, _FLOATS[dt], w, _arg(x, dt, (rows, k), dev, "x"),
            _arg(pre, dt, (rows, 2, n), dev, "pre"), _arg(dout, dt, (rows, n), dev, "dout"), _arg(dx, dt, (rows, k), dev, "dx"),
            grads, rows, k, n, act, batch, text_len, cu_ptr, ws, nbytes)


def scale_stride(cols: int) -> int:
    """Bytes in a row of E8M0 scales: one for each 128 columns, in whole groups of four."""
    return 4 * -(-cols // 512)


def hilo_quantize_blocks(x, codes, scales, block_rows: int = 1, cu=None, stream=None):
    """E4M3 codes (uint8 [rows][cols]) of x and E8M0 scales (uint8 [rows / block_rows][scale_stride(cols)]), one for each
    block of block_rows (1 or 128) rows and 128 columns; cu: the boundaries, whose last one bounds the rows."""
    dev, dtype = _on_device(x), _float_code(x)
    if x.dim() != 2:
        raise ValueError("x: expected [rows][cols]")
    if block_rows not in (1, 128):
        raise HiloError("hilo_quantize_blocks", 4)
    end = None
    if cu is not None:
        b, end = _packed(cu, dev)
        end += 4 * b
    rows, cols = x.shape
    _launch("hilo_quantize_blocks", dev, stream, dtype, _arg(x, x.dtype, x.shape, dev, "x"), rows, cols, block_rows, end,
            _arg(codes, torch.uint8, x.shape, dev, "codes"),
            _arg(scales, torch.uint8, (-(-rows // block_rows), scale_stride(cols)), dev, "scales"))


def quantize_block_weights(w, b=None, w_gate=None, b_gate=None, stream=None) -> dict:
    """A product's weights for linear_weights_fp8: codes and scales of w [out][in] and w_gate, the biases kept."""
    d = {"b": b, "b_gate": b_gate}
    for name, sname, t in (("w", "s", w), ("w_gate", "s_gate", w_gate)):
        if t is None:
            continue
        d[name] = torch.empty(t.shape, dtype=torch.uint8, device=t.device)
        d[sname] = torch.empty(-(-t.shape[0] // 128), scale_stride(t.shape[1]), dtype=torch.uint8, device=t.device)
        hilo_quantize_blocks(t, d[name], d[sname], 128, stream=stream)
    return d


def linear_weights_fp8(ws: Sequence[dict]):
    """Weights of hilo_linear_fp8: {"w": uint8 [out][in], "s": uint8 [out / 128][scale_stride(in)], "b": [out] or None, and
    "w_gate", "s_gate", "b_gate" with a gate} of the image and the text stream (one dict: of both).  Keeps the tensors alive."""
    ws = list(ws)
    for d in ws:
        if d.get("w") is None or d.get("s") is None or (d.get("w_gate") is None) != (d.get("s_gate") is None):
            raise ValueError("weights and scales go together")
    return _gated_pointers(hilo_linear_w_fp8, ws, torch.uint8)


def hilo_linear_fp8_workspace_bytes(rows: int, in_dim: int, out_dim: int, gated: bool = False) -> int:
    return 0 if (in_dim | out_dim) >> 31 else lib().hilo_linear_fp8_workspace_bytes(rows, in_dim, out_dim, 1 if gated else 0)


def hilo_linear_fp8(w, x, out, cu, text_len: int = 0, *, x_scale=None, out_scale=None, act: int = ACT_NONE, workspace=None,
                    stream=None):
    """hilo_linear on E4M3 codes with block scales: x uint8 codes with x_scale [rows][scale_stride(in)], or float rows,
    quantised here; out of a float type, or with out_scale [rows][scale_stride(out)] uint8 codes (a gate only).  Float tensors
    and biases are of one type; where there is none, sums and activations are rounded only to codes."""
    dev, rows, n, k, batch, cu_ptr = _product_rows("hilo_linear_fp8", w, out, w.shape[0], cu, text_len, act)
    u8, floats = torch.uint8, []
    if out_scale is None:
        floats.append(("out", out.dtype))
    if x_scale is None:
        floats.append(("x", x.dtype))
    if w.bias is not None:
        floats.append(("b", w.bias))
    dt = floats[0][1] if floats else torch.float32
    for name, t in floats:
        if t is not dt:
            raise ValueError(f"{name}: {t}, other tensors {dt}")
    if dt not in _FLOATS:
        raise ValueError(f"float32 or bfloat16 expected, not {dt}")
    ws, nbytes = _workspace(workspace, dev)
    _launch("hilo_linear_fp8", dev, stream, _FLOATS[dt], w, _arg(x, dt if x_scale is None else u8, (rows, k), dev, "x"),
            _arg(x_scale, u8, (rows, scale_stride(k)), dev, "x_scale"), _arg(out, dt if out_scale is None else u8, (rows, n), dev, "out"),
            _arg(out_scale, u8, (rows, scale_stride(n)), dev, "out_scale"), rows, k, n, act, batch, text_len, cu_ptr, ws, nbytes)


def hilo_profile_enable(on: bool):
    _check("hilo_profile_enable", lib().hilo_profile_enable(1 if on else 0))


def hilo_profile_read(kind: int):
    ms = ctypes.c_double()
    n = ctypes.c_int64()
    _check("hilo_profile_read", lib().hilo_profile_read(int(kind), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def hilo_profile_kinds() -> int:
    return lib().hilo_profile_kinds()


def hilo_profile_name(kind: int) -> str:
    return lib().hilo_profile_name(int(kind)).decode()
