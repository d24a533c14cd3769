"""Python binding over libicarus.so: argument marshalling only.

Every step of the layer runs in the library's gfx950 kernels; torch is used for device
memory and streams.  Function names mirror the C ABI (include/icarus.h).  If the library
is missing this module raises at import time: there is no CPU or eager fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from dataclasses import dataclass

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libicarus.so")

PROJ = ("q", "k", "v", "o", "gate", "up", "down")
NPROJ = 7
F32, BF16 = 0, 1

STATUS = {0: "OK", 1: "INVALID_ARG", 2: "SHAPE", 3: "ALIGNMENT", 4: "MODEL_ID", 5: "ROW_ORDER",
          6: "CAPACITY", 7: "UNSUPPORTED", 8: "HIP"}

EXPORTS = ("icarus_create", "icarus_destroy", "icarus_last_error", "icarus_workspace_bytes",
           "icarus_validate_decode", "icarus_prefill_kv", "icarus_decode_step", "icarus_attn_shared_kv",
           "icarus_set_kernel_mode", "icarus_timing_enable", "icarus_timing_read", "icarus_bench_copy", "icarus_bench_mfma", "icarus_stack_create", "icarus_stack_destroy",
           "icarus_stack_last_error", "icarus_stack_workspace_bytes", "icarus_stack_prefill", "icarus_stack_decode",
           "icarus_cache_create", "icarus_cache_destroy", "icarus_cache_last_error", "icarus_cache_acquire", "icarus_cache_extend",
           "icarus_cache_commit", "icarus_cache_release", "icarus_cache_get_stats", "icarus_set_full_decoders",
           "icarus_validate_block_tables", "icarus_set_attn_piece_limit", "icarus_attn_shared_kv_static", "icarus_bench_read",
           "icarus_gemm_tile_order", "icarus_gemm_choice", "icarus_gemm_group_tile", "icarus_append_in_tiles", "icarus_prefill_plan", "icarus_row_order", "icarus_gemm",
           "icarus_beam_workspace_bytes", "icarus_beam_select", "icarus_fork_workspace_bytes", "icarus_fork_sequences", "icarus_copy_blocks",
           "icarus_attn_prefix_workspace_bytes", "icarus_attn_prefix",
           "icarus_extend_sequences", "icarus_rope_append", "icarus_key_bounds", "icarus_select_workspace_bytes", "icarus_select_blocks",
           "icarus_attn_blocks_workspace_bytes", "icarus_attn_blocks")

PHASES = ("norm", "lora", "gemm_qkv", "rope_append", "attn", "attn_merge", "gemm_o", "gemm_gateup", "gemm_down",
          "elementwise")


class IcarusError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"icarus status {status} ({STATUS.get(status, '?')}): {message}")
        self.status = status
        self.status_name = STATUS.get(status, "?")


class _Cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "block_size", "num_blocks", "n_models",
        "lora_rank", "lora_target_mask", "dtype", "qk_norm", "max_position", "kv_dtype")] + [
        ("rope_theta", C.c_double), ("rms_eps", C.c_double), ("lora_scale", C.c_double),
        ("k_scale", C.c_double), ("v_scale", C.c_double)]


class _Base(C.Structure):
    _fields_ = [("w", C.c_void_p * NPROJ), ("norm_attn", C.c_void_p), ("norm_ffn", C.c_void_p),
                ("q_norm", C.c_void_p), ("k_norm", C.c_void_p)]


class _Lora(C.Structure):
    _fields_ = [("A", C.c_void_p * NPROJ), ("B", C.c_void_p * NPROJ)]


class _Full(C.Structure):
    _fields_ = [("w", C.c_void_p * NPROJ)]


class _StackCfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("vocab", C.c_int32), ("layers", C.POINTER(C.c_void_p)),
                ("embed", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)]


class _CacheCfg(C.Structure):
    _fields_ = [("num_blocks", C.c_int32), ("block_size", C.c_int32), ("key_by_model", C.c_int32)]


class _CacheStats(C.Structure):
    _fields_ = [("lookups", C.c_int64), ("hit_tokens", C.c_int64), ("miss_tokens", C.c_int64), ("evictions", C.c_int64),
                ("live", C.c_int32), ("cached", C.c_int32), ("free_blocks", C.c_int32), ("peak_live", C.c_int32)]


class _Gemm(C.Structure):
    _fields_ = [("x", C.c_void_p), ("w", C.c_void_p * 3), ("t", C.c_void_p), ("b", C.c_void_p * 2), ("resid", C.c_void_p),
                ("y", C.c_void_p), ("partials", C.c_void_p), ("rows", C.c_int32), ("k", C.c_int32), ("n", C.c_int32 * 3),
                ("n_segs", C.c_int32), ("fused", C.c_int32), ("models", C.c_int32), ("rank", C.c_int32),
                ("tile_rows", C.c_int32), ("tile_cols", C.c_int32), ("staged", C.c_int32), ("slices", C.c_int32)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2603_13281_amd.build` "
                          "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    lib.icarus_create.restype = C.c_int
    lib.icarus_create.argtypes = [C.POINTER(_Cfg), C.POINTER(_Base), C.POINTER(_Lora), C.POINTER(vp)]
    lib.icarus_destroy.restype = None
    lib.icarus_destroy.argtypes = [vp]
    lib.icarus_last_error.restype = C.c_char_p
    lib.icarus_last_error.argtypes = [vp]
    lib.icarus_workspace_bytes.restype = sz
    lib.icarus_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.icarus_validate_decode.restype = C.c_int
    lib.icarus_validate_decode.argtypes = [vp, i32, i32, vp, i32, vp, vp]
    lib.icarus_prefill_kv.restype = C.c_int
    lib.icarus_prefill_kv.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.icarus_decode_step.restype = C.c_int
    lib.icarus_decode_step.argtypes = [vp, vp, vp, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.icarus_attn_shared_kv.restype = C.c_int
    lib.icarus_attn_shared_kv.argtypes = [vp, vp, vp, vp, i32, i32, vp, i32, vp, vp, vp, sz, vp]
    lib.icarus_attn_shared_kv_static.restype = C.c_int
    lib.icarus_attn_shared_kv_static.argtypes = [vp, vp, vp, vp, i32, i32, vp, i32, vp, vp, vp]
    lib.icarus_validate_block_tables.restype = C.c_int
    lib.icarus_validate_block_tables.argtypes = [vp, vp, i32, i32, vp, vp]
    lib.icarus_set_attn_piece_limit.restype = C.c_int
    lib.icarus_set_attn_piece_limit.argtypes = [vp, i32]
    lib.icarus_set_kernel_mode.restype = C.c_int
    lib.icarus_set_kernel_mode.argtypes = [vp, i32]
    lib.icarus_timing_enable.restype = C.c_int
    lib.icarus_timing_enable.argtypes = [vp, i32]
    lib.icarus_timing_read.restype = C.c_int
    lib.icarus_timing_read.argtypes = [vp, vp, vp]
    lib.icarus_bench_copy.restype = C.c_int
    lib.icarus_bench_copy.argtypes = [vp, vp, sz, vp]
    lib.icarus_bench_read.restype = C.c_int
    lib.icarus_bench_read.argtypes = [vp, sz, vp, vp]
    lib.icarus_bench_mfma.restype = C.c_int
    lib.icarus_bench_mfma.argtypes = [vp, C.c_int32, C.c_int32, vp]
    lib.icarus_row_order.restype = C.c_int
    lib.icarus_row_order.argtypes = [vp, i32, vp, vp]
    lib.icarus_gemm_tile_order.restype = C.c_int
    lib.icarus_gemm_tile_order.argtypes = [i32] * 6 + [vp, i32, vp]
    lib.icarus_gemm_choice.restype = C.c_int
    lib.icarus_gemm_choice.argtypes = [i32, i32, vp, i32, i32, i32, i32, i32, vp]
    lib.icarus_gemm_group_tile.restype = C.c_int
    lib.icarus_gemm_group_tile.argtypes = [vp, i32, vp]
    lib.icarus_append_in_tiles.restype = i32
    lib.icarus_append_in_tiles.argtypes = [vp, i32, i32]
    lib.icarus_prefill_plan.restype = C.c_int
    lib.icarus_prefill_plan.argtypes = [vp, i32, vp, vp, vp, i32, vp]
    lib.icarus_gemm.restype = C.c_int
    lib.icarus_gemm.argtypes = [C.POINTER(_Gemm), vp]
    lib.icarus_stack_create.restype = C.c_int
    lib.icarus_stack_create.argtypes = [C.POINTER(_StackCfg), C.POINTER(vp)]
    lib.icarus_stack_destroy.restype = None
    lib.icarus_stack_destroy.argtypes = [vp]
    lib.icarus_stack_last_error.restype = C.c_char_p
    lib.icarus_stack_last_error.argtypes = [vp]
    lib.icarus_stack_workspace_bytes.restype = sz
    lib.icarus_stack_workspace_bytes.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
    lib.icarus_stack_prefill.restype = C.c_int
    lib.icarus_stack_prefill.argtypes = [vp, C.POINTER(vp), vp, C.c_int32, C.c_int32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.icarus_stack_decode.restype = C.c_int
    lib.icarus_stack_decode.argtypes = [vp, C.POINTER(vp), vp, C.c_int32, C.c_int32, vp, C.c_int32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    i32, pi32 = C.c_int32, C.POINTER(C.c_int32)
    lib.icarus_cache_create.restype = C.c_int
    lib.icarus_cache_create.argtypes = [C.POINTER(_CacheCfg), C.POINTER(vp)]
    lib.icarus_cache_destroy.restype = None
    lib.icarus_cache_destroy.argtypes = [vp]
    lib.icarus_cache_last_error.restype = C.c_char_p
    lib.icarus_cache_last_error.argtypes = [vp]
    lib.icarus_cache_acquire.restype = C.c_int
    lib.icarus_cache_acquire.argtypes = [vp, vp, i32, i32, i32, vp, i32, pi32, pi32]
    lib.icarus_cache_extend.restype = C.c_int
    lib.icarus_cache_extend.argtypes = [vp, vp, i32, pi32, i32]
    lib.icarus_cache_commit.restype = C.c_int
    lib.icarus_cache_commit.argtypes = [vp, vp, i32, i32, vp, i32]
    lib.icarus_cache_release.restype = C.c_int
    lib.icarus_cache_release.argtypes = [vp, vp, i32]
    lib.icarus_set_full_decoders.restype = C.c_int
    lib.icarus_set_full_decoders.argtypes = [vp, C.POINTER(_Full)]
    i64 = C.c_int64
    lib.icarus_extend_sequences.restype = C.c_int
    lib.icarus_extend_sequences.argtypes = [vp, i32, vp, vp, vp, vp, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.icarus_rope_append.restype = C.c_int
    lib.icarus_rope_append.argtypes = [vp, vp, i64, i32, vp, vp, vp, vp, vp]
    lib.icarus_key_bounds.restype = C.c_int
    lib.icarus_key_bounds.argtypes = [vp, vp, vp, i32, i32, vp, vp, i32, vp, vp, vp]
    lib.icarus_select_workspace_bytes.restype = sz
    lib.icarus_select_workspace_bytes.argtypes = [vp, i32, i32]
    lib.icarus_select_blocks.restype = C.c_int
    lib.icarus_select_blocks.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, i32, vp, i32, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.icarus_attn_blocks_workspace_bytes.restype = sz
    lib.icarus_attn_blocks_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.icarus_attn_blocks.restype = C.c_int
    lib.icarus_attn_blocks.argtypes = [vp, vp, vp, vp, i32, i32, vp, i32, vp, i32, vp, vp, i32, vp, vp, sz, vp]
    lib.icarus_beam_workspace_bytes.restype = sz
    lib.icarus_beam_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.icarus_beam_select.restype = C.c_int
    lib.icarus_beam_select.argtypes = [vp, vp, i32, i32, i64, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.icarus_fork_workspace_bytes.restype = sz
    lib.icarus_fork_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.icarus_fork_sequences.restype = C.c_int
    lib.icarus_fork_sequences.argtypes = [vp, i32, i32, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.icarus_copy_blocks.restype = C.c_int
    lib.icarus_copy_blocks.argtypes = [vp, vp, vp, i32, vp, vp, i32, vp]
    lib.icarus_attn_prefix_workspace_bytes.restype = sz
    lib.icarus_attn_prefix_workspace_bytes.argtypes = [vp, i32, i32, i32, i32]
    lib.icarus_attn_prefix.restype = C.c_int
    lib.icarus_attn_prefix.argtypes = [vp, vp, vp, vp, i32, i32, vp, i32, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.icarus_cache_get_stats.restype = C.c_int
    lib.icarus_cache_get_stats.argtypes = [vp, C.POINTER(_CacheStats)]
    return lib


_lib = _load()


def lib():
    return _lib


@dataclass
class LayerConfig:
    d_model: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    d_ffn: int
    block_size: int
    num_blocks: int
    n_models: int = 0
    lora_rank: int = 0
    lora_target_mask: int = 0
    bf16: bool = True
    qk_norm: bool = False
    max_position: int = 1 << 17
    rope_theta: float = 5e5
    rms_eps: float = 1e-5
    lora_scale: float = 2.0
    kv_fp8: bool = False      # the KV pool holds FP8 E4M3 codes: value = code * k_scale (K) or v_scale (V)
    k_scale: float = 1.0
    v_scale: float = 1.0

    def _c(self) -> _Cfg:
        return _Cfg(self.d_model, self.n_q_heads, self.n_kv_heads, self.head_dim, self.d_ffn, self.block_size,
                    self.num_blocks, self.n_models, self.lora_rank, self.lora_target_mask,
                    BF16 if self.bf16 else F32, int(self.qk_norm), self.max_position, 1 if self.kv_fp8 else 0,
                    float(self.rope_theta), float(self.rms_eps), float(self.lora_scale), float(self.k_scale), float(self.v_scale))

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.bf16 else torch.float32

    @property
    def pool_dtype(self):
        """Element type of the KV pool tensor (FP8 codes are handed over as raw bytes)."""
        return torch.uint8 if self.kv_fp8 else self.torch_dtype

    def pool_shape(self):
        """[num_blocks, n_kv_heads, 2, block_size*head_dim]: plane 0 = K [Bk, D], plane 1 = V^T [D, Bk]."""
        return (self.num_blocks, self.n_kv_heads, 2, self.block_size * self.head_dim)


def _ptr(t) -> C.c_void_p:
    if t is None:
        return C.c_void_p(0)
    if isinstance(t, torch.Tensor):
        assert t.is_contiguous(), "tensors passed to the library must be contiguous"
        return C.c_void_p(t.data_ptr())
    if isinstance(t, np.ndarray):
        return C.c_void_p(t.ctypes.data)
    if isinstance(t, int):
        return C.c_void_p(t)
    raise TypeError(type(t))


def _host_i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _want(t, what: str, dtype, shape=None, device=None):
    """Marshalling guard: a device tensor handed to the library must have the element type, the shape and the
    device the C signature assumes (a numpy-default int64 block table would be read as pairs of int32)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{what}: dtype {t.dtype}, the library reads {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{what}: on {t.device}, expected {device}")
    if not t.is_cuda:
        raise ValueError(f"{what}: must be a device tensor")


def bench_copy(src: torch.Tensor, dst: torch.Tensor):
    """dst <- src by the library's plain copy kernel (profiler counter calibration)."""
    n = src.numel() * src.element_size()
    rc = _lib.icarus_bench_copy(_ptr(src), _ptr(dst), n, C.c_void_p(torch.cuda.current_stream(src.device).cuda_stream))
    if rc != 0:
        raise IcarusError(rc, "icarus_bench_copy failed")


def bench_read(src: torch.Tensor, reps: int = 5) -> float:
    """Seconds per pass of the library's streaming-read kernel over `src` (whole 8 KB chunks), best of `reps`."""
    n = src.numel() * src.element_size() // 8192 * 8192
    out = torch.zeros(1, dtype=torch.int32, device=src.device)
    stream = C.c_void_p(torch.cuda.current_stream(src.device).cuda_stream)
    best = None
    for _ in range(reps + 1):
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        ev[0].record()
        rc = _lib.icarus_bench_read(_ptr(src), n, _ptr(out), stream)
        ev[1].record()
        if rc != 0:
            raise IcarusError(rc, "icarus_bench_read failed")
        torch.cuda.synchronize()
        t = ev[0].elapsed_time(ev[1]) * 1e-3
        best = t if best is None else min(best, t)
    return best


def bench_mfma(waves: int, iters: int, device="cuda:0") -> float:
    """Seconds of the library's register-resident bf16 MFMA loop (flops: 2*32*32*16*8*iters*waves)."""
    out = torch.empty(waves * 64, dtype=torch.float32, device=device)
    stream = C.c_void_p(torch.cuda.current_stream(out.device).cuda_stream)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    if _lib.icarus_bench_mfma(_ptr(out), waves, max(1, iters // 16), stream) != 0:      # warm-up
        raise IcarusError(8, "icarus_bench_mfma failed")
    ev[0].record()
    rc = _lib.icarus_bench_mfma(_ptr(out), waves, iters, stream)
    ev[1].record()
    if rc != 0:
        raise IcarusError(rc, "icarus_bench_mfma failed")
    torch.cuda.synchronize()
    return ev[0].elapsed_time(ev[1]) * 1e-3


def gemm_tile_order(row_tiles: int, col_tiles: int, k_slices: int, tile_rows: int, tile_cols: int, per_cu: int = 1) -> np.ndarray:
    """[workgroups, 4]: XCD, row tile, column tile and K slice of a GEMM's workgroups in launch order (host only)."""
    cap = row_tiles * col_tiles * k_slices + 64
    out, n = np.zeros((cap, 4), dtype=np.int32), C.c_int32()
    rc = _lib.icarus_gemm_tile_order(row_tiles, col_tiles, k_slices, tile_rows, tile_cols, per_cu, out.ctypes.data, cap, C.byref(n))
    if rc != 0:
        raise IcarusError(rc, "icarus_gemm_tile_order failed")
    return out[:min(cap, n.value)]


def row_order(row_model) -> np.ndarray:
    """Entries row | (model + 1) << 16 (-1: none) in which a decode call's row kernels take its rows; empty: as they come (host only)."""
    model = np.ascontiguousarray(row_model, dtype=np.int32)
    out, n = np.zeros(len(model) + 16, dtype=np.int32), C.c_int32()
    rc = _lib.icarus_row_order(model.ctypes.data, len(model), out.ctypes.data, C.byref(n))
    if rc != 0:
        raise IcarusError(rc, "icarus_row_order failed")
    return out[:n.value]


def gemm_choice(rows: int, k: int, n, fused: bool = False, adapter_cols: int = 0, max_slices: int = 12, taken: bool = False):
    """(tile rows, tile columns, mark of 192 and 160 rows by 256, K slices) of a GEMM's launch (host only); n: outputs per segment."""
    seg = np.ascontiguousarray(np.atleast_1d(n), dtype=np.int32)
    out = np.zeros(4, dtype=np.int32)
    rc = _lib.icarus_gemm_choice(rows, k, seg.ctypes.data, len(seg), int(fused), adapter_cols, max_slices, int(taken), out.ctypes.data)
    if rc != 0:
        raise IcarusError(rc, "icarus_gemm_choice failed")
    return int(out[0]), int(out[1]), bool(out[2]), int(out[3])


def gemm_group_tile(group_rows):
    """(rows, columns) of the tile the grouped GEMMs take for groups of these row counts (host only)."""
    n = np.ascontiguousarray(group_rows, dtype=np.int32)
    out = np.zeros(2, dtype=np.int32)
    rc = _lib.icarus_gemm_group_tile(n.ctypes.data, len(n), out.ctypes.data)
    if rc != 0:
        raise IcarusError(rc, "icarus_gemm_group_tile failed")
    return int(out[0]), int(out[1])


def gemm(x, w, tile, slices: int = 1, fused: bool = False, t=None, b=None, resid=None) -> torch.Tensor:
    """One GEMM in a given launch: x [rows, k], w a list of [n, k] (fused: gate, up), t [rows, models * rank (x 2 fused)], b a list of
    [models, n, rank], resid [rows, n]; tile as gemm_choice returns it.  Float [rows, sum n], or bf16 with resid or fused."""
    rows, k = x.shape
    _want(x, "x", torch.bfloat16, (rows, k))
    n = [int(v.shape[0]) for v in w]
    for v in w:
        _want(v, "w", torch.bfloat16, (v.shape[0], k), x.device)
    a = _Gemm(rows=rows, k=k, n_segs=1 if fused else len(w), fused=int(fused), tile_rows=tile[0], tile_cols=tile[1], staged=int(tile[2]), slices=slices)
    if len(w) > 3 or (fused and (len(w) != 2 or n[0] != n[1])):
        raise ValueError("w: up to three matrices, or gate and up of one shape")
    for i, v in enumerate(w):
        a.w[i], a.n[i] = v.data_ptr(), n[i]
    cols = n[0] if fused else sum(n)
    if t is not None:
        models, _, rank = b[0].shape
        _want(t, "t", torch.bfloat16, (rows, models * rank * (2 if fused else 1)), x.device)
        for i, v in enumerate(b):
            _want(v, "b", torch.bfloat16, (models, n[0], rank), x.device)
            a.b[i] = v.data_ptr()
        a.t, a.models, a.rank = t.data_ptr(), models, rank
    if resid is not None:
        _want(resid, "resid", torch.bfloat16, (rows, cols), x.device)
        a.resid = resid.data_ptr()
    y = torch.empty(rows, cols, dtype=torch.bfloat16 if fused or resid is not None else torch.float32, device=x.device)
    part = torch.empty(slices if slices > 1 else 0, rows, cols, dtype=torch.float32, device=x.device)
    a.x, a.y, a.partials = x.data_ptr(), y.data_ptr(), part.data_ptr() if slices > 1 else None
    rc = _lib.icarus_gemm(C.byref(a), C.c_void_p(torch.cuda.current_stream(x.device).cuda_stream))
    if rc != 0:
        raise IcarusError(rc, "icarus_gemm failed")
    return y


class SequenceMap:
    """Device arrays that IcarusLayer.extend_sequences fills, kept by the caller (a captured graph replays into the same ones): kv_lens [S],
    row_start [S + 1], row_seq, row_pos, row_slot [max_rows], counts [2] (free ids taken, sequences refused); one allocation of each type."""

    def __init__(self, n_seqs: int, max_rows: int, device):
        S, R = int(n_seqs), int(max_rows)
        self.n_seqs, self.max_rows = S, R
        self.row_slot = torch.empty(R, dtype=torch.int64, device=device)
        ints = torch.empty(2 * S + 3 + 2 * R, dtype=torch.int32, device=device)
        self.kv_lens, self.row_start, self.counts, self.row_seq, self.row_pos = ints.split([S, S + 1, 2, R, R])


class BeamMap:
    """Device arrays that IcarusLayer.beam_select fills, kept by the caller: parents, tokens, done (int32) and scores (float32) of groups * width beams."""

    def __init__(self, groups: int, width: int, device):
        self.groups, self.width = int(groups), int(width)
        S = self.groups * self.width
        self.parents, self.tokens, self.done = torch.empty(3 * S, dtype=torch.int32, device=device).split(S) if S else [torch.empty(0, dtype=torch.int32, device=device)] * 3
        self.scores = torch.empty(S, dtype=torch.float32, device=device)


class ForkMap:
    """Device arrays that IcarusLayer.fork_sequences fills, kept by the caller: kv_lens [S], block_tables [S, max_blocks], copy_src and copy_dst [S] for copy_blocks,
    counts [3] (free ids taken, children refused, blocks freed); S = groups * width.  A step reads one and fills another, so a loop keeps two."""

    def __init__(self, groups: int, width: int, max_blocks: int, device):
        self.groups, self.width, self.max_blocks = int(groups), int(width), int(max_blocks)
        S = self.groups * self.width
        ints = torch.empty(3 * S + 3, dtype=torch.int32, device=device)
        self.kv_lens, self.copy_src, self.copy_dst, self.counts = ints.split([S, S, S, 3])
        self.block_tables = torch.zeros(S, self.max_blocks, dtype=torch.int32, device=device)


# The calls with lengths on the device take a few microseconds on the GPU, so their marshalling is kept short: one look at a tensor in the common case,
# _want's message where something is wrong.
def _need(t, what: str, dtype, shape, index: int):
    """A contiguous tensor of this type and shape on CUDA device `index`."""
    if not (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous()):
        _want(t, what, dtype, shape, torch.device("cuda", index))


def _index_of(t, what: str, dtype) -> int:
    """CUDA device of a tensor of this type."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype is not dtype:
        raise TypeError(f"{what}: dtype {t.dtype}, the library reads {dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what}: must be a device tensor")
    return t.get_device()


def _launch(index: int, call, *args) -> int:
    """call(*args, stream) on the current stream of CUDA device `index`, which is made the current device meanwhile."""
    before = torch._C._cuda_getDevice()
    if before == index:
        return call(*args, torch._C._cuda_getCurrentRawStream(index))
    with torch.cuda.device(index):
        return call(*args, torch._C._cuda_getCurrentRawStream(index))


class IcarusLayer:
    """One layer context.  base / lora hold torch tensors (device, storage dtype) the caller owns;
    this object keeps references so that they outlive the context.

    base: dict "q","k","v","o","gate","up","down" -> [out,in]; "norm_attn","norm_ffn" -> [d];
          "q_norm","k_norm" -> [D] when qk_norm.
    lora: dict p -> (A [M,r,in_p], B [M,out_p,r]) or None.
    """

    def __init__(self, cfg: LayerConfig, base: dict, lora: dict | None = None):
        self.cfg = cfg
        self._refs = []
        cb = _Base()
        for i, p in enumerate(PROJ):
            cb.w[i] = self._keep(base[p])
        for name in ("norm_attn", "norm_ffn", "q_norm", "k_norm"):
            if base.get(name) is not None:
                setattr(cb, name, self._keep(base[name]))
        cl = _Lora()
        if lora:
            for i, p in enumerate(PROJ):
                if lora.get(p) is not None:
                    cl.A[i] = self._keep(lora[p][0])
                    cl.B[i] = self._keep(lora[p][1])
        cc = cfg._c()
        h = C.c_void_p()
        rc = _lib.icarus_create(C.byref(cc), C.byref(cb), C.byref(cl), C.byref(h))
        if rc != 0:
            raise IcarusError(rc, _lib.icarus_last_error(None).decode())
        self._h = h
        self._ws = None

    def _keep(self, t):
        if isinstance(t, torch.Tensor):
            assert t.is_contiguous()
            self._refs.append(t)
            return t.data_ptr()
        return int(t)  # raw address (host-only validation tests)

    def close(self):
        if getattr(self, "_h", None):
            _lib.icarus_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != 0:
            raise IcarusError(rc, _lib.icarus_last_error(self._h).decode())

    # -- C ABI mirrors ---------------------------------------------------------------
    def set_full_decoders(self, full: dict | None):
        """full: p -> device tensor [n_models, out_p, in_p] for p in q, o, gate, up, down (private weights of every
        decoder, instead of the adapters); None switches back to the adapters.  The tensors are kept alive here."""
        if full is None:
            self._check(_lib.icarus_set_full_decoders(self._h, None))
            self._full_keep = None
            return
        fw = _Full()
        for i, p in enumerate(PROJ):
            if p in full and full[p] is not None:
                fw.w[i] = full[p].data_ptr()
        self._check(_lib.icarus_set_full_decoders(self._h, C.byref(fw)))
        self._full_keep = dict(full)

    def set_kernel_mode(self, mode: int):
        self._check(_lib.icarus_set_kernel_mode(self._h, mode))

    def timing_enable(self, on: bool):
        self._check(_lib.icarus_timing_enable(self._h, int(on)))

    def timing_read(self) -> dict:
        """{phase: (milliseconds, launches)} accumulated since the last read."""
        ms = np.zeros(len(PHASES), dtype=np.float64)
        n = np.zeros(len(PHASES), dtype=np.int32)
        self._check(_lib.icarus_timing_read(self._h, _ptr(ms), _ptr(n)))
        return {p: (float(ms[i]), int(n[i])) for i, p in enumerate(PHASES)}

    def workspace_bytes(self, max_rows: int, max_seqs: int, max_ctx: int) -> int:
        return int(_lib.icarus_workspace_bytes(self._h, max_rows, max_seqs, max_ctx))

    def prefill_plan(self, ctx_lens, chunk_lens) -> np.ndarray:
        """[pieces, 5]: first row, rows, first token, tokens, partial slot (-1: none) of each piece of the prefill attention."""
        ctx, chunk = _host_i32(ctx_lens), _host_i32(chunk_lens)
        out, n = np.zeros((0, 5), dtype=np.int32), C.c_int32()
        for cap in (0, None):
            if cap is None:
                out = np.zeros((n.value, 5), dtype=np.int32)
            self._check(_lib.icarus_prefill_plan(self._h, len(ctx), ctx.ctypes.data, chunk.ctypes.data, out.ctypes.data, len(out), C.byref(n)))
        return out

    def append_in_tiles(self, rows: int, tiles: int) -> bool:
        return bool(_lib.icarus_append_in_tiles(self._h, rows, tiles))

    def set_attn_piece_limit(self, tokens: int):
        """Longest piece of the decode attention's plan, in tokens (0 = automatic); for tests and measurements."""
        self._check(_lib.icarus_set_attn_piece_limit(self._h, int(tokens)))
        self._ws = None

    def validate_block_tables(self, block_tables, ctx_lens, extra=None):
        """Host-side check of a HOST copy of the block tables ([S, max_blocks] int32)."""
        bt = np.ascontiguousarray(block_tables)
        if bt.dtype != np.int32 or bt.ndim != 2:
            raise TypeError(f"block_tables: need a 2-d int32 array, got {bt.dtype} with {bt.ndim} dims")
        ctx_lens = _host_i32(ctx_lens)
        if len(ctx_lens) != bt.shape[0]:
            raise ValueError(f"ctx_lens has {len(ctx_lens)} entries for {bt.shape[0]} table rows")
        ex = None if extra is None else _host_i32(extra)
        if ex is not None and len(ex) != bt.shape[0]:
            raise ValueError(f"extra has {len(ex)} entries for {bt.shape[0]} table rows")
        self._check(_lib.icarus_validate_block_tables(self._h, _ptr(bt), bt.shape[1], bt.shape[0], _ptr(ctx_lens), _ptr(ex)))

    def _check_call(self, kv_pool, block_tables, n_seq_meta, what_meta, x=None, x_cols=None, rows=None, outs=()):
        """Shapes, dtypes and devices of a call's tensors against what the C signature assumes."""
        dev = block_tables.device if isinstance(block_tables, torch.Tensor) else None
        _want(block_tables, "block_tables", torch.int32)
        if block_tables.dim() != 2:
            raise ValueError(f"block_tables: need [S, max_blocks], got {tuple(block_tables.shape)}")
        if block_tables.shape[0] != n_seq_meta:
            raise ValueError(f"{what_meta} has {n_seq_meta} entries for {block_tables.shape[0]} block-table rows")
        _want(kv_pool, "kv_pool", self.cfg.pool_dtype, None, dev)
        want = self.cfg.pool_shape()
        if kv_pool.dim() != 4 or tuple(kv_pool.shape[1:]) != want[1:] or kv_pool.shape[0] < want[0]:
            raise ValueError(f"kv_pool: shape {tuple(kv_pool.shape)}, expected at least {want[0]} blocks of {want[1:]}")
        if x is not None:
            _want(x, "input rows", self.cfg.torch_dtype, (rows, x_cols), dev)
        for name, t, dtype, shape in outs:
            if t is not None:
                _want(t, name, dtype, shape, dev)

    def validate_decode(self, max_blocks, ctx_lens, row_seq, row_model):
        ctx_lens, row_seq, row_model = _host_i32(ctx_lens), _host_i32(row_seq), _host_i32(row_model)
        self._check(_lib.icarus_validate_decode(self._h, max_blocks, len(ctx_lens), _ptr(ctx_lens), len(row_seq),
                                                _ptr(row_seq), _ptr(row_model)))

    def _workspace(self, rows, seqs, max_ctx, device):
        need = self.workspace_bytes(rows, seqs, max_ctx)
        if self._ws is None or self._ws.numel() < need or self._ws.device != device:
            self._ws = torch.empty(need, dtype=torch.uint8, device=device)
        return self._ws

    @staticmethod
    def _stream(device):
        return C.c_void_p(torch.cuda.current_stream(device).cuda_stream)

    def prefill_kv(self, kv_pool, block_tables, ctx_lens, chunk_lens, x_in, x_out=None, slot_out=None,
                   workspace=None, want_out=True):
        ctx_lens, chunk_lens = _host_i32(ctx_lens), _host_i32(chunk_lens)
        if len(ctx_lens) != len(chunk_lens):
            raise ValueError("ctx_lens and chunk_lens differ in length")
        total = int(chunk_lens.sum())
        self._check_call(kv_pool, block_tables, len(ctx_lens), "ctx_lens", x_in, self.cfg.d_model, total,
                         (("x_out", x_out if want_out else None, self.cfg.torch_dtype, (total, self.cfg.d_model)),
                          ("slot_out", slot_out, torch.int64, (total,))))
        S, max_blocks = block_tables.shape
        if want_out and x_out is None:
            x_out = torch.empty_like(x_in)
        if not want_out:
            x_out = None
        max_ctx = int((ctx_lens + chunk_lens).max()) if S else 0
        ws = workspace if workspace is not None else self._workspace(total, S, max_ctx, x_in.device)
        self._check(_lib.icarus_prefill_kv(self._h, _ptr(kv_pool), _ptr(block_tables), max_blocks, S, _ptr(ctx_lens),
                                           _ptr(chunk_lens), _ptr(x_in), _ptr(x_out), _ptr(slot_out), _ptr(ws),
                                           ws.numel(), self._stream(x_in.device)))
        return x_out

    def decode_step(self, kv_pool, block_tables, ctx_lens, row_seq, row_model, x_in, x_out=None, slot_out=None,
                    workspace=None):
        ctx_lens, row_seq, row_model = _host_i32(ctx_lens), _host_i32(row_seq), _host_i32(row_model)
        R = len(row_seq)
        if len(row_model) != R:
            raise ValueError("row_seq and row_model differ in length")
        self._check_call(kv_pool, block_tables, len(ctx_lens), "ctx_lens", x_in, self.cfg.d_model, R,
                         (("x_out", x_out, self.cfg.torch_dtype, (R, self.cfg.d_model)), ("slot_out", slot_out, torch.int64, (len(ctx_lens),))))
        S, max_blocks = block_tables.shape
        if x_out is None:
            x_out = torch.empty_like(x_in)
        max_ctx = int(ctx_lens.max()) + 1 if S else 0
        ws = workspace if workspace is not None else self._workspace(R, S, max_ctx, x_in.device)
        self._check(_lib.icarus_decode_step(self._h, _ptr(kv_pool), _ptr(block_tables), max_blocks, S, _ptr(ctx_lens),
                                            R, _ptr(row_seq), _ptr(row_model), _ptr(x_in), _ptr(x_out), _ptr(slot_out),
                                            _ptr(ws), ws.numel(), self._stream(x_in.device)))
        return x_out

    def _check_attn(self, q, kv_pool, block_tables, kv_lens, row_seq, out):
        R = len(row_seq)
        self._check_call(kv_pool, block_tables, len(kv_lens), "kv_lens")
        _want(q, "q", self.cfg.torch_dtype, None, block_tables.device)
        if q.numel() != R * self.cfg.n_q_heads * self.cfg.head_dim:
            raise ValueError(f"q has {q.numel()} elements for {R} rows of {self.cfg.n_q_heads} x {self.cfg.head_dim}")
        if out is not None:
            _want(out, "out", self.cfg.torch_dtype, tuple(q.shape), block_tables.device)

    def attn_shared_kv_static(self, q, kv_pool, block_tables, kv_lens, row_seq, out):
        """icarus_attn_shared_kv_static: no workspace, nothing allocated (the caller passes `out`)."""
        kv_lens, row_seq = _host_i32(kv_lens), _host_i32(row_seq)
        self._check_attn(q, kv_pool, block_tables, kv_lens, row_seq, out)
        S, max_blocks = block_tables.shape
        self._check(_lib.icarus_attn_shared_kv_static(self._h, _ptr(q), _ptr(kv_pool), _ptr(block_tables), max_blocks, S,
                                                      _ptr(kv_lens), len(row_seq), _ptr(row_seq), _ptr(out), self._stream(q.device)))
        return out

    def attn_shared_kv(self, q, kv_pool, block_tables, kv_lens, row_seq, out=None, workspace=None):
        kv_lens, row_seq = _host_i32(kv_lens), _host_i32(row_seq)
        self._check_attn(q, kv_pool, block_tables, kv_lens, row_seq, out)
        S, max_blocks = block_tables.shape
        R = len(row_seq)
        if out is None:
            out = torch.empty_like(q)
        max_ctx = int(kv_lens.max()) if S else 0
        ws = workspace if workspace is not None else self._workspace(R, S, max_ctx, q.device)
        self._check(_lib.icarus_attn_shared_kv(self._h, _ptr(q), _ptr(kv_pool), _ptr(block_tables), max_blocks, S,
                                               _ptr(kv_lens), R, _ptr(row_seq), _ptr(out), _ptr(ws), ws.numel(),
                                               self._stream(q.device)))
        return out

    # -- lengths on the device (include/icarus_blocks.h) -----------------------------
    def _table(self, block_tables):
        """Sequences, width and device of a block table."""
        index = _index_of(block_tables, "block_tables", torch.int32)
        if block_tables.dim() != 2:
            raise ValueError(f"block_tables: need [S, max_blocks], got {tuple(block_tables.shape)}")
        S, max_blocks = block_tables.shape
        _need(block_tables, "block_tables", torch.int32, (S, max_blocks), index)
        return S, max_blocks, index

    def _pool(self, kv_pool, index):
        c = self.cfg
        have = kv_pool.shape if isinstance(kv_pool, torch.Tensor) else ()
        _need(kv_pool, "kv_pool", c.pool_dtype, (max(c.num_blocks, have[0] if have else 0), c.n_kv_heads, 2, c.block_size * c.head_dim), index)

    def _bounds(self, codes, scales, index):
        c = self.cfg
        _need(codes, "codes", torch.int8, (c.num_blocks, c.n_kv_heads, 2, c.head_dim), index)
        _need(scales, "scales", torch.float32, (c.num_blocks, c.n_kv_heads), index)

    def _rows(self, q, what, index) -> int:
        """Number of rows of queries [R, Hq, D]."""
        R = q.shape[0] if isinstance(q, torch.Tensor) and q.dim() else 0
        _need(q, what, self.cfg.torch_dtype, (R, self.cfg.n_q_heads, self.cfg.head_dim), index)
        return R

    def _lists(self, blocks, counts, S, index) -> int:
        """Width of the lists of blocks [S, Hkv, width]."""
        width = blocks.shape[-1] if isinstance(blocks, torch.Tensor) and blocks.dim() else 0
        _need(blocks, "blocks", torch.int32, (S, self.cfg.n_kv_heads, width), index)
        _need(counts, "counts", torch.int32, (S,), index)
        return width

    def new_key_bounds(self, device="cuda"):
        """(codes, scales) for key_bounds and select_blocks, for all blocks of the pool."""
        c = self.cfg
        return (torch.zeros(c.num_blocks, c.n_kv_heads, 2, c.head_dim, dtype=torch.int8, device=device),
                torch.ones(c.num_blocks, c.n_kv_heads, dtype=torch.float32, device=device))

    def extend_sequences(self, seq_map, ctx_lens, new_lens, block_tables, free_ids, free_used, streams=None):
        """Fills `seq_map` (a SequenceMap) and the new entries of block_tables; all arrays are device tensors.  Returns seq_map."""
        S, max_blocks, index = self._table(block_tables)
        m = seq_map
        if m.n_seqs != S:
            raise ValueError(f"seq_map is for {m.n_seqs} sequences, block_tables has {S}")
        one, n_free = (S,), free_ids.shape[0]
        _need(ctx_lens, "ctx_lens", torch.int32, one, index)
        _need(new_lens, "new_lens", torch.int32, one, index)
        if streams is not None:
            _need(streams, "streams", torch.int32, one, index)
        _need(m.kv_lens, "seq_map", torch.int32, one, index)
        _need(free_ids, "free_ids", torch.int32, (n_free,), index)
        _need(free_used, "free_used", torch.int32, (1,), index)
        self._check(_launch(index, _lib.icarus_extend_sequences, self._h, S, ctx_lens.data_ptr(), new_lens.data_ptr(),
                            None if streams is None else streams.data_ptr(), block_tables.data_ptr(), max_blocks, free_ids.data_ptr(), n_free,
                            free_used.data_ptr(), m.max_rows, m.kv_lens.data_ptr(), m.row_start.data_ptr(), m.row_seq.data_ptr(),
                            m.row_pos.data_ptr(), m.row_slot.data_ptr(), m.counts.data_ptr()))
        return m

    def rope_append(self, qkv, row_pos, row_slot, kv_pool, q_out=None):
        """qkv [R, >= (Hq + 2 Hkv) * D], rows may be strided.  Returns q_out [R, Hq, D]; rows with a negative position are left as they were."""
        c = self.cfg
        index = _index_of(qkv, "qkv", c.torch_dtype)
        width = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim
        if qkv.dim() != 2 or qkv.shape[1] < width or qkv.stride(1) != 1 or (qkv.shape[0] > 1 and qkv.stride(0) < width):
            raise ValueError(f"qkv: shape {tuple(qkv.shape)} with strides {tuple(qkv.stride())}, expected rows of {width} contiguous elements")
        R = qkv.shape[0]
        _need(row_pos, "row_pos", torch.int32, (R,), index)
        _need(row_slot, "row_slot", torch.int64, (R,), index)
        self._pool(kv_pool, index)
        if q_out is None:
            q_out = torch.zeros(R, c.n_q_heads, c.head_dim, dtype=c.torch_dtype, device=qkv.device)
        _need(q_out, "q_out", c.torch_dtype, (R, c.n_q_heads, c.head_dim), index)
        self._check(_launch(index, _lib.icarus_rope_append, self._h, qkv.data_ptr(), max(qkv.stride(0), width), R, row_pos.data_ptr(),
                            row_slot.data_ptr(), q_out.data_ptr(), kv_pool.data_ptr()))
        return q_out

    def key_bounds(self, kv_pool, block_tables, from_lens, to_lens, codes, scales, max_new: int = 0):
        """Bounds of the keys of the blocks that hold positions from_lens .. to_lens - 1, into codes and scales (new_key_bounds)."""
        S, max_blocks, index = self._table(block_tables)
        self._pool(kv_pool, index)
        _need(from_lens, "from_lens", torch.int32, (S,), index)
        _need(to_lens, "to_lens", torch.int32, (S,), index)
        self._bounds(codes, scales, index)
        self._check(_launch(index, _lib.icarus_key_bounds, self._h, kv_pool.data_ptr(), block_tables.data_ptr(), max_blocks, S, from_lens.data_ptr(),
                            to_lens.data_ptr(), max_new, codes.data_ptr(), scales.data_ptr()))

    def select_blocks(self, q, codes, scales, block_tables, kv_lens, row_start, blocks, counts, first: int = 1, last: int = 2,
                      seq_rows: int = 0, workspace=None):
        """blocks [S, Hkv, top_k] and counts [S] receive each sequence's selected blocks.  seq_rows: as for attn_blocks, not needed here.  workspace: bytes for one call at a time, by default of its own."""
        S, max_blocks, index = self._table(block_tables)
        R = self._rows(q, "q", index)
        _need(row_start, "row_start", torch.int32, (S + 1,), index)
        _need(kv_lens, "kv_lens", torch.int32, (S,), index)
        self._bounds(codes, scales, index)
        top_k = self._lists(blocks, counts, S, index)
        if workspace is None:
            workspace = torch.empty(_lib.icarus_select_workspace_bytes(self._h, S, max_blocks), dtype=torch.uint8, device=q.device)
        elif not isinstance(workspace, torch.Tensor) or workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError("workspace: need a contiguous tensor on the device of the others")
        self._check(_launch(index, _lib.icarus_select_blocks, self._h, q.data_ptr(), codes.data_ptr(), scales.data_ptr(), block_tables.data_ptr(), max_blocks,
                            S, kv_lens.data_ptr(), R, row_start.data_ptr(), seq_rows, top_k, first, last, blocks.data_ptr(), counts.data_ptr(),
                            workspace.data_ptr(), workspace.nbytes))
        return blocks, counts

    def attn_blocks(self, q, kv_pool, block_tables, kv_lens, row_start, blocks, counts, out=None, seq_rows: int = 0, workspace=None):
        """Attention of the rows row_start[s] .. row_start[s + 1] - 1 over the listed blocks of sequence s; rows of no sequence are left as they were.
        workspace: as for select_blocks."""
        S, max_blocks, index = self._table(block_tables)
        R = self._rows(q, "q", index)
        self._pool(kv_pool, index)
        _need(row_start, "row_start", torch.int32, (S + 1,), index)
        _need(kv_lens, "kv_lens", torch.int32, (S,), index)
        width = self._lists(blocks, counts, S, index)
        if out is None:
            out = torch.zeros_like(q)
        self._rows(out, "out", index)
        if out.shape[0] != R:
            raise ValueError(f"out has {out.shape[0]} rows, q {R}")
        if workspace is None:
            workspace = torch.empty(_lib.icarus_attn_blocks_workspace_bytes(self._h, S, R, width), dtype=torch.uint8, device=q.device)
        elif not isinstance(workspace, torch.Tensor) or workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError("workspace: need a contiguous tensor on the device of the others")
        self._check(_launch(index, _lib.icarus_attn_blocks, self._h, q.data_ptr(), kv_pool.data_ptr(), block_tables.data_ptr(), max_blocks, S,
                            kv_lens.data_ptr(), R, row_start.data_ptr(), seq_rows, blocks.data_ptr(), counts.data_ptr(), width, out.data_ptr(),
                            workspace.data_ptr(), workspace.nbytes))
        return out

    # -- sequences that branch (include/icarus_branches.h) ---------------------------
    @staticmethod
    def _scratch(workspace, need, index):
        """The caller's workspace, or one of its own for this call."""
        if workspace is None:
            return torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", index))
        if not isinstance(workspace, torch.Tensor) or workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError("workspace: need a contiguous tensor on the device of the others")
        return workspace

    def beam_select(self, logits, scores, beams, row_start=None, done=None, eos: int = -1, workspace=None):
        """Best continuations of each group of beams.width beams, into `beams` (a BeamMap).  logits [R, vocab] float32 or bfloat16, rows may be strided; a beam takes its last row of
        row_start [S + 1], without it beam i has row i; a finished one needs none.  scores [S] float32, done [S] int32 of the beams now.  Returns beams."""
        m, S = beams, beams.groups * beams.width
        dt = logits.dtype if isinstance(logits, torch.Tensor) else None
        index = _index_of(logits, "logits", dt if dt is torch.bfloat16 else torch.float32)
        if logits.dim() != 2 or (logits.shape[0] and logits.shape[1] > 1 and logits.stride(1) != 1) or (logits.shape[0] > 1 and logits.stride(0) < logits.shape[1]):
            raise ValueError(f"logits: shape {tuple(logits.shape)} with strides {tuple(logits.stride())}, expected rows of contiguous elements")
        R, vocab = logits.shape
        _need(scores, "scores", torch.float32, (S,), index)
        if row_start is not None:
            _need(row_start, "row_start", torch.int32, (S + 1,), index)
        if done is not None:
            _need(done, "done", torch.int32, (S,), index)
        _need(m.parents, "beams", torch.int32, (S,), index)
        workspace = self._scratch(workspace, _lib.icarus_beam_workspace_bytes(self._h, m.groups, m.width, vocab), index)
        self._check(_launch(index, _lib.icarus_beam_select, self._h, logits.data_ptr(), BF16 if dt is torch.bfloat16 else F32, vocab,
                            max(logits.stride(0), vocab) if R > 1 else vocab, R, m.groups, m.width, None if row_start is None else row_start.data_ptr(), scores.data_ptr(),
                            None if done is None else done.data_ptr(), eos, m.parents.data_ptr(), m.tokens.data_ptr(), m.scores.data_ptr(), m.done.data_ptr(),
                            workspace.data_ptr(), workspace.nbytes))
        return m

    def fork_sequences(self, parents, kv_lens, block_tables, forked, free_ids, free_used, shared=None, workspace=None):
        """Lengths and tables of the children that `parents` names, into `forked` (a ForkMap), and the free list.  shared [groups]: leading columns of the tables that belong to the
        common prefix.  Behind them two sequences with children may not name the same partly filled block: for the first fork of samples of one prompt, shared counts the prompt's last block too.
        Returns forked."""
        S, max_blocks, index = self._table(block_tables)
        m = forked
        if S != m.groups * m.width or max_blocks != m.max_blocks:
            raise ValueError(f"forked is for {m.groups} groups of {m.width} sequences of {m.max_blocks} blocks, block_tables has shape {(S, max_blocks)}")
        n_free = free_ids.shape[0] if isinstance(free_ids, torch.Tensor) and free_ids.dim() else 0
        _need(parents, "parents", torch.int32, (S,), index)
        _need(kv_lens, "kv_lens", torch.int32, (S,), index)
        _need(free_ids, "free_ids", torch.int32, (n_free,), index)
        _need(free_used, "free_used", torch.int32, (1,), index)
        if shared is not None:
            _need(shared, "shared", torch.int32, (m.groups,), index)
        _need(m.block_tables, "forked", torch.int32, (S, max_blocks), index)
        workspace = self._scratch(workspace, _lib.icarus_fork_workspace_bytes(self._h, m.groups, m.width, max_blocks), index)
        self._check(_launch(index, _lib.icarus_fork_sequences, self._h, m.groups, m.width, parents.data_ptr(), kv_lens.data_ptr(), block_tables.data_ptr(), max_blocks,
                            None if shared is None else shared.data_ptr(), free_ids.data_ptr(), n_free, free_used.data_ptr(), m.kv_lens.data_ptr(), m.block_tables.data_ptr(),
                            m.copy_src.data_ptr(), m.copy_dst.data_ptr(), m.counts.data_ptr(), workspace.data_ptr(), workspace.nbytes))
        return m

    def copy_blocks(self, arrays, src, dst):
        """Block src[i] of each of `arrays` (pools, codes, scales: tensors of at least num_blocks blocks) to block dst[i]; -1: no copy."""
        index = _index_of(src, "src", torch.int32)
        n = src.shape[0] if src.dim() else 0
        _need(src, "src", torch.int32, (n,), index)
        _need(dst, "dst", torch.int32, (n,), index)
        blocks, at, size = self.cfg.num_blocks, array("q"), array("q")
        for t in arrays:
            if not isinstance(t, torch.Tensor) or not t.dim() or t.get_device() != index or t.size(0) < blocks or not t.is_contiguous():
                raise ValueError(f"arrays: need contiguous tensors of at least {blocks} blocks on the device of src")
            at.append(t.data_ptr())
            size.append(t.stride(0) * t.element_size())
        self._check(_launch(index, _lib.icarus_copy_blocks, self._h, at.buffer_info()[0], size.buffer_info()[0], len(at), src.data_ptr(), dst.data_ptr(), n))

    def attn_prefix(self, q, kv_pool, block_tables, kv_lens, row_start, group_start, prefix_lens, out=None, workspace=None):
        """Attention of the rows row_start[s] .. row_start[s + 1] - 1 over sequence s; the leading blocks of prefix_lens[g] tokens that the sequences group_start[g] .. group_start[g + 1] - 1
        share are read once.  Rows of no sequence or group are left as they were."""
        S, max_blocks, index = self._table(block_tables)
        R = self._rows(q, "q", index)
        self._pool(kv_pool, index)
        G = prefix_lens.shape[0] if isinstance(prefix_lens, torch.Tensor) and prefix_lens.dim() else 0
        _need(row_start, "row_start", torch.int32, (S + 1,), index)
        _need(kv_lens, "kv_lens", torch.int32, (S,), index)
        _need(group_start, "group_start", torch.int32, (G + 1,), index)
        _need(prefix_lens, "prefix_lens", torch.int32, (G,), index)
        if out is None:
            out = torch.zeros_like(q)
        self._rows(out, "out", index)
        if out.shape[0] != R:
            raise ValueError(f"out has {out.shape[0]} rows, q {R}")
        workspace = self._scratch(workspace, _lib.icarus_attn_prefix_workspace_bytes(self._h, S, G, R, max_blocks), index)
        self._check(_launch(index, _lib.icarus_attn_prefix, self._h, q.data_ptr(), kv_pool.data_ptr(), block_tables.data_ptr(), max_blocks, S, kv_lens.data_ptr(), R,
                            row_start.data_ptr(), G, group_start.data_ptr(), prefix_lens.data_ptr(), out.data_ptr(), workspace.data_ptr(), workspace.nbytes))
        return out


class IcarusStack:
    """A stack of IcarusLayer contexts with token embedding, final norm and LM head (marshalling only).
    layers: list of IcarusLayer (kept alive); embed, final_norm, lm_head: device tensors, storage dtype."""

    def __init__(self, layers, embed, final_norm, lm_head):
        self.layers = list(layers)
        self._t = [embed.contiguous(), final_norm.contiguous(), lm_head.contiguous()]
        self.vocab = int(lm_head.shape[0])
        arr = (C.c_void_p * len(self.layers))(*[l._h for l in self.layers])
        self._arr = arr
        cfg = _StackCfg(len(self.layers), self.vocab, C.cast(arr, C.POINTER(C.c_void_p)), self._t[0].data_ptr(),
                        self._t[1].data_ptr(), self._t[2].data_ptr())
        h = C.c_void_p()
        rc = _lib.icarus_stack_create(C.byref(cfg), C.byref(h))
        if rc != 0:
            raise IcarusError(rc, _lib.icarus_stack_last_error(None).decode())
        self._h = h
        self._ws = None

    def close(self):
        if getattr(self, "_h", None):
            _lib.icarus_stack_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc != 0:
            raise IcarusError(rc, _lib.icarus_stack_last_error(self._h).decode())

    def workspace_bytes(self, max_rows, max_seqs, max_ctx, max_logit_rows) -> int:
        return int(_lib.icarus_stack_workspace_bytes(self._h, max_rows, max_seqs, max_ctx, max_logit_rows))

    def _workspace(self, rows, seqs, max_ctx, logit_rows, device):
        need = self.workspace_bytes(rows, seqs, max_ctx, logit_rows)
        if self._ws is None or self._ws.numel() < need or self._ws.device != device:
            self._ws = torch.empty(need, dtype=torch.uint8, device=device)
        return self._ws

    @staticmethod
    def _pools(kv_pools):
        return (C.c_void_p * len(kv_pools))(*[p.data_ptr() for p in kv_pools])

    def prefill(self, kv_pools, block_tables, ctx_lens, chunk_lens, tokens, want_logits=False):
        """Returns (next_token [S] int32 device, logits [S, vocab] float32 device or None)."""
        ctx_lens, chunk_lens, tokens = _host_i32(ctx_lens), _host_i32(chunk_lens), _host_i32(tokens)
        S, max_blocks = block_tables.shape
        dev = block_tables.device
        R = int(chunk_lens.sum())
        nxt = torch.empty(S, dtype=torch.int32, device=dev)
        logits = torch.empty((S, self.vocab), dtype=torch.float32, device=dev) if want_logits else None
        ws = self._workspace(R, S, int((ctx_lens + chunk_lens).max()) if S else 0, S, dev)
        stream = C.c_void_p(torch.cuda.current_stream(dev).cuda_stream)
        self._check(_lib.icarus_stack_prefill(self._h, self._pools(kv_pools), _ptr(block_tables), max_blocks, S, _ptr(ctx_lens),
                                              _ptr(chunk_lens), _ptr(tokens), _ptr(nxt), _ptr(logits), _ptr(ws), ws.numel(), stream))
        return nxt, logits

    def decode(self, kv_pools, block_tables, ctx_lens, row_seq, row_model, seq_token, seq_next=None, want_logits=False):
        """seq_token: device int32 [S].  Returns (row_next [R] int32 device, logits [R, vocab] or None);
        seq_next (device int32 [S], may be seq_token itself) receives each sequence's last row's token."""
        ctx_lens, row_seq, row_model = _host_i32(ctx_lens), _host_i32(row_seq), _host_i32(row_model)
        S, max_blocks = block_tables.shape
        dev = block_tables.device
        R = len(row_seq)
        row_next = torch.empty(R, dtype=torch.int32, device=dev)
        logits = torch.empty((R, self.vocab), dtype=torch.float32, device=dev) if want_logits else None
        ws = self._workspace(R, S, int(ctx_lens.max()) + 1 if S else 0, R, dev)
        stream = C.c_void_p(torch.cuda.current_stream(dev).cuda_stream)
        self._check(_lib.icarus_stack_decode(self._h, self._pools(kv_pools), _ptr(block_tables), max_blocks, S, _ptr(ctx_lens), R,
                                             _ptr(row_seq), _ptr(row_model), _ptr(seq_token), _ptr(row_next), _ptr(seq_next),
                                             _ptr(logits), _ptr(ws), ws.numel(), stream))
        return row_next, logits


class PrefixCache:
    """icarus_cache_*: the cross-model prefix-cache manager (host side).  Marshalling only."""

    def __init__(self, num_blocks: int, block_size: int, key_by_model: bool):
        self.num_blocks, self.block_size, self.key_by_model = int(num_blocks), int(block_size), bool(key_by_model)
        self._h = C.c_void_p()
        cfg = _CacheCfg(self.num_blocks, self.block_size, int(self.key_by_model))
        rc = _lib.icarus_cache_create(C.byref(cfg), C.byref(self._h))
        if rc != 0:
            raise IcarusError(rc, (_lib.icarus_cache_last_error(None) or b"").decode())

    def close(self):
        if getattr(self, "_h", None):
            _lib.icarus_cache_destroy(self._h)
            self._h = None

    __del__ = close

    def _check(self, rc):
        if rc != 0:
            raise IcarusError(rc, (_lib.icarus_cache_last_error(self._h) or b"").decode())

    @staticmethod
    def _i32(a):
        return np.ascontiguousarray(a, dtype=np.int32)

    def acquire(self, tokens, model: int, reserve: int = 0):
        """-> (block ids of the sequence, number of leading tokens whose K/V is already cached)"""
        t = self._i32(tokens)
        cap = (len(t) + reserve + self.block_size - 1) // self.block_size
        out = np.empty(max(cap, 1), dtype=np.int32)
        nb, nc = C.c_int32(0), C.c_int32(0)
        self._check(_lib.icarus_cache_acquire(self._h, t.ctypes.data, len(t), int(model), int(reserve), out.ctypes.data, cap,
                                              C.byref(nb), C.byref(nc)))
        return out[: nb.value].tolist(), nc.value

    def extend(self, blocks, n_tokens_total: int):
        cap = max(len(blocks), (int(n_tokens_total) + self.block_size - 1) // self.block_size, 1)
        buf = np.empty(cap, dtype=np.int32)
        buf[: len(blocks)] = blocks
        nb = C.c_int32(len(blocks))
        self._check(_lib.icarus_cache_extend(self._h, buf.ctypes.data, cap, C.byref(nb), int(n_tokens_total)))
        return buf[: nb.value].tolist()

    def commit(self, tokens, model: int, blocks):
        t, b = self._i32(tokens), self._i32(blocks)
        self._check(_lib.icarus_cache_commit(self._h, t.ctypes.data, len(t), int(model), b.ctypes.data, len(b)))

    def release(self, blocks):
        b = self._i32(blocks)
        self._check(_lib.icarus_cache_release(self._h, b.ctypes.data, len(b)))

    def counts(self) -> dict:
        st = _CacheStats()
        self._check(_lib.icarus_cache_get_stats(self._h, C.byref(st)))
        return dict(lookups=st.lookups, hit_tokens=st.hit_tokens, miss_tokens=st.miss_tokens, evictions=st.evictions,
                    peak_live=st.peak_live, live=st.live, cached=st.cached, free=st.free_blocks)
