"""Thin ctypes binding of the C ABI declared in include/rom.h: argument marshalling only.

Every function takes torch tensors that already live where the ABI wants them (CUDA for data,
none on the host except sizes) and forwards raw pointers.  Nothing here computes anything; when
the compiled library is missing the import of `lib()` fails loudly -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librom_b200.so")

ROM_F32, ROM_BF16 = 0, 1
ROM_FLAG_SIMT_GEMM = 1
ROM_FLAG_DEBUG_CHECKS = 2
ROM_FLAG_TEST_STALL = 4
ROM_FLAG_FUSED_SMALL = 8
ROM_OK = 0

EXPORTS = ("rom_workspace_size", "rom_route", "rom_scan", "rom_layer_forward", "rom_workspace_find",
           "rom_get_status", "rom_status_string", "rom_last_launch_count", "rom_layer_forward_profile",
           "rom_num_stages", "rom_stage_name", "rom_route_noalloc", "rom_route_balance",
           "rom_ffn_moe_workspace_size", "rom_ffn_moe_forward", "rom_layer_step", "rom_layer_forward_host",
           "rom_scan_workspace_size", "rom_debug_check", "rom_scan_backward_workspace_size", "rom_scan_backward",
           "rom_layer_backward_workspace_size", "rom_layer_backward", "rom_mamba2_workspace_size", "rom_mamba2_layer_forward",
           "rom_conv_ragged", "rom_scan_ragged_workspace_size", "rom_scan_ragged", "rom_conv_step", "rom_scan_step",
           "rom_ffn_moe_step_workspace_size", "rom_ffn_moe_step",
           "rom_linattn_ragged_workspace_size", "rom_linattn_ragged", "rom_linattn_step", "rom_linattn_backward_workspace_size", "rom_linattn_backward",
           "rom_qk_norm_rope", "rom_qk_norm_rope_backward_workspace_size", "rom_qk_norm_rope_backward")


class RomConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "L", "d_model", "d_inner", "d_state", "d_conv", "dt_rank", "E", "K", "dtype",
                 "gate_mode", "disc_mode", "flags", "small_proj_experts")]


class RomWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("W_r", "b_r", "W_inz", "w_conv", "b_conv", "W_x", "W_dt", "b_dt", "A", "D", "W_out")]


class RomGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("dW_r", "db_r", "dW_inz", "dw_conv", "db_conv", "dW_x", "dW_dt", "db_dt", "dA", "dD", "dW_out")]


class RomMamba2Weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("W_r", "b_r", "W_in", "w_conv", "b_conv", "dt_bias", "A", "D", "w_norm", "W_out")]


class RomRagged(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seq", "rows", "n_slots")] + [(n, ctypes.c_void_p) for n in ("seq_start", "slot", "resume")]


class RomLinattnConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_heads", "n_qk_heads", "d_k", "d_v", "dtype", "flags")] + [("scale", ctypes.c_float)]


class RomQkConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_q_heads", "n_k_heads", "d_head", "rot_dim", "interleaved", "dtype")] + [("eps", ctypes.c_float)]


class RomError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load librom_b200.so (built in-tree by paper_2506_18145_b200.build).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2506_18145_b200.build` "
                              "(there is no CPU or PyTorch fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p, szp = ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)
        cfgp = ctypes.POINTER(RomConfig)
        L.rom_workspace_size.argtypes = [cfgp, szp]
        L.rom_scan_workspace_size.argtypes = [cfgp, szp]
        L.rom_debug_check.argtypes = [cfgp, vp, ctypes.c_size_t, vp]
        L.rom_scan_backward_workspace_size.argtypes = [cfgp, szp]
        L.rom_layer_backward_workspace_size.argtypes = [cfgp, szp]
        L.rom_mamba2_workspace_size.argtypes = [cfgp, ctypes.c_int32, szp]
        L.rom_mamba2_layer_forward.argtypes = [cfgp, ctypes.c_int32, ctypes.POINTER(RomMamba2Weights), vp, vp, i32p, vp, i32p, vp, ctypes.c_size_t, vp]
        L.rom_layer_backward.argtypes = [cfgp, ctypes.POINTER(RomWeights), vp, vp, vp, ctypes.POINTER(RomGrads), vp, ctypes.c_size_t, vp]
        L.rom_scan_backward.argtypes = [cfgp] + [vp] * 19 + [ctypes.c_size_t, vp]
        L.rom_route.argtypes = [cfgp, vp, vp, vp, i32p, vp, i32p, i32p, i32p, i32p, vp, ctypes.c_size_t, vp]
        L.rom_route_noalloc.argtypes = [cfgp, vp, vp, vp, i32p, vp, i32p, i32p, i32p, i32p, vp]
        L.rom_route_balance.argtypes = [cfgp, vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.rom_ffn_moe_workspace_size.argtypes = [cfgp, ctypes.c_int32, szp]
        L.rom_ffn_moe_forward.argtypes = [cfgp, ctypes.c_int32, vp, vp, vp, i32p, vp, vp, vp, ctypes.c_size_t, vp]
        L.rom_scan.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.rom_layer_forward.argtypes = [cfgp, ctypes.POINTER(RomWeights), vp, vp, i32p, vp, i32p, vp, ctypes.c_size_t, vp]
        L.rom_layer_forward_host.argtypes = [cfgp, ctypes.POINTER(RomWeights), vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.rom_layer_step.argtypes = [cfgp, ctypes.POINTER(RomWeights), vp, vp, vp, vp, i32p, vp, vp, ctypes.c_size_t, vp]
        L.rom_workspace_find.argtypes = [cfgp, ctypes.c_char_p, szp, szp]
        L.rom_get_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int32)]
        L.rom_status_string.argtypes = [ctypes.c_int]
        L.rom_status_string.restype = ctypes.c_char_p
        L.rom_last_launch_count.argtypes = []
        L.rom_layer_forward_profile.argtypes = [cfgp, ctypes.POINTER(RomWeights), vp, vp, vp, ctypes.c_size_t, vp,
                                                ctypes.POINTER(ctypes.c_float), ctypes.c_int]
        i32, i64, ragp = ctypes.c_int32, ctypes.c_int64, ctypes.POINTER(RomRagged)
        L.rom_conv_ragged.argtypes = [cfgp, ragp, vp, i64, vp, vp, vp, vp, vp, vp]
        L.rom_scan_ragged_workspace_size.argtypes = [cfgp, i32, i32, szp]
        L.rom_scan_ragged.argtypes = [cfgp, ragp, vp, vp, vp, vp, vp, i64, vp, vp, i64, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.rom_conv_step.argtypes = [cfgp, vp, i64, vp, vp, vp, i32, vp, vp, vp, vp]
        L.rom_scan_step.argtypes = [cfgp, vp, vp, vp, vp, vp, i64, vp, vp, i64, vp, i32, vp, vp, vp, vp]
        L.rom_ffn_moe_step_workspace_size.argtypes = [cfgp, i32, szp]
        L.rom_ffn_moe_step.argtypes = [cfgp, i32, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        linp, qkp, size_t = ctypes.POINTER(RomLinattnConfig), ctypes.POINTER(RomQkConfig), ctypes.c_size_t
        L.rom_linattn_ragged_workspace_size.argtypes = L.rom_linattn_backward_workspace_size.argtypes = [linp, i32, i32, szp]
        L.rom_linattn_ragged.argtypes = [linp, ragp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, size_t, vp]
        L.rom_linattn_step.argtypes = [linp, i32, vp, i64, vp, i64, vp, i64, vp, vp, i32, vp, vp, vp, vp]
        L.rom_linattn_backward.argtypes = [linp, ragp, vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp, vp, size_t, vp]
        L.rom_qk_norm_rope.argtypes = [qkp, i32, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, i64, vp]
        L.rom_qk_norm_rope_backward_workspace_size.argtypes = [qkp, i32, szp]
        L.rom_qk_norm_rope_backward.argtypes = [qkp, i32, vp, vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, size_t, vp]
        L.rom_num_stages.argtypes = []
        L.rom_stage_name.argtypes = [ctypes.c_int]
        L.rom_stage_name.restype = ctypes.c_char_p
        for name in EXPORTS:
            if name not in ("rom_status_string", "rom_stage_name"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().rom_status_string(int(code)).decode()


def make_config(B, L, d_model, d_inner, d_state, d_conv, dt_rank, E, K, dtype, gate_mode=0, disc_mode=0, flags=0,
                small_proj_experts=0) -> RomConfig:
    dt = {"f32": ROM_F32, "bf16": ROM_BF16, torch.float32: ROM_F32, torch.bfloat16: ROM_BF16}[dtype]
    return RomConfig(B, L, d_model, d_inner, d_state, d_conv, dt_rank, E, K, dt, gate_mode, disc_mode, flags, small_proj_experts)


def config_from_shape(shape, gate_mode=0, disc_mode=0, flags=0, small_proj_experts=0) -> RomConfig:
    """shape: a synth.RomShape.  small_proj_experts: 0 = shared x Proj / dt Proj, shape.E = one per expert."""
    return make_config(shape.B, shape.L, shape.d_model, shape.d_inner, shape.d_state, shape.d_conv, shape.dt_rank,
                       shape.E, shape.K, shape.dtype, gate_mode, disc_mode, flags, small_proj_experts)


def _ptr(t: Optional[torch.Tensor], cuda: bool = True) -> Optional[int]:
    if t is None:
        return None
    if cuda and not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream], device: Optional[int] = None) -> int:
    # (the current stream's handle alone: 0.2 us, where the Stream object around it takes 3.3)
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device is None else device)


def workspace_size(cfg: RomConfig) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_workspace_size(ctypes.byref(cfg), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_workspace_size")
    return int(n.value)


def scan_workspace_size(cfg: RomConfig) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_scan_workspace_size(ctypes.byref(cfg), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_scan_workspace_size", "rom_debug_check", "rom_scan_backward_workspace_size", "rom_scan_backward",
           "rom_layer_backward_workspace_size", "rom_layer_backward", "rom_mamba2_workspace_size", "rom_mamba2_layer_forward")
    return int(n.value)


def workspace_find(cfg: RomConfig, name: str):
    off, n = ctypes.c_size_t(0), ctypes.c_size_t(0)
    rc = lib().rom_workspace_find(ctypes.byref(cfg), name.encode(), ctypes.byref(off), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_workspace_find")
    return int(off.value), int(n.value)


def alloc_workspace(cfg: RomConfig, device="cuda") -> torch.Tensor:
    return torch.empty(workspace_size(cfg), dtype=torch.uint8, device=device)


def rom_route(cfg, x, W_r, b_r, topk_idx, gates, counts, offsets, perm, inv_perm, ws, stream=None, check=True) -> int:
    rc = lib().rom_route(ctypes.byref(cfg), _ptr(x), _ptr(W_r), _ptr(b_r), _ptr(topk_idx), _ptr(gates), _ptr(counts),
                         _ptr(offsets), _ptr(perm), _ptr(inv_perm), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_route")
    return rc


def rom_route_noalloc(cfg, x, W_r, b_r, topk_idx, gates, counts, offsets, perm, inv_perm, stream=None, check=True) -> int:
    """rom_route without a workspace argument: the scratch is a fixed array inside the library
    (limits and sharing rules are stated beside the declaration in include/rom.h)."""
    rc = lib().rom_route_noalloc(ctypes.byref(cfg), _ptr(x), _ptr(W_r), _ptr(b_r), _ptr(topk_idx), _ptr(gates), _ptr(counts),
                                 _ptr(offsets), _ptr(perm), _ptr(inv_perm), _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_route_noalloc")
    return rc


def rom_route_balance(cfg, x, W_r, b_r, alpha, F, Pbar, loss, ws, stream=None, check=True) -> int:
    rc = lib().rom_route_balance(ctypes.byref(cfg), _ptr(x), _ptr(W_r), _ptr(b_r), ctypes.c_float(alpha), _ptr(F), _ptr(Pbar),
                                 _ptr(loss), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_route_balance")
    return rc


def rom_scan(cfg, u, delta, A, Bm, Cm, D, z, h0, y, h_last, ws=None, stream=None, check=True) -> int:
    rc = lib().rom_scan(ctypes.byref(cfg), _ptr(u), _ptr(delta), _ptr(A), _ptr(Bm), _ptr(Cm), _ptr(D), _ptr(z), _ptr(h0),
                        _ptr(y), _ptr(h_last), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_scan")
    return rc


def scan_backward_workspace_size(cfg: RomConfig) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_scan_backward_workspace_size(ctypes.byref(cfg), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_scan_backward_workspace_size")
    return int(n.value)


def rom_scan_backward(cfg, dy, u, delta, A, Bm, Cm, D, z, h0, dh_last, du, ddelta, dA, dBm, dCm, dD, dz, dh0, ws,
                      stream=None, check=True) -> int:
    rc = lib().rom_scan_backward(ctypes.byref(cfg), _ptr(dy), _ptr(u), _ptr(delta), _ptr(A), _ptr(Bm), _ptr(Cm), _ptr(D), _ptr(z),
                                 _ptr(h0), _ptr(dh_last), _ptr(du), _ptr(ddelta), _ptr(dA), _ptr(dBm), _ptr(dCm), _ptr(dD),
                                 _ptr(dz), _ptr(dh0), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_scan_backward")
    return rc


def layer_backward_workspace_size(cfg: RomConfig) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_layer_backward_workspace_size(ctypes.byref(cfg), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_layer_backward_workspace_size")
    return int(n.value)


def make_grads(g: Dict[str, Optional[torch.Tensor]]) -> RomGrads:
    return RomGrads(*[_ptr(g.get(n)) for n, _ in RomGrads._fields_])


def rom_layer_backward(cfg, weights: RomWeights, x, dout, dx, grads: RomGrads, ws, stream=None, check=True) -> int:
    rc = lib().rom_layer_backward(ctypes.byref(cfg), ctypes.byref(weights), _ptr(x), _ptr(dout), _ptr(dx), ctypes.byref(grads), _ptr(ws),
                                  ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_layer_backward")
    return rc


def mamba2_workspace_size(cfg: RomConfig, headdim: int) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_mamba2_workspace_size(ctypes.byref(cfg), int(headdim), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_mamba2_workspace_size")
    return int(n.value)


def make_mamba2_weights(w: Dict[str, Optional[torch.Tensor]]) -> RomMamba2Weights:
    return RomMamba2Weights(*[_ptr(w.get(n)) for n, _ in RomMamba2Weights._fields_])


def rom_mamba2_layer_forward(cfg, headdim, weights: RomMamba2Weights, x, out, topk_idx_out, gates_out, counts_out, ws, stream=None, check=True) -> int:
    rc = lib().rom_mamba2_layer_forward(ctypes.byref(cfg), int(headdim), ctypes.byref(weights), _ptr(x), _ptr(out), _ptr(topk_idx_out),
                                        _ptr(gates_out), _ptr(counts_out), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_mamba2_layer_forward")
    return rc


def make_weights(w: Dict[str, Optional[torch.Tensor]]) -> RomWeights:
    return RomWeights(*[_ptr(w.get(n)) for n, _ in RomWeights._fields_])


def rom_layer_forward(cfg, weights: RomWeights, x, out, topk_idx_out, gates_out, counts_out, ws, stream=None, check=True) -> int:
    rc = lib().rom_layer_forward(ctypes.byref(cfg), ctypes.byref(weights), _ptr(x), _ptr(out), _ptr(topk_idx_out),
                                 _ptr(gates_out), _ptr(counts_out), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_layer_forward")
    return rc


def ffn_moe_workspace_size(cfg: RomConfig, d_ff: int) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_ffn_moe_workspace_size(ctypes.byref(cfg), int(d_ff), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_ffn_moe_workspace_size")
    return int(n.value)


def rom_ffn_moe_forward(cfg, d_ff, W_gu, W_down, x, topk_idx, gates, out, ws, stream=None, check=True) -> int:
    rc = lib().rom_ffn_moe_forward(ctypes.byref(cfg), int(d_ff), _ptr(W_gu), _ptr(W_down), _ptr(x), _ptr(topk_idx), _ptr(gates),
                                   _ptr(out), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_ffn_moe_forward")
    return rc


def rom_layer_forward_host(cfg, weights: RomWeights, x_host, out_host, x_dev, out_dev, ws, stream=None, check=True) -> int:
    """x_host / out_host: CPU tensors (pinned for asynchronous copies); x_dev / out_dev: CUDA staging tensors."""
    rc = lib().rom_layer_forward_host(ctypes.byref(cfg), ctypes.byref(weights), _ptr(x_host, cuda=False), _ptr(out_host, cuda=False),
                                      _ptr(x_dev), _ptr(out_dev), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_layer_forward_host")
    return rc


def rom_layer_step(cfg, weights: RomWeights, x, conv_state, ssm_state, out, topk_idx_out, gates_out, ws, stream=None, check=True) -> int:
    rc = lib().rom_layer_step(ctypes.byref(cfg), ctypes.byref(weights), _ptr(x), _ptr(conv_state), _ptr(ssm_state), _ptr(out),
                              _ptr(topk_idx_out), _ptr(gates_out), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_layer_step")
    return rc


_STORAGE = {ROM_F32: torch.float32, ROM_BF16: torch.bfloat16}


def _elsewhere(t: torch.Tensor, device: int) -> ValueError:
    return ValueError(f"a tensor is on device {t.device}, the call runs on cuda:{device}")


def _at(t: Optional[torch.Tensor], device: int, n: int = 0, dtype: Optional[torch.dtype] = None) -> Optional[int]:
    """Address of a contiguous tensor of a serving call, of which the call reads or writes n elements of the given type.  These launch on the current device: what
    lies on another one (or on the host) is refused."""
    if t is None:
        return None
    if t.get_device() != device:
        raise _elsewhere(t, device)
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    if t.numel() < n or (dtype is not None and t.dtype is not dtype):
        raise ValueError(f"a tensor of {t.numel()} elements of {t.dtype} where the call needs {n} of {dtype}")
    return t.data_ptr()


def _rows_at(t: Optional[torch.Tensor], device: int, n_rows: int = 0, n_columns: int = 0, dtype: Optional[torch.dtype] = None):
    """(address, elements between rows) of a [rows, width] tensor whose rows are contiguous; a column slice of wider rows is one."""
    if t is None:
        return None, 0
    if t.get_device() != device:
        raise _elsewhere(t, device)
    pitch = t.stride()
    if len(pitch) != 2 or pitch[1] != 1:
        raise ValueError("expected a tensor [rows, width] with contiguous rows")
    rows, width = t.shape
    if rows < n_rows or width < n_columns or (dtype is not None and t.dtype is not dtype):
        raise ValueError(f"a tensor [{rows}, {width}] of {t.dtype} where the call needs [{n_rows}, {n_columns}] of {dtype}")
    return t.data_ptr(), pitch[0] if rows > 1 else width      # (a single row has no pitch: torch may say anything)


def _sequences(seqs: RomRagged, device: int):
    if getattr(seqs, "device", device) != device:
        raise ValueError(f"the sequences are on cuda:{seqs.device}, the call runs on cuda:{device}")
    return ctypes.byref(seqs)


def _slots(a: Optional[torch.Tensor], b: Optional[torch.Tensor]) -> int:
    """Slots of the state pools of a call (0 without both, which the library refuses)."""
    if a is None or b is None:
        return 0
    n = a.shape[0]
    if b is not a and b.shape[0] != n:
        raise ValueError("the pools differ in their slots")
    return n


def _bc(Bm, Cm, device: int, n_rows: int, d_state: int):
    """Addresses of B and C and their common pitch."""
    (pb, ldb), (pc, ldc) = _rows_at(Bm, device, n_rows, d_state, torch.float32), _rows_at(Cm, device, n_rows, d_state, torch.float32)
    if ldb != ldc:
        raise ValueError("Bm and Cm differ in their pitch")
    return pb, pc, ldb


def make_ragged(rows: int, n_slots: int, seq_start, slot=None, resume=None) -> RomRagged:
    """Sequences packed in buffers of `rows` rows.  The tensors (int32, on the device) may change in place between calls."""
    n_seq = seq_start.numel() - 1
    for t, n in ((seq_start, n_seq + 1), (slot, n_seq), (resume, n_seq)):
        if t is not None and (t.dtype != torch.int32 or t.numel() != n):
            raise ValueError("expected int32 tensors: n_seq + 1 offsets, n_seq slots, n_seq flags")
    r = RomRagged(n_seq, rows, n_slots, _ptr(seq_start), _ptr(slot), _ptr(resume))
    r.tensors = (seq_start, slot, resume)      # (they live as long as the addresses do)
    r.device = seq_start.get_device()
    for t in (slot, resume):
        if t is not None and t.get_device() != r.device:
            raise ValueError("the sequences' tensors are on different devices")
    return r


def rom_conv_ragged(cfg, seqs: RomRagged, x, w_conv, b_conv, win_in, win_out, y, stream=None, check=True) -> int:
    """x: [rows, d_inner], rows may be a column slice of wider ones; y is not x."""
    d, De, rows, k, T, f32 = torch.cuda.current_device(), cfg.d_inner, seqs.rows, cfg.d_conv, _STORAGE.get(cfg.dtype), torch.float32
    (px, ldx), py, pool = _rows_at(x, d, rows, De, T), _at(y, d, rows * De, T), seqs.n_slots * (k - 1) * De
    if px == py and px:
        raise ValueError("y is x")
    rc = lib().rom_conv_ragged(ctypes.byref(cfg), _sequences(seqs, d), px, ldx, _at(w_conv, d, k * De, T), _at(b_conv, d, De, f32), _at(win_in, d, pool, f32),
                               _at(win_out, d, pool, f32), py, _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_conv_ragged")
    return rc


def scan_ragged_workspace_size(cfg: RomConfig, n_seq: int, rows: int) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_scan_ragged_workspace_size(ctypes.byref(cfg), int(n_seq), int(rows), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_scan_ragged_workspace_size")
    return int(n.value)


def rom_scan_ragged(cfg, seqs: RomRagged, u, delta, A, Bm, Cm, D, z, h_in, h_out, y, ws, stream=None, check=True) -> int:
    """Bm, Cm: [rows, d_state] of one pitch; z: [rows, d_inner]; both may be column slices of wider rows."""
    d, De, N, rows, T, f32 = torch.cuda.current_device(), cfg.d_inner, cfg.d_state, seqs.rows, _STORAGE.get(cfg.dtype), torch.float32
    n, pool = rows * De, seqs.n_slots * De * N
    (pb, pc, ld), (pz, ldz) = _bc(Bm, Cm, d, rows, N), _rows_at(z, d, rows, De, T)
    rc = lib().rom_scan_ragged(ctypes.byref(cfg), _sequences(seqs, d), _at(u, d, n, T), _at(delta, d, n, f32), _at(A, d, De * N, f32), pb, pc, ld, _at(D, d, De, f32), pz, ldz,
                               _at(h_in, d, pool, f32), _at(h_out, d, pool, f32), _at(y, d, n, T), _at(ws, d), ws.numel() if ws is not None else 0, _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_scan_ragged")
    return rc


def rom_conv_step(cfg, x, w_conv, b_conv, slot, win_in, win_out, y, stream=None, check=True) -> int:
    d, B, De, k, T, f32 = torch.cuda.current_device(), cfg.B, cfg.d_inner, cfg.d_conv, _STORAGE.get(cfg.dtype), torch.float32
    (px, ldx), n_slots = _rows_at(x, d, B, De, T), _slots(win_in, win_out)
    pool = n_slots * (k - 1) * De
    rc = lib().rom_conv_step(ctypes.byref(cfg), px, ldx, _at(w_conv, d, k * De, T), _at(b_conv, d, De, f32), _at(slot, d, B, torch.int32), n_slots, _at(win_in, d, pool, f32),
                             _at(win_out, d, pool, f32), _at(y, d, B * De, T), _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_conv_step")
    return rc


def rom_scan_step(cfg, u, delta, A, Bm, Cm, D, z, slot, h_in, h_out, y, stream=None, check=True) -> int:
    d, B, De, N, T, f32 = torch.cuda.current_device(), cfg.B, cfg.d_inner, cfg.d_state, _STORAGE.get(cfg.dtype), torch.float32
    (pb, pc, ld), (pz, ldz), n_slots = _bc(Bm, Cm, d, B, N), _rows_at(z, d, B, De, T), _slots(h_in, h_out)
    n, pool = B * De, n_slots * De * N
    rc = lib().rom_scan_step(ctypes.byref(cfg), _at(u, d, n, T), _at(delta, d, n, f32), _at(A, d, De * N, f32), pb, pc, ld, _at(D, d, De, f32), pz, ldz, _at(slot, d, B, torch.int32),
                             n_slots, _at(h_in, d, pool, f32), _at(h_out, d, pool, f32), _at(y, d, n, T), _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_scan_step")
    return rc


def ffn_moe_step_workspace_size(cfg: RomConfig, d_ff: int) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_ffn_moe_step_workspace_size(ctypes.byref(cfg), int(d_ff), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_ffn_moe_step_workspace_size")
    return int(n.value)


def rom_ffn_moe_step(cfg, d_ff, W_gu, W_down, x, topk_idx, gates, out, ws, stream=None, check=True) -> int:
    d, T, f32, F = torch.cuda.current_device(), _STORAGE.get(cfg.dtype), torch.float32, int(d_ff)
    tokens, Dm, E = cfg.B * cfg.L, cfg.d_model, cfg.E
    n, w = tokens * Dm, E * F * Dm
    chosen = tokens * cfg.K
    rc = lib().rom_ffn_moe_step(ctypes.byref(cfg), F, _at(W_gu, d, 2 * w, T), _at(W_down, d, w, T), _at(x, d, n, T), _at(topk_idx, d, chosen, torch.int32),
                                _at(gates, d, chosen, f32), _at(out, d, n, T), _at(ws, d), ws.numel() if ws is not None else 0, _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_ffn_moe_step")
    return rc


_DTYPES = {"f32": ROM_F32, "bf16": ROM_BF16, torch.float32: ROM_F32, torch.bfloat16: ROM_BF16}


def make_linattn_config(n_heads, n_qk_heads, d_k, d_v, dtype, scale: Optional[float] = None, flags=0) -> RomLinattnConfig:
    """scale: None = d_k ** -0.5."""
    return RomLinattnConfig(n_heads, n_qk_heads, d_k, d_v, _DTYPES[dtype], flags, d_k ** -0.5 if scale is None else scale)


def _linattn_size(name: str, cfg: RomLinattnConfig, n_seq: int, rows: int) -> int:
    n = ctypes.c_size_t(0)
    rc = getattr(lib(), name)(ctypes.byref(cfg), int(n_seq), int(rows), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, name)
    return int(n.value)


def linattn_ragged_workspace_size(cfg: RomLinattnConfig, n_seq: int, rows: int) -> int:
    return _linattn_size("rom_linattn_ragged_workspace_size", cfg, n_seq, rows)


def linattn_backward_workspace_size(cfg: RomLinattnConfig, n_seq: int, rows: int) -> int:
    return _linattn_size("rom_linattn_backward_workspace_size", cfg, n_seq, rows)


def rom_linattn_ragged(cfg, seqs: RomRagged, q, k, v, log_decay, s_in, s_out, o, ws, stream=None, check=True) -> int:
    """q, k: [rows, n_qk_heads * d_k], v: [rows, n_heads * d_v], each may be a column slice of wider rows; o: [rows, n_heads * d_v], contiguous, none of them."""
    d, rows, T, f32 = torch.cuda.current_device(), seqs.rows, _STORAGE.get(cfg.dtype), torch.float32
    wqk, wv, pool = cfg.n_qk_heads * cfg.d_k, cfg.n_heads * cfg.d_v, seqs.n_slots * cfg.n_heads * cfg.d_k * cfg.d_v
    (pq, ldq), (pk, ldk), (pv, ldv) = _rows_at(q, d, rows, wqk, T), _rows_at(k, d, rows, wqk, T), _rows_at(v, d, rows, wv, T)
    rc = lib().rom_linattn_ragged(ctypes.byref(cfg), _sequences(seqs, d), pq, ldq, pk, ldk, pv, ldv, _at(log_decay, d, cfg.n_heads, f32), _at(s_in, d, pool, f32),
                                  _at(s_out, d, pool, f32), _at(o, d, rows * wv, T), _at(ws, d), ws.numel() if ws is not None else 0, _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_linattn_ragged")
    return rc


def rom_linattn_step(cfg, q, k, v, log_decay, slot, s_in, s_out, o, stream=None, check=True) -> int:
    """One token of q.shape[0] sequences; slot: int32 [B] or None."""
    if q is None or q.dim() != 2:
        raise ValueError("expected q [B, n_qk_heads * d_k]")
    d, B, T, f32, n_slots = torch.cuda.current_device(), q.shape[0], _STORAGE.get(cfg.dtype), torch.float32, _slots(s_in, s_out)
    wqk, wv, pool = cfg.n_qk_heads * cfg.d_k, cfg.n_heads * cfg.d_v, n_slots * cfg.n_heads * cfg.d_k * cfg.d_v
    (pq, ldq), (pk, ldk), (pv, ldv) = _rows_at(q, d, B, wqk, T), _rows_at(k, d, B, wqk, T), _rows_at(v, d, B, wv, T)
    rc = lib().rom_linattn_step(ctypes.byref(cfg), B, pq, ldq, pk, ldk, pv, ldv, _at(log_decay, d, cfg.n_heads, f32), _at(slot, d, B, torch.int32), n_slots,
                                _at(s_in, d, pool, f32), _at(s_out, d, pool, f32), _at(o, d, B * wv, T), _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_linattn_step")
    return rc


def rom_linattn_backward(cfg, seqs: RomRagged, dout, q, k, v, log_decay, s_in, ds_out, dq, dk, dv, ds_in, ws, stream=None, check=True) -> int:
    """dout: [rows, n_heads * d_v], dq, dk: [rows, n_qk_heads * d_k], contiguous; dv: [rows, n_heads * d_v], may be a column slice of wider rows."""
    d, rows, T, f32 = torch.cuda.current_device(), seqs.rows, _STORAGE.get(cfg.dtype), torch.float32
    wqk, wv, pool = cfg.n_qk_heads * cfg.d_k, cfg.n_heads * cfg.d_v, seqs.n_slots * cfg.n_heads * cfg.d_k * cfg.d_v
    (pq, ldq), (pk, ldk), (pv, ldv), (pdv, lddv) = _rows_at(q, d, rows, wqk, T), _rows_at(k, d, rows, wqk, T), _rows_at(v, d, rows, wv, T), _rows_at(dv, d, rows, wv, T)
    rc = lib().rom_linattn_backward(ctypes.byref(cfg), _sequences(seqs, d), _at(dout, d, rows * wv, T), pq, ldq, pk, ldk, pv, ldv, _at(log_decay, d, cfg.n_heads, f32),
                                    _at(s_in, d, pool, f32), _at(ds_out, d, pool, f32), _at(dq, d, rows * wqk, T), _at(dk, d, rows * wqk, T), pdv, lddv,
                                    _at(ds_in, d, pool, f32), _at(ws, d), ws.numel() if ws is not None else 0, _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_linattn_backward")
    return rc


def make_qk_config(n_q_heads, n_k_heads, d_head, rot_dim, dtype, eps=1e-6, interleaved=False) -> RomQkConfig:
    return RomQkConfig(n_q_heads, n_k_heads, d_head, rot_dim, int(interleaved), _DTYPES[dtype], eps)


def _rotation(cfg, pos, inv_freq, d: int, rows: int):
    n = rows if cfg.rot_dim else 0
    return _at(pos, d, n, torch.int32), _at(inv_freq, d, cfg.rot_dim // 2, torch.float32)


def rom_qk_norm_rope(cfg, q, k, w_q, w_k, pos, inv_freq, q_out, k_out, stream=None, check=True) -> int:
    """q, q_out: [rows, n_q_heads * d_head]; k, k_out: [rows, n_k_heads * d_head]; each may be a column slice of wider rows, an output may be its input."""
    if q is None or q.dim() != 2:
        raise ValueError("expected q [rows, n_q_heads * d_head]")
    d, rows, T, f32 = torch.cuda.current_device(), q.shape[0], _STORAGE.get(cfg.dtype), torch.float32
    wq, wk = cfg.n_q_heads * cfg.d_head, cfg.n_k_heads * cfg.d_head
    (pq, ldq), (pk, ldk), (pyq, ldyq), (pyk, ldyk) = _rows_at(q, d, rows, wq, T), _rows_at(k, d, rows, wk, T), _rows_at(q_out, d, rows, wq, T), _rows_at(k_out, d, rows, wk, T)
    ppos, pfreq = _rotation(cfg, pos, inv_freq, d, rows)
    rc = lib().rom_qk_norm_rope(ctypes.byref(cfg), rows, pq, ldq, pk, ldk, _at(w_q, d, cfg.d_head, f32), _at(w_k, d, cfg.d_head, f32), ppos, pfreq, pyq, ldyq, pyk, ldyk,
                                _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_qk_norm_rope")
    return rc


def qk_norm_rope_backward_workspace_size(cfg: RomQkConfig, rows: int) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().rom_qk_norm_rope_backward_workspace_size(ctypes.byref(cfg), int(rows), ctypes.byref(n))
    if rc != ROM_OK:
        raise RomError(rc, "rom_qk_norm_rope_backward_workspace_size")
    return int(n.value)


def rom_qk_norm_rope_backward(cfg, dq_out, dk_out, q, k, w_q, w_k, pos, inv_freq, dq, dk, dw_q, dw_k, ws, stream=None, check=True) -> int:
    """dq_out, dk_out: contiguous; q, k, dq, dk: as q and k of rom_qk_norm_rope; dw_q, dw_k: None exactly where w_q, w_k are."""
    if q is None or q.dim() != 2:
        raise ValueError("expected q [rows, n_q_heads * d_head]")
    d, rows, T, f32 = torch.cuda.current_device(), q.shape[0], _STORAGE.get(cfg.dtype), torch.float32
    wq, wk, w = cfg.n_q_heads * cfg.d_head, cfg.n_k_heads * cfg.d_head, cfg.d_head
    (pq, ldq), (pk, ldk), (pyq, ldyq), (pyk, ldyk) = _rows_at(q, d, rows, wq, T), _rows_at(k, d, rows, wk, T), _rows_at(dq, d, rows, wq, T), _rows_at(dk, d, rows, wk, T)
    ppos, pfreq = _rotation(cfg, pos, inv_freq, d, rows)
    rc = lib().rom_qk_norm_rope_backward(ctypes.byref(cfg), rows, _at(dq_out, d, rows * wq, T), _at(dk_out, d, rows * wk, T), pq, ldq, pk, ldk, _at(w_q, d, w, f32),
                                         _at(w_k, d, w, f32), ppos, pfreq, pyq, ldyq, pyk, ldyk, _at(dw_q, d, w, f32), _at(dw_k, d, w, f32), _at(ws, d),
                                         ws.numel() if ws is not None else 0, _stream(stream, d))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_qk_norm_rope_backward")
    return rc


def rom_debug_check(cfg, ws, stream=None, check=True) -> int:
    rc = lib().rom_debug_check(ctypes.byref(cfg), _ptr(ws), ws.numel(), _stream(stream))
    if check and rc != ROM_OK:
        raise RomError(rc, "rom_debug_check")
    return rc


def rom_get_status(ws, stream=None) -> int:
    code = ctypes.c_int32(0)
    rc = lib().rom_get_status(_ptr(ws), _stream(stream), ctypes.byref(code))
    if rc != ROM_OK:
        raise RomError(rc, "rom_get_status")
    return int(code.value)


def last_launch_count() -> int:
    return int(lib().rom_last_launch_count())


def stage_names():
    L = lib()
    return [L.rom_stage_name(i).decode() for i in range(L.rom_num_stages())]


def rom_layer_forward_profile(cfg, weights: RomWeights, x, out, ws, stream=None):
    """Returns {stage name: milliseconds} of one forward (synchronises the stream)."""
    L = lib()
    n = L.rom_num_stages()
    ms = (ctypes.c_float * n)()
    rc = L.rom_layer_forward_profile(ctypes.byref(cfg), ctypes.byref(weights), _ptr(x), _ptr(out), _ptr(ws), ws.numel(),
                                     _stream(stream), ms, n)
    if rc != ROM_OK:
        raise RomError(rc, "rom_layer_forward_profile")
    return dict(zip(stage_names(), [float(v) for v in ms]))
