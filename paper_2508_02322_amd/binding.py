"""Thin ctypes binding over libcamera_hip.so (include/camera.h).

Argument marshalling only: every step of the path runs in the HIP kernels
behind the C ABI.  torch is used for device memory and the current stream.
There is no CPU fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libcamera_hip.so")

F32, BF16 = 0, 1
ACCUMULATE, NO_FINALIZE, DISTILL_TAIL = 1, 2, 4
MAX_ALTERNATIVES, DISTILL_STATS = 256, 5
K_ROUTE, K_BUCKET, K_GEMM, K_DOWN_NORM, K_FINALIZE, K_RANK, K_GATHER, K_DOWN_GEMM, K_COMBINE = range(9)
KERNEL_NAMES = ["route", "bucket", "gemm", "down_norm", "finalize", "rank", "gather", "down_gemm", "combine",
                "compact_hidden", "compact_down", "logprobs", "distill", "gated_grad"]

EXPORTS = ["camera_create", "camera_destroy", "camera_last_error", "camera_version", "camera_route_topk",
           "camera_score_layer", "camera_select_prune", "camera_select_prune_noalloc", "camera_select_prune_multi", "camera_alloc_bits", "camera_rank_decisions",
           "camera_gather_micro_experts", "camera_input_channel_energy", "camera_layer_forward", "camera_layer_forward_compact", "camera_output_error",
           "camera_token_logprobs", "camera_token_logprobs_backward", "camera_distill_topk", "camera_distill_topk_backward",
           "camera_gated_ffn", "camera_gated_ffn_backward", "camera_profile_enable", "camera_profile_read"]

_c = ctypes
_vp, _i, _i64, _f, _d = _c.c_void_p, _c.c_int, _c.c_int64, _c.c_float, _c.c_double


class CameraError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"camera status {code}: {message}")
        self.code = code
        self.message = message


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} is missing: build it with `python -m paper_2508_02322_amd.build` (there is no fallback path)")
    lib = ctypes.CDLL(path)
    lib.camera_create.argtypes = [_c.POINTER(_vp), _i]
    lib.camera_destroy.argtypes = [_vp]
    lib.camera_last_error.argtypes = [_vp]
    lib.camera_last_error.restype = _c.c_char_p
    lib.camera_version.argtypes = []
    lib.camera_route_topk.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _vp, _i64, _vp, _i, _i, _i, _vp, _vp]
    lib.camera_score_layer.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _vp, _vp, _i, _i, _i64, _vp, _vp, _i64,
                                       _vp, _i64, _f, _i, _vp, _vp, _vp, _vp]
    lib.camera_select_prune.argtypes = [_vp, _vp, _vp, _i64, _c.POINTER(_i64), _i, _d, _vp, _vp, _vp, _vp]
    lib.camera_select_prune_noalloc.argtypes = [_vp, _vp, _vp, _i64, _c.POINTER(_i64), _i, _d, _vp, _vp, _vp]
    lib.camera_select_prune_multi.argtypes = [_vp, _vp, _vp, _i64, _c.POINTER(_i64), _i, _i, _c.POINTER(_d), _vp, _vp]
    lib.camera_alloc_bits.argtypes = [_vp, _vp, _vp, _i64, _c.POINTER(_i64), _i, _i, _c.POINTER(_i),
                                      _c.POINTER(_d), _vp, _vp, _vp]
    lib.camera_rank_decisions.argtypes = [_vp, _vp, _vp, _i64, _c.POINTER(_i64), _i, _i, _c.POINTER(_d), _vp, _vp, _i,
                                          _c.POINTER(_i), _c.POINTER(_d), _vp, _vp, _vp]
    lib.camera_gather_micro_experts.argtypes = [_vp, _vp, _i, _i, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _i64,
                                                _i64, _vp, _i, _vp, _vp, _vp]
    lib.camera_input_channel_energy.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _vp, _i, _i, _vp]
    lib.camera_layer_forward.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _vp, _vp, _i, _i, _i64, _vp, _vp, _i64,
                                         _vp, _i64, _vp, _i, _vp]
    lib.camera_layer_forward_compact.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _vp, _vp, _i, _i, _i,
                                                 _c.POINTER(_c.c_int32), _i, _vp, _vp, _vp, _i, _vp]
    lib.camera_output_error.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp]
    lib.camera_token_logprobs.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _f, _vp, _i, _vp, _vp, _vp, _vp, _vp]
    lib.camera_token_logprobs_backward.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _f, _vp, _vp, _vp, _vp, _vp, _i, _vp, _i64]
    lib.camera_distill_topk.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _f, _vp, _vp, _i, _i, _vp, _vp]
    lib.camera_distill_topk_backward.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _f, _vp, _vp, _i, _vp, _vp, _i, _vp, _i64]
    lib.camera_gated_ffn.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _vp]
    lib.camera_gated_ffn_backward.argtypes = [_vp, _vp, _vp, _i, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _vp]
    lib.camera_profile_enable.argtypes = [_vp, _i]
    lib.camera_profile_read.argtypes = [_vp, _i, _c.POINTER(_d), _c.POINTER(_i64)]
    for name in EXPORTS:
        if name != "camera_last_error":
            getattr(lib, name).restype = _i
    return lib


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _require(cond: bool, message: str):
    """Layouts the library cannot see from a pointer and one stride: refuse them here instead of reading wrong bytes."""
    if not cond:
        raise CameraError(-2, message)


def _check_matrix(t, name: str, like=None):
    """[rows, cols] with unit inner stride (the row stride is passed on)."""
    if t is None:
        return
    if t.dim() != 2 or t.stride(1) != 1:
        _require(False, f"{name}: must be 2-D with unit inner stride (got strides {tuple(t.stride())})")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        _require(False, f"{name}: dtype / device differ from X")


def _check_experts(t, name: str, like=None):
    """[N_E, rows, cols] with contiguous rows exactly cols apart (the expert stride is passed on)."""
    if t is None:
        return
    _require(t.dim() == 3 and t.stride(2) == 1 and t.stride(1) == t.shape[2],
             f"{name}: must be [experts, rows, cols] with rows contiguous and cols apart (got strides {tuple(t.stride())})")
    if like is not None:
        _require(t.dtype == like.dtype and t.device == like.device, f"{name}: dtype / device differ from X")


def _check_flat(t, name: str, dtype=None, device=None):
    if t is None:
        return
    if not t.is_contiguous():
        _require(False, f"{name}: must be contiguous")
    if dtype is not None and t.dtype != dtype:
        _require(False, f"{name}: must be {dtype}")
    if device is not None and t.device != device:
        _require(False, f"{name}: on another device")


def _row_stride(t) -> int:
    """Elements between rows; a matrix of at most one row has none of its own (torch leaves any value there)."""
    return t.shape[1] if t.shape[0] <= 1 else t.stride(0)


# The current stream's handle by itself where torch has it: a Stream object around it takes 2 us, a sixth of a small call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(device) -> int:
    return _raw_stream(device.index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


class Camera:
    """One library context on one GPU.  Methods mirror the C entry points and
    allocate their outputs with torch on the context's device."""

    def __init__(self, device: int = 0, lib_path: str = LIB_PATH):
        self.lib = load_library(lib_path)
        self.device = torch.device("cuda", device)
        self._ctx = _vp()
        rc = self.lib.camera_create(_c.byref(self._ctx), device)
        if rc != 0:
            raise CameraError(rc, self.lib.camera_last_error(None).decode())

    def close(self):
        if getattr(self, "_ctx", None) is not None and self._ctx.value:
            self.lib.camera_destroy(self._ctx)
            self._ctx = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != 0:
            raise CameraError(rc, self.lib.camera_last_error(self._ctx).decode())

    @staticmethod
    def _check_layer(X, topk_idx, topk_w, W_gate, W_up, W_down):
        _check_matrix(X, "X")
        _check_experts(W_gate, "W_gate", like=X)
        _check_experts(W_up, "W_up", like=X)
        _check_experts(W_down, "W_down", like=X)
        _check_flat(topk_idx, "topk_idx", torch.int32, X.device)
        _check_flat(topk_w, "topk_w", torch.float32, X.device)
        if W_gate is not None and W_up is not None:
            _require(W_gate.shape == W_up.shape and W_gate.stride(0) == W_up.stride(0), "W_gate / W_up: shapes or expert strides differ")
        if W_gate is not None:
            _require(W_gate.shape[2] == X.shape[1], "W_gate: d_model differs from X")
        if W_gate is not None and W_down is not None:
            _require(W_down.shape[0] == W_gate.shape[0] and W_down.shape[1] == W_gate.shape[2] and W_down.shape[2] == W_gate.shape[1],
                     "W_down: must be [experts, d_model, d_ff]")

    # ---- entry points ------------------------------------------------------
    def route_topk(self, X, W_r, bias, top_k: int, renorm: bool = True):
        _check_matrix(X, "X")
        _check_matrix(W_r, "W_r", like=X)
        _check_flat(bias, "bias", torch.float32, X.device)
        n, d = X.shape
        n_experts = W_r.shape[0]
        idx = torch.empty((n, top_k), dtype=torch.int32, device=self.device)
        w = torch.empty((n, top_k), dtype=torch.float32, device=self.device)
        self._check(self.lib.camera_route_topk(
            self._ctx, _stream_handle(self.device), _ptr(X), _dtype_code(X), n, d, X.stride(0), _ptr(W_r),
            W_r.stride(0), _ptr(bias), n_experts, top_k, int(renorm), _ptr(idx), _ptr(w)))
        return idx, w

    def score_layer(self, X, topk_idx, topk_w, W_gate, W_up, W_down, alpha: float, flags: int = 0, out=None):
        """W_gate / W_up [N_E, d_ff, d_model], W_down [N_E, d_model, d_ff] (None with NO_FINALIZE).
        Returns dict(phi2, phi_inf, omega2, energy); pass `out` to reuse / accumulate into buffers."""
        self._check_layer(X, topk_idx, topk_w, W_gate, W_up, W_down)
        n, d = X.shape
        n_experts, d_ff, _ = W_gate.shape
        n_micro = n_experts * d_ff
        if out is not None:
            for k, v in out.items():
                _check_flat(v, k, torch.float32, X.device)
        if out is None:
            out = {k: torch.empty(n_micro, dtype=torch.float32, device=self.device)
                   for k in ("phi2", "phi_inf", "omega2", "energy")}
        top_k = 0 if topk_idx is None else topk_idx.shape[1]
        self._check(self.lib.camera_score_layer(
            self._ctx, _stream_handle(self.device), _ptr(X), _dtype_code(X), n, d, X.stride(0), _ptr(topk_idx),
            _ptr(topk_w), top_k, n_experts, d_ff, _ptr(W_gate), _ptr(W_up), W_gate.stride(0), _ptr(W_down),
            0 if W_down is None else W_down.stride(0), float(alpha), flags, _ptr(out["phi2"]), _ptr(out["phi_inf"]),
            _ptr(out.get("omega2")), _ptr(out.get("energy"))))
        return out

    def select_prune(self, energy, seg_offsets: Sequence[int], ratio: float, want_idx=False, want_rank=False):
        _check_flat(energy, "energy", torch.float32)
        n_micro = energy.numel()
        n_seg = len(seg_offsets) - 1
        seg = (_i64 * (n_seg + 1))(*seg_offsets)
        keep = torch.empty(n_micro, dtype=torch.uint8, device=self.device)
        per_expert = torch.empty(n_seg, dtype=torch.int32, device=self.device)
        # kept_idx is sized for the worst case; the caller trims it with per_expert.sum()
        kept_idx = torch.empty(n_micro, dtype=torch.int32, device=self.device) if want_idx else None
        rank = torch.empty(n_micro, dtype=torch.int32, device=self.device) if want_rank else None
        self._check(self.lib.camera_select_prune(
            self._ctx, _stream_handle(self.device), _ptr(energy), n_micro, seg, n_seg, float(ratio), _ptr(keep),
            _ptr(per_expert), _ptr(kept_idx), _ptr(rank)))
        return keep, per_expert, kept_idx, rank

    def select_prune_noalloc(self, energy, seg_offsets: Sequence[int], ratio: float, keep, per_expert, kept_idx=None):
        """camera_select_prune_noalloc: the caller brings every output (keep uint8 [n_micro], per_expert int32
        [n_seg], kept_idx int32 [>= kept] or None); the call itself allocates nothing on the device."""
        _check_flat(energy, "energy", torch.float32)
        _check_flat(keep, "keep", torch.uint8, energy.device)
        _check_flat(per_expert, "per_expert", torch.int32, energy.device)
        _check_flat(kept_idx, "kept_idx", torch.int32, energy.device)
        n_seg = len(seg_offsets) - 1
        seg = (_i64 * (n_seg + 1))(*seg_offsets)
        self._check(self.lib.camera_select_prune_noalloc(
            self._ctx, _stream_handle(self.device), _ptr(energy), energy.numel(), seg, n_seg, float(ratio), _ptr(keep),
            _ptr(per_expert), _ptr(kept_idx)))

    def select_prune_multi(self, energy, seg_offsets, ratios, out=None):
        """Masks at several rising ratios from one ranking pass: (keep_bits uint8 [n_micro] with bit k = kept at
        ratios[k], kept_per_expert int32 [len(ratios), n_seg])."""
        _check_flat(energy, "energy", torch.float32)
        n_micro = energy.numel()
        n_seg = len(seg_offsets) - 1
        seg = (_i64 * (n_seg + 1))(*seg_offsets)
        if out is None:
            out = (torch.empty(n_micro, dtype=torch.uint8, device=self.device),
                   torch.empty((len(ratios), n_seg), dtype=torch.int32, device=self.device))
        self._check(self.lib.camera_select_prune_multi(
            self._ctx, _stream_handle(self.device), _ptr(energy), n_micro, seg, n_seg, len(ratios),
            (_d * len(ratios))(*[float(r) for r in ratios]), _ptr(out[0]), _ptr(out[1])))
        return out

    def alloc_bits(self, energy, seg_offsets: Sequence[int], bits: Sequence[int], ratios: Sequence[float],
                   want_perm=False):
        _check_flat(energy, "energy", torch.float32)
        n_micro = energy.numel()
        n_seg = len(seg_offsets) - 1
        n_levels = len(bits)
        seg = (_i64 * (n_seg + 1))(*seg_offsets)
        bit_of = torch.empty(n_micro, dtype=torch.uint8, device=self.device)
        level_count = torch.empty((n_seg, n_levels), dtype=torch.int32, device=self.device)
        perm = torch.empty(n_micro, dtype=torch.int32, device=self.device) if want_perm else None
        self._check(self.lib.camera_alloc_bits(
            self._ctx, _stream_handle(self.device), _ptr(energy), n_micro, seg, n_seg, n_levels,
            (_i * n_levels)(*bits), (_d * len(ratios))(*ratios), _ptr(bit_of), _ptr(level_count), _ptr(perm)))
        return bit_of, level_count, perm

    def rank_decisions(self, energy, seg_offsets, prune_ratios, bits, level_ratios, want_perm=False, out=None):
        """The CAMERA-P masks at several rising ratios and one CAMERA-Q bit allocation from one pass over the
        ranking: (keep_bits, kept_per_expert [len(prune_ratios), n_seg], bit_of, level_count [n_seg, len(bits)], perm)."""
        _check_flat(energy, "energy", torch.float32)
        n_micro = energy.numel()
        n_seg = len(seg_offsets) - 1
        seg = (_i64 * (n_seg + 1))(*seg_offsets)
        if out is None:
            out = (torch.empty(n_micro, dtype=torch.uint8, device=self.device),
                   torch.empty((len(prune_ratios), n_seg), dtype=torch.int32, device=self.device),
                   torch.empty(n_micro, dtype=torch.uint8, device=self.device),
                   torch.empty((n_seg, len(bits)), dtype=torch.int32, device=self.device),
                   torch.empty(n_micro, dtype=torch.int32, device=self.device) if want_perm else None)
        self._check(self.lib.camera_rank_decisions(
            self._ctx, _stream_handle(self.device), _ptr(energy), n_micro, seg, n_seg, len(prune_ratios),
            (_d * len(prune_ratios))(*[float(r) for r in prune_ratios]), _ptr(out[0]), _ptr(out[1]), len(bits),
            (_i * len(bits))(*bits), (_d * len(level_ratios))(*[float(r) for r in level_ratios]), _ptr(out[2]), _ptr(out[3]),
            _ptr(out[4])))
        return out

    def gather_micro_experts(self, W_gate, W_up, W_down, index, count=None, index_base=0, out=None, down_row_align=1):
        """Kept gate / up rows and down columns of one group of experts (Algorithm 2, lines 10-13).
        W_gate, W_up [N_E, d_ff, d_model], W_down [N_E, d_model, d_ff] (any of them may be None: skipped);
        index int32 [n_index] global indices grouped by expert; count int32 [N_E] or None (d_ff each);
        down_row_align: the rows of every W_down block are padded with zeros to a multiple of it.
        Returns (gate_out [n_index, d_model], up_out, down_out flat: sized for the longest padding when
        allocated here, [d_model][ld(e)] blocks one after the other)."""
        ref = W_gate if W_gate is not None else (W_up if W_up is not None else W_down)
        for name, t in (("W_gate", W_gate), ("W_up", W_up), ("W_down", W_down)):
            _check_experts(t, name)
        _check_flat(index, "index", torch.int32, ref.device)
        _check_flat(count, "count", torch.int32, ref.device)
        n_experts = ref.shape[0]
        d_ff, d_model = (ref.shape[1], ref.shape[2]) if ref is not W_down else (ref.shape[2], ref.shape[1])
        n_index = index.numel()
        stride_gu = (W_gate if W_gate is not None else W_up).stride(0) if (W_gate is not None or W_up is not None) else 0
        if out is None:
            mk = lambda src, shape: None if src is None else torch.empty(shape, dtype=src.dtype, device=self.device)
            padded = n_index + n_experts * (int(down_row_align) - 1)
            out = (mk(W_gate, (n_index, d_model)), mk(W_up, (n_index, d_model)), mk(W_down, (padded * d_model,)))
        self._check(self.lib.camera_gather_micro_experts(
            self._ctx, _stream_handle(self.device), _dtype_code(ref), n_experts, d_ff, d_model, _ptr(W_gate), _ptr(W_up),
            stride_gu, _ptr(W_down), W_down.stride(0) if W_down is not None else 0, _ptr(index), n_index,
            int(index_base), _ptr(count), int(down_row_align), _ptr(out[0]), _ptr(out[1]), _ptr(out[2])))
        return out

    def input_channel_energy(self, X, topk_idx, n_experts: int, out=None):
        """h [n_experts, d_model] float32: per expert, the sum over its routed tokens of X[j, c]^2 (the statistic the
        column-wise comparison variant CAMERA-Q-dagger ranks the input channels of W_up / W_gate by)."""
        _check_matrix(X, "X")
        _check_flat(topk_idx, "topk_idx", torch.int32, X.device)
        n, d = X.shape
        if out is None:
            out = torch.empty((n_experts, d), dtype=torch.float32, device=self.device)
        _check_flat(out, "h", torch.float32, X.device)
        self._check(self.lib.camera_input_channel_energy(
            self._ctx, _stream_handle(self.device), _ptr(X), _dtype_code(X), n, d, X.stride(0), _ptr(topk_idx),
            0 if topk_idx is None else topk_idx.shape[1], int(n_experts), _ptr(out)))
        return out

    def layer_forward(self, X, topk_idx, topk_w, W_gate, W_up, W_down, keep_mask=None, Y=None, accumulate=False):
        """Layer output over the kept micro-experts of one group of experts (Eq. 1-2); Y float32 [n, d_model]."""
        self._check_layer(X, topk_idx, topk_w, W_gate, W_up, W_down)
        _check_flat(keep_mask, "keep_mask", torch.uint8, X.device)
        _check_flat(Y, "Y", torch.float32, X.device)
        n, d = X.shape
        n_experts, d_ff, _ = W_gate.shape
        top_k = 0 if topk_idx is None else topk_idx.shape[1]
        if Y is None:
            Y = torch.empty((n, d), dtype=torch.float32, device=self.device)
        self._check(self.lib.camera_layer_forward(
            self._ctx, _stream_handle(self.device), _ptr(X), _dtype_code(X), n, d, X.stride(0), _ptr(topk_idx),
            _ptr(topk_w), top_k, n_experts, d_ff, _ptr(W_gate), _ptr(W_up), W_gate.stride(0), _ptr(W_down),
            W_down.stride(0), _ptr(keep_mask), ACCUMULATE if accumulate else 0, _ptr(Y)))
        return Y

    def layer_forward_compact(self, X, topk_idx, topk_w, count, W_gate_c, W_up_c, W_down_c, n_shared=0,
                              down_row_align=1, Y=None, accumulate=False):
        """Layer output from compacted weights (the outputs of gather_micro_experts, with the same
        down_row_align); count: per-expert kept micro-experts as a sequence of Python ints, the last n_shared
        of them shared experts (every token, weight 1).  Y float32 [n, d_model]."""
        _check_matrix(X, "X")
        for name, t in (("W_gate_c", W_gate_c), ("W_up_c", W_up_c), ("W_down_c", W_down_c)):
            # (a dtype other than bf16 is the library's to refuse: it names what it supports)
            _check_flat(t, name, X.dtype if X.dtype == torch.bfloat16 else None, X.device)
        _check_flat(topk_idx, "topk_idx", torch.int32, X.device)
        _check_flat(topk_w, "topk_w", torch.float32, X.device)
        _check_flat(Y, "Y", torch.float32, X.device)
        n, d = X.shape
        counts = [int(c) for c in count]
        top_k = 0 if topk_idx is None else topk_idx.shape[1]
        if Y is None:
            Y = torch.empty((n, d), dtype=torch.float32, device=self.device)
        self._check(self.lib.camera_layer_forward_compact(
            self._ctx, _stream_handle(self.device), _ptr(X), _dtype_code(X), n, d, X.stride(0), _ptr(topk_idx),
            _ptr(topk_w), top_k, len(counts) - int(n_shared), int(n_shared), (_c.c_int32 * len(counts))(*counts),
            int(down_row_align), _ptr(W_gate_c), _ptr(W_up_c), _ptr(W_down_c), ACCUMULATE if accumulate else 0, _ptr(Y)))
        return Y

    def output_error(self, Y, Y_hat):
        """Per-token [n, 4]: ||y - y_hat||^2, ||y||^2, ||y_hat||^2, <y, y_hat>."""
        _check_flat(Y, "Y", torch.float32)
        _check_flat(Y_hat, "Y_hat", torch.float32, Y.device)
        n, d = Y.shape
        out = torch.empty((n, 4), dtype=torch.float32, device=self.device)
        self._check(self.lib.camera_output_error(self._ctx, _stream_handle(self.device), _ptr(Y), _ptr(Y_hat), n, d,
                                                 _ptr(out)))
        return out

    # ---- judging and repairing a pruned model ------------------------------
    def _check_here(self, t, name: str):
        if t.device != self.device:
            _require(False, f"{name}: on {t.device}, the context is on {self.device}")

    def _check_logits(self, logits, per_row=()):
        """Logits as a matrix, and float32 / int32 tensors with a value (or a fixed number of values) for every row of it."""
        _check_matrix(logits, "logits")
        self._check_here(logits, "logits")
        for t, name, dtype, shape in per_row:
            if t is None:
                continue
            _check_flat(t, name, dtype, logits.device)
            if t.shape != shape:
                _require(False, f"{name}: must be {list(shape)} (got {list(t.shape)})")

    def _gradient_rows(self, logits, dlogits, accumulate):
        if dlogits is None:
            _require(not accumulate, "accumulate: needs dlogits")
            return torch.empty(logits.shape, dtype=logits.dtype, device=self.device)
        _check_matrix(dlogits, "dlogits", like=logits)
        _require(dlogits.shape == logits.shape, "dlogits: shape differs from logits")
        return dlogits

    def token_logprobs(self, logits, targets=None, top_k: int = 0, temperature: float = 1.0):
        """Log probabilities of given tokens: logits [n, vocab] (bf16 / f32, unit inner stride, any row stride), targets int32 [n]
        (outside [0, vocab): no target there, log probability 0) or None.  Returns dict(logprob [n], entropy [n], stats [n, 2]) and,
        with top_k > 0, top_idx int32 [n, top_k] / top_logprob [n, top_k]: the most likely tokens, equal logits to the lower index,
        -1 where a masked row has fewer.  `logprob` is missing without targets; `stats` is what the backward call takes."""
        n = logits.shape[0]
        self._check_logits(logits, [(targets, "targets", torch.int32, (n,))])
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=self.device)  # noqa: E731
        out = {} if targets is None else {"logprob": new(n)}
        out.update(entropy=new(n), stats=new(n, 2))
        if top_k > 0:
            out.update(top_idx=new(n, top_k, dtype=torch.int32), top_logprob=new(n, top_k))
        self._check(self.lib.camera_token_logprobs(
            self._ctx, _stream_handle(self.device), _ptr(logits), _dtype_code(logits), n, logits.shape[1], _row_stride(logits),
            float(temperature), _ptr(targets), int(top_k), _ptr(out.get("logprob")), _ptr(out["entropy"]), _ptr(out["stats"]),
            _ptr(out.get("top_idx")), _ptr(out.get("top_logprob"))))
        return out

    def token_logprobs_backward(self, logits, targets, stats, grad_logprob=None, entropy=None, grad_entropy=None,
                                temperature: float = 1.0, dlogits=None, accumulate=False):
        """Gradient with respect to the logits of sum(grad_logprob * logprob) + sum(grad_entropy * entropy); stats and entropy as
        token_logprobs left them.  dlogits: written there (accumulate: added to it); it may be `logits` itself."""
        n = logits.shape[0]
        f32 = torch.float32
        self._check_logits(logits, [(targets, "targets", torch.int32, (n,)), (stats, "stats", f32, (n, 2)),
                                    (grad_logprob, "grad_logprob", f32, (n,)), (entropy, "entropy", f32, (n,)),
                                    (grad_entropy, "grad_entropy", f32, (n,))])
        dlogits = self._gradient_rows(logits, dlogits, accumulate)
        self._check(self.lib.camera_token_logprobs_backward(
            self._ctx, _stream_handle(self.device), _ptr(logits), _dtype_code(logits), n, logits.shape[1], _row_stride(logits),
            float(temperature), _ptr(targets), _ptr(stats), _ptr(entropy), _ptr(grad_logprob), _ptr(grad_entropy),
            ACCUMULATE if accumulate else 0, _ptr(dlogits), _row_stride(dlogits)))
        return dlogits

    def distill_topk(self, logits, teacher_idx, teacher_logprob, temperature: float = 1.0, tail=False):
        """Kullback-Leibler divergence of softmax(logits / temperature) from a teacher of which the most likely tokens are known:
        teacher_idx int32 [n, k], teacher_logprob [n, k] (top_idx and top_logprob of token_logprobs on the teacher's logits).
        tail: the tokens that the teacher does not list are one more class (teacher_logprob taken at this temperature); else the
        teacher's distribution is softmax(teacher_logprob / temperature) over the listed ones: logits, or log probabilities at temperature
        1, since here they are divided by the temperature.  Returns dict(loss [n], stats [n, 5])."""
        n = logits.shape[0]
        k = teacher_idx.shape[-1]
        self._check_logits(logits, [(teacher_idx, "teacher_idx", torch.int32, (n, k)),
                                    (teacher_logprob, "teacher_logprob", torch.float32, (n, k))])
        out = {"loss": torch.empty(n, dtype=torch.float32, device=self.device),
               "stats": torch.empty((n, DISTILL_STATS), dtype=torch.float32, device=self.device)}
        self._check(self.lib.camera_distill_topk(
            self._ctx, _stream_handle(self.device), _ptr(logits), _dtype_code(logits), n, logits.shape[1], _row_stride(logits),
            float(temperature), _ptr(teacher_idx), _ptr(teacher_logprob), k, DISTILL_TAIL if tail else 0, _ptr(out["loss"]),
            _ptr(out["stats"])))
        return out

    def distill_topk_backward(self, logits, teacher_idx, teacher_logprob, stats, grad_loss, temperature: float = 1.0, tail=False,
                              dlogits=None, accumulate=False):
        """Gradient with respect to the logits of sum(grad_loss * loss); stats as distill_topk left them, the other arguments as it
        had them.  dlogits: written there (accumulate: added to it); it may be `logits` itself."""
        n = logits.shape[0]
        k = teacher_idx.shape[-1]
        self._check_logits(logits, [(teacher_idx, "teacher_idx", torch.int32, (n, k)),
                                    (teacher_logprob, "teacher_logprob", torch.float32, (n, k)),
                                    (stats, "stats", torch.float32, (n, DISTILL_STATS)), (grad_loss, "grad_loss", torch.float32, (n,))])
        dlogits = self._gradient_rows(logits, dlogits, accumulate)
        self._check(self.lib.camera_distill_topk_backward(
            self._ctx, _stream_handle(self.device), _ptr(logits), _dtype_code(logits), n, logits.shape[1], _row_stride(logits),
            float(temperature), _ptr(teacher_idx), _ptr(teacher_logprob), k, _ptr(stats), _ptr(grad_loss),
            (ACCUMULATE if accumulate else 0) | (DISTILL_TAIL if tail else 0), _ptr(dlogits), _row_stride(dlogits)))
        return dlogits

    def _check_gated(self, X, W_gate, W_up):
        _check_matrix(X, "X")
        self._check_here(X, "X")
        for t, name in ((W_gate, "W_gate"), (W_up, "W_up")):
            _check_matrix(t, name, like=X)
            _check_flat(t, name)
            _require(t.shape[1] == X.shape[1], f"{name}: d_model differs from X")
        _require(W_gate.shape == W_up.shape, "W_gate / W_up: shapes differ")

    def gated_ffn(self, X, W_gate, W_up, want_pre=False, H=None):
        """H [n, d_ff] = silu(X W_gate^T) * (X W_up^T) for the micro-experts of one expert: X [n, d_model], W_gate, W_up
        [d_ff, d_model].  want_pre: returns (H, pre), pre [n, 2, P] float32 the two projections that the backward call takes.
        H allocated here has rows of a whole number of 16-byte vectors (a view of the first d_ff columns).  In a given H the columns
        from d_ff to the next whole vector are set to zero."""
        self._check_gated(X, W_gate, W_up)
        n, d_ff = X.shape[0], W_gate.shape[0]
        v = 16 // X.element_size()
        whole = (d_ff + v - 1) // v * v
        if H is None:
            H = torch.empty((n, whole), dtype=X.dtype, device=self.device)[:, :d_ff]
        else:
            _check_matrix(H, "H", like=X)
            _require(tuple(H.shape) == (n, d_ff), "H: must be [n, d_ff]")
            end = H.storage_offset() + (n - 1) * H.stride(0) + whole
            _require(n == 0 or end * H.element_size() <= H.untyped_storage().nbytes(), "H: its last row ends inside a 16-byte vector")
        pre = torch.empty((n, 2, (d_ff + 7) // 8 * 8), dtype=torch.float32, device=self.device) if want_pre else None
        self._check(self.lib.camera_gated_ffn(
            self._ctx, _stream_handle(self.device), _ptr(X), _dtype_code(X), n, X.shape[1], _row_stride(X), _ptr(W_gate), _ptr(W_up),
            d_ff, _ptr(H), H.stride(0) if n > 1 else whole, _ptr(pre)))  # a single row has no stride
        return (H, pre) if want_pre else H

    def gated_ffn_backward(self, X, W_gate, W_up, dH, pre=None, want=(True, True, True)):
        """(dX, dW_gate, dW_up) from dH [n, d_ff]; pre as gated_ffn left it, or None: the projections are computed again.  want:
        which of the three (None in the place of the others)."""
        self._check_gated(X, W_gate, W_up)
        n, d_ff = X.shape[0], W_gate.shape[0]
        _check_matrix(dH, "dH", like=X)
        _require(tuple(dH.shape) == (n, d_ff), "dH: must be [n, d_ff]")
        if pre is not None:
            _check_flat(pre, "pre", torch.float32, X.device)
            _require(tuple(pre.shape) == (n, 2, (d_ff + 7) // 8 * 8), "pre: must be as gated_ffn returned it")
        new = lambda like, wanted: torch.empty(like.shape, dtype=X.dtype, device=self.device) if wanted else None  # noqa: E731
        dX, dW_gate, dW_up = new(X, want[0]), new(W_gate, want[1]), new(W_up, want[2])
        self._check(self.lib.camera_gated_ffn_backward(
            self._ctx, _stream_handle(self.device), _ptr(X), _dtype_code(X), n, X.shape[1], _row_stride(X), _ptr(W_gate), _ptr(W_up),
            d_ff, _ptr(pre), _ptr(dH), _row_stride(dH), _ptr(dX), X.shape[1], _ptr(dW_gate), _ptr(dW_up)))
        return dX, dW_gate, dW_up

    # ---- profiling ---------------------------------------------------------
    def profile_enable(self, on: bool):
        self._check(self.lib.camera_profile_enable(self._ctx, int(on)))

    def profile_read(self, kernel_id: int):
        ms, count = _d(), _i64()
        self._check(self.lib.camera_profile_read(self._ctx, kernel_id, _c.byref(ms), _c.byref(count)))
        return ms.value, count.value
