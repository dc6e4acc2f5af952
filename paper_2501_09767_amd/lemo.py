"""Thin binding over the C-ABI HIP library (include/lemo.h).  Argument marshalling only, of the most frequent calls in native code
(csrc/native.cpp) where they are plain.

Every function takes torch tensors that live on the GPU, passes their ``data_ptr()`` and the current
HIP stream to the library call of the same name, and raises ``LemoError`` on a negative return code.
No arithmetic of the method happens here, and there is NO fallback: if ``liblemo_hip.so`` has not
been built the import of this module fails.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import warnings
from typing import NamedTuple, Optional

import torch

F32, BF16 = 0, 1
CAUSAL, EXCLUDE_SELF = 1, 2
SCATTER_ACCUMULATE, SCATTER_ZERO_PAD = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblemo_hip.so")
NATIVE_PATH = os.path.join(_HERE, "lemo_native.so")

EXPORTS = ("lemo_strerror", "lemo_keep_k", "lemo_kept_count", "lemo_score_workspace_bytes",
           "lemo_score_segments", "lemo_score_segments_static", "lemo_score_rowstats", "lemo_score_colsums", "lemo_score_head_mean",
           "lemo_select_topk", "lemo_head_mean_select_topk", "lemo_launch_floor", "lemo_probe_sweep_issue_mix", "lemo_gather_gemm", "lemo_gather_gemm_add", "lemo_scatter_grad",
           "lemo_score_blocks_workspace_bytes", "lemo_score_blocks", "lemo_threshold_init", "lemo_select_threshold",
           "lemo_kept_attention_workspace_bytes", "lemo_kept_attention",
           "lemo_gather_gemm_dw_workspace_bytes", "lemo_gather_gemm_dw", "lemo_gather_gemm_dx",
           "lemo_norm_residual", "lemo_norm_residual_grad_workspace_bytes", "lemo_norm_residual_grad",
           "lemo_block_means", "lemo_select_blocks", "lemo_block_attention_workspace_bytes", "lemo_block_attention",
           "lemo_block_attention_grad_workspace_bytes", "lemo_block_attention_grad", "lemo_block_means_step", "lemo_select_blocks_step",
           "lemo_block_attention_step_workspace_bytes", "lemo_block_attention_step")


class LemoError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {_lib.lemo_strerror(code).decode()} ({code})")


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_2501_09767_amd.build). "
                          "There is no CPU fallback for the hot path.")
    lib = ctypes.CDLL(LIB_PATH)
    i64, i32, u32, vp, f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32, ctypes.c_void_p, ctypes.c_float
    lib.lemo_strerror.restype = ctypes.c_char_p
    lib.lemo_strerror.argtypes = [ctypes.c_int]
    lib.lemo_keep_k.restype = i32
    lib.lemo_keep_k.argtypes = [i32, ctypes.c_double]
    lib.lemo_kept_count.restype = i64
    lib.lemo_kept_count.argtypes = [i64, i32, i32]
    lib.lemo_score_workspace_bytes.restype = ctypes.c_int
    lib.lemo_score_workspace_bytes.argtypes = [i64, i32, i32, i32, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
    lib.lemo_score_segments.restype = ctypes.c_int
    lib.lemo_score_segments.argtypes = [vp, vp, i64, i32, i32, i32, ctypes.c_int, i64, i64, i64, i64, f32, i32, u32,
                                        vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.lemo_score_segments_static.restype = ctypes.c_int
    lib.lemo_score_segments_static.argtypes = [vp, vp, i64, i32, i32, i32, ctypes.c_int, i64, i64, i64, i64, f32, i32, u32, vp, vp]
    lib.lemo_score_rowstats.restype = ctypes.c_int
    lib.lemo_score_rowstats.argtypes = [vp, vp, i64, i32, i32, i32, ctypes.c_int, i64, i64, i64, i64, f32, u32, vp, vp]
    lib.lemo_score_colsums.restype = ctypes.c_int
    lib.lemo_score_colsums.argtypes = [vp, vp, i64, i32, i32, i32, ctypes.c_int, i64, i64, i64, i64, f32, i32, u32, vp, vp, vp, vp]
    lib.lemo_score_head_mean.restype = ctypes.c_int
    lib.lemo_score_head_mean.argtypes = [vp, vp, i64, i32, u32, vp, vp]
    lib.lemo_score_blocks_workspace_bytes.restype = ctypes.c_int
    lib.lemo_score_blocks_workspace_bytes.argtypes = [i64, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.lemo_score_blocks.restype = ctypes.c_int
    lib.lemo_score_blocks.argtypes = [vp, vp, i64, i32, i32, i32, ctypes.c_int, i64, i64, i64, i64, f32, i32, u32, i32,
                                      vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.lemo_threshold_init.restype = ctypes.c_int
    lib.lemo_threshold_init.argtypes = [vp, i64, vp, vp]
    lib.lemo_select_threshold.restype = ctypes.c_int
    lib.lemo_select_threshold.argtypes = [vp, i64, i32, f32, vp, vp, vp, vp]
    lib.lemo_kept_attention_workspace_bytes.restype = ctypes.c_int
    lib.lemo_kept_attention_workspace_bytes.argtypes = [i64, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.lemo_kept_attention.restype = ctypes.c_int
    lib.lemo_kept_attention.argtypes = [vp, vp, vp, i64, i32, i32, i32, ctypes.c_int, i64, i64, i64, i64, i64, i64, vp, i64, f32, u32,
                                        vp, i64, i64, vp, ctypes.c_size_t, vp]
    lib.lemo_gather_gemm_dw_workspace_bytes.restype = ctypes.c_int
    lib.lemo_gather_gemm_dw_workspace_bytes.argtypes = [i64, i32, i32, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
    lib.lemo_gather_gemm_dw.restype = ctypes.c_int
    lib.lemo_gather_gemm_dw.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp, i64, i32, i32, ctypes.c_int, vp, ctypes.c_size_t, vp]
    lib.lemo_head_mean_select_topk.restype = ctypes.c_int
    lib.lemo_head_mean_select_topk.argtypes = [vp, vp, i64, i32, u32, i32, i32, vp, vp, vp]
    lib.lemo_launch_floor.restype = ctypes.c_int
    lib.lemo_launch_floor.argtypes = [vp]
    lib.lemo_probe_sweep_issue_mix.restype = ctypes.c_int
    lib.lemo_probe_sweep_issue_mix.argtypes = [i32, u32, vp, ctypes.POINTER(i32), vp]
    lib.lemo_gather_gemm_dx.restype = ctypes.c_int
    lib.lemo_gather_gemm_dx.argtypes = [vp, i64, i64, vp, i64, vp, i64, i64, vp, i32, i32, ctypes.c_int, vp]
    lib.lemo_select_topk.restype = ctypes.c_int
    lib.lemo_select_topk.argtypes = [vp, i64, i32, i32, vp, vp]
    lib.lemo_gather_gemm.restype = ctypes.c_int
    lib.lemo_gather_gemm.argtypes = [vp, i64, i64, vp, i64, vp, i64, vp, vp, i64, i32, i32, ctypes.c_int, vp]
    lib.lemo_gather_gemm_add.restype = ctypes.c_int
    lib.lemo_gather_gemm_add.argtypes = [vp, i64, i64, vp, i64, vp, i64, vp, vp, i64, i64, vp, i32, i32, ctypes.c_int, vp]
    lib.lemo_scatter_grad.restype = ctypes.c_int
    lib.lemo_scatter_grad.argtypes = [vp, i64, vp, i64, vp, i64, i64, i32, ctypes.c_int, ctypes.c_int, i32, vp]
    lib.lemo_norm_residual.restype = ctypes.c_int
    lib.lemo_norm_residual.argtypes = [vp, i64, vp, i64, vp, i64, i64, vp, i64, vp, vp, i32, vp, vp, i32, f32, f32, f32, vp, i64, vp, i32, ctypes.c_int,
                                       u32, vp]
    lib.lemo_norm_residual_grad_workspace_bytes.restype = ctypes.c_int
    lib.lemo_norm_residual_grad_workspace_bytes.argtypes = [i64, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.lemo_norm_residual_grad.restype = ctypes.c_int
    lib.lemo_norm_residual_grad.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, i32, vp, i32, f32, f32, vp, vp, i64, vp, i64,
                                            vp, vp, vp, vp, vp, i32, ctypes.c_int, u32, vp, ctypes.c_size_t, vp]
    size = ctypes.POINTER(ctypes.c_size_t)
    kinds = {"p": vp, "l": i64, "i": i32, "f": f32, "u": u32, "z": ctypes.c_size_t, "s": size}
    for name, args in (("block_means", "pliiillipp"), ("select_blocks", "pliiiillplliiiupp"), ("block_attention_workspace_bytes", "lliiiiiis"),
                       ("block_attention", "pppll" "iiii" "llllll" "piiil" "fu" "pllp" "pzp"), ("block_attention_grad_workspace_bytes", "lliiiiiis"),
                       ("block_attention_grad", "pppppp" "ll" "iiii" "llllllllll" "piiil" "fu" "ppp" "pzp"), ("block_means_step", "piliiilllpipp"),
                       ("select_blocks_step", "piiiiillplpiipp"), ("block_attention_step_workspace_bytes", "iiiiiis"),
                       ("block_attention_step", "pppil" "iiii" "llllllll" "ppii" "f" "pll" "pzp")):
        fn = getattr(lib, "lemo_" + name)
        fn.restype = ctypes.c_int
        fn.argtypes = [kinds[k] for k in args]
    return lib


_lib = _load()


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"expected float32 or bfloat16, got {t.dtype}")


def _dev(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("tensors must live on the GPU")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    # the current stream of the current device, without the Stream object that torch.cuda.current_stream() builds around it
    # (0.3 us instead of 2.9, of about 9 us that a call of a small layer takes on the host); the function is not part of
    # torch's public interface, so a torch without it takes the public way
    if _raw_stream is None:
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))


class _NoNative:
    """In the place of the native module: every call goes the long way."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_native():
    # csrc/native.cpp: the calls that a layer makes over and over, in the plain case, without the steps in Python below; anything
    # else it leaves to them (it answers None and has done nothing).  backward of a small binary32 layer, three calls: 22 us
    # enqueued from Python, 9.6 so.  It is bound to the torch it was built with; the steps in Python need liblemo_hip.so alone.
    try:
        loader = importlib.machinery.ExtensionFileLoader("lemo_native", NATIVE_PATH)
        module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("lemo_native", NATIVE_PATH, loader=loader))
        loader.exec_module(module)
        if module.torch_version != torch.__version__:
            raise ImportError(f"built with torch {module.torch_version}, not {torch.__version__}")
    except ImportError as e:
        warnings.warn(f"{NATIVE_PATH} is not used ({e}): calls are marshalled in Python.  python -m paper_2501_09767_amd.build makes it.", RuntimeWarning)
        return _NoNative()
    if _raw_stream is not None:
        module.set_stream_source(torch.cuda.current_device, _raw_stream)
    return module


_native = _load_native()


def _check(rc: int, what: str):
    if rc != 0:
        raise LemoError(rc, what)


# --------------------------------------------------------------------------------- host helpers

def lemo_keep_k(L: int, ratio: float) -> int:
    return int(_lib.lemo_keep_k(L, ratio))


def lemo_kept_count(S: int, L: int, k: int) -> int:
    return int(_lib.lemo_kept_count(S, L, k))


def lemo_score_workspace_bytes(S: int, H: int, H_kv: int, d: int, dtype: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.lemo_score_workspace_bytes(S, H, H_kv, d, dtype, ctypes.byref(n)), "lemo_score_workspace_bytes")
    return int(n.value)


# --------------------------------------------------------------------------------- the four calls

def lemo_score_segments(Q: torch.Tensor, K: torch.Tensor, L: int, flags: int = CAUSAL | EXCLUDE_SELF,
                        scale: float = 0.0, scores: Optional[torch.Tensor] = None,
                        colsum_per_head: Optional[torch.Tensor] = None, diag_per_head: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Q [S,H,d], K [S,H_kv,d] (last dim contiguous) -> scores [S] float32."""
    rc = _native.score_segments(Q, K, L, flags, scale, scores, colsum_per_head, diag_per_head, workspace)
    if rc is not None:
        _check(rc, "lemo_score_segments")
        return scores
    _dev(Q, K, scores, colsum_per_head, diag_per_head, workspace)
    if Q.dim() != 3 or K.dim() != 3 or Q.stride(2) != 1 or K.stride(2) != 1:
        raise ValueError("Q must be [S,H,d] and K [S,H_kv,d] with head_dim contiguous")
    S, H, d = Q.shape
    if K.shape[0] != S or K.shape[2] != d or _dt(K) != _dt(Q):
        raise ValueError("Q/K mismatch")
    Hkv = K.shape[1]
    if scores is None:
        scores = torch.empty(S, dtype=torch.float32, device=Q.device)
    need = lemo_score_workspace_bytes(S, H, Hkv, d, _dt(Q))
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=Q.device)
    for o, shape in ((scores, (S,)), (colsum_per_head, (H, S)), (diag_per_head, (H, S))):
        if o is not None and (o.dtype != torch.float32 or tuple(o.shape) != shape or not o.is_contiguous()):
            raise ValueError("output tensors must be contiguous float32 of shape [S] / [H,S]")
    _check(_lib.lemo_score_segments(_ptr(Q), _ptr(K), S, H, Hkv, d, _dt(Q), Q.stride(0), Q.stride(1), K.stride(0),
                                    K.stride(1), float(scale), int(L), int(flags), _ptr(scores), _ptr(colsum_per_head),
                                    _ptr(diag_per_head), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                    _stream()), "lemo_score_segments")
    return scores


def lemo_score_segments_static(Q: torch.Tensor, K: torch.Tensor, L: int, scores: torch.Tensor,
                               flags: int = CAUSAL | EXCLUDE_SELF, scale: float = 0.0) -> torch.Tensor:
    """lemo_score_segments without a workspace (the library's built-in scratch; H*S <= 2**20).  Allocates nothing:
    `scores` [S] float32 must be passed in."""
    a = _qk_args(Q, K)
    _dev(scores)
    if scores.dtype != torch.float32 or tuple(scores.shape) != (a[2],) or not scores.is_contiguous():
        raise ValueError("scores must be contiguous float32 [S]")
    _check(_lib.lemo_score_segments_static(*a, float(scale), int(L), int(flags), _ptr(scores), _stream()),
           "lemo_score_segments_static")
    return scores


def _qk_args(Q: torch.Tensor, K: torch.Tensor):
    _dev(Q, K)
    if Q.dim() != 3 or K.dim() != 3 or Q.stride(2) != 1 or K.stride(2) != 1:
        raise ValueError("Q must be [S,H,d] and K [S,H_kv,d] with head_dim contiguous")
    S, H, d = Q.shape
    if K.shape[0] != S or K.shape[2] != d or _dt(K) != _dt(Q):
        raise ValueError("Q/K mismatch")
    return (_ptr(Q), _ptr(K), S, H, K.shape[1], d, _dt(Q), Q.stride(0), Q.stride(1), K.stride(0), K.stride(1))


def _plane(t: Optional[torch.Tensor], H: int, S: int, device) -> torch.Tensor:
    if t is None:
        return torch.empty((H, S), dtype=torch.float32, device=device)
    _dev(t)
    if t.dtype != torch.float32 or tuple(t.shape) != (H, S) or not t.is_contiguous():
        raise ValueError("per-head planes must be contiguous float32 [H,S]")
    return t


def lemo_score_rowstats(Q: torch.Tensor, K: torch.Tensor, flags: int = CAUSAL | EXCLUDE_SELF, scale: float = 0.0,
                        lse2: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Sweep 1 of the scoring: base-2 log-sum-exp of every query row -> [H,S] float32."""
    a = _qk_args(Q, K)
    lse2 = _plane(lse2, a[3], a[2], Q.device)
    _check(_lib.lemo_score_rowstats(*a, float(scale), int(flags), _ptr(lse2), _stream()), "lemo_score_rowstats")
    return lse2


def lemo_score_colsums(Q: torch.Tensor, K: torch.Tensor, L: int, lse2: torch.Tensor, flags: int = CAUSAL | EXCLUDE_SELF,
                       scale: float = 0.0, colsum_per_head: Optional[torch.Tensor] = None,
                       diag_per_head: Optional[torch.Tensor] = None):
    """Sweep 2 of the scoring: per-head column sums and diagonal -> two [H,S] float32 tensors."""
    a = _qk_args(Q, K)
    lse2 = _plane(lse2, a[3], a[2], Q.device)
    col = _plane(colsum_per_head, a[3], a[2], Q.device)
    dg = _plane(diag_per_head, a[3], a[2], Q.device)
    _check(_lib.lemo_score_colsums(*a, float(scale), int(L), int(flags), _ptr(lse2), _ptr(col), _ptr(dg), _stream()),
           "lemo_score_colsums")
    return col, dg


def lemo_score_head_mean(colsum_per_head: torch.Tensor, diag_per_head: torch.Tensor, flags: int = CAUSAL | EXCLUDE_SELF,
                         scores: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Head mean of (column sums - [EXCLUDE_SELF] diagonal) -> scores [S] float32."""
    H, S = colsum_per_head.shape
    col = _plane(colsum_per_head, H, S, colsum_per_head.device)
    dg = _plane(diag_per_head, H, S, colsum_per_head.device)
    if scores is None:
        scores = torch.empty(S, dtype=torch.float32, device=col.device)
    elif scores.dtype != torch.float32 or tuple(scores.shape) != (S,) or not scores.is_contiguous() or not scores.is_cuda:
        raise ValueError("scores must be contiguous float32 [S] on the GPU")
    _check(_lib.lemo_score_head_mean(_ptr(col), _ptr(dg), S, H, int(flags), _ptr(scores), _stream()), "lemo_score_head_mean")
    return scores


BLOCKS_PROBABILITIES, BLOCKS_POSITIVE_LOGITS = 0, 1


def lemo_score_blocks_workspace_bytes(S: int, H: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.lemo_score_blocks_workspace_bytes(S, H, ctypes.byref(n)), "lemo_score_blocks_workspace_bytes")
    return int(n.value)


def lemo_score_blocks(Q: torch.Tensor, K: torch.Tensor, b: int, flags: int = CAUSAL | EXCLUDE_SELF, scale: float = 0.0,
                      mode: int = BLOCKS_PROBABILITIES, lse2: Optional[torch.Tensor] = None, want_score_blocks: bool = True,
                      score_blocks: Optional[torch.Tensor] = None, token_blocks: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None):
    """Block-wise informativeness -> (score_blocks [nb,nb] float32 or None, token_blocks [nb] float32), nb = ceil(S/b)."""
    a = _qk_args(Q, K)
    S, H = a[2], a[3]
    nb = (S + b - 1) // b if b > 0 else 0
    if lse2 is not None:
        lse2 = _plane(lse2, H, S, Q.device)
    if score_blocks is None and want_score_blocks:
        score_blocks = torch.empty((nb, nb), dtype=torch.float32, device=Q.device)
    if token_blocks is None:
        token_blocks = torch.empty(nb, dtype=torch.float32, device=Q.device)
    for o, shape in ((score_blocks, (nb, nb)), (token_blocks, (nb,))):
        if o is not None:
            _dev(o)
            if o.dtype != torch.float32 or tuple(o.shape) != shape or not o.is_contiguous():
                raise ValueError("score_blocks / token_blocks must be contiguous float32 [nb,nb] / [nb]")
    if workspace is None:
        workspace = torch.empty(lemo_score_blocks_workspace_bytes(S, H), dtype=torch.uint8, device=Q.device)
    _dev(workspace)
    _check(_lib.lemo_score_blocks(*a, float(scale), int(b), int(flags), int(mode), _ptr(lse2), _ptr(score_blocks), _ptr(token_blocks),
                                  _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()), "lemo_score_blocks")
    return score_blocks, token_blocks


def lemo_threshold_init(token_blocks: torch.Tensor, threshold: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Mean token-block score (Alg. 1 step 1) -> float32 [1] on the GPU."""
    _dev(token_blocks, threshold)
    if token_blocks.dtype != torch.float32 or token_blocks.dim() != 1 or not token_blocks.is_contiguous():
        raise ValueError("token_blocks must be contiguous float32 [nb]")
    if threshold is None:
        threshold = torch.empty(1, dtype=torch.float32, device=token_blocks.device)
    elif threshold.dtype != torch.float32 or threshold.numel() != 1:
        raise ValueError("threshold must be one float32")
    _check(_lib.lemo_threshold_init(_ptr(token_blocks), token_blocks.numel(), _ptr(threshold), _stream()), "lemo_threshold_init")
    return threshold


def lemo_select_threshold(token_blocks: torch.Tensor, S: int, b: int, threshold, kept_idx: Optional[torch.Tensor] = None,
                          kept_count: Optional[torch.Tensor] = None):
    """Tokens of the blocks with score >= threshold (a float, or a float32 GPU tensor of one element)
    -> (kept_idx int32 [S], of which the first kept_count[0] entries are valid, kept_count int32 [1])."""
    _dev(token_blocks, kept_idx, kept_count)
    if token_blocks.dtype != torch.float32 or token_blocks.dim() != 1 or not token_blocks.is_contiguous() \
            or (b > 0 and token_blocks.numel() != (S + b - 1) // b):
        raise ValueError("token_blocks must be contiguous float32 [ceil(S/b)]")
    if kept_idx is None:
        kept_idx = torch.empty(S, dtype=torch.int32, device=token_blocks.device)
    elif kept_idx.dtype != torch.int32 or kept_idx.numel() < S or not kept_idx.is_contiguous():
        raise ValueError("kept_idx must be contiguous int32 with room for S entries")
    if kept_count is None:
        kept_count = torch.empty(1, dtype=torch.int32, device=token_blocks.device)
    elif kept_count.dtype != torch.int32 or kept_count.numel() != 1:
        raise ValueError("kept_count must be one int32")
    t_dev = None
    t_host = 0.0
    if isinstance(threshold, torch.Tensor):
        _dev(threshold)
        if threshold.dtype != torch.float32 or threshold.numel() != 1:
            raise ValueError("a device threshold must be one float32")
        t_dev = threshold
    else:
        t_host = float(threshold)
    _check(_lib.lemo_select_threshold(_ptr(token_blocks), int(S), int(b), t_host, _ptr(t_dev), _ptr(kept_idx), _ptr(kept_count),
                                      _stream()), "lemo_select_threshold")
    return kept_idx, kept_count


def lemo_select_topk(scores: torch.Tensor, L: int, k: int, kept_idx: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scores [S] float32 -> kept_idx [M] int32, ascending."""
    rc = _native.select_topk(scores, L, k, kept_idx)
    if rc is not None:
        _check(rc, "lemo_select_topk")
        return kept_idx
    _dev(scores, kept_idx)
    if scores.dtype != torch.float32 or scores.dim() != 1 or not scores.is_contiguous():
        raise ValueError("scores must be contiguous float32 [S]")
    S = scores.shape[0]
    M = lemo_kept_count(S, L, k)
    if M < 0:
        raise LemoError(-2, "lemo_kept_count")
    if kept_idx is None:
        kept_idx = torch.empty(M, dtype=torch.int32, device=scores.device)
    elif kept_idx.dtype != torch.int32 or kept_idx.numel() != M or not kept_idx.is_contiguous():
        raise ValueError("kept_idx must be contiguous int32 [M]")
    _check(_lib.lemo_select_topk(_ptr(scores), S, int(L), int(k), _ptr(kept_idx), _stream()), "lemo_select_topk")
    return kept_idx


def lemo_head_mean_select_topk(colsum_per_head: torch.Tensor, diag_per_head: torch.Tensor, L: int, k: int,
                               flags: int = CAUSAL | EXCLUDE_SELF, scores: Optional[torch.Tensor] = None,
                               kept_idx: Optional[torch.Tensor] = None):
    """Head mean + per-segment top-k in one launch -> (scores [S] float32, kept_idx [M] int32)."""
    H, S = colsum_per_head.shape
    col = _plane(colsum_per_head, H, S, colsum_per_head.device)
    dg = _plane(diag_per_head, H, S, colsum_per_head.device)
    M = lemo_kept_count(S, L, k)
    if M < 0:
        raise LemoError(-2, "lemo_kept_count")
    if scores is None:
        scores = torch.empty(S, dtype=torch.float32, device=col.device)
    elif scores.dtype != torch.float32 or tuple(scores.shape) != (S,) or not scores.is_contiguous() or not scores.is_cuda:
        raise ValueError("scores must be contiguous float32 [S] on the GPU")
    if kept_idx is None:
        kept_idx = torch.empty(M, dtype=torch.int32, device=col.device)
    elif kept_idx.dtype != torch.int32 or kept_idx.numel() != M or not kept_idx.is_contiguous() or not kept_idx.is_cuda:
        raise ValueError("kept_idx must be contiguous int32 [M] on the GPU")
    _check(_lib.lemo_head_mean_select_topk(_ptr(col), _ptr(dg), S, H, int(flags), int(L), int(k), _ptr(scores), _ptr(kept_idx), _stream()),
           "lemo_head_mean_select_topk")
    return scores, kept_idx


def lemo_launch_floor() -> None:
    """One empty kernel on the current stream (measurement aid)."""
    _check(_lib.lemo_launch_floor(_stream()), "lemo_launch_floor")


def lemo_probe_sweep_issue_mix(tiles_per_wave: int, sink: torch.Tensor, operand_seed: int = 0) -> int:
    """Enqueue the register-only instruction mix of the scoring sweeps (measurement aid) -> wavefronts launched.
    operand_seed 0: constant operands; non-zero: pseudo-random operands that change from MFMA to MFMA."""
    _dev(sink)
    if sink.dtype != torch.float32 or sink.numel() < 1:
        raise ValueError("sink must hold one float32")
    waves = ctypes.c_int32(0)
    _check(_lib.lemo_probe_sweep_issue_mix(int(tiles_per_wave), int(operand_seed) & 0xffffffff, _ptr(sink), ctypes.byref(waves), _stream()), "lemo_probe_sweep_issue_mix")
    return int(waves.value)


def lemo_gather_gemm(X: torch.Tensor, kept_idx: Optional[torch.Tensor], W: torch.Tensor,
                     bias: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
                     M: Optional[int] = None) -> torch.Tensor:
    """Y[m,:] = X[kept_idx[m],:] @ W.T (+ bias).  X [S,C], W [N,C], rows contiguous."""
    rc = _native.gather_gemm(X, kept_idx, W, bias, Y, M)
    if rc is not None:
        _check(rc, "lemo_gather_gemm")
        return Y
    _dev(X, kept_idx, W, bias, Y)
    if X.dim() != 2 or W.dim() != 2 or X.stride(1) != 1 or W.stride(1) != 1 or X.shape[1] != W.shape[1] or _dt(X) != _dt(W):
        raise ValueError("X must be [S,C], W [N,C], same dtype, rows contiguous")
    S, C = X.shape
    N = W.shape[0]
    if kept_idx is not None:
        if kept_idx.dtype != torch.int32 or kept_idx.dim() != 1 or not kept_idx.is_contiguous():
            raise ValueError("kept_idx must be contiguous int32 [M]")
        if M is None:
            M = kept_idx.numel()
        elif kept_idx.numel() < M:
            raise ValueError("kept_idx is shorter than M")
    elif M is None:
        M = S
    if bias is not None and (bias.dtype != X.dtype or tuple(bias.shape) != (N,) or not bias.is_contiguous()):
        raise ValueError("bias must be [N] of the input dtype")
    if Y is None:
        Y = torch.empty((M, N), dtype=X.dtype, device=X.device)
    elif Y.dtype != X.dtype or Y.dim() != 2 or Y.shape[0] < M or Y.shape[1] != N or Y.stride(1) != 1:
        raise ValueError("Y must be [M,N] of the input dtype, rows contiguous")
    _check(_lib.lemo_gather_gemm(_ptr(X), S, X.stride(0), _ptr(kept_idx), M, _ptr(W), W.stride(0), _ptr(bias), _ptr(Y),
                                 Y.stride(0) if M > 0 else N, C, N, _dt(X), _stream()), "lemo_gather_gemm")
    return Y


def lemo_gather_gemm_add(X: torch.Tensor, kept_idx: Optional[torch.Tensor], W: torch.Tensor, R: torch.Tensor,
                         out_idx: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                         M: Optional[int] = None) -> torch.Tensor:
    """In place: R[out_idx[m],:] += X[kept_idx[m],:] @ W.T (+ bias).  X [S,C], W [N,C], R [S_out,N], rows contiguous."""
    rc = _native.gather_gemm_add(X, kept_idx, W, R, out_idx, bias, M)
    if rc is not None:
        _check(rc, "lemo_gather_gemm_add")
        return R
    _dev(X, kept_idx, W, bias, R, out_idx)
    if X.dim() != 2 or W.dim() != 2 or X.stride(1) != 1 or W.stride(1) != 1 or X.shape[1] != W.shape[1] or _dt(X) != _dt(W):
        raise ValueError("X must be [S,C], W [N,C], same dtype, rows contiguous")
    S, C = X.shape
    N = W.shape[0]
    for name, ix in (("kept_idx", kept_idx), ("out_idx", out_idx)):
        if ix is not None:
            if ix.dtype != torch.int32 or ix.dim() != 1 or not ix.is_contiguous():
                raise ValueError(f"{name} must be contiguous int32 [M]")
            if M is None:
                M = ix.numel()
            elif ix.numel() < M:
                raise ValueError(f"{name} is shorter than M")
    if M is None:
        M = S
    if bias is not None and (bias.dtype != X.dtype or tuple(bias.shape) != (N,) or not bias.is_contiguous()):
        raise ValueError("bias must be [N] of the input dtype")
    if R.dtype != X.dtype or R.dim() != 2 or R.shape[1] != N or R.stride(1) != 1:
        raise ValueError("R must be [S_out,N] of the input dtype, rows contiguous")
    _check(_lib.lemo_gather_gemm_add(_ptr(X), S, X.stride(0), _ptr(kept_idx), M, _ptr(W), W.stride(0), _ptr(bias), _ptr(R),
                                     R.stride(0), R.shape[0], _ptr(out_idx), C, N, _dt(X), _stream()), "lemo_gather_gemm_add")
    return R


def lemo_kept_attention_workspace_bytes(M: int, H_kv: int, d: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.lemo_kept_attention_workspace_bytes(M, H_kv, d, ctypes.byref(n)), "lemo_kept_attention_workspace_bytes")
    return int(n.value)


def lemo_kept_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, kept_idx: Optional[torch.Tensor], flags: int = CAUSAL,
                        scale: float = 0.0, O: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        M: Optional[int] = None) -> torch.Tensor:
    """Attention over the kept rows of Q [S,H,d], K, V [S,H_kv,d] -> compact O [M,H,d]."""
    rc = _native.kept_attention(Q, K, V, kept_idx, flags, scale, O, workspace, M)
    if rc is not None:
        _check(rc, "lemo_kept_attention")
        return O
    a = _qk_args(Q, K)
    _dev(V, kept_idx, O, workspace)
    S, H, Hkv, d = a[2], a[3], a[4], a[5]
    if V.dim() != 3 or tuple(V.shape) != tuple(K.shape) or V.stride(2) != 1 or V.dtype != K.dtype:
        raise ValueError("V must match K: [S,H_kv,d], head_dim contiguous")
    if kept_idx is not None:
        if kept_idx.dtype != torch.int32 or kept_idx.dim() != 1 or not kept_idx.is_contiguous():
            raise ValueError("kept_idx must be contiguous int32 [M]")
        if M is None:
            M = kept_idx.numel()
        elif kept_idx.numel() < M:
            raise ValueError("kept_idx is shorter than M")
    elif M is None:
        M = S
    if O is None:
        O = torch.empty((M, H, d), dtype=Q.dtype, device=Q.device)
    elif O.dtype != Q.dtype or O.dim() != 3 or O.shape[0] < M or O.shape[1] != H or O.shape[2] != d or O.stride(2) != 1:
        raise ValueError("O must be [M,H,d] of the input dtype, head_dim contiguous")
    if workspace is None:
        workspace = torch.empty(lemo_kept_attention_workspace_bytes(M, Hkv, d), dtype=torch.uint8, device=Q.device)
    _check(_lib.lemo_kept_attention(a[0], a[1], _ptr(V), *a[2:11], V.stride(0), V.stride(1), _ptr(kept_idx), M, float(scale), int(flags), _ptr(O),
                                    O.stride(0) if M > 0 else H * d, O.stride(1) if M > 0 else d, _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream()), "lemo_kept_attention")
    return O


def lemo_gather_gemm_dx(dY: torch.Tensor, W: torch.Tensor, dX: torch.Tensor, out_idx: Optional[torch.Tensor]) -> torch.Tensor:
    """In place: dX[out_idx[m],:] += dY[m,:] @ W.  dY [M,N], W [N,C] (as stored for the forward), dX [S_out,C]."""
    rc = _native.gather_gemm_dx(dY, W, dX, out_idx)
    if rc is not None:
        _check(rc, "lemo_gather_gemm_dx")
        return dX
    _dev(dY, W, dX, out_idx)
    if dY.dim() != 2 or W.dim() != 2 or dX.dim() != 2 or _dt(dY) != _dt(W) or _dt(dX) != _dt(W) or W.stride(1) != 1 or dX.stride(1) != 1 \
            or dY.shape[1] != W.shape[0] or dX.shape[1] != W.shape[1] or (dY.shape[0] > 0 and dY.stride(1) != 1):
        raise ValueError("dY must be [M,N], W [N,C], dX [S_out,C], same dtype, rows contiguous")
    M, N = dY.shape
    C = W.shape[1]
    if out_idx is not None and (out_idx.dtype != torch.int32 or out_idx.dim() != 1 or out_idx.numel() != M or not out_idx.is_contiguous()):
        raise ValueError("out_idx must be contiguous int32 [M]")
    _check(_lib.lemo_gather_gemm_dx(_ptr(dY), dY.stride(0) if M > 0 else N, M, _ptr(W), W.stride(0), _ptr(dX), dX.stride(0), dX.shape[0],
                                    _ptr(out_idx), C, N, _dt(W), _stream()), "lemo_gather_gemm_dx")
    return dX


def lemo_gather_gemm_dw_workspace_bytes(M: int, C: int, N: int, dtype: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.lemo_gather_gemm_dw_workspace_bytes(M, C, N, dtype, ctypes.byref(n)), "lemo_gather_gemm_dw_workspace_bytes")
    return int(n.value)


def lemo_gather_gemm_dw(dY: torch.Tensor, X: torch.Tensor, kept_idx: Optional[torch.Tensor], dW: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dW[n,c] = sum_m dY[m,n] * X[kept_idx[m],c].  dY [M,N], X [S,C] -> dW [N,C]."""
    rc = _native.gather_gemm_dw(dY, X, kept_idx, dW, workspace)
    if rc is not None:
        _check(rc, "lemo_gather_gemm_dw")
        return dW
    _dev(dY, X, kept_idx, dW, workspace)
    if dY.dim() != 2 or X.dim() != 2 or _dt(dY) != _dt(X) or X.stride(1) != 1 or (dY.shape[0] > 0 and dY.stride(1) != 1):
        raise ValueError("dY must be [M,N] and X [S,C], same dtype, rows contiguous")
    M, N = dY.shape
    S, C = X.shape
    if kept_idx is not None and (kept_idx.dtype != torch.int32 or kept_idx.dim() != 1 or kept_idx.numel() != M or not kept_idx.is_contiguous()):
        raise ValueError("kept_idx must be contiguous int32 [M]")
    if dW is None:
        dW = torch.empty((N, C), dtype=X.dtype, device=X.device)
    elif dW.dtype != X.dtype or tuple(dW.shape) != (N, C) or dW.stride(1) != 1:
        raise ValueError("dW must be [N,C] of the input dtype, rows contiguous")
    if workspace is None:
        need = lemo_gather_gemm_dw_workspace_bytes(M, C, N, _dt(X))
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device) if need else None
    _check(_lib.lemo_gather_gemm_dw(_ptr(dY), dY.stride(0) if M > 0 else N, _ptr(X), S, X.stride(0), _ptr(kept_idx), M, _ptr(dW),
                                    dW.stride(0), C, N, _dt(X), _ptr(workspace),
                                    workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                    _stream()), "lemo_gather_gemm_dw")
    return dW


def lemo_scatter_grad(G: torch.Tensor, kept_idx: torch.Tensor, dX: torch.Tensor, mode: int = SCATTER_ACCUMULATE) -> torch.Tensor:
    """In place: dX[kept_idx[m],:] += G[m,:] (ACCUMULATE) or dX = zero-padded G (ZERO_PAD)."""
    rc = _native.scatter_grad(G, kept_idx, dX, mode)
    if rc is not None:
        _check(rc, "lemo_scatter_grad")
        return dX
    _dev(G, kept_idx, dX)
    if G.dim() != 2 or dX.dim() != 2 or G.shape[1] != dX.shape[1] or dX.stride(1) != 1 or (G.shape[0] > 0 and G.stride(1) != 1):
        raise ValueError("G must be [M,C] and dX [S,C], rows contiguous")
    if kept_idx.dtype != torch.int32 or kept_idx.dim() != 1 or kept_idx.numel() != G.shape[0] or not kept_idx.is_contiguous():
        raise ValueError("kept_idx must be contiguous int32 [M]")
    M, C = G.shape
    _check(_lib.lemo_scatter_grad(_ptr(G), G.stride(0) if M > 0 else C, _ptr(kept_idx), M, _ptr(dX), dX.stride(0),
                                  dX.shape[0], C, _dt(G), _dt(dX), int(mode), _stream()), "lemo_scatter_grad")
    return dX


# --------------------------------------------------------------------------------- norms around a block

NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GATE_SIGMOID = 1


class NormGrads(NamedTuple):
    """What lemo_norm_residual_grad returns beside dR: None where there is nothing to take a gradient of."""
    dY: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]      # [M,C], or [C] float32 for a gate that all rows share
    dw_post: Optional[torch.Tensor]    # [C] float32, like the three below
    db_post: Optional[torch.Tensor]
    dw_next: Optional[torch.Tensor]
    db_next: Optional[torch.Tensor]


def _here(*ts):
    """Tensors of a call: on the device that is current, whose stream the call goes to."""
    _dev(*ts)
    for t in ts:
        if t is not None and t.device.index != torch.cuda.current_device():
            raise ValueError("tensors must live on the current device")


def _index(t: Optional[torch.Tensor], M: int, name: str):
    if t is not None and (t.dtype != torch.int32 or tuple(t.shape) != (M,) or not t.is_contiguous()):
        raise ValueError(f"{name} must be contiguous int32 [M]")


def _rows_of(t: Optional[torch.Tensor], M: int, C: int, dtype, name: str) -> int:
    """Row stride of an [M,C] operand that may be missing."""
    if t is None:
        return C
    if t.dim() != 2 or tuple(t.shape) != (M, C) or t.dtype != dtype or (t.stride(1) != 1 and C > 1 and M > 0):
        raise ValueError(f"{name} must be [{M},{C}] of the residual's dtype, rows contiguous")
    return t.stride(0) if M > 1 else C


def _channels(t: Optional[torch.Tensor], C: int, dtype, name: str):
    if t is not None and (tuple(t.shape) != (C,) or t.dtype != dtype or not t.is_contiguous()):
        raise ValueError(f"{name} must be contiguous [{C}] of {dtype}")


def _norm_args(Y, R, kept_idx, gate, w_post, b_post, w_next, b_next):
    """Sizes and strides shared by the norm calls: M, S, C, ldy, ld_gate, ldr."""
    if R.dim() != 2 or (R.stride(1) != 1 and R.shape[1] > 1):
        raise ValueError("R must be [S,C], rows contiguous")
    _dt(R)
    S, C = R.shape
    M = Y.shape[0] if Y is not None and Y.dim() == 2 else kept_idx.numel() if kept_idx is not None else S
    _index(kept_idx, M, "kept_idx")
    ld_gate = 0
    if gate is not None and gate.dim() == 1:
        _channels(gate, C, R.dtype, "gate")
    else:
        ld_gate = _rows_of(gate, M, C, R.dtype, "gate")
    for name, t in (("w_post", w_post), ("b_post", b_post), ("w_next", w_next), ("b_next", b_next)):
        _channels(t, C, R.dtype, name)
    return M, S, C, _rows_of(Y, M, C, R.dtype, "Y"), ld_gate, R.stride(0) if S > 1 else C


def lemo_norm_residual(Y: Optional[torch.Tensor], R: torch.Tensor, kept_idx: Optional[torch.Tensor] = None, *, gate: Optional[torch.Tensor] = None,
                       post: int = NORM_NONE, next: int = NORM_RMS, w_post: Optional[torch.Tensor] = None, b_post: Optional[torch.Tensor] = None,
                       w_next: Optional[torch.Tensor] = None, b_next: Optional[torch.Tensor] = None, eps: float = 1e-5, residual_scale: float = 1.0,
                       block_scale: float = 1.0, flags: int = 0, N: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None):
    """In place: R[kept_idx] = residual_scale * R[kept_idx] + block_scale * gate * post(Y) -> (N = next(R[kept_idx]) [M,C] or None,
    stats [M,4] float32).  Y [M,C] or None, R [S,C], gate [M,C] or one row [C]."""
    done = _native.norm_residual(Y, R, kept_idx, gate, post, next, w_post, b_post, w_next, b_next, eps, residual_scale, block_scale, flags, N, stats)
    if done is not None:
        _check(done[0], "lemo_norm_residual")
        return done[1], done[2]
    _here(Y, R, kept_idx, gate, w_post, b_post, w_next, b_next, N, stats)
    M, S, C, ldy, ldg, ldr = _norm_args(Y, R, kept_idx, gate, w_post, b_post, w_next, b_next)
    if N is None and next != NORM_NONE:
        N = torch.empty((M, C), dtype=R.dtype, device=R.device)
    ldn = _rows_of(N, M, C, R.dtype, "N")
    if stats is None:
        stats = torch.empty((M, 4), dtype=torch.float32, device=R.device)
    elif stats.dtype != torch.float32 or tuple(stats.shape) != (M, 4) or not stats.is_contiguous():
        raise ValueError("stats must be contiguous float32 [M,4]")
    _check(_lib.lemo_norm_residual(_ptr(Y), ldy, _ptr(gate), ldg, _ptr(R), ldr, S, _ptr(kept_idx), M, _ptr(w_post), _ptr(b_post), int(post),
                                   _ptr(w_next), _ptr(b_next), int(next), float(eps), float(residual_scale), float(block_scale), _ptr(N), ldn,
                                   _ptr(stats), C, _dt(R), int(flags), _stream()), "lemo_norm_residual")
    return N, stats


def lemo_norm_residual_grad_workspace_bytes(M: int, C: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.lemo_norm_residual_grad_workspace_bytes(M, C, ctypes.byref(n)), "lemo_norm_residual_grad_workspace_bytes")
    return int(n.value)


def lemo_norm_residual_grad(dN: Optional[torch.Tensor], dR: torch.Tensor, R: torch.Tensor, Y: Optional[torch.Tensor], kept_idx: Optional[torch.Tensor],
                            stats: torch.Tensor, *, gate: Optional[torch.Tensor] = None, post: int = NORM_NONE, next: int = NORM_RMS,
                            w_post: Optional[torch.Tensor] = None, b_post: Optional[torch.Tensor] = None, w_next: Optional[torch.Tensor] = None,
                            residual_scale: float = 1.0, block_scale: float = 1.0, flags: int = 0, workspace: Optional[torch.Tensor] = None,
                            dY: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None, weights: bool = True) -> NormGrads:
    """Gradients of lemo_norm_residual: dR [S,C] (of the new residual rows) becomes that of the old ones in place; returns the others.
    R, Y, gate, stats as the forward call left or took them.  dY may be dN, dgate (of a gate with rows of its own) may be gate; weights=False
    leaves out the sums for the norms' weights and biases."""
    done = _native.norm_residual_grad(dN, dR, R, Y, kept_idx, stats, gate, post, next, w_post, b_post, w_next, residual_scale, block_scale, flags, workspace,
                                      dY, dgate, weights)
    if done is not None:
        _check(done[0], "lemo_norm_residual_grad")
        return NormGrads(*done[1:])
    _here(dN, dR, R, Y, kept_idx, stats, gate, w_post, b_post, w_next, workspace, dY, dgate)
    M, S, C, ldy, ldg, ldr = _norm_args(Y, R, kept_idx, gate, w_post, b_post, w_next, None)
    if tuple(dR.shape) != (S, C) or dR.dtype != R.dtype or (dR.stride(1) != 1 and C > 1):
        raise ValueError("dR must be [S,C] of the residual's dtype, rows contiguous")
    if stats.dtype != torch.float32 or tuple(stats.shape) != (M, 4) or not stats.is_contiguous():
        raise ValueError("stats must be contiguous float32 [M,4]")
    lddn = _rows_of(dN, M, C, R.dtype, "dN")

    def rows():
        return torch.empty((M, C), dtype=R.dtype, device=R.device)

    def sums(wanted):
        return torch.empty(C, dtype=torch.float32, device=R.device) if wanted else None

    shared = gate is not None and gate.dim() == 1
    if (dY is not None and Y is None) or (dgate is not None and gate is None):
        raise ValueError("dY needs Y, dgate needs a gate")
    if dY is None and Y is not None:
        dY = rows()
    dgate_sum = _filled(dgate, (C,), torch.float32, R.device, "dgate") if shared else None
    dgate = None if shared else rows() if dgate is None and gate is not None else dgate
    lddy, lddg = _rows_of(dY, M, C, R.dtype, "dY"), _rows_of(dgate, M, C, R.dtype, "dgate")
    dw_post, db_post = sums(weights and post != NORM_NONE), sums(weights and post != NORM_NONE and (b_post is not None or post == NORM_LAYER))
    dw_next, db_next = sums(weights and next != NORM_NONE), sums(weights and next != NORM_NONE)
    needs = dgate_sum is not None or dw_post is not None or dw_next is not None
    workspace, size = _scratch(workspace, lemo_norm_residual_grad_workspace_bytes(M, C) if needs else 0, R.device)
    _check(_lib.lemo_norm_residual_grad(_ptr(dN), lddn, _ptr(dR), dR.stride(0) if S > 1 else C, S, _ptr(R), ldr, _ptr(Y), ldy, _ptr(gate), ldg,
                                        _ptr(kept_idx), M, _ptr(w_post), _ptr(b_post), int(post), _ptr(w_next), int(next), float(residual_scale),
                                        float(block_scale), _ptr(stats), _ptr(dY), lddy, _ptr(dgate), lddg, _ptr(dw_post), _ptr(db_post), _ptr(dw_next),
                                        _ptr(db_next), _ptr(dgate_sum), C, _dt(R), int(flags), _ptr(workspace), size, _stream()), "lemo_norm_residual_grad")
    return NormGrads(dY, dgate_sum if shared else dgate, dw_post, db_post, dw_next, db_next)


# --------------------------------------------------------------------------------- attention over chosen key blocks

def _heads(t: torch.Tensor, dims: int, name: str):
    if t.dim() != dims or t.stride(-1) != 1:
        raise ValueError(f"{name} must have {dims} dimensions, the last (head_dim) contiguous")
    _dt(t)


def _fits(t: torch.Tensor, shape, dtype, name: str):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {dtype} {list(shape)}")


def _filled(t: Optional[torch.Tensor], shape, dtype, device, name: str) -> torch.Tensor:
    """A contiguous result of the caller's, or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _fits(t, shape, dtype, name)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _blocks_of(n: int, b: int) -> int:
    if b <= 0:
        raise ValueError("block sizes must be positive")
    return -(-n // b)


def _bytes(name: str, *args) -> int:
    n = ctypes.c_size_t(0)
    _check(getattr(_lib, name)(*args, ctypes.byref(n)), name)
    return int(n.value)


def _scratch(workspace: Optional[torch.Tensor], need: int, device):
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, 0 if workspace is None else workspace.numel() * workspace.element_size()


def lemo_block_means(K: torch.Tensor, b: int, means: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Mean key of every block of b tokens: K [S,H_kv,d] -> [ceil(S/b),H_kv,d] float32."""
    done = _native.block_means(K, b, means)
    if done is not None:
        _check(done[0], "lemo_block_means")
        return done[1]
    _here(K, means)
    _heads(K, 3, "K")
    S, Hkv, d = K.shape
    means = _filled(means, (_blocks_of(S, b), Hkv, d), torch.float32, K.device, "means")
    _check(_lib.lemo_block_means(_ptr(K), S, Hkv, d, _dt(K), K.stride(0), K.stride(1), int(b), _ptr(means), _stream()), "lemo_block_means")
    return means


def lemo_select_blocks(Q: torch.Tensor, means: torch.Tensor, S_k: int, b: int, bq: int, T: int, flags: int = CAUSAL, q_start: int = 0,
                       blocks: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The T key blocks that each block of bq queries lists, per KV head -> [ceil(S_q/bq),H_kv,T] int32, ascending, -1 behind them."""
    done = _native.select_blocks(Q, means, S_k, b, bq, T, flags, q_start, blocks)
    if done is not None:
        _check(done[0], "lemo_select_blocks")
        return done[1]
    _here(Q, means, blocks)
    _heads(Q, 3, "Q")
    S, H, d = Q.shape
    Hkv = means.shape[1] if means.dim() == 3 else 0
    _filled(means, (_blocks_of(S_k, b), Hkv, d), torch.float32, Q.device, "means")
    blocks = _filled(blocks, (_blocks_of(S, bq), Hkv, T), torch.int32, Q.device, "blocks")
    _check(_lib.lemo_select_blocks(_ptr(Q), S, H, Hkv, d, _dt(Q), Q.stride(0), Q.stride(1), _ptr(means), int(S_k), int(q_start), int(b), int(bq), int(T),
                                   int(flags), _ptr(blocks), _stream()), "lemo_select_blocks")
    return blocks


def _attention_sizes(Q, K, V, blocks, b, bq):
    for name, t in (("Q", Q), ("K", K), ("V", V)):
        _heads(t, 3, name)
    S, H, d = Q.shape
    _fits(K, (K.shape[0], K.shape[1], d), Q.dtype, "K")
    _fits(V, K.shape, Q.dtype, "V")
    if blocks.dim() != 3:
        raise ValueError("blocks must be [query blocks, H_kv, T]")
    _filled(blocks, (_blocks_of(S, bq), K.shape[1], blocks.shape[2]), torch.int32, Q.device, "blocks")
    _blocks_of(S, b)
    return S, K.shape[0], H, K.shape[1], d, blocks.shape[2]


def lemo_block_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, blocks: torch.Tensor, b: int, bq: int, flags: int = CAUSAL, scale: float = 0.0,
                         q_start: int = 0, O: Optional[torch.Tensor] = None, lse2: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None):
    """Attention of Q [S_q,H,d] over the key blocks that `blocks` lists, K and V [S_k,H_kv,d] -> (O [S_q,H,d], lse2 [H,S_q] float32)."""
    done = _native.block_attention(Q, K, V, blocks, b, bq, flags, scale, q_start, O, lse2, workspace)
    if done is not None:
        _check(done[0], "lemo_block_attention")
        return done[1], done[2]
    _here(Q, K, V, blocks, O, lse2, workspace)
    S, Sk, H, Hkv, d, T = _attention_sizes(Q, K, V, blocks, b, bq)
    if O is None:
        O = torch.empty((S, H, d), dtype=Q.dtype, device=Q.device)
    _heads(O, 3, "O")
    _fits(O, (S, H, d), Q.dtype, "O")
    lse2 = _filled(lse2, (H, S), torch.float32, Q.device, "lse2")
    workspace, size = _scratch(workspace, _bytes("lemo_block_attention_workspace_bytes", S, Sk, H, Hkv, d, T, int(b), int(bq)), Q.device)
    _check(_lib.lemo_block_attention(_ptr(Q), _ptr(K), _ptr(V), S, Sk, H, Hkv, d, _dt(Q), Q.stride(0), Q.stride(1), K.stride(0), K.stride(1), V.stride(0),
                                     V.stride(1), _ptr(blocks), T, int(b), int(bq), int(q_start), float(scale), int(flags), _ptr(O), O.stride(0),
                                     O.stride(1), _ptr(lse2), _ptr(workspace), size, _stream()), "lemo_block_attention")
    return O, lse2


def lemo_block_attention_grad(dO: torch.Tensor, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, O: torch.Tensor, lse2: torch.Tensor, blocks: torch.Tensor,
                              b: int, bq: int, flags: int = CAUSAL, scale: float = 0.0, q_start: int = 0, dQ: Optional[torch.Tensor] = None,
                              dK: Optional[torch.Tensor] = None, dV: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Gradients of lemo_block_attention, O and lse2 as it left them -> (dQ [S_q,H,d], dK [S_k,H_kv,d], dV [S_k,H_kv,d])."""
    done = _native.block_attention_grad(dO, Q, K, V, O, lse2, blocks, b, bq, flags, scale, q_start, dQ, dK, dV, workspace)
    if done is not None:
        _check(done[0], "lemo_block_attention_grad")
        return done[1], done[2], done[3]
    _here(dO, Q, K, V, O, lse2, blocks, dQ, dK, dV, workspace)
    S, Sk, H, Hkv, d, T = _attention_sizes(Q, K, V, blocks, b, bq)
    for name, t in (("dO", dO), ("O", O)):
        _heads(t, 3, name)
        _fits(t, (S, H, d), Q.dtype, name)
    _filled(lse2, (H, S), torch.float32, Q.device, "lse2")
    dQ = _filled(dQ, (S, H, d), Q.dtype, Q.device, "dQ")
    dK = _filled(dK, (Sk, Hkv, d), Q.dtype, Q.device, "dK")
    dV = _filled(dV, (Sk, Hkv, d), Q.dtype, Q.device, "dV")
    workspace, size = _scratch(workspace, _bytes("lemo_block_attention_grad_workspace_bytes", S, Sk, H, Hkv, d, T, int(b), int(bq)), Q.device)
    _check(_lib.lemo_block_attention_grad(_ptr(dO), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(lse2), S, Sk, H, Hkv, d, _dt(Q), dO.stride(0), dO.stride(1),
                                          Q.stride(0), Q.stride(1), K.stride(0), K.stride(1), V.stride(0), V.stride(1), O.stride(0), O.stride(1),
                                          _ptr(blocks), T, int(b), int(bq), int(q_start), float(scale), int(flags), _ptr(dQ), _ptr(dK), _ptr(dV),
                                          _ptr(workspace), size, _stream()), "lemo_block_attention_grad")
    return dQ, dK, dV


def _lengths(lengths: torch.Tensor, B: int):
    _filled(lengths, (B,), torch.int32, None, "lengths")


def lemo_block_means_step(K: torch.Tensor, lengths: torch.Tensor, b: int, means: torch.Tensor) -> torch.Tensor:
    """In place: the mean of the block that the newest token of each sequence has filled, if it has.  K [B,S_max,H_kv,d], lengths [B] int32,
    means [B,ceil(S_max/b),H_kv,d] float32."""
    _here(K, lengths, means)
    _heads(K, 4, "K")
    B, S, Hkv, d = K.shape
    _lengths(lengths, B)
    _filled(means, (B, _blocks_of(S, b), Hkv, d), torch.float32, K.device, "means")
    _check(_lib.lemo_block_means_step(_ptr(K), B, S, Hkv, d, _dt(K), K.stride(0), K.stride(1), K.stride(2), _ptr(lengths), int(b), _ptr(means), _stream()),
           "lemo_block_means_step")
    return means


def lemo_select_blocks_step(Q: torch.Tensor, means: torch.Tensor, lengths: torch.Tensor, b: int, T: int, blocks: Optional[torch.Tensor] = None,
                            S_max: Optional[int] = None) -> torch.Tensor:
    """Key blocks for the newest token of each sequence: Q [B,H,d], means [B,ceil(S_max/b),H_kv,d] float32 -> [B,H_kv,T] int32.
    S_max: the cache's tokens (all that the means cover if not given)."""
    done = _native.select_blocks_step(Q, means, lengths, b, T, blocks, S_max)
    if done is not None:
        _check(done[0], "lemo_select_blocks_step")
        return done[1]
    _here(Q, means, lengths, blocks)
    _heads(Q, 3, "Q")
    B, H, d = Q.shape
    if means.dim() != 4:
        raise ValueError("means must be [B, blocks, H_kv, d]")
    nb, Hkv = means.shape[1], means.shape[2]
    S_max = nb * b if S_max is None else S_max
    if _blocks_of(S_max, b) != nb:
        raise ValueError("means must be [B, ceil(S_max / b), H_kv, d]")
    _filled(means, (B, nb, Hkv, d), torch.float32, Q.device, "means")
    _lengths(lengths, B)
    blocks = _filled(blocks, (B, Hkv, T), torch.int32, Q.device, "blocks")
    _check(_lib.lemo_select_blocks_step(_ptr(Q), B, H, Hkv, d, _dt(Q), Q.stride(0), Q.stride(1), _ptr(means), int(S_max), _ptr(lengths), int(b), int(T),
                                        _ptr(blocks), _stream()), "lemo_select_blocks_step")
    return blocks


def lemo_block_attention_step(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, lengths: torch.Tensor, blocks: torch.Tensor, b: int, scale: float = 0.0,
                              O: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the newest token of each sequence over its listed blocks: Q [B,H,d], K and V [B,S_max,H_kv,d] -> O [B,H,d]."""
    done = _native.block_attention_step(Q, K, V, lengths, blocks, b, scale, O, workspace)
    if done is not None:
        _check(done[0], "lemo_block_attention_step")
        return done[1]
    _here(Q, K, V, lengths, blocks, O, workspace)
    _heads(Q, 3, "Q")
    _heads(K, 4, "K")
    _heads(V, 4, "V")
    B, H, d = Q.shape
    S, Hkv = K.shape[1], K.shape[2]
    _fits(K, (B, S, Hkv, d), Q.dtype, "K")
    _fits(V, (B, S, Hkv, d), Q.dtype, "V")
    _lengths(lengths, B)
    if blocks.dim() != 3:
        raise ValueError("blocks must be [B, H_kv, T]")
    T = blocks.shape[2]
    _filled(blocks, (B, Hkv, T), torch.int32, Q.device, "blocks")
    if O is None:
        O = torch.empty((B, H, d), dtype=Q.dtype, device=Q.device)
    _heads(O, 3, "O")
    _fits(O, (B, H, d), Q.dtype, "O")
    workspace, size = _scratch(workspace, _bytes("lemo_block_attention_step_workspace_bytes", B, H, Hkv, d, T, int(b)), Q.device)
    _check(_lib.lemo_block_attention_step(_ptr(Q), _ptr(K), _ptr(V), B, S, H, Hkv, d, _dt(Q), Q.stride(0), Q.stride(1), K.stride(0), K.stride(1), K.stride(2),
                                          V.stride(0), V.stride(1), V.stride(2), _ptr(lengths), _ptr(blocks), T, int(b), float(scale), _ptr(O), O.stride(0),
                                          O.stride(1), _ptr(workspace), size, _stream()), "lemo_block_attention_step")
    return O
