"""Python binding of libcmc: the CMC two-tier decode path on GB300.

Argument marshalling only.  Each function checks the tensors it is given
(device, dtype, contiguity, shapes), derives the sizes, and calls the C ABI
with raw device pointers and the current torch CUDA stream.  Every step of the
computation runs in the library's CUDA kernels; there is no CPU path.

Tensor layouts (row-major, last index fastest):

  question_emb  fp32 [B, D]            cme_bank  fp32 [B, N, D]
  q             bf16 [B, L, Hq, d]     out       bf16 [B, L, Hq, d]
  tier1_k/v     bf16 [B, L, Hkv, N, d] idx       int32 [B, k]
  ring_k/v      bf16 [B, L, Hkv, W, d] pos       int64 [B]
  k_new/v_new   bf16 [B, L, Hkv, d]

and of the cache in 8 bits (T tokens, see cmc.h for the format):

  kv            float8_e4m3fn  [B, L, Hkv, 2, T, d]   keys, then values
  scales        float8_e8m0fnu [B, L, Hkv, 2, q8_scale_bytes(T)]

and where the cache's tokens have weights (what they received in attention):

  tier1_weight  fp32 [B, L, Hkv, N]    ring_weight  fp32 [B, L, Hkv, W]

Tier-1 selection in the attention calls: an ``idx`` tensor [B, k] gathers
rows of the bank by index at every step; ``idx=None`` takes every row of
``tier1_k``/``tier1_v`` in order (k = N), which is how the dense Tier-1 cache
made once per question by :func:`tier1_gather` is passed.
"""

from __future__ import annotations

import ctypes
import functools
import os
from typing import Dict, Optional, Tuple

import torch

from ._lib import CmcCopy, CmcDims, CmcQkPrep, check, lib, DEVFLAG_BAD_INDEX, DEVFLAG_BAD_POS, DEVFLAG_TIMEOUT

__all__ = [
    "CmcDims",
    "DecodeWorkspace",
    "denoise",
    "bridge_epilogue",
    "score_select",
    "score_select_workspace_size",
    "question_select",
    "window_append",
    "two_tier_decode_attn",
    "decode_step",
    "tier1_gather",
    "decode_attn_workspace_size",
    "decode_attn_plan",
    "quantize_cache",
    "dequantize_cache",
    "window_append_q8",
    "two_tier_decode_attn_q8",
    "decode_step_q8",
    "decode_attn_q8_plan",
    "decode_attn_q8_workspace_size",
    "decode_q8_status",
    "q8_scale_bytes",
    "qk_norm_rope",
    "window_prefill",
    "two_tier_decode_attn_weighted",
    "decode_step_weighted",
    "evict_cache",
    "decode_attn_weighted_plan",
    "decode_attn_weighted_workspace_size",
    "weighted_cache_status",
    "set_l2_prefetch_tiles",
    "dims_of",
    "stage_copies",
    "DEVFLAG_BAD_INDEX",
    "DEVFLAG_BAD_POS",
    "DEVFLAG_TIMEOUT",
]


# With CMC_NVTX set (not "0") when the module is imported, every device call
# below is wrapped in an NVTX range named after it ("cmc.decode_step", ...),
# for profiler timelines; otherwise the functions are left as they are.
_NVTX = os.environ.get("CMC_NVTX", "") not in ("", "0")


def _ranged(fn):
    if not _NVTX:
        return fn
    name = "cmc." + fn.__name__

    @functools.wraps(fn)
    def wrapped(*args, **kwargs):
        torch.cuda.nvtx.range_push(name)
        try:
            return fn(*args, **kwargs)
        finally:
            torch.cuda.nvtx.range_pop()
    return wrapped


# The functions below are called once per decode step, so what they do on the
# host counts: a step of a small decoder takes the GPU 5 us.  Pointers and
# streams are passed to ctypes as plain integers (the argument types are
# declared), the current stream is read without building a Stream object, and
# a tensor that passes is looked at through as few attributes as will do.

def _p(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _stream(device: torch.device) -> int:
    index = device.index
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if index is None else index)


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, ndim: int, device=None) -> None:
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == ndim
            and t.is_contiguous() and (device is None or t.get_device() == device.index)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor (the library has no CPU path)")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got shape {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")


# ----------------------------------------------------------------------------
# Graph-based context denoising
# ----------------------------------------------------------------------------

@_ranged
def denoise(emb: torch.Tensor, *, n_tokens: Optional[torch.Tensor] = None, g: int = 3,
            tau: float = 0.05, keep_every: int = 16,
            workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Positions of the tokens kept by the graph-based denoising, int32
    [B, n_max] ascending then -1, and their counts int32 [B]; see
    cmc_denoise.  Defaults: the paper's g = 3, tau = 0.05, keep-minimum 16.
    A given ``workspace`` must have been zero-filled before its first use and
    serves one (B, n_max)."""
    _need(emb, "emb", torch.float32, 3)
    dev = emb.device
    B, n_max, H = emb.shape
    if n_tokens is not None:
        _need(n_tokens, "n_tokens", torch.int32, 1, dev)
        if int(n_tokens.shape[0]) != B:
            raise ValueError("n_tokens must be [B]")
    kept = torch.empty((B, n_max), dtype=torch.int32, device=dev)
    count = torch.empty(B, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = _counter_workspace("denoise", B, n_max, dev)
    st = lib().cmc_denoise(_p(emb), _p(n_tokens), B, n_max, H, g, float(tau), keep_every,
                           _p(kept), _p(count), _p(workspace),
                           workspace.numel() * workspace.element_size(), _stream(dev))
    check(st, "cmc_denoise")
    return kept, count


# ----------------------------------------------------------------------------
# MemoryBridge output
# ----------------------------------------------------------------------------

@_ranged
def bridge_epilogue(x: torch.Tensor, nu: float, *, gamma: Optional[torch.Tensor] = None,
                    beta: Optional[torch.Tensor] = None, eps: float = 1e-5,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Decoder-ready CMEs from the MemoryBridge MLP output x (fp32 [..., D]):
    LayerNorm, nu tanh, and the 2 nu norm cap; see cmc_bridge_epilogue."""
    _need(x, "x", torch.float32, x.dim())
    dev = x.device
    D = int(x.shape[-1])
    rows = x.numel() // D if D else 0
    for t, name in ((gamma, "gamma"), (beta, "beta")):
        if t is not None:
            _need(t, name, torch.float32, 1, dev)
            if int(t.shape[0]) != D:
                raise ValueError(f"{name} must be [{D}]")
    if out is None:
        out = torch.empty_like(x)
    _need(out, "out", torch.float32, x.dim(), dev)
    if out.shape != x.shape:
        raise ValueError("out must have the shape of x")
    st = lib().cmc_bridge_epilogue(_p(x), _p(gamma), _p(beta), rows, D, float(eps), float(nu),
                                   _p(out), _stream(dev))
    check(st, "cmc_bridge_epilogue")
    return out


# ----------------------------------------------------------------------------
# Tier-1: scoring and selection
# ----------------------------------------------------------------------------

def score_select_workspace_size(B: int, N: int) -> int:
    return int(lib().cmc_score_select_workspace_size(B, N))


_counter_ws_cache: Dict[Tuple, torch.Tensor] = {}


def _counter_workspace(kind: str, B: int, n: int, device: torch.device) -> torch.Tensor:
    """A zero-filled workspace, one per (kind, device, stream, B, n): its
    counters and histograms start at zero, and every call leaves them so.
    Where they lie depends on the shape, and shapes of one size exist (B = 1,
    4,096 CMEs and B = 2, 1,024), so the size alone is no key: the one's
    scores would be the other's histograms."""
    key = (kind, device.index, _stream(device), B, n)
    ws = _counter_ws_cache.get(key)
    if ws is None:
        size = {"denoise": lib().cmc_denoise_workspace_size,
                "select": lib().cmc_score_select_workspace_size,
                "question": lib().cmc_question_select_workspace_size}[kind]
        ws = torch.zeros(int(size(B, n)), dtype=torch.uint8, device=device)
        _counter_ws_cache[key] = ws
    return ws


@_ranged
def score_select(question_emb: torch.Tensor, cme_bank: torch.Tensor, k: int, *,
                 idx_out: Optional[torch.Tensor] = None,
                 scores_out: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Top-k CMEs by cosine similarity to the question vector, as int32 [B, k]
    indices in ascending (document) order.  See cmc_score_select.  A given
    ``workspace`` must have been zero-filled before its first use and serves
    one (B, N)."""
    _need(cme_bank, "cme_bank", torch.float32, 3)
    dev = cme_bank.device
    _need(question_emb, "question_emb", torch.float32, 2, dev)
    B, N, D = cme_bank.shape
    if tuple(question_emb.shape) != (B, D):
        raise ValueError(f"question_emb shape {tuple(question_emb.shape)} != {(B, D)}")
    if idx_out is None:
        idx_out = torch.empty((B, k), dtype=torch.int32, device=dev)
    _need(idx_out, "idx_out", torch.int32, 2, dev)
    if tuple(idx_out.shape) != (B, k):
        raise ValueError(f"idx_out shape {tuple(idx_out.shape)} != {(B, k)}")
    if scores_out is not None:
        _need(scores_out, "scores_out", torch.float32, 2, dev)
        if tuple(scores_out.shape) != (B, N):
            raise ValueError(f"scores_out shape {tuple(scores_out.shape)} != {(B, N)}")
    if workspace is None:
        workspace = _counter_workspace("select", B, N, dev)
    ws_bytes = workspace.numel() * workspace.element_size()
    st = lib().cmc_score_select(_p(question_emb), _p(cme_bank), B, N, D, k, _p(idx_out),
                                _p(scores_out), _p(workspace), ws_bytes, _stream(dev))
    check(st, "cmc_score_select")
    return idx_out


@_ranged
def question_select(question_tokens: torch.Tensor, cme_bank: torch.Tensor, k: int, *,
                    q_len: Optional[torch.Tensor] = None,
                    chunk_offset: Optional[torch.Tensor] = None,
                    ctx_len: Optional[torch.Tensor] = None, W: Optional[int] = None,
                    workspace: Optional[torch.Tensor] = None):
    """The question-side prologue; see cmc_question_select.  Returns
    (q_vec fp32 [B, D], idx int32 [B, k], alpha int32 [B] or None,
    start int32 [B] or None); alpha and start when chunk_offset, ctx_len
    and W are given.  A given ``workspace`` must have been zero-filled before
    its first use and serves one (B, N)."""
    _need(cme_bank, "cme_bank", torch.float32, 3)
    dev = cme_bank.device
    _need(question_tokens, "question_tokens", torch.float32, 3, dev)
    B, N, D = cme_bank.shape
    Bq, Lq, Dq = question_tokens.shape
    if (Bq, Dq) != (B, D):
        raise ValueError(f"question_tokens shape {tuple(question_tokens.shape)} != ({B}, Lq, {D})")
    if q_len is not None:
        _need(q_len, "q_len", torch.int32, 1, dev)
        if int(q_len.shape[0]) != B:
            raise ValueError("q_len must be [B]")
    locate = chunk_offset is not None
    if locate:
        _need(chunk_offset, "chunk_offset", torch.int32, 2, dev)
        _need(ctx_len, "ctx_len", torch.int32, 1, dev)
        if tuple(chunk_offset.shape) != (B, N) or int(ctx_len.shape[0]) != B or W is None:
            raise ValueError("chunk_offset [B, N], ctx_len [B] and W are needed together")
    q_vec = torch.empty((B, D), dtype=torch.float32, device=dev)
    idx = torch.empty((B, k), dtype=torch.int32, device=dev)
    alpha = torch.empty(B, dtype=torch.int32, device=dev) if locate else None
    start = torch.empty(B, dtype=torch.int32, device=dev) if locate else None
    if workspace is None:
        workspace = _counter_workspace("question", B, N, dev)
    st = lib().cmc_question_select(
        _p(question_tokens), _p(q_len), Lq, _p(cme_bank), B, N, D, k, _p(chunk_offset),
        _p(ctx_len), int(W or 0), _p(q_vec), _p(idx), _p(alpha), _p(start), _p(workspace),
        workspace.numel() * workspace.element_size(), _stream(dev))
    check(st, "cmc_question_select")
    return q_vec, idx, alpha, start


# ----------------------------------------------------------------------------
# Decode attention
# ----------------------------------------------------------------------------

def dims_of(q: torch.Tensor, tier1_k: torch.Tensor, idx: Optional[torch.Tensor],
            ring_k: torch.Tensor) -> CmcDims:
    return CmcDims(*_sizes(q, tier1_k, idx, ring_k))


def _sizes(q, tier1_k, idx, ring_k) -> Tuple:
    B, L, Hq, d = q.shape
    Bk, Lk, Hkv, N, dk = tier1_k.shape
    Br, Lr, Hr, W, dr = ring_k.shape
    k = N if idx is None else int(idx.shape[1])
    if (Bk, Lk, dk) != (B, L, d) or (Br, Lr, Hr, dr) != (B, L, Hkv, d):
        raise ValueError(f"inconsistent shapes: q {tuple(q.shape)}, tier1 {tuple(tier1_k.shape)}, "
                         f"ring {tuple(ring_k.shape)}")
    if idx is not None and int(idx.shape[0]) != B:
        raise ValueError(f"idx shape {tuple(idx.shape)} does not match batch {B}")
    return B, L, Hq, Hkv, d, N, k, W


def decode_attn_workspace_size(dims: CmcDims) -> int:
    return int(lib().cmc_decode_attn_workspace_size(ctypes.byref(dims)))


def decode_attn_plan(dims: CmcDims, fused: bool = True, rope: bool = False) -> Tuple[int, int]:
    """(grid size, kernel launches per call) of the attention entry points for
    `dims` on the current device; see cmc_decode_attn_plan."""
    ctas, launches = ctypes.c_int(0), ctypes.c_int(0)
    mode = 2 if rope else (1 if fused else 0)
    st = lib().cmc_decode_attn_plan(ctypes.byref(dims), mode, ctypes.byref(ctas),
                                    ctypes.byref(launches))
    check(st, "cmc_decode_attn_plan")
    return int(ctas.value), int(launches.value)


def decode_attn_q8_workspace_size(dims: CmcDims) -> int:
    return int(lib().cmc_decode_attn_q8_workspace_size(ctypes.byref(dims)))


def decode_attn_weighted_workspace_size(dims: CmcDims) -> int:
    return int(lib().cmc_decode_attn_weighted_workspace_size(ctypes.byref(dims)))


class DecodeWorkspace:
    """Zero-filled device workspace for the attention entry points (with ``q8`` for
    those over a cache in 8 bits, with ``weighted`` for those that accumulate weights; any
    of the three for :func:`window_prefill` and :func:`evict_cache` of as many sequences).

    Holds the device status word and the fp32 partial results of keys split
    between CTAs.  Calls sharing one workspace must be ordered on one stream."""

    def __init__(self, dims: CmcDims, device: torch.device, q8: bool = False, weighted: bool = False):
        if q8 and weighted:
            raise ValueError("a workspace is of one kind: q8 or weighted")
        n = (decode_attn_q8_workspace_size(dims) if q8
             else decode_attn_weighted_workspace_size(dims) if weighted
             else decode_attn_workspace_size(dims))
        if n == 0:
            raise ValueError(f"unsupported dims {dims.key()}")
        self._set(dims, torch.zeros(n, dtype=torch.uint8, device=device))

    def _set(self, dims: CmcDims, buf: torch.Tensor) -> None:
        self.dims = dims
        self.nbytes = buf.numel()
        self.buf = buf
        self.ptr = buf.data_ptr()
        self.index = buf.get_device()  # -1 on the host

    def status(self, clear: bool = True) -> int:
        """CMC_DEVFLAG_* bits raised by kernels since the last clear (synchronises)."""
        flags = ctypes.c_uint32(0)
        st = lib().cmc_read_status(_p(self.buf), 1 if clear else 0, ctypes.byref(flags),
                                   _stream(self.buf.device))
        check(st, "cmc_read_status")
        return int(flags.value)


def _elsewhere_workspace(workspace: DecodeWorkspace, index: int) -> ValueError:
    return ValueError(f"workspace is on {workspace.buf.device}, expected cuda:{index}")


_ws_cache: Dict[Tuple, DecodeWorkspace] = {}


def _workspace_for(sizes: Tuple, dims: CmcDims, device: torch.device, stream: int
                   ) -> DecodeWorkspace:
    key = (device.index, stream, sizes)
    ws = _ws_cache.get(key)
    if ws is None:
        ws = DecodeWorkspace(dims, device)
        _ws_cache[key] = ws
    return ws


def _attn_args(q, tier1_k, tier1_v, idx, ring_k, ring_v, pos, out):
    _need(q, "q", torch.bfloat16, 4)
    dev = q.device
    _need(tier1_k, "tier1_k", torch.bfloat16, 5, dev)
    _need(tier1_v, "tier1_v", torch.bfloat16, 5, dev)
    _need(ring_k, "ring_k", torch.bfloat16, 5, dev)
    _need(ring_v, "ring_v", torch.bfloat16, 5, dev)
    _need(pos, "pos", torch.int64, 1, dev)
    if idx is not None:
        _need(idx, "idx", torch.int32, 2, dev)
    if tier1_v.shape != tier1_k.shape or ring_v.shape != ring_k.shape:
        raise ValueError("K and V tensors must have the same shapes")
    sizes = _sizes(q, tier1_k, idx, ring_k)
    if int(pos.shape[0]) != sizes[0]:
        raise ValueError(f"pos shape {tuple(pos.shape)} does not match batch {sizes[0]}")
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", torch.bfloat16, 4, dev)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    return sizes, dev, out


def _scale(scale: Optional[float]) -> float:
    return 0.0 if scale is None else float(scale)


def _offset(rope_offset: int) -> int:
    """For the library: what it refuses stays refused, where ctypes would cut it to 64 bits."""
    return rope_offset if 0 <= rope_offset <= 1 << 32 else -1


@_ranged
def two_tier_decode_attn(q, tier1_k, tier1_v, idx, ring_k, ring_v, pos, *,
                         scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                         workspace: Optional[DecodeWorkspace] = None) -> torch.Tensor:
    """Decode attention over [Tier-1 rows at idx | occupied ring slots]; see
    cmc_two_tier_decode_attn.  Returns bf16 [B, L, Hq, d]."""
    sizes, dev, out = _attn_args(q, tier1_k, tier1_v, idx, ring_k, ring_v, pos, out)
    dims, stream = CmcDims(*sizes), _stream(dev)
    if workspace is not None and workspace.index != dev.index:
        raise _elsewhere_workspace(workspace, dev.index)
    ws = workspace if workspace is not None else _workspace_for(sizes, dims, dev, stream)
    st = lib().cmc_two_tier_decode_attn(
        _p(q), _p(tier1_k), _p(tier1_v), _p(idx), _p(ring_k), _p(ring_v), _p(pos),
        ctypes.byref(dims), _scale(scale), _p(out), _p(ws.buf), ws.nbytes, stream)
    if st:
        check(st, "cmc_two_tier_decode_attn")
    return out


@_ranged
def decode_step(q, tier1_k, tier1_v, idx, ring_k, ring_v, pos, k_new, v_new, *,
                scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                workspace: Optional[DecodeWorkspace] = None,
                rope_theta: Optional[float] = None, rope_offset: int = 0) -> torch.Tensor:
    """Fused decode step: append (k_new, v_new) to the ring, then attend; see
    cmc_decode_step.  Updates ring_k, ring_v and pos in place.

    With ``rope_theta`` the step is that of a real GQA layer (see
    cmc_decode_step_rope): q and k_new are given before rotary embedding and
    are rotated at position ``rope_offset + pos[b]`` inside the launch."""
    sizes, dev, out = _attn_args(q, tier1_k, tier1_v, idx, ring_k, ring_v, pos, out)
    _need(k_new, "k_new", torch.bfloat16, 4, dev)
    _need(v_new, "v_new", torch.bfloat16, 4, dev)
    B, L, _, Hkv, d = sizes[:5]
    want = (B, L, Hkv, d)
    if k_new.shape != want or v_new.shape != want:
        raise ValueError(f"k_new/v_new must be {want}")
    dims, stream = CmcDims(*sizes), _stream(dev)
    if workspace is not None and workspace.index != dev.index:
        raise _elsewhere_workspace(workspace, dev.index)
    ws = workspace if workspace is not None else _workspace_for(sizes, dims, dev, stream)
    if rope_theta is None:
        st = lib().cmc_decode_step(
            _p(q), _p(tier1_k), _p(tier1_v), _p(idx), _p(ring_k), _p(ring_v), _p(pos),
            _p(k_new), _p(v_new), ctypes.byref(dims), _scale(scale), _p(out), _p(ws.buf),
            ws.nbytes, stream)
        if st:
            check(st, "cmc_decode_step")
    else:
        st = lib().cmc_decode_step_rope(
            _p(q), _p(tier1_k), _p(tier1_v), _p(idx), _p(ring_k), _p(ring_v), _p(pos),
            _p(k_new), _p(v_new), ctypes.byref(dims), _scale(scale), float(rope_theta),
            _offset(int(rope_offset)), _p(out), _p(ws.buf), ws.nbytes, stream)
        if st:
            check(st, "cmc_decode_step_rope")
    return out


def set_l2_prefetch_tiles(tiles: int) -> None:
    """Box tiles per CTA the attention launches made afterwards prefetch into
    L2 before their grid dependency wait (a hint); see
    cmc_set_l2_prefetch_tiles.  Default 5 (one stream of launches; fewer where
    a launch's plan gains from that); 0 suits
    several streams of independent requests' launches."""
    check(lib().cmc_set_l2_prefetch_tiles(int(tiles)), "cmc_set_l2_prefetch_tiles")


@_ranged
def tier1_gather(bank_k: torch.Tensor, bank_v: torch.Tensor, idx: torch.Tensor, *,
                 out_k: Optional[torch.Tensor] = None, out_v: Optional[torch.Tensor] = None,
                 workspace: Optional[DecodeWorkspace] = None
                 ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Dense Tier-1 cache of the selected rows, bf16 [B, L, Hkv, k, d] each for
    K and V; see cmc_tier1_gather.  Out-of-range indices raise
    DEVFLAG_BAD_INDEX in ``workspace``'s status word when one is given."""
    _need(bank_k, "bank_k", torch.bfloat16, 5)
    dev = bank_k.device
    _need(bank_v, "bank_v", torch.bfloat16, 5, dev)
    _need(idx, "idx", torch.int32, 2, dev)
    if bank_v.shape != bank_k.shape:
        raise ValueError("bank_v must have the shape of bank_k")
    B, L, Hkv, N, d = bank_k.shape
    k = int(idx.shape[1])
    if int(idx.shape[0]) != B:
        raise ValueError(f"idx shape {tuple(idx.shape)} does not match batch {B}")
    want = (B, L, Hkv, k, d)
    if out_k is None:
        out_k = torch.empty(want, dtype=torch.bfloat16, device=dev)
    if out_v is None:
        out_v = torch.empty(want, dtype=torch.bfloat16, device=dev)
    for t, name in ((out_k, "out_k"), (out_v, "out_v")):
        _need(t, name, torch.bfloat16, 5, dev)
        if tuple(t.shape) != want:
            raise ValueError(f"{name} must be {want}")
    dims = CmcDims(B, L, Hkv, Hkv, d, N, k, 1)
    if workspace is not None and workspace.index != dev.index:
        raise _elsewhere_workspace(workspace, dev.index)
    status = None if workspace is None else workspace.buf
    st = lib().cmc_tier1_gather(_p(bank_k), _p(bank_v), _p(idx), ctypes.byref(dims), _p(out_k),
                                _p(out_v), _p(status), _stream(dev))
    check(st, "cmc_tier1_gather")
    return out_k, out_v


@_ranged
def window_append(ring_k: torch.Tensor, ring_v: torch.Tensor, pos: torch.Tensor,
                  k_new: torch.Tensor, v_new: torch.Tensor) -> None:
    """Append one token per sequence to the Tier-2 ring; see cmc_window_append."""
    _need(ring_k, "ring_k", torch.bfloat16, 5)
    dev = ring_k.device
    _need(ring_v, "ring_v", torch.bfloat16, 5, dev)
    _need(pos, "pos", torch.int64, 1, dev)
    _need(k_new, "k_new", torch.bfloat16, 4, dev)
    _need(v_new, "v_new", torch.bfloat16, 4, dev)
    B, L, Hkv, W, d = ring_k.shape
    if ring_v.shape != ring_k.shape:
        raise ValueError("ring_v must have the shape of ring_k")
    if tuple(k_new.shape) != (B, L, Hkv, d) or tuple(v_new.shape) != (B, L, Hkv, d):
        raise ValueError(f"k_new/v_new must be {(B, L, Hkv, d)}")
    if int(pos.shape[0]) != B:
        raise ValueError("pos must be [B]")
    dims = CmcDims(B, L, Hkv, Hkv, d, 1, 0, W)
    st = lib().cmc_window_append(_p(ring_k), _p(ring_v), _p(pos), _p(k_new), _p(v_new),
                                 ctypes.byref(dims), _stream(dev))
    check(st, "cmc_window_append")


# ----------------------------------------------------------------------------
# The two-tier cache in 8 bits
# ----------------------------------------------------------------------------

_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice
_E4M3 = torch.float8_e4m3fn
_E8M0 = torch.float8_e8m0fnu


def q8_scale_bytes(rows: int) -> int:
    """Powers of two of an 8-bit cache of `rows` tokens, per (unit, K or V):
    4 ceil(rows / 128)."""
    return (rows + 127) // 128 * 4


def _need_q8(kv: torch.Tensor, scales: torch.Tensor, name: str, device) -> Tuple:
    """Checks an 8-bit cache; returns its shape."""
    _need(kv, name + "_kv", _E4M3, 6, device)
    _need(scales, name + "_scales", _E8M0, 5, device)
    shape = kv.shape
    if shape[3] != 2:
        raise ValueError(f"{name}_kv must be [B, L, Hkv, 2, T, d], got shape {tuple(shape)}")
    if scales.shape != (shape[0], shape[1], shape[2], 2, q8_scale_bytes(shape[4])):
        raise ValueError(f"{name}_scales shape {tuple(scales.shape)} does not go with {name}_kv "
                         f"{tuple(shape)}")
    return shape


def _need_new(k_new, v_new, want, dev) -> None:
    """Checks a new token's rows."""
    _need(k_new, "k_new", torch.bfloat16, 4, dev)
    _need(v_new, "v_new", torch.bfloat16, 4, dev)
    if k_new.shape != want or v_new.shape != want:
        raise ValueError(f"k_new/v_new must be {want}")


def _need_rows(idx, count, source, dim, dev) -> int:
    """Checks the row index and the token counts of a call; returns the rows
    (without an index all of `source`, whose dimension `dim` they are)."""
    B = source.shape[0]
    if count is not None:
        _need(count, "count", torch.int64, 1, dev)
        if count.shape[0] != B:
            raise ValueError("count must be [B]")
    if idx is None:
        return source.shape[dim]
    _need(idx, "idx", torch.int32, 2, dev)
    if idx.shape[0] != B:
        raise ValueError(f"idx shape {tuple(idx.shape)} does not match batch {B}")
    return idx.shape[1]


def _elsewhere(index: int, fn, *args) -> int:
    """Calls a library function with the tensors' device current (a launch goes to
    the current one)."""
    with torch.cuda.device(index):
        return fn(*args)


# Shapes that go together, and the sizes that they give: what a call can tell from
# its tensors' shapes alone is worked out once for each combination of them.  What
# is left for every call are the types, layouts and devices.  (The host side of a
# decode step's call takes longer than the GPU needs for some 60 MB of cache.)
_shapes_cache: Dict[Tuple, Tuple] = {}
_SHAPES_MOST = 4096  # combinations kept; beyond, each call works its own out


def _kept(key: Tuple, value: Tuple) -> Tuple:
    if len(_shapes_cache) < _SHAPES_MOST:
        _shapes_cache[key] = value
    return value


def _as(dtype: torch.dtype, index: int, *tensors) -> bool:
    """Whether all tensors (None: none) have this type and device and are contiguous.
    (Raises AttributeError for what is no tensor; a call then checks them one by one.)"""
    for t in tensors:
        if t is not None and (t.dtype is not dtype or t.get_device() != index
                              or not t.is_contiguous()):
            return False
    return True


@_ranged
def quantize_cache(k: torch.Tensor, v: torch.Tensor, idx: Optional[torch.Tensor] = None, *,
                   count: Optional[torch.Tensor] = None, out_kv: Optional[torch.Tensor] = None,
                   out_scales: Optional[torch.Tensor] = None,
                   workspace: Optional[DecodeWorkspace] = None
                   ) -> Tuple[torch.Tensor, torch.Tensor]:
    """An 8-bit cache (kv, scales) of rows of a bf16 bank or ring k, v [B, L, Hkv, N, d]:
    all N, or those that ``idx`` [B, k] names.  Rows from ``count[b]`` on (int64 [B]; a
    ring's pos will do) hold no token.  See cmc_quantize_cache.  Out-of-range
    indices raise DEVFLAG_BAD_INDEX in ``workspace``'s status word, and a copy that did not arrive in time
    DEVFLAG_TIMEOUT; without a workspace neither is reported."""
    _need(k, "k", torch.bfloat16, 5)
    dev = k.device
    index = dev.index
    if not isinstance(v, torch.Tensor) or not _as(torch.bfloat16, index, v) or v.shape != k.shape:
        _need(v, "v", torch.bfloat16, 5, dev)
        raise ValueError("v must have the shape of k")
    if workspace is not None and workspace.index != index:
        raise _elsewhere_workspace(workspace, index)
    rows = _need_rows(idx, count, k, 3, dev)
    key = ("quantize", k.shape, rows)
    kept = _shapes_cache.get(key)
    if kept is None:
        B, L, Hkv, N, d = k.shape
        dims = CmcDims(B, L, Hkv, Hkv, d, N, rows, 1)
        kept = _kept(key, ((B, L, Hkv, 2, rows, d), (B, L, Hkv, 2, q8_scale_bytes(rows)), dims,
                           ctypes.byref(dims)))
    shape, sshape, _, dims = kept
    given = out_kv is not None or out_scales is not None
    if out_kv is None:
        out_kv = torch.empty(shape, dtype=_E4M3, device=dev)
    if out_scales is None:
        out_scales = torch.empty(sshape, dtype=_E8M0, device=dev)
    if given and _need_q8(out_kv, out_scales, "out", dev) != shape:
        raise ValueError(f"out_kv must be {shape}")
    fn = lib().cmc_quantize_cache
    args = (k.data_ptr(), v.data_ptr(), _p(idx), _p(count), dims, out_kv.data_ptr(),
            out_scales.data_ptr(), 0 if workspace is None else workspace.ptr, _raw_stream(index))
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_quantize_cache")
    return out_kv, out_scales


@_ranged
def dequantize_cache(kv: torch.Tensor, scales: torch.Tensor, idx: Optional[torch.Tensor] = None, *,
                     out_k: Optional[torch.Tensor] = None, out_v: Optional[torch.Tensor] = None,
                     workspace: Optional[DecodeWorkspace] = None
                     ) -> Tuple[torch.Tensor, torch.Tensor]:
    """K and V of an 8-bit cache in bf16 [B, L, Hkv, rows, d]: all its rows, or
    those that ``idx`` [B, k] names.  See cmc_dequantize_cache."""
    _need(kv, "kv", _E4M3, 6)
    dev = kv.device
    index = dev.index
    if workspace is not None and workspace.index != index:
        raise _elsewhere_workspace(workspace, index)
    rows = _need_rows(idx, None, kv, 4, dev)
    kept = None
    if isinstance(scales, torch.Tensor) and _as(_E8M0, index, scales):
        key = ("dequantize", kv.shape, scales.shape, rows)
        kept = _shapes_cache.get(key)
    if kept is None:
        B, L, Hkv, _, N, d = _need_q8(kv, scales, "cache", dev)
        dims = CmcDims(B, L, Hkv, Hkv, d, N, rows, 1)
        kept = _kept(key, ((B, L, Hkv, rows, d), dims, ctypes.byref(dims)))
    want, _, dims = kept
    outs = []
    for t, name in ((out_k, "out_k"), (out_v, "out_v")):
        if t is None:
            t = torch.empty(want, dtype=torch.bfloat16, device=dev)
        else:
            _need(t, name, torch.bfloat16, 5, dev)
            if t.shape != want:
                raise ValueError(f"{name} must be {want}")
        outs.append(t)
    out_k, out_v = outs
    fn = lib().cmc_dequantize_cache
    args = (kv.data_ptr(), scales.data_ptr(), _p(idx), dims, out_k.data_ptr(), out_v.data_ptr(),
            0 if workspace is None else workspace.ptr, _raw_stream(index))
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_dequantize_cache")
    return out_k, out_v


@_ranged
def window_append_q8(ring_kv: torch.Tensor, ring_scales: torch.Tensor, pos: torch.Tensor,
                     k_new: torch.Tensor, v_new: torch.Tensor) -> None:
    """Append one token per sequence to an 8-bit ring, in place; see
    cmc_window_append_q8."""
    _need(ring_kv, "ring_kv", _E4M3, 6)
    dev = ring_kv.device
    index = dev.index
    kept = None
    try:
        if (_as(_E8M0, index, ring_scales) and _as(torch.int64, index, pos)
                and _as(torch.bfloat16, index, k_new, v_new)):
            key = ("append", ring_kv.shape, ring_scales.shape, pos.shape, k_new.shape, v_new.shape)
            kept = _shapes_cache.get(key)
    except AttributeError:
        pass
    if kept is None:
        B, L, Hkv, _, W, d = _need_q8(ring_kv, ring_scales, "ring", dev)
        _need(pos, "pos", torch.int64, 1, dev)
        if int(pos.shape[0]) != B:
            raise ValueError("pos must be [B]")
        _need_new(k_new, v_new, (B, L, Hkv, d), dev)
        dims = CmcDims(B, L, Hkv, Hkv, d, 1, 0, W)
        kept = _kept(key, (dims, ctypes.byref(dims)))
    fn = lib().cmc_window_append_q8
    args = (ring_kv.data_ptr(), ring_scales.data_ptr(), pos.data_ptr(), k_new.data_ptr(),
            v_new.data_ptr(), kept[1], _raw_stream(index))
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_window_append_q8")


def _attn_q8_dims(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, new) -> CmcDims:
    """Checks the tensors of an attention call over 8-bit caches one by one."""
    _need(q, "q", torch.bfloat16, 4)
    dev = q.device
    B, L, Hq, d = q.shape
    ring = _need_q8(ring_kv, ring_scales, "ring", dev)
    Hkv, W = ring[2], ring[4]
    k = 0
    if tier1_kv is not None or tier1_scales is not None:
        t1 = _need_q8(tier1_kv, tier1_scales, "tier1", dev)
        k = t1[4]
        if t1 != (B, L, Hkv, 2, k, d):
            raise ValueError(f"inconsistent shapes: q {tuple(q.shape)}, tier1_kv {tuple(t1)}, "
                             f"ring_kv {tuple(ring)}")
    if ring != (B, L, Hkv, 2, W, d):
        raise ValueError(f"inconsistent shapes: q {tuple(q.shape)}, ring_kv {tuple(ring)}")
    _need(pos, "pos", torch.int64, 1, dev)
    if int(pos.shape[0]) != B:
        raise ValueError(f"pos shape {tuple(pos.shape)} does not match batch {B}")
    if new is not None:
        _need_new(*new, (B, L, Hkv, d), dev)
    dims = CmcDims(B, L, Hq, Hkv, d, max(k, 1), k, W)
    if decode_attn_q8_workspace_size(dims) == 0:
        raise ValueError(f"unsupported dims {dims.key()}")
    return dims


def _attn_q8_kept(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, new, name) -> Tuple:
    """Checks the tensors of an attention call over 8-bit caches one by one; what the call keeps for
    shapes like these: (the library function, dims by reference, dims, the workspaces of its
    batch size by device and stream)."""
    dims = _attn_q8_dims(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, new)
    key = (q.shape, ring_kv.shape, ring_scales.shape, pos.shape,
           None if tier1_kv is None else tier1_kv.shape,
           None if tier1_scales is None else tier1_scales.shape)
    return _kept(key if new is None else key + (new[0].shape, new[1].shape),
                 (getattr(lib(), name), ctypes.byref(dims), dims,
                  _q8_workspaces.setdefault(dims.B, {})))


_q8_workspaces: Dict[int, Dict[Tuple[int, int], DecodeWorkspace]] = {}


def _attn_q8_workspace(kept: Dict, index: int, stream: int, dims: CmcDims) -> DecodeWorkspace:
    """A workspace for a call that is given none.  One is kept per stream and batch size; a call that
    is being captured gets one of its graph's own, since the kept ones are zero-filled
    once, outside of it, and other calls use them."""
    ws = DecodeWorkspace(dims, torch.device("cuda", index), q8=True)
    if not (stream and torch._C._cuda_isCurrentStreamCapturing()):
        kept[index, stream] = ws
    return ws


def decode_q8_status(device: Optional[torch.device] = None, clear: bool = True) -> int:
    """DEVFLAG_* bits that the attention calls over a cache in 8 bits which were given no ``workspace`` have
    raised on `device` (None: the current one) since the last clear; waits for all work on it.  Calls captured into a
    graph are not among them: give those a workspace to see theirs."""
    index = None if device is None else torch.device(device).index
    if index is None:
        index = torch.cuda.current_device()
    flags = 0
    with torch.cuda.device(index):
        torch.cuda.synchronize()
        for kept in list(_q8_workspaces.values()):
            for (i, _), ws in list(kept.items()):
                if i == index:
                    flags |= ws.status(clear)
        torch.cuda.synchronize()  # cleared before any stream's next call
    return flags


def _check_out(out: torch.Tensor, q: torch.Tensor) -> None:
    _need(out, "out", torch.bfloat16, 4, q.device)
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")


@_ranged
def two_tier_decode_attn_q8(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, *,
                            scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                            workspace: Optional[DecodeWorkspace] = None) -> torch.Tensor:
    """Decode attention over [Tier-1 | occupied ring slots], both caches in 8 bits
    (tier1_kv and tier1_scales None: the ring alone); see
    cmc_two_tier_decode_attn_q8.  Returns bf16 [B, L, Hq, d].  ``workspace`` is a
    DecodeWorkspace(dims, device, q8=True); without one the call keeps one per stream and
    batch size (see :func:`decode_q8_status`), and a captured call gets one of its own, zero-filled at every
    replay."""
    kept, index = None, -1
    try:
        index = q.get_device()
        if (index >= 0 and _as(torch.bfloat16, index, q) and _as(_E4M3, index, ring_kv, tier1_kv)
                and _as(_E8M0, index, ring_scales, tier1_scales) and _as(torch.int64, index, pos)):
            kept = _shapes_cache.get((q.shape, ring_kv.shape, ring_scales.shape, pos.shape,
                                      None if tier1_kv is None else tier1_kv.shape,
                                      None if tier1_scales is None else tier1_scales.shape))
    except AttributeError:
        pass
    if kept is None:
        kept = _attn_q8_kept(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, None,
                             "cmc_two_tier_decode_attn_q8")
    fn, ref, dims, workspaces = kept
    if out is None:
        out = torch.empty_like(q)
    else:
        _check_out(out, q)
    stream = _raw_stream(index)
    if workspace is None:
        # (the default stream, 0, is never captured)
        if not (stream and torch._C._cuda_isCurrentStreamCapturing()):
            workspace = workspaces.get((index, stream))
        if workspace is None:
            workspace = _attn_q8_workspace(workspaces, index, stream, dims)
    elif workspace.index != index:
        raise _elsewhere_workspace(workspace, index)
    args = (q.data_ptr(), 0 if tier1_kv is None else tier1_kv.data_ptr(),
            0 if tier1_scales is None else tier1_scales.data_ptr(), ring_kv.data_ptr(),
            ring_scales.data_ptr(), pos.data_ptr(), ref, 0.0 if scale is None else scale,
            out.data_ptr(), workspace.ptr, workspace.nbytes, stream)
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_two_tier_decode_attn_q8")
    return out


@_ranged
def decode_step_q8(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, k_new, v_new, *,
                   scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                   workspace: Optional[DecodeWorkspace] = None,
                   rope_theta: Optional[float] = None, rope_offset: int = 0) -> torch.Tensor:
    """Fused decode step over a cache in 8 bits: append (k_new, v_new) to the ring, then
    attend; see cmc_decode_step_q8.  Updates ring_kv, ring_scales and pos in place.
    ``rope_theta`` and ``rope_offset`` as for :func:`decode_step`, ``workspace`` as for
    :func:`two_tier_decode_attn_q8`."""
    if rope_theta is None:
        rope_theta = 0.0
    elif not rope_theta > 0:
        raise ValueError("rope_theta must be positive")
    kept, index = None, -1
    try:
        index = q.get_device()
        if (index >= 0 and _as(torch.bfloat16, index, q, k_new, v_new)
                and _as(_E4M3, index, ring_kv, tier1_kv)
                and _as(_E8M0, index, ring_scales, tier1_scales) and _as(torch.int64, index, pos)):
            kept = _shapes_cache.get((q.shape, ring_kv.shape, ring_scales.shape, pos.shape,
                                      None if tier1_kv is None else tier1_kv.shape,
                                      None if tier1_scales is None else tier1_scales.shape,
                                      k_new.shape, v_new.shape))
    except AttributeError:
        pass
    if kept is None:
        kept = _attn_q8_kept(q, tier1_kv, tier1_scales, ring_kv, ring_scales, pos, (k_new, v_new),
                             "cmc_decode_step_q8")
    fn, ref, dims, workspaces = kept
    if out is None:
        out = torch.empty_like(q)
    else:
        _check_out(out, q)
    stream = _raw_stream(index)
    if workspace is None:
        # (the default stream, 0, is never captured)
        if not (stream and torch._C._cuda_isCurrentStreamCapturing()):
            workspace = workspaces.get((index, stream))
        if workspace is None:
            workspace = _attn_q8_workspace(workspaces, index, stream, dims)
    elif workspace.index != index:
        raise _elsewhere_workspace(workspace, index)
    args = (q.data_ptr(), 0 if tier1_kv is None else tier1_kv.data_ptr(),
            0 if tier1_scales is None else tier1_scales.data_ptr(), ring_kv.data_ptr(),
            ring_scales.data_ptr(), pos.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), ref,
            0.0 if scale is None else scale, rope_theta, _offset(rope_offset), out.data_ptr(),
            workspace.ptr, workspace.nbytes, stream)
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_decode_step_q8")
    return out


def decode_attn_q8_plan(dims: CmcDims, fused: bool = True) -> int:
    """Grid size of the attention over a cache in 8 bits (always one kernel); see
    cmc_decode_attn_q8_plan."""
    ctas = ctypes.c_int(0)
    check(lib().cmc_decode_attn_q8_plan(ctypes.byref(dims), 1 if fused else 0, ctypes.byref(ctas)),
          "cmc_decode_attn_q8_plan")
    return int(ctas.value)


# ----------------------------------------------------------------------------
# Prefill into the cache, weights of its tokens, eviction by weight
# ----------------------------------------------------------------------------

_F32 = torch.float32
_byref = ctypes.byref
_weighted_workspaces: Dict[int, Dict[Tuple[int, int], DecodeWorkspace]] = {}


def _int32(x: int) -> int:
    """For the library: what it refuses stays refused, where ctypes would cut it to 32 bits."""
    return x if 0 <= x < 1 << 31 else -1


def _kept_workspaces(dims: CmcDims) -> Dict:
    """The workspaces that calls of this batch size choose themselves, by device and stream."""
    return _weighted_workspaces.setdefault(dims.B, {})


def _new_workspace(dims: CmcDims, index: int, before: Optional[DecodeWorkspace]) -> DecodeWorkspace:
    """A workspace whose flags and counters are those of the one `before`, or zero; what lies behind them, the products of
    long units, may hold anything."""
    ws = DecodeWorkspace.__new__(DecodeWorkspace)
    ws._set(dims, torch.empty(decode_attn_weighted_workspace_size(dims), dtype=torch.uint8,
                              device=torch.device("cuda", index)))
    head = ws.buf[:int(lib().cmc_cache_workspace_size(dims.B))]
    head.zero_() if before is None else head.copy_(before.buf[:head.numel()])
    return ws


def _own_workspace(kept: Dict, index: int, stream: int, dims: CmcDims, need: int) -> DecodeWorkspace:
    """A workspace of `need` bytes for a call that is given none.  One is kept per batch size and stream, and replaced by
    a larger one where a call's units are too long for it; a call that is being captured gets one of its graph's
    own, since the kept ones are zeroed once, outside of it, and other calls use them.  (The
    default stream, 0, is never captured.)"""
    if stream and torch._C._cuda_isCurrentStreamCapturing():
        return _new_workspace(dims, index, None)
    ws = kept.get((index, stream))
    if ws is None or ws.nbytes < need:
        ws = kept[index, stream] = _new_workspace(dims, index, ws)
    return ws


def weighted_cache_status(device: Optional[torch.device] = None, clear: bool = True) -> int:
    """DEVFLAG_* bits that the calls of this section which were given no ``workspace`` have raised on
    `device` (None: the current one) since the last clear; waits for all work on it.  Calls captured
    into a graph are not among them: give those a workspace to see theirs."""
    index = None if device is None else torch.device(device).index
    if index is None:
        index = torch.cuda.current_device()
    flags = 0
    with torch.cuda.device(index):
        torch.cuda.synchronize()
        for kept in list(_weighted_workspaces.values()):
            for (i, _), ws in list(kept.items()):
                if i == index:
                    flags |= ws.status(clear)
        torch.cuda.synchronize()  # cleared before any stream's next call
    return flags


def _prep(q_weight, k_weight, eps, rope_theta, rope_offset, evicted, B, L, d, dev):
    """The cmc_qk_prep of a call, by reference, or None for neither norm nor rotation."""
    if rope_theta is None:
        if q_weight is None and k_weight is None:
            return None
        rope_theta = 0.0
    elif not rope_theta > 0:
        raise ValueError("rope_theta must be positive")
    qw = kw = moved = 0
    if q_weight is not None:
        _need(q_weight, "q_weight", _F32, 2, dev)
        if q_weight.shape != (L, d):
            raise ValueError(f"q_weight must be {(L, d)}")
        qw = q_weight.data_ptr()
    if k_weight is not None:
        _need(k_weight, "k_weight", _F32, 2, dev)
        if k_weight.shape != (L, d):
            raise ValueError(f"k_weight must be {(L, d)}")
        kw = k_weight.data_ptr()
    if evicted is not None:
        _need_evicted(evicted, B, dev)
        moved = evicted.data_ptr()
    return _byref(CmcQkPrep(qw, kw, moved, rope_theta, _offset(rope_offset), eps))


def _need_evicted(evicted, B, dev) -> None:
    _need(evicted, "evicted", torch.int64, 1, dev)
    if evicted.shape[0] != B:
        raise ValueError("evicted must be [B]")


def _need_tokens(t, name, B, L, T, d, dev) -> Tuple[int, int]:
    """Checks the heads of T tokens, bf16 [B, L, T, H, d] (or, with T = 1, [B, L, H, d]): (H, elements from one
    token to the next).  Only a token's heads need be dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not torch.bfloat16 or t.device != dev:
        _need(t, name, torch.bfloat16, 5, dev)
    shape = t.shape if t.dim() == 5 else t.shape[:2] + (1,) + t.shape[2:]
    if t.dim() not in (4, 5) or shape[:3] != (B, L, T) or shape[4] != d:
        raise ValueError(f"{name} must be [{B}, {L}, {T}, heads, {d}], got shape {tuple(t.shape)}")
    stride = t.stride() if t.dim() == 5 else t.stride()[:2] + (0,) + t.stride()[2:]
    H = shape[3]
    step = None  # from one token to the next: that of the innermost dimension with several
    below = 1
    for n, s in ((T, stride[2]), (L, stride[1]), (B, stride[0])):
        if n > 1:
            if step is None:
                step = s // below if s % below == 0 else -1
            if s != step * below:
                step = -1
                break
            below *= n
    if step is None:
        step = H * d
    if (d > 1 and stride[4] != 1) or (H > 1 and stride[3] != d) or step < H * d:
        raise ValueError(f"{name}: a token's heads must be dense and tokens evenly spaced, got strides {t.stride()}")
    return H, step


def _tokens_like(t, shape, name, dev, given):
    """The output of a call for heads of `shape`: the tensor given, checked, or a new one."""
    if given is None:
        return torch.empty_like(t) if t.is_contiguous() else torch.empty(shape, dtype=torch.bfloat16, device=dev)
    _need(given, name, torch.bfloat16, len(shape), dev)
    if given.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}")
    return given


def _token_sizes(t, name) -> Tuple[int, int, int, int]:
    """(B, L, T, d) of the heads of tokens, [B, L, T, H, d] or [B, L, H, d]."""
    if not isinstance(t, torch.Tensor) or t.dim() not in (4, 5):
        _need(t, name, torch.bfloat16, 5)
    if t.dim() == 5:
        B, L, T, _, d = t.shape
    else:
        (B, L, _, d), T = t.shape, 1
    return B, L, T, d


def _need_pos(pos, B, dev) -> None:
    _need(pos, "pos", torch.int64, 1, dev)
    if pos.shape[0] != B:
        raise ValueError(f"pos shape {tuple(pos.shape)} does not match batch {B}")


@_ranged
def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, pos: torch.Tensor, *,
                 q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, rope_theta: Optional[float] = None, rope_offset: int = 0,
                 evicted: Optional[torch.Tensor] = None, out_q: Optional[torch.Tensor] = None,
                 out_k: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """RMS norm (where gains q_weight, k_weight fp32 [L, d] are given) and rotary embedding (where
    rope_theta is) of query heads q [B, L, T, Hq, d] and key heads k [B, L, T, Hkv, d], or of one
    token's [B, L, H, d], at positions rope_offset + evicted[b] + pos[b] + t; see cmc_qk_norm_rope.  q and k
    may be parts of a projection's output.  Returns both, dense; out_q and out_k may be q and k."""
    B, L, T, d = _token_sizes(q, "q")
    dev = q.device
    index = dev.index
    if not isinstance(k, torch.Tensor):
        _need(k, "k", torch.bfloat16, 5)
    key = ("norm", q.shape, q.stride(), k.shape, k.stride())
    kept = _shapes_cache.get(key)
    if (kept is None or q.dtype is not torch.bfloat16 or k.dtype is not torch.bfloat16
            or k.get_device() != index):
        Hq, sq = _need_tokens(q, "q", B, L, T, d, dev)
        Hkv, sk = _need_tokens(k, "k", B, L, T, d, dev)
        dims = CmcDims(B, L, Hq, Hkv, d, 1, 0, 1)
        kept = _kept(key, (sq, sk, ctypes.byref(dims), dims))
    sq, sk, dims, _ = kept
    _need_pos(pos, B, dev)
    prep = _prep(q_weight, k_weight, eps, rope_theta, rope_offset, evicted, B, L, d, dev)
    out_q = _tokens_like(q, q.shape, "out_q", dev, out_q)
    out_k = _tokens_like(k, k.shape, "out_k", dev, out_k)
    fn = lib().cmc_qk_norm_rope
    args = (q.data_ptr(), sq, k.data_ptr(), sk, T, pos.data_ptr(), dims, prep, out_q.data_ptr(),
            out_k.data_ptr(), _raw_stream(index))
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_qk_norm_rope")
    return out_q, out_k


@_ranged
def window_prefill(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, ring_k: torch.Tensor,
                   ring_v: torch.Tensor, pos: torch.Tensor, *,
                   ring_weight: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                   q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                   eps: float = 1e-6, rope_theta: Optional[float] = None, rope_offset: int = 0,
                   evicted: Optional[torch.Tensor] = None, out_q: Optional[torch.Tensor] = None,
                   workspace: Optional[DecodeWorkspace] = None) -> Optional[torch.Tensor]:
    """Appends the first count[b] (int64 [B]; None: all) of T tokens k, v [B, L, T, Hkv, d] to the ring, in place, after the
    norm and rotation of :func:`qk_norm_rope`, and returns the queries q [B, L, T, Hq, d] likewise (None: no
    queries); see cmc_window_prefill.  The weights of the slots written become 0 (what the prompt's own queries give its
    tokens is for the caller to add).  Rows of the queries from count[b] on are not written (of a new tensor they are
    undefined)."""
    B, L, T, d = _token_sizes(k, "k")
    dev = k.device
    index = dev.index
    if not isinstance(v, torch.Tensor) or not isinstance(ring_k, torch.Tensor):
        _need(v, "v", torch.bfloat16, 5)
        _need(ring_k, "ring_k", torch.bfloat16, 5)
    if q is not None and not isinstance(q, torch.Tensor):
        _need(q, "q", torch.bfloat16, 5)
    key = ("prefill", None if q is None else q.shape, None if q is None else q.stride(), k.shape, k.stride(),
           v.shape, v.stride(), ring_k.shape)
    kept = _shapes_cache.get(key)
    if (kept is None or k.dtype is not torch.bfloat16 or v.dtype is not torch.bfloat16
            or v.get_device() != index
            or (q is not None and (q.dtype is not torch.bfloat16 or q.get_device() != index))):
        Hkv, sk = _need_tokens(k, "k", B, L, T, d, dev)
        Hv, sv = _need_tokens(v, "v", B, L, T, d, dev)
        if Hv != Hkv:
            raise ValueError("v must have the heads of k")
        Hq, sq = (Hkv, 0) if q is None else _need_tokens(q, "q", B, L, T, d, dev)
        _need(ring_k, "ring_k", torch.bfloat16, 5, dev)
        W = ring_k.shape[3]
        if ring_k.shape != (B, L, Hkv, W, d):
            raise ValueError(f"ring_k must be {(B, L, Hkv, W, d)}, got shape {tuple(ring_k.shape)}")
        dims = CmcDims(B, L, Hq, Hkv, d, 1, 0, W)
        own = CmcDims(B, 1, 1, 1, 64, 1, 0, 1)  # a workspace that goes by the batch size alone
        kept = _kept(key, (sq, sk, sv, ctypes.byref(dims), own, _kept_workspaces(own), dims))
    sq, sk, sv, ref, own, workspaces, _ = kept
    _need(ring_k, "ring_k", torch.bfloat16, 5, dev)
    _need(ring_v, "ring_v", torch.bfloat16, 5, dev)
    if ring_v.shape != ring_k.shape:
        raise ValueError("ring_v must have the shape of ring_k")
    _need_pos(pos, B, dev)
    if ring_weight is not None:
        _need_weight(ring_weight, "ring_weight", ring_k, dev)
    if count is not None:
        _need(count, "count", torch.int64, 1, dev)
        if count.shape[0] != B:
            raise ValueError("count must be [B]")
    prep = _prep(q_weight, k_weight, eps, rope_theta, rope_offset, evicted, B, L, d, dev)
    if q is not None:
        out_q = _tokens_like(q, q.shape, "out_q", dev, out_q)
    elif out_q is not None:
        raise ValueError("out_q without q")
    stream = _raw_stream(index)
    if workspace is None:
        workspace = _own_workspace(workspaces, index, stream, own, 0)
    elif workspace.index != index:
        raise _elsewhere_workspace(workspace, index)
    fn = lib().cmc_window_prefill
    args = (_p(q), sq, k.data_ptr(), sk, v.data_ptr(), sv, T, ring_k.data_ptr(), ring_v.data_ptr(),
            _p(ring_weight), pos.data_ptr(), _p(count), ref, prep, _p(out_q), workspace.ptr,
            workspace.nbytes, stream)
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_window_prefill")
    return out_q


def _need_weight(weight, name, rows, dev) -> None:
    """Checks the weights that go with rows [B, L, Hkv, T, d]."""
    _need(weight, name, _F32, 4, dev)
    if weight.shape != rows.shape[:4]:
        raise ValueError(f"{name} must be {tuple(rows.shape[:4])}, got shape {tuple(weight.shape)}")


def _weighted_kept(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v, ring_weight, pos, new, key) -> Tuple:
    """Checks the tensors of a weighted attention call one by one; what the call keeps for shapes like
    these: (dims by reference, dims, the workspaces by device and stream, the bytes of one)."""
    _need(q, "q", torch.bfloat16, 4)
    dev = q.device
    B, L, Hq, d = q.shape
    for t, name in ((ring_k, "ring_k"), (ring_v, "ring_v")):
        _need(t, name, torch.bfloat16, 5, dev)
    Hkv, W = ring_k.shape[2], ring_k.shape[3]
    if ring_k.shape != (B, L, Hkv, W, d) or ring_v.shape != ring_k.shape:
        raise ValueError(f"inconsistent shapes: q {tuple(q.shape)}, ring {tuple(ring_k.shape)}, "
                         f"{tuple(ring_v.shape)}")
    _need_weight(ring_weight, "ring_weight", ring_k, dev)
    k = 0
    if tier1_k is not None or tier1_v is not None or tier1_weight is not None:
        for t, name in ((tier1_k, "tier1_k"), (tier1_v, "tier1_v")):
            _need(t, name, torch.bfloat16, 5, dev)
        k = tier1_k.shape[3]
        if tier1_k.shape != (B, L, Hkv, k, d) or tier1_v.shape != tier1_k.shape:
            raise ValueError(f"inconsistent shapes: q {tuple(q.shape)}, tier1 {tuple(tier1_k.shape)}, "
                             f"{tuple(tier1_v.shape)}")
        _need_weight(tier1_weight, "tier1_weight", tier1_k, dev)
    _need_pos(pos, B, dev)
    if new is not None:
        _need_new(*new, (B, L, Hkv, d), dev)
    dims = CmcDims(B, L, Hq, Hkv, d, max(k, 1), k, W)
    need = decode_attn_weighted_workspace_size(dims)
    if need == 0:
        raise ValueError(f"unsupported dims {dims.key()}")
    kept = (ctypes.byref(dims), dims, _kept_workspaces(dims), need)
    return kept if key is None else _kept(key, kept)


def _weighted_call(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v, ring_weight, pos, new):
    """Checks of a weighted attention call, most of them once for each combination of shapes."""
    kept, key = None, None
    try:
        index = q.get_device()
        k_new, v_new = (None, None) if new is None else new
        if (index >= 0 and _as(torch.bfloat16, index, q, tier1_k, tier1_v, ring_k, ring_v, k_new, v_new)
                and _as(_F32, index, tier1_weight, ring_weight) and _as(torch.int64, index, pos)):
            key = ("weighted", q.shape, None if tier1_k is None else tier1_k.shape,
                   None if tier1_v is None else tier1_v.shape,
                   None if tier1_weight is None else tier1_weight.shape, ring_k.shape, ring_v.shape,
                   ring_weight.shape, pos.shape, None if new is None else (k_new.shape, v_new.shape))
            kept = _shapes_cache.get(key)
    except AttributeError:
        pass
    if kept is None:
        kept = _weighted_kept(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v, ring_weight, pos, new, key)
    return kept


@_ranged
def two_tier_decode_attn_weighted(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v, ring_weight, pos, *,
                                  scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                                  workspace: Optional[DecodeWorkspace] = None) -> torch.Tensor:
    """Decode attention over [Tier-1 | occupied ring slots] (tier1_* None: the ring alone) that adds to each
    key's weight, in place, the probabilities that its KV head's queries gave it; see
    cmc_two_tier_decode_attn_weighted.  Returns bf16 [B, L, Hq, d].  ``workspace`` is a DecodeWorkspace(dims,
    device, weighted=True); without one the call keeps one per batch size and stream, as large as the longest units have
    asked for (see :func:`weighted_cache_status`), and a captured call gets one of its own, its flags and counters
    zeroed at every replay."""
    ref, dims, workspaces, need = _weighted_call(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v,
                                                 ring_weight, pos, None)
    index = q.get_device()
    if out is None:
        out = torch.empty_like(q)
    else:
        _check_out(out, q)
    stream = _raw_stream(index)
    if workspace is None:
        workspace = _own_workspace(workspaces, index, stream, dims, need)
    elif workspace.index != index:
        raise _elsewhere_workspace(workspace, index)
    fn = lib().cmc_two_tier_decode_attn_weighted
    args = (q.data_ptr(), _p(tier1_k), _p(tier1_v), _p(tier1_weight), ring_k.data_ptr(), ring_v.data_ptr(),
            ring_weight.data_ptr(), pos.data_ptr(), ref, 0.0 if scale is None else scale, out.data_ptr(),
            workspace.ptr, workspace.nbytes, stream)
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_two_tier_decode_attn_weighted")
    return out


@_ranged
def decode_step_weighted(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v, ring_weight, pos, k_new, v_new, *,
                         scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                         workspace: Optional[DecodeWorkspace] = None,
                         q_weight: Optional[torch.Tensor] = None,
                         k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                         rope_theta: Optional[float] = None, rope_offset: int = 0,
                         evicted: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Fused decode step with weights: append (k_new, v_new), whose weight starts at 0, then attend as
    :func:`two_tier_decode_attn_weighted`; see cmc_decode_step_weighted.  Updates ring_k, ring_v, pos and the
    weights in place.  With q_weight, k_weight or rope_theta, q and k_new are given before the norm and
    rotation of :func:`qk_norm_rope`, at position rope_offset + evicted[b] + pos[b]."""
    ref, dims, workspaces, need = _weighted_call(q, tier1_k, tier1_v, tier1_weight, ring_k, ring_v,
                                                 ring_weight, pos, (k_new, v_new))
    index = q.get_device()
    prep = _prep(q_weight, k_weight, eps, rope_theta, rope_offset, evicted, dims.B, dims.L, dims.d, q.device)
    if out is None:
        out = torch.empty_like(q)
    else:
        _check_out(out, q)
    stream = _raw_stream(index)
    if workspace is None:
        workspace = _own_workspace(workspaces, index, stream, dims, need)
    elif workspace.index != index:
        raise _elsewhere_workspace(workspace, index)
    fn = lib().cmc_decode_step_weighted
    args = (q.data_ptr(), _p(tier1_k), _p(tier1_v), _p(tier1_weight), ring_k.data_ptr(), ring_v.data_ptr(),
            ring_weight.data_ptr(), pos.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), ref,
            0.0 if scale is None else scale, prep, out.data_ptr(), workspace.ptr, workspace.nbytes, stream)
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_decode_step_weighted")
    return out


def decode_attn_weighted_plan(dims: CmcDims, fused: bool = True) -> int:
    """Grid size of the weighted attention (always one kernel); see cmc_decode_attn_weighted_plan."""
    ctas = ctypes.c_int(0)
    check(lib().cmc_decode_attn_weighted_plan(ctypes.byref(dims), 1 if fused else 0, ctypes.byref(ctas)),
          "cmc_decode_attn_weighted_plan")
    return int(ctas.value)


def _evict_kept(k, v, weight, keep, pos, evicted, out_k, out_v, out_weight, out_pos, key) -> Tuple:
    """Checks the tensors of an eviction one by one; what the call keeps for shapes like these: (dims by
    reference, the dims of its workspace, the workspaces by device and stream, dims, the shapes of the outputs' rows and
    of the index)."""
    dev = k.device
    _need(v, "v", torch.bfloat16, 5, dev)
    if v.shape != k.shape:
        raise ValueError("v must have the shape of k")
    _need_weight(weight, "weight", k, dev)
    B, L, Hkv, T, d = k.shape
    keep = int(keep)
    if not 1 <= keep <= T:
        keep = -1  # refused by the library
    if pos is not None:
        _need_pos(pos, B, dev)
    if evicted is not None:
        _need_evicted(evicted, B, dev)
    if out_pos is not None:
        _need(out_pos, "out_pos", torch.int64, 1, dev)
        if out_pos.shape[0] != B:
            raise ValueError("out_pos must be [B]")
    given = [(t, name, dtype, ndim) for t, name, dtype, ndim in
             ((out_k, "out_k", torch.bfloat16, 5), (out_v, "out_v", torch.bfloat16, 5),
              (out_weight, "out_weight", _F32, 4)) if t is not None]
    for t, name, dtype, ndim in given:
        _need(t, name, dtype, ndim, dev)
    want = (B, L, Hkv, given[0][0].shape[3] if given else max(keep, 1), d)
    for t, name, _, ndim in given:
        if t.shape != want[:ndim]:
            raise ValueError(f"{name} must be {want[:ndim]}")
    dims = CmcDims(B, L, Hkv, Hkv, d, T, keep, want[3])
    own = CmcDims(B, 1, 1, 1, 64, 1, 0, 1)  # a workspace that goes by the batch size alone
    kept = (_byref(dims), own, _kept_workspaces(own), dims, want, (B, L, Hkv, max(keep, 0)))
    return kept if key is None else _kept(key, kept)


@_ranged
def evict_cache(k: torch.Tensor, v: torch.Tensor, weight: torch.Tensor, keep: int, *,
                pos: Optional[torch.Tensor] = None, recent: int = 0,
                evicted: Optional[torch.Tensor] = None, out_k: Optional[torch.Tensor] = None,
                out_v: Optional[torch.Tensor] = None, out_weight: Optional[torch.Tensor] = None,
                out_pos: Optional[torch.Tensor] = None, workspace: Optional[DecodeWorkspace] = None
                ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Keeps, of the tokens of a cache k, v [B, L, Hkv, T, d] (all T rows, or with ``pos`` a ring's), the ``recent``
    youngest and the heaviest others, ``keep`` in all for every unit, moved together in order of age; see
    cmc_evict_cache.  Returns (k, v, weight, idx, pos): the cache, by default new tensors of ``keep`` rows (rows that
    no token is kept for are not written), the rows kept, int32 [B, L, Hkv, keep] then -1, and the tokens
    that each sequence holds now, int64 [B].  ``out_k``, ``out_v``, ``out_weight`` may be larger than ``keep`` rows,
    or k, v and weight themselves (a ring that has not wrapped, or ends at its last row); ``out_pos`` may be
    pos.  ``evicted`` (int64 [B]) grows by the tokens taken out."""
    _need(k, "k", torch.bfloat16, 5)
    dev = k.device
    index = dev.index
    kept = key = None
    try:
        if (_as(torch.bfloat16, index, v, out_k, out_v) and _as(_F32, index, weight, out_weight)
                and _as(torch.int64, index, pos, evicted, out_pos)):
            key = ("evict", k.shape, v.shape, weight.shape, keep, None if out_k is None else out_k.shape,
                   None if out_v is None else out_v.shape, None if out_weight is None else out_weight.shape,
                   None if pos is None else pos.shape, None if evicted is None else evicted.shape,
                   None if out_pos is None else out_pos.shape)
            kept = _shapes_cache.get(key)
    except AttributeError:
        pass
    if kept is None:
        kept = _evict_kept(k, v, weight, keep, pos, evicted, out_k, out_v, out_weight, out_pos, key)
    ref, own, workspaces, _, want, idx_shape = kept
    if out_k is None:
        out_k = torch.empty(want, dtype=torch.bfloat16, device=dev)
    if out_v is None:
        out_v = torch.empty(want, dtype=torch.bfloat16, device=dev)
    if out_weight is None:
        out_weight = torch.empty(want[:4], dtype=_F32, device=dev)
    idx = torch.empty(idx_shape, dtype=torch.int32, device=dev)
    if out_pos is None:
        out_pos = torch.empty(k.shape[0], dtype=torch.int64, device=dev) if pos is None else torch.empty_like(pos)
    stream = _raw_stream(index)
    if workspace is None:
        workspace = _own_workspace(workspaces, index, stream, own, 0)
    elif workspace.index != index:
        raise _elsewhere_workspace(workspace, index)
    fn = lib().cmc_evict_cache
    args = (k.data_ptr(), v.data_ptr(), weight.data_ptr(), _p(pos), ref, _int32(int(recent)), out_k.data_ptr(),
            out_v.data_ptr(), out_weight.data_ptr(), idx.data_ptr(), out_pos.data_ptr(), _p(evicted),
            workspace.ptr, workspace.nbytes, stream)
    st = fn(*args) if index == _current_device() else _elsewhere(index, fn, *args)
    if st:
        check(st, "cmc_evict_cache")
    return out_k, out_v, out_weight, idx, out_pos


# ----------------------------------------------------------------------------
# Staging copies (host <-> device traffic of a decode loop)
# ----------------------------------------------------------------------------

@_ranged
def stage_copies(pairs, *, wait_first: bool = False, device: Optional[torch.device] = None) -> None:
    """Copy each (src, dst) tensor pair, byte for byte, in one kernel launch on
    the current stream; see cmc_stage_copies.  Host tensors must be pinned
    (their memory is then mapped for the device).  With wait_first=False the
    copies overlap the kernel before the call on the stream (the caller keeps
    that kernel off every source and destination) and the launch completes
    after it."""
    pairs = list(pairs)
    if len(pairs) > 4:
        raise ValueError("at most 4 copies per call")
    arr = (CmcCopy * max(1, len(pairs)))()
    dev = device
    for i, (src, dst) in enumerate(pairs):
        for t, name in ((src, "src"), (dst, "dst")):
            if not isinstance(t, torch.Tensor) or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous tensor")
            if not t.is_cuda and not t.is_pinned():
                raise ValueError(f"{name} must be a CUDA tensor or pinned host memory")
            if t.is_cuda:
                if dev is None:
                    dev = t.device
                elif t.device != dev:
                    raise ValueError("all device tensors must be on one device")
        nb = src.numel() * src.element_size()
        if dst.numel() * dst.element_size() != nb:
            raise ValueError("src and dst sizes differ")
        arr[i].src = src.data_ptr()
        arr[i].dst = dst.data_ptr()
        arr[i].bytes = nb
    if dev is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    st = lib().cmc_stage_copies(ctypes.cast(arr, ctypes.c_void_p), len(pairs),
                                1 if wait_first else 0, _stream(dev))
    check(st, "cmc_stage_copies")
