"""LiteVLM select + prefill hot path on MI355X (gfx950).

Thin Python binding over the C ABI of liblitevlm.so: it checks tensor
placement and shapes, allocates outputs with PyTorch (device memory and the
current stream are all PyTorch provides) and passes raw pointers. Every step of
the path runs in the library's HIP kernels:

    psm_forward(...)       the Patch Selection Module's view logits from the query embeddings
    patch_select(...)      view selection and per-view patch masking
    token_score_topk(...)  visual-token scoring, top-k and gather compaction
    prefill_attn(...)      causal GQA prefill attention over the packed sequence
    decode_attn(...)       extend-one decode attention over the compacted KV cache
    tsm_qk(...)            the Token Selection Module's scoring q and k from hidden states
    cache4_append(...)     rows of K and V into a cache held in 4 bits (cache4_empty makes one,
                           cache4_read reads rows back)
    cache4_attn(...)       attention of each sample's newest tokens over that cache
    cache4_evict(...)      its rows of largest accumulated attention weight, in a new cache
    verify_draft(...)      drafted tokens against the target's probabilities
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence

import torch

from . import _abi
from ._abi import LiteVLMError, load  # noqa: F401

__all__ = ["patch_select", "token_score_topk", "select_score_topk", "prefill_attn", "decode_attn", "tsm_qk", "tsm_fold_gain",
           "gather_hidden", "psm_forward", "cache4_empty", "cache4_append", "cache4_read", "cache4_attn",
           "cache4_attn_workspace_bytes", "cache4_evict", "verify_draft", "verify_draft_workspace_bytes",
           "dtype_code",
           "workspace_bytes", "decode_workspace_bytes", "LiteVLMError", "load"]


def dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return _abi.F32
    if t == torch.bfloat16:
        return _abi.BF16
    if t in (torch.float8_e4m3fn, torch.uint8):
        return _abi.FP8_E4M3
    raise TypeError(f"unsupported dtype {t}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensors must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _stream(device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def patch_select(view_logit: torch.Tensor, view_offsets: Sequence[int], S: int,
                 w_lexical: float = 0.0, threshold: float = 0.5,
                 view_lexical: Optional[torch.Tensor] = None):
    """View selection + patch mask. view_logit: fp32 [B, N] on the GPU.
    Returns (view_keep uint8 [B,N], token_keep uint8 [B,S], n_visual_kept int32 [B])."""
    lib = load()
    B, N = view_logit.shape
    dev = view_logit.device
    view_keep = torch.empty((B, N), dtype=torch.uint8, device=dev)
    token_keep = torch.empty((B, S), dtype=torch.uint8, device=dev)
    n_vis = torch.empty((B,), dtype=torch.int32, device=dev)
    off = (ctypes.c_int32 * (N + 1))(*[int(x) for x in view_offsets])
    st = lib.litevlm_patch_select(B, N, S, off, _ptr(view_logit), _ptr(view_lexical),
                                  float(w_lexical), float(threshold), _ptr(view_keep),
                                  _ptr(token_keep), _ptr(n_vis), _stream(dev))
    _abi.check(st, "litevlm_patch_select")
    return view_keep, token_keep, n_vis


def workspace_bytes(B: int, S: int, V_full: int, Hq: int, Hkv: int, D: int,
                    query_rows: Optional[int] = None) -> int:
    if query_rows is None:
        return int(load().litevlm_token_score_topk_workspace(B, S, V_full, Hq, Hkv, D))
    return int(load().litevlm_token_score_topk_rows_workspace(B, S, V_full, Hq, Hkv, D, int(query_rows)))


def token_score_topk(q: torch.Tensor, k: torch.Tensor, v: Optional[torch.Tensor],
                     token_keep: Optional[torch.Tensor], keep_ratio: float, V_full: int,
                     softmax_scale: Optional[float] = None, q_scale: float = 1.0,
                     k_scale: float = 1.0, v_scale: float = 1.0, gather: bool = True,
                     workspace: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                     query_rows: Optional[int] = None, noalloc: bool = False) -> dict:
    """Scores, top-k and compaction. q: [B,S,Hq,D], k/v: [B,S,Hkv,D] (fp32, bf16 or
    E4M3 bytes). Returns a dict of device tensors: scores [B,V_full] fp32,
    kept_index [B*S] int32 (packed, valid up to cu_seqlens[B]), cu_seqlens [B+1],
    and when gather is set qc [B*S,Hq,D], kc/vc [B*S,Hkv,D] (valid rows likewise).
    ``out`` may supply preallocated tensors under the same keys (plus "workspace").
    query_rows = n scores with the last n text tokens as the only query rows
    (litevlm_token_score_topk_rows); None uses every text token. noalloc calls
    litevlm_token_score_topk_noalloc, whose workspace is the library's own
    device array (no workspace tensor is made or passed)."""
    lib = load()
    B, S, Hq, D = q.shape
    Hkv = k.shape[2]
    dev = q.device
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(D)
    o = dict(out or {})
    o.setdefault("scores", torch.empty((B, V_full), dtype=torch.float32, device=dev))
    o.setdefault("kept_index", torch.empty((B * S,), dtype=torch.int32, device=dev))
    o.setdefault("cu_seqlens", torch.empty((B + 1,), dtype=torch.int32, device=dev))
    if gather:
        o.setdefault("qc", torch.empty((B * S, Hq, D), dtype=q.dtype, device=dev))
        o.setdefault("kc", torch.empty((B * S, Hkv, D), dtype=k.dtype, device=dev))
        o.setdefault("vc", torch.empty((B * S, Hkv, D), dtype=v.dtype, device=dev))
    if noalloc:
        if query_rows is not None or workspace is not None:
            raise ValueError("the no-alloc call scores every text row and takes no workspace")
        st = lib.litevlm_token_score_topk_noalloc(
            dtype_code(q.dtype), B, S, V_full, Hq, Hkv, D, _ptr(q), _ptr(k), _ptr(v), float(softmax_scale),
            float(q_scale), float(k_scale), float(v_scale), _ptr(token_keep), float(keep_ratio),
            _ptr(o["scores"]), _ptr(o["kept_index"]), _ptr(o["cu_seqlens"]), _ptr(o.get("qc")),
            _ptr(o.get("kc")), _ptr(o.get("vc")), _stream(dev))
        _abi.check(st, "litevlm_token_score_topk_noalloc")
        return o
    nbytes = workspace_bytes(B, S, V_full, Hq, Hkv, D, query_rows)
    ws = workspace if workspace is not None else o.get("workspace")
    if ws is None:
        ws = torch.empty((max(nbytes, 1),), dtype=torch.uint8, device=dev)
    o["workspace"] = ws
    common = (_ptr(q), _ptr(k), _ptr(v), float(softmax_scale), float(q_scale), float(k_scale),
              float(v_scale), _ptr(token_keep), float(keep_ratio), _ptr(o["scores"]),
              _ptr(o["kept_index"]), _ptr(o["cu_seqlens"]), _ptr(o.get("qc")), _ptr(o.get("kc")),
              _ptr(o.get("vc")), _ptr(ws), ws.numel() * ws.element_size(), _stream(dev))
    if query_rows is None:
        st = lib.litevlm_token_score_topk(dtype_code(q.dtype), B, S, V_full, Hq, Hkv, D, *common)
        _abi.check(st, "litevlm_token_score_topk")
    else:
        st = lib.litevlm_token_score_topk_rows(dtype_code(q.dtype), B, S, V_full, Hq, Hkv, D,
                                               int(query_rows), *common)
        _abi.check(st, "litevlm_token_score_topk_rows")
    return o


def select_score_topk(view_logit: torch.Tensor, view_offsets: Sequence[int], q: torch.Tensor,
                      k: torch.Tensor, v: Optional[torch.Tensor], keep_ratio: float, V_full: int,
                      w_lexical: float = 0.0, threshold: float = 0.5,
                      view_lexical: Optional[torch.Tensor] = None, softmax_scale: Optional[float] = None,
                      q_scale: float = 1.0, k_scale: float = 1.0, v_scale: float = 1.0, gather: bool = True,
                      token_keep: bool = True, workspace: Optional[torch.Tensor] = None,
                      out: Optional[dict] = None) -> dict:
    """patch_select and token_score_topk in one call (litevlm_select_score_topk):
    the returned dict holds token_score_topk's tensors plus view_keep [B,N],
    n_visual_kept [B] and, when token_keep is set, the token mask [B,S]."""
    lib = load()
    B, S, Hq, D = q.shape
    Hkv = k.shape[2]
    N = view_logit.shape[1]
    dev = q.device
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(D)
    o = dict(out or {})
    o.setdefault("scores", torch.empty((B, V_full), dtype=torch.float32, device=dev))
    o.setdefault("kept_index", torch.empty((B * S,), dtype=torch.int32, device=dev))
    o.setdefault("cu_seqlens", torch.empty((B + 1,), dtype=torch.int32, device=dev))
    o.setdefault("view_keep", torch.empty((B, N), dtype=torch.uint8, device=dev))
    o.setdefault("n_visual_kept", torch.empty((B,), dtype=torch.int32, device=dev))
    if token_keep:
        o.setdefault("token_keep", torch.empty((B, S), dtype=torch.uint8, device=dev))
    if gather:
        o.setdefault("qc", torch.empty((B * S, Hq, D), dtype=q.dtype, device=dev))
        o.setdefault("kc", torch.empty((B * S, Hkv, D), dtype=k.dtype, device=dev))
        o.setdefault("vc", torch.empty((B * S, Hkv, D), dtype=v.dtype, device=dev))
    nbytes = workspace_bytes(B, S, V_full, Hq, Hkv, D)
    ws = workspace if workspace is not None else o.get("workspace")
    if ws is None:
        ws = torch.empty((max(nbytes, 1),), dtype=torch.uint8, device=dev)
    o["workspace"] = ws
    off = (ctypes.c_int32 * (N + 1))(*[int(x) for x in view_offsets])
    st = lib.litevlm_select_score_topk(
        dtype_code(q.dtype), B, S, V_full, Hq, Hkv, D, N, off, _ptr(view_logit), _ptr(view_lexical),
        float(w_lexical), float(threshold), _ptr(q), _ptr(k), _ptr(v), float(softmax_scale), float(q_scale),
        float(k_scale), float(v_scale), float(keep_ratio), _ptr(o["view_keep"]), _ptr(o.get("token_keep")),
        _ptr(o["n_visual_kept"]), _ptr(o["scores"]), _ptr(o["kept_index"]), _ptr(o["cu_seqlens"]),
        _ptr(o.get("qc")), _ptr(o.get("kc")), _ptr(o.get("vc")), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(dev))
    _abi.check(st, "litevlm_select_score_topk")
    return o


def prefill_attn(qc: torch.Tensor, kc: torch.Tensor, vc: torch.Tensor, cu_seqlens: torch.Tensor,
                 max_seqlen: int, B: Optional[int] = None, causal: bool = True,
                 softmax_scale: Optional[float] = None, q_scale: float = 1.0, k_scale: float = 1.0,
                 v_scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Causal GQA attention over packed sequences. qc: [rows,Hq,D], kc/vc: [rows,Hkv,D]
    with rows >= cu_seqlens[B]. Output [rows,Hq,D] in out_dtype (bf16 by default,
    fp32 for fp32 input); rows past cu_seqlens[B] are left untouched."""
    lib = load()
    rows, Hq, D = qc.shape
    Hkv = kc.shape[1]
    if B is None:
        B = cu_seqlens.numel() - 1
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(D)
    if out_dtype is None:
        out_dtype = torch.float32 if qc.dtype == torch.float32 else torch.bfloat16
    o = out if out is not None else torch.empty((rows, Hq, D), dtype=out_dtype, device=qc.device)
    st = lib.litevlm_prefill_attn(
        dtype_code(qc.dtype), dtype_code(o.dtype), B, Hq, Hkv, D, _ptr(qc), _ptr(kc), _ptr(vc),
        _ptr(cu_seqlens), int(max_seqlen), float(softmax_scale), float(q_scale), float(k_scale),
        float(v_scale), 1 if causal else 0, _ptr(o), _stream(qc.device))
    _abi.check(st, "litevlm_prefill_attn")
    return o


def decode_workspace_bytes(in_dtype: torch.dtype, B: int, Hq: int, Hkv: int, D: int,
                           max_seqlen: int) -> int:
    return int(load().litevlm_decode_attn_workspace(dtype_code(in_dtype), B, Hq, Hkv, D, int(max_seqlen)))


def decode_attn(q1: torch.Tensor, k1: torch.Tensor, v1: torch.Tensor, kc: torch.Tensor,
                vc: torch.Tensor, cu_seqlens: torch.Tensor, max_seqlen: int,
                softmax_scale: Optional[float] = None, q_scale: float = 1.0, k_scale: float = 1.0,
                v_scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
                out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One decode step per sample over the compacted cache. q1: [B,Hq,D], k1/v1:
    [B,Hkv,D] (the new token), kc/vc: [rows,Hkv,D] with rows >= cu_seqlens[B].
    Returns [B,Hq,D] in out_dtype (bf16 by default, fp32 for fp32 input)."""
    lib = load()
    B, Hq, D = q1.shape
    Hkv = k1.shape[1]
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(D)
    if out_dtype is None:
        out_dtype = torch.float32 if q1.dtype == torch.float32 else torch.bfloat16
    o = out if out is not None else torch.empty((B, Hq, D), dtype=out_dtype, device=q1.device)
    nbytes = decode_workspace_bytes(q1.dtype, B, Hq, Hkv, D, max_seqlen)
    ws = workspace if workspace is not None else torch.empty((max(nbytes, 1),), dtype=torch.uint8,
                                                             device=q1.device)
    st = lib.litevlm_decode_attn(
        dtype_code(q1.dtype), dtype_code(o.dtype), B, Hq, Hkv, D, _ptr(q1), _ptr(k1), _ptr(v1),
        _ptr(kc), _ptr(vc), _ptr(cu_seqlens), int(max_seqlen), float(softmax_scale), float(q_scale),
        float(k_scale), float(v_scale), _ptr(o), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(q1.device))
    _abi.check(st, "litevlm_decode_attn")
    return o


def tsm_fold_gain(w: torch.Tensor, gamma: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """bf16 w [rows, cols] times the fp32 gain gamma [cols] per column, rounded to bf16."""
    rows, cols = w.shape
    o = out if out is not None else torch.empty_like(w)
    st = load().litevlm_tsm_fold_gain(rows, cols, _ptr(w), _ptr(gamma), _ptr(o), _stream(w.device))
    _abi.check(st, "litevlm_tsm_fold_gain")
    return o


def tsm_qk(hidden: torch.Tensor, token_keep: Optional[torch.Tensor], V_full: int, w_q: torch.Tensor,
           w_k: torch.Tensor, Hq: int, Hkv: int, D: int, eps: float = 1e-5, rope_theta: float = 1e6,
           q: Optional[torch.Tensor] = None, k: Optional[torch.Tensor] = None):
    """Scoring queries (text rows) and keys (kept rows) of the Token Selection
    Module from bf16 hidden states [B,S,Dm]; w_q/w_k carry the folded RMS gain.
    Returns (q [B,S,Hq,D], k [B,S,Hkv,D]) in bf16; q's visual rows and the key
    rows of dropped tokens are untouched."""
    B, S, Dm = hidden.shape
    dev = hidden.device
    q = q if q is not None else torch.empty((B, S, Hq, D), dtype=torch.bfloat16, device=dev)
    k = k if k is not None else torch.empty((B, S, Hkv, D), dtype=torch.bfloat16, device=dev)
    st = load().litevlm_tsm_qk(B, S, V_full, Dm, Hq, Hkv, D, _ptr(hidden), _ptr(token_keep), _ptr(w_q),
                               _ptr(w_k), float(eps), float(rope_theta), _ptr(q), _ptr(k), _stream(dev))
    _abi.check(st, "litevlm_tsm_qk")
    return q, k


def gather_hidden(hidden: torch.Tensor, kept_index: torch.Tensor, cu_seqlens: torch.Tensor,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Packed copies of the kept rows of hidden [B,S,...] (rows cu_seqlens[b].. of the
    result for sample b): out [B*S, ...] with rows past cu_seqlens[B] untouched."""
    B, S = hidden.shape[0], hidden.shape[1]
    row_bytes = hidden[0, 0].numel() * hidden.element_size()
    o = out if out is not None else torch.empty((B * S,) + tuple(hidden.shape[2:]), dtype=hidden.dtype,
                                                device=hidden.device)
    st = load().litevlm_gather_hidden(B, S, row_bytes, _ptr(hidden), _ptr(kept_index), _ptr(cu_seqlens),
                                      _ptr(o), _stream(hidden.device))
    _abi.check(st, "litevlm_gather_hidden")
    return o


def psm_forward(emb: torch.Tensor, params: torch.Tensor, n_heads: int, d_ff: int, n_views: int,
                n_layers: int, out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """View logits [B, n_views] fp32 from fp32 token embeddings [B, T, d] and the
    flat fp32 parameter vector (order documented in include/litevlm.h)."""
    lib = load()
    B, T, d = emb.shape
    dev = emb.device
    o = out if out is not None else torch.empty((B, n_views), dtype=torch.float32, device=dev)
    if workspace is None:
        nbytes = int(lib.litevlm_psm_workspace(B, T, d, n_heads, d_ff))
        workspace = torch.empty((max(nbytes, 1),), dtype=torch.uint8, device=dev)
    st = lib.litevlm_psm_forward(B, T, d, n_heads, d_ff, n_views, n_layers, _ptr(emb), _ptr(params),
                                 params.numel(), _ptr(o), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(dev))
    _abi.check(st, "litevlm_psm_forward")
    return o


# ------------------------------------------------------------------ the 4-bit cache, drafted tokens

def _arg(name: str, t: torch.Tensor, dtype, shape: tuple, dev: int) -> int:
    """Address of an argument that has this type, shape and device index (-1: the host), densely laid out."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on device {dev}, got "
                     f"{t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}")


# the current stream's handle without a Stream object around it (1 us a call), the
# current device without a look whether there is one (0.2 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _enqueue(call: str, dev: int, *args) -> None:
    """Runs a call on the current stream of device `dev`, which need not be the current one."""
    if dev < 0:
        raise ValueError(f"{call}: tensors must live on the GPU")
    fn = getattr(load(), call)
    if dev == _current_device():
        st = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            st = fn(*args, _raw_stream(dev))
    if st:
        _abi.check(st, call)


def _float_code(name: str, t: torch.Tensor) -> int:
    if t.dtype is torch.bfloat16:
        return _abi.BF16
    if t.dtype is torch.float32:
        return _abi.F32
    raise TypeError(f"{name}: float32 or bfloat16 expected, got {t.dtype}")


_NO_WORKSPACE = 16  # what a workspace query answers for a call that needs none


def _workspace(t: Optional[torch.Tensor], dev: int) -> tuple:
    """Address and bytes of a workspace, if there is one."""
    if t is None:
        return None, 0
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on device {dev}, got one on {t.device}")
    return t.data_ptr(), t.nbytes


def _cache_shape(cache: torch.Tensor, D: int, dev: int):
    """(B, Hkv, cap) of a cache tensor of head dim D on device `dev`, and its address."""
    if D not in (64, 128):
        raise ValueError(f"head dim {D}: 64 or 128 expected")
    B, Hkv, n = cache.shape
    cap, rest = divmod(n, D + D // 16)
    if rest:
        raise ValueError(f"a cache of head dim {D} has {D + D // 16} bytes a position, not {n} for all of them")
    return B, Hkv, cap, _arg("cache", cache, torch.uint8, (B, Hkv, n), dev)


def cache4_empty(B: int, Hkv: int, D: int, cap: int, device="cuda") -> torch.Tensor:
    """A 4-bit cache of `cap` positions (a multiple of 32) for each sample and KV head: uint8
    [B, Hkv, cap * (D + D/16)], laid out as include/litevlm.h says; every value is 0."""
    n = int(load().litevlm_cache4_bytes(B, Hkv, D, cap))
    if n == 0:
        raise ValueError(f"no 4-bit cache for B={B} Hkv={Hkv} D={D} cap={cap}")
    return torch.zeros((B, Hkv, n // (B * Hkv)), dtype=torch.uint8, device=device)


def cache4_append(cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_new: torch.Tensor, start: torch.Tensor,
                  max_new: int, weight: Optional[torch.Tensor] = None) -> None:
    """Quantises packed rows k, v [rows,Hkv,D] (fp32 or bf16) into the cache: rows cu_new[b].. of
    sample b go to positions start[b].. (at most max_new a sample). weight [B,Hkv,cap] is set to
    0 at those positions."""
    rows, _, D = k.shape
    dev = cache.get_device()
    B, Hkv, cap, cptr = _cache_shape(cache, D, dev)
    shape = (rows, Hkv, D)
    # an empty tensor has no address; one that is never read stands in
    _enqueue("litevlm_cache4_append", dev, _float_code("k", k), B, Hkv, D, cap, max_new,
             _arg("k", k, k.dtype, shape, dev) or cptr, _arg("v", v, k.dtype, shape, dev) or cptr,
             _arg("cu_new", cu_new, torch.int32, (B + 1,), dev), _arg("start", start, torch.int32, (B,), dev), cptr,
             None if weight is None else _arg("weight", weight, torch.float32, (B, Hkv, cap), dev))


def cache4_read(cache: torch.Tensor, D: int, cu_rows: torch.Tensor, start: torch.Tensor, max_rows: int,
                rows: Optional[int] = None, dtype: torch.dtype = torch.bfloat16, out: Optional[tuple] = None):
    """The values of cached rows: rows cu_rows[b].. of the packed result are positions start[b]..
    of sample b. Returns (k, v) [rows,Hkv,D]; without `out` they have `rows` rows of `dtype`, and rows
    past cu_rows[B] are not written. `rows` is at least cu_rows[B]: the default, B * max_rows, is
    where no sample asks for more than max_rows."""
    dev = cache.get_device()
    B, Hkv, cap, cptr = _cache_shape(cache, D, dev)
    fresh = out is None
    if fresh:
        shape = (B * max_rows if rows is None else rows, Hkv, D)
        out = (torch.empty(shape, dtype=dtype, device=cache.device), torch.empty(shape, dtype=dtype, device=cache.device))
    k, v = out
    shape = (k.shape[0], Hkv, D)
    kptr, vptr = _arg("k", k, k.dtype, shape, dev), _arg("v", v, k.dtype, shape, dev)
    if shape[0] and not fresh:
        n, end = k.nbytes, cptr + B * Hkv * cap * (D + D // 16)
        if abs(kptr - vptr) < n or cptr < kptr + n and kptr < end or cptr < vptr + n and vptr < end:
            raise ValueError("out: k, v and the cache overlap")
    _enqueue("litevlm_cache4_read", dev, _float_code("k", k), B, Hkv, D, cap, max_rows, cptr,
             _arg("start", start, torch.int32, (B,), dev), _arg("cu_rows", cu_rows, torch.int32, (B + 1,), dev),
             kptr or cptr, vptr or cptr + 16)
    return k, v


def cache4_attn_workspace_bytes(dtype: torch.dtype, B: int, Hq: int, Hkv: int, D: int, max_q: int, max_len: int,
                                weight_rows: int = 0) -> int:
    return int(load().litevlm_cache4_attn_workspace(dtype_code(dtype), B, Hq, Hkv, D, max_q, max_len, weight_rows))


def cache4_attn(cache: torch.Tensor, q: torch.Tensor, cu_q: torch.Tensor, lengths: torch.Tensor, max_q: int,
                max_len: int, softmax_scale: Optional[float] = None, weight: Optional[torch.Tensor] = None,
                weight_out: Optional[torch.Tensor] = None, weight_rows: int = 0, out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the packed queries q [rows,Hq,D] (fp32 or bf16; those of sample b are its newest
    tokens, whose keys and values are in the cache) over the first lengths[b] cached rows. With
    weight_rows > 0, weight_out [B,Hkv,cap] = weight + the attention that each row receives from
    each sample's first weight_rows queries (weight None: 0; weight_out None: in place).
    Returns [rows,Hq,D] in q's type."""
    rows, Hq, D = q.shape
    dev = cache.get_device()
    B, Hkv, cap, cptr = _cache_shape(cache, D, dev)
    code = _float_code("q", q)
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(D)
    fresh = out is None
    if fresh:
        out = torch.empty_like(q)
    qptr, optr = _arg("q", q, q.dtype, (rows, Hq, D), dev), _arg("out", out, q.dtype, (rows, Hq, D), dev)
    win = wout = None
    if weight_rows:
        if weight is not None:
            win = _arg("weight", weight, torch.float32, (B, Hkv, cap), dev)
        if weight_out is None:
            if weight is None:
                raise ValueError("weight_rows > 0 needs weight or weight_out")
            wout = win
        else:
            wout = _arg("weight_out", weight_out, torch.float32, (B, Hkv, cap), dev)
    if rows and not fresh:
        n, nw = rows * Hq * D * (4 if code == _abi.F32 else 2), B * Hkv * cap * 4
        end = optr + n
        if (qptr < end and optr < qptr + n or cptr < end and optr < cptr + B * Hkv * cap * (D + D // 16)
                or wout is not None and (wout < end and optr < wout + nw
                                         or win is not None and win < end and optr < win + nw)):
            raise ValueError("out: overlaps q, the cache or a weight")
    if workspace is None:
        n = load().litevlm_cache4_attn_workspace(code, B, Hq, Hkv, D, max_q, max_len, weight_rows)
        if n > _NO_WORKSPACE:
            workspace = torch.empty((n,), dtype=torch.uint8, device=q.device)
    _enqueue("litevlm_cache4_attn", dev, code, B, Hq, Hkv, D, cap, max_q, max_len, weight_rows,
             qptr or cptr, _arg("cu_q", cu_q, torch.int32, (B + 1,), dev), cptr,
             _arg("lengths", lengths, torch.int32, (B,), dev), softmax_scale, optr or cptr + 16, win, wout,
             *_workspace(workspace, dev))
    return out


def cache4_evict(cache: torch.Tensor, D: int, weight: torch.Tensor, lengths: torch.Tensor, budget: int, recent: int,
                 max_len: int, cap_out: Optional[int] = None, out: Optional[dict] = None) -> dict:
    """Keeps at most `budget` rows of each sample and KV head: the last `recent` ones and those of
    largest weight [B,Hkv,cap]. Returns a dict of new tensors: cache (of cap_out positions, by
    default budget rounded up to 32), weight [B,Hkv,cap_out], lengths [B] and kept_index
    [B,Hkv,budget], all valid up to lengths[b]. ``out`` may supply them under the same keys."""
    dev, device = cache.get_device(), cache.device
    B, Hkv, cap, cptr = _cache_shape(cache, D, dev)
    o = dict(out or {})
    if "cache" not in o:
        o["cache"] = cache4_empty(B, Hkv, D, (budget + 31) // 32 * 32 if cap_out is None else cap_out, device)
    B2, H2, cap_out, optr = _cache_shape(o["cache"], D, dev)
    if (B2, H2) != (B, Hkv):
        raise ValueError(f"the new cache is for {B2} samples and {H2} heads, not {B} and {Hkv}")
    if "weight" not in o:
        o["weight"] = torch.empty((B, Hkv, cap_out), dtype=torch.float32, device=device)
    if "lengths" not in o:
        o["lengths"] = torch.empty((B,), dtype=torch.int32, device=device)
    if "kept_index" not in o:
        o["kept_index"] = torch.empty((B, Hkv, budget), dtype=torch.int32, device=device)
    _enqueue("litevlm_cache4_evict", dev, B, Hkv, D, cap, cap_out, max_len, budget, recent, cptr,
             _arg("weight", weight, torch.float32, (B, Hkv, cap), dev),
             _arg("lengths", lengths, torch.int32, (B,), dev), optr,
             _arg("out weight", o["weight"], torch.float32, (B, Hkv, cap_out), dev),
             _arg("out lengths", o["lengths"], torch.int32, (B,), dev),
             _arg("out kept_index", o["kept_index"], torch.int32, (B, Hkv, budget), dev))
    return o


def verify_draft_workspace_bytes(B: int, max_draft: int, V: int) -> int:
    return int(load().litevlm_verify_draft_workspace(B, max_draft, V))


def verify_draft(draft: torch.Tensor, target: torch.Tensor, proposal: Optional[torch.Tensor], u: torch.Tensor,
                 r: torch.Tensor, n_draft: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
                 out: Optional[dict] = None, workspace: Optional[torch.Tensor] = None) -> dict:
    """Drafted tokens draft [B,m] (int32) against target probabilities [B,m+1,V] (fp32 or bf16) and
    the draft model's [B,m,V] (None: the drafts were not drawn), with uniform numbers u [B,m] and
    r [B]. Returns a dict: tokens [B,m+1] (the accepted drafts, one drawn token, then -1),
    n_accepted [B] and, with `lengths`, lengths [B] without the refused drafts' rows. ``out`` may
    supply them under the same keys."""
    B, m = draft.shape
    V = target.shape[2]
    dev, device = draft.get_device(), draft.device
    code = _float_code("target", target)
    o = dict(out or {})
    if "tokens" not in o:
        o["tokens"] = torch.empty((B, m + 1), dtype=torch.int32, device=device)
    if "n_accepted" not in o:
        o["n_accepted"] = torch.empty((B,), dtype=torch.int32, device=device)
    lin = lout = None
    if lengths is not None:
        lin = _arg("lengths", lengths, torch.int32, (B,), dev)
        if "lengths" not in o:
            o["lengths"] = torch.empty((B,), dtype=torch.int32, device=device)
        lout = _arg("out lengths", o["lengths"], torch.int32, (B,), dev)
    if workspace is None:
        n = load().litevlm_verify_draft_workspace(B, m, V)
        if n > _NO_WORKSPACE:
            workspace = torch.empty((n,), dtype=torch.uint8, device=device)
    _enqueue("litevlm_verify_draft", dev, code, B, m, V, _arg("draft", draft, torch.int32, (B, m), dev),
             None if n_draft is None else _arg("n_draft", n_draft, torch.int32, (B,), dev),
             _arg("target", target, target.dtype, (B, m + 1, V), dev),
             None if proposal is None else _arg("proposal", proposal, target.dtype, (B, m, V), dev),
             _arg("u", u, torch.float32, (B, m), dev), _arg("r", r, torch.float32, (B,), dev), lin,
             _arg("out tokens", o["tokens"], torch.int32, (B, m + 1), dev),
             _arg("out n_accepted", o["n_accepted"], torch.int32, (B,), dev), lout, *_workspace(workspace, dev))
    return o
