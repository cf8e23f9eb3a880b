"""Python binding of libsrt (include/srt.h): argument marshalling only.

Every function here has the name of the C entry point it calls, takes torch
tensors that already live on the GPU, passes their device pointers and the
current HIP stream, and raises ``SrtError`` on a non-zero status.  All work
is done by the HIP kernels in libsrt.so; there is no fallback: if the
library is missing, every call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import types
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsrt.so")

SRT_OK, SRT_ERR_INVALID, SRT_ERR_CAPACITY, SRT_ERR_HIP, SRT_ERR_UNSUPPORTED = 0, -1, -2, -3, -4
SRT_FLAG_CAPACITY, SRT_FLAG_STREAM, SRT_FLAG_PROMPT = 1, 2, 4
_NAMES = {SRT_ERR_INVALID: "SRT_ERR_INVALID", SRT_ERR_CAPACITY: "SRT_ERR_CAPACITY",
          SRT_ERR_HIP: "SRT_ERR_HIP", SRT_ERR_UNSUPPORTED: "SRT_ERR_UNSUPPORTED"}

# Every symbol include/srt.h declares.
EXPORTS = ("srt_trie_workspace_bytes", "srt_trie_init", "srt_trie_insert", "srt_trie_reset_streams",
           "srt_trie_status", "srt_trie_export", "srt_draft", "srt_tree_attn_scratch_bytes",
           "srt_tree_attn", "srt_accept_scratch_bytes", "srt_accept", "srt_accept_lmhead_scratch_bytes",
           "srt_accept_lmhead", "srt_commit", "srt_version", "srt_accept_noalloc",
           "srt_tree_attn_quant_scratch_bytes", "srt_tree_attn_quant", "srt_kv_append", "srt_commit_quant",
           "srt_kv_read", "srt_accept_rules", "srt_seen_add")
SRT_ACCEPT_NOALLOC_MAX_BATCH = 4096  # include/srt.h


class SrtError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed: {_NAMES.get(status, status)}")
        self.status = status


class TrieConfig(ctypes.Structure):
    _fields_ = [("n_prompts", ctypes.c_int32), ("max_streams", ctypes.c_int32),
                ("max_depth", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("node_capacity", ctypes.c_int64)]


class DraftParams(ctypes.Structure):
    _fields_ = [("max_match", ctypes.c_int32), ("max_nodes", ctypes.c_int32),
                ("max_depth", ctypes.c_int32), ("chain", ctypes.c_int32),
                ("budget_alpha", ctypes.c_double), ("min_score", ctypes.c_double)]


class KvQuantArgs(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_int32) for k in ("kv_type", "Hkv", "d", "page", "max_pages", "reserved")] +
                [("num_pages", ctypes.c_int64)] +
                [(k, ctypes.c_void_p) for k in ("k_pages", "v_pages", "k_scale", "v_scale", "k_tail", "v_tail",
                                                "block_table", "ctx_len")])


class RulesArgs(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("seen", "repetition", "frequency", "presence", "bias_offsets",
                                                "bias_tokens", "bias_values", "mask")] +
                [("n_bias", ctypes.c_int32), ("reserved", ctypes.c_int32)])


_lib = None
_P, _I32, _I64, _SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t


def lib() -> ctypes.CDLL:
    """The loaded libsrt.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built (run __graft_entry__.build())")
        L = ctypes.CDLL(LIB_PATH)
        sig = {
            "srt_trie_workspace_bytes": (_SZ, [ctypes.POINTER(TrieConfig)]),
            "srt_trie_init": (ctypes.c_int, [_P, _SZ, ctypes.POINTER(TrieConfig), _P]),
            "srt_trie_insert": (ctypes.c_int, [_P, _I32, _P, _P, _P, _P, _I32, _P]),
            "srt_trie_reset_streams": (ctypes.c_int, [_P, _I32, _P, _P]),
            "srt_trie_status": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_int64), _P]),
            "srt_trie_export": (ctypes.c_int, [_P, _I32, _I64, _P, _P, _P, ctypes.POINTER(ctypes.c_int64), _P]),
            "srt_draft": (ctypes.c_int, [_P, _I32, _P, _P, _P, ctypes.POINTER(DraftParams), _P, _P, _P, _P, _P, _P]),
            "srt_tree_attn_scratch_bytes": (_SZ, [_I32] * 7),
            "srt_tree_attn": (ctypes.c_int, [_I32] * 7 + [_I64] + [_P] * 7 + [ctypes.c_float, _P, _P, _SZ, _P]),
            "srt_accept_scratch_bytes": (_SZ, [_I32]),
            "srt_accept": (ctypes.c_int, [_I32] * 4 + [_P, _P, ctypes.c_float] + [_P] * 7 + [_P, _SZ, _P]),
            "srt_accept_noalloc": (ctypes.c_int, [_I32] * 4 + [_P, _P, ctypes.c_float] + [_P] * 7 + [_P]),
            "srt_accept_lmhead_scratch_bytes": (_SZ, [_I32, _I32, _I32]),
            "srt_accept_lmhead": (ctypes.c_int, [_I32] * 5 + [_P, _P, _P, ctypes.c_float] + [_P] * 7 + [_P, _SZ, _P]),
            "srt_commit": (ctypes.c_int, [_I32] * 6 + [_I64] + [_P] * 4 + [_I32] + [_P] * 3 + [_I32, _P, _P, _P]),
            "srt_tree_attn_quant_scratch_bytes": (_SZ, [ctypes.POINTER(KvQuantArgs)] + [_I32] * 3),
            "srt_tree_attn_quant": (ctypes.c_int, [ctypes.POINTER(KvQuantArgs)] + [_I32] * 3 + [_P] * 3 + [_I64, _P, _P] +
                                    [ctypes.c_float, _P, _P, _SZ, _P]),
            "srt_kv_append": (ctypes.c_int, [ctypes.POINTER(KvQuantArgs), _I32, _I32, _P, _P, _I64, _P, _P]),
            "srt_commit_quant": (ctypes.c_int, [ctypes.POINTER(KvQuantArgs), _I32, _I32, _P, _P, _I64, _I32] + [_P] * 3 +
                                 [_I32] + [_P] * 3),
            "srt_kv_read": (ctypes.c_int, [ctypes.POINTER(KvQuantArgs), _I32, _I32] + [_P] * 4),
            "srt_accept_rules": (ctypes.c_int, [_I32] * 4 + [_P, _P, ctypes.c_float, ctypes.POINTER(RulesArgs)] +
                                 [_P] * 8 + [_SZ, _P]),
            "srt_seen_add": (ctypes.c_int, [_P, _I32, _I32, _P, _P, _I32, _I32, _I32, _P]),
            "srt_version": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def _check(fn: str, st: int):
    if st != SRT_OK:
        raise SrtError(fn, st)


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _on(stream):
    """Context in which buffers the binding allocates for a call belong to
    the stream the call is enqueued on: torch's caching allocator then never
    hands them out again while that stream may still use them."""
    return torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext()


def _scratch_call(fn: str, call, scratch, need: int, device, stream):
    """call(scratch) with the caller's buffer if there is one and the library
    takes it (it says so before anything is enqueued), else with one of
    ``need`` bytes."""
    st = SRT_ERR_CAPACITY if scratch is None else call(scratch)
    if st == SRT_ERR_CAPACITY and (scratch is None or scratch.numel() < need):
        with _on(stream):
            scratch = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
        st = call(scratch)
    _check(fn, st)


def _ptr(t: Optional[torch.Tensor], dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


# --------------------------------------------------------------------------- cache

def srt_trie_workspace_bytes(n_prompts: int, max_streams: int, max_depth: int, node_capacity: int) -> int:
    cfg = TrieConfig(n_prompts, max_streams, max_depth, 0, node_capacity)
    return int(lib().srt_trie_workspace_bytes(ctypes.byref(cfg)))


def srt_trie_init(ws: torch.Tensor, n_prompts: int, max_streams: int, max_depth: int, node_capacity: int,
                  stream=None):
    cfg = TrieConfig(n_prompts, max_streams, max_depth, 0, node_capacity)
    _check("srt_trie_init", lib().srt_trie_init(_ptr(ws, torch.uint8, "ws"), ws.numel(), ctypes.byref(cfg),
                                               _stream(stream)))


def srt_trie_insert(ws: torch.Tensor, prompt_ids, stream_ids, tokens, lengths, stream=None):
    n = int(prompt_ids.numel())
    stride = int(tokens.shape[1]) if tokens.dim() == 2 else max(1, int(tokens.numel()))
    _check("srt_trie_insert", lib().srt_trie_insert(
        _ptr(ws, torch.uint8, "ws"), n, _ptr(prompt_ids, torch.int32, "prompt_ids"),
        _ptr(stream_ids, torch.int32, "stream_ids"), _ptr(tokens, torch.int32, "tokens"),
        _ptr(lengths, torch.int32, "lengths"), stride, _stream(stream)))


def srt_trie_reset_streams(ws: torch.Tensor, stream_ids, stream=None):
    _check("srt_trie_reset_streams", lib().srt_trie_reset_streams(
        _ptr(ws, torch.uint8, "ws"), int(stream_ids.numel()), _ptr(stream_ids, torch.int32, "stream_ids"),
        _stream(stream)))


def srt_trie_status(ws: torch.Tensor, stream=None) -> dict:
    info = (ctypes.c_int64 * 4)()
    st = lib().srt_trie_status(_ptr(ws, torch.uint8, "ws"), info, _stream(stream))
    if st not in (SRT_OK, SRT_ERR_CAPACITY):
        raise SrtError("srt_trie_status", st)
    return {"flags": int(info[0]), "nodes": int(info[1]), "node_capacity": int(info[2]),
            "slots": int(info[3]), "status": st}


def srt_trie_export(ws: torch.Tensor, prompt_id: int, max_nodes: int, stream=None):
    """(parent, token, count) int64 numpy arrays of the prompt's cache, BFS order."""
    dev = ws.device
    parent = torch.empty(max(1, max_nodes), dtype=torch.int32, device=dev)
    token = torch.empty_like(parent)
    count = torch.empty_like(parent)
    n = ctypes.c_int64(0)
    st = lib().srt_trie_export(_ptr(ws, torch.uint8, "ws"), prompt_id, max_nodes, _ptr(parent), _ptr(token),
                               _ptr(count), ctypes.byref(n), _stream(stream))
    _check("srt_trie_export", st)
    k = n.value
    return (parent[:k].cpu().numpy().astype("int64"), token[:k].cpu().numpy().astype("int64"),
            count[:k].cpu().numpy().view("uint32").astype("int64"))


# --------------------------------------------------------------------------- draft

def srt_draft(ws: torch.Tensor, prompt_ids, ctx_tail, ctx_len, max_match: int, max_nodes: int, max_depth: int,
              budget_alpha: float = 0.0, out=None, stream=None, min_score: float = 0.0, chain: bool = False) -> dict:
    B = int(prompt_ids.numel())
    if ctx_tail.shape != (B, max_match):
        raise ValueError("ctx_tail must be [B, max_match]")
    dev = prompt_ids.device
    if out is None:
        with _on(stream):
            out = {k: torch.empty((B, max_nodes), dtype=torch.int32, device=dev)
                   for k in ("tree_tokens", "tree_parent", "tree_depth")}
            out["n_nodes"] = torch.empty(B, dtype=torch.int32, device=dev)
            out["match_len"] = torch.empty(B, dtype=torch.int32, device=dev)
    prm = DraftParams(max_match, max_nodes, max_depth, int(bool(chain)), float(budget_alpha), float(min_score))
    _check("srt_draft", lib().srt_draft(
        _ptr(ws, torch.uint8, "ws"), B, _ptr(prompt_ids, torch.int32, "prompt_ids"),
        _ptr(ctx_tail, torch.int32, "ctx_tail"), _ptr(ctx_len, torch.int32, "ctx_len"), ctypes.byref(prm),
        _ptr(out["tree_tokens"], torch.int32), _ptr(out["tree_parent"], torch.int32),
        _ptr(out["tree_depth"], torch.int32), _ptr(out["n_nodes"], torch.int32),
        _ptr(out["match_len"], torch.int32), _stream(stream)))
    return out


# --------------------------------------------------------------------------- attention

def srt_tree_attn_scratch_bytes(B: int, N: int, Hq: int, Hkv: int, d: int, page: int, max_pages: int) -> int:
    return int(lib().srt_tree_attn_scratch_bytes(B, N, Hq, Hkv, d, page, max_pages))


def srt_tree_attn(q, k_cache, v_cache, block_table, ctx_len, tree_parent, n_nodes, scale: float,
                  out=None, scratch=None, stream=None):
    """q [B,N,Hq,d] bf16; caches [P,Hkv,page,d] bf16; block_table [B,max_pages] int32."""
    B, N, Hq, d = q.shape
    P, Hkv, page, d2 = k_cache.shape
    if d2 != d or v_cache.shape != k_cache.shape:
        raise ValueError("cache shape mismatch")
    max_pages = int(block_table.shape[1])
    need = srt_tree_attn_scratch_bytes(B, N, Hq, Hkv, d, page, max_pages)
    if out is None:
        with _on(stream):
            out = torch.empty_like(q)
    args = (B, N, Hq, Hkv, d, page, max_pages, P, _ptr(q, torch.bfloat16, "q"),
            _ptr(k_cache, torch.bfloat16, "k_cache"), _ptr(v_cache, torch.bfloat16, "v_cache"),
            _ptr(block_table, torch.int32, "block_table"), _ptr(ctx_len, torch.int32, "ctx_len"),
            _ptr(tree_parent, torch.int32, "tree_parent"), _ptr(n_nodes, torch.int32, "n_nodes"), float(scale),
            _ptr(out, torch.bfloat16, "out"))
    _scratch_call("srt_tree_attn", lambda x: lib().srt_tree_attn(*args, _ptr(x, name="scratch"), x.numel(), _stream(stream)),
                  scratch, need, q.device, stream)
    return out


# --------------------------------------------------------------------------- acceptance

def _walk_outputs(B: int, max_depth: int, dev) -> dict:
    return {"n_accepted": torch.empty(B, dtype=torch.int32, device=dev),
            "out_tokens": torch.empty((B, max_depth + 1), dtype=torch.int32, device=dev),
            "out_nodes": torch.empty((B, max_depth + 1), dtype=torch.int32, device=dev),
            "n_emitted": torch.empty(B, dtype=torch.int32, device=dev)}


def _check_walk_outputs(out, B: int, max_depth: int):
    """The outputs of a walk are of its sizes (the kernels write all of them)."""
    for name, t, shape in _outputs_with_shapes(out, B, max_depth):
        if t.shape != shape:
            raise ValueError(f"out: {name} must be {list(shape)}")


def _check_walk_room(out, B: int, max_depth: int):
    """The outputs of a walk have room for what the kernels write."""
    for name, t, shape in _outputs_with_shapes(out, B, max_depth):
        if t.numel() < math.prod(shape):
            raise ValueError(f"out: {name} must be {list(shape)}")


def _outputs_with_shapes(out, B: int, max_depth: int):
    rows, table = (B,), (B, max_depth + 1)
    for name, shape in (("n_accepted", rows), ("out_tokens", table), ("out_nodes", table), ("n_emitted", rows)):
        t = out.get(name) if name == "n_emitted" else out[name]  # (that one is optional)
        if t is not None:
            yield name, t, shape


def srt_accept_scratch_bytes(B: int) -> int:
    return int(lib().srt_accept_scratch_bytes(B))


def srt_accept(logits, gumbel, inv_temperature: float, tree_tokens, tree_parent, n_nodes, max_depth: int,
               out=None, scratch=None, stream=None) -> dict:
    """logits [B,N,V] fp32; gumbel [B,max_depth+1,V] fp32 or None (greedy)."""
    B, N, V = logits.shape
    if gumbel is not None and tuple(gumbel.shape) != (B, max_depth + 1, V):
        raise ValueError("gumbel must be [B, max_depth+1, V]")
    dev = logits.device
    if out is not None:
        _check_walk_room(out, B, max_depth)
    need = srt_accept_scratch_bytes(B)
    with _on(stream):
        if out is None:
            out = _walk_outputs(B, max_depth, dev)
        if scratch is None or scratch.numel() < need:
            scratch = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    _check("srt_accept", lib().srt_accept(
        B, N, V, max_depth, _ptr(logits, torch.float32, "logits"), _ptr(gumbel, torch.float32, "gumbel"),
        float(inv_temperature), _ptr(tree_tokens, torch.int32, "tree_tokens"),
        _ptr(tree_parent, torch.int32, "tree_parent"), _ptr(n_nodes, torch.int32, "n_nodes"),
        _ptr(out["n_accepted"], torch.int32), _ptr(out["out_tokens"], torch.int32),
        _ptr(out["out_nodes"], torch.int32), _ptr(out.get("n_emitted"), torch.int32), _ptr(scratch, name="scratch"),
        scratch.numel(), _stream(stream)))
    return out


def srt_accept_noalloc(logits, gumbel, inv_temperature: float, tree_tokens, tree_parent, n_nodes, max_depth: int,
                       out, stream=None) -> dict:
    """srt_accept with the library's fixed per-device scratch array: the
    caller passes preallocated outputs (``out`` as srt_accept returns it) and
    nothing is allocated, here or in the library.  B <= 4096."""
    B, N, V = logits.shape
    if gumbel is not None and tuple(gumbel.shape) != (B, max_depth + 1, V):
        raise ValueError("gumbel must be [B, max_depth+1, V]")
    _check_walk_room(out, B, max_depth)
    _check("srt_accept_noalloc", lib().srt_accept_noalloc(
        B, N, V, max_depth, _ptr(logits, torch.float32, "logits"), _ptr(gumbel, torch.float32, "gumbel"),
        float(inv_temperature), _ptr(tree_tokens, torch.int32, "tree_tokens"),
        _ptr(tree_parent, torch.int32, "tree_parent"), _ptr(n_nodes, torch.int32, "n_nodes"),
        _ptr(out["n_accepted"], torch.int32), _ptr(out["out_tokens"], torch.int32),
        _ptr(out["out_nodes"], torch.int32), _ptr(out.get("n_emitted"), torch.int32), _stream(stream)))
    return out


def srt_accept_lmhead_scratch_bytes(B: int, N: int, V: int) -> int:
    return int(lib().srt_accept_lmhead_scratch_bytes(B, N, V))


def srt_accept_lmhead(hidden, w_head, gumbel, inv_temperature: float, tree_tokens, tree_parent, n_nodes,
                      max_depth: int, out=None, scratch=None, stream=None) -> dict:
    """hidden [B,N,d_model] bf16; w_head [V,d_model] bf16; gumbel [B,max_depth+1,V]
    fp32 or None (greedy).  Outputs as srt_accept."""
    B, N, dm = hidden.shape
    V, dm2 = w_head.shape
    if dm2 != dm:
        raise ValueError("w_head must be [V, d_model]")
    if gumbel is not None and tuple(gumbel.shape) != (B, max_depth + 1, V):
        raise ValueError("gumbel must be [B, max_depth+1, V]")
    if tuple(tree_tokens.shape) != (B, N) or tuple(tree_parent.shape) != (B, N):
        raise ValueError("tree arrays must be [B, N]")
    dev = hidden.device
    need = srt_accept_lmhead_scratch_bytes(B, N, V)
    if out is not None:
        _check_walk_room(out, B, max_depth)
    else:
        with _on(stream):
            out = _walk_outputs(B, max_depth, dev)
    args = (B, N, dm, V, max_depth, _ptr(hidden, torch.bfloat16, "hidden"), _ptr(w_head, torch.bfloat16, "w_head"),
            _ptr(gumbel, torch.float32, "gumbel"), float(inv_temperature),
            _ptr(tree_tokens, torch.int32, "tree_tokens"), _ptr(tree_parent, torch.int32, "tree_parent"),
            _ptr(n_nodes, torch.int32, "n_nodes"), _ptr(out["n_accepted"], torch.int32),
            _ptr(out["out_tokens"], torch.int32), _ptr(out["out_nodes"], torch.int32),
            _ptr(out.get("n_emitted"), torch.int32))
    _scratch_call("srt_accept_lmhead",
                  lambda x: lib().srt_accept_lmhead(*args, _ptr(x, name="scratch"), x.numel(), _stream(stream)),
                  scratch, need, dev, stream)
    return out


# --------------------------------------------------------------------------- commit

def srt_commit(k_cache, v_cache, block_table, ctx_len, n_accepted, out_tokens, out_nodes, n_nodes_max: int,
               ctx_tail=None, draft_len=None, stream=None):
    """Moves the accepted nodes' K/V into place and advances ctx_len (and, if
    given, ctx_tail [B, Qmax] / draft_len [B]) in place."""
    B = int(ctx_len.numel())
    P, Hkv, page, d = k_cache.shape
    if v_cache.shape != k_cache.shape:
        raise ValueError("cache shape mismatch")
    dmax = int(out_tokens.shape[1]) - 1
    qmax = int(ctx_tail.shape[1]) if ctx_tail is not None else 0
    _check("srt_commit", lib().srt_commit(
        B, int(n_nodes_max), Hkv, d, page, int(block_table.shape[1]), P,
        _ptr(k_cache, torch.bfloat16, "k_cache"), _ptr(v_cache, torch.bfloat16, "v_cache"),
        _ptr(block_table, torch.int32, "block_table"), _ptr(ctx_len, torch.int32, "ctx_len"), dmax,
        _ptr(n_accepted, torch.int32, "n_accepted"), _ptr(out_tokens, torch.int32, "out_tokens"),
        _ptr(out_nodes, torch.int32, "out_nodes"), qmax, _ptr(ctx_tail, torch.int32, "ctx_tail"),
        _ptr(draft_len, torch.int32, "draft_len"), _stream(stream)))


# --------------------------------------------------------------------------- 8-bit KV cache

KV_TYPES = {torch.float8_e4m3fn: 0, torch.int8: 1}  # SRT_KV_E4M3, SRT_KV_INT8


def _arg(t, dtype, device, name):
    """Address of a tensor of this type on this device, packed."""
    if t.dtype is not dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on {device}, got {t.dtype} on {t.device}")
    return t.data_ptr()


def _maybe(t, dtype, device, name):
    return None if t is None else _arg(t, dtype, device, name)


def _stream_of(device, stream):
    """The given stream, or the current one of the tensors' device."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device.index)


@contextlib.contextmanager
def _device(device):
    """The library's current device is the tensors' own."""
    if not device.type == "cuda":
        raise ValueError(f"the tensors must be CUDA (HIP) tensors, not on {device}")
    with torch.cuda.device(device) if device.index != torch.cuda.current_device() else contextlib.nullcontext():
        yield


def _on_device(device, call, *args):
    """call(*args) with the library's current device the tensors' own."""
    if device.index == torch._C._cuda_getDevice():
        return call(*args)
    with torch.cuda.device(device):
        return call(*args)


def _kept_tensor(i):
    """Tensor i of a handle; only itself can be assigned to it (as in ctx_len += 1)."""
    def assign(self, t):
        if t is not self._tensors[i]:
            raise AttributeError("the handle keeps the tensors that it is made of: make another one")
    return property(lambda self: self._tensors[i], assign)


class KvQuant:
    """A KV cache held in 8 bits (srt_kv_quant of include/srt.h): pages
    [P,Hkv,page,d] of torch.float8_e4m3fn or torch.int8, a scale for each page
    and KV head [P,Hkv] fp32, the open page of every sequence [B,Hkv,page,d]
    bf16, block_table [B,max_pages] and ctx_len [B] int32.  It keeps the tensors
    it is made of; they are updated in place, and are not to be replaced (another
    set of tensors is another cache)."""

    k_pages, v_pages, k_scale, v_scale, k_tail, v_tail, block_table, ctx_len = (_kept_tensor(i) for i in range(8))
    tensors = property(lambda self: self._tensors)

    def __init__(self, k_pages, v_pages, k_scale, v_scale, k_tail, v_tail, block_table, ctx_len):
        if k_pages.dim() != 4 or k_pages.dtype not in KV_TYPES:
            raise ValueError("k_pages must be [P, Hkv, page, d] of torch.float8_e4m3fn or torch.int8")
        P, Hkv, page, d = k_pages.shape
        B = int(ctx_len.numel())
        if v_pages.shape != k_pages.shape or tuple(k_scale.shape) != (P, Hkv) or v_scale.shape != k_scale.shape:
            raise ValueError("pages or scales: shape mismatch")
        if tuple(k_tail.shape) != (B, Hkv, page, d) or v_tail.shape != k_tail.shape:
            raise ValueError("tails must be [B, Hkv, page, d]")
        if block_table.dim() != 2 or block_table.shape[0] != B or ctx_len.dim() != 1:
            raise ValueError("block_table must be [B, max_pages], ctx_len [B]")
        self.B, self.num_pages, self.Hkv, self.page, self.d = B, P, Hkv, page, d
        self.max_pages, self.device = int(block_table.shape[1]), k_pages.device
        if self.device.type != "cuda":
            raise ValueError("k_pages must be a CUDA (HIP) tensor")
        self._tensors = (k_pages, v_pages, k_scale, v_scale, k_tail, v_tail, block_table, ctx_len)
        dtypes = (k_pages.dtype,) * 2 + (torch.float32,) * 2 + (torch.bfloat16,) * 2 + (torch.int32,) * 2
        names = [k for k, _ in KvQuantArgs._fields_[7:]]
        self._args = KvQuantArgs(KV_TYPES[k_pages.dtype], Hkv, d, page, self.max_pages, 0, P,
                                 *[_arg(t, x, self.device, n) for t, x, n in zip(self._tensors, dtypes, names)])
        self._ref = ctypes.byref(self._args)


def _new_rows(kv: KvQuant, k_new, v_new):
    """(T, elements from one token to the next) of new vectors [B,T,Hkv,d]:
    a token's heads side by side, sequences T tokens apart."""
    if (k_new.dim() != 4 or v_new.shape != k_new.shape or k_new.dtype is not torch.bfloat16 or
            v_new.dtype is not torch.bfloat16 or k_new.device != kv.device or v_new.device != kv.device):
        raise ValueError(f"k_new and v_new must be [B, T, Hkv, d] of bfloat16 on {kv.device}")
    B, T, H, d = k_new.shape
    if B != kv.B or H != kv.Hkv or d != kv.d or T < 1:
        raise ValueError("k_new and v_new must be [B, T, Hkv, d] of the cache's B, Hkv and d")
    lead = [_lead(x.stride(), B, T, H, d) for x in (k_new, v_new)]
    if lead[0] < 0 or lead[0] != lead[1]:
        raise ValueError("k_new and v_new must have the same strides: a token's heads side by side, sequences T tokens apart")
    return T, lead[0]


def _lead(s, B, T, H, d):
    ld = s[1] if T > 1 else s[0] if B > 1 else H * d
    return -1 if s[3] != 1 or (H > 1 and s[2] != d) or (B > 1 and s[0] != T * ld) or ld < H * d else ld


def srt_tree_attn_quant_scratch_bytes(kv: KvQuant, N: int, Hq: int) -> int:
    return int(lib().srt_tree_attn_quant_scratch_bytes(kv._ref, kv.B, N, Hq))


def srt_tree_attn_quant(q, kv: KvQuant, k_new, v_new, tree_parent, n_nodes, scale: float, out=None, scratch=None,
                        stream=None):
    """q [B,N,Hq,d] bf16; k_new, v_new [B,N,Hkv,d] bf16: the tree's own vectors."""
    N, ld = _new_rows(kv, k_new, v_new)
    B, dev = kv.B, kv.device
    if q.dim() != 4 or q.shape[0] != B or q.shape[1] != N or q.shape[3] != kv.d or (out is not None and
                                                                                     out.shape != q.shape):
        raise ValueError("q and out must be [B, N, Hq, d]")
    if tree_parent.shape != (B, N) or n_nodes.numel() != B:
        raise ValueError("tree_parent must be [B, N], n_nodes [B]")
    Hq = q.shape[2]
    if out is None:
        with _device(dev), _on(stream):
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if scratch is None:
        with _device(dev), _on(stream):
            scratch = torch.empty(srt_tree_attn_quant_scratch_bytes(kv, N, Hq), dtype=torch.uint8, device=dev)
    elif scratch.device != dev or not scratch.is_contiguous():
        raise ValueError(f"scratch must be a contiguous tensor on {dev}")
    args = (kv._ref, B, N, Hq, _arg(q, torch.bfloat16, dev, "q"), k_new.data_ptr(), v_new.data_ptr(), ld,
            _arg(tree_parent, torch.int32, dev, "tree_parent"), _arg(n_nodes, torch.int32, dev, "n_nodes"), scale,
            _arg(out, torch.bfloat16, dev, "out"))
    call = lambda x: _on_device(dev, lib().srt_tree_attn_quant, *args, x.data_ptr(), x.numel() * x.element_size(),
                                _stream_of(dev, stream))
    st = call(scratch)
    need = srt_tree_attn_quant_scratch_bytes(kv, N, Hq) if st == SRT_ERR_CAPACITY else 0
    if need > scratch.numel() * scratch.element_size():
        with _device(dev), _on(stream):
            st = call(torch.empty(need, dtype=torch.uint8, device=dev))
    _check("srt_tree_attn_quant", st)
    return out


def srt_kv_append(kv: KvQuant, k_new, v_new, counts, stream=None):
    """Appends the first counts[b] of the rows k_new, v_new [B,T,Hkv,d]; ctx_len grows in place."""
    T, ld = _new_rows(kv, k_new, v_new)
    if counts.numel() != kv.B:
        raise ValueError("counts must be [B]")
    _check("srt_kv_append", _on_device(
        kv.device, lib().srt_kv_append, kv._ref, kv.B, T, k_new.data_ptr(), v_new.data_ptr(), ld,
        _arg(counts, torch.int32, kv.device, "counts"), _stream_of(kv.device, stream)))


def srt_commit_quant(kv: KvQuant, k_new, v_new, n_accepted, out_tokens, out_nodes, ctx_tail=None, draft_len=None,
                     stream=None):
    """Appends the root and the accepted nodes of the tree whose vectors are
    k_new, v_new [B,N,Hkv,d]; advances ctx_len (and, if given, ctx_tail [B,Qmax]
    / draft_len [B]) in place."""
    N, ld = _new_rows(kv, k_new, v_new)
    B, dev, i32 = kv.B, kv.device, torch.int32
    if out_tokens.dim() != 2 or out_tokens.shape[0] != B or out_nodes.shape != out_tokens.shape:
        raise ValueError("out_tokens and out_nodes must be [B, Dmax + 1]")
    if n_accepted.numel() != B or (draft_len is not None and draft_len.numel() != B):
        raise ValueError("n_accepted and draft_len must be [B]")
    if ctx_tail is not None and (ctx_tail.dim() != 2 or ctx_tail.shape[0] != B):
        raise ValueError("ctx_tail must be [B, Qmax]")
    _check("srt_commit_quant", _on_device(
        dev, lib().srt_commit_quant, kv._ref, B, N, k_new.data_ptr(), v_new.data_ptr(), ld, out_tokens.shape[1] - 1,
        _arg(n_accepted, i32, dev, "n_accepted"), _arg(out_tokens, i32, dev, "out_tokens"),
        _arg(out_nodes, i32, dev, "out_nodes"), ctx_tail.shape[1] if ctx_tail is not None else 0,
        _maybe(ctx_tail, i32, dev, "ctx_tail"), _maybe(draft_len, i32, dev, "draft_len"), _stream_of(dev, stream)))


def srt_kv_read(kv: KvQuant, start, T: int, out=None, stream=None):
    """Positions start[b] .. start[b] + T - 1 as bf16 (k, v) [B,T,Hkv,d]; rows
    outside the context are left as they are (zero if ``out`` is not given)."""
    if start.numel() != kv.B or T < 1:
        raise ValueError("start must be [B], T >= 1")
    shape, dev = (kv.B, T, kv.Hkv, kv.d), kv.device
    if out is None:
        with _device(dev), _on(stream):
            out = [torch.zeros(shape, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    if len(out) != 2 or out[0].shape != shape or out[1].shape != shape:
        raise ValueError("out must be two tensors [B, T, Hkv, d]")
    _check("srt_kv_read", _on_device(
        dev, lib().srt_kv_read, kv._ref, kv.B, T, _arg(start, torch.int32, dev, "start"),
        _arg(out[0], torch.bfloat16, dev, "k_out"), _arg(out[1], torch.bfloat16, dev, "v_out"), _stream_of(dev, stream)))
    return out


# --------------------------------------------------------------------------- sampling rules

class Rules:
    """Sampling rules of a batch (srt_rules of include/srt.h), each optional:
    seen [B,V] int16 (the bits of the count words), repetition, frequency,
    presence [B] fp32, bias lists (bias_offsets [B+1] int32, bias_tokens int32,
    bias_values fp32), mask [B,N,ceil(V/32)] int32 (bits of allowed tokens).  It
    keeps the tensors it is made of; their contents may change between calls, the
    tensors themselves are not to be replaced."""

    _TYPES = {"seen": torch.int16, "repetition": torch.float32, "frequency": torch.float32, "presence": torch.float32,
              "bias_offsets": torch.int32, "bias_tokens": torch.int32, "bias_values": torch.float32,
              "mask": torch.int32}

    def __init__(self, **tensors):
        for name in tensors:
            if name not in self._TYPES:
                raise ValueError(f"no such rule: {name}")
        self.tensors = types.MappingProxyType({k: tensors.get(k) for k in self._TYPES})
        t = self.tensors
        has = [t[k] is not None for k in ("bias_offsets", "bias_tokens", "bias_values")]
        if any(has) != all(has):
            raise ValueError("bias lists need bias_offsets, bias_tokens and bias_values")
        if all(has) and t["bias_tokens"].numel() != t["bias_values"].numel():
            raise ValueError("bias_tokens and bias_values differ in length")
        n_bias = int(t["bias_tokens"].numel()) if all(has) else 0
        given = [x for x in t.values() if x is not None]
        self.device = given[0].device if given else None
        self._args = RulesArgs(*[_maybe(t[k], x, self.device, k) for k, x in self._TYPES.items()], n_bias, 0)
        self._ref = ctypes.byref(self._args)

    def check(self, B: int, N: int, V: int, device):
        if self.device is not None and self.device != device:
            raise ValueError(f"the rules are on {self.device}, not on {device}")
        want = {"seen": (B, V), "repetition": (B,), "frequency": (B,), "presence": (B,), "bias_offsets": (B + 1,),
                "mask": (B, N, (V + 31) // 32)}
        for name, shape in want.items():
            t = self.tensors[name]
            if t is not None and t.shape != shape:
                raise ValueError(f"{name} must be {list(shape)}")


def srt_accept_rules(logits, gumbel, inv_temperature: float, rules: Rules, tree_tokens, tree_parent, n_nodes,
                     max_depth: int, out=None, scratch=None, stream=None) -> dict:
    """srt_accept under sampling rules; a walk that finds every token forbidden
    ends with -1 and n_emitted = n_accepted."""
    B, N, V = logits.shape
    if gumbel is not None and gumbel.shape != (B, max_depth + 1, V):
        raise ValueError("gumbel must be [B, max_depth+1, V]")
    if tree_tokens.shape != (B, N) or tree_parent.shape != (B, N) or n_nodes.numel() != B:
        raise ValueError("tree arrays must be [B, N], n_nodes [B]")
    dev, f32, i32 = logits.device, torch.float32, torch.int32
    rules.check(B, N, V, dev)
    if out is not None:
        _check_walk_outputs(out, B, max_depth)
    if out is None or scratch is None or scratch.numel() * scratch.element_size() < srt_accept_scratch_bytes(B):
        with _device(dev), _on(stream):
            if out is None:
                out = _walk_outputs(B, max_depth, dev)
            if scratch is None or scratch.numel() * scratch.element_size() < srt_accept_scratch_bytes(B):
                scratch = torch.empty(max(srt_accept_scratch_bytes(B), 1), dtype=torch.uint8, device=dev)
    if scratch.device != dev or not scratch.is_contiguous():
        raise ValueError(f"scratch must be a contiguous tensor on {dev}")
    _check("srt_accept_rules", _on_device(
        dev, lib().srt_accept_rules, B, N, V, max_depth, _arg(logits, f32, dev, "logits"),
        _maybe(gumbel, f32, dev, "gumbel"), inv_temperature, rules._ref, _arg(tree_tokens, i32, dev, "tree_tokens"),
        _arg(tree_parent, i32, dev, "tree_parent"), _arg(n_nodes, i32, dev, "n_nodes"),
        _arg(out["n_accepted"], i32, dev, "n_accepted"), _arg(out["out_tokens"], i32, dev, "out_tokens"),
        _arg(out["out_nodes"], i32, dev, "out_nodes"), _maybe(out.get("n_emitted"), i32, dev, "n_emitted"),
        scratch.data_ptr(), scratch.numel() * scratch.element_size(), _stream_of(dev, stream)))
    return out


def srt_seen_add(seen, tokens, lengths, prompt: bool = False, reset: bool = False, stream=None):
    """Enters tokens [B,T] (the first lengths[b] of a row) into the count rows
    seen [B,V] int16, in place."""
    if seen.dim() != 2 or tokens.dim() != 2 or tokens.shape[0] != seen.shape[0] or lengths.numel() != seen.shape[0]:
        raise ValueError("seen must be [B, V], tokens [B, T], lengths [B]")
    dev = seen.device
    _check("srt_seen_add", _on_device(
        dev, lib().srt_seen_add, _arg(seen, torch.int16, dev, "seen"), seen.shape[0], seen.shape[1],
        _arg(tokens, torch.int32, dev, "tokens"), _arg(lengths, torch.int32, dev, "lengths"), tokens.shape[1],
        int(bool(prompt)), int(bool(reset)), _stream_of(dev, stream)))


def srt_version() -> str:
    return lib().srt_version().decode()
