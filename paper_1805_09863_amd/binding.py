"""ctypes binding of libkbest (the C ABI in include/kbest.h).

Argument marshalling only: every step of the output layer runs in the HIP
kernels of libkbest.  PyTorch supplies device memory and the current stream.
There is no fallback: if the library is missing, loading it raises.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkbest.so")

KB_OK, KB_ERR_INVALID_ARG, KB_ERR_UNSUPPORTED, KB_ERR_WORKSPACE, KB_ERR_HIP = range(5)
KB_F32, KB_BF16 = 0, 1
KB_MAX_K = 16

_lib = None

_P = ctypes.c_void_p
_I = ctypes.c_int
_SZ = ctypes.c_size_t

_F = ctypes.c_float
_L = ctypes.c_int64


class _Cache(ctypes.Structure):
    """kb_cache of include/kbest_cache.h."""
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("pages", ctypes.c_int32), ("seqs", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("k", _P), ("v", _P), ("table", _P)]


_C = ctypes.POINTER(_Cache)

# name -> (restype, argtypes), mirroring include/kbest.h, include/kbest_standin.h and include/kbest_cache.h
SIGNATURES = {
    "kb_abi_version": (_I, []),
    "kb_status_string": (ctypes.c_char_p, [_I]),
    "kb_last_error": (ctypes.c_char_p, []),
    "kb_kbest_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _I]),
    "kb_kbest_plan": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P]),
    "kb_kbest_step": (_I, [_I, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "kb_kbest_step_events": (_I, [_I, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ, _P,
                                  _P, _P]),
    "kb_kbest_step_scratch_max": (_SZ, []),
    "kb_kbest_step_noalloc": (_I, [_I, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "kb_argmax_workspace_bytes": (_SZ, [_I, _I, _I, _I]),
    "kb_argmax_step": (_I, [_I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "kb_unfused_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _I]),
    "kb_kbest_step_unfused": (_I, [_I, _I, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _SZ,
                                   _P, _I, _P]),
    "kb_beam_finish": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P]),
    "kb_beam_backtrace": (_I, [_I, _I, _I, ctypes.c_float, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "kb_compact_workspace_bytes": (_SZ, [_I]),
    "kb_compact_batch": (_I, [_I, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "kb_compact_beams": (_I, [_I, _I, _P, _P, _P, _P, _P, _P, _P]),
    "kb_gather_rows": (_I, [_I, _P, _P, _P, _P, _SZ, _P]),
    "kb_shard_splits": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P]),
    "kb_shard_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I]),
    "kb_shard_partials": (_I, [_I, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "kb_merge_partials": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    # decoder stand-in of the synthetic decode loop (include/kbest_standin.h)
    "kb_standin_alive": (_I, [_I, _P, _I, _I, _P, _P, _P, _P]),
    "kb_standin_next_h": (_I, [_I, _P, _I, _I, _I, _P, _P, _P, _P, _SZ, _P]),
    "kb_standin_step": (_I, [_I, _P, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P, _SZ, _P]),
    # attention cache (include/kbest_cache.h)
    "kb_cache_append": (_I, [_C, _I, _P, _I, _P, _L, _P, _L, _P, _L, _I, _I, _P, _P, _F, _P, _P, _P, _P, _P, _P]),
    "kb_cache_attend_workspace_bytes": (_SZ, [_C, _I, _I, _I, _I]),
    "kb_cache_attend": (_I, [_C, _I, _P, _I, _P, _L, _F, _P, _P, _I, _P, _P, _P, _P, _P, _SZ, _P]),
    "kb_cache_evict": (_I, [_C, _I, _P, _P, _I, _I, _I, _P, _P, _P, _P, _I, _P, _P, _P, _P, _P]),
}


class KBestError(RuntimeError):
    def __init__(self, status: int, detail: str):
        self.status = status
        super().__init__(f"libkbest status {status}: {detail}")


def lib() -> ctypes.CDLL:
    """Load libkbest.so once; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                              "or python -m paper_1805_09863_amd._build")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status: int):
    if status != KB_OK:
        raise KBestError(status, lib().kb_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    # a plain int: the declared argtypes (c_void_p) convert it, at a fraction
    # of the cost of building a c_void_p per pointer
    return None if t is None else t.data_ptr()


def _ptr_host(t: Optional[torch.Tensor]):
    """Address of a pinned host tensor (checked by the caller) that kernels write."""
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, device: Optional[torch.device] = None) -> int:
    """The hipStream_t to launch on: ``stream``'s, else the current stream of
    ``device`` (by default the current device), read as a raw handle without
    building a torch.cuda.Stream object."""
    if stream is None:
        if _raw_stream is not None:
            idx = device.index if device is not None and device.index is not None else torch.cuda.current_device()
            return _raw_stream(idx)
        stream = torch.cuda.current_stream(device)
    return stream.cuda_stream


def _dtype_code(t: torch.Tensor, what: str = "h and W") -> int:
    if t.dtype == torch.float32:
        return KB_F32
    if t.dtype == torch.bfloat16:
        return KB_BF16
    raise TypeError(f"{what} must be float32 or bfloat16, got {t.dtype}")


def _need(t: torch.Tensor, name: str, dtype=None, dim=None, numel=None):
    """Every tensor handed to the library as a pointer: on the GPU, contiguous,
    of the given type and rank, and (numel) at least that many elements."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a tensor on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if dim is not None and t.dim() != dim:
        raise ValueError(f"{name} must have {dim} dimensions")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} has {t.numel()} elements, {numel} needed")


def _need_ws(ws: torch.Tensor, nbytes: int, name: str = "ws"):
    _need(ws, name)
    if ws.numel() * ws.element_size() < nbytes:
        raise ValueError(f"{name} has {ws.numel() * ws.element_size()} bytes, {nbytes} needed")


def _need_outs(out, names, dtypes, numel):
    if len(out) != len(names):
        raise ValueError(f"out must hold {len(names)} tensors ({', '.join(names)})")
    for t, n, d in zip(out, names, dtypes):
        _need(t, n, dtype=d, numel=numel)


def abi_version() -> int:
    return lib().kb_abi_version()


_ws_bytes_cache: dict = {}


def kbest_workspace_bytes(dtype: int, N: int, H: int, V: int, k: int, S: int) -> int:
    # a pure function of the shape (for one loaded library and tile override):
    # asked once per shape
    L = lib()
    key = (id(L), os.environ.get("KB_TILE"), dtype, N, H, V, k, S)
    n = _ws_bytes_cache.get(key)
    if n is None:
        n = _ws_bytes_cache[key] = int(L.kb_kbest_workspace_bytes(dtype, N, H, V, k, S))
    return n


KB_KERNEL_NAMES = ("few", "wide", "dma", "reg")
_PLAN_FIELDS = ("kernel", "tile_rows", "tile_words", "row_tiles", "splits", "tiles_per_split")


def kbest_plan(dtype: int, N: int, H: int, V: int, k: int, aligned: bool = True) -> dict:
    """The projection plan kbest_step chooses for this shape (kb_kbest_plan):
    kernel ("few", "wide", "dma" or "reg"), tile rows and words, row tiles,
    vocabulary splits and tiles per split.  ``aligned``: whether h, W and b
    sit at 16-byte aligned addresses (torch allocations do)."""
    esz = 2 if dtype == KB_BF16 else 4
    base = 1 << 20 if aligned else (1 << 20) + esz
    out = (ctypes.c_int32 * 6)()
    _check(lib().kb_kbest_plan(dtype, N, H, V, k, base, base, (1 << 20) if aligned else (1 << 20) + 4, out))
    plan = dict(zip(_PLAN_FIELDS, list(out)))
    plan["kernel"] = KB_KERNEL_NAMES[plan["kernel"]] if N > 0 else None
    return plan


def workspace(nbytes: int, device=None) -> torch.Tensor:
    """A device byte buffer usable as a workspace (torch allocations are 256-B aligned)."""
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device or "cuda")


def _empty(like: torch.Tensor, shape, stream, dtype=None) -> torch.Tensor:
    """Memory of the stream that the call runs on: what the caller's current stream has freed may still be
    in use there, and what is dropped after the call is still in use on the call's."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def kbest_step(h: torch.Tensor, W: torch.Tensor, b: torch.Tensor, prev_score: torch.Tensor,
               sent_offsets: torch.Tensor, k: int, *, S: Optional[int] = None,
               out: Optional[tuple] = None, ws: Optional[torch.Tensor] = None,
               row_lse: Optional[torch.Tensor] = None, stream=None, events: Optional[tuple] = None):
    """One decode step of the output layer: returns (token, parent, score), each S x k.

    ``h`` is N x H, ``W`` is H x V (float32 or bfloat16, same type), ``b`` V
    float32, ``prev_score`` N float32, ``sent_offsets`` S+1 int32, all on the
    GPU.  ``out`` may supply preallocated (token, parent, score), ``ws`` a
    workspace of at least ``kbest_workspace_bytes`` bytes, ``row_lse`` an N
    float32 tensor to receive each row's log-sum-exp, ``events`` a pair of
    raw hipEvent_t handles recorded around the projection kernel.
    """
    _need(h, "h", dim=2)
    _need(W, "W", dtype=h.dtype, dim=2)
    _need(b, "b", dtype=torch.float32, dim=1)
    _need(prev_score, "prev_score", dtype=torch.float32, dim=1)
    _need(sent_offsets, "sent_offsets", dtype=torch.int32, dim=1)
    dt = _dtype_code(h)
    N, H = h.shape
    H2, V = W.shape
    if H2 != H or b.shape[0] != V or prev_score.shape[0] != N:
        raise ValueError("shape mismatch among h, W, b, prev_score")
    S = sent_offsets.shape[0] - 1 if S is None else S
    if sent_offsets.shape[0] != S + 1:
        raise ValueError("sent_offsets must have S+1 entries")
    dev = h.device
    if out is None:
        tok = _empty(h, (S, k), stream, torch.int32)
        par = _empty(h, (S, k), stream, torch.int32)
        sc = _empty(h, (S, k), stream, torch.float32)
    else:
        _need_outs(out, ("token", "parent", "score"), (torch.int32, torch.int32, torch.float32), S * k)
        tok, par, sc = out
    need = kbest_workspace_bytes(dt, N, H, V, k, S)
    if ws is None:
        ws = _empty(h, max(need, 1), stream, torch.uint8)
    _need_ws(ws, need)
    if row_lse is not None:
        _need(row_lse, "row_lse", dtype=torch.float32, numel=N)
    L = lib()
    args = [dt, N, H, V, k, S, _ptr(h), _ptr(W), _ptr(b), _ptr(prev_score), _ptr(sent_offsets),
            _ptr(tok), _ptr(par), _ptr(sc), _ptr(row_lse), _ptr(ws), ws.numel() * ws.element_size(),
            _stream(stream, dev)]
    if events is None:
        _check(L.kb_kbest_step(*args))
    else:
        _check(L.kb_kbest_step_events(*args, ctypes.c_void_p(events[0]), ctypes.c_void_p(events[1])))
    return tok, par, sc


def kbest_step_noalloc(h: torch.Tensor, W: torch.Tensor, b: torch.Tensor, prev_score: torch.Tensor,
                       sent_offsets: torch.Tensor, k: int, *, out: tuple, S: Optional[int] = None,
                       row_lse: Optional[torch.Tensor] = None, stream=None):
    """kbest_step without a workspace (include/kbest.h, kb_kbest_step_noalloc): the
    library's fixed per-device scratch array takes the partials, so nothing is
    allocated, here or in the library; ``out`` = (token, parent, score) must be given."""
    _need(h, "h", dim=2)
    _need(W, "W", dtype=h.dtype, dim=2)
    _need(b, "b", dtype=torch.float32, dim=1)
    _need(prev_score, "prev_score", dtype=torch.float32, dim=1)
    _need(sent_offsets, "sent_offsets", dtype=torch.int32, dim=1)
    dt = _dtype_code(h)
    N, H = h.shape
    H2, V = W.shape
    if H2 != H or b.shape[0] != V or prev_score.shape[0] != N:
        raise ValueError("shape mismatch among h, W, b, prev_score")
    S = sent_offsets.shape[0] - 1 if S is None else S
    if sent_offsets.shape[0] != S + 1:
        raise ValueError("sent_offsets must have S+1 entries")
    _need_outs(out, ("token", "parent", "score"), (torch.int32, torch.int32, torch.float32), S * k)
    if row_lse is not None:
        _need(row_lse, "row_lse", dtype=torch.float32, numel=N)
    tok, par, sc = out
    _check(lib().kb_kbest_step_noalloc(dt, N, H, V, k, S, _ptr(h), _ptr(W), _ptr(b), _ptr(prev_score),
                                       _ptr(sent_offsets), _ptr(tok), _ptr(par), _ptr(sc), _ptr(row_lse),
                                       _stream(stream)))
    return tok, par, sc


def argmax_workspace_bytes(dtype: int, N: int, H: int, V: int) -> int:
    return int(lib().kb_argmax_workspace_bytes(dtype, N, H, V))


def argmax_step(h: torch.Tensor, W: torch.Tensor, b: torch.Tensor, *, out: Optional[tuple] = None,
                ws: Optional[torch.Tensor] = None, stream=None):
    """Greedy (beam 1) step (Algorithms 5 and 6): returns (token[N] int32, logit[N] float32),
    the best word of every row of h @ W + b and its raw score, without a softmax."""
    _need(h, "h", dim=2)
    _need(W, "W", dtype=h.dtype, dim=2)
    _need(b, "b", dtype=torch.float32, dim=1)
    dt = _dtype_code(h)
    N, H = h.shape
    H2, V = W.shape
    if H2 != H or b.shape[0] != V:
        raise ValueError("shape mismatch among h, W, b")
    if out is None:
        tok = _empty(h, N, stream, torch.int32)
        val = _empty(h, N, stream, torch.float32)
    else:
        _need_outs(out, ("token", "logit"), (torch.int32, torch.float32), N)
        tok, val = out
    need = argmax_workspace_bytes(dt, N, H, V)
    if ws is None:
        ws = _empty(h, max(need, 1), stream, torch.uint8)
    _need_ws(ws, need)
    _check(lib().kb_argmax_step(dt, N, H, V, _ptr(h), _ptr(W), _ptr(b), _ptr(tok), _ptr(val), _ptr(ws),
                                ws.numel() * ws.element_size(), _stream(stream)))
    return tok, val


def unfused_workspace_bytes(dtype: int, N: int, H: int, V: int, k: int, S: int) -> int:
    return int(lib().kb_unfused_workspace_bytes(dtype, N, H, V, k, S))


def kbest_step_unfused(h: torch.Tensor, W: torch.Tensor, b: torch.Tensor, prev_score: torch.Tensor,
                       sent_offsets: torch.Tensor, k: int, *, mode: int = 0, out: Optional[tuple] = None,
                       ws: Optional[torch.Tensor] = None, row_lse: Optional[torch.Tensor] = None,
                       events: Optional[list] = None, stream=None):
    """The unfused baseline of kbest_step (mode 0: Algorithm 3; mode 1: Algorithm 4
    over stored scores); ``events`` is a list of raw hipEvent_t handles recorded
    at the stage boundaries (see include/kbest.h)."""
    _need(h, "h", dim=2)
    _need(W, "W", dtype=h.dtype, dim=2)
    _need(b, "b", dtype=torch.float32, dim=1)
    _need(prev_score, "prev_score", dtype=torch.float32, dim=1)
    _need(sent_offsets, "sent_offsets", dtype=torch.int32, dim=1)
    dt = _dtype_code(h)
    N, H = h.shape
    V = W.shape[1]
    S = sent_offsets.shape[0] - 1
    if out is None:
        out = tuple(_empty(h, (S, k), stream, t) for t in (torch.int32, torch.int32, torch.float32))
    _need_outs(out, ("token", "parent", "score"), (torch.int32, torch.int32, torch.float32), S * k)
    tok, par, sc = out
    need = unfused_workspace_bytes(dt, N, H, V, k, S)
    if ws is None:
        ws = _empty(h, max(need, 1), stream, torch.uint8)
    _need_ws(ws, need)
    if row_lse is not None:
        _need(row_lse, "row_lse", dtype=torch.float32, numel=N)
    ev = None
    if events:
        ev = (ctypes.c_void_p * len(events))(*[ctypes.c_void_p(e) for e in events])
    _check(lib().kb_kbest_step_unfused(mode, dt, N, H, V, k, S, _ptr(h), _ptr(W), _ptr(b), _ptr(prev_score),
                                       _ptr(sent_offsets), _ptr(tok), _ptr(par), _ptr(sc), _ptr(row_lse),
                                       _ptr(ws), ws.numel() * ws.element_size(), ev,
                                       len(events) if events else 0, _stream(stream)))
    return tok, par, sc


def compact_workspace_bytes(M: int) -> int:
    return int(lib().kb_compact_workspace_bytes(M))


def compact_batch(alive: torch.Tensor, entry_sentence: Optional[torch.Tensor] = None, *,
                  out: Optional[tuple] = None, ws: Optional[torch.Tensor] = None, stream=None):
    """Stable removal of finished entries from a batch of M entries (Algorithm 2).

    ``alive`` is M uint8 on the GPU; ``entry_sentence`` (optional) M int32,
    the non-decreasing sentence id of every entry.  Returns device tensors
    (keep_idx[M], kept_count[1], new_sent_offsets, new_S[1]); only the first
    kept_count / new_S + 1 entries are meaningful.  Without entry_sentence the
    last two are None.  ``out`` may supply (keep_idx, kept_count,
    new_sent_offsets, new_S); new_sent_offsets needs one more entry than
    entry_sentence has distinct ids (M + 1 always suffices).
    """
    _need(alive, "alive", dtype=torch.uint8, dim=1)
    M = alive.numel()
    if entry_sentence is not None:
        _need(entry_sentence, "entry_sentence", dtype=torch.int32, dim=1, numel=M)
    if out is None:
        keep = _empty(alive, max(M, 1), stream, torch.int32)
        kept = _empty(alive, 1, stream, torch.int32)
        noff = _empty(alive, M + 1, stream, torch.int32) if entry_sentence is not None else None
        nS = _empty(alive, 1, stream, torch.int32) if entry_sentence is not None else None
    else:
        keep, kept, noff, nS = out
        _need(keep, "keep_idx", dtype=torch.int32, numel=M)
        _need(kept, "kept_count", dtype=torch.int32, numel=1)
        if noff is not None:
            _need(noff, "new_sent_offsets", dtype=torch.int32, numel=1)
        if nS is not None:
            _need(nS, "new_S", dtype=torch.int32, numel=1)
    need = compact_workspace_bytes(M)
    if ws is None and need > 0:
        ws = _empty(alive, need, stream, torch.uint8)
    if ws is not None:
        _need_ws(ws, need)
    nbytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().kb_compact_batch(M, _ptr(alive), _ptr(keep), _ptr(kept), _ptr(entry_sentence), _ptr(noff),
                                  _ptr(nS), _ptr(ws), nbytes, _stream(stream)))
    return keep, kept, noff, nS


def compact_beams(alive: torch.Tensor, S: int, k: int, *, out: Optional[tuple] = None, stream=None):
    """Stable removal of finished entries from the S x k output of a step (Algorithm 2).

    ``alive`` is S*k uint8 on the GPU.  Returns device tensors
    (keep_idx[S*k], kept_count[1], new_sent_offsets[S+1], kept_sentence[S], new_S[1]);
    only the first kept_count / new_S (+1) entries are meaningful.
    """
    _need(alive, "alive", dtype=torch.uint8)
    if alive.numel() != S * k:
        raise ValueError("alive must have S*k entries")
    if out is None:
        keep, kept, noff, ksent, nS = (_empty(alive, n, stream, torch.int32)
                                       for n in (max(S * k, 1), 1, S + 1, max(S, 1), 1))
    else:
        keep, kept, noff, ksent, nS = out
        _need(keep, "keep_idx", dtype=torch.int32, numel=S * k)
        _need(kept, "kept_count", dtype=torch.int32, numel=1)
        if noff is not None:
            _need(noff, "new_sent_offsets", dtype=torch.int32, numel=S + 1)
        if ksent is not None:
            _need(ksent, "kept_sentence", dtype=torch.int32, numel=S)
        if nS is not None:
            _need(nS, "new_S", dtype=torch.int32, numel=1)
    _check(lib().kb_compact_beams(S, k, _ptr(alive), _ptr(keep), _ptr(kept), _ptr(noff), _ptr(ksent),
                                  _ptr(nS), _stream(stream)))
    return keep, kept, noff, ksent, nS


def gather_rows(src: torch.Tensor, idx: torch.Tensor, *, n_dev: Optional[torch.Tensor] = None,
                n_max: Optional[int] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[i] = src[idx[i]] for i < min(n_max, n_dev[0]) (rows of src along dim 0)."""
    _need(src, "src")
    n_max = idx.shape[0] if n_max is None else n_max
    _need(idx, "idx", dtype=torch.int32, dim=1, numel=n_max)
    if n_dev is not None:
        _need(n_dev, "n_dev", dtype=torch.int32, numel=1)
    row_bytes = src[0].numel() * src.element_size() if src.shape[0] > 0 else 0
    if out is None:
        out = _empty(src, (n_max,) + tuple(src.shape[1:]), stream)
    _need(out, "out", dtype=src.dtype, numel=n_max * (src[0].numel() if src.shape[0] > 0 else 0))
    if n_max == 0:
        return out
    _check(lib().kb_gather_rows(n_max, _ptr(n_dev), _ptr(idx), _ptr(src), _ptr(out), row_bytes,
                                _stream(stream)))
    return out


# ---------------------------------------------------------------- decoder stand-in
def shard_splits(h: torch.Tensor, W_shard: torch.Tensor, b_shard: torch.Tensor, k: int) -> int:
    """Number of vocabulary splits shard_partials writes for these operands."""
    N, H = h.shape
    out = ctypes.c_int(0)
    _check(lib().kb_shard_splits(_dtype_code(h), N, H, W_shard.shape[1], k, _ptr(h), _ptr(W_shard), _ptr(b_shard),
                                 ctypes.byref(out)))
    return int(out.value)


def shard_partials(h: torch.Tensor, W_shard: torch.Tensor, b_shard: torch.Tensor, k: int, word_base: int,
                   stats: torch.Tensor, lists: torch.Tensor, *, ws: Optional[torch.Tensor] = None, stream=None):
    """One vocabulary shard's fused projection (see include/kbest.h): its splits'
    statistics into ``stats`` (splits x N x 2 float32) and k-best lists into
    ``lists`` (splits x N x k x 2 int32, global words), normally slices of the
    combined arrays that merge_partials reduces."""
    _need(h, "h", dim=2)
    _need(W_shard, "W_shard", dtype=h.dtype, dim=2)
    _need(b_shard, "b_shard", dtype=torch.float32, dim=1)
    _need(stats, "stats", dtype=torch.float32)
    _need(lists, "lists", dtype=torch.int32)
    N, H = h.shape
    if W_shard.shape[0] != H or b_shard.shape[0] != W_shard.shape[1]:
        raise ValueError("shape mismatch among h, W_shard, b_shard")
    V_shard = W_shard.shape[1]
    P = shard_splits(h, W_shard, b_shard, k)
    if stats.numel() < P * N * 2 or lists.numel() < P * N * k * 2:
        raise ValueError(f"stats / lists too small for {P} splits")
    dt = _dtype_code(h)
    need = int(lib().kb_shard_workspace_bytes(dt, N, H, V_shard, k))
    if ws is None:
        ws = _empty(h, max(need, 1), stream, torch.uint8)
    _need_ws(ws, need)
    _check(lib().kb_shard_partials(dt, N, H, V_shard, word_base, k, _ptr(h), _ptr(W_shard), _ptr(b_shard),
                                   _ptr(stats), _ptr(lists), _ptr(ws), ws.numel() * ws.element_size(),
                                   _stream(stream)))
    return P


def merge_partials(stats: torch.Tensor, lists: torch.Tensor, P: int, V: int, k: int, prev_score: torch.Tensor,
                   sent_offsets: torch.Tensor, *, out: Optional[tuple] = None,
                   row_lse: Optional[torch.Tensor] = None, stream=None):
    """Reduce the combined partials of all shards (P splits in total) and merge the
    beam: returns (token, parent, score), each S x k, as kbest_step does."""
    _need(stats, "stats", dtype=torch.float32)
    _need(lists, "lists", dtype=torch.int32)
    _need(prev_score, "prev_score", dtype=torch.float32, dim=1)
    _need(sent_offsets, "sent_offsets", dtype=torch.int32, dim=1)
    N = prev_score.shape[0]
    S = sent_offsets.shape[0] - 1
    if stats.numel() < P * N * 2 or lists.numel() < P * N * k * 2:
        raise ValueError(f"stats / lists too small for {P} splits")
    if out is None:
        out = tuple(_empty(prev_score, (S, k), stream, t) for t in (torch.int32, torch.int32, torch.float32))
    _need_outs(out, ("token", "parent", "score"), (torch.int32, torch.int32, torch.float32), S * k)
    tok, par, sc = out
    if row_lse is not None:
        _need(row_lse, "row_lse", dtype=torch.float32, numel=N)
    _check(lib().kb_merge_partials(N, V, k, S, P, _ptr(stats), _ptr(lists), _ptr(prev_score), _ptr(sent_offsets),
                                   _ptr(tok), _ptr(par), _ptr(sc), _ptr(row_lse), _stream(stream)))
    return tok, par, sc


def standin_alive(sid: torch.Tensor, lengths: torch.Tensor, S: int, k: int, t: int, *, out: torch.Tensor,
                  S_dev: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[s*k + r] = (s < min(S, S_dev[0]) and t < lengths[sid[s]] - 1) for s < S
    (include/kbest_standin.h)."""
    _need(sid, "sid", dtype=torch.int32, numel=S)
    _need(lengths, "lengths", dtype=torch.int32)
    _need(out, "out", dtype=torch.uint8, numel=S * k)
    if S_dev is not None:
        _need(S_dev, "S_dev", dtype=torch.int32, numel=1)
    _check(lib().kb_standin_alive(S, _ptr(S_dev), k, t, _ptr(sid), _ptr(lengths), _ptr(out), _stream(stream)))
    return out


def standin_step(sid: torch.Tensor, lengths: torch.Tensor, score: torch.Tensor, S: int, k: int, t: int, *,
                 out: tuple, S_dev: Optional[torch.Tensor] = None, alive: Optional[torch.Tensor] = None,
                 counts_host: Optional[torch.Tensor] = None, next_state: Optional[tuple] = None, stream=None):
    """The loop step's bookkeeping in one launch (include/kbest_standin.h): the
    EOS mask, its compaction and the gathers of the surviving scores and sentence
    ids.  ``out`` = (keep_idx[S*k], counts[2], new_sent_offsets[S+1],
    prev_next[S*k] float32, sid_next[S]); returns it.  ``counts_host``, a pinned
    int32 host tensor of 3, receives the counts too, then the tag t + 1 (a host
    that polls [2] may read [0] and [1] once the tag is there).  ``next_state`` = (table, T, next_h): the surviving
    entries' states of step t + 1 gathered into next_h (rows x H, like table)
    in the same launch."""
    keep, counts, noff, prev_next, sid_next = out
    _need(sid, "sid", dtype=torch.int32, numel=S)
    _need(lengths, "lengths", dtype=torch.int32)
    _need(score, "score", dtype=torch.float32, numel=S * k)
    _need(keep, "keep_idx", dtype=torch.int32, numel=S * k)
    _need(counts, "counts", dtype=torch.int32, numel=2)
    _need(noff, "new_sent_offsets", dtype=torch.int32, numel=S + 1)
    _need(prev_next, "prev_next", dtype=torch.float32, numel=S * k)
    _need(sid_next, "sid_next", dtype=torch.int32, numel=S)
    if S_dev is not None:
        _need(S_dev, "S_dev", dtype=torch.int32, numel=1)
    if alive is not None:
        _need(alive, "alive", dtype=torch.uint8, numel=S * k)
    if counts_host is not None:
        if not isinstance(counts_host, torch.Tensor) or counts_host.is_cuda or not counts_host.is_pinned():
            raise TypeError("counts_host must be a pinned host tensor")
        if counts_host.dtype != torch.int32 or counts_host.numel() < 3 or not counts_host.is_contiguous():
            raise ValueError("counts_host must be 3 contiguous int32")
    table = next_h = None
    T, row_bytes = 0, 0
    if next_state is not None:
        table, T, next_h = next_state
        _need(table, "table", dim=2)
        _need(next_h, "next_h", dtype=table.dtype, numel=S * k * table.shape[1])
        row_bytes = table.shape[1] * table.element_size()
    _check(lib().kb_standin_step(S, _ptr(S_dev), k, t, _ptr(sid), _ptr(lengths), _ptr(score), _ptr(keep),
                                 _ptr(counts), _ptr(noff), _ptr(prev_next), _ptr(sid_next), _ptr(alive),
                                 _ptr_host(counts_host), _ptr(table), T, _ptr(next_h), row_bytes,
                                 _stream(stream)))
    return out


def standin_next_h(table: torch.Tensor, keep: torch.Tensor, sid: torch.Tensor, k: int, T: int, t: int,
                   n_max: int, *, n_dev: Optional[torch.Tensor] = None, out: torch.Tensor, stream=None):
    """out[i] = table[(sid[keep[i] // k] * T + t) * k + keep[i] % k] for i < min(n_max, n_dev[0])."""
    _need(table, "table")
    _need(keep, "keep", dtype=torch.int32, numel=n_max)
    _need(sid, "sid", dtype=torch.int32)
    _need(out, "out", dtype=table.dtype, numel=n_max * table[0].numel())
    if n_dev is not None:
        _need(n_dev, "n_dev", dtype=torch.int32, numel=1)
    row_bytes = table[0].numel() * table.element_size()
    _check(lib().kb_standin_next_h(n_max, _ptr(n_dev), k, T, t, _ptr(keep), _ptr(sid), _ptr(table), _ptr(out),
                                   row_bytes, _stream(stream)))
    return out


# ---------------------------------------------------------------- per-hypothesis EOS
def beam_finish(S: int, k: int, t: int, T: int, eos: int, token, parent, score, sent_id, beam, prev_keep,
                prev_hist_base: int, hist_base: int, hist_token, hist_parent, fin: tuple, alive, stream=None):
    """After a step: take each sentence's first beam[s] continuations, record the step's
    history, move EOS (or last-step) continuations to the finished store ``fin`` =
    (count, score, len, hist), shrink the beams and fill ``alive`` (include/kbest.h)."""
    fc, fs, fl, fh = fin
    n = S * k
    for x, nm, d, m in ((token, "token", torch.int32, n), (parent, "parent", torch.int32, n),
                        (score, "score", torch.float32, n), (sent_id, "sent_id", torch.int32, S),
                        (beam, "beam", torch.int32, S), (hist_token, "hist_token", torch.int32, hist_base + n),
                        (hist_parent, "hist_parent", torch.int32, hist_base + n),
                        (fc, "fin_count", torch.int32, S), (alive, "alive", torch.uint8, n)):
        _need(x, nm, dtype=d, numel=m)
    S0 = fc.numel()             # the finished store holds k slots per original sentence
    for x, nm, d in ((fs, "fin_score", torch.float32), (fl, "fin_len", torch.int32), (fh, "fin_hist", torch.int32)):
        _need(x, nm, dtype=d, numel=S0 * k)
    if prev_keep is not None:
        _need(prev_keep, "prev_keep", dtype=torch.int32, numel=S)
    _check(lib().kb_beam_finish(S, k, t, T, eos, _ptr(token), _ptr(parent), _ptr(score), _ptr(sent_id), _ptr(beam),
                                _ptr(prev_keep), prev_hist_base, hist_base, _ptr(hist_token), _ptr(hist_parent),
                                _ptr(fc), _ptr(fs), _ptr(fl), _ptr(fh), _ptr(alive), _stream(stream)))


def beam_backtrace(S0: int, k: int, T: int, alpha: float, fin: tuple, hist_token, hist_parent, *, out=None,
                   stream=None):
    """Best finished hypothesis of every sentence by score / len**alpha, and its tokens:
    returns (tokens[S0, T], len[S0], score[S0], normalised score[S0])."""
    fc, fs, fl, fh = fin
    if out is None:
        out = (_empty(fc, (S0, T), stream, torch.int32), _empty(fc, S0, stream, torch.int32),
               _empty(fc, S0, stream, torch.float32), _empty(fc, S0, stream, torch.float32))
    for x, nm_, d in ((fc, "fin_count", torch.int32), (fs, "fin_score", torch.float32),
                      (fl, "fin_len", torch.int32), (fh, "fin_hist", torch.int32)):
        _need(x, nm_, dtype=d, numel=S0 * (1 if nm_ == "fin_count" else k))
    _need(hist_token, "hist_token", dtype=torch.int32)
    _need(hist_parent, "hist_parent", dtype=torch.int32)
    _need_outs(out[:1], ("tokens",), (torch.int32,), S0 * T)
    _need_outs(out[1:], ("len", "score", "norm"), (torch.int32, torch.float32, torch.float32), S0)
    toks, ln, sc, nm = out
    _check(lib().kb_beam_backtrace(S0, k, T, float(alpha), _ptr(fc), _ptr(fs), _ptr(fl), _ptr(fh), _ptr(hist_token),
                                   _ptr(hist_parent), _ptr(toks), _ptr(ln), _ptr(sc), _ptr(nm), _stream(stream)))
    return toks, ln, sc, nm


# ---------------------------------------------------------------- attention cache
# A step's calls take a few microseconds on the device: their tensors are
# checked in one expression each, and the message is worked out only for one
# that fails.
def _refuse(t, name: str, dtype, numel: int, dev: int):
    _need(t, name, dtype=dtype, numel=numel)
    raise ValueError(f"{name} is on {t.device}, the cache on cuda:{dev}")


def _ask(t, name: str, dtype, numel: int, dev: int) -> int:
    """Address of a contiguous tensor of ``dtype`` with at least ``numel`` elements on GPU ``dev``."""
    try:
        if t.dtype is dtype and t.get_device() == dev and t.is_contiguous() and t.numel() >= numel:
            return t.data_ptr()
    except AttributeError:
        pass
    return _refuse(t, name, dtype, numel, dev)


def _ask_as(t, name: str, dtype, shape: tuple, dev: int) -> int:
    """_ask for a tensor of ``shape``, or of more rows of the same dimensions, or laid out as that is: flat, or
    divided otherwise along the same rows.  A last dimension that is longer is another distance of two rows."""
    try:
        if t.shape == shape and t.dtype is dtype and t.get_device() == dev and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    p, inner, got = _ask(t, name, dtype, math.prod(shape), dev), shape[1:], t.shape
    if (len(got) <= 1 or got[-len(inner):] == inner or got[1:] == inner[1:]
            or math.prod(got[1:]) == math.prod(inner) and (len(got) == 2 or got[1] == inner[0])):
        return p
    raise ValueError(f"{name} must have rows of {' x '.join(map(str, inner))}, got {tuple(got)}")


_INT_MAX = 2 ** 31 - 1
_I32, _F32 = torch.int32, torch.float32
_CODES = {torch.float32: KB_F32, torch.bfloat16: KB_BF16}


def _refuse_sizes(**sizes):
    """Raised before ctypes would cut a size to 32 bits."""
    for name, x in sizes.items():
        if not -_INT_MAX <= x <= _INT_MAX:
            raise ValueError(f"{name} = {x}: beyond 32 bits")


_device_now = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _run(fn, dev: int, stream, *args):
    """fn(*args, stream) with the tensors' device current; an error raised."""
    st = _raw_stream(dev) if stream is None and _raw_stream is not None else _stream(stream, torch.device("cuda", dev))
    if _device_now() == dev:
        status = fn(*args, st)
    else:
        with torch.cuda.device(dev):
            status = fn(*args, st)
    if status:
        _check(status)


def _cache(k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor):
    """(kb_cache, GPU index, type, key-value heads, dim, slots of a sequence, sequences)."""
    if not isinstance(k_cache, torch.Tensor) or not k_cache.is_cuda:
        raise TypeError("k_cache must be a tensor on the GPU")
    dtype, dev, shape = k_cache.dtype, k_cache.get_device(), k_cache.shape
    try:
        whole = (k_cache.is_contiguous() and v_cache.dtype is dtype and v_cache.get_device() == dev
                 and v_cache.is_contiguous() and table.dtype is _I32 and table.get_device() == dev
                 and table.is_contiguous())
    except AttributeError:
        whole = False
    if not whole:
        for t, name, kind in ((k_cache, "k_cache", dtype), (v_cache, "v_cache", dtype), (table, "table", _I32)):
            _ask(t, name, kind, 0, dev)
    if len(shape) != 4 or v_cache.shape != shape:
        raise ValueError("k_cache and v_cache must be pages x heads x page_size x dim, the same shape")
    if table.dim() != 2:
        raise ValueError("table must be seqs x max_pages")
    pages, heads, page_size, dim = shape
    seqs, max_pages = table.shape
    if pages | heads | page_size | dim | seqs | max_pages > _INT_MAX:
        _refuse_sizes(pages=pages, heads=heads, page_size=page_size, dim=dim, seqs=seqs, max_pages=max_pages)
    code = _CODES.get(dtype)
    if code is None:
        _dtype_code(k_cache, "k_cache")
    return (_Cache(code, heads, dim, page_size, pages, seqs, max_pages, k_cache.data_ptr(), v_cache.data_ptr(),
                   table.data_ptr()), dev, dtype, heads, dim, max_pages * page_size, seqs)


def _ask_rows(t: torch.Tensor, name: str, dtype, R: int, heads: Optional[int], dim: int, dev: int):
    """(address, distance of two rows in values, heads) of R x heads x dim whose rows may lie apart, as
    parts of a wider projection's do."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a tensor on the GPU")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the cache on cuda:{dev}")
    shape = t.shape
    if len(shape) != 3 or shape[0] != R or shape[2] != dim or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must be {R} x {'heads' if heads is None else heads} x {dim}, got {tuple(shape)}")
    heads = shape[1]
    if R | heads > _INT_MAX:
        _refuse_sizes(rows=R, **{f"heads of {name}": heads})
    step, apart, one = t.stride()
    if one != 1 or (heads > 1 and apart != dim):
        raise ValueError(f"{name}: the heads of a row must lie one after the other, without gaps")
    if R <= 1:
        step = heads * dim
    elif step < heads * dim:
        raise ValueError(f"{name}: rows must not overlap")
    return t.data_ptr(), step, heads


def cache_append(k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, length: torch.Tensor,
                 k: torch.Tensor, v: torch.Tensor, *, q: Optional[torch.Tensor] = None,
                 pos: Optional[torch.Tensor] = None, freq: Optional[torch.Tensor] = None, interleaved: bool = False,
                 amplitude: float = 1.0, seq: Optional[torch.Tensor] = None, n_dev: Optional[torch.Tensor] = None,
                 position: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                 q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """The keys and values of R new tokens into their slots of the cache, queries and
    keys turned by their rotary positions (kb_cache_append).

    ``k_cache``, ``v_cache`` are pages x heads x page_size x dim (float32 or bfloat16),
    ``table`` seqs x max_pages int32.  Row r is a token of sequence ``seq[r]`` (r) and
    goes to slot ``length[r] - 1``.  ``k``, ``v`` are R x heads x dim and ``q`` R x
    q_heads x dim; their rows may be parts of a wider projection's.  ``freq`` (float64,
    radians per position, see rotary_frequencies) turns the first ``2 * len(freq)``
    values of a head, in pairs half of that apart or, ``interleaved``, side by side.
    ``position`` (int32) and ``weight`` (float32), seqs x heads x slots, receive the new
    slots' ``pos`` and 0.  Returns the turned queries (``q_out``), None without ``q``.
    """
    c, dev, dtype, heads, dim, cap, seqs = _cache(k_cache, v_cache, table)
    lp = _ask(length, "length", _I32, 0, dev)
    R = length.numel()
    kp, k_stride, _ = _ask_rows(k, "k", dtype, R, heads, dim, dev)
    vp, v_stride, _ = _ask_rows(v, "v", dtype, R, heads, dim, dev)
    q_heads = q_stride = rot = 0
    qp = op = fp = None
    if q is not None:
        qp, q_stride, q_heads = _ask_rows(q, "q", dtype, R, None, dim, dev)
        if q_out is None:
            q_out = _empty(q, (R, q_heads, dim), stream)
        op = _ask_as(q_out, "q_out", dtype, (R, q_heads, dim), dev)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if freq is not None:
        fp = _ask(freq, "freq", torch.float64, 0, dev)
        rot = 2 * freq.numel()
        if rot > _INT_MAX:
            _refuse_sizes(**{"values that freq turns": rot})
    pp = None if pos is None else _ask(pos, "pos", _I32, R, dev)
    sp = None if seq is None else _ask(seq, "seq", _I32, R, dev)
    nd = None if n_dev is None else _ask(n_dev, "n_dev", _I32, 1, dev)
    at = None if position is None else _ask_as(position, "position", _I32, (seqs, heads, cap), dev)
    wp = None if weight is None else _ask_as(weight, "weight", _F32, (seqs, heads, cap), dev)
    _run(lib().kb_cache_append, dev, stream, c, R, nd, q_heads, qp, q_stride, kp, k_stride, vp, v_stride, rot,
         1 if interleaved else 0, pp, fp, amplitude, sp, lp, op, at, wp)
    return q_out


def cache_attend_workspace_bytes(k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, R: int,
                                 q_heads: int, max_len: Optional[int] = None, weights: bool = False) -> int:
    """Bytes that cache_attend's ``ws`` needs for R rows of q_heads heads (``weights``: with ``weight_out``)."""
    c, _, _, _, _, cap, _ = _cache(k_cache, v_cache, table)
    max_len = cap if max_len is None else min(max_len, cap)
    _refuse_sizes(R=R, q_heads=q_heads, max_len=max_len)
    return int(lib().kb_cache_attend_workspace_bytes(c, R, q_heads, max_len, int(weights)))


def cache_attend(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor,
                 length: torch.Tensor, *, scale: Optional[float] = None, max_len: Optional[int] = None,
                 seq: Optional[torch.Tensor] = None, n_dev: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                 weight_in: Optional[torch.Tensor] = None, weight_out: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of one new token a row (``q``: R x q_heads x dim) over the first
    ``length[r]`` cached slots of its sequence (kb_cache_attend): returns R x q_heads x dim.

    ``scale`` defaults to 1 / sqrt(dim), ``max_len``, a host-side bound of the lengths,
    to the slots of the table.  ``lse`` (R x q_heads float32) receives the scores'
    log-sum-exp.  ``weight_out`` (seqs x heads x slots float32) receives ``weight_in``
    (zeros; may be the same tensor) plus each slot's probability, summed over the query
    heads that share a key-value head: what cache_evict goes by.  ``ws`` may supply a
    workspace of at least ``cache_attend_workspace_bytes`` bytes.
    """
    c, dev, dtype, heads, dim, cap, seqs = _cache(k_cache, v_cache, table)
    lp = _ask(length, "length", _I32, 0, dev)
    R = length.numel()
    qp, q_stride, q_heads = _ask_rows(q, "q", dtype, R, None, dim, dev)
    if out is None:
        out = _empty(q, (R, q_heads, dim), stream)
    op = _ask_as(out, "out", dtype, (R, q_heads, dim), dev)
    ep = None if lse is None else _ask_as(lse, "lse", _F32, (R, q_heads), dev)
    sp = None if seq is None else _ask(seq, "seq", _I32, R, dev)
    nd = None if n_dev is None else _ask(n_dev, "n_dev", _I32, 1, dev)
    wi = None if weight_in is None else _ask_as(weight_in, "weight_in", _F32, (seqs, heads, cap), dev)
    wo = None if weight_out is None else _ask_as(weight_out, "weight_out", _F32, (seqs, heads, cap), dev)
    if max_len is None or max_len > cap:
        max_len = cap
    elif max_len < 1:
        _refuse_sizes(max_len=max_len)
    L = lib()
    need = L.kb_cache_attend_workspace_bytes(c, R, q_heads, max_len, 0 if wo is None else 1)
    if ws is None and need > 0:
        ws = _empty(q, need, stream, torch.uint8)
    wp, ws_bytes = None, 0
    if ws is not None:
        _need_ws(ws, need)
        wp, ws_bytes = _ask(ws, "ws", ws.dtype, 0, dev), ws.numel() * ws.element_size()
    _run(L.kb_cache_attend, dev, stream, c, R, nd, q_heads, qp, q_stride, dim ** -0.5 if scale is None else scale, sp,
         lp, max_len, op, ep, wi, wo, wp, ws_bytes)
    return out


def cache_evict(k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, length: torch.Tensor, keep: int, *,
                weight: torch.Tensor, position: Optional[torch.Tensor] = None, newest: Optional[torch.Tensor] = None,
                first: int = 0, recent: int = 0, out_table: Optional[torch.Tensor] = None,
                out: Optional[tuple] = None, n_dev: Optional[torch.Tensor] = None, stream=None):
    """Sequences' caches back to ``keep`` slots, head by head those of greatest ``weight``
    and those whose ``position`` is below ``first`` or above ``newest - recent``
    (kb_cache_evict).  Returns (length, weight, position, source): the new lengths, the
    kept slots' weights and positions, and the slot each came from.

    Without ``out_table`` the rows move within their own pages; with it (R x pages int32)
    the kept ones are put there.  Every slot below ``length`` and every place that is
    kept must have a page: holes are not looked for, and one among them leaves a place
    whose weight and position are not those of the row in it.  ``out`` may supply the four results (position None where
    ``position`` is; length and, in place, weight and position may be the inputs).
    """
    c, dev, _, heads, _, cap, seqs = _cache(k_cache, v_cache, table)
    lp = _ask(length, "length", _I32, 0, dev)
    R = length.numel()
    if not 0 <= keep | first | recent | R <= _INT_MAX:
        _refuse_sizes(keep=keep, first=first, recent=recent, rows=R)
    wp = _ask_as(weight, "weight", _F32, (seqs, heads, cap), dev)
    pp = None if position is None else _ask_as(position, "position", _I32, (seqs, heads, cap), dev)
    ne = None if newest is None else _ask(newest, "newest", _I32, R, dev)
    nd = None if n_dev is None else _ask(n_dev, "n_dev", _I32, 1, dev)
    if out_table is None:
        out_table = table
    tp = _ask(out_table, "out_table", _I32, 0, dev)
    if out_table.dim() != 2 or out_table.shape[0] < R:
        raise ValueError(f"out_table must have at least {R} rows of pages, got {tuple(out_table.shape)}")
    out_pages = out_table.shape[1]
    if out_pages > _INT_MAX:
        _refuse_sizes(**{"columns of out_table": out_pages})
    out_cap = out_pages * c.page_size
    if out is None:
        at, shape = k_cache.device, (R, heads, out_cap)
        with torch.cuda.stream(stream):
            out = (torch.empty(R, dtype=_I32, device=at), torch.zeros(shape, dtype=_F32, device=at),
                   None if position is None else torch.full(shape, -1, dtype=_I32, device=at),
                   torch.empty((R, heads, max(keep, 0)), dtype=_I32, device=at))
    if len(out) != 4:
        raise ValueError("out must hold 4 tensors (length, weight, position, source)")
    out_length, out_weight, out_position, source = out
    olp = _ask(out_length, "out length", _I32, R, dev)
    owp = _ask_as(out_weight, "out weight", _F32, (R, heads, out_cap), dev)
    opp = None if out_position is None else _ask_as(out_position, "out position", _I32, (R, heads, out_cap), dev)
    sp = _ask_as(source, "source", _I32, (R, heads, keep), dev) if keep > 0 else _ask(source, "source", _I32, 0, dev)
    _run(lib().kb_cache_evict, dev, stream, c, R, nd, lp, keep, first, recent, ne, wp, pp, tp, out_pages, olp, owp, opp,
         sp)
    return out


def rotary_frequencies(rot_dim: int, *, base: float = 10000.0, factor: float = 1.0,
                       trained_length: Optional[int] = None, slow: float = 1.0, fast: float = 32.0,
                       device=None) -> torch.Tensor:
    """Radians per position of the rot_dim / 2 pairs, float64: base ** (-2 i / rot_dim).

    For contexts ``factor`` times longer than the trained ones every frequency is divided
    by it; with ``trained_length``, only those of pairs that make at most ``slow`` turns
    over that length, those of pairs that make ``fast`` and more stay, and the ones
    between are blended linearly in the number of turns.
    """
    if rot_dim < 2 or rot_dim % 2 != 0:
        raise ValueError(f"rot_dim = {rot_dim}: an even number of values")
    if not base > 0 or not factor > 0 or not fast > slow or (trained_length is not None and trained_length < 1):
        raise ValueError(f"base = {base}, factor = {factor}, trained_length = {trained_length}, slow = {slow}, "
                         f"fast = {fast}")
    w = base ** (-2.0 * torch.arange(rot_dim // 2, dtype=torch.float64) / rot_dim)
    if trained_length is None:
        w = w / factor
    else:
        turns = trained_length * w / (2 * math.pi)
        stay = ((turns - slow) / (fast - slow)).clamp(0.0, 1.0)
        w = w * stay + w / factor * (1.0 - stay)
    return w.to(device or "cuda")
