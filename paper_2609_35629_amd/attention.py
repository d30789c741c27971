"""Rotary positions, prompt attention and decoding over a shared prompt.

What a decoder runs around the team tables: :func:`rope` and
:func:`rope_append` turn queries and keys by their positions (and write a step's
rows into the cache), :func:`prompt_attention` is the prompt's own attention,
:func:`prefix_decode` the exact step of several sequences over one prompt.

Tensors may be any views whose rows of ``d`` elements are contiguous and start
at multiples of 16 bytes (a projection's ``[B, T, H, d]`` seen as ``[B, H, T, d]``,
say).  Every call runs on the tensors' device, on its current stream unless
``stream`` is given.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple, Union

import torch

from . import _lib
from ._lib import SantappError, check


def _fail(message: str):
    raise SantappError(_lib.EINVAL, message)


def _code(t: torch.Tensor, name: str) -> int:
    if t.dtype == torch.bfloat16:
        return _lib.BF16
    if t.dtype == torch.float32:
        return _lib.FP32
    raise SantappError(_lib.EDTYPE, f"unsupported dtype {t.dtype} of {name}")


def _rows(t: torch.Tensor, name: str, shape, device) -> _lib.Rows:
    """The view ``t`` [B, H, T, d] as the library takes it."""
    if not t.is_cuda or t.device != device:
        _fail(f"{name} must be a GPU tensor on {device}")
    if tuple(t.shape) != tuple(shape):
        _fail(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.numel() and t.stride(3) != 1:
        _fail(f"{name}: rows must be contiguous")
    return _lib.Rows(t.data_ptr(), *t.stride()[:3])


def _array(t: Optional[torch.Tensor], name: str, shape, dtype, device):
    """Address of an optional dense array."""
    if t is None:
        return None
    if not t.is_cuda or t.device != device:
        _fail(f"{name} must be a GPU tensor on {device}")
    if tuple(t.shape) != tuple(shape):
        _fail(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype != dtype:
        _fail(f"{name} has dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        _fail(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


class _On:
    """The device of a call's tensors as the current one, and the stream."""

    def __init__(self, t: torch.Tensor, name: str, stream):
        if not t.is_cuda:
            _fail(f"{name} must be a GPU tensor")
        self.device = t.device
        if stream is not None and stream.device != t.device:
            _fail(f"the stream is on {stream.device}, {name} on {t.device}")
        s = stream if stream is not None else torch.cuda.current_stream(t.device)
        self.stream = ctypes.c_void_p(s.cuda_stream)
        self._guard = torch.cuda.device(t.device)

    def __enter__(self):
        self._guard.__enter__()
        return self

    def __exit__(self, *e):
        self._guard.__exit__(*e)
        return False


def _heads(t: torch.Tensor, name: str) -> torch.Tensor:
    """``[B, H, d]`` (one token) as ``[B, H, 1, d]``."""
    if t.dim() == 3:
        return t.unsqueeze(2)
    if t.dim() != 4:
        _fail(f"{name} must be [B, H, T, d] or [B, H, d]")
    return t


def _same_memory(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether the address ranges of two tensors meet."""
    if not a.numel() or not b.numel():
        return False

    def ends(t):
        last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
        return t.data_ptr(), t.data_ptr() + (last + 1) * t.element_size()
    (a0, a1), (b0, b1) = ends(a), ends(b)
    return a0 < b1 and b0 < a1


def _scratch(workspace: Optional[torch.Tensor], need: int, device) -> Tuple[Optional[ctypes.c_void_p], int,
                                                                           Optional[torch.Tensor]]:
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    elif not workspace.is_cuda or workspace.device != device:
        _fail(f"workspace must be a GPU tensor on {device}")
    elif not workspace.is_contiguous():
        _fail("workspace must be contiguous")
    if workspace is None:
        return None, 0, None
    return ctypes.c_void_p(workspace.data_ptr()), workspace.numel() * workspace.element_size(), workspace


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------


def rope_frequencies(rot: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                     original_length: int = 0, low: float = 1.0, high: float = 32.0,
                     device="cuda") -> torch.Tensor:
    """Radians per position ``[rot / 2]`` (fp64) of the pairs of ``rot`` rotated
    dims: ``base ** (-2 i / rot)``, stretched for contexts ``factor`` times the
    trained length:

    - ``"linear"``: every frequency divided by ``factor``;
    - ``"base"``: the base raised to ``base * factor ** (rot / (rot - 2))``, so
      that the slowest frequency is divided by ``factor`` and the fastest kept;
    - ``"bands"``: a frequency that turns at least ``high`` times within
      ``original_length`` positions is kept, one that turns at most ``low`` times
      divided by ``factor``, linear in the number of turns between.
    """
    if rot < 2 or rot % 2:
        _fail("rot must be a positive even number")
    if not (base > 0 and math.isfinite(base)) or not (factor > 0 and math.isfinite(factor)):
        _fail("base and factor must be positive")
    if scaling == "base":
        if rot == 2:
            _fail("base scaling needs more than one frequency")
        base = base * factor ** (rot / (rot - 2))
    f = float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaling == "linear":
        f = f / factor
    elif scaling == "bands":
        if original_length < 1 or not low < high:
            _fail("bands need original_length and low < high")
        keep = ((original_length * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    elif scaling not in (None, "base"):
        _fail(f"unknown scaling {scaling!r}")
    return f.to(device)


def _rotation(freqs: torch.Tensor, interleaved: bool, magnitude: float, device) -> _lib.Rotation:
    f = _array(freqs, "freqs", (freqs.numel(),), torch.float64, device)
    return _lib.Rotation(f, freqs.numel(), int(bool(interleaved)), float(magnitude))


def rope(x: torch.Tensor, freqs: torch.Tensor, positions: Optional[torch.Tensor] = None, first: int = 0,
         interleaved: bool = False, magnitude: float = 1.0, out: Optional[torch.Tensor] = None,
         out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """Rows ``x [B, H, T, d]`` (or ``[B, H, d]``: one token) turned by their
    positions: the first ``2 len(freqs)`` dims of a row in pairs (i, i + len(freqs)),
    or (2 i, 2 i + 1) if ``interleaved``, by ``position * freqs[i]``, times
    ``magnitude``; the rest copied.  Token t is at ``positions [B, T]`` (int32;
    any value) or at ``first + t``.  ``out`` may be ``x`` itself."""
    with _On(x, "x", stream) as on:
        x4 = _heads(x, "x")
        B, H, T, d = x4.shape
        if out is None:
            out = torch.empty_like(x4, dtype=out_dtype or x.dtype, memory_format=torch.contiguous_format).view(x.shape)
        elif out_dtype is not None and out.dtype != out_dtype:
            _fail(f"out has dtype {out.dtype}, expected {out_dtype}")
        if out.shape != x.shape:
            _fail(f"out has shape {tuple(out.shape)}, expected {tuple(x.shape)}")
        o4 = _heads(out, "out")
        if _same_memory(o4, x4) and not (o4.data_ptr() == x4.data_ptr() and o4.stride() == x4.stride() and
                                         o4.dtype == x4.dtype):
            _fail("out overlaps x without being x")
        if positions is not None and positions.dim() == 1:
            positions = positions.unsqueeze(1)
        pos = _array(positions, "positions", (B, T), torch.int32, on.device)
        r = _rotation(freqs, interleaved, magnitude, on.device)
        xr, yr = _rows(x4, "x", (B, H, T, d), on.device), _rows(o4, "out", (B, H, T, d), on.device)
        check(_lib.load().santapp_rope(ctypes.byref(r), ctypes.byref(xr), _code(x, "x"), B, H, T, d, pos, int(first),
                                       ctypes.byref(yr), _code(out, "out"), on.stream))
    return out


def rope_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, cache_K: torch.Tensor,
                cache_V: torch.Tensor, freqs: torch.Tensor, at: Union[int, torch.Tensor],
                positions: Optional[torch.Tensor] = None, first: int = 0, interleaved: bool = False,
                magnitude: float = 1.0, q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """T new tokens of every sequence in one launch: ``k [B, Hkv, T, d]`` turned
    into rows ``at[b] + t`` of ``cache_K [B, Hkv, capacity, d]``, ``v`` copied to
    the same rows of ``cache_V``, ``q [B, Hq, T, d]`` turned into ``q_out`` (new
    and fp32 unless given), which is returned.  ``[B, H, d]`` is one token;
    ``q`` may be None.  ``at``: the rows in use, one number or int32 ``[B]``
    (the caller advances it; rows outside the cache are dropped when it is a
    tensor, refused when it is a number).  Token t is at ``positions [B, T]`` or
    at ``first + at[b] + t``."""
    with _On(k, "k", stream) as on:
        k4, v4 = _heads(k, "k"), _heads(v, "v")
        B, Hkv, T, d = k4.shape
        if v.dtype != k.dtype or cache_V.dtype != cache_K.dtype:
            _fail("k and v, and the two caches, must have one type each")
        if cache_K.dim() != 4:
            _fail("cache_K must be [B, Hkv, capacity, d]")
        cap = cache_K.shape[2]
        kr, vr = _rows(k4, "k", (B, Hkv, T, d), on.device), _rows(v4, "v", (B, Hkv, T, d), on.device)
        ck = _rows(cache_K, "cache_K", (B, Hkv, cap, d), on.device)
        cv = _rows(cache_V, "cache_V", (B, Hkv, cap, d), on.device)
        Hq, qr, qo, qc, oc = 0, None, None, _lib.BF16, _lib.BF16
        ins = [k4, v4]
        outs = [cache_K, cache_V]
        if q is not None:
            q4 = _heads(q, "q")
            Hq = q4.shape[1]
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=torch.float32, device=on.device)
            if q_out.shape != q.shape:
                _fail(f"q_out has shape {tuple(q_out.shape)}, expected {tuple(q.shape)}")
            o4 = _heads(q_out, "q_out")
            qr = ctypes.byref(_rows(q4, "q", (B, Hq, T, d), on.device))
            qo = ctypes.byref(_rows(o4, "q_out", (B, Hq, T, d), on.device))
            qc, oc = _code(q, "q"), _code(q_out, "q_out")
            if not (o4.data_ptr() == q4.data_ptr() and o4.stride() == q4.stride() and q.dtype == q_out.dtype):
                ins.append(q4)
            outs.append(o4)
        elif q_out is not None:
            _fail("q_out without q")
        for i, o in enumerate(outs):
            if any(_same_memory(o, x) for x in ins + outs[:i]):
                _fail("the caches and q_out must not overlap the inputs or each other")
        row0, rows = 0, None
        if isinstance(at, torch.Tensor):
            rows = _array(at, "at", (B,), torch.int32, on.device)
        else:
            row0 = int(at)
        if positions is not None and positions.dim() == 1:
            positions = positions.unsqueeze(1)
        pos = _array(positions, "positions", (B, T), torch.int32, on.device)
        r = _rotation(freqs, interleaved, magnitude, on.device)
        check(_lib.load().santapp_rope_append(
            ctypes.byref(r), qr, qc, qo, oc, ctypes.byref(kr), ctypes.byref(vr), _code(k, "k"), ctypes.byref(ck),
            ctypes.byref(cv), _code(cache_K, "cache_K"), cap, B, Hq, Hkv, T, d, rows, row0, pos, int(first), on.stream))
    return q_out


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------


def _score(scale, softcap, slopes, window, Hq, device) -> _lib.Score:
    return _lib.Score(float(scale), float(softcap), _array(slopes, "slopes", (Hq,), torch.float32, device), int(window))


def prompt_workspace(B: int, Hq: int, Hkv: int, T: int, N: int, d: int, dtype: torch.dtype = torch.bfloat16,
                     window: int = 0, documents: bool = False, device="cuda") -> torch.Tensor:
    """Workspace of :func:`prompt_attention` at these sizes (uninitialised)."""
    return torch.empty(max(_prompt_bytes(B, Hq, Hkv, T, N, d, dtype, window, documents, torch.device(device)), 1),
                       dtype=torch.uint8, device=device)


def _prompt_bytes(B, Hq, Hkv, T, N, d, dtype, window, documents, device) -> int:
    n = ctypes.c_size_t()
    with torch.cuda.device(device):
        check(_lib.load().santapp_prompt_workspace_bytes(B, Hq, Hkv, T, N, d,
                                                         _lib.BF16 if dtype == torch.bfloat16 else _lib.FP32,
                                                         int(window), int(documents), ctypes.byref(n)))
    return n.value


def prompt_attention(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, causal: bool = True,
                     offset: Optional[int] = None, window: int = 0, softcap: float = 0.0,
                     slopes: Optional[torch.Tensor] = None, documents: Optional[torch.Tensor] = None,
                     prefix: Optional[torch.Tensor] = None, scale: float = 0.0, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Softmax attention of query tokens ``q [B, Hq, T, d]`` over ``K, V
    [B, Hkv, N, d]`` (one type, bf16 or fp32); ``out`` like ``q``.

    Query t is token ``offset + t`` of the sequence (default: the last T).  It
    attends key j if ``causal`` is false, j is not behind it, or j < ``prefix[b]``;
    if it is nearer than ``window`` (> 0); and if both tokens' ``documents
    [B, N]`` (int32) are equal and not negative.  Scores are ``scale q.k`` (0:
    1 / sqrt(d)), capped by ``softcap * tanh(s / softcap)`` when ``softcap`` > 0, less
    ``slopes[h]`` per token of distance.  A query that attends nothing gets 0."""
    with _On(q, "q", stream) as on:
        if q.dim() != 4 or K.dim() != 4:
            _fail("q and K must be [B, H, tokens, d]")
        B, Hq, T, d = q.shape
        Hkv, N = K.shape[1], K.shape[2]
        if K.dtype != q.dtype or V.dtype != q.dtype:
            _fail(f"q, K and V must have one type, got {q.dtype}, {K.dtype}, {V.dtype}")
        code = _code(q, "q")
        if offset is None:
            offset = N - T if N >= T or causal else 0
        if out is None:
            out = torch.empty_like(q, memory_format=torch.preserve_format if _dense(q) else torch.contiguous_format)
        if out.dtype != q.dtype:
            _fail(f"out has dtype {out.dtype}, expected {q.dtype}")
        if any(_same_memory(out, x) for x in (q, K, V)):
            _fail("out must not overlap q, K or V")
        qr, orr = _rows(q, "q", (B, Hq, T, d), on.device), _rows(out, "out", (B, Hq, T, d), on.device)
        kr, vr = _rows(K, "K", (B, Hkv, N, d), on.device), _rows(V, "V", (B, Hkv, N, d), on.device)
        sc = _score(scale, softcap, slopes, window, Hq, on.device)
        docs = _array(documents, "documents", (B, N), torch.int32, on.device)
        pre = _array(prefix, "prefix", (B,), torch.int32, on.device)
        need = 0
        if workspace is None:
            need = _prompt_bytes(B, Hq, Hkv, T, N, d, q.dtype, window, documents is not None, on.device)
        ws, ws_bytes, keep = _scratch(workspace, need, on.device)
        check(_lib.load().santapp_prompt_attention(
            ctypes.byref(sc), ctypes.byref(qr), ctypes.byref(kr), ctypes.byref(vr), code, B, Hq, Hkv, T, N, d,
            int(bool(causal)), int(offset), docs, pre, ctypes.byref(orr), ws, ws_bytes, on.stream))
        _hold(keep, workspace, stream)
    return out


def _dense(t: torch.Tensor) -> bool:
    """Whether the view covers its memory without gaps or repeats, rows whole."""
    n = 1
    for size, stride in sorted(zip(t.shape, t.stride()), key=lambda x: (x[1], x[0])):
        if size != 1 and stride != n:
            return False
        n *= size
    return t.stride(3) == 1


def _hold(keep, given, stream):
    """A workspace made for a call on a stream that is not the current one must
    not be given out again before that stream has passed it."""
    if keep is not None and given is None and stream is not None:
        keep.record_stream(stream)


def prefix_workspace(P: int, S: int, Hq: int, Hkv: int, N: int, T: int, d: int, dtype: torch.dtype = torch.bfloat16,
                     device="cuda") -> torch.Tensor:
    """Workspace of :func:`prefix_decode` at these sizes (uninitialised)."""
    return torch.empty(max(_prefix_bytes(P, S, Hq, Hkv, N, T, d, dtype, torch.device(device)), 1), dtype=torch.uint8,
                       device=device)


def _prefix_bytes(P, S, Hq, Hkv, N, T, d, dtype, device) -> int:
    n = ctypes.c_size_t()
    with torch.cuda.device(device):
        check(_lib.load().santapp_prefix_workspace_bytes(P, S, Hq, Hkv, N, T, d,
                                                         _lib.BF16 if dtype == torch.bfloat16 else _lib.FP32,
                                                         ctypes.byref(n)))
    return n.value


def prefix_decode(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, suffix_K: Optional[torch.Tensor] = None,
                  suffix_V: Optional[torch.Tensor] = None, T: Optional[int] = None,
                  lengths: Optional[torch.Tensor] = None, prefix_lengths: Optional[torch.Tensor] = None,
                  positions: Optional[torch.Tensor] = None, window: int = 0, softcap: float = 0.0,
                  slopes: Optional[torch.Tensor] = None, scale: float = 0.0, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One exact decode step of several sequences per prompt: ``q [B, Hq, d]``
    fp32 -> ``out [B, Hq, d]`` fp32.

    Sequence b attends prompt ``b // (B / P)`` of ``K, V [P, Hkv, N, d]`` (its
    first ``prefix_lengths[p]`` rows; int32) and the first ``T`` (default: all) or
    ``lengths[b]`` rows of its own suffix ``[B, Hkv, capacity, d]``.  Scores as in
    :func:`prompt_attention`; for ``window`` and ``slopes`` the query stands at
    ``positions[b]`` (int32; default: its last row)."""
    with _On(q, "q", stream) as on:
        if q.dim() != 3 or K.dim() != 4:
            _fail("q must be [B, Hq, d], K [P, Hkv, N, d]")
        B, Hq, d = q.shape
        P, Hkv, N = K.shape[:3]
        if P < 1 or B % P:
            _fail(f"{B} sequences over {P} prompts")
        if V.dtype != K.dtype:
            _fail("K and V must have one type")
        qp = _array(q, "q", (B, Hq, d), torch.float32, on.device)
        code = _code(K, "K")
        kr, vr = _rows(K, "K", (P, Hkv, N, d), on.device), _rows(V, "V", (P, Hkv, N, d), on.device)
        sk = sv = None
        if suffix_K is None:
            if T or lengths is not None:
                _fail("suffix rows requested without a suffix buffer")
            T = 0
        else:
            if suffix_V is None or suffix_K.dtype != K.dtype or suffix_V.dtype != K.dtype:
                _fail("suffix_K and suffix_V must have the type of K")
            if suffix_K.dim() != 4:
                _fail("suffix_K must be [B, Hkv, capacity, d]")
            cap = suffix_K.shape[2]
            sk = ctypes.byref(_rows(suffix_K, "suffix_K", (B, Hkv, cap, d), on.device))
            sv = ctypes.byref(_rows(suffix_V, "suffix_V", (B, Hkv, cap, d), on.device))
            T = cap if T is None else int(T)
            if T < 0 or T > cap:
                _fail(f"T={T} outside the suffix buffer's {cap} rows")
        if out is None:
            out = torch.empty((B, Hq, d), dtype=torch.float32, device=on.device)
        op = _array(out, "out", (B, Hq, d), torch.float32, on.device)
        if any(_same_memory(out, x) for x in (q, K, V, suffix_K, suffix_V) if x is not None):
            _fail("out must not overlap q or the caches")
        sc = _score(scale, softcap, slopes, window, Hq, on.device)
        lens = _array(lengths, "lengths", (B,), torch.int32, on.device)
        plens = _array(prefix_lengths, "prefix_lengths", (P,), torch.int32, on.device)
        pos = _array(positions, "positions", (B,), torch.int32, on.device)
        need = 0
        if workspace is None:
            need = _prefix_bytes(P, B // P, Hq, Hkv, N, T, d, K.dtype, on.device)
        ws, ws_bytes, keep = _scratch(workspace, need, on.device)
        check(_lib.load().santapp_prefix_decode(
            ctypes.byref(sc), qp, ctypes.byref(kr), ctypes.byref(vr), code, P, B // P, Hq, Hkv, N, d, plens, sk, sv, T,
            lens, pos, op, ws, ws_bytes, on.stream))
        _hold(keep, workspace, stream)
    return out
