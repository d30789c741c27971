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
from typing import Optional, Union

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


def _on(t: torch.Tensor, name: str, stream):
    """``(device, current device, stream handle)`` of a call over ``t``."""
    if not t.is_cuda:
        _fail(f"{name} must be a GPU tensor")
    device = t.device
    if stream is None:
        stream = torch.cuda.current_stream(device)
    elif stream.device != device:
        _fail(f"the stream is on {stream.device}, {name} on {device}")
    return device, torch.cuda.current_device(), stream.cuda_stream


def _call(device, current: int, function, *args) -> None:
    """A library call with ``device`` as the current one."""
    if device.index == current:
        check(function(*args))
    else:
        with torch.cuda.device(device):
            check(function(*args))


def _misfit(t, name: str, shape, device, dtype=None):
    """The error of a tensor that is not what a call needs."""
    if not t.is_cuda or t.device != device:
        _fail(f"{name} must be a GPU tensor on {device}")
    if t.shape != shape:
        _fail(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        _fail(f"{name} has dtype {t.dtype}, expected {dtype}")
    _fail(f"{name}: rows must be contiguous" if dtype is None else f"{name} must be contiguous")


def _rows(t: torch.Tensor, name: str, shape, device) -> _lib.Rows:
    """The view ``t`` [B, H, T, d] as the library takes it."""
    s = t.stride()
    if t.device != device or t.shape != shape or (s[3] != 1 and t.numel()):
        _misfit(t, name, shape, device)
    return _lib.Rows(t.data_ptr(), s[0], s[1], s[2])


def _array(t: Optional[torch.Tensor], name: str, shape, dtype, device):
    """Address of an optional dense array."""
    if t is None:
        return None
    if t.device != device or t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        _misfit(t, name, shape, device, dtype)
    return t.data_ptr()


def _heads(t: torch.Tensor, name: str) -> torch.Tensor:
    """``[B, H, d]`` (one token) as ``[B, H, 1, d]``."""
    if t.dim() == 4:
        return t
    if t.dim() != 3:
        _fail(f"{name} must be [B, H, T, d] or [B, H, d]")
    return t.unsqueeze(2)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A new tensor of the stream that will write it: memory of another
    stream's could still be in use there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _scratch(workspace: Optional[torch.Tensor], size, device, stream):
    """Address and bytes of the caller's workspace, or of a new one of
    ``size()`` bytes (and that tensor)."""
    if workspace is None:
        need = size()
        if not need:
            return None, 0, None
        workspace = _empty(need, torch.uint8, device, stream)
        return workspace.data_ptr(), need, workspace
    if workspace.device != device or not workspace.is_contiguous():
        _misfit(workspace, "workspace", workspace.shape, device, workspace.dtype)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


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
    n = freqs.numel()
    return _lib.Rotation(_array(freqs, "freqs", (n,), torch.float64, device), n, bool(interleaved), magnitude)


def rope(x: torch.Tensor, freqs: torch.Tensor, positions: Optional[torch.Tensor] = None, first: int = 0,
         interleaved: bool = False, magnitude: float = 1.0, out: Optional[torch.Tensor] = None,
         out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """Rows ``x [B, H, T, d]`` (or ``[B, H, d]``: one token) turned by their
    positions: the first ``2 len(freqs)`` dims of a row in pairs (i, i + len(freqs)),
    or (2 i, 2 i + 1) if ``interleaved``, by ``position * freqs[i]``, times
    ``magnitude``; the rest copied.  Token t is at ``positions [B, T]`` (int32;
    any value) or at ``first + t``.  ``out`` may be ``x`` itself."""
    device, current, s = _on(x, "x", stream)
    x4 = _heads(x, "x")
    if out is None:
        out = _empty(x.shape, out_dtype or x.dtype, device, stream)
    elif out_dtype is not None and out.dtype != out_dtype:
        _fail(f"out has dtype {out.dtype}, expected {out_dtype}")
    o4 = _heads(out, "out")
    shape = x4.shape
    B, H, T, d = shape
    if positions is not None and positions.dim() == 1:
        positions = positions.unsqueeze(1)
    pos = _array(positions, "positions", (B, T), torch.int32, device)
    r = _rotation(freqs, interleaved, magnitude, device)
    _call(device, current, _lib.load().santapp_rope, r, _rows(x4, "x", shape, device), _code(x, "x"), B, H, T, d, pos,
          int(first), _rows(o4, "out", shape, device), _code(out, "out"), s)
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
    device, current, s = _on(k, "k", stream)
    k4, v4 = _heads(k, "k"), _heads(v, "v")
    shape = k4.shape
    B, Hkv, T, d = shape
    if v.dtype != k.dtype or cache_V.dtype != cache_K.dtype:
        _fail("k and v, and the two caches, must have one type each")
    if cache_K.dim() != 4:
        _fail("cache_K must be [B, Hkv, capacity, d]")
    cap = cache_K.shape[2]
    held = (B, Hkv, cap, d)
    Hq, qr, qo, qc, oc = 0, None, None, 0, 0
    if q is not None:
        q4 = _heads(q, "q")
        Hq = q4.shape[1]
        if q_out is None:
            q_out = _empty(q.shape, torch.float32, device, stream)
        qs = (B, Hq, T, d)
        qr, qo = _rows(q4, "q", qs, device), _rows(_heads(q_out, "q_out"), "q_out", qs, device)
        qc, oc = _code(q, "q"), _code(q_out, "q_out")
    elif q_out is not None:
        _fail("q_out without q")
    row0, rows = 0, None
    if isinstance(at, torch.Tensor):
        rows = _array(at, "at", (B,), torch.int32, device)
    else:
        row0 = int(at)
    if positions is not None and positions.dim() == 1:
        positions = positions.unsqueeze(1)
    pos = _array(positions, "positions", (B, T), torch.int32, device)
    _call(device, current, _lib.load().santapp_rope_append, _rotation(freqs, interleaved, magnitude, device), qr, qc, qo,
          oc, _rows(k4, "k", shape, device), _rows(v4, "v", shape, device), _code(k, "k"),
          _rows(cache_K, "cache_K", held, device), _rows(cache_V, "cache_V", held, device), _code(cache_K, "cache_K"), cap,
          B, Hq, Hkv, T, d, rows, row0, pos, int(first), s)
    return q_out


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------


def _score(scale, softcap, slopes, window, Hq, device) -> _lib.Score:
    return _lib.Score(scale, softcap, _array(slopes, "slopes", (Hq,), torch.float32, device), int(window))


def prompt_workspace(B: int, Hq: int, Hkv: int, T: int, N: int, d: int, dtype: torch.dtype = torch.bfloat16,
                     window: int = 0, documents: bool = False, device="cuda") -> torch.Tensor:
    """Workspace of :func:`prompt_attention` at these sizes (uninitialised)."""
    n = ctypes.c_size_t()
    with torch.cuda.device(device):
        check(_lib.load().santapp_prompt_workspace_bytes(B, Hq, Hkv, T, N, d, _dtype(dtype), window, documents,
                                                         ctypes.byref(n)))
    return torch.empty(max(n.value, 1), dtype=torch.uint8, device=device)


def _dtype(dtype: torch.dtype) -> int:
    if dtype not in (torch.bfloat16, torch.float32):
        raise SantappError(_lib.EDTYPE, f"unsupported dtype {dtype}")
    return _lib.BF16 if dtype == torch.bfloat16 else _lib.FP32


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
    device, current, s = _on(q, "q", stream)
    if q.dim() != 4 or K.dim() != 4:
        _fail("q and K must be [B, H, tokens, d]")
    shape = q.shape
    B, Hq, T, d = shape
    Hkv, N = K.shape[1], K.shape[2]
    dtype = q.dtype
    if K.dtype != dtype or V.dtype != dtype:
        _fail(f"q, K and V must have one type, got {dtype}, {K.dtype}, {V.dtype}")
    code = _code(q, "q")
    if offset is None:
        offset = N - T if N >= T or causal else 0
    if out is None:
        if stream is None:
            out = torch.empty_like(q)  # q's order of dimensions where q is dense
        else:
            with torch.cuda.stream(stream):
                out = torch.empty_like(q)
    elif out.dtype != dtype:
        _fail(f"out has dtype {out.dtype}, expected {dtype}")
    keys = (B, Hkv, N, d)
    qr, kr, vr = _rows(q, "q", shape, device), _rows(K, "K", keys, device), _rows(V, "V", keys, device)
    orr = _rows(out, "out", shape, device)
    docs = _array(documents, "documents", (B, N), torch.int32, device)
    pre = _array(prefix, "prefix", (B,), torch.int32, device)
    lib = _lib.load()

    def size():
        n = ctypes.c_size_t()
        _call(device, current, lib.santapp_prompt_workspace_bytes, B, Hq, Hkv, T, N, d, code, int(window), docs is not None, n)
        return n.value
    ws, ws_bytes, hold = _scratch(workspace, size, device, stream)
    _call(device, current, lib.santapp_prompt_attention, _score(scale, softcap, slopes, window, Hq, device), qr, kr, vr, code,
          B, Hq, Hkv, T, N, d, bool(causal), int(offset), docs, pre, orr, ws, ws_bytes, s)
    return out


def prefix_workspace(P: int, S: int, Hq: int, Hkv: int, N: int, T: int, d: int, dtype: torch.dtype = torch.bfloat16,
                     device="cuda") -> torch.Tensor:
    """Workspace of :func:`prefix_decode` at these sizes (uninitialised)."""
    n = ctypes.c_size_t()
    with torch.cuda.device(device):
        check(_lib.load().santapp_prefix_workspace_bytes(P, S, Hq, Hkv, N, T, d, _dtype(dtype), ctypes.byref(n)))
    return torch.empty(max(n.value, 1), dtype=torch.uint8, device=device)


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
    device, current, s = _on(q, "q", stream)
    if q.dim() != 3 or K.dim() != 4:
        _fail("q must be [B, Hq, d], K [P, Hkv, N, d]")
    shape = q.shape
    B, Hq, d = shape
    P, Hkv, N, _ = K.shape
    if P < 1 or B % P:
        _fail(f"{B} sequences over {P} prompts")
    S = B // P
    dtype = K.dtype
    if V.dtype != dtype:
        _fail("K and V must have one type")
    code = _code(K, "K")
    sk = sv = None
    if suffix_K is None:
        if T or lengths is not None:
            _fail("suffix rows requested without a suffix buffer")
        T = 0
    else:
        if suffix_V is None or suffix_K.dtype != dtype or suffix_V.dtype != dtype:
            _fail("suffix_K and suffix_V must have the type of K")
        if suffix_K.dim() != 4:
            _fail("suffix_K must be [B, Hkv, capacity, d]")
        cap = suffix_K.shape[2]
        held = (B, Hkv, cap, d)
        sk, sv = _rows(suffix_K, "suffix_K", held, device), _rows(suffix_V, "suffix_V", held, device)
        T = cap if T is None else int(T)
        if T < 0 or T > cap:
            _fail(f"T={T} outside the suffix buffer's {cap} rows")
    if out is None:
        out = _empty(shape, torch.float32, device, stream)
    keys = (P, Hkv, N, d)
    kr, vr = _rows(K, "K", keys, device), _rows(V, "V", keys, device)
    lib = _lib.load()

    def size():
        n = ctypes.c_size_t()
        _call(device, current, lib.santapp_prefix_workspace_bytes, P, S, Hq, Hkv, N, T, d, code, n)
        return n.value
    ws, ws_bytes, hold = _scratch(workspace, size, device, stream)
    _call(device, current, lib.santapp_prefix_decode, _score(scale, softcap, slopes, window, Hq, device),
          _array(q, "q", shape, torch.float32, device), kr, vr, code, P, S, Hq, Hkv, N, d, _array(prefix_lengths, "prefix_lengths", (P,), torch.int32, device), sk, sv, T,
          _array(lengths, "lengths", (B,), torch.int32, device), _array(positions, "positions", (B,), torch.int32, device),
          _array(out, "out", shape, torch.float32, device), ws, ws_bytes, s)
    return out
