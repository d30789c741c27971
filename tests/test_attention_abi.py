"""Refusals of the rotation, prompt-attention and shared-prefix entry points:
host-side checks that answer before anything is launched (no GPU needed; the
addresses are never dereferenced)."""
import ctypes
import functools
import os
import subprocess
import sys

import pytest
import torch

import paper_2609_35629_amd as sp
from paper_2609_35629_amd import _lib
from tests.test_api_sanitizers import ROOT, _asan_runtime

FAKE, ODD = 1 << 20, (1 << 20) + 8
BF16, FP32 = _lib.BF16, _lib.FP32


def rows(data=FAKE, b=1 << 16, h=1 << 12, t=128):
    return ctypes.byref(_lib.Rows(data, b, h, t))


def rotation(freqs=FAKE, pairs=32, inter=0, magnitude=1.0):
    return ctypes.byref(_lib.Rotation(freqs, pairs, inter, magnitude))


def score(scale=0.0, cap=0.0, slopes=None, window=0):
    return ctypes.byref(_lib.Score(scale, cap, slopes, window))


def refused(status, text, code=_lib.EINVAL):
    assert status == code, (status, _lib.load().santapp_last_error())
    assert text.encode() in _lib.load().santapp_last_error(), _lib.load().santapp_last_error()


def test_rope_refusals():
    L = _lib.load()

    def call(rot=None, x=None, xd=BF16, B=1, H=2, T=4, d=64, pos=None, out=None, od=BF16):
        return L.santapp_rope(rot or rotation(), x or rows(), xd, B, H, T, d, pos, 0, out or rows(), od, None)
    refused(call(B=0), "invalid sizes")
    refused(call(H=0), "invalid sizes")
    refused(call(T=-1), "invalid sizes")
    refused(call(xd=7), "dtype", _lib.EDTYPE)
    refused(call(od=-1), "dtype", _lib.EDTYPE)
    refused(call(d=96), "head dim", _lib.ELIMIT)
    refused(call(rot=rotation(freqs=None)), "freqs")
    refused(call(rot=rotation(freqs=FAKE + 4)), "freqs must be 8-byte aligned")
    refused(call(rot=rotation(pairs=0)), "pairs")
    refused(call(rot=rotation(pairs=33)), "pairs")
    refused(call(rot=rotation(inter=2)), "interleaved")
    refused(call(rot=rotation(magnitude=float("nan"))), "magnitude")
    refused(call(pos=ctypes.c_void_p(FAKE + 2)), "positions")
    refused(call(x=rows(None)), "x is NULL")
    refused(call(x=rows(ODD)), "x must be 16-byte aligned")
    refused(call(x=rows(t=100)), "multiples of 16 bytes")
    refused(call(x=rows(t=-64)), "not negative")
    refused(call(out=rows(t=56)), "rows overlap")       # closer than a row
    refused(call(out=rows(h=128, t=128)), "rows overlap")
    refused(call(out=rows(t=0)), "rows overlap")
    refused(call(out=rows(FAKE + 128)), "out overlaps x")
    refused(call(out=rows(t=256)), "out overlaps x")
    refused(call(od=FP32), "out overlaps x")            # in place, but of another type
    refused(call(B=1 << 16, T=1 << 16), "too many rows", _lib.ELIMIT)
    assert call(T=0, x=rows(None)) == _lib.OK           # nothing to do
    assert L.santapp_rope(None, rows(), BF16, 1, 1, 1, 64, None, 0, rows(), BF16, None) == _lib.EINVAL


def test_rope_append_refusals():
    L = _lib.load()
    far = [FAKE + (i << 24) for i in range(8)]

    def call(q=None, Hq=0, k=None, v=None, kd=BF16, ck=None, cv=None, cd=BF16, cap=16, B=1, Hkv=2, T=4, d=64, at=None,
             at0=0, qo=None, qd=BF16, od=FP32):
        return L.santapp_rope_append(rotation(), q, qd, qo, od, k or rows(), v or rows(), kd, ck or rows(), cv or rows(), cd,
                                     cap, B, Hq, Hkv, T, d, at, at0, None, 0, None)
    refused(call(cap=0), "invalid sizes")
    refused(call(Hkv=0), "invalid sizes")
    refused(call(Hq=4), "q must be given")
    refused(call(q=rows()), "q must be given")
    refused(call(q=rows(), Hq=4, qo=rows(None)), "q_out is NULL")
    refused(call(q=rows(), Hq=4), "q_out is NULL")
    refused(call(q=rows(), Hq=4, qo=rows(), qd=9), "dtype", _lib.EDTYPE)
    refused(call(kd=9), "dtype", _lib.EDTYPE)
    refused(call(cd=9), "dtype", _lib.EDTYPE)
    refused(call(at0=13), "outside the cache")
    refused(call(at0=-1), "outside the cache")
    refused(call(at0=2 ** 31 - 1), "outside the cache")
    refused(call(at=ctypes.c_void_p(FAKE + 1)), "at must be 4-byte aligned")
    refused(call(k=rows(ODD)), "k must be 16-byte aligned")
    refused(call(v=rows(None)), "v is NULL")
    refused(call(ck=rows(t=32)), "cache_K: rows overlap")
    refused(call(cv=rows(h=32)), "cache_V: rows overlap")  # (64: two heads side by side in a token of 128)
    refused(call(d=32), "head dim", _lib.ELIMIT)
    apart = dict(k=rows(far[0]), v=rows(far[1]), ck=rows(far[2]), cv=rows(far[3]))
    refused(call(**dict(apart, ck=rows(far[0] + 16))), "cache_K overlaps k")
    refused(call(**dict(apart, cv=rows(far[1]))), "cache_V overlaps v")
    refused(call(**dict(apart, cv=rows(far[2]))), "cache_V overlaps cache_K")
    refused(call(**apart, q=rows(far[4]), Hq=2, qo=rows(far[4])), "q_out overlaps q")  # of another type
    refused(call(**apart, q=rows(far[4]), Hq=2, qo=rows(far[2])), "cache_K overlaps q_out")
    assert call(T=0) == _lib.OK


def test_prompt_refusals():
    L = _lib.load()

    def call(sc=None, q=None, K=None, V=None, dt=BF16, B=1, Hq=4, Hkv=2, T=4, N=16, d=64, causal=1, offset=12, docs=None,
             prefix=None, out=None, ws=FAKE, wb=1 << 40):
        return L.santapp_prompt_attention(sc or score(), q or rows(), K or rows(), V or rows(), dt, B, Hq, Hkv, T, N, d,
                                          causal, offset, docs, prefix, out or rows(), ctypes.c_void_p(ws), wb, None)
    refused(call(B=0), "invalid sizes")
    refused(call(N=-1), "invalid sizes")
    refused(call(Hq=3), "multiple of Hkv")
    refused(call(Hq=0), "multiple of Hkv")
    refused(call(dt=2), "dtype", _lib.EDTYPE)
    refused(call(d=80), "head dim", _lib.ELIMIT)
    refused(call(N=1 << 24, offset=0), "2^24", _lib.ELIMIT)
    refused(call(T=1 << 29, N=1 << 23, causal=0), "too many rows", _lib.ELIMIT)
    refused(call(B=1 << 20, Hq=1 << 12, Hkv=1 << 12, T=1, offset=0), "too many rows", _lib.ELIMIT)
    for bad in (dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=1e-39), dict(scale=1e31)):
        refused(call(sc=score(**bad)), "scale")
    for bad in (-1.0, float("nan"), 1e-35, 1e32):
        refused(call(sc=score(cap=bad)), "softcap")
    refused(call(sc=score(window=-1)), "window")
    refused(call(sc=score(slopes=FAKE + 2)), "slopes")
    refused(call(causal=2), "causal")
    refused(call(causal=0, prefix=ctypes.c_void_p(FAKE)), "prefix")
    refused(call(docs=ctypes.c_void_p(FAKE + 1)), "documents")
    refused(call(offset=13), "not tokens")
    refused(call(offset=-1), "not tokens")
    refused(call(offset=2 ** 31 - 1), "not tokens")
    refused(call(causal=0, offset=13, sc=score(window=3)), "not tokens")
    refused(call(causal=0, offset=13, sc=score(slopes=FAKE)), "not tokens")
    refused(call(causal=0, offset=13, docs=ctypes.c_void_p(FAKE)), "not tokens")
    refused(call(q=rows(ODD)), "q must be 16-byte aligned")
    refused(call(K=rows(None)), "K is NULL")
    refused(call(V=rows(t=4)), "V: distances")
    refused(call(V=rows(t=1 << 30)), "bytes apart", _lib.ELIMIT)
    refused(call(out=rows(t=0)), "out: rows overlap")
    refused(call(), "out overlaps q")
    call = functools.partial(call, out=rows(FAKE + (1 << 28)))
    refused(call(K=rows(FAKE + (1 << 28))), "out overlaps K")
    refused(call(ws=ODD), "workspace must be 16-byte aligned")
    n = ctypes.c_size_t()
    args = (1, 28, 4, 1, 32768, 128, BF16, 0, 1)
    assert L.santapp_prompt_workspace_bytes(*args, ctypes.byref(n)) == _lib.OK and n.value > 0
    big = dict(Hq=28, Hkv=4, T=1, N=32768, d=128, offset=32767, docs=ctypes.c_void_p(FAKE))
    refused(call(**big, wb=n.value - 1), "workspace of", _lib.EWORKSPACE)
    refused(call(**big, ws=None), "workspace of", _lib.EWORKSPACE)
    refused(L.santapp_prompt_workspace_bytes(*args, None), "bytes")
    refused(L.santapp_prompt_workspace_bytes(1, 27, 4, 1, 32768, 128, BF16, 0, 0, ctypes.byref(n)), "multiple of Hkv")
    refused(L.santapp_prompt_workspace_bytes(1, 28, 4, 1, 32768, 128, BF16, -1, 0, ctypes.byref(n)), "window")
    assert call(T=0, offset=16, q=rows(None)) == _lib.OK
    assert L.santapp_prompt_attention(None, rows(), rows(), rows(), BF16, 1, 4, 2, 4, 16, 64, 1, 12, None, None, rows(), None,
                                      0, None) == _lib.EINVAL


def test_prefix_refusals():
    L = _lib.load()

    def call(sc=None, q=FAKE, K=None, V=None, dt=BF16, P=1, S=2, Hq=4, Hkv=2, N=16, d=64, plens=None, sK=None, sV=None,
             T=8, lens=None, pos=None, out=FAKE, ws=FAKE, wb=1 << 40):
        vp = ctypes.c_void_p
        return L.santapp_prefix_decode(sc or score(), vp(q), K or rows(), V or rows(), dt, P, S, Hq, Hkv, N, d, plens,
                                       sK or rows(), sV or rows(), T, lens, pos, vp(out), vp(ws), wb, None)
    refused(call(q=None), "q and out")
    refused(call(out=None), "q and out")
    refused(call(q=ODD), "16-byte aligned")
    refused(call(ws=ODD), "16-byte aligned")
    refused(call(P=0), "invalid sizes")
    refused(call(S=0), "invalid sizes")
    refused(call(T=-1), "invalid sizes")
    refused(call(Hq=5), "multiple of Hkv")
    refused(call(dt=5), "dtype", _lib.EDTYPE)
    refused(call(d=256), "head dim", _lib.ELIMIT)
    refused(call(N=1 << 24), "2^24", _lib.ELIMIT)
    refused(call(S=1 << 21), "too many rows", _lib.ELIMIT)
    refused(call(sc=score(window=-2)), "window")
    refused(call(lens=ctypes.c_void_p(FAKE + 2)), "lengths")
    refused(call(K=rows(None)), "K is NULL")
    refused(call(sK=rows(None)), "suffix_K is NULL")
    refused(call(sV=rows(ODD)), "suffix_V must be 16-byte aligned")
    refused(call(), "out overlaps q")
    call = functools.partial(call, out=FAKE + (1 << 28))
    refused(call(sV=rows(FAKE + (1 << 28))), "out overlaps suffix_V")
    n = ctypes.c_size_t()
    assert L.santapp_prefix_workspace_bytes(1, 2, 4, 2, 16, 8, 64, BF16, ctypes.byref(n)) == _lib.OK and n.value > 0
    refused(call(wb=n.value - 1), "workspace of", _lib.EWORKSPACE)
    refused(call(ws=None), "workspace of", _lib.EWORKSPACE)
    refused(L.santapp_prefix_workspace_bytes(1, 2, 4, 2, 16, 8, 64, BF16, None), "bytes")
    refused(L.santapp_prefix_workspace_bytes(1, 0, 4, 2, 16, 8, 64, BF16, ctypes.byref(n)), "invalid sizes")


def test_binding_refuses_host_tensors():
    x, f = torch.zeros(1, 2, 3, 64), torch.zeros(32, dtype=torch.float64)
    for call in (lambda: sp.rope(x, f), lambda: sp.rope_append(x, x, x, x, x, f, 0), lambda: sp.prompt_attention(x, x, x),
                 lambda: sp.prefix_decode(x[:, :, 0], x, x)):
        with pytest.raises(sp.SantappError) as e:
            call()
        assert e.value.status == _lib.EINVAL and "GPU tensor" in str(e.value)


def test_frequency_refusals():
    for bad in (dict(rot=0), dict(rot=7), dict(rot=8, factor=0.0), dict(rot=8, base=-1.0), dict(rot=8, scaling="steps"),
                dict(rot=2, scaling="base", factor=2.0), dict(rot=8, scaling="bands", factor=2.0),
                dict(rot=8, scaling="bands", factor=2.0, original_length=10, low=3.0, high=3.0)):
        with pytest.raises(sp.SantappError):
            sp.rope_frequencies(device="cpu", **bad)


CHILD = r"""
import sys
from paper_2609_35629_amd import _lib
_lib.load(sys.argv[1])
import tests.test_attention_abi as T
T.test_rope_refusals()
T.test_rope_append_refusals()
T.test_prompt_refusals()
T.test_prefix_refusals()
print("sanitized attention api ok")
"""


def test_refusals_under_asan_and_ubsan(tmp_path):
    rt = _asan_runtime()
    if rt is None:
        pytest.skip("clang's ASan runtime is not installed")
    from paper_2609_35629_amd import build as B
    so = B.build_host_sanitized(str(tmp_path / "libsantapp_san.so"))
    env = dict(os.environ, LD_PRELOAD=rt, PYTHONPATH=ROOT, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-c", CHILD, so], env=env, capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0 and "sanitized attention api ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
