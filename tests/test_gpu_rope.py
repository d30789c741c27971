"""Rotary positions and the append of a step's rows against 64-bit arithmetic."""
import math

import pytest
import torch

import paper_2609_35629_amd as sp
from tests import attention_ref as ref

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def _rand(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g, dtype=F).to(dtype)


def _close(got, want, bound, name):
    err = (got.cpu().double() - want).abs()
    worst = (err - bound).max().item()
    assert worst <= 0, (name, worst, err.max().item())


@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (128, 128, True), (128, 64, False), (64, 32, True),
                                         (64, 16, False), (128, 20, False), (64, 2, True), (128, 126, True)])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (F, F), (BF, F), (F, BF)])
def test_rope(d, rot, inter, dtype, out_dtype):
    B, H, T = 2, 5, 37
    x = _rand((B, H, T, d), dtype, rot)
    freqs = sp.rope_frequencies(rot, device="cuda")
    pos = torch.randint(-5000, 200000, (B, T), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    for positions, at in ((pos.cuda(), pos), (None, (torch.arange(T) + 131000).expand(B, T))):
        got = sp.rope(x.cuda(), freqs, positions=positions, first=131000, interleaved=inter, magnitude=1.25,
                      out_dtype=out_dtype)
        assert got.dtype == out_dtype and got.is_contiguous()
        want = ref.rope(x, freqs.cpu(), at, inter, 1.25)
        _close(got, want, ref.rope_bound(x, freqs.cpu(), out_dtype, inter, 1.25), (d, rot, inter))


@pytest.mark.parametrize("B,H,T", [(1, 1, 1), (1, 28, 1), (3, 7, 1000), (64, 4, 1), (1, 2, 9001)])
def test_rope_sizes(B, H, T):
    x = _rand((B, H, T, 128), BF, T)
    freqs = sp.rope_frequencies(128)
    got = sp.rope(x.cuda(), freqs, first=7)
    want = ref.rope(x, freqs.cpu(), (torch.arange(T) + 7).expand(B, T))
    _close(got, want, ref.rope_bound(x, freqs.cpu(), BF), (B, H, T))


def test_far_positions_keep_their_angles():
    # the largest int32 position: 2^31 radians, still right to fp32
    x = _rand((1, 2, 3, 64), F, 0)
    freqs = sp.rope_frequencies(64)
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31, 16777217]], dtype=torch.int32)
    got = sp.rope(x.cuda(), freqs, positions=pos.cuda())
    # p f is rounded to 2^-53 of itself on both sides: 2^31 2^-52 radians
    _close(got, ref.rope(x, freqs.cpu(), pos), ref.rope_bound(x, freqs.cpu(), F) + 2.0 ** -19 * x.double().abs().max(),
           "far")


def test_views_in_place_and_inverse():
    B, H, T, d = 2, 6, 50, 64
    x = _rand((B, T, H, d), F, 1)
    freqs = sp.rope_frequencies(d)
    want = ref.rope(x.transpose(1, 2), freqs.cpu(), torch.arange(T).expand(B, T))
    bound = ref.rope_bound(x.transpose(1, 2), freqs.cpu(), F)
    xd = x.cuda().transpose(1, 2)  # as a projection leaves it
    _close(sp.rope(xd, freqs), want, bound, "view")
    wide = torch.zeros((B, H, T, 3 * d), device="cuda")
    out = sp.rope(xd, freqs, out=wide[..., d:2 * d])
    _close(out, want, bound, "strided out")
    assert wide[..., :d].abs().max() == 0 and wide[..., 2 * d:].abs().max() == 0
    y = xd.clone()
    sp.rope(y, freqs, out=y)
    _close(y, want, bound, "in place")
    back = sp.rope(y, freqs, positions=-torch.arange(T, dtype=torch.int32, device="cuda").expand(B, T).contiguous())
    _close(back, x.transpose(1, 2).double(), 4 * bound, "inverse")
    # a row repeated for every head and token
    one = _rand((1, 1, 1, d), F, 2).cuda()
    got = sp.rope(one.expand(B, H, T, d), freqs)
    _close(got, ref.rope(one.cpu().expand(B, H, T, d), freqs.cpu(), torch.arange(T).expand(B, T)),
           ref.rope_bound(one.cpu().expand(B, H, T, d), freqs.cpu(), F), "expanded")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d,rot,inter", [(128, 128, True), (128, 90, False), (64, 30, True), (64, 64, False)])
def test_in_place_of_any_pairs(dtype, d, rot, inter):
    x = _rand((2, 3, 70, d), dtype, rot).cuda()
    freqs = sp.rope_frequencies(rot)
    want = sp.rope(x, freqs, interleaved=inter, first=9)
    assert sp.rope(x, freqs, interleaved=inter, first=9, out=x) is x
    assert torch.equal(x, want)


def test_gradient_is_the_rotation_back():
    """<g, d rope(x)> = <rope(g, -p), dx>: the gradient by the call with negated
    positions, against the formula's and against differences."""
    B, H, T, d, m = 1, 2, 5, 64, 1.5
    freqs = sp.rope_frequencies(d)
    pos = torch.tensor([[0, 3, 100, 131071, 12345]], dtype=torch.int32)
    x, g, dx = _rand((B, H, T, d), F, 1), _rand((B, H, T, d), F, 2), _rand((B, H, T, d), F, 3)
    grad = sp.rope(g.cuda(), freqs, positions=-pos.cuda(), magnitude=m).cpu().double()
    x64 = x.double().requires_grad_(True)
    ref_out = _ref_differentiable(x64, freqs.cpu(), pos, m)
    ref_out.backward(g.double())
    assert ((grad - x64.grad).abs() <= ref.rope_bound(g, freqs.cpu(), F, False, m)).all()
    # linear in x: a difference of any length is exact but for roundings
    y1 = sp.rope((x + dx).cuda(), freqs, positions=pos.cuda(), magnitude=m).cpu().double()
    y0 = sp.rope(x.cuda(), freqs, positions=pos.cuda(), magnitude=m).cpu().double()
    bound = (ref.rope_bound(x.abs() + dx.abs(), freqs.cpu(), F, False, m) * 3 * g.double().abs()).sum()
    assert abs(((y1 - y0) * g.double()).sum() - (grad * ((x + dx).double() - x.double())).sum()) <= bound


def _ref_differentiable(x, freqs, positions, m):
    R = freqs.numel()
    a = positions.double()[:, None, :, None] * freqs
    u, w = x[..., :R], x[..., R:2 * R]
    return torch.cat([m * (u * a.cos() - w * a.sin()), m * (w * a.cos() + u * a.sin())], -1)


@pytest.mark.parametrize("kv,cache,qt", [(BF, BF, BF), (F, F, F), (F, BF, BF), (BF, F, F)])
@pytest.mark.parametrize("T,inter,rot", [(1, False, 128), (5, True, 64), (3, False, 12)])
def test_append(kv, cache, qt, T, inter, rot):
    B, Hq, Hkv, cap, d = 3, 6, 2, 40, 128
    q, k, v = _rand((B, Hq, T, d), qt, 1), _rand((B, Hkv, T, d), kv, 2), _rand((B, Hkv, T, d), kv, 3)
    freqs = sp.rope_frequencies(rot)
    at = torch.tensor([0, 17, cap - T], dtype=torch.int32)
    old_K, old_V = _rand((B, Hkv, cap, d), cache, 4), _rand((B, Hkv, cap, d), cache, 5)
    cK, cV = old_K.cuda(), old_V.cuda()
    got = sp.rope_append(q.cuda(), k.cuda(), v.cuda(), cK, cV, freqs, at.cuda(), first=1000, interleaved=inter)
    pos = at[:, None] + torch.arange(T) + 1000
    assert got.dtype == F
    _close(got, ref.rope(q, freqs.cpu(), pos, inter), ref.rope_bound(q, freqs.cpu(), F, inter), "q")
    wk, wb = ref.rope(k, freqs.cpu(), pos, inter), ref.rope_bound(k, freqs.cpu(), cache, inter)
    new = torch.zeros(B, cap, dtype=torch.bool)
    for b in range(B):
        a = int(at[b])
        new[b, a:a + T] = True
        _close(cK[b, :, a:a + T], wk[b], wb[b] + (0 if cache == kv else wk[b].abs() * ref.HALF[cache]), "k")
        assert torch.equal(cV[b, :, a:a + T].cpu(), v[b].to(cache))
    keep = ~new[:, None, :, None].expand(B, Hkv, cap, d)
    assert torch.equal(cK.cpu()[keep], old_K[keep]) and torch.equal(cV.cpu()[keep], old_V[keep])


def test_append_outside_the_cache_and_without_queries():
    B, Hkv, cap, d, T = 4, 2, 8, 64, 3
    k, v = _rand((B, Hkv, T, d), F, 1), _rand((B, Hkv, T, d), F, 2)
    freqs = sp.rope_frequencies(d)
    guard = torch.full((B + 2, Hkv, cap, d), 7.0, device="cuda")
    guard_V = guard.clone()
    at = torch.tensor([-1, 6, 8, 2 ** 31 - 1], dtype=torch.int32)  # first row out, last row out, all out, all out
    assert sp.rope_append(None, k.cuda(), v.cuda(), guard[1:-1], guard_V[1:-1], freqs, at.cuda()) is None
    got = guard_V.cpu()
    assert (got[0] == 7).all() and (got[-1] == 7).all()
    assert torch.equal(got[1, :, 0:2], v[0, :, 1:]) and (got[1, :, 2:] == 7).all()
    assert torch.equal(got[2, :, 6:8], v[1, :, :2]) and (got[2, :, :6] == 7).all()
    assert (got[3] == 7).all() and (got[4] == 7).all()
    # one number for every sequence; one token per sequence as [B, H, d]
    c = torch.zeros((B, Hkv, cap, d), device="cuda")
    cv = torch.zeros_like(c)
    q = _rand((B, 4, d), F, 3)
    out = sp.rope_append(q.cuda(), k[:, :, 0].cuda(), v[:, :, 0].cuda(), c, cv, freqs, 5, first=10)
    assert out.shape == q.shape
    assert torch.equal(cv[:, :, 5].cpu(), v[:, :, 0])
    _close(out.unsqueeze(2), ref.rope(q.unsqueeze(2), freqs.cpu(), torch.full((B, 1), 15)),
           ref.rope_bound(q.unsqueeze(2), freqs.cpu(), F), "q")


def test_frequencies():
    rot, base, L = 64, 10000.0, 4096
    f = sp.rope_frequencies(rot, base, device="cpu")
    i = torch.arange(rot // 2, dtype=torch.float64)
    assert torch.allclose(f, base ** (-2 * i / rot), rtol=1e-14)
    assert torch.equal(sp.rope_frequencies(rot, base, "linear", 8.0, device="cpu"), f / 8.0)
    g = sp.rope_frequencies(rot, base, "base", 8.0, device="cpu")
    assert math.isclose(g[0], f[0]) and math.isclose(g[-1], f[-1] / 8.0, rel_tol=1e-12)
    h = sp.rope_frequencies(rot, base, "bands", 8.0, original_length=L, low=1.0, high=32.0, device="cpu")
    turns = L * f / (2 * math.pi)
    assert torch.equal(h[turns >= 32], f[turns >= 32])
    assert torch.allclose(h[turns <= 1], f[turns <= 1] / 8.0, rtol=1e-14)
    between = (turns > 1) & (turns < 32)
    keep = (turns - 1) / 31
    assert between.any() and torch.allclose(h[between], (f * (keep + (1 - keep) / 8))[between], rtol=1e-14)
