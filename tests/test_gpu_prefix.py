"""Shared-prefix decoding against 64-bit arithmetic, row by row."""
import math

import pytest
import torch

import paper_2609_35629_amd as sp
from tests import attention_ref as ref

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def _rand(shape, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (size * torch.randn(shape, generator=g, dtype=F)).to(dtype)


def check(q, K, V, sK=None, sV=None, lengths=None, prefix_lengths=None, positions=None, T=None, window=0, softcap=0.0,
          slopes=None, scale=0.0, rows=None, got=None):
    B, Hq, d = q.shape
    P, Hkv, N = K.shape[:3]
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    if got is None:
        got = sp.prefix_decode(q.cuda(), K.cuda(), V.cuda(), dev(sK), dev(sV), T=T, lengths=dev(lengths),
                               prefix_lengths=dev(prefix_lengths), positions=dev(positions), window=window,
                               softcap=softcap, slopes=dev(slopes), scale=scale)
    got = got.cpu().double()
    cap = 0 if sK is None else sK.shape[2] if T is None else T
    for b, h in rows or [(b, h) for b in range(B) for h in range(Hq)]:
        p, kv = b // (B // P), h // (Hq // Hkv)
        n = N if prefix_lengths is None else min(max(int(prefix_lengths[p]), 0), N)
        t = cap if lengths is None else min(max(int(lengths[b]), 0), cap)
        k, v = K[p, kv, :n], V[p, kv, :n]
        if t:
            k, v = torch.cat([k, sK[b, kv, :t]]), torch.cat([v, sV[b, kv, :t]])
        at = torch.arange(n + t)
        dist = (at - (n + t - 1 if positions is None else int(positions[b]))).abs()
        r = ref.attend(q[b, h], k, v, dist, dist < window if window else torch.ones(n + t, dtype=torch.bool),
                       scale or d ** -0.5, softcap, 0.0 if slopes is None else float(slopes[h]))
        err = (got[b, h] - r.out).abs()
        assert (err <= r.bound).all(), ((b, h), err.max().item(), (err / r.bound.clamp_min(1e-300)).max().item())
    return got


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("P,S,Hq,Hkv,N,T", [(1, 1, 1, 1, 1, 0), (1, 1, 7, 1, 300, 5), (1, 9, 4, 4, 65, 1), (2, 3, 6, 2, 129, 33),
                                            (1, 40, 4, 2, 200, 0), (1, 5, 28, 4, 2000, 7), (3, 2, 40, 1, 70, 40),
                                            (1, 3, 2, 1, 0, 50)])
def test_sizes(dtype, d, P, S, Hq, Hkv, N, T):
    q = _rand((P * S, Hq, d), F, 1, 1.5)
    K, V = _rand((P, Hkv, N, d), dtype, 2), _rand((P, Hkv, N, d), dtype, 3)
    sK, sV = (_rand((P * S, Hkv, T, d), dtype, s) for s in (4, 5)) if T else (None, None)
    check(q, K, V, sK, sV)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("case", ["ragged", "window", "window-prefix", "slopes", "cap", "positions", "all", "T"])
def test_lengths_and_scores(dtype, case):
    P, S, Hq, Hkv, N, T, d = 2, 4, 6, 2, 150, 45, 64
    q = _rand((P * S, Hq, d), F, 1, 1.5)
    K, V = _rand((P, Hkv, N, d), dtype, 2), _rand((P, Hkv, N, d), dtype, 3)
    sK, sV = _rand((P * S, Hkv, T, d), dtype, 4), _rand((P * S, Hkv, T, d), dtype, 5)
    lens = torch.tensor([0, 1, T, 44, -3, T + 9, 32, 33], dtype=torch.int32)
    plens = torch.tensor([0, 100], dtype=torch.int32)
    slopes = 2.0 ** -torch.arange(1, Hq + 1, dtype=F)
    pos = torch.tensor([5, 2 ** 31 - 1, -2 ** 31, 0, 99, 100, 131, 3], dtype=torch.int32)
    kw = {"ragged": dict(lengths=lens, prefix_lengths=plens), "window": dict(window=20),
          "window-prefix": dict(window=80, lengths=lens, prefix_lengths=plens), "slopes": dict(slopes=slopes, lengths=lens),
          "cap": dict(softcap=3.0), "positions": dict(positions=pos, slopes=slopes * 0, window=30),
          "all": dict(window=60, lengths=lens, prefix_lengths=plens, slopes=slopes, softcap=10.0, scale=0.2,
                      positions=torch.arange(P * S, dtype=torch.int32) * 17), "T": dict(T=13)}[case]
    got = check(q, K, V, sK, sV, **kw)
    if case == "ragged":
        assert (got[0] == 0).all()  # neither prompt nor suffix


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_behind_the_lengths_hold_anything(dtype, bad):
    P, S, Hq, Hkv, N, T, d = 2, 3, 8, 2, 190, 70, 128
    q = _rand((P * S, Hq, d), F, 1)
    K, V = _rand((P, Hkv, N, d), dtype, 2), _rand((P, Hkv, N, d), dtype, 3)
    sK, sV = _rand((P * S, Hkv, T, d), dtype, 4), _rand((P * S, Hkv, T, d), dtype, 5)
    lens = torch.tensor([0, 1, 31, 32, 69, 70], dtype=torch.int32)
    plens = torch.tensor([33, 161], dtype=torch.int32)
    want = check(q, K, V, sK, sV, lengths=lens, prefix_lengths=plens)
    for p in range(P):
        K[p, :, plens[p]:], V[p, :, plens[p]:] = bad, bad
    for b in range(P * S):
        sK[b, :, lens[b]:], sV[b, :, lens[b]:] = bad, bad
    got = sp.prefix_decode(q.cuda(), K.cuda(), V.cuda(), sK.cuda(), sV.cuda(), lengths=lens.cuda(),
                           prefix_lengths=plens.cuda())
    assert torch.equal(got.cpu().double(), want)


def test_a_value_that_is_not_finite_reaches_its_sequences_only():
    P, S, Hq, Hkv, N, T, d = 1, 3, 4, 2, 500, 20, 64
    q = _rand((P * S, Hq, d), F, 1)
    K, V = _rand((P, Hkv, N, d), BF, 2), _rand((P, Hkv, N, d), BF, 3)
    sK, sV = _rand((P * S, Hkv, T, d), BF, 4), _rand((P * S, Hkv, T, d), BF, 5)
    lens = torch.tensor([20, 10, 0], dtype=torch.int32)
    args = lambda: (q.cuda(), K.cuda(), V.cuda(), sK.cuda(), sV.cuda())  # noqa: E731
    kw = dict(lengths=lens.cuda(), window=200)
    want = sp.prefix_decode(*args(), **kw).cpu()
    V[0, 0, 315, 7] = math.inf   # near enough for the sequences of 10 and 0 suffix rows (positions 509, 499)
    sV[1, 1, 3, 2] = math.nan
    got = sp.prefix_decode(*args(), **kw).cpu()
    hit = torch.zeros_like(want, dtype=torch.bool)
    hit[1, 0:2, 7] = hit[2, 0:2, 7] = True
    assert (got[hit] == math.inf).all()
    nan = torch.zeros_like(hit)
    nan[1, 2:4, 2] = True
    assert got[nan].isnan().all()
    rest = ~(hit | nan)
    assert torch.allclose(got[rest], want[rest], rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("S,N", [(1, 131072), (64, 20011), (13, 32768)])
def test_long(S, N):
    Hq, Hkv, T, d = 28, 4, 130, 128
    q = _rand((S, Hq, d), F, 1, 1.5)
    K, V = _rand((1, Hkv, N, d), BF, 2), _rand((1, Hkv, N, d), BF, 3)
    sK, sV = _rand((S, Hkv, T, d), BF, 4), _rand((S, Hkv, T, d), BF, 5)
    check(q, K, V, sK, sV, rows=[(0, 0), (S - 1, Hq - 1), (S // 2, 9), (S // 3, 20)])


def test_equals_the_dense_step_of_every_sequence():
    P, S, Hq, Hkv, N, T, d = 2, 4, 28, 4, 1500, 40, 128
    q = _rand((P * S, Hq, d), F, 1)
    K, V = _rand((P, Hkv, N, d), BF, 2), _rand((P, Hkv, N, d), BF, 3)
    sK, sV = _rand((P * S, Hkv, T, d), BF, 4), _rand((P * S, Hkv, T, d), BF, 5)
    got = sp.prefix_decode(q.cuda(), K.cuda(), V.cuda(), sK.cuda(), sV.cuda(), T=17)
    dense = sp.dense_decode(q.cuda(), K.repeat_interleave(S, 0).cuda(), V.repeat_interleave(S, 0).cuda(), sK.cuda(),
                            sV.cuda(), T=17)
    # the dense step carries its weights to 16 bits
    assert ((got - dense).norm() / dense.norm()).item() <= 2.0 ** -15
    # views: a cache kept token by token
    Kt, Vt = (x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (K, V))
    assert torch.equal(sp.prefix_decode(q.cuda(), Kt, Vt, sK.cuda(), sV.cuda(), T=17), got)


def test_graph_replays_and_streams():
    P, S, Hq, Hkv, N, T, d = 1, 6, 28, 4, 4096, 64, 128
    q = _rand((P * S, Hq, d), F, 1).cuda()
    K, V = _rand((P, Hkv, N, d), BF, 2).cuda(), _rand((P, Hkv, N, d), BF, 3).cuda()
    sK, sV = _rand((P * S, Hkv, T, d), BF, 4).cuda(), _rand((P * S, Hkv, T, d), BF, 5).cuda()
    k, v = _rand((P * S, Hkv, d), BF, 6).cuda(), _rand((P * S, Hkv, d), BF, 7).cuda()
    q_raw = _rand((P * S, Hq, d), BF, 8).cuda()
    freqs = sp.rope_frequencies(d)
    lens = torch.arange(P * S, dtype=torch.int32, device="cuda")
    one = torch.ones_like(lens)

    def step():
        sp.rope_append(q_raw, k, v, sK, sV, freqs, lens, first=N, q_out=q)
        lens.add_(one)
        return sp.prefix_decode(q, K, V, sK, sV, lengths=lens)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    state = [x.clone() for x in (sK, sV, lens)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for _ in range(4):
        before = [x.clone() for x in (sK, sV, lens)]
        g.replay()
        torch.cuda.synchronize()
        got, after = out.clone(), [x.clone() for x in (sK, sV, lens)]
        for x, y in zip((sK, sV, lens), before):
            x.copy_(y)
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert all(torch.equal(x, y) for x, y in zip((sK, sV, lens), after))
    assert not torch.equal(lens, state[2])
