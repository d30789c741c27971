"""Rotary positions, prompt attention and shared-prefix decoding as measurable cases.

Each case is one call of the package's public API.  ``run`` makes that call
where ``own`` is true; otherwise it computes the same operator from elementary
torch operations in 32 bits (angles in 64), rounded once at the end.  ``exact``
is the definition in 64 bits.

Shapes are those of the package's workloads (28 query and 4 KV heads of 128,
prompts of 8K, 32K and 131072 tokens) and of its tests, or generic odd sizes.
"""
from __future__ import annotations

import math

import torch

own = False

# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------


def _rope(name, B, T, Hq=28, Hkv=4, d=128, rot=128, inter=False, dtype="bf16", first=0, factor=1.0):
    return dict(name=name, kind="rope", B=B, T=T, Hq=Hq, Hkv=Hkv, d=d, rot=rot, inter=inter, dtype=dtype, first=first,
                factor=factor)


def _append(name, B, T, cap, Hq=28, Hkv=4, d=128, rot=128, inter=False, dtype="bf16", first=32768, factor=1.0):
    return dict(_rope(name, B, T, Hq, Hkv, d, rot, inter, dtype, first, factor), kind="append", cap=cap)


def _prompt(name, B, T, N, Hq=28, Hkv=4, d=128, dtype="bf16", causal=True, window=0, cap=0.0, slopes=False, docs=0,
            prefix=0):
    return dict(name=name, kind="prompt", B=B, T=T, N=N, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, causal=causal, window=window,
                cap=cap, slopes=slopes, docs=docs, prefix=prefix)


def _shared(name, P, S, N, T, Hq=28, Hkv=4, d=128, dtype="bf16", window=0, cap=0.0, slopes=False, ragged=False):
    return dict(name=name, kind="shared", P=P, S=S, N=N, T=T, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, window=window, cap=cap,
                slopes=slopes, ragged=ragged)


def listed():
    return [
        # one interactive sequence after a 32K prompt: the new token's q, k, v
        _append("append-1", B=1, T=1, cap=512),
        # a batch of answers far into a stretched context, half of the head rotated, interleaved pairs
        _append("append-64-partial", B=64, T=1, cap=1024, rot=64, inter=True, first=120000, factor=4.0),
        # the queries of a whole 32K prompt
        _rope("rope-32k", B=1, T=32768),
        # a short odd prompt of fp32 caches with capped scores
        _prompt("prompt-fp32-1009", B=2, T=1009, N=1009, Hq=16, Hkv=4, d=64, dtype="fp32", cap=30.0),
        # a few drafted tokens checked against a 32K prompt
        _prompt("prompt-5-of-32k", B=1, T=5, N=32768),
        # several short prompts packed into one row, padding behind the last
        _prompt("prompt-packed-8k", B=1, T=8192, N=8192, docs=7),
        # instructions read in both directions, answers forward, a bias by distance
        _prompt("prompt-prefix-4001", B=4, T=4001, N=4001, Hq=8, Hkv=8, d=64, slopes=True, prefix=1000),
        # a whole long prompt: the largest
        _prompt("prompt-16k", B=1, T=16384, N=16384, Hq=16, Hkv=4),
        # one sequence, capped scores
        _shared("shared-1-8k", P=1, S=1, N=8192, T=64, cap=50.0),
        # eight answers to one 32K prompt
        _shared("shared-8-32k", P=1, S=8, N=32768, T=128),
        # two prompts of unequal length, three answers each, fp32 caches, a window over the end
        _shared("shared-fp32-8191", P=2, S=3, N=8191, T=33, Hq=16, Hkv=4, d=64, dtype="fp32", window=5000, slopes=True,
                ragged=True),
        # a large sample of answers of many lengths to one long document
        _shared("shared-64-131k", P=1, S=64, N=131072, T=512, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "prompt", "prompt", "prompt", "shared", "shared"])
    dtype = "bf16" if rng.random() < 0.7 else "fp32"
    d = 128 if rng.random() < 0.6 else 64
    Hq, Hkv = rng.choice([(28, 4), (28, 4), (16, 4), (32, 8), (12, 2), (8, 8), (6, 1)])
    if kind in ("rope", "append"):
        rot = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
        inter, factor, first = rng.random() < 0.5, rng.choice([1.0, 1.0, 4.0, 8.0]), _log_int(rng, 1, 131072)
        if kind == "rope":
            T = _log_int(rng, 1, 32768)
            B = rng.randint(1, max(1, min(8, 32768 // T)))
            return dict(_rope("", B, T, Hq, Hkv, d, rot, inter, dtype, first, factor), name=None)
        B, T, cap = _log_int(rng, 1, 256), _log_int(rng, 1, 64), rng.randint(64, 1024)
        return dict(_append("", B, T, cap, Hq, Hkv, d, rot, inter, dtype, first, factor), name=None)
    if kind == "prompt":
        N = _log_int(rng, 1, 16384 if dtype == "bf16" else 8192)
        T = N if rng.random() < 0.6 else _log_int(rng, 1, N)
        Hq, Hkv = (8, 2) if N * T * Hq > 16 * 16384 * 8192 else (Hq, Hkv)
        B = rng.randint(1, max(1, min(8, 16 * 16384 * 8192 // (N * T * Hq))))
        mask = rng.choice(["causal", "causal", "full", "window", "docs", "prefix"])
        return dict(_prompt("", B, T, N, Hq, Hkv, d, dtype, causal=mask != "full",
                            window=_log_int(rng, 1, N) if mask == "window" else 0, cap=rng.choice([0.0, 0.0, 30.0]),
                            slopes=rng.random() < 0.3, docs=rng.randint(2, 9) if mask == "docs" else 0,
                            prefix=_log_int(rng, 1, N) if mask == "prefix" else 0), name=None)
    N = _log_int(rng, 1, 131072 if dtype == "bf16" else 32768)
    P = rng.randint(1, max(1, min(4, 131072 // N)))
    S = _log_int(rng, 1, max(1, min(128, (64 if dtype == "bf16" else 32) * 131072 // (N * P * max(1, Hq // 28)))))
    if dtype == "fp32":
        S = min(S, 32)
    return dict(_shared("", P, S, N, rng.randint(0, 512), Hq, Hkv, d, dtype,
                        window=_log_int(rng, 1, N) if rng.random() < 0.2 else 0, cap=rng.choice([0.0, 0.0, 50.0]),
                        slopes=rng.random() < 0.3, ragged=rng.random() < 0.6), name=None)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------


def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _freqs(case):
    """Radians per position [rot / 2] in 64 bits; a stretched context slows the
    slow frequencies (those that turn less than once in 32768 positions) by
    its factor, leaves the fast ones and blends between."""
    R = case["rot"] // 2
    f = 10000.0 ** (-torch.arange(R, dtype=torch.float64) / R)
    keep = ((32768 * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return (f * (keep + (1 - keep) / case["factor"])).cuda()


def _documents(case):
    """Document of every token of a packed row: lengths that grow along the
    row, the last sixteenth padding (-1)."""
    N, n = case["N"], case["docs"]
    full = N - N // 16
    at = torch.arange(N, dtype=torch.float64)
    doc = (n * ((at + 0.5) / max(full, 1)) ** (1 / 1.5)).floor().clamp(max=n - 1).to(torch.int32)
    doc[full:] = -1
    return doc


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _torch_dtype(case)

    def rows(*shape, size=1.0, to=dt):
        return (size * torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)).to(to)

    def whole(lo, hi, n):
        return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)

    st = dict(case=case)
    d, Hq, Hkv = case["d"], case["Hq"], case["Hkv"]
    if case["kind"] in ("rope", "append"):
        B, T = case["B"], case["T"]
        st["freqs"] = _freqs(case)
        st["magnitude"] = 1.0 + 0.1 * math.log(case["factor"])
        # as a projection leaves them: token by token, the heads of a token together
        st["q"] = rows(B, T, Hq, d).transpose(1, 2)
        if case["kind"] == "append":
            st["k"], st["v"] = rows(B, T, Hkv, d).transpose(1, 2), rows(B, T, Hkv, d).transpose(1, 2)
            st["cache_K"], st["cache_V"] = rows(B, Hkv, case["cap"], d), rows(B, Hkv, case["cap"], d)
            st["at"] = whole(0, case["cap"] - T, B)
        return st
    if case["kind"] == "prompt":
        B, T, N = case["B"], case["T"], case["N"]
        # queries lean towards a key of their own, as trained heads' do
        st["K"], st["V"] = rows(B, Hkv, N, d), rows(B, Hkv, N, d)
        st["q"] = rows(B, Hq, T, d, size=1.5)
        st["documents"] = _documents(case).cuda().repeat(B, 1) if case["docs"] else None
        st["prefix"] = whole(0, min(2 * case["prefix"], N), B) if case["prefix"] else None
    else:
        P, S, N, T = case["P"], case["S"], case["N"], case["T"]
        st["K"], st["V"] = rows(P, Hkv, N, d), rows(P, Hkv, N, d)
        st["sK"] = rows(P * S, Hkv, T, d) if T else None
        st["sV"] = rows(P * S, Hkv, T, d) if T else None
        st["q"] = rows(P * S, Hq, d, size=1.5, to=torch.float32)
        st["lengths"] = whole(0, T, P * S) if case["ragged"] and T else None
        st["prefix_lengths"] = whole(max(1, N // 2), N, P) if case["ragged"] else None
    st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device="cuda") / Hq) if case["slopes"] else None
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------


def _rotate(x, positions, st):
    """x [B, H, T, d] in 32 bits rotated to positions [B, T]."""
    R, m = st["freqs"].numel(), st["magnitude"]
    a = positions[:, None, :, None].double() * st["freqs"]
    c, s = (m * torch.cos(a)).float(), (m * torch.sin(a)).float()
    x = x.float()
    y = x.clone()
    if st["case"]["inter"]:
        x1, x2 = x[..., 0:2 * R:2], x[..., 1:2 * R:2]
        y[..., 0:2 * R:2], y[..., 1:2 * R:2] = x1 * c - x2 * s, x2 * c + x1 * s
    else:
        x1, x2 = x[..., :R], x[..., R:2 * R]
        y[..., :R], y[..., R:2 * R] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


def _capped(s, cap):
    return s.div_(cap).tanh_().mul_(cap) if cap else s


def _weights(s):
    """exp(s - max) in place and its sums; rows of -inf give nothing."""
    m = s.amax(-1, keepdim=True).clamp_min(-1e30)
    e = s.sub_(m).exp_()
    return e, e.sum(-1, keepdim=True), m


def _plain_prompt(st):
    case = st["case"]
    B, Hq, T, d = st["q"].shape
    Hkv, N = case["Hkv"], case["N"]
    G = Hq // Hkv
    s = torch.matmul((st["q"].float() / math.sqrt(d)).reshape(B, Hkv, G * T, d), st["K"].float().transpose(2, 3))
    s = _capped(s, case["cap"]).view(B, Hkv, G, T, N)
    j = torch.arange(N, device="cuda")
    p = torch.arange(N - T, N, device="cuda")[:, None]
    if st["slopes"] is not None:
        s.sub_(st["slopes"].view(Hkv, G, 1, 1) * (p - j).abs().float())
    bar = torch.zeros((1, T, N), dtype=torch.bool, device="cuda")
    if case["causal"]:
        bar = bar | (j > p)
    if st["prefix"] is not None:
        bar = bar & (j >= st["prefix"][:, None, None])
    if case["window"]:
        bar = bar | ((p - j).abs() >= case["window"])
    if st["documents"] is not None:
        doc = st["documents"]
        bar = bar | (doc[:, N - T:, None] != doc[:, None, :]) | (doc[:, None, :] < 0)
    s.masked_fill_(bar[:, None, None], -math.inf)
    e, total, _ = _weights(s)
    o = torch.matmul(e.view(B, Hkv, G * T, N), st["V"].float()).view(B, Hkv, G, T, d)
    return (o / total.clamp_min(1e-30)).reshape(B, Hq, T, d).to(st["q"].dtype)


def _plain_shared(st):
    case = st["case"]
    P, S, N, T, Hkv, d = (case[k] for k in ("P", "S", "N", "T", "Hkv", "d"))
    G, cap, window = case["Hq"] // Hkv, case["cap"], case["window"]
    q = (st["q"] / math.sqrt(d)).view(P, S, Hkv, G, d)
    n = st["prefix_lengths"] if st["prefix_lengths"] is not None else torch.full((P,), N, device="cuda")
    t = st["lengths"] if st["lengths"] is not None else torch.full((P * S,), T, device="cuda")
    n, t = n.view(P, 1, 1, 1, 1), t.view(P, S, 1, 1, 1)
    pos, j = n + t - 1, torch.arange(N, device="cuda")
    slopes = st["slopes"].view(Hkv, G, 1) if st["slopes"] is not None else None
    qp = q.transpose(1, 2).reshape(P, Hkv, S * G, d)
    s = _capped(torch.matmul(qp, st["K"].float().transpose(2, 3)), cap).view(P, Hkv, S, G, N).transpose(1, 2)
    if slopes is not None:
        s.sub_(slopes * (pos - j).abs().float())
    bar = j >= n
    if window:
        bar = bar | ((pos - j).abs() >= window)
    e, l1, m1 = _weights(s.masked_fill_(bar, -math.inf))
    o1 = torch.matmul(e.transpose(1, 2).reshape(P, Hkv, S * G, N), st["V"].float())
    o1 = o1.view(P, Hkv, S, G, d).transpose(1, 2)
    if not T:
        return (o1 / l1.clamp_min(1e-30)).reshape(P * S, case["Hq"], d)
    i = torch.arange(T, device="cuda")
    s = _capped(torch.matmul(q.reshape(P * S, Hkv, G, d), st["sK"].float().transpose(2, 3)), cap).view(P, S, Hkv, G, T)
    dist = (t - 1 - i).abs()
    if slopes is not None:
        s.sub_(slopes * dist.float())
    bar = i >= t
    if window:
        bar = bar | (dist >= window)
    e, l2, m2 = _weights(s.masked_fill_(bar, -math.inf))
    o2 = torch.matmul(e.view(P * S, Hkv, G, T), st["sV"].float()).view(P, S, Hkv, G, d)
    m = torch.maximum(m1, m2)
    w1, w2 = (m1 - m).exp(), (m2 - m).exp()
    return ((w1 * o1 + w2 * o2) / (w1 * l1 + w2 * l2).clamp_min(1e-30)).reshape(P * S, case["Hq"], d)


def run(st):
    case = st["case"]
    if case["kind"] == "rope":
        if own:
            import paper_2609_35629_amd as sp
            return sp.rope(st["q"], st["freqs"], first=case["first"], interleaved=case["inter"], magnitude=st["magnitude"])
        at = torch.arange(case["first"], case["first"] + case["T"], device="cuda").expand(case["B"], -1)
        return _rotate(st["q"], at, st).to(st["q"].dtype)
    if case["kind"] == "append":
        if own:
            import paper_2609_35629_amd as sp
            return sp.rope_append(st["q"], st["k"], st["v"], st["cache_K"], st["cache_V"], st["freqs"], st["at"],
                                  first=case["first"], interleaved=case["inter"], magnitude=st["magnitude"]), \
                st["cache_K"], st["cache_V"]
        row = st["at"][:, None].long() + torch.arange(case["T"], device="cuda")
        b = torch.arange(case["B"], device="cuda")[:, None]
        at = row + case["first"]
        st["cache_K"].transpose(1, 2)[b, row] = _rotate(st["k"], at, st).to(st["k"].dtype).transpose(1, 2)
        st["cache_V"].transpose(1, 2)[b, row] = st["v"].transpose(1, 2)
        return _rotate(st["q"], at, st), st["cache_K"], st["cache_V"]
    if case["kind"] == "prompt":
        if own:
            import paper_2609_35629_amd as sp
            return sp.prompt_attention(st["q"], st["K"], st["V"], causal=case["causal"], window=case["window"],
                                       softcap=case["cap"], slopes=st["slopes"], documents=st["documents"],
                                       prefix=st["prefix"])
        return _plain_prompt(st)
    if own:
        import paper_2609_35629_amd as sp
        return sp.prefix_decode(st["q"], st["K"], st["V"], st["sK"], st["sV"], lengths=st["lengths"],
                                prefix_lengths=st["prefix_lengths"], window=case["window"], softcap=case["cap"],
                                slopes=st["slopes"])
    return _plain_shared(st)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------


def work(case):
    size, d, Hq, Hkv = 2 if case["dtype"] == "bf16" else 4, case["d"], case["Hq"], case["Hkv"]
    if case["kind"] in ("rope", "append"):
        tokens = case["B"] * case["T"]
        flops = 3 * tokens * Hq * case["rot"]
        if case["kind"] == "rope":
            return dict(bytes=2 * tokens * Hq * d * size, flops=flops)
        return dict(bytes=tokens * d * (Hq * (size + 4) + 4 * Hkv * size), flops=flops + 3 * tokens * Hkv * case["rot"])
    if case["kind"] == "prompt":
        B, T, N = case["B"], case["T"], case["N"]
        lo, hi = _reach(case)
        if case["docs"]:
            doc = _documents(case)
            pairs = sum(_causal_pairs(int((doc[N - T:] == i).sum()), int((doc == i).sum()), case["causal"])
                        for i in range(case["docs"]))
        else:
            pairs = int((hi - lo).clamp_min(0).sum())
        keys = int(hi.max() - lo.min()) if T else 0
        return dict(bytes=size * d * B * (2 * Hq * T + 2 * Hkv * keys), flops=4 * d * B * Hq * pairs)
    P, S, N, T = case["P"], case["S"], case["N"], case["T"]
    n, t = (0.75 * N, 0.5 * T) if case["ragged"] else (N, T)
    if case["window"]:
        t = min(t, case["window"])
        n = min(n, case["window"] - t)
    return dict(bytes=int(2 * size * d * Hkv * P * (n + S * t) + 8 * P * S * Hq * d), flops=int(4 * d * P * S * Hq * (n + t)))


def _causal_pairs(q, k, causal):
    return q * k - (q * (q - 1) // 2 if causal else 0)


def _reach(case):
    """[lo, hi) of the keys each query of a prompt may attend (documents
    aside), with the expected prefix."""
    T, N, w = case["T"], case["N"], case["window"]
    p = torch.arange(N - T, N)
    hi = p + 1 if case["causal"] else torch.full_like(p, N)
    if case["prefix"]:
        hi = hi.clamp_min(min(case["prefix"], N))
    if w:
        hi = torch.minimum(hi, p + w)
    return (p - w + 1).clamp_min(0) if w else torch.zeros_like(p), hi


def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    d, Hq, Hkv = case["d"], case["Hq"], case["Hkv"]
    G = Hq // Hkv
    if case["kind"] in ("rope", "append"):
        R, T = case["rot"] // 2, case["T"]
        at = st["at"].to(f64)[:, None] if case["kind"] == "append" else torch.zeros((case["B"], 1), dtype=f64, device="cuda")
        turn = torch.exp(1j * (at + case["first"] + torch.arange(T, device="cuda"))[..., None] * st["freqs"])  # [B, T, R]

        def rotated(x):
            z = x[..., :2 * R].to(f64)
            z = z.unflatten(-1, (R, 2)) if case["inter"] else z.unflatten(-1, (2, R)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None] * st["magnitude"])
            z = z if case["inter"] else z.transpose(-1, -2)
            return torch.cat([z.reshape(*x.shape[:-1], 2 * R), x[..., 2 * R:].to(f64)], -1)

        if case["kind"] == "rope":
            return rotated(st["q"])
        K, V, k = st["cache_K"].to(f64), st["cache_V"].to(f64), rotated(st["k"])
        for b, a in enumerate(st["at"].tolist()):
            K[b, :, a:a + T], V[b, :, a:a + T] = k[b], st["v"][b].to(f64)
        return rotated(st["q"]), K, V

    def attend(q, K, V, h, pos, at, ok):
        """q [G or T, d] of head h at positions pos over rows at, where ok."""
        s = q.to(f64) @ K.to(f64).T * d ** -0.5
        if case["cap"]:
            s = case["cap"] * torch.tanh(s / case["cap"])
        far = (pos[:, None] - at).abs()
        if st["slopes"] is not None:
            s = s - st["slopes"][h].to(f64) * far
        if case["window"]:
            ok = ok & (far < case["window"])
        s = torch.where(ok, s, -math.inf)
        return torch.nan_to_num(torch.softmax(s, -1), nan=0.0) @ V.to(f64)

    if case["kind"] == "prompt":
        B, T, N = case["B"], case["T"], case["N"]
        at = torch.arange(N, device="cuda")
        pos = at[N - T:]
        out = torch.empty((B, Hq, T, d), dtype=f64, device="cuda")
        for b in range(B):
            ok = (at <= pos[:, None]) if case["causal"] else torch.ones((T, N), dtype=torch.bool, device="cuda")
            if st["prefix"] is not None:
                ok = ok | (at < st["prefix"][b])
            if st["documents"] is not None:
                doc = st["documents"][b]
                ok = ok & (doc[pos][:, None] == doc) & (doc >= 0)
            for h in range(Hq):
                out[b, h] = attend(st["q"][b, h], st["K"][b, h // G], st["V"][b, h // G], h, pos, at, ok)
        return out
    out = torch.empty((case["P"] * case["S"], Hq, d), dtype=f64, device="cuda")
    if out.shape[0] * Hq * (case["N"] + case["T"]) > 1 << 31:
        return None
    lens = st["lengths"].tolist() if st["lengths"] is not None else [case["T"]] * out.shape[0]
    plens = st["prefix_lengths"].tolist() if st["prefix_lengths"] is not None else [case["N"]] * case["P"]
    for b, t in enumerate(lens):
        p = b // case["S"]
        n = plens[p]
        at = torch.arange(n + t, device="cuda")
        for h in range(Hq):
            K, V = st["K"][p, h // G, :n], st["V"][p, h // G, :n]
            if t:
                K, V = torch.cat([K, st["sK"][b, h // G, :t]]), torch.cat([V, st["sV"][b, h // G, :t]])
            out[b, h] = attend(st["q"][b, h][None], K, V, h, at[-1:], at, torch.ones_like(at, dtype=torch.bool))[0]
    return out
