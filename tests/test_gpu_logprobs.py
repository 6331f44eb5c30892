"""resq_token_logprobs / _bwd on the GPU against the float64 oracle.

Bounds (U = 2^-24): with z = (x - max) / T, a lane's exponential is off by at most 4 U (1 + |z|)
relative (two roundings of its argument, one of the result), and a sum of V terms by the longest
chain of additions, below V / 256 + 64, times U.  So log S is off by at most
    eS = U (V / 256 + 64) + 4 U (1 + A),   A = sum p |z|,
logp by eS + 4 U (|z| + |logp|), and H = log S - sum p z by
    eS (1 + A) + U (V / 256 + 64) A + 4 U sum p |z| (1 + |z|) + 4 U |H|.
The gradient's p is off by 8 U (2 + |z| + log S) relative (the argument's roundings), and the rest is
a few roundings of each term.  Indices and maxima are exact."""
import numpy as np
import pytest

from oracle import operators as O
from _gpu_util import log

pytestmark = pytest.mark.gpu

U, UB, TINY = 2.0 ** -24, 2.0 ** -8, 2.0 ** -120
INF = np.inf
LOWEST = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38}


def _t(a, dtype, pad=0, shift=0):
    import torch
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    a = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dt)
    m, v = a.shape
    buf = torch.full((m * (v + pad) + shift,), 50.0, dtype=dt, device="cuda")
    view = buf[shift:].view(m, v + pad)[:, :v]
    view.copy_(a.cuda())
    return view


def _np(t):
    return t.double().cpu().numpy()


def _close(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    # outputs are float32: a value past (2 - 2^-24) 2^127, the midpoint between the largest float32 and
    # 2^128, rounds to infinity (a masked logit of the lowest value at a temperature below 1)
    want = np.where(np.abs(want) >= (2 - 2.0 ** -24) * 2.0 ** 127, np.copysign(INF, want), want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= tol + TINY) & np.isfinite(want))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, first {np.argwhere(bad)[0].tolist()}: {got[bad][0]} for {want[bad][0]}"


def _bounds(x, t):
    v = x.shape[1]
    mx = x.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        z = np.where(np.isneginf(x), 0.0, (x - np.where(np.isfinite(mx), mx, 0.0)) / t)
        e = np.where(np.isneginf(x), 0.0, np.exp(z))
        s = e.sum(1, keepdims=True)
        p = np.where(s > 0, e / np.where(s > 0, s, 1.0), 0.0)
    A = (p * np.abs(z)).sum(1)
    chain = U * (v / 256 + 64)
    eS = chain + 4 * U * (1 + A)
    eH = eS * (1 + A) + chain * A + 4 * U * (p * np.abs(z) * (1 + np.abs(z))).sum(1)
    return z, p, eS, eH


def _check(tx, targets, t, k, ws=None):
    import torch
    import paper_2607_26515_amd as P
    x = _np(tx)
    tt = None if targets is None else torch.from_numpy(np.asarray(targets, np.int64)).cuda()
    got = P.token_logprobs(tx, tt, temperature=t, top_k=k, ws=ws)
    want = O.token_logprobs(x, targets, t, k)
    assert set(got) == set(want)
    z, p, eS, eH = _bounds(x, t)
    st, ws_ = _np(got["stats"]), want["stats"]
    assert np.array_equal(st[:, 0], ws_[:, 0], equal_nan=True)
    _close(st[:, 1], ws_[:, 1], eS + 2 * U * np.abs(np.nan_to_num(ws_[:, 1], neginf=0, posinf=0)), "log sum")
    _close(st[:, 2], ws_[:, 2], eH + 4 * U * np.abs(ws_[:, 2]), "entropy")
    if targets is not None:
        at = np.clip(targets, 0, x.shape[1] - 1)[:, None]
        lp = np.nan_to_num(want["logp"], neginf=0)
        _close(_np(got["logp"]), want["logp"], eS + 4 * U * (np.abs(np.take_along_axis(z, at, 1)[:, 0]) + np.abs(lp)), "logp")
    if k:
        assert np.array_equal(got["top_index"].cpu().numpy(), want["top_index"])
        val = np.nan_to_num(want["top_logp"], neginf=0)
        _close(_np(got["top_logp"]), want["top_logp"], eS[:, None] + 8 * U * (np.abs(val) + np.abs(ws_[:, 1:2])), "top")
    return got


SIZES = [(1, 1), (1, 2), (3, 7), (2, 31), (5, 513), (1, 4096), (1, 4097), (7, 5001), (1, 50021), (3, 131072),
         (130, 2050), (1100, 777), (40, 32003)]


@pytest.mark.parametrize("m,v", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_matches_the_oracle(m, v, dtype):
    r = np.random.default_rng(m + v)
    for i, (t, k, banned) in enumerate([(1.0, 0, 0.0), (0.7, 1, 0.1), (1.3, 5, 0.0), (1.0, 32, 0.6), (0.25, 20, 0.0)]):
        log(f"logprobs m={m} v={v} {dtype} T={t} k={k}")
        x = r.normal(size=(m, v)) * 3 + r.normal() * 20
        x[np.arange(m), r.integers(0, v, m)] += 10
        x[:, r.random(v) < banned] = -INF
        targets = r.integers(0, v, m)
        targets[r.random(m) < 0.2] = -1
        _check(_t(x, dtype, pad=(0, 1, 8)[i % 3], shift=i % 2), targets, t, k)


@pytest.mark.parametrize("m,v", [(1, 70000), (6, 9000), (600, 1500)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_runs_and_orders(m, v, dtype):
    """Equal rows, rows of two values, rising and falling rows, few distinct values, signed zeros,
    alternatives that all lie side by side: indices are exact, ties to the lowest index."""
    r = np.random.default_rng(7)
    rows = [np.zeros(v), np.where(np.arange(v) % 3 == 1, 1.0, 0.5), np.linspace(-8, 8, v), np.linspace(8, -8, v),
            r.integers(-2, 3, v).astype(float), np.where(np.arange(v) % 2, 0.0, -0.0),
            np.where((np.arange(v) > v // 2) & (np.arange(v) < v // 2 + 40), 9.0, r.normal(size=v))]
    for i, row in enumerate(rows):
        log(f"logprobs ties row {i} m={m} v={v} {dtype}")
        x = np.broadcast_to(row, (m, v))
        for k in (1, 7, 32):
            _check(_t(x, dtype), r.integers(0, v, m), 1.0, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [40, 3000, 40000])
def test_masks(v, dtype):
    """Rows of -inf alone, of one token, of the type's lowest value (alone and beside others), of
    fewer tokens than alternatives; huge logits; targets outside the vocabulary."""
    low = LOWEST[dtype]
    r = np.random.default_rng(v)
    x = np.full((9, v), -INF)
    x[1, v // 2] = -3.0
    x[2] = low
    x[3] = low
    x[3, 5] = 1.0
    x[4] = r.normal(size=v)
    x[4, 10:] = low
    x[5, [3, 30, 31]] = [2.0, 2.0, 1.0]
    x[6] = r.normal(size=v) * 1e4 + 3e5
    x[7] = r.normal(size=v)
    x[8] = r.normal(size=v)
    targets = np.array([4, v // 2, 7, 5, 2, 30, 1, v, -5])
    for t in (1.0, 0.5, 2.0):
        got = _check(_t(x, dtype), targets, t, 6)
        assert np.isnan(_np(got["logp"])[7])
    _check(_t(x, dtype), None, 1.0, 6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [33, 20000])
def test_bad_logits_stay_in_their_row(v, dtype):
    import torch
    import paper_2607_26515_amd as P
    r = np.random.default_rng(1)
    x = r.normal(size=(5, v))
    x[1, 20] = np.nan
    x[2, 3] = INF
    x[3] = -INF
    x[3, 9] = np.nan
    t = torch.zeros(5, dtype=torch.int64, device="cuda")
    tx = _t(x, dtype)
    o = P.token_logprobs(tx, t, top_k=4)
    for row in (1, 2, 3):
        assert torch.isnan(o["logp"][row]) and torch.isnan(o["stats"][row, 1:]).all()
    g = P.token_logprobs_bwd(tx, t, o["stats"], torch.ones(5, device="cuda"), out="f32")
    assert torch.isfinite(g[[0, 4]]).all()
    keep = [0, 4]
    want = O.token_logprobs(_np(tx)[keep], np.zeros(2, int), 1.0, 4)
    assert np.array_equal(o["top_index"][keep].cpu().numpy(), want["top_index"])
    assert np.allclose(_np(o["logp"])[keep], want["logp"], atol=1e-4)


@pytest.mark.parametrize("m,v", SIZES)
@pytest.mark.parametrize("dtype,out", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_backward_matches_the_oracle(m, v, dtype, out):
    import torch
    import paper_2607_26515_amd as P
    r = np.random.default_rng(m * 3 + v)
    for i, (t, ent, lp, banned) in enumerate([(1.0, True, True, 0.0), (0.7, False, True, 0.3), (1.4, True, False, 0.1)]):
        log(f"logprobs_bwd m={m} v={v} {dtype} {out} T={t}")
        x = r.normal(size=(m, v)) * 3
        x[:, r.random(v) < banned] = -INF
        if m > 4:
            x[4] = -INF
        targets = r.integers(0, v, m)
        targets[r.random(m) < 0.2] = -1
        tx = _t(x, dtype, pad=(0, 1, 8)[i % 3], shift=i % 2)
        tt = torch.from_numpy(targets).cuda()
        stats = P.token_logprobs(tx, tt, temperature=t)["stats"]
        a = torch.from_numpy(r.normal(size=m).astype(np.float32)).cuda() if lp else None
        b = torch.from_numpy(r.normal(size=m).astype(np.float32)).cuda() if ent else None
        buf = torch.full((m, v + 3), 5.0, dtype=torch.bfloat16 if out == "bf16" else torch.float32, device="cuda")
        g = P.token_logprobs_bwd(tx, tt, stats, a, b, temperature=t, out=out, dlogits=buf[:, :v])
        assert (buf[:, v:] == 5).all()
        xn, sn = _np(tx), _np(stats)
        an, bn = np.zeros(m) if a is None else np.abs(_np(a)), np.zeros(m) if b is None else np.abs(_np(b))
        want = O.token_logprobs_bwd(xn, targets, sn, None if a is None else _np(a), None if b is None else _np(b), t)
        with np.errstate(invalid="ignore"):
            z = np.where(np.isneginf(xn), 0.0, (xn - sn[:, :1]) / t)
            q = np.where(np.isneginf(xn) | np.isneginf(sn[:, :1]), 0.0, np.exp(z - sn[:, 1:2]))
        z, ls = np.nan_to_num(z, neginf=0, posinf=0), np.nan_to_num(np.abs(sn[:, 1:2]), posinf=0, neginf=0)
        mag = an[:, None] + bn[:, None] * (np.abs(z) + ls + np.abs(sn[:, 2:3]))
        tol = (8 * U * (2 + np.abs(z) + ls) * q * mag + 8 * U * q * bn[:, None] * (np.abs(z) + ls)
               + 4 * U * an[:, None] * (np.arange(v)[None, :] == targets[:, None])) / t
        _close(_np(g), want, tol + (UB if out == "bf16" else U) * np.abs(want), "dlogits")


def test_backward_in_place_and_bad_targets():
    import torch
    import paper_2607_26515_amd as P
    for dt, out in ((torch.float32, "f32"), (torch.bfloat16, "bf16")):
        g = torch.Generator(device="cuda").manual_seed(3)
        x = torch.randn((6, 9001), generator=g, device="cuda").to(dt)
        t = torch.tensor([1, 9000, 9001, -1, 0, 1 << 40], device="cuda")
        stats = P.token_logprobs(x, t)["stats"]
        a = torch.randn(6, generator=g, device="cuda")
        ref = P.token_logprobs_bwd(x, t, stats, a, a, out=out)
        y = x.clone()
        P.token_logprobs_bwd(y, t, stats, a, a, out=out, dlogits=y)
        assert torch.equal(y[[0, 1, 3, 4]], ref[[0, 1, 3, 4]])
        assert torch.isnan(ref[[2, 5]]).all() and torch.isnan(y[[2, 5]]).all() and (ref[3] == 0).all()


@pytest.mark.parametrize("m,v,k", [(1, 131072, 20), (9, 40000, 5), (1500, 600, 3)])
def test_same_bits_every_time_and_split_or_whole(m, v, k):
    """Repeats give the same bits, and so do other streams; a row's indices are the same alone (split
    over many workgroups) and in a large batch (one workgroup)."""
    import torch
    import paper_2607_26515_amd as P
    g = torch.Generator(device="cuda").manual_seed(m)
    x = torch.randn((m, v), generator=g, device="cuda").bfloat16()
    t = torch.randint(0, v, (m,), generator=g, device="cuda")
    ref = P.token_logprobs(x, t, top_k=k)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for other in (P.token_logprobs(x, t, top_k=k), P.token_logprobs(x, t, top_k=k, stream=s)):
        torch.cuda.synchronize()
        for key in ref:
            assert torch.equal(ref[key], other[key]), key
    alone = P.token_logprobs(x[:1], t[:1], top_k=k)
    assert torch.equal(alone["top_index"], ref["top_index"][:1])
