"""resq_block_norm_fwd / _bwd on the GPU against the float64 oracle.

Tolerances are bounds, computed per element from the arithmetic (U = 2^-24 half an ulp of float32,
UB = 2^-8 half an ulp of bf16):

* a row factor takes five float32 roundings after an (effectively exact) float64 sum, three of them
  under the square root: below 4 U relative;
* an output element is a product of a few such values, so its float32 error is a small multiple of
  U times the sum of its terms' magnitudes, and a bf16 output is rounded once more (UB);
* a float32 sum of d terms is off by at most (longest chain of additions) U times the sum of the
  magnitudes; no lane adds more than 16 terms, then six shuffles and up to 15 waves follow: below 48;
* a column sum adds at most m terms in float32 before float64 takes over.
"""
import itertools

import numpy as np
import pytest

from oracle import operators as O
from _gpu_util import log

pytestmark = pytest.mark.gpu

U, UB, TINY = 2.0 ** -24, 2.0 ** -8, 1e-37
EPS = 1e-6


def _t(a, dtype, pad=0):
    """Device tensor of the type, rows `pad` elements further apart; the gap holds 7."""
    import torch
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    a = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    if a.dim() == 1 or pad == 0:
        return a.to(dt).cuda()
    buf = torch.full((a.shape[0], a.shape[1] + pad), 7.0, dtype=dt, device="cuda")
    buf[:, :a.shape[1]] = a.to(dt).cuda()
    return buf[:, :a.shape[1]]


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _within(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    bad = ~(np.abs(got - want) <= tol + TINY)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0].tolist()}: "
                           f"{got[bad][0]!r} for {want[bad][0]!r}, allowed {np.broadcast_to(tol, got.shape)[bad][0]:.3e}")


def _half(dtype):
    return UB if dtype == "bf16" else U


class Case:
    def __init__(self, m, d, hd, yd, post, gate, pre, pad=0, alpha=0.75, seed=0, gate_dtype="f32"):
        r = np.random.default_rng(seed + 1000 * m + d)
        self.m, self.d, self.hd, self.yd, self.alpha, self.pad = m, d, hd, yd, alpha, pad
        self.h = _t(r.normal(size=(m, d)) * (1 + 30 * (r.random(d) < 0.02)), hd, pad)
        self.y = _t(r.normal(size=(m, d)) * 0.5, yd, pad)
        self.gpost = _t(1 + 0.2 * r.normal(size=d), "bf16") if post else None
        self.gpre = _t(1 + 0.2 * r.normal(size=d), "bf16") if pre else None
        self.gate = None if gate is None else _t(r.normal(size=d if gate == "channel" else (m, 1)), gate_dtype)
        self.kw = dict(gamma_post=self.gpost, gate=self.gate, alpha=alpha, gamma_pre=self.gpre)
        self.r = r


def _check_forward(c, out, x, rstd):
    want, rp = O.block_update(_np(c.h), _np(c.y), _np(c.gpost), _np(c.gate), c.alpha, EPS)
    branch = np.abs(want - _np(c.h))
    _within(_np(out), want, _half(c.hd) * np.abs(want) + 12 * U * (np.abs(want) + np.abs(_np(c.h)) + branch), "h_out")
    if c.gpost is not None:
        _within(_np(rstd[0]), rp, 4 * U * rp, "rstd post")
    else:
        assert (rstd[0] == 0).all()
    if c.gpre is None:
        assert x is None and (rstd[1] == 0).all()
        return
    wx, rh = O.rms_norm(_np(out), _np(c.gpre), EPS)
    _within(_np(rstd[1]), rh, 4 * U * rh, "rstd pre")
    _within(_np(x), wx, (UB + 8 * U) * np.abs(wx), "x")


SIZES = [(1, 1), (1, 2048), (3, 7), (5, 64), (2, 511), (4, 513), (33, 1999), (70, 128), (257, 2048), (2, 4097),
         (3, 8200), (2, 16384), (1, 16381)]


@pytest.mark.parametrize("m,d", SIZES)
@pytest.mark.parametrize("hd,yd", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
def test_forward_matches_the_oracle(m, d, hd, yd):
    import paper_2607_26515_amd as P
    for i, (post, gate, pre) in enumerate(itertools.product([True, False], [None, "channel", "token"], [True, False])):
        c = Case(m, d, hd, yd, post, gate, pre, pad=(0, 1, 8)[i % 3], seed=i, gate_dtype=("f32", "bf16")[i % 2])
        log(f"block_norm m={m} d={d} {hd} {yd} post={post} gate={gate} pre={pre} pad={c.pad}")
        out, x, rstd = P.block_norm(c.h, c.y, eps=EPS, **c.kw)
        _check_forward(c, out, x, rstd)


def test_forward_alone_in_place_and_into_views():
    """The norm of h alone; h_out = h; outputs that are views: the gaps between rows keep their
    values, and so does everything with save=False."""
    import torch
    import paper_2607_26515_amd as P
    for hd in ("bf16", "f32"):
        c = Case(9, 205, hd, "f32", True, "channel", True, pad=3)
        out, x, rstd = P.block_norm(c.h, gamma_pre=c.gpre, eps=EPS)
        assert out is c.h
        wx, rh = O.rms_norm(_np(c.h), _np(c.gpre), EPS)
        _within(_np(x), wx, (UB + 8 * U) * np.abs(wx), "x")
        assert (rstd[0] == 0).all()
        ref, xr, rr = P.block_norm(c.h, c.y, eps=EPS, **c.kw)
        buf = torch.full((9, 211), 5.0, dtype=c.h.dtype, device="cuda")
        xbuf = torch.full((9, 208), 3.0, dtype=torch.bfloat16, device="cuda")
        o2, x2, r2 = P.block_norm(c.h, c.y, eps=EPS, save=False, h_out=buf[:, :205], x=xbuf[:, :205], **c.kw)
        assert r2 is None and torch.equal(o2, ref) and torch.equal(x2, xr)
        assert (buf[:, 205:] == 5).all() and (xbuf[:, 205:] == 3).all()
        h = c.h.clone()
        o3, x3, r3 = P.block_norm(h, c.y, eps=EPS, h_out=h, **c.kw)
        assert o3 is h and torch.equal(h, ref) and torch.equal(x3, xr) and torch.equal(r3, rr)


def test_x_is_the_input_the_fused_producer_forms():
    """The X of block_norm, given to the plain linear, gives the fused linear's Y bit for bit."""
    import torch
    import paper_2607_26515_amd as P
    for fmt, m, d, n in (("hif4", 37, 2048, 96), ("mxfp4", 5, 3584, 64)):
        c = Case(m, d, "bf16", "f32", False, None, True, seed=3)
        w = _t(c.r.normal(size=(n, d)) * 0.02, "bf16")
        wp = P.prepare_weights(*P.quantize(w, fmt), fmt)
        out, x, _ = P.block_norm(c.h, c.y, eps=EPS, **c.kw)
        a = P.linear_fwd_prepared(x, wp, n, fmt, "2:4")
        b = P.linear_fwd_rmsnorm(out, c.gpre, EPS, wp, n, fmt, "2:4")
        assert torch.equal(a, b)


def test_zero_rows_large_rows_and_bad_rows():
    """A row of zeros, rows near float32's limits, and a NaN that stays in its own row."""
    import torch
    import paper_2607_26515_amd as P
    d = 300
    h, y = np.zeros((5, d)), np.zeros((5, d))
    r = np.random.default_rng(5)
    h[1], y[1] = r.normal(size=d) * 1e30, r.normal(size=d) * 1e25
    h[2], y[2] = r.normal(size=d) * 1e-30, r.normal(size=d) * 1e-25
    h[3], y[3] = r.normal(size=d), r.normal(size=d)
    h[4], y[4] = r.normal(size=d), r.normal(size=d)
    y[3, 17] = np.nan
    c = Case(5, d, "f32", "f32", True, None, True, alpha=1.0)
    c.h, c.y = _t(h, "f32"), _t(y, "f32")
    out, x, rstd = P.block_norm(c.h, c.y, eps=EPS, **c.kw)
    assert torch.isnan(out[3]).all() and torch.isnan(x[3]).all()
    keep = [0, 1, 2, 4]
    c.h, c.y = c.h[keep], c.y[keep]
    _check_forward(c, out[keep], x[keep], rstd[:, keep])
    assert (out[0] == 0).all() and (x[0] == 0).all()


def _backward_bounds(c, dx, dh, rstd, h_out):
    """The oracle's gradients and, per output, the bound of the module's docstring."""
    a = np.abs
    h, y, e0 = _np(h_out), _np(c.y), np.zeros((c.m, c.d)) if dh is None else _np(dh)
    rp, rh = _np(rstd[0]), _np(rstd[1])
    want = O.block_norm_bwd(h, y, rp, rh, None if dx is None else _np(dx), e0, _np(c.gpost), _np(c.gate), c.alpha, _np(c.gpre))
    tol = {}
    e_abs = a(e0)
    e_err = np.zeros_like(e0)
    if c.gpre is not None:
        u, n = a(_np(dx) * _np(c.gpre)), a(h) * rh[:, None]
        cabs = (u * n).mean(1, keepdims=True)
        e_abs = a(e0) + rh[:, None] * (u + n * cabs)
        e_err = 8 * U * e_abs + 56 * U * rh[:, None] * n * cabs
        tol["dgamma_pre"] = (c.m + 16) * U * (a(_np(dx)) * n).sum(0)
    n = a(y) if c.gpost is None else a(y) * rp[:, None]
    gp = 1.0 if c.gpost is None else a(_np(c.gpost))
    gt = 1.0 if c.gate is None else a(_np(c.gate))
    al = a(c.alpha)
    w = al * gp * n
    tol["dh"] = e_err + _half(c.hd) * a(want["dh"])
    if c.gate is not None:
        if np.ndim(gt) == 2:
            tol["dgate"] = (w * e_err).sum(1, keepdims=True) + 72 * U * (w * e_abs).sum(1, keepdims=True)
        else:
            tol["dgate"] = (w * e_err).sum(0) + (c.m + 24) * U * (w * e_abs).sum(0)
    dt, dt_err = al * gt * e_abs, al * gt * (e_err + 4 * U * e_abs)
    dy_err = dt_err * np.ones_like(y)
    if c.gpost is not None:
        tol["dgamma_post"] = (dt_err * n).sum(0) + (c.m + 16) * U * (dt * n).sum(0)
        k_abs = (gt * w * e_abs).mean(1, keepdims=True)
        k_err = (gt * w * e_err).mean(1, keepdims=True) + 80 * U * k_abs
        dy_err = rp[:, None] * (dt_err * gp + n * k_err + 8 * U * (dt * gp + n * k_abs))
    tol["dy"] = dy_err
    return want, tol


@pytest.mark.parametrize("m,d", SIZES + [(1100, 96), (600, 1000)])
@pytest.mark.parametrize("hd,yd,xd,out", [("bf16", "f32", "f32", "bf16"), ("bf16", "bf16", "bf16", "f32"),
                                          ("f32", "f32", "f32", "f32"), ("f32", "bf16", "f32", "bf16"),
                                          ("bf16", "f32", "bf16", "bf16"), ("f32", "f32", "bf16", "f32")])
def test_backward_matches_the_oracle(m, d, hd, yd, xd, out):
    import paper_2607_26515_amd as P
    for i, (post, gate, pre) in enumerate(itertools.product([True, False], [None, "channel", "token"], [True, False])):
        c = Case(m, d, hd, yd, post, gate, pre, pad=(0, 1, 8)[i % 3], seed=10 + i, gate_dtype=("f32", "bf16")[i % 2])
        log(f"block_norm_bwd m={m} d={d} {hd} {yd} {xd} {out} post={post} gate={gate} pre={pre}")
        h_out, _, rstd = P.block_norm(c.h, c.y, eps=EPS, **c.kw)
        dx = _t(c.r.normal(size=(m, d)) * 0.01, xd, c.pad) if pre else None
        dh = _t(c.r.normal(size=(m, d)) * 0.01, hd, c.pad) if i % 4 != 1 or not pre else None
        g = P.block_norm_bwd(h_out, rstd, dx=dx, dh=dh, y=c.y, out=out, **c.kw)
        want, tol = _backward_bounds(c, dx, dh, rstd, h_out)
        for name, v in want.items():
            if v is None:
                assert g[name] is None, name
                continue
            assert g[name].shape == v.shape, name
            extra = _half(out) * np.abs(v) if name == "dy" else U * np.abs(v)
            _within(_np(g[name]), v, tol[name] + extra, name)


def test_backward_of_parts_and_empty_batches():
    """Single gradients equal those of the full call; y is not needed without a norm or gate; a
    batch of no rows has zero column sums."""
    import torch
    import paper_2607_26515_amd as P
    c = Case(40, 515, "bf16", "f32", True, "channel", True)
    h_out, _, rstd = P.block_norm(c.h, c.y, eps=EPS, **c.kw)
    dx, dh = _t(c.r.normal(size=(40, 515)), "f32"), _t(c.r.normal(size=(40, 515)), "bf16")
    full = P.block_norm_bwd(h_out, rstd, dx=dx, dh=dh, y=c.y, **c.kw)
    some = P.block_norm_bwd(h_out, rstd, dx=dx, dh=dh, y=c.y, want_dh=False, want_dy=False, **c.kw)
    assert some["dh"] is None and some["dy"] is None
    for k in ("dgamma_post", "dgamma_pre", "dgate"):
        assert torch.equal(full[k], some[k])
    plain = P.block_norm_bwd(h_out, rstd, dx=dx, dh=dh, alpha=0.5, gamma_pre=c.gpre)
    assert torch.equal(plain["dh"], full["dh"])
    e = full["dh"].double()
    _within(_np(plain["dy"]), _np(0.5 * e), 2.1 * UB * np.abs(_np(0.5 * e)), "dy")  # of the unrounded e
    with pytest.raises(P.ResqError):
        P.block_norm_bwd(h_out, rstd, dx=dx, dh=dh, **c.kw)  # the norm after the block needs y
    none = torch.empty((0, 515), dtype=torch.bfloat16, device="cuda")
    g = P.block_norm_bwd(none, torch.empty((2, 0), device="cuda"), dx=none, y=none, gamma_post=c.gpost, gamma_pre=c.gpre,
                         gate=c.gate)
    for k in ("dgamma_post", "dgamma_pre", "dgate"):
        assert (g[k] == 0).all() and g[k].shape == (515,)


def test_backward_in_place_through_the_c_entry():
    """dH may be dH_out: the same gradients, bit for bit."""
    import torch
    import paper_2607_26515_amd as P
    from paper_2607_26515_amd import resq as B
    m, d = 21, 770
    c = Case(m, d, "f32", "bf16", True, None, True)
    h_out, _, rstd = P.block_norm(c.h, c.y, eps=EPS, **c.kw)
    dx, dh = _t(c.r.normal(size=(m, d)), "f32"), _t(c.r.normal(size=(m, d)), "f32")
    ref = P.block_norm_bwd(h_out, rstd, dx=dx, dh=dh, y=c.y, **c.kw)
    ws, nb = P.workspace(B.OP_BLOCK_NORM_BWD, 0, 0, m, d)
    dy = torch.empty((m, d), dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    rc = P.resq_block_norm_bwd(h_out.data_ptr(), 1, m, d, d, c.y.data_ptr(), 0, d, c.gpost.data_ptr(), 0, 0, 0, c.alpha,
                               c.gpre.data_ptr(), rstd.data_ptr(), dx.data_ptr(), 1, d, dh.data_ptr(), d, dh.data_ptr(), d,
                               dy.data_ptr(), 0, d, 0, 0, 0, ws.data_ptr(), nb, s)
    assert rc == B.OK, P.resq_last_error()
    assert torch.equal(dh, ref["dh"]) and torch.equal(dy, ref["dy"])


def test_same_bits_every_time_and_on_other_streams():
    import torch
    import paper_2607_26515_amd as P
    c = Case(700, 1024, "bf16", "f32", True, "channel", True)
    dx, dh = _t(c.r.normal(size=(700, 1024)), "f32"), _t(c.r.normal(size=(700, 1024)), "bf16")

    def both(stream=None):
        o, x, r = P.block_norm(c.h, c.y, eps=EPS, stream=stream, **c.kw)
        g = P.block_norm_bwd(o, r, dx=dx, dh=dh, y=c.y, stream=stream, **c.kw)
        return [o, x, r, *g.values()]

    ref = both()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for got in (both(), both(s)):
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, got))
