"""Sizes and layouts at the limits of the operators around the linears: more rows than one grid
dimension holds, rows longer than fit one workgroup's registers or LDS beside others, in-place calls
whose last accesses are moved back, alternatives that all lie with one lane."""
import numpy as np
import pytest

from oracle import operators as O
from _gpu_util import dev_bf16, host, log
from test_gpu_block_norm import EPS, Case, _backward_bounds, _check_forward, _half, _np, _t, _within
from test_gpu_logprobs import _check, _t as _rows
from test_gpu_matvec import FMTS, U, _case

pytestmark = pytest.mark.gpu


def test_more_rows_than_a_grid_dimension_holds():
    import torch
    import paper_2607_26515_amd as P
    m, v = (1 << 25) + 3, 3  # 2^25 workgroups of 128 threads
    log(f"logprobs m={m} v={v}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    base, t = torch.randn((1024, v), generator=gen, device="cuda").bfloat16(), torch.arange(1024, device="cuda") % v
    want = P.token_logprobs(base, t, top_k=1)
    times = (m + 1023) // 1024
    x, tt = base.repeat(times, 1)[:m], t.repeat(times)[:m]
    got = P.token_logprobs(x, tt, top_k=1)
    for k in want:
        w = want[k].repeat(times, *[1] * (want[k].dim() - 1))[:m]
        assert torch.equal(got[k], w), k
    one = torch.ones(m, device="cuda")
    g = P.token_logprobs_bwd(x, tt, got["stats"], one)
    w = P.token_logprobs_bwd(base, t, want["stats"], one[:1024])
    assert torch.equal(g, w.repeat(times, 1)[:m])
    del x, tt, got, g, one
    m, d = (1 << 20) + 77, 520  # a workgroup per row
    log(f"block_norm m={m} d={d}")
    h, y = torch.randn((1024, d), generator=gen, device="cuda").bfloat16(), torch.randn((1024, d), generator=gen, device="cuda").bfloat16()
    gamma = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    times = (m + 1023) // 1024
    want = P.block_norm(h, y, gamma_post=gamma, gamma_pre=gamma)
    got = P.block_norm(h.repeat(times, 1)[:m], y.repeat(times, 1)[:m], gamma_post=gamma, gamma_pre=gamma)
    for a, b in zip(got[:2], want[:2]):
        assert torch.equal(a, b.repeat(times, 1)[:m])
    assert torch.equal(got[2], want[2].repeat(1, times)[:, :m])


def _whole(m, d):
    """X lies whole in LDS: the order of a sum depends on n and d alone."""
    return 40960 + m * ((d + 511) // 512 * 1024 + 16) <= 163840


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("d", [3648, 5504, 11008, 18944, 28416, 60032])
def test_matvec_of_long_rows_takes_windows_of_k(fmt, d):
    """X does not fit a workgroup's LDS for all tokens, at the end for one: right, the same every time,
    and the same token by token as long as the tokens fit."""
    import torch
    import paper_2607_26515_amd as P
    for n in (41, 1100 if d < 20000 else 70):  # fewer and more quads of rows than CUs
        log(f"matvec {fmt} d={d} n={n}")
        xb, wb, x, w = _case(fmt, 16, d, n, d + n)
        qc, qs = P.quantize(dev_bf16(wb), fmt, axis=1)
        tx = dev_bf16(xb)
        want, tol = x @ w.T, d * U * (np.abs(x) @ np.abs(w).T)
        same = None
        for m in (16, 13, 9, 8, 7, 5, 4, 3, 2, 1):
            log(f"  m={m}")
            y = P.matvec_w4a16(tx[:m], qc, qs, fmt)
            assert (np.abs(host(y) - want[:m]) <= tol[:m]).all(), m
            assert torch.equal(y, P.matvec_w4a16(tx[:m], qc, qs, fmt)), m
            if _whole(m, d):
                same = y if same is None else same
                assert torch.equal(y, same[:m]), m
            assert torch.equal(P.matvec_w4a16(tx[:m], qc, qs, fmt, out="bf16"), y.bfloat16()), m
        # rows of X at odd addresses and strides, NaN between and behind them
        for gap, shift in ((1, 0), (2, 1), (0, 3)):
            buf = torch.full((16 * (d + gap) + shift + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
            view = buf[shift:shift + 16 * (d + gap)].view(16, d + gap)[:, :d]
            view.copy_(tx.view(torch.bfloat16))
            assert torch.equal(P.matvec_w4a16(view, qc, qs, fmt), P.matvec_w4a16(tx, qc, qs, fmt)), (gap, shift)


@pytest.mark.parametrize("fmt", FMTS)
def test_matvec_of_more_quads_than_wait_in_lds(fmt):
    """More than 48 quads of rows to a workgroup, in windows of K, against the weights read out exactly."""
    import torch
    import paper_2607_26515_amd as P
    m, d, n = 16, 4160, 50003
    log(f"matvec {fmt} m={m} d={d} n={n}")
    gen = torch.Generator(device="cuda").manual_seed(4)
    qc, qs = P.quantize((torch.randn((n, d), generator=gen, device="cuda") * 0.02).bfloat16(), fmt)
    x = torch.randn((m, d), generator=gen, device="cuda").bfloat16()
    y = P.matvec_w4a16(x, qc, qs, fmt).double()
    w = P.linear_w4a16(torch.eye(d, device="cuda").bfloat16(), qc, qs, fmt).double()  # Q(W)^T
    want, mags = x.double() @ w, x.double().abs() @ w.abs()
    assert ((y - want).abs() <= d * U * mags).all()


@pytest.mark.parametrize("d", [9, 515, 1023, 8201, 12345, 16381])
@pytest.mark.parametrize("hd", ["bf16", "f32"])
def test_in_place_where_the_last_access_is_moved_back(d, hd):
    import torch
    import paper_2607_26515_amd as P
    from paper_2607_26515_amd import resq as B
    m = 37
    for post, gate in ((False, None), (False, "token"), (True, "channel")):
        log(f"in place d={d} {hd} post={post} gate={gate}")
        c = Case(m, d, hd, "f32", post, gate, True, seed=5)
        ref = P.block_norm(c.h, c.y, eps=EPS, **c.kw)
        _check_forward(c, *ref)
        h = c.h.clone()
        got = P.block_norm(h, c.y, eps=EPS, h_out=h, **c.kw)
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
        dx, dh = _t(c.r.normal(size=(m, d)) * 0.01, "f32"), _t(c.r.normal(size=(m, d)) * 0.01, hd)
        g = P.block_norm_bwd(ref[0], ref[2], dx=dx, dh=dh, y=c.y, **c.kw)
        want, tol = _backward_bounds(c, dx, dh, ref[2], ref[0])
        for name, v in want.items():
            if v is not None:
                _within(_np(g[name]), v, tol[name] + (_half("bf16") if name == "dy" else U) * np.abs(v), name)
        ws, nb = P.workspace(B.OP_BLOCK_NORM_BWD, 0, 0, m, d)
        code, mode = (B.IN_F32, {None: B.GATE_NONE, "channel": B.GATE_CHANNEL, "token": B.GATE_TOKEN}[gate])
        hc = B.IN_F32 if hd == "f32" else B.IN_BF16
        rc = P.resq_block_norm_bwd(ref[0].data_ptr(), hc, m, d, d, c.y.data_ptr(), 1, d, B._p(c.gpost), B._p(c.gate), code, mode,
                                   c.alpha, c.gpre.data_ptr(), ref[2].data_ptr(), dx.data_ptr(), 1, d, dh.data_ptr(), d,
                                   dh.data_ptr(), d, 0, 0, d, 0, 0, 0, ws.data_ptr(), nb, torch.cuda.current_stream().cuda_stream)
        assert rc == B.OK, P.resq_last_error()
        assert torch.equal(dh, g["dh"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v", [(1, 131072), (2, 8192), (1100, 8192), (600, 20000), (1, 8193), (1030, 8193)])
def test_alternatives_that_lie_with_one_lane(m, v, dtype):
    """The largest elements all in the groups of eight that one lane reads, for either number of waves,
    from an aligned row and from one that begins inside a group."""
    r = np.random.default_rng(v)
    for lanes, shift in ((128, 0), (512, 0), (128, 3), (512, 5)):
        log(f"logprobs one lane m={m} v={v} {dtype} lanes={lanes} shift={shift}")
        x = r.normal(size=(m, v))
        at = np.arange(v)
        x[:, (at + shift) // 8 % lanes == 17] += 30
        _check(_rows(x, dtype, pad=shift, shift=shift), r.integers(0, v, m), 1.0, 32)


@pytest.mark.parametrize("v", [1, 5, 8, 9, 8191, 8192, 8193, 12289])
def test_rows_at_every_offset(v):
    """Rows that begin at each 2-byte offset from a 16-byte boundary, shorter and longer than the way to it."""
    r = np.random.default_rng(v)
    for dtype, offsets in (("bf16", 8), ("f32", 4)):
        for shift in range(offsets):
            x = np.round(r.normal(size=(3, v)) * 3, 1)
            _check(_rows(x, dtype, pad=1, shift=shift), r.integers(0, v, 3), 0.9, min(v, 4))


def test_profiler_families():
    import torch
    import paper_2607_26515_amd as P
    c = Case(5, 256, "bf16", "f32", True, None, True)
    logits = torch.zeros((2, 40000), device="cuda")
    t = torch.zeros(2, dtype=torch.int64, device="cuda")
    qw = P.quantize(c.h, "mxfp4")
    P.resq_profile_enable(1)
    try:
        P.resq_profile_reset()
        o, _, rstd = P.block_norm(c.h, c.y, **c.kw)
        P.block_norm_bwd(o, rstd, dx=c.y, y=c.y, **c.kw)
        P.matvec_w4a16(c.h, *qw, "mxfp4")
        s = P.token_logprobs(logits, t)["stats"]
        P.token_logprobs_bwd(logits, t, s, torch.ones(2, device="cuda"))
        torch.cuda.synchronize()
        for name, calls in (("block_norm", 2), ("matvec", 1), ("logprobs", 2)):
            got = P.resq_profile_read(name)
            assert got[0] == calls and 0 < got[1] < 1000, (name, got)
    finally:
        P.resq_profile_enable(0)


def test_readme_examples_run_one_after_the_other():
    import os
    import re
    import torch
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    env = {}
    for block in re.findall(r"```python\n(.*?)```", text, re.S):
        exec(compile(block, "README.md", "exec"), env)  # noqa: S102 - the repository's own README
    torch.cuda.synchronize()
    assert env["h"].shape == env["x"].shape == (4, 2048) and env["q"].shape == (4, 2560)
    assert env["t"]["logp"].shape == (4,) and env["t"]["logp"][2] == 0 and env["t"]["top_index"].shape == (4, 5)
    assert env["dq"].shape == (4, 2560) and (env["dq"][2] == 0).all()
    assert env["g"]["dh"].shape == env["g"]["dy"].shape == (4, 2048) and env["g"]["dgamma_pre"].shape == (2048,)
    assert bool(torch.isfinite(env["g"]["dgamma_pre"]).all()) and bool(torch.isfinite(env["t"]["top_logp"][[0, 1, 3]]).all())
