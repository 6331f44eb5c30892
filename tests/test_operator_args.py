"""Refusals of the operators around the linears, on the host: every entry point rejects bad
arguments before anything is enqueued (no GPU is needed), empty calls succeed, and the Python
wrappers reject tensors of other devices, types and shapes."""
import ctypes

import pytest
import torch

import paper_2607_26515_amd as P
from paper_2607_26515_amd import resq as B

PTR = 1 << 20  # never dereferenced: every call here is refused, or empty
NAN = float("nan")


def fwd(**kw):
    a = dict(H=PTR, h_dtype=0, m=4, d=64, ldh=64, Y=PTR, y_dtype=1, ldy=64, gamma_post=PTR, gate=0, gate_dtype=0,
             gate_mode=0, alpha=1.0, gamma_pre=PTR, eps=1e-6, H_out=PTR, ldho=64, X=PTR, ldx=64, rstd=PTR)
    a.update(kw)
    return P.resq_block_norm_fwd(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(H=0), B.ERR_ARG), (dict(h_dtype=2), B.ERR_ARG), (dict(y_dtype=-1), B.ERR_ARG), (dict(m=-1), B.ERR_ARG),
    (dict(d=-1), B.ERR_ARG), (dict(ldh=63), B.ERR_ARG), (dict(ldy=63), B.ERR_ARG), (dict(ldho=63), B.ERR_ARG),
    (dict(ldx=63), B.ERR_ARG), (dict(H=PTR + 1), B.ERR_ARG), (dict(Y=PTR + 2), B.ERR_ARG), (dict(X=0), B.ERR_ARG),
    (dict(X=PTR + 1), B.ERR_ARG), (dict(H_out=0), B.ERR_ARG), (dict(gamma_post=PTR + 1), B.ERR_ARG),
    (dict(rstd=PTR + 2), B.ERR_ARG), (dict(gate_mode=3), B.ERR_ARG), (dict(gate_mode=1), B.ERR_ARG),
    (dict(gate_mode=1, gate=PTR, gate_dtype=9), B.ERR_ARG), (dict(gate_mode=2, gate=PTR + 2, gate_dtype=1), B.ERR_ARG),
    (dict(eps=0.0), B.ERR_ARG), (dict(eps=NAN), B.ERR_ARG), (dict(eps=float("inf")), B.ERR_ARG),
    (dict(alpha=NAN), B.ERR_ARG), (dict(Y=0), B.ERR_ARG), (dict(Y=0, gamma_post=0, gamma_pre=0), B.ERR_ARG),
    (dict(Y=0, gamma_post=0, gate_mode=1, gate=PTR), B.ERR_ARG),
    (dict(d=16385, ldh=16385, ldy=16385, ldho=16385, ldx=16385), B.ERR_UNSUPPORTED), (dict(m=1 << 31), B.ERR_UNSUPPORTED),
])
def test_block_norm_fwd_refuses(kw, code):
    assert fwd(**kw) == code
    assert P.resq_last_error() != ""


def bwd(**kw):
    a = dict(H=PTR, h_dtype=0, m=4, d=64, ldh=64, Y=PTR, y_dtype=1, ldy=64, gamma_post=PTR, gate=PTR, gate_dtype=0,
             gate_mode=1, alpha=1.0, gamma_pre=PTR, rstd=PTR, dX=PTR, dx_dtype=1, lddx=64, dH_out=PTR, lddho=64, dH=PTR,
             lddh=64, dY=PTR, dy_dtype=0, lddy=64, dgamma_post=PTR, dgamma_pre=PTR, dgate=PTR, workspace=PTR,
             workspace_bytes=1 << 30)
    a.update(kw)
    return P.resq_block_norm_bwd(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(H=0), B.ERR_ARG), (dict(Y=0), B.ERR_ARG), (dict(dX=0), B.ERR_ARG), (dict(rstd=0), B.ERR_ARG),
    (dict(h_dtype=2), B.ERR_ARG), (dict(y_dtype=5), B.ERR_ARG), (dict(dx_dtype=2), B.ERR_ARG), (dict(dy_dtype=2), B.ERR_ARG),
    (dict(ldh=3), B.ERR_ARG), (dict(ldy=3), B.ERR_ARG), (dict(lddx=3), B.ERR_ARG), (dict(lddho=3), B.ERR_ARG),
    (dict(lddh=3), B.ERR_ARG), (dict(lddy=3), B.ERR_ARG), (dict(m=-1), B.ERR_ARG), (dict(gate=0), B.ERR_ARG),
    (dict(gate_mode=0), B.ERR_ARG), (dict(gamma_post=0), B.ERR_ARG), (dict(gamma_pre=0), B.ERR_ARG),
    (dict(dH=0, dY=0, dgamma_post=0, dgamma_pre=0, dgate=0), B.ERR_ARG), (dict(dgate=PTR + 2), B.ERR_ARG),
    (dict(dX=PTR + 2), B.ERR_ARG), (dict(dH_out=PTR + 1), B.ERR_ARG),
    (dict(workspace=0), B.ERR_WORKSPACE), (dict(workspace=PTR + 8), B.ERR_WORKSPACE), (dict(workspace_bytes=16), B.ERR_WORKSPACE),
    (dict(d=1 << 15, ldh=1 << 15), B.ERR_UNSUPPORTED),
])
def test_block_norm_bwd_refuses(kw, code):
    assert bwd(**kw) == code
    assert P.resq_last_error() != ""


def matvec(**kw):
    a = dict(fmt=0, X=PTR, m=4, d=64, ldx=64, qw_codes=PTR, qw_scales=PTR, n=8, Y=PTR, y_dtype=1, ldy=8)
    a.update(kw)
    return P.resq_matvec_w4a16(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(fmt=2), B.ERR_ARG), (dict(m=-1), B.ERR_ARG), (dict(n=-1), B.ERR_ARG), (dict(X=0), B.ERR_ARG), (dict(Y=0), B.ERR_ARG),
    (dict(qw_codes=0), B.ERR_ARG), (dict(qw_scales=0), B.ERR_ARG), (dict(ldx=63), B.ERR_ARG), (dict(ldy=7), B.ERR_ARG),
    (dict(y_dtype=2), B.ERR_ARG), (dict(X=PTR + 1), B.ERR_ARG), (dict(Y=PTR + 2), B.ERR_ARG), (dict(qw_codes=PTR + 8), B.ERR_ARG),
    (dict(fmt=1, qw_scales=PTR + 2), B.ERR_ARG), (dict(d=48), B.ERR_SHAPE), (dict(fmt=1, d=96, ldx=96), B.ERR_SHAPE),
    (dict(m=17), B.ERR_UNSUPPORTED), (dict(n=1 << 31, ldy=1 << 31), B.ERR_UNSUPPORTED),
])
def test_matvec_refuses(kw, code):
    assert matvec(**kw) == code
    assert P.resq_last_error() != ""


def lp(**kw):
    a = dict(logits=PTR, dtype=1, m=4, V=100, ld=100, targets=PTR, temperature=1.0, logp=PTR, stats=PTR, top_k=2,
             top_logp=PTR, top_index=PTR, workspace=PTR, workspace_bytes=1 << 30)
    a.update(kw)
    return P.resq_token_logprobs(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(logits=0), B.ERR_ARG), (dict(dtype=3), B.ERR_ARG), (dict(m=-1), B.ERR_ARG), (dict(V=-1), B.ERR_ARG),
    (dict(ld=99), B.ERR_ARG), (dict(targets=0), B.ERR_ARG), (dict(targets=PTR + 4), B.ERR_ARG), (dict(stats=0), B.ERR_ARG),
    (dict(temperature=0.0), B.ERR_ARG), (dict(temperature=-1.0), B.ERR_ARG), (dict(temperature=NAN), B.ERR_ARG),
    (dict(temperature=float("inf")), B.ERR_ARG), (dict(temperature=1e-30), B.ERR_ARG), (dict(top_k=-1), B.ERR_ARG),
    (dict(top_k=33), B.ERR_ARG), (dict(top_logp=0), B.ERR_ARG), (dict(top_index=0), B.ERR_ARG), (dict(logits=PTR + 2), B.ERR_ARG),
    (dict(V=0), B.ERR_SHAPE), (dict(V=1 << 31, ld=1 << 31), B.ERR_UNSUPPORTED),
    (dict(m=1, V=100000, ld=100000, workspace=0), B.ERR_WORKSPACE),
    (dict(m=1, V=100000, ld=100000, workspace=PTR + 8), B.ERR_WORKSPACE),
    (dict(m=1, V=100000, ld=100000, workspace_bytes=8), B.ERR_WORKSPACE),
])
def test_token_logprobs_refuses(kw, code):
    assert lp(**kw) == code
    assert P.resq_last_error() != ""


def lpb(**kw):
    a = dict(logits=PTR, dtype=1, m=4, V=100, ld=100, targets=PTR, temperature=1.0, stats=PTR, dlogp=PTR, dentropy=PTR,
             dlogits=PTR, out_dtype=0, ldd=100)
    a.update(kw)
    return P.resq_token_logprobs_bwd(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(logits=0), B.ERR_ARG), (dict(targets=0), B.ERR_ARG), (dict(stats=0), B.ERR_ARG), (dict(dlogits=0), B.ERR_ARG),
    (dict(out_dtype=2), B.ERR_ARG), (dict(ldd=99), B.ERR_ARG), (dict(dlogp=PTR + 2), B.ERR_ARG),
    (dict(temperature=0.0), B.ERR_ARG), (dict(V=0), B.ERR_SHAPE), (dict(m=1 << 40), B.ERR_UNSUPPORTED),
])
def test_token_logprobs_bwd_refuses(kw, code):
    assert lpb(**kw) == code
    assert P.resq_last_error() != ""


def test_empty_calls_succeed():
    assert fwd(m=0, H=0, Y=PTR, H_out=0, X=0) == B.OK
    assert matvec(m=0, X=0, Y=0) == B.OK and matvec(n=0, Y=0, ldy=0) == B.OK
    assert lp(m=0, logits=0) == B.OK and lpb(m=0, logits=0, dlogits=0) == B.OK
    assert fwd(m=0, H=0, H_out=0, X=0, gate_mode=2, gate=0) == B.OK  # a gate of no rows
    assert P.resq_last_error() == ""


def test_workspace_sizes():
    size = P.resq_workspace_size
    assert size(B.OP_BLOCK_NORM_BWD, 0, 0, 0, 64, 0) == 0 and size(B.OP_BLOCK_NORM_BWD, 0, 0, -1, 64, 0) == 0
    assert size(B.OP_BLOCK_NORM_BWD, 0, 0, 4, 1 << 15, 0) == 0  # beyond the widths it takes
    assert 0 < size(B.OP_BLOCK_NORM_BWD, 0, 0, 1, 64, 0) <= size(B.OP_BLOCK_NORM_BWD, 0, 0, 4096, 64, 0)
    assert size(B.OP_TOKEN_LOGPROBS, 0, 0, 1, 131072, 0) > 0
    assert size(B.OP_TOKEN_LOGPROBS, 0, 0, 1, 131072, 33) == 0
    # a row per workgroup needs no scratch
    assert size(B.OP_TOKEN_LOGPROBS, 0, 0, 1 << 20, 131072, 20) == 0


def test_python_refuses_host_tensors_and_bad_shapes():
    b = torch.bfloat16
    h, x = torch.zeros(4, 64, dtype=b), torch.zeros(4, 64, dtype=b)
    codes, scales = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.uint8)
    logits, t, stats = torch.zeros(4, 100), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 3)
    g = torch.ones(64, dtype=b)
    for call in (lambda: P.block_norm(h, x, gamma_pre=g), lambda: P.block_norm_bwd(h, torch.zeros(2, 4), dx=x, gamma_pre=g),
                 lambda: P.matvec_w4a16(x, codes, scales, "mxfp4"), lambda: P.token_logprobs(logits, t),
                 lambda: P.token_logprobs_bwd(logits, t, stats, torch.zeros(4))):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: P.block_norm(h, x[:, :32]), lambda: P.block_norm(h[0]), lambda: P.block_norm(h, x, gate=torch.zeros(3)),
                 lambda: P.block_norm(h.t(), x.t()), lambda: P.block_norm(h[:1].expand(4, 64), x),
                 lambda: P.block_norm(h, x, gamma_pre=g[:5]), lambda: P.matvec_w4a16(x, codes[:, :16], scales, "mxfp4"),
                 lambda: P.matvec_w4a16(x, codes, scales[:4], "mxfp4"), lambda: P.token_logprobs(logits, t[:2]),
                 lambda: P.token_logprobs(logits[0]), lambda: P.token_logprobs_bwd(logits, t, stats[:2], torch.zeros(4)),
                 lambda: P.token_logprobs_bwd(logits, t, stats, torch.zeros(3)),
                 lambda: P.token_logprobs_bwd(logits, t, stats, torch.zeros(4), out="f16")):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: P.block_norm(h.half(), x), lambda: P.block_norm(h, x, gamma_pre=g.float()),
                 lambda: P.matvec_w4a16(x.float(), codes, scales, "mxfp4"), lambda: P.matvec_w4a16(x, codes, scales.int(), "mxfp4"),
                 lambda: P.token_logprobs(logits, t.int()), lambda: P.token_logprobs(logits.double(), t),
                 lambda: P.token_logprobs_bwd(logits, t, stats.double(), torch.zeros(4))):
        with pytest.raises(TypeError):
            call()


def test_refused_calls_keep_the_error_message_of_their_entry_point():
    lib = ctypes.CDLL(P.library_path())
    assert lib is not None
    assert matvec(m=17) == B.ERR_UNSUPPORTED and "resq_linear_w4a16" in P.resq_last_error()
    assert fwd(Y=0) == B.ERR_ARG and "gamma_pre" in P.resq_last_error()


def test_limits_of_lengths():
    """The longest row of the few-token product, the longest norm, and one step past each."""
    assert matvec(d=(1 << 30) - 64, ldx=1 << 30, qw_codes=0) == B.ERR_ARG  # gets as far as the operands
    assert matvec(d=1 << 30, ldx=1 << 30) == B.ERR_UNSUPPORTED
    assert fwd(d=16384, ldh=16384, ldy=16384, ldho=16384, ldx=16384, H=0) == B.ERR_ARG
    assert fwd(d=16385, ldh=16385, ldy=16385, ldho=16385, ldx=16385) == B.ERR_UNSUPPORTED
    assert lp(m=1 << 31) == B.ERR_UNSUPPORTED and lpb(m=1 << 31) == B.ERR_UNSUPPORTED
    assert fwd(m=1 << 31) == B.ERR_UNSUPPORTED and bwd(m=1 << 31) == B.ERR_UNSUPPORTED


def test_in_place_needs_equal_types_and_strides():
    other = PTR + (1 << 12)
    assert fwd(ldho=80, rstd=PTR + 2) == B.ERR_ARG and "rstd" not in P.resq_last_error()
    assert bwd(lddh=80, workspace=0) == B.ERR_ARG
    assert bwd(lddh=80, dH=other, workspace=0) == B.ERR_WORKSPACE  # gets as far as the workspace
    assert bwd(m=1, lddh=80, workspace=0) == B.ERR_WORKSPACE       # one row has no stride
    assert lpb(stats=0) == B.ERR_ARG and "in place" in P.resq_last_error()  # float32 logits, bf16 gradient
    assert lpb(dtype=0, ldd=104, stats=0) == B.ERR_ARG and "in place" in P.resq_last_error()
    assert lpb(dlogits=other, ldd=104, stats=0) == B.ERR_ARG and "in place" not in P.resq_last_error()
