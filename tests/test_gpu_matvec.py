"""resq_matvec_w4a16 on the GPU against the float64 oracle.  Products of bf16 and FP4 values are
exact in float32, and a sum of d terms is off by at most d 2^-24 times the sum of their magnitudes,
whatever its order; a bf16 result is rounded once more (2^-8)."""
import numpy as np
import pytest

from oracle import formats as F
from synth import activations, bf16_bits_to_f32, rng_tree, weights
from _gpu_util import Y_TOL, dev_bf16, host, log, normwise_err

pytestmark = pytest.mark.gpu

FMTS = ["mxfp4", "hif4"]
U, UB = 2.0 ** -24, 2.0 ** -8


def _case(fmt, m, d, n, seed):
    rx, rw = rng_tree(seed, 2)
    xb, wb = activations(rx, m, d, 0.01, 50.0), weights(rw, n, d)
    codes, scales = F.quantize(fmt, bf16_bits_to_f32(wb))
    w = F.dequantize(fmt, codes, scales)
    return xb, wb, bf16_bits_to_f32(xb).astype(np.float64), w


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("m,d,n", [(1, 64, 1), (1, 64, 15), (2, 128, 17), (16, 192, 33), (3, 2048, 100), (1, 2048, 2560),
                                   (5, 1088, 64), (16, 4160, 300), (8, 320, 1000), (1, 18944, 40), (13, 11008, 130),
                                   (4, 256, 20011), (16, 64, 3000), (9, 8128, 257)])
def test_matches_the_oracle(fmt, m, d, n):
    import torch
    import paper_2607_26515_amd as P
    log(f"matvec {fmt} m={m} d={d} n={n}")
    xb, wb, x, w = _case(fmt, m, d, n, m + d + n)
    qc, qs = P.quantize(dev_bf16(wb), fmt, axis=1)
    want, mags = x @ w.T, np.abs(x) @ np.abs(w).T
    y = P.matvec_w4a16(dev_bf16(xb), qc, qs, fmt)
    assert y.dtype == torch.float32 and y.shape == (m, n)
    assert (np.abs(host(y) - want) <= d * U * mags).all()
    assert normwise_err(host(y), want) <= Y_TOL
    yb = P.matvec_w4a16(dev_bf16(xb), qc, qs, fmt, out="bf16")
    assert torch.equal(yb, y.bfloat16())  # the float32 result, rounded once


def test_mxfp4_rows_of_an_odd_number_of_blocks():
    import paper_2607_26515_amd as P
    for d in (32, 96, 160, 224, 1056):
        xb, wb, x, w = _case("mxfp4", 6, d, 50, d)
        qc, qs = P.quantize(dev_bf16(wb), "mxfp4", axis=1)
        y = host(P.matvec_w4a16(dev_bf16(xb), qc, qs, "mxfp4"))
        assert (np.abs(y - x @ w.T) <= d * U * (np.abs(x) @ np.abs(w).T)).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_identity_weights_return_every_bf16_value(fmt):
    """W = c I returns c X bit for bit, for every finite bf16 value of X but those whose multiple
    by c is not a float32 (none for c = 1; for c = 1.75 the largest overflow to inf alike)."""
    import torch
    import paper_2607_26515_amd as P
    d, c = 4096, {"mxfp4": 1.0, "hif4": 1.75}[fmt]
    bits = np.arange(65536, dtype=np.uint32).astype(np.uint16).reshape(16, d)
    finite = (bits & 0x7F80) != 0x7F80
    bits = np.where(finite, bits, 0).astype(np.uint16)
    w = (torch.eye(d) * c).bfloat16().cuda()
    qc, qs = P.quantize(w, fmt, axis=1)
    y = host(P.matvec_w4a16(dev_bf16(bits), qc, qs, fmt))
    with np.errstate(over="ignore"):
        want = bf16_bits_to_f32(bits) * np.float32(c)
    big = np.abs(want) >= 2.0 ** -126  # below float32's normal range products may be flushed
    assert np.array_equal(y[big], want[big])
    assert (np.abs(y[~big]) <= 2.0 ** -126).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_strides_offsets_and_gaps(fmt):
    """X rows at odd strides and addresses, Y rows with gaps that keep their values, Y in place of a
    given tensor."""
    import torch
    import paper_2607_26515_amd as P
    m, d, n = 7, 576, 45
    xb, wb, x, w = _case(fmt, m, d, n, 5)
    qc, qs = P.quantize(dev_bf16(wb), fmt, axis=1)
    ref = P.matvec_w4a16(dev_bf16(xb), qc, qs, fmt)
    buf = torch.full((m * (d + 5) + 3,), float("nan"), dtype=torch.bfloat16, device="cuda")
    view = buf[3:3 + m * (d + 5)].view(m, d + 5)[:, :d]
    view.copy_(dev_bf16(xb).view(torch.bfloat16))
    for out, dt in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        y = torch.full((m, n + 3), 9.0, dtype=dt, device="cuda")
        got = P.matvec_w4a16(view, qc, qs, fmt, out=out, y=y[:, :n])
        assert torch.equal(got, ref.to(dt)) and (y[:, n:] == 9).all()


def test_empty_and_zero_length():
    import torch
    import paper_2607_26515_amd as P
    for fmt, sd in (("mxfp4", torch.uint8), ("hif4", torch.int32)):
        y = P.matvec_w4a16(torch.empty((3, 0), dtype=torch.bfloat16, device="cuda"),
                           torch.empty((5, 0), dtype=torch.uint8, device="cuda"), torch.empty((5, 0), dtype=sd, device="cuda"), fmt)
        assert y.shape == (3, 5) and (y == 0).all()
    with pytest.raises(P.ResqError) as e:
        P.matvec_w4a16(torch.zeros((17, 64), dtype=torch.bfloat16, device="cuda"),
                       torch.zeros((4, 32), dtype=torch.uint8, device="cuda"), torch.zeros((4, 2), dtype=torch.uint8, device="cuda"), "mxfp4")
    assert e.value.code == -3


@pytest.mark.parametrize("fmt", FMTS)
def test_rows_do_not_depend_on_each_other(fmt):
    """A token's result is the same alone and among others, and every run gives the same bits."""
    import torch
    import paper_2607_26515_amd as P
    xb, wb, _, _ = _case(fmt, 16, 3008, 500, 8)
    qc, qs = P.quantize(dev_bf16(wb), fmt, axis=1)
    x = dev_bf16(xb)
    y = P.matvec_w4a16(x, qc, qs, fmt)
    assert torch.equal(y, P.matvec_w4a16(x, qc, qs, fmt))
    for m in (1, 2, 3, 4, 5, 8, 9, 15):
        assert torch.equal(y[:m], P.matvec_w4a16(x[:m], qc, qs, fmt)), m
