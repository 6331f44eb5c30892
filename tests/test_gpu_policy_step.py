"""The operators around the linears run together, as a policy's steps run them, and in captured
graphs.  Every stage is compared with the float64 oracle on that stage's own inputs, so no error of
an earlier one enters a bound."""
import numpy as np
import pytest

from oracle import operators as O
from oracle import resq as Q
from _gpu_util import Y_TOL, log, normwise_err

pytestmark = pytest.mark.gpu

EPS = 1e-6
UB = 2.0 ** -8


def _np(t):
    return t.double().cpu().numpy()


def _bf16(a):
    import torch
    return torch.from_numpy(np.asarray(a, np.float32)).bfloat16().cuda()


def _close_bf16(got, want, slack):
    """A bf16 rounding (2^-8 of the value) and `slack` times the largest value of the row."""
    want = np.asarray(want)
    assert (np.abs(_np(got) - want) <= UB * np.abs(want) + slack * np.abs(want).max(axis=1, keepdims=True)).all()


@pytest.mark.parametrize("fmt", ["mxfp4", "hif4"])
@pytest.mark.parametrize("m", [1, 3, 16])
def test_decode_step(fmt, m):
    """The last sequences of a rollout: block update and norm, a 4-bit projection, the block update
    after it, the final norm, the logits' projection, and the tokens' log probabilities."""
    import torch
    import paper_2607_26515_amd as P
    log(f"decode step {fmt} m={m}")
    d, V = 512, 2000
    r = np.random.default_rng(m)
    h, y = _bf16(r.normal(size=(m, d))), torch.from_numpy(r.normal(size=(m, d)).astype(np.float32)).cuda()
    g1, g2 = _bf16(1 + 0.1 * r.normal(size=d)), _bf16(1 + 0.1 * r.normal(size=d))
    w = P.quantize(_bf16(r.normal(size=(d, d)) * 0.05), fmt)
    head = P.quantize(_bf16(r.normal(size=(V, d)) * 0.05), fmt)
    h1, x1, _ = P.block_norm(h, y, gamma_pre=g1, eps=EPS, save=False)
    o = P.matvec_w4a16(x1, *w, fmt)
    h2, x2, _ = P.block_norm(h1, o, gamma_pre=g2, eps=EPS, save=False)
    logits = P.matvec_w4a16(x2, *head, fmt)
    tokens = logits.argmax(1)
    out = P.token_logprobs(logits, tokens, top_k=5)
    scales = [s.cpu().numpy().view(np.uint32) if fmt == "hif4" else s.cpu().numpy() for s in (w[1], head[1])]
    want = O.matvec(fmt, _np(x1), w[0].cpu().numpy(), scales[0])
    assert normwise_err(_np(o), want) <= Y_TOL
    _close_bf16(h2, O.block_update(_np(h1), _np(o))[0], 1e-6)
    _close_bf16(x2, O.rms_norm(_np(h2), _np(g2), EPS)[0], 1e-6)
    assert normwise_err(_np(logits), O.matvec(fmt, _np(x2), head[0].cpu().numpy(), scales[1])) <= Y_TOL
    lp = O.token_logprobs(_np(logits), tokens.cpu().numpy(), 1.0, 5)
    assert np.array_equal(out["top_index"].cpu().numpy(), lp["top_index"])
    assert torch.equal(out["top_index"][:, 0].long(), tokens) and torch.equal(out["top_logp"][:, 0], out["logp"])
    # log S at 2000 logits within |z| < 20: (2000 / 256 + 64 + 84) 2^-24 < 1e-5
    assert np.abs(_np(out["logp"]) - lp["logp"]).max() < 1e-5


@pytest.mark.parametrize("fmt", ["mxfp4", "hif4"])
def test_training_step(fmt):
    """One layer and the logits of a training policy, forward and backward: norm, FP4 linear, block
    update with norms and gate, FP4 logits, log probabilities; then their gradients through
    resq_linear_bwd, whose bf16 dY and float32 dX the operators hand over as they are."""
    import torch
    import paper_2607_26515_amd as P
    log(f"training step {fmt}")
    m, d, V = 128, 256, 512
    r = np.random.default_rng(11)
    h = _bf16(r.normal(size=(m, d)))
    gp, g1, g2 = (_bf16(1 + 0.1 * r.normal(size=d)) for _ in range(3))
    gate = _bf16(0.8 + 0.1 * r.normal(size=d))
    w, head = _bf16(r.normal(size=(d, d)) * 0.06), _bf16(r.normal(size=(V, d)) * 0.06)
    targets = torch.from_numpy(r.integers(0, V, m)).cuda()
    targets[:20] = -1
    _, x1, r1 = P.block_norm(h, gamma_pre=g1, eps=EPS)
    y = P.linear_fwd(x1, *P.quantize(w, fmt), fmt, "none")
    kw = dict(gamma_post=gp, gate=gate, alpha=0.5, gamma_pre=g2)
    h2, x2, r2 = P.block_norm(h, y, eps=EPS, **kw)
    logits = P.linear_fwd(x2, *P.quantize(head, fmt), fmt, "none")
    out = P.token_logprobs(logits, targets)
    # maximise the mean log probability with an entropy bonus
    n = int((targets >= 0).sum())
    a = torch.full((m,), -1.0 / n, device="cuda")
    b = torch.full((m,), -0.01 / n, device="cuda")
    dlogits = P.token_logprobs_bwd(logits, targets, out["stats"], a, b)
    dx2, dhead = P.linear_bwd(dlogits, x2, head, fmt)
    g = P.block_norm_bwd(h2, r2, dx=dx2, y=y, **kw)
    dx1, dw = P.linear_bwd(g["dy"], x1, w, fmt)
    g1out = P.block_norm_bwd(h, r1, dx=dx1, dh=g["dh"], gamma_pre=g1, want_dy=False)

    t = targets.cpu().numpy()
    want = O.token_logprobs(_np(logits), t)
    assert np.abs(_np(out["logp"]) - want["logp"]).max() < 1e-5
    wl = O.token_logprobs_bwd(_np(logits), t, _np(out["stats"]), _np(a), _np(b))
    _close_bf16(dlogits, wl, 1e-5)
    assert (dlogits[:20] == 0).all()

    def f32(v):
        return v.float().cpu().numpy()

    o = Q.resq_backward(fmt, f32(dlogits), f32(x2), f32(head))
    assert normwise_err(_np(dx2), o["dx64"]) <= Y_TOL and normwise_err(_np(dhead), o["dw64"]) <= Y_TOL
    o = O.block_norm_bwd(_np(h2), _np(y), _np(r2[0]), _np(r2[1]), _np(dx2), np.zeros((m, d)), _np(gp), _np(gate), 0.5, _np(g2))
    _close_bf16(g["dh"], o["dh"], 1e-5)
    _close_bf16(g["dy"], o["dy"], 1e-5)
    for k in ("dgamma_post", "dgamma_pre", "dgate"):
        assert normwise_err(_np(g[k]), o[k]) <= Y_TOL, k
    o = Q.resq_backward(fmt, f32(g["dy"]), f32(x1), f32(w))
    assert normwise_err(_np(dx1), o["dx64"]) <= Y_TOL and normwise_err(_np(dw), o["dw64"]) <= Y_TOL
    o = O.block_norm_bwd(_np(h), np.zeros((m, d)), None, _np(r1[1]), _np(dx1), _np(g["dh"]), None, None, 1.0, _np(g1))
    _close_bf16(g1out["dh"], o["dh"], 1e-5)
    assert normwise_err(_np(g1out["dgamma_pre"]), o["dgamma_pre"]) <= Y_TOL
    assert g1out["dy"] is None and g1out["dgate"] is None


def test_graph_replays_match_eager():
    """Every operator captured in two graphs with inputs of their own, replayed in turn with eager
    calls between: each replay gives the eager result bit for bit."""
    import torch
    import paper_2607_26515_amd as P
    print("graph of the operators around the linears", flush=True)
    m, d, V = 4, 1024, 40000
    gen = torch.Generator(device="cuda").manual_seed(1)

    def inputs():
        rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
        return dict(h=rnd(m, d).bfloat16(), y=rnd(m, d), g=(1 + 0.1 * rnd(d)).bfloat16(), gate=rnd(d), logits=rnd(m, V),
                    t=torch.randint(0, V, (m,), generator=gen, device="cuda"), a=rnd(m), dx=rnd(m, d))

    w = P.quantize((torch.randn((512, d), generator=gen, device="cuda") * 0.02).bfloat16(), "hif4")

    def step(i, stream=None):
        h, x, r = P.block_norm(i["h"], i["y"], gamma_post=i["g"], gate=i["gate"], gamma_pre=i["g"], stream=stream)
        z = P.matvec_w4a16(x, *w, "hif4", stream=stream)
        o = P.token_logprobs(i["logits"], i["t"], top_k=8, stream=stream)
        dl = P.token_logprobs_bwd(i["logits"], i["t"], o["stats"], i["a"], i["a"], stream=stream)
        b = P.block_norm_bwd(h, r, dx=i["dx"], y=i["y"], gamma_post=i["g"], gate=i["gate"], gamma_pre=i["g"], stream=stream)
        return [h, x, r, z, dl, *o.values(), *b.values()]

    sets = [inputs(), inputs()]
    ref = [[v.clone() for v in step(i)] for i in sets]
    cs = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs, outs = [], []
    with torch.cuda.stream(cs):
        for i in sets:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=cs):
                outs.append(step(i, cs))
            graphs.append(g)
        for rep in range(3):
            for k in (0, 1):
                for v in outs[k]:
                    v.fill_(7)
                graphs[k].replay()
                step(sets[1 - k], cs)
                cs.synchronize()
                for got, want in zip(outs[k], ref[k]):
                    assert torch.equal(got, want)


def test_rows_beyond_32_bit_offsets():
    """Operands whose rows lie 2 GiB and more apart: offsets pass 32 bits in bytes and elements."""
    import torch
    import paper_2607_26515_amd as P
    stride = (1 << 31) + 8  # elements
    print("rows 4 GiB apart", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(2)
    d = 1000
    buf = torch.empty(2 * stride + d, dtype=torch.bfloat16, device="cuda")
    view = torch.as_strided(buf, (3, d), (stride, 1))
    x = torch.randn((3, d), generator=gen, device="cuda").bfloat16()
    view.copy_(x)
    g = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    t = torch.tensor([1, 2, 999], device="cuda")
    y = torch.randn((3, d), generator=gen, device="cuda")
    for a, b in ((P.block_norm(view, y, gamma_pre=g), P.block_norm(x, y, gamma_pre=g)),):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    a, b = P.token_logprobs(view, t, top_k=3), P.token_logprobs(x, t, top_k=3)
    assert all(torch.equal(a[k], b[k]) for k in a)
    dl = P.token_logprobs_bwd(x, t, b["stats"], torch.ones(3, device="cuda"))
    assert torch.equal(P.token_logprobs_bwd(view, t, a["stats"], torch.ones(3, device="cuda"), dlogits=view), dl)
    view.copy_(x)
    w = P.quantize((torch.randn((64, 960), generator=gen, device="cuda") * 0.02).bfloat16(), "mxfp4")
    assert torch.equal(P.matvec_w4a16(view[:, :960], *w, "mxfp4"), P.matvec_w4a16(x[:, :960].contiguous(), *w, "mxfp4"))
