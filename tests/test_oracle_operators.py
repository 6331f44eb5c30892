"""The float64 oracle of the operators around the linears against facts fixed outside it: central
differences for every gradient, closed forms for uniform and one-hot rows, and torch's own
functions where they exist."""
import numpy as np
import pytest

from oracle import formats as F
from oracle import operators as O


def _rng(seed):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("gate", [None, "channel", "token"])
def test_block_norm_gradients_against_differences(post, pre, gate):
    """f = <A, h'> + <B, x>: every gradient against (f(+s) - f(-s)) / 2s, whose own error is
    s^2 |f'''| / 6 + 2^-52 |f| / s, below 1e-8 here for s = 1e-5."""
    r = _rng(1)
    m, d, alpha, eps = 3, 5, 0.7, 1e-3
    v = {"h": r.normal(size=(m, d)), "y": r.normal(size=(m, d))}
    if post:
        v["gamma_post"] = 1 + 0.3 * r.normal(size=d)
    if pre:
        v["gamma_pre"] = 1 + 0.3 * r.normal(size=d)
    if gate:
        v["gate"] = r.normal(size=d if gate == "channel" else (m, 1))
    A, B = r.normal(size=(m, d)), r.normal(size=(m, d))

    def forward(v):
        h, rp = O.block_update(v["h"], v["y"], v.get("gamma_post"), v.get("gate"), alpha, eps)
        x, rh = O.rms_norm(h, v["gamma_pre"], eps) if pre else (None, None)
        return h, rp, x, rh

    def f(v):
        h, _, x, _ = forward(v)
        return (A * h).sum() + ((B * x).sum() if pre else 0.0)

    h, rp, _, rh = forward(v)
    g = O.block_norm_bwd(h, v["y"], rp, rh, B, A, v.get("gamma_post"), v.get("gate"), alpha, v.get("gamma_pre"))
    for name in v:
        got = g["d" + name]
        assert got.shape == v[name].shape
        for i in np.ndindex(v[name].shape):
            s = 1e-5
            hi, lo = {**v, name: v[name].copy()}, {**v, name: v[name].copy()}
            hi[name][i] += s
            lo[name][i] -= s
            assert abs((f(hi) - f(lo)) / (2 * s) - got[i]) < 1e-7, name


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_logprob_gradients_against_differences(temperature):
    r = _rng(2)
    m, v = 4, 7
    x = r.normal(size=(m, v)) * 2
    x[1, 3] = -np.inf
    t = np.array([0, 6, 2, -1])
    a, b = r.normal(size=m), r.normal(size=m)

    def f(x):
        o = O.token_logprobs(x, t, temperature)
        return (a * o["logp"]).sum() + (b * o["stats"][:, 2]).sum()

    g = O.token_logprobs_bwd(x, t, O.token_logprobs(x, t, temperature)["stats"], a, b, temperature)
    for i in np.ndindex(x.shape):
        s = 1e-5
        hi, lo = x.copy(), x.copy()
        hi[i] += s
        lo[i] -= s
        assert abs((f(hi) - f(lo)) / (2 * s) - g[i]) < 1e-7
    assert (g[3] == 0).all() and g[1, 3] == 0


def test_logprobs_closed_forms():
    v = 16
    o = O.token_logprobs(np.zeros((1, v)), np.array([3]), 1.0, 4)
    assert np.allclose(o["logp"], -np.log(v)) and np.allclose(o["stats"][0], [0, np.log(v), np.log(v)])
    assert o["top_index"][0].tolist() == [0, 1, 2, 3]  # ties: the lowest index first
    x = np.full((2, v), -np.inf)
    x[0, 5] = 2.0
    o = O.token_logprobs(x, np.array([5, 5]), 0.5, 3)
    assert o["logp"].tolist() == [0.0, -np.inf]
    assert o["stats"].tolist() == [[2.0, 0.0, 0.0], [-np.inf, -np.inf, 0.0]]
    assert o["top_index"].tolist() == [[5, -1, -1], [-1, -1, -1]]


def test_logprobs_against_torch():
    import torch
    r = _rng(3)
    x = torch.from_numpy(r.normal(size=(5, 33)) * 3)
    t = torch.from_numpy(r.integers(0, 33, 5))
    o = O.token_logprobs(x.numpy(), t.numpy(), 0.8)
    lq = torch.log_softmax(x / 0.8, 1)
    assert np.allclose(o["logp"], lq.gather(1, t[:, None])[:, 0].numpy(), rtol=1e-12, atol=1e-13)
    assert np.allclose(o["stats"][:, 2], torch.distributions.Categorical(logits=x / 0.8).entropy().numpy(), atol=1e-12)


@pytest.mark.parametrize("fmt", ["mxfp4", "hif4"])
def test_matvec_is_the_product_with_the_dequantized_weights(fmt):
    r = _rng(4)
    w = r.normal(size=(3, 128)).astype(np.float32)
    codes, scales = F.quantize(fmt, w)
    x = r.normal(size=(2, 128))
    want = x @ F.dequantize(fmt, codes, scales).T
    assert np.array_equal(O.matvec(fmt, x, F.pack_nibbles(codes), scales), want)
