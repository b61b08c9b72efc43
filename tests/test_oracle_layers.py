"""Pins of oracle/layers.py: its gradients by differences of its forwards, and those against torch in float64."""
import numpy as np
import pytest

from oracle import layers as ol

torch = pytest.importorskip("torch")
STEP = 1e-6


def differences(f, x, got):
    """(central differences at STEP: rounding of sums of some tens, 2^-53 over STEP, is the larger part)"""
    for at in np.ndindex(*x.shape):
        was = x[at]
        x[at] = was + STEP
        hi = f()
        x[at] = was - STEP
        lo = f()
        x[at] = was
        assert abs((hi - lo) / (2 * STEP) - got[at]) < 1e-7, at


@pytest.mark.parametrize("N,D", [(1, 1), (3, 2), (4, 7)])
def test_norm(N, D):
    g = np.random.default_rng([N, D])
    x, dy, gamma, beta = g.standard_normal((N, D)), g.standard_normal((N, D)), g.standard_normal(D), g.standard_normal(D)
    y, stats, ey, es = ol.norm_fwd(x, gamma, beta, 0.1, "fp32")
    t = torch.nn.functional.layer_norm(*(torch.from_numpy(v) if isinstance(v, np.ndarray) else v
                                         for v in (x, (D,), gamma, beta)), eps=0.1).numpy()
    np.testing.assert_allclose(y, t, rtol=0, atol=1e-13)
    assert (ey >= 0).all() and (es >= 0).all()
    ref, _ = ol.norm_bwd(x, gamma, stats, dy, "fp32")
    f = lambda: float((dy * ol.norm_fwd(x, gamma, beta, 0.1, "fp32")[0]).sum())  # noqa: E731
    for v, k in ((x, "dx"), (gamma, "dgamma"), (beta, "dbeta")):
        differences(f, v, ref[k])


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu", "swiglu"])
def test_linear(act):
    g = np.random.default_rng(7)
    N, K, F = 4, 5, 6
    C = 2 * F if act == "swiglu" else F
    x, W, b = g.standard_normal((N, K)), g.standard_normal((K, C)), g.standard_normal(C)
    res, dy = g.standard_normal((N, F)), g.standard_normal((N, F))
    y, z, ey, ez = ol.linear_fwd(x, W, b, act, res, "fp32")
    tz = torch.from_numpy(x @ W + b)
    t = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
         "swiglu": lambda v: torch.nn.functional.silu(v[:, :F]) * v[:, F:]}[act](tz).numpy() + res
    np.testing.assert_allclose(y, t, rtol=0, atol=1e-13)
    ref, _ = ol.linear_bwd(x, W, z, dy, act, "fp32")
    f = lambda: float((dy * ol.linear_fwd(x, W, b, act, res, "fp32")[0]).sum())  # noqa: E731
    for v, k in ((x, "dx"), (W, "dW"), (b, "db")):
        differences(f, v, ref[k])
