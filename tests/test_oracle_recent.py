"""Pins of oracle/recent.py: the attention by plain loops, its gradients by differences."""
import numpy as np
import pytest

from oracle import recent as orec


def by_loops(q, K, V, offsets, targets, ends=None, window=0, slopes=None, scale=None, cap=0.0):
    N, h, d = q.shape
    g = h // K.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out, lse = np.zeros(q.shape), np.full((N, h), -np.inf)
    for b in range(len(offsets) - 1):
        L = offsets[b + 1] - offsets[b]
        for i in range(targets[b], targets[b + 1]):
            e = L if ends is None else min(max(int(ends[i]), 0), L)
            lo = max(0, e - window) if window else 0
            for y in range(h):
                s = []
                for j in range(lo, e):
                    x = scale * float(q[i, y] @ K[offsets[b] + j, y // g])
                    if cap:
                        x = cap * np.tanh(x / cap)
                    s.append(x - (0.0 if slopes is None else slopes[y] * (e - 1 - j)))
                if s:
                    w = np.exp(s)
                    lse[i, y] = np.log(w.sum())
                    out[i, y] = (w / w.sum()) @ V[offsets[b] + lo:offsets[b] + e, y // g]
    return out, lse


CASES = {
    "plain": {}, "cap": dict(cap=0.7), "bias": dict(slopes=np.array([0.5, 0.1, 0.0, 0.2])), "window": dict(window=3),
    "ends": dict(ends=np.array([4, 0, -3, 9, 2, 1, 7, 5])),
    "all": dict(cap=1.5, slopes=np.array([0.5, 0.1, 0.0, 0.2]), window=2, ends=np.array([4, 0, 3, 9, 2, 1, 7, 5]), scale=0.8),
}


def inputs():
    g = np.random.default_rng(5)
    offsets, targets = np.array([0, 5, 5, 12]), np.array([0, 3, 4, 7])   # a target and two tokens behind the last user
    return [g.standard_normal(s) for s in ((8, 4, 6), (14, 2, 6), (14, 2, 6))], offsets, targets, g.standard_normal((8, 4, 6))


@pytest.mark.parametrize("name", CASES)
def test_forward_by_loops(name):
    (q, K, V), offsets, targets, _ = inputs()
    out, lse, eo, el = orec.fwd(q, K, V, offsets, targets, **CASES[name])
    ro, rl = by_loops(q, K, V, offsets, targets, **CASES[name])
    np.testing.assert_allclose(out, ro, rtol=0, atol=1e-13)
    np.testing.assert_allclose(lse, rl, rtol=0, atol=1e-13)
    assert (eo >= 0).all() and (el >= 0).all()


@pytest.mark.parametrize("name", CASES)
def test_gradients_by_differences(name):
    (q, K, V), offsets, targets, dout = inputs()
    g, _ = orec.bwd(q, K, V, offsets, targets, dout, **CASES[name])
    step = 1e-5
    for x, k in ((q, "dq"), (K, "dK"), (V, "dV")):
        for at in np.ndindex(*x.shape):
            was = x[at]
            f = []
            for s in (step, -step):
                x[at] = was + s
                f.append(float((dout * by_loops(q, K, V, offsets, targets, **CASES[name])[0]).sum())
                         if at[-1] == 0 else float((dout * orec.fwd(q, K, V, offsets, targets, **CASES[name])[0]).sum()))
            x[at] = was
            # (central differences: off by step^2 / 6 of third derivatives, and 2^-53 of sums of some tens over step)
            assert abs((f[0] - f[1]) / (2 * step) - g[k][at]) < 1e-8, (k, at)
    assert not g["dK"][12:].any() and not g["dV"][12:].any() and not g["dq"][7:].any()
