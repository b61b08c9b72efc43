"""GPU tests of layer norm and linear layers (sa_layer_norm_*, sa_linear_*) against the fp64
oracle, element by element within the bounds that oracle/layers.py derives."""
import numpy as np
import pytest

from oracle import layers as ol
from oracle.recent import HALF

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def sa():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_08443_amd import sa_sketch
    sa_sketch.lib()
    return sa_sketch


def values(dtype, shape, seed, sd=1.0, mean=0.0):
    g = np.random.default_rng([8443, seed, *shape])
    return torch.from_numpy((g.standard_normal(shape) * sd + mean).astype(np.float32)).to(DT[dtype])


def f8(t):
    return t.double().numpy()


def within(got, ref, off, what):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape, what
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    worst = np.max(np.abs(got - ref) / np.maximum(off, 1e-30), initial=0.0)
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound"


NORM = [(1, 1), (1, 64), (3, 63), (130, 64), (65, 100), (33, 128), (17, 129), (40, 256), (9, 500), (50, 512), (70, 1024),
        (5, 1023), (300, 1024), (7, 2048), (3, 2050), (5, 4096), (6, 5001), (4, 8192), (3, 9001), (2, 20000)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,D", NORM)
def test_norm(sa, N, D, dtype):
    print(f"norm {N}x{D} {dtype}", flush=True)
    x = values(dtype, (N, D), 1, 1.5, 0.7)
    gamma, beta, dy = values(dtype, (D,), 2, 0.1, 1.0), values(dtype, (D,), 3, 0.1), values(dtype, (N, D), 4)
    y, stats = sa.layer_norm_fwd(x.cuda(), gamma.cuda(), beta.cuda(), eps=1e-5)
    ry, rs, ey, es = ol.norm_fwd(f8(x), f8(gamma), f8(beta), 1e-5, dtype)
    assert y.dtype == DT[dtype] and stats.dtype == torch.float32
    within(y, ry, ey, "y")
    within(stats, rs, es, "stats")
    given = torch.from_numpy(rs.astype(np.float32))
    got = sa.layer_norm_bwd(x.cuda(), gamma.cuda(), given.cuda(), dy.cuda())
    ref, off = ol.norm_bwd(f8(x), f8(gamma), f8(given), f8(dy), dtype)
    assert got["dx"].dtype == DT[dtype] and got["dgamma"].dtype == got["dbeta"].dtype == torch.float32
    for k in ref:
        within(got[k], ref[k], off[k], k)


def test_norm_of_rows_far_from_zero(sa):
    """The squares are summed around the mean."""
    x = values("fp32", (40, 1000), 5, 1e-2, 1000.0)
    one, zero = torch.ones(1000), torch.zeros(1000)
    y, stats = sa.layer_norm_fwd(x.cuda(), one.cuda(), zero.cuda(), eps=0.0)
    ry, rs, ey, es = ol.norm_fwd(f8(x), f8(one), f8(zero), 0.0, "fp32")
    within(y, ry, ey, "y")
    within(stats, rs, es, "stats")


def test_norm_of_equal_values(sa):
    x = torch.full((3, 777), 2.5, dtype=torch.bfloat16)
    gamma, beta = values("bf16", (777,), 6), values("bf16", (777,), 7)
    y, stats = sa.layer_norm_fwd(x.cuda(), gamma.cuda(), beta.cuda(), eps=1e-5)
    assert torch.equal(y.cpu(), beta.expand(3, -1))
    np.testing.assert_allclose(stats.cpu().numpy()[:, 1], 1e-5 ** -0.5, rtol=1e-6)


@pytest.mark.parametrize("D", [64, 100, 1024])
def test_norm_of_strided_rows_in_place(sa, D):
    """Rows inside wider ones, y and dx in their inputs' place, a row with a NaN beside the others."""
    wide = values("bf16", (37, D + 24), 8).cuda()
    x = wide[:, 8:8 + D]
    gamma, beta = values("bf16", (D,), 9).cuda(), values("bf16", (D,), 10).cuda()
    y, stats = sa.layer_norm_fwd(x, gamma, beta)
    y2, _ = sa.layer_norm_fwd(x.contiguous(), gamma, beta)
    assert torch.equal(y, y2)
    z = x.contiguous()
    sa.layer_norm_fwd(z, gamma, beta, y=z)
    assert torch.equal(y, z)
    dy = values("bf16", (37, D), 11).cuda()
    ref = sa.layer_norm_bwd(x, gamma, stats, dy)
    d2 = dy.clone()
    got = sa.layer_norm_bwd(x, gamma, stats, d2, dx=d2)
    for k in ref:
        assert torch.equal(got[k], ref[k]), k
    z = x.contiguous()
    z[5, 3] = float("nan")
    y3, _ = sa.layer_norm_fwd(z, gamma, beta)
    assert torch.isnan(y3[5]).all() and torch.equal(torch.cat([y3[:5], y3[6:]]), torch.cat([y[:5], y[6:]]))


def test_norm_without_rows(sa):
    for D in (64, 20000):
        x, w = torch.empty(0, D, dtype=torch.bfloat16, device="cuda"), torch.ones(D, dtype=torch.bfloat16, device="cuda")
        y, stats = sa.layer_norm_fwd(x, w, w)
        assert y.shape == (0, D) and stats.shape == (0, 2)
        g = sa.layer_norm_bwd(x, w, stats, y)
        assert not g["dgamma"].any() and not g["dbeta"].any()


LINEAR = [(1, 1, 1), (1, 64, 64), (1, 1024, 1024), (2, 256, 512), (5, 200, 331), (64, 64, 64), (100, 128, 96), (130, 72, 40),
          (257, 320, 264), (300, 512, 1024), (1000, 63, 65), (77, 1030, 128), (16, 192, 8), (3, 4096, 24),
          # sizes that run on copies padded to whole pieces, and tiles whose last rows, columns and k end inside
          (96, 1024, 256), (200, 1096, 600), (700, 1001, 903), (1300, 999, 640), (900, 640, 1111)]
ACTS = ["none", "relu", "gelu", "silu", "swiglu"]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("N,K,F", LINEAR)
def test_linear_forward(sa, N, K, F, act, dtype):
    print(f"linear {N}x{K}x{F} {act} {dtype}", flush=True)
    C = 2 * F if act == "swiglu" else F
    x, W, b = values(dtype, (N, K), 1), values(dtype, (K, C), 2, K ** -0.5), values(dtype, (C,), 3)
    res = values(dtype, (N, F), 4)
    for bias, residual, want in ((b, res, True), (None, None, False), (None, res, True), (b, None, False)):
        y, pre = sa.linear_fwd(x.cuda(), W.cuda(), bias=None if bias is None else bias.cuda(), act=act,
                               residual=None if residual is None else residual.cuda(), want_pre=want)
        ry, rz, ey, ez = ol.linear_fwd(f8(x), f8(W), None if bias is None else f8(bias), act,
                                       None if residual is None else f8(residual), dtype)
        assert y.dtype == DT[dtype]
        within(y, ry, ey, "y")
        if want:
            assert pre.dtype == DT[dtype]
            within(pre, rz, ez, "pre")
        else:
            assert pre is None


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("N,K,F", LINEAR)
def test_linear_backward(sa, N, K, F, act, dtype):
    print(f"linear_bwd {N}x{K}x{F} {act} {dtype}", flush=True)
    C = 2 * F if act == "swiglu" else F
    x, W, pre, dy = values(dtype, (N, K), 1), values(dtype, (K, C), 2, K ** -0.5), values(dtype, (N, C), 3, 2.0), values(dtype, (N, F), 4)
    ref, off = ol.linear_bwd(f8(x), f8(W), f8(pre), f8(dy), act, dtype)
    for wdt in ([None] if dtype == "fp32" else [None, torch.float32]):
        got = sa.linear_bwd(x.cuda(), W.cuda(), dy.cuda(), bias=True, act=act, pre=None if act == "none" else pre.cuda(),
                            weight_dtype=wdt)
        assert set(got) == {"dx", "dW", "db"}
        for k in got:
            want = DT[dtype] if k == "dx" or wdt is None else wdt
            assert got[k].dtype == want
            half = HALF["bf16"] if want == torch.bfloat16 else HALF["fp32"]
            within(got[k], ref[k], off[k] + half * np.abs(ref[k]), k)
    got = sa.linear_bwd(x.cuda(), W.cuda(), dy.cuda(), act=act, pre=None if act == "none" else pre.cuda())
    assert set(got) == {"dx", "dW"}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("N,K,F", [(1, 64, 64), (5, 200, 331), (64, 64, 64), (300, 512, 1024), (700, 1001, 903), (1000, 63, 65)])
def test_linear_result_in_the_residuals_place(sa, N, K, F, act, dtype):
    C = 2 * F if act == "swiglu" else F
    x, W, res = values(dtype, (N, K), 1).cuda(), values(dtype, (K, C), 2, K ** -0.5).cuda(), values(dtype, (N, F), 4).cuda()
    y, _ = sa.linear_fwd(x, W, act=act, residual=res)
    out = res.clone()
    got, _ = sa.linear_fwd(x, W, act=act, residual=out, y=out)
    assert got is out and torch.equal(out, y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,K,F,extra", [(1, 64, 64, 8), (5, 200, 331, 3), (130, 256, 512, 64), (300, 512, 128, 5), (257, 72, 1000, 8)])
def test_linear_of_strided_rows(sa, N, K, F, extra, dtype):
    wide = values(dtype, (N, K + extra), 1).cuda()
    x, W, dy = wide[:, :K], values(dtype, (K, F), 2, K ** -0.5).cuda(), values(dtype, (N, F), 3).cuda()
    close = x.contiguous()
    y, _ = sa.linear_fwd(x, W)
    ry, _, ey, _ = ol.linear_fwd(f8(close.cpu()), f8(W.cpu()), None, "none", None, dtype)
    within(y, ry, ey, "y")
    got = sa.linear_bwd(x, W, dy, bias=True)
    ref, off = ol.linear_bwd(f8(close.cpu()), f8(W.cpu()), None, f8(dy.cpu()), "none", dtype)
    for k in got:
        within(got[k], ref[k], off[k] + HALF[dtype] * np.abs(ref[k]), k)


def test_linear_without_rows(sa):
    for act in ACTS:
        x, W = torch.empty(0, 64, device="cuda"), torch.ones(64, 64, device="cuda")
        F = 32 if act == "swiglu" else 64
        y, pre = sa.linear_fwd(x, W, act=act, want_pre=True)
        assert y.shape == (0, F) and pre.shape == (0, 64)
        g = sa.linear_bwd(x, W, y, bias=True, act=act, pre=pre)
        assert g["dx"].shape == (0, 64) and not g["dW"].any() and not g["db"].any()


def test_linear_rows_that_are_no_numbers(sa):
    """A row's NaN or infinity stays in its row, forward and in dx, on copies with padding too."""
    for N, K, F in ((300, 512, 256), (300, 333, 199), (40, 1000, 64)):
        x, W, dy = values("bf16", (N, K), 1).cuda(), values("bf16", (K, F), 2).cuda(), values("bf16", (N, F), 3).cuda()
        y, _ = sa.linear_fwd(x, W)
        dx = sa.linear_bwd(x, W, dy)["dx"]
        for bad in (float("nan"), float("inf")):
            z, dz = x.clone(), dy.clone()
            z[7, K - 1], dz[7, F - 1] = bad, bad
            got, _ = sa.linear_fwd(z, W)
            gx = sa.linear_bwd(x, W, dz)["dx"]
            for a, b in ((got, y), (gx, dx)):
                assert torch.equal(a[:7], b[:7]) and torch.equal(a[8:], b[8:])
                assert not torch.isfinite(a[7]).any()


def test_bad_tensors_are_refused(sa):
    from paper_2609_08443_amd.sa_sketch import SAError
    x, W = torch.zeros(4, 64, device="cuda"), torch.zeros(64, 64, device="cuda")
    one = torch.ones(64, device="cuda")
    stats = torch.zeros(4, 2, device="cuda")
    for call in (lambda: sa.linear_fwd(x[:1].expand(4, -1), W), lambda: sa.linear_fwd(x.t(), W),
                 lambda: sa.linear_fwd(x, W.t()), lambda: sa.linear_fwd(x, W.bfloat16()), lambda: sa.linear_fwd(x, W, act="tanh"),
                 lambda: sa.linear_fwd(x, W, bias=one[:63]), lambda: sa.linear_fwd(x, W, residual=x[:3]),
                 lambda: sa.linear_fwd(x.half(), W.half()), lambda: sa.linear_fwd(x, W.cpu()),
                 lambda: sa.linear_fwd(x, W[:, :63].contiguous(), act="swiglu"), lambda: sa.linear_fwd(x[:, 1:33], W[:32]),
                 lambda: sa.linear_bwd(x, W, x, act="relu"), lambda: sa.linear_bwd(x, W, x, weight_dtype=torch.bfloat16),
                 lambda: sa.linear_bwd(x, W, x, workspace=torch.empty(1, dtype=torch.uint8, device="cuda")),
                 lambda: sa.layer_norm_fwd(x[:1].expand(4, -1), one, one), lambda: sa.layer_norm_fwd(x, one[:3], one),
                 lambda: sa.layer_norm_fwd(x, one, one, eps=-1.0), lambda: sa.layer_norm_fwd(x[0], one, one),
                 lambda: sa.layer_norm_bwd(x, one, stats[:3], x), lambda: sa.layer_norm_bwd(x, one, stats, x.t().contiguous()),
                 lambda: sa.layer_norm_bwd(x, one, stats, x, workspace=torch.empty(1, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(SAError):
            call()
