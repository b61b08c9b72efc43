"""Pins of the sketch cache's oracle (oracle/cache.py) and the refusals of the cache's
entry points, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle import stca as ostca
from paper_2609_08443_amd import sa_sketch as sa

FMTS = ("fp4", "fp8")


def test_representable_values():
    assert oc.magnitudes("fp4").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(oc.magnitudes("fp8"), codes)


@pytest.mark.parametrize("fmt", FMTS)
def test_no_value_is_off_by_more_than_half_a_step(fmt):
    """Against the value itself in the normal range, against the group's least step below it."""
    rng = np.random.default_rng(3)
    half = {"fp4": 2.0 ** -2, "fp8": 2.0 ** -4}[fmt]      # finfo.eps / 2 of e2m1 and e4m3
    least = {"fp4": 0.5, "fp8": 2.0 ** -9}[fmt]
    for sd in (1.0, 1e-20, 1e25):
        x = rng.standard_normal((40, 75)).astype(np.float32).astype(np.float64) * sd
        codes, scales = oc.quantise(x, fmt)
        v = oc.dequantise(codes, scales, fmt)
        step = np.repeat(np.ldexp(least, scales.astype(int) - 127), oc.GROUP, 1)[:, :75]
        assert np.all(np.abs(v - x) <= np.maximum(half * np.abs(x), step / 2))
        # and the exponent is the least that does it: the largest magnitude is past half the range
        top = np.abs(v).reshape(40, 75)[:, :32].max(1) / np.ldexp(1.0, scales[:, 0].astype(int) - 127)
        assert np.all(top >= {"fp4": 3.0, "fp8": 224.0}[fmt])


def test_fp8_rounding_is_torchs():
    x = np.linspace(-464, 464, 7001).astype(np.float32)
    x = np.concatenate([x, np.geomspace(1e-5, 464, 3000).astype(np.float32)])
    row = np.stack([x, np.full_like(x, 464.0)], 1).astype(np.float64)   # beside 464: e = 0
    codes, scales = oc.quantise(row, "fp8")
    assert np.all(scales == 127)
    ref = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    np.testing.assert_array_equal(codes[:, 0], ref.numpy())


def test_fp4_ties_go_to_even_codes():
    x = np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, -5.0, -7.0, 0.0, -0.0]])
    codes, scales = oc.quantise(x, "fp4")
    assert scales[0, 0] == 127
    assert oc.dequantise(codes, scales, "fp4")[0].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 0, -1, -4, -6, 0, 0]
    assert codes[0, 8] == 8 and codes[0, 13] == 8      # the sign of a zero is kept


@pytest.mark.parametrize("fmt", FMTS)
def test_exponent_at_its_limits(fmt):
    L = oc.LIMIT[fmt]
    for e in (-99, -3, 0, 40):
        assert oc.exponent(np.ldexp(L, e), fmt) == e
        assert oc.exponent(np.nextafter(np.ldexp(L, e), np.inf), fmt) == e + 1
    assert oc.exponent(0.0, fmt) == oc.E_MIN and oc.exponent(1e-40, fmt) == oc.E_MIN
    # the largest fp32 magnitudes: the exponent is held, the value saturates below infinity
    big = float(np.finfo(np.float32).max)
    codes, scales = oc.quantise(np.array([[big, -big]]), fmt)
    assert scales[0, 0] == 127 + oc.E_MAX[fmt]
    v = oc.dequantise(codes, scales, fmt)[0]
    assert v[0] == np.ldexp({"fp4": 6.0, "fp8": 448.0}[fmt], oc.E_MAX[fmt]) == -v[1]
    assert np.isfinite(np.float32(v[0]))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("k,D", [(1, 1), (8, 32), (9, 33), (13, 100), (16, 64)])
def test_slot_layout(fmt, k, D):
    assert sa.cache_slot_bytes(k, D, fmt) == oc.slot_bytes(k, D, fmt)
    G = -(-D // 32)
    at, sat = oc.places(k, D, fmt)
    # every code and scale byte has its own place, codes before scales, all in the slot
    assert len(np.unique(at)) == k * D and len(np.unique(sat)) == k * G
    codes = -(-k // 8) * G * 8 * 32 * oc.BITS[fmt] // 8
    assert at.max() * oc.BITS[fmt] // 8 < codes <= sat.min() and sat.max() < oc.slot_bytes(k, D, fmt)
    x = np.random.default_rng(k + D).standard_normal((k, D))
    n = max(1, k - 3)
    slot = np.random.default_rng(1).integers(0, 256, oc.slot_bytes(k, D, fmt)).astype(np.uint8)
    before = slot.copy()
    oc.pack(slot, x, n, fmt)
    c, s = oc.quantise(x[:n], fmt)
    np.testing.assert_array_equal(oc.unpack(slot, n, k, D, fmt)[:n], oc.dequantise(c, s, fmt))
    assert not oc.unpack(slot, n, k, D, fmt)[n:].any()
    # rows behind the last one are left as they were
    atp = oc.places(k, G * 32, fmt)[0]
    np.testing.assert_array_equal(slot[atp[n:] * oc.BITS[fmt] // 8], before[atp[n:] * oc.BITS[fmt] // 8])
    np.testing.assert_array_equal(slot[sat[n:]], before[sat[n:]])


def test_non_finite_groups_read_as_nan():
    x = np.ones((1, 96))
    x[0, 3], x[0, 40] = np.inf, np.nan
    c, s = oc.quantise(x, "fp4")
    v = oc.dequantise(c, s, "fp4")[0]
    assert np.isnan(v[:64]).all() and np.all(v[64:] == 1)


def test_cached_attention_is_stca_on_the_valid_rows():
    rng = np.random.default_rng(5)
    B, R, k, D, h = 3, 2, 9, 12, 3
    X, q = rng.standard_normal((B, k, D)), rng.standard_normal((B, R, D))
    W = [rng.standard_normal((D, D)) for _ in range(3)]
    dout = rng.standard_normal((B, R, D))
    out, lse = oc.stca_cached_fwd(X, [k, 0, 4], q, *W, h)
    full, flse = ostca.stca_fwd(X, q, *W, h)
    np.testing.assert_array_equal(out[0], full[0])
    assert not out[1].any() and np.all(lse[1] == -np.inf)
    np.testing.assert_array_equal(out[2], ostca.stca_fwd(X[2:, :4], q[2:], *W, h)[0][0])
    # the gradients against central differences of the masked forward
    g = oc.stca_cached_bwd(X, [k, 0, 4], q, *W, h, dout)
    assert not g["dq"][1].any()
    for i, name in enumerate(("dq", "dWq", "dWk", "dWv")):
        args = [q, *W]
        d = rng.standard_normal(args[i].shape)
        f = lambda t: np.sum(dout * oc.stca_cached_fwd(  # noqa: E731
            X, [k, 0, 4], *[a + (t * d if j == i else 0) for j, a in enumerate(args)], h)[0])
        num = (f(1e-5) - f(-1e-5)) / 2e-5
        assert abs(num - np.sum(g[name] * d)) <= 1e-6 * max(1.0, abs(num))


# ---------------------------------------------------------------- refusals (nothing is enqueued)

P = 1 << 12


def test_slot_bytes_of_invalid_sizes():
    L = sa.lib()
    for k, D, fmt in ((0, 64, 0), (4, 0, 0), (-1, 64, 0), (4, 64, 2), (1 << 20, 1 << 20, 0)):
        assert L.sa_cache_slot_bytes(k, D, fmt) == 0
    with pytest.raises(sa.SAError):
        sa.cache_slot_bytes(4, 64, "fp6")


def test_cache_write_and_read_reject_bad_arguments():
    L = sa.lib()
    w = dict(X=P, dt=0, slots=P, rows=None, B=2, k=8, D=64, fmt=0, cache=P, crows=P, n=4)

    def write(**kw):
        a = dict(w, **kw)
        return L.sa_cache_write(a["X"], a["dt"], a["slots"], a["rows"], a["B"], a["k"], a["D"], a["fmt"], a["cache"],
                                a["crows"], a["n"], None)

    def read(**kw):
        a = dict(w, **kw)
        return L.sa_cache_read(a["cache"], a["crows"], a["n"], a["slots"], a["B"], a["k"], a["D"], a["fmt"], a["X"],
                               a["dt"], None)
    for f in (write, read):
        for bad in (dict(X=None), dict(slots=None), dict(cache=None), dict(crows=None), dict(B=-1), dict(k=0),
                    dict(D=0), dict(n=-1), dict(fmt=2), dict(fmt=-1), dict(dt=5), dict(X=P + 4), dict(cache=P + 8),
                    dict(slots=P + 8), dict(crows=P + 4)):
            assert f(**bad) == 1, bad
            assert L.sa_last_error().decode() != ""
        assert f(k=1 << 16, D=1 << 16) == 2
        assert f(B=1 << 40) == 2
        assert f(B=0, X=None, slots=None, cache=None, crows=None) == 0
    assert write(n=0, cache=None, crows=None) == 0     # no slot to write
    assert write(rows=P + 4) == 1


def cached_call(fwd, **kw):
    L = sa.lib()
    a = dict(cache=P, crows=P, n=4, slots=P, fmt=1, q=P, Wq=P, Wk=P, Wv=P, B=2, R=3, k=64, D=128, h=2, scale=0.125,
             dt=0, out=P, odt=0, lse=None, dout=P, dq=P, dWq=P, dWk=P, dWv=P, ws=None, wsb=0)
    a.update(kw)
    head = [a[n] for n in ("cache", "crows", "n", "slots", "fmt", "q", "Wq", "Wk", "Wv", "B", "R", "k", "D", "h",
                           "scale", "dt")]
    if fwd:
        return L.sa_stca_cached_fwd(*head, a["out"], a["odt"], a["lse"], a["ws"], a["wsb"], None)
    return L.sa_stca_cached_bwd(*head, a["dout"], a["dq"], a["dWq"], a["dWk"], a["dWv"], a["odt"], a["ws"], a["wsb"],
                                None)


@pytest.mark.parametrize("fwd", [True, False])
def test_cached_stca_rejects_bad_arguments(fwd):
    outs = ("out",) if fwd else ("dout", "dq", "dWq", "dWk", "dWv")
    for name in ("cache", "crows", "slots", "q", "Wq", "Wk", "Wv") + outs:
        assert cached_call(fwd, **{name: None}) == 1, name
        assert cached_call(fwd, **{name: P + 4}) == 1, name
    for bad in (dict(R=0), dict(k=0), dict(D=0), dict(h=0), dict(h=3), dict(scale=0.0), dict(scale=float("nan")),
                dict(dt=7), dict(odt=7), dict(fmt=3), dict(n=-1), dict(B=-1)):
        assert cached_call(fwd, **bad) == 1, bad
    assert cached_call(fwd, dt=1, odt=0) == 2           # fp32 inputs, bf16 results
    assert cached_call(fwd, B=65536) == 2
    assert cached_call(fwd, B=0) == (0 if fwd else 1)
    assert cached_call(fwd) == 3
    size = sa.stca_cached_fwd_workspace_size if fwd else sa.stca_cached_bwd_workspace_size
    need = size(2, 3, 64, 128, 2, 0)
    assert need > 0
    assert cached_call(fwd, ws=P, wsb=need - 1) == 3
    assert cached_call(fwd, ws=P + 4, wsb=need) == 3
    assert size(2, 3, 64, 128, 3, 0) == 0 and size(2, 0, 64, 128, 2, 0) == 0


@pytest.mark.parametrize("fwd", [True, False])
def test_sizes_past_a_launch_are_refused(fwd):
    """a launch holds fewer than 2^32 threads"""
    L = sa.lib()
    io = (P, P, 1 << 20, P)
    assert L.sa_cache_read(*io, 1 << 24, 1, 32, 0, P, 0, None) == 2      # one workgroup a user
    assert L.sa_cache_write(P, 0, P, None, 1 << 24, 1, 32, 0, P, P, 1 << 20, None) == 2
    size = sa.stca_cached_fwd_workspace_size if fwd else sa.stca_cached_bwd_workspace_size
    assert cached_call(fwd, B=65535, R=256, h=8, k=1, D=8, dt=1, odt=1) == 2   # 2^27 rows of the softmax
    assert size(65535, 256, 1, 8, 8, 1) == 0 and size(65535, 64, 1, 8, 8, 1) > 0
    # bf16: workgroups of more rows instead
    assert size(65535, 300, 4, 1024, 16, 0) > 0


def test_binding_refuses_a_stream_of_another_device():
    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 0
    with pytest.raises(sa.SAError):
        sa._on(torch.device("cuda", 0), Stream())


def test_binding_refuses_what_is_not_a_cache():
    rows = torch.zeros(4, dtype=torch.int32)
    data = torch.zeros((4, sa.cache_slot_bytes(8, 64, "fp4")), dtype=torch.uint8)
    slots = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(sa.SAError):                     # not on a GPU
        sa.cache_read(sa.SketchCache(data, rows, 8, 64, "fp4"), slots)
    with pytest.raises(sa.SAError):
        sa.cache_read(sa.SketchCache(data, rows, 8, 64, "int4"), slots)
    with pytest.raises(sa.SAError):
        sa.sketch_cache(4, 0, 64, device="cpu")
    c = sa.sketch_cache(3, 8, 64, "fp8", device="cpu")
    assert c.data.shape == (3, oc.slot_bytes(8, 64, "fp8")) and not c.rows.any()
    assert isinstance(c.data.data_ptr(), int) and ctypes.sizeof(ctypes.c_void_p) == 8
