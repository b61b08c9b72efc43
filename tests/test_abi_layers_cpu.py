"""Host-side checks of the recent attention, layer norm and linear layers that need no GPU: bad
arguments are refused, by the C entry points and by the binding, before anything is enqueued."""
import ctypes
import struct

import pytest

from paper_2609_08443_amd import sa_sketch as sa

torch = pytest.importorskip("torch")

A = 1 << 12   # a pointer on 16 bytes that is never followed
NAN, INF = float("nan"), float("inf")
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


def recent(q=A, K=A, V=A, qs=(0, 0), ks=(0, 0), vs=(0, 0), offsets=A, targets=A, ends=0, slopes=0, B=2, T=10, N=3, h=2, hk=1,
           d=64, window=0, scale=0.125, cap=0.0, dtype=sa.SA_BF16):
    return sa._RECENT_ATTN.pack(q, K, V, *qs, *ks, *vs, offsets, targets, ends, slopes, B, T, N, h, hk, d, window, scale, cap, dtype)


BAD_RECENT = [
    (dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(N=-1), INVALID), (dict(h=0), INVALID), (dict(hk=0), INVALID),
    (dict(d=0), INVALID), (dict(window=-1), INVALID), (dict(h=3, hk=2), INVALID), (dict(h=1, hk=2), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID),
    (dict(cap=-1.0), INVALID), (dict(cap=NAN), INVALID), (dict(cap=INF), INVALID), (dict(dtype=7), INVALID),
    (dict(d=32), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(h=65537), UNSUPPORTED),
    (dict(T=1 << 31), UNSUPPORTED), (dict(N=1 << 31), UNSUPPORTED), (dict(N=1 << 30, h=2), UNSUPPORTED),
    (dict(B=(1 << 31) - 1), UNSUPPORTED), (dict(B=(1 << 31) - 3, T=1000), UNSUPPORTED),
    (dict(q=0), INVALID), (dict(K=0), INVALID), (dict(V=0), INVALID), (dict(offsets=0), INVALID), (dict(targets=0), INVALID),
    (dict(q=A + 8), INVALID), (dict(K=A + 2), INVALID), (dict(V=A + 4), INVALID), (dict(offsets=A + 8), INVALID),
    (dict(targets=A + 8), INVALID), (dict(ends=A + 4), INVALID), (dict(slopes=A + 4), INVALID),
    (dict(qs=(132, 64)), INVALID), (dict(ks=(128, 4)), INVALID), (dict(vs=(-128, 64)), INVALID), (dict(vs=(128, -64)), INVALID),
    (dict(scale=3e38), UNSUPPORTED), (dict(cap=3e38), UNSUPPORTED), (dict(cap=1e-39), UNSUPPORTED),
    (dict(ks=(1 << 24, 64)), UNSUPPORTED), (dict(qs=(128, 1 << 23)), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,code", BAD_RECENT)
def test_recent_attn_rejects_bad_arguments(kw, code):
    L = sa.lib()
    a = recent(**kw)
    grads = sa._RECENT_ATTN_GRADS.pack(A, A, A, 0, 0, 0, 0, 0, 0)
    assert L.sa_recent_attn_fwd(a, A, None, A, 1 << 40, None) == code
    assert L.sa_last_error().decode() != ""
    assert L.sa_recent_attn_bwd(a, A, A, A, grads, A, 1 << 40, None) == code
    assert L.sa_last_error().decode() != ""


def test_recent_attn_layout():
    """The binding's layout of the arguments is the compiler's."""
    class Args(ctypes.Structure):
        _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "K", "V")] + [(f"s{i}", ctypes.c_int64) for i in range(6)] +
                    [(n, ctypes.c_void_p) for n in ("offsets", "targets", "ends", "slopes")] +
                    [(n, ctypes.c_int64) for n in "BTN"] + [(n, ctypes.c_int32) for n in ("h", "hk", "d", "window")] +
                    [("scale", ctypes.c_float), ("cap", ctypes.c_float), ("dtype", ctypes.c_int)])
    assert ctypes.sizeof(Args) == sa._RECENT_ATTN.size
    a = Args.from_buffer_copy(recent(B=5, T=6, N=7, h=8, hk=4, d=64, window=9, scale=0.5, cap=0.25, dtype=sa.SA_FP32))
    assert (a.B, a.T, a.N, a.h, a.hk, a.d, a.window, a.scale, a.cap, a.dtype) == (5, 6, 7, 8, 4, 64, 9, 0.5, 0.25, sa.SA_FP32)
    assert sa._RECENT_ATTN_GRADS.size == 3 * struct.calcsize("P") + 6 * 8


def test_recent_attn_rejects_bad_outputs():
    L = sa.lib()
    a = recent()
    g = lambda *v: sa._RECENT_ATTN_GRADS.pack(*v)  # noqa: E731
    fine = g(A, A, A, 0, 0, 0, 0, 0, 0)
    assert L.sa_recent_attn_fwd(None, A, None, A, 1 << 40, None) == INVALID
    assert L.sa_recent_attn_fwd(a, None, None, A, 1 << 40, None) == INVALID
    assert L.sa_recent_attn_fwd(a, A + 8, None, A, 1 << 40, None) == INVALID
    assert L.sa_recent_attn_fwd(a, A, A + 4, A, 1 << 40, None) == INVALID
    for args in ((None, A, A, fine), (A, None, A, fine), (A, A, None, fine), (A, A, A, None), (A + 8, A, A, fine),
                 (A, A, A, g(0, A, A, 0, 0, 0, 0, 0, 0)), (A, A, A, g(A, 0, A, 0, 0, 0, 0, 0, 0)),
                 (A, A, A, g(A, A, A + 8, 0, 0, 0, 0, 0, 0)), (A, A, A, g(A, A, A, 4, 0, 0, 0, 0, 0)),
                 (A, A, A, g(A, A, A, -128, 0, 0, 0, 0, 0)),
                 # rows or heads on each other
                 (A, A, A, g(A, A, A, 64, 64, 0, 0, 0, 0)), (A, A, A, g(A, A, A, 128, 32, 0, 0, 0, 0)),
                 (A, A, A, g(A, A, A, 0, 0, 32, 64, 0, 0)), (A, A, A, g(A, A, A, 0, 0, 0, 0, 56, 64))):
        assert L.sa_recent_attn_bwd(a, *args, A, 1 << 40, None) == INVALID
        assert L.sa_last_error().decode() != ""
    need = L.sa_recent_attn_fwd_workspace_size(a)
    assert need > 0
    for ws, n in ((None, 1 << 40), (A, need - 1), (A + 8, 1 << 40)):
        assert L.sa_recent_attn_fwd(a, A, None, ws, n, None) == WORKSPACE
    need = L.sa_recent_attn_bwd_workspace_size(a)
    for ws, n in ((None, 1 << 40), (A, need - 1), (A + 8, 1 << 40)):
        assert L.sa_recent_attn_bwd(a, A, A, A, fine, ws, n, None) == WORKSPACE
    assert L.sa_recent_attn_fwd_workspace_size(recent(d=96)) == 0
    assert L.sa_recent_attn_fwd(recent(N=0, q=0), None, None, None, 0, None) == OK
    assert L.sa_recent_attn_bwd(recent(N=0, T=0, q=0, K=0, V=0), None, None, None, None, None, 0, None) == OK


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [sa.SA_BF16, sa.SA_FP32])
def test_recent_attn_workspace_goes_by_sizes_alone(dtype, d):
    """As large for any ends, window, scale and strides; little against K and V."""
    L = sa.lib()
    for B, T, N, h, hk in ((1, 1, 1, 1, 1), (100, 80000, 4000, 8, 2), (1, 10000, 1, 16, 16), (4000, 8000, 4000, 2, 1)):
        base = dict(B=B, T=T, N=N, h=h, hk=hk, d=d, dtype=dtype)
        for size in (L.sa_recent_attn_fwd_workspace_size, L.sa_recent_attn_bwd_workspace_size):
            n = size(recent(**base))
            assert n > 0
            for kw in (dict(ends=A), dict(slopes=A, window=5, cap=2.0), dict(scale=2.0), dict(ks=(4096, 64), qs=(8192, 128))):
                assert size(recent(**base, **kw)) == n


def norm_fwd(x=A, ld=0, gamma=A, beta=A, N=3, D=64, eps=1e-5, dtype=sa.SA_BF16, y=A, stats=A):
    return sa.lib().sa_layer_norm_fwd(x, ld, gamma, beta, N, D, eps, dtype, y, stats, None)


def norm_bwd(x=A, ld=0, gamma=A, stats=A, dy=A, N=3, D=64, dtype=sa.SA_BF16, dx=A, dgamma=A, dbeta=A, ws=A, wsb=1 << 40):
    return sa.lib().sa_layer_norm_bwd(x, ld, gamma, stats, dy, N, D, dtype, dx, dgamma, dbeta, ws, wsb, None)


NORM_SIZES = [(dict(N=-1), INVALID), (dict(D=0), INVALID), (dict(dtype=5), INVALID), (dict(ld=-1), INVALID),
              (dict(D=(1 << 24) + 1), UNSUPPORTED), (dict(N=1 << 40), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", NORM_SIZES + [
    (dict(eps=-1e-9), INVALID), (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID), (dict(x=None), INVALID),
    (dict(gamma=None), INVALID), (dict(beta=None), INVALID), (dict(y=None), INVALID), (dict(x=A + 1), INVALID),
    (dict(y=A + 2, dtype=sa.SA_FP32), INVALID), (dict(stats=A + 4), INVALID)])
def test_layer_norm_fwd_rejects_bad_arguments(kw, code):
    assert norm_fwd(**kw) == code and sa.lib().sa_last_error().decode() != ""


@pytest.mark.parametrize("kw,code", NORM_SIZES + [
    (dict(x=None), INVALID), (dict(gamma=None), INVALID), (dict(stats=None), INVALID), (dict(dy=None), INVALID),
    (dict(dx=None), INVALID), (dict(dgamma=None), INVALID), (dict(dbeta=None), INVALID), (dict(dy=A + 1), INVALID),
    (dict(stats=A + 4), INVALID), (dict(dgamma=A + 2), INVALID), (dict(ws=None), WORKSPACE), (dict(wsb=1), WORKSPACE),
    (dict(ws=A + 8), WORKSPACE), (dict(N=0, dgamma=None), INVALID)])
def test_layer_norm_bwd_rejects_bad_arguments(kw, code):
    assert norm_bwd(**kw) == code and sa.lib().sa_last_error().decode() != ""


def linear_fwd(x=A, ld=0, W=2 * A, bias=None, residual=None, N=3, K=64, F=64, act=0, dtype=sa.SA_BF16, y=3 * A, pre=None, ws=A,
               wsb=1 << 50):
    return sa.lib().sa_linear_fwd(x, ld, W, bias, residual, N, K, F, act, dtype, y, pre, ws, wsb, None)


def linear_bwd(x=A, ld=0, W=2 * A, pre=3 * A, dy=4 * A, N=3, K=64, F=64, act=0, dtype=sa.SA_BF16, dx=5 * A, dW=6 * A, db=A, wdt=sa.SA_FP32, ws=A,
               wsb=1 << 50):
    return sa.lib().sa_linear_bwd(x, ld, W, pre, dy, N, K, F, act, dtype, dx, dW, db, wdt, ws, wsb, None)


LINEAR_SIZES = [(dict(N=-1), INVALID), (dict(K=0), INVALID), (dict(F=0), INVALID), (dict(act=5), INVALID), (dict(act=-1), INVALID),
                (dict(dtype=9), INVALID), (dict(ld=-8), INVALID), (dict(N=1 << 29), UNSUPPORTED), (dict(K=(1 << 20) + 1), UNSUPPORTED),
                (dict(F=(1 << 19) + 1, act=4), UNSUPPORTED), (dict(K=1 << 20, F=1 << 11), UNSUPPORTED),
                (dict(N=1 << 28, F=256), UNSUPPORTED), (dict(F=0x7fffffff, act=4), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", LINEAR_SIZES + [
    (dict(x=None), INVALID), (dict(W=None), INVALID), (dict(y=None), INVALID), (dict(x=A + 2), INVALID), (dict(W=A + 8), INVALID),
    (dict(y=A), INVALID), (dict(y=2 * A), INVALID), (dict(pre=3 * A), INVALID), (dict(pre=A), INVALID),
    (dict(bias=A + 2), INVALID), (dict(residual=A + 8), INVALID), (dict(y=A + 4), INVALID), (dict(pre=A + 4), INVALID),
    (dict(K=63, ws=None), WORKSPACE), (dict(K=63, wsb=1), WORKSPACE), (dict(K=63, ws=A + 8), WORKSPACE)])
def test_linear_fwd_rejects_bad_arguments(kw, code):
    assert linear_fwd(**kw) == code and sa.lib().sa_last_error().decode() != ""


@pytest.mark.parametrize("kw,code", LINEAR_SIZES + [
    (dict(x=None), INVALID), (dict(W=None), INVALID), (dict(dy=None), INVALID), (dict(act=1, pre=None), INVALID),
    (dict(dx=A), INVALID), (dict(dx=2 * A), INVALID), (dict(dx=3 * A), INVALID), (dict(dx=4 * A), INVALID),
    (dict(dx=A + 8), INVALID), (dict(dW=A + 4), INVALID), (dict(db=A + 4), INVALID), (dict(pre=A + 2, act=2), INVALID),
    (dict(wdt=4), INVALID), (dict(dtype=sa.SA_FP32, wdt=sa.SA_BF16), UNSUPPORTED), (dict(ws=None), WORKSPACE),
    (dict(wsb=1), WORKSPACE), (dict(ws=A + 8), WORKSPACE)])
def test_linear_bwd_rejects_bad_arguments(kw, code):
    assert linear_bwd(**kw) == code and sa.lib().sa_last_error().decode() != ""


def test_no_rows_need_nothing():
    assert norm_fwd(N=0, x=None, y=None) == OK
    assert linear_fwd(N=0, x=None, y=None, ws=None, wsb=0) == OK
    assert sa.lib().sa_linear_fwd_workspace_size(0, 63, 64, 0, sa.SA_BF16, 0) == 0


@pytest.fixture
def any_device(monkeypatch):
    """The binding's checks of tensors, on the CPU: what they let through would stop at the device."""
    monkeypatch.setattr(sa, "_gpu_code", lambda t, name: (sa._dtype_code(t), t.device))

    def stop(*args):
        raise AssertionError("not refused")
    monkeypatch.setattr(sa, "_on", stop)


def batch():
    kv = torch.zeros(10, 2, 2, 64)
    o = torch.tensor([0, 6, 10])
    return dict(q=torch.zeros(3, 4, 64), K=kv[:, 0], V=kv[:, 1], offsets=o, targets=torch.tensor([0, 1, 3]))


def test_good_tensors_reach_the_device(any_device):
    with pytest.raises(AssertionError):
        sa.recent_attn_fwd(**batch())
    with pytest.raises(AssertionError):
        sa.linear_fwd(torch.zeros(3, 8), torch.zeros(8, 4))
    with pytest.raises(AssertionError):
        sa.layer_norm_fwd(torch.zeros(3, 8), torch.zeros(8), torch.zeros(8))


z = torch.zeros


@pytest.mark.parametrize("kw", [
    dict(q=z(3, 256)), dict(q=z(3, 4, 64).half()), dict(q=z(3, 4, 64).transpose(1, 2).contiguous().transpose(1, 2)),
    dict(q=z(1, 4, 64).expand(3, 4, 64)), dict(q=z(3, 1, 64).expand(3, 4, 64)), dict(K=z(1, 2, 64).expand(10, 2, 64)),
    dict(V=z(10, 1, 64).expand(10, 2, 64)), dict(V=z(10, 2, 64, dtype=torch.bfloat16)), dict(V=z(9, 2, 64)), dict(K=z(10, 128)),
    dict(offsets=torch.tensor([0, 6, 10], dtype=torch.int32)), dict(offsets=z(0, dtype=torch.int64)), dict(targets=torch.tensor([0, 3])),
    dict(targets=torch.tensor([[0, 1, 3]])), dict(ends=z(3, dtype=torch.int64)), dict(ends=z(4, dtype=torch.int32)),
    dict(slopes=z(3)), dict(slopes=z(4, dtype=torch.float64)), dict(window=1 << 31), dict(window=1.5), dict(scale="x"),
    dict(window=-(1 << 40)), dict(cap=None)])
def test_binding_refuses_recent_attn(any_device, kw):
    with pytest.raises(sa.SAError):
        sa.recent_attn_fwd(**{**batch(), **kw})


@pytest.mark.parametrize("kw", [dict(out=z(3, 4, 32)), dict(lse=z(4, 3)), dict(dout=z(3, 4, 64, dtype=torch.bfloat16)),
                                dict(dout=z(1, 4, 64).expand(3, 4, 64)), dict(lse=z(3, 4, dtype=torch.float64))])
def test_binding_refuses_recent_attn_bwd(any_device, kw):
    args = dict(batch(), out=z(3, 4, 64), lse=z(3, 4), dout=z(3, 4, 64))
    with pytest.raises(sa.SAError):
        sa.recent_attn_bwd(**{**args, **kw})


@pytest.mark.parametrize("args,kw", [
    ((z(1, 8).expand(3, 8), z(8, 4)), {}), ((z(3, 8).t(), z(3, 4)), {}), ((z(3, 8), z(4, 8)), {}), ((z(3, 8), z(4, 8).t()), {}),
    ((z(3, 8), z(8, 5)), dict(act="swiglu")), ((z(3, 8), z(8, 4)), dict(act="tanh")), ((z(3, 8), z(8, 4)), dict(bias=z(5))),
    ((z(3, 8), z(8, 4)), dict(residual=z(3, 8))), ((z(3, 2, 8), z(8, 4)), {}), ((z(3, 8).double(), z(8, 4).double()), {})])
def test_binding_refuses_linear(any_device, args, kw):
    with pytest.raises(sa.SAError):
        sa.linear_fwd(*args, **kw)


@pytest.mark.parametrize("kw", [dict(act="relu"), dict(dy=z(3, 5)), dict(act="gelu", pre=z(4, 4)), dict(dy=z(1, 4).expand(3, 4))])
def test_binding_refuses_linear_bwd(any_device, kw):
    with pytest.raises(sa.SAError):
        sa.linear_bwd(**{**dict(x=z(3, 8), W=z(8, 4), dy=z(3, 4)), **kw})


@pytest.mark.parametrize("args", [(z(8), z(8), z(8)), (z(3, 8), z(7), z(8)), (z(3, 8), z(8), z(8, dtype=torch.bfloat16)),
                                  (z(1, 8).expand(3, 8), z(8), z(8)), (z(3, 16)[:, ::2], z(8), z(8))])
def test_binding_refuses_layer_norm(any_device, args):
    with pytest.raises(sa.SAError):
        sa.layer_norm_fwd(*args)


def test_tensors_off_the_gpu_are_refused():
    b = batch()
    for call in (lambda: sa.recent_attn_fwd(**b), lambda: sa.linear_fwd(z(3, 8), z(8, 4)), lambda: sa.layer_norm_fwd(z(3, 8), z(8), z(8)),
                 lambda: sa.recent_attn_bwd(**b, out=z(3, 4, 64), lse=z(3, 4), dout=z(3, 4, 64)),
                 lambda: sa.linear_bwd(z(3, 8), z(8, 4), z(3, 4)), lambda: sa.layer_norm_bwd(z(3, 8), z(8), z(3, 2), z(3, 8))):
        with pytest.raises(sa.SAError, match="expected a GPU"):
            call()
