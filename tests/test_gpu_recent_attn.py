"""GPU tests of the attention over recent histories (sa_recent_attn_fwd, sa_recent_attn_bwd)
against the fp64 oracle, element by element within the bounds that oracle/recent.py derives."""
import numpy as np
import pytest

from oracle import recent as orec

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


def csr(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)


class Batch:
    """Seeded inputs: host fp64 values that the dtype holds, and their device tensors."""

    def __init__(self, tokens, targets, h, hk, d, dtype, ends=None, window=0, cap=0.0, slopes=False, seed=0, packed=True,
                 tail=(0, 0), scale=None):
        g = np.random.default_rng([8443, seed, h, hk, d, sum(tokens), sum(targets)])
        self.off, self.tgt = csr(tokens), csr(targets)
        T, N = int(self.off[-1]) + tail[0], int(self.tgt[-1]) + tail[1]
        val = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).to(DT[dtype])  # noqa: E731
        self.q, self.dout = val(N, h, d), val(N, h, d)
        kv = val(T, 2, hk, d)
        self.K, self.V = kv[:, 0], kv[:, 1]
        self.kv = kv.cuda()
        self.dtype, self.packed = dtype, packed
        self.ends = None
        if ends == "random":
            n = np.repeat(tokens, targets)
            self.ends = np.floor(g.random(N) * (np.concatenate([n, np.zeros(tail[1])]) + 1)).astype(np.int32)
        elif ends is not None:
            self.ends = np.asarray(ends, np.int32)
        self.slopes = 2.0 ** (-8.0 * np.arange(1, h + 1) / h) if slopes else None
        self.kw = dict(window=window, cap=cap)
        if scale is not None:
            self.kw["scale"] = scale
        if self.slopes is not None:
            self.slopes = self.slopes.astype(np.float32)

    def device(self):
        c = lambda x: None if x is None else (torch.from_numpy(x) if isinstance(x, np.ndarray) else x).cuda()  # noqa: E731
        K, V = (self.kv[:, 0], self.kv[:, 1]) if self.packed else (self.kv[:, 0].contiguous(), self.kv[:, 1].contiguous())
        return (c(self.q), K, V, c(self.off), c(self.tgt)), dict(ends=c(self.ends), slopes=c(self.slopes), **self.kw)

    def oracle(self):
        n = lambda x: x.double().numpy()  # noqa: E731
        return (n(self.q), n(self.K), n(self.V), self.off, self.tgt), dict(ends=self.ends, slopes=self.slopes, dtype=self.dtype,
                                                                          **self.kw)


def within(got, ref, off, what):
    got = got.detach().double().cpu().numpy()
    assert np.array_equal(np.isneginf(got), np.isneginf(ref)), what
    fin = np.isfinite(ref)
    assert np.all(np.isfinite(got[fin])), f"{what}: not finite"
    worst = np.max(np.abs(got[fin] - ref[fin]) / np.maximum(off[fin], 1e-30), initial=0.0)
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound"


def check_fwd(sa, b):
    args, kw = b.device()
    out, lse = sa.recent_attn_fwd(*args, **kw)
    oargs, okw = b.oracle()
    ro, rl, eo, el = orec.fwd(*oargs, **okw)
    assert out.dtype == DT[b.dtype] and lse.dtype == torch.float32
    within(out, ro, eo, "out")
    within(lse, rl, el, "lse")
    return out, lse


def check_bwd(sa, b):
    args, kw = b.device()
    oargs, okw = b.oracle()
    ro, rl, _, _ = orec.fwd(*oargs, **okw)
    out = torch.from_numpy(ro).to(DT[b.dtype]).cuda()
    lse = torch.from_numpy(rl.astype(np.float32)).cuda()
    got = sa.recent_attn_bwd(*args, out, lse, b.dout.cuda(), **kw)
    ref, off = orec.bwd(*oargs, b.dout.double().numpy(), **okw)
    assert set(got) == {"dq", "dK", "dV"}
    for k in got:
        assert got[k].dtype == DT[b.dtype]
        within(got[k], ref[k], off[k], k)
    return got


CASES = {
    # one token, one target
    "one": dict(tokens=[1], targets=[1], h=1, hk=1),
    # users without tokens, without targets, without both
    "holes": dict(tokens=[0, 5, 0, 33, 7, 0], targets=[3, 0, 0, 2, 1, 4], h=2, hk=2),
    # single targets over histories around the unit of 128 keys
    "single": dict(tokens=[127, 128, 129, 1, 31, 32, 33, 700], targets=[1] * 8, h=4, hk=4),
    # shared heads: rows of a target side by side
    "shared": dict(tokens=[100, 65, 3], targets=[1, 9, 2], h=8, hk=2),
    "shared_by_three": dict(tokens=[200, 64], targets=[5, 50], h=6, hk=2),
    "one_key_head": dict(tokens=[90, 300], targets=[7, 3], h=9, hk=1),
    # many targets: tiles of 128 rows and their ends
    "many": dict(tokens=[64, 300, 10], targets=[127, 129, 256], h=2, hk=2),
    "many_shared": dict(tokens=[257], targets=[150], h=6, hk=2),
    # a long user among short ones, cut by many pieces
    "long": dict(tokens=[3, 5000, 17], targets=[2, 1, 1], h=2, hk=1),
    "long_many": dict(tokens=[2500, 40], targets=[70, 100], h=2, hk=2),
    # what a target sees
    "ends": dict(tokens=[50, 200, 0, 129], targets=[9, 40, 3, 60], h=2, hk=2, ends="random"),
    "ends_single": dict(tokens=[50, 200, 128, 600], targets=[1, 2, 1, 3], h=4, hk=2, ends="random"),
    "window": dict(tokens=[50, 400], targets=[9, 70], h=2, hk=2, ends="random", window=37),
    "window_alone": dict(tokens=[50, 400, 64], targets=[1, 2, 1], h=2, hk=2, window=64),
    "cap": dict(tokens=[77, 140], targets=[5, 64], h=2, hk=1, cap=2.0),
    "bias": dict(tokens=[77, 340], targets=[5, 3], h=4, hk=2, slopes=True),
    "all": dict(tokens=[77, 340, 0, 10], targets=[5, 33, 2, 90], h=4, hk=2, slopes=True, cap=3.0, ends="random", window=90),
    "apart": dict(tokens=[30, 70], targets=[3, 60], h=4, hk=2, packed=False),
    # rows and tokens behind the last user's
    "tail": dict(tokens=[30, 70], targets=[3, 60], h=2, hk=2, tail=(37, 150)),
    "tail_single": dict(tokens=[30, 70], targets=[1, 1], h=2, hk=2, tail=(200, 5)),
    # rows around what one pass over the keys takes (64, or 32 at d = 128), beside users with more; several chunks
    "few_rows": dict(tokens=[700, 31, 1500, 256, 4], targets=[32, 33, 64, 63, 1], h=1, hk=1, ends="random"),
    "few_and_many": dict(tokens=[513, 2100, 65, 0, 300], targets=[65, 3, 200, 5, 0], h=2, hk=2, ends="random"),
    "few_shared": dict(tokens=[600, 1030], targets=[8, 9], h=8, hk=2, cap=5.0, window=300),
    "chunks": dict(tokens=[255, 256, 257, 3000, 1, 511, 513], targets=[2, 1, 2, 40, 1, 3, 1], h=2, hk=1),
    # no user at all
    "no_users": dict(tokens=[], targets=[], h=2, hk=2, tail=(5, 3)),
    "ends_out_of_range": dict(tokens=[20, 9], targets=[3, 2], h=1, hk=1, ends=[-5, 21, 2 ** 31 - 1, 0, 9]),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_forward(sa, dtype, d, name):
    print(f"fwd {name} d={d} {dtype}", flush=True)
    check_fwd(sa, Batch(d=d, dtype=dtype, **CASES[name]))


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_backward(sa, dtype, d, name):
    print(f"bwd {name} d={d} {dtype}", flush=True)
    check_bwd(sa, Batch(d=d, dtype=dtype, **CASES[name]))


# ---------------------------------------------------------------- what is no number stays with those who see it

BAD = [float("nan"), float("inf"), float("-inf")]


def spoilt(b, where, at, value):
    """The batch with one value of K, V, q or dout set."""
    t = {"K": b.K, "V": b.V, "q": b.q, "dout": b.dout}[where]
    t[at] = value
    if where in "KV":
        b.kv = torch.stack([b.K, b.V], 1).cuda()
    return b


@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("targets", [[3, 5], [150, 40]])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("where", ["K", "V"])
def test_forward_of_tokens_that_are_no_numbers(sa, where, dtype, targets, cap):
    """Targets whose window leaves such a token out, and other users, have the results that they have without it."""
    case = dict(tokens=[300, 70], targets=targets, h=4, hk=2, d=64, dtype=dtype, ends="random", window=200, cap=cap)
    good = Batch(**case)
    args, kw = good.device()
    ref, rlse = sa.recent_attn_fwd(*args, **kw)
    user = np.repeat([0, 1], targets)
    for value in BAD:
        for token in (0, 31, 150, 299):
            b = spoilt(Batch(**case), where, (token, 1, 5), value)
            args, kw = b.device()
            out, lse = sa.recent_attn_fwd(*args, **kw)
            e = np.minimum(b.ends, np.array([300, 70])[user])
            sees = (user == 0) & (token < e) & (token >= np.maximum(0, e - 200))
            clean = torch.from_numpy(~sees).cuda()
            assert torch.equal(out[clean], ref[clean]) and torch.equal(lse[clean], rlse[clean]), (value, token)
            assert torch.equal(out[:, :2], ref[:, :2])          # the heads that read key head 0
            if where == "V" and sees.any():
                hit = out[~clean][:, 2:]
                assert not torch.isfinite(hit[:, :, 5]).any(), (value, token)
                rest = [d for d in range(64) if d != 5]
                assert torch.equal(hit[:, :, rest], ref[~clean][:, 2:][:, :, rest])


@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("targets", [[3, 5], [150, 40]])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("where", ["K", "V", "q", "dout"])
def test_backward_of_what_is_no_number(sa, where, dtype, targets, cap):
    """Gradients of targets and tokens that have nothing to do with it are as they are without it."""
    case = dict(tokens=[300, 70], targets=targets, h=4, hk=2, d=64, dtype=dtype, ends="random", window=200, cap=cap)
    user = np.repeat([0, 1], targets)

    def grads(b):
        args, kw = b.device()
        out, lse = sa.recent_attn_fwd(*args, **kw)
        return sa.recent_attn_bwd(*args, out, lse, b.dout.cuda(), **kw)

    ref = grads(Batch(**case))
    tok_user = np.repeat([0, 1], [300, 70])
    for value in BAD:
        for at in (0, 2):
            b = Batch(**case)
            e = np.minimum(b.ends, np.array([300, 70])[user])
            lo = np.maximum(0, e - 200)
            if where in "KV":
                token = (0, 31, 250)[at]
                g = grads(spoilt(b, where, (token, 1, 5), value))
                rows = (user == 0) & (token < e) & (token >= lo)      # targets that see the token
            else:
                g = grads(spoilt(b, where, (at, 3, 5), value))        # query head 3 of one target
                rows = np.arange(len(user)) == at
            # tokens that such a target sees
            j = np.concatenate([np.arange(300), np.arange(70)])
            toks = np.array([any(user[i] == tok_user[t] and lo[i] <= j[t] < e[i] for i in np.flatnonzero(rows))
                             for t in range(370)])
            if where in "KV":
                toks[token] = True
            rows, toks = torch.from_numpy(rows).cuda(), torch.from_numpy(toks).cuda()
            assert torch.equal(g["dq"][~rows], ref["dq"][~rows]), (value, at)
            assert torch.equal(g["dK"][~toks], ref["dK"][~toks]), (value, at)
            assert torch.equal(g["dV"][~toks], ref["dV"][~toks]), (value, at)
            assert torch.equal(g["dK"][:, 0], ref["dK"][:, 0]) and torch.equal(g["dV"][:, 0], ref["dV"][:, 0])


@pytest.mark.parametrize("targets", [[3, 5], [150, 40]])
def test_padding_that_is_no_number(sa, targets):
    """Targets that see nothing and rows and tokens behind the last user's may hold anything."""
    case = dict(tokens=[300, 70], targets=targets, h=4, hk=2, d=64, dtype="bf16", ends="random", tail=(33, 20))

    def run(fill):
        b = Batch(**case)
        n = sum(targets)
        b.ends[1] = 0
        for t in (b.q, b.dout):
            t[1] = fill
            t[n:] = fill
        b.K[370:] = fill
        b.V[370:] = fill
        b.kv = torch.stack([b.K, b.V], 1).cuda()
        args, kw = b.device()
        out, lse = sa.recent_attn_fwd(*args, **kw)
        return out, lse, sa.recent_attn_bwd(*args, out, lse, b.dout.cuda(), **kw)

    out, lse, g = run(1.0)
    for fill in BAD:
        o, l, h = run(fill)
        assert torch.equal(o, out) and torch.equal(l, lse)
        for k in g:
            assert torch.equal(h[k], g[k]), k
    n = sum(targets)
    assert not out[n:].any() and torch.isneginf(lse[n:]).all() and not g["dq"][n:].any()
    assert not g["dK"][370:].any() and not g["dV"][370:].any()
