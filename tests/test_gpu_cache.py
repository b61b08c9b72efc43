"""GPU tests of the sketch cache (sa_cache_write, sa_cache_read) and of the attention
over it (sa_stca_cached_fwd, sa_stca_cached_bwd) against the fp64 oracle.

Tolerances.  What is written and read back is exact, byte for byte.  The attention's
results are compared by 2-norm, per user (outputs, dq) or whole (weights).  A rounding
to bf16 is off by at most 2^-8 of the value (finfo.eps / 2), so independent ones of n
quantities in a chain add up to at most sqrt(n) 2^-8: five in the forward (q W_Q, u,
the weights, the aggregates, a bf16 result), eight in the gradients (those of the
forward that they contain, dout, dc, ds, du, dp, the result).  fp32 mode: a sum of N
terms in any order is off by about sqrt(N) 2^-24 of its terms' norm; the chain has four
sums of D, two of k and, for the weights, one of B R: the bound is twice their total.
lse: fp32 as the outputs, absolute; bf16 mode moves a logit by the two roundings before
it, 2 * 2^-8 of sum |scale u X| at most, about 3 of whose standard deviations (2^-8 |s|
sqrt(2 / 3)) bound it over a few thousand logits: 2^-6 max |s|.
"""
import numpy as np
import pytest

from oracle import cache as oc

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


def rng_of(*key):
    return np.random.default_rng([8443, *key])


def as_dtype(x, dtype):
    """fp32 values that the dtype represents."""
    t = torch.from_numpy(np.asarray(x, np.float32))
    return t.to(DT[dtype])


def raw_cache(sa, n_slots, k, D, fmt, seed=0):
    """A cache whose unwritten bytes are random (NaN codes and scales among them)."""
    g = rng_of(seed, 77)
    c = sa.sketch_cache(n_slots, k, D, fmt)
    c.data.copy_(torch.from_numpy(g.integers(0, 256, tuple(c.data.shape)).astype(np.uint8)))
    return c


def same(a, b):
    """Equal, NaN in the same places."""
    np.testing.assert_array_equal(np.asarray(a, np.float64), np.asarray(b, np.float64))


# ---------------------------------------------------------------- writing and reading

IO_CASES = [  # k, D, rows of the users, slots
    (1, 1, [1], [0]),
    (8, 32, [8, 8], [1, 0]),
    (9, 33, [9, 0, 5], [2, 0, 3]),
    (16, 64, [16, 3], [3, 1]),
    (33, 100, [33, 17, 1, 40], [4, 0, 2, 1]),          # rows above k count as k
    (70, 320, [70, 64, 13], [1, -1, 5]),               # no slot; a slot outside the cache
    (130, 72, [100, 130], [2, 0]),
    (5, 1030, [5, 4], [0, 1]),
]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("k,D,rows,slots", IO_CASES)
def test_write_and_read_are_exact(sa, fmt, dtype, k, D, rows, slots):
    print(f"io k={k} D={D} {fmt} {dtype}", flush=True)
    g = rng_of(k, D)
    B = len(rows)
    x = g.standard_normal((B, k, D)) * np.exp(3 * g.standard_normal((B, k, 1)))
    x[0, 0, : D // 2] = 0.0
    t = as_dtype(x, dtype)
    n_slots = 5
    c = raw_cache(sa, n_slots, k, D, fmt)
    want = c.data.cpu().numpy().copy()
    counts = np.zeros(n_slots, np.int32)
    for b in range(B):
        if 0 <= slots[b] < n_slots:
            counts[slots[b]] = min(max(rows[b], 0), k)
            oc.pack(want[slots[b]], t[b].double().numpy(), counts[slots[b]], fmt)
    s = torch.tensor(slots, device="cuda")
    sa.cache_write(c, t.cuda(), s, torch.tensor(rows, dtype=torch.int32, device="cuda"))
    got = sa.cache_read(c, s, dtype=DT[dtype])
    got32 = sa.cache_read(c, s, dtype=torch.float32)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(c.rows.cpu().numpy(), counts)
    np.testing.assert_array_equal(c.data.cpu().numpy(), want)
    for b in range(B):
        hit = 0 <= slots[b] < n_slots
        ref = oc.unpack(want[slots[b]], counts[slots[b]], k, D, fmt) if hit else np.zeros((k, D))
        same(got[b].double().cpu().numpy(), ref)
        same(got32[b].cpu().numpy(), ref)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_every_magnitude_rounds_as_defined(sa, fmt):
    """Values around every rounding border, at exponents over the whole range, and the
    values that no exponent reaches."""
    top = oc.LIMIT[fmt]
    mags = oc.magnitudes(fmt)
    mid = (mags[1:] + mags[:-1]) / 2
    v = np.concatenate([mags, mid, np.nextafter(mid.astype(np.float32), 0), np.nextafter(mid.astype(np.float32), 9e9)])
    v = np.concatenate([v, -v])
    rows = [np.append(p, top) for p in np.array_split(v, -(-v.size // 31))]      # each group's largest is L: e as given
    rows = np.stack([np.pad(p, (0, 32 - p.size)) for p in rows])
    x = np.concatenate([np.ldexp(rows, e) for e in (-101, -100, -3, 0, 60, 115)]).astype(np.float32)
    big = np.finfo(np.float32).max
    odd = np.zeros((6, 32), np.float32)
    odd[0, :3] = [big, -big, 1.0]
    odd[1, :3] = [1e-38, 1e-45, -1e-45]
    odd[2, 5], odd[3, 31], odd[4, 0] = np.inf, np.nan, -np.inf
    x = np.concatenate([x, odd])
    t = torch.from_numpy(x)[None]
    c = raw_cache(sa, 1, x.shape[0], 32, fmt)
    s = torch.zeros(1, dtype=torch.int64, device="cuda")
    sa.cache_write(c, t.cuda(), s)
    codes, scales = oc.quantise(x, fmt)
    same(sa.cache_read(c, s, dtype=torch.float32)[0].cpu().numpy(), oc.dequantise(codes, scales, fmt))
    want = np.zeros(c.data.shape[1], np.uint8)
    oc.pack(want, x.astype(np.float64), x.shape[0], fmt)
    used = oc.places(x.shape[0], 32, fmt)[1].max() + 1
    if x.shape[0] % 8 == 0:
        np.testing.assert_array_equal(c.data[0, :used].cpu().numpy(), want[:used])


@pytest.mark.parametrize("B", [2, 40, 1025, 3000])
def test_of_two_users_with_one_slot_the_last_is_kept(sa, B):
    k, D, n_slots = 3, 40, 7
    g = rng_of(B)
    slots = g.integers(-1, n_slots, B)
    slots[-2:] = 2
    rows = g.integers(0, k + 1, B)
    t = as_dtype(g.standard_normal((B, k, D)), "fp32")
    c = raw_cache(sa, n_slots, k, D, "fp8", B)
    want, counts = c.data.cpu().numpy().copy(), np.zeros(n_slots, np.int32)
    for b in range(B):
        if slots[b] >= 0 and not np.any(slots[b + 1:] == slots[b]):
            counts[slots[b]] = rows[b]
            oc.pack(want[slots[b]], t[b].double().numpy(), rows[b], "fp8")
    for _ in range(2):
        sa.cache_write(c, t.cuda(), torch.from_numpy(slots).cuda(), torch.from_numpy(rows.astype(np.int32)).cuda())
        np.testing.assert_array_equal(c.data.cpu().numpy(), want)
        np.testing.assert_array_equal(c.rows.cpu().numpy(), counts)


def test_slots_beyond_four_gigabytes(sa):
    """Slot offsets past 32 bits: a cache of 5 GB, its first and last slots."""
    k, D = 512, 1024
    n_slots = 5_000_000_000 // sa.cache_slot_bytes(k, D, "fp8")
    c = sa.sketch_cache(n_slots, k, D, "fp8")
    assert c.data.numel() > 1 << 32
    t = torch.randn((2, k, D), device="cuda")
    s = torch.tensor([n_slots - 1, 0], device="cuda")
    sa.cache_write(c, t, s)
    got = sa.cache_read(c, s, dtype=torch.float32)
    small = sa.sketch_cache(2, k, D, "fp8")
    sa.cache_write(small, t, torch.tensor([0, 1], device="cuda"))
    assert torch.equal(got, sa.cache_read(small, torch.tensor([0, 1], device="cuda"), dtype=torch.float32))
    q = torch.randn((2, 3, D), device="cuda").bfloat16()
    w = [(torch.randn((D, D), device="cuda") / 32).bfloat16() for _ in range(3)]
    out, _ = sa.stca_cached_fwd(c, s, q, *w, 16)
    assert torch.equal(out, sa.stca_cached_fwd(small, torch.tensor([0, 1], device="cuda"), q, *w, 16)[0])


# ---------------------------------------------------------------- attention over the cache


def problem(sa, B, R, k, D, h, fmt, dtype, rows, slots, seed=0, sharp=1.0):
    """A cache with written slots and stale bytes, targets and weights, and the oracle's
    inputs: the values of the valid rows."""
    g = rng_of(B, R, k, D, seed)
    n_slots = max(slots) + 2
    c = raw_cache(sa, n_slots, k, D, fmt, seed)
    host = c.data.cpu().numpy().copy()
    counts = np.zeros(n_slots, np.int32)
    for s, n in dict(zip(slots, rows)).items():
        if s >= 0:
            # (packed by the oracle: these tests stand apart from the write)
            oc.pack(host[s], g.standard_normal((k, D)), n, fmt)
            counts[s] = n
    c.data.copy_(torch.from_numpy(host))
    c.rows.copy_(torch.from_numpy(counts))
    n = [int(counts[s]) if s >= 0 else 0 for s in slots]
    X = np.stack([oc.unpack(host[max(s, 0)], m, k, D, fmt) for s, m in zip(slots, n)])
    q = as_dtype(g.standard_normal((B, R, D)) * sharp, dtype)
    W = [as_dtype(g.standard_normal((D, D)) / np.sqrt(D), dtype) for _ in range(3)]
    dout = as_dtype(g.standard_normal((B, R, D)), dtype)
    return c, torch.tensor(slots, device="cuda"), X, n, q, W, dout


def norm_err(got, ref, axes):
    num = np.sqrt((np.square(got - ref)).sum(axis=axes))
    den = np.sqrt(np.square(ref).sum(axis=axes))
    assert np.all(num[den == 0] == 0)
    return (num / np.where(den == 0, 1, den)).max()


def bounds(dtype, k, D, BR):
    if dtype == "bf16":
        return 5 ** 0.5 * 2.0 ** -8, 8 ** 0.5 * 2.0 ** -8
    chain = 2 * 2.0 ** -24 * (4 * D ** 0.5 + 2 * k ** 0.5)
    return chain, chain + 2 * 2.0 ** -24 * BR ** 0.5


def check_fwd(sa, p, h, dtype, out_dtype):
    c, s, X, n, q, W, _ = p
    out, lse = sa.stca_cached_fwd(c, s, q.cuda(), *[w.cuda() for w in W], h, out_dtype=DT[out_dtype], want_lse=True)
    torch.cuda.synchronize()
    ref, rlse = oc.stca_cached_fwd(X, n, q.double().numpy(), *[w.double().numpy() for w in W], h)
    tol, _ = bounds(dtype, X.shape[1], X.shape[2], 1)
    assert out.dtype == DT[out_dtype]
    err = norm_err(out.double().cpu().numpy(), ref, (1, 2))
    assert err <= tol, ("out", err, tol)
    lse = lse.cpu().numpy()
    empty = np.isneginf(rlse)
    np.testing.assert_array_equal(np.isneginf(lse), empty)
    if not empty.all():
        s_max = np.abs(rlse[~empty]).max() + np.log(X.shape[1])
        lt = 2.0 ** -6 * max(1.0, s_max) if dtype == "bf16" else tol * max(1.0, s_max)
        assert np.abs(lse[~empty] - rlse[~empty]).max() <= lt
    return out


def check_bwd(sa, p, h, dtype, grad_dtype):
    c, s, X, n, q, W, dout = p
    g = sa.stca_cached_bwd(c, s, q.cuda(), *[w.cuda() for w in W], h, dout.to(DT[grad_dtype]).cuda())
    torch.cuda.synchronize()
    ref = oc.stca_cached_bwd(X, n, q.double().numpy(), *[w.double().numpy() for w in W], h,
                             dout.to(DT[grad_dtype]).double().numpy())
    _, tol = bounds(dtype, X.shape[1], X.shape[2], q.shape[0] * q.shape[1])
    for name in ("dq", "dWq", "dWk", "dWv"):
        assert g[name].dtype == DT[grad_dtype]
        got = g[name].double().cpu().numpy()
        err = norm_err(got, ref[name], (1, 2) if name == "dq" else (0, 1))
        assert err <= tol, (name, err, tol)
    return g


# B, R, k, D, h, rows, slots: one row and one target; odd sizes; empty users, misses and a
# shared slot; rows ending inside a tile, an octet or at one; heads of odd width; long sketches
STCA_CASES = [
    (1, 1, 1, 1, 1, [1], [0]),
    (1, 1, 5, 32, 1, [5], [0]),
    (2, 1, 64, 128, 2, [64, 1], [1, 0]),
    (3, 5, 40, 96, 3, [40, 0, 17], [2, 0, 1]),
    (4, 3, 33, 60, 3, [33, 32, 31, 9], [0, 1, -1, 3]),
    (3, 7, 100, 100, 5, [100, 65, 100], [0, 1, 0]),
    (2, 16, 130, 256, 4, [130, 129], [1, 0]),
    (2, 20, 96, 320, 5, [96, 64], [0, 1]),
    (1, 40, 512, 512, 8, [509], [0]),
    (2, 4, 600, 128, 2, [600, 257], [1, 0]),
    (2, 2, 1100, 64, 2, [1100, 1025], [0, 1]),
    (1, 3, 300, 1024, 16, [300], [0]),
    (2, 70, 72, 72, 3, [72, 50], [0, 1]),
    (1, 2, 48, 1100, 11, [47], [0]),            # wider than 1024
    (5, 1, 20, 64, 4, [0, 0, 20, 0, 3], [0, 1, 2, -1, 4]),
]


def many(B, k, empty=True):
    """Rows and slots of a batch: full and short sketches, some empty, a miss."""
    g = rng_of(B, k, 5)
    rows = np.minimum(g.integers(1, 2 * k, B), k)
    if empty:
        rows[1::5] = 0
    slots = g.permutation(B)
    slots[2] = -1
    return rows.tolist(), slots.tolist()


# batches large enough for workgroups of one head's targets: heads of 32, 64, 96 and 128,
# one to four 16s of targets, one chunk of keys and several
HEAD_CASES = [(43, 12, 24, 96, 3), (32, 13, 33, 256, 4), (32, 20, 300, 256, 4), (65, 12, 20, 256, 2),
              (45, 17, 100, 288, 3), (11, 40, 150, 384, 12), (11, 64, 384, 384, 12), (9, 70, 130, 512, 16)]
STCA_CASES += [c + many(c[0], c[2]) for c in HEAD_CASES]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,R,k,D,h,rows,slots", STCA_CASES)
def test_forward_matches_oracle(sa, B, R, k, D, h, rows, slots, dtype, fmt):
    print(f"fwd B={B} R={R} k={k} D={D} h={h} {dtype} {fmt}", flush=True)
    check_fwd(sa, problem(sa, B, R, k, D, h, fmt, dtype, rows, slots), h, dtype, dtype)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,R,k,D,h,rows,slots", STCA_CASES)
def test_backward_matches_oracle(sa, B, R, k, D, h, rows, slots, dtype, fmt):
    print(f"bwd B={B} R={R} k={k} D={D} h={h} {dtype} {fmt}", flush=True)
    check_bwd(sa, problem(sa, B, R, k, D, h, fmt, dtype, rows, slots), h, dtype, dtype)


# ---------------------------------------------------------------- larger batches


def reference64(X, n, q, W, h, dout):
    """(out, lse, gradients) of the masked attention in float64 on the device, all users
    at once, keys X W_K and values X W_V formed, the gradients by differentiation."""
    B, k, D = X.shape
    R, dh = q.shape[1], D // h
    leaves = [t.double().requires_grad_(True) for t in (q, *W)]
    Q = (leaves[0] @ leaves[1]).view(B, R, h, dh).transpose(1, 2)
    K = (X @ leaves[2]).view(B, k, h, dh).transpose(1, 2)
    V = (X @ leaves[3]).view(B, k, h, dh).transpose(1, 2)
    s = (Q @ K.transpose(2, 3).contiguous()) / dh ** 0.5                    # [B, h, R, k]
    valid = torch.arange(k, device=X.device) < n[:, None]
    s = s.masked_fill(~valid[:, None, None, :], -torch.inf)
    lse = torch.logsumexp(s, -1)
    alpha = torch.where(n[:, None, None, None] > 0, torch.exp(s - lse[..., None].nan_to_num(neginf=0.0)), 0.0)
    out = (alpha @ V).transpose(1, 2).reshape(B, R, D)
    g = torch.autograd.grad(out, leaves, dout.double())
    return out.detach(), lse.detach().transpose(1, 2), dict(zip(("dq", "dWq", "dWk", "dWv"), g))


# every form of the forward and of the backward: workgroups of one head's targets in one to
# four 16s, of all of a user's rows, of split keys, keys in one chunk and several, the
# separate products (the backward's for many keys at the widest, too); widths that are no
# multiple of a head's 32, of 8, of 2
BIG_CASES = [(16, 40, 130, 1024, 16), (16, 60, 300, 1024, 16), (64, 16, 140, 1024, 16), (64, 8, 1100, 1024, 16),
             (300, 1, 100, 1024, 16), (50, 30, 90, 600, 5), (60, 33, 70, 333, 3), (3, 300, 700, 1024, 16),
             (20, 33, 1030, 1024, 16), (100, 40, 40, 96, 3), (40, 100, 300, 256, 2), (16, 16, 140, 1024, 16),
             (32, 40, 100, 1024, 32), (64, 20, 60, 512, 16), (2, 4, 600, 1000, 8), (8, 60, 150, 999, 9),
             (128, 20, 60, 1000, 5), (40, 50, 200, 768, 8), (1, 300, 2500, 1024, 8), (2, 20, 90, 1600, 10),
             (40, 300, 130, 96, 3), (40, 300, 520, 20, 1), (100, 300, 130, 20, 1), (1, 1, 130, 20, 1),
             (20, 9, 1100, 512, 4), (7, 30, 900, 288, 3), (6, 5, 1500, 500, 5), (3, 2, 4096, 256, 2), (100, 20, 600, 480, 5)]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("B,R,k,D,h", BIG_CASES)
def test_larger_batches_match_float64(sa, B, R, k, D, h, fmt):
    print(f"big B={B} R={R} k={k} D={D} h={h} {fmt}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(B + R + k + D)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    rows, slots = many(B, k, empty=B > 3) if B > 2 else ([k, max(1, k - 37)][:B], [1, 0][:B])
    n = torch.tensor(rows, device="cuda")
    slots = torch.tensor(slots, device="cuda")
    c = raw_cache(sa, max(B, 2), k, D, fmt, B)
    held = sa.sketch_cache(max(B, 2), k, D, fmt)
    held.data.copy_(c.data)
    sa.cache_write(held, normal(B, k, D), slots, n.int())
    X = sa.cache_read(held, slots, dtype=torch.float32).double()   # (exact: tested above)
    n = torch.where(slots >= 0, n, 0)
    q, dout = normal(B, R, D).bfloat16(), normal(B, R, D).bfloat16()
    W = [(normal(D, D) / D ** 0.5).bfloat16() for _ in range(3)]
    out, lse = sa.stca_cached_fwd(held, slots, q, *W, h, out_dtype=torch.bfloat16, want_lse=True)
    grads = sa.stca_cached_bwd(held, slots, q, *W, h, dout)
    ref, rlse, rgrads = reference64(X, n, q, W, h, dout)
    ftol, btol = bounds("bf16", k, D, B * R)
    off = lambda a, b: float((a.double() - b).norm() / b.norm().clamp(min=1e-300))  # noqa: E731
    assert off(out, ref) <= ftol, ("out", off(out, ref))
    for b in range(B):   # no user is wrong among many: 1.5 times the bound for the fewer values of one
        assert off(out[b], ref[b]) <= 1.5 * ftol, ("out", b, int(n[b]), off(out[b], ref[b]))
        assert off(grads["dq"][b], rgrads["dq"][b]) <= 1.5 * btol or int(n[b]) <= 2, ("dq", b, int(n[b]))
        if not int(n[b]):
            assert not out[b].any() and not grads["dq"][b].any() and torch.isneginf(lse[b]).all()
    some = n > 0
    assert float((lse[some] - rlse[some]).abs().max()) <= 2.0 ** -6 * max(1.0, float(rlse[some].abs().max()) + np.log(k))
    for name in grads:
        assert off(grads[name], rgrads[name]) <= btol, (name, off(grads[name], rgrads[name]))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,R,D,h", [(13, 5, 24, 3), (65, 1, 128, 4), (9, 71, 64, 1), (3, 64, 40, 1), (127, 1, 72, 3),
                                     (40, 125, 256, 4)])
def test_weight_gradients_over_any_number_of_targets(sa, B, R, D, h, dt):
    """sums over one target to many, around the multiples of 64 that the products take at a time,
    with gradients in either type"""
    k = 20
    print(f"targets B={B} R={R} D={D} h={h} {dt}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(B + R + D)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    c = sa.sketch_cache(B, k, D, "fp8")
    slots = torch.arange(B, device="cuda")
    sa.cache_write(c, normal(B, k, D), slots)
    X = sa.cache_read(c, slots, dtype=torch.float32).double()
    q, dout = normal(B, R, D).bfloat16(), normal(B, R, D).to(dt)
    W = [(normal(D, D) / D ** 0.5).bfloat16() for _ in range(3)]
    grads = sa.stca_cached_bwd(c, slots, q, *W, h, dout)
    n = torch.full((B,), k, device="cuda")
    _, _, ref = reference64(X, n, q, W, h, dout)
    _, btol = bounds("bf16", k, D, B * R)
    for name, want in ref.items():
        assert grads[name].dtype == dt
        off = float((grads[name].double() - want).norm() / want.norm())
        assert off <= btol, (name, off)


def test_fp32_results_of_bf16_inputs(sa):
    p = problem(sa, 3, 6, 70, 128, 2, "fp8", "bf16", [70, 0, 41], [0, 1, 2])
    check_fwd(sa, p, 2, "bf16", "fp32")
    check_bwd(sa, p, 2, "bf16", "fp32")
    with pytest.raises(sa.SAError):
        sa.stca_cached_fwd(p[0], p[1], p[4].float().cuda(), *[w.float().cuda() for w in p[5]], 2,
                           out_dtype=torch.bfloat16)


def test_no_user_has_rows(sa):
    for dtype in ("bf16", "fp32"):
        p = problem(sa, 2, 3, 24, 64, 2, "fp4", dtype, [0, 0], [-1, 1])
        out = check_fwd(sa, p, 2, dtype, dtype)
        assert not out.any()
        g = check_bwd(sa, p, 2, dtype, dtype)
        assert not any(v.any() for v in g.values())


def test_a_nan_row_stays_with_its_users(sa):
    """A sketch with a NaN group gives its own users NaN and nobody else."""
    for dtype in ("bf16", "fp32"):
        p = problem(sa, 3, 2, 40, 64, 2, "fp4", dtype, [40, 40, 12], [0, 1, 2])
        c, s, X, n, q, W, _ = p
        clean, _ = sa.stca_cached_fwd(c, s, q.cuda(), *[w.cuda() for w in W], 2)
        at = oc.places(40, 64, "fp4")[1][7, 1]
        c.data[1, int(at)] = 255
        out, _ = sa.stca_cached_fwd(c, s, q.cuda(), *[w.cuda() for w in W], 2)
        assert torch.isnan(out[1]).all() and torch.equal(out[0], clean[0]) and torch.equal(out[2], clean[2])


def test_sharp_logits(sa):
    """Logits of tens: weights of one row, others underflow.  One rounding of 2^-8 in a
    logit of 60 moves it by 0.2, so bf16 mode is compared in fp32 inputs only."""
    check_fwd(sa, problem(sa, 2, 5, 90, 128, 2, "fp8", "fp32", [90, 33], [0, 1], sharp=40.0), 2, "fp32", "fp32")


def test_results_are_the_same_bits_again(sa):
    p = problem(sa, 3, 9, 200, 256, 4, "fp4", "bf16", [200, 77, 5], [0, 1, 2])
    c, s, _, _, q, W, dout = p
    a = [q.cuda()] + [w.cuda() for w in W]
    first, grads = sa.stca_cached_fwd(c, s, *a, 4)[0], sa.stca_cached_bwd(c, s, *a, 4, dout.cuda())
    for _ in range(3):
        assert torch.equal(first, sa.stca_cached_fwd(c, s, *a, 4)[0])
        again = sa.stca_cached_bwd(c, s, *a, 4, dout.cuda())
        assert all(torch.equal(grads[x], again[x]) for x in grads)


# ---------------------------------------------------------------- together, as they are used


def test_request_path_captured_and_replayed(sa):
    """Refresh, read back and attend in one captured graph on its own stream and
    workspace: replays with new inputs equal the eager calls."""
    B, R, k, D, h = 3, 4, 100, 256, 4
    g = rng_of(11)
    c = sa.sketch_cache(6, k, D, "fp4")
    Xs = torch.empty((B, k, D), device="cuda")
    q = torch.empty((B, R, D), device="cuda", dtype=torch.bfloat16)
    W = [as_dtype(g.standard_normal((D, D)) / 16, "bf16").cuda() for _ in range(3)]
    slots = torch.tensor([4, 1, 2], device="cuda")
    rows = torch.tensor([100, 37, 64], dtype=torch.int32, device="cuda")
    dout = as_dtype(g.standard_normal((B, R, D)), "bf16").cuda()

    def step():
        sa.cache_write(c, Xs, slots, rows)
        back = sa.cache_read(c, slots)
        out, lse = sa.stca_cached_fwd(c, slots, q, *W, h, out_dtype=torch.bfloat16, want_lse=True)
        return [back, out, lse] + list(sa.stca_cached_bwd(c, slots, q, *W, h, dout).values())

    Xs.normal_(), q.normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        Xs.copy_(torch.from_numpy(g.standard_normal((B, k, D)).astype(np.float32)))
        q.copy_(as_dtype(g.standard_normal((B, R, D)), "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_on_a_stream_of_the_callers(sa):
    """Everything on a side stream, behind work that the default stream has not done."""
    p = problem(sa, 2, 3, 50, 64, 2, "fp8", "bf16", [50, 20], [0, 1])
    c, s, _, _, q, W, dout = p
    a = [q.cuda()] + [w.cuda() for w in W]
    ref, gref = sa.stca_cached_fwd(c, s, *a, 2)[0], sa.stca_cached_bwd(c, s, *a, 2, dout.cuda())
    side = torch.cuda.Stream()
    d = dout.cuda()
    torch.cuda.synchronize()
    out, _ = sa.stca_cached_fwd(c, s, *a, 2, stream=side)
    g = sa.stca_cached_bwd(c, s, *a, 2, d, stream=side)
    back = sa.cache_read(c, s, stream=side)
    side.synchronize()
    assert torch.equal(out, ref) and all(torch.equal(g[x], gref[x]) for x in g)
    assert torch.equal(back, sa.cache_read(c, s))


def test_outputs_of_the_caller(sa):
    p = problem(sa, 2, 3, 50, 64, 2, "fp8", "bf16", [50, 20], [0, 1])
    c, s, _, _, q, W, _ = p
    a = [q.cuda()] + [w.cuda() for w in W]
    ref, _ = sa.stca_cached_fwd(c, s, *a, 2)
    out = torch.full((2, 3, 64), 7.0, device="cuda")
    ws = torch.empty(sa.stca_cached_fwd_workspace_size(2, 3, 50, 64, 2, sa.SA_BF16), dtype=torch.uint8, device="cuda")
    got, _ = sa.stca_cached_fwd(c, s, *a, 2, out=out, workspace=ws)
    assert got is out and torch.equal(out, ref)
    for bad in (dict(out=torch.empty((2, 3, 65), device="cuda")), dict(workspace=ws[:-256]), dict(workspace=ws.cpu())):
        with pytest.raises(sa.SAError):
            sa.stca_cached_fwd(c, s, *a, 2, **bad)
    with pytest.raises(sa.SAError):
        sa.cache_read(c, s, out=torch.empty((2, 64, 50), dtype=torch.bfloat16, device="cuda").transpose(1, 2))
    with pytest.raises(sa.SAError):
        sa.cache_write(c, torch.empty((2, 50, 64), device="cuda"), s.int())


def test_no_users(sa):
    c = sa.sketch_cache(3, 10, 64, "fp4")
    s = torch.empty(0, dtype=torch.int64, device="cuda")
    sa.cache_write(c, torch.empty((0, 10, 64), device="cuda"), s)
    assert sa.cache_read(c, s).shape == (0, 10, 64)
    W = [torch.zeros((64, 64), dtype=torch.bfloat16, device="cuda")] * 3
    out, _ = sa.stca_cached_fwd(c, s, torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"), *W, 2)
    assert out.shape == (0, 2, 64) and not c.rows.any()
