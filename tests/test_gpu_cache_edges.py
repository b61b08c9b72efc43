"""GPU tests of the sketch cache and of the attention over it at the edges of what a call
may hold: targets of users without rows, sketches of one or two rows, sharp logits, row
counts that no write has left, bytes at every rounding border, sizes past 32 bits.

Tolerances.  A rounding to bf16 is off by at most half a step, 2^-8 of the value
(finfo.eps / 2), so n independent ones in a chain add up to at most sqrt(n) 2^-8 by
2-norm; how many stands at each test.  Everything else is compared bit by bit.
"""
import numpy as np
import pytest

from oracle import cache as oc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def sa():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_08443_amd import sa_sketch
    sa_sketch.lib()
    return sa_sketch


def generator(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(8443 + sum(p * int(x) for p, x in zip((1, 3, 7, 11, 13), key)))
    return lambda *shape: torch.randn(shape, generator=g, device="cuda")


def off(a, b):
    return float((a.double() - b).norm() / b.norm())


# B, R, k, D, h: one head's targets a workgroup and all of a user's rows, keys in one chunk and in
# several, heads of odd width, separate products (wider than 1024; the widest with many keys), sums over
# whole 64s of targets and not
FORMS = [(11, 40, 150, 384, 12), (32, 40, 100, 1024, 16), (9, 70, 130, 512, 16), (300, 1, 100, 1024, 16),
         (60, 33, 70, 333, 3), (100, 40, 40, 96, 3), (12, 5, 200, 256, 4), (20, 9, 1100, 512, 4), (6, 5, 1500, 500, 5),
         (7, 2, 4096, 256, 2), (6, 2, 60, 1100, 11), (10, 16, 1100, 1024, 16), (200, 20, 600, 64, 2), (40, 300, 520, 20, 1),
         (40, 20, 600, 512, 8)]


def batch(sa, B, R, k, D, h, rows, dt=BF, fmt="fp8"):
    """A written cache, slots, targets, weights and upstream gradients; the last user has no slot."""
    normal = generator(B, R, k, D, h)
    c = sa.sketch_cache(B + 1, k, D, fmt)
    slots = torch.randperm(B, device="cuda")
    sa.cache_write(c, normal(B, k, D), slots, torch.tensor(rows, dtype=torch.int32, device="cuda"))
    slots[-1] = -1
    q, dout = normal(B, R, D).to(dt), normal(B, R, D).to(dt)
    W = [(normal(D, D) / D ** 0.5).to(dt) for _ in range(3)]
    return c, slots, q, W, dout


# ---------------------------------------------------------------- users without rows


@pytest.mark.parametrize("dt,gdt", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("B,R,k,D,h", FORMS)
def test_targets_of_users_without_rows_may_hold_anything(sa, B, R, k, D, h, dt, gdt):
    """A padded batch: misses and empty slots, whose q and dout are NaN and infinities, give and
    add nothing, as if they were zeros."""
    print(f"no rows B={B} R={R} k={k} D={D} h={h} {dt} {gdt}", flush=True)
    rows = [k if b % 3 else 0 for b in range(B)]
    c, slots, q, W, dout = batch(sa, B, R, k, D, h, rows, dt)
    slots[1] = c.data.shape[0] + 5                      # outside the cache
    none = torch.tensor([b % 3 == 0 or b in (1, B - 1) for b in range(B)], device="cuda")
    dout = dout.to(gdt)
    q[none], dout[none] = 0, 0
    out, lse = sa.stca_cached_fwd(c, slots, q, *W, h, want_lse=True)
    want = sa.stca_cached_bwd(c, slots, q, *W, h, dout)
    assert not out[none].any() and torch.isneginf(lse[none]).all() and not want["dq"][none].any()
    assert all(torch.isfinite(g).all() and g.any() for g in want.values())
    for bad in (float("nan"), float("inf")):
        q[none], dout[none] = bad, bad
        q[none, :, ::3] = -bad
        got, glse = sa.stca_cached_fwd(c, slots, q, *W, h, want_lse=True)
        assert torch.equal(got, out) and torch.equal(glse, lse)
        grads = sa.stca_cached_bwd(c, slots, q, *W, h, dout)
        for name in want:
            assert torch.equal(grads[name], want[name]), (name, bad)


# ---------------------------------------------------------------- row counts


@pytest.mark.parametrize("B", [5, 1024, 1025, 3000])
def test_a_write_takes_any_row_count(sa, B):
    """Counts past k (of a cache of longer sketches, or memory that nobody has cleared) read as k
    rows, and a write to their slots is a write, whatever the batch's size."""
    k, D, n_slots = 3, 40, 6000
    normal = generator(B)
    c = sa.sketch_cache(n_slots, k, D, "fp8")
    c.data.fill_(255)
    left = torch.tensor([k + 1, 100, B + k, B + 5000, 2 ** 31 - 1, -1, -2 ** 31, k + 1 + B // 2], dtype=torch.int32)
    c.rows.copy_(left.repeat(n_slots // 8 + 1)[:n_slots])
    before = c.rows.clone()
    slots = torch.randperm(n_slots, device="cuda")[:B]
    slots[B // 2] = slots[B - 1]                        # the last of the two stays
    n = torch.randint(0, k + 1, (B,), device="cuda", dtype=torch.int32)
    x = normal(B, k, D)
    sa.cache_write(c, x, slots, n)
    want = before.clone()
    want[slots[B // 2 + 1:]], want[slots[:B // 2]] = n[B // 2 + 1:], n[:B // 2]
    assert torch.equal(c.rows, want)
    clean = sa.sketch_cache(n_slots, k, D, "fp8")
    for at in range(0, B, 512):
        sa.cache_write(clean, x[at:at + 512].contiguous(), slots[at:at + 512].clone(), n[at:at + 512].clone())
    assert torch.equal(sa.cache_read(c, slots), sa.cache_read(clean, slots))


# ---------------------------------------------------------------- bytes at the rounding borders


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_bytes_at_every_rounding_border(sa, fmt):
    """Codes (the sign of a zero among them) and scale bytes of the whole slot, around every border
    between two codes, at exponents over the whole range and past it, and of groups with an infinity
    or a NaN.  Rows and the bytes behind them that nobody writes stay."""
    mags = oc.magnitudes(fmt)
    mid = ((mags[1:] + mags[:-1]) / 2).astype(np.float32)
    v = np.concatenate([mags, mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(9e9))])
    v = np.concatenate([v, -v])
    x = np.zeros((-(-v.size // 31), 32))
    for i, part in enumerate(np.array_split(v, x.shape[0])):   # (each group's last is the limit: its exponent as given)
        x[i, :part.size] = part
    x[:, 31] = oc.LIMIT[fmt]
    big = float(np.finfo(np.float32).max)
    x = np.concatenate([np.ldexp(x, e) for e in (-130, -101, -100, -99, -3, 0, 60, 115)])
    odd = np.zeros((8, 32))
    odd[0, :3] = [big, -big, 1.0]
    odd[1, :4] = [1e-38, 1e-45, -1e-45, -0.0]
    odd[2, :2], odd[3, 30:], odd[4, 0] = [1.0, np.inf], [np.nan, -0.0], -np.inf
    odd[5] = -0.0
    odd[6, 0] = np.ldexp(oc.LIMIT[fmt], oc.E_MAX[fmt])
    odd[7, 0] = np.nextafter(np.float32(odd[6, 0]), np.float32(big))
    x = np.concatenate([x, odd]).astype(np.float32)
    k = -(-x.shape[0] // 8) * 8 + 8                      # an octet behind the rows, and a short one before it
    x = np.concatenate([x, np.ones((k - x.shape[0], 32), np.float32)])
    n = k - 11
    c = sa.sketch_cache(1, k, 32, fmt)
    c.data.copy_(torch.from_numpy(np.random.default_rng(3).integers(0, 256, tuple(c.data.shape)).astype(np.uint8)))
    want = c.data[0].cpu().numpy().copy()
    slot = torch.zeros(1, dtype=torch.int64, device="cuda")
    sa.cache_write(c, torch.from_numpy(x)[None].cuda(), slot, torch.tensor([n], dtype=torch.int32, device="cuda"))
    oc.pack(want, x.astype(np.float64), n, fmt)
    np.testing.assert_array_equal(c.data[0].cpu().numpy(), want)


# ---------------------------------------------------------------- short sketches, sharp logits, NaN


def reference64(X, n, q, W, h, dout, scale):
    """(out, lse, gradients) of the attention over each user's first n rows, in float64, keys X W_K
    and values X W_V formed, the gradients by differentiation."""
    B, k, D = X.shape
    R, dh = q.shape[1], D // h
    leaves = [t.double().requires_grad_(True) for t in (q, *W)]
    split = lambda t, m: t.view(B, m, h, dh).transpose(1, 2)                           # noqa: E731
    Q, K, V = split(leaves[0] @ leaves[1], R), split(X @ leaves[2], k), split(X @ leaves[3], k)
    s = scale * (Q @ K.transpose(2, 3).contiguous())
    s = s.masked_fill((torch.arange(k, device=X.device) >= n[:, None])[:, None, None, :], -torch.inf)
    some = (n > 0)[:, None, None, None]
    lse = torch.logsumexp(s, -1, keepdim=True)
    alpha = torch.where(some, torch.exp(s - torch.where(some, lse, 0.0)), 0.0)
    out = (alpha @ V).transpose(1, 2).reshape(B, R, D)
    g = torch.autograd.grad(out, leaves, dout.double())
    return out.detach(), lse.detach()[..., 0].transpose(1, 2), dict(zip(("dq", "dWq", "dWk", "dWv"), g))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,R,k,D,h", FORMS)
def test_sketches_of_one_and_two_rows(sa, B, R, k, D, h, dt):
    """One row: its weight is 1, and the targets' gradient exactly zero.  Two rows and three: the
    eight roundings of the gradients (q W_Q, u, the weights, dc, ds, du, dp, the result),
    all users of that length together; fp32: a sum of N terms is off by about sqrt(N) 2^-24 of its
    terms' norm, of D in four products, here times 8."""
    print(f"short B={B} R={R} k={k} D={D} h={h} {dt}", flush=True)
    rows = [(1, 2, 3, 1, 2, k)[b % 6] for b in range(B)]
    c, slots, q, W, dout = batch(sa, B, R, k, D, h, rows, dt, "fp4")
    n = torch.tensor(rows, device="cuda")
    n[-1] = 0
    X = sa.cache_read(c, slots, dtype=F32).double()
    out, lse = sa.stca_cached_fwd(c, slots, q, *W, h, out_dtype=dt, want_lse=True)
    grads = sa.stca_cached_bwd(c, slots, q, *W, h, dout)
    ref, rlse, rgrads = reference64(X, n, q, W, h, dout, (D // h) ** -0.5)
    tol = 8 ** 0.5 * 2.0 ** -8 if dt == BF else 8 * 4 * D ** 0.5 * 2.0 ** -24
    assert not grads["dq"][n == 1].any()
    for m in (1, 2, 3):
        at = n == m
        assert off(out[at], ref[at]) <= tol, m
        assert float((lse[at] - rlse[at]).abs().max()) <= 2 * tol * max(1.0, float(rlse[at].abs().max()))
        if m > 1 and bool(at.any()):
            assert off(grads["dq"][at], rgrads["dq"][at]) <= tol, m
    for name in rgrads:
        assert off(grads[name], rgrads[name]) <= tol, name


SHARP = FORMS + [(2, 4, 600, 128, 2), (1, 1, 3000, 256, 4), (1, 300, 2500, 1024, 8), (40, 20, 600, 128, 2),
                 (16, 60, 300, 1024, 16), (64, 8, 1100, 1024, 16)]


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("B,R,k,D,h", SHARP)
def test_sharp_logits_in_bf16(sa, B, R, k, D, h, fmt):
    """Logits of tens, the largest of a user's first target at its last key, behind one nearly as large
    at its first: maxima that rise from chunk to chunk and from split to split.  W_Q and W_K are
    identities, so that q W_Q and u are exact in bf16 and the logits those of float64 but for
    fp32 sums: |q_i| is about 6, a logit's standard deviation 6, the planted ones 29 and 40.
    Roundings left: forward, the weights, the aggregates and a bf16 result; gradients, fewer than
    eight (the weights or ds, the aggregates, dc, du, dp, the result).  lse: a sum of dh fp32 products whose norm is
    |q_i| |X_i|, its maximum's product with the scale and two hardware functions, 8 times 2^-24
    of their sizes."""
    print(f"sharp B={B} R={R} k={k} D={D} h={h} {fmt}", flush=True)
    normal = generator(B, R, k, D, h)
    dh = D // h
    q = (normal(B, R, D) * (6 / dh ** 0.5)).to(BF)
    n = torch.full((B,), k, device="cuda")
    n[1::2] = max(k - 3, 1)
    x = normal(B, k, D)
    x[:, 0] = 0.8 * q[:, 0].float()
    x[torch.arange(B, device="cuda"), n - 1] = 1.1 * q[:, 0].float()
    c = sa.sketch_cache(B, k, D, fmt)
    slots = torch.arange(B, device="cuda")
    sa.cache_write(c, x, slots, n.int())
    X = sa.cache_read(c, slots, dtype=F32).double()
    eye = torch.eye(D, device="cuda", dtype=BF)
    W = [eye, eye, (normal(D, D) / D ** 0.5).to(BF)]
    dout = normal(B, R, D).to(BF)
    out, lse = sa.stca_cached_fwd(c, slots, q, *W, h, scale=1.0, out_dtype=BF, want_lse=True)
    grads = sa.stca_cached_bwd(c, slots, q, *W, h, dout, scale=1.0)
    ref, rlse, rgrads = reference64(X, n, q, W, h, dout, 1.0)
    assert float(rlse.max()) > 25.0
    assert off(out, ref) <= 3 ** 0.5 * 2.0 ** -8
    assert float((lse - rlse).abs().max()) <= 8 * 2.0 ** -24 * (float(rlse.abs().max()) + 6 * dh ** 0.5)
    for name in rgrads:
        assert off(grads[name], rgrads[name]) <= 8 ** 0.5 * 2.0 ** -8, (name, off(grads[name], rgrads[name]))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,R,k,D,h", FORMS)
def test_a_nan_group_in_the_backward(sa, B, R, k, D, h, dt):
    """It gives its own user's targets NaN and the weights' sums, and nobody else's targets."""
    c, slots, q, W, dout = batch(sa, B, R, k, D, h, [k] * B, dt)
    clean = sa.stca_cached_bwd(c, slots, q, *W, h, dout)
    c.data[slots[1], int(oc.places(k, D, "fp8")[1][k // 2, -1])] = 255
    grads = sa.stca_cached_bwd(c, slots, q, *W, h, dout)
    rest = torch.arange(B, device="cuda") != 1
    assert torch.equal(grads["dq"][rest], clean["dq"][rest])
    assert torch.isnan(grads["dq"][1]).all()
    assert all(torch.isnan(grads[w]).all() for w in ("dWq", "dWk", "dWv"))


# ---------------------------------------------------------------- sizes past 32 bits


def test_more_than_four_giga_values_of_targets(sa):
    """4.26 million targets at D = 1024, 2^32 + 67 million values: gradients asked for in fp32 are,
    rounded, those asked for in bf16 of the same dout bit for bit, and the last user's are a small
    call's (by 2-norm the eight roundings of the gradients)."""
    B, R, k, D = 65535, 65, 4, 1024
    if torch.cuda.mem_get_info()[0] < 170 << 30:
        pytest.skip("needs 170 GB")
    assert B * R * D > 1 << 32
    normal = generator(B, R)
    c = sa.sketch_cache(3, k, D, "fp8")
    sa.cache_write(c, normal(3, k, D), torch.arange(3, device="cuda"))
    slots = torch.arange(B, device="cuda") % 3
    W = [(normal(D, D) / 32).to(BF) for _ in range(3)]
    q, dout = (torch.empty((B, R, D), dtype=BF, device="cuda") for _ in range(2))
    for at in range(0, B, 4096):                     # (other targets everywhere)
        m = min(4096, B - at)
        q[at:at + m], dout[at:at + m] = normal(m, R, D), normal(m, R, D)
    ws = torch.empty(sa.stca_cached_bwd_workspace_size(B, R, k, D, 1, sa.SA_BF16), dtype=torch.uint8, device="cuda")
    half = sa.stca_cached_bwd(c, slots, q, *W, 1, dout, workspace=ws)
    single = sa.stca_cached_bwd(c, slots[-1:].clone(), q[-1:].contiguous(), *W, 1, dout[-1:].contiguous())
    assert off(half["dq"][-1:], single["dq"].double()) <= 8 ** 0.5 * 2.0 ** -8
    full = sa.stca_cached_bwd(c, slots, q, *W, 1, dout.float(), workspace=ws)
    for name in full:
        assert full[name].dtype == F32 and bool(half[name].any())
        a, b = full[name].view(-1, D), half[name].view(-1, D)
        assert all(torch.equal(a[at:at + (1 << 20)].to(BF), b[at:at + (1 << 20)]) for at in range(0, a.shape[0], 1 << 20))
    del ws, half, full, q, dout
    torch.cuda.empty_cache()
