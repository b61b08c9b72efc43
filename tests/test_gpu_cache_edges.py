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
         (7, 2, 4096, 256, 2), (6, 2, 60, 1100, 11), (10, 16, 1100, 1024, 16)]


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
