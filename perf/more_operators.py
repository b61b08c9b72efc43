"""Attention over the recent history and the layers around it: what their speed and their results are judged by.

Targets attend over the last tokens of their user's history as they lie in the packed
batch (the recent branch beside the sketch's STCA), with the norms before and the
products around it.  Each case is one pass through the public entry points of
``paper_2609_08443_amd.sa_sketch`` (``own``), or through the same operators written in
plain torch.  ``listed()`` names the cases, ``draw()`` gives others of the same ranges,
``exact()`` evaluates a case in float64.

Attention: q [N, h, d] of N targets, packed by user as ``targets`` [B + 1] says, K and V
[T, hk, d] of T tokens, packed as ``offsets`` [B + 1] says; query head i reads head
i // (h / hk).  Target i of a user with L tokens sees the tokens [max(0, e - window), e)
of them, e = ends[i] (L without ``ends``; window 0: no limit):
  s_j = scale <q_i, K_j>, with a cap s_j = cap tanh(s_j / cap), then - slope_head (e - 1 - j)
  out = sum_j softmax(s)_j V_j, lse = log sum_j exp(s_j); 0 and -inf where it sees none.
Norm: y = (x - mean) rstd gamma + beta, rstd = 1 / sqrt(var + eps), over rows of D.
Linear: z = x W + b, y = act(z) + residual; swiglu: W has 2 F columns, y = silu(z1) z2 + residual.

Values: activations, targets and upstream gradients ~ N(0, 1) (the history's rows with a
mean of their own in the norm), weights ~ N(0, 1/fan-in), norms' weights near one.
Ragged cases have between one and L tokens a user (log-uniform), every seventh none;
targets of "prefix" cases end anywhere in their user's history, some before its first token.

Kinds:
  attn, attn_grad       sa_recent_attn_fwd, sa_recent_attn_bwd
  norm, norm_grad       sa_layer_norm_fwd, sa_layer_norm_bwd
  linear, linear_grad   sa_linear_fwd, sa_linear_bwd
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
EPS = 1e-5


def listed():
    return [
        # one request with a single target over 10K recent tokens: latency
        dict(name="attn_one", kind="attn", dtype="bf16", B=1, R=1, L=10000, h=16, hk=16, d=64, ragged=False, prefix=False,
             window=0, cap=0.0, bias=False, packed=True, spread=0),
        # a server's batch of single targets of users with short and long histories, heads in groups of four, nearer tokens preferred
        dict(name="attn_users", kind="attn", dtype="bf16", B=256, R=1, L=10000, h=16, hk=4, d=64, ragged=True, prefix=False,
             window=0, cap=0.0, bias=True, packed=True, spread=5),
        # candidate scoring: 300 targets a user over 10K tokens; the largest
        dict(name="attn_candidates", kind="attn", dtype="bf16", B=16, R=300, L=10000, h=16, hk=16, d=64, ragged=False, prefix=False,
             window=0, cap=0.0, bias=False, packed=False, spread=0),
        # a training step's gradients: 40 targets a user, each seeing what came before its request, scores capped
        dict(name="attn_grads", kind="attn_grad", dtype="bf16", B=16, R=40, L=10000, h=16, hk=16, d=64, ragged=False, prefix=True,
             window=0, cap=30.0, bias=False, packed=True, spread=3),
        # gradients in single precision, sizes off every tile, shared heads, bias and window together
        dict(name="attn_grads_fp32_odd", kind="attn_grad", dtype="fp32", B=9, R=7, L=700, h=6, hk=3, d=128, ragged=True, prefix=True,
             window=150, cap=20.0, bias=True, packed=False, spread=2),
        # the norm before a single target's projections: the smallest call
        dict(name="norm_one", kind="norm", dtype="bf16", N=1, D=1024),
        # the norm of a batch's recent histories
        dict(name="norm_history", kind="norm", dtype="bf16", N=100000, D=1024),
        # its gradients in training, a ragged number of tokens
        dict(name="norm_grads", kind="norm_grad", dtype="bf16", N=61003, D=1024),
        # a single target's output projection on the residual stream
        dict(name="linear_one", kind="linear", dtype="bf16", N=1, K=1024, F=1024, act="none", bias=True, residual=True),
        # the history's feed-forward, its gated half
        dict(name="linear_ffn", kind="linear", dtype="bf16", N=40000, K=1024, F=2048, act="swiglu", bias=False, residual=False),
        # a small layer in single precision, sizes off every tile
        dict(name="linear_fp32_odd", kind="linear", dtype="fp32", N=1001, K=200, F=331, act="gelu", bias=True, residual=True),
        # gradients of the gated half over a ragged batch
        dict(name="linear_grads", kind="linear_grad", dtype="bf16", N=10007, K=1024, F=2048, act="swiglu", bias=True, residual=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn_grad", "attn_grad", "norm", "norm_grad", "linear", "linear", "linear_grad"])
    while True:
        c = dict(kind=kind, dtype="bf16" if rng.random() < 0.75 else "fp32")
        if kind.startswith("attn"):
            hk = rng.choice([1, 2, 4, 4, 8, 16, rng.randrange(1, 13)])
            c.update(B=_log_int(rng, 1, 256), L=_log_int(rng, 1, 20000), d=rng.choice([64, 64, 128]), hk=hk,
                     h=hk * rng.choice([1, 1, 2, 4, 8, rng.randrange(1, 9)]),
                     R=rng.choice([1, 1, _log_int(rng, 2, 300), _log_int(rng, 2, 60)]),
                     ragged=rng.random() < 0.6, prefix=rng.random() < 0.5, window=rng.choice([0, 0, _log_int(rng, 1, 10000)]),
                     cap=rng.choice([0.0, 0.0, 15.0, 50.0]), bias=rng.random() < 0.4, packed=rng.random() < 0.5,
                     spread=rng.randrange(1000))
            if c["h"] > 32 or c["B"] * c["L"] * c["hk"] * c["d"] > 3.3e8:
                continue
            if c["B"] * c["R"] * c["h"] * c["L"] > (7.6e8 if kind == "attn" else 2e8):   # the plain form's scores
                continue
        elif kind.startswith("norm"):
            c.update(N=_log_int(rng, 1, 100000), D=rng.choice([64, 128, 256, 512, 1024, 1024, 2048, _log_int(rng, 1, 9000)]))
            if c["N"] * c["D"] > 1e8:
                continue
        else:
            size = lambda: rng.choice([64, 128, 256, 512, 1024, 1024, 2048, _log_int(rng, 1, 2500)])  # noqa: E731
            c.update(N=rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 60000), _log_int(rng, 1, 60000)]), K=size(), F=size(),
                     act=rng.choice(["none", "none", "relu", "gelu", "silu", "swiglu", "swiglu"]), bias=rng.random() < 0.6,
                     residual=rng.random() < 0.4)
        w = work(c)
        if w["flops"] <= (3e10 if c["dtype"] == "fp32" else 3e11) and w["bytes"] <= 1.5e9:
            return c


# ---------------------------------------------------------------- a case's sizes


def _users(case):
    """Tokens and targets of every user."""
    B, L, R = case["B"], case["L"], case["R"]
    n, r = np.full(B, L, np.int64), np.full(B, R, np.int64)
    if case["ragged"]:
        rng = np.random.default_rng(8443 + case["spread"])
        n = np.clip(np.rint(np.exp(rng.uniform(0.0, math.log(L), B))), 1, L).astype(np.int64)
        if B > 3:
            n[np.arange(B) % 7 == 3] = 0
        if R > 1:   # single targets: every user has one
            r = rng.integers(0, R, B, endpoint=True)
            r[0] = max(r[0], 1)
    return n, r


def _ends(case):
    """Every target's end in its user's history."""
    n, r = _users(case)
    ends = np.repeat(n, r)
    if case["prefix"]:
        ends = np.floor(np.random.default_rng(977 + case["spread"]).random(ends.size) * (ends + 1)).astype(np.int64)
    return ends


def _cols(case):
    return case["F"] * (2 if case["act"] == "swiglu" else 1)


def work(case):
    el = 2 if case["dtype"] == "bf16" else 4
    if case["kind"].startswith("norm"):
        N, D = case["N"], case["D"]
        if case["kind"] == "norm":      # x in, y out, gamma, beta; two statistics a row
            return {"bytes": el * (2 * N * D + 2 * D) + 8 * N, "flops": 8 * N * D}
        return {"bytes": el * (3 * N * D + D) + 8 * N + 8 * D, "flops": 14 * N * D}
    if case["kind"].startswith("linear"):
        N, K, F, C = case["N"], case["K"], case["F"], _cols(case)
        if case["kind"] == "linear":
            return {"bytes": el * (N * K + K * C + C * case["bias"] + N * F * (1 + case["residual"])), "flops": 2 * N * K * C}
        pre = 0 if case["act"] == "none" else N * C
        return {"bytes": el * (2 * N * K + 2 * K * C + N * F + pre + C * case["bias"]), "flops": 4 * N * K * C}
    n, _ = _users(case)
    ends, h, hk, d = _ends(case), case["h"], case["hk"], case["d"]
    seen = np.minimum(ends, case["window"]) if case["window"] else ends
    N, pairs, T = ends.size, float(seen.sum()), int(n.sum())
    if case["kind"] == "attn":
        return {"bytes": el * (2 * T * hk * d + 2 * N * h * d), "flops": 4 * pairs * h * d}
    return {"bytes": el * (4 * T * hk * d + 4 * N * h * d) + 4 * N * h, "flops": 10 * pairs * h * d}


# ---------------------------------------------------------------- inputs


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(1_000_003 * seed + 8443)
    dt = _dt(case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE)

    t = {"case": case}
    if case["kind"].startswith("norm"):
        N, D = case["N"], case["D"]
        t["x"] = (normal(N, D) * torch.exp(0.5 * normal(N, 1)) + normal(N, 1)).to(dt)
        t["gamma"], t["beta"] = (1 + 0.1 * normal(D)).to(dt), (0.1 * normal(D)).to(dt)
        if case["kind"] == "norm_grad":
            t["dy"] = normal(N, D).to(dt)
        return t
    if case["kind"].startswith("linear"):
        N, K, C = case["N"], case["K"], _cols(case)
        t["x"], t["W"] = normal(N, K).to(dt), (normal(K, C) * K ** -0.5).to(dt)
        t["b"] = normal(C).to(dt) if case["bias"] else None
        t["res"] = normal(N, case["F"]).to(dt) if case["residual"] and case["kind"] == "linear" else None
        if case["kind"] == "linear_grad":
            t["dy"] = normal(N, case["F"]).to(dt)
        return t
    n, r = _users(case)
    T, N, h, hk, d = int(n.sum()), int(r.sum()), case["h"], case["hk"], case["d"]
    csr = lambda v: torch.from_numpy(np.concatenate([[0], np.cumsum(v)]).astype(np.int64)).to(DEVICE)  # noqa: E731
    t["offsets"], t["targets"] = csr(n), csr(r)
    t["ends"] = torch.from_numpy(_ends(case).astype(np.int32)).to(DEVICE) if case["prefix"] else None
    t["slopes"] = torch.from_numpy(np.exp2(-8.0 * np.arange(1, h + 1) / h).astype(np.float32)).to(DEVICE) if case["bias"] else None
    t["q"] = normal(N, h, d).to(dt)
    if case["packed"]:   # keys and values side by side, as one projection writes them
        kv = normal(T, 2, hk, d).to(dt)
        t["K"], t["V"] = kv[:, 0], kv[:, 1]
    else:
        t["K"], t["V"] = normal(T, hk, d).to(dt), normal(T, hk, d).to(dt)
    if case["kind"] == "attn_grad":
        t["dout"] = normal(N, h, d).to(dt)
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    # what the forward pass of a training step left for the backward
    if case["kind"] == "attn_grad":
        t["out"], t["lse"] = _attn_plain(t, case)
    elif case["kind"] == "norm_grad":
        t["stats"] = _norm_plain(t)[1]
    elif case["kind"] == "linear_grad":
        t["pre"] = None if case["act"] == "none" else _pre_plain(t).to(_dt(case))
    return t


# ---------------------------------------------------------------- one pass


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2609_08443_amd import sa_sketch as sa
        if kind.startswith("attn"):
            a = dict(ends=s["ends"], window=case["window"], slopes=s["slopes"], cap=case["cap"])
            if kind == "attn_grad":
                return sa.recent_attn_bwd(s["q"], s["K"], s["V"], s["offsets"], s["targets"], s["out"], s["lse"], s["dout"], **a)
            out, lse = sa.recent_attn_fwd(s["q"], s["K"], s["V"], s["offsets"], s["targets"], want_lse=case["dtype"] == "fp32", **a)
            return out if lse is None else (out, lse)
        if kind == "norm":
            return sa.layer_norm_fwd(s["x"], s["gamma"], s["beta"], eps=EPS)
        if kind == "norm_grad":
            return sa.layer_norm_bwd(s["x"], s["gamma"], s["stats"], s["dy"])
        if kind == "linear":
            return sa.linear_fwd(s["x"], s["W"], bias=s["b"], act=case["act"], residual=s["res"])[0]
        return sa.linear_bwd(s["x"], s["W"], s["dy"], bias=case["bias"], act=case["act"], pre=s["pre"])
    if kind == "attn":
        out, lse = _attn_plain(s, case)
        return out if case["dtype"] == "bf16" else (out, lse)
    if kind == "attn_grad":
        return _attn_grad_plain(s, case)
    if kind == "norm":
        return _norm_plain(s)
    if kind == "norm_grad":
        return _norm_grad_plain(s)
    if kind == "linear":
        y = _act(_pre_plain(s), case["act"])
        return (y if s["res"] is None else y + s["res"].float()).to(_dt(case))
    return _linear_grad_plain(s, case)


def _scores(s, case):
    """Padded operands in fp32 and the masked scores of every user's targets: [B, hk, R g, L]."""
    B, R, L, h, hk, d = (case[x] for x in ("B", "R", "L", "h", "hk", "d"))
    g, dev = h // hk, s["q"].device
    off, tgt = s["offsets"], s["targets"]
    n, j, i = off[1:] - off[:-1], torch.arange(L, device=dev), torch.arange(R, device=dev)
    at = (off[:-1, None] + j).clamp(max=s["K"].shape[0] - 1)        # [B, L]
    to = (tgt[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)        # [B, R]
    rows = lambda x: x[to].float().view(B, R, hk, g, d).permute(0, 2, 1, 3, 4).reshape(B, hk, R * g, d)  # noqa: E731
    keys = lambda x: x[at].float().permute(0, 2, 1, 3).contiguous()  # noqa: E731
    K, V, q = keys(s["K"]), keys(s["V"]), rows(s["q"])              # [B, hk, L, d], [B, hk, R g, d]
    x = torch.matmul(q, K.transpose(2, 3).contiguous()) * d ** -0.5
    t = None
    if case["cap"]:
        t = torch.tanh(x / case["cap"])
        x = case["cap"] * t
    e = n[:, None].expand(B, R) if s["ends"] is None else s["ends"].long()[to]
    lo = (e - case["window"]).clamp(min=0) if case["window"] else torch.zeros_like(e)
    seen = ((j >= lo[:, :, None]) & (j < e[:, :, None])).repeat_interleave(g, 1)[:, None]     # [B, 1, R g, L]
    if s["slopes"] is not None:
        back = (e[:, :, None] - 1 - j).float().repeat_interleave(g, 1)[:, None]
        x = x - s["slopes"].view(1, hk, 1, g, 1).expand(B, hk, R, g, 1).reshape(B, hk, R * g, 1) * back
    return q, K, V, t, torch.where(seen, x, -math.inf), rows


def _softmax(x):
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(x - top)
    z = w.sum(-1, keepdim=True)
    return w / torch.where(z > 0, z, 1.0), (top + torch.log(z))[..., 0]


def _packed_rows(x, csr, n):
    """Rows [n, ...] of padded x [B, R, ...]."""
    at = torch.arange(n, device=x.device)
    b = torch.searchsorted(csr[1:].contiguous(), at, right=True).clamp(max=csr.shape[0] - 2)
    return x[b, at - csr[b]]


def _attn_plain(s, case):
    B, R, h, hk, d = (case[x] for x in ("B", "R", "h", "hk", "d"))
    _, _, V, _, x, _ = _scores(s, case)
    p, lse = _softmax(x)
    o = torch.matmul(p, V).view(B, hk, R, h // hk, d).permute(0, 2, 1, 3, 4).reshape(B, R, h, d)
    lse = lse.view(B, hk, R, h // hk).permute(0, 2, 1, 3).reshape(B, R, h)
    N = s["q"].shape[0]
    return _packed_rows(o, s["targets"], N).to(_dt(case)), _packed_rows(lse, s["targets"], N)


def _attn_grad_plain(s, case):
    B, R, h, hk, d = (case[x] for x in ("B", "R", "h", "hk", "d"))
    g, dt = h // hk, _dt(case)
    q, K, V, t, x, rows = _scores(s, case)
    p, _ = _softmax(x)
    # places past a user's last target hold another's: none of their weight
    r = s["targets"][1:] - s["targets"][:-1]
    p = p * (torch.arange(R, device=p.device) < r[:, None]).repeat_interleave(g, 1)[:, None, :, None]
    do = rows(s["dout"])
    dV = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, V.transpose(2, 3).contiguous())
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * d ** -0.5
    if t is not None:
        ds = ds * (1 - t * t)
    dq = torch.matmul(ds, K).view(B, hk, R, g, d).permute(0, 2, 1, 3, 4).reshape(B, R, h, d)
    dK = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    back = lambda v: _packed_rows(v.permute(0, 2, 1, 3), s["offsets"], s["K"].shape[0]).to(dt)  # noqa: E731
    return {"dq": _packed_rows(dq, s["targets"], s["q"].shape[0]).to(dt), "dK": back(dK), "dV": back(dV)}


def _norm_plain(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = (x - mean) * rstd * s["gamma"].float() + s["beta"].float()
    return y.to(s["x"].dtype), torch.cat([mean, rstd], 1)


def _norm_grad_plain(s):
    x, dy = s["x"].float(), s["dy"].float()
    mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
    xh = (x - mean) * rstd
    g = dy * s["gamma"].float()
    dx = (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True)) * rstd
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _pre_plain(s):
    z = s["x"].float() @ s["W"].float()
    return z if s["b"] is None else z + s["b"].float()


def _act(z, act):
    if act == "swiglu":
        a, b = z.chunk(2, -1)
        return a * torch.sigmoid(a) * b
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z.clamp(min=0) if act == "relu" else z


def _act_grad(z, dy, act):
    if act in ("swiglu", "silu"):
        a, b = z.chunk(2, -1) if act == "swiglu" else (z, None)
        sg = torch.sigmoid(a)
        da = dy * sg * (1 + a * (1 - sg))
        return da if b is None else torch.cat([da * b, dy * a * sg], -1)
    if act == "gelu":
        return dy * (0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5)
    return torch.where(z > 0, dy, 0.0) if act == "relu" else dy


def _linear_grad_plain(s, case):
    dt, x, W, dy = _dt(case), s["x"].float(), s["W"].float(), s["dy"].float()
    dz = dy if s["pre"] is None else _act_grad(s["pre"].float(), dy, case["act"])
    out = {"dx": (dz @ W.t().contiguous()).to(dt), "dW": (x.t().contiguous() @ dz).to(dt)}
    if case["bias"]:
        out["db"] = dz.sum(0).to(dt)
    return out


# ---------------------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    t = _inputs(case, seed)
    f8 = torch.float64
    kind = case["kind"]
    if kind.startswith("norm"):
        x, gamma = t["x"].to(f8), t["gamma"].to(f8)
        mean = x.mean(1)
        rstd = 1 / torch.sqrt(x.var(1, unbiased=False) + EPS)
        if kind == "norm":
            y = torch.addcmul(t["beta"].to(f8), (x - mean[:, None]) / torch.sqrt(x.var(1, unbiased=False) + EPS)[:, None], gamma)
            return y, torch.stack([mean, rstd], 1)
        x.requires_grad_(True)
        gamma, beta = gamma.requires_grad_(True), t["beta"].to(f8).requires_grad_(True)
        m = x.mean(1, keepdim=True)
        c = x - m
        y = c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * gamma + beta
        return dict(zip(("dx", "dgamma", "dbeta"), torch.autograd.grad(y, (x, gamma, beta), t["dy"].to(f8))))
    if kind.startswith("linear"):
        if kind == "linear":
            z = torch.matmul(t["x"].to(f8), t["W"].to(f8))
            if t["b"] is not None:
                z += t["b"].to(f8)
            y = _exact_act(z, case)
            return y if t["res"] is None else y + t["res"].to(f8)
        # the gradient at the pre-activations that the forward pass kept
        x, W, dy = t["x"].to(f8), t["W"].to(f8), t["dy"].to(f8)
        dz = dy
        if case["act"] != "none":
            z = _pre_plain(t).to(_dt(case)).to(f8).requires_grad_(True)
            dz, = torch.autograd.grad(_exact_act(z, case), z, dy)
        out = {"dx": torch.matmul(dz, W.T), "dW": torch.matmul(x.T, dz)}
        return {**out, "db": dz.sum(0)} if case["bias"] else out
    # attention user by user
    h, hk, d = case["h"], case["hk"], case["d"]
    g = h // hk
    n, r = _users(case)
    ends = torch.from_numpy(_ends(case)).to(DEVICE)
    grad = kind == "attn_grad"
    N = t["q"].shape[0]
    out, lse = torch.zeros((N, h, d), dtype=f8, device=DEVICE), torch.full((N, h), -math.inf, dtype=f8, device=DEVICE)
    grads = [torch.zeros(t[x].shape, dtype=f8, device=DEVICE) for x in ("q", "K", "V")] if grad else None
    t0 = i0 = 0
    for L, R in zip(n.tolist(), r.tolist()):
        if L and R:
            rows, toks = slice(i0, i0 + R), slice(t0, t0 + L)
            leaves = [t["q"][rows].to(f8), t["K"][toks].to(f8), t["V"][toks].to(f8)]
            if grad:
                leaves = [x.requires_grad_(True) for x in leaves]
            q, K, V = leaves
            e = ends[rows]
            dist = e[:, None] - 1 - torch.arange(L, device=DEVICE)[None, :]                    # [R, L]
            seen = dist >= 0
            if case["window"]:
                seen = seen & (dist < case["window"])
            some = seen.any(1)
            for c in range(0, hk, max(1, int(1e8 / max(1, R * g * L)))):                       # heads, as memory allows
                hs = slice(c, min(hk, c + max(1, int(1e8 / max(1, R * g * L)))))
                m = hs.stop - hs.start
                qq = q[:, c * g:hs.stop * g].reshape(R, m, g, d).permute(1, 2, 0, 3).reshape(m, g * R, d)
                s = torch.matmul(qq, K[:, hs].permute(1, 2, 0)).view(m, g, R, L) / math.sqrt(d)
                if case["cap"]:
                    s = torch.tanh(s / case["cap"]) * case["cap"]
                if case["bias"]:
                    s = s - t["slopes"][c * g:hs.stop * g].to(f8).view(m, g, 1, 1) * dist
                s = s.masked_fill(~seen, -math.inf).masked_fill(~some[:, None], 0.0)
                a = torch.softmax(s, -1) * some[:, None]
                o = torch.matmul(a.view(m, g * R, L), V[:, hs].permute(1, 0, 2)).view(m, g, R, d).permute(2, 0, 1, 3).reshape(R, m * g, d)
                if grad:
                    part = torch.autograd.grad(o, leaves, t["dout"][rows, c * g:hs.stop * g].to(f8))
                    for whole, at, v in zip(grads, (rows, toks, toks), part):
                        whole[at] += v
                else:
                    out[rows, c * g:hs.stop * g] = o
                    z = torch.where(some, torch.logsumexp(s, -1), -math.inf)                   # [m, g, R]
                    lse[rows, c * g:hs.stop * g] = z.reshape(m * g, R).t()
        t0, i0 = t0 + L, i0 + R
    if grad:
        return dict(zip(("dq", "dK", "dV"), grads))
    return out if case["dtype"] == "bf16" else (out, lse)


def _exact_act(z, case):
    act = case["act"]
    if act == "swiglu":
        F = case["F"]
        return z[:, :F] / (1 + torch.exp(-z[:, :F])) * z[:, F:]
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return torch.relu(z) if act == "relu" else z
