"""The training operators in 64 bits from their definitions, with a bound on
the error of every output value, and cases to try them on.  Imported only by
tests."""
from __future__ import annotations

import math

import numpy as np
import torch

U = 2.0 ** -24                                  # half a step of fp32
HALF_STEP = {"bf16": 2.0 ** -8, "f32": U}
M32 = np.uint64(0xFFFFFFFF)


# --- random numbers -----------------------------------------------------------

def philox(counter, seed):
    """Philox4x32-10; counter: four uint64 arrays of 32-bit values."""
    c = [np.asarray(x, np.uint64) for x in counter]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & M32, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + np.uint64(0x9E3779B9)) & M32, (k[1] + np.uint64(0xBB67AE85)) & M32]
    return c


def threshold(p):
    return min(65535, round(float(np.float32(p)) * 65536))


def keep_pairs(heads, n, p, seed, offset, head=0):
    """[heads][n][n] bool: the pairs that attention dropout keeps, from `head` on."""
    i = np.arange(n, dtype=np.uint64)
    lo, hi = np.full(n, offset & 0xFFFFFFFF, np.uint64), np.full(n, offset >> 32, np.uint64)
    out = np.empty((heads, n, n), bool)
    for h in range(heads):
        a, b = (philox((i, np.full(n, 0x80000000 + 2 * (head + h) + side, np.uint64), lo, hi), seed)
                for side in (0, 1))
        z = (a[0][:, None] ^ b[0][None]) * ((a[1][:, None] + b[1][None]) & M32)
        out[h] = ((((z >> np.uint64(32)) ^ z) & M32) >> np.uint64(16)) >= np.uint64(threshold(p))
    return out


def keep_elements(count, p, seed, offset):
    g = np.arange((count + 7) // 8, dtype=np.uint64)
    w = philox((g & M32, g >> np.uint64(32), np.full_like(g, offset & 0xFFFFFFFF),
                np.full_like(g, offset >> 32)), seed)
    half = np.stack([x for word in w for x in (word & np.uint64(0xFFFF), word >> np.uint64(16))], 1)
    return half.reshape(-1)[:count] >= np.uint64(threshold(p))


# --- cases ---------------------------------------------------------------------

def make(heads, n, d, dtype, c_q, keep, seed=0, pattern="", device="cuda", scale_q=1.0):
    """Inputs with random clusters and key sets of a mean share `keep`.
    Patterns: "empty" (a cluster without keys, one without queries), "single"
    (one key per cluster), "uncovered" (a tail of queries in no cluster),
    "prefix" (every set the first keys), "last" (only the last key)."""
    g = np.random.default_rng([seed, heads, n, d, c_q])
    x = {a: torch.from_numpy(g.standard_normal((heads, n, d)).astype(np.float32) * s).to(
        torch.bfloat16 if dtype == "bf16" else torch.float32)
        for a, s in (("q", scale_q), ("k", 1.0), ("v", 1.0), ("d_o", 1.0))}
    offsets = np.zeros((heads, c_q + 1), np.int32)
    perm = np.empty((heads, n), np.int32)
    counts = np.empty((heads, c_q), np.int32)
    sel = np.full((heads, c_q, n), -1, np.int32)
    for h in range(heads):
        perm[h] = g.permutation(n)
        cuts = np.sort(g.integers(0, n + 1, c_q - 1)) if c_q > 1 else np.empty(0, int)
        if pattern == "empty" and c_q > 2:
            cuts[1] = cuts[0]                      # cluster 1 has no queries
        offsets[h] = np.concatenate([[0], cuts, [n - n // 3 if pattern == "uncovered" else n]])
        offsets[h] = np.minimum(offsets[h], offsets[h, -1])
        for c in range(c_q):
            r = n if keep >= 1.0 else int(np.clip(round(n * keep * g.uniform(0.5, 1.5)), 1, n))
            if pattern in ("single", "last"):
                r = 1
            if pattern == "empty" and c == 0:
                r = 0
            counts[h, c] = r
            keys = (np.arange(r) if pattern == "prefix" else np.array([n - 1])[:r]
                    if pattern == "last" else np.sort(g.choice(n, r, replace=False)))
            sel[h, c, :r] = keys
    x.update(offsets=torch.from_numpy(offsets), perm=torch.from_numpy(perm),
             sel_counts=torch.from_numpy(counts), sel_idx=torch.from_numpy(sel))
    x = {a: t.to(device) for a, t in x.items()}
    x["dims"] = (heads, n, d, c_q, dtype)
    return x


SETS = ("offsets", "perm", "sel_counts", "sel_idx")


def sets(x):
    return tuple(x[a] for a in SETS)


def allowed(x):
    """[heads][n][n] bool (query, key), and [heads][n] whether a cluster holds the query."""
    H, n, _, C, _ = x["dims"]
    off, perm, cnt, sel = (x[a].cpu().numpy() for a in SETS)
    ok, held = np.zeros((H, n, n), bool), np.zeros((H, n), bool)
    for h in range(H):
        for c in range(C):
            rows = perm[h, off[h, c]:off[h, c + 1]]
            held[h, rows] = True
            ok[h, rows[:, None], sel[h, c, :cnt[h, c]][None]] = True
    return ok, held


# --- forward and backward with error bounds ---------------------------------------

def reference(x, p=0.0, rng=(0, 0), scale=None, o=None, lse=None, head=0):
    """(values, bounds): dicts of float64 tensors for o and lse, and given the
    kernel's o and lse (which the gradients start from) dq, dk and dv.

    The bounds follow the calls' contract.  With u = 2^-24 and b half a step of
    the operands (2^-8 for bf16, 0 for fp32 where the products do not round):
      s      a sum of d products of exact operands, each addition off by u:
             (d + 8) u scale |q| |k|, and 4 u |s| for the scaling and exponent
      p      relative 2 max_j E_s + 16 u in the forward (the normaliser carries
             the same errors), E_s + u (4 |lse| + 16) in the backward
      o      sum of r terms p m v: p's error, b for p as an operand, (r + 8) u
             for the sum, and half a step of the output
      ds     p's error times |dp - D|, p times the errors of the sums dp and D,
             b for ds as an operand
      dq, dk sums of the ds' errors, (terms + 8) u for the sum, half a step; dq's
             ds are two operands, the second the first's rounding error, so b^2"""
    H, n, d, _, dtype = x["dims"]
    dev = x["q"].device
    b, half = (HALF_STEP["bf16"], HALF_STEP["bf16"]) if dtype == "bf16" else (0.0, U)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    q, k, v, g = (x[a].double() for a in ("q", "k", "v", "d_o"))
    ok, held = (torch.from_numpy(a).to(dev) for a in allowed(x))
    m = torch.ones(H, n, n, dtype=torch.float64, device=dev)
    if threshold(p):
        m = torch.from_numpy(keep_pairs(H, n, p, *rng, head)).to(dev) * (65536.0 / (65536 - threshold(p)))
    T = lambda t: t.transpose(1, 2).contiguous()
    mm = torch.matmul
    s = mm(q, T(k)) * scale
    e_s = (d + 8) * U * scale * mm(q.abs(), T(k.abs())) + 4 * U * s.abs()
    s = s.masked_fill(~ok, -math.inf)
    e_s = e_s.masked_fill(~ok, 0.0)
    val, tol = {}, {}
    some = ok.any(2)
    lse64 = torch.where(some, torch.logsumexp(s, 2), -math.inf)
    prob = torch.where(ok, (s - torch.where(some, lse64, 0.0)[..., None]).exp(), 0.0)
    terms = ok.sum(2).double()
    row = e_s.amax(2)
    val["lse"] = lse64
    tol["lse"] = torch.where(some, row + (terms + 8) * U + 8 * U * lse64.nan_to_num(neginf=0.0).abs() + 8 * U, 0.0)
    weight = mm(prob * m, v.abs())
    val["o"] = mm(prob * m, v)
    tol["o"] = weight * ((2 * row + 16 * U) + b + (terms + 8) * U)[..., None] + half * val["o"].abs()
    if o is not None:
        o, lse = o.double(), lse.double()
        prob = torch.where(ok, (s - torch.where(some, lse, 0.0)[..., None]).exp(), 0.0)
        rel = e_s + (U * (4 * torch.where(some, lse, 0.0).abs() + 16))[..., None]
        dp = mm(g, T(v)) * m
        e_dp = (d + 8) * U * mm(g.abs(), T(v.abs())) * m
        D, e_D = (g * o).sum(2, keepdim=True), (d + 8) * U * (g * o).abs().sum(2, keepdim=True)
        live = held[..., None]
        D, e_D = torch.where(live, D, 0.0), torch.where(live, e_D, 0.0)
        ds = prob * (dp - D)
        e_ds = ds.abs() * (rel + b) + prob * (e_dp + e_D + 4 * U * (dp.abs() + D.abs()))
        e_dq = ds.abs() * (rel + b * b) + prob * (e_dp + e_D + 4 * U * (dp.abs() + D.abs()))
        per_key = ok.sum(1).double()
        val["dq"] = scale * mm(ds, k)
        tol["dq"] = scale * mm(e_dq + (terms + 8)[..., None] * U * ds.abs(), k.abs()) + half * val["dq"].abs()
        val["dk"] = scale * mm(T(ds), q)
        tol["dk"] = scale * mm(T(e_ds) + (per_key + 8)[..., None] * U * T(ds.abs()), q.abs()) + half * val["dk"].abs()
        pm = prob * m
        e_pm = pm * (rel + b)
        val["dv"] = mm(T(pm), g)
        tol["dv"] = mm(T(e_pm) + (per_key + 8)[..., None] * U * T(pm), g.abs()) + half * val["dv"].abs()
    # second-order terms of the bounds; values below the smallest normal number
    # may be flushed to zero
    return val, {a: 1.05 * t + 1e-30 for a, t in tol.items()}, held


def assert_within(name, got, want, bound, held=None):
    got = got.double()
    if held is not None:
        h = held if got.dim() == 2 else held[..., None].expand_as(got)
        got, want, bound = got[h], want[h], bound[h]
    if not got.numel():
        return
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), name
    off = (got - want).abs()[~inf] / bound[~inf]
    worst = float(off.max()) if off.numel() else 0.0
    assert not torch.isnan(got).any(), name
    assert worst <= 1.0, f"{name}: {worst:.3g} times the bound"
