"""Attention over packed sequences and rotary positions in 64 bits from their
definitions, with a bound on the error of every output value, and cases to try
them on.  Imported only by tests."""
from __future__ import annotations

import math

import numpy as np
import torch

U = 2.0 ** -24                                  # half a step of fp32
HALF_STEP = {"bf16": 2.0 ** -8, "f32": U}
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(H, G, lq, lk, d, dtype, seed=0, before=0, after=0, room=0, scale_q=1.0, device="cuda"):
    """Sequences of lq[i] queries and lk[i] keys; `before` and `after` rows in no
    sequence, `room` more key rows than each sequence has keys."""
    g = torch.Generator().manual_seed(seed)
    oq, ok = [before], [before]
    for a, b in zip(lq, lk):
        oq.append(oq[-1] + a)
        ok.append(ok[-1] + b + room)
    nq, nk = oq[-1] + after, ok[-1] + after
    t = DTYPE[dtype]
    x = {"dims": (H, G, d, dtype), "lq": list(lq), "lk": list(lk), "oq": oq, "ok": ok,
         "rows": (nq, nk)}
    for name, shape, scale in (("q", (H, nq, d), scale_q), ("k", (G, nk, d), 1.0),
                               ("v", (G, nk, d), 1.0), ("d_o", (H, nq, d), 1.0)):
        x[name] = (scale * torch.randn(shape, generator=g)).to(device).to(t)
    i32 = dict(dtype=torch.int32, device=device)
    x["offsets_q"], x["offsets_k"] = torch.tensor(oq, **i32), torch.tensor(ok, **i32)
    x["lengths_k"] = torch.tensor(list(lk), **i32)
    return x


def inside(x):
    """Which query and key rows are in a sequence."""
    (nq, nk), dev = x["rows"], x["q"].device
    a, b = torch.zeros(nq, dtype=torch.bool, device=dev), torch.zeros(nk, dtype=torch.bool, device=dev)
    a[x["oq"][0]:x["oq"][-1]] = True
    for s, n in zip(x["ok"], x["lk"]):
        b[s:s + n] = True
    return a, b


def reference(x, causal, scale=None, o=None, lse=None):
    """(values, bounds): float64 tensors for o and lse, and given the kernel's o and
    lse (which the gradients start from) dq, dk and dv; rows in no sequence are 0
    (lse: -inf).

    With u = 2^-24 and b half a step of the operands (2^-8 for bf16, 0 for fp32
    where the products do not round):
      s      a sum of d products of exact operands, each addition off by u:
             (d + 8) u scale |q| |k|, and 4 u |s| for the scaling and exponent
      p      relative 2 max_j E_s + 16 u in the forward (the normaliser carries
             the same errors), E_s + u (4 |lse| + 16) in the backward
      o      sum of r terms p v: p's error, b for p as an operand, (r + 8) u for
             the sum, and half a step of the output
      ds     p's error times |dp - D|, p times the errors of the sums dp and D,
             b for ds as an operand
      dq, dk sums of the ds' errors, (terms + 8) u for the sum, half a step; dq's
             ds are two operands, the second the first's rounding error, so b^2"""
    H, G, d, dtype = x["dims"]
    dev, group = x["q"].device, H // G
    b, half = (HALF_STEP["bf16"], HALF_STEP["bf16"]) if dtype == "bf16" else (0.0, U)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    nq, nk = x["rows"]
    f64 = dict(dtype=torch.float64, device=dev)
    val = {"o": torch.zeros(H, nq, d, **f64), "lse": torch.full((H, nq), -math.inf, **f64)}
    tol = {"o": torch.zeros(H, nq, d, **f64), "lse": torch.zeros(H, nq, **f64)}
    if o is not None:
        for t in (val, tol):
            t["dq"] = torch.zeros(H, nq, d, **f64)
            t["dk"], t["dv"] = (torch.zeros(G, nk, d, **f64) for _ in "kv")
    for i, (n, m) in enumerate(zip(x["lq"], x["lk"])):
        if not n or not m:
            continue
        rows, keys = slice(x["oq"][i], x["oq"][i + 1]), slice(x["ok"][i], x["ok"][i] + m)
        seen = torch.ones(n, m, dtype=torch.bool, device=dev)
        if causal:
            seen = torch.arange(m, device=dev) <= (torch.arange(n, device=dev) + m - n)[:, None]
        some, terms = seen.any(1), seen.sum(1).double()
        for h in range(H):
            k, v = x["k"][h // group, keys].double(), x["v"][h // group, keys].double()
            q, g = x["q"][h, rows].double(), x["d_o"][h, rows].double()
            s = (q @ k.T) * scale
            e_s = (d + 8) * U * scale * (q.abs() @ k.abs().T) + 4 * U * s.abs()
            s, e_s = s.masked_fill(~seen, -math.inf), e_s.masked_fill(~seen, 0.0)
            lse64 = torch.where(some, torch.logsumexp(s, 1), -math.inf)
            top = torch.where(some, lse64, 0.0)
            prob = torch.where(seen, (s - top[:, None]).exp(), 0.0)
            row = e_s.amax(1)
            val["lse"][h, rows] = lse64
            tol["lse"][h, rows] = torch.where(some, row + (terms + 8) * U + 8 * U * top.abs() + 8 * U, 0.0)
            y = prob @ v
            val["o"][h, rows] = y
            tol["o"][h, rows] = (prob @ v.abs()) * (2 * row + 16 * U + b + (terms + 8) * U)[:, None] + half * y.abs()
            if o is None:
                continue
            oo = o[h, rows].double()
            L = torch.where(some, lse[h, rows].double(), 0.0)
            prob = torch.where(seen, (s - L[:, None]).exp(), 0.0)
            rel = e_s + (U * (4 * L.abs() + 16))[:, None]
            dp, e_dp = g @ v.T, (d + 8) * U * (g.abs() @ v.abs().T)
            D, e_D = (g * oo).sum(1, keepdim=True), (d + 8) * U * (g * oo).abs().sum(1, keepdim=True)
            ds = prob * (dp - D)
            sums = prob * (e_dp + e_D + 4 * U * (dp.abs() + D.abs()))
            e_ds, e_dq = ds.abs() * (rel + b) + sums, ds.abs() * (rel + b * b) + sums
            per_key = group * n
            y = scale * (ds @ k)
            val["dq"][h, rows] = y
            tol["dq"][h, rows] = scale * ((e_dq + (terms + 8)[:, None] * U * ds.abs()) @ k.abs()) + half * y.abs()
            val["dk"][h // group, keys] += scale * (ds.T @ q)
            tol["dk"][h // group, keys] += scale * ((e_ds + (per_key + 8) * U * ds.abs()).T @ q.abs())
            val["dv"][h // group, keys] += prob.T @ g
            tol["dv"][h // group, keys] += (prob * (rel + b) + (per_key + 8) * U * prob).T @ g.abs()
    for a in ("dk", "dv") if o is not None else ():
        tol[a] += half * val[a].abs()
    # second-order terms of the bounds; values below the smallest normal number
    # may be flushed to zero
    return val, {a: 1.05 * t + 1e-30 for a, t in tol.items()}


def assert_within(name, got, want, bound):
    got = got.double()
    if not got.numel():
        return
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), name
    assert not torch.isnan(got).any(), name
    off = (got - want).abs()[~inf] / bound[~inf]
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} times the bound"


def rotated(x, positions, turns, ranges, layout, factor=1.0, inverse=False):
    """(values, bounds) of a rotation, from its frequencies in units of 2^-64 turns:
    sines and cosines are off by 2^-22, their products with the factor and the pair's
    values by three roundings, and the result is rounded once."""
    half = HALF_STEP["bf16"] if x.dtype == torch.bfloat16 else U
    val = x.double().cpu().clone()
    tol = torch.full_like(val, 1e-37)   # copied channels: off by nothing, and 0 / 0 is no bound
    at = 0
    p = positions.cpu().numpy().reshape(len(ranges[0]), -1).astype(np.int64).view(np.uint64)
    w = turns.cpu().numpy().view(np.uint64)
    for a, (off, n) in enumerate(zip(*ranges)):
        with np.errstate(over="ignore"):
            turn = (p[a][:, None] * w[at:at + n // 2][None]).astype(np.float64) * 2.0 ** -64
        t = torch.from_numpy(2 * math.pi * turn * (-1 if inverse else 1))
        c, s = t.cos() * factor, t.sin() * factor
        i, j = ((slice(off, off + n, 2), slice(off + 1, off + n, 2)) if layout == "pairs" else
                (slice(off, off + n // 2), slice(off + n // 2, off + n)))
        u, v = x[..., i].double().cpu(), x[..., j].double().cpu()
        err = (u.abs() + v.abs()) * abs(factor) * (2.0 ** -22 + 4 * U)
        for where, y in ((i, u * c - v * s), (j, u * s + v * c)):
            val[..., where] = y
            tol[..., where] = err + half * y.abs() + 1e-37
        at += n // 2
    return val, tol
