"""The training attention on every way through its launches (training_paths.py), and
at 118,800 tokens on sampled rows and keys, against the definitions in 64 bits within
bounds derived per value."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2608_12780_amd import binding as B  # noqa: E402
from paper_2608_12780_amd.layer import TrainingAttention  # noqa: E402

import gpu_harness as G  # noqa: E402
import training_paths as P  # noqa: E402
import training_reference as R  # noqa: E402

U = R.U


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def run(x, p, rng):
    """Forward and backward, on outputs and a workspace full of other values."""
    H, n, d, C, dtype = x["dims"]
    a = TrainingAttention(H, n, d, C, dtype)
    a.workspace.fill_(0xA5)
    r = torch.tensor(rng, dtype=torch.int64, device="cuda")
    qkv = (x["q"], x["k"], x["v"])
    outs, grads = a.outputs(), a.gradients()
    for t in (*outs, *grads):
        t.fill_(77.0)
    a.forward(*qkv, *R.sets(x), 0.0, p, r, into=outs)
    a.backward(*qkv, *outs, x["d_o"], *R.sets(x), 0.0, p, r, into=grads)
    assert int(a.status.item()) == 0
    return dict(zip(("o", "lse", "dq", "dk", "dv"), (*outs, *grads)))


@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("heads,n,d,dtype,c_q,keep,pattern",
                         P.ORDERED + P.BY_COST + P.BY_COST_PARTS + P.LISTED_PARTS)
def test_every_way(heads, n, d, dtype, c_q, keep, pattern, p):
    G.say(f"[ways] {heads}x{n} d={d} {dtype} c_q={c_q} keep={keep} {pattern} p={p}")
    x = R.make(heads, n, d, dtype, c_q, keep, 8, pattern)
    got = run(x, p, (31, n))
    for h in range(heads) if heads < 10 else (0, heads // 2, heads - 1):
        y = {a: t[h:h + 1] for a, t in x.items() if a != "dims"}
        y["dims"] = (1, n, d, c_q, dtype)
        own = {a: t[h:h + 1] for a, t in got.items()}
        val, tol, held = R.reference(y, p, (31, n), None, own["o"], own["lse"], h)
        for a in ("o", "lse", "dq"):
            R.assert_within(a, own[a], val[a], tol[a], held)
            assert (own[a][~held] == 77.0).all(), a
        for a in ("dk", "dv"):
            R.assert_within(a, own[a], val[a], tol[a])


def make_long(heads, n, d, dtype, c_q, keep):
    """Inputs, random clusters and sets, made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(n + heads)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = {a: torch.randn(heads, n, d, generator=g, device="cuda").to(t)
         for a in ("q", "k", "v", "d_o")}
    i32 = dict(dtype=torch.int32, device="cuda")
    x["perm"] = torch.stack([torch.randperm(n, generator=g, device="cuda")
                             for _ in range(heads)]).to(torch.int32)
    cuts = torch.randint(0, n + 1, (heads, c_q - 1), generator=g, device="cuda").sort(1).values
    x["offsets"] = torch.zeros(heads, c_q + 1, **i32)
    x["offsets"][:, 1:-1] = cuts.int()
    x["offsets"][:, -1] = n
    x["sel_counts"] = torch.zeros(heads, c_q, **i32)
    x["sel_idx"] = torch.full((heads, c_q, n), -1, **i32)
    for h in range(heads):
        for c in range(c_q):
            keys = (torch.rand(n, generator=g, device="cuda") < keep).nonzero()[:, 0].int()
            x["sel_counts"][h, c] = len(keys)
            x["sel_idx"][h, c, :len(keys)] = keys
    x["dims"] = (heads, n, d, c_q, dtype)
    return x


def factors(rows, keys, h, p, rng):
    """The dropout factors of the pairs of some queries and keys of head h."""
    if not R.threshold(p):
        return 1.0
    words = []
    for side, i in enumerate((rows, keys)):
        i = i.cpu().numpy().astype(np.uint64)
        full = lambda v: np.full(len(i), v, np.uint64)
        words.append(R.philox((i, full(0x80000000 + 2 * h + side), full(rng[1] & 0xFFFFFFFF),
                               full(rng[1] >> 32)), rng[0]))
    (a0, a1, *_), (b0, b1, *_) = words
    z = (a0[:, None] ^ b0[None]) * ((a1[:, None] + b1[None]) & R.M32)
    keep = ((((z >> np.uint64(32)) ^ z) & R.M32) >> np.uint64(16)) >= np.uint64(R.threshold(p))
    return torch.from_numpy(keep).cuda() * (65536.0 / (65536 - R.threshold(p)))


def pairs(x, h, rows, keys, p, rng, o, lse):
    """Of some queries and keys of head h: values and error bounds of the logits, of the
    probabilities from the kernel's lse and of ds (training_reference.py derives them)."""
    H, n, d, C, dtype = x["dims"]
    b = R.HALF_STEP["bf16"] if dtype == "bf16" else 0.0
    scale = 1.0 / math.sqrt(d)
    q, g, o = (t[h, rows].double() for t in (x["q"], x["d_o"], o))
    k, v = (x[a][h, keys].double() for a in "kv")
    T = lambda t: t.T.contiguous()
    cluster = torch.empty(n, dtype=torch.long, device="cuda")
    off = x["offsets"][h].tolist()
    member = torch.zeros(C, n, dtype=torch.bool, device="cuda")
    for c in range(C):
        cluster[x["perm"][h, off[c]:off[c + 1]].long()] = c
        member[c, x["sel_idx"][h, c, :int(x["sel_counts"][h, c])].long()] = True
    ok = member[cluster[rows]][:, keys]
    m = factors(rows, keys, h, p, rng)
    s = q @ T(k) * scale
    e_s = ((d + 8) * U * scale * (q.abs() @ T(k.abs())) + 4 * U * s.abs()).masked_fill(~ok, 0.0)
    s = s.masked_fill(~ok, -math.inf)
    L = lse[h, rows].double()
    prob = (s - L[:, None]).exp()
    rel = e_s + (U * (4 * L.abs() + 16))[:, None]
    dp, e_dp = (g @ T(v)) * m, (d + 8) * U * (g.abs() @ T(v.abs())) * m
    D, e_D = (g * o).sum(1, keepdim=True), (d + 8) * U * (g * o).abs().sum(1, keepdim=True)
    ds = prob * (dp - D)
    sums = prob * (e_dp + e_D + 4 * U * (dp.abs() + D.abs()))
    return dict(q=q, k=k, v=v, g=g, m=m, ok=ok, s=s, e_s=e_s, ds=ds,
                e_dk=ds.abs() * (rel + b) + sums, e_dq=ds.abs() * (rel + b * b) + sums,
                pm=prob * m, e_pm=prob * m * (rel + b))


@pytest.mark.parametrize("heads,n,d,dtype,c_q,keep,p", P.LONG)
def test_long_sequences(heads, n, d, dtype, c_q, keep, p):
    G.say(f"[long] {heads}x{n} d={d} {dtype} c_q={c_q} keep={keep} p={p}")
    x, rng = make_long(heads, n, d, dtype, c_q, keep), (77, 2 ** 35 + 1)
    got = run(x, p, rng)
    b, half = (R.HALF_STEP["bf16"],) * 2 if dtype == "bf16" else (0.0, U)
    scale = 1.0 / math.sqrt(d)
    every = torch.arange(n, device="cuda")
    picked = np.random.default_rng(5).choice(n, 30, replace=False)
    some = torch.from_numpy(np.concatenate([[0, 1, 65535, 65536, n - 2, n - 1], picked])).cuda()

    def check(name, value, want, bound):
        R.assert_within(name, value, want, 1.05 * bound + 1e-30)

    T = lambda t: t.T.contiguous()
    for h in sorted({0, heads - 1}):
        z = pairs(x, h, some, every, p, rng, got["o"], got["lse"])
        terms, row = z["ok"].sum(1).double(), z["e_s"].amax(1)
        lse = torch.logsumexp(z["s"], 1)
        prob = (z["s"] - lse[:, None]).exp() * z["m"]
        check("lse", got["lse"][h, some], lse,
              row + (terms + 8) * U + 8 * U * lse.abs() + 8 * U)
        o = prob @ z["v"]
        check("o", got["o"][h, some], o, (prob @ z["v"].abs()) *
              ((2 * row + 16 * U) + b + (terms + 8) * U)[:, None] + half * o.abs())
        dq = scale * (z["ds"] @ z["k"])
        check("dq", got["dq"][h, some], dq, half * dq.abs() + scale * (
            (z["e_dq"] + (terms + 8)[:, None] * U * z["ds"].abs()) @ z["k"].abs()))
        z = pairs(x, h, every, some, p, rng, got["o"], got["lse"])
        per_key = (z["ok"].sum(0).double() + 8)[:, None] * U
        dk = scale * (T(z["ds"]) @ z["q"])
        check("dk", got["dk"][h, some], dk, half * dk.abs() + scale * (
            (T(z["e_dk"]) + per_key * T(z["ds"].abs())) @ z["q"].abs()))
        dv = T(z["pm"]) @ z["g"]
        check("dv", got["dv"][h, some], dv, half * dv.abs() + (
            (T(z["e_pm"]) + per_key * T(z["pm"])) @ z["g"].abs()))
