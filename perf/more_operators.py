"""Performance cases of rotary positions and of attention over packed sequences.

What a program asks of this library before and beside the sparse layer.  The
layer takes queries and keys after their rotary positions: ``rotate`` turns the
projections' queries and keys by them, part of the channels per axis (time,
height and width of a video, or one axis of text), in pairs of neighbours or of
halves, with frequencies stretched for contexts longer than the trained one, and
lays them out by heads; ``rotate_gradient`` turns gradients back into the
projections' layout.  ``forward`` and ``backward`` are exact attention over
sequences of different lengths packed into one array, causal or not, with query
heads in groups that share a key head, and its gradients: clips of several sizes
in one batch, prompts, chunks and single tokens behind a cache.

A case is a dict of plain values:
  kind      rotate | rotate_gradient | forward | backward
  heads, kv_heads, d, dtype (bf16 | f32)
  rotate, rotate_gradient: n (tokens), axes (channels of each axis, from channel 0
            on; the rest stays), layout (pairs | halves), theta, scaling (none |
            linear | base | ramp), stretch, start (the first token's position)
  forward, backward: sequences, tokens (queries of all sequences), spread (the
            longest sequence over the shortest), behind (keys that the longest
            cache holds before the first query, 0: as many keys as queries),
            causal, short (every third sequence has a quarter as many keys as
            queries: rows that the mask leaves empty)

``run`` with ``own`` false computes the formulas with elementary torch
operations; with ``own`` true it makes the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

DEVICE = "cuda"
own = False


def _rotation(name, kind, heads, kv_heads, n, d, axes, layout="pairs", dtype="bf16", theta=10000.0,
              scaling="none", stretch=1.0, start=0):
    c = {"kind": kind, "heads": heads, "kv_heads": kv_heads, "n": n, "d": d, "axes": axes,
         "layout": layout, "dtype": dtype, "theta": theta, "scaling": scaling, "stretch": stretch,
         "start": start}
    return dict(c, name=name) if name else c


def _attention(name, kind, heads, kv_heads, sequences, tokens, spread=1.0, behind=0, d=128,
               dtype="bf16", causal=True, short=False):
    c = {"kind": kind, "heads": heads, "kv_heads": kv_heads, "sequences": sequences,
         "tokens": tokens, "spread": spread, "behind": behind, "d": d, "dtype": dtype,
         "causal": causal, "short": short}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token of each of eight texts, stretched context: the smallest
        # call, where its launch counts
        _rotation("rotate_tokens", "rotate", 16, 4, 8, 128, "128", "halves", theta=500000.0,
                  scaling="ramp", stretch=4.0, start=30000),
        # the queries and keys of a whole 720p layer, from the fused projection
        _rotation("rotate_hy720", "rotate", 24, 24, 118800, 128, "16/56/56"),
        # a long text in fp32, part of each head turned, far positions
        _rotation("rotate_text_f32", "rotate", 8, 2, 20011, 64, "32", "halves", "f32",
                  scaling="linear", stretch=8.0, start=3000000),
        # the gradients of one GPU's share (5 of 40 heads) of the 480p model
        _rotation("rotate_gradient_wan480_share", "rotate_gradient", 5, 5, 32760, 128, "44/42/42"),
        # one new token of each of 16 texts behind caches of up to 8000 keys
        _attention("forward_tokens", "forward", 16, 4, 16, 16, 1.0, 8000),
        # the repository's Tiny size in fp32, three sequences: the smallest prompt
        _attention("forward_tiny_f32", "forward", 2, 1, 3, 256, 4.0, d=64, dtype="f32"),
        # prompts of 22 to 6600 tokens in one batch
        _attention("forward_prompts", "forward", 16, 4, 24, 30011, 300.0),
        # a chunk of 512 tokens of each of four long texts behind their caches
        _attention("forward_chunk", "forward", 16, 4, 4, 2048, 1.0, 16000),
        # the gradients of the Tiny size: the smallest backward
        _attention("backward_tiny", "backward", 2, 1, 3, 256, 4.0, d=64),
        # training on texts of different lengths, d = 64
        _attention("backward_prompts", "backward", 16, 4, 24, 30011, 300.0, d=64),
        # fp32, cross-attention lengths, rows without keys
        _attention("backward_short_f32", "backward", 4, 2, 7, 6417, 5.0, short=True, dtype="f32"),
        # two clips, one GPU's share of the 480p model's dense layer: the largest
        _attention("backward_clips", "backward", 5, 5, 2, 49140, 2.0, causal=False),
    ]


def draw(rng):
    """One more case: any kind, token counts over their logarithm, odd sizes,
    head groups, lengths and caches from a few tokens to many."""
    def size(low, high):
        return round(math.exp(rng.uniform(math.log(low), math.log(high))))

    kind = rng.choice(["rotate", "rotate", "rotate_gradient", "forward", "forward", "forward",
                       "backward", "backward", "backward"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
    if kind.startswith("rotate"):
        n = size(1, 120000)
        d, axes = rng.choice([(128, "16/56/56"), (128, "44/42/42"), (64, "16/24/24"), (64, "64"),
                              (64, "32"), (128, "128"), (128, "64")])
        scaling = rng.choice(["none", "none", "linear", "base", "ramp"])
        return _rotation("", kind, heads, kv_heads, n, d, axes, rng.choice(["pairs", "halves"]),
                         dtype, rng.choice([10000.0, 500000.0]), scaling,
                         1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                         rng.choice([0, 0, size(100, 4000000)]))
    d = 64 if rng.random() < 0.35 else 128
    sequences = size(1, 48)
    if kind == "forward" and rng.random() < 0.5:  # behind a cache
        new = rng.choice([1, 1, 1, 2, 5, 100, 400])
        behind = size(100, 16000)
        sequences = max(1, min(sequences, int(2e9 / (heads * new * behind))))
        return _attention("", kind, heads, kv_heads, sequences, sequences * new, 1.0, behind, d,
                          dtype)
    tokens = max(sequences, size(100, 32000))
    most = 4e8 if dtype == "f32" else 3e9   # elements of the score matrices
    heads, kv_heads = (heads, kv_heads) if heads * tokens ** 2 <= most else (kv_heads, kv_heads)
    tokens = max(sequences, min(tokens, int(math.sqrt(most / heads))))
    return _attention("", kind, heads, kv_heads, sequences, tokens,
                      rng.choice([1.0, 3.0, 30.0, 300.0]), 0, d, dtype, rng.random() < 0.7,
                      rng.random() < 0.2)


# --- sizes --------------------------------------------------------------------

def _lengths(case):
    """(queries, keys) of each sequence, from the case alone."""
    S, total = case["sequences"], case["tokens"]
    weight = [case["spread"] ** (i / max(S - 1, 1)) for i in range(S)]
    random.Random(31 * S + total).shuffle(weight)
    lq = [int(total * w / sum(weight)) for w in weight]
    lq[weight.index(max(weight))] += total - sum(lq)
    if case["behind"]:
        share = [1.0 - 0.9 * i / S for i in range(S)]
        return lq, [n + int(case["behind"] * x) for n, x in zip(lq, share)]
    if case["short"]:
        return lq, [n // 4 if i % 3 == 2 or S == 1 else n for i, n in enumerate(lq)]
    return lq, list(lq)


def _room(case, lk):
    """Rows of K and V that each sequence has: caches have room for more keys."""
    return [(max(lk) + 127) // 128 * 128] * len(lk) if case["behind"] else lk


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _pairs(case):
    """Query-key pairs of one head that the mask leaves."""
    total = 0
    for n, m in zip(*_lengths(case)):
        if not case["causal"]:
            total += n * m
        elif m >= n:      # the last query sees every key
            total += n * (m - n) + n * (n + 1) // 2
        else:
            total += m * (m + 1) // 2
    return total


# --- inputs -----------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _axes(case):
    return [int(x) for x in case["axes"].split("/")]


def _positions(case):
    """[axes][n]: places in a latent grid of about n tokens, or in a text."""
    n, axes = case["n"], len(_axes(case))
    i = torch.arange(n, device=DEVICE)
    if axes == 1:
        p = i[None] * (1 if n > 64 else 997)  # few tokens: of texts of different lengths
    else:
        w = max(1, round((n / 33 * 16 / 9) ** 0.5)) if n > 33 else 4
        h = max(1, round(w * 9 / 16))
        p = torch.stack([i // (h * w), i // w % h, i % w])
    return (p + case["start"]).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    s = {"case": case}
    H, G, d, t = case["heads"], case["kv_heads"], case["d"], _dtype(case)

    def randn(*shape):
        return torch.randn(*shape, generator=g, dtype=torch.float32, device=DEVICE)

    if case["kind"].startswith("rotate"):
        s["positions"] = _positions(case)
        n = case["n"]
        if case["kind"] == "rotate":  # queries and keys are parts of one projection's rows
            rows = randn(n, H + 2 * G, d).to(t)
            s["q"], s["k"] = (x.transpose(0, 1) for x in (rows[:, :H], rows[:, H:H + G]))
        else:
            s["q"], s["k"] = randn(H, n, d).to(t), randn(G, n, d).to(t)
        return s
    lq, lk = _lengths(case)
    room = _room(case, lk)
    s["lq"], s["lk"], s["oq"], s["ok"] = lq, lk, _offsets(lq), _offsets(room)
    i32 = dict(dtype=torch.int32, device=DEVICE)
    s["offsets_q"], s["offsets_k"] = (torch.tensor(x, **i32) for x in (s["oq"], s["ok"]))
    s["lengths_k"] = torch.tensor(lk, **i32) if case["behind"] else None
    # a direction that a group's queries and keys share, slow fields over the
    # tokens, and noise, as trained heads have them
    R, nq, nk = 8, sum(lq), sum(room)
    basis = randn(G, R, d)
    freq = 0.02 * torch.rand(G, R, 1, generator=g, device=DEVICE)
    phase = 2 * math.pi * torch.rand(G, R, 1, generator=g, device=DEVICE)
    common = randn(G, 1, d)

    def fields(n):
        at = torch.arange(n, dtype=torch.float32, device=DEVICE)
        waves = math.sqrt(2.0) * (2 * math.pi * freq * at + phase).cos()
        return (torch.bmm(waves.transpose(1, 2).contiguous(), basis) + common) * (0.8 / 3.0)

    s["k"] = (fields(nk) + 0.6 * randn(G, nk, d)).to(t)
    s["v"] = randn(G, nk, d).to(t)
    s["q"] = (fields(nq).repeat_interleave(H // G, 0) + 0.6 * randn(H, nq, d)).to(t)
    if case["kind"] == "backward":
        s["d_o"] = randn(H, nq, d).to(t)
        s["o"], s["lse"] = _forward(s)
    return s


# --- the plain forms ----------------------------------------------------------

def _frequencies(case, length):
    """Radians per position of each of length / 2 pairs, in 64 bits, and the
    factor on the turned channels."""
    theta, s = case["theta"], case["stretch"]
    if case["scaling"] == "base":   # the slowest pair turns s times slower
        theta *= s ** (length / (length - 2))
    f = theta ** (-torch.arange(0, length, 2, dtype=torch.float64, device=DEVICE) / length)
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "ramp":   # pairs that turn less than once over 4096 tokens fully
        share = ((4096 * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        return f * (share + (1.0 - share) / s), 1.0 + 0.1 * math.log(s)
    return f, 1.0


def _rotate(s, x):
    """x [heads][n][d] turned by its positions (or back), in its type."""
    case = s["case"]
    y, first = x.float(), 0
    parts = []
    for length, p in zip(_axes(case), s["positions"]):
        f, factor = _frequencies(case, length)
        angle = p.double()[:, None] * f
        c, n = (angle.cos() * factor).float(), (angle.sin() * factor).float()
        if case["kind"] == "rotate_gradient":
            n = -n
        z = y[..., first:first + length]
        if case["layout"] == "pairs":
            a, b = z[..., 0::2], z[..., 1::2]
            parts.append(torch.stack((a * c - b * n, a * n + b * c), -1).flatten(-2))
        else:
            a, b = z[..., :length // 2], z[..., length // 2:]
            parts += [a * c - b * n, a * n + b * c]
        first += length
    return torch.cat((*parts, y[..., first:]), -1).to(x.dtype)


def _masked(x, causal):
    """Scores [..., queries, keys] with -inf behind the last key that a query sees:
    the last query sees every key."""
    n, m = x.shape[-2:]
    if not causal:
        return x
    i, j = torch.arange(n, device=DEVICE)[:, None], torch.arange(m, device=DEVICE)
    return x.masked_fill_(j > i + (m - n), -math.inf)


def _softmax(x):
    """Weights and log-sum-exp of the last axis; rows of -inf have weights 0."""
    top = x.amax(-1, keepdim=True) if x.shape[-1] else x.new_full((*x.shape[:-1], 1), -math.inf)
    x = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    return x.div_(torch.where(total == 0.0, 1.0, total)), (top + total.log())[..., 0]


def _tokens(s):
    """A few queries of every sequence: all sequences at once, their keys padded."""
    case = s["case"]
    S, H, G, d = case["sequences"], case["heads"], case["kv_heads"], case["d"]
    n, m = case["tokens"] // S, max(s["lk"])
    lk = s["lengths_k"].long()[:, None]
    j = torch.arange(m, device=DEVICE)
    at = s["offsets_k"][:-1].long()[:, None] + j
    k, v = (x[:, at].float().reshape(G * S, m, d) for x in (s["k"], s["v"]))
    q = s["q"].float().reshape(G, H // G, S, n, d).transpose(1, 2).reshape(G * S, -1, d)
    x = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(d))
    x = x.view(G, S, H // G, n, m)
    seen = j <= (lk - n + torch.arange(n, device=DEVICE))[..., None]
    x, lse = _softmax(x.masked_fill_(~seen[:, None], -math.inf))
    o = torch.bmm(x.view(G * S, -1, m), v).view(G, S, H // G, n, d)
    return (o.transpose(1, 2).reshape(H, S * n, d).to(_dtype(case)),
            lse.transpose(1, 2).reshape(H, S * n))


def _sequence(s, i):
    """The rows of sequence i: slices of queries and of keys."""
    return slice(s["oq"][i], s["oq"][i + 1]), slice(s["ok"][i], s["ok"][i] + s["lk"][i])


def _scores(s, rows, keys):
    """[key head][its query heads and their queries][keys] scaled scores, masked."""
    case = s["case"]
    q, k = s["q"][:, rows].float(), s["k"][:, keys].float()
    H, n, d = q.shape
    G, m, _ = k.shape
    x = torch.bmm(q.reshape(G, H // G * n, d), k.transpose(1, 2).contiguous())
    return _masked(x.mul_(1.0 / math.sqrt(d)).view(H, n, m), case["causal"]).view_as(x)


def _forward(s):
    """O and the rows' log-sum-exp: sequence by sequence, or with few queries at once."""
    case = s["case"]
    H, d, n = case["heads"], case["d"], case["tokens"]
    if case["behind"] and n <= 64 * case["sequences"] and case["spread"] == 1.0:
        return _tokens(s)
    o = torch.empty(H, n, d, dtype=_dtype(case), device=DEVICE)
    lse = torch.empty(H, n, dtype=torch.float32, device=DEVICE)
    for i in range(case["sequences"]):
        rows, keys = _sequence(s, i)
        x, total = _softmax(_scores(s, rows, keys))
        o[:, rows] = torch.bmm(x, s["v"][:, keys].float()).view(H, s["lq"][i], d).to(o.dtype)
        lse[:, rows] = total.view(H, s["lq"][i])
    return o, lse


def _backward(s):
    """dQ, dK, dV from the forward's O and log-sum-exp."""
    case, t = s["case"], _dtype(s["case"])
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    dq, dk, dv = (torch.empty_like(s[x]) for x in "qkv")
    for i in range(case["sequences"]):
        rows, keys = _sequence(s, i)
        m = H // G * s["lq"][i]
        q, o, d_o = (s[x][:, rows].float().reshape(G, m, d) for x in ("q", "o", "d_o"))
        k, v = s["k"][:, keys].float(), s["v"][:, keys].float()
        lse = s["lse"][:, rows].reshape(G, m, 1)
        prob = _scores(s, rows, keys).sub_(torch.where(lse == -math.inf, 0.0, lse)).exp_()
        dv[:, keys] = torch.bmm(prob.transpose(1, 2).contiguous(), d_o).to(t)
        d_s = torch.bmm(d_o, v.transpose(1, 2).contiguous())
        d_s = d_s.sub_((d_o * o).sum(2, keepdim=True)).mul_(prob).mul_(1.0 / math.sqrt(d))
        dq[:, rows] = torch.bmm(d_s, k).view(H, s["lq"][i], d).to(t)
        dk[:, keys] = torch.bmm(d_s.transpose(1, 2).contiguous(), q).to(t)
    return dq, dk, dv


def _named(kind, outputs):
    names = {"forward": ("o", "lse"), "backward": ("dq", "dk", "dv")}.get(kind, ("q", "k"))
    return dict(zip(names, outputs))


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _named(kind, _run_own(s))
    if kind == "forward":
        return _named(kind, _forward(s))
    if kind == "backward":
        return _named(kind, _backward(s))
    return _named(kind, (_rotate(s, s["q"]), _rotate(s, s["k"])))


# --- the library's calls -------------------------------------------------------

def _run_own(s):
    from paper_2608_12780_amd import packed, rotary

    case = s["case"]
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    if case["kind"].startswith("rotate"):
        n, back = case["n"], case["kind"] == "rotate_gradient"
        if "rotary" not in s:  # what a program keeps: the frequencies, and its buffers
            scaling = None if case["scaling"] == "none" else (case["scaling"], case["stretch"])
            s["rotary"] = rotary.Rotary(d, _axes(case), theta=case["theta"],
                                        layout=case["layout"], scaling=scaling, context=4096,
                                        device=DEVICE)
            if back:  # the projection's gradient, of which V's part is not written here
                rows = torch.zeros(n, H + 2 * G, d, dtype=_dtype(case), device=DEVICE)
                s["out"] = tuple(x.transpose(0, 1) for x in (rows[:, :H], rows[:, H:H + G]))
            else:
                s["out"] = (torch.empty(H, n, d, dtype=_dtype(case), device=DEVICE),
                            torch.empty(G, n, d, dtype=_dtype(case), device=DEVICE))
        return s["rotary"].rotate(s["q"], s["positions"], s["k"], out=s["out"], inverse=back)
    if "attention" not in s:  # the buffers that a program keeps
        s["attention"] = packed.PackedAttention(H, G, s["oq"][-1], s["ok"][-1], d,
                                                case["sequences"], causal=case["causal"],
                                                dtype=case["dtype"], device=DEVICE)
    if case["kind"] == "forward":
        return s["attention"].forward(s["q"], s["k"], s["v"], s["offsets_q"], s["offsets_k"],
                                      lengths_k=s["lengths_k"])
    return s["attention"].backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["d_o"],
                                   s["offsets_q"], s["offsets_k"])


# --- what a pass cannot do without ---------------------------------------------

def work(case):
    el = 2.0 if case["dtype"] == "bf16" else 4.0
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    if case["kind"].startswith("rotate"):
        values = float(H + G) * case["n"] * d
        turned = sum(_axes(case)) / d
        return {"bytes": 2 * values * el + 4.0 * case["n"] * len(_axes(case)),
                "flops": 3.0 * values * turned}
    lq, lk = _lengths(case)
    rows, keys = float(H * sum(lq) * d), float(G * sum(lk) * d)
    pairs = float(H) * _pairs(case)
    if case["kind"] == "forward":   # two products; Q, K, V in, O and the statistics out
        return {"bytes": el * 2 * (rows + keys) + 4.0 * H * sum(lq), "flops": 4.0 * d * pairs}
    # five products; Q, K, V, O, dO and the statistics in, dQ, dK, dV out
    return {"bytes": el * 4 * (rows + keys) + 4.0 * H * sum(lq), "flops": 10.0 * d * pairs}


# --- the same in 64 bits --------------------------------------------------------

def _turned64(case, positions, x):
    """Pairs of channels as complex numbers, times unit ones (turned back: their
    conjugates)."""
    z, at = x.double().clone(), 0
    s, back = case["stretch"], case["kind"] == "rotate_gradient"
    for a, length in enumerate(_axes(case)):
        i = torch.arange(length // 2, dtype=torch.float64, device=DEVICE)
        base = case["theta"] * (s ** (length / (length - 2)) if case["scaling"] == "base" else 1.0)
        speed, size = torch.exp(-2.0 * i / length * math.log(base)), 1.0
        if case["scaling"] == "linear":
            speed = speed / s
        elif case["scaling"] == "ramp":
            turns = 4096 * speed / (2 * math.pi)
            kept = torch.clamp((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
            speed, size = speed * kept + speed / s * (1.0 - kept), 1.0 + 0.1 * math.log(s)
        angle = positions[a].double()[:, None] * speed * (-1.0 if back else 1.0)
        unit = torch.polar(torch.full_like(angle, size), angle)
        lo, hi = ((z[..., at:at + length:2], z[..., at + 1:at + length:2])
                  if case["layout"] == "pairs" else
                  (z[..., at:at + length // 2], z[..., at + length // 2:at + length]))
        w = torch.complex(lo.contiguous(), hi.contiguous()) * unit
        lo.copy_(w.real)
        hi.copy_(w.imag)
        at += length
    return z


def exact(case, seed):
    s = prepare(case, seed)
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    if case["kind"].startswith("rotate"):
        return {x: _turned64(case, s["positions"], s[x]) for x in "qk"}
    f64 = dict(dtype=torch.float64, device=DEVICE)
    n, grads = case["tokens"], case["kind"] == "backward"
    scale, group = 1.0 / math.sqrt(d), H // G
    if grads:
        out = [torch.zeros(H, n, d, **f64), *(torch.zeros(s["k"].shape, **f64) for _ in "kv")]
    else:
        out = [torch.zeros(H, n, d, **f64), torch.full((H, n), -math.inf, **f64)]
    for h in range(H):
        for i, (lq, lk) in enumerate(zip(s["lq"], s["lk"])):
            first, keys = s["oq"][i], slice(s["ok"][i], s["ok"][i] + lk)
            k, v = s["k"][h // group, keys].double(), s["v"][h // group, keys].double()
            for a in range(0, lq, 4096):
                m = min(4096, lq - a)
                rows = slice(first + a, first + a + m)
                last = a + torch.arange(m, device=DEVICE) + lk - lq   # the last key seen
                hidden = torch.arange(lk, device=DEVICE) > last[:, None]
                empty = (last < 0) if case["causal"] else torch.full_like(last, lk == 0) > 0
                if not lk:
                    continue
                x = (s["q"][h, rows].double() @ k.T) * scale
                if case["causal"]:
                    x = x.masked_fill(hidden, -math.inf)
                if not grads:
                    top = torch.where(empty, 0.0, x.amax(1))[:, None]
                    e = torch.exp(x - top)
                    total = e.sum(1)
                    out[1][h, rows] = torch.where(empty, -math.inf, top[:, 0] + total.log())
                    out[0][h, rows] = (e @ v) / torch.where(empty, 1.0, total)[:, None]
                    continue
                lse = torch.where(empty, 0.0, s["lse"][h, rows].double())
                p = torch.exp(x - lse[:, None])
                g, o = s["d_o"][h, rows].double(), s["o"][h, rows].double()
                d_x = p * (g @ v.T - (g * o).sum(1, keepdim=True)) * scale
                out[0][h, rows] = d_x @ k
                out[1][h // group, keys] += d_x.T @ s["q"][h, rows].double()
                out[2][h // group, keys] += p.T @ g
    return _named(case["kind"], out)
