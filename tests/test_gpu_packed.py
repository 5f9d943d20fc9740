"""Attention over packed sequences against its definition in 64 bits with derived
bounds: lengths from none to hundreds of sequences, head groups, rows that see no
key, parts, strides, caches, masked places that hold NaN, bad offsets, and the calls
as programs make them."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2608_12780_amd import binding as B  # noqa: E402
from paper_2608_12780_amd import layer, packed, rotary  # noqa: E402

import gpu_harness as G  # noqa: E402
import packed_reference as R  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def attention_of(x, causal, workspace=True, **kw):
    H, kv, d, dtype = x["dims"]
    return packed.PackedAttention(H, kv, *x["rows"], d, len(x["lq"]), causal, dtype,
                                  workspace=workspace, **kw)


def check(x, causal, cache=False, scale=0.0, grads=True):
    """Forward and backward within the bounds, twice the same bits, rows in no sequence
    as they were."""
    H, kv, d, dtype = x["dims"]
    a = attention_of(x, causal)
    lengths = x["lengths_k"] if cache else None
    qkv, off = (x["q"], x["k"], x["v"]), (x["offsets_q"], x["offsets_k"])
    used_q, used_k = R.inside(x)
    out = [torch.full_like(t, 7.0) for t in a.outputs()]
    a.forward(*qkv, *off, lengths_k=lengths, scale=scale, into=out)
    torch.cuda.synchronize()
    val, tol = R.reference(x, causal, scale or None)
    for name, got in zip(("o", "lse"), out):
        assert (got[:, ~used_q] == 7.0).all(), name
        R.assert_within(name, got[:, used_q], val[name][:, used_q], tol[name][:, used_q])
    again = a.forward(*qkv, *off, lengths_k=lengths, scale=scale, into=a.outputs())
    assert all(torch.equal(g[:, used_q], o[:, used_q]) for g, o in zip(again, out))
    assert int(a.status) == 0
    if not grads or cache:
        return
    into = [torch.full_like(t, 7.0) for t in a.gradients()]
    # rows in no sequence are not read
    o, lse, d_o = (t.clone() for t in (*out, x["d_o"]))
    for t in (o, lse, d_o):
        t[:, ~used_q] = math.nan
    a.backward(*qkv, o, lse, d_o, *off, scale=scale, into=into)
    torch.cuda.synchronize()
    val, tol = R.reference(x, causal, scale or None, *out)
    for name, got, used in zip(("dq", "dk", "dv"), into, (used_q, used_k, used_k)):
        assert (got[:, ~used] == 7.0).all(), name
        R.assert_within(name, got[:, used], val[name][:, used], tol[name][:, used])
    again = a.backward(*qkv, *out, x["d_o"], *off, scale=scale, into=a.gradients())
    for g, o, used in zip(again, into, (used_q, used_k, used_k)):
        assert torch.equal(g[:, used], o[:, used])
    assert int(a.status) == 0


LENGTHS = {
    "one": ([1], [1]),
    "same": ([130, 7, 257, 64], [130, 7, 257, 64]),
    "empty": ([0, 5, 0, 33, 0], [0, 5, 0, 33, 0]),
    "no_keys": ([9, 40, 3], [0, 70, 0]),
    "no_queries": ([0, 40, 0], [50, 70, 1]),
    "short": ([200, 40, 65], [10, 39, 1]),          # rows that see no key
    "chunks": ([33, 3, 128], [500, 230, 129]),
    "tokens": ([1] * 9, [64, 65, 1, 63, 700, 128, 2, 300, 127]),
    "parts": ([37], [3001]),
    "few": ([2, 1, 3, 1], [1500, 900, 3, 2100]),    # a block's waves share out the keys
    "few_ragged": ([90, 1, 0, 4], [200, 700, 5, 3]),
    "long": ([1200], [1100]),
    "seventy": ([i % 5 for i in range(70)], [(3 * i) % 7 for i in range(70)]),
}


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("heads", [(2, 2), (4, 1), (6, 2)], ids=["2of2", "4of1", "6of2"])
@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32")])
def test_lengths(d, dtype, lengths, heads, causal):
    G.say(f"[packed] {dtype} d={d} {lengths} {heads} causal={causal}")
    check(R.make(*heads, *LENGTHS[lengths], d, dtype, seed=len(lengths), before=3, after=5), causal)


@pytest.mark.parametrize("d,dtype,heads", [(128, "bf16", (8, 1)), (64, "bf16", (3, 3)), (128, "f32", (5, 1))])
def test_many_sequences(d, dtype, heads):
    """More sequences than a list's block has threads."""
    lq = [(7 * i) % 4 for i in range(1100)]
    lk = [(5 * i) % 6 for i in range(1100)]
    check(R.make(*heads, lq, lk, d, dtype, seed=3, before=1, after=2), True)


@pytest.mark.parametrize("S", [63, 64, 65])
def test_sequences_about_a_wave(S):
    check(R.make(2, 1, [(11 * i) % 40 for i in range(S)], [(13 * i) % 50 for i in range(S)], 64,
                 "bf16", seed=S), True)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (128, "f32")])
def test_large_logits_and_scale(d, dtype):
    check(R.make(4, 2, [150, 40], [150, 90], d, dtype, seed=5, scale_q=40.0), True)
    check(R.make(4, 2, [150, 40], [150, 90], d, dtype, seed=6), True, scale=0.37)


@pytest.mark.parametrize("heads", [(7, 1), (40, 8), (16, 1)], ids=["7of1", "40of8", "16of1"])
def test_head_groups(heads):
    check(R.make(*heads, [70, 33], [70, 50], 64, "bf16", seed=8), True)


def test_parts_follow_from_sizes():
    """Sums in parts are as exact as whole ones, and joined for every row of their range."""
    for lq, lk in (([1, 1], [5000, 40]), ([300], [4000]), ([64, 200], [2000, 3000])):
        check(R.make(2, 1, lq, lk, 128, "bf16", seed=9, before=2, after=3), True)
        check(R.make(2, 1, lq, lk, 64, "f32", seed=9, before=2, after=3), True)
    check(R.make(4, 1, [4000], [30], 64, "bf16", seed=9), False)     # dK, dV in parts


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32")])
def test_more_parts_than_tiles(d, dtype, causal):
    """Parts follow from the average length: a short sequence's items have fewer tiles."""
    check(R.make(8, 1, [700, 1, 40, 0], [700, 1, 60, 5], d, dtype, seed=10, before=1, after=2), causal)
    check(R.make(2, 2, [900, 3], [2, 900], d, dtype, seed=11), causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_with_room(dtype):
    """Keys behind a cache's length are not read into any result, whatever they hold."""
    x = R.make(4, 2, [1, 1, 5, 1, 70], [1, 200, 64, 0, 333], 128, dtype, seed=4, room=77)
    _, used = R.inside(x)
    for name in "kv":
        x[name][:, ~used] = math.nan
    check(x, True, cache=True)
    check(x, False, cache=True)


def test_single_tokens_continue_a_prompt():
    """A prompt's rows one by one behind a cache are its rows at once."""
    H, kv, d, n, first = 4, 2, 128, 150, 120
    x = R.make(H, kv, [n], [n], d, "bf16", seed=12)
    whole, _ = attention_of(x, True).forward(x["q"], x["k"], x["v"], x["offsets_q"], x["offsets_k"])
    step = packed.PackedAttention(H, kv, 1, n + 10, d, 1)
    room = [torch.full((kv, n + 10, d), math.nan, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    for r, name in zip(room, "kv"):
        r[:, :first] = x[name][:, :first]
    oq, ok = packed.offsets_of([1]), packed.offsets_of([n + 10])
    length = torch.zeros(1, dtype=torch.int32, device="cuda")
    val, tol = R.reference(x, True)
    for i in range(first, n):
        for r, name in zip(room, "kv"):
            r[:, i] = x[name][:, i]
        length.fill_(i + 1)
        out, lse = step.forward(x["q"][:, i:i + 1], *room, oq, ok, lengths_k=length)
        R.assert_within("o", out[:, 0], val["o"][:, i], tol["o"][:, i])
        R.assert_within("lse", lse[:, 0], val["lse"][:, i], tol["lse"][:, i])
        assert (out[:, 0].double() - whole[:, i].double()).abs().max() < 2.0 ** -7 * 4


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_masked_places_may_hold_anything(dtype, d):
    """A key that a row does not see, a NaN or an infinity among them, leaves it as it
    was, as long as its value is finite."""
    x = R.make(2, 1, [200], [200], d, dtype, seed=14)
    a = attention_of(x, True)
    off = (x["offsets_q"], x["offsets_k"])
    want = [t.clone() for t in a.forward(x["q"], x["k"], x["v"], *off)]
    k = x["k"].clone()
    k[:, 100], k[:, 150] = math.nan, math.inf
    out, lse = a.forward(x["q"], k, x["v"], *off)
    assert torch.equal(out[:, :100], want[0][:, :100]) and torch.equal(lse[:, :100], want[1][:, :100])
    assert torch.isnan(out[:, 100:150]).all() and torch.isnan(lse[:, 100:150]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_of_minus_infinity(dtype):
    """Keys whose logits are -inf weigh nothing, whole tiles of them at the start too; a
    row that sees no others has no weights."""
    x = R.make(2, 2, [300], [300], 64, dtype, seed=15)
    x["q"] = x["q"].abs() + 0.1
    k = x["k"].clone()
    k[:, :140] = -math.inf
    a = attention_of(x, True)
    out, lse = a.forward(x["q"], k, x["v"], x["offsets_q"], x["offsets_k"])
    assert (out[:, :140] == 0).all() and (lse[:, :140] == -math.inf).all()
    y = dict(x, lq=[160], lk=[160], oq=[140, 300], ok=[140, 300])
    val, tol = R.reference(y, True)
    R.assert_within("o", out[:, 140:], val["o"][:, 140:], tol["o"][:, 140:])
    R.assert_within("lse", lse[:, 140:], val["lse"][:, 140:], tol["lse"][:, 140:])


def test_bad_offsets_are_reported_and_cannot_fault():
    x = R.make(2, 1, [50, 60, 70], [50, 60, 70], 64, "bf16", seed=16, after=4)
    nq, nk = x["rows"]
    for bad in ([0, 50, 20, 180], [-5, 50, 110, 180], [0, 50, 110, 1 << 30], [1 << 30, 0, -1, 7]):
        for many in (False, True):
            off = torch.tensor(bad + [bad[-1]] * (70 if many else 0), dtype=torch.int32, device="cuda")
            a = packed.PackedAttention(2, 1, nq, nk, 64, len(off) - 1)
            o, lse = a.forward(x["q"], x["k"], x["v"], off)
            a.backward(x["q"], x["k"], x["v"], o, lse, x["d_o"], off)
            torch.cuda.synchronize()
            assert int(a.status) == 16, (bad, many)
    # each offset is the largest so far: the second sequence is empty, the third starts at 50
    a = packed.PackedAttention(2, 1, nq, nk, 64, 3)
    o, _ = a.forward(x["q"], x["k"], x["v"], torch.tensor([0, 50, 20, 180], dtype=torch.int32, device="cuda"))
    b = packed.PackedAttention(2, 1, nq, nk, 64, 2)
    want, _ = b.forward(x["q"], x["k"], x["v"], packed.offsets_of([50, 130]))
    assert torch.equal(o, want)
    # lengths beyond their room are cut to it
    lengths = torch.tensor([50, 61, -3], dtype=torch.int32, device="cuda")
    off = packed.offsets_of([50, 60, 70])
    c = packed.PackedAttention(2, 1, nq, nk, 64, 3)
    o, lse = c.forward(x["q"], x["k"], x["v"], off, lengths_k=lengths)
    assert int(c.status) == 16
    assert (o[:, 110:180] == 0).all() and (lse[:, 110:180] == -math.inf).all()
    c.status.zero_()
    want, _ = c.forward(x["q"], x["k"], x["v"], off, into=c.outputs())
    assert int(c.status) == 0 and torch.equal(o[:, :110], want[:, :110])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_where_they_lie(dtype):
    """[rows][heads][d] views of one projection in and out give the dense layout's bits."""
    H, kv, d, n = 6, 2, 64, 190
    x = R.make(H, kv, [100, 90], [100, 90], d, dtype, seed=17)
    a = attention_of(x, True)
    off = (x["offsets_q"], x["offsets_k"])
    out, lse = a.forward(x["q"], x["k"], x["v"], *off)
    want = a.backward(x["q"], x["k"], x["v"], out, lse, x["d_o"], *off)
    rows = torch.empty(n, H + 2 * kv, d, dtype=x["q"].dtype, device="cuda")
    views = [t.transpose(0, 1) for t in (rows[:, :H], rows[:, H:H + kv], rows[:, H + kv:])]
    for v, name in zip(views, "qkv"):
        v.copy_(x[name])
    o = torch.zeros(n, H, d, dtype=x["q"].dtype, device="cuda").transpose(0, 1)
    o2, lse2 = a.forward(*views, *off, into=(o, torch.empty_like(lse)))
    assert torch.equal(o2, out) and torch.equal(lse2, lse)
    d_rows = torch.zeros_like(rows)
    grads = [t.transpose(0, 1) for t in (d_rows[:, :H], d_rows[:, H:H + kv], d_rows[:, H + kv:])]
    g = x["d_o"].transpose(0, 1).contiguous().transpose(0, 1)
    a.backward(*views, o2, lse2, g, *off, into=grads)
    assert all(torch.equal(p, q) for p, q in zip(grads, want))
    # one key head for all (stride 0)
    one = packed.PackedAttention(H, H, n, n, d, 2, True, dtype)
    k, v = (x[t][:1].expand(H, n, d) for t in "kv")
    shared = packed.PackedAttention(H, 1, n, n, d, 2, True, dtype)
    p, _ = one.forward(x["q"], k, v, *off)
    q, _ = shared.forward(x["q"], x["k"][:1], x["v"][:1], *off)
    bound = 2.0 ** -7 if dtype == "bf16" else 1e-5   # two roundings of values up to 4
    assert (p.double() - q.double()).abs().max() <= 4 * bound


def test_offsets_past_32_bits():
    """Keys and values in the rows of one wide projection, more than 2^32 bytes from the
    first to the last, in a sequence's own rows and before it."""
    n, width, d = 2_200_000, 8, 128
    g = torch.Generator(device="cuda").manual_seed(30)
    rows = torch.empty(n, width, d, dtype=torch.bfloat16, device="cuda")
    for a in range(0, n, 200_000):
        rows[a:a + 200_000] = torch.randn(200_000, width, d, generator=g, device="cuda").bfloat16()
    assert rows.numel() * 2 > 1 << 32
    lq, lk = [3, 2], [2_150_000, 50_000]
    x = R.make(2, 2, lq, [1, 1], d, "bf16", seed=31)
    x.update(lk=lk, ok=[0, lk[0], n], rows=(5, n), offsets_k=packed.offsets_of(lk),
             k=rows[:, :2].transpose(0, 1), v=rows[:, 2:4].transpose(0, 1))
    check(x, True)
    # queries far apart: the same few rows of a wide projection as a dense copy of them
    m = 40
    y = R.make(2, 1, [m], [m], d, "bf16", seed=32)
    a = attention_of(y, True)
    off = y["offsets_q"]
    far = rows[::n // m][:m, 4:6].transpose(0, 1)
    with pytest.raises(B.ScopeError, match="unsupported"):   # 39 x 112640000 bytes >= 2^32
        a.forward(far, y["k"], y["v"], off)
    far = rows[::n // (2 * m)][:m, 4:6].transpose(0, 1)      # 39 x 56320000, past 2^31
    far.copy_(y["q"])
    want = [t.clone() for t in a.forward(y["q"], y["k"], y["v"], off)]
    grads = [t.clone() for t in a.backward(y["q"], y["k"], y["v"], *want, y["d_o"], off)]
    got = a.forward(far, y["k"], y["v"], off, into=a.outputs())
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    got = a.backward(far, y["k"], y["v"], *want, y["d_o"], off, into=a.gradients())
    assert all(torch.equal(p, q) for p, q in zip(got, grads))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
def test_autograd(dtype, causal):
    """`attention` gives the calls' gradients, of inputs and gradients laid out in any way."""
    x = R.make(4, 2, [60, 0, 41], [60, 3, 80], 64, dtype, seed=18, before=2, after=6)
    a = attention_of(x, causal, workspace=False)
    off = (x["offsets_q"], x["offsets_k"])
    out, lse = a.forward(x["q"], x["k"], x["v"], *off)
    want = [t.clone() for t in a.backward(x["q"], x["k"], x["v"], out, lse, x["d_o"], *off)]
    leaves = [x[n].clone().requires_grad_() for n in "qkv"]
    y = a.attention(*leaves, *off)
    assert torch.equal(y, out)
    y.backward(x["d_o"])
    assert all(torch.equal(t.grad, w) for t, w in zip(leaves, want))
    # behind a layout change, with an expanded gradient; only v asks for one
    v = x["v"].transpose(0, 1).contiguous().requires_grad_()
    g = torch.ones(1, 1, 1, dtype=x["q"].dtype, device="cuda").expand_as(out)
    (a.attention(x["q"], x["k"], v.transpose(0, 1), *off) * 1.0).backward(g)
    _, _, dv = a.backward(x["q"], x["k"], x["v"], out, lse, g.contiguous(), *off)
    assert torch.equal(v.grad.transpose(0, 1), dv)
    # a gradient that starts off 16 bytes
    leaf = x["q"].clone().requires_grad_()
    flat = torch.cat((torch.zeros(1, dtype=x["q"].dtype, device="cuda"), x["d_o"].reshape(-1)))
    a.attention(leaf, x["k"], x["v"], *off).backward(flat[1:].view_as(x["d_o"]))
    assert torch.equal(leaf.grad, want[0])


def test_gradients_against_differences():
    """dQ, dK and dV of a scalar of O, by differences of the definition in 64 bits."""
    x = R.make(2, 1, [9, 20], [12, 20], 64, "f32", seed=19)
    a = attention_of(x, True)
    off = (x["offsets_q"], x["offsets_k"])
    out, lse = a.forward(x["q"], x["k"], x["v"], *off)
    grads = a.backward(x["q"], x["k"], x["v"], out, lse, x["d_o"], *off)
    g = torch.Generator().manual_seed(1)
    for name, grad in zip("qkv", grads):
        step = torch.randn(x[name].shape, generator=g).cuda().double()
        value = []
        for e in (1e-4, -1e-4):
            y = {**x, name: x[name].double() + e * step}
            value.append(float((R.reference(y, True)[0]["o"] * x["d_o"].double()).sum()))
        slope, got = (value[0] - value[1]) / 2e-4, float((grad.double() * step).sum())
        # third-order terms of the differences, and fp32's sums of 29 x 64 products
        assert abs(slope - got) <= 1e-4 * float((grad.double() * step).abs().sum())


def test_streams_and_their_memory():
    x = R.make(2, 1, [1500], [1500], 64, "bf16", seed=20)
    off = (x["offsets_q"], x["offsets_k"])
    qkv = (x["q"], x["k"], x["v"])
    want = attention_of(x, True)
    ref = [t.clone() for t in want.forward(*qkv, *off)]
    grads = [t.clone() for t in want.backward(*qkv, *ref, x["d_o"], *off)]
    for workspace in (True, False):
        a, s = attention_of(x, True, workspace), torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        o, lse = a.forward(*qkv, *off, stream=s)
        got = a.backward(*qkv, o, lse, x["d_o"], *off, stream=s)
        s.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((o, lse, *got), (*ref, *grads)))
    # two objects at once
    objects = [attention_of(x, True) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in objects]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for a, s in zip(objects, streams):
            a.backward(*qkv, *a.forward(*qkv, *off, stream=s), x["d_o"], *off, stream=s)
    torch.cuda.synchronize()
    for a in objects:
        assert all(torch.equal(p, q) for p, q in zip((*a._out, *a._grads), (*ref, *grads)))


def test_captured_steps_follow_lengths_and_offsets():
    """A captured decode step and a captured training step, replayed with other lengths and
    offsets, between eager calls of other objects."""
    H, kv, d, S, room = 4, 2, 128, 3, 300
    g = torch.Generator().manual_seed(21)
    k, v = (torch.randn(kv, S * room, d, generator=g).cuda().bfloat16() for _ in "kv")
    q = torch.randn(H, S, d, generator=g).cuda().bfloat16()
    oq, ok = packed.offsets_of([1] * S), packed.offsets_of([room] * S)
    lengths = torch.tensor([3, 100, 299], dtype=torch.int32, device="cuda")
    step, eager = (packed.PackedAttention(H, kv, S, S * room, d, S) for _ in range(2))
    out = step.outputs()
    step.forward(q, k, v, oq, ok, lengths, into=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.forward(q, k, v, oq, ok, lengths, into=out)
    for change in ([4, 101, 300], [300, 1, 64], [0, 65, 128], [4, 101, 300]):
        lengths.copy_(torch.tensor(change, dtype=torch.int32))
        graph.replay()
        want = eager.forward(q, k, v, oq, ok, lengths)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), change
    x = R.make(H, kv, [80, 120], [80, 120], 64, "bf16", seed=22)
    train, check_ = attention_of(x, True), attention_of(x, True)
    out, grads = train.outputs(), train.gradients()
    off = x["offsets_q"]

    def pass_of(a, out, grads):
        a.forward(x["q"], x["k"], x["v"], off, into=out)
        a.backward(x["q"], x["k"], x["v"], *out, x["d_o"], off, into=grads)

    pass_of(train, out, grads)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pass_of(train, out, grads)
    for cut in (1, 80, 199, 200):
        off.copy_(torch.tensor([0, cut, 200], dtype=torch.int32))
        graph.replay()
        o, gr = check_.outputs(), check_.gradients()
        pass_of(check_, o, gr)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*out, *grads), (*o, *gr))), cut


def test_refusals():
    x = R.make(2, 1, [20], [20], 64, "bf16", seed=23)
    a = attention_of(x, True)
    off = x["offsets_q"]
    q, k, v = x["q"], x["k"], x["v"]
    for bad in ((q.float(), k, v), (q[:1], k, v), (q, k[:, :10], v), (q, k, v.cpu()),
                (q.transpose(1, 2).contiguous().transpose(1, 2), k, v)):
        with pytest.raises(ValueError):
            a.forward(*bad, off)
    with pytest.raises(ValueError):
        a.forward(q, k, v, off.long())
    with pytest.raises(ValueError):
        a.forward(q, k, v, off[:1])
    with pytest.raises(B.ScopeError):
        a.forward(q, k, v, off, into=(q, torch.empty(2, 20, device="cuda")))
    odd = torch.empty(2, 20, 68, dtype=torch.bfloat16, device="cuda")[..., :64]
    with pytest.raises(B.ScopeError):
        a.forward(odd, k, v, off)
    with pytest.raises(B.ScopeError):
        packed.PackedAttention(3, 2, 10, 10, 64, 1)
    with pytest.raises(B.ScopeError):
        packed.PackedAttention(2, 2, 10, 10, 96, 1)


def test_no_rows():
    a = packed.PackedAttention(2, 1, 0, 30, 64, 2)
    z = torch.empty(2, 0, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.randn(1, 30, 64, device="cuda").bfloat16()
    off, ok = packed.offsets_of([0, 0]), packed.offsets_of([10, 20])
    o, lse = a.forward(z, k, k.clone(), off, ok)
    grads = [torch.full_like(t, 7.0) for t in a.gradients()]
    a.backward(z, k, k.clone(), o, lse, z, off, ok, into=grads)
    torch.cuda.synchronize()
    assert o.shape == (2, 0, 64) and (grads[1] == 0).all() and (grads[2] == 0).all()
    b = packed.PackedAttention(2, 1, 30, 0, 64, 2)
    q, zk = torch.randn(2, 30, 64, device="cuda").bfloat16(), z[:1]
    o, lse = b.forward(q, zk, zk.clone(), ok, off)
    assert (o == 0).all() and (lse == -math.inf).all()
    dq, _, _ = b.backward(q, zk, zk.clone(), o, lse, q, ok, off)
    assert (dq == 0).all()


def test_dense_layer_is_one_sequence():
    """One sequence without a mask is the dense layer's attention."""
    H, n, d = 3, 333, 128
    x = R.make(H, H, [n], [n], d, "bf16", seed=24)
    dense = layer.DenseAttention(H, n, d).forward(x["q"], x["k"], x["v"])
    out, _ = attention_of(x, False).forward(x["q"], x["k"], x["v"], x["offsets_q"])
    _, tol = R.reference(x, False)
    # the dense layer's normaliser sums the rounded weights
    assert ((out.double() - dense.double()).abs() <= 2 * tol["o"] + 2.0 ** -8 * out.double().abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_projection_to_attention_and_back(dtype):
    """Rotary positions and attention as a block runs them, from one projection of
    packed clips, and the projection's gradient through both."""
    H, kv, d = 4, 2, 64
    grids = [(2, 4, 5), (1, 6, 6), (3, 3, 3)]
    lengths = [t * h * w for t, h, w in grids]
    n = sum(lengths)
    g = torch.Generator().manual_seed(25)
    t = R.DTYPE[dtype]
    rows = torch.randn(n, H + 2 * kv, d, generator=g).cuda().to(t).requires_grad_()
    positions = torch.cat([rotary.grid_positions(s) for s in grids], 1)
    turn = rotary.Rotary(d, [16, 24, 24])
    attend = packed.PackedAttention(H, kv, n, n, d, len(grids), causal=False, dtype=dtype)
    q, k, v = (rows[:, a:b].transpose(0, 1) for a, b in ((0, H), (H, H + kv), (H + kv, H + 2 * kv)))
    out = attend.attention(*turn.rotate(q, positions, k), v, packed.offsets_of(lengths))
    d_out = torch.randn(H, n, d, generator=g).cuda().to(t)
    out.backward(d_out)

    # the same in 64 bits
    r64 = rows.detach().double().requires_grad_()
    f = turn.turns.double() * (2 * math.pi * 2.0 ** -64)
    at, first = 0, 0
    angle = []
    for a, m in enumerate((16, 24, 24)):
        angle.append(positions[a].double()[:, None] * f[at:at + m // 2])
        at += m // 2
    angle = torch.cat(angle, 1)[:, None]

    def turned(x):
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), -1).flatten(2)

    q64, k64, v64 = turned(r64[:, :H]), turned(r64[:, H:H + kv]), r64[:, H + kv:]
    want, at = [], 0
    for m in lengths:
        s = slice(at, at + m)
        x = [y[s].transpose(0, 1) for y in (q64, k64.repeat_interleave(H // kv, 1), v64.repeat_interleave(H // kv, 1))]
        want.append(torch.softmax(x[0] @ x[1].transpose(1, 2) / math.sqrt(d), 2) @ x[2])
        at += m
    want = torch.cat(want, 1)
    want.backward(d_out.double())
    # roundings of the rotated inputs, of weights and of results, each half a step, and
    # their sums; in the norm
    few = 4 * R.HALF_STEP[dtype] if dtype == "bf16" else 64 * R.U
    assert float((out.double() - want).detach().norm() / want.detach().norm()) <= few
    assert float((rows.grad.double() - r64.grad).norm() / r64.grad.norm()) <= few
