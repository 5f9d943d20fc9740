"""Rotary positions against their definition in 64 bits with derived bounds: layouts,
axes, parts of a head, far and negative positions, alignments, strides, in place,
gradients and the layer's own inputs."""
import dataclasses
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2608_12780_amd import binding as B  # noqa: E402
from paper_2608_12780_amd import inputs, rotary  # noqa: E402

import gpu_harness as G  # noqa: E402
import packed_reference as R  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def make(heads, n, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(heads, n, d, generator=g).cuda().to(R.DTYPE[dtype])


def positions_of(axes, n, seed=0, low=-5, high=1 << 24):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(low, high, (axes, n), generator=g, dtype=torch.int32).cuda()


def check(turn, x, positions, got, inverse=False):
    val, tol = R.rotated(x, positions, turn.turns, turn.ranges, turn.layout, turn.factor, inverse)
    R.assert_within("y", got.cpu(), val, tol)
    # channels in no range are copied
    inside = torch.zeros(x.shape[2], dtype=torch.bool)
    for off, n in zip(*turn.ranges):
        inside[off:off + n] = True
    assert torch.equal(got[..., ~inside], x[..., ~inside])


CASES = [  # d, lengths, offsets
    (128, [16, 56, 56], None), (128, [44, 42, 42], None), (64, [16, 24, 24], None), (64, None, None),
    (64, [32], None), (64, [32], [32]), (128, [32, 16], [80, 16]), (128, [10, 6, 4], [100, 2, 50]),
    (2, [2], None), (6, [2], [4]), (40, [16], [8]), (1024, [512, 256], [0, 768]),
]


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,lengths,offsets", CASES)
def test_ranges(d, lengths, offsets, dtype, layout):
    G.say(f"[rotary] d={d} {lengths} {offsets} {dtype} {layout}")
    turn = rotary.Rotary(d, lengths, offsets, layout=layout)
    x, x2 = make(5, 33, d, dtype, 1), make(2, 33, d, dtype, 2)
    p = positions_of(len(turn.ranges[0]), 33, 3)
    for inverse in (False, True):
        y, y2 = turn.rotate(x, p, x2, inverse=inverse)
        check(turn, x, p, y, inverse)
        check(turn, x2, p, y2, inverse)
        assert torch.equal(turn.rotate(x, p, inverse=inverse), y)


@pytest.mark.parametrize("n", [0, 1, 2, 255, 1000])
@pytest.mark.parametrize("heads", [(1, 0), (3, 1), (9, 9)])
def test_sizes(n, heads):
    turn = rotary.Rotary(64, [16, 24, 24])
    x = make(heads[0], n, 64, "bf16", n)
    x2 = make(heads[1], n, 64, "bf16", n + 1) if heads[1] else None
    p = positions_of(3, n, 4, 0, 100)
    y = turn.rotate(x, p, x2)
    for a, b in zip((x, x2), y if x2 is not None else (y,)):
        check(turn, a, p, b)


def test_many_rows():
    """Rows enough for several heads a thread; a sample of them against the definition."""
    turn = rotary.Rotary(128, [44, 42, 42])
    x = torch.randn(7, 70001, 128, device="cuda").bfloat16()
    p = rotary.grid_positions((1, 1, 70001))
    y = turn.rotate(x, p)
    rows = torch.tensor([0, 1, 2047, 2048, 35000, 69999, 70000], device="cuda")
    check(turn, x[:, rows], p[:, rows], y[:, rows])


@pytest.mark.parametrize("scaling", [None, ("linear", 8.0), ("base", 4.0), ("ramp", 4.0)])
def test_stretched_contexts(scaling):
    turn = rotary.Rotary(128, theta=500000.0, layout="halves", scaling=scaling)
    x, p = make(3, 64, 128, "f32", 5), positions_of(1, 64, 6, 100000, 2 ** 31 - 1)
    check(turn, x, p, turn.rotate(x, p))
    assert torch.equal(turn.rotate(x, p[0]), turn.rotate(x, p))   # one axis: [n] too


def test_extreme_positions():
    turn = rotary.Rotary(64)
    p = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30, -2 ** 30]], dtype=torch.int32, device="cuda")
    x = make(2, 7, 64, "f32", 7)
    y = turn.rotate(x, p)
    check(turn, x, p, y)
    assert torch.equal(y[:, 0], x[:, 0])


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_where_they_lie(dtype, layout):
    """Parts of one projection in and out, at aligned and odd offsets, and in place."""
    H, kv, d, n = 4, 2, 64, 77
    turn = rotary.Rotary(d, [16, 32], layout=layout)
    p = positions_of(2, n, 8, 0, 500)
    for extra in (0, 3):   # elements before the first row, and between rows
        flat = torch.randn(extra + n * ((H + 2 * kv) * d + extra), device="cuda").to(R.DTYPE[dtype])
        rows = flat[extra:].view(n, -1)[:, :(H + 2 * kv) * d].unflatten(1, (H + 2 * kv, d))
        q, k = rows[:, :H].transpose(0, 1), rows[:, H:H + kv].transpose(0, 1)
        want = turn.rotate(q, p, k)
        check(turn, q, p, want[0])
        check(turn, k, p, want[1])
        before = rows.clone()
        into = torch.full_like(flat, 7.0)
        out = into[extra:].view(n, -1)[:, :(H + 2 * kv) * d].unflatten(1, (H + 2 * kv, d))
        views = out[:, :H].transpose(0, 1), out[:, H:H + kv].transpose(0, 1)
        got = turn.rotate(q, p, k, out=views)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert (out[:, H + kv:] == 7).all() and torch.equal(rows, before)
        assert int((into == 7).sum()) >= into.numel() - n * (H + kv) * d   # nothing else is written
        turn.rotate(q, p, k, out=(q, k))
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
        assert torch.equal(rows[:, H + kv:], before[:, H + kv:])
    one = make(1, n, d, dtype, 9)
    assert torch.equal(turn.rotate(one.expand(H, n, d), p)[2], turn.rotate(one, p)[0])


def test_values_that_are_not_finite():
    """A pair's NaN or infinity stays in its pair; copied channels keep theirs."""
    turn = rotary.Rotary(64, [32])
    x, p = make(1, 4, 64, "bf16", 10), positions_of(1, 4, 11, 1, 50)
    want = turn.rotate(x, p)
    x[0, 1, 3], x[0, 2, 40], x[0, 3, 63] = math.nan, math.inf, math.nan
    y = turn.rotate(x, p)
    assert torch.isnan(y[0, 1, 2:4]).all() and y[0, 2, 40] == math.inf and torch.isnan(y[0, 3, 63])
    same = torch.ones(1, 4, 64, dtype=torch.bool)
    same[0, 1, 2:4] = same[0, 2, 40] = same[0, 3, 63] = False
    assert torch.equal(y.cpu()[same], want.cpu()[same])


@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients(dtype, two):
    turn = rotary.Rotary(64, [16, 24], layout="halves", scaling=("ramp", 4.0))
    p = positions_of(2, 50, 12, 0, 1000)
    x, x2 = make(4, 50, 64, dtype, 13).requires_grad_(), make(2, 50, 64, dtype, 14).requires_grad_()
    g, g2 = make(4, 50, 64, dtype, 15), make(2, 50, 64, dtype, 16)
    if two:
        y, y2 = turn.rotate(x, p, x2)
        torch.autograd.backward((y, y2), (g, g2))
        assert torch.equal(x2.grad, turn.rotate(g2, p, inverse=True))
    else:
        turn.rotate(x, p).backward(g)
    assert torch.equal(x.grad, turn.rotate(g, p, inverse=True))
    check(turn, g, p, x.grad, True)
    # against differences: <rotate(x + e s) - rotate(x - e s), g> / 2 e = <s, dx>
    s = make(4, 50, 64, "f32", 17).double().cpu()
    up, down = (R.rotated(x.detach().double().cpu() + e * s, p, turn.turns, turn.ranges, turn.layout,
                          turn.factor)[0] for e in (1.0, -1.0))
    slope = float(((up - down) / 2 * g.double().cpu()).sum())
    got = float((s * x.grad.double().cpu()).sum())
    # the map is linear; dx is rounded once
    half = R.HALF_STEP[dtype] if dtype == "bf16" else 2.0 ** -20
    assert abs(slope - got) <= 2 * half * float((s * x.grad.double().cpu()).abs().sum())
    # only one of two asks for a gradient
    a = make(4, 50, 64, dtype, 18)
    leaf = make(2, 50, 64, dtype, 19).requires_grad_()
    turn.rotate(a, p, leaf)[1].backward(g2)
    assert torch.equal(leaf.grad, turn.rotate(g2, p, inverse=True))


def test_gradients_into_a_buffer_are_refused():
    turn = rotary.Rotary(64)
    x, p = make(1, 3, 64, "f32").requires_grad_(), positions_of(1, 3)
    with pytest.raises(ValueError, match="not differentiable"):
        turn.rotate(x, p, out=torch.empty(1, 3, 64, device="cuda"))
    with torch.no_grad():
        assert torch.equal(turn.rotate(x, p, out=torch.empty(1, 3, 64, device="cuda")),
                           turn.rotate(x.detach(), p))


def test_streams_and_graphs():
    turn = rotary.Rotary(128, [16, 56, 56])
    x, p = make(3, 500, 128, "bf16", 20), positions_of(3, 500, 21, 0, 100)
    want = turn.rotate(x, p)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = turn.rotate(x, p, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
    out = torch.empty_like(x)
    turn.rotate(x, p, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn.rotate(x, p, out=out)
    for add in (0, 1, 77):
        p += add
        out.zero_()
        graph.replay()
        assert torch.equal(out, turn.rotate(x, p)), add


def test_the_layers_inputs():
    """The generator's rotation of queries and keys, with its frequencies and pairs."""
    cfg = inputs.CONFIGS["tiny"]
    cos, sin = inputs._rope_tables(cfg)
    turn = rotary.Rotary(cfg.d, cfg.ranges[1], cfg.ranges[0])
    p = rotary.grid_positions(cfg.grid)
    x = make(1, cfg.n, cfg.d, "f32", 22)
    y = turn.rotate(x, p)
    unit = torch.zeros(1, cfg.n, cfg.d, device="cuda")
    unit[..., 0::2] = 1.0
    at = turn.rotate(unit, p)[0].cpu().numpy()     # (cos, sin) of every pair
    assert np.abs(at[:, 0::2] - np.asarray(cos).reshape(cfg.n, -1)).max() <= 2.0 ** -21
    assert np.abs(at[:, 1::2] - np.asarray(sin).reshape(cfg.n, -1)).max() <= 2.0 ** -21
    check(turn, x, p, y)
