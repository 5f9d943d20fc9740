"""Rotary positions and packed attention on a host without a GPU: bad arguments are
refused before anything is enqueued (the fake pointers are never dereferenced), and
the frequencies and work lists' formulas."""
import ctypes
import math
from fractions import Fraction

import pytest

torch = pytest.importorskip("torch")

from paper_2608_12780_amd import binding as B
from paper_2608_12780_amd import inputs, packed, rotary

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
ROOM = 1 << 36


def ptr(i, off=0):
    return ctypes.c_void_p((1 << 40) + i * ROOM + off)


def strides(row, head):
    return ctypes.byref(B.Strides(row, head))


NAMES = {
    "forward": ("q", "qs", "k", "ks", "v", "vs", "offsets_q", "offsets_k", "lengths_k", "scale",
                "o", "os", "lse", "workspace", "ws_bytes", "dev_status", "stream"),
    "backward": ("q", "qs", "k", "ks", "v", "vs", "o", "os", "lse", "d_o", "gs", "offsets_q",
                 "offsets_k", "scale", "dq", "dqs", "dk", "dks", "dv", "dvs", "workspace",
                 "ws_bytes", "dev_status", "stream"),
}
ROWS = {"forward": ("q", "k", "v", "o"), "backward": ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")}
STRIDES = {"q": "qs", "k": "ks", "v": "vs", "o": "os", "d_o": "gs", "dq": "dqs", "dk": "dks",
           "dv": "dvs"}


def pack(heads=16, kv_heads=4, rows_q=3000, rows_k=4000, sequences=5, d=128, dtype=B.BF16,
         causal=True):
    return B.make_pack(heads, kv_heads, rows_q, rows_k, sequences, d, dtype, causal)


def call(kind, p=None, **kw):
    args = {name: ptr(i) for i, name in enumerate(NAMES[kind])}
    args.update({s: None for s in STRIDES.values()}, scale=0.0, ws_bytes=16, stream=None,
                dev_status=None, lengths_k=None)
    args.update(kw)
    f = B.lib().scope_packed_attention if kind == "forward" else B.lib().scope_packed_attention_backward
    return f(ctypes.byref(p or pack()), *(args[n] for n in NAMES[kind]))


@pytest.mark.parametrize("kind", ["forward", "backward"])
def test_refusals(kind):
    # everything in order but the workspace, which is checked last
    assert call(kind) == WORKSPACE
    assert call(kind, workspace=None, ws_bytes=1 << 50) == WORKSPACE
    assert call(kind, workspace=ptr(30, 8), ws_bytes=1 << 50) == WORKSPACE
    if kind == "forward":
        assert call(kind, lengths_k=ptr(33)) == WORKSPACE
        assert call(kind, lengths_k=ptr(33, 2)) == INVALID
    for name in (*ROWS[kind], "offsets_q", "offsets_k", "lse"):
        assert call(kind, **{name: None}) == INVALID, name
    for i, name in enumerate(ROWS[kind]):
        assert call(kind, **{name: ptr(40 + i, 8)}) == INVALID, name
    for name in ("lse", "offsets_q", "offsets_k", "dev_status"):
        assert call(kind, **{name: ptr(40, 2)}) == INVALID, name
    for bad in (math.nan, math.inf):
        assert call(kind, scale=bad) == INVALID
    for bad in (dict(heads=0), dict(kv_heads=0), dict(heads=15), dict(rows_q=-1), dict(rows_k=-1),
                dict(sequences=0)):
        assert call(kind, pack(**bad)) == INVALID, bad
    for bad in (dict(d=96), dict(d=32), dict(dtype=7), dict(heads=65536, kv_heads=65536),
                dict(rows_q=(1 << 24) + 1), dict(rows_k=(1 << 24) + 1), dict(sequences=65537),
                dict(heads=512, rows_q=1 << 22), dict(heads=512, kv_heads=512, rows_k=1 << 22)):
        assert call(kind, pack(**bad)) == UNSUPPORTED, bad
    # no rows at all is a valid call
    assert call(kind, pack(rows_q=0, rows_k=0), q=None, k=None, v=None, o=None, lse=None,
                **({} if kind == "forward" else dict(d_o=None, dq=None, dk=None, dv=None))) == WORKSPACE
    out = ROWS[kind][-1]
    for other in ROWS[kind][:-1]:
        assert call(kind, **{out: ptr(NAMES[kind].index(other))}) == INVALID, other
    assert call(kind, **{out: ptr(NAMES[kind].index("v"), 4096)}) == INVALID


@pytest.mark.parametrize("kind", ["forward", "backward"])
def test_strides(kind):
    # [rows][heads][d], and inputs that are one row for all
    for name in ROWS[kind]:
        keys = name in ("k", "v", "dk", "dv")
        heads, rows, of = (4, 4000, STRIDES[name]) if keys else (16, 3000, STRIDES[name])
        output = name in ("o", "dq", "dk", "dv") and not (kind == "backward" and name == "o")
        assert call(kind, **{of: strides(heads * 128, 128)}) == WORKSPACE, name
        assert call(kind, **{of: strides(24 * 128, 128)}) == WORKSPACE, name
        assert call(kind, **{of: strides(0, 0)}) == (INVALID if output else WORKSPACE), name
        assert call(kind, **{of: strides(heads * 128 + 4, 128)}) == INVALID, name    # 16 bytes
        assert call(kind, **{of: strides(-128, rows * 128)}) == INVALID, name
        if output:   # rows over one another
            assert call(kind, **{of: strides(64, rows * 128)}) == INVALID, name
            assert call(kind, **{of: strides(128, rows * 64)}) == INVALID, name
        # a long cache passes 32 bits of bytes, the rows of a tile must not
        assert call(kind, **{of: strides(1 << 20, 128)}) == WORKSPACE, name
        assert call(kind, **{of: strides(1 << 26, 128)}) == UNSUPPORTED, name


def test_workspace_size():
    out = ctypes.c_size_t(0)
    f = B.lib().scope_packed_workspace_size
    assert f(ctypes.byref(pack()), None) == INVALID
    assert f(ctypes.byref(pack(d=100)), ctypes.byref(out)) == UNSUPPORTED
    for p in (pack(), pack(rows_q=0, rows_k=0), pack(sequences=65536), pack(dtype=B.F32)):
        assert f(ctypes.byref(p), ctypes.byref(out)) == OK and 0 < out.value < 1 << 31
        assert out.value % 256 == 0


def rotation(rows=100, heads=(4, 2), d=128, dtype=B.BF16, ranges=((0, 16, 72), (16, 56, 56)),
             layout="pairs", inverse=False, factor=1.0):
    return B.make_rotation(rows, heads, d, dtype, ranges, layout, inverse, factor)


def rotate(r, **kw):
    names = ("positions", "turns", "x", "xs", "y", "ys", "x2", "x2s", "y2", "y2s", "stream")
    args = {n: ptr(i) for i, n in enumerate(names)}
    args.update(xs=None, ys=None, x2s=None, y2s=None, stream=None)
    args.update(kw)
    return B.lib().scope_rotary(ctypes.byref(r), *(args[n] for n in names))


def test_rotary_refusals():
    # rows = 0 is checked as any call and enqueues nothing
    assert rotate(rotation(rows=0)) == OK
    for bad in (dict(rows=-1), dict(heads=(0, 2)), dict(heads=(4, -1)), dict(d=0),
                dict(d=127), dict(factor=math.inf), dict(factor=math.nan),
                dict(ranges=((0, 10, 72), (16, 56, 56))),          # overlap
                dict(ranges=((0, 16, 72), (16, 56, 58))),          # past d
                dict(ranges=((0,), (15,))), dict(ranges=((0,), (0,))), dict(ranges=((-2,), (16,))),
                dict(ranges=((1,), (16,)))):                       # pairs at an odd channel
        assert rotate(rotation(**{"rows": 0, **bad})) == INVALID, bad
    assert rotate(rotation(rows=0, ranges=((1,), (16,)), layout="halves")) == OK
    assert rotate(rotation(rows=0, d=1026, ranges=((0,), (16,)))) == UNSUPPORTED
    assert rotate(rotation(rows=0, heads=(65535, 1))) == UNSUPPORTED
    assert rotate(rotation(rows=0, dtype=7)) == UNSUPPORTED
    assert rotate(rotation(rows=1 << 26)) == UNSUPPORTED           # threads of a launch
    r = rotation(rows=100)
    for name in ("positions", "turns", "x", "y", "x2", "y2"):
        assert rotate(r, **{name: None}) == INVALID, name
    for name, off in (("positions", 2), ("turns", 4), ("x", 1), ("y", 1), ("x2", 1), ("y2", 1)):
        assert rotate(r, **{name: ptr(40, off)}) == INVALID, name
    x, y = ptr(2), ptr(4)
    assert rotate(r, y=ctypes.c_void_p(x.value + 256)) == INVALID             # over a part of x
    assert rotate(r, y=x, ys=strides(4 * 128, 128)) == INVALID                # in place, other strides
    assert rotate(r, y2=y) == INVALID
    assert rotate(r, ys=strides(64, 128 * 100)) == INVALID                    # rows over one another
    assert rotate(r, ys=strides(0, 0)) == INVALID
    assert rotate(r, xs=strides(-128, 0)) == INVALID


def test_rotary_object_refusals():
    with pytest.raises(ValueError):
        rotary.Rotary(64, [31], device="cpu")
    with pytest.raises(ValueError):
        rotary.Rotary(64, [8] * 4, device="cpu")
    with pytest.raises(ValueError):
        rotary.Rotary(64, layout="spiral", device="cpu")
    with pytest.raises(ValueError):
        rotary.Rotary(64, scaling=("tight", 2.0), device="cpu")
    with pytest.raises(ValueError):
        rotary.Rotary(64, [2], scaling=("base", 2.0), device="cpu")
    r = rotary.Rotary(64, device="cpu")
    x, p = torch.zeros(2, 5, 64), torch.zeros(5, dtype=torch.int32)
    for bad in (dict(x=x[0]), dict(x=x[..., :32]), dict(positions=p[:4]), dict(x2=x[:, :4]),
                dict(x2=x.bfloat16()), dict(out=(x, x)), dict(x2=x, out=x)):
        with pytest.raises(ValueError):
            r.rotate(**{"x": x, "positions": p, **bad})
    with pytest.raises(ValueError, match="GPU"):
        r.rotate(x, p)
    with pytest.raises(ValueError, match="not differentiable"):
        r.rotate(x.requires_grad_(), p, out=torch.zeros(2, 5, 64))


def test_frequencies():
    assert rotary.frequencies(8, 10000.0)[0] == pytest.approx([1, 0.1, 0.01, 0.001], rel=1e-14)
    f, factor = rotary.frequencies(8, 10000.0, ("linear", 4.0))
    assert f == pytest.approx([0.25, 0.025, 0.0025, 0.00025], rel=1e-14) and factor == 1.0
    # the fastest pair keeps its speed, the slowest is s times slower
    f, factor = rotary.frequencies(64, 10000.0, ("base", 8.0))
    plain = rotary.frequencies(64, 10000.0)[0]
    assert f[0] == plain[0] and f[-1] == pytest.approx(plain[-1] / 8, rel=1e-12) and factor == 1.0
    f, factor = rotary.frequencies(128, 500000.0, ("ramp", 4.0), context=4096)
    plain = rotary.frequencies(128, 500000.0)[0]
    assert factor == pytest.approx(1 + 0.1 * math.log(4))
    for a, b in zip(f, plain):
        turns = 4096 * b / (2 * math.pi)
        if turns >= 32:
            assert a == b
        elif turns <= 1:
            assert a == pytest.approx(b / 4, rel=1e-14)
        else:
            assert b / 4 < a < b
    # the table holds fractions of a turn in units of 2^-64
    r = rotary.Rotary(128, [16, 56, 56], device="cpu")
    want = [f / (2 * math.pi) for n in (16, 56, 56) for f in rotary.frequencies(n)[0]]
    got = [Fraction(int(t) % 2 ** 64, 2 ** 64) for t in r.turns]
    for a, b in zip(got, want):
        assert abs(a - Fraction(b)) <= Fraction(1, 2 ** 52) * Fraction(b) + Fraction(1, 2 ** 64)


def test_positions_of_a_grid():
    t, h, w = 3, 4, 5
    p = rotary.grid_positions((t, h, w), "cpu")
    assert p.dtype == torch.int32 and p.shape == (3, 60)
    at = [(a, b, c) for a in range(t) for b in range(h) for c in range(w)]
    assert p.T.tolist() == [list(x) for x in at]
    assert packed.offsets_of([3, 0, 4], "cpu").tolist() == [0, 3, 3, 7]
    assert inputs.CONFIGS["tiny"].grid == (4, 8, 8)
