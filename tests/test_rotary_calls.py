"""Rotary positions on a host without a GPU: calls that would race on their tensors are
refused before anything is enqueued (the fake pointers are never dereferenced)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2608_12780_amd import binding as B

INVALID, UNSUPPORTED = 1, 2
D = 128


def call(heads=(4, 4), n=100, **at):
    """Tensors of `n` rows at the given places, in bytes, or far from one another; xs, ys, x2s
    and y2s: their strides (row, head)."""
    strides = {k: ctypes.byref(B.Strides(*at.pop(k))) for k in list(at) if k.endswith("s")}
    names = ("positions", "turns", "x", "y", "x2", "y2")
    place = {name: (1 << 40) + (i << 36) for i, name in enumerate(names)}
    place.update(at)
    p = {name: ctypes.c_void_p(place[name]) for name in names}
    r = B.make_rotation(n, heads, D, B.BF16, ((0,), (D,)), "pairs", False, 1.0)
    return B.lib().scope_rotary(ctypes.byref(r), p["positions"], p["turns"], p["x"], strides.get("xs"),
                                p["y"], strides.get("ys"), p["x2"], strides.get("x2s"), p["y2"],
                                strides.get("y2s"), None)


A, C = 1 << 41, 1 << 42            # two tensors, of 4 heads x 100 rows
BYTES = 4 * 100 * D * 2


@pytest.mark.parametrize("at", [
    dict(x=A, x2=C, y=C, y2=A),                         # exchanged
    dict(x2=C, y=C), dict(x=A, y2=A),                   # over the other's input
    dict(x=A, x2=A, y=A),                               # in place, which the other reads too
    dict(x2=C, y=C + D * 2), dict(x=A, y2=A + BYTES - 2 * D), dict(x2=C, y=C - 2 * D),
    dict(x=A, y=A + 256), dict(y=A, y2=A), dict(y=A, y2=A + 256),
])
def test_outputs_over_another_tensor_are_refused(at):
    assert call(**at) == INVALID


def test_exchanged_parts_of_one_projection_are_refused():
    """[rows][heads][d]: queries over keys and keys over queries."""
    rows = (8 * D, D)
    assert call(x=A, x2=A + 8 * D, y=A + 8 * D, y2=A, xs=rows, x2s=rows, ys=rows, y2s=rows) == INVALID


@pytest.mark.parametrize("places", [
    lambda size: dict(x=A, y=A, x2=C, y2=C), lambda size: dict(x=A, x2=A),
    lambda size: dict(x=A, x2=A + size, y=C, y2=C + size),
    lambda size: dict(x=A, x2=A + size, y=A, y2=A + size),
], ids=["in place", "one input", "side by side", "side by side in place"])
def test_outputs_beside_the_other_tensor_are_taken(places):
    """They pass every check of memory: their number of rows alone is refused, after it."""
    n = 1 << 26
    assert call(n=n, **places(4 * n * D * 2)) == UNSUPPORTED


@pytest.mark.parametrize("row", [1 << 40, 1 << 39, (1 << 40) - 8])
@pytest.mark.parametrize("name", ["xs", "ys"])
def test_rows_out_of_64_bits_are_refused(name, row):
    """2^24 or 2^25 steps of 2^39 or 2^40 elements: 0 modulo 2^64, or beyond 2^63."""
    for n in ((1 << 24) + 1, (1 << 25) - 5, (1 << 25) + 1):
        assert call(n=n, heads=(1, 0), **{name: (row, D)}) == INVALID, n
