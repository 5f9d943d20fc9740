"""The training calls on a host without a GPU: bad arguments are refused before
anything is enqueued (the fake pointers are never dereferenced)."""
import ctypes
import math

import numpy as np
import pytest

from paper_2608_12780_amd import binding as B

import training_reference as R

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
ROOM = 1 << 36


def ptr(i, off=0):
    return ctypes.c_void_p((1 << 40) + i * ROOM + off)


def shape(heads=24, n=118800, d=128, dtype=B.BF16):
    a = d // 3 // 2 * 2
    return B.make_shape(heads, n, d, dtype, ((0, a, 2 * a), (a, a, d - 2 * a)))


NAMES = {
    "train": ("q", "k", "v", "c_q", "offsets", "perm", "sel_counts", "sel_idx", "scale", "dropout",
              "rng", "o", "lse", "workspace", "ws_bytes", "stream"),
    "backward": ("q", "k", "v", "o", "lse", "d_o", "c_q", "offsets", "perm", "sel_counts",
                 "sel_idx", "scale", "dropout", "rng", "dq", "dk", "dv", "workspace", "ws_bytes",
                 "dev_status", "stream"),
}


def call(kind, sh=None, **kw):
    names = NAMES[kind]
    args = {name: ptr(i) for i, name in enumerate(names)}
    args.update(c_q=256, scale=0.0, dropout=0.1, ws_bytes=16, stream=None, dev_status=None)
    args.update(kw)
    return getattr(B.lib(), "scope_sparse_attention_" + kind)(
        ctypes.byref(sh or shape()), *(args[n] for n in names))


@pytest.mark.parametrize("kind", ["train", "backward"])
def test_refusals(kind):
    # everything in order but the workspace, which is checked last
    assert call(kind) == WORKSPACE
    assert call(kind, dropout=0.0, rng=None) == WORKSPACE
    assert call(kind, workspace=None, ws_bytes=1 << 50) == WORKSPACE
    assert call(kind, workspace=ptr(30, 8), ws_bytes=1 << 50) == WORKSPACE
    for name in NAMES[kind]:
        if name in ("c_q", "scale", "dropout", "workspace", "ws_bytes", "stream", "dev_status"):
            continue
        assert call(kind, **{name: None}) == INVALID, name
    rows = {"q", "k", "v", "o", "d_o", "dq", "dk", "dv"} & set(NAMES[kind])
    for i, name in enumerate(sorted(rows)):
        assert call(kind, **{name: ptr(40 + i, 8)}) == INVALID, name
    assert call(kind, lse=ptr(40, 2)) == INVALID
    assert call(kind, rng=ptr(40, 4)) == INVALID
    for bad in (-0.1, 1.0, math.nan, math.inf):
        assert call(kind, dropout=bad) == INVALID
    for bad in (math.nan, math.inf):
        assert call(kind, scale=bad) == INVALID
    assert call(kind, c_q=0) == INVALID
    assert call(kind, sh=shape(n=100), c_q=101) == INVALID
    assert call(kind, c_q=1025) == UNSUPPORTED
    assert call(kind, sh=shape(d=96)) == UNSUPPORTED
    assert call(kind, sh=shape(dtype=7)) == UNSUPPORTED
    assert call(kind, sh=shape(heads=1, n=1 << 24)) == UNSUPPORTED   # 32-bit row offsets
    assert call(kind, sh=shape(heads=1, n=1 << 23, dtype=B.F32)) == UNSUPPORTED
    assert call(kind, sh=shape(heads=65535, n=512), c_q=512) == UNSUPPORTED  # 2^32 threads
    assert call(kind, sh=shape(heads=0)) == INVALID
    # outputs over inputs, also shifted
    out = "o" if kind == "train" else "dk"
    for other in ("q", "k", "v"):
        at = NAMES[kind].index(other)
        assert call(kind, **{out: ptr(at)}) == INVALID
        assert call(kind, **{out: ptr(at, 4096)}) == INVALID
    if kind == "backward":
        assert call(kind, dq=ptr(NAMES[kind].index("dv"))) == INVALID
        assert call(kind, dv=ptr(NAMES[kind].index("d_o"))) == INVALID


def test_workspace_size():
    def size(sh, c_q):
        out = ctypes.c_size_t(0)
        st = B.lib().scope_training_workspace_size(ctypes.byref(sh), c_q, ctypes.byref(out))
        return st, out.value

    st, small = size(shape(1, 1), 1)
    assert st == OK and 0 < small < 1 << 20
    st, full = size(shape(), 256)
    # key bits (one per head, cluster and key) and per-token tables
    assert st == OK and full < 24 * 118800 * (256 / 8 + 1200)
    assert size(shape(), 0)[0] == INVALID
    assert size(shape(), 1025)[0] == UNSUPPORTED
    assert size(shape(d=32), 4)[0] == UNSUPPORTED
    assert size(shape(n=100), 101)[0] == INVALID
    assert B.lib().scope_training_workspace_size(ctypes.byref(shape()), 4, None) == INVALID


def test_dropout_refusals():
    L = B.lib()

    def drop(dtype=B.BF16, count=64, x=ptr(0), r=None, p=0.1, rng=ptr(3), y=ptr(2)):
        return L.scope_dropout(dtype, count, x, r, p, rng, y, None)

    assert drop(count=0, x=None, y=None) == OK
    assert drop(count=-1) == INVALID
    assert drop(count=(1 << 40) + 1) == UNSUPPORTED
    assert drop(dtype=5) == UNSUPPORTED
    assert drop(x=None) == INVALID and drop(y=None) == INVALID and drop(rng=None) == INVALID
    assert drop(rng=ptr(3, 4)) == INVALID
    assert drop(x=ptr(0, 1)) == INVALID and drop(y=ptr(2, 1)) == INVALID
    assert drop(dtype=B.F32, r=ptr(1, 2)) == INVALID
    assert drop(y=ptr(0, 2)) == INVALID and drop(r=ptr(2, 2)) == INVALID   # shifted overlaps
    for bad in (-1e-3, 1.0, math.nan):
        assert drop(p=bad) == INVALID


def test_generator_known_answers():
    """The published vectors of Philox4x32-10, through the tests' own generator."""
    for counter, key, want in (
            ((0, 0, 0, 0), 0, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((0xFFFFFFFF,) * 4, 0xFFFFFFFFFFFFFFFF,
             (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), 0x299F31D0A4093822,
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        got = R.philox([np.array([c], np.uint64) for c in counter], key)
        assert tuple(int(w[0]) for w in got) == want


def test_pair_masks_look_independent():
    """Row, column and pairwise correlations of 1024 x 1024 masks: their sums of n
    centred bits have variance 1 when scaled; the largest of about 2^20 normal
    values lies below 7, the variance of 2^19 such values within 1%."""
    n = 1024
    for p, seed in ((0.1, 1), (0.5, 2)):
        keep = R.keep_pairs(1, n, p, seed, 0)[0].astype(np.float64)
        q = R.threshold(p) / 65536
        x = (keep - (1 - q)) / math.sqrt(q * (1 - q))
        for y in (x, x.T):
            assert abs(y.sum(1) / math.sqrt(n)).max() < 6
            corr = (y @ y.T / math.sqrt(n))[np.triu_indices(n, 1)]
            assert abs(corr).max() < 7 and abs(corr.var() - 1) < 0.01
