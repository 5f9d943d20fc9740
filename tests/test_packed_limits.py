"""The largest sizes of packed attention, on a host without a GPU: those that a launch or 32
bits cannot hold are refused, and no others."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2608_12780_amd import binding as B

OK, UNSUPPORTED = 0, 2
ROWS = 1 << 24


def status(heads, kv_heads, rows_q, rows_k, sequences=1, d=64, dtype=B.BF16):
    p, out = B.make_pack(heads, kv_heads, rows_q, rows_k, sequences, d, dtype, False), ctypes.c_size_t(0)
    return B.lib().scope_packed_workspace_size(ctypes.byref(p), ctypes.byref(out))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
def test_rows_of_a_key_head(d, dtype):
    """A key head's rows have 4 bytes of statistics each, within 32 bits."""
    assert status(64, 1, ROWS, 100, d=d, dtype=dtype) == UNSUPPORTED              # 2^30
    assert status(1024, 1, 1 << 20, 100, d=d, dtype=dtype) == UNSUPPORTED
    if dtype == B.BF16:
        assert status(64, 1, ROWS - 1, 100, d=d) == OK
        assert status(127, 1, ROWS // 2, 100, d=d) == OK
    else:                                     # 2^24 items of 64 rows, 256 threads each
        assert status(32, 1, ROWS, 100, d=d, dtype=dtype) == OK


@pytest.mark.parametrize("d", [64, 128])
def test_threads_of_a_launch(d):
    """An item of 128 rows or keys has 256 threads, in each direction."""
    most = (1 << 24) // 128                   # items of a key head, of 128: 2^32 threads
    assert status(128, 128, 10, (most - 9) * 128, d=d) == OK
    assert status(128, 128, 10, most * 128, d=d) == UNSUPPORTED
    assert status(128, 128, (most - 9) * 128, 10, d=d) == OK
    assert status(128, 128, most * 128, 10, d=d) == UNSUPPORTED
    # a token of each of many sequences
    assert status(255, 255, 65000, 65000, 65000, d=d) == OK
    assert status(256, 256, 65536, 65536, 65536, d=d) == UNSUPPORTED


@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_no_join_reads(d):
    """Lanes of a join's rows count only where there is one."""
    assert status(16, 16, ROWS, 100, d=d) == OK
    assert status(16, 16, 100, ROWS, d=d) == OK
    assert status(100, 100, ROWS, ROWS, d=d) == OK
