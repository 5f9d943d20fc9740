"""Rotary positions where rows fill the chip and a thread turns many heads of both tensors,
loaded ahead of its stores, also in place."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2608_12780_amd import binding as B  # noqa: E402
from paper_2608_12780_amd import rotary  # noqa: E402

import gpu_harness as G  # noqa: E402
import packed_reference as R  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


# d, lengths, rows (262144 threads, a unit of 16 bytes or one pair each, and a thread takes all
# heads), heads: a thread's rounds of eight end after the first tensor's heads, between, and beyond
CASES = [
    (64, [16, 24, 24], 70001, (13, 6)), (64, [32], 66000, (8, 9)), (128, [16, 56, 56], 33000, (3, 2)),
    (6, [4], 140000, (17, 1)), (64, None, 66000, (24, 0)),
]


@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,lengths,n,heads", CASES)
def test_many_heads_of_a_thread(d, lengths, n, heads, dtype, layout):
    G.say(f"[rotary heads] d={d} {lengths} {n} {heads} {dtype} {layout}")
    turn = rotary.Rotary(d, lengths, layout=layout)
    g = torch.Generator(device="cuda").manual_seed(60)
    x, x2 = (torch.randn(h, n, d, generator=g, device="cuda").to(R.DTYPE[dtype]) for h in heads)
    p = torch.randint(0, 100000, (len(turn.ranges[0]), n), generator=g, dtype=torch.int32, device="cuda")
    two = heads[1] > 0
    got = turn.rotate(x, p, x2) if two else (turn.rotate(x, p),)
    # a sample of rows against the definition
    rows = torch.tensor([0, 1, 777, n // 2, n - 2, n - 1], device="cuda")
    for a, y in zip((x, x2), got):
        val, tol = R.rotated(a[:, rows], p[:, rows], turn.turns, turn.ranges, layout)
        R.assert_within("y", y[:, rows].cpu(), val, tol)
    # every head as alone
    for a, y in zip((x, x2), got):
        for h in range(a.shape[0]):
            assert torch.equal(turn.rotate(a[h:h + 1], p)[0], y[h]), h
    # in place, and there from tensors whose tokens lie first
    b, b2 = (a.transpose(0, 1).clone(memory_format=torch.contiguous_format).transpose(0, 1)
             for a in (x, x2))
    turn.rotate(b, p, b2 if two else None, out=(b, b2) if two else b)
    turn.rotate(x, p, x2 if two else None, out=(x, x2) if two else x)
    for inplace in ((x, x2), (b, b2)):
        assert all(torch.equal(a, y) for a, y in zip(inplace, got))
