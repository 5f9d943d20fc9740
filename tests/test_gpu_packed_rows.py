"""Packed attention of so many rows that a lane for every four channels of them would need
2^32 threads."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2608_12780_amd import binding as B  # noqa: E402
from paper_2608_12780_amd import packed  # noqa: E402

import gpu_harness as G  # noqa: E402
import packed_reference as R  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def test_2_to_the_28_rows():
    """Of 16 heads: every sequence has the same keys and the same query over and over, so
    that its outputs are one row each."""
    H, nq, d, S, m = 16, 1 << 24, 64, 64, 5
    n = nq // S
    if torch.cuda.get_device_properties(0).total_memory < 100 << 30:
        pytest.skip("needs 75 GB")
    x = R.make(H, H, [1], [m], d, "bf16", seed=70)
    k, v = (x[t].repeat(1, S, 1) for t in "kv")
    q, d_o = (x[t].expand(H, nq, d) for t in ("q", "d_o"))
    a = packed.PackedAttention(H, H, nq, S * m, d, S, causal=False)
    oq, ok = packed.offsets_of([n] * S), packed.offsets_of([m] * S)
    G.say("[packed rows] forward")
    out, lse = a.forward(q, k, v, oq, ok, into=a.outputs())
    row, row_lse = out[:, :1].clone(), lse[:, :1].clone()
    val, tol = R.reference(x, False)
    R.assert_within("o", row, val["o"], tol["o"])
    R.assert_within("lse", row_lse, val["lse"], tol["lse"])
    assert all(bool((out[h] == row[h]).all()) for h in range(H)) and bool((lse == row_lse).all())
    del out
    G.say("[packed rows] backward")
    dq, dk, dv = a.backward(q, k, v, row.expand(H, nq, d), lse, d_o, oq, ok, into=a.gradients())
    val, tol = R.reference(x, False, o=row, lse=row_lse)
    R.assert_within("dq", dq[:, :1], val["dq"], tol["dq"])
    assert all(bool((dq[h] == dq[h, :1]).all()) for h in range(H))
    for name, got in (("dk", dk), ("dv", dv)):
        # n equal terms: n times the one, and the sum's roundings, (n + 8) u of its terms,
        # where the bound of one term has 9 u: dv's are p d_o, dk's scale ds q, of which a
        # row's value is the term itself
        want, bound = n * val[name], n * tol[name] + n * (n + 8) * R.U * val[name].abs()
        got = got.view(H, S, m, d)
        assert torch.equal(got, got[:, :1].expand_as(got)), name
        R.assert_within(name, got[:, 0], want, bound)


def test_a_token_of_each_of_65536_sequences():
    """Of 128 key heads: one key each, whose weight is 1, so that O is V, dV is dO, and the
    other gradients are differences of two sums of the same d products."""
    H, S, d = 128, 1 << 16, 64
    g = torch.Generator(device="cuda").manual_seed(71)
    q, k, v, d_o = (torch.randn(H, S, d, generator=g, device="cuda").bfloat16() for _ in range(4))
    a = packed.PackedAttention(H, H, S, S, d, S)
    off = packed.offsets_of([1] * S)
    G.say("[packed rows] tokens forward")
    out, lse = a.forward(q, k, v, off)
    assert torch.equal(out, v)
    G.say("[packed rows] tokens backward")
    dq, dk, dv = a.backward(q, k, v, out, lse, d_o, off)
    assert torch.equal(dv, d_o)
    scale, U = d ** -0.5, R.U
    for h in range(H):
        s = (q[h].double() * k[h].double()).sum(1) * scale
        e = (d + 8) * U * scale * (q[h].double() * k[h].double()).abs().sum(1) + 12 * U * s.abs() + 8 * U
        assert ((lse[h].double() - s).abs() <= e).all(), h
        # |ds| at most the errors of <d_o, v> and <d_o, o>; p and roundings within 5%
        ds = 1.05 * 2 * (d + 8) * U * (d_o[h].double() * v[h].double()).abs().sum(1, keepdim=True)
        assert (dq[h].double().abs() <= scale * ds * k[h].double().abs() + 1e-30).all(), h
        assert (dk[h].double().abs() <= scale * ds * q[h].double().abs() + 1e-30).all(), h
    assert int(a.status) == 0
