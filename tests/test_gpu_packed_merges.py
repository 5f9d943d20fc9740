"""Packed attention's sums in parts and in a block's waves, joined where they differ widely:
maxima far apart, parts and waves whose logits are all -inf or NaN beside finite ones."""
import math

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


# heads, queries and keys: a block of few queries with whole sums (its four waves' alone) and
# in parts, and parts of many queries
SIZES = {
    "waves": ((8, 8), [1, 3, 2, 4], [200, 255, 190, 131]),
    "few": ((4, 1), [1, 4], [3001, 2900]),
    "parts": ((2, 1), [300], [4000]),
}
TYPES = [(64, "bf16"), (128, "bf16"), (64, "f32"), (128, "f32")]


def forward(x):
    H, kv, d, dtype = x["dims"]
    a = packed.PackedAttention(H, kv, *x["rows"], d, len(x["lq"]), True, dtype)
    out, lse = a.forward(x["q"], x["k"], x["v"], x["offsets_q"], x["offsets_k"])
    return out.clone(), lse.clone()


def without(x, dead):
    """The same without the keys in `dead`, which lie before the last lq keys: a query's
    last key stays the same one."""
    kept, lk, ok = [], [], [0]
    for a, m, n in zip(x["ok"], x["lk"], x["lq"]):
        rows = [a + j for j in range(m) if not dead(j, m)]
        assert all(not dead(j, m) for j in range(m - n, m))
        kept += rows
        lk.append(len(rows))
        ok.append(ok[-1] + len(rows))
    at = torch.tensor(kept, device="cuda")
    return dict(x, k=x["k"][:, at], v=x["v"][:, at], lk=lk, ok=ok, rows=(x["rows"][0], ok[-1]))


@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("d,dtype", TYPES)
def test_maxima_far_apart(d, dtype, size):
    """Logits of a few and of hundreds, by runs of keys, rising and falling along them."""
    G.say(f"[packed merges] {dtype} d={d} {size}")
    heads, lq, lk = SIZES[size]
    for seed, rising in ((51, True), (52, False)):
        x = R.make(*heads, lq, lk, d, dtype, seed=seed, scale_q=40.0)
        size_of = torch.cat([torch.linspace(0.01, 3.0, m) if rising else torch.linspace(3.0, 0.01, m)
                             for m in lk]).cuda()
        x["k"] = (x["k"].float() * size_of[:, None]).to(x["k"].dtype)
        out, lse = forward(x)
        val, tol = R.reference(x, True)
        R.assert_within("o", out, val["o"], tol["o"])
        R.assert_within("lse", lse, val["lse"], tol["lse"])


DEAD = {  # of m keys: whole tiles and parts at the start, all but a few, and every other tile
    "start": lambda j, m: j < m // 2,
    "most": lambda j, m: j < m - 5 and j != 3,
    "end": lambda j, m: m // 3 < j < m - 4,
    "between": lambda j, m: j // 64 % 2 == 0 and j < m - 4,
}


@pytest.mark.parametrize("dead", list(DEAD))
@pytest.mark.parametrize("size", ["waves", "few"])
@pytest.mark.parametrize("d,dtype", TYPES)
def test_runs_of_minus_infinity(d, dtype, size, dead):
    """Keys whose logits are -inf are as if they were not there."""
    heads, lq, lk = SIZES[size]
    x = R.make(*heads, lq, lk, d, dtype, seed=53)
    x["q"] = x["q"].abs() + 0.1
    gone = torch.tensor([DEAD[dead](j, m) for m in lk for j in range(m)], device="cuda")
    k = x["k"].clone()
    k[:, gone] = -math.inf
    out, lse = forward(dict(x, k=k))
    val, tol = R.reference(without(x, DEAD[dead]), True)
    R.assert_within("o", out, val["o"], tol["o"])
    R.assert_within("lse", lse, val["lse"], tol["lse"])


@pytest.mark.parametrize("d,dtype", TYPES)
def test_runs_of_minus_infinity_in_parts(d, dtype):
    """Of 300 queries: a row that sees no other key has no weights."""
    x = R.make(2, 1, [300], [4000], d, dtype, seed=54)
    x["q"] = x["q"].abs() + 0.1
    first = 3800                       # query i sees the keys up to 3700 + i
    k = x["k"].clone()
    k[:, :first] = -math.inf
    out, lse = forward(dict(x, k=k))
    assert (out[:, :100] == 0).all() and (lse[:, :100] == -math.inf).all()
    y = dict(x, q=x["q"][:, 100:], d_o=x["d_o"][:, 100:], k=x["k"][:, first:], v=x["v"][:, first:],
             lq=[200], lk=[200], oq=[0, 200], ok=[0, 200], rows=(200, 200))
    val, tol = R.reference(y, True)
    R.assert_within("o", out[:, 100:], val["o"], tol["o"])
    R.assert_within("lse", lse[:, 100:], val["lse"], tol["lse"])


@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("d,dtype", TYPES)
def test_a_nan_key_reaches_those_that_see_it(d, dtype, size):
    """The last key of a sequence is seen by its last query alone, an early one by all of
    the first sequence."""
    heads, lq, lk = SIZES[size]
    x = R.make(*heads, lq, lk, d, dtype, seed=55)
    want, want_lse = forward(x)
    last = [n - 1 for n in x["oq"][1:]]
    others = torch.ones(x["rows"][0], dtype=torch.bool, device="cuda")
    others[last] = False
    for bad in (math.nan, math.inf):
        k = x["k"].clone()
        k[:, [n - 1 for n in x["ok"][1:]]] = bad
        out, lse = forward(dict(x, k=k))
        assert torch.equal(out[:, others], want[:, others]) and torch.equal(lse[:, others], want_lse[:, others])
        assert torch.isnan(out[:, last]).all() and torch.isnan(lse[:, last]).all()
    k = x["k"].clone()
    k[:, lk[0] // 3] = math.nan
    out, lse = forward(dict(x, k=k))
    n = lq[0]
    assert torch.isnan(out[:, :n]).all() and torch.isnan(lse[:, :n]).all()
    assert torch.equal(out[:, n:], want[:, n:]) and torch.equal(lse[:, n:], want_lse[:, n:])
