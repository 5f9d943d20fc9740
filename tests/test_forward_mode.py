"""Forward-mode differentiation on a host without a GPU: calls that have no derivative of that
kind say so before they reach the library, and others inside a dual level run."""
import pytest

torch = pytest.importorskip("torch")
from torch.autograd import forward_ad

from paper_2608_12780_amd import binding as B
from paper_2608_12780_amd import layer, rotary


@pytest.fixture
def calls(monkeypatch):
    """The library's calls, which do nothing here."""
    made = []
    for name in ("scope_rotary", "scope_dropout"):
        monkeypatch.setattr(B, name, lambda *a, name=name, **k: made.append(name))
    return made


def rotations():
    r = rotary.Rotary(64, device="cpu")
    p = torch.zeros(5, dtype=torch.int32)
    other = torch.ones(2, 5, 64)
    return {"x": lambda t: r.rotate(t, p), "inverse": lambda t: r.rotate(t, p, inverse=True),
            "x of two": lambda t: r.rotate(t, p, other), "x2": lambda t: r.rotate(other, p, t),
            "into out": lambda t: r.rotate(t, p, out=torch.empty(2, 5, 64)),
            "out": lambda t: r.rotate(other, p, out=t)}


def refused(calls, name, call, grad):
    x = torch.ones(2, 5, 64)
    with torch.set_grad_enabled(grad):
        with forward_ad.dual_level():
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call(forward_ad.make_dual(x, torch.ones_like(x)))
            assert not calls
            call(x)
        call(x)
        assert calls == [name] * 2
        with pytest.raises(NotImplementedError, match="forward-mode"):
            torch.func.jvp(call, (x,), (x,))
    assert len(calls) == 2


@pytest.mark.parametrize("grad", [True, False], ids=["grad", "no_grad"])
@pytest.mark.parametrize("form", list(rotations()))
def test_a_rotation_does_not_lose_a_tangent(calls, form, grad):
    refused(calls, "scope_rotary", rotations()[form], grad)


@pytest.mark.parametrize("grad", [True, False], ids=["grad", "no_grad"])
@pytest.mark.parametrize("form", ["x", "residual", "into out", "out"])
def test_dropout_does_not_lose_a_tangent(calls, form, grad):
    other, rng = torch.ones(2, 5, 64), torch.zeros(2, dtype=torch.int64)
    refused(calls, "scope_dropout",
            {"x": lambda t: layer.dropout(t, 0.5, rng),
             "residual": lambda t: layer.dropout(other, 0.5, rng, residual=t),
             "into out": lambda t: layer.dropout(t, 0.5, rng, out=torch.empty(2, 5, 64)),
             "out": lambda t: layer.dropout(other, 0.5, rng, out=t)}[form], grad)
