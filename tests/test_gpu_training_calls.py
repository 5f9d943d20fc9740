"""Calls of the training operators that their documentation allows, in the ways
programs make them: buffers that a call allocates, streams, autograd's gradients
and shapes."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from paper_2608_12780_amd import binding as B  # noqa: E402
from paper_2608_12780_amd import inputs  # noqa: E402
from paper_2608_12780_amd.layer import DenseAttention, TrainingAttention, dropout  # noqa: E402

import gpu_harness as G  # noqa: E402
import training_reference as R  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def rng_of(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def freed_block(like):
    """The address of a block that the current stream's pool has just got back;
    work queued on that stream could still be using it."""
    t = torch.empty_like(like)
    at = t.data_ptr()
    del t
    assert torch.empty_like(like).data_ptr() == at  # what an allocation here would get
    return at


def test_dropout_allocates_on_the_stream_it_runs_on():
    x = torch.randn(3_000_001, device="cuda")
    want = dropout(x, 0.2, rng_of(1, 2))
    rng, s = rng_of(1, 2), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    at = freed_block(x)
    y = dropout(x, 0.2, rng, stream=s)
    s.synchronize()
    assert y.data_ptr() != at
    assert torch.equal(y, want)


def test_held_buffers_are_allocated_on_the_stream_of_their_first_call():
    x = R.make(2, 3001, 64, "bf16", 5, 0.5, 3)
    a = TrainingAttention(2, 3001, 64, 5, "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    qkv = (x["q"], x["k"], x["v"])
    at = freed_block(x["q"])
    o, lse = a.forward(*qkv, *R.sets(x), stream=s)
    assert o.data_ptr() != at
    at = freed_block(x["q"])
    grads = a.backward(*qkv, o, lse, x["d_o"], *R.sets(x), stream=s)
    s.synchronize()
    assert at not in [t.data_ptr() for t in grads]
    want = TrainingAttention(2, 3001, 64, 5, "bf16")
    out = want.forward(*qkv, *R.sets(x))
    for got, ref in zip((o, lse, *grads), (*out, *want.backward(*qkv, *out, x["d_o"], *R.sets(x)))):
        assert torch.equal(got, ref)


@pytest.mark.parametrize("of_residual", [False, True])
def test_dropout_on_a_stream_is_differentiable(of_residual):
    x, res = torch.randn(2, 1001, device="cuda").unbind()
    leaf = (res if of_residual else x).clone().requires_grad_()
    args = (x, leaf) if of_residual else (leaf, res)
    rng, s = rng_of(4, 5), torch.cuda.Stream()
    g = torch.randn_like(x)
    s.wait_stream(torch.cuda.current_stream())
    y = dropout(args[0], 0.3, rng, residual=args[1], stream=s)
    torch.cuda.current_stream().wait_stream(s)
    y.backward(g)
    keep = torch.from_numpy(R.keep_elements(1001, 0.3, 4, 5)).cuda()
    factor = 65536.0 / (65536 - R.threshold(0.3))
    assert torch.equal(y, torch.where(keep, x * factor, 0.0) + res)
    assert torch.equal(leaf.grad, g if of_residual else torch.where(keep, g * factor, 0.0))


def test_dropout_into_a_buffer_refuses_to_lose_a_gradient():
    x, out = torch.randn(2, 100, device="cuda").unbind()
    leaf = x.clone().requires_grad_()
    for kw in (dict(), dict(residual=x), dict(stream=torch.cuda.current_stream())):
        with pytest.raises(ValueError, match="not differentiable"):
            dropout(leaf, 0.1, rng_of(1, 1), out=out, **kw)
    with pytest.raises(ValueError, match="not differentiable"):
        dropout(x, 0.1, rng_of(1, 1), residual=leaf, out=out)
    want = dropout(x, 0.1, rng_of(1, 1))
    with torch.no_grad():
        assert torch.equal(dropout(leaf, 0.1, rng_of(1, 1), out=out), want)
    assert torch.equal(dropout(x, 0.1, rng_of(1, 1), out=out), want)


def dense_case(dtype, heads=2, n=150, d=64):
    x = R.make(heads, n, d, dtype, 1, 1.0, 6)
    dense = DenseAttention(heads, n, d, dtype)
    x.update({a: getattr(dense, a) for a in R.SETS})
    return dense, x, [x[a].clone().requires_grad_() for a in "qkv"]


def want_gradients(x):
    """(dq, dk, dv) of the calls themselves."""
    H, n, d, C, dtype = x["dims"]
    a = TrainingAttention(H, n, d, C, dtype)
    qkv = (x["q"], x["k"], x["v"])
    return a.backward(*qkv, *a.forward(*qkv, *R.sets(x)), x["d_o"], *R.sets(x))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("before", [1, 3, 8])
def test_gradient_of_a_piece_at_any_offset(dtype, before):
    """The gradient behind torch.cat with a piece of odd length is a contiguous view
    that starts off the 16 bytes that the gradient call asks for."""
    dense, x, leaves = dense_case(dtype)
    out = dense.attention(*leaves)
    whole = torch.cat((torch.zeros(before, dtype=out.dtype, device="cuda"), out.flatten()))
    seen = []
    whole.register_hook(lambda g: seen.append(g[before:].data_ptr() % 16))
    whole.backward(torch.cat((torch.ones(before, device="cuda").to(out.dtype),
                              x["d_o"].flatten())))
    assert seen == [before * out.element_size() % 16]
    for leaf, want in zip(leaves, want_gradients(x)):
        assert torch.equal(leaf.grad, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_have_their_inputs_shapes(dtype):
    """[heads][n][d] under other shapes, one for each input."""
    dense, x, _ = dense_case(dtype)
    shapes = ((1, 2, 150, 64), (300, 64), (2 * 150 * 64,))
    leaves = [x[a].reshape(shape).clone().requires_grad_() for a, shape in zip("qkv", shapes)]
    out = dense.attention(*leaves)
    assert out.shape == (2, 150, 64)
    out.backward(x["d_o"])
    for leaf, want in zip(leaves, want_gradients(x)):
        assert torch.equal(leaf.grad, want.view_as(leaf))


@pytest.mark.parametrize("only", range(3))
def test_gradients_of_some_inputs(only):
    dense, x, leaves = dense_case("bf16")
    for i, leaf in enumerate(leaves):
        leaf.requires_grad_(i == only)
    dense.attention(*leaves).backward(x["d_o"])
    for i, (leaf, want) in enumerate(zip(leaves, want_gradients(x))):
        assert torch.equal(leaf.grad, want) if i == only else leaf.grad is None


def test_larger_inputs_have_no_gradient():
    """More than heads x n x d elements: their first ones are attended to, as the
    calls do, but a gradient of all of them is refused before anything runs."""
    dense, x, _ = dense_case("f32")
    with torch.no_grad():
        want = dense.attention(x["q"], x["k"], x["v"])
    for i, name in enumerate("qkv"):
        args = [x[a] for a in "qkv"]
        args[i] = torch.cat((args[i], torch.ones_like(args[i])))
        assert torch.equal(dense.attention(*args), want)
        args[i].requires_grad_()
        with pytest.raises(ValueError, match=f"{name} needs 19200 elements"):
            dense.attention(*args)
        with torch.no_grad():
            assert torch.equal(dense.attention(*args), want)


@pytest.fixture
def workspaces(monkeypatch):
    """(call, address, stream) of every training call's workspace."""
    seen = []

    def watch(name, at):
        call = getattr(B, name)

        def watched(*args):
            seen.append((name[23:], args[at].data_ptr(), torch.cuda.current_stream().cuda_stream))
            return call(*args)
        monkeypatch.setattr(B, name, watched)
    watch("scope_sparse_attention_train", 14)
    watch("scope_sparse_attention_backward", 17)
    return seen


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_layers_attention_on_two_streams(dtype, workspaces):
    """Forward and backward passes of one layer on two streams at once, each with a
    workspace that the other stream's calls do not write."""
    dense, x, _ = dense_case(dtype, 3, 1500)
    cases = [dict(x, q=x["q"] * (1 + i / 4), d_o=x["d_o"] * (1 - i / 4)) for i in range(2)]
    want = [want_gradients(y) for y in cases]
    del workspaces[:]
    streams = [torch.cuda.Stream() for _ in cases]
    leaves = [[[y[a].clone().requires_grad_() for a in "qkv"] for y in cases] for _ in range(6)]
    dense.autograd_attention()
    torch.cuda.synchronize()
    for turn in leaves:
        for s, y, own in zip(streams, cases, turn):
            with torch.cuda.stream(s):
                dense.attention(*own).backward(y["d_o"])
    torch.cuda.synchronize()
    assert len(workspaces) == 24
    of = [{at for _, at, stream in workspaces if stream == s.cuda_stream} for s in streams]
    assert of[0] and of[1] and not of[0] & of[1]
    for turn in leaves:
        for own, grads in zip(turn, want):
            for leaf, grad in zip(own, grads):
                assert torch.equal(leaf.grad, grad)


def test_layers_hold_no_workspace_for_autograd():
    """Forward and backward of several layers leave no more memory than one does."""
    held = []
    x = R.make(4, 2048, 64, "bf16", 1, 1.0, 6)
    layers = [DenseAttention(4, 2048, 64, "bf16") for _ in range(3)]
    layers[0].training_attention()
    size = layers[0].training_attention().workspace.numel()
    leaves = [x[a].requires_grad_() for a in "qkv"]
    for layer in layers[1:]:
        layer.attention(*leaves).backward(x["d_o"])
        for leaf in leaves:
            leaf.grad = None
        held.append(torch.cuda.memory_allocated())
    assert held[1] - held[0] < size / 4


def test_status_of_autograds_calls_is_the_layers():
    dense, x, leaves = dense_case("bf16")
    y = dense.attention(*leaves)
    dense.sel_idx[0, 0, 7] = 3          # not ascending
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    dense.attention(*leaves).sum().backward()
    assert int(dense.training_attention().status.item()) == 8
    assert int(dense.autograd_attention().status.item()) == 8


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32")])
def test_non_finite_rows_reach_the_same_keys_on_every_run(d, dtype):
    """Keys of few signatures, so that most positions in the keys' order are a choice
    among equals: a NaN and an infinity in Q and dO reach the keys that share a wave
    with one that their clusters keep, the same ones on every run."""
    H, n, C = 2, 9000, 24
    x = R.make(H, n, d, dtype, C, 0.5, 17)
    g = torch.Generator(device="cuda").manual_seed(3)
    group = torch.randint(0, 48, (H, n), generator=g, device="cuda")
    for h in range(H):
        for c in range(C):
            keys = (torch.rand(48, generator=g, device="cuda") < 0.3)[group[h]].nonzero()[:, 0]
            x["sel_counts"][h, c] = len(keys)
            x["sel_idx"][h, c, :len(keys)] = keys.int()
    x["q"][0, 100, 3], x["q"][1, 5000, 7] = float("nan"), float("inf")
    x["d_o"][0, 4000, 1], x["d_o"][1, 1, 2] = float("inf"), float("nan")
    a = TrainingAttention(H, n, d, C, dtype)
    qkv = (x["q"], x["k"], x["v"])
    out = a.forward(*qkv, *R.sets(x))
    bits = torch.int16 if dtype == "bf16" else torch.int32
    runs = [[t.view(bits) for t in a.backward(*qkv, *out, x["d_o"], *R.sets(x), into=a.gradients())]
            for _ in range(6)]
    assert all(int(t.view(x["q"].dtype).isnan().any(2).sum()) for t in runs[0])
    for again in runs[1:]:
        for first, t in zip(runs[0], again):
            assert torch.equal(first, t)


def test_bf16_layer_trains_end_to_end():
    """forward_train of a bf16 layer, with both dropouts and a residual: values and
    gradients are those of the calls on the sets that the layer found, and those are
    within the bounds of the definition."""
    cfg = inputs.LayerConfig("train", 2, (5, 11, 13), 128, (16, 56, 56), 12, 16, 3, 0.8,
                             inputs.ceil_tenth(5 * 11 * 13), "bf16", 8, 31)
    host = inputs.generate(cfg)
    layer = G.make_layer(cfg, materialize=False)
    q, k, v = G.to_device(host)
    init = torch.from_numpy(host.init_q).cuda(), torch.from_numpy(host.init_k).cuda()
    res, g = torch.randn(2, *q.shape, device="cuda").bfloat16().unbind()
    leaves = [t.clone().requires_grad_() for t in (q, k, v, res)]
    rng = rng_of(5, 6)
    y = layer.forward_train(*leaves[:3], *init, dropout=0.1, rng=rng, residual=leaves[3],
                            out_dropout=0.2)
    y.backward(g)
    # the same, call by call
    x = dict(q=q, k=k, v=v, dims=(cfg.heads, cfg.n, cfg.d, cfg.c_q, "bf16"),
             d_o=dropout(g, 0.2, rng), **{a: getattr(layer, a) for a in R.SETS})
    a = TrainingAttention(cfg.heads, cfg.n, cfg.d, cfg.c_q, "bf16")
    o, lse = a.forward(q, k, v, *R.sets(x), 0.0, 0.1, rng)
    grads = a.backward(q, k, v, o, lse, x["d_o"], *R.sets(x), 0.0, 0.1, rng)
    assert torch.equal(y, dropout(o, 0.2, rng, residual=res))
    assert torch.equal(leaves[3].grad, g)
    val, tol, held = R.reference(x, 0.1, (5, 6), None, o, lse)
    assert held.all()
    for name, t in (("o", o), ("lse", lse)):
        R.assert_within(name, t, val[name], tol[name])
    for leaf, t, name in zip(leaves, grads, ("dq", "dk", "dv")):
        assert torch.equal(leaf.grad, t), name
        R.assert_within(name, t, val[name], tol[name])


def test_attention_without_gradients_is_captured_and_replayed():
    """Two calls in one graph: their workspaces come from the graph's own memory."""
    dense, x, _ = dense_case("bf16", 2, 700, 128)
    q, rng = x["q"].clone(), rng_of(1, 1)
    scales = (0.0, 0.03)

    def step():
        with torch.no_grad():
            return [dense.attention(q, x["k"], x["v"], s, 0.2, rng) for s in scales]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for t in range(4):
        q.copy_(x["q"] * (1 + t / 8))
        rng.copy_(rng_of(9, t))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o, want in zip(got, step()):
            assert torch.equal(o, want), t
