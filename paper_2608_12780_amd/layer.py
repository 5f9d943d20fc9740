"""The SCOPE layer as five library calls on buffers allocated once.

ScopeLayer owns every output and the workspace for one problem size and runs
Alg. 1 end to end through the C ABI: query clustering, key-subspace
clustering, score tables, selection and sparse attention.  Nothing here
computes; it allocates device memory and sequences the calls.

For training, TrainingAttention holds the buffers of the attention with row
statistics and of its gradients, ScopeLayer.attention and
DenseAttention.attention are differentiable in q, k and v, dropout in its input
and residual, and ScopeLayer.forward_train runs the layer with both.
"""
from __future__ import annotations

import contextlib

import torch
from torch.autograd import forward_ad

from . import binding as B


def _allocating_on(stream):
    """Where a call allocates what it runs `stream` on: memory that torch's
    allocator gives out for another stream may still be in use there."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _refuse_tangents(name, *tensors):
    """Raises where forward-mode differentiation follows one of the tensors: the result
    would come without its tangent."""
    if forward_ad._current_level >= 0 and any([
            t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors]):
        raise NotImplementedError(f"{name} has no forward-mode derivative")


class TrainingAttention:
    """Attention over given clusters and key sets with the rows' log-sum-exp
    (call 6) and its gradients (call 7), on buffers allocated once.  `dropout`
    drops attention probabilities; `rng` is an int64 tensor (seed, offset) on
    the GPU, the same in backward as in forward.  Calls that may run at once
    (streams, replays of captured graphs) need an object each.  With
    workspace=False it holds no workspace: every call takes one from torch's
    allocator, for the stream it runs on, and gives it back."""

    def __init__(self, heads, n, d, c_q, dtype="bf16", device="cuda", workspace=True):
        self.heads, self.n, self.d, self.c_q = int(heads), int(n), int(d), int(c_q)
        self.dtype = B.BF16 if dtype == "bf16" else B.F32
        self.tdtype = torch.bfloat16 if self.dtype == B.BF16 else torch.float32
        self.shape = B.make_shape(heads, n, d, self.dtype, _dummy_ranges(self.d))
        self.device = torch.device(device)
        self.workspace = (B.alloc_training_workspace(self.shape, self.c_q, device) if workspace
                          else None)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self._out = self._grads = None

    def _scratch(self, stream):
        if self.workspace is not None:
            return self.workspace
        with _allocating_on(stream):
            return B.alloc_training_workspace(self.shape, self.c_q, self.device)

    def _rows(self):
        return torch.empty(self.heads, self.n, self.d, dtype=self.tdtype, device=self.device)

    def outputs(self):
        """New (out, lse) buffers."""
        return self._rows(), torch.empty(self.heads, self.n, dtype=torch.float32,
                                         device=self.device)

    def gradients(self):
        """New (dq, dk, dv) buffers."""
        return self._rows(), self._rows(), self._rows()

    def forward(self, q, k, v, offsets, perm, sel_counts, sel_idx, scale=0.0, dropout=0.0,
                rng=None, into=None, stream=None):
        """Returns (out, lse): `into`, or the buffers this object holds."""
        if into is None:
            with _allocating_on(stream):
                self._out = into = self._out or self.outputs()
        B.scope_sparse_attention_train(self.shape, q, k, v, self.c_q, offsets, perm, sel_counts,
                                       sel_idx, scale, dropout, rng, *into,
                                       self._scratch(stream), stream)
        return into

    def backward(self, q, k, v, out, lse, d_out, offsets, perm, sel_counts, sel_idx, scale=0.0,
                 dropout=0.0, rng=None, into=None, stream=None):
        """Returns (dq, dk, dv): `into`, or the buffers this object holds."""
        if into is None:
            with _allocating_on(stream):
                self._grads = into = self._grads or self.gradients()
        B.scope_sparse_attention_backward(self.shape, q, k, v, out, lse, d_out, self.c_q, offsets,
                                          perm, sel_counts, sel_idx, scale, dropout, rng, *into,
                                          self._scratch(stream), self.status, stream)
        return into


class _AttentionFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, owner, sets, scale, dropout, rng):
        attention = owner.autograd_attention()
        # the mask belongs to the values that rng holds now
        rng = rng.clone() if rng is not None else None
        out, lse = attention.forward(q, k, v, *sets, scale, dropout, rng,
                                     into=attention.outputs())
        ctx.save_for_backward(q, k, v, out, lse, *sets, *(() if rng is None else (rng,)))
        ctx.owner, ctx.scale, ctx.dropout = owner, scale, dropout
        ctx.selection = owner.selection
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_out):
        q, k, v, out, lse, offsets, perm, sel_counts, sel_idx, *rng = ctx.saved_tensors
        if ctx.owner.selection != ctx.selection:
            raise RuntimeError("the layer's clusters or key sets changed between this attention "
                               "and its backward pass")
        attention = ctx.owner.autograd_attention()
        d_out = d_out.contiguous()
        if d_out.data_ptr() % 16:  # a piece of another tensor's gradient
            d_out = d_out.clone()
        grads = attention.backward(q, k, v, out, lse, d_out, offsets, perm, sel_counts, sel_idx,
                                   ctx.scale, ctx.dropout, rng[0] if rng else None,
                                   into=attention.gradients())
        # each of its input's shape, which may name [heads][n][d] in other ways
        grads = [g.view(x.shape) if need else None
                 for g, x, need in zip(grads, (q, k, v), ctx.needs_input_grad)]
        return (*grads, None, None, None, None, None)


class _DropoutFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, rng, stream):
        rng = rng.clone() if rng is not None else None
        ctx.save_for_backward(*(() if rng is None else (rng,)))
        ctx.p = p
        y = torch.empty_like(x)
        B.scope_dropout(x, residual, p, rng, y, stream)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_y):
        dx = None
        if ctx.needs_input_grad[0]:
            d_y = d_y.contiguous()
            dx = torch.empty_like(d_y)
            B.scope_dropout(d_y, None, ctx.p, ctx.saved_tensors[0] if ctx.saved_tensors else None,
                            dx)
        return dx, d_y if ctx.needs_input_grad[1] else None, None, None, None


def dropout(x, p, rng, residual=None, out=None, stream=None):
    """x / (1 - p) where kept, else 0, plus `residual` (call 8), into `out` or a
    new tensor; differentiable in x and residual (in reverse mode; forward mode is
    refused), except into `out`, which is refused where a gradient is asked for.  `rng` is an int64 tensor (seed,
    offset) on the GPU."""
    if residual is not None and residual.shape != x.shape:
        raise ValueError(f"residual is {tuple(residual.shape)}, x {tuple(x.shape)}")
    _refuse_tangents("dropout", x, residual, out)
    if torch.is_grad_enabled() and (
            x.requires_grad or residual is not None and residual.requires_grad
            or out is not None and out.requires_grad):
        if out is not None:
            raise ValueError("dropout into `out` is not differentiable: leave `out` away, or call "
                             "it under torch.no_grad()")
        with _allocating_on(stream):  # the backward pass runs on this stream too
            return _DropoutFunction.apply(x, residual, p, rng, stream)
    y = out
    if y is None:
        with _allocating_on(stream):
            y = torch.empty_like(x)
    B.scope_dropout(x, residual, p, rng, y, stream)
    return y


_dropout = dropout  # where an argument has the name


class _Differentiable:
    """The attention of a layer as a function that torch differentiates."""

    # counts what rewrites the clusters or key sets that a backward pass reads
    selection = 0
    _training = _autograd = None

    def _calls(self, workspace):
        return TrainingAttention(self.heads, self.n, self.d, self.offsets.shape[1] - 1,
                                 "bf16" if self.dtype == B.BF16 else "f32", self.offsets.device,
                                 workspace)

    def autograd_attention(self):
        """The training calls that `attention` makes, with a workspace for each:
        one that the layer held would be written by calls on several streams at
        once, and would be memory for every layer of a model."""
        if self._autograd is None:
            self._autograd = self._calls(workspace=False)
        return self._autograd

    def training_attention(self):
        """The training calls on buffers held by the layer, made on the first use;
        its status is that of `attention`'s calls too."""
        if self._training is None:
            self._training = self._calls(workspace=True)
            self._training.status = self.autograd_attention().status
        return self._training

    def attention(self, q, k, v, scale=0.0, dropout=0.0, rng=None):
        """Attention over the clusters and key sets that the layer holds (calls
        6 and 7), on the current stream, differentiable in q, k and v, whose
        gradients have their shapes.  The sets must not be rewritten (a new
        clustering or selection) before the backward pass has run.  To capture
        a graph, call `training_attention`'s forward and backward: they
        allocate nothing when given their outputs."""
        count = self.heads * self.n * self.d
        for t, name in ((q, "q"), (k, "k"), (v, "v")):
            if torch.is_grad_enabled() and t.requires_grad and t.numel() != count:
                raise ValueError(f"{name} needs {count} elements for its gradient, "
                                 f"has {t.numel()}")
        return _AttentionFunction.apply(
            q, k, v, self, (self.offsets, self.perm, self.sel_counts, self.sel_idx), float(scale),
            float(dropout), rng)


class ScopeLayer(_Differentiable):
    def __init__(self, heads, n, d, ranges, c_q, c_m, iters, rho, k_fix,
                 dtype="bf16", device="cuda", materialize_scores=False,
                 workspace=True):
        self.heads, self.n, self.d = int(heads), int(n), int(d)
        self.ranges = (tuple(map(int, ranges[0])), tuple(map(int, ranges[1])))
        self.c_q = int(c_q)
        self.c_m = tuple(int(c) for c in c_m)
        self.iters, self.rho, self.k_fix = int(iters), float(rho), int(k_fix)
        self.dtype = B.BF16 if dtype == "bf16" else B.F32
        self.tdtype = torch.bfloat16 if self.dtype == B.BF16 else torch.float32
        self.shape = B.make_shape(heads, n, d, self.dtype, self.ranges)
        H, N, D, C = self.heads, self.n, self.d, self.c_q
        cs = sum(self.c_m)
        per_head = sum(self.c_m[m] * self.ranges[1][m] for m in range(3))
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.q_centroids = torch.empty(H, C, D, **f32)
        self.assign = torch.empty(H, N, **i32)
        self.counts = torch.empty(H, C, **i32)
        self.offsets = torch.empty(H, C + 1, **i32)
        self.perm = torch.empty(H, N, **i32)
        self.k_centroids = torch.empty(H, per_head, **f32)
        self.codes = torch.empty(H, N, **i32)
        self.tables = torch.empty(H, C, cs, **f32)
        self.scores = torch.empty(H, C, N, **f32) if materialize_scores else None
        self.base_counts = torch.empty(H, C, **i32)
        self.topp_counts = torch.empty(H, C, **i32)
        self.k_head = torch.empty(H, **i32)
        self.sel_counts = torch.empty(H, C, **i32)
        self.sel_idx = torch.empty(H, C, N, **i32)
        self.out = torch.empty(H, N, D, dtype=self.tdtype, device=device)
        self.workspace = (B.alloc_workspace(self.shape, C, self.c_m, device)
                          if workspace else None)
        self.status = torch.zeros(1, **i32)

    # the five stages -------------------------------------------------------
    def cluster_queries(self, q, init_q=None, stream=None, warm=False, iters=None):
        """warm: start from the centroids this layer holds (calls 1w)."""
        it = self.iters if iters is None else int(iters)
        self.selection += 1
        if warm:
            B.scope_cluster_queries_warm(self.shape, q, self.c_q, it, self.q_centroids,
                                         self.assign, self.counts, self.offsets, self.perm,
                                         self.workspace, self.status, stream)
            return
        B.scope_cluster_queries(self.shape, q, self.c_q, it, init_q,
                                self.q_centroids, self.assign, self.counts,
                                self.offsets, self.perm, self.workspace,
                                self.status, stream)

    def cluster_keys(self, k, init_k=None, stream=None, warm=False, iters=None):
        """warm: start from the codebooks this layer holds (call 2w)."""
        it = self.iters if iters is None else int(iters)
        if warm:
            B.scope_cluster_key_subspaces_warm(self.shape, k, self.c_m, it, self.k_centroids,
                                               self.codes, self.workspace, self.status, stream)
            return
        stride = init_k.shape[-1] if init_k is not None else 0
        B.scope_cluster_key_subspaces(self.shape, k, self.c_m, it,
                                      init_k, stride, self.k_centroids,
                                      self.codes, self.workspace, self.status,
                                      stream)

    def proxy_scores(self, stream=None):
        B.scope_proxy_scores(self.shape, self.q_centroids, self.c_q,
                             self.k_centroids, self.c_m, self.codes,
                             self.tables, self.scores, stream)

    def select(self, stream=None, use_scores=False, policy="online", rho=None):
        """policy "online" is call 4 (Eq. 10); "fixed" and "topp" are the
        Fig. 6 variants through call 4b.  rho overrides the layer's."""
        rho = self.rho if rho is None else rho
        self.selection += 1
        args = (self.shape, self.c_q, self.c_m,
                self.scores if use_scores else None, self.tables,
                self.codes, self.counts, rho, self.k_fix,
                self.base_counts, self.topp_counts, self.k_head,
                self.sel_counts, self.sel_idx, self.workspace)
        if policy == "online":
            B.scope_select(*args, stream)
        else:
            B.scope_select_policy(*args, policy, stream)

    def attend(self, q, k, v, scale=0.0, stream=None):
        B.scope_sparse_attention(self.shape, q, k, v, self.c_q, self.offsets,
                                 self.perm, self.sel_counts, self.sel_idx,
                                 scale, self.out, self.workspace, stream)

    def forward(self, q, k, v, init_q=None, init_k=None, stream=None,
                marks=None, warm=False, warm_iters=None):
        """Runs the layer; `marks(i)` (if given) is called before stage i and
        after the last one, e.g. to record timing events.  warm: the
        clusterings start from the centroids the layer holds (the previous
        denoising step's), with warm_iters iterations (default: iters)."""
        steps = (lambda: self.cluster_queries(q, init_q, stream, warm, warm_iters),
                 lambda: self.cluster_keys(k, init_k, stream, warm, warm_iters),
                 lambda: self.proxy_scores(stream),
                 lambda: self.select(stream),
                 lambda: self.attend(q, k, v, 0.0, stream))
        for i, f in enumerate(steps):
            if marks:
                marks(i)
            f()
        if marks:
            marks(len(steps))
        return self.out

    def forward_train(self, q, k, v, init_q=None, init_k=None, dropout=0.0, rng=None,
                      residual=None, out_dropout=0.0, warm=False, warm_iters=None):
        """The layer for training, on the current stream: clusters and key sets
        from q and k without gradients, the attention over them with `dropout`
        on its probabilities, then out_dropout on its output and the residual
        added (where either is given).  Differentiable in q, k, v and residual;
        one forward at a time: its backward pass comes before the next forward."""
        with torch.no_grad():
            self.cluster_queries(q.detach(), init_q, None, warm, warm_iters)
            self.cluster_keys(k.detach(), init_k, None, warm, warm_iters)
            self.proxy_scores()
            self.select()
        out = self.attention(q, k, v, 0.0, dropout, rng)
        if residual is None and not out_dropout:
            return out
        return _dropout(out, out_dropout, rng, residual)


class SparsitySchedule:
    """Where the layer runs across a DiT's layers and denoising steps (Sec. 4
    setup): the first attention layer stays dense at every step, and the
    other layers stay dense during the first `dense_fraction` of the steps
    (20% for the Wan models, 10% for HunyuanVideo), SCOPE afterwards.  The
    first SCOPE step of a layer clusters from seeded rows; later steps may
    warm-start from the previous step's centroids."""

    def __init__(self, steps, dense_fraction, dense_layers=(0,)):
        self.steps = int(steps)
        self.dense_fraction = float(dense_fraction)
        self.dense_layers = frozenset(int(x) for x in dense_layers)
        # the dense prefix in whole steps, ceil(fraction * steps) exactly
        from fractions import Fraction
        f = Fraction(str(dense_fraction)) * self.steps
        self.dense_steps = -((-f.numerator) // f.denominator)

    def dense(self, layer, step):
        return layer in self.dense_layers or step < self.dense_steps

    def warm(self, layer, step):
        """True when the previous step of this layer also ran SCOPE."""
        return not self.dense(layer, step) and step > self.dense_steps


def _dummy_ranges(d):
    """Three valid ranges for the calls that check but do not use them."""
    a = d // 3 // 2 * 2
    ln = (a, a, d - 2 * a)
    return (0, ln[0], ln[0] + ln[1]), ln


class ScopePartitionLayer(ScopeLayer):
    """The layer with the keys split into any M disjoint channel sets (App. B;
    the partition ablation of Table 3), through the partition calls: codes
    are one uint16 plane per subspace (held in an int16 tensor)."""

    def __init__(self, heads, n, d, sets, c_q, c_m, iters, rho, k_fix,
                 dtype="bf16", device="cuda", materialize_scores=False):
        self.sets = [tuple(map(int, x)) for x in sets]
        self.part = B.make_partition(self.sets, c_m)
        M = len(self.sets)
        # the query and attention calls see three placeholder ranges
        super().__init__(heads, n, d, _dummy_ranges(d), c_q, (1, 1, 1), iters,
                         rho, k_fix, dtype, device, materialize_scores,
                         workspace=False)
        self.c_m = tuple(int(c) for c in c_m)
        H, N, C = self.heads, self.n, self.c_q
        per_head = sum(self.c_m[m] * len(self.sets[m]) for m in range(M))
        self.k_centroids = torch.empty(H, per_head, dtype=torch.float32, device=device)
        self.codes = torch.empty(H, M, N, dtype=torch.int16, device=device)
        self.tables = torch.empty(H, C, sum(self.c_m), dtype=torch.float32, device=device)
        self.workspace = B.alloc_partition_workspace(self.shape, C, self.part, device)

    def cluster_keys(self, k, init_k=None, stream=None, warm=False, iters=None):
        if warm:
            raise NotImplementedError("warm starts are offered for the three RoPE ranges only")
        stride = init_k.shape[-1] if init_k is not None else 0
        B.scope_cluster_key_partition(self.shape, k, self.part,
                                      self.iters if iters is None else int(iters), init_k,
                                      stride, self.k_centroids, self.codes,
                                      self.workspace, self.status, stream)

    def proxy_scores(self, stream=None):
        B.scope_proxy_scores_partition(self.shape, self.q_centroids, self.c_q,
                                       self.k_centroids, self.part, self.codes,
                                       self.tables, self.scores, self.workspace,
                                       stream)

    def select(self, stream=None, use_scores=False, policy="online", rho=None):
        rho = self.rho if rho is None else rho
        self.selection += 1
        B.scope_select_partition(self.shape, self.c_q, self.part,
                                 self.scores if use_scores else None, self.tables,
                                 self.codes, self.counts, rho, self.k_fix,
                                 self.base_counts, self.topp_counts, self.k_head,
                                 self.sel_counts, self.sel_idx, self.workspace,
                                 policy, stream)


class DenseAttention(_Differentiable):
    """Dense attention (Eq. 1) through the same attention call: one cluster
    holding every query, whose key set is every key."""

    def __init__(self, heads, n, d, dtype="bf16", device="cuda"):
        self.heads, self.n, self.d = int(heads), int(n), int(d)
        self.dtype = B.BF16 if dtype == "bf16" else B.F32
        tdt = torch.bfloat16 if self.dtype == B.BF16 else torch.float32
        self.shape = B.make_shape(heads, n, d, self.dtype, _dummy_ranges(d))
        i32 = dict(dtype=torch.int32, device=device)
        H, N = self.heads, self.n
        self.offsets = torch.tensor([0, N], **i32).repeat(H, 1).contiguous()
        self.perm = torch.arange(N, **i32).repeat(H, 1).contiguous()
        self.sel_counts = torch.full((H, 1), N, **i32)
        self.sel_idx = torch.arange(N, **i32).repeat(H, 1).reshape(H, 1, N).contiguous()
        self.out = torch.empty(H, N, d, dtype=tdt, device=device)
        self.workspace = B.alloc_workspace(self.shape, 1, (1, 1, 1), device)

    def forward(self, q, k, v, scale=0.0, stream=None):
        B.scope_sparse_attention(self.shape, q, k, v, 1, self.offsets,
                                 self.perm, self.sel_counts, self.sel_idx,
                                 scale, self.out, self.workspace, stream)
        return self.out
