"""Exact attention over sequences packed one after the other (calls 10 and 11):
clips of several sizes in one batch, prompts, chunks and single tokens behind a
cache, causal or not, with query heads in groups that share a key head.

PackedAttention stands beside layer.DenseAttention, which attends over one
sequence; like it, it allocates buffers once and makes the library's calls.
"""
from __future__ import annotations

import torch

from . import binding as B
from .layer import _allocating_on


def offsets_of(lengths, device="cuda"):
    """int32 [sequences + 1]: where sequences of these lengths start and end."""
    at = [0]
    for n in lengths:
        at.append(at[-1] + int(n))
    return torch.tensor(at, dtype=torch.int32, device=device)


class _PackedFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, owner, offsets_q, offsets_k, scale):
        out, lse = owner._forward(owner.pack, q, k, v, offsets_q, offsets_k, None, scale,
                                  owner.outputs(), owner._workspace(None), None)
        # the sequences are those that the offsets hold now
        ctx.save_for_backward(q, k, v, out, lse, offsets_q.clone(), offsets_k.clone())
        ctx.owner, ctx.scale = owner, scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_out):
        q, k, v, out, lse, offsets_q, offsets_k = ctx.saved_tensors
        owner = ctx.owner
        if not _takes(d_out):  # expanded, or a piece of another tensor's gradient
            d_out = d_out.clone(memory_format=torch.contiguous_format)
        # rows in no sequence have no gradient
        into = tuple(torch.zeros(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        grads = owner._backward(owner.pack, q, k, v, out, lse, d_out, offsets_q, offsets_k, ctx.scale,
                                into, owner._workspace(None), None)
        return (*(g if need else None for g, need in zip(grads, ctx.needs_input_grad)),
                None, None, None, None)


def _takes(t):
    """Whether the calls take a tensor [heads][rows][d] where it lies."""
    el = t.element_size()
    return (t.stride(2) == 1 and t.data_ptr() % 16 == 0
            and all(t.shape[i] == 1 or t.stride(i) * el % 16 == 0 for i in (0, 1)))


class PackedAttention:
    """Attention of `heads` query heads, rows_q rows each, over `kv_heads` key heads of
    rows_k rows, in `sequences` sequences given by offsets at each call.  Tensors are
    [heads][rows][d] with contiguous channels and any strides of heads and rows that
    keep rows on 16 bytes.  Calls that may run at once (streams, replays of captured
    graphs) need an object each.  With workspace=False it holds no workspace: every
    call takes one from torch's allocator, for the stream it runs on."""

    def __init__(self, heads, kv_heads, rows_q, rows_k, d, sequences, causal=True, dtype="bf16",
                 device="cuda", workspace=True):
        self.dtype = B.BF16 if dtype == "bf16" else B.F32
        self.tdtype = torch.bfloat16 if self.dtype == B.BF16 else torch.float32
        sizes = (heads, kv_heads, rows_q, rows_k, sequences, d, self.dtype, causal)
        self.pack = B.make_pack(*sizes)
        # into the buffers that this object holds: they have rows of earlier calls, whose
        # offsets may have covered more
        self._clearing = B.make_pack(*sizes, clear=True)
        self.device = torch.device(device)
        B.scope_packed_workspace_size(self.pack)  # refuses what the calls would
        self.workspace = B.alloc_packed_workspace(self.pack, device) if workspace else None
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self._out = self._grads = None

    def _workspace(self, stream):
        with _allocating_on(stream):
            return B.alloc_packed_workspace(self.pack, self.device)

    def outputs(self):
        """New (out, lse) buffers; rows in no sequence are 0 and -inf."""
        p = self.pack
        return (torch.zeros(p.heads, p.rows_q, p.d, dtype=self.tdtype, device=self.device),
                torch.full((p.heads, p.rows_q), float("-inf"), dtype=torch.float32,
                           device=self.device))

    def gradients(self):
        """New (dq, dk, dv) buffers; rows in no sequence are 0."""
        p = self.pack
        return tuple(torch.zeros(h, n, p.d, dtype=self.tdtype, device=self.device)
                     for h, n in ((p.heads, p.rows_q), (p.kv_heads, p.rows_k),
                                  (p.kv_heads, p.rows_k)))

    def _forward(self, pack, q, k, v, offsets_q, offsets_k, lengths_k, scale, into, workspace,
                 stream):
        B.scope_packed_attention(pack, q, k, v, offsets_q, offsets_k, lengths_k, scale, *into,
                                 workspace, self.status, stream)
        return into

    def _backward(self, pack, q, k, v, out, lse, d_out, offsets_q, offsets_k, scale, into,
                  workspace, stream):
        B.scope_packed_attention_backward(pack, q, k, v, out, lse, d_out, offsets_q, offsets_k,
                                          scale, *into, workspace, self.status, stream)
        return into

    def forward(self, q, k, v, offsets_q, offsets_k=None, lengths_k=None, scale=0.0, into=None,
                stream=None):
        """Returns (out, lse): `into`, whose rows in no sequence stay as they are, or the
        buffers this object holds, where they are set to 0 and -inf.  offsets_q and
        offsets_k (the same where not given) are int32 [sequences + 1]; lengths_k, int32
        [sequences], the keys that each sequence's rows of k and v hold so far."""
        pack = self.pack
        if into is None:
            with _allocating_on(stream):
                self._out = into = self._out or self.outputs()
            pack = self._clearing
        offsets_k = offsets_q if offsets_k is None else offsets_k
        workspace = self._workspace(stream) if self.workspace is None else self.workspace
        return self._forward(pack, q, k, v, offsets_q, offsets_k, lengths_k, scale, into, workspace,
                             stream)

    def backward(self, q, k, v, out, lse, d_out, offsets_q, offsets_k=None, scale=0.0, into=None,
                 stream=None):
        """Returns (dq, dk, dv): `into`, whose rows in no sequence stay as they are, or the
        buffers this object holds, where they are set to 0."""
        pack = self.pack
        if into is None:
            with _allocating_on(stream):
                self._grads = into = self._grads or self.gradients()
            pack = self._clearing
        offsets_k = offsets_q if offsets_k is None else offsets_k
        workspace = self._workspace(stream) if self.workspace is None else self.workspace
        return self._backward(pack, q, k, v, out, lse, d_out, offsets_q, offsets_k, scale, into,
                              workspace, stream)

    def attention(self, q, k, v, offsets_q, offsets_k=None, scale=0.0):
        """The forward's out, on the current stream, differentiable in q, k and v.  Every
        call takes its workspace from torch's allocator.  To capture a graph, call
        forward and backward: they allocate nothing when given their outputs."""
        offsets_k = offsets_q if offsets_k is None else offsets_k
        return _PackedFunction.apply(q, k, v, self, offsets_q, offsets_k, float(scale))
