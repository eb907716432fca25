"""Thin autograd wrappers over the C ABI, so the sparse operations can sit
inside an ordinary PyTorch training step (the role of the paper's C++ wrapper that connects
forward and backward propagation to the kernels, Section 3.1).  Everything numerical still runs
in the library's HIP kernels; the nodes (csrc/torch_native.cpp) only route tensors and remember what
backward needs.

There are no second derivatives: gradients made with ``create_graph=True`` raise NotImplementedError when they are differentiated.

``SparseGraph`` owns the handle; its transpose is built on the first backward and cached in the
handle for all later epochs (Section 3.3).
"""
from __future__ import annotations

import torch

from . import binding as _b

_recorder = torch._C._get_tracing_state  # None unless torch.jit.trace is recording


class SparseGraph:
    """A CSR matrix on the GPU plus its library handle.  ``values`` may be a leaf tensor that
    requires grad; its gradient is the SDDMM of (dY, X)."""

    def __init__(self, indptr, indices, values=None, n_cols=None):
        self.indptr, self.indices, self.values = indptr, indices, values
        self.handle = _b.csr_build(indptr, indices, None if values is None else values.detach(), n_cols=n_cols)
        self.n_rows, self.n_cols, self.nnz = self.handle.n_rows, self.handle.n_cols, self.handle.nnz
        self._native = _b._native().graph(self.handle._cell, self.handle, values)

    def sync_values(self):
        """The handle reads ``values``' storage directly.  When an optimizer step has rewritten it in place
        since the last call, the arrays derived from it have to pick the new values up (the transpose's structure,
        permutation and partition stay cached).  The operations below do this themselves."""
        _b._native().graph_sync(self._native)

    def transpose(self):
        self.sync_values()
        return _b.csr_transpose_cached(self.handle)[0]


def _values_without_gradient(graph: SparseGraph, what: str):
    """Refuses where a gradient with respect to the edge values is asked for, which ``what`` does not have (under torch.no_grad() none is)."""
    if graph.values is not None and graph.values.requires_grad and torch.is_grad_enabled():
        raise NotImplementedError(what)


class _Recorded(torch.autograd.Function):
    """One of the operations below while torch.jit.trace records a program: the native nodes are not among the operations
    that a recording knows (all that it would keep is the empty output they write into), an autograd function is."""

    @staticmethod
    def forward(ctx, run, values, X):
        Y = X.new_empty(0)  # (an output has to be made while the recorder looks on)
        recorder = _recorder()
        torch._C._set_tracing_state(None)
        try:
            with torch.enable_grad():
                ctx.leaves = [t if t is None else t.detach().requires_grad_(need)
                              for t, need in zip((values, X), ctx.needs_input_grad[1:])]
                ctx.output = run(*ctx.leaves)
            Y.set_(ctx.output.detach())
        finally:
            torch._C._set_tracing_state(recorder)
        ctx.save_for_backward(X)  # (X overwritten, or a second backward without retain_graph: refused)
        return Y

    @staticmethod
    def backward(ctx, dY):
        ctx.saved_tensors
        wanted = [t for t, need in zip(ctx.leaves, ctx.needs_input_grad[1:]) if need]
        got = iter(torch.autograd.grad(ctx.output, wanted, dY, retain_graph=True, create_graph=torch.is_grad_enabled()))
        return (None, *(next(got) if need else None for need in ctx.needs_input_grad[1:]))


def spmm(graph: SparseGraph, X):
    """Differentiable Y = A X (with respect to X and, if ``graph.values`` requires grad, to the values).
    X is kept for the backward only where the values have a gradient.  Without one the backward needs nothing of the
    forward, as with torch's own linear operations: X may be overwritten before it, and it may run again without
    ``retain_graph``."""
    if _recorder() is not None:
        return _Recorded.apply(lambda values, X: _b._nat.ag_spmm(graph._native, values, X), graph.values, X)
    return _b._nat.ag_spmm(graph._native, graph.values, X)


def matmul(graph: SparseGraph, X, reduce: str = "sum"):
    """The paper's matmul(sparse, dense, reduce) (Section 3.5): reduce in 'sum' | 'mean' | 'min' | 'max'.
    Differentiable with respect to X; with respect to the edge values for 'sum' only.  min / max remember the
    position of the winning entry per output element for the backward."""
    if reduce == "sum":
        return spmm(graph, X)
    if reduce not in ("mean", "min", "max"):
        raise ValueError("reduce must be 'sum', 'mean', 'min' or 'max'")
    _values_without_gradient(graph, "gradients with respect to the edge values exist for reduce='sum' only")
    if _recorder() is not None:
        return _Recorded.apply(lambda _, X: _b._nat.ag_reduce(graph._native, X, _b.REDUCE[reduce]), None, X)
    return _b._nat.ag_reduce(graph._native, X, _b.REDUCE[reduce])


def fusedmm(graph: SparseGraph, X):
    """Differentiable sigmoid FusedMM: y_i = sum_j a_ij sigmoid(<x_i, x_j>) x_j (with respect to X only)."""
    _values_without_gradient(graph, "FusedMM has no gradient with respect to the edge values")
    if _recorder() is not None:
        return _Recorded.apply(lambda _, X: _b._nat.ag_fused(graph._native, X), None, X)
    return _b._nat.ag_fused(graph._native, X)


class _RecordedRows(torch.autograd.Function):
    """_Recorded for the operators below: any number of tensors, one output or several."""

    @staticmethod
    def forward(ctx, run, *tensors):
        recorder = _recorder()
        torch._C._set_tracing_state(None)
        try:
            with torch.enable_grad():
                ctx.leaves = [t if t is None else t.detach().requires_grad_(need) for t, need in zip(tensors, ctx.needs_input_grad[1:])]
                out = run(*ctx.leaves)
        finally:
            torch._C._set_tracing_state(recorder)
        several = isinstance(out, tuple)
        ctx.outputs = out if several else (out,)
        first = next(t for t in tensors if t is not None)
        results = tuple(first.new_empty(0, dtype=o.dtype) for o in ctx.outputs)  # (made while the recorder looks on)
        torch._C._set_tracing_state(None)
        try:
            for r, o in zip(results, ctx.outputs):
                r.set_(o.detach())
        finally:
            torch._C._set_tracing_state(recorder)
        ctx.mark_non_differentiable(*(r for r, o in zip(results, ctx.outputs) if not o.requires_grad))
        ctx.save_for_backward(*(t for t in tensors if t is not None))
        return results if several else results[0]

    @staticmethod
    def backward(ctx, *grads):
        ctx.saved_tensors
        wanted = [t for t, need in zip(ctx.leaves, ctx.needs_input_grad[1:]) if need]
        pairs = [(o, g) for o, g in zip(ctx.outputs, grads) if o.requires_grad]
        got = iter(torch.autograd.grad([o for o, _ in pairs], wanted, [g for _, g in pairs], retain_graph=True,
                                       create_graph=torch.is_grad_enabled()))
        return (None, *(next(got) if need else None for need in ctx.needs_input_grad[1:]))


def layer_norm(X, weight=None, bias=None, eps: float = 1e-5):
    """Differentiable layer norm over the rows of X (fp32, bf16 or fp16; weight and bias fp32 or of X's type)."""
    nat = _b._native()
    if _recorder() is not None:
        return _RecordedRows.apply(lambda X, weight, bias: nat.ag_layer_norm(X, weight, bias, float(eps)), X, weight, bias)
    return nat.ag_layer_norm(X, weight, bias, float(eps))


def label_logprob(Z, labels, top: int = 0):
    """(logprob, entropy) of the rows of scores Z (fp32, bf16 or fp16) for int64 labels, both fp32 and differentiable with respect to Z;
    a label outside [0, classes) names no class: log probability 0, no gradient.  With top > 0 also the log probabilities and the
    classes (int32) of that many best alternatives, which have no gradient: (logprob, entropy, top_logprob, top_index)."""
    nat = _b._native()
    if _recorder() is not None:
        return _RecordedRows.apply(lambda Z, labels: nat.ag_label_logprob(Z, labels, int(top)), Z, labels)
    return nat.ag_label_logprob(Z, labels, int(top))


def attention(graph: SparseGraph, Q, K, V, heads: int, kv_heads=None, *, scale=None, bias: bool = False):
    """Differentiable attention over the graph's entries (with respect to Q, K and V): per head, Y[i] = sum over row i's entries (i, j) of
    softmax(scale <Q[i], K[j]> (+ the entry's value with bias=True)) V[j].  Q [rows, heads * c], K, V [columns, kv_heads * c], fp32, bf16 or
    fp16; heads is a multiple of kv_heads (default: heads); scale: c ** -0.5 unless given."""
    if bias:
        _values_without_gradient(graph, "the attention has no gradient with respect to the edge values")
    kv_heads = heads if kv_heads is None else kv_heads
    scale = None if scale is None else float(scale)
    call = lambda Q, K, V: _b._nat.ag_attention(graph._native, Q, K, V, int(heads), int(kv_heads), scale, _b.ISP_BIAS_BY_A if bias else 0)
    if _recorder() is not None:
        return _RecordedRows.apply(call, Q, K, V)
    return call(Q, K, V)
