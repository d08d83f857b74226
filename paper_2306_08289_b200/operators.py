"""Operators of a language model's gradient event, on torch tensors: embedding lookup and its gradient, the vocabulary
loss with its gradients, orthogonalisation of matrix updates.

Thin wrappers of the a2cid2_embed*, a2cid2_vocab_loss* and a2cid2_orthogonalize* entry points of include/a2cid2.h (formulas
and conventions there). A matrix argument is a CUDA tensor of float32 or bfloat16 whose last dimension is contiguous; it may be a
view into an engine's rows, e.g. `eng.x[w, off:off + v * h].view(v, h)` for worker w's table and the same slice of `eng.g` for its
gradient, so that gradients land where the event kernels read them. Work is queued on torch's current stream of the tensors' device,
or on `stream`; results and workspaces are allocated through torch on that stream. An argument the library cannot take raises
`binding.A2Error`.

The operators are no part of torch's autograd: gradients are calls of their own here. A tensor that requires a gradient is refused while torch
records (call under `torch.no_grad()`, or pass it detached), for its result would have no gradient.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import operator

import torch

from . import binding as B

NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)  # a quintic whose iterates send every singular value into about [0.7, 1.2]

_sizes: dict = {}
_DTYPES = {torch.float32: B.A2_F32, torch.bfloat16: B.A2_BF16}


def _refuse(text):
    raise B.A2Error(B.A2_EINVAL, text)


def _refuse_recorded(name, t):
    if t.requires_grad and torch.is_grad_enabled():
        _refuse(f"{name} requires a gradient, which these operators do not record: call under torch.no_grad() or pass {name}.detach()")


def _matrix(name, t, like=None, shape=None, ndim=2):
    """Checks a matrix (or a batch of them) and returns its row pitch."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name} must be a CUDA tensor")
    if t.dtype not in _DTYPES:
        _refuse(f"{name} must be float32 or bfloat16")
    _refuse_recorded(name, t)
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        _refuse(f"{name} must have the type and device of the other matrices")
    dims, strides = t.shape, t.stride()
    if len(dims) != ndim or (shape is not None and dims != shape):
        _refuse(f"{name} has shape {tuple(dims)}" + (f", {tuple(shape)} needed" if shape is not None else f", {ndim} dimensions needed"))
    if dims[-1] != 1 and strides[-1] != 1:
        _refuse(f"the last dimension of {name} must be contiguous")
    return strides[-2] if dims[-2] > 1 else max(dims[-1], 1)


def _vector(name, t, n, dtype, device):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} vector of {n} elements on {device}")
    _refuse_recorded(name, t)
    return t.data_ptr()


class _Queue:
    """The context in which a call allocates and queues: the tensors' device and the stream. Entering it gives the raw stream. `given` are the
    caller's tensors (or None), `made` collects results allocated here: with a stream of the caller's, torch's allocator is told that the
    former are used on it and that the latter are used on the caller's current one, so that neither is handed out again too early."""

    __slots__ = ("device", "stream", "given", "made", "inner")

    def __init__(self, device, stream, *given):
        self.device, self.stream, self.given, self.made, self.inner = device, stream, given, [], None

    def __enter__(self):
        if self.stream is None and torch._C._cuda_getDevice() == self.device.index:
            return torch._C._cuda_getCurrentRawStream(self.device.index)  # nothing to switch: the usual case, kept short
        if self.stream is not None and self.stream.device != self.device:
            _refuse(f"the stream is one of {self.stream.device}, the tensors are on {self.device}")
        self.inner = contextlib.ExitStack()
        self.inner.enter_context(torch.cuda.device(self.device))
        stream = torch.cuda.current_stream(self.device) if self.stream is None else self.stream
        self.inner.enter_context(torch.cuda.stream(stream))
        return stream.cuda_stream

    def __exit__(self, *exc):
        if self.inner is None:
            return False
        self.inner.__exit__(*exc)
        if self.stream is not None:
            caller = torch.cuda.current_stream(self.device)
            for t in self.given:
                if isinstance(t, torch.Tensor):
                    t.record_stream(self.stream)
            for t in self.made:
                t.record_stream(caller)
        return False


def _workspace(like, size_of, *args):
    """A workspace of the size the library asks for: (tensor or None, address, bytes). The size depends on the arguments alone, so the
    library is asked once for each."""
    size = _sizes.get((size_of, args))
    if size is None:
        need = C.c_int64()
        B._check(getattr(B.lib(), size_of)(*args, C.byref(need)))
        if len(_sizes) >= 4096:
            _sizes.clear()
        size = _sizes[size_of, args] = need.value
    if size == 0:
        return None, None, 0
    ws = torch.empty(size, dtype=torch.uint8, device=like.device)
    return ws, ws.data_ptr(), size


def embed(table, ids, scale=1.0, out=None, stream=None):
    """out[t] = scale * table[ids[t]]; a row of zeros where ids[t] lies outside the table. table [vocab, width], ids int32 [n]."""
    pitch = _matrix("table", table)
    n, (vocab, width) = ids.numel() if isinstance(ids, torch.Tensor) else 0, table.shape
    ids_p = _vector("ids", ids, n, torch.int32, table.device)
    queue = _Queue(table.device, stream, table, ids, out)
    with queue as s:
        if out is None:
            out, out_pitch = torch.empty(n, width, dtype=table.dtype, device=table.device), width
            queue.made.append(out)
        else:
            out_pitch = _matrix("out", out, table, (n, width))
        B._check(B.lib().a2cid2_embed(table.data_ptr(), vocab, width, pitch, ids_p, n, scale, out.data_ptr(), out_pitch,
                                      _DTYPES[table.dtype], s))
    return out


def embed_grad(grad_out, ids, vocab, scale=1.0, out=None, accumulate=False, stream=None):
    """The gradient of `embed` for its table: out[v] = scale * sum of grad_out[t] over ids[t] = v, out [vocab, width].
    With accumulate it is added to `out`, which must then be given."""
    pitch = _matrix("grad_out", grad_out)
    n, width = grad_out.shape
    ids_p = _vector("ids", ids, n, torch.int32, grad_out.device)
    if accumulate and out is None:
        _refuse("accumulate needs out")
    try:
        vocab = operator.index(vocab)
    except TypeError:
        _refuse("vocab must be a whole number")
    queue = _Queue(grad_out.device, stream, grad_out, ids, out)
    with queue as s:
        ws, ws_p, size = _workspace(grad_out, "a2cid2_embed_grad_workspace", vocab, width, n)  # checks the sizes
        if out is None:
            out = torch.empty(vocab, width, dtype=grad_out.dtype, device=grad_out.device)
            queue.made.append(out)
        out_pitch = _matrix("out", out, grad_out, (vocab, width))
        B._check(B.lib().a2cid2_embed_grad(grad_out.data_ptr(), pitch, ids_p, n, vocab, width, scale, int(accumulate), out.data_ptr(),
                                           out_pitch, _DTYPES[grad_out.dtype], ws_p, size, s))
    return out


def _vocab_loss(hidden, head, targets, weights, scale, grad_hidden, grad_head, stream):
    hidden_pitch = _matrix("hidden", hidden)
    head_pitch = _matrix("head", head, hidden)
    (n, width), vocab, device = hidden.shape, head.shape[0], hidden.device
    if head.shape[1] != width:
        _refuse(f"hidden has {width} columns, head {head.shape[1]}")
    targets_p = _vector("targets", targets, n, torch.int32, device)
    weights_p = None if weights is None else _vector("weights", weights, n, torch.float32, device)
    queue = _Queue(device, stream, hidden, head, targets, weights, grad_hidden, grad_head)
    with queue as s:
        grads = []
        for name, g, like in (("grad_hidden", grad_hidden, hidden), ("grad_head", grad_head, head)):
            if g is True:
                g = torch.empty(like.shape, dtype=like.dtype, device=device)
                queue.made.append(g)
            pitch = 0 if g is None else _matrix(name, g, like, like.shape)
            grads += [g, None if g is None else g.data_ptr(), pitch]
        gh, gh_p, gh_pitch, gw, gw_p, gw_pitch = grads
        loss = torch.empty(n, dtype=torch.float32, device=device)
        lse = torch.empty(n, dtype=torch.float32, device=device)
        queue.made += (loss, lse)
        dtype = _DTYPES[hidden.dtype]
        ws, ws_p, size = _workspace(hidden, "a2cid2_vocab_loss_workspace", n, width, vocab, int(gh is not None or gw is not None), dtype)
        B._check(B.lib().a2cid2_vocab_loss(hidden.data_ptr(), hidden_pitch, head.data_ptr(), head_pitch, targets_p, n, width, vocab,
                                           weights_p, scale, loss.data_ptr(), lse.data_ptr(), gh_p, gh_pitch, gw_p, gw_pitch, dtype,
                                           ws_p, size, s))
    return loss, lse, gh, gw


def vocab_loss(hidden, head, targets, stream=None):
    """(loss, lse), float32 [n]: softmax cross entropy of hidden [n, width] over the rows of head [vocab, width], and the logarithm of each
    token's sum of exponentials. loss is 0 where targets[t] (int32) lies outside the vocabulary."""
    return _vocab_loss(hidden, head, targets, None, 1.0, None, None, stream)[:2]


def vocab_loss_grad(hidden, head, targets, weights=None, scale=1.0, grad_hidden=True, grad_head=True, stream=None):
    """(loss, lse, grad_hidden, grad_head): as `vocab_loss`, with the gradients of sum_t scale * weights[t] * loss[t] (weights float32 [n], ones
    if None). grad_hidden and grad_head are True (allocate), None (leave out) or the tensor to write."""
    return _vocab_loss(hidden, head, targets, weights, scale, grad_hidden, grad_head, stream)


def orthogonalize(mats, steps=5, coeffs=NEWTON_SCHULZ, eps=1e-7, scale=1.0, out=None, stream=None):
    """Newton-Schulz orthogonalisation of a matrix [rows, cols] or a batch [mats, rows, cols] (e.g. one matrix of every worker's row:
    `eng.g[:, off:off + r * c].view(-1, r, c)`). out may be `mats` itself."""
    if isinstance(mats, torch.Tensor) and mats.dim() == 2:
        if out is not None:
            _matrix("out", out, mats, mats.shape)
        return orthogonalize(mats[None], steps, coeffs, eps, scale, None if out is None else out[None], stream)[0]
    pitch = _matrix("mats", mats, ndim=3)
    if len(coeffs) != 3:
        _refuse("coeffs are three numbers")
    n, rows, cols = mats.shape
    queue = _Queue(mats.device, stream, mats, out)
    with queue as s:
        if out is None:
            out = torch.empty(mats.shape, dtype=mats.dtype, device=mats.device)
            queue.made.append(out)
        out_pitch = _matrix("out", out, mats, mats.shape, ndim=3)
        dtype = _DTYPES[mats.dtype]
        ws, ws_p, size = _workspace(mats, "a2cid2_orthogonalize_workspace", n, rows, cols, dtype)
        B._check(B.lib().a2cid2_orthogonalize(mats.data_ptr(), mats.stride(0), pitch, n, rows, cols, steps, *coeffs, eps, scale, out.data_ptr(),
                                              out.stride(0), out_pitch, dtype, ws_p, size, s))
    return out


def check(stream=None):
    """Waits for the stream (torch's current one if None) and raises `binding.A2Error` if a kernel of the products gave up a wait on its device
    since this was last raised. Until then every operator on that device raises it too."""
    stream = torch.cuda.current_stream() if stream is None else stream
    with torch.cuda.device(stream.device):
        B._check(B.lib().a2cid2_operators_check(stream.cuda_stream))
