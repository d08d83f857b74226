"""Operators of a language model's gradient event, on torch tensors: embedding lookup and its gradient, the vocabulary
loss with its gradients, orthogonalisation of matrix updates, the root-mean-square norm (also to 8 bits) and its gradient, routing to
experts and its gradient, the norm of a gradient and its clipping.

Thin wrappers of the a2cid2_embed*, a2cid2_vocab_loss*, a2cid2_orthogonalize*, a2cid2_rms_norm*, a2cid2_dequantize_e4m3, a2cid2_route* and
a2cid2_*_gradient* entry points of include/a2cid2.h (formulas and conventions there). A matrix argument is a CUDA tensor of float32 or bfloat16 whose last dimension is contiguous; it may be a
view into an engine's rows, e.g. `eng.x[w, off:off + v * h].view(v, h)` for worker w's table and the same slice of `eng.g` for its
gradient, so that gradients land where the event kernels read them. Work is queued on torch's current stream of the tensors' device,
or on `stream`; results and workspaces are allocated through torch on that stream. An argument the library cannot take raises
`binding.A2Error`.

The operators are no part of torch's autograd: gradients are calls of their own here. A tensor that requires a gradient is refused while torch
records (call under `torch.no_grad()`, or pass it detached), for its result would have no gradient.
"""
from __future__ import annotations

import array
import contextlib
import ctypes as C
import importlib
import operator
import warnings

import torch

from . import binding as B
from . import build

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


_calls = None


class _NoCalls:
    """In the place of the module below where that cannot be loaded: every call is left to the code in Python."""

    def __getattr__(self, name):
        return lambda *arguments: None


def _usual():
    """The module that takes the usual calls (csrc/torch_calls.cpp): its functions return None for what they leave to the code below them."""
    global _calls
    if _calls is None:
        B.lib()  # says so if nothing has been built
        try:
            if build.calls_version() != torch.__version__:
                raise ImportError(f"it was built for torch {build.calls_version()}, this is {torch.__version__}")
            module = importlib.import_module(__package__ + "._calls")
            module.set_error(B.A2Error)
        except ImportError as e:
            warnings.warn(f"the host side of the operators' usual calls cannot be loaded ({e}), so small calls take some 5 to 25 us longer: "
                          "build it with `python -m paper_2306_08289_b200.build`", RuntimeWarning, stacklevel=3)
            module = _NoCalls()
        _calls = module
    return _calls


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
    vocab = _whole("vocab", vocab)
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


def _whole(name, v):
    try:
        return operator.index(v)
    except TypeError:
        _refuse(f"{name} must be a whole number")


def _norm_inputs(x, weight, residual, sum_out):
    """(pitches of x, residual and sum_out, address of weight) after their checks."""
    x_pitch = _matrix("x", x)
    shape = x.shape
    weight_p = None if weight is None else _vector("weight", weight, shape[1], x.dtype, x.device)
    r_pitch = 0 if residual is None else _matrix("residual", residual, x, shape)
    if sum_out is not None and residual is None:
        _refuse("sum_out needs a residual")
    s_pitch = shape[1] if sum_out is None else _matrix("sum_out", sum_out, x, shape)
    return x_pitch, r_pitch, s_pitch, weight_p


def rms_norm(x, weight=None, residual=None, eps=1e-6, out=None, sum_out=None, stream=None):
    """s / sqrt(mean(s^2) + eps) * weight for every row of s = x + residual; x, residual [n, width], weight [width] of their type. Without a residual
    returns the result, with one (result, s). out may be x or residual, sum_out x or residual."""
    if stream is None and out is None and sum_out is None:
        done = _usual().rms_norm(x, weight, residual, eps)
        if done is not None:
            return done
    x_pitch, r_pitch, s_pitch, weight_p = _norm_inputs(x, weight, residual, sum_out)
    n, width = x.shape
    queue = _Queue(x.device, stream, x, weight, residual, out, sum_out)
    with queue as s:
        if out is None:
            out, out_pitch = torch.empty(n, width, dtype=x.dtype, device=x.device), width
            queue.made.append(out)
        else:
            out_pitch = _matrix("out", out, x, x.shape)
        if residual is not None and sum_out is None:
            sum_out = torch.empty(n, width, dtype=x.dtype, device=x.device)
            queue.made.append(sum_out)
        B._check(B.lib().a2cid2_rms_norm(x.data_ptr(), x_pitch, None if residual is None else residual.data_ptr(), r_pitch, weight_p, n, width, eps,
                                         None if sum_out is None else sum_out.data_ptr(), s_pitch, out.data_ptr(), out_pitch, _DTYPES[x.dtype], s))
    return out if residual is None else (out, sum_out)


def rms_norm_quantized(x, weight=None, residual=None, eps=1e-6, block=128, sum_out=None, stream=None):
    """As `rms_norm` with the result in 8 bits: (values float8_e4m3fn [n, width], scales float32 [n, blocks]), and s where there is a residual. A scale
    is that of `block` columns (32, 64, 128, or 0 for a whole row): the result is values * scale (`dequantize`)."""
    if stream is None and sum_out is None:
        done = _usual().rms_norm_quantized(x, weight, residual, eps, block)
        if done is not None:
            return done
    x_pitch, r_pitch, s_pitch, weight_p = _norm_inputs(x, weight, residual, sum_out)
    n, width = x.shape
    block = _whole("block", block)
    if block not in (0, 32, 64, 128):
        _refuse("block is 32, 64, 128 or 0 for whole rows")
    queue = _Queue(x.device, stream, x, weight, residual, sum_out)
    with queue as s:
        values = torch.empty(n, width, dtype=torch.float8_e4m3fn, device=x.device)
        scales = torch.empty(n, -(-width // block) if block else 1, dtype=torch.float32, device=x.device)
        queue.made += (values, scales)
        if residual is not None and sum_out is None:
            sum_out = torch.empty(n, width, dtype=x.dtype, device=x.device)
            queue.made.append(sum_out)
        B._check(B.lib().a2cid2_rms_norm_e4m3(x.data_ptr(), x_pitch, None if residual is None else residual.data_ptr(), r_pitch, weight_p, n, width, eps,
                                              None if sum_out is None else sum_out.data_ptr(), s_pitch, block, values.data_ptr(), width, scales.data_ptr(),
                                              _DTYPES[x.dtype], s))
    return (values, scales) if residual is None else (values, scales, sum_out)


def dequantize(values, scales, dtype=torch.bfloat16, out=None, stream=None):
    """values * scales in float32 or bfloat16, for what `rms_norm_quantized` returns. The columns of a scale follow from the shapes: the whole row for
    one scale a row of more than 128 columns, else 32, 64 or 128."""
    if stream is None and out is None and dtype in _DTYPES:
        done = _usual().dequantize(values, scales, _DTYPES[dtype])
        if done is not None:
            return done
    if not isinstance(values, torch.Tensor) or not values.is_cuda or values.dtype != torch.float8_e4m3fn or values.dim() != 2:
        _refuse("values must be a CUDA matrix of float8_e4m3fn")
    n, width = values.shape
    if width != 1 and values.stride(1) != 1:
        _refuse("the last dimension of values must be contiguous")
    if not isinstance(scales, torch.Tensor) or scales.dtype != torch.float32 or scales.device != values.device or scales.dim() != 2 \
            or scales.shape[0] != n or not scales.is_contiguous():
        _refuse(f"scales must be a contiguous torch.float32 matrix of {n} rows on {values.device}")
    _refuse_recorded("scales", scales)
    if dtype not in _DTYPES:
        _refuse("dtype must be float32 or bfloat16")
    blocks = scales.shape[1]
    block = 0 if blocks == 1 else next((b for b in (32, 64, 128) if -(-width // b) == blocks), None)
    if block is None:
        _refuse(f"{blocks} scales a row for {width} columns")
    queue = _Queue(values.device, stream, values, scales, out)
    with queue as s:
        if out is None:
            out, out_pitch = torch.empty(n, width, dtype=dtype, device=values.device), width
            queue.made.append(out)
        else:
            out_pitch = _matrix("out", out, None, (n, width))
            if out.dtype != dtype or out.device != values.device:
                _refuse(f"out must be {dtype} on {values.device}")
        B._check(B.lib().a2cid2_dequantize_e4m3(values.data_ptr(), values.stride(0) if n > 1 else width, scales.data_ptr(), n, width, block, out.data_ptr(), out_pitch,
                                                _DTYPES[dtype], s))
    return out


def rms_norm_grad(grad_out, x, weight=None, eps=1e-6, grad_sum=None, grad_x=True, grad_weight=True, stream=None):
    """(grad_x, grad_weight): the gradients of `rms_norm` for its rows x (with a residual: the s it returned; grad_sum is then the gradient that reaches s
    by its other use, and grad_x that of both x and the residual). grad_x and grad_weight are True (allocate), None (leave out) or
    the tensor to write; without a weight grad_weight is None. grad_x may be grad_out, grad_sum or x."""
    if stream is None and (grad_x is True or grad_x is None) and (grad_weight is True or grad_weight is None):
        done = _usual().rms_norm_grad(grad_out, x, weight, eps, grad_sum, grad_x, grad_weight)
        if done is not None:
            return done
    g_pitch = _matrix("grad_out", grad_out)
    x_pitch = _matrix("x", x, grad_out, grad_out.shape)
    (n, width), dtype, device = x.shape, x.dtype, x.device
    weight_p = None if weight is None else _vector("weight", weight, width, dtype, device)
    s_pitch = 0 if grad_sum is None else _matrix("grad_sum", grad_sum, x, x.shape)
    if weight is None and grad_weight is True:
        grad_weight = None
    if grad_x is not None and grad_x is not True:
        gx_pitch = _matrix("grad_x", grad_x, x, x.shape)
    else:
        gx_pitch = width
    if grad_weight is not None and grad_weight is not True:
        _vector("grad_weight", grad_weight, width, dtype, device)
    queue = _Queue(device, stream, grad_out, x, weight, grad_sum, grad_x, grad_weight)
    with queue as s:
        if grad_x is True:
            grad_x = torch.empty(n, width, dtype=dtype, device=device)
            queue.made.append(grad_x)
        if grad_weight is True:
            grad_weight = torch.empty(width, dtype=dtype, device=device)
            queue.made.append(grad_weight)
        code = _DTYPES[dtype]
        ws, ws_p, size = _workspace(x, "a2cid2_rms_norm_grad_workspace", n, width, int(grad_weight is not None), code)
        B._check(B.lib().a2cid2_rms_norm_grad(grad_out.data_ptr(), g_pitch, x.data_ptr(), x_pitch, weight_p, None if grad_sum is None else grad_sum.data_ptr(), s_pitch,
                                              n, width, eps, None if grad_x is None else grad_x.data_ptr(), gx_pitch,
                                              None if grad_weight is None else grad_weight.data_ptr(), code, ws_p, size, s))
    return grad_x, grad_weight


_SCORES = {"softmax": B.A2_SCORE_SOFTMAX, "sigmoid": B.A2_SCORE_SIGMOID}
_GROUP_SCORES = {"max": B.A2_GROUP_BEST, "top2": B.A2_GROUP_TWO_BEST}


def _named(name, v, known):
    code = known.get(v) if isinstance(v, str) else None
    if code is None:
        _refuse(f"{name} must be one of {', '.join(known)}")
    return code


def route(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_score="max", renormalize=True, scale=1.0, stream=None):
    """(ids int32 [n, k], weights float32 [n, k], counts int32 [n_experts]): the k experts of every token of logits [n, n_experts], best first, their weights
    and how many tokens have chosen each. score "softmax" or "sigmoid"; bias float32 [n_experts] is added to the scores for the choice alone; of `groups` groups of
    experts the `top_groups` best are open (group_score "max": by their best expert, "top2": by the sum of their two best). Weights are scale * score, divided by
    the chosen scores' sum with renormalize. Logits of -inf or the type's lowest value are experts that are not available; ids are -1 where too few are."""
    if stream is None and isinstance(score, str) and isinstance(group_score, str):
        done = _usual().route(logits, k, _SCORES.get(score), bias, groups, top_groups, _GROUP_SCORES.get(group_score), bool(renormalize), scale)
        if done is not None:
            return done
    pitch = _matrix("logits", logits)
    n, experts = logits.shape
    device = logits.device
    bias_p = None if bias is None else _vector("bias", bias, experts, torch.float32, device)
    k = _whole("k", k)
    score, group_score = _named("score", score, _SCORES), _named("group_score", group_score, _GROUP_SCORES)
    if not 1 <= k <= experts:
        _refuse(f"need 1 <= k <= {experts}")
    queue = _Queue(device, stream, logits, bias)
    with queue as s:
        ids = torch.empty(n, k, dtype=torch.int32, device=device)
        weights = torch.empty(n, k, dtype=torch.float32, device=device)
        counts = torch.empty(experts, dtype=torch.int32, device=device)
        queue.made += (ids, weights, counts)
        B._check(B.lib().a2cid2_route(logits.data_ptr(), pitch, n, experts, k, score, bias_p, _whole("groups", groups), _whole("top_groups", top_groups), group_score,
                                      int(bool(renormalize)), scale, ids.data_ptr(), weights.data_ptr(), counts.data_ptr(), _DTYPES[logits.dtype], s))
    return ids, weights, counts


def route_grad(logits, ids, grad_weights, score="softmax", renormalize=True, scale=1.0, out=None, stream=None):
    """The gradient of `route`'s weights for its logits, the choice held fixed: ids are what it returned, grad_weights float32 [n, k] the gradient of its weights; score,
    renormalize and scale as given to it. Entries whose id is -1 do not matter. out may be logits."""
    if stream is None and out is None and isinstance(score, str):
        done = _usual().route_grad(logits, ids, grad_weights, _SCORES.get(score), bool(renormalize), scale)
        if done is not None:
            return done
    pitch = _matrix("logits", logits)
    n, experts = logits.shape
    device = logits.device
    for name, t, dtype in (("ids", ids, torch.int32), ("grad_weights", grad_weights, torch.float32)):
        if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device or t.dim() != 2 or t.shape[0] != n or not t.is_contiguous():
            _refuse(f"{name} must be a contiguous {dtype} matrix of {n} rows on {device}")
        _refuse_recorded(name, t)
    if ids.shape != grad_weights.shape:
        _refuse("ids and grad_weights differ in shape")
    score = _named("score", score, _SCORES)
    queue = _Queue(device, stream, logits, ids, grad_weights, out)
    with queue as s:
        if out is None:
            out, out_pitch = torch.empty(n, experts, dtype=logits.dtype, device=device), experts
            queue.made.append(out)
        else:
            out_pitch = _matrix("out", out, logits, logits.shape)
        B._check(B.lib().a2cid2_route_grad(logits.data_ptr(), pitch, ids.data_ptr(), grad_weights.data_ptr(), n, experts, ids.shape[1], score, int(bool(renormalize)),
                                           scale, out.data_ptr(), out_pitch, _DTYPES[logits.dtype], s))
    return out


def _rows_of(name, shape, strides, out_strides):
    """(rows, cols, pitch, out_pitch) of a tensor whose elements may be visited in any order, the same one on both sides."""
    dims = sorted(((a, b, n) for n, a, b in zip(shape, strides, out_strides) if n != 1), reverse=True)
    merged = []
    for a, b, n in dims:
        if merged and merged[-1][0] == a * n and merged[-1][1] == b * n:
            merged[-1] = (a, b, n * merged[-1][2])
        else:
            merged.append((a, b, n))
    if merged and merged[-1][:2] == (1, 1):
        cols = merged.pop()[2]
    else:
        cols = 1
    if len(merged) > 1 or any(a < cols or b < cols for a, b, _ in merged):
        _refuse(f"{name} has strides {tuple(strides)}: rows at one distance from each other are needed")
    return (merged[0][2], cols, merged[0][0], merged[0][1]) if merged else (1, cols, cols, cols)


def _gradients(tensors, per_worker, out):
    """(descriptions for the library, number of workers, device) of a list of tensors."""
    if isinstance(tensors, torch.Tensor) or isinstance(out, torch.Tensor):
        _refuse("tensors and out are lists of tensors")
    tensors = list(tensors)
    if not tensors:
        _refuse("no tensors")
    out = tensors if out is None else list(out)
    if len(out) != len(tensors):
        _refuse(f"{len(tensors)} tensors, but {len(out)} to write to")
    device, workers, words = None, None, []
    for t, o in zip(tensors, out):
        for v in (t,) if o is t else (t, o):
            if not isinstance(v, torch.Tensor) or not v.is_cuda:
                _refuse("a gradient's tensors must be CUDA tensors")
            if v.dtype not in _DTYPES:
                _refuse("a gradient's tensors must be float32 or bfloat16")
            _refuse_recorded("a gradient's tensor", v)
            if device is None:
                device = v.device
            elif v.device != device:
                _refuse("a gradient's tensors must be on one device")
        shape = t.shape
        if o is not t and (o.shape != shape or o.dtype != t.dtype):
            _refuse(f"a tensor of shape {tuple(shape)} and type {t.dtype} has an output of shape {tuple(o.shape)} and type {o.dtype}")
        numel = t.numel()
        if per_worker:
            if not shape:
                _refuse("a worker's tensors have a first dimension of workers")
            if workers is None:
                workers = shape[0]
            elif shape[0] != workers:
                _refuse(f"tensors of {workers} and of {shape[0]} workers")
            strides, out_strides = t.stride(), o.stride()
            ws, out_ws = (strides[0], out_strides[0]) if workers > 1 else (0, 0)
            shape, strides, out_strides = shape[1:], strides[1:], out_strides[1:]
            numel = numel // workers if workers else 0
        elif t.is_contiguous() and (o is t or o.is_contiguous()):
            words += (t.data_ptr(), o.data_ptr(), 0, 0, 1, numel, numel, numel, _DTYPES[t.dtype])
            continue
        else:
            ws = out_ws = 0
            strides, out_strides = t.stride(), o.stride()
        rows, cols, pitch, out_pitch = _rows_of("a gradient's tensor", shape, strides, out_strides) if numel else (0, 0, 0, 0)
        words += (t.data_ptr(), o.data_ptr(), ws, out_ws, rows, cols, pitch, out_pitch, _DTYPES[t.dtype])
    return tensors, out, array.array("q", words), workers if per_worker else 1, device


def _clip(tensors, max_norm, zero_nonfinite, per_worker, out, stream):
    if stream is None:
        done = _usual().clip(tensors, out, bool(per_worker), max_norm, bool(zero_nonfinite))
        if done is not None:
            return done
    tensors, out, words, workers, device = _gradients(tensors, per_worker, out)
    queue = _Queue(device, stream, *tensors, *out)
    with queue as s:
        norms = torch.empty((workers,) if per_worker else (), dtype=torch.float32, device=device)
        queue.made.append(norms)
        ws, ws_p, size = _workspace(norms, "a2cid2_clip_gradients_workspace", len(tensors), workers)
        table = words.buffer_info()[0]
        if max_norm is None:
            B._check(B.lib().a2cid2_gradient_norms(table, len(tensors), workers, norms.data_ptr(), ws_p, size, s))
        else:
            B._check(B.lib().a2cid2_clip_gradients(table, len(tensors), workers, max_norm, int(bool(zero_nonfinite)), norms.data_ptr(), ws_p, size, s))
    return norms


def gradient_norms(tensors, per_worker=False, stream=None):
    """The 2-norm of all elements of a list of tensors (float32 or bfloat16, also mixed), a float32 scalar on their device. With per_worker all have the workers as their first
    dimension (e.g. parts of the engine's rows, `eng.g[:, off:off + r * c].view(-1, r, c)`) and a norm is that of a worker: float32 [workers]."""
    return _clip(tensors, None, False, per_worker, None, stream)


def clip_gradients(tensors, max_norm, per_worker=False, zero_nonfinite=False, out=None, stream=None):
    """Multiplies the tensors by min(1, max_norm / norm), in place or into the list `out` of tensors of the same shapes and types, and returns the norms before that
    (as `gradient_norms`). Tensors whose norm is not finite are left as they are, or with zero_nonfinite become zeros."""
    if max_norm is None:
        _refuse("max_norm must be a number")
    return _clip(tensors, max_norm, zero_nonfinite, per_worker, out, stream)


def check(stream=None):
    """Waits for the stream (torch's current one if None) and raises `binding.A2Error` if a kernel of the products gave up a wait on its device
    since this was last raised. Until then every operator on that device raises it too."""
    stream = torch.cuda.current_stream() if stream is None else stream
    with torch.cuda.device(stream.device):
        B._check(B.lib().a2cid2_operators_check(stream.cuda_stream))
