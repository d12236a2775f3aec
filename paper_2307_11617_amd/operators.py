"""The operators that take tensors instead of a context (include/rfast.h, same names): low-rank adapters beside a shared
projection, rows sent to experts and back, token embeddings, softmax cross-entropy and the clipped policy loss with their gradients, and AdamW over many tensors.

Every call runs on the current stream of its tensors' device and neither waits nor reads anything back, so that it can be captured
into a graph.  Workspaces come from torch's allocator with each call: calls on different streams, and graphs, share none.
What the library cannot see (extents, types, devices of tensors) is checked here, before any launch.
None takes part in torch's autograd: inputs that require gradients are read as they are and results require none; gradients are the backward
calls' own results."""
from __future__ import annotations

import ctypes as C
from typing import Any, NamedTuple

import numpy as np

from .binding import RFastError, RfastAdamwOptions, RfastAdamwTensor, RfastLoraShape, lib, rfast_last_error

F32, BF16 = 0, 1
_torch = _types = _stream_of = None


def _t():
    global _torch, _types, _stream_of
    if _torch is None:
        import torch
        _torch, _types = torch, {torch.float32: F32, torch.bfloat16: BF16}
        # (the handle alone, where torch offers it: a Stream object costs a microsecond more than the call it is made for)
        _stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _torch


def _need(ok, msg):
    if not ok:
        raise RFastError(-1, msg)


def _sizes(*counts):
    """Counts go to the library in 32 bits, which ctypes would cut to."""
    if max(counts) > 0x7FFFFFFF:
        raise RFastError(-1, f"sizes out of range: {max(counts)}")


def _counters(steps):
    if not all(0 <= s <= 0x7FFFFFFF for s in steps):  # (before anything cuts them to their type)
        raise RFastError(-4, "steps out of range")


def _type(t, name):
    k = _types.get(t.dtype)
    if k is None:
        raise RFastError(-1, f"{name}: need float32 or bfloat16, got {t.dtype}")
    return k


def _call(device, f, *args):
    """f on the current stream of `device` (its last argument), with that device current."""
    index = device.index
    if index == _torch.cuda.current_device():
        code = f(*args, _stream_of(index))
    else:
        with _torch.cuda.device(index):
            code = f(*args, _stream_of(index))
    if code != 0:
        raise RFastError(code, rfast_last_error(None))


def _matrix(t, name, rows, cols, dtype, device):
    """Distance of the rows of a [rows][cols] tensor whose columns are neighbours."""
    if t.shape != (rows, cols) or t.device != device or (dtype is not None and t.dtype != dtype):
        raise RFastError(-1, f"{name}: need a tensor of shape ({rows}, {cols}) and type {dtype or t.dtype} on {device}, "
                             f"got {tuple(t.shape)}, {t.dtype} on {t.device}")
    if t.is_contiguous():
        return cols if cols > 0 else 1
    if cols > 1 and t.stride(1) != 1:
        raise RFastError(-1, f"{name}: the elements of a row must be neighbours")
    return t.stride(0) if rows > 1 else max(cols, 1)


def _new(device, dtype, rows, cols=None):
    """An uninitialised tensor (with strides given torch is a third faster than without: 1.3 us)."""
    if cols is None:
        return _torch.empty_strided((rows,), (1,), dtype=dtype, device=device)
    return _torch.empty_strided((rows, cols), (cols or 1, 1), dtype=dtype, device=device)


def _vector(t, name, count, dtype, device):
    if t.dtype != dtype or t.device != device or t.numel() != count or not t.is_contiguous():
        raise RFastError(-1, f"{name}: need a contiguous {dtype} tensor of {count} elements on {device}")
    return t.data_ptr()


def rfast_softmax_xent(logits, labels, grad_scale=1.0, grad_dtype=None, grad=None, loss=None, lse=None, rows=None):
    """(loss, grad) of rows of logits [T][K] (float32 or bfloat16) with labels int32 [T] (outside [0, K): padding): loss float32 [T],
    grad = grad_scale (softmax - onehot) in grad_dtype (default: the logits').  grad: tensor to write to, `logits` itself for its place, or False for no gradient.
    lse: float32 [T] to receive log sum exp.  rows: int32 [1] on the device; only that many rows are taken, the others of the
    outputs are not written."""
    torch = _t()
    if logits.dim() != 2 or not logits.is_cuda or logits.shape[1] < 1:
        raise RFastError(-1, "logits: need a matrix on the GPU with at least one class")
    T, K = logits.shape
    _sizes(T, K)
    dev = logits.device
    ld, lt = _matrix(logits, "logits", T, K, None, dev), _type(logits, "logits")
    p_labels = _vector(labels, "labels", T, torch.int32, dev)
    if loss is None:
        loss = torch.empty(T, dtype=torch.float32, device=dev)
        p_loss = loss.data_ptr()
    else:
        p_loss = _vector(loss, "loss", T, torch.float32, dev)
    p_lse = None if lse is None else _vector(lse, "lse", T, torch.float32, dev)
    if grad is None:
        grad = torch.empty((T, K), dtype=grad_dtype or logits.dtype, device=dev)
        ldg, gt, p_grad = K, _type(grad, "grad"), grad.data_ptr()
    elif grad is False:
        grad, p_grad, gt, ldg = None, None, F32, 0
    else:
        _need(grad_dtype is None or grad.dtype == grad_dtype, "grad: its type is not grad_dtype")
        ldg, gt, p_grad = _matrix(grad, "grad", T, K, None, dev), _type(grad, "grad"), grad.data_ptr()
    p_rows = None if rows is None else _vector(rows, "rows", 1, torch.int32, dev)
    _call(dev, lib().rfast_softmax_xent, T, K, logits.data_ptr(), lt, ld, p_labels, grad_scale, p_loss, p_lse, p_grad, gt, ldg, p_rows)
    return loss, grad


def rfast_policy_loss(logits, actions, old_logp, advantage, reference=None, weight=None, clip=(0.2, 0.2), beta=0.0, grad_scale=1.0,
                      grad_dtype=None, grad=None, loss=None, logp=None, rows=None):
    """(loss, grad) of the clipped policy loss of rows of logits [T][K] (float32 or bfloat16): actions int32 [T] (outside [0, K): padding);
    old_logp, advantage and, where given, reference and weight float32 [T].  With r = exp(logp - old_logp) a row's loss is
    weight (-min(r advantage, clip(r, 1 - clip[0], 1 + clip[1]) advantage) + beta (exp(q) - q - 1)), q = reference - logp (no second term without
    one), grad its derivative by the logits times grad_scale.  grad_dtype, grad, loss, rows: as in rfast_softmax_xent.  logp: float32 [T] to receive
    log probabilities of the actions."""
    torch = _t()
    f32 = torch.float32
    if logits.dim() != 2 or not logits.is_cuda or logits.shape[1] < 1:
        raise RFastError(-1, "logits: need a matrix on the GPU with at least one class")
    T, K = logits.shape
    _sizes(T, K)
    dev = logits.device
    ld, lt = _matrix(logits, "logits", T, K, None, dev), _type(logits, "logits")
    given = (_vector(actions, "actions", T, torch.int32, dev), _vector(old_logp, "old_logp", T, f32, dev), _vector(advantage, "advantage", T, f32, dev),
             None if reference is None else _vector(reference, "reference", T, f32, dev),
             None if weight is None else _vector(weight, "weight", T, f32, dev))
    loss = _new(dev, f32, T) if loss is None else loss
    p_loss = _vector(loss, "loss", T, f32, dev)
    p_logp = None if logp is None else _vector(logp, "logp", T, f32, dev)
    if grad is None:
        grad = _new(dev, grad_dtype or logits.dtype, T, K)
        ldg, gt, p_grad = K, _type(grad, "grad"), grad.data_ptr()
    elif grad is False:
        grad, p_grad, gt, ldg = None, None, F32, 0
    else:
        _need(grad_dtype is None or grad.dtype == grad_dtype, "grad: its type is not grad_dtype")
        ldg, gt, p_grad = _matrix(grad, "grad", T, K, None, dev), _type(grad, "grad"), grad.data_ptr()
    p_rows = None if rows is None else _vector(rows, "rows", 1, torch.int32, dev)
    _call(dev, lib().rfast_policy_loss, T, K, logits.data_ptr(), lt, ld, *given, clip[0], clip[1], beta, grad_scale, p_loss, p_logp, p_grad, gt, ldg,
          p_rows)
    return loss, grad


# ------------------------------------------------------------------------------------------------------- embeddings
def rfast_embedding(table, tokens, scale=1.0, out=None, out_dtype=None):
    """Rows scale table[token] of a table [V][d] (float32 or bfloat16), tokens int32 [T] (outside [0, V): padding, a row of zeros), in out_dtype
    (default: the table's)."""
    torch = _t()
    _need(table.dim() == 2 and table.is_cuda, "table: need a matrix on the GPU")
    (V, d), T, dev = table.shape, tokens.numel(), table.device
    _sizes(T, V, d)
    ld = _matrix(table, "table", V, d, None, dev)
    if out is None:
        out, ld_out = _new(dev, out_dtype or table.dtype, T, d), max(d, 1)
    else:
        _need(out_dtype is None or out.dtype == out_dtype, "out: its type is not out_dtype")
        ld_out = _matrix(out, "out", T, d, None, dev)
    _call(dev, lib().rfast_embedding, T, V, d, table.data_ptr(), _type(table, "table"), ld, _vector(tokens, "tokens", T, torch.int32, dev), scale,
          out.data_ptr(), _type(out, "out"), ld_out)
    return out


def rfast_embedding_backward_workspace_bytes(rows, vocabulary, d):
    _sizes(rows, vocabulary, d)
    return int(lib().rfast_embedding_backward_workspace_bytes(rows, vocabulary, d))


def rfast_embedding_backward(dy, tokens, vocabulary, scale=1.0, grad=None, grad_dtype=None, accumulate=False):
    """Gradient [vocabulary][d] of rfast_embedding's table for dy [T][d] (float32 or bfloat16), in grad_dtype (default float32): every row is
    written, zeros where no token is.  accumulate: added to what `grad` holds, rows without a token stay as they are."""
    torch = _t()
    _need(dy.dim() == 2 and dy.is_cuda, "dy: need a matrix on the GPU")
    (T, d), dev, V = dy.shape, dy.device, int(vocabulary)
    _sizes(T, V, d)
    ld = _matrix(dy, "dy", T, d, None, dev)
    p_tokens = _vector(tokens, "tokens", T, torch.int32, dev)
    if grad is None:
        _need(not accumulate, "accumulate: need the gradient to add to")
        _need(V >= 1, "need a vocabulary of at least one")
        grad, ld_grad = _new(dev, grad_dtype or torch.float32, V, d), max(d, 1)
    else:
        _need(grad_dtype is None or grad.dtype == grad_dtype, "grad: its type is not grad_dtype")
        ld_grad = _matrix(grad, "grad", V, d, None, dev)
    nbytes = rfast_embedding_backward_workspace_bytes(T, V, d)
    ws = _new(dev, torch.uint8, nbytes)
    _call(dev, lib().rfast_embedding_backward, T, V, d, dy.data_ptr(), _type(dy, "dy"), ld, p_tokens, scale, grad.data_ptr(), _type(grad, "grad"),
          ld_grad, 1 if accumulate else 0, ws.data_ptr(), nbytes)
    return grad


# ---------------------------------------------------------------------------------------- rows to experts and back
class RFastRoute(NamedTuple):
    """What a router decided for T rows: expert int32 [T][k] and weight float32 [T][k]; the pairs (row, choice) sorted by expert: row_ptr int32
    [experts + 1], place int32 [T][k] (where a pair is, -1: nowhere) and order int32 [T k] (which pair is there)."""
    expert: Any
    weight: Any
    row_ptr: Any
    place: Any
    order: Any


def rfast_route_workspace_bytes(pairs, experts):
    _sizes(pairs, experts)
    return int(lib().rfast_route_workspace_bytes(pairs, experts))


def rfast_route(logits, k, normalise=True):
    """The k experts of every row of logits [T][experts] (float32 or bfloat16; at most 1024 experts, k at most 64) with the largest logits (of equal
    ones the lowest; masked ones, -infinity, never: expert -1, weight 0), their weights (exp(logit) over the sum of the chosen, or of all if
    normalise is false), and the order of the pairs by expert."""
    torch = _t()
    _need(logits.dim() == 2 and logits.is_cuda, "logits: need a matrix on the GPU")
    (T, E), dev, k = logits.shape, logits.device, int(k)
    _need(1 <= k <= min(E, 64) and E <= 1024, "need 1 to 1024 experts and k from 1 to min(experts, 64)")
    _sizes(T * k)
    ld, lt = _matrix(logits, "logits", T, E, None, dev), _type(logits, "logits")
    i32 = torch.int32
    r = RFastRoute(_new(dev, i32, T, k), _new(dev, torch.float32, T, k), _new(dev, i32, E + 1), _new(dev, i32, T, k), _new(dev, i32, T * k))
    nbytes = rfast_route_workspace_bytes(T * k, E)
    ws = _new(dev, torch.uint8, nbytes)
    _call(dev, lib().rfast_route, T, E, k, logits.data_ptr(), lt, ld, 1 if normalise else 0, *[t.data_ptr() for t in r], ws.data_ptr(), nbytes)
    return r


def rfast_route_plan(expert, experts):
    """(row_ptr, place, order) of experts (or adapters) chosen elsewhere: expert int32 of any shape, numbers outside [0, experts) go nowhere; place has
    its shape."""
    torch = _t()
    P, dev, i32 = expert.numel(), expert.device, torch.int32
    _need(expert.is_cuda, "expert: need a tensor on the GPU")
    _sizes(P, experts)
    _need(experts >= 1, "need at least one expert")
    p_expert = _vector(expert, "expert", P, i32, dev)
    row_ptr, place, order = _new(dev, i32, experts + 1), torch.empty(expert.shape, dtype=i32, device=dev), _new(dev, i32, P)
    nbytes = rfast_route_workspace_bytes(P, experts)
    ws = _new(dev, torch.uint8, nbytes)
    _call(dev, lib().rfast_route_plan, P, experts, p_expert, row_ptr.data_ptr(), place.data_ptr(), order.data_ptr(), ws.data_ptr(), nbytes)
    return row_ptr, place, order


def rfast_route_backward(logits, expert, weight, dweight, normalise=True, dlogits=None, grad_dtype=None):
    """Gradient [T][experts] of rfast_route's logits for dweight float32 [T][k]; expert and weight as it returned them; in grad_dtype (default: the
    logits')."""
    torch = _t()
    _need(logits.dim() == 2 and logits.is_cuda and expert.dim() == 2, "need logits [rows][experts] on the GPU and expert [rows][k]")
    (T, E), dev, k = logits.shape, logits.device, expert.shape[1]
    _sizes(T, E, k)
    ld, lt = _matrix(logits, "logits", T, E, None, dev), _type(logits, "logits")
    given = (_vector(expert, "expert", T * k, torch.int32, dev), _vector(weight, "weight", T * k, torch.float32, dev),
             _vector(dweight, "dweight", T * k, torch.float32, dev))
    if dlogits is None:
        dlogits, ld_out = _new(dev, grad_dtype or logits.dtype, T, E), max(E, 1)
    else:
        _need(grad_dtype is None or dlogits.dtype == grad_dtype, "dlogits: its type is not grad_dtype")
        ld_out = _matrix(dlogits, "dlogits", T, E, None, dev)
    _call(dev, lib().rfast_route_backward, T, E, k, logits.data_ptr(), lt, ld, 1 if normalise else 0, *given, dlogits.data_ptr(),
          _type(dlogits, "dlogits"), ld_out)
    return dlogits


def _pairs(place, dev):
    _need(place.dim() == 2, "place: need a matrix [rows][k]")
    T, k = place.shape
    _sizes(T * k)
    return T, k, _vector(place, "place", T * k, _torch.int32, dev)


def rfast_route_gather(x, place, out=None):
    """Rows sorted by expert, [T k][d]: row place[t][j] is x[t] (x [T][d], float32 or bfloat16).  Rows that are nobody's place are not written: they
    stay as they are in `out` (whose rows may be any number; a place outside is none), and hold anything without one.  Its gradient is
    rfast_route_combine(dout, place)."""
    torch = _t()
    _need(x.dim() == 2 and x.is_cuda, "x: need a matrix on the GPU")
    (T, d), dev = x.shape, x.device
    ld = _matrix(x, "x", T, d, None, dev)
    rows, k, p_place = _pairs(place, dev)
    _need(rows == T, "place: need one row per row of x")
    if out is None:
        out = _new(dev, x.dtype, T * k, d)
    _need(out.dim() == 2, "out: need a matrix")
    P = out.shape[0]
    _sizes(P, d)
    ld_out = _matrix(out, "out", P, d, x.dtype, dev)
    _call(dev, lib().rfast_route_gather, T, k, d, x.data_ptr(), _type(x, "x"), ld, p_place, out.data_ptr(), P, ld_out)
    return out


def rfast_route_combine(rows, place, weight=None, out=None, out_dtype=None):
    """y [T][d], y[t] = sum over j of weight[t][j] rows[place[t][j]], of rows sorted by expert [P][d] (float32 or bfloat16); weight float32 [T][k] (None: 1); a
    place outside [0, P) counts for nothing.  In out_dtype (default: the rows')."""
    torch = _t()
    _need(rows.dim() == 2 and rows.is_cuda, "rows: need a matrix on the GPU")
    (P, d), dev = rows.shape, rows.device
    _sizes(P, d)
    ld = _matrix(rows, "rows", P, d, None, dev)
    T, k, p_place = _pairs(place, dev)
    p_weight = None if weight is None else _vector(weight, "weight", T * k, torch.float32, dev)
    if out is None:
        out, ld_out = _new(dev, out_dtype or rows.dtype, T, d), max(d, 1)
    else:
        _need(out_dtype is None or out.dtype == out_dtype, "out: its type is not out_dtype")
        ld_out = _matrix(out, "out", T, d, None, dev)
    _call(dev, lib().rfast_route_combine, T, k, d, rows.data_ptr(), _type(rows, "rows"), P, ld, p_place, p_weight, out.data_ptr(), _type(out, "out"),
          ld_out)
    return out


def rfast_route_combine_backward(rows, place, weight, dy, drows=None, dweight=None):
    """(drows, dweight) of rfast_route_combine for dy [T][d] of the rows' type: drows [P][d] of that type (rows that are nobody's place are not written:
    they stay as they are in `drows`, and hold anything without one), dweight float32 [T][k].  Either may be False: not wanted."""
    torch = _t()
    _need(rows.dim() == 2 and rows.is_cuda, "rows: need a matrix on the GPU")
    (P, d), dev = rows.shape, rows.device
    _sizes(P, d)
    ld = _matrix(rows, "rows", P, d, None, dev)
    T, k, p_place = _pairs(place, dev)
    p_weight = None if weight is None else _vector(weight, "weight", T * k, torch.float32, dev)
    ld_dy = _matrix(dy, "dy", T, d, rows.dtype, dev)
    ld_out = d
    if drows is None:
        drows = _new(dev, rows.dtype, P, d)
    elif drows is not False:
        ld_out = _matrix(drows, "drows", P, d, rows.dtype, dev)
    if dweight is None:
        dweight = _new(dev, torch.float32, T, k)
    p_dweight = None if dweight is False else _vector(dweight, "dweight", T * k, torch.float32, dev)
    _call(dev, lib().rfast_route_combine_backward, T, k, d, rows.data_ptr(), _type(rows, "rows"), P, ld, p_place, p_weight, dy.data_ptr(), ld_dy,
          None if drows is False else drows.data_ptr(), ld_out, p_dweight)
    return (None if drows is False else drows), (None if dweight is False else dweight)


def rfast_lora_workspace_bytes(shape, which):
    """which: 0 forward, 1 backward without dx, 2 backward with dx."""
    return int(lib().rfast_lora_workspace_bytes(C.byref(shape), which))


_shapes = {}


def _lora_shape(*sizes):
    """(RfastLoraShape by reference, its workspaces in bytes) of these sizes."""
    got = _shapes.get(sizes)
    if got is None:
        if len(_shapes) >= 4096:
            _shapes.clear()
        _sizes(*sizes[:6])
        shape = RfastLoraShape(*sizes)
        got = _shapes[sizes] = (C.byref(shape), tuple(int(lib().rfast_lora_workspace_bytes(C.byref(shape), k)) for k in range(3)))
    return got


def _lora(x, w, a, b, row_ptr, adapter, y_type, ld_y, scale, which):
    torch = _torch
    bf16, dev = torch.bfloat16, x.device
    if x.dim() != 2 or not x.is_cuda or w.dim() != 2 or a.dim() != 3:
        raise RFastError(-1, "need x [rows][d] on the GPU, w [K][d], a [adapters][rank][d], b [adapters][K][rank]")
    T, d = x.shape
    K, (n, r, _) = w.shape[0], a.shape
    for t, name, want in ((w, "w", (K, d)), (a, "a", (n, r, d)), (b, "b", (n, K, r))):
        if t.shape != want or t.dtype != bf16 or t.device != dev or not t.is_contiguous():
            raise RFastError(-1, f"{name}: need a contiguous bfloat16 tensor of shape {want} on {dev}, got {t.dtype}, {tuple(t.shape)} on {t.device}")
    ld_x = _matrix(x, "x", T, d, bf16, dev)
    S = row_ptr.numel() - 1
    p_ptr = _vector(row_ptr, "row_ptr", S + 1, torch.int32, dev)
    p_ad = None if adapter is None else _vector(adapter, "adapter", S, torch.int32, dev)
    shape, nbytes = _lora_shape(T, S, n, d, K, r, ld_x, ld_y, y_type, scale)
    nbytes = nbytes[which]
    if nbytes == 0 and T > 0:
        raise RFastError(-1, "sizes out of range (at least one segment; rank 1 .. 64)")
    ws = torch.empty(nbytes or 256, dtype=torch.uint8, device=dev)
    return dev, ld_x, (shape, x.data_ptr(), w.data_ptr(), a.data_ptr(), b.data_ptr(), p_ptr, p_ad), (ws.data_ptr(), nbytes or 256), ws


def rfast_lora_forward(x, w, a, b, row_ptr, adapter=None, scale=1.0, out=None, out_dtype=None):
    """y_t = w x_t + scale b_a a_a x_t for the rows of every segment: x bfloat16 [T][d], w [K][d], a [adapters][rank][d], b
    [adapters][K][rank], row_ptr int32 [segments + 1], adapter int32 [segments] (None: segment s has adapter s; a number outside
    [0, adapters): no adapter).  Returns y [T][K] in out_dtype (default bfloat16); rows behind the last segment are not
    written: they stay as they are in `out`, and hold anything without one."""
    torch = _t()
    _need(x.dim() == 2 and w.dim() == 2, "need matrices x [rows][d] and w [K][d]")
    T, K = x.shape[0], w.shape[0]
    if out is None:
        out, ld_y = torch.empty((T, K), dtype=out_dtype or torch.bfloat16, device=x.device), max(K, 1)
    else:
        _need(out_dtype is None or out.dtype == out_dtype, "out: its type is not out_dtype")
        ld_y = _matrix(out, "out", T, K, None, x.device)
    dev, _, given, work, _keep = _lora(x, w, a, b, row_ptr, adapter, _type(out, "out"), ld_y, scale, 0)
    _call(dev, lib().rfast_lora_forward, *given, out.data_ptr(), *work)
    return out


def rfast_lora_backward(x, w, a, b, row_ptr, adapter, dy, scale=1.0, need_dx=True, dx=None, da=None, db=None):
    """(dx, da, db) of rfast_lora_forward for dy bfloat16 [T][K], w frozen: dx bfloat16 [T][d] (None unless need_dx or a tensor to write to
    is given, its rows as far apart as x's; rows behind the last segment are not written), da float32 [adapters][rank][d], db
    float32 [adapters][K][rank]."""
    torch = _t()
    _need(x.dim() == 2 and w.dim() == 2, "need matrices x [rows][d] and w [K][d]")
    T, d = x.shape
    ld_y = _matrix(dy, "dy", T, w.shape[0], torch.bfloat16, x.device)
    with_dx = need_dx or dx is not None
    dev, ld_x, given, work, _keep = _lora(x, w, a, b, row_ptr, adapter, BF16, ld_y, scale, 2 if with_dx else 1)
    if dx is not None:
        _need(_matrix(dx, "dx", T, d, torch.bfloat16, dev) == ld_x or T <= 1, "dx: its rows must be as far apart as x's")
    elif with_dx:
        dx = torch.empty_strided((T, d), (ld_x, 1), dtype=torch.bfloat16, device=dev)
    da = torch.empty(a.shape, dtype=torch.float32, device=dev) if da is None else da
    db = torch.empty(b.shape, dtype=torch.float32, device=dev) if db is None else db
    _call(dev, lib().rfast_lora_backward, *given, dy.data_ptr(), None if dx is None else dx.data_ptr(),
          _vector(da, "da", a.numel(), torch.float32, dev), _vector(db, "db", b.numel(), torch.float32, dev), *work)
    return dx, da, db


# ------------------------------------------------------------------------------------------------------------- AdamW
def rfast_adamw_workspace_bytes(tensors):
    """tensors: a ctypes array of RfastAdamwTensor."""
    return int(lib().rfast_adamw_workspace_bytes(len(tensors), tensors))


def rfast_adamw_create(tensors, options, workspace):
    _t()
    h = C.c_void_p()
    _call(workspace.device, lambda stream: lib().rfast_adamw_create(C.byref(h), len(tensors), tensors, C.byref(options),
                                                                    workspace.data_ptr(), workspace.numel(), stream))
    return h


def rfast_adamw_step(h, gamma, active, device):
    """active: uint8 device tensor, one flag per tensor, or None."""
    _call(device, lib().rfast_adamw_step, h, gamma, None if active is None else active.data_ptr())


def rfast_adamw_steps(h, out, device):
    """out: int32 host array, one number per tensor."""
    _call(device, lib().rfast_adamw_steps, h, out.ctypes.data_as(C.c_void_p))
    return out


def rfast_adamw_set_steps(h, steps, device):
    _call(device, lib().rfast_adamw_set_steps, h, steps.ctypes.data_as(C.c_void_p))


def rfast_adamw_destroy(h):
    lib().rfast_adamw_destroy(h)


class RFastAdamW:
    """AdamW over a list of tensors with one launch per step; moments in 32 or 8 bits.

    params, grads: contiguous float32 or bfloat16 tensors of one device, the same tensors at every step (gradients are read where they
    were given).  m, v: the moments, made as zeros where not given (state_bits 32: float32; 8: uint8 or float8_e4m3fn codes of m and
    sqrt(v), with m_scale and v_scale float32 [ceil(count / 256)]).  weight_decay: one number or one per tensor.  copies: bfloat16 tensors (or None each) that receive the
    new parameters rounded.  steps: taken before, one number or one per tensor.
    A graph that holds steps needs the object for as long as it is replayed."""

    def __init__(self, params, grads, m=None, v=None, m_scale=None, v_scale=None, state_bits=32, betas=(0.9, 0.999), eps=1e-8,
                 weight_decay=0.0, copies=None, steps=0):
        torch = _t()
        self.handle = None
        params, grads = list(params), list(grads)
        n = len(params)
        _need(n >= 1, "need at least one tensor")
        _need(state_bits in (8, 32), "state_bits must be 8 or 32")
        self.device = params[0].device
        _need(params[0].is_cuda, "params: need tensors on the GPU")

        made = []  # memory of this object's own

        def listed(value, name, make):
            if value is None:
                value = [make(p) for p in params]
                made.extend(value)
            value = list(value)
            _need(len(value) == n, f"{name}: need one per parameter")
            return value

        def numbers(value, name):
            return listed([value] * n if isinstance(value, (int, float)) else value, name, None)

        grads = listed(grads, "grads", None)
        state = torch.float32 if state_bits == 32 else torch.uint8
        self.params, self.grads = params, grads
        self.m = listed(m, "m", lambda p: torch.zeros(p.numel(), dtype=state, device=self.device))
        self.v = listed(v, "v", lambda p: torch.zeros(p.numel(), dtype=state, device=self.device))
        if state_bits == 8:
            def scales(p):
                return torch.zeros((p.numel() + 255) // 256, dtype=torch.float32, device=self.device)
            self.m_scale, self.v_scale = listed(m_scale, "m_scale", scales), listed(v_scale, "v_scale", scales)
        else:
            _need(m_scale is None and v_scale is None, "scales belong to states in 8 bits")
            self.m_scale = self.v_scale = [None] * n
        self.copies = [None] * n if copies is None else listed(copies, "copies", None)
        decay, steps = numbers(weight_decay, "weight_decay"), numbers(steps, "steps")
        _counters(steps)
        tensors = (RfastAdamwTensor * n)()
        pt, gt = _type(params[0], "params"), _type(grads[0], "grads")
        states = (torch.float32,) if state_bits == 32 else (torch.uint8, torch.float8_e4m3fn)
        for i, (p, g) in enumerate(zip(params, grads)):
            c = p.numel()
            _need(self.m[i].dtype in states and self.v[i].dtype in states, f"tensor {i}: need moments of type {states[0]}")
            tensors[i] = RfastAdamwTensor(
                _vector(p, f"params[{i}]", c, params[0].dtype, self.device), _vector(g, f"grads[{i}]", c, grads[0].dtype, self.device),
                _vector(self.m[i], f"m[{i}]", c, self.m[i].dtype, self.device), _vector(self.v[i], f"v[{i}]", c, self.v[i].dtype, self.device),
                None if state_bits == 32 else _vector(self.m_scale[i], f"m_scale[{i}]", (c + 255) // 256, torch.float32, self.device),
                None if state_bits == 32 else _vector(self.v_scale[i], f"v_scale[{i}]", (c + 255) // 256, torch.float32, self.device),
                None if self.copies[i] is None else _vector(self.copies[i], f"copies[{i}]", c, torch.bfloat16, self.device),
                c, decay[i], steps[i])
        nbytes = rfast_adamw_workspace_bytes(tensors)
        _need(nbytes > 0, "sizes out of range")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self._made = made + [self.workspace]
        self._streams = {torch.cuda.current_stream(self.device).cuda_stream}  # those that the allocator knows to use that memory
        self.handle = rfast_adamw_create(tensors, RfastAdamwOptions(pt, gt, state_bits, betas[0], betas[1], eps), self.workspace)

    def step(self, gamma, active=None):
        """One step with step size gamma; active: uint8 [tensors] on the device, zero for tensors that stay as they are."""
        if active is not None:
            _vector(active, "active", len(self.params), _torch.uint8, self.device)
        if _stream_of(self.device.index) not in self._streams:  # the allocator has to know, or it hands the memory on too early
            stream = _torch.cuda.current_stream(self.device)
            for t in self._made:
                t.record_stream(stream)
            self._streams.add(stream.cuda_stream)
        rfast_adamw_step(self.handle, gamma, active, self.device)

    def steps(self):
        return rfast_adamw_steps(self.handle, np.empty(len(self.params), dtype=np.int32), self.device)

    def set_steps(self, steps):
        steps = np.asarray(steps)
        _need(steps.shape == (len(self.params),), "need one number per tensor")
        _counters(steps)
        steps = np.ascontiguousarray(steps, dtype=np.int32)
        rfast_adamw_set_steps(self.handle, steps, self.device)

    def close(self):
        if self.handle is not None:
            rfast_adamw_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
