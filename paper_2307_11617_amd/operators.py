"""The operators that take tensors instead of a context (include/rfast.h, same names): low-rank adapters beside a shared
projection, softmax cross-entropy with its gradient, and AdamW over many tensors.

Every call runs on the current stream of its tensors' device and neither waits nor reads anything back, so that it can be captured
into a graph.  Workspaces come from torch's allocator with each call: calls on different streams, and graphs, share none.
What the library cannot see (extents, types, devices of tensors) is checked here, before any launch.
None takes part in torch's autograd: inputs that require gradients are read as they are and results require none; gradients are the backward
calls' own results."""
from __future__ import annotations

import ctypes as C

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
