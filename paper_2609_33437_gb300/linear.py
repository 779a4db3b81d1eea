"""Linear layers for the model whose parameters the library simulates: the products of a layer with what
surrounds them, and activations saved in 8 bits for the backward pass (include/smat.h, "linear layers").

    y         = linear(x, w, bias, act, residual)            y = act(x W^T + b) + residual
    y, saved  = linear(..., save=True)                       and h = x W^T + b in 8 bits
    dx        = linear_grad_input(dy, w, act, saved)         dx = (dy W) * act'(h^)
    dw, db    = linear_grad_weight(dy, x, act, bias=True)    dW = dy^T x^, db = sums of dy over rows
    p         = pack8(x); unpack8(p, act); act_grad8(dy, p, act)

`Linear8` is a torch.nn.Linear with an activation and a residual whose backward pass reads 8-bit activations,
`Mlp8` the two-layer MLP that saves its input and its pre-activation, one byte per element each, and nothing else.

Tensors are CUDA tensors of one dtype per call (float32 or bfloat16); activations may have any number of leading
dimensions and a row stride (the last dimension is contiguous). Argument marshalling only: every operator runs in
the library's kernels, on the current stream or the one given. The operators build no autograd graph and refuse tensors
whose gradient or tangent that would lose: call them under torch.no_grad(), in a torch.autograd.Function, or on detached
tensors; the layers are differentiable.
"""

import ctypes
import struct
from typing import Optional, Tuple, Union

import torch
import torch.autograd.forward_ad as forward_ad

from . import smat as S

GROUP = 32
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "quick_gelu": 4, "silu": 5}

_LINEAR = struct.Struct("@7P9q2i")
_GRAD_INPUT = struct.Struct("@5P8q2i")
_GRAD_WEIGHT = struct.Struct("@6P8q4i")


class Packed8:
    """A tensor in 8 bits: q int8 of the tensor's shape, e uint8 with ceil(columns / 32) in place of the columns;
    it stands for q * 2^(e - 127), e by groups of 32 columns. Packed8(q, e) takes tensors that hold these; what the
    operators make is one buffer, q's rows and then e's, of which q and e are views."""
    __slots__ = ("_q", "_e", "_buffer", "_at", "shape", "device")

    def __init__(self, q: torch.Tensor, e: torch.Tensor):
        if q.dtype is not torch.int8 or e.dtype is not torch.uint8 or q.dim() < 1 or e.dim() != q.dim():
            raise ValueError("q must be int8 and e uint8, with the same leading dimensions")
        if e.shape[:-1] != q.shape[:-1] or e.shape[-1] != -(-q.shape[-1] // GROUP):
            raise ValueError(f"e must be shaped {(*q.shape[:-1], -(-q.shape[-1] // GROUP))}")
        self._q, self._e, self._buffer = q, e, None
        self.shape, self.device = q.shape, q.device

    @classmethod
    def _make(cls, shape, rows: int, cols: int, device) -> "Packed8":
        """An empty one for the operators to fill (rows: the leading dimensions' product)."""
        p = object.__new__(cls)
        p._q = p._e = None
        p._at = -(-rows * cols // 256) * 256  # of e in the buffer
        p._buffer = torch.empty(p._at + rows * -(-cols // GROUP), dtype=torch.uint8, device=device)
        p.shape, p.device = torch.Size(shape), device
        return p

    @property
    def q(self) -> torch.Tensor:
        if self._q is None:
            self._q = self._buffer[:self.shape.numel()].view(torch.int8).view(self.shape)
        return self._q

    @property
    def e(self) -> torch.Tensor:
        if self._e is None:
            self._e = self._buffer[self._at:].view(*self.shape[:-1], -(-self.shape[-1] // GROUP))
        return self._e

    def nbytes(self) -> int:
        rows = self.shape[:-1].numel()
        return rows * (self.shape[-1] - (-self.shape[-1] // GROUP))

    def _places(self, name: str, device, rows: int, cols: int):
        """(address and row stride of q, and of e); what does not fit [rows, cols] on `device` is refused."""
        if self._buffer is not None:
            shape = self.shape
            if shape[-1] == cols and shape[:-1].numel() == rows and self.device == device:
                at = self._buffer.data_ptr()
                return at, cols, at + self._at, -(-cols // GROUP)
        return (*_like(name + ".q", self.q, torch.int8, device, rows, cols),
                *_like(name + ".e", self.e, torch.uint8, device, rows, -(-cols // GROUP)))


def _rows(name: str, t: torch.Tensor) -> Tuple[int, int, int]:
    """(rows, columns, row stride) of t with its leading dimensions flattened, without a copy."""
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a CUDA tensor")
    d = t.dim()
    if d == 2:
        rows, cols = t.shape
        ld, inner = t.stride()
        if rows == 0:  # whatever the strides say
            return 0, cols, cols
    else:
        if d == 0:
            raise ValueError(f"{name}: needs at least one dimension")
        cols, inner = t.shape[-1], t.stride(-1)
        if 0 in t.shape[:-1]:
            return 0, cols, cols
        rows, ld = 1, cols
        for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
            if n == 1:
                continue
            if rows == 1:
                ld = s
            elif s != ld * rows:
                raise ValueError(f"{name}: its leading dimensions cannot be taken as rows of one stride")
            rows *= n
    if inner != 1 and cols > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    # the stride of a single row, and of rows that a broadcast repeats, says nothing or too little
    if rows <= 1 or cols == 0:
        ld = cols
    elif ld < cols:
        raise ValueError(f"{name}: rows overlap (row stride {ld} for {cols} columns)")
    return rows, cols, ld


def _no_graph(a: torch.Tensor, b: Optional[torch.Tensor] = None, c: Optional[torch.Tensor] = None,
              d: Optional[torch.Tensor] = None) -> None:
    """The operators' results belong to no graph: refuses what autograd would lose without a word. (0.3 us of a call.)"""
    if torch.is_grad_enabled() and (a.requires_grad or (b is not None and b.requires_grad)
                                    or (c is not None and c.requires_grad) or (d is not None and d.requires_grad)):
        raise ValueError("the operator builds no graph, and an argument requires a gradient: use Linear8 or Mlp8, "
                         "torch.no_grad() or detach()")
    if forward_ad._current_level >= 0:
        for t in (a, b, c, d):
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError("an argument has a tangent, which the operator would lose: there is no forward-mode "
                                 "derivative")


def _act(act: str) -> int:
    a = ACTS.get(act)
    if a is None:
        raise ValueError(f"act: {act!r} is none of {', '.join(ACTS)}")
    return a


def _like(name: str, t: torch.Tensor, dtype, device, rows: int, cols: int) -> Tuple[int, int]:
    """(address, row stride) of a tensor that must have this type, place and size."""
    if t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name}: must be {dtype} on {device}")
    r, c, ld = _rows(name, t)
    if r != rows or c != cols:
        raise ValueError(f"{name}: {r} x {c}, not {rows} x {cols}")
    return t.data_ptr(), ld


def _vector(name: str, t: torch.Tensor, dtype, device, n: int) -> int:
    if t.dtype is not dtype or t.device != device or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name}: must be a contiguous vector of {n} {dtype} on {device}")
    return t.data_ptr()


# The current stream's handle without a Stream object around it (2.8 us of a small call otherwise).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
_functions = {}  # name -> (size query or None, function), as they are first called


def _function(name: str):
    f = _functions.get(name)
    if f is None:
        lib = S.load_library()
        f = _functions[name] = (getattr(lib, name + "_workspace_bytes", None), getattr(lib, name))
    return f


def _run(name: str, args: bytes, device):
    """Workspace, then the call, on the tensors' device and the current stream."""
    index = device.index
    if index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _run(name, args, device)
    size, f = _function(name)
    nbytes = size(args)
    if nbytes:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        st = f(args, ws.data_ptr(), nbytes, _raw_stream(index))
    else:
        st = f(args, None, 0, _raw_stream(index))
    if st:
        S.check(name, st)


def _call(name: str, device, *args):
    index = device.index
    if index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _call(name, device, *args)
    st = _function(name)[1](*args, _raw_stream(index))
    if st:
        S.check(name, st)


def _on(stream: torch.cuda.Stream, f, *args):
    """A call on a given stream: as if that stream were current, so that what it allocates belongs to that stream
    (and is not memory that the current stream's earlier work may still use)."""
    with torch.cuda.stream(stream):
        return f(*args)


def linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
           residual: Optional[torch.Tensor] = None, save: bool = False, out: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None):
    """y = act(x W^T + b) + residual; with save, (y, Packed8 of x W^T + b).

    x [..., k], w [n, k], bias [n], residual and out [..., n]; out may be the residual."""
    if stream is not None:
        return _on(stream, linear, x, w, bias, act, residual, save, out)
    _no_graph(x, w, bias, residual)
    a = _act(act)
    rows, k, ldx = _rows("x", x)
    code = S.dtype_code(x.dtype)
    dtype, device = x.dtype, x.device
    if w.dim() != 2:
        raise ValueError("w: must be a matrix")
    n = w.shape[0]
    pw, ldw = _like("w", w, dtype, device, n, k)
    shape = (*x.shape[:-1], n)
    pb = _vector("bias", bias, dtype, device, n) if bias is not None else 0
    pr, ldr = _like("residual", residual, dtype, device, rows, n) if residual is not None else (0, n)
    y = out
    if y is None:
        y = torch.empty(shape, dtype=dtype, device=device)
        py, ldy = y.data_ptr(), n
    else:
        py, ldy = _like("out", y, dtype, device, rows, n)
    saved = Packed8._make(shape, rows, n, device) if save else None
    pq, ldq, pe, lde = saved._places("saved", device, rows, n) if save else (0, n, 0, 1)
    args = _LINEAR.pack(x.data_ptr(), pw, pb, pr, py, pq, pe, rows, k, n, ldx, ldw, ldr, ldy, ldq, lde, code, a)
    _run("smat_linear", args, device)
    return (y, saved) if save else y


def linear_grad_input(dy: torch.Tensor, w: torch.Tensor, act: str = "none", saved: Optional[Packed8] = None,
                      out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """dx = (dy W) * act'(h^): back through a layer, and through the activation `act` that made the layer's input
    from the pre-activation `saved` ([..., k]; none with act "none"). dy [..., n], w [n, k]."""
    if stream is not None:
        return _on(stream, linear_grad_input, dy, w, act, saved, out)
    _no_graph(dy, w)
    a = _act(act)
    if (a != 0) != (saved is not None):
        raise ValueError("saved: needed with an activation, and only then")
    rows, n, lddy = _rows("dy", dy)
    code = S.dtype_code(dy.dtype)
    dtype, device = dy.dtype, dy.device
    if w.dim() != 2:
        raise ValueError("w: must be a matrix")
    k = w.shape[1]
    pw, ldw = _like("w", w, dtype, device, n, k)
    pq, ldq, pe, lde = saved._places("saved", device, rows, k) if saved is not None else (0, k, 0, 1)
    dx = out
    if dx is None:
        dx = torch.empty((*dy.shape[:-1], k), dtype=dtype, device=device)
        px, lddx = dx.data_ptr(), k
    else:
        px, lddx = _like("out", dx, dtype, device, rows, k)
    args = _GRAD_INPUT.pack(dy.data_ptr(), pw, pq, pe, px, rows, k, n, lddy, ldw, ldq, lde, lddx, code, a)
    _run("smat_grad_input", args, device)
    return dx


def linear_grad_weight(dy: torch.Tensor, x: Union[torch.Tensor, Packed8], act: str = "none", bias: bool = False,
                       out: Optional[torch.Tensor] = None, bias_out: Optional[torch.Tensor] = None,
                       accumulate: bool = False, stream: Optional[torch.cuda.Stream] = None):
    """(dW, db): dW = dy^T x^ [n, k] and, with bias, db [n] = dy's sums over its rows (else None).

    x is the layer's input [..., k], or its 8 bits; with `act`, the 8 bits of the pre-activation that `act` made
    the input from. With accumulate, dW is added to `out`, and db to `bias_out` where that is given."""
    if stream is not None:
        return _on(stream, linear_grad_weight, dy, x, act, bias, out, bias_out, accumulate)
    packed = isinstance(x, Packed8)
    _no_graph(dy, None if packed else x)
    a = _act(act)
    if a and not packed:
        raise ValueError("act: is applied to x in 8 bits only")
    if accumulate and out is None:
        raise ValueError("accumulate: needs out")
    if bias_out is not None and not bias:
        raise ValueError("bias_out: without bias")
    rows, n, lddy = _rows("dy", dy)
    code = S.dtype_code(dy.dtype)
    dtype, device = dy.dtype, dy.device
    k = x.shape[-1]
    px = pq = pe = 0
    ldx, ldq, lde = k, k, 1
    if packed:
        pq, ldq, pe, lde = x._places("x", device, rows, k)
    else:
        px, ldx = _like("x", x, dtype, device, rows, k)
    dw = out
    if dw is None:
        dw = torch.empty((n, k), dtype=dtype, device=device)
        pdw, lddw = dw.data_ptr(), k
    else:
        pdw, lddw = _like("out", dw, dtype, device, n, k)
    db, pdb = bias_out, 0
    if bias:
        if db is None:
            db = torch.empty(n, dtype=dtype, device=device)
        pdb = _vector("bias_out", db, dtype, device, n)
    flags = (1 if accumulate else 0) | (2 if accumulate and bias_out is not None else 0)
    args = _GRAD_WEIGHT.pack(dy.data_ptr(), px, pq, pe, pdw, pdb, rows, k, n, lddy, ldx, ldq, lde, lddw, code, a, flags,
                             0)
    _run("smat_grad_weight", args, device)
    return dw, db


def pack8(x: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> Packed8:
    """x in 8 bits."""
    if stream is not None:
        return _on(stream, pack8, x)
    _no_graph(x)
    rows, cols, ldx = _rows("x", x)
    code = S.dtype_code(x.dtype)
    p = Packed8._make(x.shape, rows, cols, x.device)
    _call("smat_pack8", x.device, x.data_ptr(), ldx, *p._places("p", x.device, rows, cols), rows, cols, code)
    return p


def unpack8(p: Packed8, act: str = "none", dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """act of the values that p stands for."""
    if stream is not None:
        return _on(stream, unpack8, p, act, dtype, out)
    a = _act(act)
    code = S.dtype_code(dtype)
    device, cols = p.device, p.shape[-1]
    rows = p.shape[:-1].numel()
    y = out
    if y is None:
        y = torch.empty(p.shape, dtype=dtype, device=device)
        py, ldy = y.data_ptr(), cols
    else:
        py, ldy = _like("out", y, dtype, device, rows, cols)
    _call("smat_unpack8", device, *p._places("p", device, rows, cols), py, ldy, rows, cols, code, a)
    return y


def act_grad8(dy: torch.Tensor, saved: Packed8, act: str, out: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """dy * act'(h^): a gradient back through an activation, from the pre-activation's 8 bits."""
    if stream is not None:
        return _on(stream, act_grad8, dy, saved, act, out)
    _no_graph(dy)
    a = _act(act)
    rows, cols, lddy = _rows("dy", dy)
    code = S.dtype_code(dy.dtype)
    places = saved._places("saved", dy.device, rows, cols)
    dh = out
    if dh is None:
        dh = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
        ph, ldh = dh.data_ptr(), cols
    else:
        ph, ldh = _like("out", dh, dy.dtype, dy.device, rows, cols)
    _call("smat_act_grad8", dy.device, dy.data_ptr(), lddy, *places, ph, ldh, rows, cols, code, a)
    return dh


def poll_errors(stream: Optional[torch.cuda.Stream] = None) -> int:
    """Read and clear the products' device error flags (0 = none; 1 = a bounded wait ran out and a result is
    unfinished, of either dtype); synchronises the stream. No call returns this, and no layer asks for it: poll where the
    program waits for the GPU anyway, before results are kept (a loss that is read, a checkpoint)."""
    v = ctypes.c_int32()
    S.check("smat_linear_poll_errors", S.load_library().smat_linear_poll_errors(S._stream_handle(stream), ctypes.byref(v)))
    return v.value


# ------------------------------------------------------------------- layers ---
def _rows_like(t: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """A layer's input as the operators take it: one that is transposed, broadcast or strided otherwise than as rows of one
    stride is written out, as torch.nn.Linear does."""
    if t is None or t.is_contiguous():
        return t
    try:
        _rows("", t)
        return t
    except ValueError:
        return t.contiguous()


def _autocast(layer, x: torch.Tensor, *rest: Optional[torch.Tensor]) -> torch.Tensor:
    """layer(x, parameters, residual) under torch.autocast: in its type, as torch.nn.Linear would be (64-bit tensors stay as they
    are). A residual of another type is added afterwards, and the result has the wider one, as beside torch.nn.Linear."""
    dtype = torch.get_autocast_dtype("cuda")
    x, *params = (t if t is None or t.dtype is torch.float64 else t.to(dtype) for t in (x, *rest[:-1]))
    residual = rest[-1]
    if residual is None or residual.dtype is x.dtype:
        return layer(x, *params, residual)
    return layer(x, *params, None) + residual


def _row_sums(dy: torch.Tensor) -> torch.Tensor:
    """db alone, of a layer whose weight is frozen: the weight gradient's own sums, with no columns of x."""
    dy = dy.reshape(-1, dy.shape[-1])
    return linear_grad_weight(dy, dy.new_empty(dy.shape[0], 0), bias=True)[1]


class _FirstOnly(torch.autograd.Function):
    """Gradients as they are; going back through them raises. `anchor` and `dy` tie them to all that they depend on, so
    that a second derivative meets this, whichever of those it is taken by."""

    @staticmethod
    def forward(ctx, anchor, dy, *grads):
        return tuple(g.view_as(g) if g is not None else None for g in grads)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("Linear8 and Mlp8 have first derivatives only: their gradients cannot be differentiated")


def _first_only(ctx, dy, gradients):
    """gradients(ctx, dy). They are made by the library's kernels and belong to no graph. Where one is asked for
    (create_graph), they refuse to be differentiated; otherwise terms of a second derivative would be left out silently. The
    residual's gradient, which is dy, has the graph that dy has."""
    if not torch.is_grad_enabled():
        return gradients(ctx, dy)
    with torch.no_grad():
        grads = gradients(ctx, dy)
    anchor = ctx.saved_tensors[-1]
    refusing = _FirstOnly.apply(anchor, dy, *(None if g is dy else g for g in grads))
    return tuple(dy if g is dy else h for g, h in zip(grads, refusing))


class _Linear8(torch.autograd.Function):
    """(y, anchor): `anchor` is empty and stands for the inputs in _FirstOnly."""

    @staticmethod
    def forward(ctx, x, w, b, residual, act):
        ctx.act = act
        ctx.set_materialize_grads(False)
        x, w, b, residual = map(_rows_like, (x, w, b, residual))
        need_h = act != "none" and any(ctx.needs_input_grad[:3])
        y = linear(x, w, b, act, residual, save=need_h)
        y, h = y if need_h else (y, None)
        p = pack8(x) if ctx.needs_input_grad[1] else None
        anchor = x.new_empty(0)
        ctx.save_for_backward(w, *((h.q, h.e) if h else (None, None)), *((p.q, p.e) if p else (None, None)), anchor)
        return y, anchor

    @staticmethod
    def backward(ctx, dy, _):
        return _first_only(ctx, dy, _Linear8._gradients)

    @staticmethod
    def _gradients(ctx, grad):
        w, hq, he, xq, xe, _ = ctx.saved_tensors
        need_x, need_w, need_b, need_r, _ = ctx.needs_input_grad
        dy = grad.contiguous()
        dh = act_grad8(dy, Packed8(hq, he), ctx.act) if hq is not None else dy
        dx = dw = db = None
        if need_x:
            dx = linear_grad_input(dh, w)
        if need_w:
            dw, db = linear_grad_weight(dh, Packed8(xq, xe), bias=need_b)
        elif need_b:
            db = _row_sums(dh)
        return dx, dw, db, (grad if need_r else None), None


class _Mlp8(torch.autograd.Function):
    """As _Linear8."""

    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, residual, act):
        ctx.act = act
        ctx.set_materialize_grads(False)
        x, w1, b1, w2, b2, residual = map(_rows_like, (x, w1, b1, w2, b2, residual))
        a, h = linear(x, w1, b1, act, save=True)
        y = linear(a, w2, b2, "none", residual)
        p = pack8(x) if ctx.needs_input_grad[1] else None
        anchor = x.new_empty(0)
        ctx.save_for_backward(w1, w2, *((p.q, p.e) if p else (None, None)), h.q, h.e, anchor)
        return y, anchor

    @staticmethod
    def backward(ctx, dy, _):
        return _first_only(ctx, dy, _Mlp8._gradients)

    @staticmethod
    def _gradients(ctx, grad):
        w1, w2, xq, xe, hq, he, _ = ctx.saved_tensors
        need_x, need_w1, need_b1, need_w2, need_b2, need_r, _ = ctx.needs_input_grad
        h = Packed8(hq, he)
        dy = grad.contiguous()
        dx = dw1 = db1 = dw2 = db2 = None
        if need_w2:
            dw2, db2 = linear_grad_weight(dy, h, ctx.act, bias=need_b2)
        elif need_b2:
            db2 = _row_sums(dy)
        if need_x or need_w1 or need_b1:
            dh = linear_grad_input(dy, w2, ctx.act, h if ctx.act != "none" else None)
            if need_w1:
                dw1, db1 = linear_grad_weight(dh, Packed8(xq, xe), bias=need_b1)
            elif need_b1:
                db1 = _row_sums(dh)
            if need_x:
                dx = linear_grad_input(dh, w1)
        return dx, dw1, db1, dw2, db2, (grad if need_r else None), None


class Linear8(torch.nn.Linear):
    """torch.nn.Linear followed by an activation and a residual; its backward pass reads the input and, with an
    activation, the pre-activation in 8 bits instead of keeping them whole. First derivatives only: one taken of its
    gradients raises RuntimeError. Inputs and weights may have any strides; torch.autocast to bf16 casts them as it does for
    torch.nn.Linear. What poll_errors says of its products is for the caller to ask."""

    def __init__(self, in_features: int, out_features: int, bias: bool = True, act: str = "none", device=None,
                 dtype=None):
        super().__init__(in_features, out_features, bias, device=device, dtype=dtype)
        _act(act)
        self.act = act

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        if torch.is_autocast_enabled("cuda"):
            return _autocast(self._forward, x, self.weight, self.bias, residual)
        return self._forward(x, self.weight, self.bias, residual)

    def _forward(self, x, w, b, residual):
        if not torch.is_grad_enabled():
            x, w, b, residual = map(_rows_like, (x, w, b, residual))
            return linear(x, w, b, self.act, residual)
        return _Linear8.apply(x, w, b, residual, self.act)[0]


class Mlp8(torch.nn.Module):
    """y = act(x W1^T + b1) W2^T + b2 + residual. Between forward and backward it holds x and the pre-activation in
    8 bits, 33 / 32 bytes per element; the second layer's input is recomputed from the pre-activation. First
    derivatives only, inputs, autocast and poll_errors as Linear8."""

    def __init__(self, features: int, hidden: int, bias: bool = True, act: str = "gelu", device=None, dtype=None):
        super().__init__()
        _act(act)
        self.act = act
        self.fc1 = torch.nn.Linear(features, hidden, bias, device=device, dtype=dtype)
        self.fc2 = torch.nn.Linear(hidden, features, bias, device=device, dtype=dtype)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        fc1, fc2 = self.fc1, self.fc2
        if torch.is_autocast_enabled("cuda"):
            return _autocast(self._forward, x, fc1.weight, fc1.bias, fc2.weight, fc2.bias, residual)
        return self._forward(x, fc1.weight, fc1.bias, fc2.weight, fc2.bias, residual)

    def _forward(self, x, w1, b1, w2, b2, residual):
        if not torch.is_grad_enabled():
            x, w1, b1, w2, b2, residual = map(_rows_like, (x, w1, b1, w2, b2, residual))
            return linear(linear(x, w1, b1, self.act), w2, b2, "none", residual)
        return _Mlp8.apply(x, w1, b1, w2, b2, residual, self.act)[0]
