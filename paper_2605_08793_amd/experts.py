"""What follows a router's choices: the buffers of one size, and the calls.

`ExpertOrder` puts the choices of RowRoute into the order of their experts, `ExpertProduct` multiplies each expert's rows by its
weights (with the gate of a gated layer) and forms the gradients to the rows and to the weights, `ExpertCombine` adds the rows of each
token up again under the router's weights (its .g_weight is what RowRoute.grad takes), and `GradClip` gives the norm over all gradients and scales them.
A gated layer of n tokens, and the way back:

    order.sort(route.idx)
    up.product(X, W_up, order.start, order.order, k)               # gated, keep=True: .Y, .saved
    down.product(up.Y, W_down, order.start)
    total.combine(down.Y, order.place, route.weight)               # .out

    total.grad(g_out, down.Y, order.place, route.weight)           # .dY, .g_weight
    down.weight_grad(total.dY, up.Y, order.start)
    down.input_grad(total.dY, W_down, order.start, saved=up.saved)  # the gradient to the gated product's sums
    up.weight_grad(down.dX, X, order.start, order.order, k)
    up.input_grad(down.dX, W_up, order.start)
    tokens.combine(up.dX, order.place)                             # the gradient to X, without the router's part

As in the row objects, no arithmetic happens here, the results stay on the device in buffers that the next call of the same object writes
again, and before the first call they hold anything: so do rows that belong to no expert.
"""
import torch

from . import binding as B
from .rows import _address, _output


class _Buffers:
    def __init__(self, device):
        self.device = torch.empty(0, device=device).device

    def _buffer(self, *shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=self.device)

    def _workspace(self, size):
        return self._buffer(max(size, 256), dtype=torch.uint8)

    def _list(self, v, n, width, name, dtype=torch.float32, optional=False):
        if v is not None and v.device != self.device:
            raise TypeError(f"{name} must be on {self.device}")
        return B._list(v, n, width, name, dtype, optional)

    def _matrix(self, t, n, m, name, dtype):
        """(address, leading dimension) of an n x m matrix; n None: any."""
        rows, cols, _, ld, at = B._scores(t, name)
        if (n is not None and rows != n) or cols != m or t.dtype != dtype or t.device != self.device:
            raise TypeError(f"{name} must be {'rows' if n is None else n} x {m} of type {dtype} on {self.device}")
        return at, ld


class ExpertOrder(_Buffers):
    """The choices of n tokens, k each, by expert.

    After `sort`: .start (experts + 1, int64: where each expert's rows begin), .order (n * k, int32: the choice i * k + l of each row, -1 behind
    the last) and .place (n, k, int32: the row of each choice, -1 for none)."""
    start, order, place, workspace = map(_output, ("_start", "_order", "_place", "_work"))

    def __init__(self, n: int, k: int, experts: int, device="cuda"):
        super().__init__(device)
        self.n, self.k, self.experts = int(n), int(k), int(experts)
        self._work = self._workspace(B.regot_expert_order_workspace_bytes(n, k, experts))
        self._start = self._buffer(self.experts + 1, dtype=torch.int64)
        self._order = self._buffer(self.n * self.k, dtype=torch.int32)
        self._place = self._buffer(self.n, self.k, dtype=torch.int32)
        self._out = [_address(t) for t in (self._start, self._order, self._place, self._work)] + [self._work.numel()]

    def sort(self, idx):
        """idx (n, k) int32: RowRoute.idx; anything outside 0 .. experts - 1 is no choice."""
        B._check(B.load().regot_expert_order(
            self.n, self.k, self.experts, self._list(idx, self.n, self.k, "idx", torch.int32), *self._out, B._row_stream(idx, None)),
            "regot_expert_order")


class ExpertProduct(_Buffers):
    """Each expert's rows times its weights: `rows` rows of d inputs and m outputs, weights (experts, m, d), or (experts, 2 m, d) where
    `gated`: the first m outputs are put through silu and multiplied by the others.

    After `product`: .Y (rows, m), and with `keep` .saved (rows, 2 m: the outputs before the gate).  After `input_grad`: .dX; after
    `weight_grad`: .dW, of type `grad_dtype` (that of the rows, or float32).  .dX and .dW can be replaced by tensors of the same shape and type (.dX by one of either width: it is
    that of the last call, and each width keeps its own)."""
    Y, saved, workspace = map(_output, ("_Y", "_saved", "_work"))

    def __init__(self, rows: int, m: int, d: int, experts: int, gated=False, keep=False, dtype=torch.bfloat16, grad_dtype=None, device="cuda"):
        super().__init__(device)
        if dtype not in B.SCORE_TYPES:
            raise TypeError("dtype must be float32, bfloat16 or float16")
        self.rows, self.m, self.d, self.experts, self.gated, self.dtype = int(rows), int(m), int(d), int(experts), bool(gated), dtype
        self.grad_dtype = dtype if grad_dtype is None else grad_dtype
        if self.grad_dtype not in (dtype, torch.float32):
            raise TypeError("grad_dtype must be float32 or the type of the rows")
        self.wide = 2 * self.m if gated else self.m
        self._Y = self._buffer(self.rows, self.m, dtype=dtype)
        self._saved = self._buffer(self.rows, 2 * self.m, dtype=dtype) if keep and gated else None
        self._work = self._workspace(B.regot_expert_weight_grad_workspace_bytes(self.rows, self.wide, self.d, self.experts))
        self.dX = self.dW = None
        self._aside = {}  # .dX by its columns, of the width that was not asked for last: a captured call may still write it

    def _run(self, X, x_rows, d, W, by, start, order, k, act, m, Y, saved, ldS):
        _, _, _, w_by, ldW, stride, w_at = W
        at, ldX = X
        to, ldY = Y
        B._check(B.load().regot_expert_product(
            self.rows, m, d, self.experts, self._list(start, self.experts + 1, 1, "start", torch.int64), at, B.SCORE_TYPES[self.dtype], ldX, x_rows,
            self._list(order, self.rows, 1, "order", torch.int32, optional=True), int(k), w_at, w_by ^ by, ldW, stride, act, to, ldY, saved, ldS,
            B._row_stream(start, None)), "regot_expert_product")

    def _weights(self, W):
        found = B._weights(W)
        if found[:3] != (self.experts, self.wide, self.d) or W.dtype != self.dtype or W.device != self.device:
            raise TypeError(f"W must be {self.experts} x {self.wide} x {self.d} of type {self.dtype} on {self.device}")
        return found

    def _out(self, name, shape, dtype):
        t = getattr(self, name)
        if name == "dX" and t is not None and t.shape != shape and t.shape in ((self.rows, self.d), (self.rows, 2 * self.d)):
            self._aside[t.shape[1]] = t
            t = self._aside.get(shape[1])
        if t is None:
            t = self._buffer(*shape, dtype=dtype)
        if t.shape != shape or t.dtype != dtype or t.device != self.device:
            raise TypeError(f"{name} must be of shape {tuple(shape)}, type {dtype}, on {self.device}")
        setattr(self, name, t)
        return t

    def product(self, X, W, start, order=None, k=1):
        """X (rows, d), or with `order` the tokens (n, d), each of k choices: ExpertOrder's .start and .order."""
        x = self._matrix(X, None, self.d, "X", self.dtype)
        self._run(x, X.shape[0], self.d, self._weights(W), 0, start, order, k, int(self.gated), self.m, (self._Y.data_ptr(), max(self.m, 1)),
                  _address(self._saved), 2 * self.m)

    def input_grad(self, dY, W, start, saved=None):
        """The gradient to the rows that `product` took, in .dX (rows, d); dY (rows, m), with `gated` (rows, 2 m): to the outputs before the gate.
        saved: the .saved of the gated product whose .Y those rows are; .dX (rows, 2 d) is then the gradient to its outputs before the gate."""
        g = self._matrix(dY, self.rows, self.wide, "dY", self.dtype)
        dX = self._out("dX", torch.Size((self.rows, self.d if saved is None else 2 * self.d)), self.dtype)
        s_at, ldS = (0, 2 * self.d) if saved is None else self._matrix(saved, self.rows, 2 * self.d, "saved", self.dtype)
        self._run(g, self.rows, self.wide, self._weights(W), 1, start, None, 1, 0 if saved is None else 2, self.d,
                  self._matrix(dX, self.rows, dX.shape[1], "dX", self.dtype), s_at, ldS)
        return dX

    def weight_grad(self, dY, X, start, order=None, k=1):
        """The gradient to the weights, in .dW (experts, m or 2 m, d); dY as for `input_grad`, X and order as `product` took them."""
        g_at, ldY = self._matrix(dY, self.rows, self.wide, "dY", self.dtype)
        at, ldX = self._matrix(X, None, self.d, "X", self.dtype)
        dW = self._out("dW", torch.Size((self.experts, self.wide, self.d)), self.grad_dtype)
        _, _, _, by, ldW, stride, to = B._weights(dW, "dW")
        if by != 0 and dW.numel():
            raise TypeError("dW must have rows of neighbours")
        B._check(B.load().regot_expert_weight_grad(
            self.rows, self.wide, self.d, self.experts, self._list(start, self.experts + 1, 1, "start", torch.int64), g_at, B.SCORE_TYPES[self.dtype], ldY,
            at, ldX, X.shape[0], self._list(order, self.rows, 1, "order", torch.int32, optional=True), int(k), to, B.SCORE_TYPES[self.grad_dtype], ldW,
            stride, self._work.data_ptr(), self._work.numel(), B._row_stream(start, None)), "regot_expert_weight_grad")
        return dW


class ExpertCombine(_Buffers):
    """The k rows of each of n tokens, of m columns, weighted and added up; `rows` rows, n * k where it is not given.

    After `combine`: .out (n, m).  After `grad`: .dY (rows, m; can be replaced by a tensor of that shape) and .g_weight (n, k)."""
    out, g_weight = map(_output, ("_total", "_g_weight"))

    def __init__(self, n: int, k: int, m: int, rows=None, dtype=torch.bfloat16, device="cuda"):
        super().__init__(device)
        if dtype not in B.SCORE_TYPES:
            raise TypeError("dtype must be float32, bfloat16 or float16")
        self.n, self.k, self.m, self.dtype = int(n), int(k), int(m), dtype
        self.rows = self.n * self.k if rows is None else int(rows)
        self._total = self._buffer(self.n, self.m, dtype=dtype)
        self._g_weight = self._buffer(self.n, self.k)
        self.dY = None

    def combine(self, Y, place, weight=None):
        """place (n, k) int32: ExpertOrder's; weight (n, k): RowRoute's, None for 1."""
        at, ldY = self._matrix(Y, self.rows, self.m, "Y", self.dtype)
        B._check(B.load().regot_expert_combine(
            self.n, self.k, self.m, self.rows, at, B.SCORE_TYPES[self.dtype], ldY, self._list(place, self.n, self.k, "place", torch.int32),
            self._list(weight, self.n, self.k, "weight", optional=True), self._total.data_ptr(), max(self.m, 1), B._row_stream(Y, None)),
            "regot_expert_combine")

    def grad(self, g_out, Y, place, weight=None):
        """The gradients of sum(g_out * out), in .dY and .g_weight; Y None: to the rows alone.  Rows of .dY that no choice has stay as they were."""
        g_at, ldG = self._matrix(g_out, self.n, self.m, "g_out", self.dtype)
        if self.dY is None:
            self.dY = self._buffer(self.rows, self.m, dtype=self.dtype)
        to, ldD = self._matrix(self.dY, self.rows, self.m, "dY", self.dtype)
        at, ldY = (0, self.m) if Y is None else self._matrix(Y, self.rows, self.m, "Y", self.dtype)
        B._check(B.load().regot_expert_combine_grad(
            self.n, self.k, self.m, self.rows, g_at, B.SCORE_TYPES[self.dtype], ldG, at, ldY, self._list(place, self.n, self.k, "place", torch.int32),
            self._list(weight, self.n, self.k, "weight", optional=True), to, ldD, 0 if Y is None else self._g_weight.data_ptr(),
            B._row_stream(g_out, None)), "regot_expert_combine_grad")
        return self.dY


class GradClip(_Buffers):
    """The norm over a list of tensors, and their scaling to a norm of at most `max_norm`, in place or to the tensors `out`.

    After `norm` or `clip`: .norm_out (1); after `clip`: .factor (1).  The tensors' addresses are looked up once: tensors that a program makes
    anew for each step belong to a new object."""
    norm_out, factor, workspace = map(_output, ("_norm", "_factor", "_work"))

    def __init__(self, tensors, out=None):
        tensors = list(tensors)
        self._kept = tensors, None if out is None else list(out)
        self._list_of = B._tensors(*self._kept)
        super().__init__(tensors[0].device if tensors else "cuda")
        self._work = self._workspace(B.regot_grad_norm_workspace_bytes(tensors))
        self._norm, self._factor = self._buffer(1), self._buffer(1)

    def norm(self):
        B._check(B.load().regot_grad_norm(
            len(self._kept[0]), self._list_of, self._norm.data_ptr(), self._work.data_ptr(), self._work.numel(), B._list_stream([self._norm], None)),
            "regot_grad_norm")

    def clip(self, max_norm):
        B._check(B.load().regot_grad_clip(
            len(self._kept[0]), self._list_of, float(max_norm), self._norm.data_ptr(), self._factor.data_ptr(), self._work.data_ptr(),
            self._work.numel(), B._list_stream([self._norm], None)), "regot_grad_clip")
