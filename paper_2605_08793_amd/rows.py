"""Row operators on a model's scores: the buffers of one size, and the calls.

The model's side of the plan that the solver works on: `RowLogprob` gives log probabilities of given columns, the entropy
and the best columns of each row under column duals (`bias`), `RowDistill` the loss of a model's rows against such sparse
targets with its gradient, `RowRoute` the k columns (experts) that each row goes to, with their weights.  As in the driver,
no arithmetic happens here, and the results stay on the device, in buffers that the next call of the same object writes
again.  (The buffers' addresses are looked up once, which is a fifth of a small call: the outputs cannot be replaced by
other tensors.  Only .dS can be, by a tensor that `grad` checks at each call.)  Before the first call they hold anything.
"""
import torch

from . import binding as B


def _address(t):
    return 0 if t is None else t.data_ptr()


def _output(name):
    return property(lambda self: getattr(self, name), doc="a buffer of the object, which its calls write")


class _Rows:
    """n rows of m scores of one type, on one device."""

    def __init__(self, n, m, dtype, device):
        self.n, self.m, self.dtype = int(n), int(m), dtype
        if dtype not in B.SCORE_TYPES:
            raise TypeError("dtype must be float32, bfloat16 or float16")
        self.device = torch.empty(0, device=device).device
        self._kept = []

    def _buffer(self, *shape, dtype=torch.float32):
        t = torch.empty(*shape, dtype=dtype, device=self.device)
        self._kept.append(t)
        return t

    def _workspace(self, size):
        return self._buffer(max(size, 256), dtype=torch.uint8)

    def _scores(self, S):
        """(n, m, address, type, leading dimension) of a call's scores, which have to be of the object's size, type and device."""
        n, m, kind, ld, at = B._scores(S)
        if n != self.n or m != self.m or S.dtype != self.dtype or S.device != self.device:
            raise TypeError(f"S must be {self.n} x {self.m} of type {self.dtype} on {self.device}")
        return n, m, at, kind, ld

    def _gradient(self, S):
        if self.dS is None:
            self.dS = self._buffer(self.n, self.m, dtype=self.dtype)
        return B._same_scores(self.dS, S)[::-1]


class RowLogprob(_Rows):
    """Log probabilities, entropy and the `k` best columns of n rows of m scores of type `dtype`.

    After `logprob`: .logprob_out (n, targets), .entropy (n), .stats (n, 2: the maximum, and the logarithm of the sum
    relative to it), .top_idx and .top_logprob (n, k).  After `grad`: .dS (n, m)."""
    logprob_out, entropy, stats, top_idx, top_logprob = map(_output, ("_logprob_out", "_entropy", "_stats", "_top_idx", "_top_logprob"))
    workspace = _output("_work")

    def __init__(self, n: int, m: int, k: int = 0, targets: int = 1, dtype=torch.bfloat16, device="cuda"):
        super().__init__(n, m, dtype, device)
        self.k, self.targets = int(k), int(targets)
        self._work = self._workspace(B.regot_row_logprob_workspace_bytes(n, m, k))
        self._logprob_out = self._buffer(n, targets) if targets else None
        self._entropy = self._buffer(n)
        self._stats = self._buffer(n, 2)
        self._top_idx = self._buffer(n, k, dtype=torch.int32) if k else None
        self._top_logprob = self._buffer(n, k) if k else None
        self.dS = None
        self._out = [_address(t) for t in (self.logprob_out, self.entropy, self.stats, self.top_idx, self.top_logprob, self.workspace)]
        self._out.append(self.workspace.numel())

    def logprob(self, S, target=None, eta=1.0, bias=None):
        """target: (n, targets) int32, -1 for none; may be left out where targets = 0."""
        B._check(B.load().regot_row_logprob(
            *self._scores(S), B._list(bias, 1, self.m, "bias", optional=True), float(eta),
            B._list(target, self.n, self.targets, "target", torch.int32, optional=self.targets == 0), self.targets, self.k,
            *self._out, B._row_stream(S, None)), "regot_row_logprob")

    def grad(self, S, target, g_logprob, g_entropy=None, eta=1.0, bias=None, stats=None, entropy=None):
        """The gradient to S of sum(g_logprob * logprob_out) + sum(g_entropy * entropy), in .dS; after `logprob` of the same
        S, bias and eta, or with the stats and entropy that it gave.  target and g_logprob may be None, for the entropy alone."""
        n, targets = self.n, 0 if target is None else self.targets
        B._check(B.load().regot_row_logprob_grad(
            *self._scores(S), B._list(bias, 1, self.m, "bias", optional=True), float(eta),
            B._list(target, n, targets, "target", torch.int32, optional=True), targets,
            self._out[2] if stats is None else B._list(stats, n, 2, "stats"),
            self._out[1] if entropy is None else B._list(entropy, n, 1, "entropy"),
            B._list(g_logprob, n, targets, "g_logprob", optional=targets == 0), B._list(g_entropy, n, 1, "g_entropy", optional=True),
            *self._gradient(S), B._row_stream(S, None)), "regot_row_logprob_grad")
        return self.dS


class RowDistill(_Rows):
    """Loss of n rows of m scores against lists of k teacher entries, with the gradient (unless grad=False).

    After `distill`: .loss (n), .grad (n, m) of S's type."""
    loss, grad, workspace = map(_output, ("_loss", "_grad", "_work"))

    def __init__(self, n: int, m: int, k: int, dtype=torch.bfloat16, device="cuda", grad=True):
        super().__init__(n, m, dtype, device)
        self.k = int(k)
        self._work = self._workspace(B.regot_row_distill_workspace_bytes(n, m, k))
        self._loss = self._buffer(n)
        self._grad = self._buffer(n, m, dtype=dtype) if grad else None
        self._out = [_address(self.loss), _address(self.grad), self.m, _address(self.workspace), self.workspace.numel()]

    def distill(self, S, t_idx, t_score, eta=1.0, row_weight=None):
        """t_idx (n, k) int32, -1 for no entry; t_score (n, k): the teacher's scores or log probabilities there, which are
        divided by eta: log probabilities (RowLogprob.top_logprob, of whatever eta) are scores at temperature 1, and belong
        to eta = 1, or are multiplied by their own eta first."""
        B._check(B.load().regot_row_distill(
            *self._scores(S), float(eta), B._list(t_idx, self.n, self.k, "t_idx", torch.int32),
            B._list(t_score, self.n, self.k, "t_score"), self.k, B._list(row_weight, self.n, 1, "row_weight", optional=True),
            *self._out, B._row_stream(S, None)), "regot_row_distill")


class RowRoute(_Rows):
    """The k columns of n rows of m scores, and their weights: .idx, .weight (n, k); .dS (n, m) after `grad`."""
    idx, weight = map(_output, ("_idx", "_weight"))

    def __init__(self, n: int, m: int, k: int, score="softmax", bias_on=None, groups=1, groups_kept=1, group_by="max",
                 renormalise=True, scale=1.0, dtype=torch.float32, device="cuda"):
        super().__init__(n, m, dtype, device)
        self.k = int(k)
        self._score, self._bias_on = B.SCORE_KINDS[score], B.BIAS_ON[bias_on]
        self._choose = self._bias_on, self._score, int(groups), int(groups_kept), B.GROUP_BY[group_by], self.k
        self._weigh = int(bool(renormalise)), float(scale)
        self._idx = self._buffer(n, k, dtype=torch.int32)
        self._weight = self._buffer(n, k)
        self.dS = None
        self._out = self.idx.data_ptr(), self.weight.data_ptr()

    def route(self, S, bias=None):
        B._check(B.load().regot_row_route(
            *self._scores(S), B._list(bias, 1, self.m, "bias", optional=True), *self._choose, *self._weigh, *self._out,
            B._row_stream(S, None)), "regot_row_route")

    def grad(self, S, g_weight):
        """The gradient to S of sum(g_weight * weight) at the choices of the last `route`, in .dS."""
        B._check(B.load().regot_row_route_grad(
            *self._scores(S), self._score, self._out[0], self.k, *self._weigh, B._list(g_weight, self.n, self.k, "g_weight"),
            *self._gradient(S), B._row_stream(S, None)), "regot_row_route_grad")
        return self.dS
