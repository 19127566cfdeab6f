"""Row operators on a model's scores: the buffers of one size, and the calls.

The model's side of the plan that the solver works on: `RowLogprob` gives log probabilities of given columns, the entropy
and the best columns of each row under column duals (`bias`), `RowDistill` the loss of a model's rows against such sparse
targets with its gradient, `RowRoute` the k columns (experts) that each row goes to, with their weights.  As in the driver,
no arithmetic happens here, and the results stay on the device, in buffers that the next call of the same object writes
again.
"""
import torch

from . import binding as B


class RowLogprob:
    """Log probabilities, entropy and the `k` best columns of n rows of m scores of type `dtype`.

    After `logprob`: .logprob_out (n, targets), .entropy (n), .stats (n, 2: the maximum, and the logarithm of the sum
    relative to it), .top_idx and .top_logprob (n, k)."""

    def __init__(self, n: int, m: int, k: int = 0, targets: int = 1, dtype=torch.bfloat16, device="cuda"):
        self.n, self.m, self.k, self.targets, self.dtype = int(n), int(m), int(k), int(targets), dtype
        self.device = torch.device(device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.workspace = torch.empty(max(B.regot_row_logprob_workspace_bytes(n, m, k), 256), dtype=torch.uint8, device=self.device)
        self.logprob_out = torch.zeros(n, targets, **f32) if targets else None
        self.entropy = torch.zeros(n, **f32)
        self.stats = torch.zeros(n, 2, **f32)
        self.top_idx = torch.zeros(n, k, dtype=torch.int32, device=self.device) if k else None
        self.top_logprob = torch.zeros(n, k, **f32) if k else None
        self.dS = None

    def logprob(self, S, target=None, eta=1.0, bias=None):
        """target: (n, targets) int32, -1 for none; may be left out where targets = 0."""
        B.regot_row_logprob(S, target, eta, self.logprob_out, self.entropy, self.stats, self.top_idx, self.top_logprob,
                            bias=bias, workspace=self.workspace)

    def grad(self, S, target, g_logprob, g_entropy=None, eta=1.0, bias=None, stats=None, entropy=None):
        """The gradient to S of sum(g_logprob * logprob_out) + sum(g_entropy * entropy), in .dS; after `logprob` of the same
        S, bias and eta, or with the stats and entropy that it gave."""
        if self.dS is None:
            self.dS = torch.empty(self.n, self.m, dtype=self.dtype, device=self.device)
        B.regot_row_logprob_grad(S, target, eta, self.stats if stats is None else stats,
                                 None if g_entropy is None else self.entropy if entropy is None else entropy,
                                 g_logprob, g_entropy, self.dS, bias=bias)
        return self.dS


class RowDistill:
    """Loss of n rows of m scores against lists of k teacher entries, with the gradient (unless grad=False).

    After `distill`: .loss (n), .grad (n, m) of S's type."""

    def __init__(self, n: int, m: int, k: int, dtype=torch.bfloat16, device="cuda", grad=True):
        self.n, self.m, self.k = int(n), int(m), int(k)
        dev = torch.device(device)
        self.workspace = torch.empty(max(B.regot_row_distill_workspace_bytes(n, m, k), 256), dtype=torch.uint8, device=dev)
        self.loss = torch.zeros(n, dtype=torch.float32, device=dev)
        self.grad = torch.empty(n, m, dtype=dtype, device=dev) if grad else None

    def distill(self, S, t_idx, t_score, eta=1.0, row_weight=None):
        """t_idx (n, k) int32, -1 for no entry; t_score (n, k): the teacher's scores or log probabilities there."""
        B.regot_row_distill(S, t_idx, t_score, eta, self.loss, self.grad, row_weight=row_weight, workspace=self.workspace)


class RowRoute:
    """The k columns of n rows of m scores, and their weights: .idx, .weight (n, k); .dS after `grad`."""

    def __init__(self, n: int, m: int, k: int, score="softmax", bias_on=None, groups=1, groups_kept=1, group_by="max",
                 renormalise=True, scale=1.0, dtype=torch.float32, device="cuda"):
        self.n, self.m, self.k, self.dtype = int(n), int(m), int(k), dtype
        self.device = torch.device(device)
        self.choose = dict(bias_on=bias_on, groups=groups, groups_kept=groups_kept, group_by=group_by)
        self.weigh = dict(score=score, renormalise=renormalise, scale=scale)
        self.idx = torch.zeros(n, k, dtype=torch.int32, device=self.device)
        self.weight = torch.zeros(n, k, dtype=torch.float32, device=self.device)
        self.dS = None

    def route(self, S, bias=None):
        B.regot_row_route(S, self.idx, self.weight, bias=bias, **self.choose, **self.weigh)

    def grad(self, S, g_weight):
        """The gradient to S of sum(g_weight * weight) at the choices of the last `route`, in .dS."""
        if self.dS is None:
            self.dS = torch.empty(self.n, self.m, dtype=self.dtype, device=self.device)
        B.regot_row_route_grad(S, self.idx, g_weight, self.dS, **self.weigh)
        return self.dS
