"""Balanced targets and balanced routing: the solver's column duals beside a model's scores.

    python -m paper_2605_08793_amd.balanced

Two uses of one idea.  Scores of n rows against m columns are the negative costs of a transport problem with uniform
marginals; its column duals beta, added to the scores, spread the rows evenly over the columns.

`train_student`: a teacher's scores of samples against prototypes are balanced by a few Sinkhorn sweeps; the best columns of
each row under those duals (RowLogprob with bias) are the targets that a linear student learns (RowDistill: loss and
gradient in one call), and its answers are looked at with RowLogprob.

`route_tokens`: a router's scores of tokens against experts are balanced in the same way; RowRoute takes the duals as its
bias, and regot_pattern_transpose puts the choices into the order of the experts.
"""
import torch

from . import binding as B
from .driver import DualPass
from .rows import RowDistill, RowLogprob, RowRoute


def column_duals(scores, eta: float, sweeps: int):
    """Duals beta (m, fp32) of the columns: rows and columns with uniform marginals, costs = -scores."""
    n, m = scores.shape
    M = (-scores).double().contiguous()
    a = torch.full((n,), 1.0 / n, dtype=torch.float64, device=M.device)
    b = torch.full((m,), 1.0 / m, dtype=torch.float64, device=M.device)
    _, beta = DualPass(n, m, device=M.device).sinkhorn_sweeps(M, a, b, eta, sweeps)
    return beta.float()


def train_student(n=2048, m=1500, features=96, k=16, eta=0.1, sweeps=10, steps=60, rate=300.0, dtype=torch.bfloat16, seed=0):
    """Returns the mean loss of each step, the share of the most used column with and without the duals, and the student's
    mean entropy and log probability of the teacher's best column at the end."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.nn.functional.normalize(torch.randn(n, features, generator=gen, device="cuda"), dim=1)
    prototypes = torch.nn.functional.normalize(torch.randn(m, features, generator=gen, device="cuda"), dim=1)
    prototypes *= 0.5 + 2.5 * torch.rand(m, 1, generator=gen, device="cuda") ** 8  # (long ones take most rows)
    teacher = (X @ prototypes.t()).to(dtype)

    beta = column_duals(teacher, eta, sweeps)
    targets, plain = (RowLogprob(n, m, k=k, targets=0, dtype=dtype) for _ in range(2))
    targets.logprob(teacher, eta=eta, bias=beta)
    plain.logprob(teacher, eta=eta)
    most = [float(torch.bincount(t.top_idx[:, 0].long(), minlength=m).max()) / n for t in (targets, plain)]

    W = torch.zeros(features, m, device="cuda")
    step, answer = RowDistill(n, m, k, dtype=dtype), RowLogprob(n, m, targets=1, dtype=dtype)
    weight = torch.full((n,), 1.0 / n, device="cuda")
    losses = []
    best = targets.top_idx[:, :1].contiguous()
    for _ in range(steps):
        scores = (X @ W).to(dtype)
        # (log probabilities are scores at temperature 1, which is the student's)
        step.distill(scores, targets.top_idx, targets.top_logprob, row_weight=weight)
        W -= rate * (X.t() @ step.grad.float())
        losses.append(step.loss.mean())
    answer.logprob((X @ W).to(dtype), best)
    return dict(loss=torch.stack(losses).tolist(), most_balanced=most[0], most_plain=most[1],
                entropy=float(answer.entropy.mean()), logprob=float(answer.logprob_out.mean()))


def route_tokens(n=4096, experts=64, k=2, sweeps=8, dtype=torch.float32, seed=0):
    """Returns the tokens of the most used expert over the mean, with the duals as bias and without, the tokens in the order of their
    experts, where each expert's begin, and the weights' gradient to the scores."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    scores = (torch.randn(n, experts, generator=gen, device="cuda") + torch.randn(experts, generator=gen, device="cuda")).to(dtype)
    beta = column_duals(scores, 1.0, sweeps)
    balanced, plain = RowRoute(n, experts, k, bias_on="logit", dtype=dtype), RowRoute(n, experts, k, dtype=dtype)
    balanced.route(scores, bias=beta)
    plain.route(scores)
    load = [float(torch.bincount(r.idx.reshape(-1).long(), minlength=experts).max()) * experts / (n * k) for r in (balanced, plain)]

    row_ptr = torch.arange(0, n * k + 1, k, dtype=torch.int64, device="cuda")
    col_idx = balanced.idx.sort(dim=1).values.reshape(-1)  # (a pattern's columns ascend in its rows)
    start = torch.empty(experts + 1, dtype=torch.int64, device="cuda")
    tokens = torch.empty(n * k, dtype=torch.int32, device="cuda")
    place = torch.empty(n * k, dtype=torch.int64, device="cuda")
    ws = torch.empty(max(B.regot_pattern_transpose_workspace_bytes(n, experts, n * k), 256), dtype=torch.uint8, device="cuda")
    B.regot_pattern_transpose(n, experts, n * k, row_ptr, col_idx, start, tokens, place, workspace=ws)
    grad = balanced.grad(scores, torch.ones_like(balanced.weight))
    return dict(load_balanced=load[0], load_plain=load[1], start=start, tokens=tokens, idx=balanced.idx, weight=balanced.weight, grad=grad)


if __name__ == "__main__":
    s = train_student()
    print(f"student: loss {s['loss'][0]:.4f} -> {s['loss'][-1]:.4f}, entropy {s['entropy']:.3f}, log probability of the target {s['logprob']:.3f}; "
          f"most used column {100 * s['most_plain']:.2f} % of the rows, balanced {100 * s['most_balanced']:.2f} %")
    r = route_tokens()
    print(f"router: most used expert {r['load_plain']:.2f} times the mean, balanced {r['load_balanced']:.2f}")
